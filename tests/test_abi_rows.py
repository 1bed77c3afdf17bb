"""Refusals of the entry points with norms and rotations, and of the paged cache's, through the C ABI and the binding: every call here fails
on its checks before anything is read or enqueued (no GPU needed).  Beside them, the arithmetic that finds a slot's page."""

import ctypes as C
import os
import subprocess

import pytest

from paper_2511_23113_amd import binding as B
from paper_2511_23113_amd import build as b

FAKE = 1 << 20         # an aligned address that is never used
STRIDES = (2 * 8 * 64, 8 * 64, 64)


def rotary(pairs=(8, 12, 12), halves=0, axes=None, freqs=None):
    n = sum(pairs)
    values = (C.c_double * max(n, 1))(*([0.5] * n if freqs is None else freqs))
    r = B.RotaryDesc(axes=len(pairs) if axes is None else axes, halves=halves, freqs=values)
    r.pairs[:len(pairs)] = pairs
    r.kept = values
    return r


def norm(kind=1, eps=1e-6, **kw):
    return B.HeadNormDesc(kind=kind, eps=eps, q_gain=FAKE, k_gain=FAKE, **kw)


def said(rc):
    return rc, B.load_library().dbsp_last_error().decode()


def ref(x):
    return None if x is None else C.byref(x)


def packed(dtype, nb, n, d, H, Hk, q, qs, k, ks, qo, qos, ko, kos, pos, pb, pt):
    return B._QK_ROWS.pack(dtype, nb, n, d, H, Hk, q or 0, *qs, k or 0, *ks, qo or 0, *qos, ko or 0, *kos, pos or 0, pb, pt)


def fwd(dtype=0, nb=2, n=8, d=64, q=FAKE, qs=STRIDES, qo=FAKE, qos=STRIDES, H=2, k=FAKE, ks=STRIDES, ko=FAKE, kos=STRIDES, Hk=2, nrm=norm(), rot=rotary(),
        pos=FAKE, pb=24, pt=3):
    rows = packed(dtype, nb, n, d, H, Hk, q, qs, k, ks, qo, qos, ko, kos, pos, pb, pt)
    return said(B.load_library().dbsp_qk_norm_rope_fwd(rows, ref(nrm), ref(rot), None))


def bwd(dtype=0, nb=2, n=8, d=64, q=FAKE, qs=STRIDES, qo=FAKE, qos=STRIDES, H=2, k=FAKE, ks=STRIDES, ko=FAKE, kos=STRIDES, Hk=2, nrm=norm(), rot=rotary(),
        pos=FAKE, pb=24, pt=3, dy=FAKE, dys=STRIDES, grads=FAKE, ws=FAKE, size=1 << 40):
    # q_out and k_out of the forward pass: dq and dk here, behind gradients of the results that are all right
    rows = packed(dtype, nb, n, d, H, Hk, q, qs, k, ks, dy, dys, dy, dys, pos, pb, pt)
    dx = [B._HEADS.pack(x or 0, *xs) for x, xs in ((qo, qos), (ko, kos))]
    return said(B.load_library().dbsp_qk_norm_rope_bwd(rows, *dx, ref(nrm), ref(rot), grads, ws, size, None))


def cache(**kw):
    x = B.PagedCacheDesc(dtype=0, B=2, Hk=2, d=64, n_pages=9, page_size=16, max_pages=4, k=FAKE, v=FAKE, pages=FAKE, pages_stride=4, lens=FAKE)
    x.k_stride[:] = x.v_stride[:] = (2 * 16 * 64, 16 * 64, 64)
    for name, value in kw.items():
        if name.endswith("_stride") and name != "pages_stride":
            getattr(x, name)[:] = value
        else:
            setattr(x, name, value)
    return x


def append(c, nrm=norm(), rot=rotary(), k=FAKE, ks=STRIDES, v=FAKE, vs=STRIDES, q=FAKE, qs=STRIDES, qo=FAKE, qos=STRIDES, H=2, n=8, new=None, pos=FAKE, pb=24, pt=3, **other):
    nb, hk, d, dtype = (c.B, c.Hk, c.d, c.dtype) if c is not None else (1, 1, 64, 0)
    rows = packed(other.get("dtype", dtype), other.get("B", nb), n, other.get("d", d), H, other.get("Hk", hk), q, qs, k, ks, qo, qos, None, STRIDES, pos, pb, pt)
    return said(B.load_library().dbsp_paged_append(ref(c), rows, B._HEADS.pack(v or 0, *vs), new, ref(nrm), ref(rot), None))


def attn(c, q=FAKE, qs=STRIDES, o=FAKE, os_=STRIDES, lse=FAKE, q_lens=None, H=2, n=1, scale=0.0, ws=FAKE, size=1 << 40):
    return said(B.load_library().dbsp_paged_attn_fwd(ref(c), q, *qs, o, *os_, lse, q_lens, H, n, 1, scale, ws, size, None))


ROWS = [
    (dict(dtype=2), "dtype"), (dict(nb=0), "positive"), (dict(n=0), "positive"), (dict(d=96), "head dim"), (dict(q=None), "(q)"), (dict(q=FAKE + 8), "q must be"),
    (dict(qs=(1024, 4, 64)), "q must be"), (dict(qs=(1024, 512, -64)), "q must be"), (dict(qs=(1024, 512, (1 << 24) + 8)), "q must be"), (dict(qo=None), "null"),
    (dict(qos=(1024, 512, 0)), "overlap"), (dict(qos=(512, 512, 64)), "overlap"), (dict(H=0), "heads"), (dict(Hk=0), "heads"), (dict(ko=None), "null"),
    (dict(kos=(1024, 0, 64)), "overlap"), (dict(nrm=norm(kind=3)), "kind"), (dict(nrm=norm(kind=-1)), "kind"), (dict(nrm=norm(eps=0.0)), "eps"),
    (dict(nrm=norm(eps=float("nan"))), "eps"), (dict(nrm=norm(eps=float("inf"))), "eps"), (dict(nrm=norm(q_bias=FAKE + 4)), "aligned"),
    (dict(rot=rotary(axes=5)), "axes"), (dict(rot=rotary(axes=-1)), "axes"), (dict(rot=rotary((8, 0))), "pairs"), (dict(rot=rotary((20, 13))), "pairs"),
    (dict(rot=rotary((5, 6), halves=1)), "multiple of 4"), (dict(rot=rotary((2,), freqs=[1.0, float("inf")])), "finite"),
    (dict(rot=rotary((2,), freqs=[float("nan"), 1.0])), "finite"), (dict(pos=None), "positions"), (dict(pos=FAKE + 2), "4-byte"), (dict(pt=-3), "positions"), (dict(pb=-1), "positions"),
]


@pytest.mark.parametrize("change, word", ROWS, ids=[f"{i}-{sorted(c)[0]}" for i, (c, _) in enumerate(ROWS)])
def test_bad_calls_of_norms_and_rotations(change, word):
    for rc, msg in (fwd(**change), bwd(**change)):
        assert rc == B.DBSP_EINVAL and word in msg


def test_too_many_tokens_or_heads():
    for call in (fwd, bwd):
        assert call(nb=1 << 16, n=1 << 15)[0] == B.DBSP_ESHAPE
        big = (1 << 30, 64, 64)
        assert call(nb=1, n=1 << 29, H=1 << 9, qs=(0, 1 << 40, 64), qos=(0, 1 << 40, 64))[0] in (B.DBSP_ESHAPE, B.DBSP_EINVAL)
        assert call(nb=1, n=1, H=1 << 30, k=None, qs=big, qos=big)[0] == B.DBSP_ESHAPE


BACKWARD = [
    (dict(dy=None), "q_out"), (dict(dys=(1024, 4, 64)), "q_out"), (dict(nrm=None), "no gains"), (dict(nrm=norm(kind=0)), "no gains"), (dict(grads=FAKE + 4), "16-byte"),
    (dict(ws=None), "workspace"), (dict(ws=FAKE + 16), "256-byte"), (dict(size=100), "holds 100 bytes"),
]


@pytest.mark.parametrize("change, word", BACKWARD, ids=[f"{i}-{sorted(c)[0]}" for i, (c, _) in enumerate(BACKWARD)])
def test_bad_backward_calls(change, word):
    rc, msg = bwd(**change)
    assert rc == B.DBSP_EINVAL and word in msg


def test_backward_workspaces():
    lib, n = B.load_library(), C.c_int64()
    assert lib.dbsp_qk_norm_rope_bwd_workspace(1, 32760, 128, 40, 40, None) == B.DBSP_EINVAL
    assert lib.dbsp_qk_norm_rope_bwd_workspace(1, 0, 128, 40, 40, C.byref(n)) == B.DBSP_EINVAL and n.value == 0
    assert lib.dbsp_qk_norm_rope_bwd_workspace(1, 10, 128, 0, 40, C.byref(n)) == B.DBSP_EINVAL
    for shape in ((1, 1, 64, 1, 0), (1, 32760, 128, 40, 40), (64, 4096, 64, 200, 8)):
        assert lib.dbsp_qk_norm_rope_bwd_workspace(*shape, C.byref(n)) == B.DBSP_OK
        assert 0 < n.value <= 1 << 23 and n.value % 256 == 0


PAGED = [
    (dict(dtype=7), "dtype"), (dict(d=80), "head dim"), (dict(B=0), "positive"), (dict(Hk=0), "positive"), (dict(n_pages=0), "positive"), (dict(page_size=0), "positive"),
    (dict(max_pages=-1), "positive"), (dict(k=None), "null"), (dict(v=None), "null"), (dict(pages=None), "null"), (dict(lens=None), "null"), (dict(k=FAKE + 4), "16-byte"),
    (dict(k_stride=(2048, 1024, 60)), "multiples of 8"), (dict(v_stride=(2048, 1024, -64)), "multiples of 8"), (dict(v_stride=(2048, 1024, (1 << 24) + 8)), "2^24"),
    (dict(k_stride=((1 << 30) + 8, 1024, 64)), "2^30"), (dict(pages_stride=-4), "pages_stride"), (dict(pages=FAKE + 2), "4-byte"), (dict(lens=FAKE + 1), "4-byte"),
]


@pytest.mark.parametrize("change, word", PAGED, ids=[f"{i}-{sorted(c)[0]}" for i, (c, _) in enumerate(PAGED)])
def test_bad_paged_caches_are_refused_by_every_entry_point(change, word):
    c = cache(**change)
    for rc, msg in (append(c), attn(c)):
        assert rc == B.DBSP_EINVAL and word in msg
    n = C.c_int64(5)
    assert B.load_library().dbsp_paged_attn_workspace(C.byref(c), 2, 1, C.byref(n)) == B.DBSP_EINVAL and n.value == 0


def test_paged_caches_that_are_too_large():
    for c in (cache(max_pages=1 << 27, page_size=8, pages_stride=1 << 27), cache(B=1 << 20, Hk=1 << 11)):
        assert append(c)[0] == B.DBSP_ESHAPE and attn(c)[0] == B.DBSP_ESHAPE
    assert append(None)[0] == B.DBSP_EINVAL and attn(None)[0] == B.DBSP_EINVAL


APPEND = [
    (dict(k=None), "(k)"), (dict(v=None), "(v)"), (dict(qo=None), "(q_out)"), (dict(n=0), "positive"), (dict(H=0), "H must"), (dict(ks=(1024, 512, 60)), "k must"),
    (dict(vs=(1024, 512, 60)), "v must"), (dict(qos=(1024, 512, 0)), "overlap"), (dict(new=FAKE + 2), "new_lens"), (dict(pos=None), "positions"),
    (dict(nrm=norm(eps=-1.0)), "eps"), (dict(rot=rotary((33,))), "pairs"),
]


@pytest.mark.parametrize("change, word", APPEND, ids=[f"{i}-{sorted(c)[0]}" for i, (c, _) in enumerate(APPEND)])
def test_bad_appends(change, word):
    rc, msg = append(cache(), **change)
    assert rc == B.DBSP_EINVAL and word in msg


def test_appended_rows_that_are_not_the_caches():
    for change in (dict(dtype=1), dict(B=3), dict(d=128), dict(Hk=1)):
        rc, msg = append(cache(), **change)
        assert rc == B.DBSP_ESHAPE and "the cache's" in msg
    lib = B.load_library()
    assert lib.dbsp_paged_append(C.byref(cache()), None, None, None, None, None, None) == B.DBSP_EINVAL
    assert lib.dbsp_qk_norm_rope_fwd(None, None, None, None) == B.DBSP_EINVAL
    rows = packed(0, 2, 8, 64, 2, 2, FAKE, STRIDES, FAKE, STRIDES, FAKE, STRIDES, FAKE, STRIDES, None, 0, 0)
    assert said(lib.dbsp_qk_norm_rope_bwd(rows, None, None, None, None, None, None, 0, None))[1].endswith("(dq)")
    assert said(lib.dbsp_paged_append(C.byref(cache()), rows, None, None, None, None, None))[1].endswith("(v)")


def test_pools_that_are_written_do_not_overlap():
    for change in (dict(k_stride=(2048, 1024, 0)), dict(v_stride=(1024, 1024, 64)), dict(k_stride=(0, 1024, 64))):
        rc, msg = append(cache(**change))
        assert rc == B.DBSP_EINVAL and "overlap" in msg


ATTN = [
    (dict(q=None), "(q)"), (dict(o=None), "(o)"), (dict(H=0), "positive"), (dict(n=0), "positive"), (dict(qs=(1024, 4, 64)), "q must"), (dict(os_=(0, 512, 64)), "overlap"),
    (dict(lse=FAKE + 2), "4-byte"), (dict(q_lens=FAKE + 2), "4-byte"), (dict(scale=float("nan")), "softmax_scale"), (dict(scale=1e-35), "softmax_scale"),
    (dict(scale=float("inf")), "softmax_scale"), (dict(ws=FAKE + 64), "256-byte"),
]


@pytest.mark.parametrize("change, word", ATTN, ids=[f"{i}-{sorted(c)[0]}" for i, (c, _) in enumerate(ATTN)])
def test_bad_paged_attention_calls(change, word):
    rc, msg = attn(cache(), **change)
    assert rc == B.DBSP_EINVAL and word in msg


def test_paged_attention_shapes_and_workspaces():
    rc, msg = attn(cache(), H=3)
    assert rc == B.DBSP_ESHAPE and "multiple" in msg
    assert attn(cache(), n=1 << 30)[0] == B.DBSP_ESHAPE
    lib, n = B.load_library(), C.c_int64()

    def need(c, H, Nq):
        assert lib.dbsp_paged_attn_workspace(C.byref(c), H, Nq, C.byref(n)) == B.DBSP_OK
        return n.value
    assert need(cache(), 2, 1) == 0                      # one launch
    long = cache(max_pages=8192, pages_stride=8192)
    assert 0 < need(long, 2, 1) < 1 << 24 and n.value % 256 == 0
    assert need(long, 32, 8) < 1 << 28
    rc, msg = attn(long, ws=None)
    assert rc == B.DBSP_EINVAL and "workspace" in msg
    rc, msg = attn(long, size=100)
    assert rc == B.DBSP_EINVAL and "holds 100 bytes" in msg
    assert lib.dbsp_paged_attn_workspace(C.byref(long), 2, 1, None) == B.DBSP_EINVAL


def test_tensors_that_are_not_on_a_gpu_are_refused():
    import torch
    x, i = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        B.qk_norm_rope_fwd(x, x)
    with pytest.raises(ValueError, match="GPU"):
        B.qk_norm_rope_bwd(x, x, x, x)
    with pytest.raises(ValueError, match="GPU"):
        B.PagedKVCache(x, x, i[None], i)
    with pytest.raises(ValueError, match="bf16 or fp16"):
        B.PagedKVCache(x.float(), x.float(), i[None], i)
    with pytest.raises(ValueError, match="GPU"):
        B.HeadNorm(torch.ones(64))
    with pytest.raises(ValueError, match="kind"):
        B.HeadNorm(kind="batch")


def test_rotaries():
    r = B.Rotary((2, 3), theta=100.0)
    assert r.freqs == pytest.approx((1.0, 0.1, 1.0, 100.0 ** (-1 / 3), 100.0 ** (-2 / 3)))
    assert B.Rotary((2,), freqs=[3, 4]).freqs == (3.0, 4.0)
    for bad in (dict(pairs=()), dict(pairs=(1, 2, 3, 4, 5)), dict(pairs=(0, 3)), dict(pairs=(2,), freqs=[1.0])):
        with pytest.raises(ValueError):
            B.Rotary(**bad)


def test_a_slots_page_by_multiplication(tmp_path):
    # the division by the page size as the kernels form it, against the division: at every slot near a page's end or the largest slot
    src = tmp_path / "pages.cpp"
    src.write_text("""
#include "paged_params.hpp"
extern "C" int wrong(int page_size, int step) {
  uint32_t mul, shift;
  paged_divisor(page_size, mul, shift);
  auto bad = [&](int64_t slot) { return slot >= 0 && slot < ((int64_t)1 << 30) + 64 && paged_quotient((int)slot, mul, shift) != (int)(slot / page_size); };
  for (int64_t s = 0; s < ((int64_t)1 << 30) + 64; s += step)
    for (int64_t x = s / page_size * page_size - 1; x <= s / page_size * page_size + 1; ++x)
      if (bad(x)) return 1;
  for (int64_t x = ((int64_t)1 << 30) - 1000; x < ((int64_t)1 << 30) + 64; ++x)
    if (bad(x)) return 1;
  return 0;
}
""")
    out = tmp_path / "pages.so"
    subprocess.run([b._hipcc(), "-x", "hip", "--cuda-host-only", "-shared", "-fPIC", "-O1", str(src), "-o", str(out), "-I", b.CSRC, "-I", os.path.join(b.ROOT, "include")],
                   check=True, capture_output=True, timeout=120)
    lib = C.CDLL(str(out))
    for page_size in [*range(1, 70), 96, 100, 127, 128, 129, 255, 256, 1000, 4095, 4096, 65537, (1 << 29) - 1, 1 << 29, (1 << 30) - 1]:
        assert lib.wrong(page_size, 99991) == 0
