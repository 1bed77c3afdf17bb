"""The cache entry points' refusals and workspace sizes, through the C ABI: every call here fails on its checks before anything is
read or enqueued (no GPU needed)."""

import ctypes as C

import pytest

from paper_2511_23113_amd import binding as B

FAKE = 1 << 20         # an aligned address that is never used


def desc(**kw):
    d = B.CacheDesc(dtype=0, B=2, Hk=2, d=64, n_prefix=100, capacity=64, prefix_k=FAKE, prefix_v=FAKE, k=FAKE, v=FAKE, lens=FAKE, weights=FAKE, positions=FAKE)
    for x in (d.prefix_k_stride, d.prefix_v_stride):
        x[:] = (100 * 64, 64)
    for x in (d.k_stride, d.v_stride):
        x[:] = (2 * 64 * 64, 64 * 64, 64)
    for name, value in kw.items():
        if name.endswith("_stride"):
            getattr(d, name)[:] = value
        else:
            setattr(d, name, value)
    return d


def attn(d, q=FAKE, qs=(256, 64, 64), o=FAKE, os_=(256, 64, 64), lse=FAKE, q_lens=None, H=4, Nq=1, scale=0.0, decay=1.0, ws=FAKE, n=1 << 40):
    lib = B.load_library()
    rc = lib.dbsp_cache_attn_fwd(C.byref(d) if d is not None else None, q, *qs, o, *os_, lse, q_lens, H, Nq, 1, scale, decay, ws, n, None)
    return rc, lib.dbsp_last_error().decode()


def evict(d, budget=32, sinks=0, keep_from=None, ws=FAKE, n=1 << 40):
    lib = B.load_library()
    rc = lib.dbsp_cache_evict(C.byref(d) if d is not None else None, budget, sinks, keep_from, ws, n, None)
    return rc, lib.dbsp_last_error().decode()


BAD_CACHES = [
    (dict(dtype=2), "dtype"), (dict(d=96), "head dim"), (dict(B=0), "positive"), (dict(Hk=-1), "positive"), (dict(n_prefix=-1), "negative"),
    (dict(capacity=-1), "negative"), (dict(prefix_v=None), "prefix"), (dict(k=None), "null"), (dict(lens=None), "lens"),
    (dict(k=FAKE + 8), "aligned"), (dict(prefix_k=FAKE + 2), "aligned"), (dict(k_stride=(8192, 4096, 60)), "multiples of 8"),
    (dict(v_stride=(8192, -64, 64)), "multiples of 8"), (dict(v_stride=(8192, 4096, (1 << 24) + 8)), "2^24"), (dict(prefix_k_stride=(6400, 4)), "multiples of 8"),
    (dict(weights=FAKE + 2), "4-byte"),
]


@pytest.mark.parametrize("change, word", BAD_CACHES, ids=[str(sorted(c)) + w for c, w in BAD_CACHES])
def test_bad_caches_are_refused_by_every_entry_point(change, word):
    for rc, msg in (attn(desc(**change)), evict(desc(**change))):
        assert rc == B.DBSP_EINVAL and word in msg
    n = C.c_int64(7)
    assert B.load_library().dbsp_cache_attn_workspace(C.byref(desc(**change)), 4, 1, 1, 1, C.byref(n)) == B.DBSP_EINVAL and n.value == 0


BAD_CALLS = [
    (dict(q=None), "null"), (dict(o=None), "null"), (dict(ws=None), "null"), (dict(H=0), "positive"), (dict(Nq=0), "positive"), (dict(q=FAKE + 8), "aligned"),
    (dict(qs=(256, 4, 64)), "multiples of 8"), (dict(os_=(256, 0, 64)), "overlap"), (dict(os_=(64, 64, 64)), "overlap"), (dict(lse=FAKE + 1), "4-byte"),
    (dict(q_lens=FAKE + 1), "4-byte"), (dict(scale=float("nan")), "softmax_scale"), (dict(scale=float("inf")), "softmax_scale"), (dict(scale=1e-35), "softmax_scale"), (dict(decay=float("nan")), "decay"),
    (dict(decay=float("inf")), "decay"), (dict(ws=FAKE + 16), "256-byte"), (dict(n=100), "holds 100 bytes"),
]


@pytest.mark.parametrize("change, word", BAD_CALLS, ids=[str(sorted(c)) + w for c, w in BAD_CALLS])
def test_bad_attention_calls(change, word):
    rc, msg = attn(desc(), **change)
    assert rc == B.DBSP_EINVAL and word in msg


def test_attention_shapes_and_missing_weights():
    assert attn(None)[0] == B.DBSP_EINVAL
    rc, msg = attn(desc(), H=3)
    assert rc == B.DBSP_ESHAPE and "multiple" in msg
    assert attn(desc(), Nq=1 << 30)[0] == B.DBSP_ESHAPE
    assert attn(desc(capacity=1 << 30))[0] == B.DBSP_ESHAPE
    assert attn(desc(B=1 << 29, Hk=1 << 10), H=1 << 10)[0] == B.DBSP_ESHAPE
    rc, msg = attn(desc(weights=None))
    assert rc == B.DBSP_EINVAL and "no weights" in msg
    lib = B.load_library()
    assert lib.dbsp_cache_attn_workspace(C.byref(desc()), 4, 1, 1, 1, None) == B.DBSP_EINVAL


def test_bad_evictions():
    assert evict(None)[0] == B.DBSP_EINVAL
    for change, word in ((dict(budget=0), "budget"), (dict(sinks=-1), "sinks"), (dict(keep_from=FAKE + 2), "4-byte"), (dict(ws=None), "null"),
                         (dict(ws=FAKE + 4), "256-byte"), (dict(n=0), "holds 0 bytes")):
        rc, msg = evict(desc(), **change)
        assert rc == B.DBSP_EINVAL and word in msg
    for change, word in ((dict(weights=None), "weights"), (dict(positions=None), "positions"), (dict(k_stride=(0, 4096, 64)), "overlap"),
                         (dict(v_stride=(8192, 4096, 0)), "overlap"), (dict(v_stride=(4096, 4096, 64)), "overlap")):
        rc, msg = evict(desc(**change))
        assert rc == B.DBSP_EINVAL and word in msg
    # nothing can be over a budget of the whole capacity
    assert evict(desc(), budget=64)[0] == B.DBSP_OK
    assert evict(desc(capacity=0), budget=64)[0] == B.DBSP_OK


def test_workspaces_grow_with_the_call_and_stay_moderate():
    lib, n = B.load_library(), C.c_int64()

    def need(d, H, Nq, weights=0, causal=1):
        assert lib.dbsp_cache_attn_workspace(C.byref(d), H, Nq, causal, weights, C.byref(n)) == B.DBSP_OK
        return n.value
    assert need(desc(), 4, 1) == 0         # one launch
    small = need(desc(n_prefix=1000), 4, 1)
    assert 0 < small < 1 << 22 and small % 256 == 0
    assert need(desc(n_prefix=1000), 4, 1, 1) > small
    # of long prompts only the last rounds' row tiles are cut
    assert need(desc(B=4, Hk=40, capacity=9000), 40, 9000) == 0
    assert need(desc(B=4, Hk=40, capacity=9000), 40, 9000, causal=0) < 1 << 28
    assert need(desc(n_prefix=1 << 20), 4, 1) < 1 << 30
    assert lib.dbsp_cache_evict_workspace(C.byref(desc()), 48, C.byref(n)) == B.DBSP_OK and n.value == 256 + 2 * 256


def test_tensors_that_are_not_on_a_gpu_are_refused():
    import torch
    k = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        B.KVCache(k, k, torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError, match="prefix_k and prefix_v"):
        B.KVCache(k, k, None)
    with pytest.raises(ValueError, match="bf16 or fp16"):
        B.KVCache(k.float(), k.float(), torch.zeros(1, dtype=torch.int32))
