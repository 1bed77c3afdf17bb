"""What the binding's objects do where a tensor that they keep is given other memory: `x.data = y`, as a module's half(), to() and cpu() do with
every parameter, or resize_().  The object has to go by where its tensors are at a call, and must not let go of what it goes by.  No GPU needed:
tensors of the host pass for ones on a GPU, and calls note what they are given."""

import gc

import pytest
import torch

from paper_2511_23113_amd import binding as B


class OnGpu(torch.Tensor):
    """A tensor of the host that says that it is on a GPU."""
    is_cuda = True


def on_gpu(x):
    return torch.Tensor._make_subclass(OnGpu, x)


class Noting:
    """Of the library: every call notes its arguments, and workspaces are of 256 bytes."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_workspace"):
                args[-1]._obj.value = 256
            else:
                self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def lib(monkeypatch):
    B._torch_module()
    B.load_library()
    noting = Noting()
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    monkeypatch.setattr(B, "_lib", noting)
    here = object.__new__(B._Rows)
    here.device, here._index, here._at, here._bytes = torch.device("cpu"), -1, None, {}
    monkeypatch.setitem(B._rows_on, -1, here)
    B._ROW_TYPES.update({torch.bfloat16: 0, torch.float16: 1})
    return noting


def norm_given(lib):
    """The norm that the last call was given, as it stood when the call was made or after it: objects keep one description."""
    name, args = lib.calls[-1]
    at = {"dbsp_qk_norm_rope_fwd": 1, "dbsp_qk_norm_rope_bwd": 3, "dbsp_paged_append": 4}[name]
    return args[at]._obj


def rows(dtype=torch.bfloat16):
    return torch.zeros(1, 2, 8, 64, dtype=dtype), torch.zeros(1, 1, 8, 64, dtype=dtype)


@pytest.mark.parametrize("which", ["q_gain", "k_gain", "q_bias", "k_bias"])
def test_gains_that_move(lib, which):
    given = {n: on_gpu(torch.ones(64)) for n in ("q_gain", "k_gain", "q_bias", "k_bias")}
    norm = B.HeadNorm(**given)
    q, k = rows()
    calls = (lambda: B.qk_norm_rope_fwd(q, k, norm=norm), lambda: B.qk_norm_rope_bwd(q, k, q, k, norm=norm))
    for call in calls:
        given[which].data = torch.full((64,), 2.0)
        call()
        assert getattr(norm_given(lib), which) == given[which].data_ptr()
        for other in given:
            assert getattr(norm_given(lib), other) == given[other].data_ptr()


def test_gains_of_another_type(lib):
    # a module's half(): the same parameters, other memory, another type
    given = [on_gpu(torch.ones(64)) for _ in range(2)]
    norm = B.HeadNorm(*given)
    q, k = rows()
    B.qk_norm_rope_fwd(q, k, norm=norm)
    assert norm_given(lib).gains_f32 == 1
    given[0].data = given[0].data.bfloat16()
    with pytest.raises(ValueError, match="differ"):
        B.qk_norm_rope_fwd(q, k, norm=norm)
    given[1].data = given[1].data.bfloat16()
    B.qk_norm_rope_fwd(q, k, norm=norm)
    assert norm_given(lib).gains_f32 == 0 and norm_given(lib).k_gain == given[1].data_ptr()
    with pytest.raises(ValueError, match="rows' type"):
        B.qk_norm_rope_fwd(*rows(torch.float16), norm=norm)
    given[0].data = torch.ones(128)
    for _ in range(2):                     # and again, not only the first time
        with pytest.raises(ValueError):
            B.qk_norm_rope_fwd(q, k, norm=norm)


def test_gains_that_are_resized(lib):
    x = torch.ones(64)
    norm = B.HeadNorm(on_gpu(x))
    norm.given["q_gain"].resize_(1 << 20)
    with pytest.raises(ValueError, match="rows' type"):
        B.qk_norm_rope_fwd(*rows(), norm=norm)


def test_memory_that_a_description_names_is_kept(lib):
    # (else memory that comes to lie where a gain was, of another type or size, would pass for it)
    x = torch.ones(64)
    gain = on_gpu(x)
    norm = B.HeadNorm(gain)
    at = norm._desc.q_gain
    gain.data = torch.ones(64)
    del x
    gc.collect()
    taken = [torch.empty(64) for _ in range(64)]
    assert at not in [y.data_ptr() for y in taken]
    B.qk_norm_rope_fwd(*rows(), norm=norm)
    assert norm_given(lib).q_gain == gain.data_ptr() != at


def paged():
    x = {"k": torch.zeros(9, 1, 16, 64, dtype=torch.bfloat16), "v": torch.zeros(9, 1, 16, 64, dtype=torch.bfloat16), "pages": torch.zeros(1, 4, dtype=torch.int32),
         "lens": torch.zeros(1, dtype=torch.int32)}
    return {n: on_gpu(y) for n, y in x.items()}


def contiguous():
    x = {"k": torch.zeros(1, 1, 40, 64, dtype=torch.bfloat16), "v": torch.zeros(1, 1, 40, 64, dtype=torch.bfloat16), "lens": torch.zeros(1, dtype=torch.int32),
         "prefix_k": torch.zeros(1, 9, 64, dtype=torch.bfloat16), "prefix_v": torch.zeros(1, 9, 64, dtype=torch.bfloat16), "weights": torch.zeros(1, 1, 40),
         "positions": torch.zeros(1, 1, 40, dtype=torch.int32)}
    return {n: on_gpu(y) for n, y in x.items()}


def calls_of(cache):
    q, k = rows()
    if isinstance(cache, B.PagedKVCache):
        return [lambda: B.paged_append(cache, k, k), lambda: B.paged_attn_fwd(cache, q[:, :, :1])]
    return [lambda: B.cache_attn_fwd(cache, q[:, :, :1], decay=1.0), lambda: B.cache_evict(cache, 20)]


@pytest.mark.parametrize("make, of, which", [(paged, B.PagedKVCache, n) for n in paged()] + [(contiguous, B.KVCache, n) for n in contiguous()])
def test_a_caches_tensors_that_move(lib, make, of, which):
    given = make()
    cache = of(**given)
    for call in calls_of(cache):
        given[which].data = given[which].data.clone()
        call()
        desc = lib.calls[-1][1][0]._obj
        for name, x in given.items():
            assert getattr(desc, name) == x.data_ptr()


def test_a_cache_of_other_sizes(lib):
    # the pool grows, its pages are wider, and the table gets longer
    given = paged()
    cache = B.PagedKVCache(**given)
    attend = calls_of(cache)[1]
    attend()
    given["k"].data, given["v"].data = (torch.zeros(30, 24, 1, 64, dtype=torch.bfloat16).transpose(1, 2) for _ in range(2))
    given["pages"].data = torch.zeros(1, 7, dtype=torch.int32)
    attend()
    desc = lib.calls[-1][1][0]._obj
    assert (desc.n_pages, desc.page_size, desc.max_pages, desc.pages_stride, cache.page_size) == (30, 24, 7, 7, 24) and list(desc.k_stride) == [24 * 64, 64, 64]
    given["lens"].data = torch.zeros(2, dtype=torch.int32)
    for _ in range(2):
        with pytest.raises(ValueError, match="lens"):
            attend()
    given["lens"].data = torch.zeros(1, dtype=torch.int32)
    given["v"].data = given["v"].data.half()
    with pytest.raises(ValueError, match="v must"):
        attend()


def test_a_prefix_that_moves_serves_other_batches(lib):
    given = {n: x for n, x in contiguous().items() if n.startswith("prefix")}
    cache = B.KVCache(**given)
    for b in (1, 3):
        given["prefix_v"].data = given["prefix_v"].data.clone()
        B.cache_attn_fwd(cache, torch.zeros(b, 2, 1, 64, dtype=torch.bfloat16))
        desc = lib.calls[-1][1][0]._obj
        assert desc.B == b and desc.prefix_v == given["prefix_v"].data_ptr()


@pytest.mark.parametrize("dims", range(6))
def test_appended_rows_of_other_dimensions(lib, dims):
    cache, k = B.PagedKVCache(**paged()), rows()[1]
    x = torch.zeros((1, 1, 8, 64, 1, 1)[:dims], dtype=torch.bfloat16)
    for bad in (dict(q=x), dict(k=x), dict(v=x), dict(q=k, q_out=x), dict(positions=x.int(), rotary=B.Rotary((8, 8)))):
        if dims != 4 or "positions" in bad:
            with pytest.raises(ValueError):
                B.paged_append(cache, **{"k": k, "v": k, **bad})


def test_a_gain_whose_memory_is_gone(lib):
    # (its address is NULL then, which would pass for a gain that is not given)
    gain = on_gpu(torch.ones(64))
    norm = B.HeadNorm(gain)
    gain.untyped_storage().resize_(0)
    for call in (lambda: B.qk_norm_rope_fwd(*rows(), norm=norm), lambda: B.HeadNorm(gain)):
        with pytest.raises(ValueError, match="memory"):
            call()
    gain.untyped_storage().resize_(256)
    B.qk_norm_rope_fwd(*rows(), norm=norm)
    assert norm_given(lib).q_gain == gain.data_ptr() != 0
