"""Sizes that no launch can have are refused before anything is enqueued: HIP launches fewer than 2^32 threads along a dimension.  Host
only, through the sizes' entry points and calls on addresses that are never used."""

import ctypes as C

import pytest

from paper_2511_23113_amd import binding as B
from test_abi_cache import attn, desc, evict


def size(d, H, Nq, weights):
    n = C.c_int64(7)
    return B.load_library().dbsp_cache_attn_workspace(C.byref(d), H, Nq, 1, weights, C.byref(n)), n.value


# a (sequence, KV head) a workgroup of 256 threads; a prefix that is pooled, whose parts leave 16 rows a workgroup to be joined
@pytest.mark.parametrize("cache, H, Nq", [(dict(B=1 << 23, n_prefix=0, capacity=8), 2, 1), (dict(B=1 << 23, Hk=1, n_prefix=2000, capacity=0), 1, 40)])
def test_attention_of_more_than_a_launch_holds(cache, H, Nq):
    for weights in (0, 1) if cache["capacity"] else (0,):
        assert size(desc(**cache), H, Nq, weights) == (B.DBSP_ESHAPE, 0)
        assert attn(desc(**cache), H=H, Nq=Nq, decay=1.0 if weights else -1.0)[0] == B.DBSP_ESHAPE
        fewer = dict(cache, B=cache["B"] // 4)
        assert size(desc(**fewer), H, Nq, weights)[0] == B.DBSP_OK


@pytest.mark.parametrize("capacity, most", [(8, (1 << 24) - 1), (1025, (1 << 23) - 1), (4097, (1 << 22) - 1), (40000, (1 << 22) - 1)])
def test_eviction_of_more_than_a_launch_holds(capacity, most):
    n = C.c_int64(7)
    lib = B.load_library()
    assert lib.dbsp_cache_evict_workspace(C.byref(desc(B=most, Hk=1, capacity=capacity)), 4, C.byref(n)) == B.DBSP_OK
    assert lib.dbsp_cache_evict_workspace(C.byref(desc(B=most + 1, Hk=1, capacity=capacity)), 4, C.byref(n)) == B.DBSP_ESHAPE and n.value == 0
    assert evict(desc(B=most + 1, Hk=1, capacity=capacity), budget=4)[0] == B.DBSP_ESHAPE
