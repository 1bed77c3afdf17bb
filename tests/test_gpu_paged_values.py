"""Attention over a paged cache on the GPU, to the last bits: what O is off by beside its own rounding.

Queries have one value that is not zero, so a score is one product and its error that of the few roundings behind it.  u = 2^-24.  A score of s is
off by 3 u |s| (the scale, its product with log2 e, the argument) and by the exponential's unit, so a probability by 2 u (3 |s| + 2), relative
and with its sum; as two numbers of the inputs' type by 2^-16 more in bf16 (half a step of each, 2^-8 2^-8) and 2^-21 in fp16 (a step of the first,
2^-10, half a step of the second, 2^-11), or half of fp16's least step, 2^-25, where the largest
probability is 2^10 (FLOOR).  Sums over n keys: (n + 64) u in any order.  O is rounded once: h |O|."""

import numpy as np
import pytest

from oracle import rows as orows
from test_gpu_paged import filled, pool_of, table_of
from test_gpu_rows import host, torch_types

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
FLOOR = {"bf16": 0.0, "fp16": 2.0 ** -35}      # of a probability, in terms of the largest one of the row


def check(got, O, A, seen, s, dtype, top_v):
    import torch
    h = torch.finfo(torch_types(dtype)).eps / 2
    two = 2.0 ** -16 if dtype == "bf16" else 2.0 ** -21
    n = seen[..., None]
    err = (2 * U * (3 * s + 2) + two + (n + 64) * U) * A + n * FLOOR[dtype] * top_v
    tol = h * (np.abs(O) + err) + err + (2.0 ** -25 if dtype == "fp16" else 0.0)
    off = np.abs(got - O)
    assert (off <= tol).all(), f"O is {np.max(off / tol):.3g} of its tolerance"


# B, H, Hk, Nq, d, page, lens, dtype: row tiles of 16, 32, 48 and 64 rows, whole, in parts and in runs
CASES = {
    "few_keys": (3, 2, 1, 1, 64, 16, [1, 2, 5], "bf16"),
    "a_tile": (4, 8, 2, 1, 128, 16, [40, 63, 64, 65], "bf16"),
    "a_tile_fp16": (4, 8, 2, 1, 64, 24, [40, 63, 64, 65], "fp16"),
    "tiles": (2, 6, 2, 7, 64, 16, [200, 333], "bf16"),
    "tiles_fp16": (2, 15, 3, 5, 128, 7, [200, 333], "fp16"),
    "rows_48": (1, 48, 1, 1, 128, 16, [300], "bf16"),
    "rows_64": (2, 64, 1, 1, 64, 32, [90, 300], "fp16"),
    "rows_71": (1, 71, 1, 1, 128, 16, [300], "bf16"),
    "parts": (1, 2, 1, 1, 64, 64, [3000], "bf16"),
    "parts_fp16": (1, 4, 2, 1, 128, 64, [3000], "fp16"),
    "runs": (70, 2, 2, 2, 128, 16, [(i * 613) % 6900 + 2 for i in range(70)], "bf16"),
}


@pytest.mark.parametrize("name", CASES)
def test_o_is_rounded_once(name):
    import torch
    import paper_2511_23113_amd as dbsp
    B, H, Hk, Nq, d, page, lens, dtype = CASES[name]
    rng = np.random.default_rng(20)
    per = -(-max(lens) // page)
    n_pages = B * per + 1
    k, v = pool_of(n_pages, Hk, page, d, dtype, rng, "heads")
    t, table = table_of(B, per, n_pages, lens, page, rng)
    filled(k, v, t, lens, rng)
    q = torch.zeros(B, H, Nq, d, dtype=torch_types(dtype), device="cuda")
    q[..., 3] = torch.from_numpy(8 * rng.random(size=(B, H, Nq))).cuda()
    cache = dbsp.PagedKVCache(k, v, table, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    o, _ = dbsp.paged_attn_fwd(cache, q, causal=False, softmax_scale=0.125)
    hq, hk, hv = host(q), host(k), host(v)
    O, _, A, seen = orows.paged_attention(hq, hk, hv, t, lens, [Nq] * B, False, 0.125)
    top_k, top_v = (np.abs(x[np.isfinite(x)]).max() for x in (hk, hv))
    check(host(o), O, A, seen, 0.125 * hq.max() * top_k, dtype, top_v)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("n, sink", [(64, 0), (64, 63), (2, 0), (3000, 0), (3000, 2999), (640, 333)])
def test_keys_far_below_the_largest_one(dtype, n, sink):
    # one key has nearly all of the attention and a value of 0: O is what the others have, each of them 10 to 22 below in its score
    import torch
    import paper_2511_23113_amd as dbsp
    H, d, page = 16, 64, 16
    per = -(-n // page)
    k, v = (torch.zeros(per, 1, page, d, dtype=torch_types(dtype), device="cuda") for _ in range(2))
    t = np.random.default_rng(21).permutation(per).astype(np.int32)[None]
    k[..., 3], v[:] = -1.0, torch.linspace(100, 60000, d, device="cuda")
    place = int(t[0, sink // page]), 0, sink % page
    k[place], v[place] = 0.0, 0.0
    q = torch.zeros(1, H, 1, d, dtype=k.dtype, device="cuda")
    q[0, :, 0, 3] = 10 + 0.75 * torch.arange(H, device="cuda")
    cache = dbsp.PagedKVCache(k, v, torch.from_numpy(t).cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"))
    o, lse = dbsp.paged_attn_fwd(cache, q, softmax_scale=1.0)
    O, LSE, A, seen = orows.paged_attention(host(q), host(k), host(v), t, [n], [1], True, 1.0)
    check(host(o), O, A, seen, 21.25, dtype, float(v.max()))
    # the sum: a lane adds four keys a tile, so n / 64 additions in turn and 2 + 2 + 2 + 8 in trees and merges, u of it each; the largest score is 0 and the
    # others' errors, 2 u (3 * 21.25 + 2) of less than 0.14, are below 19 u; 4 u for the logarithm, its factor and rounding
    assert np.abs(host(lse) - LSE).max() <= (n / 64 + 37) * U
