"""Attention over a key/value cache on the GPU where values are as large as their type allows."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

# B, H, Hk, Nq, d, P, cap, lens: up to 32 rows a (sequence, KV head), 33 .. 128, more over few and over many tiles, and parts that are joined
LARGEST = {
    "few_rows": (3, 8, 2, 4, 64, 0, 64, [4, 5, 8]),
    "few_rows_in_parts": (2, 8, 2, 4, 128, 700, 64, [4, 5]),
    "rows_80": (3, 8, 2, 20, 64, 0, 64, [20, 21, 23]),
    "rows_128_in_parts": (1, 8, 2, 32, 128, 0, 800, [33]),
    "rows_300": (2, 2, 1, 150, 64, 0, 200, [150, 160]),
    "many_rows_in_parts": (2, 2, 1, 150, 128, 0, 50000, [150, 160]),
    "many_rows": (1, 8, 8, 1500, 64, 0, 1500, [1500]),
}


@pytest.mark.parametrize("name", LARGEST)
def test_values_at_the_top_of_fp16(name):
    """O lies between the least and the largest v that its query sees, so where v is the type's largest number O is it too.  Rounded
    probabilities may sum to more than they did by half a step, relative 2^-11, and 65,520 = 65,504 (1 + 2.4e-4) would be rounded to infinity."""
    import torch
    import paper_2511_23113_amd as dbsp
    B, H, Hk, Nq, d, P, cap, lens = LARGEST[name]
    rng = np.random.default_rng(sorted(LARGEST).index(name))
    rand = lambda *s: torch.from_numpy(rng.normal(size=s)).half().cuda()      # noqa: E731
    top = torch.where(torch.arange(d, device="cuda") % 2 == 0, 65504.0, -65504.0).half()
    q, k, v = 2 * rand(B, H, Nq, d), rand(B, Hk, cap, d), top.expand(B, Hk, cap, d).contiguous()
    pk, pv = (rand(Hk, P, d), top.expand(Hk, P, d).contiguous()) if P else (None, None)
    o, _ = dbsp.cache_attn_fwd(dbsp.KVCache(k, v, torch.tensor(lens, dtype=torch.int32, device="cuda"), pk, pv), q, causal=True)
    # below the top: probabilities' half step 2^-11, O's own; sums of up to 50,000 f32 terms stay far below
    assert bool(torch.isfinite(o).all())
    off = (o.double() / top.double() - 1).abs().max()
    assert off <= 2 * 2.0 ** -11 * 1.01


@pytest.mark.parametrize("H, Nq, cap", [(2, 2, 128), (4, 20, 128), (4, 20, 2000), (2, 250, 128), (2, 250, 40000)])
def test_one_key_with_all_of_a_rows_attention_at_the_top_of_fp16(H, Nq, cap):
    """The key that counts comes in the second tile, by less above the first tile's largest score than what raises the running max: its
    probability is formed as e^s, s in 3 .. 5.5, and rounded."""
    import torch
    import paper_2511_23113_amd as dbsp
    B, d = 12, 64
    s = torch.linspace(3.0, 5.5, B * H * Nq, device="cuda").view(B, H, Nq)
    q = torch.zeros(B, H, Nq, d, device="cuda")
    q[..., 0] = 8 * s                      # (scores are q.k / 8)
    k = torch.zeros(B, 1, cap, d, device="cuda")
    k[:, :, 1:64, 0], k[:, :, 64, 0] = -30.0, 1.0
    v = torch.full((B, 1, cap, d), 65504.0, device="cuda")
    lens = torch.full((B,), 65, dtype=torch.int32, device="cuda")
    o, _ = dbsp.cache_attn_fwd(dbsp.KVCache(k.half(), v.half(), lens), q.half(), causal=False)
    assert bool(torch.isfinite(o).all())
    assert (o.double() / 65504 - 1).abs().max() <= 2 * 2.0 ** -11 * 1.01


def test_infinities_and_nan_in_a_query_stay_its_own():
    """A query that is not finite gets what it gives; the others' rows are those of a call without it, to a rounding."""
    import torch
    import paper_2511_23113_amd as dbsp
    for Nq in (1, 20, 150):
        rng = np.random.default_rng(Nq)
        q, k, v = (torch.from_numpy(rng.normal(size=s)).half().cuda() for s in ((1, 4, Nq, 64), (1, 2, 200, 64), (1, 2, 200, 64)))
        lens = torch.tensor([200], dtype=torch.int32, device="cuda")
        want, want_lse = dbsp.cache_attn_fwd(dbsp.KVCache(k, v, lens), q, causal=False)
        q[0, 1, Nq // 2] = float("nan")
        o, lse = dbsp.cache_attn_fwd(dbsp.KVCache(k, v, lens), q, causal=False)
        assert o[0, 1, Nq // 2].isnan().all()
        o[0, 1, Nq // 2], lse[0, 1, Nq // 2] = want[0, 1, Nq // 2], want_lse[0, 1, Nq // 2]
        # other running maxima: probabilities rounded anew, half a step each, and O
        assert ((o.float() - want.float()).abs() <= 4 * 2.0 ** -11 * v.float().abs().max()).all() and (lse - want_lse).abs().max() <= 1e-5
