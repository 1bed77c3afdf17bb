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


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H, Nq, cap, P", [(2, 2, 250, 0), (2, 2, 250, 900), (4, 20, 250, 0), (4, 20, 250, 900), (2, 250, 700, 0), (2, 250, 40000, 0)])
def test_scores_as_large_as_they_may_be(H, Nq, cap, P, dtype):
    """Scores of up to 2^26, whole multiples of 2^18 and so exact in f32: a row has the value of its largest score's key.  That key's probability is formed
    against a running max that is rounded to f32, a factor of at most 2^4 for all of the row's keys alike; LSE holds it."""
    import torch
    import paper_2511_23113_amd as dbsp
    B, d, dt = 3, 64, {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
    g = torch.Generator(device="cuda").manual_seed(H * Nq + P)
    sign = torch.where(torch.rand(B, H, Nq, device="cuda", generator=g) < 0.5, -1.0, 1.0)
    q = torch.zeros(B, H, Nq, d, device="cuda")
    q[..., 0] = 256 * sign
    n = 250
    k = torch.zeros(B, 1, cap, d, device="cuda")
    k[:, 0, :n, 0] = torch.stack([torch.randperm(n, device="cuda", generator=g) for _ in range(B)]) + 5.0
    v = torch.randn(B, 1, cap, d, device="cuda", generator=g).to(dt)
    pk, pv = torch.zeros(1, P, d, device="cuda"), torch.randn(1, P, d, device="cuda", generator=g).to(dt)
    pk[..., 0] = 100.0 + torch.arange(P, device="cuda") % 3           # neither the largest nor the smallest
    lens = torch.full((B,), n, dtype=torch.int32, device="cuda")
    cache = dbsp.KVCache(k.to(dt), v, lens, *((pk.to(dt), pv) if P else ()))
    o, lse = dbsp.cache_attn_fwd(cache, q.to(dt), causal=False, softmax_scale=1024.0)
    at = torch.where(sign > 0, k[:, 0, :n, 0].argmax(-1)[:, None, None], k[:, 0, :n, 0].argmin(-1)[:, None, None])
    want = v[torch.arange(B, device="cuda")[:, None, None], 0, at].double()
    top = 2.0 ** 18 * torch.where(sign > 0, n + 4.0, -5.0).double()
    h = torch.finfo(dt).eps / 2
    assert ((o.double() - want).abs() <= 2 * h * want.abs() * (1 + h)).all()
    assert ((lse.double() - top).abs() <= 2.0 ** -22 * top.abs()).all()


@pytest.mark.parametrize("H, Nq, cap", [(2, 2, 300), (2, 2, 3000), (4, 20, 300), (4, 20, 3000), (2, 250, 300), (2, 250, 40000)])
def test_bf16_values_of_up_to_2_to_the_80(H, Nq, cap):
    """f32 sums of 40,000 keys' values, with probabilities of up to 2^10 before they are divided by their sum, stay below 2^106."""
    import torch
    import paper_2511_23113_amd as dbsp
    g = torch.Generator(device="cuda").manual_seed(cap)
    q, k = (torch.randn(2, n, m, 64, device="cuda", generator=g).bfloat16() for n, m in ((H, Nq), (1, cap)))
    v = torch.full((2, 1, cap, 64), 2.0 ** 80, device="cuda").bfloat16()
    lens = torch.full((2,), cap, dtype=torch.int32, device="cuda")
    o, _ = dbsp.cache_attn_fwd(dbsp.KVCache(k, v, lens), q, causal=False)
    assert (o.double() / 2.0 ** 80 - 1).abs().max() <= 2 * 2.0 ** -8 * 1.01
