"""Places of a head that the rotation does not turn: they keep their values, whatever these are, and do not touch their neighbours'."""

import pytest

pytestmark = pytest.mark.gpu

# d, pairs, halves: turned places end inside those of a lane or between lanes
LAYOUTS = [(64, (3, 5), False), (64, (8, 12), False), (128, (61,), False), (128, (20, 12), True), (64, (4,), True)]
BAD = [float("inf"), float("-inf"), float("nan")]


def places(d, pairs, halves):
    """Unturned ones: the first, one amid, the last."""
    R = sum(pairs)
    return 2 * R, (2 * R + d) // 2, d - 1


def make(d, dtype, seed=0):
    import torch
    torch.manual_seed(seed)
    q, k = (torch.randn(2, h, 19, d, device="cuda").to(dtype) for h in (3, 1))
    return q, k


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("d, pairs, halves", LAYOUTS)
def test_without_a_norm_they_are_copied(d, pairs, halves, dtype):
    import torch
    import paper_2511_23113_amd as dbsp
    q, k = make(d, getattr(torch, dtype))
    rotary = dbsp.Rotary(pairs, halves=halves)
    pos = torch.randint(0, 99, (19, len(pairs)), device="cuda", dtype=torch.int32)
    R = sum(pairs)
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    lens = torch.full((2,), 19, dtype=torch.int32, device="cuda")

    def call(q, k):
        pool = torch.zeros(2, 4, 1, 16, d, dtype=k.dtype, device="cuda")
        q_out = dbsp.paged_append(dbsp.PagedKVCache(pool[0], pool[1], table, lens), k, k, q=q, rotary=rotary, positions=pos)
        return (*dbsp.qk_norm_rope_fwd(q, k, rotary=rotary, positions=pos), *dbsp.qk_norm_rope_bwd(q, k, q, k, rotary=rotary, positions=pos)[:2], q_out,
                pool[0].view(2, 1, 32, d)[:, :, :19])
    want = call(q, k)
    bad_q, bad_k = q.clone(), k.clone()
    for i, at in enumerate(places(d, pairs, halves)):
        bad_q[1, 2, 5 + i, at] = bad_k[0, 0, 7 + i, at] = BAD[i]
    for x, y, z in zip((bad_q, bad_k) * 3, call(bad_q, bad_k), want):
        same = x.view(torch.int16) == y.view(torch.int16)
        assert bool(same[..., 2 * R:].all())
        off = torch.isfinite(x)
        assert torch.equal(y[off], z[off])


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("d, pairs, halves", LAYOUTS)
def test_gains_and_gradients_beside_them(d, pairs, halves, kind):
    import torch
    import paper_2511_23113_amd as dbsp
    q, k = make(d, torch.bfloat16)
    gains = {n: 1 + 0.2 * torch.randn(d, device="cuda") for n in ("q_gain", "k_gain", "q_bias", "k_bias")}
    rotary = dbsp.Rotary(pairs, halves=halves)
    pos = torch.randint(0, 99, (19, len(pairs)), device="cuda", dtype=torch.int32)
    more = dict(norm=dbsp.HeadNorm(**gains, kind=kind), rotary=rotary, positions=pos)
    for at in places(d, pairs, halves):
        others = torch.arange(d, device="cuda") != at
        # gains and biases that are no numbers there
        want = dbsp.qk_norm_rope_fwd(q, k, **more)
        for name in gains:
            was = gains[name][at].clone()
            for bad in BAD:
                gains[name][at] = bad
                got = dbsp.qk_norm_rope_fwd(q, k, **more)
                assert all(torch.equal(x[..., others], y[..., others]) for x, y in zip(got, want))
                assert not bool(torch.isfinite(got[name[0] == "k"][..., at]).any())
            gains[name][at] = was
        # gradients that are none there: those of the other places' gains and biases are what they were
        dy = make(d, torch.bfloat16, seed=1)
        want = dbsp.qk_norm_rope_bwd(q, k, *dy, **more)[2]
        for bad in BAD:
            for x in dy:
                x[1, 0, 11, at] = bad
            got = dbsp.qk_norm_rope_bwd(q, k, *dy, **more)[2]
            assert all(torch.equal(got[n][others], want[n][others]) and not torch.isfinite(got[n][at]) for n in gains)
