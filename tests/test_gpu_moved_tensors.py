"""Calls on the GPU with objects whose tensors have been given other memory since they were made: by a module's half() and to(), by an assignment to
.data.  What was there before is overwritten, so a call that still went by it would show."""

import pytest

pytestmark = pytest.mark.gpu


def test_gains_of_a_module():
    import torch
    import paper_2511_23113_amd as dbsp
    torch.manual_seed(0)
    gains = torch.nn.ParameterDict({n: torch.nn.Parameter(1 + 0.2 * torch.randn(64, device="cuda"), requires_grad=False) for n in ("q_gain", "k_gain")})
    q, k, dq, dk = (torch.randn(2, h, 37, 64, device="cuda").bfloat16() for h in (4, 2, 4, 2))
    norm = dbsp.HeadNorm(**gains)

    def both(norm):
        return (*dbsp.qk_norm_rope_fwd(q, k, norm=norm), *dbsp.qk_norm_rope_bwd(q, k, dq, dk, norm=norm))

    def same():
        got, want = both(norm), both(dbsp.HeadNorm(**{n: x.detach().clone() for n, x in gains.items()}))
        assert all(torch.equal(x, y) for x, y in zip(got[:4], want[:4])) and all(torch.equal(got[4][n], want[4][n]) for n in gains)
    same()
    old = [x.detach() for x in gains.values()]
    gains.bfloat16()                       # the rows' type
    for x in old:
        x.fill_(float("nan"))
    same()
    gains.cpu()
    with pytest.raises(ValueError):
        both(norm)
    gains.cuda().float()
    same()
    gains["k_gain"].data = torch.full((64,), 3.0, device="cuda")
    same()
    with torch.no_grad():                  # and in place, as an optimizer's step
        gains["q_gain"].mul_(0.5)
    same()


def test_caches_whose_tensors_move():
    import torch
    import paper_2511_23113_amd as dbsp
    torch.manual_seed(1)
    rand = lambda *s: torch.randn(*s, device="cuda").bfloat16()      # noqa: E731
    of_pages = [rand(12, 2, 16, 64), rand(12, 2, 16, 64), torch.randperm(12, device="cuda").int().view(2, 6), torch.tensor([90, 33], dtype=torch.int32, device="cuda")]
    of_slots = [rand(2, 2, 96, 64), rand(2, 2, 96, 64), torch.tensor([90, 33], dtype=torch.int32, device="cuda")]
    paged, slots, q, k, v = dbsp.PagedKVCache(*of_pages), dbsp.KVCache(*of_slots), rand(2, 4, 1, 64), rand(2, 2, 1, 64), rand(2, 2, 1, 64)
    for x in of_pages + of_slots:
        was = x.detach()
        x.data = x.data.clone()
        was.fill_(-1 if was.dtype == torch.int32 else float("nan"))
        others = [y.clone() for y in of_pages]
        dbsp.paged_append(paged, k, v)
        dbsp.paged_append(dbsp.PagedKVCache(*others), k, v)
        assert all(torch.equal(y, z) for y, z in zip(of_pages, others))
        for got, want in ((dbsp.paged_attn_fwd(paged, q), dbsp.paged_attn_fwd(dbsp.PagedKVCache(*others), q)),
                          (dbsp.cache_attn_fwd(slots, q), dbsp.cache_attn_fwd(dbsp.KVCache(*(y.clone() for y in of_slots)), q))):
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and bool(torch.isfinite(got[1]).all())
