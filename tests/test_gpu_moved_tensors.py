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
