"""Norms and rotations of queries and keys on the GPU, and their gradients, against the float64 oracle: norms, axes, pairings, head layouts,
strides, sizes from one token on, in place, on other streams, in graphs.

Tolerances, from the arithmetic (u = 2^-24, h half a step of the rows' type, relative).  The sum of d <= 128 squares is of non-negative f32 terms, at
most 4 + 5 additions deep: with the factor 1 / d, eps and the reciprocal root (one unit, 2u) r is off by at most (10 / 2 + 1 + 2) u < 16 u, so
x r by 17 u of itself.  With a mean, that is off by at most 12 u mean|x|, which shifts (x - mu) r by 13 u mean|x| r =: s, and r by 2 s at
most, relative.  Gain and bias: 2 u of each term.  Angles are off by 2^-52 |position freq| (two products of 64 bits) and, in turns, by half an
f32 step below 1 / 2 (2 pi 2^-26); sine and cosine by four units more (4 u, math library): 2^-21 + 2^-51 |position freq| in all.  A pair's
results are off by the sum of its values' errors and by that times the sum of their sizes, and 3 u of it from products and sum.
The result is rounded once: h of it, in fp16 at least half of 2^-24."""

import numpy as np
import pytest

from oracle import rows as orows

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-6


def torch_types(name):
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16}[name]


def host(x):
    return x.double().cpu().numpy()


def half_step(dtype, y):
    import torch
    return torch.finfo(torch_types(dtype)).eps / 2 * np.abs(y) + (2.0 ** -25 if dtype == "fp16" else 0.0)


def pair_sum(x, R, halves):
    """At a pair's places the sum over both."""
    y = np.array(x, copy=True)
    i, j = orows.pair_places(R, halves)
    y[..., i] = y[..., j] = x[..., i] + x[..., j]
    return y


def angle_error(a, d, halves):
    """At every place."""
    e = np.zeros(a.shape[:-1] + (d,))
    i, j = orows.pair_places(a.shape[-1], halves)
    e[..., i] = e[..., j] = 2.0 ** -21 + 2.0 ** -51 * np.abs(a)
    return e


def hat_error(x, hat, r, kind):
    if kind == "rms":
        return 17 * U * np.abs(hat)
    s = 13 * U * np.abs(x).mean(-1, keepdims=True) * r
    return 17 * U * np.abs(hat) + s * (1 + 2 * np.abs(hat))


def fwd_tolerance(x, y, kind, gain, bias, a, halves, dtype):
    if kind == "none":
        size, err = np.abs(x), np.zeros_like(x)
    else:
        hat, r = orows.normed(x, kind, EPS)
        size = np.abs(hat * gain) + np.abs(bias)
        err = hat_error(x, hat, r, kind) * np.abs(gain) + 2 * U * size
    if a is not None:
        R, d = a.shape[-1], x.shape[-1]
        err, size = pair_sum(err, R, halves), pair_sum(size, R, halves)
        err = err * (1 + 2.0 ** -20) + (angle_error(a, d, halves) + 3 * U) * size
    return half_step(dtype, np.abs(y) + err) + err


def make(case, seed=0):
    """The case's tensors on the GPU, as views into a projection's output where `fused`."""
    import torch
    import paper_2511_23113_amd as dbsp
    rng = np.random.default_rng(seed)
    B, N, H, Hk, d, dt = case["B"], case["N"], case["H"], case["Hk"], case["d"], torch_types(case["dtype"])

    def rand(*shape, scale=1.0):
        return torch.from_numpy(rng.normal(size=shape) * scale).to(dt).cuda()
    if case["fused"]:
        x = rand(B, N, H + 2 * Hk + 1, d)
        q, k = x[:, :, 1:H + 1].transpose(1, 2), x[:, :, H + 1:H + 1 + Hk].transpose(1, 2) if Hk else None
    else:
        q, k = rand(B, H, N, d), rand(B, Hk, N, d) if Hk else None
    gains = {}
    if case["kind"] != "none":
        names = [n for n in case["gains"].split(",") if n]
        wide = torch.float32 if case["wide"] else dt
        gains = {n: torch.from_numpy(rng.normal(size=d) * 0.3 + (1.0 if n.endswith("gain") else 0.0)).to(wide).cuda() for n in names}
    norm = None if case["kind"] == "none" else dbsp.HeadNorm(kind=case["kind"], eps=EPS, **gains)
    rotary = dbsp.Rotary(case["pairs"], halves=case["halves"]) if case["pairs"] else None
    positions = None
    if case["pairs"] and case["pos"] != "none":
        shape = (B, N, len(case["pairs"])) if case["pos"] == "each" else (N, len(case["pairs"]))
        positions = torch.from_numpy(rng.integers(-5, case.get("far", 3000), size=shape).astype(np.int32)).cuda()
    return dict(q=q, k=k, gains=gains, norm=norm, rotary=rotary, positions=positions, rand=rand)


def host_angles(case, s):
    if not case["pairs"]:
        return None
    B, N = case["B"], case["N"]
    pos = np.arange(N)[:, None] if s["positions"] is None else s["positions"].cpu().numpy()
    if pos.ndim == 2:
        pos = np.broadcast_to(pos, (B,) + pos.shape)
    return orows.angles(pos, case["pairs"], s["rotary"].freqs)[:, None]          # [B, 1, N, R]


def gain_of(s, name, d, none):
    x = s["gains"].get(name)
    return np.full(d, none) if x is None else host(x)


def C(B=1, N=1, H=1, Hk=1, d=64, dtype="bf16", kind="rms", gains="q_gain,k_gain", wide=True, pairs=(32,), halves=False, pos="shared", fused=True, **more):
    return dict(B=B, N=N, H=H, Hk=Hk, d=d, dtype=dtype, kind=kind, gains=gains, wide=wide, pairs=pairs, halves=halves, pos=pos, fused=fused, **more)


ALL = "q_gain,k_gain,q_bias,k_bias"
CASES = {
    "one_token": C(),
    "one_token_halves": C(halves=True, dtype="fp16", d=128, pairs=(64,), pos="none"),
    "no_keys": C(N=37, H=3, Hk=0, gains="q_gain", pos="none"),
    "rotation_alone": C(B=2, N=19, H=5, Hk=2, d=128, kind="none", pairs=(16, 24, 24)),
    "rotation_alone_halves": C(B=2, N=19, H=5, Hk=2, kind="none", pairs=(6, 10, 12), halves=True, dtype="fp16", pos="each"),
    "norm_alone": C(B=3, N=33, H=2, Hk=1, kind="layer", gains=ALL, pairs=None, wide=False),
    "neither": C(B=2, N=5, H=3, Hk=3, kind="none", pairs=None),
    "three_axes": C(B=1, N=211, H=7, Hk=7, d=128, pairs=(22, 21, 21), pos="shared"),
    "four_axes_some_places": C(B=2, N=65, H=9, Hk=3, d=128, pairs=(3, 5, 7, 11), dtype="fp16", pos="each", wide=False),
    "some_places_halves": C(B=2, N=65, H=9, Hk=3, pairs=(3, 5, 4), halves=True, kind="layer", gains=ALL, dtype="bf16", pos="each"),
    "one_pair": C(N=7, H=2, Hk=2, pairs=(1,), d=64, pos="none"),
    "no_gains": C(N=50, H=4, Hk=2, gains="", kind="layer", dtype="fp16"),
    "biases_alone": C(N=50, H=4, Hk=2, gains="q_bias,k_bias", kind="rms", wide=False, dtype="fp16"),
    "q_gain_alone": C(N=50, H=4, Hk=2, gains="q_gain", kind="rms"),
    "plain_layout": C(B=2, N=129, H=3, Hk=1, d=128, pairs=(64,), fused=False, halves=True),
    "far_positions": C(N=40, H=2, Hk=2, d=128, pairs=(32, 32), far=2 ** 31 - 1, pos="each"),
    "many_heads": C(B=1, N=3, H=130, Hk=65, d=64, pairs=(8, 12, 12), halves=True),
    "many_tokens": C(B=2, N=1500, H=3, Hk=2, d=64, kind="layer", gains=ALL, pairs=(8, 12, 12), dtype="fp16"),
    # more heads than a workgroup's share, and a share that no group's heads divide
    "dealt_heads": C(B=1, N=2500, H=11, Hk=5, d=128, pairs=(22, 21, 21)),
}


def run_fwd(case, s, **out):
    import paper_2511_23113_amd as dbsp
    return dbsp.qk_norm_rope_fwd(s["q"], s["k"], norm=s["norm"], rotary=s["rotary"], positions=s["positions"], **out)


@pytest.mark.parametrize("name", CASES)
def test_forward(name):
    import torch
    case = CASES[name]
    s = make(case)
    got = run_fwd(case, s)
    torch.cuda.synchronize()
    a, d = host_angles(case, s), case["d"]
    for x, y, which in ((s["q"], got[0], "q"), (s["k"], got[1], "k")):
        if x is None:
            assert y is None
            continue
        gain, bias = gain_of(s, which + "_gain", d, 1.0), gain_of(s, which + "_bias", d, 0.0)
        want = orows.rows_fwd(host(x), case["kind"], gain, bias, EPS, a, case["halves"])
        tol = fwd_tolerance(host(x), want, case["kind"], gain, bias, a, case["halves"], case["dtype"])
        assert y.is_contiguous() and y.dtype == x.dtype
        off = np.abs(host(y) - want)
        assert (off <= tol).all(), f"{which} is {np.max(off / tol):.3g} of its tolerance"
    if case["kind"] == "none" and not case["pairs"]:
        assert torch.equal(got[0], s["q"])


@pytest.mark.parametrize("name", [n for n in CASES if n not in ("neither",)])
def test_backward(name):
    import torch
    import paper_2511_23113_amd as dbsp
    case = CASES[name]
    s = make(case)
    B, N, H, Hk, d, kind = (case[n] for n in ("B", "N", "H", "Hk", "d", "kind"))
    dq_out, dk_out = s["rand"](B, H, N, d), s["rand"](B, Hk, N, d) if Hk else None
    if case["fused"]:                      # the gradient of a projection's output, of which other parts stay as they are
        whole = torch.full((B, N, H + 2 * Hk + 1, d), 7.0, dtype=s["q"].dtype, device="cuda")
        dq, dk = whole[:, :, 1:H + 1].transpose(1, 2), whole[:, :, H + 1:H + 1 + Hk].transpose(1, 2) if Hk else None
    else:
        dq = dk = None
    dq, dk, gains = dbsp.qk_norm_rope_bwd(s["q"], s["k"], dq_out, dk_out, norm=s["norm"], rotary=s["rotary"], positions=s["positions"], dq=dq, dk=dk)
    again = dbsp.qk_norm_rope_bwd(s["q"], s["k"], dq_out, dk_out, norm=s["norm"], rotary=s["rotary"], positions=s["positions"])
    torch.cuda.synchronize()
    assert set(gains) == set(s["gains"]) and torch.equal(dq, again[0]) and all(torch.equal(gains[n], again[2][n]) for n in gains)
    if case["fused"]:
        assert (whole[:, :, 0] == 7).all() and (whole[:, :, H + 1 + Hk:] == 7).all()
    a = host_angles(case, s)
    for x, dy, dx, which in ((s["q"], dq_out, dq, "q"), (s["k"], dk_out, dk, "k")):
        if x is None:
            continue
        gain = gain_of(s, which + "_gain", d, 1.0)
        x, dy = host(x), host(dy)
        want, want_gain, want_bias = orows.rows_bwd(x, dy, kind, gain, EPS, a, case["halves"])
        # dn is off by the angles' errors; then, term by term, what the formula makes of it and of the errors of x r and r
        if a is None:
            dn, dn_err = np.abs(dy), np.zeros_like(dy)
        else:
            dn = np.abs(orows.rotate(dy, -a, case["halves"]))
            dn_err = (angle_error(a, d, case["halves"]) + 3 * U) * pair_sum(np.abs(dy), a.shape[-1], case["halves"])
        if kind == "none":
            err = dn_err
        else:
            hat, r = orows.normed(x, kind, EPS)
            hat_err, hat = hat_error(x, hat, r, kind), np.abs(hat)
            r_err = 16 * U + (2 * 13 * U * np.abs(x).mean(-1, keepdims=True) * r if kind == "layer" else 0.0)
            e, e_err = dn * np.abs(gain), dn_err * np.abs(gain) + U * dn * np.abs(gain)
            mean = lambda y: y.mean(-1, keepdims=True)      # noqa: E731
            along, along_err = mean(e * hat), mean(e_err * hat + e * hat_err) + 16 * U * mean(e * hat)
            m0, m0_err = (mean(e), mean(e_err) + 16 * U * mean(e)) if kind == "layer" else (0.0, 0.0)
            size = e + along * hat + m0
            err = r * (e_err + along * hat_err + along_err * hat + m0_err + (r_err + 4 * U) * size) * (1 + 2.0 ** -10)
        tol = half_step(case["dtype"], np.abs(want) + err) + err
        off = np.abs(host(dx) - want)
        assert (off <= tol).all(), f"d{which} is {np.max(off / tol):.3g} of its tolerance"
        if kind == "none":
            continue
        # sums: a lane's in turn, then a tree and the workgroups' partial sums, in any case no deeper than all rows and 32 additions
        rows = x[..., 0].size
        for what, found, terms, terms_err in (("gain", want_gain, dn * hat, dn_err * hat + dn * hat_err), ("bias", want_bias, dn, dn_err)):
            if f"{which}_{what}" in gains:
                tol = (terms_err + U * terms).sum((0, 1, 2)) + (rows + 32) * U * terms.sum((0, 1, 2)) + 1e-30
                off = np.abs(host(gains[f"{which}_{what}"]) - found)
                assert (off <= tol).all(), f"{which}_{what} is {np.max(off / tol):.3g} of its tolerance"


@pytest.mark.parametrize("kind, halves", [("rms", False), ("layer", True)])
def test_gradients_against_differences(kind, halves):
    # of the sum of products with dy, formed in float64 from the forward kernel's results: both sides' roundings at the places that differ, and
    # what a difference over so wide a step is off by itself, which the float64 definition tells
    import torch
    import paper_2511_23113_amd as dbsp
    case = C(N=2, H=1, Hk=1, d=64, dtype="fp16", kind=kind, gains=ALL, pairs=(8, 12, 12), halves=halves, fused=False)
    s = make(case, seed=5)
    dq_out, dk_out = s["rand"](1, 1, 2, 64), s["rand"](1, 1, 2, 64)
    dq, _, gains = dbsp.qk_norm_rope_bwd(s["q"], s["k"], dq_out, dk_out, norm=s["norm"], rotary=s["rotary"], positions=s["positions"])
    dy, a = host(dq_out), host_angles(case, s)

    def slope(up, down, span):
        y = [host(run_fwd(case, dict(s, q=x))[0]) for x in (up, down)]
        rounding = np.where(y[0] != y[1], np.abs(dy) * (half_step("fp16", y[0]) + half_step("fp16", y[1])) * 1.1, 0).sum() / span
        return ((y[0] - y[1]) * dy).sum() / span, rounding

    def exact(x):
        return (orows.rows_fwd(host(x), kind, host(s["gains"]["q_gain"]), host(s["gains"]["q_bias"]), EPS, a, halves) * dy).sum()
    want = orows.rows_bwd(host(s["q"]), dy, kind, host(s["gains"]["q_gain"]), EPS, a, halves)[0]
    for at in np.abs(want).ravel().argsort()[-4:]:
        up, down = s["q"].clone(), s["q"].clone()
        up.view(-1)[at] += 0.5
        down.view(-1)[at] -= 0.5
        span = float(up.view(-1)[at].double() - down.view(-1)[at].double())
        found, rounding = slope(up, down, span)
        wide = abs((exact(up) - exact(down)) / span - want.ravel()[at])
        g = float(dq.reshape(-1)[at])
        assert rounding + wide < 0.5 * abs(g)
        assert abs(found - g) <= rounding + wide + half_step("fp16", abs(g)) * 1.1
    for name in ("q_gain", "q_bias"):
        old = s["gains"][name][9].clone()
        both = []
        for sign in (1, -1):
            s["gains"][name][9] = old + sign * 0.5
            both.append(host(run_fwd(case, s)[0]))
        s["gains"][name][9] = old
        rounding = np.where(both[0] != both[1], np.abs(dy) * (half_step("fp16", both[0]) + half_step("fp16", both[1])) * 1.1, 0).sum()
        assert abs(((both[0] - both[1]) * dy).sum() - float(gains[name][9])) <= rounding + 1e-4


@pytest.mark.parametrize("halves", [False, True])
def test_in_place(halves):
    import torch
    import paper_2511_23113_amd as dbsp
    case = C(B=2, N=70, H=6, Hk=3, d=128, pairs=(16, 20), halves=halves)
    s = make(case)
    want = run_fwd(case, s)
    dy = s["rand"](2, 6, 70, 128), s["rand"](2, 3, 70, 128)
    want_back = dbsp.qk_norm_rope_bwd(s["q"], s["k"], *dy, norm=s["norm"], rotary=s["rotary"], positions=s["positions"])
    dq, dk, gains = dbsp.qk_norm_rope_bwd(s["q"], s["k"], *dy, norm=s["norm"], rotary=s["rotary"], positions=s["positions"], dq=dy[0], dk=dy[1])
    assert torch.equal(dq, want_back[0]) and torch.equal(dk, want_back[1]) and torch.equal(gains["k_gain"], want_back[2]["k_gain"])
    got = run_fwd(case, s, q_out=s["q"], k_out=s["k"])
    assert got[0] is s["q"] and torch.equal(s["q"], want[0]) and torch.equal(s["k"], want[1])


def test_infinite_rows_spoil_no_other():
    import torch
    case = C(N=40, H=3, Hk=2, d=64, fused=False)
    s = make(case)
    want = run_fwd(case, s)
    s["q"][0, 1, 7, 3], s["k"][0, 0, 39, 0] = float("inf"), float("nan")
    got = run_fwd(case, s)
    rest = torch.ones(3, 40, dtype=torch.bool, device="cuda")
    rest[1, 7] = False
    assert torch.equal(got[0][0][rest], want[0][0][rest]) and torch.equal(got[1][0, :, :39], want[1][0, :, :39])


def test_zero_rows_and_large_ones():
    import torch
    case = C(N=3, H=1, Hk=1, d=64, dtype="fp16", kind="rms", gains="", fused=False)
    s = make(case)
    s["q"][0, 0, 0], s["q"][0, 0, 1] = 0, 60000.0
    got = run_fwd(case, s)[0]
    assert (got[0, 0, 0] == 0).all() and torch.isfinite(got).all()
    np.testing.assert_allclose((host(got)[0, 0, 1] ** 2).sum(), 64, rtol=64 * 2.0 ** -11)


@pytest.mark.parametrize("pairs, halves", [((22, 21, 21), False), ((22, 21, 21), True), ((20, 21, 11), True)])
def test_large_tensors_are_their_pieces(pairs, halves):
    # 40 + 40 heads of 14,001 tokens (573 MB in and out, past the caches where lines are stored whole) against thirds of them, which go through the caches: the same bits
    import torch
    import paper_2511_23113_amd as dbsp
    N, d = 14001, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(1, N, 80, d, device="cuda", generator=g).bfloat16()
    dy = torch.randn(1, 80, N, d, device="cuda", generator=g).bfloat16()
    norm = dbsp.HeadNorm(*(1 + 0.1 * torch.randn(2, d, device="cuda", generator=g)))
    rotary = dbsp.Rotary(pairs, halves=halves)
    pos = torch.randint(0, 100, (N, 3), device="cuda", generator=g, dtype=torch.int32)

    def both(a, b):
        q, k = x[:, a:b, :40].transpose(1, 2), x[:, a:b, 40:].transpose(1, 2)
        more = dict(norm=norm, rotary=rotary, positions=pos[a:b])
        return (*dbsp.qk_norm_rope_fwd(q, k, **more), *dbsp.qk_norm_rope_bwd(q, k, dy[:, :40, a:b], dy[:, 40:, a:b], **more))
    whole, third = both(0, N), N // 3
    sums = {"q_gain": 0, "k_gain": 0}
    for a in range(0, N, third):
        part = both(a, a + third)
        for i in range(4):
            assert torch.equal(whole[i][:, :, a:a + third], part[i])
        for name in sums:
            sums[name] = sums[name] + part[4][name].double()
    # sums of 560,040 terms |dn xh| of 0.64 on average: two tiles of 40 heads a lane, 2 + 4 additions of lanes and waves, 8 + 6 of the 512
    # workgroups' sums, less than 128 in all for a term on either side
    for name in sums:
        assert float((whole[4][name].double() - sums[name]).abs().max()) <= 2 * 128 * U * 560040 * 0.8


def test_strides_past_32_bits():
    import torch
    import paper_2511_23113_amd as dbsp
    # two sequences more than 2^32 bytes apart: one tensor of 11 GB, of which little is touched
    whole = torch.empty(2, 5 << 29, dtype=torch.bfloat16, device="cuda")
    q = whole.as_strided((2, 2, 9, 64), (5 << 29, 64, 128, 1))
    q.copy_(torch.randn(2, 2, 9, 64, device="cuda"))
    rotary = dbsp.Rotary((32,))
    want = dbsp.qk_norm_rope_fwd(q.contiguous(), rotary=rotary)[0]
    assert torch.equal(dbsp.qk_norm_rope_fwd(q, rotary=rotary)[0], want)
    dbsp.qk_norm_rope_fwd(q, rotary=rotary, q_out=q)
    assert torch.equal(q, want)


def test_other_streams_and_graphs():
    import torch
    import paper_2511_23113_amd as dbsp
    case = C(B=2, N=600, H=4, Hk=2, d=64, kind="layer", gains=ALL, pairs=(8, 12, 12))
    s = make(case)
    dy = s["rand"](2, 4, 600, 64), s["rand"](2, 2, 600, 64)
    more = dict(norm=s["norm"], rotary=s["rotary"], positions=s["positions"])

    def both(**kw):
        return (*dbsp.qk_norm_rope_fwd(s["q"], s["k"], **more, **kw), *dbsp.qk_norm_rope_bwd(s["q"], s["k"], *dy, **more, **kw))

    def same(x, y):
        return all(torch.equal(i, j) for i, j in zip(x[:4], y[:4])) and all(torch.equal(x[4][n], y[4][n]) for n in y[4])
    want = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream, torch.cuda.default_stream(), 0):
        with torch.cuda.stream(torch.cuda.Stream()):
            got = both(stream=stream)
        torch.cuda.synchronize()
        assert same(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for i in range(3):
        s["q"].mul_(1.5 if i else 1.0)
        s["positions"].add_(i)
        s["gains"]["q_gain"].add_(0.25 * i)
        for x in got[:4]:
            x.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert same(got, both())
        torch.cuda.synchronize()


def test_two_calls_at_once():
    import torch
    import paper_2511_23113_amd as dbsp
    case = C(B=1, N=3000, H=8, Hk=4, d=128, kind="rms", pairs=(64,))
    s = [make(case, seed=i) for i in range(2)]
    dy = [(x["rand"](1, 8, 3000, 128), x["rand"](1, 4, 3000, 128)) for x in s]

    def call(i, **kw):
        return dbsp.qk_norm_rope_bwd(s[i]["q"], s[i]["k"], *dy[i], norm=s[i]["norm"], rotary=s[i]["rotary"], positions=s[i]["positions"], **kw)
    want = [call(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = [call(i, stream=streams[i]) for i in range(2)]
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1]) and all(torch.equal(x[2][n], y[2][n]) for n in y[2])


def test_refusals_on_the_gpu():
    import torch
    import paper_2511_23113_amd as dbsp
    q, k = torch.zeros(2, 4, 9, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, 9, 64, dtype=torch.bfloat16, device="cuda")
    rotary = dbsp.Rotary((8, 12, 12))
    pos = torch.zeros(9, 3, dtype=torch.int32, device="cuda")
    for bad in (dict(k=k[:1]), dict(k=k.half()), dict(k=k[:, :, :8]), dict(q_out=k), dict(k_out=k), dict(positions=pos.long()), dict(positions=pos[:8]),
                dict(positions=pos[:, :2]), dict(positions=pos.cpu()), dict(positions=pos[None].repeat(3, 1, 1)),
                dict(norm=dbsp.HeadNorm(torch.ones(128, device="cuda"))), dict(norm=dbsp.HeadNorm(torch.ones(64, device="cuda").half()))):
        with pytest.raises(ValueError):
            dbsp.qk_norm_rope_fwd(q, rotary=rotary, **{"positions": pos, **bad})
    with pytest.raises(ValueError):
        dbsp.HeadNorm(torch.ones(64, device="cuda"), torch.ones(64, device="cuda").half())
    with pytest.raises(ValueError):
        dbsp.qk_norm_rope_fwd(q[..., ::2], rotary=rotary, positions=pos)
    with pytest.raises(dbsp.DbspError, match="positions"):
        dbsp.qk_norm_rope_fwd(q, rotary=rotary)
    with pytest.raises(dbsp.DbspError, match="head dim"):
        dbsp.qk_norm_rope_fwd(q[..., :32])
    with pytest.raises(ValueError):
        dbsp.qk_norm_rope_bwd(q, k, q, None)
    with pytest.raises(ValueError):
        dbsp.qk_norm_rope_bwd(q, None, q, k)
    with pytest.raises(dbsp.DbspError, match="overlap"):
        dbsp.qk_norm_rope_fwd(q, q_out=q[:1].expand(2, 4, 9, 64))
