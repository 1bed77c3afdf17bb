"""Attention over a key/value cache on the GPU against the float64 oracle: head layouts, lengths, odd sizes, strides, padded
batches, rows without a key, weights; captures, streams, long offsets.

Tolerances, from the arithmetic (h: half a step of the type, relative).  O: every probability is rounded to the type (h A with
A = sum p |v|), O itself too (h |O|); fp16 probabilities below 2^-14 of the running max are off by at most 2^-25 each; scores are
f32 sums of d exact products, off by at most (d + 8) 2^-24 S with S = scale max sum |q k|, which shifts LSE by that and p relative
by twice that.  LSE and W are f32: a few more steps of 2^-24 of their values, and of as many terms as W sums."""

import numpy as np
import pytest

from oracle import cache as oc

pytestmark = pytest.mark.gpu


def torch_types(name):
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16}[name]


def make(B, H, Hk, Nq, d, P, cap, dtype, seed, layout="plain", grow=0.0):
    """q, k, v, prefix_k, prefix_v on the GPU; layouts other than plain are views as projections leave them."""
    import torch
    rng = np.random.default_rng(seed)
    dt = torch_types(dtype)

    def rand(*shape, along=None):
        x = rng.normal(size=shape)
        if along is not None and grow:
            x = x * (1 + grow * np.arange(shape[along]) / shape[along]).reshape([-1 if i == along else 1 for i in range(len(shape))])
        return torch.from_numpy(x).to(dt).cuda()
    if layout == "plain":
        q = rand(B, H, Nq, d)
        k, v = (rand(B, Hk, cap, d, along=2), rand(B, Hk, cap, d)) if cap else (None, None)
        pk, pv = (rand(Hk, P, d), rand(Hk, P, d)) if P else (None, None)
    else:                                  # token-major, K and V of a token side by side, heads of q cut out of a wider projection
        q = rand(B, Nq, H + 2, d)[:, :, 1:H + 1].transpose(1, 2)
        kv = rand(B, max(cap, 1), 2, Hk, d, along=1)
        k, v = (kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2)) if cap else (None, None)
        pkv = rand(max(P, 1), Hk, 2 * d)
        pk, pv = (pkv[..., :d].transpose(0, 1), pkv[..., d:].transpose(0, 1)) if P else (None, None)
    return q, k, v, pk, pv


def host(x):
    return None if x is None else x.double().cpu().numpy()


def check(q, k, v, pk, pv, lens, q_lens, causal, dtype, decay=None, scale=0.0, out_layout="plain", seed=0):
    import torch
    import paper_2511_23113_amd as dbsp
    B, H, Nq, d = q.shape
    Hk, cap = (k.shape[1], k.shape[2]) if k is not None else (pk.shape[0], 0)
    dev_lens = None if k is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    weights = None
    if decay is not None:
        weights = torch.from_numpy(np.random.default_rng(seed + 9).random((B, Hk, cap)).astype(np.float32)).cuda()
        for b in range(B):
            weights[b, :, lens[b]:] = float("nan")       # not in use: never touched
    before = host(weights)
    cache = dbsp.KVCache(k, v, dev_lens, pk, pv, weights=weights)
    o = torch.full((B, Nq, H, d), 7.0, dtype=q.dtype, device="cuda").transpose(1, 2) if out_layout != "plain" else torch.full((B, H, Nq, d), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((B, H, Nq), 7.0, device="cuda")
    dev_q_lens = None if q_lens is None else torch.tensor(q_lens, dtype=torch.int32, device="cuda")
    dbsp.cache_attn_fwd(cache, q, q_lens=dev_q_lens, causal=causal, decay=decay, o=o, lse=lse, softmax_scale=scale)
    torch.cuda.synchronize()
    compare(q, k, v, pk, pv, lens, q_lens, causal, dtype, host(o), host(lse), before, host(weights), decay, scale)
    return o, lse


def compare(q, k, v, pk, pv, lens, q_lens, causal, dtype, got_o, got_lse, before, got_w, decay, scale):
    import torch
    B, H, Nq, d = q.shape
    hq, hk, hv, hpk, hpv = (host(x) for x in (q, k, v, pk, pv))
    s = scale or d ** -0.5
    O, LSE, A, W = oc.cache_attention(hq, lens, hk, hv, hpk, hpv, q_lens, causal, s)
    h = torch.finfo(torch_types(dtype)).eps / 2
    there = ~np.isnan(LSE)
    assert (got_lse[~there] == 7.0).all() and (got_o[~there] == 7.0).all()
    n_keys = (hpk.shape[1] if hpk is not None else 0) + (hk.shape[2] if hk is not None else 0)
    top_k = max([np.abs(x[np.isfinite(x)]).max(initial=0.0) for x in (hpk, hk) if x is not None and x.size] + [0.0])
    score_err = (d + 8) * 2.0 ** -24 * s * np.nanmax(np.abs(np.where(there[..., None], hq, 0)).sum(-1)) * top_k
    none = there & (LSE == -np.inf)
    assert (got_lse[none] == -np.inf).all() and (got_o[none] == 0).all()
    some = there & ~none
    if some.any():
        top_v = max([np.abs(x[np.isfinite(x)]).max(initial=0.0) for x in (hpv, hv) if x is not None and x.size] + [0.0])
        tol = h * (A + np.abs(O)) * (1 + h) + 2 * score_err * A + (n_keys * 2.0 ** -25 * top_v if dtype == "fp16" else 0) + 2.0 ** -20 * A + 2.0 ** -25
        off = np.abs(got_o - O)
        assert (off[some] <= tol[some]).all(), f"O is {np.max((off / tol)[some]):.3g} of its tolerance"
        tol_lse = score_err + 2.0 ** -21 * (1 + np.abs(LSE))
        off = np.abs(np.where(some, got_lse - np.where(some, LSE, 0), 0))
        assert (off[some] <= tol_lse[some]).all(), f"LSE is off by {np.max(off[some]):.3g}, may be {np.min(tol_lse[some]):.3g}"
    if decay is not None:
        rows = Nq * (H // hk.shape[1])
        for b in range(B):
            n = lens[b]
            want = (decay * before[b, :, :n] if decay else 0.0) + W[b, :, :n]
            top_lse = np.abs(LSE[b][some[b]]).max() if some[b].any() else 0.0
            tol = W[b, :, :n] * (2 * score_err + 2.0 ** -21 * (1 + top_lse) + (rows + 8) * 2.0 ** -24) + 4 * 2.0 ** -24 * np.abs(want) + 1e-30
            off = np.abs(got_w[b, :, :n] - want)
            assert (off <= tol).all(), f"weights are {np.max(off / tol):.3g} of their tolerance"
            assert np.isnan(got_w[b, :, n:]).all()


# B, H, Hk, Nq, d, P, cap, lens, q_lens, causal, dtype, decay
CASES = {
    "one_key": (1, 1, 1, 1, 64, 0, 8, [1], None, True, "bf16", 0.0),
    "no_key": (2, 2, 1, 1, 64, 0, 8, [0, 3], None, True, "bf16", 1.0),
    "prefix_only": (3, 4, 2, 1, 128, 65, 0, None, None, True, "fp16", None),
    "prefix_only_one_sequence": (1, 4, 4, 5, 64, 64, 0, None, None, True, "bf16", None),
    "empty_own": (2, 2, 2, 1, 64, 63, 16, [0, 0], [0, 1], True, "bf16", 1.0),
    "tile_borders": (5, 2, 2, 1, 128, 64, 200, [63, 64, 65, 127, 129], None, True, "bf16", 1.0),
    "odd_group": (3, 14, 2, 3, 64, 129, 300, [3, 299, 190], None, True, "fp16", 0.5),
    "rows_129": (2, 3, 1, 43, 128, 100, 90, [43, 90], None, True, "bf16", 1.0),
    "pooled_rows_cross_a_tile": (7, 10, 2, 4, 128, 150, 70, [4, 70, 33, 64, 65, 5, 20], None, True, "fp16", 1.0),
    "padded": (4, 4, 2, 9, 64, 70, 130, [9, 130, 64, 0], [9, 4, 0, 0], True, "bf16", 0.9),
    "more_new_than_used": (3, 2, 2, 9, 64, 0, 32, [3, 9, 0], None, True, "bf16", 1.0),
    "more_new_than_used_prefix": (3, 2, 2, 9, 64, 31, 32, [3, 9, 0], [9, 5, 9], True, "fp16", 0.0),
    "frame": (2, 4, 2, 70, 128, 130, 210, [210, 140], None, False, "bf16", 1.0),
    "prompt": (2, 2, 1, 150, 64, 0, 150, [150, 97], [150, 97], True, "bf16", 1.0),
    "prompt_no_prefix_fp16": (1, 3, 3, 257, 128, 0, 300, [257], None, True, "fp16", 0.0),
    "prompt_rows_from_the_end": (2, 10, 2, 130, 128, 20, 140, [140, 130], [130, 77], True, "fp16", 1.0),
    "prompt_in_parts": (1, 2, 2, 700, 64, 0, 700, [700], None, True, "bf16", None),
    "prompt_after_others": (1, 2, 1, 200, 128, 77, 600, [431], None, True, "bf16", 1.0),
    "prompt_weights_in_parts": (1, 4, 2, 620, 64, 0, 700, [689], None, True, "bf16", 0.5),
    "frame_weights_in_parts": (1, 3, 1, 500, 128, 30, 700, [601], [433], False, "fp16", 1.0),
    "many_sequences": (300, 2, 1, 1, 64, 40, 20, [i % 21 for i in range(300)], None, True, "bf16", 1.0),
    "many_sequences_in_parts": (100, 2, 1, 1, 64, 400, 300, [(7 * i) % 301 for i in range(100)], None, True, "fp16", 0.5),
    "many_rows_in_parts": (40, 8, 2, 16, 64, 300, 60, [16 + i for i in range(40)], [i % 17 for i in range(40)], True, "bf16", 1.0),
    "one_kv_head_of_40": (3, 40, 1, 1, 128, 500, 300, [300, 0, 65], None, True, "bf16", 1.0),
    "one_kv_head_of_200": (2, 200, 1, 1, 64, 70, 300, [300, 129], None, True, "fp16", 1.0),
    "rows_100": (3, 20, 2, 10, 128, 400, 200, [200, 10, 77], [10, 3, 0], True, "bf16", 0.0),
    "frame_in_parts": (1, 2, 2, 300, 128, 2000, 700, [611], None, False, "bf16", 1.0),
    "long_prefix": (2, 4, 2, 1, 64, 5000, 100, [100, 57], None, True, "bf16", 1.0),
    "long_own": (1, 2, 1, 2, 128, 0, 7000, [6999], None, True, "fp16", 1.0),
    "one_head_many_parts": (1, 1, 1, 1, 64, 20000, 1000, [999], None, True, "bf16", 0.3),
}


@pytest.mark.parametrize("layout", ["plain", "views"])
@pytest.mark.parametrize("name", CASES)
def test_against_the_oracle(name, layout):
    B, H, Hk, Nq, d, P, cap, lens, q_lens, causal, dtype, decay = CASES[name]
    seed = 100 + list(CASES).index(name)
    q, k, v, pk, pv = make(B, H, Hk, Nq, d, P, cap, dtype, seed, layout)
    if cap:                                # what is not in use may hold anything
        for b in range(B):
            k[b, :, lens[b]:] = float("nan")
            v[b, :, lens[b]:] = float("inf")
    if q_lens is not None:
        for b in range(B):
            q[b, :, q_lens[b]:] = float("nan")
    check(q, k, v, pk, pv, lens, q_lens, causal, dtype, decay, out_layout=layout, seed=seed)


# Many rows over many slots: the kernel for many queries.  Slots far behind the lengths, row tiles cut into parts and whole ones,
# the longest first or not, rows that end inside a tile.
MANY = {
    "rows_129": (2, 3, 1, 43, 128, 100, 50000, [43, 90], None, True, "bf16", 1.0),
    "frame": (2, 4, 2, 70, 128, 13000, 12000, [210, 140], None, False, "bf16", 1.0),
    "prompt": (2, 2, 1, 150, 64, 0, 70000, [150, 97], [150, 97], True, "bf16", 1.0),
    "no_prefix_fp16": (1, 3, 3, 257, 128, 0, 22000, [22000], None, True, "fp16", 0.0),
    "rows_from_the_end": (2, 10, 2, 130, 128, 20, 8200, [140, 7001], [130, 77], True, "fp16", 1.0),
    "longest_first": (1, 4, 4, 2100, 64, 0, 4200, [2500], None, True, "bf16", None),
    "longest_first_all_slots": (1, 4, 4, 1300, 128, 0, 4700, [4700], [1277], True, "bf16", 0.7),
    "after_others": (1, 2, 1, 200, 128, 48000, 600, [431], None, True, "bf16", 1.0),
    "weights_in_parts": (1, 4, 2, 620, 64, 0, 13500, [689], None, True, "bf16", 0.5),
    "weights_of_all_slots": (1, 4, 2, 620, 64, 0, 13500, [13500], None, True, "fp16", 0.0),
    "frame_weights_in_parts": (1, 3, 1, 500, 128, 15300, 900, [801], [433], False, "fp16", 1.0),
    "one_kv_head_of_200": (2, 200, 1, 1, 64, 65970, 300, [300, 129], None, True, "fp16", 1.0),
    "more_new_than_used": (2, 4, 2, 90, 64, 0, 33000, [70, 0], None, True, "bf16", 1.0),
    "prefix_only": (2, 2, 1, 130, 128, 33000, 0, None, [130, 11], True, "bf16", None),
    "many_sequences": (26, 2, 2, 600, 64, 0, 1100, [600 - 23 * i for i in range(26)], [600 - 23 * i for i in range(26)], True, "bf16", 1.0),
    "many_sequences_behind_a_prefix": (9, 6, 3, 650, 128, 20, 670, [670 - 50 * i for i in range(9)], [max(0, 650 - 90 * i) for i in range(9)], True, "fp16", None),
    "many_sequences_all_see": (9, 6, 3, 650, 128, 20, 670, [670 - 80 * i for i in range(9)], [650 - 60 * i for i in range(9)], False, "bf16", 1.0),
}


@pytest.mark.parametrize("name", MANY)
def test_many_rows_against_the_oracle(name):
    B, H, Hk, Nq, d, P, cap, lens, q_lens, causal, dtype, decay = MANY[name]
    seed = 300 + list(MANY).index(name)
    q, k, v, pk, pv = make(B, H, Hk, Nq, d, P, cap, dtype, seed, "views")
    for b in range(B if cap else 0):
        k[b, :, lens[b]:] = float("nan")
        v[b, :, lens[b]:] = float("inf")
    for b in range(B if q_lens is not None else 0):
        q[b, :, q_lens[b]:] = float("nan")
    check(q, k, v, pk, pv, lens, q_lens, causal, dtype, decay, out_layout="views", seed=seed)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_scores_that_rise_along_many_rows_keys(dtype):
    q, k, v, pk, pv = make(2, 4, 2, 90, 128, 12000, 900, dtype, 71, grow=9.0)
    check(q, k, v, pk, pv, [900, 555], None, True, dtype, 1.0, scale=0.21)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_scores_that_rise_along_the_keys_and_an_explicit_scale(dtype):
    # the running max has to be raised again and again, in the prefix, in the own keys and from part to part
    q, k, v, pk, pv = make(2, 4, 2, 3, 128, 700, 900, dtype, 7, grow=9.0)
    check(q, k, v, pk, pv, [900, 555], None, True, dtype, 1.0, scale=0.21)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_a_key_that_has_most_of_a_rows_attention_costs_no_rounding(dtype, d):
    """The rounding of a probability p_i by a factor 1 + e_i, |e_i| <= h, moves sum p_i v_i / sum p_i by e_i p_i (v_i - O) where both sums are
    of the rounded ones: O is off by at most h sum p_i |v_i - O| and its own rounding, h |O|, not by h sum p_i |v_i|."""
    import torch
    import paper_2511_23113_amd as dbsp
    h = torch.finfo(torch_types(dtype)).eps / 2
    q, k, v, _, _ = make(6, 4, 2, 2, d, 0, 700, dtype, 72)
    q = (q.float() * 4).to(q.dtype)
    lens = torch.tensor([700, 600, 500, 64, 333, 699], dtype=torch.int32, device="cuda")
    o, lse = dbsp.cache_attn_fwd(dbsp.KVCache(k, v, lens), q, causal=False)
    for b in range(6):
        n = int(lens[b])
        kk, vv = (x[b, :, :n].double().cpu().repeat_interleave(2, 0) for x in (k, v))
        x = q[b].double().cpu() @ kk.transpose(1, 2) / d ** 0.5
        P = torch.softmax(x, -1)
        O = P @ vv
        spread = (P[..., None] * (vv[:, None] - O[:, :, None]).abs()).sum(2)
        top = vv.abs().max()
        # scores: f32 sums of d products; fp16: probabilities below its normal range, half a step of 2^-24 each, of a row whose sum is at least 1
        score_err = 4 * d * 2.0 ** -24 * (q[b].double().abs().cpu() @ kk.abs().transpose(1, 2) / d ** 0.5).max()
        tol = h * O.abs() * (1 + 2 * h) + h * (1 + 4 * h) * spread + 2 * score_err * top + (n * 2.0 ** -25 * top if dtype == "fp16" else 0) + 2.0 ** -20 * top
        off = (o[b].double().cpu() - O).abs()
        assert (off <= tol).all(), f"{float((off / tol).max()):.3g} of the tolerance"
        assert (lse[b].double().cpu() - torch.logsumexp(x, -1)).abs().max() <= score_err + 2.0 ** -20 * (1 + x.abs().max())


def test_lengths_out_of_range_are_taken_as_the_nearest_in_range():
    import torch
    import paper_2511_23113_amd as dbsp
    q, k, v, pk, pv = make(3, 2, 2, 4, 64, 10, 16, "bf16", 8)
    outs = []
    for lens, q_lens in (([99, -5, 7], [9, 4, -1]), ([16, 0, 7], [4, 4, 0])):
        o, lse = torch.zeros_like(q), torch.zeros(3, 2, 4, device="cuda")
        cache = dbsp.KVCache(k, v, torch.tensor(lens, dtype=torch.int32, device="cuda"), pk, pv)
        dbsp.cache_attn_fwd(cache, q, q_lens=torch.tensor(q_lens, dtype=torch.int32, device="cuda"), o=o, lse=lse)
        outs.append((o, lse))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_offsets_past_32_bits():
    # tokens 2 MiB apart: 2300 of them reach past 4 GiB
    import torch
    import paper_2511_23113_amd as dbsp
    n, step = 2300, 1 << 20
    buffer = torch.empty(n * step, dtype=torch.bfloat16, device="cuda")
    q, k, v, _, _ = make(1, 2, 1, 1, 64, 0, n, "bf16", 9)
    far_k, far_v = (torch.as_strided(buffer, (1, 1, n, 64), (n * step, 8, step, 1), at) for at in (0, 64))
    far_k.copy_(k)
    far_v.copy_(v)
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    near, far = (dbsp.cache_attn_fwd(dbsp.KVCache(a, b, lens), q) for a, b in ((k, v), (far_k, far_v)))
    assert torch.equal(near[0], far[0]) and torch.equal(near[1], far[1])
    # as a prefix
    near, far = (dbsp.cache_attn_fwd(dbsp.KVCache(prefix_k=a[0], prefix_v=b[0]), q) for a, b in ((k, v), (far_k, far_v)))
    assert torch.equal(near[0], far[0])
    check(q, k, v, None, None, [n], None, True, "bf16")


def test_one_prefix_serves_batches_of_any_size():
    import torch
    import paper_2511_23113_amd as dbsp
    cache = None
    for B, Nq, q_lens in ((1, 3, [2]), (5, 3, [3, 0, 1, 2, 3]), (2, 300, [300, 170])):
        q, _, _, pk, pv = make(B, 4, 2, Nq, 64, 400, 0, "bf16", 13)
        if cache is None:
            keep = pk, pv
            cache = dbsp.KVCache(prefix_k=pk, prefix_v=pv)
        o, lse = torch.full_like(q, 7.0), torch.full((B, 4, Nq), 7.0, device="cuda")
        dbsp.cache_attn_fwd(cache, q, q_lens=torch.tensor(q_lens, dtype=torch.int32, device="cuda"), o=o, lse=lse)
        compare(q, None, None, *keep, None, q_lens, True, "bf16", host(o), host(lse), None, None, None, 0.0)


def test_strides_of_dimensions_of_one_say_nothing():
    import torch
    import paper_2511_23113_amd as dbsp
    q, k, v, pk, pv = make(1, 1, 1, 1, 64, 1, 1, "bf16", 14)
    lens = torch.ones(1, dtype=torch.int32, device="cuda")
    want = dbsp.cache_attn_fwd(dbsp.KVCache(k, v, lens, pk, pv), q)
    odd = [torch.as_strided(x, x.shape, (3,) * (x.dim() - 1) + (1,)) for x in (q, k, v, pk, pv)]
    got = dbsp.cache_attn_fwd(dbsp.KVCache(*odd[1:3], lens, *odd[3:]), odd[0])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_prefix_is_as_good_as_own_keys():
    import torch
    import paper_2511_23113_amd as dbsp
    q, k, v, pk, pv = make(6, 8, 2, 2, 128, 500, 100, "bf16", 11)
    lens = torch.tensor([2, 100, 50, 64, 7, 99], dtype=torch.int32, device="cuda")
    o, lse = dbsp.cache_attn_fwd(dbsp.KVCache(k, v, lens, pk, pv), q)
    both = [torch.cat([p[None].expand(6, -1, -1, -1), x], 2) for p, x in ((pk, k), (pv, v))]
    o2, lse2 = dbsp.cache_attn_fwd(dbsp.KVCache(*both, lens + 500), q)
    # two ways to cut the same sums: probabilities rounded against other running maxima, each half a step, and O itself
    assert (lse - lse2).abs().max() <= 1e-5
    assert ((o.float() - o2.float()).abs() <= 4 * 2.0 ** -8 * (o.float().abs() + v.float().abs().max())).all()


def test_a_batch_that_shares_its_cache_through_stride_zero():
    import torch
    import paper_2511_23113_amd as dbsp
    q, k, v, _, _ = make(1, 2, 2, 1, 64, 0, 90, "bf16", 12)
    qs = torch.cat([q, q + 1, q - 1])
    lens = torch.tensor([90, 33, 1], dtype=torch.int32, device="cuda")
    o, lse = dbsp.cache_attn_fwd(dbsp.KVCache(k.expand(3, -1, -1, -1), v.expand(3, -1, -1, -1), lens), qs)
    for b in range(3):
        ob, lb = dbsp.cache_attn_fwd(dbsp.KVCache(k, v, lens[b:b + 1]), qs[b:b + 1])
        assert (o[b] - ob[0]).abs().max() <= 2 * 2.0 ** -8 * v.abs().max() and (lse[b] - lb[0]).abs().max() <= 1e-5


def _state(seed=21):
    import torch
    q, k, v, pk, pv = make(5, 6, 2, 3, 128, 900, 800, "bf16", seed)
    lens = torch.tensor([800, 3, 444, 0, 65], dtype=torch.int32, device="cuda")
    return q, k, v, lens, pk, pv, torch.rand(5, 2, 800, device="cuda")


def test_the_same_call_gives_the_same_bits():
    import torch
    import paper_2511_23113_amd as dbsp
    q, k, v, lens, pk, pv, w = _state()
    outs = []
    for _ in range(3):
        cache = dbsp.KVCache(k, v, lens, pk, pv, weights=w.clone())
        outs.append((*dbsp.cache_attn_fwd(cache, q, decay=0.5), cache.weights))
    for other in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], other))


def test_a_captured_call_follows_the_lengths_of_each_replay():
    import torch
    import paper_2511_23113_amd as dbsp
    q, k, v, lens, pk, pv, w = _state(22)
    q_lens = torch.tensor([3, 2, 3, 3, 0], dtype=torch.int32, device="cuda")
    cache, other = (dbsp.KVCache(k, v, lens, pk, pv, weights=x) for x in (w.clone(), w.clone()))
    o, lse, o2, lse2 = (torch.zeros(s, dtype=t, device="cuda") for s, t in [((5, 6, 3, 128), torch.bfloat16), ((5, 6, 3), torch.float32)] * 2)
    dbsp.cache_attn_fwd(other, q, q_lens=q_lens, decay=1.0, o=o2, lse=lse2)
    other.weights.copy_(w)
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        dbsp.cache_attn_fwd(cache, q, q_lens=q_lens, decay=1.0, o=o, lse=lse)
    for step in range(4):
        lens.copy_(torch.tensor([[800, 3, 444, 0, 65], [1, 799, 2, 64, 128], [700, 700, 700, 700, 700], [5, 3, 3, 9, 1]][step]))
        q_lens.copy_(torch.tensor([[3, 2, 3, 3, 0], [1, 3, 2, 0, 3], [3, 3, 3, 3, 3], [0, 0, 1, 3, 1]][step]))
        for x in (o, lse, o2, lse2):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        dbsp.cache_attn_fwd(other, q, q_lens=q_lens, decay=1.0, o=o2, lse=lse2)
        torch.cuda.synchronize()
        assert torch.equal(o, o2) and torch.equal(lse, lse2) and torch.equal(cache.weights, other.weights)


def test_two_captured_calls_may_share_a_workspace_that_they_use_in_turn():
    import torch
    import paper_2511_23113_amd as dbsp
    states = [_state(s) for s in (51, 52)]
    caches = [dbsp.KVCache(k, v, lens, pk, pv, weights=w) for q, k, v, lens, pk, pv, w in states]
    ws = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    outs = [(torch.empty_like(s[0]), torch.empty(5, 6, 3, device="cuda")) for s in states]
    graphs = []
    for c, s, (o, lse) in zip(caches, states, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            dbsp.cache_attn_fwd(c, s[0], decay=0.0, o=o, lse=lse, workspace=ws)
    want = [(*dbsp.cache_attn_fwd(c, s[0], decay=0.0), c.weights.clone()) for c, s in zip(caches, states)]
    for step in range(6):
        i = (0, 1, 1, 0, 1, 0)[step]
        outs[i][0].zero_()
        caches[i].weights.zero_()
        graphs[i].replay()
        torch.cuda.synchronize()
        got, used = (*outs[i], caches[i].weights), torch.arange(800, device="cuda") < states[i][3][:, None, None]
        assert torch.equal(got[0], want[i][0]) and torch.equal(got[1], want[i][1]) and torch.equal(got[2] * used, want[i][2] * used)


def test_no_slots_and_no_prefix():
    import torch
    import paper_2511_23113_amd as dbsp
    q, k, v, pk, pv = make(2, 2, 2, 3, 64, 5, 7, "bf16", 15)
    empty, none = torch.empty(2, 2, 0, 64, dtype=q.dtype, device="cuda"), torch.empty(2, 0, 64, dtype=q.dtype, device="cuda")
    lens = torch.tensor([4, 7], dtype=torch.int32, device="cuda")
    for cache, other in ((dbsp.KVCache(empty, empty, lens * 0, pk, pv), dbsp.KVCache(prefix_k=pk, prefix_v=pv)),
                         (dbsp.KVCache(k, v, lens, none, none), dbsp.KVCache(k, v, lens))):
        a, b = dbsp.cache_attn_fwd(cache, q), dbsp.cache_attn_fwd(other, q)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    o, lse = dbsp.cache_attn_fwd(dbsp.KVCache(empty, empty, lens * 0, none, none), q)
    assert (o == 0).all() and (lse == -float("inf")).all()


def test_two_streams_at_once_and_a_stream_by_argument():
    import torch
    import paper_2511_23113_amd as dbsp
    states = [_state(s) for s in (31, 32)]
    caches = [dbsp.KVCache(k, v, lens, pk, pv) for q, k, v, lens, pk, pv, w in states]
    want = [dbsp.cache_attn_fwd(c, s[0]) for c, s in zip(caches, states)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for i in range(2):
            got[i].append(dbsp.cache_attn_fwd(caches[i], states[i][0], stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for o, lse in got[i]:
            assert torch.equal(o, want[i][0]) and torch.equal(lse, want[i][1])


def test_calls_on_two_streams_do_not_share_memory_that_one_of_them_still_uses():
    """What a call takes for itself and gives back when it returns, while its kernels wait, is not what a call on another stream gets."""
    import torch
    import paper_2511_23113_amd as dbsp
    q, k, v, lens, pk, pv, w = _state(33)
    want = dbsp.cache_attn_fwd(dbsp.KVCache(k, v, lens, pk, pv, weights=w), q, decay=0.0)
    caches = [dbsp.KVCache(k, v, lens, pk, pv, weights=torch.zeros_like(w)) for _ in range(2)]
    blocks, got, other, real = [], [], torch.cuda.Stream(), dbsp.KVCache._empty

    def noting(*a):
        x = real(*a)
        blocks.append(x.data_ptr())
        return x

    torch.cuda.synchronize()
    try:
        dbsp.KVCache._empty = noting
        for i in range(6):
            got.append(dbsp.cache_attn_fwd(caches[i % 2], q, decay=0.0, stream=other if i % 2 else None))
    finally:
        dbsp.KVCache._empty = real
    assert len(blocks) == 18 and not {x for i, x in enumerate(blocks) if i // 3 % 2} & {x for i, x in enumerate(blocks) if not i // 3 % 2}
    torch.cuda.synchronize()
    used = torch.arange(800, device="cuda") < lens[:, None, None]
    for o, lse in got:
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    assert all(torch.equal(c.weights * used, w * used) for c in caches)


def test_a_workspace_of_the_caller_and_none_that_is_too_small():
    import torch
    import paper_2511_23113_amd as dbsp
    q, k, v, lens, pk, pv, w = _state(41)
    cache = dbsp.KVCache(k, v, lens, pk, pv)
    want = dbsp.cache_attn_fwd(cache, q)
    ws = torch.full((1 << 28,), 255, dtype=torch.uint8, device="cuda")      # NaNs wherever it is looked at before it is written
    got = dbsp.cache_attn_fwd(cache, q, workspace=ws)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with pytest.raises(dbsp.DbspError, match="the workspace holds 256"):
        dbsp.cache_attn_fwd(cache, q, workspace=ws[:256])


def test_refusals_of_the_binding():
    import torch
    import paper_2511_23113_amd as dbsp
    q, k, v, lens, pk, pv, w = _state(42)
    cache = dbsp.KVCache(k, v, lens, pk, pv)
    for bad in (lambda: dbsp.cache_attn_fwd(cache, q.half()), lambda: dbsp.cache_attn_fwd(cache, q[:4]), lambda: dbsp.cache_attn_fwd(cache, q[..., :64]),
                lambda: dbsp.cache_attn_fwd(cache, q, decay=1.0), lambda: dbsp.cache_attn_fwd(cache, q, o=q[:, :, :1]),
                lambda: dbsp.cache_attn_fwd(cache, q, lse=torch.zeros(5, 6, 3, device="cuda", dtype=torch.float64)),
                lambda: dbsp.cache_attn_fwd(cache, q, q_lens=lens.long()), lambda: dbsp.cache_attn_fwd(cache, q.transpose(2, 3)),
                lambda: dbsp.cache_attn_fwd(cache, q, decay=-1.0), lambda: dbsp.KVCache(k, v[:, :, :9], lens), lambda: dbsp.KVCache(k, v.half(), lens),
                lambda: dbsp.KVCache(k, v, lens.long()), lambda: dbsp.KVCache(k, v, lens, weights=w[:, :, :9]), lambda: dbsp.KVCache(k, v, lens, pk[:1], pv[:1]),
                lambda: dbsp.KVCache(k, v, lens, positions=w), lambda: dbsp.cache_evict(dbsp.KVCache(prefix_k=pk, prefix_v=pv), 4)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(dbsp.DbspError, match="multiple"):
        dbsp.cache_attn_fwd(cache, q[:, :5])
    with pytest.raises(dbsp.DbspError, match="16-byte"):
        dbsp.cache_attn_fwd(cache, torch.empty(5 * 6 * 3 * 128 + 4, dtype=q.dtype, device="cuda")[4:].view(5, 6, 3, 128))
    with pytest.raises(dbsp.DbspError, match="overlap"):
        dbsp.cache_attn_fwd(cache, q, o=torch.empty(5, 6, 1, 128, dtype=q.dtype, device="cuda").expand(-1, -1, 3, -1))
