"""The paged key/value cache on the GPU against the float64 oracle: appending with norm and rotation on the way, and attention of new tokens, over
pages of any size, in any order, some of them none; ragged and empty sequences; strides, streams, graphs, and both together.

Tolerances.  Appended keys and rotated queries: those of the forward pass of norms and rotations; values and everything else bit for bit.
Attention, with h half a step of the type, relative: every probability is rounded to the type (h A with A = sum p |v|), O itself too (h |O|); fp16
probabilities below 2^-14 of the running max are off by at most 2^-25 each; scores are f32 sums of d exact products, off by at most
(d + 8) 2^-24 S with S = scale max sum |q k|, which shifts LSE by that and p relative by twice that.  LSE is f32: a few more steps of
2^-24 of its value, and of as many terms."""

import numpy as np
import pytest

from oracle import rows as orows
from test_gpu_rows import ALL, EPS, fwd_tolerance, host, torch_types

pytestmark = pytest.mark.gpu


def pool_of(n_pages, Hk, page, d, dtype, rng, layout):
    """K and V of a pool, of any layout, with NaN wherever nothing has been written."""
    import torch
    dt = torch_types(dtype)
    if layout == "heads":                  # [n_pages, Hk, page, d]
        k, v = (torch.full((n_pages, Hk, page, d), float("nan"), dtype=dt, device="cuda") for _ in range(2))
    elif layout == "slots":                # [n_pages, page, Hk, d]
        k, v = (torch.full((n_pages, page, Hk, d), float("nan"), dtype=dt, device="cuda").transpose(1, 2) for _ in range(2))
    else:                                  # K and V of a page side by side, and something behind each slot
        x = torch.full((n_pages, 2, page, Hk, d + 8), float("nan"), dtype=dt, device="cuda")
        k, v = x[:, 0, :, :, :d].transpose(1, 2), x[:, 1, :, :, :d].transpose(1, 2)
    return k, v


def table_of(B, per, n_pages, lens, page, rng, gone=(), wide=0):
    """int32 [B, per] on the GPU, the sequences' pages in random order; entries behind the length, and (b, i) of `gone`, are no pages."""
    import torch
    t = rng.permutation(n_pages)[:B * per].reshape(B, per).astype(np.int32)
    for b in range(B):
        t[b, -(-max(lens[b], 0) // page):] = [-1, n_pages, 2 ** 31 - 1, -2 ** 31][b % 4]
    for i, (b, at) in enumerate(gone):
        t[b, at] = [-1, n_pages, -7, 2 ** 31 - 1][i % 4]
    whole = torch.full((B, per + wide), 123456789, dtype=torch.int32, device="cuda")
    whole[:, :per] = torch.from_numpy(t).cuda()
    return t, whole[:, :per]


def filled(pool_k, pool_v, table, lens, rng, grow=0.0):
    """Random keys and values in the used slots whose page is there."""
    import torch
    n_pages, Hk, page, d = pool_k.shape
    for b, n in enumerate(lens):
        for i in range(-(-n // page)):
            p = int(table[b, i])
            if not 0 <= p < n_pages:
                continue
            m = min(page, n - i * page)
            x = rng.normal(size=(2, Hk, m, d)) * (1 + grow * i)
            pool_k[p, :, :m], pool_v[p, :, :m] = (torch.from_numpy(y).to(pool_k.dtype).cuda() for y in x)


def check_attn(got_o, got_lse, q, pool_k, pool_v, table, lens, q_lens, causal, dtype, scale):
    import torch
    d = q.shape[-1]
    hq, hk, hv = host(q), host(pool_k), host(pool_v)
    O, LSE, A, seen = orows.paged_attention(hq, hk, hv, table, lens, q_lens, causal, scale)
    h = torch.finfo(torch_types(dtype)).eps / 2
    there = ~np.isnan(LSE)
    assert (got_lse[~there] == 7.0).all() and (got_o[~there] == 7.0).all()
    none = there & (LSE == -np.inf)
    assert (got_lse[none] == -np.inf).all() and (got_o[none] == 0).all()
    some = there & ~none
    if not some.any():
        return
    top_k, top_v = (np.abs(x[np.isfinite(x)]).max() for x in (hk, hv))
    score_err = (d + 8) * 2.0 ** -24 * scale * np.nanmax(np.abs(np.where(there[..., None], hq, 0)).sum(-1)) * top_k
    tol = h * (A + np.abs(O)) * (1 + h) + 2 * score_err * A + (seen[..., None] * 2.0 ** -25 * top_v if dtype == "fp16" else 0) + 2.0 ** -20 * A + 2.0 ** -25
    off = np.abs(got_o - O)
    assert (off[some] <= tol[some]).all(), f"O is {np.max((off / tol)[some]):.3g} of its tolerance"
    tol_lse = score_err + 2.0 ** -21 * (1 + np.abs(LSE))
    off = np.abs(np.where(some, got_lse - np.where(some, LSE, 0), 0))
    assert (off[some] <= tol_lse[some]).all(), f"LSE is off by {np.max(off[some]):.3g}, may be {np.min(tol_lse[some]):.3g}"


# B, H, Hk, Nq, d, page, lens, q_lens, causal, dtype, layout, gone
ATTN = {
    "one_key": (1, 1, 1, 1, 64, 16, [1], None, True, "bf16", "heads", []),
    "no_key": (3, 2, 1, 1, 64, 16, [0, 3, 0], None, True, "bf16", "heads", []),
    "page_of_one": (2, 4, 2, 1, 64, 1, [37, 65], None, True, "fp16", "slots", [(0, 5), (1, 64)]),
    "pages_end_inside_tiles": (2, 8, 2, 1, 128, 24, [600, 71], None, True, "bf16", "slots", []),
    "odd_pages": (2, 6, 3, 1, 128, 7, [130, 777], None, True, "fp16", "beside", [(1, 0), (1, 50), (0, 18)]),
    "pages_of_100": (3, 10, 2, 1, 64, 100, [1000, 99, 641], None, True, "bf16", "beside", []),
    "one_large_page": (1, 8, 8, 1, 128, 2000, [1999], None, True, "bf16", "heads", []),
    "all_pages_gone": (2, 4, 2, 1, 64, 16, [40, 40], None, True, "bf16", "heads", [(0, 0), (0, 1), (0, 2)]),
    "long_gap": (1, 4, 1, 1, 128, 16, [3000], None, True, "bf16", "slots", [(0, i) for i in range(3, 170)]),
    "many_heads_a_group": (2, 40, 2, 1, 128, 16, [900, 33], None, True, "bf16", "heads", []),
    "sixty_four_rows": (2, 64, 1, 1, 64, 32, [800, 1500], None, True, "fp16", "slots", []),
    "odd_rows": (1, 71, 1, 1, 64, 16, [1300], None, True, "bf16", "slots", [(0, 3)]),
    "odd_rows_128": (1, 71, 1, 1, 128, 16, [1300], None, True, "bf16", "slots", [(0, 3)]),
    "forty_rows": (2, 16, 2, 5, 64, 16, [900, 70], [5, 3], True, "bf16", "heads", [(0, 30)]),
    "forty_rows_128": (2, 16, 2, 5, 128, 24, [900, 70], [5, 3], True, "fp16", "slots", [(0, 30)]),
    "forty_eight_rows_128": (1, 48, 1, 1, 128, 16, [700], None, True, "bf16", "heads", []),
    "sixty_four_rows_128": (2, 32, 1, 2, 128, 16, [700, 1300], None, True, "bf16", "beside", [(1, 9)]),
    "drafts": (3, 6, 2, 7, 64, 24, [7, 333, 0], [7, 3, 0], True, "fp16", "heads", [(1, 2)]),
    "drafts_128": (3, 15, 3, 5, 128, 16, [900, 5, 64], [5, 4, 1], True, "bf16", "slots", []),
    "more_queries_than_keys": (2, 4, 2, 9, 64, 16, [4, 100], [9, 9], True, "bf16", "heads", []),
    "frame": (2, 4, 2, 33, 64, 48, [400, 90], None, False, "bf16", "beside", []),
    "many_tokens": (1, 4, 2, 150, 128, 16, [1000], None, True, "bf16", "heads", [(0, 60)]),
    "many_sequences": (130, 2, 1, 1, 64, 16, [i * 37 % 1100 for i in range(130)], None, True, "bf16", "heads", []),
    "whole_batch_uncut": (70, 32, 16, 1, 64, 32, [i * 11 % 200 for i in range(70)], None, True, "fp16", "heads", []),
    "cut_into_many_parts": (1, 2, 1, 1, 64, 64, [20000], None, True, "fp16", "heads", [(0, 100)]),
    # long enough for runs over several row tiles: more than 64 sequences, some without new tokens or keys; several row tiles a KV head
    "runs": (70, 4, 2, 2, 128, 16, [(i * 613) % 6900 for i in range(70)], [i % 3 for i in range(70)], True, "bf16", "slots", [(1, 5), (9, 0), (33, 60)]),
    "runs_short_row_tiles": (100, 4, 4, 1, 128, 32, [(i * 371) % 2000 for i in range(100)], None, True, "bf16", "heads", [(7, 1), (50, 0)]),
    "runs_64": (70, 2, 2, 1, 64, 24, [(i * 1013) % 5000 for i in range(70)], None, True, "fp16", "heads", [(2, 3), (69, 0)]),
    "runs_forty_rows": (3, 8, 1, 5, 128, 64, [46000, 44000, 47001], [5, 5, 4], True, "bf16", "heads", [(0, 100), (1, 0)]),
    "runs_row_tiles": (2, 65, 1, 1, 128, 64, [47000, 43000], None, True, "bf16", "heads", [(0, 100), (1, 0)]),
    "runs_row_tiles_64": (2, 65, 1, 2, 64, 64, [47000, 43001], [1, 2], True, "fp16", "slots", [(0, 100)]),
    "exact_tiles": (2, 4, 4, 1, 128, 64, [1024, 640], None, True, "bf16", "heads", []),
}


@pytest.mark.parametrize("name", ATTN)
def test_attention(name):
    import torch
    import paper_2511_23113_amd as dbsp
    B, H, Hk, Nq, d, page, lens, q_lens, causal, dtype, layout, gone = ATTN[name]
    rng = np.random.default_rng(3)
    per = -(-max(max(lens), 1) // page) + 1
    n_pages = B * per + 2
    k, v = pool_of(n_pages, Hk, page, d, dtype, rng, layout)
    t, table = table_of(B, per, n_pages, lens, page, rng, gone, wide=3)
    filled(k, v, t, lens, rng, grow=0.02 if max(lens) < 5000 else 0.0)
    q = torch.from_numpy(rng.normal(size=(B, Nq, H + 1, d))).to(torch_types(dtype)).cuda()[:, :, 1:].transpose(1, 2)
    o = torch.full((B, Nq, H, d), 7.0, dtype=q.dtype, device="cuda").transpose(1, 2)
    lse = torch.full((B, H, Nq), 7.0, device="cuda")
    if q_lens is not None:
        for b in range(B):
            q[b, :, q_lens[b]:] = float("nan")
    dev_q_lens = None if q_lens is None else torch.tensor(q_lens, dtype=torch.int32, device="cuda")
    cache = dbsp.PagedKVCache(k, v, table, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    dbsp.paged_attn_fwd(cache, q, q_lens=dev_q_lens, causal=causal, o=o, lse=lse)
    torch.cuda.synchronize()
    check_attn(host(o), host(lse), q, k, v, t, lens, [Nq] * B if q_lens is None else q_lens, causal, dtype, d ** -0.5)
    if q_lens is None:                     # the same bits again, in tensors of the call's own; and without LSE, by another scale
        again = dbsp.paged_attn_fwd(cache, q, causal=causal)
        assert torch.equal(again[0], o) and torch.equal(again[1], lse)
        assert dbsp.paged_attn_fwd(cache, q, causal=causal, want_lse=False)[1] is None
        o, lse = dbsp.paged_attn_fwd(cache, q, causal=causal, softmax_scale=0.03)
        check_attn(host(o), host(lse), q, k, v, t, lens, [Nq] * B, causal, dtype, 0.03)


@pytest.mark.parametrize("lo, hi", [(0, 40), (900, 1100)])
def test_thousands_of_sequences(lo, hi):
    # more than 64 blocks of 64 sequences: short ones with a few long ones among them, whose row tiles are cut into parts, and longer ones, in runs
    import torch
    import paper_2511_23113_amd as dbsp
    rng = np.random.default_rng(12)
    B, H, d, page, n_pages, per = 4230, 2, 64, 16, 200, 100
    k, v = (torch.from_numpy(rng.normal(size=(n_pages, 1, page, d))).half().cuda() for _ in range(2))
    table = rng.integers(-1, n_pages, size=(B, per)).astype(np.int32)
    lens = rng.integers(lo, hi, size=B)
    lens[rng.integers(0, B, 20)] = 1600
    q = torch.from_numpy(rng.normal(size=(B, H, 1, d))).half().cuda()
    cache = dbsp.PagedKVCache(k, v, torch.from_numpy(table).cuda(), torch.from_numpy(lens.astype(np.int32)).cuda())
    o, lse = dbsp.paged_attn_fwd(cache, q)
    check_attn(host(o), host(lse), q, k, v, table, lens, [1] * B, True, "fp16", d ** -0.5)


def test_the_order_of_pages_changes_no_bit():
    import torch
    import paper_2511_23113_amd as dbsp
    rng = np.random.default_rng(4)
    B, H, Hk, d, page, lens = 2, 8, 2, 128, 16, [1500, 407]
    per, n_pages = 100, 210
    outs = []
    data = torch.from_numpy(rng.normal(size=(2, B, per, Hk, page, d))).bfloat16().cuda()
    q = torch.from_numpy(rng.normal(size=(B, H, 1, d))).bfloat16().cuda()
    for seed in range(3):
        t, table = table_of(B, per, n_pages, [per * page] * B, page, np.random.default_rng(seed))
        k, v = pool_of(n_pages, Hk, page, d, "bf16", rng, ["heads", "slots", "beside"][seed])
        for b in range(B):
            k[table[b].long()], v[table[b].long()] = data[0, b], data[1, b]
        cache = dbsp.PagedKVCache(k, v, table, torch.tensor(lens, dtype=torch.int32, device="cuda"))
        outs.append(dbsp.paged_attn_fwd(cache, q))
    assert all(torch.equal(o, outs[0][0]) and torch.equal(l, outs[0][1]) for o, l in outs[1:])


def test_large_scores_and_late_maxima():
    # keys that grow along the cache: the running max is raised again and again; and scores of either sign far from 0
    import torch
    import paper_2511_23113_amd as dbsp
    rng = np.random.default_rng(5)
    k, v = pool_of(40, 2, 16, 64, "fp16", rng, "heads")
    t, table = table_of(1, 30, 40, [470], 16, rng)
    filled(k, v, t, [470], rng, grow=0.6)
    q = torch.from_numpy(3 * rng.normal(size=(1, 4, 1, 64))).half().cuda()
    cache = dbsp.PagedKVCache(k, v, table, torch.tensor([470], dtype=torch.int32, device="cuda"))
    o, lse = dbsp.paged_attn_fwd(cache, q, softmax_scale=0.5)
    assert float(lse.abs().max()) > 100
    check_attn(host(o), host(lse), q, k, v, t, [470], [1], True, "fp16", 0.5)


def test_lengths_out_of_range_are_clamped():
    import torch
    import paper_2511_23113_amd as dbsp
    rng = np.random.default_rng(6)
    k, v = pool_of(12, 2, 16, 64, "bf16", rng, "heads")
    t, table = table_of(2, 5, 12, [80, 80], 16, rng)
    filled(k, v, t, [80, 80], rng)
    q = torch.from_numpy(rng.normal(size=(2, 4, 2, 64))).bfloat16().cuda()
    lens, q_lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([2 ** 31 - 1, -5], [7, 2 ** 31 - 1]))
    o, lse = dbsp.paged_attn_fwd(dbsp.PagedKVCache(k, v, table, lens), q, q_lens=q_lens)
    check_attn(host(o), host(lse), q, k, v, t, [80, 0], [2, 2], True, "bf16", 64 ** -0.5)
    q_lens.fill_(-3)
    lse.fill_(7.0)
    dbsp.paged_attn_fwd(dbsp.PagedKVCache(k, v, table, lens), q, q_lens=q_lens, o=o, lse=lse)
    assert (lse == 7).all()
    # and appending: tokens before slot 0 are left out, lengths past the end are the end
    pools = k.clone(), v.clone()
    x = torch.from_numpy(rng.normal(size=(2, 2, 3, 64))).bfloat16().cuda()
    lens.copy_(torch.tensor([2 ** 31 - 1, 2]))
    q_out = torch.full_like(x, 7.0)
    dbsp.paged_append(dbsp.PagedKVCache(*pools, table, lens), x, x, q=x, q_out=q_out)
    want = orows.paged_append(host(k), host(v), t, [80, 2], host(x), host(x), [3, 3])
    assert np.array_equal(host(pools[0]), want[0], equal_nan=True) and np.array_equal(host(pools[1]), want[1], equal_nan=True)
    assert torch.equal(q_out[0], x[0]) and (q_out[1, :, 0] == 7).all() and torch.equal(q_out[1, :, 1:], x[1, :, 1:])


def test_pools_past_32_bits():
    # pages more than 2^32 bytes, and more than 2^31 elements, into the pool
    import torch
    import paper_2511_23113_amd as dbsp
    page, d, n_pages = 16, 128, 700_000
    pool = torch.empty(2, n_pages, 1, page, d, dtype=torch.bfloat16, device="cuda")
    table = torch.tensor([[n_pages - 1, 3, n_pages - 200, 640_000]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([60], dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(7)
    x = torch.from_numpy(rng.normal(size=(3, 1, 1, 60, d))).bfloat16().cuda()
    cache = dbsp.PagedKVCache(pool[0], pool[1], table, lens)
    dbsp.paged_append(cache, x[0], x[1])
    for i in range(4):
        m = min(page, 60 - i * page)
        at = int(table[0, i])
        assert torch.equal(pool[:, at, 0, :m], x[:2, 0, 0, i * page:i * page + m])
    q = x[2][:, :, :1]
    o, lse = dbsp.paged_attn_fwd(cache, q)
    s = (q.float() @ x[0].float().transpose(-1, -2)) * d ** -0.5
    assert float((lse - torch.logsumexp(s, -1)).abs().max()) < 1e-4
    assert float((o.float() - torch.softmax(s, -1) @ x[1].float()).abs().max()) < 2.0 ** -6


# B, H, Hk, Nn, d, page, lens, new_lens, dtype, layout, gone, kind, gains, pairs, halves, pos
APPEND = {
    "one_token": (1, 1, 1, 1, 64, 16, [1], None, "bf16", "heads", [], "none", "", (32,), True, "none"),
    "values_alone": (2, 0, 2, 3, 64, 16, [20, 3], None, "bf16", "slots", [], "none", "", None, False, "none"),
    "next_tokens": (5, 8, 2, 1, 128, 16, [1, 16, 17, 900, 33], None, "bf16", "heads", [], "rms", "q_gain,k_gain", (64,), True, "none"),
    "page_of_one": (2, 2, 1, 9, 64, 1, [9, 40], None, "fp16", "slots", [(1, 33)], "none", "", (8, 12, 12), False, "each"),
    "prompt": (2, 6, 3, 211, 128, 24, [211, 500], None, "bf16", "beside", [], "rms", "q_gain,k_gain", (22, 21, 21), False, "shared"),
    "ragged": (4, 4, 2, 50, 64, 7, [50, 13, 0, 300], [50, 13, 0, 1], "fp16", "slots", [(0, 2), (3, 42)], "layer", ALL, (8, 12, 12), True, "each"),
    "no_queries": (2, 0, 5, 17, 128, 100, [130, 99], None, "bf16", "heads", [], "rms", "k_gain", (16, 24), False, "each"),
    "some_places": (1, 3, 1, 33, 128, 48, [70], None, "fp16", "beside", [], "none", "", (3, 5), False, "each"),
    "more_new_than_used": (2, 2, 2, 8, 64, 16, [5, 30], None, "bf16", "heads", [], "none", "", (32,), False, "none"),
}


@pytest.mark.parametrize("name", APPEND)
def test_append(name):
    import torch
    import paper_2511_23113_amd as dbsp
    B, H, Hk, Nn, d, page, lens, new_lens, dtype, layout, gone, kind, gain_names, pairs, halves, pos = APPEND[name]
    rng = np.random.default_rng(8)
    dt = torch_types(dtype)
    per = -(-max(lens) // page) + 1
    n_pages = B * per + 2
    pool_k, pool_v = pool_of(n_pages, Hk, page, d, dtype, rng, layout)
    t, table = table_of(B, per, n_pages, lens, page, rng, gone, wide=1)
    before = host(pool_k), host(pool_v)
    x = torch.from_numpy(rng.normal(size=(B, Nn, H + 2 * Hk, d))).to(dt).cuda()
    q = x[:, :, :H].transpose(1, 2) if H else None
    k, v = x[:, :, H:H + Hk].transpose(1, 2), x[:, :, H + Hk:].transpose(1, 2)
    gains = {n: torch.from_numpy(1 + 0.3 * rng.normal(size=d)).to(dt).cuda() for n in gain_names.split(",") if n}
    norm = None if kind == "none" else dbsp.HeadNorm(kind=kind, eps=EPS, **gains)
    rotary = dbsp.Rotary(pairs, halves=halves) if pairs else None
    positions = None
    if pos != "none":
        positions = torch.from_numpy(rng.integers(0, 5000, size=(B, Nn, len(pairs)) if pos == "each" else (Nn, len(pairs))).astype(np.int32)).cuda()
    q_out = torch.full((B, H, Nn, d), 7.0, dtype=dt, device="cuda") if H else None
    cache = dbsp.PagedKVCache(pool_k, pool_v, table, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    dev_new = None if new_lens is None else torch.tensor(new_lens, dtype=torch.int32, device="cuda")
    assert dbsp.paged_append(cache, k, v, new_lens=dev_new, q=q, q_out=q_out, norm=norm, rotary=rotary, positions=positions) is q_out
    torch.cuda.synchronize()
    new = [Nn] * B if new_lens is None else new_lens
    slots = np.array([[lens[b] - new[b] + i for i in range(Nn)] for b in range(B)])
    a = None
    if pairs:
        at = slots[..., None] if positions is None else np.broadcast_to(positions.cpu().numpy(), (B, Nn, len(pairs)))
        a = orows.angles(at, pairs, rotary.freqs)[:, None]
    value = lambda n, none: host(gains[n]) if n in gains else np.full(d, none)      # noqa: E731
    hk = orows.rows_fwd(host(k), kind, value("k_gain", 1.0), value("k_bias", 0.0), EPS, a, halves)
    tol = fwd_tolerance(host(k), hk, kind, value("k_gain", 1.0), value("k_bias", 0.0), a, halves, dtype)
    # what is written, where, and how far off it may be; all else as it was
    want_k, want_v = orows.paged_append(*before, t, lens, hk, host(v), new)
    tol_k, _ = orows.paged_append(np.zeros_like(before[0]), before[1], t, lens, tol, host(v), new)
    got_k, got_v = host(pool_k), host(pool_v)
    assert np.array_equal(got_v, want_v, equal_nan=True) and np.array_equal(np.isnan(got_k), np.isnan(want_k))
    there = ~np.isnan(want_k)
    assert (np.abs(got_k - want_k)[there] <= tol_k[there]).all()
    if H:
        hq = orows.rows_fwd(host(q), kind, value("q_gain", 1.0), value("q_bias", 0.0), EPS, a, halves)
        tol = fwd_tolerance(host(q), hq, kind, value("q_gain", 1.0), value("q_bias", 0.0), a, halves, dtype)
        got = host(q_out)
        for b in range(B):
            written = (np.arange(Nn) < new[b]) & (slots[b] >= 0)
            assert (got[b][:, ~written] == 7).all()
            assert (np.abs(got[b] - hq[b])[:, written] <= tol[b][:, written]).all()


def test_shared_pages_and_the_same_page_twice():
    # two sequences with the same beginning, and a table that names one page twice
    import torch
    import paper_2511_23113_amd as dbsp
    rng = np.random.default_rng(9)
    k, v = pool_of(8, 2, 16, 64, "bf16", rng, "heads")
    t = np.array([[3, 5, 1, 1], [3, 5, 6, -1]], dtype=np.int32)
    lens = [64, 40]
    filled(k, v, t, lens, rng)
    k[6], v[6] = k[0].nan_to_num(0.5), v[0].nan_to_num(0.25)
    q = torch.from_numpy(rng.normal(size=(2, 4, 1, 64))).bfloat16().cuda()
    cache = dbsp.PagedKVCache(k, v, torch.from_numpy(t).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    o, lse = dbsp.paged_attn_fwd(cache, q)
    check_attn(host(o), host(lse), q, k, v, t, lens, [1, 1], True, "bf16", 64 ** -0.5)
    # both append to the one page: either's row is there, whole
    x = torch.from_numpy(rng.normal(size=(2, 2, 1, 64))).bfloat16().cuda()
    table = torch.tensor([[4], [4]], dtype=torch.int32, device="cuda")
    dbsp.paged_append(dbsp.PagedKVCache(k, v, table, torch.tensor([9, 9], dtype=torch.int32, device="cuda")), x, x)
    for h in range(2):
        assert any(torch.equal(k[4, h, 8], x[b, h, 0]) for b in range(2)) and any(torch.equal(v[4, h, 8], x[b, h, 0]) for b in range(2))


@pytest.mark.parametrize("halves", [False, True])
def test_queries_in_place(halves):
    import torch
    import paper_2511_23113_amd as dbsp
    s = generator(3, 7, 2, 128, 16, 8)
    s["lens"].copy_(torch.tensor([100, 5, 30]))
    x = s["rand"](3, 5, 11, 128)
    q, k, v = (x[:, :, a:b].transpose(1, 2) for a, b in ((0, 7), (7, 9), (9, 11)))
    new = torch.tensor([5, 2, 0], dtype=torch.int32, device="cuda")
    more = dict(new_lens=new, norm=s["norm"], rotary=dbsp.Rotary((20, 12), halves=halves), positions=torch.randint(0, 99, (3, 5, 2), device="cuda", dtype=torch.int32))
    want = dbsp.paged_append(s["cache"], k, v, q=q, q_out=q.clone(), **more)
    pools = s["k"].clone(), s["v"].clone()
    assert dbsp.paged_append(s["cache"], k, v, q=q, q_out=q, **more) is q
    assert torch.equal(q, want) and torch.equal(s["k"], pools[0]) and torch.equal(s["v"], pools[1])


def generator(B, H, Hk, d, page, per, seed=10):
    """A program that generates token by token: what it has in hand, and a step."""
    import torch
    import paper_2511_23113_amd as dbsp
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()      # noqa: E731
    n_pages = B * per
    k, v = rand(n_pages, Hk, page, d), rand(n_pages, Hk, page, d)
    table = torch.randperm(n_pages, device="cuda", generator=g).view(B, per).int()
    lens = torch.randint(1, 300, (B,), device="cuda", generator=g, dtype=torch.int32)
    cache = dbsp.PagedKVCache(k, v, table, lens)
    norm = dbsp.HeadNorm(1 + 0.1 * torch.randn(d, device="cuda", generator=g), 1 + 0.1 * torch.randn(d, device="cuda", generator=g), eps=EPS)
    rotary = dbsp.Rotary((d // 2,), halves=True)
    x = rand(B, 1, H + 2 * Hk, d)

    def step(stream=None, **out):
        q_out = dbsp.paged_append(cache, x[:, :, H:H + Hk].transpose(1, 2), x[:, :, H + Hk:].transpose(1, 2), q=x[:, :, :H].transpose(1, 2), norm=norm, rotary=rotary, stream=stream)
        return dbsp.paged_attn_fwd(cache, q_out, stream=stream, **out)
    return dict(cache=cache, x=x, k=k, v=v, table=table, lens=lens, norm=norm, rotary=rotary, step=step, rand=rand)


def test_token_by_token():
    # a whole run: a prompt by the block-sparse path's operators and appended at once, then tokens one by one; each step against attention over
    # all that has been generated, formed from the same tokens in float64
    import torch
    import paper_2511_23113_amd as dbsp
    B, H, Hk, d, page, prompt, steps = 2, 4, 2, 64, 24, 128, 30
    s = generator(B, H, Hk, d, page, 12)
    x = s["rand"](B, prompt + steps, H + 2 * Hk, d)
    part = lambda a, b: [y.transpose(1, 2) for y in (x[:, a:b, :H], x[:, a:b, H:H + Hk], x[:, a:b, H + Hk:])]      # noqa: E731
    q, k, v = part(0, prompt)
    # the prompt's own attention: all blocks of its 128 tokens, from the rows that the forward pass makes, heads of K repeated for their groups
    rows_q, rows_k = dbsp.qk_norm_rope_fwd(q, k, norm=s["norm"], rotary=s["rotary"])
    plan = dbsp.plan_sparse_attn(np.ones((H, 2, 2), np.uint8), 64)
    o_sparse, lse_sparse = dbsp.sparse_attn_fwd(plan, rows_q, rows_k.repeat_interleave(H // Hk, 1), v.repeat_interleave(H // Hk, 1).contiguous())
    s["lens"].fill_(prompt)
    q_out = dbsp.paged_append(s["cache"], k, v, q=q, norm=s["norm"], rotary=s["rotary"])
    assert torch.equal(q_out, rows_q)
    o, lse = dbsp.paged_attn_fwd(s["cache"], q_out, causal=False)
    # (both are within their roundings of the same attention: h for the probabilities and h for O, each)
    assert float((o.float() - o_sparse.float()).abs().max()) <= 4 * 2.0 ** -8 * float(v.abs().max()) and float((lse - lse_sparse).abs().max()) < 1e-3
    gain = [host(g) for g in s["norm"].given.values()]
    for i in range(prompt, prompt + steps):
        s["lens"].add_(1)
        q, k, v = part(i, i + 1)
        q_out = dbsp.paged_append(s["cache"], k, v, q=q, norm=s["norm"], rotary=s["rotary"])
        o, lse = dbsp.paged_attn_fwd(s["cache"], q_out)
        if i % 10 == 0:
            t, lens = s["table"].cpu().numpy(), [i + 1] * B
            check_attn(host(o), host(lse), q_out, s["k"], s["v"], t, lens, [1] * B, True, "bf16", d ** -0.5)
            a = orows.angles(np.arange(i + 1)[:, None], s["rotary"].pairs, s["rotary"].freqs)[None, None]
            hk = host(x[:, :i + 1, H:H + Hk].transpose(1, 2))
            want = orows.rows_fwd(hk, "rms", gain[1], 0.0, EPS, a, True)
            tol = fwd_tolerance(hk, want, "rms", gain[1], 0.0, a, True, "bf16")
            for b in range(B):
                places = [orows.slot_place(t[b], j, page, s["k"].shape[0]) for j in range(i + 1)]
                got = np.stack([host(s["k"][p, :, at]) for p, at in places], 1)
                assert (np.abs(got - want[b]) <= tol[b]).all()


def test_graphs_follow_lengths_and_pages():
    import torch
    s = generator(3, 8, 2, 128, 16, 80)
    s["step"]()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = s["step"]()
    for i in range(4):
        s["lens"].add_(1 + 150 * i)
        s["x"].copy_(s["rand"](*s["x"].shape))
        if i == 2:
            s["table"][1, 3] = -1
            s["table"].copy_(s["table"].flip(0))
        o.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        pools = s["k"].clone(), s["v"].clone()
        want = s["step"]()
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1]) and torch.equal(pools[0], s["k"]) and torch.equal(pools[1], s["v"])


def test_two_graphs_and_an_eager_call_each_have_their_workspace():
    import torch
    import paper_2511_23113_amd as dbsp
    s = [generator(2, 4, 2, 64, 16, 200, seed=i) for i in range(3)]
    for x in s:
        x["lens"].fill_(2900)
    want = [x["step"]() for x in s]
    graphs, outs = [], []
    for x in s[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(x["step"]())
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        got = s[2]["step"]()
        torch.cuda.synchronize()
        for (o, lse), (wo, wl) in zip([*outs, got], want):
            assert torch.equal(o, wo) and torch.equal(lse, wl)
    assert isinstance(s[0]["cache"], dbsp.PagedKVCache)


def test_a_table_that_all_sequences_share():
    import torch
    import paper_2511_23113_amd as dbsp
    rng = np.random.default_rng(11)
    k, v = pool_of(6, 2, 16, 64, "bf16", rng, "heads")
    t, table = table_of(1, 5, 6, [75], 16, rng)
    filled(k, v, t, [75], rng)
    q = torch.from_numpy(rng.normal(size=(3, 4, 1, 64))).bfloat16().cuda()
    lens = [75, 20, 60]
    o, lse = dbsp.paged_attn_fwd(dbsp.PagedKVCache(k, v, table.expand(3, -1), torch.tensor(lens, dtype=torch.int32, device="cuda")), q)
    check_attn(host(o), host(lse), q, k, v, np.repeat(t, 3, 0), lens, [1, 1, 1], True, "bf16", 64 ** -0.5)


def test_tensors_of_another_device_than_the_current_one(monkeypatch):
    import torch
    import paper_2511_23113_amd as dbsp
    s = generator(2, 4, 2, 64, 16, 4)
    q = s["rand"](2, 4, 1, 64)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for call in (lambda: s["step"](), lambda: dbsp.paged_attn_fwd(s["cache"], q), lambda: dbsp.qk_norm_rope_fwd(q), lambda: dbsp.qk_norm_rope_bwd(q, None, q, None)):
        with pytest.raises(ValueError, match="another device"):
            call()


def test_other_streams():
    import torch
    s = generator(3, 8, 2, 64, 16, 100)
    s["lens"].fill_(1000)
    want = s["step"]()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream, torch.cuda.default_stream(), 0):
        with torch.cuda.stream(torch.cuda.Stream()):
            got = s["step"](stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_workspace_of_the_callers():
    import torch
    import paper_2511_23113_amd as dbsp
    s = generator(1, 4, 2, 64, 16, 400)
    s["lens"].fill_(6000)
    want = s["step"]()
    q = s["rand"](1, 4, 1, 64)
    want = dbsp.paged_attn_fwd(s["cache"], q)
    need = next(iter(s["cache"]._bytes.values()))
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    got = dbsp.paged_attn_fwd(s["cache"], q, workspace=ws[:need])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and (ws[need:] == 255).all()
    with pytest.raises(dbsp.DbspError, match="workspace holds"):
        dbsp.paged_attn_fwd(s["cache"], q, workspace=ws[:256])


def test_refusals_on_the_gpu():
    import torch
    import paper_2511_23113_amd as dbsp
    s = generator(2, 4, 2, 64, 16, 4)
    cache, x = s["cache"], s["rand"](2, 2, 3, 64)
    q = s["rand"](2, 4, 3, 64)
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (dict(k=x[:1], v=x[:1]), dict(v=x[:, :1]), dict(v=x.half()), dict(q=q[:, :, :2]), dict(q_out=q), dict(q=q, q_out=x), dict(new_lens=lens.long()),
                dict(new_lens=lens[:1]), dict(new_lens=lens.cpu()), dict(norm=dbsp.HeadNorm(torch.ones(128, device="cuda")))):
        with pytest.raises(ValueError):
            dbsp.paged_append(cache, **{"k": x, "v": x, **bad})
    with pytest.raises(dbsp.DbspError, match="positions"):
        dbsp.paged_append(cache, x, x, rotary=dbsp.Rotary((8, 8)))
    for bad in (dict(q=q[:1]), dict(q=q.half()), dict(q=q[..., ::2]), dict(o=q[:, :2]), dict(lse=lens), dict(q_lens=lens.long()), dict(workspace=lens)):
        with pytest.raises(ValueError):
            dbsp.paged_attn_fwd(cache, **{"q": q, **bad})
    with pytest.raises(dbsp.DbspError, match="multiple"):
        dbsp.paged_attn_fwd(cache, s["rand"](2, 3, 1, 64))
    for bad in (dict(v=s["v"][:-1]), dict(v=s["v"].half()), dict(pages=s["table"].long()), dict(pages=s["table"][0]), dict(lens=lens[:1]), dict(lens=lens.cpu())):
        with pytest.raises(ValueError):
            dbsp.PagedKVCache(**{"k": s["k"], "v": s["v"], "pages": s["table"], "lens": lens, **bad})
