"""Cases by which the speed of the key/value cache's operators is measured, over the range that a program meets which
generates piece by piece: attention of new tokens over a prefix that all sequences share and over each sequence's own cache,
with the keys' weights summed up beside it, and the eviction of the keys that weigh least.

A case is a dict of plain values.  Attention cases (kind "attn"): B sequences, H query and Hk key/value heads, Nq new tokens,
head dim d, P tokens of shared prefix, `cap` slots of each sequence's own cache, of which between lo / 1000 and hi / 1000 are
used; `ragged`: the sequences bring different numbers of new tokens; `decay`: None, or the factor of the weights before.
Eviction cases (kind "evict"): Hk heads of B sequences are cut back to `budget` slots; `sinks` and `recent` positions stay.
"""

import math

import torch

own = False


def attn(name, B, H, Hk, Nq, d, P, cap, lo, hi, dtype, causal=True, ragged=False, decay=None):
    return dict(name=name, kind="attn", B=B, H=H, Hk=Hk, Nq=Nq, d=d, P=P, cap=cap, lo=lo, hi=hi, dtype=dtype, causal=causal, ragged=ragged,
                decay=decay)


def evict(name, B, Hk, d, cap, lo, hi, budget, dtype, sinks=4, recent=32):
    return dict(name=name, kind="evict", B=B, Hk=Hk, d=d, cap=cap, lo=lo, hi=hi, budget=budget, dtype=dtype, sinks=sinks, recent=recent)


def listed():
    return [
        # the smallest call: one sequence's next token behind a short text prompt (latency, launches, host work)
        attn("first_tokens", 1, 2, 2, 1, 64, 77, 64, 300, 600, "bf16"),
        # next tokens of 16 samples from one prompt, a head of its own for every query head, weights kept for eviction
        attn("token_step", 16, 24, 24, 1, 128, 4096, 2304, 300, 1000, "bf16", decay=1.0),
        # next tokens of many samples that share their conditioning frames, grouped heads: the prefix's products fill tiles
        attn("shared_tokens", 64, 40, 8, 1, 128, 16384, 4096, 100, 900, "bf16"),
        # a few sequences behind a very long shared context: nearly all of the time is the stream of its keys and values
        attn("long_prefix", 6, 16, 4, 1, 128, 131072, 8200, 200, 1000, "fp16", decay=1.0),
        # a few drafted tokens a sequence, not as many for each, with forgetting weights
        attn("drafts", 24, 30, 10, 7, 64, 1000, 1500, 50, 1000, "fp16", ragged=True, decay=0.9),
        # one latent frame of 30 x 52 tokens at a time (bidirectional inside), two earlier frames in the cache, long context
        attn("frame", 2, 40, 40, 1560, 128, 8190, 4680, 1000, 1000, "bf16", causal=False, decay=1.0),
        # a prompt's first pass: causal, behind a short shared text
        attn("prompt", 1, 48, 48, 4101, 64, 226, 4200, 990, 1000, "bf16"),
        # the smallest eviction
        evict("evict_small", 1, 2, 64, 96, 900, 1000, 48, "fp16", recent=8),
        # steady state: every few tokens the caches are cut back to their budget, and next to nothing has to move
        evict("evict_step", 32, 8, 128, 2304, 890, 900, 2048, "bf16"),
        # after a prompt: long caches of different lengths are cut to a small budget
        evict("evict_prompt", 4, 24, 128, 16500, 400, 1000, 2048, "bf16"),
        # one very long sequence, cut to an eighth
        evict("evict_long", 1, 8, 128, 131100, 995, 1000, 16000, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """One more case of the same ranges; no more bytes or operations than the largest listed one, and scores that the plain
    form can hold."""
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    while True:
        d, dtype, B = rng.choice([64, 128]), rng.choice(["bf16", "fp16"]), _log_int(rng, 1, 64)
        Hk = _log_int(rng, 2, 48)
        hi = rng.randint(100, 1000)
        lo = rng.randint(20, hi)
        if rng.random() < 0.35:
            cap = _log_int(rng, 64, 131100)
            case = evict(None, B, Hk, d, cap, lo, hi, max(8, cap * hi * rng.randint(50, 990) // 1000000), dtype, sinks=rng.choice([0, 4, 16]), recent=rng.choice([0, 8, 64]))
            big = 0
        else:
            Nq = rng.choice([1, 1, _log_int(rng, 2, 64), _log_int(rng, 64, 4500)])
            cap = max(Nq, _log_int(rng, 64, 8200))
            P = rng.choice([0, _log_int(rng, 32, 131072), _log_int(rng, 32, 131072)])
            case = attn(None, B, Hk * rng.choice([1, 1, 2, 4, 5, 8]), Hk, Nq, d, P, cap, lo, hi, dtype, causal=rng.random() < 0.7,
                        ragged=B > 1 and Nq > 1 and rng.random() < 0.4, decay=rng.choice([None, 1.0, 0.9, 0.0]))
            big = B * case["H"] * Nq * (P + cap)
        del case["name"]
        held = 4 * B * Hk * cap * d
        if big <= 1 << 31 and held <= 4 << 30 and all(work(case)[k] <= most[k] for k in most):
            return case


def _used(case):
    return (case["lo"] + case["hi"]) / 2000 * case["cap"]


def work(case):
    """K, V and the queries once, the outputs once; a product of d for a score and one for its value, and of the own keys' scores
    no second time.  Eviction: weights and positions once, and the rows that move, read and written."""
    B, d, n = case["B"], case["d"], _used(case)
    if case["kind"] == "evict":
        moved = case["budget"] * max(0.0, 1 - case["budget"] / n)
        return {"bytes": B * case["Hk"] * (8 * n + moved * (8 * d + 16)), "flops": B * case["Hk"] * 4 * n}
    H, Hk, Nq, P = case["H"], case["Hk"], case["Nq"], case["P"]
    queries = B * H * Nq * (0.5 if case["ragged"] else 1.0)
    seen = n - (min(n, Nq) / 2 if case["causal"] else 0)
    moved = 4 * d * Hk * (P + B * n) + queries * (4 * d + 4) + (8 * B * Hk * n if case["decay"] is not None else 0)
    return {"bytes": moved, "flops": 4 * d * queries * (P + seen)}


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float16
    B, Hk, d, cap = case["B"], case["Hk"], case["d"], case["cap"]

    def keys(*shape):           # a few of them draw much more attention than the others
        return (torch.randn(*shape, d, device=dev, generator=g) * torch.exp(0.4 * torch.randn(*shape, 1, device=dev, generator=g))).to(dt)

    used = torch.randint(cap * case["lo"] // 1000, cap * case["hi"] // 1000 + 1, (B,), device=dev, generator=g, dtype=torch.int32)
    s = dict(case=case, k=keys(B, Hk, cap), v=torch.randn(B, Hk, cap, d, device=dev, generator=g).to(dt))
    if case["kind"] == "evict":
        # what changes in a pass and is set back before it lies in one buffer: lens, positions, weights (heavy-tailed, a tenth never attended to)
        s["small"] = torch.empty(B + 2 * B * Hk * cap, device=dev, dtype=torch.int32)
        s["lens"], s["positions"], s["weights"] = _small(s["small"], B, Hk, cap)
        s["lens"].copy_(used)
        order = torch.rand(B, Hk, cap, device=dev, generator=g)
        order[:, :, case["budget"]:] = 1 + torch.arange(cap - case["budget"], device=dev)      # new tokens lie behind what earlier passes mixed
        s["positions"].copy_(order.argsort(-1).argsort(-1))
        s["weights"].copy_(torch.rand(B, Hk, cap, device=dev, generator=g) ** 6 * (torch.rand(B, Hk, cap, device=dev, generator=g) > 0.1))
        s["as_before"] = s["small"].clone()
        s["keep_from"] = (used - case["recent"]).to(torch.int32)
    else:
        H, Nq, P = case["H"], case["Nq"], case["P"]
        s["q"] = torch.randn(B, H, Nq, d, device=dev, generator=g).to(dt)
        s["q_lens"] = torch.randint(0, Nq + 1, (B,), device=dev, generator=g, dtype=torch.int32) if case["ragged"] else None
        # a sequence's new tokens are in its cache
        new = s["q_lens"] if case["ragged"] else Nq
        s["lens"] = torch.clamp(torch.maximum(used, torch.zeros_like(used) + new), max=cap)
        s["prefix_k"] = keys(Hk, P) if P else None
        s["prefix_v"] = torch.randn(Hk, P, d, device=dev, generator=g).to(dt) if P else None
        s["weights"] = torch.rand(B, Hk, cap, device=dev, generator=g) if case["decay"] is not None else None
        s["o"] = torch.zeros_like(s["q"])                  # rows behind a sequence's new tokens stay as they are
        s["lse"] = torch.zeros(B, H, Nq, device=dev)
    if own:
        import paper_2511_23113_amd as dbsp
        s["cache"] = dbsp.KVCache(s["k"], s["v"], s["lens"], prefix_k=s.get("prefix_k"), prefix_v=s.get("prefix_v"), weights=s["weights"],
                                  positions=s.get("positions"))
        s["attn"], s["evict"] = dbsp.cache_attn_fwd, dbsp.cache_evict
    return s


def _small(buffer, B, Hk, cap):
    n = B * Hk * cap
    return buffer[:B], buffer[B:B + n].view(B, Hk, cap), buffer[B + n:].view(torch.float32).view(B, Hk, cap)


def run(s):
    case = s["case"]
    if case["kind"] == "evict":
        s["small"].copy_(s["as_before"])
        if own:
            s["evict"](s["cache"], case["budget"], sinks=case["sinks"], keep_from=s["keep_from"])
        else:
            _evict_plain(s["k"], s["v"], s["lens"], s["weights"], s["positions"], case["budget"], case["sinks"], s["keep_from"])
        return {"k": s["k"], "v": s["v"], "lens": s["lens"], "weights": s["weights"], "positions": s["positions"]}
    if own:
        s["attn"](s["cache"], s["q"], q_lens=s["q_lens"], causal=case["causal"], decay=case["decay"], o=s["o"], lse=s["lse"])
    else:
        _attn_plain(s)
    out = {"o": s["o"], "lse": s["lse"]}
    if case["decay"] is not None:
        out["weights"] = s["weights"]
    return out


def _attn_plain(s):
    case, q, lens = s["case"], s["q"], s["lens"].long()
    B, H, Nq, d = q.shape
    Hk, P, cap = case["Hk"], case["P"], case["cap"]
    G = H // Hk
    new = s["q_lens"].long() if s["q_lens"] is not None else torch.full_like(lens, Nq)
    t = torch.arange(Nq, device=q.device)
    slot = torch.arange(cap, device=q.device)
    until = (lens - new)[:, None] + t + 1 if case["causal"] else lens[:, None].expand(B, Nq)      # [B, Nq] own slots that a query sees
    seen = slot < torch.minimum(until, lens[:, None])[:, :, None]                                 # [B, Nq, cap]
    qf = (q.float() * (1 / math.sqrt(d))).view(B, Hk, G * Nq, d)
    scores = (qf @ s["k"].float().transpose(-1, -2)).view(B, Hk, G, Nq, cap)
    scores = torch.where(seen[:, None, None], scores, -math.inf)
    top = scores.amax(-1, keepdim=True)
    if P:
        qp = qf.transpose(0, 1).reshape(Hk, B * G * Nq, d)
        before = (qp @ s["prefix_k"].float().transpose(-1, -2)).view(Hk, B, G, Nq, P).transpose(0, 1)
        top = torch.maximum(top, before.amax(-1, keepdim=True))
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(scores - top)
    del scores
    total = p.sum(-1, keepdim=True)
    v = torch.where((slot < lens[:, None])[:, None, :, None], s["v"].float(), 0.0)
    o = (p.view(B, Hk, G * Nq, cap) @ v).view(B, Hk, G, Nq, d)
    if P:
        pp = torch.exp(before - top)
        del before
        total = total + pp.sum(-1, keepdim=True)
        o = o + (pp.transpose(0, 1).reshape(Hk, B * G * Nq, P) @ s["prefix_v"].float()).view(Hk, B, G, Nq, d).transpose(0, 1)
        del pp
    some = total > 0
    o = torch.where(some, o / total, 0.0).view(B, H, Nq, d)
    lse = torch.where(some, top + torch.log(total), -math.inf).view(B, H, Nq)
    there = (t < new[:, None])[:, None]                                                           # [B, 1, Nq]
    s["o"].copy_(torch.where(there[..., None], o.to(q.dtype), s["o"]))
    s["lse"].copy_(torch.where(there, lse, s["lse"]))
    if case["decay"] is not None:
        share = torch.where(there[:, :, None, :, None] & some, p / total, 0.0).sum((2, 3))
        s["weights"].copy_(torch.where((slot < lens[:, None])[:, None], case["decay"] * s["weights"] + share, s["weights"]))


def _evict_plain(k, v, lens, weights, positions, budget, sinks, keep_from):
    B, Hk, cap, d = k.shape
    slot = torch.arange(cap, device=k.device)
    valid = (slot < lens[:, None])[:, None]                                                       # [B, 1, cap]
    cut = (lens > budget)[:, None, None]
    stays = (positions < sinks) | (positions >= keep_from[:, None, None])
    rank = torch.where(weights.isnan(), -math.inf, weights.double())
    rank = torch.where(stays, 1e300, rank.clamp(max=1e299))
    rank = torch.where(valid, rank, -math.inf)
    # (a slot that is not used comes behind every used one: a stable sort, and used slots lie in front)
    first = rank.sort(dim=-1, descending=True, stable=True).indices[..., :budget]
    kept = torch.zeros_like(stays).scatter_(-1, first, torch.ones_like(first, dtype=torch.bool)) & valid
    hole, filler = cut & ~kept & (slot < budget), cut & kept & (slot >= budget)
    # the n-th filler's slot in place n, then every hole takes its own
    fill = torch.zeros(B, Hk, cap + 1, device=k.device, dtype=torch.long)
    fill.scatter_(-1, torch.where(filler, filler.cumsum(-1) - 1, cap), slot.expand(B, Hk, cap))
    source = torch.where(hole, fill.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0)), slot)[..., :budget]
    rows = source[..., None].expand(B, Hk, source.shape[-1], d)
    k[:, :, :budget], v[:, :, :budget] = k.gather(2, rows), v.gather(2, rows)
    weights[:, :, :budget], positions[:, :, :budget] = weights.gather(2, source), positions.gather(2, source)
    weights.masked_fill_(cut & valid & (slot >= budget), 0.0)
    lens.clamp_(max=budget)


def exact(case, seed):
    s = prepare(case, seed)
    return _evict_exact(s) if case["kind"] == "evict" else _attn_exact(s)


def _attn_exact(s):
    """Sequence by sequence, over the keys that it has and no others, in 64 bits; long query lists a part at a time."""
    case = s["case"]
    H, Hk, Nq, d, P = case["H"], case["Hk"], case["Nq"], case["d"], case["P"]
    G = H // Hk
    o, lse = s["o"].double(), s["lse"].double()
    weights = None if case["decay"] is None else s["weights"].double()
    none = torch.empty(Hk, 0, d, device=o.device, dtype=torch.float64)
    pk, pv = (s["prefix_k"].double(), s["prefix_v"].double()) if P else (none, none)
    for b, n in enumerate(s["lens"].tolist()):
        new = Nq if s["q_lens"] is None else int(s["q_lens"][b])
        keys, values = torch.cat([pk, s["k"][b, :, :n].double()], 1), torch.cat([pv, s["v"][b, :, :n].double()], 1)
        if weights is not None:
            weights[b, :, :n] *= case["decay"]
        step = max(1, 300_000_000 // max(1, H * (P + n)))
        for a in range(0, new, step):
            e = min(new, a + step)
            logits = torch.einsum("kgtd,knd->kgtn", s["q"][b].view(Hk, G, Nq, d)[:, :, a:e].double(), keys) / math.sqrt(d)
            if case["causal"]:
                ahead = torch.arange(n, device=o.device)[None] > (n - new + torch.arange(a, e, device=o.device))[:, None]
                logits[..., P:].masked_fill_(ahead, -math.inf)
            z = torch.logsumexp(logits, -1)
            prob = torch.exp(logits - torch.where(z == -math.inf, 0.0, z)[..., None])
            del logits
            o[b].view(Hk, G, Nq, d)[:, :, a:e] = torch.einsum("kgtn,knd->kgtd", prob, values)
            lse[b].view(Hk, G, Nq)[:, :, a:e] = z
            if weights is not None:
                weights[b, :, :n] += prob[..., P:].sum((1, 2))
    out = {"o": o, "lse": lse}
    if weights is not None:
        out["weights"] = weights
    return out


def _evict_exact(s):
    """Head by head: who stays, from the definition, and where it goes."""
    case, budget = s["case"], s["case"]["budget"]
    k, v, weights, positions = s["k"].double(), s["v"].double(), s["weights"].double(), s["positions"].clone()
    for b, n in enumerate(s["lens"].tolist()):
        if n <= budget:
            continue
        for h in range(case["Hk"]):
            w, at = s["weights"][b, h, :n].double(), s["positions"][b, h, :n]
            safe = (at < case["sinks"]) | (at >= s["keep_from"][b])
            ranked = torch.cat([safe.nonzero()[:, 0], (~safe).nonzero()[:, 0][torch.argsort(w[~safe], descending=True, stable=True)]])
            stay = ranked[:budget].sort().values
            late = stay[stay >= budget]
            free = torch.ones(budget, dtype=torch.bool, device=k.device)
            free[stay[stay < budget]] = False
            free = free.nonzero()[:, 0]
            for x in (k, v, weights, positions):
                x[b, h, free] = x[b, h, late]
            weights[b, h, budget:n] = 0
    return {"k": k, "v": v, "lens": s["lens"].clamp(max=budget), "weights": weights, "positions": positions}
