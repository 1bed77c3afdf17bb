"""Cases by which the speed of the operators around attention is measured: norms and rotations that make queries and keys of a
projection's output, forwards and backwards, and a paged key/value cache, to which new tokens are appended and over which they attend.

A case is a dict of plain values.  Rows (kind "rows", and "grad" for the backward pass): B sequences of N tokens, H query and Hk key
heads of dim d, cut out of one projection [B, N, (H + 2 Hk) d].  `norm`: "none", "rms" or "layer" of each head; `wide`: its gains are
f32.  `pairs`: how many pairs of a head each axis turns, neighbouring places or (`halves`) places half the turned ones apart;
`grid`: the tokens' grid over these axes; `far`: sequences begin at positions up to that on the first axis.
Paged cases (kind "append" and "attn"): a pool of pages of `page` slots, of which sequence b has those that its table names, in any order,
for lens[b] slots, between lo / 1000 and hi / 1000 of `cap`.  Nn new tokens, all of them or (`ragged`) up to that many; `gone`: thousandths
of the pages that a sequence has given back.
"""

import math

import torch

own = False
THETA = 10000.0


def rows(name, B, N, H, Hk, d, dtype, norm, pairs, grid, halves=False, wide=False, far=0, kind="rows"):
    return dict(name=name, kind=kind, B=B, N=N, H=H, Hk=Hk, d=d, dtype=dtype, norm=norm, pairs=pairs, grid=grid, halves=halves, wide=wide, far=far)


def grad(*args, **more):
    return rows(*args, kind="grad", **more)


def append(name, B, Nn, H, Hk, d, page, cap, lo, hi, dtype, norm, pairs, grid, halves=False, wide=False, ragged=False):
    return dict(name=name, kind="append", B=B, Nn=Nn, H=H, Hk=Hk, d=d, page=page, cap=cap, lo=lo, hi=hi, dtype=dtype, norm=norm, pairs=pairs, grid=grid,
                halves=halves, wide=wide, ragged=ragged, gone=0)


def attn(name, B, Nn, H, Hk, d, page, cap, lo, hi, dtype, causal=True, ragged=False, gone=0):
    return dict(name=name, kind="attn", B=B, Nn=Nn, H=H, Hk=Hk, d=d, page=page, cap=cap, lo=lo, hi=hi, dtype=dtype, causal=causal, ragged=ragged, gone=gone)


def listed():
    return [
        # the smallest call: a short text's queries and keys, one axis (latency, launches, host work)
        rows("rows_text", 1, 77, 2, 2, 64, "bf16", "rms", "32", "77"),
        # a video layer at 480p: 21 latent frames of 30 x 52 tokens, three axes, neighbouring places
        rows("rows_video", 1, 32760, 40, 40, 128, "bf16", "rms", "22,21,21", "21,30,52", wide=True),
        # clips of a d = 64 model, grouped key heads, layer norm with bias, halves, an odd number of tokens far into a stream
        rows("rows_clips", 3, 4101, 30, 10, 64, "fp16", "layer", "8,12,12", "3,37,37", halves=True, far=100000),
        # fine-tuning a video layer: gradients of projections and gains
        grad("grad_video", 1, 17550, 40, 40, 128, "bf16", "rms", "16,24,24", "13,30,45", wide=True),
        # fine-tuning on small odd clips: layer norm, halves, some places not turned
        grad("grad_clips", 2, 509, 6, 2, 64, "fp16", "layer", "6,10,12", "2,15,17", halves=True, far=5000),
        # the next token of many sequences goes to its cache: latency
        append("append_token", 64, 1, 40, 8, 128, 16, 1200, 100, 900, "bf16", "none", "64", "0", halves=True),
        # a prompt's keys and values, normed and turned on three axes, pages that are no power of two
        append("append_prompt", 2, 4101, 30, 10, 64, 48, 8400, 500, 1000, "fp16", "rms", "8,12,12", "3,37,37", wide=True, ragged=True),
        # the smallest attention: one sequence's next token over a few pages
        attn("paged_first", 1, 1, 2, 2, 64, 16, 64, 300, 900, "bf16"),
        # next tokens of many sequences of different lengths, grouped heads
        attn("paged_tokens", 32, 1, 40, 8, 128, 16, 4400, 200, 1000, "bf16"),
        # two sequences with very long caches: the stream of keys and values
        attn("paged_long", 2, 1, 16, 4, 128, 64, 131100, 700, 1000, "fp16"),
        # a few drafted tokens a sequence, not as many for each, some pages given back, pages that end inside tiles
        attn("paged_drafts", 24, 7, 30, 10, 64, 24, 1500, 50, 1000, "fp16", ragged=True, gone=100),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """One more case of the same ranges; no more bytes or operations than the largest listed one, and no more than the plain
    forms can hold."""
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    while True:
        d, dtype, kind = rng.choice([64, 128]), rng.choice(["bf16", "fp16"]), rng.choice(["rows", "grad", "append", "attn", "attn"])
        Hk = _log_int(rng, 1, 40)
        H = Hk * rng.choice([1, 1, 2, 3, 5, 8])
        turned = d // 2 if rng.random() < 0.7 else d // 2 - 4 * rng.randint(1, 4)
        axes = rng.choice([1, 2, 3, 3, 4])
        cuts = sorted(rng.sample(range(1, turned), axes - 1))
        pairs = ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [turned]))
        turn = dict(norm=rng.choice(["none", "rms", "rms", "layer"]), pairs=pairs, halves=rng.random() < 0.5, wide=rng.random() < 0.5)
        B = _log_int(rng, 1, 64)
        if kind in ("rows", "grad"):
            N = _log_int(rng, 1, 33000)
            side = max(1, int((N / 3) ** (1 / max(1, axes - 1))))
            grid = ",".join(str(n) for n in [-(-N // side ** (axes - 1))] + [side] * (axes - 1))
            case = rows(None, B, N, H, Hk, d, dtype, grid=grid, far=rng.choice([0, 1000, 1000000]), kind=kind, **turn)
            held = 4 * B * N * (H + 2 * Hk) * d
        else:
            lo = rng.randint(0, 1000)
            hi = rng.randint(lo, 1000)
            page, cap = rng.choice([1, 8, 16, 16, 24, 32, 48, 64, 100, 128, 256]), _log_int(rng, 16, 131100)
            ragged = rng.random() < 0.4
            if kind == "append":
                Nn = min(cap, _log_int(rng, 1, 5000))
                side = max(1, int((Nn / 3) ** (1 / max(1, axes - 1))))
                grid = "0" if axes == 1 else ",".join(str(n) for n in [-(-Nn // side ** (axes - 1))] + [side] * (axes - 1))
                case = append(None, B, Nn, H, Hk, d, page, cap, lo, hi, dtype, grid=grid, ragged=ragged, **turn)
            else:
                Nn = min(cap, rng.choice([1, 1, _log_int(rng, 2, 16)]))
                case = attn(None, B, Nn, H, Hk, d, page, cap, lo, hi, dtype, causal=rng.random() < 0.7, ragged=ragged, gone=rng.choice([0, 0, 50, 300]))
            held = 4 * B * Hk * (cap + page) * d + 4 * B * H * Nn * d
        del case["name"]
        if held <= 1 << 30 and B * H * case.get("Nn", 1) * case.get("cap", 1) <= 1 << 28 and all(work(case)[k] <= most[k] for k in most):
            return case


def work(case):
    """What comes in once, what goes out once; of a cache's attention a product of d for a score and one for its value, over the keys in use."""
    B, H, Hk, d = case["B"], case["H"], case["Hk"], case["d"]
    if case["kind"] in ("rows", "grad"):
        elements = B * case["N"] * (H + Hk) * d
        axes = len(case["pairs"].split(","))
        return {"bytes": (4 if case["kind"] == "rows" else 6) * elements + 4 * axes * case["N"] * (B if case["far"] else 1), "flops": (10 if case["kind"] == "rows" else 20) * elements}
    new = B * case["Nn"] * (0.5 if case["ragged"] else 1.0)
    if case["kind"] == "append":
        return {"bytes": 4 * new * (H + 2 * Hk) * d, "flops": 10 * new * (H + Hk) * d}
    keys = B * (case["lo"] + case["hi"]) / 2000 * case["cap"] * (1 - case["gone"] / 1000)
    return {"bytes": 4 * d * Hk * keys + new * H * (4 * d + 4), "flops": 4 * d * H * new / B * keys}


def _pairs(case):
    return tuple(int(n) for n in case["pairs"].split(","))


def _freqs(pairs):
    return [THETA ** (-i / n) for n in pairs for i in range(n)]


def _grid_positions(case, n, g, dev):
    """int32 [n, axes], or [B, n, axes] where the sequences begin at different places; None: the slots are the positions."""
    if case["grid"] == "0":
        return None
    sides = [int(x) for x in case["grid"].split(",")]
    at, left = [], torch.arange(n, device=dev)
    for side in reversed(sides):
        at.append(left % side)
        left = left // side
    at = torch.stack(at[::-1], -1).to(torch.int32)
    if case.get("far"):
        at = at.repeat(case["B"], 1, 1)
        at[..., 0] += torch.randint(0, case["far"] + 1, (case["B"], 1), device=dev, generator=g, dtype=torch.int32)
    return at.contiguous()


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float16
    B, H, Hk, d = case["B"], case["H"], case["Hk"], case["d"]

    def rand(*shape):
        return torch.randn(*shape, device=dev, generator=g)

    def keys(*shape):           # rows of different size, as projections give them
        return (rand(*shape, d) * torch.exp(0.4 * rand(*shape, 1))).to(dt)

    s = dict(case=case)
    if case["kind"] != "attn":
        s["pairs"] = _pairs(case)
        s["freqs"] = torch.tensor(_freqs(s["pairs"]), dtype=torch.float64, device=dev)
        s["axis"] = torch.repeat_interleave(torch.arange(len(s["pairs"]), device=dev), torch.tensor(s["pairs"], device=dev))
        s["gains"] = {}
        if case["norm"] != "none":
            for name in ("q_gain", "k_gain") + (("q_bias", "k_bias") if case["norm"] == "layer" else ()):
                x = 0.2 * rand(d) + (1.0 if name.endswith("gain") else 0.0)
                s["gains"][name] = x if case["wide"] else x.to(dt)
        s["eps"] = 1e-6
    if case["kind"] in ("rows", "grad"):
        N = case["N"]
        x = keys(B, N, H + 2 * Hk)
        s["q"], s["k"] = x[:, :, :H].transpose(1, 2), x[:, :, H:H + Hk].transpose(1, 2)
        s["positions"] = _grid_positions(case, N, g, dev)
        if case["kind"] == "rows":
            s["q_out"], s["k_out"] = torch.empty(B, H, N, d, dtype=dt, device=dev), torch.empty(B, Hk, N, d, dtype=dt, device=dev)
        else:
            s["dq_out"], s["dk_out"] = rand(B, H, N, d).to(dt), rand(B, Hk, N, d).to(dt)
            dx = torch.zeros_like(x)
            s["dq"], s["dk"] = dx[:, :, :H].transpose(1, 2), dx[:, :, H:H + Hk].transpose(1, 2)
    else:
        Nn, page, cap = case["Nn"], case["page"], case["cap"]
        per = -(-cap // page)
        n_pages = B * per + 3
        # page-major, the heads of a page behind one another
        s["pool_k"], s["pool_v"] = keys(n_pages, Hk, page), rand(n_pages, Hk, page, d).to(dt)
        used = torch.randint(cap * case["lo"] // 1000, cap * case["hi"] // 1000 + 1, (B,), device=dev, generator=g, dtype=torch.int32)
        s["new_lens"] = torch.randint(0, Nn + 1, (B,), device=dev, generator=g, dtype=torch.int32) if case["ragged"] else None
        new = s["new_lens"] if case["ragged"] else torch.full_like(used, Nn)
        s["lens"] = torch.maximum(used, new)                # the new tokens' slots are counted in
        table = torch.randperm(n_pages, device=dev, generator=g)[:B * per].view(B, per)
        slots = page * torch.arange(per, device=dev)[None]
        there = slots < s["lens"][:, None]
        if case["gone"]:
            there &= (torch.rand(B, per, device=dev, generator=g) >= case["gone"] / 1000) | (slots + page > (s["lens"] - new)[:, None])
        s["table"] = torch.where(there, table, -1).to(torch.int32)
        if case["kind"] == "append":
            x = keys(B, Nn, H + 2 * Hk)
            s["q"], s["k"], s["v"] = x[:, :, :H].transpose(1, 2), x[:, :, H:H + Hk].transpose(1, 2), x[:, :, H + Hk:].transpose(1, 2)
            s["q_out"] = torch.zeros(B, H, Nn, d, dtype=dt, device=dev)       # rows behind a sequence's new tokens stay as they are
            s["positions"] = _grid_positions(case, Nn, g, dev)
        else:
            s["q"] = rand(B, H, Nn, d).to(dt)
            s["o"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros(B, H, Nn, device=dev)
    if own:
        import paper_2511_23113_amd as dbsp
        s["dbsp"] = dbsp
        if case["kind"] != "attn":
            s["rotary"] = dbsp.Rotary(s["pairs"], theta=THETA, halves=case["halves"])
            s["norm"] = None if case["norm"] == "none" else dbsp.HeadNorm(kind=case["norm"], eps=s["eps"], **s["gains"])
        if case["kind"] in ("append", "attn"):
            s["cache"] = dbsp.PagedKVCache(s["pool_k"], s["pool_v"], s["table"], s["lens"])
    return s


def run(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "rows":
        if own:
            s["dbsp"].qk_norm_rope_fwd(s["q"], s["k"], norm=s["norm"], rotary=s["rotary"], positions=s["positions"], q_out=s["q_out"], k_out=s["k_out"])
        else:
            cos, sin = _turns(s, s["positions"])
            for name in ("q", "k"):
                s[name + "_out"].copy_(_turn(s, _normed(s, s[name], name)[0], cos, sin).to(s["q"].dtype))
        return {"q": s["q_out"], "k": s["k_out"]}
    if kind == "grad":
        if own:
            _, _, gains = s["dbsp"].qk_norm_rope_bwd(s["q"], s["k"], s["dq_out"], s["dk_out"], norm=s["norm"], rotary=s["rotary"], positions=s["positions"],
                                                     dq=s["dq"], dk=s["dk"])
        else:
            gains = {}
            cos, sin = _turns(s, s["positions"])
            for name in ("q", "k"):
                dx, gain, bias = _grad_plain(s, name, cos, sin)
                s["d" + name].copy_(dx.to(s["q"].dtype))
                gains.update({name + "_gain": gain, name + "_bias": bias})
        return {"dq": s["dq"], "dk": s["dk"], **{name: gains[name] for name in s["gains"]}}
    if kind == "append":
        if own:
            s["dbsp"].paged_append(s["cache"], s["k"], s["v"], new_lens=s["new_lens"], q=s["q"], q_out=s["q_out"], norm=s["norm"], rotary=s["rotary"],
                                   positions=s["positions"])
        else:
            _append_plain(s)
        return {"k": s["pool_k"], "v": s["pool_v"], "q": s["q_out"]}
    if own:
        s["dbsp"].paged_attn_fwd(s["cache"], s["q"], q_lens=s["new_lens"], causal=case["causal"], o=s["o"], lse=s["lse"])
    else:
        _attn_plain(s)
    return {"o": s["o"], "lse": s["lse"]}


def _turns(s, positions):
    """Cosines and sines [.., 1, n, pairs] of every token's angles, which are formed in 64 bits."""
    angles = positions.double()[..., s["axis"]] * s["freqs"]
    angles = angles.unsqueeze(-3)
    return angles.cos().float(), angles.sin().float()


def _normed(s, x, name):
    """The head's norm in 32 bits: the result, the values before gain and bias, and the factor 1 / root."""
    x, case = x.float(), s["case"]
    if case["norm"] == "none":
        return x, x, None
    if case["norm"] == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"])
    hat = x * r
    y = hat * s["gains"][name + "_gain"].float()
    return (y + s["gains"][name + "_bias"].float() if case["norm"] == "layer" else y), hat, r


def _turn(s, x, cos, sin):
    n = cos.shape[-1]
    y = x.clone()
    if s["case"]["halves"]:
        a, b = x[..., :n], x[..., n:2 * n]
        y[..., :n], y[..., n:2 * n] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
        y[..., 0:2 * n:2], y[..., 1:2 * n:2] = a * cos - b * sin, a * sin + b * cos
    return y


def _grad_plain(s, name, cos, sin):
    dn = _turn(s, s["d" + name + "_out"].float(), cos, -sin)
    if s["case"]["norm"] == "none":
        return dn, None, None
    _, hat, r = _normed(s, s[name], name)
    gain = (dn * hat).sum((0, 1, 2), dtype=torch.float64).float()
    bias = dn.sum((0, 1, 2), dtype=torch.float64).float()
    e = dn * s["gains"][name + "_gain"].float()
    dx = e - hat * (e * hat).mean(-1, keepdim=True)
    if s["case"]["norm"] == "layer":
        dx = dx - e.mean(-1, keepdim=True)
    return dx * r, gain, bias


def _append_plain(s):
    case, lens = s["case"], s["lens"].long()
    Nn, page = case["Nn"], case["page"]
    new = s["new_lens"].long() if s["new_lens"] is not None else torch.full_like(lens, Nn)
    t = torch.arange(Nn, device=lens.device)
    there = t < new[:, None]                                                 # [B, Nn]
    slot = torch.where(there, (lens - new)[:, None] + t, 0)
    cos, sin = _turns(s, slot[..., None] if s["positions"] is None else s["positions"])
    q, k = (_turn(s, _normed(s, s[name], name)[0], cos, sin).to(s["q"].dtype) for name in ("q", "k"))
    s["q_out"].copy_(torch.where(there[:, None, :, None], q, s["q_out"]))
    page_of = s["table"].long().gather(1, slot // page)
    at, tok = there.nonzero(as_tuple=True)
    where = page_of[at, tok], slot[at, tok] % page
    s["pool_k"][where[0], :, where[1]] = k[at, :, tok]
    s["pool_v"][where[0], :, where[1]] = s["v"][at, :, tok]


def _attn_plain(s):
    case, q, lens, table = s["case"], s["q"], s["lens"].long(), s["table"].long()
    B, H, Nq, d = q.shape
    Hk, page = case["Hk"], case["page"]
    G, cap = H // Hk, table.shape[1] * page
    new = s["new_lens"].long() if s["new_lens"] is not None else torch.full_like(lens, Nq)
    t, slot = torch.arange(Nq, device=q.device), torch.arange(cap, device=q.device)
    held = (table >= 0).repeat_interleave(page, 1) & (slot < lens[:, None])                       # [B, cap]
    until = (lens - new)[:, None] + t + 1 if case["causal"] else lens[:, None].expand(B, Nq)
    seen = held[:, None] & (slot < until[:, :, None])                                             # [B, Nq, cap]

    def gathered(pool):
        x = pool[table.clamp(min=0)].transpose(1, 2).reshape(B, Hk, cap, d).float()
        return x.masked_fill_(~held[:, None, :, None], 0.0)
    scores = ((q.float() * (1 / math.sqrt(d))).view(B, Hk, G * Nq, d) @ gathered(s["pool_k"]).transpose(-1, -2)).view(B, Hk, G, Nq, cap)
    scores = torch.where(seen[:, None, None], scores, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(scores - top)
    del scores
    total = p.sum(-1, keepdim=True)
    o = (p.view(B, Hk, G * Nq, cap) @ gathered(s["pool_v"])).view(B, Hk, G, Nq, d)
    some = total > 0
    o = torch.where(some, o / total, 0.0).view(B, H, Nq, d)
    lse = torch.where(some, top + torch.log(total), -math.inf).view(B, H, Nq)
    there = (t < new[:, None])[:, None]
    s["o"].copy_(torch.where(there[..., None], o.to(q.dtype), s["o"]))
    s["lse"].copy_(torch.where(there, lse, s["lse"]))


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attn":
        return _attn_exact(s)
    if case["kind"] == "append":
        return _append_exact(s)
    positions = s["positions"] if s["positions"].dim() == 3 else s["positions"][None]
    out = {}
    for name in ("q", "k"):
        x = s[name].double()
        if case["kind"] == "rows":
            out[name] = _row_exact(s, x, positions[:, None], {n: w.double() for n, w in s["gains"].items()}, name)
            continue
        x = x.detach().requires_grad_()
        gains = {n: w.double().requires_grad_() for n, w in s["gains"].items() if n.startswith(name)}
        y = _row_exact(s, x, positions[:, None], gains, name)
        found = torch.autograd.grad(y, [x, *gains.values()], s["d" + name + "_out"].double())
        out["d" + name] = found[0]
        out.update(zip(gains, found[1:]))
        del y, found
    return out


def _row_exact(s, x, positions, gains, name):
    """Norm and rotation in 64 bits, pairs as complex numbers."""
    case = s["case"]
    if case["norm"] != "none":
        if case["norm"] == "layer":
            x = x - x.sum(-1, keepdim=True) / case["d"]
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["d"] + s["eps"]) * gains[name + "_gain"]
        if case["norm"] == "layer":
            x = x + gains[name + "_bias"]
    n, pieces, first = sum(s["pairs"]), [], 0
    for axis, count in enumerate(s["pairs"]):
        angle = positions[..., axis, None].double() * torch.tensor(_freqs(s["pairs"])[first:first + count], dtype=torch.float64, device=x.device)
        pieces.append(torch.polar(torch.ones_like(angle), angle))
        first += count
    if case["halves"]:
        z = torch.complex(x[..., :n].contiguous(), x[..., n:2 * n].contiguous()) * torch.cat(pieces, -1)
        return torch.cat([z.real, z.imag, x[..., 2 * n:]], -1)
    z = torch.view_as_complex(x[..., :2 * n].unflatten(-1, (n, 2)).contiguous()) * torch.cat(pieces, -1)
    return torch.cat([torch.view_as_real(z).flatten(-2), x[..., 2 * n:]], -1)


def _append_exact(s):
    """Sequence by sequence, the new tokens that it has."""
    case, page = s["case"], s["case"]["page"]
    gains = {n: w.double() for n, w in s["gains"].items()}
    k, v, q = s["pool_k"].double(), s["pool_v"].double(), s["q_out"].double()
    for b, n in enumerate(s["lens"].tolist()):
        new = case["Nn"] if s["new_lens"] is None else int(s["new_lens"][b])
        slots = torch.arange(n - new, n, device=k.device)
        positions = slots[:, None] if s["positions"] is None else s["positions"][:new]
        pages, places = s["table"][b].long()[slots // page], slots % page
        q[b, :, :new] = _row_exact(s, s["q"][b, :, :new].double(), positions[None], gains, "q")
        k[pages, :, places] = _row_exact(s, s["k"][b, :, :new].double(), positions[None], gains, "k").transpose(0, 1)
        v[pages, :, places] = s["v"][b, :, :new].double().transpose(0, 1)
    return {"k": k, "v": v, "q": q}


def _attn_exact(s):
    """Sequence by sequence, over the keys that it holds and no others, in 64 bits."""
    case, page = s["case"], s["case"]["page"]
    H, Hk, Nq, d = case["H"], case["Hk"], case["Nn"], case["d"]
    o, lse = s["o"].double(), s["lse"].double()
    for b, n in enumerate(s["lens"].tolist()):
        new = Nq if s["new_lens"] is None else int(s["new_lens"][b])
        slots = torch.arange(n, device=o.device)
        pages = s["table"][b].long()[slots // page]
        slots, pages = slots[pages >= 0], pages[pages >= 0]
        keys, values = (s[name][pages, :, slots % page].double().transpose(0, 1) for name in ("pool_k", "pool_v"))
        logits = torch.einsum("kgtd,knd->kgtn", s["q"][b].view(Hk, H // Hk, Nq, d)[:, :, :new].double(), keys) / math.sqrt(d)
        if case["causal"]:
            logits.masked_fill_(slots[None] > (n - new + torch.arange(new, device=o.device))[:, None], -math.inf)
        z = torch.logsumexp(logits, -1)
        prob = torch.exp(logits - torch.where(z == -math.inf, 0.0, z)[..., None])
        o[b].view(Hk, H // Hk, Nq, d)[:, :, :new] = torch.einsum("kgtn,knd->kgtd", prob, values)
        lse[b].view(Hk, H // Hk, Nq)[:, :, :new] = z
    return {"o": o, "lse": lse}
