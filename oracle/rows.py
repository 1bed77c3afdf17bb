"""Plain definitions of the norms and rotations of queries and keys, and of a paged cache's operators, in float64 (no reference code
exists; the definitions are those of dbsp.h)."""

from __future__ import annotations

import numpy as np

from .cache import seen_slots


def pair_places(R: int, halves: bool):
    """Places of the first and second values of the R pairs."""
    p = np.arange(R)
    return (p, p + R) if halves else (2 * p, 2 * p + 1)


def angles(positions, pairs, freqs):
    """positions [..., axes] -> [..., R]."""
    axis = np.repeat(np.arange(len(pairs)), pairs)
    return np.asarray(positions, dtype=np.float64)[..., axis] * np.asarray(freqs, dtype=np.float64)


def rotate(x, a, halves: bool):
    """x [..., d] by the angles a [..., R]; -a takes it back."""
    y = np.array(x, dtype=np.float64, copy=True)
    i, j = pair_places(a.shape[-1], halves)
    c, s = np.cos(a), np.sin(a)
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., i] * s + x[..., j] * c
    return y


def normed(x, kind: str, eps: float):
    """(x - mu) r and r."""
    x = np.asarray(x, dtype=np.float64)
    if kind == "layer":
        x = x - x.mean(-1, keepdims=True)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x * r, r


def rows_fwd(x, kind, gain, bias, eps, a, halves):
    x = np.asarray(x, dtype=np.float64)
    n = x if kind == "none" else normed(x, kind, eps)[0] * gain + bias
    return n if a is None else rotate(n, a, halves)


def rows_bwd(x, dy, kind, gain, eps, a, halves):
    """dx, and the gradients of gain and bias, summed over all but the last dimension."""
    dn = np.asarray(dy, dtype=np.float64) if a is None else rotate(np.asarray(dy, dtype=np.float64), -a, halves)
    if kind == "none":
        return dn, None, None
    hat, r = normed(x, kind, eps)
    e = dn * gain
    dx = e - (e * hat).mean(-1, keepdims=True) * hat
    if kind == "layer":
        dx = dx - e.mean(-1, keepdims=True)
    over = tuple(range(dn.ndim - 1))
    return r * dx, (dn * hat).sum(over), dn.sum(over)


def slot_place(pages, slot: int, page_size: int, n_pages: int):
    """(page, place in it) of a slot of a sequence with this table, or None."""
    page = int(pages[slot // page_size])
    return (page, slot % page_size) if 0 <= page < n_pages else None


def paged_append(pool_k, pool_v, pages, lens, k, v, new_lens):
    """New pools, from rows [B, Hk, Nn, d] as they are (normed and rotated already)."""
    pool_k, pool_v = np.array(pool_k, copy=True), np.array(pool_v, copy=True)
    n_pages, _, page_size, _ = pool_k.shape
    for b, n in enumerate(lens):
        for t in range(new_lens[b]):
            slot = n - new_lens[b] + t
            at = slot_place(pages[b], slot, page_size, n_pages) if slot >= 0 else None
            if at is not None:
                pool_k[at[0], :, at[1]], pool_v[at[0], :, at[1]] = k[b, :, t], v[b, :, t]
    return pool_k, pool_v


def paged_attention(q, pool_k, pool_v, pages, lens, q_lens, causal, scale):
    """q [B,H,Nq,d].  Returns O, LSE (NaN where a sequence has no such query), the sum of p |v| beside every O, and how many keys each row
    sees."""
    B, H, Nq, d = q.shape
    n_pages, Hk, page_size, _ = pool_k.shape
    O, A, LSE = np.full((B, H, Nq, d), np.nan), np.full((B, H, Nq, d), np.nan), np.full((B, H, Nq), np.nan)
    seen = np.zeros((B, H, Nq), dtype=np.int64)
    for b in range(B):
        n, new = int(lens[b]), int(q_lens[b])
        slots = np.arange(n)
        page = np.asarray(pages[b], dtype=np.int64)[slots // page_size]
        there = (page >= 0) & (page < n_pages)
        for t in range(new):
            here = slots[there & (slots < seen_slots(n, new, t, causal))]
            at, off = page[here], here % page_size
            for h in range(H):
                hk = h // (H // Hk)
                seen[b, h, t] = len(here)
                if not len(here):
                    O[b, h, t], A[b, h, t], LSE[b, h, t] = 0.0, 0.0, -np.inf
                    continue
                K, V = pool_k[at, hk, off].astype(np.float64), pool_v[at, hk, off].astype(np.float64)
                s = scale * (K @ q[b, h, t].astype(np.float64))
                e = np.exp(s - s.max())
                p = e / e.sum()
                O[b, h, t], A[b, h, t], LSE[b, h, t] = p @ V, p @ np.abs(V), s.max() + np.log(e.sum())
    return O, LSE, A, seen
