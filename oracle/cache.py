"""Plain definitions of the key/value cache's operators, in float64 and one query at a time (no reference code exists; the
definitions are those of dbsp.h)."""

from __future__ import annotations

import numpy as np


def seen_slots(length: int, q_len: int, t: int, causal: bool) -> int:
    """Own slots that query t of q_len new tokens sees: all used ones, causal those up to its own."""
    return max(0, min(length, length - q_len + t + 1)) if causal else length


def cache_attention(q, lens, k=None, v=None, prefix_k=None, prefix_v=None, q_lens=None, causal=True, scale=None):
    """q [B,H,Nq,d]; k, v [B,Hk,cap,d]; prefix_k, prefix_v [Hk,P,d]; lens, q_lens [B].  Returns O, LSE (NaN where a sequence has no
    such query), the sum of p |v| beside every O, and the weights [B,Hk,cap] that the own keys draw."""
    B, H, Nq, d = q.shape
    Hk = (k.shape[1] if k is not None else prefix_k.shape[0])
    cap = k.shape[2] if k is not None else 0
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    O, A, LSE = np.full((B, H, Nq, d), np.nan), np.full((B, H, Nq, d), np.nan), np.full((B, H, Nq), np.nan)
    W = np.zeros((B, Hk, cap))
    for b in range(B):
        n, new = (int(lens[b]) if k is not None else 0), (Nq if q_lens is None else int(q_lens[b]))
        for h in range(H):
            hk = h // (H // Hk)
            keys = [prefix_k[hk]] if prefix_k is not None else []
            values = [prefix_v[hk]] if prefix_v is not None else []
            P = prefix_k.shape[1] if prefix_k is not None else 0
            if k is not None:
                keys.append(k[b, hk, :n])
                values.append(v[b, hk, :n])
            K, V = np.concatenate(keys).astype(np.float64), np.concatenate(values).astype(np.float64)
            for t in range(new):
                m = P + seen_slots(n, new, t, causal)
                if m == 0:
                    O[b, h, t], A[b, h, t], LSE[b, h, t] = 0.0, 0.0, -np.inf
                    continue
                s = scale * (K[:m] @ q[b, h, t].astype(np.float64))
                top = s.max()
                e = np.exp(s - top)
                p = e / e.sum()
                O[b, h, t], A[b, h, t], LSE[b, h, t] = p @ V[:m], p @ np.abs(V[:m]), top + np.log(e.sum())
                W[b, hk, :m - P] += p[P:]
    return O, LSE, A, W


def keepers(weights, positions, length: int, budget: int, sinks: int, keep_from) -> list:
    """Slots of one (sequence, head) that stay, ascending."""
    def rank(i):
        safe = positions[i] < sinks or (keep_from is not None and positions[i] >= keep_from)
        w = -np.inf if np.isnan(weights[i]) else float(weights[i])
        return (0 if safe else 1, 0.0 if safe else -w, i)
    return sorted(sorted(range(length), key=rank)[:budget])


def cache_evict(k, v, weights, positions, lens, budget: int, sinks: int = 0, keep_from=None):
    """New k, v, weights, positions, lens."""
    k, v, weights, positions, lens = (np.array(x, copy=True) for x in (k, v, weights, positions, lens))
    B, Hk = k.shape[:2]
    for b in range(B):
        n = int(lens[b])
        if n <= budget:
            continue
        for h in range(Hk):
            stay = keepers(weights[b, h], positions[b, h], n, budget, sinks, None if keep_from is None else int(keep_from[b]))
            there = set(stay)
            holes = [i for i in range(budget) if i not in there]
            for to, frm in zip(holes, [i for i in stay if i >= budget]):
                for x in (k, v, weights, positions):
                    x[b, h, to] = x[b, h, frm]
            weights[b, h, budget:n] = 0
        lens[b] = budget
    return k, v, weights, positions, lens
