"""Oracle of the operators around the step, in float64 numpy with plain loops:
block attention over a shared prefix and a paged cache, the attention weight
each key received, eviction by it, and verification of drafts from given
probabilities.  Beside each computed value stands the size that its rounding
errors scale with, so that tests can derive their tolerances."""
from __future__ import annotations

import numpy as np


def own_rows(pages, table, n, page_size):
    """[n, Hkv, D] of one sequence from [n_pages, page_size, Hkv, D] pages."""
    out = np.zeros((n,) + pages.shape[2:], dtype=np.float64)
    for j in range(n):
        out[j] = pages[table[j // page_size], j % page_size]
    return out


def sees(n, L, i, mask_row):
    """Which of n own slots block position i sees; mask_row None: all."""
    vis = np.ones(n, dtype=bool)
    if mask_row is not None:
        bits = int(mask_row) & ((1 << 64) - 1)
        for j in range(max(0, n - L), n):
            vis[j] = (bits >> (j - (n - L))) & 1
    return vis


def block_attention(q, own_k, own_v, prefix, mask, scale):
    """q [B, L, H, D]; own_k, own_v lists of [n_b, Hkv, D]; prefix None or (k, v)
    [P, Hkv, D]; mask None or [B, L] ints.  Returns out, lse, the sums of
    p |v|, and the largest scale * sum |q k| of a row."""
    B, L, H, D = q.shape
    out, mag = np.zeros((B, L, H, D)), np.zeros((B, L, H, D))
    lse, size = np.full((B, L, H), -np.inf), np.zeros((B, L, H))
    for b in range(B):
        n, Hkv = own_k[b].shape[:2]
        for i in range(L):
            vis = sees(n, L, i, None if mask is None else mask[b, i])
            k, v = own_k[b][vis], own_v[b][vis]
            if prefix is not None:
                k, v = np.concatenate([prefix[0], k]), np.concatenate([prefix[1], v])
            if len(k) == 0:
                continue
            for h in range(H):
                kh, vh = k[:, h // (H // Hkv)], v[:, h // (H // Hkv)]
                s = scale * (kh @ q[b, i, h])
                m = s.max()
                if m == -np.inf:
                    continue
                p = np.exp(s - m)
                lse[b, i, h] = m + np.log(p.sum())
                p /= p.sum()
                out[b, i, h], mag[b, i, h] = p @ vh, p @ np.abs(vh)
                size[b, i, h] = scale * (np.abs(kh) @ np.abs(q[b, i, h])).max()
    return out, lse, mag, size


def cache_score(q, own_k, lse, mask, scale, decay, score):
    """(new scores, their error scale): [B, Hkv, cap]."""
    B, L, H, _ = q.shape
    out, err = np.zeros_like(score, dtype=np.float64), np.zeros_like(score, dtype=np.float64)
    for b in range(B):
        n, Hkv = own_k[b].shape[:2]
        G = H // Hkv
        for hk in range(Hkv):
            out[b, hk, :n] = decay * score[b, hk, :n]
            err[b, hk, :n] = np.abs(out[b, hk, :n])
            for i in range(L):
                vis = sees(n, L, i, None if mask is None else mask[b, i])
                for h in range(hk * G, hk * G + G):
                    if lse[b, i, h] == -np.inf:
                        continue
                    k = own_k[b][vis, hk]
                    p = np.exp(scale * (k @ q[b, i, h]) - lse[b, i, h])
                    out[b, hk, :n][vis] += p
                    err[b, hk, :n][vis] += p * (2 + abs(lse[b, i, h]) + scale * (np.abs(k) @ np.abs(q[b, i, h])))
    return out, err


def cache_evict(score, pos, n, next_pos, budget, recent):
    """One head of one sequence: (score, pos, moves as (source, target) pairs)."""
    cap = len(score)
    out_s, out_p = np.zeros(cap, dtype=score.dtype), np.full(cap, -1, dtype=pos.dtype)
    m = min(n, budget)
    out_s[:m], out_p[:m] = score[:m], pos[:m]
    moves = []
    if n > budget:
        def order(j):
            if pos[j] >= next_pos - recent:
                return (0, 0.0, j)
            return (2, 0.0, j) if np.isnan(score[j]) else (1, -float(score[j]), j)
        kept = set(sorted(range(n), key=order)[:m])
        moves = list(zip([j for j in range(m, n) if j in kept], [j for j in range(m) if j not in kept]))
        for s, d in moves:
            out_s[d], out_p[d] = score[s], pos[s]
    return out_s, out_p, moves


def draft_verify(target, draft, tok, n, u, noise):
    """One block: (accepted, token, whether rounding can change either)."""
    a = 0
    close = False
    while a < n:
        lhs, rhs = float(u[a]) * float(draft[a, tok[a]]), float(target[a, tok[a]])
        close |= abs(lhs - rhs) <= 2.0 ** -22 * max(abs(lhs), abs(rhs)) and lhs != rhs
        if not lhs < rhs:
            break
        a += 1
    p = target[a].astype(np.float64)
    w = np.maximum(p - draft[a], 0.0) if a < n else p
    if not (w > 0).any():
        w = p
    with np.errstate(divide="ignore", invalid="ignore"):
        r = np.where(w > 0, w / noise.astype(np.float64), 0.0)
    if not (r > 0).any():
        return a, -1, close
    order = np.argsort(-r, kind="stable")
    best = int(order[0])
    if len(r) > 1 and r[order[1]] != r[best]:
        close |= bool(r[order[1]] > r[best] * (1 - 2.0 ** -21))
    return a, best, close
