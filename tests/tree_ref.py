"""64-bit references of the operators on trees of drafted tokens, from their definitions, on the CPU."""
import math

import numpy as np
import torch


def random_tree(rng, n, ways):
    """Parents of n rows: ways 1 a chain, else about `ways` children a row."""
    if ways == 1:
        return np.arange(-1, n - 1).astype(np.int32)
    return np.array([-1] + [max(0, (i - 1) // ways - int(rng.integers(0, 3))) for i in range(1, n)], np.int32)


def ancestors(parent):
    """bool [n][n]: column c of row i is row i or an ancestor of it; parents out of range count as none."""
    n = len(parent)
    seen = np.zeros((n, n), bool)
    for i, p in enumerate(parent):
        if 0 <= p < i:
            seen[i] = seen[p]
        seen[i, i] = True
    return seen


def pack(seen, words):
    """Rows of bools as int32 words, the lowest column in the lowest bit."""
    out = np.zeros((seen.shape[0], words), np.uint32)
    for i, c in zip(*np.nonzero(seen)):
        out[i, c // 32] |= np.uint32(1 << (c % 32))
    return out.view(np.int32)


def attention(q, k, v, dk, dv, q_pos, seen, scale, window=0):
    """One sequence, one layer: q [rows][H][d], cache k, v [Hkv][kv][*], drafted dk, dv [Hkv][rows][*], seen
    [rows][rows]: outputs and log-sum-exps.  Rows that see nothing: zeros and -inf."""
    rows, H = q.shape[:2]
    G = H // k.shape[0]
    kv = k.shape[1]
    out, lse = np.zeros((rows, H, v.shape[2])), np.full((rows, H), -np.inf)
    j = np.arange(kv)
    for i in range(rows):
        at = int(q_pos[i])
        context = j <= at
        tree = seen[i].copy()
        if window:
            context &= j > at - window
            tree &= q_pos.astype(np.int64) > at - window
        if not context.any() and not tree.any():
            continue
        for h in range(H):
            g = h // G
            keys = np.concatenate([k[g][context], dk[g][tree]])
            values = np.concatenate([v[g][context], dv[g][tree]])
            with np.errstate(invalid="ignore"):
                x = keys @ q[i, h] * scale
                m = x.max()
                p = np.exp(x - m)
                out[i, h] = p @ values / p.sum()
                lse[i, h] = m + math.log(p.sum())
    return out, lse


def weights(p):
    """Probabilities as verification takes them."""
    p = np.asarray(p, np.float64)
    return np.where((p > 0) & np.isfinite(p), p, 0.0)


def verify(target, draft, tokens, parent, u_accept, u_sample, max_path):
    """One sequence: (accepted rows, next token), by the definition."""
    n, V = target.shape
    if n == 0:
        return [], -1
    cur, path = 0, [0]
    while True:
        p = weights(target[cur])
        w, b, found = p.copy(), 1.0, None
        a = 0.0
        if len(path) < max_path:
            for c in range(cur + 1, n):
                x = tokens[c]
                if parent[c] != cur or not 0 <= x < V:
                    continue
                q = 1.0 if draft is None else weights(draft[cur])[x]
                if w[x] > 0 and float(u_accept[c]) * q * b < w[x]:
                    found = c
                    break
                if draft is None:
                    b -= w[x]
                    w[x] = 0
                else:
                    a += b
                    w = np.maximum(p - a * weights(draft[cur]), 0)
                    b = math.fsum(w)
        if found is None:
            break
        cur = found
        path.append(cur)
    if not w.any():
        w = p
    if not w.any():
        return path, -1
    run = np.cumsum(w)
    hit = np.nonzero((run > float(u_sample) * run[-1]) & (w > 0))[0]
    return path, int(hit[0]) if len(hit) else int(np.nonzero(w)[0][-1])


def near_tie(target, draft, tokens, parent, u_accept, u_sample, max_path, eps=1e-12):
    """Whether a comparison of the walk or the draw is closer than 64-bit sums in another order may decide."""
    lo = verify(target, draft, tokens, parent, np.asarray(u_accept, np.float64) * (1 - eps), float(u_sample) * (1 - eps), max_path)
    hi = verify(target, draft, tokens, parent, np.asarray(u_accept, np.float64) * (1 + eps), float(u_sample) * (1 + eps), max_path)
    return lo != hi


def as_tensor(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)
