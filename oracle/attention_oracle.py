"""fp64 CPU oracle of the calls around a verification step's attention, written from their formulas (test infrastructure only).

Inputs are float64 arrays that hold the stored values.  A batch is tree_off [S + 1] over token rows; `sees` is a list with one
boolean [T, T] matrix per sequence.
"""
import numpy as np


def ancestors(parents):
    """sees[t, j]: token j is t itself or one of its ancestors.  parents[t] < t, or -1 for a child of the last cached token."""
    n = len(parents)
    sees = np.zeros((n, n), dtype=bool)
    for t, p in enumerate(parents):
        if p >= 0:
            sees[t] = sees[p]
        sees[t, t] = True
    return sees


def chain(n):
    return np.tril(np.ones((n, n), dtype=bool))


def pack(sees_list, M, max_tree, fill=0):
    """Packed bits [M, ceil(max_tree / 32)] int32; rows of no sequence and bits past a tree's end hold `fill`'s bits."""
    words = (max_tree + 31) // 32
    bits = np.full((M, 32 * words), bool(fill))
    row = 0
    for s in sees_list:
        bits[row:row + len(s), :s.shape[1]] = s
        row += len(s)
    return np.packbits(bits, axis=1, bitorder="little").view("<u4").astype(np.uint32).view(np.int32)


def attention(q, kt, vt, kc, vc, lens, off, sees, scale):
    """(out [M, H, D], lse [M, H], bound [M, H, D], spread [M, H]): bound = sum_j p_j |v_j|, spread = the largest
    scale * sum_i |q_i k_ji| over the keys that are seen.  What a row does not see has no part, whatever it holds."""
    M, H, D = q.shape
    G = H // kt.shape[1]
    out, bound = np.zeros((M, H, D)), np.zeros((M, H, D))
    lse, spread = np.full((M, H), -np.inf), np.zeros((M, H))
    for s, n in enumerate(lens):
        for h in range(H):
            for t in range(off[s + 1] - off[s]):
                row = off[s] + t
                seen = np.flatnonzero(sees[s][t])
                k = np.concatenate([kc[s, h // G, :n], kt[off[s] + seen, h // G]]) if kc is not None else kt[off[s] + seen, h // G]
                v = np.concatenate([vc[s, h // G, :n], vt[off[s] + seen, h // G]]) if vc is not None else vt[off[s] + seen, h // G]
                if len(k) == 0:
                    continue
                with np.errstate(all="ignore"):
                    a = scale * (k @ q[row, h])
                    top = a.max()
                    if top == -np.inf:
                        continue
                    p = np.exp(a - top)
                    total = p.sum()
                    lse[row, h] = top + np.log(total)
                    p /= total
                    out[row, h] = (p[:, None] * v).sum(axis=0)
                    bound[row, h] = (p[:, None] * np.abs(v)).sum(axis=0)
                    spread[row, h] = scale * (np.abs(k) @ np.abs(q[row, h])).max()
    return out, lse, bound, spread


def weights(q, kt, kc, lens, off, sees, scale, lse, row_weight=None, w_in=None, decay=1.0, capacity=None):
    """(cache_w [S, Hk, capacity], tree_w [M, Hk], the same two of |row_weight| instead).  Entries behind a length: w_in or 0."""
    M, H, D = q.shape
    S, Hk = len(lens), kt.shape[1]
    G = H // Hk
    rw = np.ones(M) if row_weight is None else row_weight
    cap = capacity if kc is None else kc.shape[2]
    cw, tw = np.zeros((S, Hk, cap)), np.zeros((M, Hk))
    acw, atw = np.zeros_like(cw), np.zeros_like(tw)
    for s, n in enumerate(lens):
        for h in range(H):
            for t in range(off[s + 1] - off[s]):
                row = off[s] + t
                if lse[row, h] == -np.inf:
                    continue
                if n:
                    p = np.exp(scale * (kc[s, h // G, :n] @ q[row, h]) - lse[row, h])
                    cw[s, h // G, :n] += rw[row] * p
                    acw[s, h // G, :n] += abs(rw[row]) * p
                seen = off[s] + np.flatnonzero(sees[s][t])
                p = np.exp(scale * (kt[seen, h // G] @ q[row, h]) - lse[row, h])
                tw[seen, h // G] += rw[row] * p
                atw[seen, h // G] += abs(rw[row]) * p
        if w_in is not None:
            cw[s, :, :n] += decay * w_in[s, :, :n]
            acw[s, :, :n] += np.abs(decay * w_in[s, :, :n])
    return cw, tw, acw, atw


def kept_entries(w, n, budget, recent):
    """Indices that stay of n entries with weights w, ascending."""
    if n <= budget:
        return np.arange(n)
    first = n - recent
    order = sorted(range(first), key=lambda i: (0, -float(w[i]), i) if w[i] == w[i] else (1, 0.0, i))
    return np.array(sorted(order[:budget - recent]) + list(range(first, n)), dtype=np.int64)


def block_norm(y, residual, post_norm=False, w_post=None, gate=None, sigmoid=False, scale=1.0, w_pre=None, eps=0.0):
    """(r, x, |scale gate z|); gate broadcasts against [M, d]."""
    z = y
    if post_norm:
        z = y / np.sqrt((y * y).mean(axis=1, keepdims=True) + eps) * (1.0 if w_post is None else w_post)
    if gate is not None:
        z = z * (1.0 / (1.0 + np.exp(-gate)) if sigmoid else gate)
    z = scale * z
    r = z if residual is None else residual + z
    x = r / np.sqrt((r * r).mean(axis=1, keepdims=True) + eps) * (1.0 if w_pre is None else w_pre)
    return r, x, np.abs(z)
