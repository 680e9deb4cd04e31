"""fp64 CPU oracle of the calls around a serving step (head norm and rotation, paged cache, attention of single tokens, draft
verification), written from their formulas (test infrastructure only).  Inputs are float64 arrays that hold the stored values."""
import numpy as np


def places(lens, off, sees):
    """Place of every token row of the sequences: entries in front of its tree plus its depth there."""
    return np.concatenate([n + s.sum(axis=1) - 1 for n, s in zip(lens, sees)]) if len(lens) else np.zeros(0)


def head_rope(x, w, place, freq, rot, interleaved=False, norm=False, eps=0.0):
    """(out, |parts|) of heads x [M, H, D]: the second is what roundings of the result's terms are relative to."""
    if norm:
        x = x / np.sqrt((x * x).mean(axis=2, keepdims=True) + eps) * (1.0 if w is None else w)
    out, size = x.copy(), np.abs(x)
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        angle = place * freq[i]
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        size[..., a] = size[..., b] = np.hypot(x[..., a], x[..., b])
    return out, size


def codes_i8(rows):
    """(codes, scales float32) of rows [..., D]."""
    amax = np.abs(rows).max(axis=-1).astype(np.float32)
    with np.errstate(all="ignore"):
        inv = np.minimum(np.float32(127) / amax, np.finfo(np.float32).max)
        scale = amax / np.float32(127)
        odd = ~np.isfinite(rows).all(axis=-1)
        codes = np.rint(np.where(odd[..., None], 0.0, rows) * np.where(odd, 0, inv).astype(np.float64)[..., None])
    return codes, np.where(odd, np.float32(np.nan), scale)


def codes_e4m3(rows):
    """(values of the codes, scales float32)."""
    odd = ~np.isfinite(rows).all(axis=-1)
    rows = np.where(odd[..., None], 0.0, rows)
    scale = np.zeros(rows.shape[:-1])
    for at in np.ndindex(scale.shape):
        amax, e = np.abs(rows[at]).max(), -126
        while amax > 448.0 * 2.0 ** e:
            e += 1
        scale[at] = 2.0 ** e
    y = rows / scale[..., None]
    _, exponent = np.frexp(y)  # |y| = m 2^exponent, m in [0.5, 1)
    step = 2.0 ** (np.maximum(exponent - 1, -6) - 3)
    return np.rint(y / step) * step, np.where(odd, np.nan, scale).astype(np.float32)


def attention(q, keys, values, scale):
    """(out [S, H, D], lse [S, H], sum_j p_j |v_j|, largest scale sum_i |q_i k_ji|) of one token of each sequence; keys, values: lists of
    [Hk, n, D]."""
    S, H, D = q.shape
    out, bound, lse, spread = np.zeros_like(q), np.zeros_like(q), np.full((S, H), -np.inf), np.zeros((S, H))
    for s in range(S):
        G = H // keys[s].shape[0]
        for h in range(H):
            k, v = keys[s][h // G], values[s][h // G]
            if len(k) == 0:
                continue
            with np.errstate(all="ignore"):
                a = scale * (k @ q[s, h])
                top = a.max()
                if top == -np.inf:
                    continue
                p = np.exp(a - top)
                total = p.sum()
                lse[s, h] = top + np.log(total)
                p /= total
                out[s, h] = (p[:, None] * v).sum(axis=0)
                bound[s, h] = (p[:, None] * np.abs(v)).sum(axis=0)
                spread[s, h] = scale * (np.abs(k) @ np.abs(q[s, h])).max()
    return out, lse, bound, spread


def distribution(row, heat):
    """Softmax of a row at a temperature (not above 0: 1 at the first largest logit), or None."""
    top = row.max() if not np.isnan(row).any() else np.inf
    if not np.isfinite(top):
        return None
    if not heat > 0:
        p = np.zeros(len(row))
        p[int(np.argmax(row))] = 1.0
        return p
    p = np.exp((row - top) / min(max(heat, 2.0 ** -60), 2.0 ** 60))
    return p / p.sum()


def verify(logits, tokens, sees, u_accept, u_sample, max_path, heat=1.0, draft=None):
    """(path, next token) of one sequence: rows of logits [T, V], sees [T, T]."""
    T, V = logits.shape
    if T == 0:
        return [], -1
    parent = [-1] + [max((j for j in range(t) if sees[t, j]), default=-1) for t in range(1, T)]
    path = [0]
    while True:
        u = path[-1]
        p, step = distribution(logits[u], heat), None
        if p is not None:
            for t in range(u + 1, T):
                if parent[t] != u or not 0 <= tokens[t] < V:
                    continue
                x = tokens[t]
                if draft is not None and heat > 0:
                    q = distribution(draft[u], heat)
                    if q is None:
                        continue
                else:
                    q = np.zeros(V)
                    q[x] = 1.0
                if (u_accept[t] if heat > 0 else 0.0) * q[x] < p[x]:
                    step = t
                    break
                rest = np.maximum(p - q, 0.0)
                if rest.sum() > 0:
                    p = rest / rest.sum()
        if step is None:
            break
        if len(path) == max_path:
            return path, int(tokens[step])
        path.append(step)
    if p is None:
        return path, -1
    total = np.cumsum(p)
    past = np.flatnonzero(total > (u_sample if heat > 0 else 0.0) * total[-1])
    return path, int(past[0] if len(past) else np.flatnonzero(p > 0)[-1])
