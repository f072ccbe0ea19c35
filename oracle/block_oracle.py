"""Plain fp64 forms of the operators of a hybrid stack's other layers: the two norms, the paged cache's append with its
rotation, and attention of single and of packed new tokens over it.  NumPy, one sequence, head and token at a time where
that is what the definition says; test infrastructure only, shares no code with the HIP path."""
import numpy as np


def _f64(t):
    if t is None:
        return None
    if hasattr(t, "detach"):
        t = t.detach().double().cpu().numpy() if t.is_floating_point() else t.detach().cpu().numpy()
    return np.asarray(t, dtype=np.float64) if np.asarray(t).dtype.kind == "f" else np.asarray(t)


def silu(z):
    with np.errstate(over="ignore"):
        return z / (1.0 + np.exp(-z))


def norm_gated(y, z, weight, eps, groups=1, norm_first=False):
    y, z, weight = _f64(y), _f64(z), _f64(weight)
    rows, width = y.shape
    out = np.empty_like(y)
    n = width // groups
    for g in range(groups):
        c = slice(g * n, (g + 1) * n)
        u = y[:, c] if norm_first else y[:, c] * silu(z[:, c])
        u = u / np.sqrt(np.mean(u * u, axis=1, keepdims=True) + eps) * weight[c]
        out[:, c] = u * silu(z[:, c]) if norm_first else u
    return out


def norm_residual(residual, x, weight, scale, eps):
    r = scale * _f64(x) + (0.0 if residual is None else _f64(residual))
    return r / np.sqrt(np.mean(r * r, axis=1, keepdims=True) + eps) * _f64(weight), r


def new_tokens(cu, lens, tokens, capacity):
    """(packed index, sequence, position) of every new token that is in a sequence; negative: it has no place in it."""
    def place(pos):
        return pos if pos < capacity else -1
    lens = np.maximum(_f64(lens), 0)
    if cu is None:
        return [(b, b, place(int(lens[b]) - 1)) for b in range(len(lens))]
    cu = [int(v) for v in _f64(cu)]
    out = []
    for b in range(len(lens)):
        lo, hi = max(cu[b], 0), min(cu[b + 1], tokens)
        out += [(t, b, place(int(lens[b]) - (hi - t))) for t in range(lo, hi)]
    return out


def rotate(v, pos, cos, sin, interleaved):
    """v (heads, headdim) turned by position pos."""
    half = cos.shape[1]
    out = v.copy()
    a, b = (np.arange(half) * 2, np.arange(half) * 2 + 1) if interleaved else (np.arange(half), np.arange(half) + half)
    out[:, a] = v[:, a] * cos[pos] - v[:, b] * sin[pos]
    out[:, b] = v[:, b] * cos[pos] + v[:, a] * sin[pos]
    return out


def append(q, k, v, k_cache, v_cache, table, lens, cu=None, rope=None, interleaved=False, q_out=None):
    """Returns (q_out, k_cache, v_cache); tokens without a place keep what ``q_out`` holds, or NaN."""
    q, k, v, k_cache, v_cache, table = (_f64(t) for t in (q, k, v, k_cache, v_cache, table))
    k_cache, v_cache = k_cache.copy(), v_cache.copy()
    npages, _, page, _ = k_cache.shape
    out = None if q is None else (np.full_like(q, np.nan) if q_out is None else _f64(q_out).copy())
    cos, sin = (None, None) if rope is None else (_f64(rope[0]), _f64(rope[1]))
    for t, b, pos in new_tokens(cu, lens, k.shape[0], table.shape[1] * page):
        if pos < 0:
            continue
        if out is not None:
            out[t] = q[t] if cos is None else rotate(q[t], pos, cos, sin, interleaved)
        where = table[b, pos // page]
        if 0 <= where < npages:
            k_cache[where, :, pos % page] = k[t] if cos is None else rotate(k[t], pos, cos, sin, interleaved)
            v_cache[where, :, pos % page] = v[t]
    return out, k_cache, v_cache


def attention(q, k_cache, v_cache, table, lens, cu=None, scale=None, window=0, y=None):
    """Rows of tokens outside every sequence keep what ``y`` holds, or NaN."""
    q, table, lens = _f64(q), _f64(table), _f64(lens)
    k_cache, v_cache = (t.detach().float().cpu().numpy() if hasattr(t, "detach") else t for t in (k_cache, v_cache))
    npages, nkv, page, D = k_cache.shape
    H = q.shape[1]
    scale = D ** -0.5 if scale is None else scale
    out = np.full(q.shape, np.nan) if y is None else _f64(y).copy()
    held = {}
    for t, b, pos in new_tokens(cu, lens, q.shape[0], table.shape[1] * page):
        if b not in held:
            n = int(np.clip(lens[b], 0, table.shape[1] * page))
            at = np.arange(n)
            where = table[b][at // page] if n else np.zeros(0, dtype=np.int64)
            there = (where >= 0) & (where < npages)
            at, where = at[there], where[there]
            held[b] = at, k_cache[where, :, at % page].astype(np.float64), v_cache[where, :, at % page].astype(np.float64)
        at, k, v = held[b]
        seen = at <= pos
        if window > 0:
            seen &= at > pos - window
        out[t] = 0.0
        if not seen.any():
            continue
        k, v = k[seen], v[seen]
        for h in range(H):
            s = k[:, h // (H // nkv)] @ q[t, h] * scale
            p = np.exp(s - s.max())
            out[t, h] = (p / p.sum()) @ v[:, h // (H // nkv)]
    return out
