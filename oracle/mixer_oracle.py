"""fp64 oracle of the selective scan, of its convolution over packed prompts, and of the append with normed heads.  NumPy, a
token at a time where that is what the definition says; test infrastructure only, shares no code with the HIP path.  With
``magnitude`` a function returns the sums of the absolute values of its terms, which rounding errors are relative to."""
import numpy as np

from oracle import block_oracle, ssd_oracle
from oracle.block_oracle import _f64, silu


def sequences(cu, tokens):
    """(sequence, first token, last + 1), boundaries cut to the tokens."""
    cu = [min(max(int(v), 0), tokens) for v in _f64(cu)]
    return [(q, cu[q], max(cu[q], cu[q + 1])) for q in range(len(cu) - 1)]


def conv1d_varlen(u, weight, bias, cu, conv_state=None, activation="silu", z=None):
    """Returns (z, new cache); tokens of no sequence keep what ``z`` holds, or NaN."""
    u = _f64(u)
    tokens, C = u.shape
    k = _f64(weight).shape[1]
    out = np.full(u.shape, np.nan) if z is None else _f64(z).copy()
    spans = sequences(cu, tokens)
    caches = np.zeros((len(spans), C, k - 1)) if conv_state is None else _f64(conv_state).copy()
    for q, lo, hi in spans:
        if hi > lo:
            out[lo:hi], caches[q] = (v[0] for v in ssd_oracle.conv1d_prefill(u[None, lo:hi], weight, bias, caches[q:q + 1], activation))
    return out, caches


def selective_scan(x, d, A, B, C, D, cu, z=None, h0=None, y=None, magnitude=False):
    """``d``: the final step sizes.  Returns (y, final states); tokens of no sequence keep what ``y`` holds, or NaN."""
    x, d, A, B, C = (_f64(t) for t in (x, d, A, B, C))
    D = np.zeros(x.shape[1]) if D is None else _f64(D)
    spans = sequences(cu, x.shape[0])
    final = np.zeros((len(spans),) + A.shape) if h0 is None else _f64(h0).copy()
    gate = np.ones_like(x) if z is None else silu(_f64(z))
    if magnitude:
        x, B, C, D, final, gate = (np.abs(t) for t in (x, B, C, D, final, gate))
    out = np.full(x.shape, np.nan) if y is None else _f64(y).copy()
    for q, lo, hi in spans:
        h = final[q]
        for t in range(lo, hi):
            h = np.exp(d[t][:, None] * A) * h + (d[t] * x[t])[:, None] * B[t]
            out[t] = (h @ C[t] + D * x[t]) * gate[t]
        final[q] = h
    return out, final


def normed_heads(v, weight, eps):
    """v (tokens, heads, headdim)."""
    v = _f64(v)
    return v / np.sqrt(np.mean(v * v, axis=2, keepdims=True) + eps) * _f64(weight)


def append_norm(q, k, v, q_weight, k_weight, k_cache, v_cache, table, lens, cu=None, rope=None, interleaved=False, eps=1e-5, q_out=None,
                magnitude=False):
    """Returns (q_out, k_cache, v_cache) as ``block_oracle.append``."""
    q = None if q is None else normed_heads(q, q_weight, eps)
    k = normed_heads(k, k_weight, eps)
    if magnitude:  # |a cos| + |b sin| and so on
        q, k = (None if t is None else np.abs(t) for t in (q, k))
        rope = None if rope is None else (np.abs(_f64(rope[0])), np.abs(_f64(rope[1])))
        if rope is not None:
            first = block_oracle.append(q, k, v, k_cache, v_cache, table, lens, cu, rope, interleaved, q_out)
            second = block_oracle.append(q, k, v, k_cache, v_cache, table, lens, cu, (rope[0], -rope[1]), interleaved, q_out)
            return tuple(None if a is None else np.fmax(np.abs(a), np.abs(b)) for a, b in zip(first, second))
    return block_oracle.append(q, k, v, k_cache, v_cache, table, lens, cu, rope, interleaved, q_out)
