"""The plain 64-bit form of attention with capped scores and windows, and the bound its outputs keep.

As in tests/serving.py, with what capping adds to a score's error.  cap * tanh(s / cap) moves no more than s does, so an error of s stays
what it is.  On the bf16 matrix cores a score is 2 cap * u + const, u = -1 / (1 + e), e = exp2(x): x is rounded once (2^-24 of it), e is
right to 2^-23, the sum and the reciprocal to 2^-24 each; u moves by u (1 + u) <= 1/4 of e's relative error.  That is
2 cap * (2^-25 + 2^-24 + 2^-24) plus |s| * 2^-24: within cap * 2^-22 + |s| * 2^-23.  In fp32 kernels tanh is right to 8 half steps."""
import numpy as np

from serving import U32


def visible_rows(n, context, mask_rows=None, window=0, rel=None):
    """[n, context + n] bool."""
    among = np.tril(np.ones((n, n), bool))
    i = np.arange(n)
    if mask_rows is not None:
        among &= ((mask_rows[:, i // 64] >> (i % 64).astype(np.uint64)) & np.uint64(1)).astype(bool)
    see = np.concatenate([np.ones((n, context), bool), among], axis=1)
    if window:
        new = context + (i if rel is None else np.asarray(rel, np.int64))
        see &= new[:, None] - np.concatenate([np.arange(context), new])[None, :] < window
    return see


def scored_plain(q, k, v, visible, scale, cap, weight_half, out_half, exact):
    """One sequence, float64 in: (out, bound).  Keys that a row does not see are left out, whatever they hold."""
    n, Hq, d = q.shape
    G = Hq // k.shape[1]
    out, bound = np.zeros((n, Hq, d)), np.zeros((n, Hq, d))
    clean = np.where(np.isfinite(k), k, 0.0), np.where(np.isfinite(v), v, 0.0)
    whole = np.isfinite(k).all() and np.isfinite(v).all()
    for h in range(Hq):
        kk, vv = clean[0][:, h // G], clean[1][:, h // G]
        s, t = q[:, h] @ kk.T * scale, np.abs(q[:, h]) @ np.abs(kk).T * scale
        e = (d + 2) * U32 * np.where(visible, t, 0.0).max(1, keepdims=True)
        if cap:
            e = e + (8 * U32 * np.where(visible, np.abs(s), 0.0).max(1, keepdims=True) if exact else
                     cap * 2.0 ** -22 + 2 * U32 * np.where(visible, np.abs(s), 0.0).max(1, keepdims=True))
            s = cap * np.tanh(s / cap)
        s = np.where(visible, s, -np.inf)
        top = s.max(1, keepdims=True)
        top = np.where(np.isfinite(top), top, 0.0)
        w = np.exp(s - top)
        l = w.sum(1, keepdims=True)
        l = np.where(l > 0, l, 1.0)
        o, a = w @ vv / l, w @ np.abs(vv) / l
        spread = np.where(visible, np.abs(s - top) + np.abs(top), 0.0).max(1, keepdims=True)
        if cap and not exact:
            spread = np.maximum(spread, cap)                  # (what is scaled and subtracted is 2 cap u, up to 2 cap)
        e = e + 4 * U32 * spread
        out[:, h] = o
        keys = visible.sum(1, keepdims=True)
        bound[:, h] = a * (2 * e + (2 * keys + 32) * U32 + weight_half) + out_half * np.abs(o) + 1e-30
    if not whole:                                             # rows that see something odd: not compared
        odd = ~(np.isfinite(k).all((1, 2)) & np.isfinite(v).all((1, 2)))
        out[(visible & odd[None, :]).any(1)] = np.nan
    return out, bound
