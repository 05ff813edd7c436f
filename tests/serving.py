"""Plain 64-bit forms of the paged cache's calls and of prompt attention, inputs for them, and the bounds their outputs keep.

The attention bound, element by element, from the arithmetic of the kernels (u = 2^-24, half a step of fp32):
  scores are fp32 sums of d exact or once-rounded products: off by at most (d + 2) u sum|q k|, as exponents that times the scale,
  plus 4 u |exponent| for the scaling, the maximum's subtraction and the exponential itself; a weight is off by that, relative;
  sums of n weights (and of weights times values) are off by n u, relative to the sum of their sizes; merging parts adds a few u.
  So out = sum w v / sum w is within A (2 e + (2 n + 32) u) of the exact value, A = sum w |v| / sum w, e the scores' error.
  bf16 on the matrix cores rounds a weight once (half a step: 2^-8 of it) and the output once (2^-8 of it).
"""
import math

import numpy as np
import torch

U32 = 2.0 ** -24
HALF = {torch.float32: U32, torch.bfloat16: 2.0 ** -8}


def page_table(lengths, page, seed, spare=3, extra_columns=2):
    """Pages in no order: (table [n_seq, most + extra_columns] int32, pages of the pool).  Entries that are not reached: -1."""
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in lengths]
    pool = sum(need) + spare
    order = rng.permutation(pool).astype(np.int32)
    table = np.full((len(need), max(need + [0]) + extra_columns), -1, np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return table, pool


def random_mask(sizes, seed, self_bit=True):
    """Ancestor masks of random trees [sum, words] uint64 and their depths."""
    rng = np.random.default_rng(seed)
    words = max(1, -(-max(sizes) // 64))
    rows, depths = [], []
    for n in sizes:
        m, depth = np.zeros((n, words), np.uint64), np.zeros(n, np.int32)
        for j in range(n):
            if j:
                up = int(rng.integers(max(0, j - 40), j))
                m[j], depth[j] = m[up], depth[up] + 1
            m[j, j // 64] |= np.uint64(1) << np.uint64(j % 64)
        rows.append(m)
        depths.append(depth)
    return np.concatenate(rows), np.concatenate(depths)


def visible_rows(n, context, mask_rows=None):
    """[n, context + n] bool."""
    among = np.tril(np.ones((n, n), bool))
    if mask_rows is not None:
        i = np.arange(n)
        among &= ((mask_rows[:, i // 64] >> (i % 64).astype(np.uint64)) & np.uint64(1)).astype(bool)
    return np.concatenate([np.ones((n, context), bool), among], axis=1)


def attend_plain(q, k, v, visible, scale, weight_half=0.0, out_half=U32):
    """One sequence, numpy in: q [n, Hq, d], k, v [keys, Hkv, d].  Returns (out, bound), float64.  Keys that a row does not see are
    left out of its sums, whatever they hold."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n, Hq, d = q.shape
    G = Hq // k.shape[1]
    out, bound = np.zeros((n, Hq, d)), np.zeros((n, Hq, d))
    clean = np.isfinite(k).all() and np.isfinite(v).all()
    for h in range(Hq):
        kk, vv = k[:, h // G], v[:, h // G]
        if clean:
            s, t = q[:, h] @ kk.T * scale, np.abs(q[:, h]) @ np.abs(kk).T * scale
            s = np.where(visible, s, -np.inf)
            top = s.max(1, keepdims=True)
            top = np.where(np.isfinite(top), top, 0.0)
            w = np.exp(s - top)
            l = w.sum(1, keepdims=True)
            some = l > 0
            l = np.where(some, l, 1.0)
            o, a = w @ vv / l, w @ np.abs(vv) / l
            spread = np.where(visible, np.abs(s - top) + np.abs(top), 0.0).max(1, keepdims=True)
            e = (d + 2) * U32 * np.where(visible, t, 0.0).max(1, keepdims=True) + 4 * U32 * spread
        else:
            o, a, e = np.zeros((n, d)), np.zeros((n, d)), np.zeros((n, 1))
            for j in range(n):
                see = np.nonzero(visible[j])[0]
                if len(see) == 0:
                    continue
                s = kk[see] @ q[j, h] * scale
                w = np.exp(s - s.max())
                o[j], a[j] = w @ vv[see] / w.sum(), w @ np.abs(vv[see]) / w.sum()
                e[j] = (d + 2) * U32 * (np.abs(kk[see]) @ np.abs(q[j, h])).max() * scale + 4 * U32 * 2 * np.abs(s).max()
        out[:, h] = o
        keys = visible.sum(1, keepdims=True)
        bound[:, h] = a * (2 * e + (2 * keys + 32) * U32 + weight_half) + out_half * np.abs(o) + 1e-30
    return out, bound


def rounds_weights(dtype, head_dim):
    return HALF[torch.bfloat16] if dtype is torch.bfloat16 and head_dim in (64, 128) else 0.0


class Paged:
    """A batch over a paged cache: random contexts in the pool, new tokens' rows in it as well (as if appended)."""

    def __init__(self, new, context, Hq, Hkv, d, dtype, page, seed, mask=None, layers=0, both_in_one=False, device="cuda"):
        import paper_2410_11744_amd as dy
        g = torch.Generator().manual_seed(seed)
        mk = lambda *sh: torch.randn(sh, generator=g, dtype=torch.float32).to(dtype)
        self.new, self.context, self.Hq, self.Hkv, self.d, self.dtype, self.page = list(new), list(context), Hq, Hkv, d, dtype, page
        self.total = sum(new)
        self.row0 = np.concatenate([[0], np.cumsum(new)])
        self.table, pool = page_table([c + n for c, n in zip(context, new)], page, seed)
        self.q = mk(self.total, Hq, d)
        lead = (layers,) if layers else ()
        if both_in_one:
            kv = mk(*lead, pool, 2, page, Hkv, d)
            self.kv_dev = kv.to(device)
            self.k, self.v = kv.select(-4, 0).clone(), kv.select(-4, 1).clone()
            k_dev, v_dev = self.kv_dev.select(-4, 0), self.kv_dev.select(-4, 1)
        else:
            self.k, self.v = mk(*lead, pool, page, Hkv, d), mk(*lead, pool, page, Hkv, d)
            k_dev, v_dev = self.k.to(device), self.v.to(device)
        self.mask = mask
        self.mask_dev = None if mask is None else torch.from_numpy(mask.view(np.int64)).to(device)
        self.batch = dy.Batch.from_sizes(new, context)
        self.cache = dy.PagedCache(k_dev, v_dev, torch.from_numpy(self.table).to(device))
        self.q_dev = self.q.to(device)
        self.scale = 1.0 / math.sqrt(d)

    def place(self, s, position):
        return int(self.table[s, position // self.page]), position % self.page

    def rows(self, s):
        """(k, v) of sequence s, context and new tokens, as float64."""
        n = self.context[s] + self.new[s]
        pages = torch.from_numpy(self.table[s, :-(-n // self.page)].astype(np.int64))
        return tuple(t[pages].flatten(0, 1)[:n].double().numpy() for t in (self.k, self.v))

    def check(self, out, only=None):
        """out against the plain form, within its bound; returns the largest share of the bound used."""
        got = out.double().cpu().numpy()
        wh, oh, worst = rounds_weights(self.dtype, self.d), HALF[self.dtype], 0.0
        for s, n in enumerate(self.new):
            if n == 0 or (only is not None and s not in only):
                continue
            a = self.row0[s]
            k, v = self.rows(s)
            words = None if self.mask is None else self.mask[a:a + n]
            want, bound = attend_plain(self.q[a:a + n].double().numpy(), k, v, visible_rows(n, self.context[s], words), self.scale, wh, oh)
            worst = max(worst, compare(got[a:a + n], want, bound, f"sequence {s}"))
        return worst


def compare(got, want, bound, what):
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)), f"{what}: finite where the plain form is not, or the other way round"
    share = np.abs(got[fine] - want[fine]) / bound[fine]
    assert share.size == 0 or share.max() <= 1.0, f"{what}: off by {share.max():.2f} times the bound at {np.unravel_index(np.argmax(np.where(fine, np.abs(got - want) / bound, 0)), got.shape)}"
    return float(share.max()) if share.size else 0.0


def rotate_plain(x, position, inv_freq, interleaved):
    """x [n, heads, d] rotated, float64, and the bound of an fp32 kernel that rounds to the type of `x` once: cos and sin within
    4 half steps (the fraction of a turn, its sine), two products and a sum."""
    y = x.double().numpy().copy()
    half = len(inv_freq)
    a = np.asarray(position, np.float64)[:, None, None] * np.asarray(inv_freq, np.float64)
    i, j = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    u, w = y[..., i].copy(), y[..., j].copy()
    y[..., i], y[..., j] = u * np.cos(a) - w * np.sin(a), u * np.sin(a) + w * np.cos(a)
    bound = np.zeros_like(y)
    size = np.abs(u) + np.abs(w)
    bound[..., i] = bound[..., j] = 8 * U32 * size + 1e-13 * np.abs(a) * size
    return y, bound + HALF[x.dtype] * np.abs(y) + (1e-30 if half else 0.0)
