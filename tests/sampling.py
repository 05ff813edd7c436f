"""The plain 64-bit form of dyspec_sample and dyspec_filter_logits, row by row on the host.

Tokens and counts have to be equal.  The kernel's weights are off by at most 2^-46 of the row's largest and 4e-14 of themselves, so a
draw or a border of top-p could differ where u * total or p * total lies closer to a sum than V * 2^-46: nearest() says how near the
nearest one was (relative to the largest weight), and inputs that come nearer than that are not compared (none of the seeded ones do;
equal weights of 1, whose sums are exact in both, are compared whatever lies there)."""
import numpy as np

TOP_U = np.float64(1.0) - 2.0 ** -24


def plain_row(x, uniform, temperature, top_k=0, top_p=1.0, min_p=0.0):
    """x: one row, float64.  Returns (kept [V] bool, token, prob, nearest)."""
    V = len(x)
    kept = np.zeros(V, bool)
    if np.isnan(x).any() or (x == np.inf).any() or not np.isfinite(x).any():
        return kept, -1, 0.0, np.inf
    order = np.argsort(-x, kind="stable")
    near = np.inf
    if temperature == 0:
        kept[order[0]] = True
        return kept, int(order[0]), 1.0, near
    best = order[:top_k] if top_k else order
    with np.errstate(over="ignore", under="ignore"):
        w = np.exp((x[best] - x[best[0]]) / np.float64(np.float32(temperature)))
    n = len(best)
    if top_p < 1:
        sums, target = np.cumsum(w), np.float64(np.float32(top_p)) * w.sum()
        n = 1 + int(np.searchsorted(sums[:-1], target, side="left"))
        near = min(near, np.abs(sums - target).min())
    n = min(n, int(np.count_nonzero(w >= np.float64(np.float32(min_p)))))
    kept[best[:n]] = True
    index = np.sort(best[:n])
    with np.errstate(over="ignore", under="ignore"):
        w = np.exp((x[index] - x[best[0]]) / np.float64(np.float32(temperature)))
    u = 0.0 if np.isnan(uniform) else min(max(np.float64(uniform), 0.0), TOP_U)
    sums = np.cumsum(w)
    target = u * sums[-1]
    near = min(near, np.abs(sums - target).min())
    at = int(np.searchsorted(sums, target, side="right"))
    return kept, int(index[at]), w[at] / sums[-1], near


def plain_rows(logits, rows, uniform, temperature, top_k, top_p, min_p):
    """Whole tables: (filtered float64, tokens, probs, counts, rows that can be compared)."""
    x = logits.double().cpu().numpy()
    of = np.repeat(np.arange(len(rows)), rows)
    out, tokens, probs, counts, fine = np.full(x.shape, -np.inf), [], [], [], []
    for r, s in enumerate(of):
        kept, token, prob, near = plain_row(x[r], uniform[r], temperature[s], top_k[s], top_p[s], min_p[s])
        out[r, kept] = x[r, kept]
        tokens.append(token), probs.append(prob), counts.append(int(kept.sum()))
        top = x[r, kept].max() if kept.any() else 0.0
        fine.append(near > x.shape[1] * 2.0 ** -46 or bool((x[r, kept] == top).all()))
    return out, np.asarray(tokens), np.asarray(probs), np.asarray(counts), np.asarray(fine)
