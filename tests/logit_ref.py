"""Plain 64-bit forms of the operators on rows of logits, for their tests."""
import numpy as np


def order_of(z):
    """Indices by falling value, ties by rising index (-0 equals +0)."""
    return np.argsort(-z, kind="stable")


def softmax_lse(x):
    m = x.max()
    if not np.isfinite(m):
        return m
    return m + np.log(np.exp(x - m).sum())


def kept_tokens(z, T, k, p, min_p):
    """(kept indices in vocabulary order, their shares, distance of the nearest
    undecided comparison as a relative weight)."""
    V = len(z)
    e = np.exp((z - z.max()) / T)
    order = order_of(z)
    keep = np.zeros(V, bool)
    keep[order[:k] if 0 < k < V else order] = True
    cut = min(min_p, 1.0)
    margin = np.inf
    if cut > 0:
        live = e[e > 0]
        rel = np.abs(live / cut - 1.0)
        if cut < 1.0:
            margin = min(margin, rel.min())
        keep &= (e >= cut) | (e == 1.0)
    if p < 1.0:
        run = order[keep[order]]
        w = e[run]
        cum = np.cumsum(w)
        target = max(p, 0.0) * cum[-1]
        n = int(np.searchsorted(cum, target, side="left")) + 1
        n = min(n, len(run))
        margin = min(margin, np.abs(cum - target).min() / cum[-1])
        keep[:] = False
        keep[run[:n]] = True
    ix = np.flatnonzero(keep)
    w = e[ix]
    return ix, w / w.sum(), margin


def distill(z, tv, ti, tlse, tau, w):
    """(loss, (lse, lse_rest), gradient) of one row."""
    V = len(z)
    x = z / tau
    given = (ti >= 0) & (ti < V)
    if w == 0 or not given.any():
        return 0.0, (0.0, 0.0), np.zeros(V)
    t = tv[given] / tau
    at = ti[given]
    norm = softmax_lse(t) if tlse is None else tlse
    lq = t - norm
    q = np.exp(lq)
    rest = 0.0 if tlse is None else max(0.0, 1.0 - q.sum())
    lse = softmax_lse(x)
    outside = np.ones(V, bool)
    outside[at] = False
    lse_rest = softmax_lse(x[outside]) if outside.any() else -np.inf
    kl = (q * (lq - (x[at] - lse))).sum()
    if rest > 0:
        kl += rest * (np.log(rest) - (lse_rest - lse))
    whole = q.sum() + rest
    p = np.exp(x - lse)
    share = rest * np.exp(lse - lse_rest) if rest > 0 and lse_rest > -np.inf else 0.0
    g = p * np.where(outside, whole - share, whole)
    np.subtract.at(g, at, q)
    return w * tau * tau * kl, (lse, lse_rest), w * tau * g
