"""Sampling by its definition in float64, for the tests: numpy only."""
import numpy as np

CUT = 2.0 ** -45


def kept_weights(x, temperature, top_k, top_p, min_p):
    """Weights (float64, the largest 1) of the tokens that the settings keep of logits x, 0 for the others."""
    x = np.asarray(x, dtype=np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    V = x.size
    if (x == -np.inf).all():
        return np.zeros(V)
    order = np.lexsort((np.arange(V), -x))
    top = x[order[0]]
    w = np.zeros(V)
    if not temperature > 0:
        w[order[0]] = 1.0
        return w
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(x == top, 1.0, np.exp((x - top) / np.float64(np.float32(temperature))))
    w[(w < CUT) | (x == -np.inf)] = 0.0
    n = top_k if 0 < top_k < V else V
    run = np.cumsum(w[order])
    if np.float32(top_p) < 1:
        n = min(n, 1 + int(np.searchsorted(run[:n], np.float64(np.float32(top_p)) * run[n - 1], side="left")))
    keep = np.zeros(V, dtype=bool)
    keep[order[:max(n, 1)]] = True
    keep &= w >= min(np.float64(np.float32(min_p)), 1.0)
    return np.where(keep, w, 0.0)


def pick(w, u):
    """The first index whose running sum passes u of the whole; -1 of nothing."""
    if not (w > 0).any():
        return -1
    run = np.cumsum(w)
    return min(int(np.searchsorted(run, min(max(np.float64(u), 0.0), 1.0) * run[-1], side="right")),
               int(np.flatnonzero(w)[-1]))


def verify(x, draft, u_accept, u, settings, q=None):
    """One window: logits x [T, V]; returns (accepted, token)."""
    T, V = x.shape
    if T == 0:
        return 0, -1
    for t in range(T):
        w = kept_weights(x[t], *settings)
        p = w / w.sum() if w.sum() > 0 else w
        if t == T - 1:
            return T, pick(p, u)
        d = int(draft[t])
        inside = 0 <= d < V
        qx = (1.0 if q is None else float(q[t, d])) if inside else 1.0
        if inside and np.float64(u_accept[t]) * qx < p[d]:
            continue
        rest = p.copy()
        if q is not None:
            rest = np.maximum(p - q[t].astype(np.float64), 0.0)
        elif inside:
            rest[d] = 0.0
        return t + 1, pick(rest if rest.sum() > 0 else p, u)
