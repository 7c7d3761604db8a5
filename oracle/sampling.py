"""One token per row of logits in float64, from the definition: a sort, three
prefixes of the sorted order, inversion in order of index."""
import numpy as np


def sample(l, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """l [vocab] float64 (values of the stored logits) -> token (-1: none)."""
    l = np.where(np.isnan(l), -np.inf, np.asarray(l, np.float64))
    m = l.max()
    if m == -np.inf:
        return -1
    order = np.argsort(-l, kind="stable")           # ties: lowest index first
    if not temperature > 0 or top_k == 1 or min_p > 1:
        return int(order[0])
    if m == np.inf:
        w = (l == np.inf).astype(np.float64)
    else:
        with np.errstate(over="ignore", invalid="ignore"):
            w = np.where(l == -np.inf, 0.0, np.exp((l - m) / temperature))
    ws = w[order]
    n = len(l) if top_k <= 0 else min(top_k, len(l))
    if top_p < 1:
        c = np.cumsum(ws[:n])
        n = max(1, min(n, int(np.searchsorted(c, top_p * c[-1], side="left")) + 1))
    if min_p > 0:
        n = max(1, min(n, int((ws >= min_p).sum())))
    kept = np.zeros_like(w)
    kept[order[:n]] = ws[:n]
    c = np.cumsum(kept)
    u = min(max(u, 0.0), float(np.float32(1) - np.float32(2.0 ** -24))) if u == u else 0.0
    return int(np.searchsorted(c, u * c[-1], side="right"))
