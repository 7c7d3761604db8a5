"""Verification of drafted tokens in float64, from the definition."""
import numpy as np


def kept(l, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The distribution that sampling draws from, [vocab] (all 0: nothing can be drawn)."""
    l = np.where(np.isnan(l), -np.inf, np.asarray(l, np.float64))
    m = l.max()
    out = np.zeros(len(l))
    if m == -np.inf:
        return out
    order = np.argsort(-l, kind="stable")
    if not temperature > 0 or top_k == 1 or min_p > 1:
        out[order[0]] = 1.0
        return out
    if m == np.inf:
        w = (l == np.inf).astype(np.float64)
    else:
        w = np.where(l == -np.inf, 0.0, np.exp((l - m) / temperature))
    ws = w[order]
    n = len(l) if top_k <= 0 else min(top_k, len(l))
    if top_p < 1:
        c = np.cumsum(ws[:n])
        n = max(1, min(n, int(np.searchsorted(c, top_p * c[-1], side="left")) + 1))
    if min_p > 0:
        n = max(1, min(n, int((ws >= min_p).sum())))
    out[order[:n]] = ws[:n]
    return out / out.sum()


def _u(u):
    return min(max(u, 0.0), float(np.float32(1) - np.float32(2.0 ** -24))) if u == u else 0.0


def verify(target, draft, drafted, n_draft, u_accept, u_token, **params):
    """target [width][vocab], draft [width - 1][vocab] or None -> (tokens, n_out) of one slot."""
    width, vocab = target.shape
    if n_draft < 0:
        return [-1] * width, 0
    tokens = []
    r = None
    for i in range(min(n_draft, width - 1)):
        p, x = kept(target[i], **params), int(drafted[i])
        inside = 0 <= x < vocab
        if draft is None:
            q = np.zeros(vocab)
            q[x if inside else 0] = 1.0 if inside else 0.0
        else:
            q = kept(draft[i], **params)
        if inside and (draft is None or q.any()) and _u(u_accept[i]) * q[x] < p[x]:
            tokens.append(x)
            continue
        r = np.maximum(0.0, p - q)
        if r.sum() == 0:
            r = p
        break
    if r is None:
        r = kept(target[len(tokens)], **params)
    c = np.cumsum(r)
    token = int(np.searchsorted(c, _u(u_token) * c[-1], side="right")) if c[-1] > 0 else -1
    tokens.append(token)
    return tokens + [-1] * (width - len(tokens)), len(tokens)
