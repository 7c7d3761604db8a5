"""The 4-bit form of keys and values, and a batch whose cache holds it, in float64.

A block of 32 elements shares a power of two 2^e, the smallest (from 2^-125 to
2^125) that takes its largest magnitude to at most 7; an element is the nearest
of 0, 1/2, 1, 3/2, 2, 3, 4, 6 times 2^e (ties to the one with an even place in
that list), with its sign.  A block with an infinity or a NaN is NaN.
"""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def round_bf16(x):
    """float64 values rounded to the nearest bf16 (normal range)."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32).astype(np.float64)


def stored(x):
    """The values that x [..., multiple of 32] is held as."""
    x = np.asarray(x, np.float64)
    v = x.reshape(-1, 32)
    out = np.empty_like(v)
    ok = np.isfinite(v).all(1)
    out[~ok] = np.nan
    w = v[ok]
    a = np.abs(w).max(1)
    e = np.full(len(w), 125)
    for k in range(124, -126, -1):      # the smallest that will do, from above
        e = np.where(a <= 7 * 2.0 ** k, k, e)
    s = 2.0 ** e[:, None]
    t = np.abs(w) / s
    d = np.abs(t[..., None] - GRID)
    lo = d.argmin(-1)                   # of two equally near, the lower ...
    hi = np.minimum(lo + 1, 7)
    tie = (np.take_along_axis(d, hi[..., None], -1)[..., 0] == np.take_along_axis(d, lo[..., None], -1)[..., 0]) & (hi != lo)
    out[ok] = np.sign(w) * GRID[np.where(tie & (lo % 2 == 1), hi, lo)] * s   # ... unless that place is odd
    return out.reshape(x.shape)


def attend(q, k, v, scale):
    """One query row over its tokens: q [d], k, v [n][d] -> (output [d], sum p |v| / sum p)."""
    s = (k @ q) * scale
    p = np.exp(s - s.max())
    p /= p.sum()
    return p @ v, p @ np.abs(v)


class Batch4:
    """A batch's slots as lists of stored tokens: k[b], v[b] are [layers][heads][n][d], None when free."""

    def __init__(self, layers, batch, hq, hkv, d):
        self.layers, self.batch, self.hq, self.hkv, self.d = layers, batch, hq, hkv, d
        self.k, self.v = [None] * batch, [None] * batch

    def embed(self, slots, ks, vs):
        for b, k, v in zip(slots, ks, vs):
            assert self.k[b] is None
            self.k[b], self.v[b] = stored(k), stored(v)

    def evict(self, slots):
        for b in slots:
            assert self.k[b] is not None
            self.k[b] = self.v[b] = None

    def move(self, src, dst):
        for s, t in zip(src, dst):
            assert self.k[t] is None
            self.k[t], self.v[t], self.k[s], self.v[s] = self.k[s], self.v[s], None, None

    def step(self, q, k_new, v_new, prompts=None, scale=None):
        """q [layers][batch][T][hq][d], k_new, v_new [layers][batch][T][hkv][d]; prompts {slot: length}.
        Returns {(layer, slot, position): (out, bound) of [hq][d]}; the new tokens are stored."""
        prompts = prompts or {}
        scale = self.d ** -0.5 if scale is None else scale
        T, G, out = q.shape[2], self.hq // self.hkv, {}
        for b in range(self.batch):
            for l in range(self.layers):
                if b in prompts:
                    p = prompts[b]
                    for i in range(p):
                        at = T - p + i
                        got = [attend(q[l, b, at, h], k_new[l, b, T - p:at + 1, h // G], v_new[l, b, T - p:at + 1, h // G],
                                      scale) for h in range(self.hq)]
                        out[l, b, at] = tuple(np.array(x) for x in zip(*got))
                elif self.k[b] is not None:
                    got = []
                    for h in range(self.hq):
                        k = np.concatenate([self.k[b][l, h // G], k_new[l, b, :1, h // G]])
                        v = np.concatenate([self.v[b][l, h // G], v_new[l, b, :1, h // G]])
                        got.append(attend(q[l, b, 0, h], k, v, scale))
                    out[l, b, 0] = tuple(np.array(x) for x in zip(*got))
                else:
                    out[l, b, 0] = (np.zeros((self.hq, self.d)), np.zeros((self.hq, self.d)))
            new = (lambda x, t0, n: stored(x[:, b, t0:t0 + n].transpose(0, 2, 1, 3)))
            if b in prompts:
                p = prompts[b]
                self.k[b], self.v[b] = new(k_new, T - p, p), new(v_new, T - p, p)
            elif self.k[b] is not None:
                self.k[b] = np.concatenate([self.k[b], new(k_new, 0, 1)], 2)
                self.v[b] = np.concatenate([self.v[b], new(v_new, 0, 1)], 2)
        return out
