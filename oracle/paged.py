"""A cache in pages in float64 and Python integers, from the definitions: the tables
of a step, and attention of new tokens over all tokens or a window and first ones."""
import numpy as np


class Tables:
    """Lengths, tables and the stack of free pages (the last element is its top)."""

    def __init__(self, batch, n_pages, max_pages, page, window=0, sinks=0, order=None):
        self.page, self.max_pages, self.window, self.sinks = page, max_pages, window, sinks
        self.stack = list(reversed(range(n_pages) if order is None else [int(x) for x in order]))
        self.table = [[-1] * max_pages for _ in range(batch)]
        self.lens = [0] * batch
        self.upto = [0] * batch      # blocks handed out (those given back behind the window among them)
        self.n_new = [0] * batch     # new tokens of the last step (0 where pages were lacking)

    def step(self, n_new, keep=None, width=1):
        """Returns (slot_map, missing)."""
        batch, P = len(self.lens), self.page
        back = []
        want = [0] * batch
        for b in range(batch):
            k = 0 if keep is None else int(keep[b])
            row = self.table[b]
            if k < 0:
                self.lens[b] = 0
                gone = range(self.upto[b])
                self.upto[b] = 0
                want[b] = -(-max(0, int(n_new[b])) // P)
            else:
                self.lens[b] += min(k, self.n_new[b])
                want[b] = -(-(self.lens[b] + max(0, int(n_new[b]))) // P)
                low = self.lens[b] - self.window + 1 if self.window else 0     # the first token the window shows
                gone = [j for j in range(self.upto[b])
                        if j >= want[b] or (j * P >= self.sinks and (j + 1) * P <= low)]
            for j in gone:
                if row[j] >= 0:
                    back.append(row[j])
                    row[j] = -1
            self.upto[b] = min(self.upto[b], want[b])
        self.stack += reversed(back)
        need, free = 0, len(self.stack)
        slot_map, missing = [], []
        for b in range(batch):
            more = max(0, want[b] - self.upto[b])
            short = 0
            if want[b] > self.max_pages:
                short = more
            else:
                need += more
                if more and need > free:
                    short = more
            missing.append(short)
            n = 0 if short else max(0, int(n_new[b]))
            if not short:
                for j in range(self.upto[b], want[b]):
                    self.table[b][j] = self.stack.pop()
                self.upto[b] = want[b]
            self.n_new[b] = n
            places = []
            for i in range(width):
                t = self.lens[b] + i
                places.append(self.table[b][t // P] * P + t % P if i < n else -1)
            slot_map.append(places)
        return slot_map, missing


def visible(p, n, window, sinks):
    """Which of n tokens a token at position p sees."""
    j = np.arange(n)
    return (j <= p) & ((j > p - window) | (j < sinks) if window else True)


def attention(q, k, v, length, window=0, sinks=0, scale=None):
    """q [t][hq][d] at positions length .., k, v [hkv][length + t][d] -> [t][hq][d]."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    t, hq, d = q.shape
    g = hq // k.shape[0]
    scale = d ** -0.5 if scale is None else scale
    out = np.zeros(q.shape)
    for i in range(t):
        see = visible(length + i, k.shape[1], window, sinks)
        for h in range(hq):
            s = scale * (k[h // g][see] @ q[i, h])
            w = np.exp(s - s.max())
            out[i, h] = (w / w.sum()) @ v[h // g][see]
    return out
