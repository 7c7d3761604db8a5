"""Steps over a pool of pages that runs dry: what each step brings and how many of its tokens
its end says stay, whether or not the slot's pages were there (as a verification's n_out does,
which knows nothing of pages); and what the slots then hold."""
import numpy as np


def schedule(seed, batch, steps, width, most, leave=0.08):
    """(n_new, keep) of every step; the keep of step i is passed to step i + 1.  Some steps bring up to
    `most` tokens to a slot, the others up to `width`."""
    r = np.random.default_rng(seed)
    for _ in range(steps):
        n_new = [int(r.integers(0, (width if r.random() < 0.8 else most) + 1)) for _ in range(batch)]
        how = r.random(batch)
        yield n_new, [-1 if h < leave else 2 ** 31 - 1 if h > 0.96 else n + 3 if h > 0.88 else int(r.integers(0, n + 1))
                      for h, n in zip(how, n_new)]


class Held:
    """Each slot's tokens by number, as lists: a step's are appended if the slot lacks no pages."""

    def __init__(self, batch):
        self.tokens, self.new, self.next = [[] for _ in range(batch)], [[] for _ in range(batch)], 0

    def end(self, keep):
        for b, k in enumerate(keep):
            self.tokens[b] = [] if k < 0 else self.tokens[b] + self.new[b][:k]
            self.new[b] = []

    def begin(self, n_new, missing):
        for b, (n, m) in enumerate(zip(n_new, missing)):
            if m == 0:
                self.new[b] = list(range(self.next, self.next + n))
                self.next += n
