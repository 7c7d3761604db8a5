"""Steps over a pool of pages that runs dry, on the GPU: what a slot without pages is told to
keep is not there, and attention is over the tokens that were appended and kept, alone."""
import numpy as np
import pytest
import torch

from oracle import paged as O
from paper_2410_18701_amd.paged import PagedCache
from tests.paged_schedule import Held, schedule
from tests.test_gpu_paged import close, f64, i32, rand

pytestmark = pytest.mark.gpu


def test_keep_more_than_there_is():
    """As many tokens stay as the last step brought, whatever keep says."""
    c = PagedCache(1, 2, 2, 1, 64, 8, 4, page=32)
    c.begin(i32([40, 129]))
    assert c.missing.tolist() == [0, 5]
    c.begin(i32([0, 0]), keep=i32([2 ** 31 - 1, 2 ** 31 - 1]))
    assert c.lens.tolist() == [40, 0]
    c.begin(i32([2 ** 31 - 1, 1]), keep=i32([2 ** 31 - 1, 2 ** 31 - 1]))
    assert c.lens.tolist() == [40, 0]
    assert c.missing.tolist()[0] > 0 and c.missing.tolist()[1] == 0 and c.slot_map.tolist()[0] == [-1]


@pytest.mark.parametrize("seed", range(3))
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
def test_tables(window, sinks, seed):
    batch, width, page, n_pages = 5, 5, 32, 9
    c = PagedCache(1, batch, 2, 1, 64, n_pages, 4, page=page, width=width, window=window, sinks=sinks)
    t, held, keep, lacked = O.Tables(batch, n_pages, 4, page, window, sinks), Held(batch), [0] * batch, 0
    for n_new, next_keep in schedule(seed, batch, 60, width, 3 * page):
        places = c.begin(i32(n_new), keep=i32(keep))
        want, missing = t.step(n_new, keep, width)
        held.end(keep)
        assert c.lens.tolist() == t.lens == [len(x) for x in held.tokens]
        assert c.table.tolist() == t.table and places.tolist() == want and c.missing.tolist() == missing
        held.begin(n_new, missing)
        keep, lacked = next_keep, lacked + sum(m > 0 for m in missing)
    assert lacked > 10


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 2)])
def test_attention(window, sinks, dtype):
    """Old tokens of other queries lie in the pages; keys and values of every appended token are
    known by its number."""
    batch, width, page, d = 4, 5, 32, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    c = PagedCache(1, batch, 4, 2, d, 5, 4, page=page, width=width, window=window, sinks=sinks, dtype=dtype)
    c.kv.fill_(float("nan"))
    held, keep, lacked, checked = Held(batch), [0] * batch, 0, 0
    ks, vs = [], []
    for n_new, next_keep in schedule(7, batch, 70, width, width, leave=0.03):
        c.begin(i32(n_new), keep=i32(keep))
        held.end(keep)
        missing = c.missing.tolist()
        held.begin(n_new, missing)
        assert c.lens.tolist() == [len(x) for x in held.tokens]
        q = rand(g, batch, width, 4, d, dtype=dtype)
        k, v = (rand(g, batch, width, 2, d, dtype=dtype) for _ in range(2))
        out = c.decode_attn(0, q, k, v, out=torch.full_like(q, 7.0))
        for b in range(batch):
            n = len(held.new[b])
            ks += [f64(k[b, i]) for i in range(n)]
            vs += [f64(v[b, i]) for i in range(n)]
            assert (out[b, n:] == 7.0).all()
            if n:
                at = held.tokens[b] + held.new[b]
                kk, vv = (np.stack([x[i] for i in at], 1) for x in (ks, vs))
                close(out[b, :n], O.attention(f64(q[b, :n]), kk, vv, len(held.tokens[b]), window, sinks),
                      np.abs(vv).max(), dtype)
                checked += 1
        keep, lacked = next_keep, lacked + sum(m > 0 for m in missing)
    assert lacked > 10 and checked > 100
