"""The cache in pages on the GPU: tables against the oracle's, copies bit for
bit, attention against 64-bit arithmetic.

Tolerances.  Keys, values and queries are what the oracle gets, products of two
bf16 numbers are exact in fp32.  A score is a sum of d <= 128 products, off by at
most d 2^-24 times the sum of their magnitudes: of normal numbers about 0.64 d,
times scale d^-1/2, below 128 * 2^-24 * 0.8 * 128 / 11.3 = 2^-13.9 for d = 128
(8 % above the mean sum of magnitudes: over 3 of its deviations; keys here are at
most 1.5 of a normal number's).  A weight's relative error is that, 2^-17 for its
16 bits and some 2^-22 for its exponential; a mean of values with weights off by at
most e each is off by at most 2 e max|v|.  With 1.5 2^-13.9 + 2^-17 < 2^-13.2: fp32
within 2^-12 max|v|, and bf16 by half a step of its result, 2^-8 of it, more."""
import numpy as np
import pytest
import torch

from oracle import paged as O
from paper_2410_18701_amd.paged import PagedCache

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def rand(g, *shape, dtype="bf16", gain=1.0):
    return (gain * torch.randn(shape, generator=g, device="cuda")).to(DT[dtype])


def f64(t):
    return t.detach().double().cpu().numpy()


def close(out, want, vmax, dtype):
    err = np.abs(f64(out) - want)
    tol = 2.0 ** -12 * vmax + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0.0)
    assert np.isfinite(f64(out)).all() and (err <= tol).all(), float((err / tol).max())


class Twin:
    """A PagedCache beside each query's keys and values as rows."""

    def __init__(self, seed=0, layers=1, batch=3, hq=4, hkv=2, d=64, page=32, width=1, window=0, sinks=0, dtype="bf16",
                 max_pages=None, n_pages=None, lens=(), poison=False):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        need = sum(-(-(n + 2 * width + 2) // page) for n in lens) + batch
        self.max_pages = max_pages or -(-(max(lens, default=1) + 4 * width + 4) // page)
        order = torch.randperm(n_pages or need, generator=torch.Generator().manual_seed(seed)).int().cuda()
        self.c = PagedCache(layers, batch, hq, hkv, d, n_pages or need, self.max_pages, page=page, width=width,
                            window=window, sinks=sinks, dtype=dtype, order=order)
        if poison:
            self.c.kv.fill_(float("nan"))
            if self.c._ws is not None:
                self.c._ws.fill_(0xFF)
        self.layers, self.hq, self.hkv, self.d, self.dtype, self.width = layers, hq, hkv, d, dtype, width
        self.window, self.sinks, self.batch = window, sinks, batch
        self.ks = [rand(self.g, layers, hkv, 0, d, dtype=dtype) for _ in range(batch)]
        self.vs = [x.clone() for x in self.ks]
        lens = list(lens) + [0] * (batch - len(lens))
        self.lens = lens
        self.c.begin(i32(lens))
        live = [b for b in range(batch) if lens[b]]
        for b in live:
            self.ks[b] = rand(self.g, layers, hkv, lens[b], d, dtype=dtype, gain=1.5)
            self.vs[b] = rand(self.g, layers, hkv, lens[b], d, dtype=dtype)
        self.c.embed(live, [lens[b] for b in live], [self.ks[b] for b in live], [self.vs[b] for b in live])

    def step(self, n_new, keep, check=True):
        """One step over all layers; keep: how many of the last step's tokens stay."""
        self.c.begin(i32(n_new), keep=i32(keep))
        q = rand(self.g, self.layers, self.batch, self.width, self.hq, self.d, dtype=self.dtype)
        k, v = (rand(self.g, self.layers, self.batch, self.width, self.hkv, self.d, dtype=self.dtype) for _ in range(2))
        for b in range(self.batch):
            n = max(0, keep[b] + (self.lens[b] if self.started else 0))
            self.ks[b], self.vs[b] = self.ks[b][:, :, :n], self.vs[b][:, :, :n]
            self.lens[b] = self.ks[b].shape[2]
            t = min(n_new[b], self.width)
            self.ks[b] = torch.cat([self.ks[b], k[:, b, :t].transpose(1, 2)], 2)
            self.vs[b] = torch.cat([self.vs[b], v[:, b, :t].transpose(1, 2)], 2)
        outs = []
        for l in range(self.layers):
            out = torch.full_like(q[l], 7.0)
            self.c.decode_attn(l, q[l], k[l], v[l], out=out)
            outs.append(out)
            if check:
                self.check(l, q[l], out, n_new)
        self.last = (q, k, v)
        return outs

    started = False      # the prompts' own step is the first

    def first(self, n_new):
        out = self.step(n_new, list(self.lens))
        self.started = True
        return out

    def check(self, layer, q, out, n_new):
        for b in range(self.batch):
            t = n_new[b]
            assert (out[b, t:] == 7.0).all()               # rows behind the last are left as they were
            if t == 0:
                continue
            k, v = f64(self.ks[b][layer]), f64(self.vs[b][layer])
            want = O.attention(f64(q[b, :t]), k, v, self.lens[b], self.window, self.sinks)
            close(out[b, :t], want, np.abs(v).max(), self.dtype)


# ------------------------------------------------------------------ tables --
@pytest.mark.parametrize("batch,page,window,sinks,seed", [
    (1, 32, 0, 0, 0), (5, 64, 0, 0, 1), (64, 32, 0, 0, 2), (512, 32, 0, 0, 3), (7, 256, 0, 0, 4), (5, 32, 40, 3, 5),
    (33, 64, 1, 0, 6), (20, 32, 200, 70, 7), (9, 128, 300, 128, 8)])
def test_tables(batch, page, window, sinks, seed):
    """Queries come, grow, are cut back and leave, in a pool that is too small at times."""
    r = np.random.default_rng(seed)
    max_pages, width = 12, 5
    n_pages = max(3, batch * 5)
    order = r.permutation(n_pages)
    c = PagedCache(1, batch, 2, 1, 64, n_pages, max_pages, page=page, width=width, window=window, sinks=sinks,
                   order=i32(order))
    t = O.Tables(batch, n_pages, max_pages, page, window, sinks, order)
    keep = None
    for step in range(40):
        n_new = [int(r.choice([0, 1, 1, 2, 3, 5, 5, r.integers(0, 14 * page)])) if r.random() < 0.9 else -3
                 for _ in range(batch)]
        places = c.begin(i32(n_new), keep=None if keep is None else i32(keep))
        want, missing = t.step(n_new, keep, width)
        assert c.lens.tolist() == t.lens, step
        assert c.table.tolist() == t.table, step
        assert places.tolist() == want, step
        assert c.missing.tolist() == missing, step
        keep = [int(r.choice([0, max(0, n), max(0, n // 2), max(0, n), -1])) for n in n_new]
    c.begin(i32([0] * batch), keep=i32([-1] * batch))
    assert c._state[0].item() == n_pages and (c.table == -1).all() and (c.lens == 0).all()


def test_tables_keep_more_than_there_is():
    """Tokens without a page are not kept, whatever keep says; lens stays within the table."""
    c = PagedCache(1, 2, 2, 1, 64, 8, 4, page=32)
    c.begin(i32([40, 129]))
    assert c.missing.tolist() == [0, 5]
    c.begin(i32([0, 0]), keep=i32([2 ** 31 - 1, 2 ** 31 - 1]))
    assert c.lens.tolist() == [64, 0]
    c.begin(i32([2 ** 31 - 1, 1]))
    assert c.missing.tolist()[0] > 0 and c.missing.tolist()[1] == 0 and c.slot_map.tolist()[0] == [-1]


# ------------------------------------------------------------------ copies --
@pytest.mark.parametrize("dtype,d,page", [("bf16", 128, 64), ("bf16", 64, 32), ("f32", 128, 256), ("f32", 64, 128)])
def test_embed_extract(dtype, d, page):
    """Bit for bit, odd lengths, NaN payloads among them; slots beside them keep theirs."""
    lens = [1, 31, 32, 33, 300, 257]
    t = Twin(1, layers=2, batch=6, hkv=3, hq=3, d=d, page=page, dtype=dtype, lens=lens)
    t.ks[2][0, 0, 3, 5] = float("nan")
    t.ks[2][0, 1, 3, 6] = -0.0
    t.c.embed([2], [32], [t.ks[2]], [t.vs[2]])
    ks, vs = t.c.extract([4, 2, 0, 1, 5, 3], [300, 32, 1, 31, 257, 33])
    bits = torch.int16 if dtype == "bf16" else torch.int32
    for i, b in enumerate([4, 2, 0, 1, 5, 3]):
        assert torch.equal(ks[i].view(bits), t.ks[b].view(bits)) and torch.equal(vs[i].view(bits), t.vs[b].view(bits))
    ks, vs = t.c.extract([4], [77])                        # a prefix
    assert torch.equal(ks[0], t.ks[4][:, :, :77]) and torch.equal(vs[0], t.vs[4][:, :, :77])


def test_many_queries_in_one_call():
    lens = [(7 * b) % 50 + 1 for b in range(70)]           # more than one launch holds
    t = Twin(2, batch=70, lens=lens)
    ks, vs = t.c.extract(list(range(70)), lens)
    assert all(torch.equal(ks[b], t.ks[b]) and torch.equal(vs[b], t.vs[b]) for b in range(70))


# --------------------------------------------------------------- attention --
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,page,width", [(4, 4, 64, 32, 1), (8, 1, 128, 64, 1), (4, 2, 128, 256, 3),
                                                 (8, 2, 64, 128, 16), (16, 2, 128, 32, 8), (2, 2, 64, 64, 16),
                                                 (16, 2, 64, 32, 3)])
def test_attention(dtype, hq, hkv, d, page, width):
    lens = [1, 31, 32, 33, 100, 700, 0, 255]
    t = Twin(3, layers=2, batch=9, hq=hq, hkv=hkv, d=d, page=page, width=width, dtype=dtype, lens=lens, poison=True)
    n_new = [min(width, x) for x in (1, 2, width, width, 1, width, 3, 0, 0)]
    t.first(n_new)                                          # slot 6: new tokens alone; 7: none; 8: free
    t.step([min(width, x) for x in (width, 1, 2, 0, 5, 1, 1, 2, 0)], [max(0, n - 1) for n in n_new])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 0), (32, 4), (33, 32), (64, 33), (100, 5), (333, 100),
                                          (5000, 3)])
def test_window(dtype, window, sinks):
    lens = [1, 5, 64, 129, 400, 1001]
    t = Twin(4, batch=6, hq=4, hkv=2, d=64, page=32, width=4, window=window, sinks=sinks, dtype=dtype, lens=lens,
             poison=True)
    n_new = [1, 4, 4, 2, 4, 3]
    t.first(n_new)
    for keep in ([1, 2, 4, 1, 0, 3], [4, 4, 4, 4, 4, 4], [1, 1, 1, 1, 1, 1]):
        t.step([4] * 6, keep)


@pytest.mark.parametrize("dtype,d,width", [("bf16", 128, 1), ("bf16", 128, 5), ("f32", 64, 2)])
def test_long_queries_are_divided(dtype, d, width):
    lens = [20000, 3, 9999, 511, 257]
    t = Twin(5, batch=5, hq=8, hkv=2, d=d, page=64, width=width, dtype=dtype, lens=lens, poison=True)
    t.first([width, 1, width, width, 1])
    assert int(t.c._state[1]) > 60                          # work items


@pytest.mark.parametrize("hq,hkv,width", [(2, 1, 1), (8, 8, 4), (8, 1, 3)])
def test_the_largest_batch(hq, hkv, width):
    r = np.random.default_rng(hq)
    lens = [int(x) for x in r.integers(0, 300, 512)]
    t = Twin(17, batch=512, hq=hq, hkv=hkv, d=64, page=32, width=width, lens=lens, max_pages=16)
    n_new = [int(x) for x in r.integers(0, width + 1, 512)]
    t.first(n_new)
    ks, vs = t.c.extract([5, 511], [lens[5] + n_new[5], lens[511] + n_new[511]])      # the new tokens are in the pages
    assert torch.equal(ks[0], t.ks[5]) and torch.equal(vs[1], t.vs[511])


@pytest.mark.parametrize("hq,width,lens", [(32, 1, [70000] * 7 + [65000]), (64, 16, [40000])])
def test_items_of_many_blocks(hq, width, lens):
    """Items of more than 64 blocks a wave (and a workgroup's), whose pages are looked up in turns."""
    g = torch.Generator(device="cuda").manual_seed(18)
    batch, hkv, d = len(lens), 32, 64
    c = PagedCache(1, batch, hq, hkv, d, sum(-(-(n + width) // 128) for n in lens), 600, page=128, width=width)
    c.begin(i32(lens))
    ks, vs = ([rand(g, 1, hkv, n, d) for n in lens] for _ in range(2))
    c.embed(list(range(batch)), lens, ks, vs)
    c.begin(i32([width] * batch), keep=i32(lens))
    q, k, v = rand(g, batch, width, hq, d), rand(g, batch, width, hkv, d), rand(g, batch, width, hkv, d)
    out = c.decode_attn(0, q, k, v, out=torch.zeros_like(q))
    assert int(c._state[1]) * 64 * (4 if width == 1 else 1) < sum(-(-n // 32) for n in lens)     # work items
    for b in (0, batch - 1):
        for h in (0, 31):
            kk, vv = (torch.cat([x[b][0, h], y[b, :, h]])[None] for x, y in ((ks, k), (vs, v)))
            heads = slice(h * hq // hkv, (h + 1) * hq // hkv)
            want = O.attention(f64(q[b, :, heads]), f64(kk), f64(vv), lens[b])
            close(out[b, :, heads], want, float(vv.abs().max()), "bf16")


def test_offsets_past_32_bits():
    """A pool of 2^31 and more elements, a query in its last pages."""
    n_pages = 33 * 2 ** 31 // (8 * 256 * 128) // 32
    order = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device="cuda")
    c = PagedCache(1, 2, 8, 8, 128, n_pages, 4, page=256, order=order)
    g = torch.Generator(device="cuda").manual_seed(6)
    ks, vs = (rand(g, 1, 8, 700, 128) for _ in range(2))
    c.begin(i32([700, 0]))
    assert int(c.table[0, 0]) == n_pages - 1
    c.embed([0], [700], [ks], [vs])
    c.begin(i32([1, 0]), keep=i32([700, 0]))
    q, k, v = rand(g, 2, 1, 8, 128), rand(g, 2, 1, 8, 128), rand(g, 2, 1, 8, 128)
    out = c.decode_attn(0, q, k, v, out=torch.zeros_like(q))
    kk, vv = torch.cat([ks[0], k[0].transpose(0, 1)], 1), torch.cat([vs[0], v[0].transpose(0, 1)], 1)
    close(out[0], O.attention(f64(q[0]), f64(kk), f64(vv), 700), float(vv.abs().max()), "bf16")
    got = c.extract([0], [701])
    assert torch.equal(got[0][0][0], kk) and torch.equal(got[1][0][0], vv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_unseen_infinities(dtype, bad):
    """A draft's infinite or NaN key and value reach that draft and those behind it alone; tokens
    outside the window nobody."""
    t = Twin(7, batch=2, hq=8, hkv=2, d=64, page=32, width=6, window=50, sinks=2, dtype=dtype, lens=[300, 70])
    t.ks[0][:, :, 30:250], t.vs[0][:, :, 30:250] = bad, bad
    t.c.embed([0], [300], [t.ks[0]], [t.vs[0]])
    t.c.begin(i32([6, 6]), keep=i32([300, 70]))
    q = rand(t.g, 2, 6, 8, 64, dtype=dtype)
    k, v = (rand(t.g, 2, 6, 2, 64, dtype=dtype) for _ in range(2))
    v[:, 3, 1, 5], k[:, 5] = bad, bad
    out = t.c.decode_attn(0, q, k, v, out=torch.zeros_like(q))
    for b, n in enumerate((300, 70)):
        kk = torch.cat([t.ks[b][0], k[b].transpose(0, 1)], 1)
        vv = torch.cat([t.vs[b][0], v[b].transpose(0, 1)], 1)
        for i in range(5):
            o, want = out[b, i], O.attention(f64(q[b, i:i + 1]), f64(kk[:, :n + i + 1]), f64(vv[:, :n + i + 1]), n + i, 50, 2)
            if i >= 3:                                      # column 5 of kv-head 1: what the formula says
                assert not torch.isfinite(o[4:, 5]).any()
                assert np.array_equal(np.isnan(f64(o)), np.isnan(want[0])) and \
                    np.array_equal(np.isposinf(f64(o)), np.isposinf(want[0]))
                o[4:, 5], want[0, 4:, 5] = 0, 0
            tol = 2.0 ** -12 * 5 + 2.0 ** -7 * np.abs(want[0]) + 2.0 ** -8 * 5 * (i >= 3)   # a block in 8 bits
            assert (np.abs(f64(o) - want[0]) <= tol).all(), (b, i)


def test_large_scores_and_equal_ones():
    t = Twin(8, batch=1, hq=2, hkv=1, d=64, width=2, dtype="f32", lens=[600])
    t.c.begin(i32([2]), keep=i32([600]))
    q = torch.zeros(1, 2, 2, 64, device="cuda")
    q[0, 1] = 1e4 * rand(t.g, 2, 64, dtype="f32")
    k, v = (rand(t.g, 1, 2, 1, 64, dtype="f32") for _ in range(2))
    out = t.c.decode_attn(0, q, k, v, out=torch.zeros_like(q))
    kk, vv = torch.cat([t.ks[0][0], k[0].transpose(0, 1)], 1), torch.cat([t.vs[0][0], v[0].transpose(0, 1)], 1)
    close(out[0, 0], np.broadcast_to(f64(vv[0, :601]).mean(0), (2, 64)), float(vv.abs().max()), "f32")
    s = f64(kk[0]) @ f64(q[0, 1]).T
    assert np.allclose(f64(out[0, 1]), f64(vv[0])[s.argmax(0)], atol=1e-5)   # scores thousands apart


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scale_and_keys_already_there(dtype):
    t = Twin(9, batch=2, hq=4, hkv=2, d=64, width=3, dtype=dtype, lens=[90, 10])
    outs = t.first([3, 2])
    q, k, v = t.last
    again = t.c.decode_attn(0, q[0], None, None, out=torch.full_like(q[0], 7.0))
    assert torch.equal(again, outs[0])
    out = t.c.decode_attn(0, q[0], k[0], v[0], out=torch.zeros_like(q[0]), scale=0.3)
    for b, n in ((0, 3), (1, 2)):
        vv = f64(t.vs[b][0])
        close(out[b, :n], O.attention(f64(q[0, b, :n]), f64(t.ks[b][0]), vv, t.lens[b], scale=0.3), 4 * np.abs(vv).max(), dtype)


def test_a_slot_without_pages_takes_no_part():
    t = Twin(10, batch=3, hq=2, hkv=1, d=64, page=32, width=2, lens=[32, 32, 32], n_pages=4, max_pages=4)
    t.c.begin(i32([2, 2, 1]), keep=i32([32, 32, 32]))
    assert t.c.missing.tolist() == [0, 1, 1]
    q, k, v = rand(t.g, 3, 2, 2, 64), rand(t.g, 3, 2, 1, 64), rand(t.g, 3, 2, 1, 64)
    before = t.c.extract([1, 2], [32, 32])
    out = t.c.decode_attn(0, q, k, v, out=torch.full_like(q, 7.0))
    assert (out[1:] == 7.0).all() and (out[0] != 7.0).all()
    after = t.c.extract([1, 2], [32, 32])
    assert all(torch.equal(x, y) for x, y in zip(before[0] + before[1], after[0] + after[1]))


def test_prompts_are_left_alone():
    """A step in which one slot brings a prompt: the others decode."""
    t = Twin(11, batch=2, hq=2, hkv=2, d=64, width=1, lens=[50], n_pages=40, max_pages=20)
    t.c.begin(i32([1, 200]), keep=i32([50, 0]))
    ks, vs = (rand(t.g, 1, 2, 200, 64) for _ in range(2))
    t.c.embed([1], [200], [ks], [vs])
    q, k, v = rand(t.g, 2, 1, 2, 64), rand(t.g, 2, 1, 2, 64), rand(t.g, 2, 1, 2, 64)
    out = t.c.decode_attn(0, q, k, v, out=torch.full_like(q, 7.0))
    assert (out[1] == 7.0).all()
    kk, vv = torch.cat([t.ks[0][0], k[0].transpose(0, 1)], 1), torch.cat([t.vs[0][0], v[0].transpose(0, 1)], 1)
    close(out[0], O.attention(f64(q[0]), f64(kk), f64(vv), 50), float(vv.abs().max()), "bf16")
    assert torch.equal(t.c.extract([1], [200])[0][0], ks)


def test_rope():
    from paper_2410_18701_amd import baton as B
    t = Twin(12, batch=3, hq=4, hkv=2, d=64, width=3, lens=[5, 0, 70000], max_pages=2200)
    t.c.begin(i32([3, 3, 2]), keep=i32([5, 0, 70000]))
    qkv = rand(t.g, 3, 3, 8 * 64)
    q, k, v = rand(t.g, 3, 3, 4, 64), rand(t.g, 3, 3, 2, 64), rand(t.g, 3, 3, 2, 64)
    B.baton_paged_rope_qkv(t.c.desc, qkv, 3, q, k, v, 10000.0, torch.cuda.current_stream())
    x = f64(qkv).reshape(3, 3, 8, 64)
    pos = np.array([5, 0, 70000])[:, None] + np.arange(3)
    ang = pos[:, :, None] * 10000.0 ** (-np.arange(32) / 32)
    c, s = np.cos(ang)[:, :, None], np.sin(ang)[:, :, None]
    y = np.concatenate([x[..., :32] * c - x[..., 32:] * s, x[..., :32] * s + x[..., 32:] * c], -1)
    # half a step, and 2^-20 of the pair for the fp32 sine and cosine and their products
    mag = np.concatenate([np.hypot(x[..., :32], x[..., 32:])] * 2, -1)
    tol = 2.0 ** -8 * np.abs(y) + 2.0 ** -20 * mag
    assert (np.abs(f64(q) - y[:, :, :4]) <= tol[:, :, :4]).all() and (np.abs(f64(k) - y[:, :, 4:6]) <= tol[:, :, 4:6]).all()
    assert torch.equal(v.flatten(), qkv.view(3, 3, 8, 64)[:, :, 6:].flatten())


def test_other_stream_and_repeats():
    t = Twin(13, batch=4, hq=8, hkv=2, d=128, page=64, width=2, lens=[3000, 5, 900, 64])
    outs = t.first([2, 1, 2, 2])
    q, k, v = t.last
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = [t.c.decode_attn(0, q[0], k[0], v[0], out=torch.full_like(q[0], 7.0)) for _ in range(5)]
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(x, outs[0]) for x in again)


def test_captured_steps():
    """Steps captured once and replayed: lengths, tables and results follow what the device holds."""
    def make():
        t = Twin(14, batch=3, hq=4, hkv=2, d=64, page=32, width=3, lens=[60, 700, 1], n_pages=60, max_pages=30)
        t.c.begin(i32([0, 0, 0]), keep=i32([60, 700, 1]))
        return t

    t, e = make(), make()
    n_new, keep = i32([3, 2, 1]), i32([0, 0, 0])
    q, k, v = rand(t.g, 3, 3, 4, 64), rand(t.g, 3, 3, 2, 64), rand(t.g, 3, 3, 2, 64)
    out = torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.c.begin(n_new, keep=keep)
        t.c.decode_attn(0, q, k, v, out=out)
    for i in range(12):
        new, kept = [(1, 2, 3), (3, 3, 3), (2, 0, 1)][i % 3], [(0, 0, 0), (1, 1, 2), (3, 2, 1)][i % 3]
        n_new.copy_(i32(new))
        keep.copy_(i32(kept))
        for x in (q, k, v):
            x.copy_(rand(t.g, *x.shape))
        out.zero_()
        graph.replay()
        e.c.begin(i32(new), keep=i32(kept))
        want = e.c.decode_attn(0, q, k, v, out=torch.zeros_like(q))
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(t.c.table, e.c.table) and torch.equal(t.c.lens, e.c.lens), i


def test_from_the_aligned_cache_and_back():
    """Queries of a BatonCache, extracted, go into pages, and out of them back, bit for bit."""
    from paper_2410_18701_amd.cache import BatonCache
    g = torch.Generator(device="cuda").manual_seed(15)
    ring = BatonCache(2, 3, 4, 2, 64, 300)
    ks, vs = ([rand(g, 2, 2, n, 64) for n in (40, 131)] for _ in range(2))
    ring.embed([0, 2], [40, 131], ks, vs)
    c = PagedCache(2, 3, 4, 2, 64, 20, 8, page=32)
    c.begin(i32([131, 0, 40]))
    k1, v1 = ring.extract([0, 2])
    c.embed([2, 0], [40, 131], k1, v1)
    k2, v2 = c.extract([0, 2], [131, 40])
    ring.evict([0, 2])
    ring.embed([1, 0], [131, 40], k2, v2)
    k3, v3 = ring.extract([0, 1])
    assert all(torch.equal(x, y) for x, y in zip(k3 + v3, ks + vs))


def test_wrapper_refusals_on_the_gpu():
    t = Twin(16, batch=2, hq=2, hkv=1, d=64, lens=[5, 5])
    q, k = rand(t.g, 2, 1, 2, 64), rand(t.g, 2, 1, 1, 64)
    for bad in (lambda: t.c.begin(torch.zeros(2, dtype=torch.int64, device="cuda")), lambda: t.c.begin(i32([1])),
                lambda: t.c.begin(i32([1, 1]), keep=i32([1])), lambda: t.c.begin(torch.zeros(2, dtype=torch.int32)),
                lambda: t.c.decode_attn(0, q[:1], k, k), lambda: t.c.decode_attn(0, q.float(), k, k),
                lambda: t.c.decode_attn(0, q.cpu(), k, k), lambda: t.c.embed([0], [5], [t.ks[0].cpu()], [t.vs[0]]),
                lambda: t.c.embed([0], [4], [t.ks[0]], [t.vs[0]]), lambda: t.c.embed([0, 1], [5], [t.ks[0]], [t.vs[0]]),
                lambda: t.c.reset(order=i32([0]))):
        with pytest.raises(ValueError):
            bad()
