"""A cache held in 4 bits on the GPU against its float64 model (oracle/mxfp4.py):
the tokens bit for bit after every operation, attention within its roundings.

Tolerance of an output element, from the roundings alone: each softmax weight
is rounded to bf16 (at most 2^-8 of it) before its product with the value, so
the weighted sum is off by at most 2^-8 A, A = sum p |v| / sum p; the output's own
rounding adds 2^-8 |out|; scores, exponentials and sums in fp32 (a few hundred
terms, scores below 2^6) stay within 2^-13 A."""
import numpy as np
import pytest
import torch

from oracle import mxfp4 as X
from paper_2410_18701_amd import baton as B
from paper_2410_18701_amd.cache import BatonCache

pytestmark = pytest.mark.gpu


def bf16(t):
    """float64 bf16 values -> device tensor (exact)."""
    return torch.from_numpy(np.ascontiguousarray(t, np.float32)).cuda().to(torch.bfloat16)


def val(t):
    return t.double().cpu().numpy()


class Pair:
    """A GPU cache and its model, driven together."""

    def __init__(self, layers, batch, hq, hkv, d, capacity, seed=0, split=None, layout="by_layer", noalloc=False):
        self.c = BatonCache(layers, batch, hq, hkv, d, capacity, dtype="mxfp4", layout=layout)
        self.m = X.Batch4(layers, batch, hq, hkv, d)
        self.rng = np.random.default_rng(seed)
        self.saved, self.worst, self.noalloc = {}, 0.0, noalloc
        if split:
            self.c.set_split_tokens(split)

    def draw(self, *shape, spread=1.0):
        return X.round_bf16(spread * self.rng.standard_normal(shape) * np.exp2(self.rng.integers(-2, 3, shape[-1])))

    def embed(self, slots, lens):
        ks, vs = ([self.draw(self.m.layers, self.m.hkv, n, self.m.d) for n in lens] for _ in range(2))
        self.c.embed(slots, lens, [bf16(x) for x in ks], [bf16(x) for x in vs])
        self.m.embed(slots, ks, vs)
        self.check()

    def evict(self, slots, **kw):
        self.c.evict(slots, **kw)
        self.m.evict(slots)

    def extract(self, slots, name):
        ks, vs = self.c.extract(slots)
        for b, k, v in zip(slots, ks, vs):
            assert np.array_equal(val(k), self.m.k[b], equal_nan=True) and np.array_equal(val(v), self.m.v[b], equal_nan=True)
        self.saved[name] = (ks, vs, [(self.m.k[b], self.m.v[b]) for b in slots])

    def embed_saved(self, slots, name):
        ks, vs, model = self.saved.pop(name)
        self.c.embed(slots, [k.shape[2] for k in ks], ks, vs)
        for b, (k, v) in zip(slots, model):
            self.m.k[b], self.m.v[b] = k, v     # stored once: the same values again
        self.check()

    def move(self, src, dst):
        self.c.move(src, dst)
        self.m.move(src, dst)
        self.check()

    def check(self):
        """Every live slot's tokens, bit for bit."""
        live = [b for b in range(self.m.batch) if self.m.k[b] is not None]
        assert [n > 0 for n in self.c.tokens()] == [k is not None for k in self.m.k]
        assert [self.c.tokens()[b] for b in live] == [self.m.k[b].shape[2] for b in live]
        if live:
            ks, vs = self.c.extract(live)
            for b, k, v in zip(live, ks, vs):
                assert np.array_equal(val(k), self.m.k[b], equal_nan=True), f"keys of slot {b}"
                assert np.array_equal(val(v), self.m.v[b], equal_nan=True), f"values of slot {b}"

    def step(self, prompts=None, scale=0.0, spread=1.0, q=None):
        m, prompts = self.m, prompts or {}
        T = max(prompts.values(), default=1)
        if prompts:
            self.c.shape_insert(list(prompts), list(prompts.values()))
        q = self.draw(m.layers, m.batch, T, m.hq, m.d, spread=spread) if q is None else q
        k, v = (self.draw(m.layers, m.batch, T, m.hkv, m.d) for _ in range(2))
        got = []
        for l in range(m.layers):
            args = [bf16(x[l]) if T > 1 or prompts else bf16(x[l, :, 0]) for x in (q, k, v)]
            out = torch.full_like(args[0], 7.0)
            if self.noalloc:
                B.baton_decode_attn_noalloc(self.c.handle, l, *args, out, scale, torch.cuda.current_stream())
            else:
                self.c.decode_attn(l, *args, out=out, scale=scale)
            got.append(val(out).reshape(m.batch, T, m.hq, m.d))
        self.c.advance()
        want = m.step(q, k, v, prompts, scale or None)
        for l in range(m.layers):
            for b in range(m.batch):
                for t in range(T):
                    if (l, b, t) not in want:
                        assert (got[l][b, t] == 7.0).all(), "a position that holds no token was written"
                        continue
                    o, a = want[l, b, t]
                    tol = 2.0 ** -8 * (a + np.abs(o)) + 2.0 ** -13 * a + 1e-30
                    err = np.abs(got[l][b, t] - o) / tol
                    assert err.max() <= 1, f"layer {l} slot {b} position {t}: {err.max():.3g} of the tolerance"
                    self.worst = max(self.worst, err.max())
        self.check()


SHAPES = [(1, 3, 4, 4, 64), (2, 3, 8, 4, 64), (1, 3, 8, 2, 64), (1, 3, 16, 2, 64),
          (1, 3, 4, 4, 128), (1, 3, 4, 2, 128), (2, 3, 8, 2, 128), (1, 3, 16, 2, 128)]


def _sid(s):
    return f"{s[0]}x{s[1]}-{s[2]}/{s[3]}x{s[4]}"


@pytest.mark.parametrize("d", [64, 128])
def test_format_of_every_bf16_value(d):
    """Blocks that hold every bf16 pattern as an element and as the largest one,
    zeros, subnormals, infinities and NaN: stored and copied out by the
    definition, and stored again with the same bytes."""
    bits = np.arange(65536, dtype=np.uint32)
    every = (bits << 16).view(np.float32).astype(np.float64)
    rng = np.random.default_rng(3)
    alone = np.zeros((65536, 32))
    alone[bits, rng.integers(0, 32, 65536)] = every              # the largest of its block
    with np.errstate(all="ignore"):
        mixed = every[rng.permutation(65536)].reshape(-1, 32)    # any beside any
        near = np.where(np.isfinite(every), every, 1.0)[:, None] * rng.choice([0.03, 0.25, 0.4, 0.6, 0.9, 1.0], (65536, 32))
    near = X.round_bf16(near)
    x = np.concatenate([alone, mixed, near]).reshape(-1, d)
    tiny = (np.abs(x) < 2.0 ** -126) & (x != 0)
    n = len(x)
    c = BatonCache(1, 1, 1, 1, d, -(-(n + 1) // 16) * 16, dtype="mxfp4")
    raw = torch.from_numpy(x.astype(np.float32).reshape(1, 1, n, d)).cuda().to(torch.bfloat16)
    assert tiny.any()
    c.embed([0], [n], [raw], [raw.flip(2).contiguous()])
    (k,), (v,) = c.extract([0])
    want = X.stored(x)
    assert np.array_equal(val(k)[0, 0], want, equal_nan=True)
    assert np.array_equal(val(v)[0, 0, ::-1], want, equal_nan=True)
    assert np.array_equal(val(c.logical("k"))[0, 0, 0], want, equal_nan=True)
    before = c.k.clone(), c.v.clone()
    c.evict([0], scrub=False, release=False)
    c.embed([0], [n], [k], [v])
    assert torch.equal(before[0], c.k) and torch.equal(before[1], c.v)


@pytest.mark.parametrize("shape", SHAPES, ids=_sid)
def test_rows_around_the_block_edges(shape):
    """Rows of one token, around 64 and 128 (a wave's blocks) and around the
    split, a slot free throughout; over the ring's end."""
    layers, _, hq, hkv, d = shape
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 191, 256, 257, 383, 385]
    p = Pair(layers, len(lens) + 1, hq, hkv, d, 400, seed=d + hq, split=128)
    p.embed(list(range(len(lens))), lens)
    for _ in range(3):
        p.step()
    assert p.c.query()[1] != 0      # base has moved: the window wraps
    print(f"[kv4] {shape}: {p.worst:.3g} of the tolerance", flush=True)


@pytest.mark.parametrize("shape", [(1, 1, 4, 4, 64), (1, 1, 8, 4, 64), (1, 1, 16, 4, 64), (1, 1, 16, 2, 64),
                                   (1, 1, 4, 4, 128), (1, 1, 4, 2, 128), (1, 1, 8, 2, 128), (1, 1, 16, 2, 128)], ids=_sid)
def test_weights_are_kept_past_bf16(shape):
    """Sums of a few values that nearly cancel: the softmax weights are rounded no more
    than to 2^-16 of each, so beside the output's own rounding an element is off by
    that and the 2^-13 of fp32 arithmetic times sum p |v| / sum p."""
    layers, _, hq, hkv, d = shape
    lens = [1 + b % 29 for b in range(58)] + [300, 64]
    p = Pair(layers, len(lens), hq, hkv, d, 320, seed=hq, split=128)
    p.embed(list(range(len(lens))), lens)
    q, k, v = (p.draw(layers, len(lens), 1, h, d) for h in (hq, hkv, hkv))
    got = val(p.c.decode_attn(0, *(bf16(x[0, :, 0]) for x in (q, k, v))))
    worst = 0.0
    for (_, b, _), (o, a) in p.m.step(q, k, v).items():
        err = np.abs(got[b] - o) / (2.0 ** -8 * np.abs(o) + (2.0 ** -16 + 2.0 ** -13) * a + 1e-30)
        worst = max(worst, err.max())
    print(f"[kv4] {shape}: {worst:.3g} of the tolerance", flush=True)
    assert worst <= 1


def test_an_infinite_value_of_the_step_itself():
    """The step's own value takes part as given: an infinity comes out as one."""
    for hq, hkv, d in ((2, 2, 64), (8, 1, 64), (2, 2, 128), (4, 2, 128), (4, 1, 128), (8, 1, 128)):
        c = BatonCache(1, 3, hq, hkv, d, 48, dtype="mxfp4")
        k, v = (torch.randn(1, hkv, 30, d, device="cuda").bfloat16() for _ in range(2))
        c.embed([0, 2], [30, 30], [k, k], [v, v])
        q, kn, vn = (torch.randn(3, h, d, device="cuda").bfloat16() for h in (hq, hkv, hkv))
        vn[0, 0, 5], vn[0, 0, d - 1] = float("inf"), -float("inf")
        out = c.decode_attn(0, q, kn, vn)
        g = hq // hkv
        assert (out[0, :g, 5] == float("inf")).all() and (out[0, :g, d - 1] == -float("inf")).all()
        out[0, :g, 5] = out[0, :g, d - 1] = 0.0
        assert out.isfinite().all()


@pytest.mark.parametrize("shape", SHAPES, ids=_sid)
@pytest.mark.parametrize("layout", ["by_layer", "separate"])
def test_story(shape, layout):
    """Arrivals, steps, preemption and return, moves, release, evictions with
    and without scrubbing, prompts prefilled inside the batch and the holes they leave."""
    layers, batch, hq, hkv, d = shape
    p = Pair(layers, batch + 2, hq, hkv, d, 320, seed=hkv, layout=layout, split=64)
    p.embed([0, 2], [37, 90])
    p.step()
    p.extract([2], "low")
    p.evict([2])
    p.embed([2, 1], [12, 130])          # grows on the left
    p.step()
    p.move([2], [4])
    p.step()
    p.evict([1], scrub=False)
    p.embed_saved([3], "low")
    p.step(prompts={1: 9, 2: 33})       # holes of 32 columns in the other rows
    p.step()
    p.step(prompts={})
    p.evict([0, 4], scrub=True)
    p.move([3], [0])                    # a row with holes, over owed placeholders
    p.step()
    p.move([0], [3])
    p.step(prompts={0: 1})
    p.step(prompts={4: 70})
    for _ in range(2):
        p.step()
    p.extract([3, 1], "pair")
    p.evict([3, 1])
    p.step()
    p.embed_saved([1, 3], "pair")
    p.step()
    print(f"[kv4] {shape}: {p.worst:.3g} of the tolerance", flush=True)


@pytest.mark.parametrize("shape", [(1, 3, 4, 4, 64), (1, 3, 16, 2, 128), (1, 3, 3, 3, 128)], ids=_sid)
def test_many_holes(shape):
    """Rows of different ages through many holes: gathered items."""
    layers, batch, hq, hkv, d = shape
    p = Pair(layers, 5, hq, hkv, d, 512, seed=11, noalloc=True)
    p.embed([0, 1], [50, 3])
    for i in range(24):
        b = 2 + i % 3
        if p.m.k[b] is not None:
            p.evict([b], scrub=i % 2 == 0)
        p.step(prompts={b: 2 + i % 5})
        if i % 4 == 0:
            p.step()
    print(f"[kv4] {shape}: {p.worst:.3g} of the tolerance", flush=True)


@pytest.mark.parametrize("d,hq,hkv", [(128, 8, 1), (64, 2, 2)])
@pytest.mark.parametrize("scale", [2.0, -0.5])
def test_peaked_scores(d, hq, hkv, scale):
    """Scores up to some hundreds: one token has nearly all the weight, maxima
    rise late, others underflow.  Scores of that size are themselves off by up
    to d 2^-24 of the sum of their terms; the weights' error is that times the
    score, so values of one sign and equal magnitude make the outputs tell."""
    p = Pair(1, 2, hq, hkv, d, 784, seed=5, split=256)
    p.embed([0, 1], [700, 133])
    q = X.round_bf16(0.25 * p.rng.standard_normal((1, 2, 1, hq, d)))
    p.step(scale=scale, q=q)
    p.step(scale=scale, q=q)


def test_a_stored_nan_reaches_its_row_alone():
    """An infinity in a key makes its whole row NaN, in a value its block of 32; other rows are untouched."""
    d, n = 128, 100
    c = BatonCache(1, 3, 2, 2, d, 112, dtype="mxfp4")
    k, v = torch.randn(3, 1, 2, n, d, device="cuda").bfloat16(), torch.randn(3, 1, 2, n, d, device="cuda").bfloat16()
    k[0, 0, 1, 70, 5] = float("inf")
    v[1, 0, 0, 3, 40] = float("nan")
    c.embed([0, 1, 2], [n] * 3, list(k), list(v))
    x = [torch.randn(3, 2, d, device="cuda").bfloat16() for _ in range(3)]
    out = c.decode_attn(0, *x).isnan()
    assert out[0, 1].all() and not out[0, 0].any()
    assert out[1, 0, 32:64].all() and not out[1, 0, :32].any() and not out[1, 0, 64:].any() and not out[1, 1].any()
    assert not out[2].any()


def test_more_tiles_than_one_launch():
    """32 queries of one to three tokens over 128 layers of 64 heads: 524,288 tiles to an embed."""
    layers, slots, heads, d = 128, 32, 64, 64
    c = BatonCache(layers, slots, heads, heads, d, 16, dtype="mxfp4")
    lens = [1 + b % 3 for b in range(slots)]
    ks, vs = ([torch.randn(layers, heads, n, d, device="cuda").bfloat16() for n in lens] for _ in range(2))
    c.embed(list(range(slots)), lens, ks, vs)
    gk, gv = c.extract(list(range(slots)))
    for b in (0, 1, 30, 31):
        for got, src in ((gk[b], ks[b]), (gv[b], vs[b])):
            for l in (0, 77, 127):
                assert np.array_equal(val(got[l]), X.stored(val(src[l])))
    again = BatonCache(layers, slots, heads, heads, d, 16, dtype="mxfp4")
    again.embed(list(range(slots)), lens, gk, gv)
    assert torch.equal(c.k, again.k) and torch.equal(c.v, again.v)


def test_placeholders():
    """Every byte that is no live token's holds the placeholder after scrubbing, and what the fill asks for."""
    for fill in (None, 0x5A):
        c = BatonCache(2, 2, 2, 2, 64, 48, dtype="mxfp4", fill_bits=fill)
        byte = 0xFF if fill is None else fill
        assert (c.k == byte).all() and (c.v == byte).all()
        x = torch.randn(2, 2, 20, 64, device="cuda").bfloat16()
        c.embed([1], [20], [x], [x])
        assert not (c.k[:, 1] == byte).all() and (c.k[:, 0] == byte).all()
        c.evict([1])
        c.flush()
        assert (c.k == byte).all() and (c.v == byte).all()


def test_long_rows_and_offsets_past_32_bits():
    """Two rows far into a ring of 4.6 GB of K: lengths of 20,000 over heads of 128."""
    cap, hkv, d, n = 1 << 16, 64, 128, 20000
    c = BatonCache(1, 17, hkv, hkv, d, cap, dtype="mxfp4", assume_filled=True, layout="separate")
    assert c.k[0].numel() > 1 << 32
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(1, hkv, n, d, device="cuda", generator=g).bfloat16() for _ in range(2))
    c.embed([16], [n], [k], [v])
    (ks,), (vs,) = c.extract([16])
    x = [torch.randn(17, hkv, d, device="cuda", generator=g).bfloat16() for _ in range(3)]
    out = c.decode_attn(0, *x)
    assert (out[:16] == 0).all()
    for h in (0, 31, 63):
        assert np.array_equal(val(ks[0, h, ::997]), X.stored(val(k[0, h, ::997])))
        kk, vv = np.concatenate([val(ks[0, h]), val(x[1][16, h])[None]]), np.concatenate([val(vs[0, h]), val(x[2][16, h])[None]])
        o, a = X.attend(val(x[0][16, h]), kk, vv, d ** -0.5)
        err = np.abs(val(out[16, h]) - o)
        assert (err <= 2.0 ** -8 * (a + np.abs(o)) + 2.0 ** -13 * a).all()


def test_host_round_trip():
    """Tokens parked in pinned host memory and brought back."""
    from paper_2410_18701_amd.scaling import BatchScaler
    c = BatonCache(2, 3, 4, 2, 64, 128, dtype="mxfp4")
    x = [torch.randn(2, 2, n, 64, device="cuda").bfloat16() for n in (30, 95, 20)]
    c.embed([0, 1, 2], [30, 95, 20], x, x)
    (k0,), (v0,) = c.extract([1])
    s = BatchScaler(c, 200)
    assert s.shrink() == [1]
    c.evict([0])
    assert s.grow() == [0]
    (k1,), (v1,) = c.extract([0])
    torch.cuda.synchronize()
    assert torch.equal(k0, k1) and torch.equal(v0, v1)


def test_step_in_a_hip_graph():
    """A captured step replays bit for bit like the eager one, other work between the replays."""
    caches = []
    for _ in range(2):
        p = Pair(2, 4, 8, 2, 128, 320, seed=7, split=64)
        p.embed([0, 1, 3], [200, 3, 77])
        p.evict([3])                      # owed placeholders are written in the captured step
        caches.append(p.c)
    eager, graphed = caches
    x = [torch.randn(2, 4, h, 128, device="cuda").bfloat16() for h in (8, 2, 2)]
    want = [eager.decode_attn(l, *(t[l] for t in x)) for l in range(2)]
    outs = [torch.empty_like(o) for o in want]
    graphed.workspace()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for l in range(2):
            graphed.decode_attn(l, *(t[l] for t in x), out=outs[l])
    for _ in range(3):
        for o in outs:
            o.fill_(float("nan"))
        torch.randn(1 << 16, device="cuda").sum()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    assert torch.equal(eager.k, graphed.k) and torch.equal(eager.v, graphed.v)
