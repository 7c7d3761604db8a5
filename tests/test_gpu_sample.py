"""Sampling on the GPU against its float64 definition (oracle/sampling.py): the
same token for the same numbers, everywhere."""
import numpy as np
import pytest
import torch

from oracle.sampling import sample
from paper_2410_18701_amd.layer import Sampler

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def run(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    f = lambda v, t: None if v is None else torch.tensor(v, dtype=t, device="cuda")  # noqa: E731
    rows, vocab = logits.shape
    got = Sampler(rows, vocab)(logits, f(u, torch.float32), f(temperature, torch.float32), f(top_k, torch.int32),
                               f(top_p, torch.float32), f(min_p, torch.float32))
    return got.cpu().tolist()


def check(logits, u, **params):
    got = run(logits, u, **params)
    l = logits.double().cpu().numpy()
    f32 = lambda x: float(np.float32(x))  # noqa: E731
    for r in range(len(got)):
        p = {k: (int(v[r]) if k == "top_k" else f32(v[r])) for k, v in params.items() if v is not None}
        want = sample(l[r], f32(u[r]), **p)
        assert got[r] == want, f"row {r}: {got[r]}, not {want}, with u {u[r]} and {p}"


def draw_params(rng, rows):
    return dict(temperature=rng.choice([0.0, 0.2, 0.7, 1.0, 1.3, 5.0], rows).tolist(),
                top_k=rng.choice([0, 1, 2, 7, 40, 1000, 5000, 1 << 30], rows).tolist(),
                top_p=rng.choice([0.0, 0.01, 0.5, 0.9, 0.99, 0.9999, 1.0, 2.0], rows).tolist(),
                min_p=rng.choice([0.0, 0.0, 1e-4, 0.05, 0.5, 1.0, 1.5], rows).tolist())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 8, 9, 63, 64, 511, 1000, 4097, 32000, 50257, 131072, 300001])
def test_vocabularies(dtype, vocab):
    rng = np.random.default_rng(vocab)
    rows = 48 if vocab < 100000 else 20
    logits = torch.from_numpy(rng.standard_normal((rows, vocab)).astype(np.float32) * 2.5).cuda().to(DT[dtype])
    check(logits, rng.random(rows).tolist(), **draw_params(rng, rows))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_each_parameter_alone_and_none(dtype):
    rng = np.random.default_rng(5)
    rows = 300     # more rows than compute units
    logits = torch.from_numpy(rng.standard_normal((rows, 3000)).astype(np.float32) * 3).cuda().to(DT[dtype])
    u = rng.random(rows).tolist()
    check(logits, u)
    for name, v in draw_params(rng, rows).items():
        check(logits, u, **{name: v})


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [40000, 5000, 100])
def test_ties(dtype, vocab):
    """Equal logits: prefixes end inside a tie, the lowest indices are kept; more
    of one value than a list holds; a few values only."""
    rng = np.random.default_rng(vocab)
    rows = 32
    flat = np.zeros((rows, vocab), np.float32)
    flat[1::2] = rng.choice([0.0, -0.0, 0.5, 1.0], (rows // 2, vocab))
    flat[2, 17] = 3.0
    ks = rng.choice([1, 2, 3, 50, vocab // 2, vocab - 1, vocab], rows)
    check(torch.from_numpy(flat).cuda().to(DT[dtype]), rng.random(rows).tolist(), top_k=ks.tolist(),
          top_p=rng.choice([1.0, 0.5, 0.25, 0.9], rows).tolist())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_crowded_bins(dtype):
    """A far outlier and a high temperature squeeze all other tokens into a bin."""
    rng = np.random.default_rng(2)
    rows, vocab = 16, 30000
    l = rng.standard_normal((rows, vocab)).astype(np.float32)
    l[:, 5] = -1e6
    check(torch.from_numpy(l).cuda().to(DT[dtype]), rng.random(rows).tolist(), temperature=[1e6] * rows,
          top_k=rng.choice([0, 3, 2500, 20000], rows).tolist(), top_p=rng.choice([0.1, 0.5, 0.99, 1.0], rows).tolist())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [5000, 32000, 128000])
def test_a_nucleus_above_a_crowded_cut_by_count(dtype, vocab):
    """top_k past what a list holds ends among thousands of different values of one
    bin (most of the row lies more than 32 temperatures below the maximum), top_p in
    a bin of few: each prefix by its own sums, wherever in the row the weight is."""
    rng = np.random.default_rng(vocab + len(dtype))
    combos = [(t, k, p) for t in (0.1, 0.3) for k in (2000, vocab // 3, vocab - 1) for p in (0.5, 0.9, 0.99)]
    us = (np.arange(8) + rng.random()) / 8
    t, k, p, u = (list(x) for x in zip(*[c + (float(x),) for c in combos for x in us]))
    l = rng.standard_normal((len(u), vocab)).astype(np.float32) * 4
    l[::3, :vocab // 4] += 3.0            # the weight in the first quarter of the row, ...
    l[1::3, vocab * 3 // 4:] += 3.0       # ... in the last, anywhere
    check(torch.from_numpy(l).cuda().to(DT[dtype]), u, temperature=t, top_k=k, top_p=p)


def test_many_neighbours_of_a_large_vocabulary():
    """More kept tokens side by side than one range of the list's draw takes."""
    vocab, n = 1 << 21, 1500
    l = np.full((3, vocab), -np.inf, np.float32)
    rng = np.random.default_rng(8)
    for r, first in enumerate((0, 4096, vocab - n)):
        l[r, first:first + n] = rng.standard_normal(n)
    l[1, 5] = 0.0
    logits = torch.from_numpy(l).cuda()
    for u in (0.0, 0.25, 0.5, 0.999999):
        check(logits, [u] * 3, min_p=[1e-6] * 3)
        check(logits, [u] * 3, top_k=[1200] * 3)
        check(logits, [u] * 3, top_p=[0.97] * 3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_and_infinite_logits(dtype):
    inf, low = float("inf"), -3.3895313892515355e38
    v = 400
    base = np.linspace(-3, 3, v).astype(np.float32)
    cases = [np.full(v, -inf), np.full(v, np.nan), np.full(v, low)]
    one = np.full(v, -inf)
    one[123] = -5.0
    cases.append(one)
    masked = base.copy()
    masked[::2] = -inf
    cases.append(masked)
    lowest = base.copy()
    lowest[10:] = low
    cases.append(lowest)
    nans = base.copy()
    nans[390:] = np.nan
    cases.append(nans)
    infs = base.copy()
    infs[[7, 200, 201]] = inf
    infs[5] = np.nan
    cases.append(infs)
    logits = torch.from_numpy(np.stack(cases).astype(np.float32)).cuda().to(DT[dtype])
    n = len(cases)
    for u in (0.0, 0.3, 0.7, 0.999):
        check(logits, [u] * n)
        check(logits, [u] * n, temperature=[0.5] * n, top_k=[30] * n, top_p=[0.9] * n, min_p=[0.01] * n)
        check(logits, [u] * n, temperature=[1e-30] * n, top_k=[2] * n)
        check(logits, [u] * n, temperature=[0.0] * n)
        check(logits, [u] * n, top_k=[1000] * n, min_p=[1.0] * n)
        check(logits, [u] * n, temperature=[float("inf")] * n, top_p=[0.5] * n)
    assert run(logits, [0.5] * n)[:2] == [-1, -1]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ends_of_u_and_odd_parameters(dtype):
    rng = np.random.default_rng(3)
    logits = torch.from_numpy(rng.standard_normal((9, 777)).astype(np.float32)).cuda().to(DT[dtype])
    nan = float("nan")
    us = [0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, nan, 1e-45, 0.5, 2.0 ** -30]
    check(logits, us)
    check(logits, us, top_k=[40] * 9)
    check(logits, us, temperature=[nan, -1.0, 0.0, 1e-45, 1e38, float("inf"), 1.0, 2.0, 3.0])
    check(logits, us, top_p=[nan, -1.0, 0.0, 1e-45, 1e-20, 1.0, 3.0, 1.0 - 2.0 ** -24, 0.5])
    check(logits, us, min_p=[nan, -1.0, 0.0, 1e-45, 1.0, 1.0001, 7.0, 0.5, 1e-3])
    check(logits, us, top_k=[-5, 0, 1, 2, 776, 777, 778, 1 << 30, -(1 << 31)])


def test_rows_apart_and_at_odd_addresses():
    """A slice of a wider tensor; logits that begin past a 16-byte boundary."""
    rng = np.random.default_rng(4)
    for dtype in ("bf16", "f32"):
        wide = torch.from_numpy(rng.standard_normal((13, 1031)).astype(np.float32)).cuda().to(DT[dtype])
        for first in range(9):
            check(wide[:, first:first + 1000], rng.random(13).tolist(), **draw_params(rng, 13))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [20000, 131073])
def test_largest_values_in_few_places(dtype, vocab):
    """The tokens that can be drawn lie side by side, at either end, or anywhere, also
    with equal ones and infinities among them; greedy rows take the first of equals."""
    rng = np.random.default_rng(vocab)
    l = rng.standard_normal((12, vocab)).astype(np.float32)
    l[1, 9000:9700] += 8.0
    l[2, :700] += 8.0
    l[3, -700:] += 8.0
    l[4, 11::64] += 8.0                                   # a few per lane, everywhere
    l[5, [vocab - 1, 12345, 12344, 77]] = 30.0            # equal ones
    l[6, [vocab - 2, 19000, 18999]] = np.inf
    l[7, 5000:5040] = np.inf
    l[8] = -np.inf
    l[8, vocab - 3] = -1e30
    l[9, ::2] = np.nan
    l[10, 100:] = -np.inf
    l[11, 600:] = l[11, 0]
    wide = torch.full((12, vocab + 3), 99.0, dtype=DT[dtype], device="cuda")
    wide[:, 1:vocab + 1] = torch.from_numpy(l).cuda().to(DT[dtype])
    logits = wide[:, 1:vocab + 1]
    u = rng.random(12).tolist()
    check(logits, u, temperature=[0.0] * 12)
    check(logits, u, min_p=[1.5] * 12)
    for k in (1, 2, 50, 511, 512, 513, 1024, 1025, 1536, 1537):
        check(logits, u, top_k=[k] * 12)
        check(logits, u, top_k=[k] * 12, temperature=[0.02, 0.1, 0.5] * 4)
    check(logits, u, top_k=[400] * 12, top_p=[0.9] * 12, min_p=[0.02] * 12)
    for m in (0.9, 0.05, 1e-3):
        check(logits, u, min_p=[m] * 12)
        check(logits, u, min_p=[m] * 12, top_p=[0.8] * 12)


def test_frequencies():
    """Tokens come as often as their weights say: u over a grid of 4096 places hits
    each token within one place of its share, for any rounding of the sums."""
    rng = np.random.default_rng(6)
    l = rng.standard_normal(50).astype(np.float32)
    n = 4096
    got = run(torch.from_numpy(l).cuda().repeat(n, 1), ((np.arange(n) + 0.5) / n).tolist(), top_k=[20] * n)
    keep = np.argsort(-l, kind="stable")[:20]
    w = np.zeros(50)
    w[keep] = np.exp(l[keep].astype(np.float64))
    assert (np.abs(np.bincount(got, minlength=50) - n * w / w.sum()) <= 1).all()


def test_in_a_hip_graph():
    """Parameters and random numbers are read when the graph is replayed."""
    rng = np.random.default_rng(7)
    rows, vocab = 12, 5000
    logits = torch.empty(rows, vocab, device="cuda")
    t = {k: torch.empty(rows, device="cuda", dtype=torch.int32 if k == "top_k" else torch.float32)
         for k in ("u", "temperature", "top_k", "top_p", "min_p")}
    logits.normal_()
    for x in t.values():
        x.fill_(1)
    s = Sampler(rows, vocab)
    s(logits, **t)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = s(logits, **t)
    for _ in range(3):
        logits.copy_(torch.from_numpy(rng.standard_normal((rows, vocab)).astype(np.float32) * 2))
        p = dict(draw_params(rng, rows), u=rng.random(rows).tolist())
        for k, x in t.items():
            x.copy_(torch.tensor(p[k], dtype=x.dtype))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert out.cpu().tolist() == run(logits, **p)
        check(logits, **p)
