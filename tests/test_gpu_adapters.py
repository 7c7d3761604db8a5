"""Low-rank adapters beside a shared projection on the GPU against float64.

Tolerance of an output, from the roundings alone: y is rounded once, at most
2^-8 of it; x . A^T is kept as two bf16 halves, 2^-16 of it; its fp32 sums, over
in_dim terms, and those over rank terms are off by at most 2^-24 of the sum of
magnitudes for each addition."""
import numpy as np
import pytest
import torch

from paper_2410_18701_amd import baton as B
from paper_2410_18701_amd.layer import Adapters, Gemm

pytestmark = pytest.mark.gpu


def val(t):
    return t.double().cpu().numpy()


def make(rng, rows, in_dim, part_dims, ranks):
    P, out = len(part_dims), sum(part_dims)
    t = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda().bfloat16()  # noqa: E731
    a = [t(P * r, in_dim) for r in ranks]
    b = [t(out, r) for r in ranks]
    scales = [float(np.float32(rng.uniform(-2, 2))) for _ in ranks]
    return t(rows, in_dim), a, b, scales, t(rows, out)


def want(x, a, b, scales, ids, part_dims, y0, accumulate):
    """(value, tolerance) of every output."""
    out = sum(part_dims)
    y = val(y0) if accumulate else np.zeros((len(ids), out))
    mag = np.zeros_like(y)
    x = val(x)
    for r, i in enumerate(ids):
        if i < 0:
            continue
        ai, bi, c = val(a[i]), val(b[i]), 0
        rank = bi.shape[1]
        for p, d in enumerate(part_dims):
            ap = ai[p * rank:(p + 1) * rank]
            y[r, c:c + d] += scales[i] * (bi[c:c + d] @ (ap @ x[r]))
            mag[r, c:c + d] = abs(scales[i]) * (np.abs(bi[c:c + d]) @ (np.abs(ap) @ np.abs(x[r])))
            c += d
    rank = max((t.shape[1] for t in b), default=0)
    return y, 2.0 ** -8 * np.abs(y) + (2.0 ** -16 + (x.shape[1] + 2 * rank + 128) * 2.0 ** -24) * mag + 1e-30


def check(rng, rows, in_dim, part_dims, ranks, ids, accumulate, ws_bytes=32 << 20):
    x, a, b, scales, y0 = make(rng, rows, in_dim, part_dims, ranks)
    y = y0.clone()
    g = Gemm(ws_bytes)
    ad = Adapters(a, b, scales, parts=part_dims)
    g.linear_adapters(x, ad, ids, y, accumulate=accumulate)
    o, tol = want(x, a, b, scales, ids, part_dims, y0, accumulate)
    err = np.abs(val(y) - o) / tol
    assert err.max() <= 1, f"{err.max():.3g} of the tolerance at {np.unravel_index(err.argmax(), err.shape)}"
    bare = [r for r, i in enumerate(ids) if i < 0]
    if bare:
        assert torch.equal(y[bare], y0[bare] if accumulate else torch.zeros_like(y0[bare]))
    again = y0.clone()
    g.linear_adapters(x, ad, ids, again, accumulate=accumulate)
    assert torch.equal(y, again)
    print(f"[adapters] rows {rows} in {in_dim} parts {part_dims} ranks {ranks[:4]}: {err.max():.3g} of the tolerance",
          flush=True)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("in_dim,part_dims", [(8, [8]), (40, [24]), (136, [16, 8, 40]), (1000, [1064]),
                                              (4096, [4096]), (4104, [520, 8, 264, 2000])])
@pytest.mark.parametrize("ranks", [[8], [16, 24], [64, 8, 128, 40]], ids=str)
def test_sizes(in_dim, part_dims, ranks, accumulate):
    rng = np.random.default_rng(in_dim + len(ranks))
    for rows in (1, 2, 17, 67):
        ids = [int(i) for i in rng.integers(-1, len(ranks), rows)]
        check(rng, rows, in_dim, part_dims, ranks, ids, accumulate)


@pytest.mark.parametrize("rows,n,ids", [
    (256, 1, "one"), (256, 200, "each"), (256, 256, "each"), (130, 97, "each"), (200, 3, "any"), (65, 2, "ends"),
    (64, 1, "one"), (16, 16, "each")])
def test_many_rows_and_adapters(rows, n, ids):
    """One adapter for all rows (several row blocks), one for each (several launches), and between."""
    rng = np.random.default_rng(rows * 1000 + n)
    ranks = [int(r) for r in rng.choice([8, 16, 32], n)]
    which = {"one": [0] * rows, "each": [int(i) for i in rng.permutation(max(n, rows))[:rows] % n],
             "any": [int(i) for i in rng.integers(-1, n, rows)],
             "ends": [-1] + [1] * (rows - 2) + [-1]}[ids]
    check(rng, rows, 264, [72, 200], ranks, which, accumulate=rows % 2 == 0)


@pytest.mark.parametrize("splits", [1, 2, 3, 7])
def test_workspaces(splits):
    """The smallest workspace and ones that let in_dim be divided."""
    rng = np.random.default_rng(splits)
    need = B.baton_linear_adapters_workspace_bytes(5, 2, 16)
    assert need == 5 * 2 * 16 * 4
    check(rng, 5, 4096, [64, 32], [16], [0, 0, -1, 0, 0], False, ws_bytes=need * splits)


def test_nothing_to_do():
    """No row with an adapter: zeros, or y untouched; no adapters at all."""
    x, y = torch.randn(3, 64, device="cuda").bfloat16(), torch.randn(3, 40, device="cuda").bfloat16()
    y0, g = y.clone(), Gemm()
    g.linear_adapters(x, Adapters([], [], []), [-1, -1, -1], y, accumulate=True)
    assert torch.equal(y, y0)
    g.linear_adapters(x, Adapters([], [], []), [-1, -1, -1], y)
    assert (y == 0).all()


def test_rows_do_not_mix_and_infinities_stay():
    """A row of infinities reaches its own outputs only; rows behind the last one are left as they were."""
    rng = np.random.default_rng(0)
    x, a, b, scales, y = make(rng, 21, 128, [48], [8, 16])
    x[4] = float("inf")
    x[9, 3] = float("nan")
    wide = torch.full((30, 48), 7.0, device="cuda", dtype=torch.bfloat16)
    ids = [i % 2 for i in range(21)]
    Gemm().linear_adapters(x, Adapters(a, b, scales), ids, wide[:21])
    bad = ~wide.isfinite().all(1)
    assert bad.nonzero().flatten().tolist() == [4, 9]
    assert (wide[21:] == 7.0).all()


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("rows,in_dim,part_dims,rank", [(3, 128, [48], 8), (20, 256, [40, 24], 24), (5, 136, [64], 40),
                                                        (70, 64, [32], 104)])
def test_infinities_of_b(rows, in_dim, part_dims, rank, accumulate):
    """An infinite element of B times a number other than 0 is an infinity of its sign, in its
    column alone; infinities of both signs, and an infinity times 0, are NaN."""
    rng = np.random.default_rng(rank)
    x, a, b, scales, y0 = make(rng, rows, in_dim, part_dims, [rank])
    inf = float("inf")
    b[0][1, 0], b[0][7, rank - 1], b[0][9, 3] = inf, -inf, inf
    b[0][12, 2], b[0][12, 5] = inf, -inf        # of one sign where the two products agree
    x[rows - 1] = 0.0
    scales[0] = -1.5
    y = y0.clone()
    Gemm().linear_adapters(x, Adapters(a, b, scales, parts=part_dims), [0] * rows, y, accumulate=accumulate)
    with np.errstate(invalid="ignore"):
        h, mag = val(x)[:-1] @ val(a[0]).T, np.abs(val(x)[:-1]) @ np.abs(val(a[0])).T
        assert (np.abs(h) > in_dim * 2.0 ** -24 * mag).all()   # fp32 sums have its sign
        o, tol = want(x, a, b, scales, [0] * rows, part_dims, y0, accumulate)
        got, finite = val(y), np.isfinite(o)
        assert np.array_equal(np.isnan(got), np.isnan(o))
        assert np.array_equal(got[np.isinf(o)], o[np.isinf(o)])
        assert (np.abs(got - o)[finite] <= tol[finite]).all()
    assert np.isinf(o).any() and np.isnan(o[:-1]).any() and np.isnan(o[-1]).sum() == 4


@pytest.mark.parametrize("rows", [16, 64])
@pytest.mark.parametrize("in_dim,rank", [(8, 8), (136, 16), (40, 104)])
def test_products_of_x_and_a_keep_fp32(rows, in_dim, rank):
    """x . A^T is held in fp32, not rounded below it: two rows of A, one 3 times the other,
    against columns b and -3 b of B sum to exactly 0, and what comes out instead is off by
    fp32's roundings alone.  All else of A, B is 0 and adds exactly, so those are 4 additions
    of x . A^T, the scale, the two that part it and 6 of the last sum, each at most 2^-23
    of the sum of magnitudes.  One rounding to 16 bits would be up to 2^-16 of a term."""
    out, rng = 512, np.random.default_rng(in_dim * rank)
    few = lambda *s: rng.integers(1, 32, s) * rng.choice([-1.0, 1.0], s) / 16.0  # noqa: E731  (5 bits, 3 times it 7)
    a, b = np.zeros((rank, in_dim)), np.zeros((out, rank))
    a[rank - 1, in_dim - 4:], b[:, rank - 2] = few(4), few(out)
    a[rank - 2], b[:, rank - 1] = 3 * a[rank - 1], -3 * b[:, rank - 2]
    t = lambda v: torch.from_numpy(v.astype(np.float32)).cuda().bfloat16()  # noqa: E731
    x, a, b = t(rng.standard_normal((rows, in_dim))), [t(a)], [t(b)]
    scales, y = [float(np.float32(1.37))], torch.empty(rows, out, device="cuda", dtype=torch.bfloat16)
    Gemm().linear_adapters(x, Adapters(a, b, scales), [0] * rows, y)
    mag = 1.37 * (np.abs(val(x)) @ np.abs(val(a[0])).T) @ np.abs(val(b[0])).T
    err = np.abs(val(y)) / (13 * 2.0 ** -23 * mag)
    print(f"[adapters] in {in_dim} rank {rank}: {err.max():.3g} of the tolerance", flush=True)
    assert err.max() <= 1


def test_beside_a_packed_projection_in_a_hip_graph():
    """The projection and its adapters captured and replayed, other work between the replays."""
    rng = np.random.default_rng(8)
    x, a, b, scales, _ = make(rng, 24, 512, [256, 128], [16, 32])
    g = Gemm()
    wp = g.pack((torch.randn(384, 512, device="cuda") / 16).bfloat16())
    ad = Adapters(a, b, scales, parts=[256, 128])
    ids = [i % 3 - 1 for i in range(24)]
    y, want_y = (torch.empty(24, 384, device="cuda", dtype=torch.bfloat16) for _ in range(2))

    def both(out):
        g.linear_packed(x, wp, out)
        g.linear_adapters(x, ad, ids, out, accumulate=True)
    both(want_y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(y)
    for _ in range(3):
        y.fill_(float("nan"))
        torch.randn(1 << 16, device="cuda").sum()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want_y)


def test_calls_follow_the_current_stream():
    rng = np.random.default_rng(9)
    x, a, b, scales, y = make(rng, 8, 256, [64], [16])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        Gemm().linear_adapters(x, Adapters(a, b, scales), [0] * 8, y)
        got = y.clone()
    torch.cuda.current_stream().wait_stream(side)
    o, tol = want(x, a, b, scales, [0] * 8, [64], y, False)
    assert (np.abs(val(got) - o) <= tol).all()


def test_a_workspace_elsewhere_is_refused():
    """A workspace that is not on the current device, as a Gemm made on another one has."""
    rng = np.random.default_rng(1)
    x, a, b, scales, y = make(rng, 4, 64, [32], [8])
    g = Gemm()
    g.ws = torch.empty(g.ws_bytes, dtype=torch.uint8)
    with pytest.raises(ValueError, match="current device"):
        g.linear_adapters(x, Adapters(a, b, scales), [0] * 4, y)
