"""What attention over a cache in pages keeps of its numbers: the softmax weights' bits,
fp32's, and what infinite scores give, against 64 bits."""
import numpy as np
import pytest
import torch

from oracle import paged as O
from paper_2410_18701_amd.paged import PagedCache

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
PATHS = [(1, 1), (5, 2), (16, 1), (16, 2), (16, 4)]      # width, query heads a kv-head: 1 to 64 rows


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().double().cpu().numpy()


def attend(k, v, q, k_new, v_new, dtype, scale=0.0, page=32):
    """One query: cached k, v [hkv][n][d], new ones [t][hkv][d], q [t][hq][d], all float64 arrays that
    the type holds -> (out, what 64 bits give), [t][hq][d]."""
    t, hq, d = q.shape
    hkv, n = k.shape[:2]
    dev = lambda x: torch.tensor(x, device="cuda").to(DT[dtype]).contiguous()  # noqa: E731
    c = PagedCache(1, 1, hq, hkv, d, 8 + (n + t) // page, 8 + (n + t) // page, page=page, width=t, dtype=dtype)
    c.kv.fill_(float("nan"))
    c.begin(i32([n]))
    c.embed([0], [n], [dev(k[None])], [dev(v[None])])
    c.begin(i32([t]), keep=i32([n]))
    out = c.decode_attn(0, dev(q[None]), dev(k_new[None]), dev(v_new[None]), scale=scale)
    with np.errstate(invalid="ignore"):
        want = O.attention(q, np.concatenate([k, k_new.transpose(1, 0, 2)], 1),
                           np.concatenate([v, v_new.transpose(1, 0, 2)], 1), n, scale=scale or None)
    return f64(out)[0], want


def bf16(x):
    return f64(torch.tensor(x).bfloat16())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [None, float("inf"), float("nan")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("width,group", PATHS)
def test_weights_keep_their_bits(width, group, d, bad, dtype):
    """Three tokens of weights 1, 1 and p = exp(-n / 16) whose values cancel but for their last bits:
    a weight's rounding is all that is left.  Scores are whole numbers.  Off by, in units of 2^-23:
    p < 1 times a value below 2 by 4 (the exponential 2^-23 of it, its argument 2^-24, the scale 2^-25
    of at most 1.2), the weights of 1 by 2, sums of numbers below 2 in at most three products 6; all
    that over a sum of weights of at least 2: 6 2^-23 < 2^-20.  (A weight of 16 bits is off by up to
    2^-18 of itself, here 2^-18.8.)  An infinite or NaN value in one column takes nothing from the others."""
    rng = np.random.default_rng(width + group)
    ns = (1, 2, 3, 5, 7, 9, 11, 13)
    hkv = len(ns)
    qh, k_a = rng.integers(-2, 3, (hkv, d)).astype(float), rng.integers(-2, 3, (hkv, d)).astype(float)
    qh[:, 0] = 1
    k = np.repeat(k_a[:, None], 3, 1)
    k[:, 1, 0] -= ns
    p = np.exp(-np.array(ns) / 16)[:, None]
    v_b = bf16(rng.uniform(1, 2, (hkv, d)) * rng.choice([-1, 1], (hkv, d)))
    v_a = -bf16(p * v_b)
    v = np.stack([v_a, v_b, -bf16(p * v_b + v_a)], 1)
    if bad is not None:
        v[:, 1, 5] = bad
    q = np.broadcast_to(np.repeat(qh, group, 0), (width, hkv * group, d))
    k_new = np.broadcast_to(-100 * np.sign(qh), (width, hkv, d))          # scores below -3000: no weight
    out, want = attend(k, v, q, k_new, np.broadcast_to(v_b, (width, hkv, d)), dtype, scale=1 / 16)
    if bad is not None:
        assert np.array_equal(out[..., 5], want[..., 5], equal_nan=True)
        out, want = np.delete(out, 5, 2), np.delete(want, 5, 2)
    err = np.abs(out - want) - (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0.0)
    assert err.max() <= 2.0 ** -20, err.max()


def normal(rng, dtype, *shape):
    x = rng.normal(size=shape)
    return bf16(x) if dtype == "bf16" else x.astype(np.float32).astype(np.float64)


def close(out, want, vmax, dtype):
    """As the other tests of this attention: 2^-12 of the largest value, bf16 half a step more."""
    assert np.array_equal(np.isnan(out), np.isnan(want))
    err = np.where(np.isnan(want), 0.0, np.abs(out - want)) - 2.0 ** -12 * vmax
    assert (err <= (2.0 ** -8 * np.abs(np.nan_to_num(want)) if dtype == "bf16" else 0.0)).all()


LENS_AND_PATHS = [(41, p) for p in PATHS] + [(9000, PATHS[0]), (9000, PATHS[3])]      # 9,000: several work items
SCALES = [(64, 0.0), (128, 0.0), (64, -0.2), (128, -0.3)]


def with_infinities(n, width, group, d, scale, dtype, keys, new_keys):
    """Query, keys and values of four kv-heads; keys(k, low), new_keys(k_new, low) put `low`, which gives a
    score of -inf, into some keys."""
    rng = np.random.default_rng(d + width)
    low = float("-inf") if scale >= 0 else float("inf")
    q, k, v = (normal(rng, dtype, *s) for s in ((width, 4 * group, d), (4, n, d), (4, n, d)))
    k_new, v_new = (normal(rng, dtype, width, 4, d) for _ in range(2))
    q[..., 0] = 1
    keys(k[..., 0], low)
    new_keys(k_new[..., 0], low)
    return attend(k, v, q, k_new, v_new, dtype, scale=scale) + (np.abs(v).max(),)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,scale", SCALES)
@pytest.mark.parametrize("n,path", LENS_AND_PATHS)
def test_scores_of_minus_infinity(n, path, d, scale, dtype):
    """Weight 0 where the score is -inf, as the formula has it: every second token of kv-head 0, all but one of
    kv-head 1, new ones of kv-head 2; a score of +inf in kv-head 3 is NaN."""
    def keys(k, low):
        k[0, ::2] = k[1, :-1] = low
        k[3, 5] = -low

    def new_keys(k, low):
        k[:, 1:3] = low

    out, want, vmax = with_infinities(n, *path, d, scale, dtype, keys, new_keys)
    assert np.isnan(want).sum() == want.size / 4
    close(out, want, vmax, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,scale", SCALES)
@pytest.mark.parametrize("n,path", LENS_AND_PATHS)
def test_rows_of_minus_infinity_alone(n, path, d, scale, dtype):
    """Where every score is -inf there is nothing to divide by: NaN, as the formula has it.  kv-head 0: all
    tokens; 1: all but the first; 2: all but the new ones; 3: the new ones."""
    def keys(k, low):
        k[0] = k[2] = k[1, 1:] = low

    def new_keys(k, low):
        k[:, [0, 1, 3]] = low

    out, want, vmax = with_infinities(n, *path, d, scale, dtype, keys, new_keys)
    assert np.isnan(want).sum() == want.size / 4
    close(out, want, vmax, dtype)


@pytest.mark.parametrize("n", [3, 700, 9000])
@pytest.mark.parametrize("width,group", PATHS)
@pytest.mark.parametrize("d", [64, 128])
def test_fp32_errors(d, width, group, n):
    """The size of fp32's own errors, for normal numbers and d = 128.  A score is four sums of 32 products whose
    partial sums are about 4: each addition is off by 0.29 2^-21, 80 of them by 1.3e-6, times d^-1/2 1.1e-7.
    Its distance to the maximum, up to 8, is rounded to 0.29 2^-21 (ln 2 of that in the exponential: 1.0e-7), the
    exponential to some 2^-24.  Together 1.7e-7 of each weight, so of the outputs in the mean: below 2^-21.
    Single ones, where few tokens weigh, below eight times that of the largest value."""
    rng = np.random.default_rng(n + d + width)
    q, k, v = (normal(rng, "f32", *s) for s in ((width, 2 * group, d), (2, n, d), (2, n, d)))
    k_new, v_new = (normal(rng, "f32", width, 2, d) for _ in range(2))
    out, want = attend(k, v, q, k_new, v_new, "f32")
    err = out - want
    assert np.abs(err).max() <= 2.0 ** -18 * np.abs(v).max()
    assert np.sqrt((err ** 2).mean() / (want ** 2).mean()) <= 2.0 ** -21
