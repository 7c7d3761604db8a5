"""The 4-bit form on the CPU: its definition against closed forms, the unpacking
of stored bytes, and the host checks of a 4-bit cache (nothing is enqueued)."""
import numpy as np
import pytest
import torch

from oracle import mxfp4 as X
from paper_2410_18701_amd import baton as B
from paper_2410_18701_amd.cache import row_bytes_mxfp4, unpack_mxfp4

FAKE_K, FAKE_V = 0x10000, 0x10000000


def block(*head):
    x = np.zeros(32)
    x[:len(head)] = head
    return x


def test_closed_forms():
    assert X.stored(block(6, 5, -5, 3.5, 2.5, 0.25, 0.75)).tolist()[:7] == [6, 4, -4, 4, 2, 0, 1]
    assert X.stored(block(7, 5)).tolist()[:2] == [6, 4]             # 7 is still within half a step of 6
    assert X.stored(block(7.03125, 1)).tolist()[:2] == [8, 1]       # past it the scale doubles
    assert X.stored(block()).tolist() == [0.0] * 32
    assert np.isnan(X.stored(block(np.inf, 1.0))).all()
    assert X.stored(block(1e-38)).tolist()[0] == pytest.approx(1e-38, rel=0.5)
    assert X.stored(block(3.3e38)).tolist()[0] == 6 * 2.0 ** 125


def test_half_a_step_and_idempotence():
    rng = np.random.default_rng(0)
    x = X.round_bf16(rng.standard_normal((4096, 32)) * np.exp2(rng.integers(-30, 30, (4096, 1))))
    y = X.stored(x)
    assert np.array_equal(X.stored(y), y)
    # In units of the scale an element t is off by at most half the step at t: 1 from 4 on (at t = 5, 7), 1/2 from
    # 2 on (t = 2.5, 3.5), 1/4 below.  The largest magnitude is over 3.5 and at least t, so relative to it that
    # is at most 1/5 (t = 5), 1/7 (t = 3.5) or 1/14.
    assert (np.abs(x - y) <= np.abs(x).max(1, keepdims=True) / 5).all()


def test_planted_mistakes_are_seen():
    """Other roundings and scales differ from the definition on ordinary data."""
    x = X.round_bf16(np.random.default_rng(1).standard_normal((512, 32)))
    y = X.stored(x)
    a = np.abs(x).max(1, keepdims=True)
    floor = 2.0 ** (np.floor(np.log2(a)) - 2)                        # the scale without the 7 / 8 rule
    t = np.abs(x) / floor
    z = np.sign(x) * X.GRID[np.abs(t[..., None] - X.GRID).argmin(-1)] * floor
    assert not np.array_equal(y, z)


@pytest.mark.parametrize("d", [64, 128])
def test_unpack(d):
    rng = np.random.default_rng(d)
    cap = 16
    raw = rng.integers(0, 256, (2, row_bytes_mxfp4(cap, d)), dtype=np.uint8)
    scales = raw[:, cap * d // 2:]
    scales[:] = rng.integers(2, 253, scales.shape)
    scales[0, 3] = 255
    got = unpack_mxfp4(torch.from_numpy(raw), cap, d).double().numpy()
    for r in range(2):
        for t in range(cap):
            for e in range(d):
                byte = raw[r, t * d // 2 + e // 2]
                c = byte >> 4 if e % 2 else byte & 15
                s = int(raw[r, cap * d // 2 + t * d // 32 + e // 32])
                want = np.nan if s == 255 else (-1) ** int(c > 7) * X.GRID[c & 7] * 2.0 ** (s - 127)
                assert got[r, t, e] == want or (np.isnan(want) and np.isnan(got[r, t, e]))


def desc(**kw):
    f = dict(dtype=B.BATON_MXFP4, n_layers=2, batch=4, n_q_heads=8, n_kv_heads=2, head_dim=128, capacity=304,
             k=FAKE_K, v=FAKE_V, fill_bits=B.BATON_FILL_NAN_MXFP4)
    f.update(kw)
    return B.baton_cache_desc(**f)


LAYER = 4 * 2 * 304 * 68   # bytes of a layer's rows


@pytest.mark.parametrize("kw,status", [
    (dict(capacity=300), B.BATON_EINVAL), (dict(capacity=8), B.BATON_EINVAL), (dict(head_dim=96), B.BATON_EDTYPE),
    (dict(dtype=3), B.BATON_EDTYPE), (dict(n_q_heads=6, n_kv_heads=4), B.BATON_EDTYPE),
    (dict(layer_stride=LAYER - 16), B.BATON_EINVAL), (dict(layer_stride=LAYER + 8), B.BATON_EINVAL),
    (dict(v=FAKE_K + LAYER), B.BATON_EINVAL), (dict(v=FAKE_K + LAYER, layer_stride=2 * LAYER - 16), B.BATON_EINVAL),
    (dict(capacity=1 << 25, head_dim=128), B.BATON_EINVAL), (dict(v=FAKE_V + 8), B.BATON_EINVAL),
])
def test_create_rejects(kw, status):
    with pytest.raises(B.BatonError) as e:
        B.baton_cache_create(desc(**kw), B.BATON_CREATE_ASSUME_FILLED)
    assert e.value.status == status


@pytest.mark.parametrize("kw", [dict(), dict(head_dim=64), dict(v=FAKE_K + LAYER, layer_stride=2 * LAYER),
                                dict(v=FAKE_K + 2 * LAYER), dict(capacity=16)])
def test_create_accepts(kw):
    h = B.baton_cache_create(desc(**kw), B.BATON_CREATE_ASSUME_FILLED)
    with pytest.raises(B.BatonError) as e:
        B.baton_kv_embed(h, [0], [304], [FAKE_K], [FAKE_V])
    assert e.value.status == B.BATON_ECAPACITY
    B.baton_cache_destroy(h)
