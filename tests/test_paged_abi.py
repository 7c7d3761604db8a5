"""Host checks of the cache in pages on the CPU (fake addresses: every call
returns before any device work), the wrapper's refusals, and its oracle
against closed forms."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import paged as O
from paper_2410_18701_amd import baton as B
from paper_2410_18701_amd.paged import PagedCache

K, V, T, L, S = 0x1000000, 0x9000000, 0x100000, 0x110000, 0x120000   # never dereferenced
Q, O_, W, M = 0x200000, 0x210000, 0x220000, 0x230000


def desc(**kw):
    d = dict(dtype=B.BATON_BF16, n_layers=2, batch=4, n_q_heads=8, n_kv_heads=2, head_dim=128, page=64, n_pages=100,
             max_pages=40, window=0, sinks=0, k=K, v=V, layer_stride=0, table=T, lens=L, state=S)
    d.update(kw)
    return B.baton_paged_desc(**d)


def status(call, *args):
    try:
        call(*args)
    except B.BatonError as e:
        return e.status
    return B.BATON_OK


LAYER = 100 * 64 * 2 * 128    # elements


@pytest.mark.parametrize("kw,want", [
    (dict(n_layers=0), B.BATON_EINVAL), (dict(batch=0), B.BATON_EINVAL), (dict(batch=513), B.BATON_EINVAL),
    (dict(page=16), B.BATON_EINVAL), (dict(page=96), B.BATON_EINVAL), (dict(page=512), B.BATON_EINVAL),
    (dict(n_pages=0), B.BATON_EINVAL), (dict(n_pages=1 << 25), B.BATON_EINVAL), (dict(max_pages=0), B.BATON_EINVAL),
    (dict(max_pages=(1 << 20) + 1), B.BATON_EINVAL), (dict(window=-1), B.BATON_EINVAL), (dict(sinks=-1), B.BATON_EINVAL),
    (dict(k=0), B.BATON_EINVAL), (dict(v=0), B.BATON_EINVAL), (dict(table=0), B.BATON_EINVAL),
    (dict(lens=0), B.BATON_EINVAL), (dict(state=0), B.BATON_EINVAL), (dict(k=K + 8), B.BATON_EINVAL),
    (dict(table=T + 2), B.BATON_EINVAL), (dict(lens=L + 1), B.BATON_EINVAL), (dict(state=S + 4), B.BATON_EINVAL),
    (dict(v=K), B.BATON_EINVAL), (dict(v=K + LAYER), B.BATON_EINVAL), (dict(layer_stride=LAYER - 8), B.BATON_EINVAL),
    (dict(layer_stride=-LAYER), B.BATON_EINVAL), (dict(layer_stride=LAYER + 4), B.BATON_EINVAL),
    (dict(layer_stride=2 * LAYER - 8, v=K + 2 * LAYER), B.BATON_EINVAL), (dict(layer_stride=1 << 60), B.BATON_EINVAL),
    (dict(dtype=B.BATON_MXFP4), B.BATON_EDTYPE), (dict(head_dim=96), B.BATON_EDTYPE),
    (dict(n_q_heads=6, n_kv_heads=4), B.BATON_EDTYPE), (dict(n_q_heads=32), B.BATON_EDTYPE),
], ids=lambda x: "-".join(x) if isinstance(x, dict) else str(x))
def test_descriptor_refusals(kw, want):
    """By every call alike."""
    d = desc(**kw)
    assert status(B.baton_paged_reset, d) == want
    assert status(B.baton_paged_step, d, 0, M) == want
    assert status(B.baton_paged_embed, d, [], [], [], []) == want
    assert status(B.baton_paged_extract, d, [], [], [], []) == want
    assert status(B.baton_paged_rope_qkv, d, Q, 1, Q, Q, Q, 1e4) == want
    assert status(B.baton_paged_attn, d, 0, Q, 0, 0, 1, O_, 0.0, W, 1 << 40) == want


def test_sizes():
    d = desc()
    assert status(B.baton_paged_embed, d, [], [], [], []) == B.BATON_OK       # nothing to do
    interleaved = desc(v=K + 2 * LAYER, layer_stride=2 * LAYER)
    assert status(B.baton_paged_embed, interleaved, [], [], [], []) == B.BATON_OK
    assert B.baton_paged_state_bytes(d) >= 4 * (100 + 4 * 4)
    assert B.baton_paged_state_bytes(desc(page=48)) == 0
    assert B.baton_paged_attn_workspace_bytes(d, 1) > 0
    assert B.baton_paged_attn_workspace_bytes(d, 17) == 0
    assert B.baton_paged_attn_workspace_bytes(desc(n_q_heads=16), 9) == 0
    assert B.baton_paged_attn_workspace_bytes(desc(max_pages=1), 1) == 0      # nothing to divide
    assert ctypes.sizeof(B.baton_paged_desc) == 96


@pytest.mark.parametrize("args", [
    (0, 0), (0, M + 2), (M + 1, M), (0, M, M + 2, 1, 1), (0, M, M, 0, 1), (0, M, M, 2, 1), (0, M, M, (1 << 20) + 1, 1 << 21),
    (0, M, 0, 1, 1, M + 1)])
def test_step_refusals(args):
    assert status(B.baton_paged_step, desc(), *args) == B.BATON_EINVAL


@pytest.mark.parametrize("slots,lens,k,v", [
    ([0, 0], [5, 5], [Q, Q], [Q, Q]), ([4], [5], [Q], [Q]), ([-1], [5], [Q], [Q]), ([0], [0], [Q], [Q]),
    ([0], [40 * 64 + 1], [Q], [Q]), ([0], [5], [0], [Q]), ([0], [5], [Q], [Q + 8])])
def test_copy_refusals(slots, lens, k, v):
    assert status(B.baton_paged_embed, desc(), slots, lens, k, v) == B.BATON_EINVAL
    assert status(B.baton_paged_extract, desc(), slots, lens, k, v) == B.BATON_EINVAL


def attn(d=None, layer=0, q=Q, k=Q, v=Q, width=1, out=O_, scale=0.0, ws=W, ws_bytes=1 << 30):
    return status(B.baton_paged_attn, desc() if d is None else d, layer, q, k, v, width, out, scale, ws, ws_bytes)


@pytest.mark.parametrize("kw", [
    dict(layer=2), dict(layer=-1), dict(q=0), dict(out=0), dict(k=0), dict(v=0), dict(q=Q + 8), dict(k=Q + 2),
    dict(v=Q + 4), dict(out=O_ + 8), dict(width=0), dict(width=17), dict(d=desc(n_q_heads=16), width=9),
    dict(d=desc(batch=512, n_q_heads=1 << 16, n_kv_heads=1 << 16, n_pages=1, layer_stride=0, v=1 << 40), ws_bytes=1 << 60),
    dict(scale=float("inf")), dict(scale=float("nan")), dict(ws=0), dict(ws=W + 8), dict(ws_bytes=16)],
    ids=lambda kw: "-".join(kw))
def test_attention_refusals(kw):
    assert attn(**kw) == B.BATON_EINVAL


@pytest.mark.parametrize("args,want", [
    ((0, 1, Q, Q, Q, 1e4), B.BATON_EINVAL), ((Q, 0, Q, Q, Q, 1e4), B.BATON_EINVAL), ((Q, 17, Q, Q, Q, 1e4), B.BATON_EINVAL),
    ((Q, 1, 0, Q, Q, 1e4), B.BATON_EINVAL), ((Q, 1, Q, Q, Q + 1, 1e4), B.BATON_EINVAL), ((Q, 1, Q, Q, Q, 1.0), B.BATON_EINVAL)])
def test_rope_refusals(args, want):
    assert status(B.baton_paged_rope_qkv, desc(), *args) == want
    assert status(B.baton_paged_rope_qkv, desc(dtype=B.BATON_F32), Q, 1, Q, Q, Q, 1e4) == B.BATON_EDTYPE


@pytest.mark.parametrize("kw", [dict(page=48), dict(dtype="mxfp4"), dict(width=17), dict(n_q_heads=16, width=9),
                                dict(batch=513), dict(head_dim=96)], ids=lambda kw: "-".join(kw))
def test_wrapper_refusals(kw):
    d = dict(n_layers=1, batch=2, n_q_heads=2, n_kv_heads=2, head_dim=64, n_pages=4, max_pages=2, device="cpu")
    with pytest.raises(ValueError):
        PagedCache(**{**d, **kw})


def test_oracle_tables():
    t = O.Tables(3, 8, 4, 32, order=[5, 3, 7, 0, 1, 2, 4, 6])
    assert t.step([33, 0, 32], width=2) == ([[5 * 32, 5 * 32 + 1], [-1, -1], [7 * 32, 7 * 32 + 1]], [0, 0, 0])
    assert [r[:2] for r in t.table] == [[5, 3], [-1, -1], [7, -1]]
    t.step([0, 0, 0], keep=[1, 0, 32])           # one of 33 stays: its second page goes back
    assert t.lens == [1, 0, 32] and t.stack[-1] == 3 and len(t.stack) == 6
    m, short = t.step([1, 500, 1], keep=[0, 0, 0])   # more than its table: nothing, the others all the same
    assert short == [0, 16, 0] and m == [[5 * 32 + 1], [-1], [3 * 32]]
    m, short = t.step([128, 100, 10], keep=[1, 0, -1])
    assert t.lens == [2, 0, 0]                    # 130 tokens: 5 pages, more than its table
    assert short == [4, 0, 0] and m[2] == [t.table[2][0] * 32]
    t.step([0, 0, 0], keep=[-1, -1, -1])
    assert sorted(t.stack) == list(range(8)) and all(x == -1 for r in t.table for x in r)


def test_oracle_tables_a_full_pool():
    t = O.Tables(4, 4, 4, 32)
    m, short = t.step([64, 96, 1, 0])
    assert short == [0, 3, 1, 0] and m[2] == [-1]     # need in front counts, granted or not
    assert t.n_new == [64, 0, 0, 0]


def test_oracle_window():
    t = O.Tables(1, 20, 10, 32, window=40, sinks=3)
    t.step([300])
    t.step([1], keep=[300])
    # from token 261 on: blocks 1 .. 7 hold none the window shows, block 0 holds the first tokens
    assert [x >= 0 for x in t.table[0]] == [True] + [False] * 7 + [True] * 2
    assert O.visible(300, 301, 40, 3).sum() == 43 and O.visible(2, 3, 1, 0).sum() == 1
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(1, 2, 4)), rng.normal(size=(1, 1, 4)), rng.normal(size=(1, 1, 4))
    assert np.allclose(O.attention(q, k, v, 0), np.broadcast_to(v[0, 0], (1, 2, 4)))   # one token
    k, v = np.zeros((1, 9, 4)), rng.normal(size=(1, 9, 4))
    assert np.allclose(O.attention(q, k, v, 8, window=2, sinks=1), v[0, [0, 7, 8]].mean(0))
    assert not np.allclose(O.attention(q, k, v, 8, window=3, sinks=1), v[0, [0, 7, 8]].mean(0))   # planted
