"""Host checks of the adapters and of sampling on the CPU (fake addresses:
every call returns before any device work), the oracle of sampling against
closed forms, and the wrappers' refusals."""
import ctypes

import numpy as np
import pytest
import torch

from oracle.sampling import sample
from paper_2410_18701_amd import baton as B
from paper_2410_18701_amd.layer import Adapters

X, Y, W, A, BB = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000


def table(*entries):
    t = (B.baton_adapter * max(1, len(entries)))()
    for i, e in enumerate(entries):
        t[i] = B.baton_adapter(*e)
    return t


def adapters_status(dtype=B.BATON_BF16, x=X, tab=((A, BB, 16, 1.0),), n=None, ids=(0, -1), y=Y, rows=2, out_dim=64,
                    in_dim=128, parts=None, n_parts=1, accumulate=1, ws=W, ws_bytes=1 << 20):
    try:
        B.baton_linear_adapters(dtype, x, table(*tab), len(tab) if n is None else n, list(ids), y, rows, out_dim,
                                in_dim, parts, n_parts, accumulate, ws, ws_bytes)
    except B.BatonError as e:
        return e.status
    return B.BATON_OK


@pytest.mark.parametrize("kw", [
    dict(x=0), dict(x=X + 8), dict(y=0), dict(y=Y + 2), dict(out_dim=60), dict(out_dim=0), dict(in_dim=132),
    dict(in_dim=0), dict(ids=(1, -1)), dict(ids=(-2, 0)), dict(ids=(0, 1 << 30)), dict(n=-1), dict(accumulate=2),
    dict(tab=((0, BB, 16, 1.0),)), dict(tab=((A, 0, 16, 1.0),)), dict(tab=((A + 8, BB, 16, 1.0),)),
    dict(tab=((A, BB, 0, 1.0),)), dict(tab=((A, BB, 12, 1.0),)), dict(tab=((A, BB, 136, 1.0),)),
    dict(tab=((A, BB, 16, float("nan")),)), dict(tab=((A, BB, 16, float("inf")),)),
    dict(parts=[32, 24], n_parts=2), dict(parts=[60, 4], n_parts=2), dict(parts=[72, -8], n_parts=2),
    dict(n_parts=2), dict(n_parts=0), dict(parts=[16] * 5, n_parts=5, out_dim=80), dict(ws=0), dict(ws=W + 4),
    dict(ws_bytes=2 * 16 * 4 - 1), dict(rows=257, ids=[0] * 257), dict(rows=0, ids=()),
], ids=lambda kw: "-".join(kw))
def test_adapters_refusals(kw):
    assert adapters_status(**kw) == B.BATON_EINVAL


def test_adapters_other_statuses():
    assert adapters_status(dtype=B.BATON_F32) == B.BATON_EDTYPE
    assert adapters_status(ids=(-1, -1), ws=0, ws_bytes=0) == B.BATON_OK              # nothing to do
    # an entry no row names is not looked at
    assert adapters_status(tab=((A, BB, 16, 1.0), (0, 0, 5, float("nan"))), ids=(-1, -1)) == B.BATON_OK
    assert B.baton_linear_adapters_workspace_bytes(3, 2, 24) == 3 * 2 * 24 * 4
    assert B.baton_linear_adapters_workspace_bytes(0, 1, 8) == 0
    with pytest.raises(ValueError):
        B.baton_linear_adapters(B.BATON_BF16, X, table(), 0, [0], Y, 2, 64, 64, None, 1, 0, W, 1 << 20)


def test_adapters_wrapper_refusals():
    t = lambda *s, d=torch.bfloat16: torch.zeros(s, dtype=d)  # noqa: E731
    Adapters([t(16, 64), t(8, 64)], [t(32, 16), t(32, 8)], [1.0, 2.0])
    Adapters([t(32, 64)], [t(32, 16)], [1.0], parts=[8, 24])
    for bad in (lambda: Adapters([t(16, 64)], [t(32, 8)], [1.0]), lambda: Adapters([t(16, 64)], [], [1.0]),
                lambda: Adapters([t(16, 64, d=torch.float32)], [t(32, 16)], [1.0]),
                lambda: Adapters([t(64, 16).t()], [t(32, 16)], [1.0]),
                lambda: Adapters([t(32, 64)], [t(32, 16)], [1.0], parts=[8, 8]),
                lambda: Adapters([t(8, 64), t(8, 72)], [t(32, 8), t(32, 8)], [1.0, 1.0]),
                lambda: Adapters([t(16, 64)], [t(32, 16).to("meta")], [1.0]),
                lambda: Adapters([t(8, 64), t(8, 64).to("meta")], [t(32, 8), t(32, 8)], [1.0, 1.0])):
        with pytest.raises(ValueError):
            bad()


def test_adapters_too_small_a_workspace_is_named():
    """Before the call, by the largest rank that a row uses (nothing is allocated or enqueued)."""
    from paper_2410_18701_amd.layer import Gemm
    t = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    ad = Adapters([t(16, 64), t(48, 64)], [t(32, 8), t(32, 24)], [1.0, 1.0], parts=[8, 24])
    g, x, y = Gemm(0), t(3, 64), t(3, 32)
    g.ws_bytes = 4 * 3 * 2 * 24 - 1
    with pytest.raises(ValueError, match="rank 24 needs a workspace of 576 bytes, the Gemm has 575"):
        g.linear_adapters(x, ad, [0, 1, -1], y)
    with pytest.raises(Exception) as e:          # rank 8 alone fits: refused for the tensors' device, not the workspace
        g.linear_adapters(x, ad, [0, 0, -1], y)
    assert "workspace" not in str(e.value)


def sample_status(dtype=B.BATON_BF16, logits=X, ld=100, rows=4, vocab=100, temperature=0, top_k=0, top_p=0, min_p=0,
                  u=W, tokens=Y):
    try:
        B.baton_sample(dtype, logits, ld, rows, vocab, temperature, top_k, top_p, min_p, u, tokens)
    except B.BatonError as e:
        return e.status
    return B.BATON_OK


@pytest.mark.parametrize("kw", [
    dict(logits=0), dict(logits=X + 1), dict(dtype=B.BATON_F32, logits=X + 2), dict(ld=99), dict(rows=0), dict(rows=-1),
    dict(rows=(1 << 21) + 1),
    dict(vocab=0), dict(vocab=(1 << 24) + 1, ld=1 << 25), dict(u=0), dict(u=W + 2), dict(tokens=0), dict(tokens=Y + 1),
    dict(temperature=A + 2), dict(top_k=A + 1), dict(top_p=A + 3), dict(min_p=A + 2), dict(ld=(1 << 40) + 1),
], ids=lambda kw: "-".join(kw))
def test_sample_refusals(kw):
    assert sample_status(**kw) == B.BATON_EINVAL


def test_sample_dtype():
    assert sample_status(dtype=B.BATON_MXFP4) == B.BATON_EDTYPE
    assert sample_status(dtype=9) == B.BATON_EDTYPE


def test_sampling_oracle_closed_forms():
    l = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    assert [sample(l, u) for u in (0.0, 0.09, 0.11, 0.49, 0.51, 0.69, 0.71, 0.999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert [sample(l, u, top_k=2) for u in (0.0, 0.5, 0.58, 0.99)] == [1, 1, 3, 3]
    assert [sample(l, u, top_p=0.65) for u in (0.0, 0.56, 0.58)] == [1, 1, 3]      # 0.4 < 0.65 <= 0.7
    assert [sample(l, u, min_p=0.6) for u in (0.0, 0.56, 0.58)] == [1, 1, 3]       # 0.3 / 0.4
    assert sample(l, 0.99, temperature=0.0) == 1 and sample(l, 0.99, min_p=2.0) == 1 and sample(l, 0.5, top_p=0.0) == 1
    assert sample(np.zeros(10), 0.95, top_k=3) == 2                                 # ties: lowest indices
    assert sample(np.array([0.0, np.inf, 5.0, np.inf]), 0.6) == 3
    assert sample(np.array([-np.inf, np.nan]), 0.5) == -1
    # planted: a prefix one too long or too short is another token for some u
    us = np.linspace(0, 0.999, 200)
    right = [sample(l, u, top_k=3) for u in us]
    assert right != [sample(l, u, top_k=2) for u in us] and right != [sample(l, u, top_k=4) for u in us]


def test_structure_sizes():
    assert ctypes.sizeof(B.baton_adapter) == 24
