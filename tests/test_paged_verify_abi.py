"""Host checks of the verification of a paged cache's step on the CPU (fake addresses: refused
before any device work): those of the cache and those of the verification."""
import pytest

from paper_2410_18701_amd import baton as B
from tests.test_paged_abi import desc
from tests.test_verify_abi import W, X, Y, Z


def status(d=None, dtype=B.BATON_BF16, target=X, target_ld=100, draft=Y, draft_ld=100, width=3, vocab=100, drafted=Z,
           n_draft=Z, u_accept=Z, u_token=Z, tokens=Z, n_out=Z, ws=W, ws_bytes=1 << 20):
    try:
        B.baton_paged_verify(desc() if d is None else d, dtype, target, target_ld, draft, draft_ld, width, vocab, drafted,
                             n_draft, u_accept, u_token, 0, 0, 0, 0, tokens, n_out, ws, ws_bytes)
    except B.BatonError as e:
        return e.status
    return B.BATON_OK


@pytest.mark.parametrize("kw,want", [
    (dict(batch=0), B.BATON_EINVAL), (dict(batch=513), B.BATON_EINVAL), (dict(state=0), B.BATON_EINVAL),
    (dict(page=48), B.BATON_EINVAL), (dict(head_dim=96), B.BATON_EDTYPE)])
def test_descriptor_refusals(kw, want):
    assert status(desc(**kw)) == want


@pytest.mark.parametrize("kw", [
    dict(target=0), dict(target=X + 1), dict(target_ld=99), dict(draft_ld=99), dict(width=0), dict(width=17), dict(vocab=0),
    dict(drafted=0), dict(n_draft=Z + 1), dict(u_accept=0), dict(u_token=0), dict(tokens=0), dict(n_out=0), dict(ws=0),
    dict(ws=W + 8), dict(ws_bytes=64)], ids=lambda kw: "-".join(kw))
def test_refusals(kw):
    assert status(**kw) == B.BATON_EINVAL
    assert status(dtype=B.BATON_MXFP4) == B.BATON_EDTYPE
