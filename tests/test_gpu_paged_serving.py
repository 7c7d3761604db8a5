"""Steps with drafted tokens as they would be served: DecodeLayers over a cache in
pages, drafts verified on the GPU, what was accepted kept by the next step, queries
that leave and arrive between steps.  Layers and attention against 64 bits on the GPU's
own inputs, as the other serving tests do (attention within what tests of it alone
allow); whole numbers against the oracles."""
import numpy as np
import pytest
import torch

from oracle import paged as O
from oracle.verify import verify
from paper_2410_18701_amd.cache import BatonCache
from paper_2410_18701_amd.layer import DecodeLayers, Gemm
from paper_2410_18701_amd.paged import PagedCache
from tests.test_gpu_serving import Model, check_layer, val

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prompts(m, lens):
    """Keys and values of prefilled queries, [layers][hkv][len][d]."""
    return [m.rand(m.LAYERS, m.HKV, n, m.D) for n in lens], [m.rand(m.LAYERS, m.HKV, n, m.D) for n in lens]


def paged(m, batch, width, page=32, window=0, sinks=0, n_pages=60):
    return PagedCache(m.LAYERS, batch, m.HQ, m.HKV, m.D, n_pages, 20, page=page, width=width, window=window, sinks=sinks)


def arrive(c, lens, ks, vs):
    c.begin(i32(lens + [0] * (c.batch - len(lens))))
    c.embed(list(range(len(lens))), lens, ks, vs)


def one_layer(layers, l, x):
    """Layer l on stream x (in place), and what went through it, as float64."""
    layers.layer(l, x)
    return dict({n: val(getattr(layers, n)) for n in ("q", "k", "v", "att")}, x=val(x))


def test_as_over_the_aligned_cache():
    """Queries, keys and values bit for bit; attention within both kernels' roundings: each
    output's (2^-8 of it), the aligned cache's softmax weights in bf16 (2^-8 of the mean of
    |v|) and fp32's (2^-12 of the largest)."""
    m, lens = Model(1, 2), [40, 1, 133]
    ks, vs = prompts(m, lens)
    ring = BatonCache(m.LAYERS, 4, m.HQ, m.HKV, m.D, 400)
    ring.embed([0, 1, 2], lens, ks, vs)
    c = paged(m, 4, 1)
    arrive(c, lens, ks, vs)
    a, b = (DecodeLayers(x, m.weights, Gemm(), adapters=m.adapters, head=m.head) for x in (ring, c))
    a.slot_adapter = b.slot_adapter = [1, -1, 0, -1]
    keep = i32(lens + [0])
    for step in range(4):
        x = m.rand(4, m.HID)
        c.begin(i32([1, 1, 1, 0]), keep=keep)
        keep = i32([1, 1, 1, 0])
        for l in range(m.LAYERS):           # from the same stream
            y = x.clone()
            a._normed = b._normed = None
            got, want = one_layer(b, l, y), one_layer(a, l, x)
            for n in ("q", "k", "v"):
                assert np.array_equal(got[n][:3], want[n][:3]), (step, l, n)
            err = np.abs(got["att"] - want["att"])[:3]
            vmax = max(float(t.abs().max()) for t in vs) + np.abs(want["v"]).max()
            assert (err <= 2 * 2.0 ** -8 * np.abs(want["att"][:3]) + (2.0 ** -8 + 2.0 ** -12) * vmax).all()
        ring.advance()
        u = torch.full((4,), 0.37, device="cuda")
        assert torch.equal(b.next_tokens(x, u)[:3], a.next_tokens(x, u)[:3])


@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 3)])
def test_drafts(window, sinks):
    """Twelve steps of up to three drafts, adapters beside the projections; one query leaves and another takes its slot.  The
    tables follow the oracle's with the GPU's own n_out as keep, tokens the oracle's verification
    of the GPU's own logits."""
    m, width, batch = Model(3, 2), 4, 4
    g = torch.Generator(device="cuda").manual_seed(3)
    lens = [50, 7, 180, 0]
    ks, vs = prompts(m, lens[:3])
    c = paged(m, batch, width, window=window, sinks=sinks)
    arrive(c, lens[:3], ks, vs)
    t = O.Tables(batch, 60, 20, 32, window, sinks)
    t.step(lens, width=width)
    layers = DecodeLayers(c, m.weights, Gemm(), adapters=m.adapters, head=m.head)
    layers.slot_adapter = [0, 1, -1, 0]
    emb = m.rand(m.VOCAB, m.HID)
    params = [dict(temperature=0.7), dict(top_p=0.9), dict(temperature=0.0), dict(top_k=20)]
    par = dict(temperature=torch.tensor([0.7, 1.0, 0.0, 1.0], device="cuda"), top_k=i32([0, 0, 0, 20]),
               top_p=torch.tensor([1.0, 0.9, 1.0, 1.0], device="cuda"))
    f32 = [{k: v if k == "top_k" else float(np.float32(v)) for k, v in p.items()} for p in params]
    last = torch.randint(0, m.VOCAB, (batch,), generator=g, device="cuda").int()
    keep, expected, accepted = i32(lens), [50, 7, 180, 0], 0
    held = [[[val(t[b])[l] if b < 3 else np.zeros((m.HKV, 0, m.D)) for l in range(m.LAYERS)] for t in (ks, vs)]
            for b in range(batch)]          # keys and values of each slot and layer
    for step in range(12):
        n_draft = [int(x) for x in torch.randint(0, width, (batch,), generator=g, device="cuda").tolist()]
        live = [0, 1, 2] if step < 6 else [0, 2, 3]
        n_draft = [n_draft[b] if b in live else -1 for b in range(batch)]
        if step == 6:                       # slot 1 leaves, a query of 33 tokens comes into slot 3
            k = keep.clone()
            k[1] = -1
            c.begin(i32([0, 0, 0, 33]), keep=k)
            t.step([0, 0, 0, 33], k.tolist(), width)
            expected[1], expected[3] = 0, 0
            ks, vs = prompts(m, [33])
            c.embed([3], [33], ks, vs)
            keep, expected[3] = i32([0, 0, 0, 33]), 33
            held[3] = [[val(t[0])[l] for l in range(m.LAYERS)] for t in (ks, vs)]
        # the target's own logits of the last step, changed a little, stand for a draft model
        draft = torch.randn((batch, width - 1, m.VOCAB), generator=g, device="cuda").mul(3).bfloat16()
        drafted = torch.randint(0, m.VOCAB, (batch, width - 1), generator=g, device="cuda").int()
        n_new = i32([n + 1 for n in n_draft])
        places = c.begin(n_new, keep=keep)
        want_places, missing = t.step(n_new.tolist(), keep.tolist(), width)
        assert places.tolist() == want_places and missing == [0] * batch
        assert c.lens.tolist() == t.lens == expected and c.table.tolist() == t.table
        x = emb[torch.cat([last[:, None], drafted], 1).long()].view(batch * width, -1)
        u = torch.rand(batch, width, generator=g, device="cuda")
        ua = (u[:, 1:] * (0.0 if step % 3 == 0 else 1e-3)).contiguous()      # so that some are accepted
        x = x.clone()
        pos = np.add.outer(expected, np.arange(width)).reshape(-1)
        rows = [b * width + i for b in live for i in range(n_draft[b] + 1)]
        for l in range(m.LAYERS):
            x0 = val(x)
            got = one_layer(layers, l, x)
            check_layer(m, l, x0, [i for i in layers.slot_adapter for _ in range(width)], pos, got, rows)
            for b in live:
                n, at = n_draft[b] + 1, expected[b]
                for j, name in enumerate("kv"):
                    new = got[name].reshape(batch, width, m.HKV, m.D)[b, :n].transpose(1, 0, 2)
                    held[b][j][l] = np.concatenate([held[b][j][l][:, :at], new], 1)
                k, v = held[b][0][l], held[b][1][l]
                q, o = (got[s].reshape(batch, width, m.HQ, m.D)[b, :n] for s in ("q", "att"))
                want = O.attention(q, k, v, at, window, sinks)
                assert (np.abs(o - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -12 * np.abs(v).max()).all(), (step, l, b)
        tokens, n_out = layers.accept_drafts(x, draft, drafted, i32(n_draft), ua, u[:, 0].contiguous(), **par)
        logits = val(layers.logits).reshape(batch, width, -1)
        for b in range(batch):
            want = verify(logits[b], val(draft[b]), drafted[b].tolist(), n_draft[b], ua[b].tolist(), float(u[b, 0]), **f32[b]) \
                if b in live else ([-1] * width, 0)
            assert (tokens[b].tolist(), int(n_out[b])) == want, (step, b)
        keep = n_out.clone()
        accepted += int((n_out - 1).clamp(min=0).sum())
        expected = [n + int(k) for n, k in zip(expected, keep.tolist())]
        last = tokens.gather(1, (n_out - 1).clamp(min=0).long()[:, None])[:, 0].clamp(min=0)
    assert accepted > 3


def test_refusals():
    m = Model(4, 0)
    c = paged(m, 4, 4)
    layers = DecodeLayers(c, m.weights, Gemm(), head=m.head)
    with pytest.raises(ValueError):
        layers.next_tokens(m.rand(16, m.HID), torch.zeros(16, device="cuda"))
    with pytest.raises(ValueError):
        DecodeLayers(PagedCache(1, 65, 4, 2, 64, 4, 2, width=4), m.weights, Gemm())
    ring = DecodeLayers(BatonCache(m.LAYERS, 2, m.HQ, m.HKV, m.D, 64), m.weights, Gemm(), head=m.head)
    with pytest.raises(ValueError):
        ring.accept_drafts(m.rand(2, m.HID), None, None, None, None, None)
