"""Decode steps of a batch whose queries differ, as they would be served: a cache
held in 4 bits, an adapter per slot beside every projection, the next token by
each slot's own parameters, slots evicted and refilled between the steps.
Every layer against the oracles on the GPU's own inputs: what is stored in bf16
between operations is rounded at the same places, so an element is off by the
roundings that fall the other way, the whole-layer bound of the other layer
tests (2^-5 relative, 2e-2); tokens are the same."""
import numpy as np
import pytest
import torch

import oracle.llama_layer as LL
from oracle import mxfp4 as X
from oracle.sampling import sample
from paper_2410_18701_amd import layer as PL
from paper_2410_18701_amd.cache import BatonCache

pytestmark = pytest.mark.gpu

REL, ATOL = 2.0 ** -5, 2e-2


def val(t):
    return t.double().cpu().numpy()


def close(got, want, what):
    err = np.abs(got - want) / (REL * np.abs(want) + ATOL)
    assert err.max() <= 1, f"{what}: {err.max():.3g} of the tolerance"


class Model:
    HID, HQ, HKV, D, F, VOCAB, LAYERS = 256, 4, 2, 64, 512, 1000, 2

    def __init__(self, seed, n_adapters):
        g = torch.Generator(device="cuda").manual_seed(seed)
        t = lambda *s, k=0: (torch.randn(s, generator=g, device="cuda") * 2.0 ** -k).bfloat16()  # noqa: E731
        qkv = (self.HQ + 2 * self.HKV) * self.D
        outs = dict(qkv=(qkv, self.HID), o=(self.HID, self.HQ * self.D), gate_up=(2 * self.F, self.HID),
                    down=(self.HID, self.F))
        self.parts = dict(qkv=[self.HQ * self.D, self.HKV * self.D, self.HKV * self.D], gate_up=[self.F, self.F],
                          o=None, down=None)
        self.weights = [dict({n: t(*s, k=4) for n, s in outs.items()}, norm1=t(self.HID), norm2=t(self.HID))
                        for _ in range(self.LAYERS)]
        ranks = [8, 24, 16][:n_adapters]
        self.ab = [{n: [(t(len(self.parts[n] or [0]) * r, s[1], k=4), t(s[0], r, k=3), 0.5 + i) for i, r in enumerate(ranks)]
                    for n, s in outs.items()} for _ in range(self.LAYERS)]
        self.adapters = [{n: PL.Adapters([a for a, _, _ in v], [b for _, b, _ in v], [s for _, _, s in v],
                                         parts=self.parts[n]) for n, v in layer.items()} for layer in self.ab]
        self.head = dict(norm=t(self.HID), out=t(self.VOCAB, self.HID, k=3))
        self.rand = t

    def delta(self, layer, name, x, ids):
        """float64 low-rank products of the rows of x."""
        ab, out = self.ab[layer][name], None
        for r, i in enumerate(ids):
            if i < 0:
                continue
            a, b, s = val(ab[i][0]), val(ab[i][1]), ab[i][2]
            out = np.zeros((len(ids), b.shape[0])) if out is None else out
            c, rank = 0, b.shape[1]
            for p, d in enumerate(self.parts[name] or [b.shape[0]]):
                out[r, c:c + d] = s * (b[c:c + d] @ (a[p * rank:(p + 1) * rank] @ x[r]))
                c += d
        return 0.0 if out is None else out


def check_layer(m, layer, x0, ids, pos, got, live):
    """One layer from the stream x0: q, k, v, the attention output att (of the model of
    the cache) and the stream after it."""
    r, w = X.round_bf16, {n: val(t) for n, t in m.weights[layer].items()}
    h = r(LL.rmsnorm(x0, w["norm1"], 1e-5))
    qkv = r(r(LL.linear(h, w["qkv"])) + m.delta(layer, "qkv", h, ids))
    q, k, v = LL.split_qkv(qkv, m.HQ, m.HKV, m.D)
    p = np.asarray(pos, np.float64)[:, None]
    for name, want in (("q", LL.rope(q, p, 1e4)), ("k", LL.rope(k, p, 1e4)), ("v", v)):
        close(got[name][live], want[live], f"layer {layer} {name}")
    att = got["att"].reshape(len(ids), -1)
    x = r(r(x0 + m.delta(layer, "o", att, ids)) + LL.linear(att, w["o"]))
    h = r(LL.rmsnorm(x, w["norm2"], 1e-5))
    gu = r(r(LL.linear(h, w["gate_up"])) + m.delta(layer, "gate_up", h, ids))
    act = r(LL.silu(gu[:, :m.F]) * gu[:, m.F:])
    x = r(r(x + m.delta(layer, "down", act, ids)) + LL.linear(act, w["down"]))
    close(got["x"][live], x[live], f"layer {layer} stream")


@pytest.mark.parametrize("batch", [1, 6, 70])
def test_a_batch_of_different_queries(batch):
    m = Model(batch, 3)
    rng = np.random.default_rng(batch)
    cache = BatonCache(m.LAYERS, batch, m.HQ, m.HKV, m.D, 160, dtype="mxfp4")
    model = X.Batch4(m.LAYERS, batch, m.HQ, m.HKV, m.D)
    gemm = PL.Gemm()
    layers = PL.DecodeLayers(cache, m.weights, gemm, adapters=m.adapters, head=m.head)

    def embed(slots, lens):
        ks, vs = ([m.rand(m.LAYERS, m.HKV, n, m.D) for n in lens] for _ in range(2))
        cache.embed(slots, lens, ks, vs)
        model.embed(slots, [val(x) for x in ks], [val(x) for x in vs])
        for b in slots:
            layers.slot_adapter[b] = int(rng.integers(-1, 3))

    full = list(range(batch - (batch > 3)))          # a slot stays free at first
    embed(full, [int(n) for n in rng.integers(1, 90, len(full))])
    for step in range(4):
        if step == 2 and batch > 1:
            gone = full[::3]
            cache.evict(gone)
            model.evict(gone)
            embed(gone, [int(n) for n in rng.integers(1, 120, len(gone))])
            if batch - 1 not in full:
                embed([batch - 1], [40])
        if step == 3:
            layers.slot_adapter = [-1] * batch      # the fused forms without adapters
        live = [b for b in range(batch) if model.k[b] is not None]
        ids, pos = list(layers.slot_adapter), cache.tokens()
        x = m.rand(batch, m.HID)
        seen = []
        for l in range(m.LAYERS):
            x0 = val(x)
            layers.layer(l, x)
            got = {n: val(getattr(layers, n)) for n in ("q", "k", "v", "att")}
            got["x"] = val(x)
            seen.append(got)
            check_layer(m, l, x0, ids, pos, got, live)
        cache.advance()
        q, k, v = (np.stack([g[n][:, None] for g in seen]) for n in ("q", "k", "v"))
        for (l, b, _), (o, a) in model.step(q, k, v).items():
            err = np.abs(seen[l]["att"][b] - o) - (2.0 ** -8 * (a + np.abs(o)) + 2.0 ** -13 * a)
            assert err.max() <= 0, f"step {step} layer {l} slot {b}: attention"
        params = dict(temperature=rng.choice([0.0, 0.7, 1.0], batch), top_k=rng.choice([0, 5, 50], batch),
                      top_p=rng.choice([0.5, 0.9, 1.0], batch), min_p=rng.choice([0.0, 0.05], batch))
        u = rng.random(batch)
        dev = {n: torch.tensor(p, device="cuda", dtype=torch.int32 if n == "top_k" else torch.float32)
               for n, p in params.items()}
        tokens = layers.next_tokens(x, torch.tensor(u, device="cuda", dtype=torch.float32), **dev).cpu().tolist()
        h = X.round_bf16(LL.rmsnorm(val(x), val(m.head["norm"]), 1e-5))
        logits = val(layers.logits)
        close(logits[live], LL.linear(h, val(m.head["out"]))[live], "logits")
        for b in live:
            f = {n: float(np.float32(p[b])) if n != "top_k" else int(p[b]) for n, p in params.items()}
            assert tokens[b] == sample(logits[b], float(np.float32(u[b])), **f)
    print(f"[serving] batch {batch}: {len(live)} live", flush=True)


def test_a_whole_step_in_a_hip_graph():
    """Two steps of the same batch, one captured: the captured one replays with new
    streams, parameters and random numbers like the eager one."""
    m = Model(5, 2)
    ks, vs = ([m.rand(m.LAYERS, m.HKV, n, m.D) for n in (70, 9, 33)] for _ in range(2))
    both = []
    for _ in range(2):
        cache = BatonCache(m.LAYERS, 4, m.HQ, m.HKV, m.D, 160, dtype="mxfp4")
        cache.embed([0, 1, 3], [70, 9, 33], ks, vs)
        layers = PL.DecodeLayers(cache, m.weights, PL.Gemm(), adapters=m.adapters, head=m.head)
        layers.slot_adapter = [1, -1, 0, 0]
        cache.workspace()
        both.append((cache, layers))

    x = m.rand(4, m.HID)
    t = dict(u=torch.rand(4, device="cuda"), temperature=torch.ones(4, device="cuda"),
             top_k=torch.full((4,), 20, device="cuda", dtype=torch.int32), top_p=torch.full((4,), 0.9, device="cuda"))

    def step(layers):
        y = x.clone()
        for l in range(m.LAYERS):
            layers.layer(l, y)
        return y, layers.next_tokens(y, **t)

    (eager_cache, eager), (graph_cache, graphed) = both
    want_y, want_tokens = step(eager)
    want = [(want_y.clone(), want_tokens.clone())]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y, tokens = step(graphed)
    for rep in range(3):
        y.fill_(float("nan"))
        tokens.fill_(-7)
        torch.randn(1 << 16, device="cuda").sum()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0][0]) and torch.equal(tokens, want[0][1]), f"replay {rep}"
    assert torch.equal(eager_cache.k, graph_cache.k) and torch.equal(eager_cache.v, graph_cache.v)
    # other random numbers and parameters: the replay follows them
    t["u"].copy_(torch.rand(4, device="cuda"))
    t["temperature"].fill_(0.5)
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    logits = val(graphed.logits)
    for b in (0, 1, 3):
        assert int(tokens[b]) == sample(logits[b], float(t["u"][b]), 0.5, 20, float(t["top_p"][b]))
