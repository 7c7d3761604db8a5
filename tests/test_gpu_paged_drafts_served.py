"""Steps with drafted tokens over a pool of pages that runs dry and recovers: slots without
pages are verified as free ones, bring the same tokens again, and hold in the end what they hold
in a pool with room for all.  A whole step captured and replayed, its n_out the next one's keep,
queries arriving and leaving between replays."""
import numpy as np
import pytest
import torch

from oracle import paged as O
from oracle.verify import verify
from paper_2410_18701_amd.layer import DecodeLayers, Gemm, Verifier
from paper_2410_18701_amd.paged import PagedCache
from tests.test_gpu_paged import i32, rand
from tests.test_gpu_paged_serving import paged, prompts
from tests.test_gpu_serving import Model, val

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slots_that_took_no_part_are_free(dtype):
    """Verification with the cache: what n_draft says counts only of tokens that the step took."""
    g = torch.Generator(device="cuda").manual_seed(1)
    batch, width, vocab = 7, 3, 500
    c = PagedCache(1, batch, 2, 1, 64, 9, 2, page=32, width=width)
    c.begin(i32([31, 32, 0, 1, 5, 30, 0]))
    c.begin(i32([2, 1, 0, 3, 2, 40, 40]), keep=i32([31, 32, 0, 1, 5, 30, 0]))
    assert c.missing.tolist() == [0, 0, 0, 0, 0, 2, 0]       # 70 tokens are more than two pages; slot 6 brings a prompt
    taken = [2, 1, 0, 3, 2, 0, 40]
    target = rand(g, batch, width, vocab, dtype=dtype, gain=3.0)
    draft = rand(g, batch, width - 1, vocab, dtype=dtype, gain=3.0)
    drafted = torch.randint(0, vocab, (batch, width - 1), generator=g, device="cuda").int()
    u = torch.rand(batch, width, generator=g, device="cuda")
    ua = torch.zeros(batch, width - 1, device="cuda")        # drafts of any weight are accepted
    v = Verifier(batch, width, vocab)
    for n_draft in (None, [2] * 7, [1, 0, -1, 2, 1, 2, 2], [-1, 0, 2, 0, 5, 0, 0]):
        tokens, n_out = v(target, draft, drafted, None if n_draft is None else i32(n_draft), ua, u[:, 0].contiguous(), cache=c)
        for b in range(batch):
            n = min(width - 1 if n_draft is None else n_draft[b], taken[b] - 1) if 1 <= taken[b] <= width else -1
            want = verify(val(target[b]), val(draft[b]), drafted[b].tolist(), n, ua[b].tolist(), float(u[b, 0]))
            assert (tokens[b].tolist(), int(n_out[b])) == want, (n_draft, b)
    with pytest.raises(ValueError):
        Verifier(6, width, vocab)(target[:6], draft[:6], drafted[:6], None, ua[:6], u[:6, 0].contiguous(), cache=c)


def test_a_pool_that_runs_dry_and_recovers():
    """Slot b's tokens are given; every draft is accepted (a random number of 0), so a slot goes on
    by as many as it brought, by none where it lacked pages.  Of every step the tables are the
    oracle's, attention 64 bits' over the tokens taken; in the end each slot's first layer has the bits
    that it has in a pool with room for all."""
    m, batch, width, page, want_tokens = Model(5, 0), 4, 4, 32, 90
    emb = m.rand(m.VOCAB, m.HID)
    ids = torch.randint(0, m.VOCAB, (batch, want_tokens + 8), generator=torch.Generator().manual_seed(6))

    def serve(n_pages):
        c = PagedCache(m.LAYERS, batch, m.HQ, m.HKV, m.D, n_pages, 4, page=page, width=width)
        c.kv.fill_(float("nan"))
        t = O.Tables(batch, n_pages, 4, page)
        layers = DecodeLayers(c, m.weights, Gemm(), head=m.head)
        at, keep, lacked, kv = [0] * batch, None, 0, {}
        held = [[[np.zeros((m.HKV, 0, m.D))] * 2 for _ in range(m.LAYERS)] for _ in range(batch)]
        k_list = [0] * batch
        for step in range(400):
            # a slot that has all of its tokens leaves once its cache was looked at
            left = [b for b in range(batch) if at[b] >= want_tokens and b not in kv]
            if left:
                c.begin(i32([0] * batch), keep=keep)
                t.step([0] * batch, k_list, width)
                ks, vs = c.extract(left, [want_tokens] * len(left))
                for b, k, v in zip(left, ks, vs):
                    kv[b] = torch.stack([k[0], v[0]])
                k_list = [-1 if b in left else 0 for b in range(batch)]
                keep = i32(k_list)
            if len(kv) == batch:
                return kv, lacked
            n_new = [0 if b in kv else 1 + (at[b] + b) % width for b in range(batch)]
            places = c.begin(i32(n_new), keep=keep)
            want_places, missing = t.step(n_new, k_list, width)
            assert places.tolist() == want_places and c.missing.tolist() == missing and c.table.tolist() == t.table
            live = [b for b in range(batch) if n_new[b] and not missing[b]]
            assert c.lens.tolist() == t.lens and all(t.lens[b] == at[b] for b in range(batch) if b not in kv)
            tok = torch.stack([ids[b, min(at[b], want_tokens):][:width] for b in range(batch)]).cuda()
            x = emb[tok].view(batch * width, -1).clone()
            for l in range(m.LAYERS):
                layers.layer(l, x)
                q, k, v, att = (val(getattr(layers, s)).reshape(batch, width, -1, m.D) for s in ("q", "k", "v", "att"))
                for b in live:
                    n = n_new[b]
                    rows = [np.concatenate([h, y[b, :n].transpose(1, 0, 2)], 1) for h, y in zip(held[b][l], (k, v))]
                    want = O.attention(q[b, :n], *rows, at[b])
                    err = np.abs(att[b, :n] - want)
                    assert (err <= 2.0 ** -8 * np.abs(want) + 2.0 ** -12 * np.abs(rows[1]).max()).all(), (step, l, b)
                    held[b][l] = rows
            u = torch.zeros(batch, width - 1, device="cuda")
            tokens, n_out = layers.accept_drafts(x, None, tok[:, 1:].int().contiguous(), i32([n - 1 for n in n_new]), u,
                                                 torch.full((batch,), 0.5, device="cuda"))
            k_list = n_out.tolist()
            assert k_list == [n_new[b] if b in live else 0 for b in range(batch)]
            assert all(tokens[b].tolist() == [-1] * width for b in range(batch) if b not in live)
            assert all(tokens[b, :n_new[b] - 1].tolist() == tok[b, 1:n_new[b]].tolist() for b in live)
            keep = n_out.clone()
            at = [n + k for n, k in zip(at, k_list)]
            lacked += sum(x > 0 for x in missing)
        raise AssertionError("not done")

    room, none = serve(20)
    dry, some = serve(9)
    assert none == 0 and some > 10          # (20 by the tables)
    assert all(torch.equal(room[b], dry[b]) for b in range(batch))


def test_a_captured_step():
    """begin, the layers and the verification in one graph, which reads n_out as its keep: replayed
    with queries that arrive and leave between replays, over a pool that runs dry at times, beside
    the same calls without a graph."""
    m, batch, width, n_pages = Model(8, 0), 4, 4, 9
    vocab = m.VOCAB
    g = torch.Generator(device="cuda").manual_seed(9)

    class Side:
        def __init__(self):
            self.c = paged(m, batch, width, n_pages=n_pages)
            self.c.kv.zero_()
            self.layers = DecodeLayers(self.c, m.weights, Gemm(), head=m.head)
            e = lambda *s, t=torch.int32: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
            self.x, self.n_new, self.n_draft = e(batch * width, m.HID, t=torch.bfloat16), e(batch), e(batch)
            self.draft, self.drafted = e(batch, width - 1, vocab, t=torch.bfloat16), e(batch, width - 1)
            self.ua, self.ut = e(batch, width - 1, t=torch.float32), e(batch, t=torch.float32)
            self.layers.verifier.n_out.zero_()
            self.outs = [self.layers.verifier.n_out, self.layers.verifier.tokens, self.c.lens, self.c.table, self.c.missing,
                         self.c.slot_map, self.c.kv]

        def step(self):
            self.c.begin(self.n_new, keep=self.layers.verifier.n_out)
            for l in range(m.LAYERS):
                self.layers.layer(l, self.x)
            self.layers.accept_drafts(self.x, self.draft, self.drafted, self.n_draft, self.ua, self.ut)

        def between(self, leave, slot, ks, vs):
            """The query in `leave` goes, one of ks comes into `slot`."""
            n_out, n = self.layers.verifier.n_out, ks.shape[2]
            for b in leave:
                n_out[b] = -1
            self.c.begin(i32([n if b == slot else 0 for b in range(batch)]), keep=n_out)
            took = self.c.missing[slot] == 0
            self.c.embed([slot], [n], [ks], [vs])
            n_out.zero_()
            n_out[slot] = torch.where(took, n, 0)

    a, e = Side(), Side()
    for s in (a, e):
        s.step()                                   # nothing: four free slots; warms up
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    lacked = accepted = 0
    for i in range(40):
        if i in (0, 1, 2, 3, 14, 22, 30):
            leave, slot, n = ([], i, (40, 9, 61, 30)[i]) if i < 4 else ([i % 4], i % 4, i)
            (ks,), (vs,) = prompts(m, [n])
            for s in (a, e):
                s.between(leave, slot, ks, vs)
        n_draft = torch.randint(0, width, (batch,), generator=g, device="cuda").int()
        live = torch.tensor([b <= i or i >= 4 for b in range(batch)], device="cuda")
        inputs = dict(x=rand(g, batch * width, m.HID), n_draft=torch.where(live, n_draft, -1),
                      n_new=torch.where(live, n_draft + 1, 0), draft=rand(g, batch, width - 1, vocab, gain=3.0),
                      drafted=torch.randint(0, vocab, (batch, width - 1), generator=g, device="cuda").int(),
                      ua=1e-3 * torch.rand(batch, width - 1, generator=g, device="cuda"),
                      ut=torch.rand(batch, generator=g, device="cuda"))
        for s in (a, e):
            for name, v in inputs.items():
                getattr(s, name).copy_(v)
        graph.replay()
        e.step()
        torch.cuda.synchronize()
        for x, y in zip(a.outs, e.outs):
            assert torch.equal(x, y), i
        missing, n_out = a.c.missing.tolist(), a.outs[0].tolist()
        assert all((n_out[b] == 0) == (missing[b] > 0 or not bool(live[b])) for b in range(batch))
        lacked, accepted = lacked + sum(x > 0 for x in missing), accepted + sum(max(0, n - 1) for n in n_out)
    assert lacked > 5 and accepted > 10
