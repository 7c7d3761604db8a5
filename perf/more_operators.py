"""Operators of speculative decoding over a paged cache, as timed cases: tables
of pages kept on the GPU, attention of one or a few new tokens over pages (all
of a query, or a sliding window and its first tokens), and the verification of
drafted tokens.

Where `own` is false a pass computes the operator in its plain form, in
elementary torch operations; where it is true it makes the library's calls.

kinds
  step    the new tokens' keys and values of every layer go into pages, and the
          new tokens attend over the pages: one new token per query, or some
          drafted ones behind it.  window > 0: token j is visible from position p
          if p - window < j <= p, or j < sinks and j <= p.
  tables  the tables of a step: pages for each query's new tokens and their
          places, then the step's end with every draft rejected
  arrive  prefilled queries arrive (pages, their keys and values) and are parked
          again (copied out, their pages given back), among others that stay
  verify  drafted tokens against the target's logits, from given random numbers

Passes repeat: a pass leaves the lengths, tables and pages as it found them.
"""
import math
import random

import torch

own = False   # True: the library's calls


def listed():
    return [
        # The smallest step: four queries of a few dozen tokens, where latency counts.
        dict(name="step-tiny", kind="step", dtype="bf16", layers=1, batch=4, free=0, hq=4, hkv=4, d=64, page=32, width=1,
             window=0, sinks=0, law="uniform", lo=16, hi=128, lens_seed=1),
        # An ordinary step with a head of its own per query head.
        dict(name="step-b32-L2048", kind="step", dtype="bf16", layers=1, batch=32, free=2, hq=32, hkv=32, d=128, page=64,
             width=1, window=0, sinks=0, law="uniform", lo=128, hi=2048, lens_seed=2),
        # Grouped heads and long queries: the largest.
        dict(name="step-gqa-b64-L8192", kind="step", dtype="bf16", layers=2, batch=64, free=3, hq=64, hkv=8, d=128,
             page=64, width=1, window=0, sinks=0, law="uniform", lo=256, hi=8192, lens_seed=3),
        # Up to four drafted tokens behind each query's next one; a few very long queries among short ones.
        dict(name="step-drafts-skew-L32768", kind="step", dtype="bf16", layers=1, batch=32, free=1, hq=32, hkv=4, d=128,
             page=128, width=5, window=0, sinks=0, law="skew", lo=64, hi=32768, lens_seed=4),
        # A model with a sliding window whose first tokens stay visible, long queries.
        dict(name="window-b64-L16384", kind="step", dtype="bf16", layers=1, batch=64, free=0, hq=32, hkv=8, d=128, page=64,
             width=1, window=4096, sinks=4, law="uniform", lo=512, hi=16384, lens_seed=5),
        # The same in fp32 with drafts and odd sizes: the window starts and ends inside pages.
        dict(name="window-f32-drafts", kind="step", dtype="f32", layers=1, batch=7, free=1, hq=16, hkv=8, d=64, page=32,
             width=3, window=333, sinks=5, law="uniform", lo=1, hi=3001, lens_seed=6),
        # The tables of a large batch's step with four drafts each.
        dict(name="tables-b256", kind="tables", batch=256, free=9, page=64, width=5, lo=64, hi=8192, lens_seed=7),
        # One short query comes and goes.
        dict(name="arrive-n1-L300", kind="arrive", dtype="bf16", layers=2, batch=8, n=1, hq=8, hkv=8, d=64, page=32, lo=300,
             hi=300, rest=500, lens_seed=8),
        # Several long ones, ragged, in four layers.
        dict(name="arrive-n8-L4096", kind="arrive", dtype="bf16", layers=4, batch=64, n=8, hq=32, hkv=8, d=128, page=64,
             lo=333, hi=4095, rest=2000, lens_seed=9),
        # One user's drafts, greedy ones of a small model: what a draft looked like is one token, not a distribution.
        dict(name="verify-b1-v50257", kind="verify", dtype="f32", batch=1, free=0, width=4, vocab=50257, mode="plain",
             spread=3.0, near=0.5, points=True, params_seed=10),
        # An ordinary batch, each query with its own sampling parameters and number of drafts.
        dict(name="verify-b16-v32000", kind="verify", dtype="bf16", batch=16, free=1, width=5, vocab=32000, mode="mixed",
             spread=2.5, near=0.5, points=False, params_seed=11),
        # A large batch over a large vocabulary.
        dict(name="verify-b64-v128000", kind="verify", dtype="bf16", batch=64, free=0, width=5, vocab=128000, mode="mixed",
             spread=2.0, near=0.3, points=False, params_seed=12),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["step", "step", "step", "step", "tables", "arrive", "verify", "verify", "verify"])
    if kind == "verify":
        c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), batch=_log(rng, 1, 256), width=rng.randint(1, 9),
                 vocab=_log(rng, 500, 160000), mode=rng.choice(["mixed", "mixed", "plain", "top_k", "top_p", "min_p", "greedy"]),
                 spread=round(rng.uniform(0.5, 4.0), 2), near=round(rng.uniform(0.05, 1.0), 2),
                 points=rng.random() < 0.25, params_seed=rng.randrange(1 << 20))
        while c["batch"] * (2 * c["width"] - 1) * c["vocab"] * (2 if c["dtype"] == "bf16" else 4) > 64 * 9 * 128000 * 2:
            c["batch"] = max(1, c["batch"] // 2)
        c["free"] = rng.randint(0, c["batch"] // 4)
        return c
    if kind == "tables":
        c = dict(kind=kind, batch=_log(rng, 1, 512), page=rng.choice([32, 64, 128, 256]), width=rng.randint(1, 16),
                 hi=_log(rng, 32, 32768), lens_seed=rng.randrange(1 << 20))
        c["free"], c["lo"] = rng.randint(0, c["batch"] // 4), max(1, c["hi"] // 16)
        return c
    c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), d=rng.choice([64, 128, 128]),
             page=rng.choice([32, 64, 128, 256]), lens_seed=rng.randrange(1 << 20), hkv=_log(rng, 1, 32),
             batch=_log(rng, 1, 256), layers=rng.randint(1, 4), hi=_log(rng, 32, 32768))
    group = rng.choice([1, 1, 2, 4, 8])
    while c["hkv"] * group > 64:
        c["hkv"] //= 2
    c["hq"] = c["hkv"] * group
    if kind == "arrive":
        c["n"] = rng.randint(1, min(c["batch"], 16))
        c["rest"] = rng.randint(1, 2048)
    else:
        c["width"] = rng.choice([1, 1, 1, rng.randint(2, 64 // group if group > 4 else 16)])
        c["law"] = rng.choice(["uniform", "uniform", "lognormal", "skew"])
        c["free"] = rng.randint(0, c["batch"] // 4)
        windowed = rng.random() < 0.4
        c["window"] = _log(rng, 1, c["hi"]) if windowed else 0
        c["sinks"] = rng.choice([0, 1, 4, 4, rng.randint(0, 100)]) if windowed else 0
    size = lambda: c["layers"] * c["batch"] * c["hkv"] * c["hi"] * c["d"] * (1 if c["dtype"] == "bf16" else 2)  # noqa: E731
    while size() > 2 * 64 * 8 * 8192 * 128 and c["hi"] > 32:
        c["hi"] = max(32, c["hi"] // 2)
    while c["batch"] * c.get("width", 1) * c["hq"] * c["hi"] > 32 * 5 * 32 * 32768 and c["hi"] > 32:   # scores of the plain form
        c["hi"] = max(32, c["hi"] // 2)
    c["lo"] = max(1, c["hi"] // 16)
    return c


# ------------------------------------------------------------ the schedule --
def lengths(c):
    """Tokens cached for each of the live queries (arrive: of the queries that arrive)."""
    r = random.Random(c["lens_seed"])
    lo, hi, n = c["lo"], c["hi"], c["n"] if c["kind"] == "arrive" else c["batch"] - c["free"]
    law = c.get("law", "uniform")
    if law == "lognormal":
        lens = [int(min(hi, max(lo, round(r.lognormvariate(math.log(max(2, hi / 6)), 0.8))))) for _ in range(n)]
    elif law == "skew":   # a tenth of the queries long
        long = set(r.sample(range(n), max(1, n // 10)))
        lens = [r.randint(hi // 2, hi) if b in long else r.randint(min(lo, hi), max(lo, hi // 32)) for b in range(n)]
    else:
        lens = [r.randint(lo, hi) for _ in range(n)]
    lens[max(range(n), key=lambda b: lens[b])] = hi
    return lens


def fresh(c):
    """New tokens of each slot in the step: one and some drafts of a live query, none of a free slot."""
    r = random.Random(c["lens_seed"] + 1)
    n = c["batch"] - c["free"]
    return [r.randint(1, c["width"]) for _ in range(n)] + [0] * c["free"]


def drafts(c):
    """Drafted tokens of each slot; -1 of a free one."""
    r = random.Random(c["params_seed"] + 1)
    n = c["batch"] - c["free"]
    return [r.choice([c["width"] - 1, r.randint(0, c["width"] - 1)]) for _ in range(n)] + [-1] * c["free"]


def pages(c):
    """(pages of the pool, pages of a slot at most): enough for all, and a tenth more."""
    per = lambda n: -(-n // c["page"])  # noqa: E731
    lens = lengths(c)
    total = sum(per(n + c.get("width", 1)) for n in lens)
    longest = max(lens) + c.get("width", 1)
    if c["kind"] == "arrive":
        total += (c["batch"] - c["n"]) * per(c["rest"])
        longest = max(longest, c["rest"])
    return total + total // 10 + 1, per(longest)


def _whole(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# -------------------------------------------------------------- the inputs --
def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed(seed * 1009 + salt)


def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _randn(g, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _sources(c, lens, g):
    """Keys and values of the queries, [layers][hkv][len][d]: normal, the keys
    with some channels several times as large as the others."""
    gain = torch.exp(0.5 * torch.randn((c["hkv"], 1, c["d"]), generator=g, device="cuda")).to(_type(c))
    ks = [_randn(g, c["layers"], c["hkv"], n, c["d"], dtype=_type(c)) * gain for n in lens]
    vs = [_randn(g, c["layers"], c["hkv"], n, c["d"], dtype=_type(c)) for n in lens]
    return ks, vs


def _inputs(c, g):
    """A step's queries, keys and values, [layers][batch][width][heads][d]."""
    shape = (c["layers"], c["batch"], c["width"])
    q = _randn(g, *shape, c["hq"], c["d"], dtype=_type(c))
    return (q,) + tuple(_randn(g, *shape, c["hkv"], c["d"], dtype=_type(c)) for _ in range(2))


def _order(c, seed):
    """The pool's pages in the order in which they are taken: a pool in use is in no order."""
    return torch.randperm(pages(c)[0], generator=_gen(seed, 4), device="cuda").int()


def _cache(c, seed):
    from paper_2410_18701_amd.paged import PagedCache
    n, per = pages(c)
    return PagedCache(c.get("layers", 1), c["batch"], c.get("hq", 1), c.get("hkv", 1), c.get("d", 64), n, per,
                      page=c["page"], width=c.get("width", 1), window=c.get("window", 0), sinks=c.get("sinks", 0),
                      dtype=c.get("dtype", "bf16"), order=_order(c, seed))


def _plain_cache(c, seed):
    """The plain form's cache: rows of tokens [layers][places][hkv][d], one more for what goes nowhere."""
    n, per = pages(c)
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    s = dict(page=c["page"], width=c.get("width", 1), table=z(c["batch"], per) - 1, lens=z(c["batch"]),
             covered=z(c["batch"]), pool=_order(c, seed).flip(0), count=z(1) + n)
    if "layers" in c:
        shape = (c["layers"], n * c["page"] + 1, c["hkv"], c["d"])
        s["k"], s["v"] = (torch.zeros(shape, dtype=_type(c), device="cuda") for _ in range(2))
    return s


def _params(c):
    """Each query's temperature, top_k, top_p and min_p, as requests give them."""
    r, n, mode = random.Random(c["params_seed"]), c["batch"], c["mode"]
    temperature, top_k, top_p, min_p = [], [], [], []
    for _ in range(n):
        how = r.choice(["greedy", "plain", "plain", "top_k", "top_p", "min_p", "all"]) if mode == "mixed" else mode
        temperature.append(0.0 if how == "greedy" else r.choice([0.3, 0.7, 1.0, 1.0, 1.5]))
        top_k.append(r.choice([1, 5, 40, 50, 100, 1000]) if how in ("top_k", "all") else 0)
        top_p.append(r.choice([0.1, 0.5, 0.8, 0.9, 0.95, 0.99]) if how in ("top_p", "all") else 1.0)
        min_p.append(r.choice([0.01, 0.05, 0.1]) if how in ("min_p", "all") else 0.0)
    f = lambda v, t=torch.float32: torch.tensor(v, dtype=t, device="cuda")  # noqa: E731
    return dict(temperature=f(temperature), top_k=f(top_k, torch.int32), top_p=f(top_p), min_p=f(min_p))


def prepare(case, seed):
    c = case
    if c["kind"] == "verify":
        g = _gen(seed, 3)
        b, w, v = c["batch"], c["width"], c["vocab"]
        target = c["spread"] * torch.randn((b, w, v), generator=g, device="cuda")
        draft = (target[:, :-1] + c["near"] * torch.randn((b, w - 1, v), generator=g, device="cuda")).to(_type(c))
        s = dict(c=c, target=target.to(_type(c)), draft=draft, n_draft=_whole(drafts(c)), **_params(c))
        s["u_accept"] = torch.rand((b, max(1, w - 1)), generator=g, device="cuda")[:, :w - 1].contiguous()
        s["u_token"] = torch.rand(b, generator=g, device="cuda")
        u = torch.rand(b * (w - 1), generator=g, device="cuda")
        if c["points"] or w == 1:   # the draft's likeliest tokens
            s["drafted"] = draft.argmax(-1).int()
        else:                       # drawn as the draft's own sampling does
            rows = {k: s[k].repeat_interleave(w - 1) for k in ("temperature", "top_k", "top_p", "min_p")}
            s["drafted"] = _invert(_kept(draft.flatten(0, 1), **rows), u).view(b, w - 1)
        if c["points"]:
            s["draft"] = None
        if own:
            from paper_2410_18701_amd.layer import Verifier
            s["verifier"] = Verifier(b, w, v)
        return s
    g = _gen(seed, 1)
    lens = lengths(c)
    s = dict(c=c, lens=lens)
    if c["kind"] == "tables":
        at = _whole(lens + [0] * c["free"])
        s["n_new"], s["none"] = _whole(fresh(c)), torch.zeros_like(at)
    elif c["kind"] == "arrive":
        s["ks"], s["vs"] = _sources(c, lens, g)
        s["slots"] = random.Random(c["lens_seed"] + 2).sample(range(c["batch"]), c["n"])
        at = [c["rest"]] * c["batch"]
        coming, going = [0] * c["batch"], [0] * c["batch"]
        for b, n in zip(s["slots"], lens):
            at[b], coming[b], going[b] = 0, n, -1
        at, s["n_new"], s["keep"], s["none"] = _whole(at), _whole(coming), _whole(going), _whole([0] * c["batch"])
    else:
        ks, vs = _sources(c, lens, g)
        s["q"], s["k_new"], s["v_new"] = _inputs(c, g)
        s["out"] = torch.zeros_like(s["q"])
        s["n_new"] = _whole(fresh(c))
        at = _whole(lens + [0] * c["free"])
    if own:
        cache = s["cache"] = _cache(c, seed)
        cache.begin(at)
        if c["kind"] == "step":
            cache.embed(list(range(len(lens))), lens, ks, vs)
            cache.begin(s["n_new"], keep=at)
        else:
            cache.begin(torch.zeros_like(at), keep=at)
    else:
        cache = s["cache"] = _plain_cache(c, seed)
        _begin(cache, at)
        if c["kind"] == "step":
            _embed(cache, list(range(len(lens))), lens, ks, vs)
            s["map"] = _begin(cache, s["n_new"], at)
        else:
            _begin(cache, torch.zeros_like(at), at)
    return s


# -------------------------------------------------------- the plain forms --
def _begin(s, n_new, keep=None):
    """Ends a step (keep of its tokens stay, all of the query leaves if negative) and begins the
    next one with n_new tokens: pages given back, pages taken, the places of the new tokens."""
    lens, n_new = s["lens"], n_new.clamp(min=0)
    if keep is not None:
        lens = torch.where(keep < 0, 0, lens + keep)
    want, had = (lens + n_new + s["page"] - 1) // s["page"], s["covered"]
    j = torch.arange(s["table"].shape[1], device="cuda")
    gone = (j >= want[:, None]) & (j < had[:, None])
    back = s["table"][gone]
    count = int(s["count"])
    s["pool"][count:count + len(back)] = back.flip(0)
    s["table"][gone] = -1
    count += len(back)
    need = (want - had).clamp(min=0)
    fits = (need == 0) | (torch.cumsum(need, 0) <= count)
    more = (j >= had[:, None]) & (j < want[:, None]) & fits[:, None]
    taken = int(more.sum())
    s["table"][more] = s["pool"][count - taken:count].flip(0)
    s["count"].fill_(count - taken)
    s["covered"], s["lens"] = torch.where(fits, want, had).int(), lens.int()
    i = torch.arange(s["width"], device="cuda")
    at = (lens[:, None] + i).clamp(max=len(j) * s["page"] - 1)
    place = s["table"].gather(1, (at // s["page"]).long()) * s["page"] + at % s["page"]
    return torch.where((i < n_new[:, None]) & fits[:, None], place, -1).int()


def _places(s, slot, n):
    t = torch.arange(n, device="cuda")
    return s["table"][slot].long()[t // s["page"]] * s["page"] + t % s["page"]


def _put(s, slot, n, k, v):
    at = _places(s, slot, n)
    s["k"][:, at], s["v"][:, at] = k.transpose(1, 2), v.transpose(1, 2)


def _embed(s, slots, lens, ks, vs):
    [_put(s, *x) for x in zip(slots, lens, ks, vs)]


def _attention(s, layer, q, k_new, v_new, where, n_new, window, sinks):
    """One layer: the new tokens go to their places, then softmax over what each of them sees."""
    batch, width, hq, d = q.shape
    hkv = k_new.shape[2]
    where = torch.where(where < 0, s["k"].shape[1] - 1, where).long().flatten()
    s["k"][layer][where], s["v"][layer][where] = k_new.flatten(0, 1), v_new.flatten(0, 1)
    j = torch.arange(s["table"].shape[1] * s["page"], device="cuda")
    rows = s["table"].clamp(min=0).long()[:, j // s["page"]] * s["page"] + j % s["page"]
    k = s["k"][layer][rows].permute(0, 2, 3, 1).float()                       # [batch][hkv][d][tokens]
    qs = q.float().view(batch, width, hkv, -1, d).transpose(1, 2).flatten(2, 3) * d ** -0.5
    x = (qs @ k).unflatten(2, (width, -1))
    del k
    at = (s["lens"][:, None] + torch.arange(width, device="cuda"))[:, :, None]
    sees = (j <= at) & ((j > at - window) | (j < sinks) if window else True)
    x = x.masked_fill(~sees[:, None, :, None], -math.inf)
    p = torch.exp(x - x.amax(-1, keepdim=True))
    p = (p / p.sum(-1, keepdim=True)).flatten(2, 3)
    out = p @ s["v"][layer][rows].transpose(1, 2).float()
    out = out.view(batch, hkv, width, -1, d).transpose(1, 2).reshape(q.shape)
    live = torch.arange(width, device="cuda") < n_new[:, None]
    return torch.where(live[:, :, None, None], out, 0.0).to(q.dtype)


def _kept(l, temperature, top_k, top_p, min_p):
    """Weights in 64 bits of the tokens that sampling keeps, 0 of the others: rows of logits."""
    n = l.shape[1]
    l, order = torch.sort(l.double(), dim=1, descending=True, stable=True)
    greedy = temperature <= 0
    t = torch.where(greedy, 1.0, temperature).double()[:, None]
    w = torch.exp((l - l[:, :1]) / t)
    del l
    place = torch.arange(n, device="cuda")
    k = torch.where((top_k <= 0) | (top_k > n), n, top_k)[:, None]
    w = torch.where(place < k, w, 0.0)
    before = torch.cumsum(w, 1) - w
    p = top_p.double()[:, None]
    keep = (place < k) & ((before < p * w.sum(1, keepdim=True)) | (p >= 1) | (place == 0))
    keep &= (w >= min_p.double()[:, None]) | (place == 0)
    keep &= ~greedy[:, None] | (place == 0)
    return torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0))


def _invert(w, u):
    """The first token of each row at which the running weight exceeds u times all of it."""
    c = torch.cumsum(w, 1)
    return (c <= u.double()[:, None] * c[:, -1:]).sum(1).clamp(max=w.shape[1] - 1).int()


def _verify(target, draft, drafted, n_draft, u_accept, u_token, temperature, top_k, top_p, min_p):
    """A draft is kept with probability min(1, p / q); at the first that is not, a token is drawn
    from max(0, p - q), behind the last one from p."""
    b, w, v = target.shape
    params = (temperature, top_k, top_p, min_p)
    p = _kept(target.flatten(0, 1), *(x.repeat_interleave(w) for x in params)).view(b, w, v)
    p = p / p.sum(-1, keepdim=True)
    x = drafted.long()
    i = torch.arange(w, device="cuda")
    if draft is None or w == 1:
        q = torch.zeros((b, w - 1, v), dtype=torch.float64, device="cuda").scatter_(2, x[:, :, None], 1.0)
    else:
        q = _kept(draft.flatten(0, 1), *(y.repeat_interleave(w - 1) for y in params)).view(b, w - 1, v)
        q = q / q.sum(-1, keepdim=True)
    at = lambda y: y.gather(2, x[:, :, None])[:, :, 0]  # noqa: E731
    good = (u_accept.double() * at(q) < at(p[:, :-1])) & (i[:-1] < n_draft[:, None])
    n = torch.cumprod(good.int(), 1).sum(1)
    row = torch.arange(b, device="cuda")
    r = p[row, n]
    if w > 1:
        less = (r - q[row, n.clamp(max=w - 2)]).clamp(min=0)
        less = torch.where(less.sum(1, keepdim=True) > 0, less, r)
        r = torch.where((n < n_draft)[:, None], less, r)
    token = _invert(r, u_token)
    padded = torch.cat([drafted.int(), torch.full((b, 1), -1, dtype=torch.int32, device="cuda")], 1)
    out = torch.where(i < n[:, None], padded, torch.where(i == n[:, None], token[:, None], -1))
    live = n_draft >= 0
    return torch.where(live[:, None], out, -1).int(), torch.where(live, n + 1, 0).int()


def run(s):
    c = s["c"]
    if c["kind"] == "verify":
        args = (s["target"], s["draft"], s["drafted"], s["n_draft"], s["u_accept"], s["u_token"], s["temperature"],
                s["top_k"], s["top_p"], s["min_p"])
        return s["verifier"](*args) if own else _verify(*args)
    cache = s["cache"]
    if c["kind"] == "tables":
        if own:
            places = cache.begin(s["n_new"]).clone()
            granted = cache.table.clone()
            cache.begin(s["none"], keep=s["none"])
            return places, granted, cache.table, cache.lens
        places = _begin(cache, s["n_new"])
        granted = cache["table"].clone()
        _begin(cache, s["none"], s["none"])
        return places, granted, cache["table"], cache["lens"]
    if c["kind"] == "arrive":
        if own:
            cache.begin(s["n_new"])
            cache.embed(s["slots"], s["lens"], s["ks"], s["vs"])
            ks, vs = cache.extract(s["slots"], s["lens"])
            table = cache.table.clone()
            cache.begin(s["none"], keep=s["keep"])
            return ks, vs, table
        _begin(cache, s["n_new"])
        _embed(cache, s["slots"], s["lens"], s["ks"], s["vs"])
        ks, vs = ([cache[x][:, _places(cache, b, n)].transpose(1, 2) for b, n in zip(s["slots"], s["lens"])] for x in "kv")
        table = cache["table"].clone()
        _begin(cache, s["none"], s["keep"])
        return ks, vs, table
    if own:
        return [cache.decode_attn(l, s["q"][l], s["k_new"][l], s["v_new"][l], out=s["out"][l])
                for l in range(c["layers"])]
    return [_attention(cache, l, s["q"][l], s["k_new"][l], s["v_new"][l], s["map"], s["n_new"], c["window"], c["sinks"])
            for l in range(c["layers"])]


# ------------------------------------------------------------------- work --
def work(case):
    c = case
    if c["kind"] == "verify":
        rows = sum(n + 1 + (0 if c["points"] else n) for n in drafts(c) if n >= 0)
        return {"bytes": rows * c["vocab"] * (2 if c["dtype"] == "bf16" else 4) + 24 * c["batch"] * c["width"],
                "flops": 2 * rows * c["vocab"]}
    lens = lengths(c)
    if c["kind"] == "tables":
        pairs = list(zip(lens, fresh(c)))
        taken = sum(-(-(n + t) // c["page"]) - -(-n // c["page"]) for n, t in pairs)
        n = c["batch"]
        return {"bytes": 4 * (n * c["width"] + 4 * taken + 6 * n + 2 * n * pages(c)[1]), "flops": 10 * n}
    es = 2 if c["dtype"] == "bf16" else 4
    token = c["layers"] * c["hkv"] * c["d"] * 2 * es         # bytes of K and V of one token
    if c["kind"] == "arrive":   # sources read, pages written and read, copies written
        return {"bytes": 4 * sum(lens) * token, "flops": sum(lens)}
    seen = new = pairs = 0
    for n, t in zip(lens, fresh(c)):
        w, k = c["window"] or n + t, min(c["sinks"], n + t)
        first = max(0, n - w + 1)
        seen += n + t - first + min(first, k)
        pairs += sum(min(w, p + 1) + min(max(0, p + 1 - w), k) for p in range(n, n + t))
        new += t
    return {"bytes": (seen + 2 * new) * token + 2 * new * c["layers"] * c["hq"] * c["d"] * es,
            "flops": 4 * pairs * c["layers"] * c["hq"] * c["d"]}


# ------------------------------------------------------------------ exact --
def exact(case, seed):
    c = case
    if c["kind"] in ("verify", "tables"):
        return None   # whole numbers
    g = _gen(seed, 1)
    lens = lengths(c)
    ks, vs = _sources(c, lens, g)
    if c["kind"] == "arrive":
        return [k.double() for k in ks], [v.double() for v in vs], None
    q, k_new, v_new = _inputs(c, g)
    out = torch.zeros_like(q, dtype=torch.float64)
    group = c["hq"] // c["hkv"]
    for b, (n, t) in enumerate(zip(lens, fresh(c))):
        k = torch.cat([ks[b].double(), k_new[:, b, :t].transpose(1, 2).double()], 2)   # [layers][hkv][n + t][d]
        v = torch.cat([vs[b].double(), v_new[:, b, :t].transpose(1, 2).double()], 2)
        for i in range(t):
            at = n + i
            seen = [j for j in range(min(c["sinks"], at + 1)) if j <= at - c["window"]] if c["window"] else []
            pick = torch.tensor(seen + list(range(max(0, at - c["window"] + 1) if c["window"] else 0, at + 1)), device="cuda")
            kk, vv = k[:, :, pick], v[:, :, pick]
            x = q[:, b, i].double().unflatten(1, (c["hkv"], group))                    # [layers][hkv][group][d]
            y = torch.softmax(torch.matmul(x, kk.mT.contiguous()) / math.sqrt(c["d"]), -1)
            out[:, b, i] = torch.matmul(y, vv).flatten(1, 2)
    return list(out)
