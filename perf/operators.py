"""Operators of a serving step whose queries differ, as timed cases: a KV cache
held in 4 bits with the decode attention that reads it, the low-rank adapters
of many requests beside a shared projection, and sampling with each request's
own parameters.

Where `own` is false a pass computes the operator in its plain form, in
elementary torch operations; where it is true it makes the library's calls.

kinds
  step      one decode step over a 4-bit cache in its steady state: a few
            slots' queries are replaced (bf16 keys and values, quantised as
            they are embedded), then the attention of every layer, which also
            appends the step's keys and values.  Slot b's query in cycle c is
            query (b + c) mod batch, so lengths stay where they are however
            often a pass is run.
  park      queries embedded into a 4-bit cache and copied out of it again
            (preemption): the quantisation and its inverse alone
  adapters  one adapter per row at most, their low-rank products alone
  proj      the same beside the shared projection they belong to
  sample    one token per row from logits, with given random numbers

The 4-bit form: blocks of 32 consecutive elements of a token's head share a
power of two; an element is one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 of it, with a
sign, the nearest one (ties to the even code).  The power of two is the
smallest that takes the block's largest magnitude to at most 7, which still
rounds to 6 by less than half a step.
"""
import math
import random

import torch

own = False   # True: the library's calls

BLOCK = 32


def listed():
    return [
        # The smallest step: four slots of a few dozen tokens, four short calls.
        dict(name="step-tiny", kind="step", layers=1, batch=4, free=0, hq=4, hkv=4, d=64, law="uniform", lo=16, hi=128,
             turn=1, lens_seed=1),
        # An ordinary one-layer step with a head of its own per query head.
        dict(name="step-b32-L2048", kind="step", layers=1, batch=32, free=0, hq=32, hkv=32, d=128, law="uniform",
             lo=128, hi=2048, turn=2, lens_seed=2),
        # Grouped heads, long rows, a few slots free: the largest.
        dict(name="step-gqa-b64-L8192", kind="step", layers=2, batch=64, free=3, hq=64, hkv=8, d=128, law="uniform",
             lo=256, hi=8192, turn=2, lens_seed=3),
        # A few very long rows among many short ones: the long ones have to be split.
        dict(name="step-skew-b32-L32768", kind="step", layers=1, batch=32, free=1, hq=32, hkv=4, d=128, law="skew",
             lo=64, hi=32768, turn=1, lens_seed=4),
        # Arrivals embedded and preempted queries copied out, ragged lengths.
        dict(name="park-n8-L4096", kind="park", layers=4, batch=16, n=8, hq=32, hkv=8, d=128, lo=333, hi=4095,
             lens_seed=5),
        # One request alone with an adapter on a 4096-wide projection: two short launches.
        dict(name="adapters-r1", kind="adapters", rows=1, adapters=1, used=1, rank=16, in_dim=4096, out_dim=4096,
             parts=1, bare=0, ids_seed=6),
        # A decode batch whose rows carry 24 adapters of the fused query/key/value projection; some have none.
        dict(name="adapters-qkv-r64", kind="adapters", rows=64, adapters=32, used=24, rank=32, in_dim=4096,
             out_dim=12288, parts=3, bare=7, ids_seed=7),
        # The largest batch and the widest projection (gate and up), the shared product with it.
        dict(name="proj-gate-up-r256", kind="proj", rows=256, adapters=40, used=40, rank=64, in_dim=4096,
             out_dim=22016, parts=2, bare=16, ids_seed=8),
        # One user's next token.
        dict(name="sample-r1-v32000", kind="sample", dtype="bf16", rows=1, vocab=32000, mode="mixed", spread=2.5,
             params_seed=9),
        # An ordinary batch, every row with its own parameters.
        dict(name="sample-r64-v32000", kind="sample", dtype="bf16", rows=64, vocab=32000, mode="mixed", spread=2.5,
             params_seed=10),
        # The same in fp32 with an odd vocabulary, whose rows start at odd addresses, temperature alone.
        dict(name="sample-f32-r16-v50257", kind="sample", dtype="f32", rows=16, vocab=50257, mode="plain", spread=3.0,
             params_seed=11),
        # A large batch over a large vocabulary.
        dict(name="sample-r256-v128000", kind="sample", dtype="bf16", rows=256, vocab=128000, mode="mixed", spread=2.0,
             params_seed=12),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["step", "step", "step", "park", "adapters", "adapters", "proj", "sample", "sample", "sample"])
    if kind == "sample":
        c = dict(kind=kind, dtype=rng.choice(["bf16", "f32"]), rows=_log(rng, 1, 256), vocab=_log(rng, 500, 160000),
                 mode=rng.choice(["mixed", "mixed", "plain", "top_k", "top_p", "min_p", "greedy"]),
                 spread=round(rng.uniform(0.5, 4.0), 2), params_seed=rng.randrange(1 << 20))
        while c["rows"] * c["vocab"] > 256 * 128000:
            c["rows"] //= 2
        return c
    if kind in ("adapters", "proj"):
        n = _log(rng, 1, 64)
        c = dict(kind=kind, rows=_log(rng, 1, 256), adapters=n, used=rng.randint(1, n),
                 rank=rng.choice([8, 16, 16, 24, 32, 40, 64, 104, 128]), in_dim=8 * _log(rng, 32, 1376),
                 out_dim=16 * _log(rng, 16, 1376), parts=rng.choice([1, 1, 2, 3]), ids_seed=rng.randrange(1 << 20))
        c["out_dim"] = -(-c["out_dim"] // (16 * c["parts"])) * 16 * c["parts"]
        c["bare"] = rng.randint(0, c["rows"] // 3)
        while c["in_dim"] * c["out_dim"] > 4096 * 22016 or c["in_dim"] * c["parts"] * c["rank"] * c["adapters"] > 40 * 2 * 64 * 4096:
            c["in_dim"] = max(256, c["in_dim"] // 16 * 8)
            c["adapters"] = max(1, c["adapters"] // 2)
            c["used"] = min(c["used"], c["adapters"])
        while c["rows"] * c["rank"] * max(c["out_dim"], c["parts"] * c["in_dim"]) > 256 * 22016 * 64:
            c["rows"] = max(1, c["rows"] // 2)
            c["bare"] = min(c["bare"], c["rows"] // 3)
        return c
    c = dict(kind=kind, d=rng.choice([64, 128, 128]), lens_seed=rng.randrange(1 << 20), hkv=_log(rng, 1, 32))
    group = rng.choice([1, 1, 2, 4, 8])
    while c["hkv"] * group > 64:
        c["hkv"] //= 2
    c["hq"] = c["hkv"] * group
    c["layers"], c["batch"], c["hi"] = rng.randint(1, 4), _log(rng, 1, 256), _log(rng, 32, 32768)
    if kind == "park":
        c["batch"] = min(c["batch"], 32)
        c["n"] = rng.randint(1, min(c["batch"], 16))
    else:
        c["law"] = rng.choice(["uniform", "uniform", "lognormal", "skew"])
        c["free"] = rng.randint(0, c["batch"] // 4)
        c["turn"] = rng.randint(1, max(1, (c["batch"] - c["free"]) // 16))
    cells = lambda: c["layers"] * c["batch"] * c["hkv"] * c["hi"] * c["d"]  # noqa: E731
    while cells() > 2 * 64 * 8 * 8192 * 128 and c["hi"] > 32:
        c["hi"] = max(32, c["hi"] // 2)
    c["lo"] = max(1, c["hi"] // 16)
    return c


# ------------------------------------------------------------ the schedule --
def lengths(c):
    """Tokens of each of the batch's queries."""
    r = random.Random(c["lens_seed"])
    lo, hi, n = c["lo"], c["hi"], c["n"] if c["kind"] == "park" else c["batch"] - c["free"]
    law = c.get("law", "uniform")
    if law == "lognormal":
        lens = [int(min(hi, max(lo, round(r.lognormvariate(math.log(max(2, hi / 6)), 0.8))))) for _ in range(n)]
    elif law == "skew":   # a tenth of the rows long
        long = set(r.sample(range(n), max(1, n // 10)))
        lens = [r.randint(hi // 2, hi) if b in long else r.randint(min(lo, hi), max(lo, hi // 32)) for b in range(n)]
    else:
        lens = [r.randint(lo, hi) for _ in range(n)]
    lens[max(range(n), key=lambda b: lens[b])] = hi
    return lens


def turnover(c, i):
    """(slots, queries) replaced in pass i (from 0)."""
    n, k = c["batch"] - c["free"], c["turn"]
    at = [i * k + j for j in range(k)]
    return [a % n for a in at], [(a % n + a // n + 1) % n for a in at]


def capacity(c):
    period = -(-(c["batch"] - c["free"]) // c["turn"]) if c["kind"] == "step" else 1
    return -(-(c["hi"] + period + 2) // 16) * 16


# -------------------------------------------------------------- the inputs --
def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed(seed * 1009 + salt)


def _randn(g, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _sources(c, lens, g):
    """Keys and values of the queries, [layers][hkv][len][d] bf16: normal, the
    keys with some channels several times as large as the others."""
    gain = torch.exp(0.5 * torch.randn((c["hkv"], 1, c["d"]), generator=g, device="cuda")).to(torch.bfloat16)
    ks = [_randn(g, c["layers"], c["hkv"], n, c["d"]) * gain for n in lens]
    vs = [_randn(g, c["layers"], c["hkv"], n, c["d"]) for n in lens]
    return ks, vs


def _cache(c):
    from paper_2410_18701_amd.cache import BatonCache
    return BatonCache(c["layers"], c["batch"], c["hq"], c["hkv"], c["d"], capacity(c), dtype="mxfp4")


def _store(c):
    """The plain form's cache: codes and exponents of K and V, left-aligned rows."""
    shape = (c["layers"], c["batch"], c["hkv"], capacity(c))
    codes = [torch.zeros(shape + (c["d"],), dtype=torch.int8, device="cuda") for _ in range(2)]
    exps = [torch.zeros(shape + (c["d"] // BLOCK,), dtype=torch.int16, device="cuda") for _ in range(2)]
    return dict(codes=codes, exps=exps, lens=torch.zeros(c["batch"], dtype=torch.int64, device="cuda"))


def _ids(c):
    """The adapter of each row (-1: none), in no order."""
    r = random.Random(c["ids_seed"])
    pool = r.sample(range(c["adapters"]), c["used"])
    ids = [r.choice(pool) for _ in range(c["rows"])]
    for b in r.sample(range(c["rows"]), c["bare"]):
        ids[b] = -1
    return ids


def _params(c):
    """Each row's temperature, top_k, top_p and min_p, as requests give them."""
    r, n, mode = random.Random(c["params_seed"]), c["rows"], c["mode"]
    temperature, top_k, top_p, min_p = [], [], [], []
    for _ in range(n):
        how = r.choice(["greedy", "plain", "top_k", "top_p", "min_p", "all", "all"]) if mode == "mixed" else mode
        temperature.append(0.0 if how == "greedy" else r.choice([0.3, 0.7, 1.0, 1.0, 1.5]))
        top_k.append(r.choice([1, 5, 40, 50, 100, 1000]) if how in ("top_k", "all") else 0)
        top_p.append(r.choice([0.1, 0.5, 0.8, 0.9, 0.95, 0.99]) if how in ("top_p", "all") else 1.0)
        min_p.append(r.choice([0.01, 0.05, 0.1]) if how in ("min_p", "all") else 0.0)
    f = lambda v, t=torch.float32: torch.tensor(v, dtype=t, device="cuda")  # noqa: E731
    return dict(temperature=f(temperature), top_k=f(top_k, torch.int32), top_p=f(top_p), min_p=f(min_p))


def prepare(case, seed):
    c = case
    if c["kind"] == "sample":
        g = _gen(seed, 3)
        logits = c["spread"] * torch.randn((c["rows"], c["vocab"]), generator=g, device="cuda")
        logits = logits.to(torch.bfloat16 if c["dtype"] == "bf16" else torch.float32)
        s = dict(c=c, logits=logits, u=torch.rand(c["rows"], generator=g, device="cuda"), **_params(c))
        if own:
            from paper_2410_18701_amd.layer import Sampler
            s["sampler"] = Sampler(c["rows"], c["vocab"])
        return s
    if c["kind"] in ("adapters", "proj"):
        g = _gen(seed, 2)
        n, r, i, o = c["adapters"], c["rank"], c["in_dim"], c["out_dim"]
        s = dict(c=c, ids=_ids(c), x=_randn(g, c["rows"], i), a=_randn(g, n, c["parts"] * r, i) * 2.0 ** -6,
                 b=_randn(g, n, o, r) * 2.0 ** -3, scales=[0.5 + (k % 7) / 4 for k in range(n)],
                 y=torch.empty((c["rows"], o), dtype=torch.bfloat16, device="cuda"))
        if c["kind"] == "proj":
            s["w"] = _randn(g, o, i) * 2.0 ** -6
        if own:
            from paper_2410_18701_amd.layer import Adapters, Gemm
            s["gemm"] = Gemm()
            s["adapters"] = Adapters(list(s["a"]), list(s["b"]), s["scales"], parts=[o // c["parts"]] * c["parts"])
            if c["kind"] == "proj":
                s["packed"] = s["gemm"].pack(s["w"])
        return s
    g = _gen(seed, 1)
    lens = lengths(c)
    ks, vs = _sources(c, lens, g)
    s = dict(c=c, lens=lens, ks=ks, vs=vs, i=0)
    s["q"] = _randn(g, c["layers"], c["batch"], c["hq"], c["d"])
    s["k_new"], s["v_new"] = (_randn(g, c["layers"], c["batch"], c["hkv"], c["d"]) for _ in range(2))
    live = list(range(len(lens)))
    if own:
        s["cache"] = _cache(c)
        s["cache"].embed(live, lens, ks, vs)
    else:
        s["store"] = _store(c)
        _embed(s["store"], live, lens, ks, vs)
    return s


# -------------------------------------------------------- the plain forms --
def _quantise(x):
    """bf16 [..., d] -> codes (halves: 0..12, signed) and exponents [..., d / 32]."""
    v = x.to(torch.float32).unflatten(-1, (-1, BLOCK))
    mant, e = torch.frexp(v.abs().amax(-1))                # amax = mant * 2^e, mant in [1/2, 1)
    e = torch.where(mant > 0.875, e - 2, e - 3).clamp(-127, 127)
    e = torch.where(mant == 0, torch.full_like(e, -127), e)
    t = torch.ldexp(v, -e.unsqueeze(-1)).abs()             # exact: a power of two
    step = torch.where(t < 2, 0.5, torch.where(t < 4, 1.0, 2.0))
    t = (torch.round(t / step) * step).clamp(max=6.0)      # round: ties to even
    return (2 * torch.where(v < 0, -t, t)).to(torch.int8).flatten(-2), e.to(torch.int16)


def _values(codes, exps):
    """fp32 values of codes and exponents."""
    v = codes.to(torch.float32).unflatten(-1, (-1, BLOCK))
    return torch.ldexp(v, exps.to(torch.int32).unsqueeze(-1) - 1).flatten(-2)


def _embed(store, slots, lens, ks, vs):
    for b, n, k, v in zip(slots, lens, ks, vs):
        for j, x in enumerate((k, v)):
            store["codes"][j][:, b, :, :n], store["exps"][j][:, b, :, :n] = _quantise(x)
    store["lens"][slots] = torch.tensor(lens, device="cuda")


def _attention(store, layer, q, k_new, v_new):
    """One layer: softmax over the row's cached tokens and the current one, which is then appended."""
    batch, hkv, d = k_new.shape
    lens, cap = store["lens"], store["codes"][0].shape[3]
    k, v = (_values(store["codes"][j][layer], store["exps"][j][layer]) for j in range(2))
    qs = q.to(torch.float32).view(batch, hkv, -1, d) * d ** -0.5
    s = qs @ k.transpose(-1, -2)
    s = s.masked_fill(torch.arange(cap, device="cuda") >= lens[:, None, None, None], -math.inf)
    s = torch.cat([s, (qs * k_new.to(torch.float32).unsqueeze(2)).sum(-1, keepdim=True)], -1)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    out = p[..., :cap] @ v + p[..., cap:] * v_new.to(torch.float32).unsqueeze(2)
    out = torch.where(lens[:, None, None, None] > 0, out, 0.0)   # a free slot's row
    at = torch.arange(batch, device="cuda")
    for j, x in enumerate((k_new, v_new)):
        store["codes"][j][layer, at, :, lens], store["exps"][j][layer, at, :, lens] = _quantise(x)
    return out.to(q.dtype).view_as(q)


def _adapters(c, x, a, b, scales, ids):
    """fp32 [rows][out]: each row's scale * (x . A^T) . B^T, part by part of the output; 0 without an adapter."""
    at = torch.tensor(ids, device="cuda")
    f = torch.where(at >= 0, torch.tensor(scales, device="cuda")[at], 0.0)
    h = torch.bmm(a[at].float(), x.float().unsqueeze(2)).view(-1, c["parts"], c["rank"], 1)
    w = b[at].float().view(len(ids), c["parts"], -1, c["rank"])
    return torch.matmul(w, h).flatten(1) * f[:, None]


def _sample(logits, u, temperature, top_k, top_p, min_p):
    """The plain form in 64 bits: sort, three prefixes of the sorted order, inversion in vocabulary order."""
    n = logits.shape[1]
    l, order = torch.sort(logits.double(), dim=1, descending=True, stable=True)
    greedy = temperature <= 0
    t = torch.where(greedy, 1.0, temperature).double()[:, None]
    w = torch.exp((l - l[:, :1]) / t)
    place = torch.arange(n, device="cuda")
    k = torch.where((top_k <= 0) | (top_k > n), n, top_k)[:, None]
    w = torch.where(place < k, w, 0.0)
    before = torch.cumsum(w, 1) - w                              # weight of the tokens in front
    p = top_p.double()[:, None]
    keep = (place < k) & ((before < p * w.sum(1, keepdim=True)) | (p >= 1) | (place == 0))
    keep &= (w >= min_p.double()[:, None]) | (place == 0)
    keep &= ~greedy[:, None] | (place == 0)
    w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0))
    c = torch.cumsum(w, 1)
    target = u.double()[:, None] * c[:, -1:]
    return (c <= target).sum(1).clamp(max=n - 1).to(torch.int32)


def run(s):
    c = s["c"]
    if c["kind"] == "sample":
        args = (s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
        return s["sampler"](*args) if own else _sample(*args)
    if c["kind"] in ("adapters", "proj"):
        if own:
            if c["kind"] == "proj":
                s["gemm"].linear_packed(s["x"], s["packed"], s["y"])
            return s["gemm"].linear_adapters(s["x"], s["adapters"], s["ids"], s["y"], accumulate=c["kind"] == "proj")
        y = _adapters(c, s["x"], s["a"], s["b"], s["scales"], s["ids"])
        if c["kind"] == "proj":
            y += s["x"].float() @ s["w"].float().t()
        return y.to(torch.bfloat16)
    if c["kind"] == "park":
        slots = list(range(len(s["lens"])))
        if own:
            s["cache"].evict(slots)
            s["cache"].embed(slots, s["lens"], s["ks"], s["vs"])
            ks, vs = s["cache"].extract(slots)
            return ks + vs
        _embed(s["store"], slots, s["lens"], s["ks"], s["vs"])
        return [_values(s["store"]["codes"][j][:, b, :, :n], s["store"]["exps"][j][:, b, :, :n]).to(torch.bfloat16)
                for j in range(2) for b, n in enumerate(s["lens"])]
    slots, queries = turnover(c, s["i"])
    s["i"] += 1
    lens, ks, vs = ([x[q] for q in queries] for x in (s["lens"], s["ks"], s["vs"]))
    if own:
        cache = s["cache"]
        cache.evict(slots)
        cache.embed(slots, lens, ks, vs)
        out = [cache.decode_attn(l, s["q"][l], s["k_new"][l], s["v_new"][l]) for l in range(c["layers"])]
        cache.advance()
        return out
    _embed(s["store"], slots, lens, ks, vs)
    out = [_attention(s["store"], l, s["q"][l], s["k_new"][l], s["v_new"][l]) for l in range(c["layers"])]
    s["store"]["lens"] += (s["store"]["lens"] > 0).long()
    return out


# ------------------------------------------------------------------- work --
def work(case):
    c = case
    if c["kind"] == "sample":
        n = c["rows"] * c["vocab"]
        return {"bytes": n * (2 if c["dtype"] == "bf16" else 4) + 24 * c["rows"], "flops": 2 * n}
    if c["kind"] in ("adapters", "proj"):
        ids = _ids(c)
        rows, n = sum(i >= 0 for i in ids), len({i for i in ids if i >= 0})
        per = c["parts"] * c["rank"] * c["in_dim"] + c["rank"] * c["out_dim"]
        shared = c["in_dim"] * c["out_dim"] if c["kind"] == "proj" else 0
        return {"bytes": 2 * (n * per + shared + c["rows"] * (c["in_dim"] + c["out_dim"])),
                "flops": 2 * (rows * per + c["rows"] * shared)}
    lens = lengths(c)
    vec = c["layers"] * c["hkv"] * c["d"]           # elements of K of one token
    four = 2 * vec * (1 / 2 + 1 / BLOCK)            # bytes of K and V of one token in 4 bits
    if c["kind"] == "park":   # sources read, the cache written and read, the copies written
        return {"bytes": sum(lens) * (2 * 4 * vec + 2 * four), "flops": sum(lens) * 6 * vec}
    mean = sum(lens) / len(lens)
    live = len(lens)
    heads = c["layers"] * c["hq"] * c["d"]
    return {"bytes": c["turn"] * mean * (4 * vec + four) + (sum(lens) + live) * four + live * 4 * vec
            + 4 * heads * c["batch"], "flops": 4 * heads * (sum(lens) + live)}


# ------------------------------------------------------------------ exact --
_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _stored(x):
    """64-bit values that the 4-bit form holds for x, from its definition."""
    v = x.double().reshape(-1, BLOCK)
    a = v.abs().amax(1, keepdim=True).clamp(min=2.0 ** -124)
    e = torch.ceil(torch.log2(a / 7)).clamp(-127, 127)       # the smallest with a <= 7 * 2^e ...
    e = torch.where(a > 7 * 2.0 ** e, e + 1, torch.where(a <= 7 * 2.0 ** (e - 1), e - 1, e))   # ... whatever log2 rounds
    t = v.abs() / 2.0 ** e
    r = torch.zeros_like(t)
    for j in range(1, 8):   # past the middle of two grid values, or on it where the upper code is even
        mid = (_GRID[j - 1] + _GRID[j]) / 2
        r = torch.where(t >= mid if j % 2 == 0 else t > mid, _GRID[j], r)
    return (torch.sign(v) * r * 2.0 ** e).view(x.shape)


def exact(case, seed):
    c = case
    if c["kind"] == "sample":
        return None
    if c["kind"] in ("adapters", "proj"):
        g = _gen(seed, 2)
        n, r, i, o, parts = c["adapters"], c["rank"], c["in_dim"], c["out_dim"], c["parts"]
        x, a, b = _randn(g, c["rows"], i).double(), _randn(g, n, parts * r, i) * 2.0 ** -6, _randn(g, n, o, r) * 2.0 ** -3
        y = torch.zeros((c["rows"], o), dtype=torch.float64, device="cuda")
        if c["kind"] == "proj":
            y += x @ (_randn(g, o, i) * 2.0 ** -6).double().t()
        ids = _ids(c)
        for k in sorted(set(ids) - {-1}):
            rows = [row for row, i_ in enumerate(ids) if i_ == k]
            for p in range(parts):
                h = x[rows] @ a[k, p * r:(p + 1) * r].double().t()
                cols = slice(p * o // parts, (p + 1) * o // parts)
                y[rows, cols] += (0.5 + (k % 7) / 4) * (h @ b[k, cols].double().t())
        return y
    g = _gen(seed, 1)
    lens = lengths(c)
    ks, vs = _sources(c, lens, g)
    if c["kind"] == "park":
        return [_stored(x) for x in ks + vs]
    q = _randn(g, c["layers"], c["batch"], c["hq"], c["d"]).double()
    k_new, v_new = (_randn(g, c["layers"], c["batch"], c["hkv"], c["d"]).double() for _ in range(2))
    at = {b: b for b in range(len(lens))}
    at.update(zip(*turnover(c, 0)))
    out = torch.zeros_like(q)
    for b, j in at.items():
        k = torch.cat([_stored(ks[j]), k_new[:, b].unsqueeze(2)], 2)
        v = torch.cat([_stored(vs[j]), v_new[:, b].unsqueeze(2)], 2)
        s = torch.matmul(q[:, b].unflatten(1, (c["hkv"], -1)), k.mT.contiguous()) / math.sqrt(c["d"])
        out[:, b] = torch.matmul(torch.softmax(s, -1), v).flatten(1, 2)
    return list(out)
