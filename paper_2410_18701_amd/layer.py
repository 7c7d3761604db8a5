"""A whole decode layer around the re-batched attention, as C-ABI calls.

Each method is argument marshalling for one libbaton call (paper_2410_18701_amd/
baton.py); PyTorch provides the buffers.  The layer is the paper's model's
(llama2-7b, sec. 5): RMS norm -> fused QKV projection -> rotary embedding at
each query's token count -> re-batched attention (BatonCache.decode_attn) ->
output projection added to the residual stream -> RMS norm -> gate/up
projection -> silu(gate) * up -> down projection added to the residual stream.
What each query of the batch brings of its own joins it: low-rank adapters
beside the projections, and its sampling parameters for the next token.
"""
import ctypes

from . import baton as B
from .cache import _cur_device, _cur_stream as _stream


def _on_this_gpu(what, *tensors):
    """The calls go to the current device's stream: tensors elsewhere are refused."""
    here = _cur_device()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError(f"{what}: a tensor on {t.device}, the current device is cuda:{here}")


class PackedWeight:
    """A weight in the packed form baton_linear_packed reads."""

    def __init__(self, data, out_dim, in_dim):
        self.data, self.out_dim, self.in_dim = data, out_dim, in_dim


class Adapters:
    """Low-rank adapters of one projection: a[i] [parts * rank_i][in], b[i] [out][rank_i]
    bf16 tensors, scales[i]; parts: the widths of the output's parts when the projection
    is fused along its outputs (query, key and value; gate and up), each with rows of a
    of its own.  The tensors are used in place."""

    def __init__(self, a, b, scales, parts=None):
        import torch
        if not len(a) == len(b) == len(scales):
            raise ValueError("Adapters: a, b and scales need the same length")
        self.a, self.b, self.n = list(a), list(b), len(a)
        self.parts = None if parts is None else (ctypes.c_int32 * len(parts))(*[int(p) for p in parts])
        n_parts = self.n_parts = 1 if parts is None else len(self.parts)
        self.max_rank = max((t.shape[1] for t in self.b), default=0)
        self.table = (B.baton_adapter * max(1, self.n))()
        for i, (ai, bi, s) in enumerate(zip(self.a, self.b, scales)):
            if ai.shape[0] != n_parts * bi.shape[1] or ai.shape[1] != self.a[0].shape[1] or \
                    bi.shape[0] != self.b[0].shape[0]:
                raise ValueError(f"Adapters: shapes of adapter {i} do not match")
            for t in (ai, bi):
                if t.dtype != torch.bfloat16 or not t.is_contiguous():
                    raise ValueError("Adapters: contiguous bf16 tensors only")
                if t.device != self.a[0].device:
                    raise ValueError("Adapters: tensors on different devices")
            self.table[i] = B.baton_adapter(ai.data_ptr(), bi.data_ptr(), bi.shape[1], float(s))
        self.in_dim = self.a[0].shape[1] if self.n else None
        self.out_dim = self.b[0].shape[0] if self.n else None
        if self.n and parts is not None and sum(self.parts) != self.out_dim:
            raise ValueError("Adapters: parts do not add up to the output")


class Gemm:
    """The device workspace of the projections (the partial sums of
    baton_linear_packed when it splits along in_dim), and the projection calls."""

    def __init__(self, ws_bytes=32 << 20):
        import torch
        self.ws = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda") if ws_bytes else None
        self.ws_bytes = ws_bytes

    def pack(self, w):
        """The packed form of a weight w [out][in] for linear_packed (made once per weight)."""
        import torch
        out_dim, in_dim = w.shape
        if not w.is_contiguous():
            raise ValueError("pack: contiguous tensors only")
        wp = torch.empty(B.baton_linear_packed_bytes(out_dim, in_dim) // 2, dtype=w.dtype, device=w.device)
        B.baton_linear_pack(B.BATON_BF16, w, wp, out_dim, in_dim, _stream())
        return PackedWeight(wp, out_dim, in_dim)

    def linear_packed(self, x, wp, y, accumulate=False):
        """y (+)= x . w^T with w packed by pack(); x [rows <= 256][in], y [rows][out]."""
        rows, in_dim = x.shape
        if in_dim != wp.in_dim or tuple(y.shape) != (rows, wp.out_dim):
            raise ValueError("linear_packed: shapes do not match")
        for t in (x, y):
            if not t.is_contiguous():
                raise ValueError("linear_packed: contiguous tensors only")
        B.baton_linear_packed(B.BATON_BF16, x, wp.data, y, rows, wp.out_dim, in_dim, accumulate, self.ws,
                              self.ws_bytes, _stream())
        return y

    def linear_packed_silu(self, x, wp, out):
        """out = silu(x . gate^T) * (x . up^T) for the packed [gate; up] weight wp
        (bit for bit linear_packed unsplit, then silu_mul, in one kernel)."""
        rows, in_dim = x.shape
        if in_dim != wp.in_dim or tuple(out.shape) != (rows, wp.out_dim // 2):
            raise ValueError("linear_packed_silu: shapes do not match")
        for t in (x, out):
            if not t.is_contiguous():
                raise ValueError("linear_packed_silu: contiguous tensors only")
        B.baton_linear_packed_silu(B.BATON_BF16, x, wp.data, out, rows, wp.out_dim, in_dim, _stream())
        return out

    def linear_packed_rmsnorm(self, x, wp, y, gain, eps, y_norm, accumulate=False):
        """linear_packed, then y_norm = rmsnorm(y, gain, eps) (bit for bit; one
        kernel adds the split sums and normalises when the product splits)."""
        rows, in_dim = x.shape
        if in_dim != wp.in_dim or tuple(y.shape) != (rows, wp.out_dim) or tuple(y_norm.shape) != tuple(y.shape) \
                or gain.numel() != wp.out_dim:
            raise ValueError("linear_packed_rmsnorm: shapes do not match")
        for t in (x, y, y_norm, gain):
            if not t.is_contiguous():
                raise ValueError("linear_packed_rmsnorm: contiguous tensors only")
        B.baton_linear_packed_rmsnorm(B.BATON_BF16, x, wp.data, y, rows, wp.out_dim, in_dim, accumulate, gain,
                                      eps, y_norm, self.ws, self.ws_bytes, _stream())
        return y

    def linear_adapters(self, x, adapters, row_adapter, y, accumulate=False):
        """y (+)= each row's low-rank product with its adapter: x [rows <= 256][in], y [rows][out],
        row_adapter a list of rows indices into adapters (-1: none)."""
        import torch
        rows, in_dim = x.shape
        if y.shape[0] != rows or y.dim() != 2 or len(row_adapter) != rows or \
                (adapters.n and (in_dim != adapters.in_dim or y.shape[1] != adapters.out_dim)):
            raise ValueError("linear_adapters: shapes do not match")
        for t in (x, y):
            if not t.is_contiguous() or t.dtype != torch.bfloat16:
                raise ValueError("linear_adapters: contiguous bf16 tensors only")
        if rows * adapters.n_parts * adapters.max_rank * 4 > self.ws_bytes:   # these rows may have smaller ranks
            rank = max((adapters.b[i].shape[1] for i in row_adapter if 0 <= i < adapters.n), default=0)
            need = B.baton_linear_adapters_workspace_bytes(rows, adapters.n_parts, rank)
            if need > self.ws_bytes:
                raise ValueError(f"linear_adapters: rank {rank} needs a workspace of {need} bytes, the Gemm has "
                                 f"{self.ws_bytes}")
        _on_this_gpu("linear_adapters", x, y, self.ws, *adapters.a[:1])
        B.baton_linear_adapters(B.BATON_BF16, x, adapters.table, adapters.n, row_adapter, y, rows, y.shape[1], in_dim,
                                adapters.parts, adapters.n_parts, accumulate, self.ws, self.ws_bytes, _stream())
        return y

    def close(self):
        self.ws = None


def rmsnorm(x, gain, y, eps):
    rows, dim = x.shape
    if tuple(y.shape) != (rows, dim) or gain.numel() != dim:
        raise ValueError("rmsnorm: shapes do not match")
    B.baton_rmsnorm(B.BATON_BF16, x, gain, y, rows, dim, eps, _stream())
    return y


def silu_mul(gate_up, out):
    rows, two_f = gate_up.shape
    if tuple(out.shape) != (rows, two_f // 2):
        raise ValueError("silu_mul: shapes do not match")
    B.baton_silu_mul(B.BATON_BF16, gate_up, out, rows, two_f // 2, _stream())
    return out


def rope_qkv(cache, qkv, q, k_new, v_new, theta):
    """Of a PagedCache, qkv has its width's rows per slot."""
    paged = hasattr(cache, "desc")
    rows = cache.batch * (cache.width if paged else 1)
    width = (cache.n_q_heads + 2 * cache.n_kv_heads) * cache.head_dim
    if tuple(qkv.shape) != (rows, width):
        raise ValueError("rope_qkv: qkv must be [batch][(Hq + 2 Hkv) * head_dim]")
    if q.numel() != rows * cache.n_q_heads * cache.head_dim or \
            k_new.numel() != rows * cache.n_kv_heads * cache.head_dim or v_new.numel() != k_new.numel():
        raise ValueError("rope_qkv: output sizes do not match the cache")
    if paged:
        B.baton_paged_rope_qkv(cache.desc, qkv, cache.width, q, k_new, v_new, theta, _stream())
    else:
        B.baton_rope_qkv(cache.handle, qkv, q, k_new, v_new, theta, _stream())


class Sampler:
    """One token per row of logits, with each row's own parameters (device tensors of
    rows entries, or None) and uniform random numbers u.  The tokens, int32 [rows],
    are written to the same tensor by every call."""

    def __init__(self, rows, vocab):
        import torch
        self.rows, self.vocab = rows, vocab
        self.tokens = torch.empty(rows, dtype=torch.int32, device="cuda")

    def __call__(self, logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
        """logits [rows][vocab], fp32 or bf16, rows any distance apart."""
        import torch
        if tuple(logits.shape) != (self.rows, self.vocab) or (self.vocab > 1 and logits.stride(1) != 1):
            raise ValueError("Sampler: logits must be [rows][vocab], each row dense")
        dtype = {torch.float32: B.BATON_F32, torch.bfloat16: B.BATON_BF16}.get(logits.dtype)
        if dtype is None:
            raise ValueError("Sampler: fp32 or bf16 logits")
        for name, t, want in (("u", u, torch.float32), ("temperature", temperature, torch.float32),
                              ("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32),
                              ("min_p", min_p, torch.float32)):
            if t is None and name != "u":
                continue
            if t.dtype != want or t.numel() != self.rows or not t.is_contiguous():
                raise ValueError(f"Sampler: {name} must be {self.rows} contiguous {want} values")
        _on_this_gpu("Sampler", self.tokens, logits, u, temperature, top_k, top_p, min_p)
        ld = logits.stride(0) if self.rows > 1 else self.vocab
        B.baton_sample(dtype, logits, ld, self.rows, self.vocab, temperature, top_k, top_p, min_p, u, self.tokens,
                       _stream())
        return self.tokens


class Verifier:
    """Drafted tokens against the target's logits: which are accepted, and the token behind
    them.  Both results are written to the same tensors by every call: tokens, int32
    [batch][width], the accepted drafts and the token drawn, -1 behind; n_out, int32 [batch],
    their number (0 of a free slot), which is PagedCache.begin's keep."""

    def __init__(self, batch, width, vocab):
        import torch
        self.batch, self.width, self.vocab = batch, width, vocab
        self.ws_bytes = B.baton_verify_workspace_bytes(batch, width, vocab)
        if self.ws_bytes == 0:
            raise ValueError("Verifier: sizes out of range")
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device="cuda")
        self.tokens = torch.empty((batch, width), dtype=torch.int32, device="cuda")
        self.n_out = torch.empty(batch, dtype=torch.int32, device="cuda")

    def _rows(self, what, t, n):
        """The distance of the rows of t [batch][n][vocab], which may be any but the same throughout."""
        b = self.batch
        if tuple(t.shape) != (b, n, self.vocab) or (self.vocab > 1 and t.stride(2) != 1) or \
                (b > 1 and n > 1 and t.stride(0) != n * t.stride(1)):
            raise ValueError(f"Verifier: {what} must be [batch][{n}][vocab], rows dense and evenly apart")
        return t.stride(1) if n > 1 else t.stride(0) if b > 1 else self.vocab

    def __call__(self, target, draft, drafted, n_draft, u_accept, u_token, temperature=None, top_k=None, top_p=None,
                 min_p=None, cache=None):
        """target [batch][width][vocab], draft [batch][width - 1][vocab] (or None: the drafts are
        tokens without a distribution), fp32 or bf16; drafted int32 and u_accept [batch][width - 1];
        n_draft int32 [batch] (None: all; negative: a free slot); u_token [batch].  cache: the
        PagedCache whose present step the drafts belong to, of which slots that took no part in
        it (they lacked pages) are free ones, and others have at most the drafts that it took."""
        import torch
        b, w = self.batch, self.width
        dtype = {torch.float32: B.BATON_F32, torch.bfloat16: B.BATON_BF16}.get(target.dtype)
        if dtype is None or (draft is not None and draft.dtype != target.dtype):
            raise ValueError("Verifier: fp32 or bf16 logits, target and draft alike")
        target_ld = self._rows("target", target, w)
        if w == 1:
            draft = drafted = u_accept = None
        draft_ld = self._rows("draft", draft, w - 1) if draft is not None else 0
        f32, i32 = torch.float32, torch.int32
        for name, t, want, n, needed in (
                ("drafted", drafted, i32, b * (w - 1), w > 1), ("u_accept", u_accept, f32, b * (w - 1), w > 1),
                ("u_token", u_token, f32, b, True), ("n_draft", n_draft, i32, b, False),
                ("temperature", temperature, f32, b, False), ("top_k", top_k, i32, b, False),
                ("top_p", top_p, f32, b, False), ("min_p", min_p, f32, b, False)):
            if t is None and not needed:
                continue
            if t is None or t.dtype != want or t.numel() != n or not t.is_contiguous():
                raise ValueError(f"Verifier: {name} must be {n} contiguous {want} values")
        if cache is not None and cache.batch != b:
            raise ValueError(f"Verifier: a cache of {cache.batch} slots, not {b}")
        _on_this_gpu("Verifier", self.ws, target, draft, drafted, n_draft, u_accept, u_token, temperature, top_k, top_p,
                     min_p, None if cache is None else cache.lens)
        rest = (w, self.vocab, drafted, n_draft, u_accept, u_token, temperature, top_k, top_p, min_p, self.tokens,
                self.n_out, self.ws, self.ws_bytes, _stream())
        if cache is None:
            B.baton_verify(dtype, target, target_ld, draft, draft_ld, b, *rest)
        else:
            B.baton_paged_verify(cache.desc, dtype, target, target_ld, draft, draft_ld, *rest)
        return self.tokens, self.n_out


class DecodeLayers:
    """The layers of one model over one BatonCache, or over one PagedCache, whose steps have
    its width's rows for each slot (x [batch * width][hid]: the next token and drafted ones
    behind it; batch * width <= 256), with preallocated activations.

    weights[layer]: dict of bf16 device tensors norm1 [hid], qkv [(Hq + 2 Hkv) D][hid],
    o [hid][Hq D], norm2 [hid], gate_up [2 F][hid], down [hid][F].  The projections
    run on the weight-streaming GEMM over packed copies of the weights, made here
    once.  Each residual add is fused with the normalisation that follows it (the
    output projection with norm2, the down projection with the next layer's
    norm1), so layer(l + 1) expects x as layer(l) returned it, and the gate/up
    projection with the gated activation.

    adapters[layer]: dict from names of PROJ to Adapters (qkv in parts [Hq D, Hkv D,
    Hkv D], gate_up in [F, F], the same adapter at the same index everywhere);
    slot_adapter[slot] is the index its query uses, -1 for none, and may be changed
    between steps (a captured step keeps the indices that it was captured with).  head: dict
    of norm [hid] and out [vocab][hid] (vocab a multiple of 8), for next_tokens, or
    accept_drafts over a PagedCache."""

    PROJ = ("qkv", "o", "gate_up", "down")

    def __init__(self, cache, weights, gemm, theta=10000.0, eps=1e-5, adapters=None, head=None):
        import torch
        self.cache, self.w, self.gemm, self.theta, self.eps = cache, weights, gemm, theta, eps
        Hq, Hkv, D = cache.n_q_heads, cache.n_kv_heads, cache.head_dim
        self.width = getattr(cache, "width", 1)
        Bt = cache.batch * self.width
        if Bt > B.BATON_GEMM_MAX_ROWS:
            raise ValueError(f"at most {B.BATON_GEMM_MAX_ROWS} slots (times their new tokens)")
        self.wp = [{k: gemm.pack(w[k]) for k in self.PROJ} for w in weights]
        hid = weights[0]["norm1"].numel()
        F = weights[0]["down"].shape[1]
        e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
        self.h, self.qkv = e(Bt, hid), e(Bt, (Hq + 2 * Hkv) * D)
        self.q, self.k, self.v, self.att = e(Bt, Hq, D), e(Bt, Hkv, D), e(Bt, Hkv, D), e(Bt, Hq, D)
        self.gu, self.act = e(Bt, 2 * F), e(Bt, F)
        self._normed = None   # (layer, x) whose norm1 input h already holds
        if adapters is not None and (len(adapters) != len(weights) or any(set(a) - set(self.PROJ) for a in adapters)):
            raise ValueError(f"adapters: one dict over {self.PROJ} per layer")
        self.adapters, self.slot_adapter = adapters, [-1] * cache.batch
        self.head = None
        if head is not None:
            vocab = head["out"].shape[0]
            self.head, self.head_norm = gemm.pack(head["out"]), head["norm"]
            self.logits = e(Bt, vocab)
            self.sampler = Sampler(Bt, vocab) if self.width == 1 else None
            self.verifier = Verifier(cache.batch, self.width, vocab) if hasattr(cache, "desc") else None

    def _adapt(self, layer, proj, x, y):
        """y += the low-rank products of the slots with an adapter of this projection."""
        ad = self._adapter(layer, proj)
        if ad is not None:
            rows = self.slot_adapter if self.width == 1 else [i for i in self.slot_adapter for _ in range(self.width)]
            self.gemm.linear_adapters(x, ad, rows, y, accumulate=True)

    def _adapter(self, layer, proj):
        return None if self.adapters is None or max(self.slot_adapter) < 0 else self.adapters[layer].get(proj)

    def layer(self, layer, x):
        """One layer of the decode step on the residual stream x [batch][hid] (a PagedCache:
        [batch * width][hid]; in place)."""
        w, wp, g = self.w[layer], self.wp[layer], self.gemm
        if self._normed != (layer, x.data_ptr()):   # h holds norm1(x) after the previous layer
            rmsnorm(x, w["norm1"], self.h, self.eps)
        self._normed = None
        g.linear_packed(self.h, wp["qkv"], self.qkv)
        self._adapt(layer, "qkv", self.h, self.qkv)
        rope_qkv(self.cache, self.qkv, self.q, self.k, self.v, self.theta)
        self.cache.decode_attn(layer, self.q, self.k, self.v, out=self.att)
        att = self.att.view(self.att.shape[0], -1)
        self._adapt(layer, "o", att, x)   # before the projection, whose sum the norm then takes
        g.linear_packed_rmsnorm(att, wp["o"], x, w["norm2"], self.eps, self.h, accumulate=True)
        if wp["gate_up"].out_dim % 32 == 0 and self._adapter(layer, "gate_up") is None:
            g.linear_packed_silu(self.h, wp["gate_up"], self.act)
        else:
            g.linear_packed(self.h, wp["gate_up"], self.gu)
            self._adapt(layer, "gate_up", self.h, self.gu)
            silu_mul(self.gu, self.act)
        self._adapt(layer, "down", self.act, x)
        if layer + 1 < len(self.w):
            g.linear_packed_rmsnorm(self.act, wp["down"], x, self.w[layer + 1]["norm1"], self.eps, self.h,
                                    accumulate=True)
            self._normed = (layer + 1, x.data_ptr())
        else:
            g.linear_packed(self.act, wp["down"], x, accumulate=True)
        return x

    def next_tokens(self, x, u, temperature=None, top_k=None, top_p=None, min_p=None):
        """The next token of every slot (int32 [batch], the Sampler's own tensor; a free
        slot's, or one's that lacked pages, says nothing) from the last layer's residual stream x [batch][hid]: norm,
        vocabulary projection, sampling with each slot's parameters and random number u."""
        if self.head is None or self.sampler is None:
            raise ValueError("next_tokens: no head was given" if self.head is None else
                             "next_tokens: one new token per slot (accept_drafts takes several)")
        return self.sampler(self._logits(x), u, temperature, top_k, top_p, min_p)

    def _logits(self, x):
        rmsnorm(x, self.head_norm, self.h, self.eps)
        self._normed = None
        return self.gemm.linear_packed(self.h, self.head, self.logits)

    def accept_drafts(self, x, draft, drafted, n_draft, u_accept, u_token, temperature=None, top_k=None, top_p=None,
                      min_p=None):
        """Over a PagedCache: the drafted tokens that are accepted and the token behind them
        (tokens [batch][width], n_out [batch], the Verifier's own tensors) from the last layer's
        residual stream x [batch * width][hid], whose row b width + i belongs to slot b's i-th
        new token; the other arguments as Verifier's.  n_out is the next begin's keep: 0, with no
        tokens, of a slot that took no part in the step, which brings its tokens again once
        the pool has pages."""
        if self.head is None or self.verifier is None:
            raise ValueError("accept_drafts: no head was given" if self.head is None else "accept_drafts: a PagedCache only")
        logits = self._logits(x).view(self.cache.batch, self.width, -1)
        return self.verifier(logits, draft, drafted, n_draft, u_accept, u_token, temperature, top_k, top_p, min_p,
                             cache=self.cache)
