"""PagedCache: a KV cache in pages of one pool, whose lengths live on the GPU.

Beside BatonCache (cache.py), for steps with drafted tokens: how many of a
step's new tokens stay is a device tensor (layer.Verifier's n_out), so steps
are enqueued, or captured into a graph, without the host knowing lengths.
PyTorch provides device memory and the stream; every operation is one call of
the C ABI (paper_2410_18701_amd/baton.py).
"""
from . import baton as B
from .cache import _cur_stream, torch_dtype
from .layer import _on_this_gpu


class PagedCache:
    """`batch` slots over `n_pages` pages of `page` tokens, at most max_pages of them a
    slot's; steps of up to `width` new tokens per slot.  window: a new token sees the last
    `window` tokens (itself among them) and the first `sinks`; 0: all.

    lens [batch] and table [batch][max_pages] (int32) may be read; slot_map
    [batch][width] holds the places of the step's new tokens, missing [batch] the pages a
    slot lacks (it then takes no part in the step).  order: the pages in the order in
    which they are taken (int32 [n_pages])."""

    def __init__(self, n_layers, batch, n_q_heads, n_kv_heads, head_dim, n_pages, max_pages, page=64, width=1, window=0,
                 sinks=0, dtype="bf16", device="cuda", order=None):
        import torch
        if dtype not in ("f32", "bf16"):
            raise ValueError("PagedCache: f32 or bf16")
        self.dtype, self.io_dtype = dtype, torch_dtype(dtype)
        self.n_layers, self.batch, self.width = n_layers, batch, width
        self.n_q_heads, self.n_kv_heads, self.head_dim = n_q_heads, n_kv_heads, head_dim
        self.page, self.n_pages, self.max_pages, self.window, self.sinks = page, n_pages, max_pages, window, sinks
        self.desc = B.baton_paged_desc(B.BATON_F32 if dtype == "f32" else B.BATON_BF16, n_layers, batch, n_q_heads,
                                       n_kv_heads, head_dim, page, n_pages, max_pages, window, sinks)
        state_bytes = B.baton_paged_state_bytes(self.desc)
        if state_bytes == 0:
            raise ValueError("PagedCache: sizes out of range")
        if not (1 <= width <= B.BATON_PAGED_MAX_WIDTH and width * n_q_heads // n_kv_heads <= B.BATON_PAGED_MAX_ROWS):
            raise ValueError(f"PagedCache: at most {B.BATON_PAGED_MAX_WIDTH} new tokens, {B.BATON_PAGED_MAX_ROWS} with "
                             "the query heads of a kv-head")
        whole = lambda *s: torch.empty(s, dtype=torch.int32, device=device)  # noqa: E731
        # K and V of a layer next to each other
        self.kv = torch.empty((n_layers, 2, n_pages, n_kv_heads, page * head_dim), dtype=self.io_dtype, device=device)
        self.table, self.lens = whole(batch, max_pages), whole(batch)
        self.slot_map, self.missing, self._state = whole(batch, width), whole(batch), whole(state_bytes // 4)
        self._ws_bytes = B.baton_paged_attn_workspace_bytes(self.desc, width)
        self._ws = torch.empty(self._ws_bytes, dtype=torch.uint8, device=device) if self._ws_bytes else None
        d = self.desc
        d.k, d.v = self.kv[:, 0].data_ptr(), self.kv[:, 1].data_ptr()
        d.layer_stride = self.kv.stride(0)
        d.table, d.lens, d.state = (t.data_ptr() for t in (self.table, self.lens, self._state))
        self.reset(order)

    def _numbers(self, what, t, n):
        import torch
        if t.dtype != torch.int32 or t.numel() != n or not t.is_contiguous():
            raise ValueError(f"PagedCache: {what} must be {n} contiguous int32 values")

    def reset(self, order=None):
        """Every slot free, every page in the pool."""
        if order is not None:
            self._numbers("order", order, self.n_pages)
        _on_this_gpu("PagedCache", self.lens, order)
        B.baton_paged_reset(self.desc, order, _cur_stream())

    def begin(self, n_new, keep=None):
        """Ends the last step (keep [batch]: how many of its new tokens stay, of a slot that lacked
        pages none whatever it says, < 0: the query leaves; None: none stay) and begins the next
        with n_new [batch] new tokens; returns slot_map."""
        self._numbers("n_new", n_new, self.batch)
        if keep is not None:
            self._numbers("keep", keep, self.batch)
        _on_this_gpu("PagedCache", self.lens, n_new, keep)
        B.baton_paged_step(self.desc, keep, n_new, self.slot_map, self.width, self.width, self.missing, _cur_stream())
        return self.slot_map

    def _queries(self, what, slots, lens, ks, vs):
        if not len(slots) == len(lens) == len(ks) == len(vs):
            raise ValueError(f"{what}: slots, lens, keys and values must have the same length")
        for n, k, v in zip(lens, ks, vs):
            for t in (k, v):
                if tuple(t.shape) != (self.n_layers, self.n_kv_heads, n, self.head_dim) or t.dtype != self.io_dtype or \
                        not t.is_contiguous():
                    raise ValueError(f"{what}: contiguous [n_layers][n_kv_heads][len][head_dim] tensors of the "
                                     "cache's type")
        _on_this_gpu(what, self.lens, *ks, *vs)

    def embed(self, slots, lens, k_src, v_src):
        """Whole queries, [n_layers][n_kv_heads][len][head_dim], into the pages of a step whose
        n_new are their lengths."""
        self._queries("embed", slots, lens, k_src, v_src)
        B.baton_paged_embed(self.desc, slots, lens, k_src, v_src, _cur_stream())

    def extract(self, slots, lens):
        """The first lens[i] tokens' K and V of the slots as new tensors
        [n_layers][n_kv_heads][len][head_dim] (what is in no page: undefined)."""
        import torch
        ks, vs = ([torch.empty((self.n_layers, self.n_kv_heads, n, self.head_dim), dtype=self.io_dtype,
                               device=self.lens.device) for n in lens] for _ in range(2))
        self._queries("extract", slots, lens, ks, vs)
        B.baton_paged_extract(self.desc, slots, lens, ks, vs, _cur_stream())
        return ks, vs

    def decode_attn(self, layer, q, k_new, v_new, out=None, scale=0.0):
        """Attention of the step's new tokens in one layer; k_new, v_new go into the pages (None,
        None: they are there).  q, out: [batch][width][n_q_heads][head_dim] (rows past a slot's
        new tokens of out are not written); k_new, v_new: the same with n_kv_heads."""
        import torch
        if out is None:
            out = torch.empty_like(q)
        rows = self.batch * self.width * self.head_dim
        for name, t, n in (("q", q, rows * self.n_q_heads), ("k_new", k_new, rows * self.n_kv_heads),
                           ("v_new", v_new, rows * self.n_kv_heads), ("out", out, rows * self.n_q_heads)):
            if t is not None and (t.dtype != self.io_dtype or not t.is_contiguous() or t.numel() != n):
                raise ValueError(f"{name}: expected {n} contiguous {self.io_dtype} elements")
        _on_this_gpu("decode_attn", self.lens, q, k_new, v_new, out)
        B.baton_paged_attn(self.desc, layer, q, k_new, v_new, self.width, out, scale, self._ws, self._ws_bytes,
                           _cur_stream())
        return out
