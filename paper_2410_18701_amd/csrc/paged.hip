// Host side of the cache in pages: argument checks and launches.  The C ABI is
// documented in include/baton.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <vector>

#include "baton.h"
#include "layer_ops.hpp"
#include "paged_attn.hpp"
#include "paged_ops.hpp"
#include "verify.hpp"

namespace {

bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

baton_status done() { return hipGetLastError() == hipSuccess ? BATON_OK : BATON_EHIP; }

int64_t layer_elems(const baton_paged_desc& d) { return (int64_t)d.n_pages * d.n_kv_heads * d.page * d.head_dim; }
int32_t elem_bytes(const baton_paged_desc& d) { return d.dtype == BATON_F32 ? 4 : 2; }
int64_t stride_elems(const baton_paged_desc& d) { return d.layer_stride ? d.layer_stride : layer_elems(d); }
int32_t page_shift(const baton_paged_desc& d) { return d.page == 32 ? 5 : d.page == 64 ? 6 : d.page == 128 ? 7 : 8; }

int32_t max_items(const baton_paged_desc& d) {
  return baton::paged_max_items(d.batch, d.n_kv_heads, d.max_pages, d.page);
}
baton::PagedState state_at(const baton_paged_desc& d) { return baton::paged_state(d.batch, d.n_pages, max_items(d)); }

// The sizes alone: what the byte counts go by.
baton_status check_sizes(const baton_paged_desc* d) {
  if (!d) return BATON_EINVAL;
  if (d->n_layers < 1 || d->batch < 1 || d->batch > BATON_MAX_BATCH || d->n_q_heads < 1 || d->n_kv_heads < 1 ||
      d->n_q_heads > (1 << 16) || d->n_pages < 1 || d->max_pages < 1 || d->max_pages > (1 << 20) || d->window < 0 ||
      d->sinks < 0 || d->window > (1 << 30) || d->sinks > (1 << 30))
    return BATON_EINVAL;
  if (d->page != 32 && d->page != 64 && d->page != 128 && d->page != 256) return BATON_EINVAL;
  if ((int64_t)d->n_pages * d->page >= (int64_t(1) << 31)) return BATON_EINVAL;
  if (d->dtype != BATON_F32 && d->dtype != BATON_BF16) return BATON_EDTYPE;
  if (d->head_dim != 64 && d->head_dim != 128) return BATON_EDTYPE;
  const int32_t g = d->n_q_heads / d->n_kv_heads;
  if (d->n_q_heads % d->n_kv_heads || (g != 1 && g != 2 && g != 4 && g != 8)) return BATON_EDTYPE;
  return BATON_OK;
}

baton_status check(const baton_paged_desc* d) {
  const baton_status st = check_sizes(d);
  if (st != BATON_OK) return st;
  if (!d->k || !d->v || !d->table || !d->lens || !d->state) return BATON_EINVAL;
  if (!aligned(d->k, 16) || !aligned(d->v, 16) || !aligned(d->table, 4) || !aligned(d->lens, 4) ||
      !aligned(d->state, 16))
    return BATON_EINVAL;
  // K (and V) span less than 2^56 bytes, their layers are whole 16-byte vectors apart
  // and no layer of one lies on a layer of the other.
  const int32_t es = elem_bytes(*d);
  if (d->layer_stride < 0 || (__int128)d->n_pages * d->page * d->n_kv_heads * d->head_dim * es >= ((__int128)1 << 56))
    return BATON_EINVAL;
  const int64_t layer = layer_elems(*d), stride = stride_elems(*d);
  if (stride < layer || (__int128)stride * es * d->n_layers >= ((__int128)1 << 56) || stride * es % 16)
    return BATON_EINVAL;
  const int64_t lb = layer * es, sb = stride * es, span = (int64_t)(d->n_layers - 1) * sb + lb;
  const int64_t dist = static_cast<const char*>(d->v) - static_cast<const char*>(d->k);
  const int64_t r = ((dist % sb) + sb) % sb;             // v's offset within a layer period of k
  const bool apart = dist >= span || -dist >= span;
  const bool interleaved = d->n_layers > 1 && r >= lb && r <= sb - lb;
  if (!apart && !interleaved) return BATON_EINVAL;
  return BATON_OK;
}

template <typename T, int D>
void launch_attn(const baton::PagedAttnArgs& a, int32_t items, bool split, hipStream_t s) {
  const dim3 grid((unsigned)items * a.n_kv_heads), block(baton::kWave * baton::kPagedWaves);
  hipLaunchKernelGGL((baton::paged_attn_kernel<T, D>), grid, block, 0, s, a);
  if (split)
    hipLaunchKernelGGL((baton::paged_combine_kernel<T, D>),
                       dim3((unsigned)a.batch * a.n_kv_heads, (unsigned)(a.width * a.group)), dim3(256), 0, s, a);
}

template <int ES, int D>
void launch_copy(const baton::PagedCopyArgs& a, bool out, hipStream_t s) {
  const dim3 grid((unsigned)std::min<int64_t>(a.block_end[a.n_segs - 1], 1 << 22)), block(baton::kWave);
  if (out) hipLaunchKernelGGL((baton::paged_copy_kernel<ES, D, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((baton::paged_copy_kernel<ES, D, false>), grid, block, 0, s, a);
}

baton_status copy(const baton_paged_desc* d, const int32_t* slots, int32_t n, const int32_t* lens, const void* const* k,
                  const void* const* v, bool out, hipStream_t stream) {
  const baton_status st = check(d);
  if (st != BATON_OK) return st;
  if (n < 0 || (n > 0 && (!slots || !lens || !k || !v))) return BATON_EINVAL;
  std::vector<uint8_t> seen(d->batch, 0);
  for (int32_t i = 0; i < n; ++i) {
    const int32_t s = slots[i];
    if (s < 0 || s >= d->batch || seen[s] || lens[i] < 1 || lens[i] > (int64_t)d->max_pages * d->page)
      return BATON_EINVAL;
    if (!k[i] || !v[i] || !aligned(k[i], 16) || !aligned(v[i], 16)) return BATON_EINVAL;
    seen[s] = 1;
  }
  baton::PagedCopyArgs a;
  std::memset(&a, 0, sizeof(a));
  a.k = static_cast<uint8_t*>(d->k);
  a.v = static_cast<uint8_t*>(d->v);
  a.table = d->table;
  a.layer_bytes = stride_elems(*d) * elem_bytes(*d);
  a.n_layers = d->n_layers;
  a.n_kv_heads = d->n_kv_heads;
  a.max_pages = d->max_pages;
  a.n_pages = d->n_pages;
  a.page_shift = page_shift(*d);
  for (int32_t i0 = 0; i0 < n; i0 += baton::kPagedSegs) {
    a.n_segs = std::min(n - i0, baton::kPagedSegs);
    int64_t blocks = 0;
    for (int32_t i = 0; i < a.n_segs; ++i) {
      a.slot[i] = slots[i0 + i];
      a.len[i] = lens[i0 + i];
      blocks += (int64_t)2 * d->n_layers * d->n_kv_heads * ((a.len[i] + baton::kPagedBlock - 1) / baton::kPagedBlock);
      a.block_end[i] = blocks;
      a.kext[i] = static_cast<uint8_t*>(const_cast<void*>(k[i0 + i]));
      a.vext[i] = static_cast<uint8_t*>(const_cast<void*>(v[i0 + i]));
    }
    if (d->dtype == BATON_F32) {
      if (d->head_dim == 64) launch_copy<4, 64>(a, out, stream);
      else launch_copy<4, 128>(a, out, stream);
    } else {
      if (d->head_dim == 64) launch_copy<2, 64>(a, out, stream);
      else launch_copy<2, 128>(a, out, stream);
    }
    if (done() != BATON_OK) return BATON_EHIP;
  }
  return BATON_OK;
}

}  // namespace

extern "C" {

size_t baton_paged_state_bytes(const baton_paged_desc* d) {
  return check_sizes(d) == BATON_OK ? (size_t)state_at(*d).words * 4 : 0;
}

size_t baton_paged_attn_workspace_bytes(const baton_paged_desc* d, int32_t width) {
  if (check_sizes(d) != BATON_OK || width < 1 || width * (d->n_q_heads / d->n_kv_heads) > BATON_PAGED_MAX_ROWS ||
      width > BATON_PAGED_MAX_WIDTH)
    return 0;
  const int32_t items = max_items(*d);
  if (items <= d->batch) return 0;         // no slot has two
  return (size_t)items * d->n_q_heads * width * (d->head_dim + 4) * sizeof(float);
}

baton_status baton_paged_reset(const baton_paged_desc* d, const int32_t* order, hipStream_t stream) {
  const baton_status st = check(d);
  if (st != BATON_OK) return st;
  if (!aligned(order, 4)) return BATON_EINVAL;
  const int64_t n = std::max<int64_t>((int64_t)d->batch * d->max_pages, d->n_pages);
  hipLaunchKernelGGL(baton::paged_reset_kernel, dim3((unsigned)std::min<int64_t>((n + 255) / 256, 2048)), dim3(256), 0,
                     stream, d->table, d->lens, d->state, order, d->batch, d->max_pages, d->n_pages, state_at(*d));
  return done();
}

baton_status baton_paged_step(const baton_paged_desc* d, const int32_t* keep, const int32_t* n_new, int32_t* slot_map,
                              int32_t width, int64_t map_ld, int32_t* missing, hipStream_t stream) {
  const baton_status st = check(d);
  if (st != BATON_OK) return st;
  if (!n_new || !aligned(n_new, 4) || !aligned(keep, 4) || !aligned(slot_map, 4) || !aligned(missing, 4))
    return BATON_EINVAL;
  if (slot_map && (width < 1 || width > (1 << 20) || map_ld < width || map_ld > (int64_t(1) << 40))) return BATON_EINVAL;
  baton::PagedStepArgs a;
  std::memset(&a, 0, sizeof(a));
  a.table = d->table;
  a.lens = d->lens;
  a.state = d->state;
  a.keep = keep;
  a.n_new = n_new;
  a.slot_map = slot_map;
  a.missing = missing;
  a.batch = d->batch;
  a.max_pages = d->max_pages;
  a.page_shift = page_shift(*d);
  a.window = d->window;
  a.sinks = d->sinks;
  a.n_kv_heads = d->n_kv_heads;
  a.group = d->n_q_heads / d->n_kv_heads;
  a.width = width;
  a.map_ld = map_ld;
  a.at = state_at(*d);
  hipLaunchKernelGGL(baton::paged_step_kernel, dim3(1), dim3(baton::kStepThreads), 0, stream, a);
  return done();
}

baton_status baton_paged_embed(const baton_paged_desc* d, const int32_t* slots, int32_t n, const int32_t* lens,
                               const void* const* k_src, const void* const* v_src, hipStream_t stream) {
  return copy(d, slots, n, lens, k_src, v_src, false, stream);
}

baton_status baton_paged_extract(const baton_paged_desc* d, const int32_t* slots, int32_t n, const int32_t* lens,
                                 void* const* k_dst, void* const* v_dst, hipStream_t stream) {
  return copy(d, slots, n, lens, const_cast<const void* const*>(k_dst), const_cast<const void* const*>(v_dst), true,
              stream);
}

baton_status baton_paged_rope_qkv(const baton_paged_desc* d, const void* qkv, int32_t width, void* q, void* k_new,
                                  void* v_new, float theta, hipStream_t stream) {
  const baton_status st = check(d);
  if (st != BATON_OK) return st;
  if (!qkv || !q || !k_new || !v_new || !(theta > 1.f) || !std::isfinite(theta) || width < 1 ||
      width > BATON_PAGED_MAX_WIDTH)
    return BATON_EINVAL;
  if (!aligned(qkv, 2) || !aligned(q, 2) || !aligned(k_new, 2) || !aligned(v_new, 2)) return BATON_EINVAL;
  if (d->dtype != BATON_BF16) return BATON_EDTYPE;
  baton::RopeShape a;
  a.qkv = static_cast<const uint16_t*>(qkv);
  a.q = static_cast<uint16_t*>(q);
  a.k = static_cast<uint16_t*>(k_new);
  a.v = static_cast<uint16_t*>(v_new);
  a.n_q_heads = d->n_q_heads;
  a.n_kv_heads = d->n_kv_heads;
  a.head_dim = d->head_dim;
  a.log2_theta = std::log2((double)theta);
  const int64_t blocks = (int64_t)d->batch * width * (d->n_q_heads + 2 * d->n_kv_heads);
  if (blocks >= (int64_t(1) << 26)) return BATON_EINVAL;   // fewer than 2^32 threads
  hipLaunchKernelGGL(baton::rope_qkv_at_kernel, dim3((unsigned)blocks), dim3(baton::kWave), 0, stream, a, d->lens, width);
  return done();
}

baton_status baton_paged_attn(const baton_paged_desc* d, int32_t layer, const void* q, const void* k_new,
                              const void* v_new, int32_t width, void* out, float scale, void* ws, size_t ws_bytes,
                              hipStream_t stream) {
  const baton_status st = check(d);
  if (st != BATON_OK) return st;
  const int32_t group = d->n_q_heads / d->n_kv_heads;
  if (layer < 0 || layer >= d->n_layers || !q || !out || !k_new != !v_new || !(std::fabs(scale) <= 0x1p127f))
    return BATON_EINVAL;                   // (times log2 e it is finite)
  if (width < 1 || width > BATON_PAGED_MAX_WIDTH || width * group > BATON_PAGED_MAX_ROWS) return BATON_EINVAL;
  if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(out, 16)) return BATON_EINVAL;
  const size_t need = baton_paged_attn_workspace_bytes(d, width);
  if (need && (!ws || !aligned(ws, 16) || ws_bytes < need)) return BATON_EINVAL;
  const int32_t items = max_items(*d);
  // launches of fewer than 2^32 threads
  if ((int64_t)items * d->n_kv_heads >= (int64_t(1) << 24) ||
      (int64_t)d->batch * d->n_q_heads * width >= (int64_t(1) << 24))
    return BATON_EINVAL;
  baton::PagedAttnArgs a;
  std::memset(&a, 0, sizeof(a));
  a.q = static_cast<const uint8_t*>(q);
  a.k_new = static_cast<const uint8_t*>(k_new);
  a.v_new = static_cast<const uint8_t*>(v_new);
  a.out = static_cast<uint8_t*>(out);
  const int64_t at = layer * stride_elems(*d) * elem_bytes(*d);
  a.k = static_cast<uint8_t*>(d->k) + at;
  a.v = static_cast<uint8_t*>(d->v) + at;
  a.table = d->table;
  a.state = d->state;
  a.at = state_at(*d);
  a.partial = static_cast<float*>(ws);
  const double qscale = (scale == 0.f ? 1.0 / std::sqrt((double)d->head_dim) : (double)scale) * 1.4426950408889634074;
  a.qscale = (float)qscale;
  a.qscale_rest = (float)(qscale - (double)a.qscale);
  a.batch = d->batch;
  a.n_kv_heads = d->n_kv_heads;
  a.group = group;
  a.width = width;
  a.max_pages = d->max_pages;
  a.n_pages = d->n_pages;
  a.page_shift = page_shift(*d);
  a.window = d->window;
  a.sinks = d->sinks;
  const bool split = need > 0;
  if (d->dtype == BATON_F32) {
    if (d->head_dim == 64) launch_attn<baton::F32Tag, 64>(a, items, split, stream);
    else launch_attn<baton::F32Tag, 128>(a, items, split, stream);
  } else {
    if (d->head_dim == 64) launch_attn<baton::BF16Tag, 64>(a, items, split, stream);
    else launch_attn<baton::BF16Tag, 128>(a, items, split, stream);
  }
  return done();
}

baton_status baton_paged_verify(const baton_paged_desc* d, int32_t dtype, const void* target, int64_t target_ld,
                                const void* draft, int64_t draft_ld, int32_t width, int32_t vocab,
                                const int32_t* drafted, const int32_t* n_draft, const float* u_accept,
                                const float* u_token, const float* temperature, const int32_t* top_k,
                                const float* top_p, const float* min_p, int32_t* tokens, int32_t* n_out, void* ws,
                                size_t ws_bytes, hipStream_t stream) {
  const baton_status st = check(d);
  if (st != BATON_OK) return st;
  return baton::verify(d->state + state_at(*d).n_new, dtype, target, target_ld, draft, draft_ld, d->batch, width, vocab,
                       drafted, n_draft, u_accept, u_token, temperature, top_k, top_p, min_p, tokens, n_out, ws,
                       ws_bytes, stream);
}

}  // extern "C"
