// Host side of the 4-bit cache: copies and the decode attention's launches.
// Part of baton.hip's anonymous namespace (it uses the handle's fields).
#pragma once

#ifndef BATON_KV4_WAVES
#define BATON_KV4_WAVES 4   // waves per attention workgroup
#endif

bool is_kv4(const baton_cache* c) { return c->d.dtype == BATON_MXFP4; }

// The tiles of a's segments, kSeg4Tiles to a launch.
template <int D>
baton_status launch_tiles4(baton::Seg4Args& a, int64_t tiles, hipStream_t s) {
  if (tiles > 0x7FFFFFFF) return BATON_EINVAL;
  for (a.tile0 = 0; a.tile0 < tiles; a.tile0 += baton::kSeg4Tiles) {
    const uint32_t n = std::min(baton::kSeg4Tiles, (uint32_t)tiles - a.tile0);
    hipLaunchKernelGGL(baton::seg4_kernel<D>, dim3(n), dim3(baton::kCopyThreads), 0, s, a);
    const baton_status st = hip_status(hipGetLastError());
    if (st != BATON_OK) return st;
  }
  return BATON_OK;
}

template <int D>
baton_status launch_segs4_d(const baton_cache* c, const std::vector<Seg>& segs, int mode, hipStream_t s) {
  constexpr int PPT = D / 8, TT = baton::kCopyThreads * baton::kCopyVecs / PPT;
  for (size_t off = 0; off < segs.size(); off += baton::kMaxSegs) {
    baton::Seg4Args a;
    std::memset(&a, 0, sizeof(a));
    a.k = static_cast<uint8_t*>(c->d.k);
    a.v = static_cast<uint8_t*>(c->d.v);
    a.cap = c->d.capacity;
    a.layer_bytes = c->layer_vec * 16;
    a.n_layers = c->d.n_layers;
    a.batch = c->d.batch;
    a.n_kv_heads = c->d.n_kv_heads;
    a.fill_word = fill_word(c);
    a.mode = mode;
    const size_t n = std::min<size_t>(baton::kMaxSegs, segs.size() - off);
    int64_t tiles = 0;
    int32_t used = 0;
    for (size_t i = 0; i < n; ++i) {
      const Seg& g = segs[off + i];
      if (g.len <= 0) continue;
      const int64_t ext_len = g.ext_len > 0 ? g.ext_len : g.len;
      a.slot[used] = g.slot;
      a.len[used] = g.len;
      a.col0[used] = g.col0;
      a.tiles_per_row[used] = (g.len + TT - 1) / TT;
      a.dst_slot[used] = g.dst_slot;
      a.tok_stride[used] = PPT;
      a.head_stride[used] = ext_len * PPT;
      a.ext_off[used] = (int64_t)g.ext_t0 * PPT;
      a.kext[used] = static_cast<baton::u32x4*>(const_cast<void*>(g.ks));
      a.vext[used] = static_cast<baton::u32x4*>(const_cast<void*>(g.vs));
      tiles += (int64_t)a.tiles_per_row[used] * 2 * c->d.n_layers * c->d.n_kv_heads;
      a.tile_end[used] = (uint32_t)tiles;
      ++used;
    }
    a.n_segs = used;
    const baton_status st = launch_tiles4<D>(a, tiles, s);
    if (st != BATON_OK) return st;
  }
  return BATON_OK;
}

baton_status launch_segs4(const baton_cache* c, const std::vector<Seg>& segs, int mode, hipStream_t s) {
  return c->d.head_dim == 64 ? launch_segs4_d<64>(c, segs, mode, s) : launch_segs4_d<128>(c, segs, mode, s);
}

// Quantises the prompts of a prefill step into the layer whose rows begin at
// p.k and p.v: columns base + L + T - p .. of each prefilled slot, from k_new
// and v_new [batch][T][n_kv_heads][D].
template <int D>
baton_status append_prompts4_d(const baton_cache* c, const baton::PrefillArgs& p, hipStream_t s) {
  constexpr int PPT = D / 8, TT = baton::kCopyThreads * baton::kCopyVecs / PPT;
  for (int32_t off = 0; off < p.n_ins; off += baton::kMaxSegs) {
    baton::Seg4Args a;
    std::memset(&a, 0, sizeof(a));
    a.k = reinterpret_cast<uint8_t*>(p.k);
    a.v = reinterpret_cast<uint8_t*>(p.v);
    a.cap = p.cap;
    a.n_layers = 1;
    a.batch = p.batch;
    a.n_kv_heads = p.n_kv_heads;
    int64_t tiles = 0;
    a.n_segs = std::min(baton::kMaxSegs, p.n_ins - off);
    for (int32_t i = 0; i < a.n_segs; ++i) {
      const int32_t len = p.plen[off + i];
      a.slot[i] = p.slot[off + i];
      a.len[i] = len;
      a.col0[i] = ring(p.base + p.L + p.T - len, p.cap);
      a.tiles_per_row[i] = (len + TT - 1) / TT;
      a.dst_slot[i] = -1;
      a.tok_stride[i] = (int64_t)p.n_kv_heads * PPT;
      a.head_stride[i] = PPT;
      a.ext_off[i] = ((int64_t)p.slot[off + i] * p.T + p.T - len) * p.n_kv_heads * PPT;
      a.kext[i] = reinterpret_cast<baton::u32x4*>(const_cast<uint32_t*>(p.knew));
      a.vext[i] = reinterpret_cast<baton::u32x4*>(const_cast<uint32_t*>(p.vnew));
      tiles += (int64_t)a.tiles_per_row[i] * 2 * p.n_kv_heads;
      a.tile_end[i] = (uint32_t)tiles;
    }
    const baton_status st = launch_tiles4<D>(a, tiles, s);
    if (st != BATON_OK) return st;
  }
  return BATON_OK;
}

baton_status append_prompts4(const baton_cache* c, const baton::PrefillArgs& p, hipStream_t s) {
  return c->d.head_dim == 64 ? append_prompts4_d<64>(c, p, s) : append_prompts4_d<128>(c, p, s);
}

// Automatic split.  A token's bytes are 17/64 of bf16's, so an item costs as
// much besides them as one of a quarter of the tokens would there: items are
// longer.  A workgroup of four waves with two blocks each in flight takes what a
// CU can, so an item per CU is enough (tokens / 256); and a row of n tokens in n / S
// pieces pays for each piece in the work list and the merge, about 0.25 us a
// piece, against 2 ns per token of an item, balanced at S = sqrt(128 n).  us per
// layer at S and at 256 tokens: one row of 32,768 over one kv-head 24.4 (2048) and
// 43.3, of 100,000 over eight 39 (3584) and 132, of 8192 over 32 18.5 (1024) and
// 27.4; 32 rows of up to 2048 over 32 40.0 (4096) and 53.2.
int32_t kv4_split(const baton_cache* c) {
  const baton::HoleList hl = hole_list(c);
  int64_t total = 0, longest = 0;
  for (int32_t b = 0; b < c->d.batch; ++b)
    if (c->lens[b] > 0 && c->plen[b] == 0) {
      const int64_t n = row_tokens(c, b, hl) + 1;
      total += n;
      longest = std::max(longest, n);
    }
  const int64_t s = std::max((total * c->d.n_kv_heads + 255) / 256, (int64_t)std::sqrt(128.0 * (double)longest));
  return (int32_t)std::min(kAutoSplitMax, std::max(kAutoSplitMin, (s + 63) / 64 * 64));
}

template <int D, int G>
void launch_attn4_g(const baton_cache* c, const baton::AttnArgs& a, hipStream_t s) {
  constexpr int NW = BATON_KV4_WAVES;
  const int hkv = c->d.n_kv_heads;
  hipLaunchKernelGGL((baton::attn_kv4_kernel<D, G, NW>), dim3(c->n_items * hkv), dim3(baton::kWave * NW), 0, s, a);
  if (c->n_multi > 0)
    hipLaunchKernelGGL((baton::combine_kernel<baton::BF16Tag, D, G>), dim3(c->n_multi, hkv * G), dim3(baton::kWave), 0,
                       s, a);
}

template <int D>
void launch_attn4_d(const baton_cache* c, const baton::AttnArgs& a, hipStream_t s) {
  switch (c->group) {
    case 1: launch_attn4_g<D, 1>(c, a, s); break;
    case 2: launch_attn4_g<D, 2>(c, a, s); break;
    case 4: launch_attn4_g<D, 4>(c, a, s); break;
    default: launch_attn4_g<D, 8>(c, a, s); break;
  }
}

bool launch_attn4(const baton_cache* c, const baton::AttnArgs& a, hipStream_t s) {
  if (c->d.head_dim == 64) launch_attn4_d<64>(c, a, s);
  else launch_attn4_d<128>(c, a, s);
  return true;
}
