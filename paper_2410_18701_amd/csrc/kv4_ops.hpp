// KV cache held in 4 bits: the element format, and the copies into, out of and
// within a ring of it.
//
// Format (MXFP4): 32 consecutive elements of a token's head share one scale
// byte s, the power of two 2^(s - 127); an element is a sign and one of 0, 1/2,
// 1, 3/2, 2, 3, 4, 6 times it, two to a byte, the first in the low half.  A row
// (layer, slot, kv-head) of the ring is a plane of codes [cap][D / 2] followed by
// a plane of scales [cap][D / 32]: whole 16-byte vectors of codes, and each
// token's scales one 2- or 4-byte word.
//
// A block's scale is the smallest power of two that takes its largest magnitude
// to at most 7: the format's next value after 6 would be 8, so 7 still rounds to
// 6 by half a step and no element is off by more than half a step.  Elements
// round to nearest, ties to the even code.  Storing what was stored again gives
// the same bits (the largest magnitude of a block becomes 4 or 6 times its scale,
// and both ask for that scale), so tokens copied out and embedded again are the
// same.  Scales lie in 2^-125 .. 2^125: every value is a normal bf16 number and a
// smaller block becomes zeros; at the top 2^125 saturates at 6 * 2^125.  A block
// that holds an infinity or a NaN becomes NaN as a whole: scale byte 255, codes 0.
//
// All of it is data movement, bound by HBM: 4-byte words of codes per lane (8
// elements, one 16-byte vector of bf16), the scale from the four lanes that share a
// block.  490 MB embedded or extracted (8 queries of up to 4095 tokens) in 92 to 96 us,
// 5.2 TB/s; 45 MB in 15.
#pragma once

#include "common.hpp"
#include "kv_ops.hpp"

namespace baton {

constexpr uint32_t kMxNan = 255u, kMxMin = 2u, kMxMax = 252u;

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// Bytes of one row of the ring.
__host__ __device__ constexpr int64_t kv4_row_bytes(int64_t cap, int32_t D) { return cap * (D / 2 + D / 32); }

__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kDppXor1, 0xF, 0xF, true));
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kDppXor2, 0xF, 0xF, true));
}

// The scale byte of a block whose largest bf16 magnitude bits are `amax`: the
// exponent two below the largest element's, one more above 1.75 times its power
// of two (the 31 carries from the 97th of the 128 fractions on).
__device__ __forceinline__ uint32_t mx_scale(uint32_t amax) {
  if (amax >= 0x7F80u) return kMxNan;
  const int32_t e = (int32_t)((amax + 31u) >> 7) - 2;
  return (uint32_t)min(max(e, (int32_t)kMxMin), (int32_t)kMxMax);
}

__device__ __forceinline__ float mx_scale_value(uint32_t s) { return __uint_as_float(s << 23); }

// Eight bf16 elements -> their codes and the block's scale byte.  The block is
// spread over four consecutive lanes, all of which must be active.
__device__ __forceinline__ uint32_t mx_quantise(const u32x4& w, uint32_t& scale) {
  uint32_t amax = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) amax = max(amax, max(w[j] & 0x7FFFu, (w[j] >> 16) & 0x7FFFu));
  scale = mx_scale(quad_max(amax));
  const float s = mx_scale_value(scale);
  // each word by value: a bit cast of a vector's element in place reads element 0
  const uint32_t x0 = w[0], x1 = w[1], x2 = w[2], x3 = w[3];
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x0), s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x1), s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x2), s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x3), s, 3);
  return scale == kMxNan ? 0u : c;
}

// Eight codes -> bf16, times the scale value: exact.
__device__ __forceinline__ u32x4 mx_widen(uint32_t c, float s) {
  u32x4 w;
  w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
  w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
  w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
  w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
  return w;
}

// The scale bytes of a token from the D / 8 lanes that hold it, in the first of them.
template <int D>
__device__ __forceinline__ uint32_t mx_scales(uint32_t s) {
  s |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x104, 0xF, 0xF, true) << 8;             // row_shl 4
  if constexpr (D == 128) s |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x108, 0xF, 0xF, true) << 16;
  return s;
}

// Tiles (workgroups) of a launch: some 4 GB of sources, far below 2^32 threads.
constexpr uint32_t kSeg4Tiles = 1u << 18;

// SegArgs for a 4-bit ring: segments as there, the contiguous side in bf16 with
// its own strides (a prompt's keys lie [position][head][D], a prefilled query's
// [layer][head][position][D]).  k, v and layer_vec as in SegArgs.
struct Seg4Args {
  uint8_t* k;
  uint8_t* v;
  int64_t cap;
  int64_t layer_bytes;      // from one layer's rows to the next layer's
  int32_t n_layers, batch, n_kv_heads;
  int32_t n_segs;
  uint32_t tile0;           // tile of the launch's first workgroup
  int32_t mode;             // 0: ext (or placeholder) -> ring, 1: ring -> ext, 2: ring row -> ring row
  uint32_t fill_word;       // placeholder byte, four times
  int32_t slot[kMaxSegs];
  int32_t len[kMaxSegs];
  int32_t tiles_per_row[kMaxSegs];
  int64_t col0[kMaxSegs];
  uint32_t tile_end[kMaxSegs];
  int32_t dst_slot[kMaxSegs];
  int64_t tok_stride[kMaxSegs];    // 16-byte vectors of the contiguous side: token to token,
  int64_t head_stride[kMaxSegs];   //   head to head (layers n_kv_heads heads apart),
  int64_t ext_off[kMaxSegs];       //   and to the segment's first token
  u32x4* kext[kMaxSegs];           // null: placeholders
  u32x4* vext[kMaxSegs];
};

// One block moves a tile of TT tokens of one row, 8 elements per lane and step.
// 64-bit where it counts: a segment's place and the contiguous side's.
template <int D>
__global__ void __launch_bounds__(kCopyThreads) seg4_kernel(const Seg4Args a) {
  constexpr int PPT = D / 8;                               // pieces per token
  constexpr int TT = kCopyThreads * kCopyVecs / PPT;
  const uint32_t g = a.tile0 + blockIdx.x;                 // tiles fit 31 bits
  int i = 0;
  while (i < a.n_segs - 1 && g >= a.tile_end[i]) ++i;
  const uint32_t local = g - (i > 0 ? a.tile_end[i - 1] : 0), tpr = a.tiles_per_row[i];
  const uint32_t row = local / tpr;
  const int32_t tile = (int32_t)(local - row * tpr);
  const uint32_t lh_count = a.n_layers * a.n_kv_heads;
  const bool which = row >= lh_count;                      // 0: K, 1: V
  const int32_t lh = (int32_t)(which ? row - lh_count : row);
  const int32_t layer = lh / a.n_kv_heads, h = lh - layer * a.n_kv_heads;
  const int32_t t0 = tile * TT;
  const int32_t n = min(TT, a.len[i] - t0) * PPT;          // pieces of the tile
  const int64_t row_bytes = kv4_row_bytes(a.cap, D), plane = a.cap * (D / 2);
  uint8_t* layer0 = (which ? a.v : a.k) + layer * a.layer_bytes;
  uint8_t* ring = layer0 + ((int64_t)a.slot[i] * a.n_kv_heads + h) * row_bytes;
  u32x4* ext = which ? a.vext[i] : a.kext[i];
  if (ext) ext += lh * a.head_stride[i] + a.ext_off[i] + t0 * a.tok_stride[i];
  const int64_t c0 = ring_add(a.col0[i], t0, a.cap);
  uint8_t* dst = a.mode == 2 ? layer0 + ((int64_t)a.dst_slot[i] * a.n_kv_heads + h) * row_bytes : ring;

  uint32_t code[kCopyVecs], scale[kCopyVecs];
  u32x4 w[kCopyVecs];
#pragma unroll
  for (int r = 0; r < kCopyVecs; ++r) {
    const int idx = threadIdx.x + r * kCopyThreads, t = idx / PPT, e = idx % PPT;
    code[r] = a.fill_word;
    scale[r] = a.fill_word & 255u;
    w[r] = u32x4{0, 0, 0, 0};
    if (idx < n) {
      if (a.mode != 0) {
        const int64_t col = ring_add(c0, t, a.cap);
        code[r] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(ring + col * (D / 2)) + e);
        scale[r] = ring[plane + col * (D / 32) + e / 4];
      } else if (ext) {
        w[r] = __builtin_nontemporal_load(ext + t * a.tok_stride[i] + e);
      }
    }
  }
  if (a.mode == 0 && ext) {
#pragma unroll
    for (int r = 0; r < kCopyVecs; ++r) code[r] = mx_quantise(w[r], scale[r]);   // whole waves: the block's lanes agree
  }
#pragma unroll
  for (int r = 0; r < kCopyVecs; ++r) {
    const int idx = threadIdx.x + r * kCopyThreads, t = idx / PPT, e = idx % PPT;
    if (idx >= n) continue;
    if (a.mode == 1) {
      u32x4 x = mx_widen(code[r], mx_scale_value(scale[r]));
      if (scale[r] == kMxNan) x = u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
      __builtin_nontemporal_store(x, ext + t * a.tok_stride[i] + e);
    } else {
      const int64_t col = ring_add(c0, t, a.cap);
      __builtin_nontemporal_store(code[r], reinterpret_cast<uint32_t*>(dst + col * (D / 2)) + e);
      // a token's scales, one from every fourth of its lanes, in one store
      const uint32_t all = mx_scales<D>(scale[r]);
      if (e == 0) {
        if constexpr (D == 128) *reinterpret_cast<uint32_t*>(dst + plane + col * 4) = all;
        else *reinterpret_cast<uint16_t*>(dst + plane + col * 2) = (uint16_t)all;
      }
    }
  }
}

}  // namespace baton
