// Decode attention over a cache held in 4 bits (kv4_ops.hpp has the format), on
// the matrix cores, for every grouping.  Work items, partial records and their
// merge are those of the bf16 kernels.
//
// What bounds it is HBM -- 68 bytes of K or V per token at head_dim 128, against
// 256 in bf16 -- as long as turning codes into operands costs few instructions,
// and then each item's start (its descriptor, the query, the first loads) and end:
// 39 us for 152 MB (32 rows of up to 2048 tokens, 32 heads; 3.9 TB/s), 62 for 295 MB
// (61 rows of up to 8192, 64 heads over 8; 4.8), where a copy of it that only loads
// takes 32 and 54 and a plain read of as many bytes 23 and 42.  The vector ALUs are
// active 36% and 45% of the launch, the matrix cores 11% and 18%.  Per iteration a wave
// takes 64 tokens:
//  * QK^T: A = 16 key rows x 32 of d, four tiles of 16 consecutive tokens.  The
//    contraction's order is free, so lane l takes the D / 4 elements from D / 4 *
//    (l / 16) on of its key row -- one load of 16 bytes (8 at head_dim 64), a
//    quarter row, all in one scale block -- and the query is laid out the same
//    way.  No key passes through LDS; one instruction turns two codes and the
//    block's scale into two bf16 of the operand, exactly.
//  * the scores of tile j, row 4 g + r are lane group g's register (j, r), so a
//    lane holds 16 tokens' scores of its column.
//  * PV, transposed (O^T = V^T P^T): A = V^T needs 8 tokens of one column per
//    lane.  The codes are staged in LDS as they come, and the transposing read of
//    4-bit elements hands lane i of a group of 16 the i-th column of 16 rows; the
//    rows are given in the order of the lane's own scores, so one read per 16
//    columns feeds both halves of the tokens.  A value's scale belongs to its token and its
//    block of 32 columns, so it cannot be applied to operand pairs of two tokens:
//    it multiplies the weight instead, P' = p 2^(s - 127), exactly.
//    That makes P' differ between the column blocks --
//    and a 16-column operand has columns to spare: with G query heads per kv-head,
//    REP = min(D / 32, 16 / G) columns per head each carry another block, and of the
//    16 result columns only the one with the slice's block is kept (at G = 8 and
//    head_dim 128 two blocks share a column and P' is formed twice).
//  * a weight is taken in two bf16 parts, which keep 16 bits of it (with one, the
//    outputs of a step of random values were off by 0.0020 of their size, where their own
//    rounding makes 0.0017).  Where 8 columns or fewer carry weights, the other 8 carry the
//    second parts, and the two results are added once, at the item's end; else the second
//    parts take matrix operations of their own.  A whole step takes 0.7 us longer than with
//    one part at G = 1 (56.7), at G = 8 1.4 (36.3, 32 rows of up to 32,768) and 5 (155, two
//    layers of the 61 rows above).
// The weights' sum is taken in fp32 before they are parted.
// Registers are capped for three waves per SIMD (up to 166 used); for four they spill, and
// the kernel takes 1.5 to 2 times as long.
// The step's own key and value take part as given, in bf16, and are stored in 4 bits.
#pragma once

#ifndef BATON_KV4_WPE
#define BATON_KV4_WPE 3
#endif

#include "common.hpp"
#include "decode_attn.hpp"
#include "decode_attn_mfma.hpp"
#include "kv4_ops.hpp"

namespace baton {

template <int D>
struct Kv4Geo {
  static constexpr int kKk = D / 32;                     // QK operations per 16 tokens
  static constexpr int kDt = D / 16;                     // 16-column slices
  static constexpr int kNb = D / 32;                     // scale blocks per token
  static constexpr int kRowB = D / 2;                    // bytes of codes per token
  static constexpr int kVlanes = kRowB / 16;             // lanes per V row
  static constexpr int kVLoads = kVlanes;                // V loads per 64 tokens
  static constexpr int kVTok = kWave / kVlanes;          // V rows per load
  // Padded LDS row: 20 banks (12 at head_dim 64) put the 16 rows of a
  // transposing read on disjoint banks.
  static constexpr int kLdsRow = kRowB + 16;
  static constexpr int kLdsV = 64 * kLdsRow;
  static constexpr int kLdsS = kNb * 64 * 4;             // V scales as fp32 [block][token]
};

typedef int i32x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ i32x2_t read_tr4(const uint8_t* p) {
  return __builtin_amdgcn_ds_read_tr4_b64_v2i32(
      (__attribute__((address_space(3))) i32x2_t*)(const_cast<uint8_t*>(p)));
}

// What one 64-token block needs from memory.
template <int D>
struct Kv4Block {
  uint32_t k[4][D / 32];          // tile j: the lane's quarter of key row 16 j + l % 16
  uint32_t ks[4];                 // its scale byte
  u32x4 v[Kv4Geo<D>::kVLoads];    // V rows, 16 bytes per lane
  uint32_t vs;                    // scales of token l
};

template <int D, int G, int NW>
__global__ void __launch_bounds__(kWave * NW) __attribute__((amdgpu_waves_per_eu(BATON_KV4_WPE)))
attn_kv4_kernel(const AttnArgs a) {
  using Geo = Kv4Geo<D>;
  constexpr int KK = Geo::kKk, DT = Geo::kDt, NB = Geo::kNb, VPT = D / 8, REC = D + 4;
  constexpr int REP = NB < 16 / G ? NB : 16 / G;   // columns per query head
  constexpr int NS = NB / REP;                     // blocks per column
  constexpr bool SPARE = G * REP <= 8;             // columns 8 .. 15 carry the weights' second parts
  __shared__ __attribute__((aligned(16))) uint8_t lds_v[NW][Geo::kLdsV];
  __shared__ __attribute__((aligned(16))) float lds_s[NW][NB * 64];
  __shared__ float sm_m[NW][G], sm_l[NW][G];
  static_assert(G * D * 4 <= Geo::kLdsV, "merge area");
  int32_t item, h;
  const Item desc = work_unit(a, item, h);
  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave), lane = tid % kWave;
  const int g4 = lane / 16, c16 = lane % 16;
  const int col8 = SPARE ? c16 % 8 : c16;
  const bool rest = SPARE && c16 >= 8;
  const int head = col8 / REP, hb = col8 % REP;    // this column's head (none from G on) and place
  uint8_t* lds = lds_v[w];
  float* ldss = lds_s[w];

  const int4 it = desc.span;
  const int4 rw = desc.row;
  const int b = it.x;
  const int32_t n = it.w;
  const int64_t bt = (int64_t)b * a.tw;
  uint32_t* outw = a.out + ((bt * a.n_kv_heads + h) * G) * (D / 2);
  if (n < 0) {                       // free slot: zero output rows
    for (int v = tid; v < G * VPT; v += NW * kWave) reinterpret_cast<u32x4*>(outw)[v] = u32x4{0, 0, 0, 0};
    return;
  }
  const int32_t t_begin = it.y, t_end = it.z;
  const int64_t row = (int64_t)b * a.n_kv_heads + h;
  const int64_t row_bytes = kv4_row_bytes(a.cap, D);
  uint8_t* krow = reinterpret_cast<uint8_t*>(a.k_w) + row * row_bytes;
  uint8_t* vrow = reinterpret_cast<uint8_t*>(a.v) + row * row_bytes;
  const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(krow, 0, (uint32_t)row_bytes, kBufferWord3);
  const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(vrow, 0, (uint32_t)row_bytes, kBufferWord3);
  const uint32_t cap = (uint32_t)a.cap, plane = cap * Geo::kRowB;
  const uint32_t start = (uint32_t)ring_add(a.base, a.L - n, a.cap);

  auto load_k = [&](uint32_t off, uint32_t (&k)[KK]) {
    if constexpr (D == 128) {
      const u32x4 q = load16(rk, off);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) k[kk] = q[kk];
    } else {
      const auto q = __builtin_amdgcn_raw_buffer_load_b64(rk, off, 0, BATON_ATTN_NT ? 2 : 0);
      k[0] = q[0];
      k[1] = q[1];
    }
  };
  auto load_vs = [&](uint32_t off) -> uint32_t {
    if constexpr (D == 128) return __builtin_amdgcn_raw_buffer_load_b32(rv, off, 0, 0);
    else return __builtin_amdgcn_raw_buffer_load_b16(rv, off, 0, 0);
  };

  // Query heads as the B operand in the keys' order of d, negated for a negative
  // scale, so that the largest score is the largest product.
  const float qs = fabsf(a.qscale);
  const uint32_t flip = a.qscale < 0.f ? 0x80008000u : 0u;
  bf16x8 qb[KK];
  const u32x4* qrow = reinterpret_cast<const u32x4*>(a.q) + ((bt * a.n_kv_heads + h) * G) * VPT;
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    const u32x4 qw = head < G ? qrow[head * VPT + KK * g4 + kk] : u32x4{0, 0, 0, 0};
    qb[kk] = as_bf16x8(qw ^ flip);
  }

  float m = -INFINITY, lsum = 0.f;
  f32x4 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};

  // Loads of 64 consecutive columns of the ring from col on.  Those past the row's
  // last column find other bytes of the row or, past its end, zeros.
  const uint32_t k_lane = c16 * Geo::kRowB + g4 * (D / 8), ks_lane = c16 * NB + (D == 128 ? g4 : g4 / 2);
  // Not live: beyond the buffer, which loads zeros without an access.
  constexpr uint32_t kNone = 0x80000000u;
  auto issue = [&](bool live, uint32_t col, Kv4Block<D>& x) {
    const uint32_t cb = live ? col * Geo::kRowB : kNone, sb = live ? plane + col * NB : kNone;
    const uint32_t ko = cb + k_lane, so = sb + ks_lane;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      load_k(ko + j * 16 * Geo::kRowB, x.k[j]);
      x.ks[j] = __builtin_amdgcn_raw_buffer_load_b8(rk, so + j * 16 * NB, 0, 0);
    }
    const uint32_t vo = cb + lane * 16;
#pragma unroll
    for (int u = 0; u < Geo::kVLoads; ++u) x.v[u] = load16(rv, vo + u * 1024);
    x.vs = load_vs(sb + lane * NB);
  };
  // The same for the tokens of a gather list, from place i0 on; none past its end.
  auto issue_listed = [&](int32_t i0, int32_t i1, Kv4Block<D>& x) {
    auto col = [&](int32_t i) {   // its ring column, or cap
      if (i >= i1) return cap;
      const uint32_t c = start + (uint32_t)a.gather[i];
      return c >= cap ? c - cap : c;
    };
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t c = col(i0 + 16 * j + c16);
      load_k(c < cap ? c * Geo::kRowB + g4 * (D / 8) : kNone, x.k[j]);
      x.ks[j] = __builtin_amdgcn_raw_buffer_load_b8(rk, c < cap ? plane + c * NB + (D == 128 ? g4 : g4 / 2) : kNone, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < Geo::kVLoads; ++u) {
      const uint32_t c = col(i0 + u * Geo::kVTok + lane / Geo::kVlanes);
      x.v[u] = load16(rv, c < cap ? c * Geo::kRowB + (lane % Geo::kVlanes) * 16 : kNone);
    }
    const uint32_t c = col(i0 + lane);
    x.vs = load_vs(c < cap ? plane + c * NB : kNone);
  };

  // Scores, online softmax and PV of a block whose first nv tokens are valid.
  auto block = [&](const Kv4Block<D>& x, int32_t nv) {
#pragma unroll
    for (int u = 0; u < Geo::kVLoads; ++u)
      *reinterpret_cast<u32x4*>(lds + (u * Geo::kVTok + lane / Geo::kVlanes) * Geo::kLdsRow +
                                (lane % Geo::kVlanes) * 16) = x.v[u];
    // no scale behind the last token: its weight is 0, which an infinite one (a NaN block's) would make a NaN
    const uint32_t vs = lane < nv ? x.vs : 0u;
#pragma unroll
    for (int k = 0; k < NB; ++k) ldss[k * 64 + lane] = mx_scale_value((vs >> (8 * k)) & 255u);
    float s[16];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float sc = mx_scale_value(x.ks[j]);
      f32x4 sj = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
        sj = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(mx_widen(x.k[j][kk], sc)), qb[kk], sj, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) s[4 * j + r] = sj[r];
    }
    if (nv < 64) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (16 * (e / 4) + 4 * g4 + e % 4 >= nv) s[e] = -INFINITY;
    }
    float mx = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
    mx = fmaxf(m, max_over_groups(mx) * qs);
    if (__builtin_amdgcn_ballot_w64(mx > m)) {    // some column's maximum rose
      const float f = m == -INFINITY ? 0.f : fast_exp2(m - mx);
      lsum *= f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] *= f;
      m = mx;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float p[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = fast_exp2(fmaf(s[e], qs, -ref));
      lsum += p[e];
    }
    // The second part is what the first one's rounding (SPARE; else its cutting off) leaves.
    if constexpr (SPARE) {
#pragma unroll
      for (int e = 0; e < 16; ++e) p[e] = fmaf(rest ? -1.f : 0.f, (float)(__bf16)p[e], p[e]);
    }
    const uint8_t* vt = lds + (16 * (c16 / 4) + 4 * g4 + c16 % 4) * Geo::kLdsRow;
    // P' operands: [part][set], for the tokens of tiles 0 and 1, then of 2 and 3
#pragma unroll
    for (int th = 0; th < 2; ++th) {
      constexpr int NP = SPARE ? 1 : 2;
      bf16x8 pb[NP][NS];
#pragma unroll
      for (int t = 0; t < NS; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const f32x4 sc = *reinterpret_cast<const f32x4*>(ldss + (hb * NS + t) * 64 + 16 * (2 * th + j) + 4 * g4);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float w = p[4 * (2 * th + j) + r];
            if constexpr (SPARE) {
              pb[0][t][4 * j + r] = (__bf16)(w * sc[r]);
            } else {
              const float first = __uint_as_float(__float_as_uint(w) & 0xFFFF0000u);
              pb[0][t][4 * j + r] = (__bf16)(first * sc[r]);
              pb[1][t][4 * j + r] = (__bf16)((w - first) * sc[r]);
            }
          }
        }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const i32x2_t c = read_tr4(vt + dt * 8);
        const bf16x8 v = as_bf16x8(mx_widen(c[th], 1.f));
#pragma unroll
        for (int h2 = 0; h2 < NP; ++h2)
          o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pb[h2][(dt / 2) % NS], o[dt], 0, 0, 0);
      }
    }
  };

  const bool gathered = (rw.w & kGathered) != 0;
  if (gathered) {
    for (int32_t i0 = t_begin + 64 * w; i0 < t_end; i0 += 64 * NW) {
      Kv4Block<D> x;
      issue_listed(i0, t_end, x);
      block(x, t_end - i0);
    }
  } else {
    // The item's tokens before and after the ring's end, each a run of columns, of
    // which wave w takes every NW-th block of 64; a block's loads are in flight while
    // the one before it is computed.
    const int32_t c_end = min(t_end, n), wrap = (int32_t)(cap - start);
#pragma unroll 1
    for (int part = 0; part < 2; ++part) {
      const int32_t t0 = (part == 0 ? t_begin : max(t_begin, wrap)) + 64 * w, t1 = part == 0 ? min(c_end, wrap) : c_end;
      if (t0 >= t1) continue;
      uint32_t col = part == 0 ? start + (uint32_t)t0 : (uint32_t)(t0 - wrap);
      int32_t left = t1 - t0;
      Kv4Block<D> xa, xb;
      issue(true, col, xa);
#pragma unroll 1
      while (true) {
        issue(left > 64 * NW, col + 64 * NW, xb);
        __builtin_amdgcn_sched_barrier(0);   // keep the loads ahead of the computation
        block(xa, left);
        left -= 64 * NW;
        if (left <= 0) break;
        col += 128 * NW;
        issue(left > 64 * NW, col, xa);
        __builtin_amdgcn_sched_barrier(0);
        block(xb, left);
        left -= 64 * NW;
        if (left <= 0) break;
      }
    }
  }

  // The current token, from k_new / v_new in bf16: row 0 of a tile of its own.
  // Its key and value are then quantised into the ring (by
  // the item's first wave): lane i < D / 8 has K's elements 8 i .., the next D / 8 lanes V's.
  if (w == 0 && (gathered ? (rw.w & kCurrent) != 0 : n >= t_begin && n < t_end)) {
    const u32x4* knew = reinterpret_cast<const u32x4*>(a.knew) + (bt * a.n_kv_heads + h) * VPT;
    const u32x4* vnew = reinterpret_cast<const u32x4*>(a.vnew) + (bt * a.n_kv_heads + h) * VPT;
    f32x4 sj = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const u32x4 kw = c16 == 0 ? knew[KK * g4 + kk] : u32x4{0, 0, 0, 0};
      sj = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kw), qb[kk], sj, 0, 0, 0);
    }
    const float s = g4 == 0 ? sj[0] * qs : -INFINITY;
    const float mx = fmaxf(m, max_over_groups(s));
    const float ref = mx == -INFINITY ? 0.f : mx;
    const float f = m == -INFINITY ? 0.f : fast_exp2(m - ref);
    const float p = fast_exp2(s - ref);
    lsum = lsum * f + p;
    m = mx;
    // its two parts (the second not 0, so that an infinite value meets one sign alone)
    const float first = __uint_as_float(__float_as_uint(p) & 0xFFFF0000u);
    const float second = __uint_as_float(__float_as_uint(p) | 1u) - first;
    bf16x8 pa;
#pragma unroll
    for (int e = 0; e < 8; ++e) pa[e] = (__bf16)(e == 0 ? (rest ? second : first) : e == 1 && !SPARE ? second : 0.f);
    const uint16_t* v16 = reinterpret_cast<const uint16_t*>(vnew);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const u32x4 vw = {g4 == 0 ? (uint32_t)v16[16 * dt + c16] * (SPARE ? 1u : 0x10001u) : 0u, 0u, 0u, 0u};
      o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vw), pa, o[dt] * f, 0, 0, 0);
    }
    const bool is_v = lane >= VPT;
    const int e = lane % VPT;
    uint32_t scale;
    const uint32_t code = mx_quantise(is_v ? vnew[e] : knew[e], scale);
    const uint32_t col = (uint32_t)ring_add(start, n, a.cap);
    if (lane < 2 * VPT) {
      uint8_t* dst = is_v ? vrow : krow;
      reinterpret_cast<uint32_t*>(dst + (int64_t)col * Geo::kRowB)[e] = code;
      if (e % 4 == 0) dst[(int64_t)plane + (int64_t)col * NB + e / 4] = (uint8_t)scale;
    }
  }

  // A column keeps the slices of its own blocks: lane l's o[dt][r] is column
  // 16 dt + 4 (l / 16) + r of its head.
  lsum = sum_over_groups(lsum);
  __builtin_amdgcn_wave_barrier();
  if constexpr (SPARE) {      // both parts' products added
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        o[dt][r] += __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(o[dt][r]), 0x128, 0xF, 0xF, true));   // row_ror 8
  }
  if (head < G && !rest) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      if (dt / 2 / NS == hb) *reinterpret_cast<f32x4*>(lds + (head * D + 16 * dt + 4 * g4) * 4) = o[dt];
    if (hb == 0 && g4 == 0) {
      sm_m[w][head] = m;
      sm_l[w][head] = lsum;
    }
  }
  __syncthreads();
  float* rec0 = a.partial + (((int64_t)h * a.n_items + item) * G) * REC;
  wg_merge_write<BF16Tag, D, G, NW>(sm_m, sm_l, reinterpret_cast<const float*>(&lds_v[0][0]), Geo::kLdsV / 4,
                                    rw.y == 1, outw, rec0, tid);
}

}  // namespace baton
