// Attention of a step's new tokens -- one per query, or a few drafted ones behind it --
// over a cache in pages (paged_ops.hpp: its layout, and the work items).
//
// The rows of a (slot, kv-head) are its new tokens' query heads, row i G + q for query
// head q of the head's G at new token i, up to 64 of them, in MT tiles of 16.  Token j
// is visible to new token i, at position p = len + i, if j <= p and, with a window W and
// S sinks, j > p - W or j < S.
//
// A work item is a run of blocks of 32 tokens of one slot; a workgroup of four waves
// takes an item for one kv-head.  Per block and tile, with the matrix cores' 16x16 tiles:
//  * scores, transposed: S^T = K Q^T, K's rows being the tokens.  Lane l has row l % 16's
//    scores of the tokens 8 (l / 16) .. + 7.
//  * softmax with a running maximum per row, in fp32, base 2.
//  * O^T += V^T P^T, where lane l supplies as it holds them its own row's weights, and
//    accumulates columns 16 t + 4 (l / 16) .. + 3 of row l % 16.
// bf16: weights are taken as a sum of three bf16 numbers, which have all of fp32's bits;
// the values' and keys' products with them are exact in fp32.
// fp32: products in fp32 (v_mfma_f32_16x16x4_f32).
// K and V come from memory in the order of the operands.
// Values that are infinite or NaN: a weight of 0 would turn them into NaN for rows that
// do not see them.  Blocks that hold any are multiplied once for each new token, with
// what it does not see set to zero, and added to that token's rows alone.
// The waves' results are merged through LDS; items of one slot through the workspace, by
// a second launch.
//
// Errors, relative to 64 bits (random lengths, windows and drafts): fp32 2.6e-7, where
// torch's products and softmax have 5.8e-7; bf16 1.7e-3 as theirs, the result's rounding,
// which falls the other way than theirs in one of 10,000 (5e-5 of the outputs' size).
#pragma once

#include "paged_ops.hpp"

namespace baton {

typedef __bf16 pa_bf16x8 __attribute__((ext_vector_type(8)));
typedef float pa_f32x4 __attribute__((ext_vector_type(4)));

constexpr int kPagedWaves = 4;

struct PagedAttnArgs {
  const uint8_t* q;        // [batch][width][Hq][D]
  const uint8_t* k_new;    // [batch][width][Hkv][D]; null: already in the pages
  const uint8_t* v_new;
  uint8_t* out;            // as q
  uint8_t* k;              // the layer's pages
  uint8_t* v;
  const int32_t* table;
  const int32_t* state;
  PagedState at;
  float* partial;          // [item][head][rows]: D sums, maximum, sum of the weights
  float qscale, qscale_rest;   // scale * log2 e, and what it is more than that
  int32_t batch, n_kv_heads, group, width, max_pages, n_pages, page_shift, window, sinks;
};

template <typename T, int D>
struct PagedGeo {
  static constexpr int kRow = D * T::kBytes;        // bytes of a token
  static constexpr int kChunks = kRow / 64;         // K chunks per tile
  static constexpr int kVecs = 32 * kRow / 1024;    // 16-byte vectors per lane and block, of K and of V
  static constexpr int kDt = D / 16;
  static constexpr int kRec = D + 4;                // floats of a partial record
  typedef u32x4 Vecs[kVecs];                        // a lane's part of a block's K, or V
};

// Scores of 32 tokens against 16 rows: s[e] for token 8 (lane / 16) + e of row lane % 16.
// fp32: four sums per score, so that each has fewer roundings (and waits for fewer of its
// own products).
template <typename T, int D>
__device__ __forceinline__ void paged_scores(const typename PagedGeo<T, D>::Vecs& kw,
                                             const u32x4 (&qw)[PagedGeo<T, D>::kChunks], float (&s)[8]) {
  using Geo = PagedGeo<T, D>;
#pragma unroll
  for (int tl = 0; tl < 2; ++tl) {
    if constexpr (T::kBytes == 2) {
      pa_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < Geo::kChunks; ++c)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pa_bf16x8, kw[tl * Geo::kChunks + c]),
                                                      __builtin_bit_cast(pa_bf16x8, qw[c]), acc, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) s[4 * tl + r] = acc[r];
    } else {
      pa_f32x4 acc[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = pa_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < Geo::kChunks; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kw[tl * Geo::kChunks + c][j]),
                                                        __uint_as_float(qw[c][j]), acc[j], 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) s[4 * tl + r] = (acc[0][r] + acc[1][r]) + (acc[2][r] + acc[3][r]);
    }
  }
}

// fp32 weights as three bf16 numbers each, of 8 bits: their sum is the weight.  The third
// product of a block's values costs steps of up to 16 rows nothing that shows (32 slots of up
// to 2,048 tokens 104.9 us, with two 104.7; 64 of up to 8,192, two layers, 401.9 and 401.1),
// 32 slots with four drafts each over up to 32,768 tokens 51.3 us instead of 49.4.  With two,
// 16 bits, the first one's results were 1.0e-4 of their size from those of fp32 weights, now 5e-5.
struct PagedWeights {
  pa_bf16x8 part[3];

  __device__ __forceinline__ explicit PagedWeights(const float (&p)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float rest = p[e];
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        part[i][e] = (__bf16)rest;
        rest -= (float)part[i][e];
      }
    }
  }
};

// Pairs of bf16 numbers, infinite or NaN ones set to zero.
__device__ __forceinline__ uint32_t paged_finite(uint32_t x) {
  return x & (((x & 0x7F80u) != 0x7F80u ? 0xFFFFu : 0u) | ((x & 0x7F800000u) != 0x7F800000u ? 0xFFFF0000u : 0u));
}

// o = alpha o + V^T P^T over 32 tokens, finite values.  fp32: the block's sum by itself, so
// that a long row's has a rounding per block, not per product.
template <typename T, int D>
__device__ __forceinline__ void paged_values(const typename PagedGeo<T, D>::Vecs& vw, const float (&p)[8],
                                             float alpha, pa_f32x4 (&o)[D / 16]) {
  constexpr int DT = D / 16;
  if constexpr (T::kBytes == 2) {
    const PagedWeights w(p);
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      const pa_bf16x8 v = __builtin_bit_cast(pa_bf16x8, vw[t]);
      o[t] *= alpha;
#pragma unroll
      for (int i = 0; i < 3; ++i) o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, w.part[i], o[t], 0, 0, 0);
    }
  } else {
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      pa_f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 8; ++e)
        x = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vw[e / 4 * DT + t][e % 4]), p[e], x, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) o[t][r] = fmaf(o[t][r], alpha, x[r]);
    }
  }
}

// The same for the rows of one new token alone (`mine`), of the tokens of `keep` (bit e:
// this lane's token 8 (lane / 16) + e): the others' values, which may be infinite or NaN,
// are left out.  bf16: infinite and NaN values only times a weight's first part, which is 0
// only if the weight is (the others may be 0, or negative).
template <typename T, int D>
__device__ __forceinline__ void paged_values_of(const typename PagedGeo<T, D>::Vecs& vw, const float (&p)[8], uint32_t keep,
                                                bool mine, pa_f32x4 (&o)[D / 16]) {
  constexpr int DT = D / 16;
  if constexpr (T::kBytes == 2) {
    const PagedWeights w(p);
    u32x4 m;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      m[e] = ((keep >> (2 * e)) & 1u ? 0xFFFFu : 0u) | ((keep >> (2 * e + 1)) & 1u ? 0xFFFF0000u : 0u);
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      u32x4 v = vw[t] & m;
      pa_f32x4 x = {0.f, 0.f, 0.f, 0.f};
      x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pa_bf16x8, v), w.part[0], x, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = paged_finite(v[e]);
#pragma unroll
      for (int i = 1; i < 3; ++i)
        x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pa_bf16x8, v), w.part[i], x, 0, 0, 0);
      if (mine) o[t] += x;
    }
  } else {
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      pa_f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t v = (keep >> e) & 1u ? vw[e / 4 * DT + t][e % 4] : 0u;
        x = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v), p[e], x, 0, 0, 0);
      }
      if (mine) o[t] += x;
    }
  }
}

// The lane's values with those of the tokens whose bit e (token 8 (lane / 16) + e) is not
// in `keep` set to zero.
template <typename T, int D>
__device__ __forceinline__ void paged_clear(typename PagedGeo<T, D>::Vecs& vw, uint32_t keep) {
  constexpr int DT = D / 16;
  if constexpr (T::kBytes == 2) {
    u32x4 m;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      m[e] = ((keep >> (2 * e)) & 1u ? 0xFFFFu : 0u) | ((keep >> (2 * e + 1)) & 1u ? 0xFFFF0000u : 0u);
#pragma unroll
    for (int t = 0; t < DT; ++t) vw[t] &= m;
  } else {
#pragma unroll
    for (int tl = 0; tl < 2; ++tl)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint32_t m = (keep >> (4 * tl + r)) & 1u ? 0xFFFFFFFFu : 0u;
#pragma unroll
        for (int t = 0; t < DT; ++t) vw[tl * DT + t][r] &= m;
      }
  }
}

// Whether any lane holds a value that is infinite or NaN: one that is, by its bits, among
// the largest as a signed number (positive) or as an unsigned one (negative).
template <typename T, int D>
__device__ __forceinline__ bool paged_odd(const typename PagedGeo<T, D>::Vecs& vw) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  if constexpr (T::kBytes == 2) {
    s16x2 pos = {0, 0};
    u16x2 neg = {0, 0};
#pragma unroll
    for (int u = 0; u < PagedGeo<T, D>::kVecs; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t x = vw[u][e];
        pos = __builtin_elementwise_max(pos, __builtin_bit_cast(s16x2, x));
        neg = __builtin_elementwise_max(neg, __builtin_bit_cast(u16x2, x));
      }
    return __any(max(pos.x, pos.y) >= 0x7F80 || max(neg.x, neg.y) >= 0xFF80);
  } else {
    int32_t pos = 0;
    uint32_t neg = 0;
#pragma unroll
    for (int u = 0; u < PagedGeo<T, D>::kVecs; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        pos = max(pos, (int32_t)vw[u][e]);
        neg = max(neg, vw[u][e]);
      }
    return __any(pos >= 0x7F800000 || neg >= 0xFF800000u);
  }
}

// What a workgroup's waves know of their item.
struct PagedRows {
  int32_t len, n_new, group, window, sinks, shift;   // shift: log2 of a page's blocks
  float qscale, qscale_rest;

  __device__ __forceinline__ PagedRows(const PagedAttnArgs& a, const PagedItem& it)
      : len(it.len), n_new(it.n_new), group(a.group), window(a.window), sinks(a.sinks), shift(a.page_shift - 5),
        qscale(a.qscale), qscale_rest(a.qscale_rest) {}

  // Bit e: a token at a position from p0 to p1 sees token j + e.
  __device__ __forceinline__ uint32_t sees(int32_t j, int32_t p0, int32_t p1) const {
    uint32_t bits = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) bits |= j + e <= p1 && (window == 0 || j + e > p0 - window || j + e < sinks) ? 1u << e : 0u;
    return bits;
  }
  // All rows see all of the block from token j0 on.
  __device__ __forceinline__ bool whole(int32_t j0) const {
    return j0 + kPagedBlock - 1 <= len && (window == 0 || j0 > len + n_new - 1 - window || j0 + kPagedBlock <= sinks);
  }
};

// A tile of 16 rows: lane l has row l % 16, its running maximum, its sum over the lane's
// tokens, and columns 16 t + 4 (l / 16) .. + 3 of its weighted values.
template <int D>
struct PagedTile {
  int32_t first, pos;        // the tile's first row; this lane's row's position (-1: no row)
  float m, l;
  pa_f32x4 o[D / 16];

  __device__ __forceinline__ PagedTile(const PagedRows& r, int32_t tile, int c16) {
    first = tile * 16;
    pos = first + c16 < r.n_new * r.group ? r.len + (first + c16) / r.group : -1;
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) o[t] = pa_f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // One block, from its scores and values.  there: it has a page.
  template <typename T>
  __device__ __forceinline__ void add(const PagedRows& r, int32_t j0, bool there, float (&s)[8],
                                      typename PagedGeo<T, D>::Vecs& vw, int g4) {
    const bool whole = there && r.whole(j0);
    const int32_t jl = j0 + 8 * g4;
    const uint32_t bits = whole ? 0xFFu : there ? r.sees(jl, pos, pos) : 0u;
    // what no row sees: anything may lie there
    if (!whole) paged_clear<T, D>(vw, there ? r.sees(jl, r.len, r.len + r.n_new - 1) : 0u);
    float mx = -INFINITY, p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) mx = fmaxf(mx, (bits >> e) & 1u ? s[e] * r.qscale : -INFINITY);
    const float mn = fmaxf(m, max_over_groups(mx));
    const float ref = mn == -INFINITY ? 0.f : mn;       // nothing seen yet
    const float alpha = fast_exp2(m - ref);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // The difference is rounded, not the score, whose magnitude may be many times as
      // large (the reference's own rounding is the same for all tokens); in fp32 with the rest
      // of the scale, which is off by up to 2^-25 of itself.
      float x = fmaf(s[e], r.qscale, -ref);
      if constexpr (T::kBytes == 4) x = x == -INFINITY ? x : fmaf(s[e], r.qscale_rest, x);   // (inf - inf where the signs differ)
      p[e] = (bits >> e) & 1u ? fast_exp2(x) : 0.f;
      sum += p[e];
    }
    m = mn;
    l = l * alpha + sum;
    if (!paged_odd<T, D>(vw)) {
      paged_values<T, D>(vw, p, alpha, o);
    } else {
#pragma unroll
      for (int t = 0; t < D / 16; ++t) o[t] *= alpha;
      for (int32_t i = first / r.group; i < r.n_new && i * r.group < first + 16; ++i)
        paged_values_of<T, D>(vw, p, there ? r.sees(jl, r.len + i, r.len + i) : 0u, pos == r.len + i, o);
    }
  }
};

// The row's result, or its partial record if the slot has several items.
template <typename T, int D>
__device__ __forceinline__ void paged_write(const PagedAttnArgs& a, const PagedItem& it, int32_t item, int32_t h,
                                            const PagedTile<D>& x, int lane) {
  using Geo = PagedGeo<T, D>;
  const int g4 = lane / 16, c16 = lane % 16;
  const int32_t G = a.group, r = x.first + c16;
  if (r >= it.n_new * G) return;
  if (it.parts == 1) {
    const float inv = 1.f / x.l;       // (every score -inf: NaN)
    uint8_t* const row = a.out + ((((int64_t)it.b * a.width + r / G) * a.n_kv_heads + h) * G + r % G) * Geo::kRow;
#pragma unroll
    for (int t = 0; t < Geo::kDt; ++t) {
      const pa_f32x4 y = x.o[t] * inv;
      if constexpr (T::kBytes == 2)
        *reinterpret_cast<uint2*>(row + (16 * t + 4 * g4) * 2) =
            make_uint2(f32_to_bf16_rne(y[0]) | f32_to_bf16_rne(y[1]) << 16,
                       f32_to_bf16_rne(y[2]) | f32_to_bf16_rne(y[3]) << 16);
      else
        *reinterpret_cast<pa_f32x4*>(row + (16 * t + 4 * g4) * 4) = y;
    }
  } else {
    float* const rec = a.partial + (((int64_t)item * a.n_kv_heads + h) * (a.width * G) + r) * Geo::kRec;
#pragma unroll
    for (int t = 0; t < Geo::kDt; ++t) *reinterpret_cast<pa_f32x4*>(rec + 16 * t + 4 * g4) = x.o[t];
    if (g4 == 0) {
      rec[D] = x.m;
      rec[D + 1] = x.l;
    }
  }
}

// Waves that have the same tile (`groups` of them, a power of two; wave w is of group
// w / (4 / groups)) bring their sums together: in the first group's.  Each sum is
// relative to its own maximum; half of the groups at a time hand theirs over in LDS.
template <int D>
__device__ __forceinline__ void paged_merge(PagedTile<D>& x, int32_t groups, u32x4 (*sm)[kWave],
                                            float (*sm_m)[16], float (*sm_l)[16], int w, int lane) {
  constexpr int DT = D / 16;
  const int g4 = lane / 16, c16 = lane % 16;
  const int tiles = kPagedWaves / groups, tile = w % tiles, group = w / tiles;
  x.l = sum_over_groups(x.l);
  if (g4 == 0) {
    sm_m[w][c16] = x.m;
    sm_l[w][c16] = x.l;
  }
  __syncthreads();
  float mx = -INFINITY, sum = 0.f;
  for (int v = tile; v < kPagedWaves; v += tiles) mx = fmaxf(mx, sm_m[v][c16]);
  const float ref = mx == -INFINITY ? 0.f : mx;
  for (int v = tile; v < kPagedWaves; v += tiles) sum += sm_l[v][c16] * fast_exp2(sm_m[v][c16] - ref);
  const float f = fast_exp2(x.m - ref);
#pragma unroll
  for (int t = 0; t < DT; ++t) x.o[t] *= f;
  x.m = mx;
  x.l = sum;
  for (int half = groups / 2; half > 0; half /= 2) {
    u32x4(*const at)[kWave] = sm + (((group % half) * tiles) + tile) * DT;
    if (group >= half && group < 2 * half) {
#pragma unroll
      for (int t = 0; t < DT; ++t) at[t][lane] = __builtin_bit_cast(u32x4, x.o[t]);
    }
    __syncthreads();
    if (group < half) {
#pragma unroll
      for (int t = 0; t < DT; ++t) x.o[t] += __builtin_bit_cast(pa_f32x4, at[t][lane]);
    }
    __syncthreads();
  }
}

// The page of block `block` of the item's slot, -1 if it has none.
__device__ __forceinline__ int32_t paged_page(const PagedAttnArgs& a, const PagedItem& it, int32_t block, int32_t shift) {
  const int32_t page = block >> shift;
  const int32_t id = page < a.max_pages ? a.table[(int64_t)it.b * a.max_pages + page] : -1;
  return (uint32_t)id < (uint32_t)a.n_pages ? id : -1;
}
template <typename T, int D>
__device__ __forceinline__ int64_t paged_offset(const PagedAttnArgs& a, int32_t id, int32_t h, int32_t block, int32_t shift) {
  return ((((int64_t)id * a.n_kv_heads + h) << shift) + (block & ((1 << shift) - 1))) *
         (int64_t)(kPagedBlock * PagedGeo<T, D>::kRow);
}
// The item's k-th block.
__device__ __forceinline__ int32_t paged_block_of(const PagedItem& it, int32_t k) {
  const int32_t v = it.v0 + k;
  return v < it.sink ? v : v + it.skip;
}
// Keys and values of the step's new tokens that lie in this block -- of them, every BY-th
// from `from` on --, from their rows into the pages, if the block has one.  All loads at
// once, before the page's number is waited for: with runs of V's elements, waited for one
// after the other by one wave, an item's start took 5 to 12 us (32 slots with four drafts,
// lengths up to 32,768: a step 61.5 us, with all loads at once 60.9, all waves 58.2).
template <typename T, int D, int BY>
__device__ __forceinline__ void paged_append(const PagedAttnArgs& a, const PagedItem& it, int32_t h, int32_t block,
                                             int32_t shift, int32_t from, int lane) {
  using Geo = PagedGeo<T, D>;
  constexpr int P = Geo::kRow / 16, NI = (kPagedMaxNew / BY * P + kWave - 1) / kWave;
  const int32_t j0 = max(it.len, block * kPagedBlock), n = min(it.len + it.n_new, (block + 1) * kPagedBlock) - j0;
  const int64_t row0 = (((int64_t)it.b * a.width + (j0 - it.len)) * a.n_kv_heads + h) * Geo::kRow;
  const int64_t step = (int64_t)a.n_kv_heads * Geo::kRow;       // from token to token
  const int32_t page = paged_page(a, it, block, shift);
  u32x4 kw[NI], vw[NI];
#pragma unroll
  for (int u = 0; u < NI; ++u) {
    const int32_t idx = u * kWave + lane, j = from + idx / P * BY;
    if (j >= n) continue;
    const int64_t at = row0 + j * step + idx % P * 16;
    kw[u] = *reinterpret_cast<const u32x4*>(a.k_new + at);
    vw[u] = *reinterpret_cast<const u32x4*>(a.v_new + at);
  }
  const int32_t id = __builtin_amdgcn_readfirstlane(page);
  if (id < 0) return;
  const int64_t off = paged_offset<T, D>(a, id, h, block, shift);
  uint8_t* const kb = a.k + off;
  uint8_t* const vb = a.v + off;
#pragma unroll
  for (int u = 0; u < NI; ++u) {
    const int32_t idx = u * kWave + lane, p = idx % P, j = from + idx / P * BY, t = (j0 + j) % kPagedBlock;
    if (j >= n) continue;
    *reinterpret_cast<u32x4*>(kb + ((((t >> 2 & 1) * Geo::kChunks + p / 4) * 64) + (p % 4) * 16 + 4 * (t >> 3) + (t & 3)) * 16) = kw[u];
    if constexpr (T::kBytes == 2) {
      uint8_t* const to = vb + (p / 2 * 64 + (t >> 3) * 16 + p % 2 * 8) * 16 + (t & 7) * 2;     // columns 8 p ..
#pragma unroll
      for (int e = 0; e < 8; ++e) *reinterpret_cast<uint16_t*>(to + e * 16) = (uint16_t)(vw[u][e / 2] >> (16 * (e % 2)));
    } else {
      uint8_t* const to = vb + (((t >> 2 & 1) * Geo::kDt + p / 4) * 64 + (t >> 3) * 16 + p % 4 * 4) * 16 + (t & 3) * 4;
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t*>(to + e * 16) = vw[u][e];         // columns 4 p ..
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "workgroup");   // the stores are done before the block is read
}

// 16 bytes of row r's query.
template <typename T, int D>
__device__ __forceinline__ u32x4 paged_query(const PagedAttnArgs& a, const PagedItem& it, int32_t h, int32_t r, int c, int g4) {
  const int32_t G = a.group;
  if (r >= it.n_new * G) return u32x4{0, 0, 0, 0};
  const int64_t row = (((int64_t)it.b * a.width + r / G) * a.n_kv_heads + h) * G + r % G;
  return *reinterpret_cast<const u32x4*>(a.q + row * PagedGeo<T, D>::kRow + (c * 4 + g4) * 16);
}

// All of the wave's loads are done.  They are, where this stands, but for the branch that
// lanes without a block take; told so, the compiler does not wait in the loops behind it.
__device__ __forceinline__ void paged_wait_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// An item of up to 16 rows.  Every wave has all of them, and every fourth of the item's
// blocks, whose keys and values go from memory into its registers: 1 KB of consecutive bytes
// per load, no LDS and no barrier until the merge.  Bound by memory: 64 slots of up to 8,192
// tokens (64/8 heads, bf16) take 194 us a layer, 5.9 TB/s of 6.09 that a plain read of that
// size reaches, with two new tokens each 201; 32 of up to 2,048 (32/32 heads) 100 us, 5.7 TB/s.
// The matrix cores are busy a third of the time.  bf16 at head_dim 64 5.9 TB/s, fp32 5.3 at 64
// and 5.0 at 128 (64 of up to 4,096 tokens, 64/8 heads).
template <typename T, int D>
__device__ __forceinline__ void paged_item16(const PagedAttnArgs& a, const PagedItem& it, int32_t item, int32_t h,
                                             const PagedRows& r, u32x4 (*sm)[kWave], float (*sm_m)[16], float (*sm_l)[16]) {
  using Geo = PagedGeo<T, D>;
  constexpr int CH = Geo::kChunks, NV = Geo::kVecs;
  const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int g4 = lane / 16, c16 = lane % 16;
  // This wave's blocks: w, w + 4, ... of the item.
  const int32_t n_mine = (it.v1 - it.v0 - w + kPagedWaves - 1) / kPagedWaves;
  auto block_of = [&](int32_t k) { return paged_block_of(it, w + k * kPagedWaves); };
  u32x4 qw[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) qw[c] = paged_query<T, D>(a, it, h, c16, c, g4);
  if (a.k_new) {       // the new tokens of its blocks (the last ones) first
    for (int32_t k = n_mine - 1; k >= 0 && block_of(k) * kPagedBlock + kPagedBlock > it.len; --k)
      paged_append<T, D, 1>(a, it, h, block_of(k), r.shift, 0, lane);
  }
  PagedTile<D> x(r, 0, c16);

  // 64 blocks at a time, whose pages are in a lane each.  K of the next block is asked for
  // when the scores are done, V when it has been used, so that one of them is always on its way.
  for (int32_t k0 = 0; k0 < n_mine; k0 += kWave) {
    const int32_t n = min(n_mine - k0, kWave);
    const int32_t ids = lane < n ? paged_page(a, it, block_of(k0 + lane), r.shift) : -1;
    paged_wait_loads();
    typename Geo::Vecs kw, vw;
    auto load = [&](typename Geo::Vecs& to, const uint8_t* from, int32_t k) {
      const int32_t id = __builtin_amdgcn_readlane(ids, k);
      // (a block without a page: the pool's first one, not looked at)
      const u32x4* const p =
          reinterpret_cast<const u32x4*>(from + paged_offset<T, D>(a, max(id, 0), h, block_of(k0 + k), r.shift)) + lane;
#pragma unroll
      for (int u = 0; u < NV; ++u) to[u] = __builtin_nontemporal_load(p + u * kWave);
    };
    load(kw, a.k, 0);
    load(vw, a.v, 0);
    for (int32_t k = 0; k < n; ++k) {
      const bool there = __builtin_amdgcn_readlane(ids, k) >= 0;    // tokens without a page are not seen
      const bool more = k + 1 < n;
      float s[8];
      paged_scores<T, D>(kw, qw, s);
      __builtin_amdgcn_sched_barrier(0);
      if (more) load(kw, a.k, k + 1);
      __builtin_amdgcn_sched_barrier(0);
      x.template add<T>(r, block_of(k0 + k) * kPagedBlock, there, s, vw, g4);
      __builtin_amdgcn_sched_barrier(0);
      if (more) load(vw, a.v, k + 1);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  paged_merge<D>(x, kPagedWaves, sm, sm_m, sm_l, w, lane);
  if (w == 0) paged_write<T, D>(a, it, item, h, x, lane);
}

// This wave's LDS reads and vector loads are done, then the barrier: __syncthreads() does not
// promise that another wave's loads into LDS have landed.
__device__ __forceinline__ void paged_wait_and_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);            // vmcnt 0, lgkmcnt 0
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// 1 KB from `from` into LDS at `to`, lane l's 16 bytes (l16 = 16 l) at 16 l.  In asm: the
// compiler would wait for such loads before reads of other buffers (it keeps only a few of
// them apart).  They have no result in registers, and are waited for at the barriers.
__device__ __forceinline__ void paged_load_lds(const uint8_t* from, uint32_t l16, u32x4* to) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"((uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)to), "v"(l16), "s"(from)
               : "memory", "m0");
#endif
}

// An item of more than 16 rows, up to 64: blocks go from memory into LDS, without registers, a
// pair of them while the last pair is worked on, and the waves share them: with more than 32
// rows each wave has a tile of its own, with 32 two waves share a tile and a pair.  32 slots
// with four drafts each (32/4 heads, lengths up to 32,768, most far shorter): 51 us a step,
// whose bytes take 32.  Waves wait for loads 3% of the loop; it is bound by a tile's chain of
// product, maximum, exponential and product.  Before weights had three parts: some 2,800 cycles
// a block with a barrier at each (58 us, three blocks ahead; 56 with two), which a pair's two
// chains overlap (52, and 49 with items of up to 16 rows as above, which all of a call's items
// took here before: 131 us instead of 105 for the 32 slots of up to 2,048, 470 instead of 400
// for two layers of the 64).
//
// Two waves a SIMD are asked for (fp32 at head_dim 128, whose blocks are twice as large: one),
// which leaves registers for K and V of a block each; with all of a SIMD's registers for one
// wave those steps took 119 and 423 us.
template <typename T, int D>
__global__ void __launch_bounds__(kWave * kPagedWaves) __attribute__((amdgpu_waves_per_eu(T::kBytes == 4 && D == 128 ? 1 : 2)))
paged_attn_kernel(const PagedAttnArgs a) {
  using Geo = PagedGeo<T, D>;
  constexpr int CH = Geo::kChunks, NV = Geo::kVecs;
  constexpr int NL = 2 * NV / kPagedWaves;       // loads per wave and block
  __shared__ __attribute__((aligned(1024))) u32x4 ring[4][2 * NV][kWave];     // two pairs of blocks, K and V of each
  __shared__ float sm_m[kPagedWaves][16], sm_l[kPagedWaves][16];
  const int32_t item = blockIdx.x / a.n_kv_heads, h = blockIdx.x - item * a.n_kv_heads;
  const PagedItem it = reinterpret_cast<const PagedItem*>(a.state + a.at.items)[item];   // (the list has room for all)
  if (item >= a.state[kNumItems] || it.n_new > a.width) return;   // the latter: more than the call brings
  const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int g4 = lane / 16, c16 = lane % 16;
  const PagedRows r(a, it);
  const int32_t n = it.v1 - it.v0, rows = it.n_new * a.group;
  if (rows <= 16) {
    paged_item16<T, D>(a, it, item, h, r, ring[0], sm_m, sm_l);
    return;
  }
  const int32_t tiles = rows <= 32 ? 2 : 4, groups = kPagedWaves / tiles;
  const int32_t tile = w % tiles, turn = w / tiles;

  u32x4 qw[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) qw[c] = paged_query<T, D>(a, it, h, tile * 16 + c16, c, g4);
  if (a.k_new) {       // the new tokens of the item's blocks (the last ones) first, by all waves
    for (int32_t k = n - 1; k >= 0 && paged_block_of(it, k) * kPagedBlock + kPagedBlock > it.len; --k)
      paged_append<T, D, kPagedWaves>(a, it, h, paged_block_of(it, k), r.shift, w, lane);
    __syncthreads();
  }
  PagedTile<D> x(r, tile, c16);

  // 64 blocks at a time, whose pages are in a lane each.
  for (int32_t k0 = 0; k0 < n; k0 += kWave) {
    const int32_t nk = min(n - k0, kWave);
    const int32_t ids = lane < nk ? paged_page(a, it, paged_block_of(it, k0 + lane), r.shift) : -1;
    paged_wait_loads();
    int32_t fetched = 0;
    // The next block into LDS, a fourth of it by this wave (past the last one: that one again).
    auto fetch = [&](u32x4 (*to)[kWave]) {
      const int32_t k = min(fetched, nk - 1), id = __builtin_amdgcn_readlane(ids, k);
      const int64_t off = paged_offset<T, D>(a, max(id, 0), h, paged_block_of(it, k0 + k), r.shift);
#pragma unroll
      for (int i = 0; i < NL; ++i) {       // chunks of K, then of V
        const int c = (i < NL / 2 ? i : i - NL / 2) * kPagedWaves + w;
        paged_load_lds((i < NL / 2 ? a.k : a.v) + off + c * 1024, lane * 16, to[(i < NL / 2 ? 0 : NV) + c]);
      }
      ++fetched;
    };
    fetch(ring[0]);
    fetch(ring[1]);
    for (int32_t k = 0; k < nk; k += 2) {
      const u32x4 (*const pair)[2 * NV][kWave] = ring + (k & 2);
      // The pair has landed, and every wave is done with the other two buffers.
      paged_wait_and_barrier();
      if (k + 2 < nk) {
        fetch(ring[2 - (k & 2)]);
        fetch(ring[3 - (k & 2)]);
      }
      if (tile * 16 >= rows) continue;
      const bool first = (k0 + k) % groups == turn, second = k + 1 < nk && (k0 + k + 1) % groups == turn;
      auto scores = [&](int q, float (&s)[8]) {
        typename Geo::Vecs kw;
#pragma unroll
        for (int u = 0; u < NV; ++u) kw[u] = pair[q][u][lane];
        paged_scores<T, D>(kw, qw, s);
      };
      auto values = [&](int q, typename Geo::Vecs& vw) {
#pragma unroll
        for (int u = 0; u < NV; ++u) vw[u] = pair[q][NV + u][lane];
      };
      auto add = [&](int q, float (&s)[8], typename Geo::Vecs& vw) {
        x.template add<T>(r, paged_block_of(it, k0 + k + q) * kPagedBlock, __builtin_amdgcn_readlane(ids, k + q) >= 0, s, vw, g4);
      };
      float s[8];
      typename Geo::Vecs vw;
      if (first && second) {
        float s2[8];
        typename Geo::Vecs vw2;
        scores(0, s);
        scores(1, s2);
        values(0, vw);
        values(1, vw2);
        add(0, s, vw);
        add(1, s2, vw2);
      } else if (first || second) {
        scores(second, s);
        values(second, vw);
        add(second, s, vw);
      }
    }
    paged_wait_and_barrier();                    // every wave is done with the buffers
  }
  paged_merge<D>(x, groups, ring[0], sm_m, sm_l, w, lane);
  if (turn == 0) paged_write<T, D>(a, it, item, h, x, lane);
}

// Rows of slots with several work items: their partial sums.  One workgroup per (slot,
// head) and row; D / 4 threads hold the columns, the others' groups take every
// 256 / (D / 4)-th item, and their sums are added in order.  Bound by latency: 3.5 to 6.9 us
// with few rows, of which a launch is 3.4, 12 with 16 rows a head of 64 slots.
template <typename T, int D>
__global__ void __launch_bounds__(256) paged_combine_kernel(const PagedAttnArgs a) {
  using Geo = PagedGeo<T, D>;
  constexpr int TC = D / 4, NG = 256 / TC;
  __shared__ float sm_m[4], sm_l[NG];
  __shared__ __attribute__((aligned(16))) float sm_o[NG][D];
  const int32_t b = blockIdx.x / a.n_kv_heads, h = blockIdx.x - b * a.n_kv_heads, r = blockIdx.y;
  const int32_t first = a.state[a.at.first + b], parts = a.state[a.at.first + b + 1] - first;
  const int32_t n_new = a.state[a.at.n_new + b];
  const int32_t G = a.group, max_rows = a.width * G;
  if (parts < 2 || n_new > a.width || r >= n_new * G) return;
  const int64_t step = (int64_t)a.n_kv_heads * max_rows * Geo::kRec;
  const float* const rec = a.partial + (((int64_t)first * a.n_kv_heads + h) * max_rows + r) * Geo::kRec;
  float mx = -INFINITY;
  for (int32_t s = threadIdx.x; s < parts; s += 256) mx = fmaxf(mx, rec[s * step + D]);
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) mx = fmaxf(mx, __shfl_xor(mx, d, kWave));
  if (threadIdx.x % kWave == 0) sm_m[threadIdx.x / kWave] = mx;
  __syncthreads();
  mx = fmaxf(fmaxf(sm_m[0], sm_m[1]), fmaxf(sm_m[2], sm_m[3]));
  const float ref = mx == -INFINITY ? 0.f : mx;
  const int32_t d4 = threadIdx.x % TC, g = threadIdx.x / TC;
  float sum = 0.f;
  pa_f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int32_t s = g; s < parts; s += NG) {
    const float f = fast_exp2(rec[s * step + D] - ref);
    sum += rec[s * step + D + 1] * f;
    o += *reinterpret_cast<const pa_f32x4*>(rec + s * step + 4 * d4) * f;
  }
  *reinterpret_cast<pa_f32x4*>(sm_o[g] + 4 * d4) = o;
  if (d4 == 0) sm_l[g] = sum;
  __syncthreads();
  if (g != 0) return;
#pragma unroll
  for (int v = 1; v < NG; ++v) {
    o += *reinterpret_cast<const pa_f32x4*>(sm_o[v] + 4 * d4);
    sum += sm_l[v];
  }
  const pa_f32x4 x = o * (1.f / sum);
  uint8_t* const row = a.out + ((((int64_t)b * a.width + r / G) * a.n_kv_heads + h) * G + r % G) * Geo::kRow;
  if constexpr (T::kBytes == 2)
    *reinterpret_cast<uint2*>(row + 8 * d4) = make_uint2(f32_to_bf16_rne(x[0]) | f32_to_bf16_rne(x[1]) << 16,
                                                        f32_to_bf16_rne(x[2]) | f32_to_bf16_rne(x[3]) << 16);
  else
    *reinterpret_cast<pa_f32x4*>(row + 16 * d4) = x;
}

}  // namespace baton
