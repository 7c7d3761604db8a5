// Attention of a step's new tokens -- one per query, or a few drafted ones behind it --
// over a cache in pages (paged_ops.hpp: its layout, and the work items).
//
// The rows of a (slot, kv-head) are its new tokens' query heads, row i G + q for query
// head q of the head's G at new token i, up to 64 of them, in MT tiles of 16.  Token j
// is visible to new token i, at position p = len + i, if j <= p and, with a window W and
// S sinks, j > p - W or j < S.
//
// A work item is a run of blocks of 32 tokens of one slot; a workgroup of four waves
// takes an item for one kv-head, wave w every fourth of its blocks.  Per block, with the
// matrix cores' 16x16 tiles:
//  * scores, transposed: S^T = K Q^T, K's rows being the tokens.  Lane l has row l % 16's
//    scores of the tokens 8 (l / 16) .. + 7.
//  * softmax with a running maximum per row, in fp32, base 2.
//  * O^T += V^T P^T, where lane l supplies as it holds them its own row's weights, and
//    accumulates columns 16 t + 4 (l / 16) .. + 3 of row l % 16.
// bf16: weights are taken as a sum of two bf16 numbers, so that they have 16 bits for
// their product with the values; the values' and keys' products are exact in fp32.
// fp32: products in fp32 (v_mfma_f32_16x16x4_f32).
// K and V come from memory in the order of the operands, without a trip through LDS.
// Values that are infinite or NaN: a weight of 0 would turn them into NaN for rows that
// do not see them.  Blocks that hold any are multiplied once for each new token, with
// what it does not see set to zero, and added to that token's rows alone.
// The waves' results are merged through LDS; items of one slot through the workspace, by
// a second launch.
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
  float qscale;            // scale * log2 e
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

// Keys and values of the step's new tokens that lie in this block, from their rows into
// the pages.  The wave that stores them reads the block back itself.
template <typename T, int D>
__device__ __forceinline__ void paged_append(const PagedAttnArgs& a, const PagedItem& it, int32_t h, int32_t block,
                                             uint8_t* kb, uint8_t* vb, int lane) {
  using Geo = PagedGeo<T, D>;
  const int32_t j0 = max(it.len, block * kPagedBlock), j1 = min(it.len + it.n_new, (block + 1) * kPagedBlock);
  for (int32_t j = j0; j < j1; ++j) {
    const int32_t t = j % kPagedBlock;
    const int64_t row = (((int64_t)it.b * a.width + (j - it.len)) * a.n_kv_heads + h) * Geo::kRow;
    const int tl = (t >> 2) & 1, g = t >> 3, i = 4 * g + (t & 3);
    if (lane < Geo::kRow / 16) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(a.k_new + row + lane * 16);
      *reinterpret_cast<u32x4*>(kb + (((tl * Geo::kChunks + lane / 4) * 64) + (lane % 4) * 16 + i) * 16) = w;
    }
    for (int d = lane; d < D; d += kWave) {
      if constexpr (T::kBytes == 2)
        *reinterpret_cast<uint16_t*>(vb + ((d / 16 * 64) + g * 16 + d % 16) * 16 + (t & 7) * 2) =
            reinterpret_cast<const uint16_t*>(a.v_new + row)[d];
      else
        *reinterpret_cast<uint32_t*>(vb + (((tl * Geo::kDt + d / 16) * 64) + g * 16 + d % 16) * 16 + (t & 3) * 4) =
            reinterpret_cast<const uint32_t*>(a.v_new + row)[d];
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "workgroup");   // the stores are done before the block is read
}

// Scores of 32 tokens against 16 rows: s[e] for token 8 (lane / 16) + e of row lane % 16.
template <typename T, int D>
__device__ __forceinline__ void paged_scores(const typename PagedGeo<T, D>::Vecs& kw,
                                             const u32x4 (&qw)[PagedGeo<T, D>::kChunks], float (&s)[8]) {
  using Geo = PagedGeo<T, D>;
#pragma unroll
  for (int tl = 0; tl < 2; ++tl) {
    pa_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < Geo::kChunks; ++c) {
      const u32x4 kk = kw[tl * Geo::kChunks + c], qq = qw[c];
      if constexpr (T::kBytes == 2) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pa_bf16x8, kk),
                                                      __builtin_bit_cast(pa_bf16x8, qq), acc, 0, 0, 0);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kk[j]), __uint_as_float(qq[j]), acc, 0, 0, 0);
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) s[4 * tl + r] = acc[r];
  }
}

// o += V^T P^T over 32 tokens, finite values.
template <typename T, int D>
__device__ __forceinline__ void paged_values(const typename PagedGeo<T, D>::Vecs& vw, const float (&p)[8],
                                             pa_f32x4 (&o)[D / 16]) {
  constexpr int DT = D / 16;
  if constexpr (T::kBytes == 2) {
    pa_bf16x8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      hi[e] = (__bf16)p[e];
      lo[e] = (__bf16)(p[e] - (float)hi[e]);
    }
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      const pa_bf16x8 v = __builtin_bit_cast(pa_bf16x8, vw[t]);
      o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, hi, o[t], 0, 0, 0);
      o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, lo, o[t], 0, 0, 0);
    }
  } else {
#pragma unroll
    for (int tl = 0; tl < 2; ++tl)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int t = 0; t < DT; ++t)
          o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vw[tl * DT + t][r]), p[4 * tl + r], o[t], 0, 0, 0);
  }
}

// The same for the rows of one new token alone (`mine`), of the tokens of `keep` (bit e:
// this lane's token 8 (lane / 16) + e): the others' values, which may be infinite or NaN,
// are left out.  bf16: weights of 8 bits, of which none is 0 beside an infinite value.
template <typename T, int D>
__device__ __forceinline__ void paged_values_of(const typename PagedGeo<T, D>::Vecs& vw, const float (&p)[8], uint32_t keep,
                                                bool mine, pa_f32x4 (&o)[D / 16]) {
  constexpr int DT = D / 16;
  if constexpr (T::kBytes == 2) {
    pa_bf16x8 hi;
    u32x4 m;
#pragma unroll
    for (int e = 0; e < 8; ++e) hi[e] = (__bf16)p[e];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      m[e] = ((keep >> (2 * e)) & 1u ? 0xFFFFu : 0u) | ((keep >> (2 * e + 1)) & 1u ? 0xFFFF0000u : 0u);
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      const pa_f32x4 x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pa_bf16x8, vw[t] & m), hi,
                                                                 pa_f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
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

// Whether any lane holds a value that is infinite or NaN.
template <typename T, int D>
__device__ __forceinline__ bool paged_odd(const typename PagedGeo<T, D>::Vecs& vw) {
  uint32_t any = 0;
#pragma unroll
  for (int u = 0; u < PagedGeo<T, D>::kVecs; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // an exponent of all ones carries into the bit above it
      if constexpr (T::kBytes == 2) any |= (vw[u][e] & 0x7F807F80u) + 0x00800080u;
      else any |= (vw[u][e] & 0x7F800000u) + 0x00800000u;
    }
  return __any((any & (T::kBytes == 2 ? 0x80008000u : 0x80000000u)) != 0);
}

template <typename T, int D, int MT>
__global__ void __launch_bounds__(kWave * kPagedWaves) paged_attn_kernel(const PagedAttnArgs a) {
  using Geo = PagedGeo<T, D>;
  constexpr int DT = Geo::kDt, CH = Geo::kChunks, NV = Geo::kVecs;
  constexpr bool kQInLds = MT > 1;         // registers hold one tile's queries
  constexpr int kMerge = kPagedWaves / 2 * MT * DT, kQueries = kQInLds ? MT * CH : 0;
  // The rows' queries; then the merge: half of the waves' sums at a time.
  __shared__ u32x4 sm[kMerge > kQueries ? kMerge : kQueries][kWave];
  __shared__ float sm_m[kPagedWaves][MT * 16], sm_l[kPagedWaves][MT * 16];   // rows' maxima and sums
  const int32_t item = blockIdx.x / a.n_kv_heads, h = blockIdx.x - item * a.n_kv_heads;
  if (item >= a.state[kNumItems]) return;
  const PagedItem it = reinterpret_cast<const PagedItem*>(a.state + a.at.items)[item];
  if (it.n_new > a.width) return;          // a prompt: it comes whole, with its attention done
  const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int g4 = lane / 16, c16 = lane % 16;
  const int32_t G = a.group, rows = it.n_new * G;
  const int32_t p_first = it.len, p_last = it.len + it.n_new - 1;
  const int32_t shift = a.page_shift - 5;                 // blocks per page
  const int32_t* const table = a.table + (int64_t)it.b * a.max_pages;

  // This wave's blocks: v0 + w, + 4, ...  Their pages, a lane each, 64 at a time.
  const int32_t n_mine = (it.v1 - it.v0 - w + kPagedWaves - 1) / kPagedWaves;
  auto block_of = [&](int32_t k) {
    const int32_t v = it.v0 + w + k * kPagedWaves;
    return v < it.sink ? v : v + it.skip;
  };
  auto pages_from = [&](int32_t k0) {
    const int32_t page = block_of(k0 + lane) >> shift;
    const int32_t id = k0 + lane < n_mine && page < a.max_pages ? table[page] : -1;
    return (uint32_t)id < (uint32_t)a.n_pages ? id : -1;
  };
  int32_t ids = pages_from(0);
  auto offset_of = [&](int32_t id, int32_t block) {
    return ((((int64_t)id * a.n_kv_heads + h) << shift) + (block & ((1 << shift) - 1))) *
           (int64_t)(kPagedBlock * Geo::kRow);
  };
  if (a.k_new) {       // the new tokens of its blocks (the last ones) first
    for (int32_t k = n_mine - 1; k >= 0 && block_of(k) * kPagedBlock + kPagedBlock > it.len; --k) {
      const int32_t block = block_of(k), page = block >> shift;
      const int32_t id = __builtin_amdgcn_readfirstlane(page < a.max_pages ? table[page] : -1);
      if ((uint32_t)id >= (uint32_t)a.n_pages) continue;
      const int64_t off = offset_of(id, block);
      paged_append<T, D>(a, it, h, block, a.k + off, a.v + off, lane);
    }
  }

  // The rows: their queries as the second operand, and their positions.
  u32x4 qr[CH];
  int32_t pos[MT];
  const uint8_t* const q = a.q + ((int64_t)it.b * a.width * a.n_kv_heads * G + h * G) * Geo::kRow;
  auto query = [&](int32_t r, int c) {
    return r < rows ? *reinterpret_cast<const u32x4*>(q + ((int64_t)(r / G) * a.n_kv_heads * G + r % G) * Geo::kRow +
                                                      (c * 4 + g4) * 16)
                    : u32x4{0, 0, 0, 0};
  };
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int32_t r = mt * 16 + c16;
    pos[mt] = r < rows ? it.len + r / G : -1;
  }
  if constexpr (kQInLds) {
#pragma unroll
    for (int u = w; u < MT * CH; u += kPagedWaves) sm[u][lane] = query(u / CH * 16 + c16, u % CH);
    __syncthreads();
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c) qr[c] = query(c16, c);
  }
  float m[MT], l[MT];
  pa_f32x4 o[MT][DT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    m[mt] = -INFINITY;
    l[mt] = 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t) o[mt][t] = pa_f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // K of the next block is asked for when the scores are done, V when it has been used, so
  // that one of them is always on its way.
  typename Geo::Vecs kw, vw;
  auto load = [&](typename Geo::Vecs& x, const uint8_t* from, int32_t k) {
    const int32_t id = __builtin_amdgcn_readlane(ids, k % kWave);
    // (a block without a page: the pool's first one, not looked at)
    const u32x4* const p = reinterpret_cast<const u32x4*>(from + offset_of(max(id, 0), block_of(k))) + lane;
#pragma unroll
    for (int u = 0; u < NV; ++u) x[u] = __builtin_nontemporal_load(p + u * kWave);
  };
  if (n_mine > 0) {
    load(kw, a.k, 0);
    load(vw, a.v, 0);
  }
  for (int32_t k = 0; k < n_mine; ++k) {
    const bool there = __builtin_amdgcn_readlane(ids, k % kWave) >= 0;    // tokens without a page are not seen
    const int32_t j0 = block_of(k) * kPagedBlock;
    if ((k + 1) % kWave == 0) ids = pages_from(k + 1);
    const bool more = k + 1 < n_mine;
    float s[MT][8];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if (mt > 0 && mt * 16 >= rows) break;
      if constexpr (kQInLds) {
        u32x4 qw[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) qw[c] = sm[mt * CH + c][lane];
        paged_scores<T, D>(kw, qw, s[mt]);
      } else {
        paged_scores<T, D>(kw, qr, s[mt]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (more) load(kw, a.k, k + 1);
    __builtin_amdgcn_sched_barrier(0);

    // All rows see all of the block, but where it holds new tokens or the window's start.
    const bool whole = there && j0 + kPagedBlock - 1 <= p_first &&
                       (a.window == 0 || j0 > p_last - a.window || j0 + kPagedBlock <= a.sinks);
    const int32_t jl = j0 + 8 * g4;                       // this lane's first token
    // Bit e: a token at a position from p0 to p1 sees token jl + e.
    auto sees = [&](int32_t p0, int32_t p1) {
      uint32_t bits = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int32_t j = jl + e;
        bits |= there && j <= p1 && (a.window == 0 || j > p0 - a.window || j < a.sinks) ? 1u << e : 0u;
      }
      return bits;
    };
    if (!whole) paged_clear<T, D>(vw, sees(p_first, p_last));   // what no row sees: anything may lie there
    const bool odd = paged_odd<T, D>(vw);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      if (mt > 0 && mt * 16 >= rows) break;
      if (whole) {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[mt][e] *= a.qscale;
      } else {
        const uint32_t bits = sees(pos[mt], pos[mt]);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[mt][e] = (bits >> e) & 1u ? s[mt][e] * a.qscale : -INFINITY;
      }
      float mx = s[mt][0], p[8];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[mt][e]);
      const float mn = fmaxf(m[mt], max_over_groups(mx));
      const float ref = mn == -INFINITY ? 0.f : mn;       // nothing seen yet
      const float alpha = fast_exp2(m[mt] - ref);
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = fast_exp2(s[mt][e] - ref);
        sum += p[e];
      }
      m[mt] = mn;
      l[mt] = l[mt] * alpha + sum;
#pragma unroll
      for (int t = 0; t < DT; ++t) o[mt][t] *= alpha;
      if (!odd) {
        paged_values<T, D>(vw, p, o[mt]);
      } else {
        for (int32_t i = mt * 16 / G; i < it.n_new && i * G < mt * 16 + 16; ++i)
          paged_values_of<T, D>(vw, p, sees(it.len + i, it.len + i), pos[mt] == it.len + i, o[mt]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (more) load(vw, a.v, k + 1);
    __builtin_amdgcn_sched_barrier(0);
  }

  // The waves' sums, each relative to its row's maximum in the wave, brought to the
  // largest of the four: two waves hand theirs to the other two, then one to the first.
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    l[mt] = sum_over_groups(l[mt]);
    if (g4 == 0) {
      sm_m[w][mt * 16 + c16] = m[mt];
      sm_l[w][mt * 16 + c16] = l[mt];
    }
  }
  __syncthreads();                         // (and the queries have been read)
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float mx = sm_m[0][mt * 16 + c16], sum = 0.f;
#pragma unroll
    for (int v = 1; v < kPagedWaves; ++v) mx = fmaxf(mx, sm_m[v][mt * 16 + c16]);
    const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
    for (int v = 0; v < kPagedWaves; ++v) sum += sm_l[v][mt * 16 + c16] * fast_exp2(sm_m[v][mt * 16 + c16] - ref);
    const float f = fast_exp2(m[mt] - ref);
#pragma unroll
    for (int t = 0; t < DT; ++t) o[mt][t] *= f;
    m[mt] = mx;
    l[mt] = sum;
  }
#pragma unroll
  for (int half = kPagedWaves / 2; half > 0; half /= 2) {
    if (w >= half && w < 2 * half) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int t = 0; t < DT; ++t) sm[((w - half) * MT + mt) * DT + t][lane] = __builtin_bit_cast(u32x4, o[mt][t]);
    }
    __syncthreads();
    if (w < half) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int t = 0; t < DT; ++t) o[mt][t] += __builtin_bit_cast(pa_f32x4, sm[(w * MT + mt) * DT + t][lane]);
    }
    __syncthreads();
  }
  if (w != 0) return;
  const int32_t parts = a.state[a.at.first + it.b + 1] - a.state[a.at.first + it.b];
  const int32_t max_rows = a.width * G;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int32_t r = mt * 16 + c16;
    if (r >= rows) continue;
    if (parts == 1) {
      const float inv = l[mt] == 0.f ? 0.f : 1.f / l[mt];
      uint8_t* const row = a.out + ((((int64_t)it.b * a.width + r / G) * a.n_kv_heads + h) * G + r % G) * Geo::kRow;
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const pa_f32x4 x = o[mt][t] * inv;
        if constexpr (T::kBytes == 2)
          *reinterpret_cast<uint2*>(row + (16 * t + 4 * g4) * 2) =
              make_uint2(f32_to_bf16_rne(x[0]) | f32_to_bf16_rne(x[1]) << 16,
                         f32_to_bf16_rne(x[2]) | f32_to_bf16_rne(x[3]) << 16);
        else
          *reinterpret_cast<pa_f32x4*>(row + (16 * t + 4 * g4) * 4) = x;
      }
    } else {
      float* const rec = a.partial + (((int64_t)item * a.n_kv_heads + h) * max_rows + r) * Geo::kRec;
#pragma unroll
      for (int t = 0; t < DT; ++t) *reinterpret_cast<pa_f32x4*>(rec + 16 * t + 4 * g4) = o[mt][t];
      if (g4 == 0) {
        rec[D] = m[mt];
        rec[D + 1] = l[mt];
      }
    }
  }
}

// Rows of slots with several work items: their partial sums.  One workgroup per (slot,
// head) and row; D / 4 threads hold the columns, the others' groups take every
// 256 / (D / 4)-th item, and their sums are added in order.
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
  const pa_f32x4 x = o * (sum == 0.f ? 0.f : 1.f / sum);
  uint8_t* const row = a.out + ((((int64_t)b * a.width + r / G) * a.n_kv_heads + h) * G + r % G) * Geo::kRow;
  if constexpr (T::kBytes == 2)
    *reinterpret_cast<uint2*>(row + 8 * d4) = make_uint2(f32_to_bf16_rne(x[0]) | f32_to_bf16_rne(x[1]) << 16,
                                                        f32_to_bf16_rne(x[2]) | f32_to_bf16_rne(x[3]) << 16);
  else
    *reinterpret_cast<pa_f32x4*>(row + 16 * d4) = x;
}

}  // namespace baton
