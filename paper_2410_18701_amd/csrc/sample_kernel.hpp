// One token per row of logits, from a given uniform number.
//
// With w_i = exp((l_i - max) / T), the tokens in order of (l descending, index
// ascending), and n the length of the shortest of three prefixes of that order --
// the first top_k tokens; the fewest whose weight reaches top_p times the weight
// of the first top_k; those with w >= min_p (the first one always) -- the token
// drawn is the first, in order of index, at which the weight of the kept tokens so
// far exceeds u times all of it.
//
// A result is an index, so weights and sums have to be the same whatever the order
// they are formed in, and near those of 64-bit arithmetic: a weight is
// computed in double precision (relative error about 2^-52) and rounded to a whole
// number of 2^-shift, shift = 62 - ceil(log2 V) at most 51.  Sums of whole numbers are
// exact, so atomics in any order give the same sums, and the boundary between two
// tokens is off by about sqrt(V) 2^-(shift + 1) at most.
//
// One workgroup of 16 waves per row.  The row is read once from memory into LDS (what
// does not fit is read again); wave w owns the w-th of 16 contiguous parts of
// it, 16 bytes per lane and step.
//  * prefixes: 1024 bins of equal width over the top of the values' range hold counts
//    and weights (floats' own bits would put most tokens into a few bins, whose
//    atomics then queue); a scan finds the bin in which a prefix ends; that
//    bin's tokens, a few dozen, are sorted in LDS.  More than fit (equal
//    logits, mostly) are first narrowed by bins over the bits of their floats, and if
//    one value alone has too many, its tokens are counted off in order of index.
//  * the draw: kept weights per wave, then the tokens of the wave's part in
//    which the target lies.
// exp: 2^(j / 64) from a table, times a polynomial of degree 5 on half a step: relative
// error below 2^-53, in about 20 instructions.
#pragma once

#include "common.hpp"

namespace baton {
namespace {

constexpr int kSampleThreads = 1024, kSampleWaves = kSampleThreads / kWave;
constexpr int kSampleBins = 1024;        // == kSampleThreads: a bin per thread
constexpr int kSampleList = 2048;        // tokens sorted at most
constexpr int kSampleRowBytes = 112 << 10;   // of a row kept in LDS

struct SampleArgs {
  const uint8_t* logits;
  int64_t ld;                  // elements from row to row
  int32_t vocab, shift;        // weights are whole numbers of 2^-shift
  const float* temperature;    // [rows] each; null: 1, off, off, off
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* u;
  int32_t* tokens;
};

// Floats as unsigned numbers of the same order (no NaN, no -0).
__device__ __forceinline__ uint32_t float_key(float f) {
  const uint32_t b = __float_as_uint(f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_float(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

__device__ __forceinline__ uint64_t shfl_xor_u64(uint64_t x, int m) {
  return (uint64_t)__shfl_xor((uint32_t)(x >> 32), m, kWave) << 32 | __shfl_xor((uint32_t)x, m, kWave);
}
__device__ __forceinline__ uint64_t shfl_up_u64(uint64_t x, int d) {
  return (uint64_t)__shfl_up((uint32_t)(x >> 32), d, kWave) << 32 | __shfl_up((uint32_t)x, d, kWave);
}
__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t x) {
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) x += shfl_xor_u64(x, m);
  return x;
}

// floor(f * n) (UP: rounded up) for 0 <= f < 1: exact.
template <bool UP>
__device__ __forceinline__ uint64_t times_fraction(float f, uint64_t n) {
  const uint32_t b = __float_as_uint(f);
  const int e = (int)(b >> 23);                                  // f = m * 2^(e - 150)
  const uint32_t m = e ? (b & 0x7FFFFFu) | 0x800000u : b & 0x7FFFFFu;
  const int s = 150 - (e ? e : 1);                               // >= 24
  if (m == 0 || s >= 120) return UP && m != 0 && n != 0 ? 1 : 0;
  const unsigned __int128 x = (unsigned __int128)n * m;
  return (uint64_t)((x + (UP ? ((unsigned __int128)1 << s) - 1 : 0)) >> s);
}

// Rows of T = fp32 or bf16 (EPV elements per 16 bytes).
template <typename T>
struct SampleRow {
  static constexpr int EPV = Lane16<T>::kElems;
  const uint8_t* row;      // first element
  int32_t off;             // elements of the first vector in front of it
  int32_t vocab, n_vec, n_lds;
  u32x4* lds;

  __device__ __forceinline__ void widen(int32_t i, const u32x4& w, float (&x)[EPV]) const {
    Lane16<T>::widen(w, x);
#pragma unroll
    for (int e = 0; e < EPV; ++e) {
      const int32_t at = i * EPV - off + e;
      // outside the row: NaN, which every comparison leaves out; -0 as 0
      x[e] = at >= 0 && at < vocab ? x[e] + 0.f : __uint_as_float(0x7FC00000u);
    }
  }
  // A vector from memory; at the row's ends only the elements that are the row's.
  __device__ __forceinline__ u32x4 fetch(int32_t i) const {
    const int32_t at = i * EPV - off;
    if (at >= 0 && at + EPV <= vocab) return *reinterpret_cast<const u32x4*>(row + (int64_t)at * T::kBytes);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < EPV; ++e)
      if (at + e >= 0 && at + e < vocab) {
        if constexpr (T::kBytes == 4) w[e] = reinterpret_cast<const uint32_t*>(row)[at + e];
        else w[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[at + e] << (16 * (e % 2));
      }
    return u32x4{w[0], w[1], w[2], w[3]};
  }
  __device__ __forceinline__ u32x4 load(int32_t i) const { return i < n_lds ? lds[i] : fetch(i); }
};

struct SampleShared {
  double table[64];
  uint64_t weight[kSampleBins];
  uint32_t count[kSampleBins];
  uint64_t list[kSampleList];
  uint64_t scan[kSampleWaves];
  uint64_t part[kSampleWaves];
  float fmax[kSampleWaves], fmin[kSampleWaves];
  uint32_t kmin, kmax, n_list;
  int32_t found, found_at;
  uint64_t before;
  uint32_t key, index;
};

// Inclusive prefix sum over the workgroup; `total` gets the whole.
__device__ __forceinline__ uint64_t wg_scan(SampleShared& s, uint64_t x, uint64_t& total) {
  const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const uint64_t y = shfl_up_u64(x, d);
    x += lane >= d ? y : 0;
  }
  __syncthreads();
  if (lane == kWave - 1) s.scan[w] = x;
  __syncthreads();
  uint64_t before = 0;
  total = 0;
  for (int v = 0; v < kSampleWaves; ++v) {
    before += v < w ? s.scan[v] : 0;
    total += s.scan[v];
  }
  return before + x;
}

template <typename T>
__global__ void __launch_bounds__(kSampleThreads) sample_kernel(const SampleArgs a) {
  constexpr int EPV = Lane16<T>::kElems;
  extern __shared__ __attribute__((aligned(16))) u32x4 row_lds[];
  __shared__ SampleShared s;
  const int tid = threadIdx.x, lane = tid % kWave;
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int64_t r = blockIdx.x;
  SampleRow<T> row;
  row.row = a.logits + r * a.ld * T::kBytes;
  row.off = (int32_t)((reinterpret_cast<uintptr_t>(row.row) & 15u) / T::kBytes);
  row.vocab = a.vocab;
  row.n_vec = (row.off + a.vocab + EPV - 1) / EPV;
  row.n_lds = min(row.n_vec, kSampleRowBytes / 16);
  row.lds = row_lds;
  const int32_t per = (row.n_vec + kSampleWaves - 1) / kSampleWaves;   // vectors of a wave's part
  const int32_t v0 = w * per, v1 = min(v0 + per, row.n_vec);

  const float temperature = a.temperature ? a.temperature[r] : 1.f;
  const int32_t top_k = a.top_k ? a.top_k[r] : 0;
  const float top_p = a.top_p ? a.top_p[r] : 1.f;
  const float min_p = a.min_p ? a.min_p[r] : 0.f;
  const float u = a.u[r];

  // The row into LDS; its largest value and the smallest that is finite.
  float mx = -INFINITY, mn = INFINITY;
  for (int32_t i = v0 + lane; i < v1; i += kWave) {
    const u32x4 v = row.fetch(i);
    if (i < row.n_lds) row.lds[i] = v;
    float x[EPV];
    row.widen(i, v, x);
#pragma unroll
    for (int e = 0; e < EPV; ++e) {
      mx = fmaxf(mx, x[e]);
      mn = x[e] > -INFINITY ? fminf(mn, x[e]) : mn;
    }
  }
  if (tid < 64) s.table[tid] = exp2((double)tid / 64.0);
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) {
    mx = fmaxf(mx, __shfl_xor(mx, m, kWave));
    mn = fminf(mn, __shfl_xor(mn, m, kWave));
  }
  if (lane == 0) {
    s.fmax[w] = mx;
    s.fmin[w] = mn;
  }
  if (tid == 0) s.index = 0xFFFFFFFFu;
  __syncthreads();
  for (int v = 0; v < kSampleWaves; ++v) {
    mx = fmaxf(mx, s.fmax[v]);
    mn = fminf(mn, s.fmin[v]);
  }
  if (mx == -INFINITY) {      // no token can be drawn
    if (tid == 0) a.tokens[r] = -1;
    return;
  }
  if (!(temperature > 0.f) || top_k == 1 || min_p > 1.f) {     // the first of the largest
    for (int32_t i = v0 + lane; i < v1; i += kWave) {
      float x[EPV];
      row.widen(i, row.load(i), x);
#pragma unroll
      for (int e = EPV - 1; e >= 0; --e)
        if (x[e] == mx) atomicMin(&s.index, (uint32_t)(i * EPV - row.off + e));
    }
    __syncthreads();
    if (tid == 0) a.tokens[r] = (int32_t)s.index;
    return;
  }
  if (mx == INFINITY) mn = INFINITY;   // beside an infinity nothing finite has weight

  // The weight of a value, as a whole number: 0 for what is not >= mn (a NaN, -inf).
  const double scale = 64.0 * 1.4426950408889634074 / (double)temperature, top = (double)mx;
  const double unit = __longlong_as_double((int64_t)(1023 + a.shift) << 52);
  const double least = -64.0 * (a.shift + 2);
  auto weight_of = [&](float x) -> uint64_t {
    const double d = x == mx ? 0.0 : (double)x - top;
    const double y = d * scale;                                     // 64 log2 w
    if (!(y > least)) return 0;
    const double magic = 6755399441055744.0;                        // 1.5 * 2^52: rounds to a whole number
    const double t = y + magic;
    const int32_t j = (int32_t)__double_as_longlong(t);
    const double f = (y - (t - magic)) * 0.010830424696249145;      // ln 2 / 64
    double p = fma(f, 1.0 / 120.0, 1.0 / 24.0);
    p = fma(p, f, 1.0 / 6.0);
    p = fma(p, f, 0.5);
    p = fma(p, f, 1.0);
    p = fma(p, f, 1.0);
    const double b = s.table[j & 63];
    const double pow2 = __longlong_as_double(__double_as_longlong(b) + ((int64_t)(j >> 6) << 52));
    const double z = fma(p * unit, pow2, 4503599627370496.0);       // + 2^52: rounded to a whole number
    return (uint64_t)__double_as_longlong(z) & 0xFFFFFFFFFFFFFull;
  };
  auto valid = [&](float x) { return x >= mn; };

  // Tokens kept: key above s_key, or equal to it and index at most s_index.
  uint32_t cut_key = 0, cut_index = 0xFFFFFFFFu;
  const bool want_k = top_k > 0 && top_k < a.vocab, want_p = top_p < 1.f;
  if (want_k || want_p) {
    // Bins over the top of the range: past 32 T below the maximum a weight is under 2^-46.
    const float span = fminf(mx - mn, 32.f * temperature);
    const float per_bin = span > 0.f ? (float)(kSampleBins - 1) / span : 0.f;
    auto bin_of = [&](float x) -> int {
      return x == mx ? 0 : (int)fminf((mx - x) * per_bin, (float)(kSampleBins - 1));
    };
    s.weight[tid] = 0;
    s.count[tid] = 0;
    __syncthreads();
    for (int32_t i = v0 + lane; i < v1; i += kWave) {
      float x[EPV];
      row.widen(i, row.load(i), x);
#pragma unroll
      for (int e = 0; e < EPV; ++e)
        if (valid(x[e])) {
          const int b = bin_of(x[e]);
          atomicAdd(&s.count[b], 1u);
          if (want_p) atomicAdd(reinterpret_cast<unsigned long long*>(&s.weight[b]), (unsigned long long)weight_of(x[e]));
        }
    }
    __syncthreads();
    const uint64_t bin_count = s.count[tid], bin_weight = s.weight[tid];
    uint64_t all_count, all_weight;
    const uint64_t to_count = wg_scan(s, bin_count, all_count);
    const uint64_t to_weight = wg_scan(s, bin_weight, all_weight);

    // The place at which a prefix ends: the first token, in the order, at which the
    // running count (BY_WEIGHT: weight) reaches `need`, 1 <= need <= all of it.
    // Sets s.key and s.index to it and s.before to the weight up to it.
    auto select = [&](bool by_weight, uint64_t need) {
      const uint64_t mine = by_weight ? bin_weight : bin_count, upto = by_weight ? to_weight : to_count;
      __syncthreads();
      if (upto >= need && upto - mine < need) {    // one thread
        s.found = tid;
        s.before = upto - mine;
        s.part[0] = to_weight - bin_weight;
        s.kmin = 0xFFFFFFFFu;
        s.kmax = 0;
        s.n_list = 0;
      }
      __syncthreads();
      const int bin = s.found;
      uint64_t before = s.before, weight_before = s.part[0];
      // its tokens into the list, and the range of their keys
      uint32_t lo = 0xFFFFFFFFu, hi = 0;
      for (int32_t i = v0 + lane; i < v1; i += kWave) {
        float x[EPV];
        row.widen(i, row.load(i), x);
#pragma unroll
        for (int e = 0; e < EPV; ++e)
          if (valid(x[e]) && bin_of(x[e]) == bin) {
            const uint32_t k = float_key(x[e]);
            lo = min(lo, k);
            hi = max(hi, k);
            const uint32_t at = atomicAdd(&s.n_list, 1u);
            if (at < kSampleList) s.list[at] = (uint64_t)k << 32 | (uint32_t)~(i * EPV - row.off + e);
          }
      }
      if (lo <= hi) {
        atomicMin(&s.kmin, lo);
        atomicMax(&s.kmax, hi);
      }
      __syncthreads();
      lo = s.kmin;
      hi = s.kmax;
      uint32_t n = s.n_list;
      // Too many: bins over the keys of [lo, hi] until the list holds them or one key is left.
      while (n > kSampleList && lo < hi) {
        const int sh = max(0, 22 - __clz((int)(hi - lo)));     // (hi - lo) >> sh < 1024
        __syncthreads();
        s.weight[tid] = 0;
        s.count[tid] = 0;
        __syncthreads();
        for (int32_t i = v0 + lane; i < v1; i += kWave) {
          float x[EPV];
          row.widen(i, row.load(i), x);
#pragma unroll
          for (int e = 0; e < EPV; ++e)
            if (valid(x[e])) {
              const uint32_t k = float_key(x[e]);
              if (k >= lo && k <= hi) {
                atomicAdd(&s.count[(hi - k) >> sh], 1u);
                atomicAdd(reinterpret_cast<unsigned long long*>(&s.weight[(hi - k) >> sh]),
                          (unsigned long long)(want_p ? weight_of(x[e]) : 0));
              }
            }
        }
        __syncthreads();
        const uint64_t c = s.count[tid], g = s.weight[tid];
        uint64_t total;
        const uint64_t tc = wg_scan(s, c, total), tg = wg_scan(s, g, total);
        const uint64_t m = by_weight ? g : c, t = before + (by_weight ? tg : tc);
        __syncthreads();
        if (t >= need && t - m < need) {
          s.found = tid;
          s.before = t - m;
          s.part[0] = weight_before + tg - g;
          s.n_list = (uint32_t)c;
        }
        __syncthreads();
        before = s.before;
        weight_before = s.part[0];
        n = s.n_list;
        const uint32_t top_key = hi - ((uint32_t)s.found << sh);
        lo = max(lo, top_key - ((1u << sh) - 1));
        hi = top_key;
        __syncthreads();
        if (n <= kSampleList) {      // the list, now that they fit
          if (tid == 0) s.n_list = 0;
          __syncthreads();
          for (int32_t i = v0 + lane; i < v1; i += kWave) {
            float x[EPV];
            row.widen(i, row.load(i), x);
#pragma unroll
            for (int e = 0; e < EPV; ++e)
              if (valid(x[e])) {
                const uint32_t k = float_key(x[e]);
                if (k >= lo && k <= hi) {
                  const uint32_t at = atomicAdd(&s.n_list, 1u);
                  if (at < kSampleList) s.list[at] = (uint64_t)k << 32 | (uint32_t)~(i * EPV - row.off + e);
                }
              }
          }
          __syncthreads();
        }
      }
      if (n <= kSampleList) {
        // Sort the list, largest first (bitonic; filled up with zeros).
        uint32_t size = 2;
        while (size < n) size <<= 1;
        for (uint32_t i = tid; i < size; i += kSampleThreads)
          if (i >= n) s.list[i] = 0;
        __syncthreads();
        for (uint32_t k = 2; k <= size; k <<= 1)
          for (uint32_t j = k >> 1; j > 0; j >>= 1) {
            for (uint32_t i = tid; i < size / 2; i += kSampleThreads) {
              const uint32_t p = 2 * i - (i & (j - 1)), q = p + j;
              const uint64_t x = s.list[p], y = s.list[q];
              if ((x < y) == ((p & k) == 0)) {
                s.list[p] = y;
                s.list[q] = x;
              }
            }
            __syncthreads();
          }
        // Two neighbours per thread: the first at which the sum reaches `need`.
        const uint32_t i0 = 2 * tid;
        uint64_t g[2], m[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const bool in = i0 + e < n;
          g[e] = in && want_p ? weight_of(key_float((uint32_t)(s.list[i0 + e] >> 32))) : 0;
          m[e] = by_weight ? g[e] : in ? 1 : 0;
        }
        uint64_t total;
        const uint64_t tm = before + wg_scan(s, m[0] + m[1], total) - m[1] - m[0];
        const uint64_t tg = weight_before + wg_scan(s, g[0] + g[1], total) - g[1] - g[0];
        uint64_t m_at = tm, g_at = tg;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (m_at < need && m_at + m[e] >= need) {
            s.key = (uint32_t)(s.list[i0 + e] >> 32);
            s.index = ~(uint32_t)s.list[i0 + e];
            s.before = g_at + g[e];
          }
          m_at += m[e];
          g_at += g[e];
        }
        __syncthreads();
        return;
      }
      // One value alone: its tokens counted off in order of index.
      const uint64_t each = want_p ? weight_of(key_float(lo)) : 0;
      const uint64_t left = need - before;
      const uint64_t nth = by_weight ? (left + each - 1) / each : left;      // of them, from 1
      uint32_t mine_n = 0;
      for (int32_t i = v0 + lane; i < v1; i += kWave) {
        float x[EPV];
        row.widen(i, row.load(i), x);
#pragma unroll
        for (int e = 0; e < EPV; ++e) mine_n += valid(x[e]) && float_key(x[e]) == lo;
      }
      const uint64_t wave_n = wave_sum_u64(mine_n);
      __syncthreads();
      if (lane == 0) s.part[w] = wave_n;
      __syncthreads();
      uint64_t seen = 0;
      int part = 0;
      while (part < kSampleWaves - 1 && seen + s.part[part] < nth) seen += s.part[part++];
      const int32_t p1 = min((part + 1) * per, row.n_vec);
      for (int32_t base = part * per; base < p1; base += kSampleThreads) {
        const int32_t i = base + tid;
        float x[EPV];
        uint32_t c = 0;
        if (i < p1) {
          row.widen(i, row.load(i), x);
#pragma unroll
          for (int e = 0; e < EPV; ++e) c += valid(x[e]) && float_key(x[e]) == lo;
        }
        uint64_t total;
        const uint64_t upto = seen + wg_scan(s, c, total);
        if (upto >= nth && upto - c < nth) {
          uint64_t at = upto - c;
#pragma unroll
          for (int e = 0; e < EPV; ++e)
            if (valid(x[e]) && float_key(x[e]) == lo && ++at == nth) s.index = (uint32_t)(i * EPV - row.off + e);
        }
        seen += total;
      }
      if (tid == 0) {
        s.key = lo;
        s.before = weight_before + nth * each;
      }
      __syncthreads();
    };

    uint64_t kept = all_weight;
    if (want_k && (uint64_t)top_k < all_count) {
      select(false, (uint64_t)top_k);
      cut_key = s.key;
      cut_index = s.index;
      kept = s.before;
    }
    if (want_p) {
      const uint64_t need = top_p > 0.f ? times_fraction<true>(top_p, kept) : 1;
      select(true, need < 1 ? 1 : need);
      cut_key = s.key;
      cut_index = s.index;
    }
  }

  // Weight of a token if it is kept, else 0.
  const double floor_p = (double)min_p;
  auto kept_weight = [&](float x, int32_t at) -> uint64_t {
    if (!valid(x)) return 0;
    const uint32_t k = float_key(x);
    if (k < cut_key || (k == cut_key && (uint32_t)at > cut_index)) return 0;
    if (min_p > 0.f && x != mx && exp(((double)x - top) / (double)temperature) < floor_p) return 0;
    return weight_of(x);
  };
  uint64_t sum = 0;
  for (int32_t i = v0 + lane; i < v1; i += kWave) {
    float x[EPV];
    row.widen(i, row.load(i), x);
#pragma unroll
    for (int e = 0; e < EPV; ++e) sum += kept_weight(x[e], i * EPV - row.off + e);
  }
  sum = wave_sum_u64(sum);
  __syncthreads();
  if (lane == 0) s.part[w] = sum;
  if (tid == 0) s.found_at = -1;
  __syncthreads();
  uint64_t total = 0;
  for (int v = 0; v < kSampleWaves; ++v) total += s.part[v];
  // the first token at which the running weight exceeds u * total
  const float uc = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;       // a NaN is 0
  const uint64_t target = times_fraction<false>(uc, total);
  uint64_t seen = 0;
  int part = 0;
  while (part < kSampleWaves - 1 && seen + s.part[part] <= target) seen += s.part[part++];
  const int32_t p1 = min((part + 1) * per, row.n_vec);
  for (int32_t base = part * per; base < p1; base += kSampleThreads) {
    const int32_t i = base + tid;
    float x[EPV];
    uint64_t g[EPV], mine = 0;
#pragma unroll
    for (int e = 0; e < EPV; ++e) g[e] = 0;
    if (i < p1) {
      row.widen(i, row.load(i), x);
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        g[e] = kept_weight(x[e], i * EPV - row.off + e);
        mine += g[e];
      }
    }
    uint64_t all;
    const uint64_t upto = seen + wg_scan(s, mine, all);
    if (upto > target && upto - mine <= target) {
      uint64_t at = upto - mine;
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        if (at <= target && at + g[e] > target) a.tokens[r] = i * EPV - row.off + e;
        at += g[e];
      }
    }
    seen += all;
  }
}

}  // namespace
}  // namespace baton
