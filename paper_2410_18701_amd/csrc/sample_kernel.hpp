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
// computed in double precision (relative error below 2^-49) and rounded to a whole
// number of 2^-shift, shift = 62 - ceil(log2 V) at most 51.  Sums of whole numbers are
// exact, so atomics in any order give the same sums, and the boundary between two
// tokens is off by about sqrt(V) 2^-(shift + 1) at most.
//
// One workgroup of 16 waves per row.  The row is read once from memory into LDS (what
// does not fit is read again); wave w owns the w-th of 16 contiguous parts of
// it, 16 bytes per lane and step.  What bounds it is the vector ALUs of one compute
// unit -- a weight takes about 25 instructions, a row of 32,000 all weighed 5 us; they
// are active 64 to 69% of the time that a row takes -- and the latency of its dependent
// steps, so whole passes over the row are kept few and a list of tokens in LDS takes
// their place as soon as one can.  With a row per compute unit the launch then waits for
// the slowest one (256 rows of 128,000 that differ: a unit is busy 31 of 79 us):
//  * top_k up to 512: the k-th largest of the threads' own largest values bounds
//    the k-th largest from below (up to 1024, counts in bins of the values do); the
//    tokens from there on, a few more than k, are the list.
//  * else 1024 bins of equal width over the top of the values' range hold counts
//    or weights (floats' own bits would put most tokens into a few bins, whose atomics
//    then queue); a scan finds the bin in which a prefix ends, and that bin's
//    tokens, a few dozen, are the list that gives the place exactly.  More than fit
//    (equal logits, mostly) are first narrowed by bins over the bits of their floats,
//    and if one value alone has too many, its tokens are counted off in order of index.
//  * the draw: from a list of the kept tokens where they fit one, else kept
//    weights per wave, then the tokens of the wave's part in which the target lies.
// exp: 2^(j / 128) from a table, times a polynomial of degree 4 on half a step:
// relative error below 2^-49.
// us, bf16: one row of 32,000 8 (greedy), 12 (top_k 50), 15 (temperature alone), 23 to
// 26 (top_p); 256 rows of 128,000, which LDS holds a third of, 15, 21, 46 and 72 to 85,
// of which 13.5 is the first read and 33 the bins' weights.
#pragma once

#include "common.hpp"

namespace baton {
namespace {

constexpr int kSampleThreads = 1024, kSampleWaves = kSampleThreads / kWave;
constexpr int kSampleBins = 1024;        // == kSampleThreads: a bin per thread
constexpr int kSampleList = 2048;        // tokens in a list at most, two per thread
constexpr int kSampleRank = 256;         // up to here a list is ordered by counting, not sorted
constexpr int kSampleTopK = 512;         // the largest top_k for which threads' largest values bound it
constexpr int kSampleTopKList = kSampleThreads;   // and the largest whose tokens are gathered as a list
constexpr int kSampleQuarters = 4;       // of the row, with bins of their own
constexpr int kSampleRowBytes = 80 << 10;    // of a row kept in LDS

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

// Floats (no NaN) as unsigned numbers of the same order, -0 as 0.
__device__ __forceinline__ uint32_t float_key(float f) {
  const uint32_t b = __float_as_uint(f + 0.f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_float(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

// One step of a wave's prefix sum: x plus the value DPP moves here (0 from outside).
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t dpp_add(uint64_t x) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, ROWS, 0xF, false);
  return x + ((uint64_t)hi << 32 | lo);
}
// Inclusive prefix sum over the wave: within rows of 16 lanes, then across them.
__device__ __forceinline__ uint64_t wave_scan(uint64_t x) {
  x = dpp_add<0x111, 0xF>(x);   // row_shr 1, 2, 4, 8
  x = dpp_add<0x112, 0xF>(x);
  x = dpp_add<0x114, 0xF>(x);
  x = dpp_add<0x118, 0xF>(x);
  x = dpp_add<0x142, 0xA>(x);   // lane 15 of each row into the next (rows 1 and 3)
  x = dpp_add<0x143, 0xC>(x);   // lane 31 into the upper half
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
  // Whether the 64 vectors from i0 on hold elements of the row only.
  __device__ __forceinline__ bool inside(int32_t i0) const { return i0 > 0 && (i0 + kWave) * EPV - off <= vocab; }
  // The elements of vector i; outside the row NaN, which every comparison leaves out.
  __device__ __forceinline__ void widen(int32_t i, const u32x4& w, bool all, float (&x)[EPV]) const {
    Lane16<T>::widen(w, x);
    if (all) return;
#pragma unroll
    for (int e = 0; e < EPV; ++e) {
      const int32_t at = i * EPV - off + e;
      if (at < 0 || at >= vocab) x[e] = __uint_as_float(0x7FC00000u);
    }
  }
  __device__ __forceinline__ uint32_t index(int32_t i, int e) const { return (uint32_t)(i * EPV - off + e); }
};

struct SampleShared {
  double table[128];             // 2^(i / 128 + shift)
  uint64_t weight[kSampleQuarters][kSampleBins];
  uint32_t count[kSampleBins];
  uint64_t list[kSampleList];    // tokens: (float_key, ~index), so that larger is earlier
  uint64_t lw[kSampleList];      // their weights; before they are known, scratch
  uint64_t ahead_w[kSampleRank];
  uint32_t ahead[kSampleRank];
  uint64_t scan[2][kSampleWaves];
  uint64_t part[kSampleWaves], quarter[kSampleQuarters];
  float fmax[kSampleWaves], fmin[kSampleWaves];
  uint32_t kmin, kmax, n_list, n_own;
  int32_t found, bin_whole;   // bin_whole: the cut's bin, if its tokens were one list; else -1
  uint64_t before, weight_before;
  uint64_t cut;                  // the last kept token
  uint32_t index;
};

template <typename T>
struct Sampler {
  static constexpr int EPV = Lane16<T>::kElems;
  SampleShared& s;
  SampleRow<T> row;
  int32_t per, v0, v1;        // vectors of a wave's part; this wave's
  float mx, mn;               // the largest value and the smallest that is finite
  float own;                  // the largest that this thread has read
  bool infinite;              // the largest was infinite: see get
  float per_bin;
  double scale, top, least, floor_w;   // floor_w: min_p as a weight
  int tid, lane, w, turn = 0;

  // Inclusive prefix sum over the workgroup; `total` gets the whole.
  __device__ __forceinline__ uint64_t wg_scan(uint64_t x, uint64_t& total) {
    x = wave_scan(x);
    turn ^= 1;                           // alternating, so that one barrier will do
    if (lane == kWave - 1) s.scan[turn][w] = x;
    __syncthreads();
    uint64_t t = lane < kSampleWaves ? s.scan[turn][lane] : 0;
    t = dpp_add<0x111, 0xF>(t);
    t = dpp_add<0x112, 0xF>(t);
    t = dpp_add<0x114, 0xF>(t);
    t = dpp_add<0x118, 0xF>(t);          // lanes 0 .. 15: sums up to wave `lane`
    auto from = [&](int l) {
      return (uint64_t)__builtin_amdgcn_readlane((int)(t >> 32), l) << 32 |
             (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)t, l);
    };
    total = from(kSampleWaves - 1);
    return x + (w > 0 ? from(w - 1) : 0);
  }

  // The weight of a value, before it is rounded to a whole number (0, of a NaN or -inf).
  __device__ __forceinline__ double weight(float x) const {
    const double y = fmax(((double)x - top) * scale, least);        // 128 log2 w; a NaN is least
    constexpr double kMagic = 6755399441055744.0;                   // 1.5 * 2^52: rounds to a whole number
    const double t = y + kMagic;
    const uint32_t j = (uint32_t)__double_as_longlong(t);
    const double f = y - (t - kMagic);
    constexpr double c = 0.0054152123481245727;                     // ln 2 / 128
    double p = fma(f, c * c * c * c / 24.0, c * c * c / 6.0);
    p = fma(p, f, c * c / 2.0);
    p = fma(p, f, c);
    p = fma(p, f, 1.0);
    // 2^(j / 128 + shift): the table's entry with j / 128 added to its exponent
    const double b = __longlong_as_double(__double_as_longlong(s.table[j & 127]) +
                                          ((uint64_t)((j & ~127u) << 13) << 32));
    return p * b;
  }
  __device__ __forceinline__ uint64_t whole(double wd) const {
    return (uint64_t)__double_as_longlong(wd + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;   // + 2^52
  }
  __device__ __forceinline__ uint32_t valid(float x) const { return x >= mn; }
  __device__ __forceinline__ uint64_t weight_of(float x) const { return whole(weight(x)); }
  // 0 also below min_p (the largest value never is)
  __device__ __forceinline__ uint64_t weight_if(float x, uint32_t keep) const {
    const double d = weight(x);
    const uint64_t g = whole(d);
    return keep & ((uint32_t)(d >= floor_w) | (uint32_t)(x == mx)) ? g : 0;
  }
  __device__ __forceinline__ int bin_of(float x) const {
    return (int)fminf((mx - x) * per_bin, (float)(kSampleBins - 1));
  }

  // Counts the token in its bin; those of the last one, which may be most of the row, in `deep`.
  __device__ __forceinline__ void count(float x, uint32_t& deep) {
    if (!valid(x)) return;
    const int b = bin_of(x);
    if (b == kSampleBins - 1) ++deep;
    else atomicAdd(&s.count[b], 1u);
  }

  // The elements of vector i0 + lane (i0 the same in the wave), NaN outside the row
  // and from vector `end` on.  Beside an infinity, 1 for one and NaN for all else.
  __device__ __forceinline__ void get(int32_t i0, int32_t end, float (&x)[EPV]) const {
    const int32_t i = i0 + lane;
    const bool all = row.inside(i0) && i0 + kWave <= end;
    u32x4 v = {0, 0, 0, 0};
    if (all) v = i0 + kWave <= row.n_lds ? row.lds[i] : i0 < row.n_lds && i < row.n_lds ? row.lds[i] : row.fetch(i);
    else if (i < end) v = i < row.n_lds ? row.lds[i] : row.fetch(i);
    row.widen(i, v, all, x);
    if (!all && i >= end) {
#pragma unroll
      for (int e = 0; e < EPV; ++e) x[e] = __uint_as_float(0x7FC00000u);
    }
    if (infinite) {
#pragma unroll
      for (int e = 0; e < EPV; ++e) x[e] = x[e] == INFINITY ? 1.f : __uint_as_float(0x7FC00000u);
    }
  }
  // f(i, x) for every vector of the row, each wave its part.
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
    for (int32_t i0 = v0; i0 < v1; i0 += kWave) {
      float x[EPV];
      get(i0, v1, x);
      f(i0 + lane, x);
    }
  }
  // The same for vector i, by itself.
  __device__ __forceinline__ void get_one(int32_t i, float (&x)[EPV]) const {
    row.widen(i, i < row.n_lds ? row.lds[i] : row.fetch(i), false, x);
    if (infinite) {
#pragma unroll
      for (int e = 0; e < EPV; ++e) x[e] = x[e] == INFINITY ? 1.f : __uint_as_float(0x7FC00000u);
    }
  }
  // Tokens of lo <= x <= hi for which pick(i, e, x) into the list; n_list is more than it
  // holds if they are, which ends the search.  Where only `few` threads may have seen such a value, the
  // vectors of those that have are dealt to all (with more than 3/4 of them the row is
  // passed over as it lies; a limit of 1/2 took 44 us instead of 40 at top_k 500 of 256
  // rows of 128,000, 32 instead of 28.5 at min_p 0.05).
  template <typename F>
  __device__ __forceinline__ void collect(float lo, float hi, bool few, F&& pick) {
    if (tid == 0) s.n_list = s.n_own = 0;
    __syncthreads();
    uint32_t last = 0;     // this thread's latest place
    auto take = [&](int32_t i, const float (&x)[EPV]) {
      uint32_t some = 0;
#pragma unroll
      for (int e = 0; e < EPV; ++e) some |= x[e] >= lo && x[e] <= hi ? 1u << e : 0u;
      if (last >= kSampleList) some = 0;
      while (some) {
        const int e = __builtin_ctz(some);
        some &= some - 1;
        float f = x[0];
#pragma unroll
        for (int q = 1; q < EPV; ++q) f = e == q ? x[q] : f;
        if (!pick(i, e, f)) continue;
        const uint32_t at = atomicAdd(&s.n_list, 1u);
        if (at < kSampleList) s.list[at] = (uint64_t)float_key(f) << 32 | (uint32_t)~row.index(i, e);
        last = at;
      }
    };
    uint32_t n = kSampleThreads;
    if (few) {
      if (own >= lo) s.lw[atomicAdd(&s.n_own, 1u)] = (uint64_t)tid;
      __syncthreads();
      n = s.n_own;
    }
    if (n <= kSampleThreads * 3 / 4) {
      const uint32_t steps = (uint32_t)(per + kWave - 1) / kWave;
      for (uint32_t j = tid; j < n * steps; j += kSampleThreads) {
        const int32_t step = (int32_t)(j / n), t = (int32_t)s.lw[j - (uint32_t)step * n];
        const int32_t part = t / kWave * per, i = part + step * kWave + t % kWave;
        if (i >= min(part + per, row.n_vec)) continue;
        float x[EPV];
        get_one(i, x);
        take(i, x);
      }
    } else {
      each(take);
    }
    __syncthreads();
  }
  // Values beside which no token of bins b0 .. b1 lies: bin_of's roundings are off by
  // 2^-13 of a bin, a float's by 2^-24 of it.
  __device__ __forceinline__ float bin_low(int b1) const {
    if (b1 >= kSampleBins - 1) return -INFINITY;
    const double v = top - (b1 + 1.01) / (double)per_bin;
    return (float)(v - fabs(v) * 0x1p-22);
  }
  __device__ __forceinline__ float bin_high(int b0) const {
    const double v = top - (b0 - 0.01) / (double)per_bin;
    return (float)(v + fabs(v) * 0x1p-22);
  }

  // A thread's tokens of the list with what comes before each in its order.
  struct Place {
    uint64_t id, w, before_w;
    uint32_t before;
    bool in;
  };
  // Weights of the n <= kSampleList tokens of the list, and their places.  A short
  // list is compared with itself, a longer one sorted (bitonic, largest first).
  __device__ __forceinline__ void order(uint32_t n, Place (&p)[2]) {
    if (n > kSampleRank) {
      uint32_t size = 512;
      while (size < n) size <<= 1;
      for (uint32_t i = n + tid; i < size; i += kSampleThreads) s.list[i] = 0;
      __syncthreads();
      for (uint32_t k = 2; k <= size; k <<= 1)
        for (uint32_t j = k >> 1; j > 0; j >>= 1) {
          const uint32_t i = tid;
          if (i < size / 2) {
            const uint32_t l = 2 * i - (i & (j - 1)), h = l + j;
            const uint64_t x = s.list[l], y = s.list[h];
            if ((x < y) == ((l & k) == 0)) {
              s.list[l] = y;
              s.list[h] = x;
            }
          }
          // A wave's 64 pairs at distances up to 64 are 128 elements of its own, which its
          // own operations on LDS, done in order, pass on; only others are waited for.
          if (j > kWave || (j == 1 && k > kWave)) {
            __syncthreads();
          } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
          }
        }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t i = 2 * tid + e;
        p[e].in = i < n;
        p[e].id = p[e].in ? s.list[i] : 0;
        p[e].before = i;
        const uint64_t g = weight_of(key_float((uint32_t)(p[e].id >> 32)));
        p[e].w = p[e].in ? g : 0;
        if (p[e].in) s.lw[i] = g;
      }
      uint64_t total;
      const uint64_t upto = wg_scan(p[0].w + p[1].w, total);
      p[1].before_w = upto - p[1].w;
      p[0].before_w = p[1].before_w - p[0].w;
      return;
    }
    // Token e against a quarter of the list in each of four threads.
    const uint32_t e = tid % kSampleRank, q = tid / kSampleRank;
    static_assert(kSampleThreads == 4 * kSampleRank, "four threads per token");
    const bool in = e < n;
    const uint64_t id = in ? s.list[e] : 0;
    uint64_t g = 0;
    if (q == 0) {
      g = weight_of(key_float((uint32_t)(id >> 32)));
      g = in ? g : 0;
      s.lw[e] = g;
      s.ahead[e] = 0;
      s.ahead_w[e] = 0;
    }
    __syncthreads();
    const uint32_t j0 = q * n / 4, j1 = (q + 1) * n / 4;
    uint64_t bw = 0;
    uint32_t b = 0;
    if (w % 4 * kWave < n) {
#pragma unroll 4
      for (uint32_t j = j0; j < j1; ++j) {
        const uint64_t other = s.list[j], ow = s.lw[j];
        const bool first = other > id;
        b += first;
        bw += first ? ow : 0;
      }
      atomicAdd(&s.ahead[e], b);
      atomicAdd(reinterpret_cast<unsigned long long*>(&s.ahead_w[e]), (unsigned long long)bw);
    }
    __syncthreads();
    p[0].in = q == 0 && in;
    p[0].id = q == 0 ? id : 0;
    p[0].w = g;
    p[0].before = s.ahead[e];
    p[0].before_w = s.ahead_w[e];
    p[1].in = false;
    p[1].w = p[1].before_w = p[1].id = 0;
    p[1].before = 0;
  }

  __device__ __forceinline__ int quarter_of(uint32_t index) const {
    return (int)(((int32_t)index + row.off) / EPV / (kSampleWaves / kSampleQuarters * per));
  }

  // The place at which a prefix ends: the first token, in the order, at which the
  // running count (BY_WEIGHT: weight) reaches `need`, 1 <= need <= all of it, from the
  // bins' own values and their running sums.  Sets s.cut to it and s.before to the
  // weight up to it.
  __device__ __forceinline__ void select(bool by_weight, uint64_t need, uint64_t mine, uint64_t upto,
                                         uint64_t weight_upto) {
    __syncthreads();
    if (upto >= need && upto - mine < need) {    // one thread
      s.found = tid;
      s.before = upto - mine;
      s.weight_before = weight_upto;
    }
    if (tid < kSampleQuarters) s.quarter[tid] = 0;
    __syncthreads();
    const int bin = s.found;
    uint64_t before = s.before, weight_before = s.weight_before;
    collect(bin_low(bin), bin_high(bin), false, [&](int32_t, int, float x) { return x >= mn && bin_of(x) == bin; });
    uint32_t n = s.n_list, lo = 0, hi = 0;
    if (tid == 0) s.bin_whole = n <= kSampleList ? bin : -1;
    if (n > kSampleList) {
      // Too many: bins over the keys of [lo, hi] until the list holds them or one key is left.
      // Their weights lie in lw, free until the list is ordered: s.weight keeps the bins of
      // the whole row, which the draw reads once the other prefix has ended.
      static_assert(kSampleBins <= kSampleList, "weights of the narrower bins");
      if (tid == 0) {
        s.kmin = 0xFFFFFFFFu;
        s.kmax = 0;
      }
      __syncthreads();
      lo = 0xFFFFFFFFu;
      each([&](int32_t, const float (&x)[EPV]) {
#pragma unroll
        for (int e = 0; e < EPV; ++e)
          if (valid(x[e]) && bin_of(x[e]) == bin) {
            lo = min(lo, float_key(x[e]));
            hi = max(hi, float_key(x[e]));
          }
      });
      if (lo <= hi) {
        atomicMin(&s.kmin, lo);
        atomicMax(&s.kmax, hi);
      }
      __syncthreads();
      lo = s.kmin;
      hi = s.kmax;
      while (n > kSampleList && lo < hi) {
        const int sh = max(0, 22 - __clz((int)(hi - lo)));     // (hi - lo) >> sh < 1024
        s.lw[tid] = 0;
        s.count[tid] = 0;
        __syncthreads();
        each([&](int32_t, const float (&x)[EPV]) {
#pragma unroll
          for (int e = 0; e < EPV; ++e) {
            const uint32_t k = float_key(x[e]);
            if (valid(x[e]) && k >= lo && k <= hi) {
              atomicAdd(&s.count[(hi - k) >> sh], 1u);
              atomicAdd(reinterpret_cast<unsigned long long*>(&s.lw[(hi - k) >> sh]),
                        (unsigned long long)weight_of(x[e]));
            }
          }
        });
        __syncthreads();
        const uint64_t c = s.count[tid], g = s.lw[tid];
        uint64_t total;
        const uint64_t tc = wg_scan(c, total), tg = wg_scan(g, total);
        const uint64_t m = by_weight ? g : c, t = before + (by_weight ? tg : tc);
        if (t >= need && t - m < need) {
          s.found = tid;
          s.before = t - m;
          s.weight_before = weight_before + tg - g;
          s.n_list = (uint32_t)c;
        }
        __syncthreads();
        before = s.before;
        weight_before = s.weight_before;
        n = s.n_list;
        const uint32_t top_key = hi - ((uint32_t)s.found << sh);
        lo = max(lo, top_key - ((1u << sh) - 1));
        hi = top_key;
        __syncthreads();
      }
      if (n <= kSampleList)
        collect(key_float(lo), key_float(hi), false, [&](int32_t, int, float) { return true; });
    }
    if (n <= kSampleList) {
      Place p[2];
      order(n, p);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint64_t m0 = before + (by_weight ? p[e].before_w : p[e].before), m = by_weight ? p[e].w : 1;
        if (p[e].in && m0 < need && m0 + m >= need) {
          s.cut = p[e].id;
          s.before = weight_before + p[e].before_w + p[e].w;
        }
        // this bin's share of what each quarter keeps
        if (p[e].w && m0 < need && s.bin_whole >= 0)
          atomicAdd(reinterpret_cast<unsigned long long*>(&s.quarter[quarter_of(~(uint32_t)p[e].id)]), (unsigned long long)p[e].w);
      }
      __syncthreads();
      return;
    }
    // One value alone: its tokens counted off in order of index.
    const uint64_t value = weight_of(key_float(lo));
    const uint64_t left = need - before;
    const uint64_t nth = by_weight ? (left + value - 1) / value : left;      // of them, from 1
    uint64_t wave_n = 0, total;
    each([&](int32_t, const float (&x)[EPV]) {
#pragma unroll
      for (int e = 0; e < EPV; ++e) wave_n += valid(x[e]) && float_key(x[e]) == lo;
    });
    wave_n = wave_scan(wave_n);
    if (lane == kWave - 1) s.part[w] = wave_n;
    __syncthreads();
    uint64_t seen = 0;
    int part = 0;
    while (part < kSampleWaves - 1 && seen + s.part[part] < nth) seen += s.part[part++];
    const int32_t p1 = min((part + 1) * per, row.n_vec);
    for (int32_t base = part * per; base < p1; base += kSampleThreads) {
      const int32_t i0 = base + w * kWave, i = i0 + lane;
      float x[EPV];
      uint64_t c = 0;
      get(i0, p1, x);
#pragma unroll
      for (int e = 0; e < EPV; ++e) c += valid(x[e]) && float_key(x[e]) == lo;
      const uint64_t to = seen + wg_scan(c, total);
      if (to >= nth && to - c < nth) {
        uint64_t at = to - c;
#pragma unroll
        for (int e = 0; e < EPV; ++e)
          if (valid(x[e]) && float_key(x[e]) == lo && ++at == nth)
            s.cut = (uint64_t)lo << 32 | (uint32_t)~row.index(i, e);
      }
      seen += total;
    }
    if (tid == 0) s.before = weight_before + nth * value;
    __syncthreads();
  }

  // The draw from the tokens of the list with weight g[e] (0: not kept) in the places i[e].
  __device__ __forceinline__ void draw_list(uint32_t n, float u, const uint64_t (&id)[2], const uint64_t (&g)[2],
                                            const uint32_t (&at)[2], int32_t* token) {
    // 1024 ranges of the index; then the tokens of the range in which the target lies
    s.weight[0][tid] = 0;
    __syncthreads();     // and n_list has been read
    if (tid == 0) s.n_list = 0;
    const uint32_t per_range = ((uint32_t)row.vocab + kSampleBins - 1) / kSampleBins;
    uint32_t range[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      range[e] = ~(uint32_t)id[e] / per_range;
      if (g[e]) atomicAdd(reinterpret_cast<unsigned long long*>(&s.weight[0][range[e]]), (unsigned long long)g[e]);
      if (at[e] < n) s.lw[at[e]] = g[e];
    }
    __syncthreads();
    const uint64_t mine = s.weight[0][tid];
    uint64_t total;
    const uint64_t upto = wg_scan(mine, total);
    const uint64_t target = times_fraction<false>(u, total);
    if (upto > target && upto - mine <= target) {
      s.found = tid;
      s.before = upto - mine;
    }
    __syncthreads();
    // those of them that lie in the range, gathered (unless they are more than fit)
    const uint32_t r = (uint32_t)s.found, first = r * per_range;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (g[e] && range[e] == r) {
        const uint32_t k = atomicAdd(&s.n_list, 1u);
        if (k < kSampleBins) s.count[k] = at[e];
      }
    __syncthreads();
    const uint32_t m = s.n_list, few = m <= kSampleBins ? m : n;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (g[e] && range[e] == r) {
        const uint32_t own = ~(uint32_t)id[e];
        uint64_t before = s.before;
        for (uint32_t j = 0; j < few; ++j) {
          const uint32_t l = m <= kSampleBins ? s.count[j] : j, o = ~(uint32_t)s.list[l];
          before += o >= first && o < own ? s.lw[l] : 0;
        }
        if (before <= target && before + g[e] > target) *token = (int32_t)own;
      }
  }
};

template <typename T>
__global__ void __launch_bounds__(kSampleThreads) sample_kernel(const SampleArgs a) {
  constexpr int EPV = Lane16<T>::kElems;
  extern __shared__ __attribute__((aligned(16))) u32x4 row_lds[];
  __shared__ SampleShared s;
  const int64_t r = blockIdx.x;
  SampleRow<T> row;
  row.row = a.logits + r * a.ld * T::kBytes;
  row.off = (int32_t)((reinterpret_cast<uintptr_t>(row.row) & 15u) / T::kBytes);
  row.vocab = a.vocab;
  row.n_vec = (row.off + a.vocab + EPV - 1) / EPV;
  row.n_lds = min(row.n_vec, kSampleRowBytes / 16);
  row.lds = row_lds;
  Sampler<T> p{s, row};
  const int tid = p.tid = threadIdx.x, lane = p.lane = tid % kWave;
  const int w = p.w = __builtin_amdgcn_readfirstlane(tid / kWave);
  p.per = (row.n_vec + kSampleWaves - 1) / kSampleWaves;
  p.v0 = w * p.per;
  p.v1 = min(p.v0 + p.per, row.n_vec);

  const float temperature = a.temperature ? a.temperature[r] : 1.f;
  const int32_t top_k = a.top_k ? a.top_k[r] : 0;
  const float top_p = a.top_p ? a.top_p[r] : 1.f;
  const float min_p = a.min_p ? a.min_p[r] : 0.f;
  const float u_in = a.u[r];
  const float u = u_in > 0.f ? fminf(u_in, 0x1.fffffep-1f) : 0.f;       // a NaN is 0

  // The row into LDS; its largest value and the smallest that is finite.
  float mx = -INFINITY, mn = INFINITY;
  int32_t own_i = 0;          // the first vector in which this thread saw its largest
  auto take = [&](int32_t i, const u32x4& v, bool all) {
    if (i < row.n_lds) row.lds[i] = v;
    float x[EPV];
    row.widen(i, v, all, x);
    const float before = mx;
#pragma unroll
    for (int e = 0; e < EPV; ++e) {
      mx = fmaxf(mx, x[e]);
      mn = x[e] > -INFINITY ? fminf(mn, x[e]) : mn;
    }
    own_i = mx > before ? i : own_i;
  };
  constexpr int U = 4;        // vectors in flight at once
  for (int32_t i0 = p.v0; i0 < p.v1;) {
    const int32_t i = i0 + lane;
    if (row.inside(i0) && row.inside(i0 + (U - 1) * kWave) && i0 + U * kWave <= p.v1) {
      const u32x4* src = reinterpret_cast<const u32x4*>(row.row + (int64_t)(i * EPV - row.off) * T::kBytes);
      u32x4 v[U];
#pragma unroll
      for (int q = 0; q < U; ++q) v[q] = src[q * kWave];
#pragma unroll
      for (int q = 0; q < U; ++q) take(i + q * kWave, v[q], true);
      i0 += U * kWave;
    } else {
      if (i < p.v1) take(i, row.fetch(i), row.inside(i0));
      i0 += kWave;
    }
  }
  p.own = mx;
  if (tid < 128) s.table[tid] = ldexp(exp2((double)tid / 128.0), a.shift);
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
#pragma unroll
  for (int q = 0; q < kSampleQuarters; ++q) s.weight[q][tid] = 0;
  s.count[tid] = 0;
  __syncthreads();
#pragma unroll
  for (int v = 0; v < kSampleWaves; ++v) {
    mx = fmaxf(mx, s.fmax[v]);
    mn = fminf(mn, s.fmin[v]);
  }
  // the same in every lane, which the compiler cannot see
  mx = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(mx)));
  mn = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(mn)));
  if (mx == -INFINITY) {      // no token can be drawn
    if (tid == 0) a.tokens[r] = -1;
    return;
  }
  p.infinite = mx == INFINITY;             // beside an infinity nothing finite has weight
  if (p.infinite) mx = mn = 1.f;
  if (!(temperature > 0.f) || top_k == 1 || min_p > 1.f) {     // the first of the largest
    if (p.own == (p.infinite ? INFINITY : mx)) {
      float x[EPV];
      row.widen(own_i, own_i < row.n_lds ? row.lds[own_i] : row.fetch(own_i), false, x);
      uint32_t first = 0;
#pragma unroll
      for (int e = EPV - 1; e >= 0; --e) first = x[e] == p.own ? row.index(own_i, e) : first;
      atomicMin(&s.index, first);
    }
    __syncthreads();
    if (tid == 0) a.tokens[r] = (int32_t)s.index;
    return;
  }
  if (p.infinite) p.own = p.own == INFINITY ? 1.f : -INFINITY;
  p.mx = mx;
  p.mn = mn;
  p.top = (double)mx;
  p.scale = 128.0 * 1.4426950408889634074 / (double)temperature;
  p.least = -128.0 * (a.shift + 2);        // a weight that rounds to 0
  const bool want_m = min_p > 0.f;
  p.floor_w = want_m ? ldexp((double)min_p, a.shift) : -1.0;
  // Bins over the top of the range: past 32 T below the maximum a weight is under 2^-46.
  const float span = fminf(mx - p.mn, 32.f * temperature);
  p.per_bin = span > 0.f ? fminf((float)(kSampleBins - 1) / span, 3.4e38f) : 0.f;

  const bool want_k = top_k > 0 && top_k < a.vocab;
  const bool want_p = top_p < 1.f;
  uint64_t cut = 0;       // tokens kept: list ids from here on
  uint64_t total;
  if (want_k && top_k <= kSampleTopKList) {
    // A bin up to which at least top_k tokens lie: that of the k-th largest of the
    // threads' own largest values, or, for a larger k, of the k-th largest of all.
    // The bins span the threads' largest values, whatever the temperature.
    float low = p.own > -INFINITY ? p.own : mx;
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) low = fminf(low, __shfl_xor(low, m, kWave));
    if (lane == 0) s.part[w] = __float_as_uint(low);
    __syncthreads();
#pragma unroll
    for (int v = 0; v < kSampleWaves; ++v) low = fminf(low, __uint_as_float((uint32_t)s.part[v]));
    const float weight_bins = p.per_bin;
    if (mx > low) p.per_bin = fminf((float)(kSampleBins - 2) / (mx - low), 3.4e38f);
    if (top_k <= kSampleTopK) {
      if (p.valid(p.own)) atomicAdd(&s.count[p.bin_of(p.own)], 1u);
    } else {
      p.each([&](int32_t, const float (&x)[EPV]) {
#pragma unroll
        for (int e = 0; e < EPV; ++e)
          if (x[e] >= low) atomicAdd(&s.count[p.bin_of(x[e])], 1u);
      });
    }
    __syncthreads();
    const uint64_t c = s.count[tid], to = p.wg_scan(c, total);
    if (tid == 0) s.found = kSampleBins;
    __syncthreads();
    if (to >= (uint64_t)top_k && to - c < (uint64_t)top_k) s.found = tid;
    __syncthreads();
    const int bin = s.found;       // (fewer than k counted: every bin)
    s.count[tid] = 0;
    p.collect(fmaxf(p.bin_low(bin), mn), mx, top_k <= kSampleTopK, [&](int32_t, int, float x) { return p.bin_of(x) <= bin; });
    const uint32_t n = s.n_list;
    if (n <= kSampleList) {
      typename Sampler<T>::Place q[2];
      p.order(n, q);
      uint64_t g[2], id[2];
      uint32_t at[2];
      uint64_t sum = 0;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        id[e] = q[e].id;
        at[e] = n > kSampleRank ? 2 * tid + e : e == 0 ? tid : kSampleList;
        g[e] = q[e].in && q[e].before < (uint32_t)top_k ? q[e].w : 0;
        sum += g[e];
      }
      p.wg_scan(sum, total);
      const uint64_t need = !want_p ? ~0ull : top_p > 0.f ? times_fraction<true>(top_p, total) : 1;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (q[e].before_w >= max(need, (uint64_t)1)) g[e] = 0;
        if (want_m && g[e] && !p.weight_if(key_float((uint32_t)(id[e] >> 32)), true)) g[e] = 0;
      }
      p.draw_list(n, u, id, g, at, a.tokens + r);
      return;
    }
    p.per_bin = weight_bins;
  }
  if (want_k || want_p) {
    uint64_t* const weights = s.weight[w / (kSampleWaves / kSampleQuarters)];
    uint32_t deep = 0;
    p.each([&](int32_t, const float (&x)[EPV]) {
#pragma unroll
      for (int h = 0; h < EPV; h += 4) {
        if (want_p) {
          uint64_t g[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) g[e] = p.weight_of(x[h + e]);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (g[e])
              atomicAdd(reinterpret_cast<unsigned long long*>(&weights[p.bin_of(x[h + e])]), (unsigned long long)g[e]);
        }
        if (want_k) {
#pragma unroll
          for (int e = 0; e < 4; ++e) p.count(x[h + e], deep);
        }
      }
    });
    if (deep) atomicAdd(&s.count[kSampleBins - 1], deep);
    __syncthreads();
    const uint64_t bin_count = s.count[tid];
    uint64_t bin_weight = 0;
#pragma unroll
    for (int q = 0; q < kSampleQuarters; ++q) bin_weight += s.weight[q][tid];
    uint64_t all_count, kept;
    const uint64_t to_weight = p.wg_scan(bin_weight, kept);
    const uint64_t to_count = p.wg_scan(bin_count, all_count);
    // the prefix by count, then the one by weight of what that keeps
#pragma unroll 1
    for (int by_weight = 0; by_weight < 2; ++by_weight) {
      uint64_t need = (uint64_t)top_k;
      if (by_weight) {
        if (!want_p) break;
        need = top_p > 0.f ? max(times_fraction<true>(top_p, kept), (uint64_t)1) : 1;
      } else if (!want_k || need >= all_count) {
        continue;
      }
      p.select(by_weight != 0, need, by_weight ? bin_weight : bin_count, by_weight ? to_weight : to_count,
               to_weight - bin_weight);
      cut = s.cut;
      kept = s.before;
    }
  }

  const uint32_t cut_key = (uint32_t)(cut >> 32), cut_index = ~(uint32_t)cut;
  const float cut_x = cut ? key_float(cut_key) : mn;
  auto kept = [&](int32_t i, int e, float x) {
    return (uint32_t)(x > cut_x) | ((uint32_t)(x == cut_x) & (uint32_t)(row.index(i, e) <= cut_index));
  };
  // Kept weights of a vector's tokens.
  auto weigh = [&](int32_t i, const float (&x)[EPV], uint64_t (&g)[EPV]) {
    if (cut || want_m) {
#pragma unroll
      for (int e = 0; e < EPV; ++e) g[e] = p.weight_if(x[e], kept(i, e, x[e]));
    } else {
#pragma unroll
      for (int e = 0; e < EPV; ++e) g[e] = p.weight_of(x[e]);
    }
  };
  // The kept weight of parts of the row, in order: its quarters from the bins, where
  // those and the cut's own bin say it all; else from a list of the kept tokens if
  // they fit one; else a wave's part each, weighed once more.
  int32_t p0, p1, parts = kSampleWaves;
  if (want_p && !want_m && s.bin_whole >= 0) {
    parts = kSampleQuarters;
    uint64_t sum = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int b = w % 4 * 256 + lane * 4 + e;
      sum += b < s.bin_whole ? s.weight[w / 4][b] : 0;
    }
    sum = wave_scan(sum);
    if (lane == kWave - 1) s.part[w] = sum;
    __syncthreads();
    if (tid < kSampleQuarters) {
      sum = s.quarter[tid];
      for (int v = 0; v < 4; ++v) sum += s.part[4 * tid + v];
    }
    __syncthreads();
    if (tid < kSampleQuarters) s.part[tid] = sum;
  } else {
    if (cut || want_m) {
      // a value below which min_p keeps nothing: T ln(min_p) under the maximum, and some more
      const float depth = -1.01f * temperature * logf(fmaxf(min_p, 1e-37f)) + 1e-5f * fabsf(mx) + 1e-30f;
      const float low = want_m && mx - depth > cut_x ? mx - depth : cut_x;
      p.collect(low, mx, want_m, [&](int32_t i, int e, float x) { return kept(i, e, x) != 0; });
      const uint32_t n = s.n_list;
      if (n <= kSampleList) {
        uint64_t id[2], g[2];
        uint32_t at[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          at[e] = tid + e * kSampleThreads;
          const bool in = at[e] < n;
          id[e] = in ? s.list[at[e]] : 0;
          const uint64_t v = p.weight_if(key_float((uint32_t)(id[e] >> 32)), in);
          g[e] = in ? v : 0;
        }
        p.draw_list(n, u, id, g, at, a.tokens + r);
        return;
      }
    }
    uint64_t sum = 0;
    p.each([&](int32_t i, const float (&x)[EPV]) {
      uint64_t g[EPV];
      weigh(i, x, g);
#pragma unroll
      for (int e = 0; e < EPV; ++e) sum += g[e];
    });
    sum = wave_scan(sum);
    if (lane == kWave - 1) s.part[w] = sum;
  }
  __syncthreads();
  total = 0;
  for (int v = 0; v < parts; ++v) total += s.part[v];
  // the first token at which the running weight exceeds u * total
  const uint64_t target = times_fraction<false>(u, total);
  uint64_t seen = 0;
  int part = 0;
  while (part < parts - 1 && seen + s.part[part] <= target) seen += s.part[part++];
  const int32_t wide = kSampleWaves / parts * p.per;
  p0 = part * wide;
  p1 = min(p0 + wide, row.n_vec);
  for (int32_t base = p0; base < p1; base += kSampleThreads) {
    const int32_t i0 = base + w * kWave, i = i0 + lane;
    float x[EPV];
    uint64_t g[EPV], mine = 0, all;
    p.get(i0, p1, x);
    weigh(i, x, g);
#pragma unroll
    for (int e = 0; e < EPV; ++e) mine += g[e];
    const uint64_t upto = seen + p.wg_scan(mine, all);
    if (upto > target && upto - mine <= target) {
      uint64_t at = upto - mine;
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        if (at <= target && at + g[e] > target) a.tokens[r] = (int32_t)row.index(i, e);
        at += g[e];
      }
    }
    seen += all;
    if (seen > target) break;
  }
}

}  // namespace
}  // namespace baton
