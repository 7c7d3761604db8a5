// Drafted tokens against the target's distribution, from given uniform numbers.
//
// With p the distribution that sampling draws from (sample_kernel.hpp) for the target's
// row of logits, q the draft's -- from its row of logits with the same parameters, or
// all at the drafted token -- draft x is accepted if u q(x) < p(x).  At the first draft
// that is not, a token is drawn from max(0, p - q); behind the last one, from p.  So a
// token is distributed as p whatever the draft.
//
//  1. What every row keeps, a workgroup per row: its largest value, the last token that
//     the prefixes keep, the weight of the kept ones.  Reads all logits once.
//  2. A slot's vocabulary in segments, a workgroup each: every one finds the row in which
//     the slot's drafts end, and adds up its segment's weights to draw from, as whole
//     numbers: kept weights themselves, or p - q in units of 2^-50.
//  3. A workgroup per slot: the segment in which u times their sum lies, then the token.
// Weights are those of sample_kernel.hpp, whole numbers, whose sums do not depend on an
// order: the same inputs give the same tokens.
#pragma once

#include "sample_kernel.hpp"

namespace baton {
namespace {

constexpr int kVerifyThreads = 256, kVerifyWaves = kVerifyThreads / kWave;
constexpr int kVerifySegs = 32;          // segments of the vocabulary

struct VerifyArgs {
  const uint8_t* target;       // [batch * width] rows
  const uint8_t* draft;        // [batch * (width - 1)] rows; null: the draft's distribution is its token
  int64_t target_ld, draft_ld;
  int32_t batch, width, vocab, shift, segs, per_seg;
  const int32_t* drafted;      // [batch][width - 1]
  const int32_t* n_draft;      // [batch]; null: width - 1
  const float* u_accept;       // [batch][width - 1]
  const float* u_token;        // [batch]
  const float* temperature;    // [batch] each; null: 1, off, off, off
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* tokens;             // [batch][width]
  int32_t* n_out;              // [batch]
  SampleKept* kept;            // the target's rows, then the draft's
  uint64_t* sums;              // [batch][segs] of the weights to draw from, then of p's own
};

__device__ __forceinline__ int32_t verify_drafts(const VerifyArgs& a, int32_t b) {
  return a.n_draft ? min(a.n_draft[b], a.width - 1) : a.width - 1;
}

template <typename T>
__global__ void __launch_bounds__(kSampleThreads) verify_rows_kernel(const VerifyArgs a) {
  extern __shared__ __attribute__((aligned(16))) u32x4 row_lds[];
  __shared__ SampleShared s;
  const int32_t n_target = a.batch * a.width;
  const int32_t r = blockIdx.x;
  const bool target = r < n_target;
  const int32_t per = target ? a.width : a.width - 1, at = target ? r : r - n_target;
  const int32_t b = at / per, i = at - b * per;
  const int32_t n = verify_drafts(a, b);
  if (target ? i > n : i >= n) return;
  const SampleDraw d = {a.vocab, a.shift, a.temperature ? a.temperature[b] : 1.f, a.top_k ? a.top_k[b] : 0,
                        a.top_p ? a.top_p[b] : 1.f, a.min_p ? a.min_p[b] : 0.f, 0.f};
  const uint8_t* const row = target ? a.target + at * a.target_ld * T::kBytes : a.draft + at * a.draft_ld * T::kBytes;
  sample_row<T, true>(s, row_lds, row, d, nullptr, a.kept + r);
}

// The kept weights of one row.
template <typename T>
struct VerifyRow {
  const uint8_t* row;
  SampleKept kept;
  double top, scale, least, floor;

  __device__ __forceinline__ float value(int32_t i) const {
    if constexpr (T::kBytes == 4) return reinterpret_cast<const float*>(row)[i];
    else return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(row)[i] << 16);
  }
  __device__ __forceinline__ uint64_t weight(const double* table, float x, uint32_t index) const {
    if (kept.infinite) x = x == INFINITY ? 1.f : __uint_as_float(0x7FC00000u);
    if (!(x <= kept.mx) || kept.none) return 0;                       // a NaN
    if (((uint64_t)float_key(x) << 32 | (uint32_t)~index) < kept.cut) return 0;
    if (kept.one) return 1;
    const double d = sample_weight(table, x, top, scale, least);
    return d >= floor || x == kept.mx ? sample_whole(d) : 0;
  }
};

template <typename T>
__device__ __forceinline__ VerifyRow<T> verify_row(const VerifyArgs& a, const uint8_t* rows, int64_t ld, int32_t at,
                                                   const SampleKept* kept, int32_t b) {
  VerifyRow<T> r;
  r.row = rows + at * ld * T::kBytes;
  r.kept = kept[at];
  r.top = (double)r.kept.mx;
  r.scale = sample_scale(a.temperature ? a.temperature[b] : 1.f);
  r.least = sample_least(a.shift);
  const float min_p = a.min_p ? a.min_p[b] : 0.f;
  r.floor = min_p > 0.f ? ldexp((double)min_p, a.shift) : -1.0;
  return r;
}

// The row in which a slot's drafts end, and what to draw from there.
template <typename T>
struct VerifyEnd {
  VerifyRow<T> p, q;
  int32_t n;               // accepted drafts
  int32_t minus;           // 0: p; 1: p - q; 2: p without the token `x`
  int32_t x;
  double cp, cq;           // weights to units of 2^-50 of p and of q

  // The weight of token i to draw from, of p itself in `own`.
  __device__ __forceinline__ uint64_t weight(const double* table, int32_t i, uint64_t& own) const {
    own = p.weight(table, p.value(i), (uint32_t)i);
    if (minus == 0 || own == 0) return own;
    if (minus == 2) return i == x ? 0 : own;
    const uint64_t h = q.weight(table, q.value(i), (uint32_t)i);
    const double d = (double)own * cp - (double)h * cq;
    return d > 0.0 ? sample_whole(d) : 0;
  }
};

// Accepted drafts of a slot, by the workgroup's first wave; all threads get the answer.
template <typename T>
__device__ __forceinline__ VerifyEnd<T> verify_end(const VerifyArgs& a, const double* table, int32_t b, int32_t n_draft,
                                                   int32_t* shared) {
  const int32_t i = threadIdx.x, w1 = a.width - 1;
  const SampleKept* const draft_kept = a.kept + (int64_t)a.batch * a.width;
  if (threadIdx.x < kWave) {
    bool good = false;
    if (i < n_draft) {
      const int32_t x = a.drafted[b * w1 + i];
      const float u_in = a.u_accept[b * w1 + i];
      const double u = u_in > 0.f ? fminf(u_in, 0x1.fffffep-1f) : 0.f;
      if (x >= 0 && x < a.vocab) {
        const VerifyRow<T> p = verify_row<T>(a, a.target, a.target_ld, b * a.width + i, a.kept, b);
        const double g = (double)p.weight(table, p.value(x), (uint32_t)x);
        double h = 1.0, all = 1.0;
        if (a.draft) {
          const VerifyRow<T> q = verify_row<T>(a, a.draft, a.draft_ld, b * w1 + i, draft_kept, b);
          h = (double)q.weight(table, q.value(x), (uint32_t)x);
          all = (double)q.kept.total;
        }
        good = u * h * (double)p.kept.total < g * all;
      }
    }
    const uint64_t bad = ~__ballot(good);
    if (threadIdx.x == 0) *shared = __builtin_ctzll(bad);      // lanes from n_draft on are not good
  }
  __syncthreads();
  VerifyEnd<T> e;
  const int32_t n = *shared;
  e.n = n;
  e.p = verify_row<T>(a, a.target, a.target_ld, b * a.width + n, a.kept, b);
  e.minus = 0;
  e.x = -1;
  e.cp = e.cq = 0.0;
  e.q = e.p;
  if (n < n_draft) {
    e.x = a.drafted[b * w1 + n];
    e.minus = 2;
    if (a.draft) {
      e.q = verify_row<T>(a, a.draft, a.draft_ld, b * w1 + n, draft_kept, b);
      e.minus = e.q.kept.none || e.p.kept.none ? 0 : 1;
      e.cp = 0x1p50 / (double)e.p.kept.total;
      e.cq = 0x1p50 / (double)e.q.kept.total;
    }
  }
  return e;
}

__device__ __forceinline__ uint64_t verify_sum(uint64_t x, uint64_t* shared) {
  x = wave_scan(x);
  __syncthreads();
  if (threadIdx.x % kWave == kWave - 1) shared[threadIdx.x / kWave] = x;
  __syncthreads();
  x = 0;
#pragma unroll
  for (int v = 0; v < kVerifyWaves; ++v) x += shared[v];
  return x;
}

template <typename T>
__global__ void __launch_bounds__(kVerifyThreads) verify_sums_kernel(const VerifyArgs a) {
  __shared__ double table[128];
  __shared__ uint64_t sums[kVerifyWaves];
  __shared__ int32_t accepted;
  const int32_t b = blockIdx.y, seg = blockIdx.x;
  const int32_t n_draft = verify_drafts(a, b);
  if (n_draft < 0) return;
  if (threadIdx.x < 128) table[threadIdx.x] = ldexp(exp2((double)threadIdx.x / 128.0), a.shift);
  __syncthreads();
  const VerifyEnd<T> e = verify_end<T>(a, table, b, n_draft, &accepted);
  const int32_t i0 = seg * a.per_seg, i1 = min(i0 + a.per_seg, a.vocab);
  uint64_t sum = 0, own_sum = 0;
  for (int32_t i = i0 + threadIdx.x; i < i1; i += kVerifyThreads) {
    uint64_t own;
    sum += e.weight(table, i, own);
    own_sum += own;
  }
  sum = verify_sum(sum, sums);
  own_sum = verify_sum(own_sum, sums);
  if (threadIdx.x == 0) {
    a.sums[(int64_t)b * a.segs + seg] = sum;
    a.sums[(int64_t)(a.batch + b) * a.segs + seg] = own_sum;
  }
}

template <typename T>
__global__ void __launch_bounds__(kVerifyThreads) verify_draw_kernel(const VerifyArgs a) {
  __shared__ double table[128];
  __shared__ uint64_t sums[kVerifyWaves];
  __shared__ int32_t accepted, token;
  const int32_t b = blockIdx.x, w1 = a.width - 1;
  const int32_t n_draft = verify_drafts(a, b);
  if (n_draft < 0) {                      // a free slot
    for (int32_t i = threadIdx.x; i < a.width; i += kVerifyThreads) a.tokens[b * a.width + i] = -1;
    if (threadIdx.x == 0) a.n_out[b] = 0;
    return;
  }
  if (threadIdx.x < 128) table[threadIdx.x] = ldexp(exp2((double)threadIdx.x / 128.0), a.shift);
  if (threadIdx.x == 0) token = -1;
  __syncthreads();
  VerifyEnd<T> e = verify_end<T>(a, table, b, n_draft, &accepted);
  // The segment in which the target lies.
  const uint64_t* seg_sums = a.sums + (int64_t)b * a.segs;
  uint64_t total = 0;
  for (int32_t v = 0; v < a.segs; ++v) total += seg_sums[v];
  if (total == 0) {                       // nothing of p is above q: from p
    e.minus = 0;
    seg_sums += (int64_t)a.batch * a.segs;
    for (int32_t v = 0; v < a.segs; ++v) total += seg_sums[v];
  }
  const float u_in = a.u_token[b];
  const uint64_t target = times_fraction<false>(u_in > 0.f ? fminf(u_in, 0x1.fffffep-1f) : 0.f, total);
  uint64_t seen = 0;
  int32_t seg = 0;
  while (seg < a.segs - 1 && seen + seg_sums[seg] <= target) seen += seg_sums[seg++];
  // The first token of it at which the running weight exceeds the target.
  const int32_t i0 = seg * a.per_seg, i1 = min(i0 + a.per_seg, a.vocab);
  for (int32_t base = i0; base < i1 && total > 0; base += kVerifyThreads) {
    const int32_t i = base + threadIdx.x;
    uint64_t own;
    const uint64_t g = i < i1 ? e.weight(table, i, own) : 0;
    const uint64_t upto = wave_scan(g);
    __syncthreads();
    if (threadIdx.x % kWave == kWave - 1) sums[threadIdx.x / kWave] = upto;
    __syncthreads();
    uint64_t before = seen, all = 0;
#pragma unroll
    for (int v = 0; v < kVerifyWaves; ++v) {
      before += v < (int)(threadIdx.x / kWave) ? sums[v] : 0;
      all += sums[v];
    }
    if (before + upto > target && before + upto - g <= target) token = i;
    seen += all;
    if (seen > target) break;
  }
  __syncthreads();
  for (int32_t i = threadIdx.x; i < a.width; i += kVerifyThreads)
    a.tokens[b * a.width + i] = i < e.n ? a.drafted[b * w1 + i] : i == e.n ? token : -1;
  if (threadIdx.x == 0) a.n_out[b] = e.n + 1;
}

}  // namespace
}  // namespace baton
