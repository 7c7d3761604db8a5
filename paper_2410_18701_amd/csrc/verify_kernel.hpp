// Drafted tokens against the target's distribution, from given uniform numbers.
//
// With p the distribution that sampling draws from (sample_kernel.hpp) for the target's
// row of logits, q the draft's -- from its row of logits with the same parameters, or
// all at the drafted token -- draft x is accepted if u q(x) < p(x).  At the first draft
// that is not, a token is drawn from max(0, p - q); behind the last one, from p.  So a
// token is distributed as p whatever the draft.
//
//  1. What every row keeps: its largest value, the last token that the prefixes keep, the
//     weight of the kept ones.  Reads all logits once.  Rows without prefixes, and greedy
//     ones, are added up in pieces, a workgroup each, relative to the piece's largest
//     value; the others take a workgroup each, as sampling does.
//  2. A slot's vocabulary in segments, a workgroup each: every one finds the row in which
//     the slot's drafts end, and adds up its segment's weights to draw from, as whole
//     numbers: kept weights themselves, or p - q in units of 2^-50.
//  3. A workgroup per slot: the segment's part in which u times their sum lies, then the
//     token.
// Weights are those of sample_kernel.hpp, whole numbers, whose sums do not depend on an
// order: the same inputs give the same tokens.
//
// Four launches (3.4 us each if they did nothing), 19 us for one slot of three drafts over
// 50,257, fp32.  64 slots of four drafts over 128,000, bf16, parameters of all kinds: 24 + 74 + 20
// + 9 us, of which the first two read 118 MB (20 us at a plain read's rate).
#pragma once

#include "sample_kernel.hpp"

namespace baton {
namespace {

constexpr int kVerifyThreads = 256, kVerifyWaves = kVerifyThreads / kWave;
constexpr int kVerifySegs = 32;          // segments of the vocabulary at most, a workgroup each
constexpr int kVerifyParts = kVerifySegs * kVerifyWaves;   // of a wave each
constexpr int kVerifyVecs = 4;           // 16-byte vectors of a piece per thread

// A piece of a row: its largest value and that one's first index, the weight of its tokens
// relative to it (of an infinite one, how often it is there).
struct VerifyPiece {
  uint64_t weight;
  float mx;
  uint32_t first;
};

struct VerifyArgs {
  const uint8_t* target;       // [batch * width] rows
  const uint8_t* draft;        // [batch * (width - 1)] rows; null: the draft's distribution is its token
  int64_t target_ld, draft_ld;
  int32_t batch, width, vocab, shift, segs, per_part;   // per_part: tokens of a wave's part of a segment
  const int32_t* drafted;      // [batch][width - 1]
  const int32_t* n_draft;      // [batch]; null: width - 1
  const int32_t* taken;        // [batch] new tokens that the cache's step took; null: those that n_draft says
  const float* u_accept;       // [batch][width - 1]
  const float* u_token;        // [batch]
  const float* temperature;    // [batch] each; null: 1, off, off, off
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* tokens;             // [batch][width]
  int32_t* n_out;              // [batch]
  SampleKept* kept;            // the target's rows, then the draft's
  uint64_t* sums;              // [batch][kVerifyParts] of the weights to draw from, then of p's own
  VerifyPiece* pieces;         // [rows][n_pieces]
  int32_t n_pieces, slot_rows; // rows of a slot: width, and width - 1 with a draft's logits
};

// A slot's drafts, negative if it takes no part: also where the cache's step took none of its
// tokens, or more of them (a prompt's) than there are rows.
__device__ __forceinline__ int32_t verify_drafts(const VerifyArgs& a, int32_t b) {
  const int32_t n = a.n_draft ? min(a.n_draft[b], a.width - 1) : a.width - 1;
  if (!a.taken) return n;
  const int32_t t = a.taken[b];
  return t < 1 || t > a.width ? -1 : min(n, t - 1);
}

// A slot's row i: of the target's, then of the draft's.  False if it is not needed.
struct VerifyLogits {
  int32_t b, r;                // r: of all target rows, then all draft rows
  const uint8_t* logits;
  SampleDraw draw;
  bool one, pieces;            // the first token alone; no prefixes

  template <typename T>
  __device__ __forceinline__ bool find(const VerifyArgs& a, int32_t slot, int32_t i) {
    b = slot;
    const bool target = i < a.width;
    const int32_t n = verify_drafts(a, b);
    if (target ? i > n : i - a.width >= n) return false;
    const int32_t at = target ? b * a.width + i : b * (a.width - 1) + i - a.width;
    r = target ? at : a.batch * a.width + at;
    logits = target ? a.target + at * a.target_ld * T::kBytes : a.draft + at * a.draft_ld * T::kBytes;
    draw = {a.vocab, a.shift, a.temperature ? a.temperature[b] : 1.f, a.top_k ? a.top_k[b] : 0,
            a.top_p ? a.top_p[b] : 1.f, a.min_p ? a.min_p[b] : 0.f, 0.f};
    one = !(draw.temperature > 0.f) || draw.top_k == 1 || draw.min_p > 1.f;
    pieces = one || (!(draw.top_k > 0 && draw.top_k < a.vocab) && !(draw.top_p < 1.f) && !(draw.min_p > 0.f));
    return true;
  }
};

__device__ __forceinline__ void verify_table(double* table, int32_t shift) {
  if (threadIdx.x < 128) table[threadIdx.x] = ldexp(exp2((double)threadIdx.x / 128.0), shift);
}

// A piece a workgroup, whose logits stay in registers between their maximum and their
// weights: a row is read once, by as many workgroups as its length fills.  Bound by the
// weights' arithmetic, in 64 bits: 480 rows of 128,000 take 65 us with weights, 30 if greedy.
template <typename T>
__global__ void __launch_bounds__(kVerifyThreads) verify_pieces_kernel(const VerifyArgs a) {
  constexpr int EPV = Lane16<T>::kElems, V = kVerifyVecs;
  __shared__ double table[128];
  __shared__ float sm_mx[kVerifyWaves];
  __shared__ uint64_t sm_sum[kVerifyWaves];
  __shared__ uint32_t sm_first[kVerifyWaves];
  VerifyLogits l;
  if (!l.find<T>(a, blockIdx.y / a.slot_rows, blockIdx.y % a.slot_rows) || !l.pieces) return;
  SampleRow<T> row;
  row.row = l.logits;
  row.off = (int32_t)((reinterpret_cast<uintptr_t>(row.row) & 15u) / T::kBytes);
  row.vocab = a.vocab;
  row.n_vec = (row.off + a.vocab + EPV - 1) / EPV;
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave;
  const int32_t i0 = (int32_t)blockIdx.x * (kVerifyThreads * V) + tid;
  float x[V][EPV], mx = -INFINITY;
  u32x4 v[V];
#pragma unroll
  for (int q = 0; q < V; ++q) {
    const int32_t i = i0 + q * kVerifyThreads;
    v[q] = i < row.n_vec ? row.fetch(i) : u32x4{0, 0, 0, 0};
  }
  verify_table(table, a.shift);
#pragma unroll
  for (int q = 0; q < V; ++q) {
    row.widen(i0 + q * kVerifyThreads, v[q], false, x[q]);      // NaN behind the row
#pragma unroll
    for (int e = 0; e < EPV; ++e) mx = fmaxf(mx, x[q][e]);
  }
  const float own = mx;
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) mx = fmaxf(mx, __shfl_xor(mx, m, kWave));
  if (lane == 0) sm_mx[w] = mx;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kVerifyWaves; ++u) mx = fmaxf(mx, sm_mx[u]);
  uint64_t sum = 0;
  uint32_t first = 0xFFFFFFFFu;
  if (own == mx && mx > -INFINITY) {
#pragma unroll
    for (int q = V - 1; q >= 0; --q)
#pragma unroll
      for (int e = EPV - 1; e >= 0; --e)
        if (x[q][e] == mx) {
          first = row.index(i0 + q * kVerifyThreads, e);
          sum += mx == INFINITY;
        }
  }
  if (!l.one && mx > -INFINITY && mx < INFINITY) {
    const double top = (double)mx, scale = sample_scale(l.draw.temperature), least = sample_least(a.shift);
    sum = 0;
#pragma unroll
    for (int q = 0; q < V; ++q)
#pragma unroll
      for (int e = 0; e < EPV; ++e) sum += sample_whole(sample_weight(table, x[q][e], top, scale, least));
  }
  sum = wave_scan(sum);
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) first = min(first, (uint32_t)__shfl_xor((int)first, m, kWave));
  if (lane == kWave - 1) {
    sm_sum[w] = sum;
    sm_first[w] = first;
  }
  __syncthreads();
  if (tid == 0) {
    for (int u = 1; u < kVerifyWaves; ++u) first = min(first, sm_first[u]);
    first = min(first, sm_first[0]);
    sum = 0;
    for (int u = 0; u < kVerifyWaves; ++u) sum += sm_sum[u];
    a.pieces[(int64_t)l.r * a.n_pieces + blockIdx.x] = {sum, mx, first};
  }
}

// ---- What a row of bf16 logits keeps, by counting its values ----
// Few values are bf16: a row's tokens are counted by their 65,536 possible values in LDS
// (16-bit counters in the values' order), and prefixes end within one value's tokens.  One
// pass over the row, one weight for each value that is there, and a second pass for the
// token's index.  480 rows of 128,000, two rounds of the GPU as the counters fill a compute
// unit's LDS: top_p 105 us, top_k 81, min_p 83, where bins of weights take 192, 89 and 106.
// A row: 16 us to be counted (all compute units together read 4.2 TB/s then), 11 for weights
// and prefixes, 0 to 17 until the index is found.
constexpr int kValueWords = 32768;       // two counters each

struct ValueShared {
  uint32_t count[kValueWords];
  double table[128];
  uint64_t sum[kSampleThreads];          // of each block of 64 values: its tokens' weight,
  uint32_t n[kSampleThreads];            // and their number
  uint16_t list[kSampleThreads];         // blocks that hold tokens
  uint64_t scan[kSampleWaves], high[kSampleWaves], weight, before, before_sum;
  uint32_t mx, n_list, key, nth, found, index;
};

// bf16 bits as numbers of the values' order, -0 as 0.
__device__ __forceinline__ uint32_t value_key(uint32_t h) {
  h = h == 0x8000u ? 0u : h;
  return h ^ (h & 0x8000u ? 0xFFFFu : 0x8000u);
}
__device__ __forceinline__ float key_value(uint32_t key) {
  return __uint_as_float((key & 0x8000u ? key ^ 0x8000u : ~key & 0xFFFFu) << 16);
}
constexpr uint32_t kKeyPlusInf = 0xFF80u, kKeyMinusInf = 0x007Fu;
// Where the counters of keys 2 w and 2 w + 1 lie: a thread's 32 words, four at a time, in
// other banks than its neighbours'.
__device__ __forceinline__ uint32_t value_place(uint32_t w) { return w ^ (w >> 3 & 28u); }

// Prefix sum over the workgroup's 16 waves, exclusive, and the whole.
__device__ __forceinline__ uint64_t value_scan(uint64_t x, uint64_t* shared, uint64_t& total) {
  const int lane = threadIdx.x % kWave, w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint64_t y = wave_scan(x);
  __syncthreads();
  if (lane == kWave - 1) shared[w] = y;
  __syncthreads();
  const uint64_t t = wave_scan(lane < kSampleWaves ? shared[lane] : 0);    // lane l: up to wave l
  auto from = [&](int l) {
    return (uint64_t)__builtin_amdgcn_readlane((int)(t >> 32), l) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)t, l);
  };
  total = from(kSampleWaves - 1);
  return y - x + (w > 0 ? from(w - 1) : 0);
}

// False (for all threads): a value is there too often for its counter.
__device__ __forceinline__ bool verify_values_row(ValueShared& s, const VerifyLogits& l, SampleKept* out) {
  constexpr int EPV = 8, U = 4;
  const SampleDraw& d = l.draw;
  SampleRow<BF16Tag> row;
  row.row = l.logits;
  row.off = (int32_t)((reinterpret_cast<uintptr_t>(row.row) & 15u) / 2);
  row.vocab = d.vocab;
  row.n_vec = (row.off + d.vocab + EPV - 1) / EPV;
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave;
  for (int i = tid; i < kValueWords / 4; i += kSampleThreads) reinterpret_cast<u32x4*>(s.count)[i] = u32x4{0, 0, 0, 0};
  verify_table(s.table, d.shift);
  if (tid == 0) s.mx = s.n_list = 0;
  __syncthreads();
  auto in_row = [&](int32_t i, int e) { return (uint32_t)(i * EPV - row.off + e) < (uint32_t)d.vocab; };
  auto add = [&](int32_t i, const u32x4& v) {
    const bool all = in_row(i, 0) && in_row(i, EPV - 1);
#pragma unroll
    for (int e = 0; e < EPV; ++e) {
      const uint32_t k = value_key(v[e / 2] >> (16 * (e % 2)) & 0xFFFFu);
      if (all || in_row(i, e)) atomicAdd(&s.count[value_place(k >> 1)], 1u << (16 * (k & 1)));
    }
  };
  for (int32_t i = tid; i < row.n_vec; i += U * kSampleThreads) {
    u32x4 v[U];
#pragma unroll
    for (int q = 0; q < U; ++q)
      if (i + q * kSampleThreads < row.n_vec) v[q] = row.fetch(i + q * kSampleThreads);
#pragma unroll
    for (int q = 0; q < U; ++q)
      if (i + q * kSampleThreads < row.n_vec) add(i + q * kSampleThreads, v[q]);
  }
  __syncthreads();
  // This thread's 64 values, from the largest on: those of block 1023 - tid.
  const uint32_t block = kSampleThreads - 1 - tid;
  uint32_t most = 0, n = 0;
#pragma unroll
  for (int j = 0; j < 32; j += 4) {
    const u32x4 c = *reinterpret_cast<const u32x4*>(&s.count[value_place(block * 32 + j)]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      n += (c[e] & 0xFFFFu) + (c[e] >> 16);
      const uint32_t k = block * 64 + 2 * (j + e);
      if (c[e] & 0xFFFFu && k > kKeyMinusInf && k <= kKeyPlusInf) most = k;
      if (c[e] >> 16 && k + 1 > kKeyMinusInf && k + 1 <= kKeyPlusInf) most = k + 1;
    }
  }
  s.sum[block] = 0;
  s.n[block] = 0;
  if (n) s.list[atomicAdd(&s.n_list, 1u)] = (uint16_t)block;
  if (most) atomicMax(&s.mx, most);
  uint64_t total;
  value_scan(n, s.scan, total);
  if (total != (uint64_t)d.vocab) return false;
  const uint32_t top_key = s.mx;
  if (top_key == 0) {
    if (tid == 0) *out = {0, 0, 0.f, 0, 0, 1};
    return true;
  }
  const bool infinite = top_key == kKeyPlusInf;      // beside an infinity nothing finite has weight
  const float mx = infinite ? 1.f : key_value(top_key);
  const double top = (double)mx, scale = sample_scale(d.temperature), least = sample_least(d.shift);
  const bool want_k = d.top_k > 0 && d.top_k < d.vocab, want_p = d.top_p < 1.f, want_m = d.min_p > 0.f;
  const double floor_w = want_m ? ldexp((double)d.min_p, d.shift) : -1.0;
  // Key k's tokens that can be drawn, and a token's weight.
  auto tokens = [&](uint32_t k) {
    const uint32_t m = s.count[value_place(k >> 1)] >> (16 * (k & 1)) & 0xFFFFu;
    return k <= top_key && k > kKeyMinusInf && !(infinite && k < top_key) ? m : 0u;
  };
  auto weight = [&](uint32_t k) { return sample_weight(s.table, infinite ? 1.f : key_value(k), top, scale, least); };
  // The blocks' sums: a wave per block, a lane per value.
  uint64_t high = 0;                                 // of the tokens that min_p keeps
  for (uint32_t q = w; q < s.n_list; q += kSampleWaves) {
    const uint32_t b = s.list[q], k = b * 64 + lane, m = tokens(k);
    const double x = weight(k);
    const uint64_t g = sample_whole(x) * m, sum = wave_scan(g), count = wave_scan(m);
    high += x >= floor_w || k == top_key ? g : 0;
    if (lane == kWave - 1) {
      s.sum[b] = sum;
      s.n[b] = (uint32_t)count;
    }
  }
  high = wave_scan(high);
  if (lane == kWave - 1) s.high[w] = high;
  __syncthreads();
  const uint64_t count = s.n[block], sum = s.sum[block];
  uint64_t all_count, kept, kept_high = 0;
  if (want_m)
    for (int v = 0; v < kSampleWaves; ++v) kept_high += s.high[v];
  const uint64_t count_before = value_scan(count, s.scan, all_count);
  const uint64_t sum_before = value_scan(sum, s.scan, kept);
  bool cut = false;
#pragma unroll 1
  for (int by_weight = 0; by_weight < 2; ++by_weight) {
    uint64_t need = (uint64_t)d.top_k;
    if (by_weight) {
      if (!want_p) break;
      need = d.top_p > 0.f ? max(times_fraction<true>(d.top_p, kept), (uint64_t)1) : 1;
    } else if (!want_k || need >= all_count) {
      continue;
    }
    const uint64_t before = by_weight ? sum_before : count_before, mine = by_weight ? sum : count;
    __syncthreads();                                 // the last prefix's end has been read
    if (before < need && before + mine >= need) {    // one thread
      s.found = block;
      s.before = before;
      s.before_sum = sum_before;
    }
    __syncthreads();
    if (w == 0) {                                    // the block's values, the largest first
      const uint32_t k = s.found * 64 + kWave - 1 - lane, m = tokens(k);
      const uint64_t g = sample_whole(weight(k)), step = by_weight ? g : 1;
      const uint64_t at = s.before + wave_scan(step * m) - step * m, at_sum = s.before_sum + wave_scan(g * m) - g * m;
      if (at < need && at + step * m >= need) {      // one lane
        const uint64_t nth = (need - at + step - 1) / step;
        s.key = k;
        s.nth = nth == m ? 0 : (uint32_t)nth;        // 0: all of them
        s.weight = at_sum + nth * g;
      }
    }
    __syncthreads();
    kept = s.weight;
    cut = true;
  }
  kept = min(kept, want_m ? kept_high : kept);
  const uint32_t key = s.key, nth = s.nth;
  uint32_t index = 0xFFFFFFFFu;                      // the last kept token's; all of a value: behind its last
  if (cut && nth) {
    // The nth token of value `key`: four vectors of each thread at a time, counted, until
    // they hold it.
    uint64_t seen = 0, all;
    for (int32_t base = 0; base < row.n_vec && seen < nth; base += U * kSampleThreads) {
      uint32_t b[U], m = 0;
      u32x4 v[U];
#pragma unroll
      for (int q = 0; q < U; ++q)
        if (base + tid * U + q < row.n_vec) v[q] = row.fetch(base + tid * U + q);
#pragma unroll
      for (int q = 0; q < U; ++q) {
        b[q] = 0;
        if (base + tid * U + q < row.n_vec) {
#pragma unroll
          for (int e = 0; e < EPV; ++e)
            b[q] |= value_key(v[q][e / 2] >> (16 * (e % 2)) & 0xFFFFu) == key && in_row(base + tid * U + q, e) ? 1u << e : 0u;
        }
        m += __popc(b[q]);
      }
      uint64_t at = seen + value_scan(m, s.scan, all);
      if (at < nth && at + m >= nth) {
#pragma unroll
        for (int q = 0; q < U; ++q)
          for (; b[q]; b[q] &= b[q] - 1)
            if (++at == nth) s.index = row.index(base + tid * U + q, __builtin_ctz(b[q]));
      }
      seen += all;
    }
    __syncthreads();
    index = s.index;
  }
  if (tid == 0) {
    const uint64_t id = (uint64_t)float_key(infinite ? 1.f : key_value(key)) << 32 | (uint32_t)~index;
    *out = {cut ? id : 0, kept, mx, infinite, 0, 0};
  }
  return true;
}

// A row a workgroup: what it keeps, or its pieces' sum.  Unlike sums and draws, no part of
// it can be left out for a rejected draft: which ones are is known only afterwards.
template <typename T>
__global__ void __launch_bounds__(kSampleThreads) verify_rows_kernel(const VerifyArgs a) {
  constexpr bool kValues = T::kBytes == 2;
  constexpr size_t kRow = (sizeof(SampleShared) + 15) / 16;            // of the row's copy, in vectors
  static_assert(!kValues || sizeof(ValueShared) <= sizeof(SampleShared) + kSampleRowBytes, "either fits");
  extern __shared__ __attribute__((aligned(16))) u32x4 lds[];
  SampleShared& s = *reinterpret_cast<SampleShared*>(lds);
  VerifyLogits l;
  if (!l.find<T>(a, blockIdx.x / a.slot_rows, blockIdx.x % a.slot_rows)) return;
  const int32_t r = l.r;
  if (!l.pieces) {
    if constexpr (kValues) {
      if (verify_values_row(*reinterpret_cast<ValueShared*>(lds), l, a.kept + r)) return;
      __syncthreads();
    }
    sample_row<T, true>(s, lds + kRow, l.logits, l.draw, nullptr, a.kept + r);
    return;
  }
  // From the row's pieces, by the first wave.
  verify_table(s.table, a.shift);
  __syncthreads();
  if (threadIdx.x >= kWave) return;
  const VerifyPiece* const pieces = a.pieces + (int64_t)r * a.n_pieces;
  float mx = -INFINITY;
  for (int32_t i = threadIdx.x; i < a.n_pieces; i += kWave) mx = fmaxf(mx, pieces[i].mx);
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) mx = fmaxf(mx, __shfl_xor(mx, m, kWave));
  const double scale = sample_scale(l.draw.temperature), least = sample_least(a.shift), unit = ldexp(1.0, -a.shift);
  double sum = 0.0;
  uint32_t first = 0xFFFFFFFFu;
  for (int32_t i = threadIdx.x; i < a.n_pieces; i += kWave) {
    const VerifyPiece p = pieces[i];
    if (p.mx == mx) first = min(first, p.first);
    if (p.mx == mx) sum += (double)p.weight;
    else if (mx < INFINITY && p.mx > -INFINITY)
      sum += (double)p.weight * (sample_weight(s.table, p.mx, (double)mx, scale, least) * unit);
  }
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) {
    sum += __shfl_xor(sum, m, kWave);
    first = min(first, (uint32_t)__shfl_xor((int)first, m, kWave));
  }
  if (threadIdx.x != 0) return;
  const bool infinite = mx == INFINITY;
  const float top = infinite ? 1.f : mx;
  const uint64_t one = ldexp(1.0, a.shift);          // the weight of an infinite one
  if (mx == -INFINITY) a.kept[r] = {0, 0, 0.f, 0, 0, 1};
  else if (l.one) a.kept[r] = {(uint64_t)float_key(top) << 32 | (uint32_t)~first, 1, top, infinite, 1, 0};
  else a.kept[r] = {0, infinite ? (uint64_t)sum * one : (uint64_t)rint(sum), top, infinite, 0, 0};
}

// The kept weights of one row.
template <typename T>
struct VerifyRow {
  const uint8_t* row;
  SampleKept kept;
  double top, scale, least, floor;
  float low;                   // the last kept token's value

  __device__ __forceinline__ float value(int32_t i) const {
    if constexpr (T::kBytes == 4) return reinterpret_cast<const float*>(row)[i];
    else return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(row)[i] << 16);
  }
  __device__ __forceinline__ uint64_t weight(const double* table, float x, uint32_t index) const {
    if (kept.infinite) x = x == INFINITY ? 1.f : __uint_as_float(0x7FC00000u);
    if (!(x >= low)) return 0;                                        // below the last kept value, or a NaN
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
  r.low = r.kept.none ? INFINITY : r.kept.cut ? key_float((uint32_t)(r.kept.cut >> 32)) : -INFINITY;
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

  // The weight of token i to draw from, of p itself in `own`; xp, xq: its logits.
  __device__ __forceinline__ uint64_t weight(const double* table, int32_t i, float xp, float xq, uint64_t& own) const {
    own = p.weight(table, xp, (uint32_t)i);
    if (minus == 0 || own == 0) return own;
    if (minus == 2) return i == x ? 0 : own;
    const uint64_t h = q.weight(table, xq, (uint32_t)i);
    const double d = (double)own * cp - (double)h * cq;
    return d > 0.0 ? sample_whole(d) : 0;
  }
  // The logits of N tokens from `i` on, `step` apart, below `end` (the others' are -inf).
  template <int N>
  __device__ __forceinline__ void values(int32_t i, int32_t step, int32_t end, float (&xp)[N], float (&xq)[N]) const {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int32_t at = i + e * step < end ? i + e * step : end - 1;
      xp[e] = p.value(at);
      xq[e] = minus == 1 ? q.value(at) : 0.f;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) xp[e] = i + e * step < end ? xp[e] : -INFINITY;
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
    if (i < w1) {            // all drafts' loads at once, whatever their number
      const int32_t x = a.drafted[b * w1 + i], at = x >= 0 && x < a.vocab ? x : 0;
      const float u_in = a.u_accept[b * w1 + i];
      const double u = u_in > 0.f ? fminf(u_in, 0x1.fffffep-1f) : 0.f;
      const VerifyRow<T> p = verify_row<T>(a, a.target, a.target_ld, b * a.width + i, a.kept, b);
      VerifyRow<T> q = p;
      if (a.draft) q = verify_row<T>(a, a.draft, a.draft_ld, b * w1 + i, draft_kept, b);
      const float xp = p.value(at), xq = a.draft ? q.value(at) : 0.f;
      if (i < n_draft && x == at) {
        const double g = (double)p.weight(table, xp, (uint32_t)x);
        const double h = a.draft ? (double)q.weight(table, xq, (uint32_t)x) : 1.0;
        const double all = a.draft ? (double)q.kept.total : 1.0;
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

// A segment a workgroup, in parts of a wave each, in whole 16-byte vectors where rows start
// at them.  Every workgroup finds the accepted drafts by itself, from two numbers a draft,
// which saves a launch.  Bound by the weights' arithmetic and that chain of loads: 64 slots
// of 128,000 20 us (by single elements 28).
template <typename T>
__global__ void __launch_bounds__(kVerifyThreads) verify_sums_kernel(const VerifyArgs a) {
  __shared__ double table[128];
  __shared__ int32_t accepted;
  const int32_t b = blockIdx.y, part = blockIdx.x * kVerifyWaves + threadIdx.x / kWave;
  const int32_t n_draft = verify_drafts(a, b);
  if (n_draft < 0) return;
  verify_table(table, a.shift);
  __syncthreads();
  const VerifyEnd<T> e = verify_end<T>(a, table, b, n_draft, &accepted);
  const int32_t i0 = min(part * a.per_part, a.vocab);          // (2^24 tokens at most)
  int32_t i1 = min(i0 + a.per_part, a.vocab);
  uint64_t sum = 0, own_sum = 0;
  if (e.p.kept.one) {                     // one token alone, whose index is known
    const int32_t i = (int32_t)~(uint32_t)e.p.kept.cut;
    if (threadIdx.x % kWave == 0 && i >= i0 && i < i1) sum = e.weight(table, i, e.p.value(i), e.minus == 1 ? e.q.value(i) : 0.f, own_sum);
    i1 = 0;
  }
  const int32_t lane = threadIdx.x % kWave;
  // Rows that start at 16 bytes: V vectors of a lane at a time (parts begin at whole ones).
  constexpr int EPV = Lane16<T>::kElems, V = 4;
  int32_t base = i0;
  if (((reinterpret_cast<uintptr_t>(e.p.row) | (e.minus == 1 ? reinterpret_cast<uintptr_t>(e.q.row) : 0)) & 15u) == 0) {
    const int32_t end = i1 > i0 ? i0 + (i1 - i0) / EPV * EPV : i0;
    for (; base < end; base += V * EPV * kWave) {
      u32x4 vp[V], vq[V];
#pragma unroll
      for (int q = 0; q < V; ++q) {
        const int32_t at = min(base + (q * kWave + lane) * EPV, end - EPV) / EPV;
        vp[q] = reinterpret_cast<const u32x4*>(e.p.row)[at];
        vq[q] = e.minus == 1 ? reinterpret_cast<const u32x4*>(e.q.row)[at] : u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int q = 0; q < V; ++q) {
        const int32_t i = base + (q * kWave + lane) * EPV;
        if (i >= end) continue;
        float xp[EPV], xq[EPV];
        Lane16<T>::widen(vp[q], xp);
        Lane16<T>::widen(vq[q], xq);
#pragma unroll
        for (int k = 0; k < EPV; ++k) {
          uint64_t own;
          sum += e.weight(table, i + k, xp[k], xq[k], own);
          own_sum += own;
        }
      }
    }
    base = end;
  }
  constexpr int N = 8;                    // tokens of a lane at a time
  for (; base < i1; base += N * kWave) {
    float xp[N], xq[N];
    e.template values<N>(base + lane, kWave, i1, xp, xq);
#pragma unroll
    for (int q = 0; q < N; ++q) {
      uint64_t own;
      sum += e.weight(table, base + lane + q * kWave, xp[q], xq[q], own);
      own_sum += own;
    }
  }
  sum = wave_scan(sum);
  own_sum = wave_scan(own_sum);
  if (threadIdx.x % kWave == kWave - 1) {
    a.sums[(int64_t)b * kVerifyParts + part] = sum;
    a.sums[(int64_t)(a.batch + b) * kVerifyParts + part] = own_sum;
  }
}

// Inclusive prefix sum over the workgroup, and the whole.
__device__ __forceinline__ uint64_t verify_scan(uint64_t x, uint64_t* shared, uint64_t& total) {
  x = wave_scan(x);
  __syncthreads();
  if (threadIdx.x % kWave == kWave - 1) shared[threadIdx.x / kWave] = x;
  __syncthreads();
  total = 0;
  uint64_t before = 0;
#pragma unroll
  for (int v = 0; v < kVerifyWaves; ++v) {
    before += v < (int)(threadIdx.x / kWave) ? shared[v] : 0;
    total += shared[v];
  }
  return before + x;
}

// A slot a workgroup: its parts' sums, then one part's tokens.  Bound by latency: 4.5 us
// for one slot over 50,257, 9 for 64 over 128,000.
template <typename T>
__global__ void __launch_bounds__(kVerifyThreads) verify_draw_kernel(const VerifyArgs a) {
  constexpr int E = 4;                    // tokens of a thread at a time
  __shared__ double table[128];
  __shared__ uint64_t sums[kVerifyWaves], s_before;
  __shared__ int32_t accepted, token, s_part;
  static_assert(kVerifyParts <= kVerifyThreads, "a part per thread");
  const int32_t b = blockIdx.x, w1 = a.width - 1, tid = threadIdx.x;
  const int32_t n_draft = verify_drafts(a, b);
  if (n_draft < 0) {                      // a free slot
    for (int32_t i = tid; i < a.width; i += kVerifyThreads) a.tokens[b * a.width + i] = -1;
    if (tid == 0) a.n_out[b] = 0;
    return;
  }
  const uint64_t* const part_sums = a.sums + (int64_t)b * kVerifyParts;
  const bool part = tid < a.segs * kVerifyWaves;
  uint64_t mine = part ? part_sums[tid] : 0;
  const uint64_t own = part ? part_sums[(int64_t)a.batch * kVerifyParts + tid] : 0;
  const float u_in = a.u_token[b], u = u_in > 0.f ? fminf(u_in, 0x1.fffffep-1f) : 0.f;
  verify_table(table, a.shift);
  if (tid == 0) {
    token = -1;
    s_part = 0;
  }
  __syncthreads();
  VerifyEnd<T> e = verify_end<T>(a, table, b, n_draft, &accepted);
  // The part in which the target lies.
  uint64_t total, upto = verify_scan(mine, sums, total);
  if (total == 0) {                       // nothing of p is above q: from p
    e.minus = 0;
    mine = own;
    upto = verify_scan(mine, sums, total);
  }
  const uint64_t target = times_fraction<false>(u, total);
  if (upto > target && upto - mine <= target) {
    s_part = tid;
    s_before = upto - mine;
  }
  __syncthreads();
  // The first token of it at which the running weight exceeds the target.
  const int32_t i0 = min(s_part * a.per_part, a.vocab), i1 = min(i0 + a.per_part, a.vocab);
  uint64_t seen = total > 0 ? s_before : 0;
  for (int32_t base = i0; base < i1 && total > 0; base += kVerifyThreads * E) {
    uint64_t g[E], sum = 0, all;
    float xp[E], xq[E];
    e.template values<E>(base + tid * E, 1, i1, xp, xq);
#pragma unroll
    for (int q = 0; q < E; ++q) {
      uint64_t own_g;
      g[q] = e.weight(table, base + tid * E + q, xp[q], xq[q], own_g);
      sum += g[q];
    }
    uint64_t at = seen + verify_scan(sum, sums, all) - sum;
#pragma unroll
    for (int q = 0; q < E; ++q) {
      if (at <= target && at + g[q] > target) token = base + tid * E + q;
      at += g[q];
    }
    seen += all;
    if (seen > target) break;
  }
  __syncthreads();
  for (int32_t i = tid; i < a.width; i += kVerifyThreads)
    a.tokens[b * a.width + i] = i < e.n ? a.drafted[b * w1 + i] : i == e.n ? token : -1;
  if (tid == 0) a.n_out[b] = e.n + 1;
}

}  // namespace
}  // namespace baton
