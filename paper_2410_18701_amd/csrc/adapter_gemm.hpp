// Low-rank adapters of many requests beside a shared projection:
//   y[r] (+)= scale_g * (x[r] . A_g^T) . B_g^T,  g the adapter of row r,
// in two launches over the rows sorted by adapter (in one where both are short,
// adapter_small_kernel).  What bounds both is reading
// the adapters' weights once (and, for a few small ones, the launches' latency):
// a batch of 64 rows over 24 adapters does 1 to 3 flops per byte.
//  * down: h = x . A^T, [rows][parts * rank].  A workgroup takes 16 of an
//    adapter's rows of A, up to 64 of its batch rows and a range of k; its four
//    waves divide the range and add through LDS.  Ranges are taken so that
//    the launch has a few waves per SIMD whatever the number of adapters; each
//    range's sums go to the workspace in fp32.
//  * up: the ranges' sums are added in order, scaled, and split into three bf16
//    parts, which keep all 24 bits, staged in LDS; then 16 x 16 tiles of
//    y = h . B^T, every wave its own columns, the next 32 columns of B and of y's
//    first rows on their way meanwhile.  The second and third part cost a matrix
//    operation each on operands of B that are in registers (up to 0.1 us of the times
//    below); with one part h would be rounded to 8 bits, with two to 16, which still
//    turns one rounding of y in some 250 the other way.
// Sums are fp32 in a fixed order: the same call gives the same bits.
// us down / up: 64 rows of 24 adapters of rank 32, 4096 to 3 parts of 4096 (35 MB)
// 7.0 / 8.3; 240 rows of 40 of rank 64, 4096 to 2 of 11008 (177 MB with y) 15.0 / 32.3.
#pragma once

#include <type_traits>

#include "common.hpp"

namespace baton {
namespace {

typedef __bf16 ad_bf16x8 __attribute__((ext_vector_type(8)));
typedef float ad_f32x4 __attribute__((ext_vector_type(4)));

constexpr int kAdapterWaves = 4;
constexpr int kAdapterRows = 64;      // batch rows a workgroup takes at most
constexpr int kAdapterMaxRank = 128;  // == BATON_ADAPTER_MAX_RANK
constexpr int kAdapterGroups = 96;    // adapters per launch (the arguments are 4 KB at most)
constexpr int kAdapterMaxRows = 256;  // == BATON_GEMM_MAX_ROWS
constexpr int kAdapterParts = 3;      // bf16 parts of x . A^T

// The rows of one adapter: places [begin, next group's begin) of the sorted rows.
struct AdapterGroup {
  const uint16_t* a;    // [parts * rank][K]; null: rows without an adapter
  const uint16_t* b;    // [N][rank]
  float scale;
  int16_t rank, begin;
  int32_t down_end, up_end;   // workgroups up to this group's last one, of each launch
};

struct AdapterArgs {
  const uint16_t* x;    // [rows][K]
  uint16_t* y;          // [rows][N]
  float* h;             // [splits][rows][hs]
  int32_t K, N, rows, hs, parts, splits, n_groups, accumulate;
  int32_t kt;           // 32-wide steps of k per split
  int32_t cols;         // columns of y per wave, a multiple of 32
  int32_t part_end[4];  // columns of y up to the end of each part
  AdapterGroup g[kAdapterGroups];
  int16_t end;          // sorted rows of this launch end here
  uint16_t row[kAdapterMaxRows];   // sorted place -> batch row
};
static_assert(sizeof(AdapterArgs) <= 4096, "kernel arguments");

// f in three bf16 parts that sum to it within 2^-23 of it.  Each is what the one before
// left, cut off (the last rounded) with its last bit set, so that all have f's sign and
// none is 0 where f is not: times an infinity of B all are the same infinity, and times 0
// all are 0 (numbers under 2^-80, whose last part is too small for bf16, lose it).  An
// infinity or a NaN (a product's, so a quiet one) is every part.
__device__ __forceinline__ void adapter_split(float f, uint32_t (&part)[kAdapterParts]) {
  const uint32_t b = __float_as_uint(f);
  part[0] = b >> 16;
  const uint32_t r = __float_as_uint(__uint_as_float(b | 1u) - __uint_as_float(b & 0xFFFF0000u));
  part[1] = r >> 16;
  part[2] = f32_to_bf16_rne(__uint_as_float(r | 1u) - __uint_as_float(r & 0xFFFF0000u));
  if ((b & 0x7F800000u) == 0x7F800000u) part[1] = part[2] = part[0];
}

// The parts of four elements v, staged one below the other `plane` elements apart.
__device__ __forceinline__ void adapter_stage(const ad_f32x4& v, uint16_t* at, int32_t plane) {
  uint32_t part[4][kAdapterParts];
#pragma unroll
  for (int e = 0; e < 4; ++e) adapter_split(v[e], part[e]);
#pragma unroll
  for (int q = 0; q < kAdapterParts; ++q)
    *reinterpret_cast<uint2*>(at + q * plane) =
        make_uint2(part[0][q] | part[1][q] << 16, part[2][q] | part[3][q] << 16);
}

__device__ __forceinline__ ad_bf16x8 ad_vec(const u32x4& w) { return __builtin_bit_cast(ad_bf16x8, w); }

// The group of workgroup i of a launch.
template <bool UP>
__device__ __forceinline__ int adapter_group(const AdapterArgs& a, int32_t i) {
  int lo = 0, hi = a.n_groups - 1;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (i < (UP ? a.g[mid].up_end : a.g[mid].down_end)) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

__global__ void __launch_bounds__(kWave * kAdapterWaves) adapter_down_kernel(const AdapterArgs a) {
  __shared__ ad_f32x4 part[kAdapterWaves][kAdapterRows / 16][kWave];
  const int gi = adapter_group<false>(a, blockIdx.x);
  const AdapterGroup& g = a.g[gi];
  const int local = (int)blockIdx.x - (gi > 0 ? a.g[gi - 1].down_end : 0);
  const int n_r = a.parts * g.rank, tiles = (n_r + 15) / 16;
  const int tile = local % tiles, rest = local / tiles, split = rest % a.splits, rb = rest / a.splits;
  const int first = g.begin + rb * kAdapterRows;
  const int n = min((gi + 1 < a.n_groups ? a.g[gi + 1].begin : a.end) - first, kAdapterRows);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int g4 = lane / 16, c16 = lane % 16;
  const int n_rt = (n + 15) / 16;      // tiles of batch rows
  // this wave's steps of k
  const int per = (a.kt + kAdapterWaves - 1) / kAdapterWaves;
  const int s0 = split * a.kt + w * per, s1 = min(min(s0 + per, (split + 1) * a.kt), (a.K + 31) / 32);
  // rows past the last one read it again; their sums are not stored
  const uint16_t* ar = g.a + (int64_t)min(tile * 16 + c16, n_r - 1) * a.K + 8 * g4;
  const uint16_t* xr[kAdapterRows / 16];
#pragma unroll
  for (int t = 0; t < kAdapterRows / 16; ++t)
    xr[t] = a.x + (int64_t)a.row[first + min(16 * t + c16, n - 1)] * a.K + 8 * g4;
  ad_f32x4 acc[kAdapterRows / 16];
#pragma unroll
  for (int t = 0; t < kAdapterRows / 16; ++t) acc[t] = ad_f32x4{0.f, 0.f, 0.f, 0.f};
  const u32x4 zero = {0, 0, 0, 0};
  auto run = [&](auto nt_tag) {
    constexpr int NT = decltype(nt_tag)::value, U = NT == 1 ? 8 : NT == 2 ? 4 : 2;   // U steps' loads in flight
    for (int s = s0; s < s1; s += U) {
      u32x4 aw[U], xw[U][NT];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int k = 32 * (s + i);
        const bool in = s + i < s1 && k + 8 * g4 < a.K;   // K is a multiple of 8
        aw[i] = in ? *reinterpret_cast<const u32x4*>(ar + k) : zero;
#pragma unroll
        for (int t = 0; t < NT; ++t) xw[i][t] = in ? *reinterpret_cast<const u32x4*>(xr[t] + k) : zero;
      }
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t)
          acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ad_vec(aw[i]), ad_vec(xw[i][t]), acc[t], 0, 0, 0);
    }
  };
  if (n_rt == 1) run(std::integral_constant<int, 1>{});
  else if (n_rt == 2) run(std::integral_constant<int, 2>{});
  else run(std::integral_constant<int, 4>{});
#pragma unroll
  for (int t = 0; t < kAdapterRows / 16; ++t)
    if (t < n_rt) part[w][t][lane] = acc[t];
  __syncthreads();
  // wave t adds tile t's sums: lane l has rows 4 (l / 16) .. + 3 of A for batch row l % 16
  if (w >= n_rt) return;
  ad_f32x4 sum = part[0][w][lane];
#pragma unroll
  for (int v = 1; v < kAdapterWaves; ++v) sum += part[v][w][lane];
  const int r = 16 * w + c16, j = tile * 16 + 4 * g4;
  if (r < n && j < n_r)     // n_r is a multiple of 8
    *reinterpret_cast<ad_f32x4*>(a.h + ((int64_t)split * a.rows + first + r) * a.hs + j) = sum;
}

// Workgroup `local` of a group's row blocks rb x columns, taken part by part, `wide` at
// a time: its part p and first column c0; c_end is the part's end.
__device__ __forceinline__ void adapter_columns(const AdapterArgs& a, int local, int wide, int& rb, int& p, int& c0,
                                                int& c_end) {
  int per_rb = 0;
  for (int q = 0; q < a.parts; ++q) per_rb += (a.part_end[q] - (q > 0 ? a.part_end[q - 1] : 0) + wide - 1) / wide;
  rb = local / per_rb;
  int chunk = local - rb * per_rb;
  for (p = 0;; ++p) {
    const int b0 = p > 0 ? a.part_end[p - 1] : 0, cnt = (a.part_end[p] - b0 + wide - 1) / wide;
    c0 = b0 + chunk * wide;
    c_end = a.part_end[p];
    if (chunk < cnt || p == a.parts - 1) return;
    chunk -= cnt;
  }
}

// Elements between two staged rows of h, of NKK 32-wide steps: padded by 16 bytes.
template <int NKK>
constexpr int adapter_row() { return 32 * NKK + 8; }

// Ranks up to 32 * NKK; the parts of `lds_rows` rows of h (whole tiles of 16) are
// staged in the launch's dynamic LDS.
template <int NKK>
__global__ void __launch_bounds__(kWave * kAdapterWaves) adapter_up_kernel(const AdapterArgs a, const int32_t lds_rows) {
  constexpr int ROW = adapter_row<NKK>();
  extern __shared__ __attribute__((aligned(16))) uint16_t hs[];
  const int32_t plane = lds_rows * ROW;
  const int gi = adapter_group<true>(a, blockIdx.x);
  const AdapterGroup& g = a.g[gi];
  const int local = (int)blockIdx.x - (gi > 0 ? a.g[gi - 1].up_end : 0);
  int rb, p, c0, c_end;
  adapter_columns(a, local, kAdapterWaves * a.cols, rb, p, c0, c_end);
  const int first = g.begin + rb * kAdapterRows;
  const int n = min((gi + 1 < a.n_groups ? a.g[gi + 1].begin : a.end) - first, kAdapterRows);
  const int rank = g.rank, n_rt = (n + 15) / 16;
  const int tid = threadIdx.x, lane = tid % kWave, g4 = lane / 16, c16 = lane % 16;
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const u32x4 zero = {0, 0, 0, 0};
  const int w0 = c0 + w * a.cols, w1 = min(w0 + a.cols, c_end);
  // B of 32 columns: row 4 g + r of tile j is column 8 g + 4 j + r, so a lane ends
  // with 8 neighbouring columns of its batch row.  Columns past the last read it again.
  auto load_b = [&](int c, u32x4 (&bw)[2][NKK]) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int col = min(c + 8 * (c16 / 4) + 4 * j + c16 % 4, c_end - 1);
      const uint16_t* br = g.b + (int64_t)col * rank + 8 * g4;
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk)
        bw[j][kk] = 32 * kk + 8 * g4 < rank ? *reinterpret_cast<const u32x4*>(br + 32 * kk) : zero;
    }
  };
  // y of the first tile of batch rows at those columns
  const int64_t y_row = (int64_t)a.row[first + min(c16, n - 1)] * a.N + 8 * g4;
  auto load_y = [&](int c) {
    return a.accumulate && c16 < n && c + 8 * g4 < w1 ? *reinterpret_cast<const u32x4*>(a.y + y_row + c) : zero;
  };
  u32x4 bw[2][NKK], old = zero;
  if (w0 < w1) {
    load_b(w0, bw);
    old = load_y(w0);
  }
  // h of the part, four elements per thread and step; zeros up to whole operands
  constexpr int kQuads = NKK * 8;
  for (int i = tid; i < n_rt * 16 * kQuads; i += kWave * kAdapterWaves) {
    const int r = i / kQuads, j = 4 * (i % kQuads);
    ad_f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (r < n && j < rank) {
      const float* src = a.h + (int64_t)(first + r) * a.hs + p * rank + j;
#pragma unroll 4
      for (int s = 0; s < a.splits; ++s) v += *reinterpret_cast<const ad_f32x4*>(src + (int64_t)s * a.rows * a.hs);
    }
    adapter_stage(v * g.scale, hs + r * ROW + j, plane);
  }
  __syncthreads();
  for (int c = w0; c < w1; c += 32) {
    u32x4 next[2][NKK], next_old = zero;
    if (c + 32 < w1) {      // on their way while these columns are computed
      load_b(c + 32, next);
      next_old = load_y(c + 32);
    }
    for (int t = 0; t < n_rt; ++t) {
      const int r = 16 * t + c16;
      const bool ok = r < n && c + 8 * g4 < w1;     // w1 is a multiple of 8
      u32x4* yp = reinterpret_cast<u32x4*>(a.y + (int64_t)a.row[first + min(r, n - 1)] * a.N + c + 8 * g4);
      if (t > 0) old = ok && a.accumulate ? *yp : zero;
      ad_f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) {
#pragma unroll
        for (int q = kAdapterParts - 1; q >= 0; --q) {
          const ad_bf16x8 h = ad_vec(*reinterpret_cast<const u32x4*>(hs + q * plane + r * ROW + 32 * kk + 8 * g4));
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ad_vec(bw[j][kk]), h, acc[j], 0, 0, 0);
        }
      }
      u32x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        o[e] = f32_to_bf16_rne(bf16_lo(old[e]) + acc[e / 2][2 * (e % 2)]) |
               f32_to_bf16_rne(bf16_hi(old[e]) + acc[e / 2][2 * (e % 2) + 1]) << 16;
      if (ok) *yp = o;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) bw[j][kk] = next[j][kk];
    old = next_old;
  }
}

// Both products in one launch, for calls of few small adapters, where the launches
// are the time: up to 16 rows and rank 32 a group.  Every workgroup forms the whole h
// of its part -- its 16 waves divide k and add through LDS -- for 512 columns of y, so
// A is read from the caches once for each 512 columns.
constexpr int kAdapterSmallWaves = 16, kAdapterSmallRank = 32, kAdapterSmallRows = 16;
constexpr int kAdapterSmallCols = 32 * kAdapterSmallWaves;

// AT = 16-row tiles of A: ranks up to 16 or 32.
template <int AT>
__global__ void __launch_bounds__(kWave * kAdapterSmallWaves) adapter_small_kernel(const AdapterArgs a) {
  constexpr int NW = kAdapterSmallWaves, ROW = adapter_row<1>(), U = 8 / AT;   // U steps' loads in flight
  __shared__ ad_f32x4 part[NW][AT][kWave];
  __shared__ __attribute__((aligned(16))) uint16_t hs[kAdapterParts][16 * ROW];
  const int gi = adapter_group<true>(a, blockIdx.x);
  const AdapterGroup& g = a.g[gi];
  const int local = (int)blockIdx.x - (gi > 0 ? a.g[gi - 1].up_end : 0);
  int rb, p, c0, c_end;
  adapter_columns(a, local, kAdapterSmallCols, rb, p, c0, c_end);   // rb = 0
  const int first = g.begin, n = (gi + 1 < a.n_groups ? a.g[gi + 1].begin : a.end) - first;
  const int rank = g.rank;
  const int tid = threadIdx.x, lane = tid % kWave, g4 = lane / 16, c16 = lane % 16;
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const u32x4 zero = {0, 0, 0, 0};
  const int row = a.row[first + min(c16, n - 1)];     // rows past the last read it again
  // this wave's 32 columns of B and y, on their way while h is formed
  const int c = c0 + 32 * w;
  const bool ok = c16 < n && c + 8 * g4 < c_end;
  u32x4* const yp = reinterpret_cast<u32x4*>(a.y + (int64_t)row * a.N + c + 8 * g4);
  u32x4 bw[2], old = zero;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int col = min(c + 8 * (c16 / 4) + 4 * j + c16 % 4, c_end - 1);
    bw[j] = 8 * g4 < rank ? *reinterpret_cast<const u32x4*>(g.b + (int64_t)col * rank + 8 * g4) : zero;
  }
  if (ok && a.accumulate) old = *yp;
  const int steps = rank > 0 ? (a.K + 31) / 32 : 0, per = (steps + NW - 1) / NW;
  const int s0 = w * per, s1 = min(s0 + per, steps);
  const uint16_t* xr = a.x + (int64_t)row * a.K + 8 * g4;
  const uint16_t* ar[AT];
#pragma unroll
  for (int t = 0; t < AT; ++t)
    ar[t] = g.a + ((int64_t)p * rank + max(min(16 * t + c16, rank - 1), 0)) * a.K + 8 * g4;
  ad_f32x4 acc[AT];
#pragma unroll
  for (int t = 0; t < AT; ++t) acc[t] = ad_f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s = s0; s < s1; s += U) {
    u32x4 xw[U], aw[U][AT];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int k = 32 * (s + i);
      const bool in = s + i < s1 && k + 8 * g4 < a.K;
      xw[i] = in ? *reinterpret_cast<const u32x4*>(xr + k) : zero;
#pragma unroll
      for (int t = 0; t < AT; ++t) aw[i][t] = in ? *reinterpret_cast<const u32x4*>(ar[t] + k) : zero;
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int t = 0; t < AT; ++t)
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ad_vec(aw[i][t]), ad_vec(xw[i]), acc[t], 0, 0, 0);
  }
#pragma unroll
  for (int t = 0; t < AT; ++t) part[w][t][lane] = acc[t];
  __syncthreads();
  if (w < 2) {     // wave t: 4 ranks from 16 t + 4 (l / 16) on of batch row l % 16
    ad_f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (w < AT) {
#pragma unroll
      for (int q = 0; q < NW; ++q) v += part[q][w][lane];
    }
    const int j = 16 * w + 4 * g4;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = c16 < n && j + e < rank ? v[e] * g.scale : 0.f;
    adapter_stage(v, hs[0] + c16 * ROW + j, 16 * ROW);
  }
  __syncthreads();
  ad_bf16x8 h[kAdapterParts];
#pragma unroll
  for (int q = 0; q < kAdapterParts; ++q) h[q] = ad_vec(*reinterpret_cast<const u32x4*>(hs[q] + c16 * ROW + 8 * g4));
  u32x4 o;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    ad_f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = kAdapterParts - 1; q >= 0; --q) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ad_vec(bw[j]), h[q], d, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 2; ++e)
      o[2 * j + e] = f32_to_bf16_rne(bf16_lo(old[2 * j + e]) + d[2 * e]) |
                     f32_to_bf16_rne(bf16_hi(old[2 * j + e]) + d[2 * e + 1]) << 16;
  }
  if (ok) *yp = o;
}

}  // namespace
}  // namespace baton
