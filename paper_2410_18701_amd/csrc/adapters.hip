// Host side of the low-rank adapters: argument checks, the rows sorted by
// adapter, the two launches.  The C ABI is documented in include/baton.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "baton.h"
#include "adapter_gemm.hpp"

static_assert(BATON_ADAPTER_MAX_RANK == baton::kAdapterMaxRank, "staged rank");
static_assert(BATON_GEMM_MAX_ROWS == baton::kAdapterMaxRows, "row list");

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace

extern "C" {

size_t baton_linear_adapters_workspace_bytes(int32_t rows, int32_t n_parts, int32_t max_rank) {
  if (rows < 1 || n_parts < 1 || max_rank < 1) return 0;
  return (size_t)rows * n_parts * max_rank * sizeof(float);
}

baton_status baton_linear_adapters(int32_t dtype, const void* x, const baton_adapter* adapters, int32_t n_adapters,
                                   const int32_t* row_adapter, void* y, int32_t rows, int32_t out_dim,
                                   int32_t in_dim, const int32_t* part_dims, int32_t n_parts, int32_t accumulate,
                                   void* ws, size_t ws_bytes, hipStream_t stream) {
  using namespace baton;
  if (!x || !y || !row_adapter || n_adapters < 0 || (n_adapters > 0 && !adapters)) return BATON_EINVAL;
  if (rows < 1 || rows > BATON_GEMM_MAX_ROWS || out_dim < 8 || out_dim % 8 || in_dim < 8 || in_dim % 8 ||
      in_dim > (1 << 24) || out_dim > (1 << 24) || (accumulate != 0 && accumulate != 1))
    return BATON_EINVAL;
  if (n_parts < 1 || n_parts > BATON_ADAPTER_MAX_PARTS || (n_parts > 1 && !part_dims)) return BATON_EINVAL;
  if (dtype != BATON_BF16) return BATON_EDTYPE;
  if (!aligned16(x) || !aligned16(y)) return BATON_EINVAL;
  AdapterArgs a;
  std::memset(&a, 0, sizeof(a));
  int64_t end = 0;
  for (int32_t p = 0; p < n_parts; ++p) {
    const int32_t d = part_dims ? part_dims[p] : out_dim;
    if (d < 8 || d % 8 || d > out_dim) return BATON_EINVAL;
    end += d;
    a.part_end[p] = (int32_t)end;
  }
  if (end != out_dim) return BATON_EINVAL;
  int32_t used_rank = 0;
  for (int32_t r = 0; r < rows; ++r) {
    const int32_t i = row_adapter[r];
    if (i < -1 || i >= n_adapters) return BATON_EINVAL;
    if (i < 0) continue;
    const baton_adapter& d = adapters[i];
    if (!d.a || !d.b || !aligned16(d.a) || !aligned16(d.b) || d.rank < 8 || d.rank % 8 ||
        d.rank > BATON_ADAPTER_MAX_RANK || !std::isfinite(d.scale))
      return BATON_EINVAL;
    used_rank = std::max(used_rank, d.rank);
  }
  // Rows sorted by adapter, those without one first (skipped when they keep y).
  uint64_t key[BATON_GEMM_MAX_ROWS];   // (adapter + 1, row)
  int32_t n_order = 0;
  for (int32_t r = 0; r < rows; ++r)
    if (row_adapter[r] >= 0 || !accumulate) key[n_order++] = (uint64_t)(row_adapter[r] + 1) << 32 | (uint64_t)r;
  if (n_order == 0) return BATON_OK;
  std::sort(key, key + n_order);
  const size_t per_split = baton_linear_adapters_workspace_bytes(rows, n_parts, used_rank);
  if (used_rank > 0 && (!ws || !aligned16(ws) || ws_bytes < per_split)) return BATON_EINVAL;

  a.x = static_cast<const uint16_t*>(x);
  a.y = static_cast<uint16_t*>(y);
  a.h = static_cast<float*>(ws);
  a.K = in_dim;
  a.N = out_dim;
  a.rows = rows;
  a.hs = n_parts * used_rank;
  a.parts = n_parts;
  a.accumulate = accumulate;
  const int32_t steps = (in_dim + 31) / 32;
  for (int32_t at = 0; at < n_order;) {
    // the next groups, up to a launch's number of them
    int64_t units = 0;           // workgroups of the down launch for each split
    int32_t max_rank = 0, lds_rows = 0;
    a.n_groups = 0;
    while (at < n_order && a.n_groups < kAdapterGroups) {
      const int64_t i = (int64_t)(key[at] >> 32) - 1;
      AdapterGroup& g = a.g[a.n_groups++];
      g.a = i < 0 ? nullptr : static_cast<const uint16_t*>(adapters[i].a);
      g.b = i < 0 ? nullptr : static_cast<const uint16_t*>(adapters[i].b);
      g.rank = (int16_t)(i < 0 ? 0 : adapters[i].rank);
      g.scale = i < 0 ? 0.f : adapters[i].scale;
      g.begin = (int16_t)at;
      const int32_t from = at;
      for (; at < n_order && (int64_t)(key[at] >> 32) - 1 == i; ++at) a.row[at] = (uint16_t)key[at];
      const int32_t rbs = (at - from + kAdapterRows - 1) / kAdapterRows;
      g.up_end = rbs;            // row blocks; made into workgroups below
      max_rank = std::max(max_rank, (int32_t)g.rank);
      lds_rows = std::max(lds_rows, std::min((at - from + 15) / 16 * 16, (int32_t)kAdapterRows));
      units += (int64_t)rbs * ((n_parts * g.rank + 15) / 16);
    }
    a.end = (int16_t)at;
    const dim3 block(kWave * kAdapterWaves);
    int32_t small = 0;     // workgroups of the single launch for each row block
    for (int32_t p = 0; p < n_parts; ++p)
      small += (a.part_end[p] - (p > 0 ? a.part_end[p - 1] : 0) + kAdapterSmallCols - 1) / kAdapterSmallCols;
    // One launch while a part's A is up to 128 KB, which each workgroup reads, and the
    // workgroups make one round.  us by both, calls from Python: one row of rank 16,
    // 4096 to 4096 8.7 / 10.4, 11008 to 4096 16.2 / 10.1; 32 adapters of rank 8, 2048 to
    // 2048 8.0 / 11.1; of rank 16, 4096 to 4096: 8 9.3 / 10.0, 32 (256 workgroups) 10.8 /
    // 11.2, 64 19.2 / 12.0.
    if (max_rank <= kAdapterSmallRank && lds_rows <= kAdapterSmallRows && (int64_t)max_rank * in_dim <= 1 << 16 &&
        (int64_t)a.n_groups * small <= 256) {
      for (int32_t i = 0; i < a.n_groups; ++i) a.g[i].up_end = (i + 1) * small;
      const dim3 grid((unsigned)(a.n_groups * small)), wide(kWave * kAdapterSmallWaves);
      if (max_rank <= 16) hipLaunchKernelGGL(adapter_small_kernel<1>, grid, wide, 0, stream, a);
      else hipLaunchKernelGGL(adapter_small_kernel<2>, grid, wide, 0, stream, a);
      if (hipGetLastError() != hipSuccess) return BATON_EHIP;
      continue;
    }
    // Ranges of k: 1024 workgroups in all or a few more, at most one range for every 1024
    // columns begun -- eight steps of 32 (the loads a wave has in flight at once) for each
    // of four waves at a multiple of 1024, five at least past the first.  us of both
    // launches, 256 rows of 40 adapters of rank 64, 4096 to 2 x 11008: with 512 workgroups 53.7, with
    // 1024 50.2; 64 rows of 24 of rank 32, 4096 to 12288: 15.3, with four steps a wave 16.3.
    const int64_t fit = per_split ? (int64_t)(ws_bytes / per_split) : 1;
    int64_t splits = units > 0 ? (1024 + units - 1) / units : 1;
    splits = std::max<int64_t>(1, std::min({splits, (int64_t)(steps + 31) / 32, fit, (int64_t)64}));
    a.kt = (int32_t)((steps + splits - 1) / splits);
    a.splits = (steps + a.kt - 1) / a.kt;
    // Columns of y per wave: about 4096 waves in all, 32 to 128 columns (the first of
    // those cases with up to 256 49.2, 128 44.4, 64 44.6).
    int64_t rbs = 0;
    for (int32_t i = 0; i < a.n_groups; ++i) rbs += a.g[i].up_end;
    a.cols = (int32_t)std::max<int64_t>(32, std::min<int64_t>(128, (rbs * out_dim / 4096 + 31) / 32 * 32));
    int32_t per_rb = 0;
    const int32_t wide = kAdapterWaves * a.cols;
    for (int32_t p = 0; p < n_parts; ++p)
      per_rb += (a.part_end[p] - (p > 0 ? a.part_end[p - 1] : 0) + wide - 1) / wide;
    int64_t down = 0, up = 0;
    for (int32_t i = 0; i < a.n_groups; ++i) {
      AdapterGroup& g = a.g[i];
      const int64_t rb = g.up_end;
      down += rb * ((n_parts * g.rank + 15) / 16) * a.splits;
      up += rb * per_rb;
      g.down_end = (int32_t)down;
      g.up_end = (int32_t)up;
    }
    if (down > 0) hipLaunchKernelGGL(adapter_down_kernel, dim3((unsigned)down), block, 0, stream, a);
    auto launch_up = [&](auto kernel, int32_t row) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)up), block, (size_t)lds_rows * row * kAdapterParts * sizeof(uint16_t), stream, a, lds_rows);
    };
    if (max_rank <= 32) launch_up(adapter_up_kernel<1>, adapter_row<1>());
    else if (max_rank <= 64) launch_up(adapter_up_kernel<2>, adapter_row<2>());
    else launch_up(adapter_up_kernel<4>, adapter_row<4>());
    if (hipGetLastError() != hipSuccess) return BATON_EHIP;
  }
  return BATON_OK;
}

}  // extern "C"
