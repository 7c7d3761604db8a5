// A KV cache in pages: its layout, the step that keeps its tables, and copies of
// whole queries into pages and out of them.
//
// A page holds `page` tokens (32, 64, 128 or 256) of one layer and kv-head, as blocks
// of 32 tokens in the order in which the matrix cores take them, so that attention
// loads them straight into registers, 1 KB of consecutive bytes per instruction:
//  * keys: token t of a block is row 4 (t / 8) + t % 4 of tile (t / 4) % 2 (the rows
//    whose scores lane group g of the result holds are then tokens 8 g .. 8 g + 7).  A
//    tile is a run of 1 KB chunks of 64 bytes of every row, lane l of a chunk holding
//    16 bytes: row l % 16, bytes 16 (l / 16) .. of the chunk.
//  * values, transposed: 16 columns of head_dim a chunk, lane l holding column l % 16
//    of the tokens 8 (l / 16) ..: eight of them in bf16, four in fp32, where a chunk
//    per column slice and tile holds the tile's.
#pragma once

#include "wave_scan.hpp"

namespace baton {

constexpr int kPagedBlock = 32;          // tokens per block
constexpr int kPagedMaxNew = 16;         // == BATON_PAGED_MAX_WIDTH
// Workgroups of an attention launch, about, and blocks per work item, at least.  A compute
// unit holds two workgroups of bf16 at head_dim 128 and of fp32 at 64 (512 on the GPU), three
// of bf16 at 64, one of fp32 at 128; the step, which makes the items, knows neither type nor
// head_dim, and the numbers are those that served the first best.
//  * Up to 16 rows per head, 2048: four rounds even out lengths, and every item costs its
//    start and its part of the second launch.  With 1024, 2048 and 4096 a step of 32 slots
//    of up to 2,048 tokens (32/32 heads) took 112, 104 and 103 us, two layers of 64 slots of
//    up to 8,192 (64/8 heads) 400, 401 and 413.
//  * More rows, 512, for all of a call's items if any slot has more: an item's start (its
//    loads into LDS, its merge) is longer.  32 slots of very different lengths up to 32,768
//    (32/4 heads) with four drafts each: 53.3 us with 448, 51.7 with 512, 59.4 with 640 and
//    55.8 with 1024, by how full the last round of workgroups is.
//  * 8 blocks, two a wave.  With 4, 8 and 16 a step of four slots of up to 128 tokens took
//    13.6, 11.3 and 10.9 us, one of seven in fp32 with a window of 333 13.3, 13.8 and 15.9.
constexpr int kPagedItems = 2048;
constexpr int kPagedRowItems = 512;      // more than 16 rows
constexpr int kPagedMinBlocks = 8;

// A work item, one of a slot's `parts`: visible blocks v0 .. v1 - 1 of slot b.
// Visible block v is the query's block v (v < sink) or v + skip.
struct PagedItem {
  int32_t b, v0, v1, parts;
  int32_t len, n_new, sink, skip;
};

// The library's part of a paged cache's device memory, in 32-bit words: header, four
// numbers per slot, the stack of free pages, the step's work items.
struct PagedState {
  int64_t covered, released, n_new, first, stack, items, words;
};
enum { kFreePages = 0, kNumItems = 1, kPagedHeader = 16 };

__host__ __device__ inline int32_t paged_max_items(int32_t batch, int32_t n_kv_heads, int32_t max_pages, int32_t page) {
  const int64_t per_slot = ((int64_t)max_pages * (page / kPagedBlock) + kPagedMinBlocks - 1) / kPagedMinBlocks;
  const int64_t most = kPagedItems / n_kv_heads + 1 + batch;
  return (int32_t)(per_slot * batch < most ? per_slot * batch : most);
}

__host__ __device__ inline PagedState paged_state(int32_t batch, int32_t n_pages, int32_t max_items) {
  PagedState s;
  s.covered = kPagedHeader;             // blocks of pages the table has handed out
  s.released = s.covered + batch;       // where those the window has left behind end
  s.n_new = s.released + batch;         // the step's new tokens
  s.first = s.n_new + batch;            // a slot's first work item, batch + 1
  s.stack = s.first + batch + 1;
  s.items = (s.stack + n_pages + 7) / 8 * 8;
  s.words = s.items + 8 * (int64_t)max_items;
  return s;
}

struct PagedStepArgs {
  int32_t* table;
  int32_t* lens;
  int32_t* state;
  const int32_t* keep;      // null: 0
  const int32_t* n_new;
  int32_t* slot_map;        // null: not wanted
  int32_t* missing;         // null: not wanted
  int64_t map_ld;
  int32_t batch, max_pages, page_shift, window, sinks, n_kv_heads, group, width;
  PagedState at;
};

constexpr int kStepThreads = 512;        // == BATON_MAX_BATCH: a thread per slot

// Exclusive prefix sum over the workgroup's threads, and the whole.  `sums` alternate, so
// that one barrier does.
__device__ __forceinline__ uint64_t step_scan(uint64_t x, uint64_t* sums, uint64_t& total) {
  const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
  const uint64_t y = wave_scan(x);
  if (lane == kWave - 1) sums[w] = y;
  __syncthreads();
  uint64_t before = 0;
  total = 0;
#pragma unroll
  for (int v = 0; v < kStepThreads / kWave; ++v) {
    before += v < w ? sums[v] : 0;
    total += sums[v];
  }
  return before + y - x;
}

// The slot whose range of an exclusive prefix sum holds k (of empty ones none).
__device__ __forceinline__ int32_t step_find(const int32_t* first, int32_t n, int32_t k) {
  int32_t lo = 0, hi = n;               // first[lo] <= k < first[hi]
  while (hi - lo > 1) {
    const int32_t mid = (lo + hi) / 2;
    if (first[mid] <= k) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Ends a step and begins the next: lengths, pages given back and taken, places of the
// new tokens, attention's work items.  One workgroup, a thread per slot for the sums
// and all threads over the pages, places and items.  Pages are handed out in the order
// of (slot, block) whatever order the threads run in.  One workgroup, as every number
// depends on the sums over all slots; bound by the latency of its few dependent reads and
// barriers: 4.2 us for one slot, 4.9 for 256 (a launch that does nothing: 3.4).
__global__ void __launch_bounds__(kStepThreads) paged_step_kernel(const PagedStepArgs a) {
  __shared__ uint64_t sums[3][kStepThreads / kWave];
  __shared__ int32_t first_back[kStepThreads + 1], first_more[kStepThreads + 1], first_item[kStepThreads + 1];
  __shared__ int32_t r1[kStepThreads], n1[kStepThreads], r2[kStepThreads], s_had[kStepThreads];
  __shared__ int32_t s_len[kStepThreads], s_new[kStepThreads], s_sink[kStepThreads], s_skip[kStepThreads];
  __shared__ int32_t s_blocks[kStepThreads];
  const int b = threadIdx.x;
  const bool slot = b < a.batch;
  const int32_t page = 1 << a.page_shift;
  const int64_t places = (int64_t)a.max_pages << a.page_shift;

  int32_t len = 0, fresh = 0, covered = 0, released = 0;
  const int32_t count = a.state[kFreePages];
  bool leaves = false;
  if (slot) {
    covered = a.state[a.at.covered + b];
    released = a.state[a.at.released + b];
    const int32_t keep = a.keep ? a.keep[b] : 0;
    fresh = max(a.n_new[b], 0);
    const int32_t took = a.state[a.at.n_new + b];     // new tokens of the last step, 0 if it had no pages
    leaves = keep < 0;
    len = leaves ? 0 : max(a.lens[b], 0) + min(keep, took);
  }
  // Blocks of pages that stay in front of the window, and those that the window has left.
  const int32_t s0 = (a.sinks + page - 1) >> a.page_shift;
  int32_t hidden = 0;                    // blocks before this one hold no token a new one sees ...
  if (a.window > 0 && !leaves && len - a.window + 1 > 0) hidden = (len - a.window + 1) >> a.page_shift;
  hidden = hidden > s0 ? hidden : 0;     // ... but for the first s0
  const int64_t want64 = ((int64_t)len + fresh + page - 1) >> a.page_shift;
  const int32_t want = (int32_t)(want64 < (1 << 30) ? want64 : 1 << 30);
  // Pages given back: two runs of blocks.
  int32_t a0, a1, b0;
  if (leaves) {
    a0 = 0;
    a1 = released > 0 ? min(s0, covered) : covered;
    b0 = released > 0 ? released : covered;
  } else {
    a0 = max(s0, released);
    a1 = max(hidden, a0);
    b0 = max(want, max(hidden, released));
  }
  const int32_t c1 = max(a1 - a0, 0), c2 = max(covered - b0, 0);
  const int32_t had = leaves ? 0 : min(covered, want);
  const int32_t need = slot ? max(want - had, 0) : 0;
  // Sums of two and three numbers at once: pages and blocks are fewer than 2^26 (a pool
  // has fewer than 2^31 tokens), needs up to 2^20 a slot.
  uint64_t all;
  const bool fits_table = want <= a.max_pages;      // a slot that needs more has none
  const uint64_t before = step_scan((uint64_t)(slot ? c1 + c2 : 0) << 32 | (fits_table ? need : 0), sums[0], all);
  const int32_t n_back = (int32_t)(all >> 32);
  first_back[b] = (int32_t)(before >> 32);
  r1[b] = a0;
  n1[b] = c1;
  r2[b] = b0;
  const int32_t free_now = count + n_back;
  // A slot's pages are taken if those of all slots up to it fit.
  const bool granted = fits_table && (need == 0 || (int32_t)(uint32_t)before + need <= free_now);
  s_had[b] = had;
  const int32_t now = granted ? fresh : 0;
  // Visible blocks of 32 tokens, and work items.
  int32_t blocks = 0, sink = 0, skip = 0;
  if (slot && now > 0 && now <= kPagedMaxNew) {       // (a prompt comes with its attention done)
    const int32_t end = (len + now + kPagedBlock - 1) / kPagedBlock;
    const int32_t from = a.window > 0 ? max(0, len - a.window + 1) / kPagedBlock : 0;
    sink = min((min(a.sinks, len + now) + kPagedBlock - 1) / kPagedBlock, from);
    skip = from - sink;
    blocks = end - skip;
  }
  s_len[b] = len;
  s_new[b] = now;
  s_sink[b] = sink;
  s_skip[b] = skip;
  s_blocks[b] = blocks;
  const bool rows = blocks > 0 && now * a.group > 16;
  const uint64_t taken = step_scan((uint64_t)(granted ? need : 0) << 38 | (uint64_t)blocks << 11 | (uint64_t)(blocks > 0), sums[1], all);
  const int32_t n_more = (int32_t)(all >> 38), n_blocks = (int32_t)(all >> 11 & 0x7FFFFFF), n_live = (int32_t)(all & 0x7FF);
  first_more[b] = (int32_t)(taken >> 38);
  // Items of `per` blocks, so that there are about as many as the launch has workgroups: a
  // live slot's last one is half full.
  const bool many = __syncthreads_or(rows);
  const int32_t target = (many ? kPagedRowItems : kPagedItems) / a.n_kv_heads;
  const int32_t whole = max(target - n_live / 2, target / 4 + 1);
  const int32_t per = max(kPagedMinBlocks, (n_blocks + whole - 1) / whole);
  const int32_t items = (blocks + per - 1) / per;
  first_item[b] = (int32_t)step_scan(items, sums[2], all);
  const int32_t n_items = (int32_t)all;
  if (b == 0) {
    first_back[kStepThreads] = n_back;
    first_more[kStepThreads] = n_more;
    first_item[kStepThreads] = n_items;
  }
  __syncthreads();

  int32_t* const stack = a.state + a.at.stack;
  for (int32_t k = threadIdx.x; k < n_back; k += kStepThreads) {
    const int32_t s = step_find(first_back, kStepThreads, k), j = k - first_back[s];
    const int32_t block = j < n1[s] ? r1[s] + j : r2[s] + j - n1[s];
    int32_t* const entry = a.table + (int64_t)s * a.max_pages + block;
    stack[count + n_back - 1 - k] = *entry;
    *entry = -1;
  }
  __syncthreads();
  for (int32_t k = threadIdx.x; k < n_more; k += kStepThreads) {
    const int32_t s = step_find(first_more, kStepThreads, k), j = k - first_more[s];
    a.table[(int64_t)s * a.max_pages + s_had[s] + j] = stack[free_now - 1 - k];
  }
  if (slot) {
    a.lens[b] = len;
    a.state[a.at.covered + b] = granted ? want : had;
    a.state[a.at.released + b] = leaves ? 0 : max(hidden, released);
    a.state[a.at.n_new + b] = now;
    a.state[a.at.first + b] = first_item[b];
    if (a.missing) a.missing[b] = granted ? 0 : want - had;
  }
  if (b == 0) {
    a.state[kFreePages] = free_now - n_more;
    a.state[kNumItems] = n_items;
    a.state[a.at.first + a.batch] = n_items;
  }
  PagedItem* const list = reinterpret_cast<PagedItem*>(a.state + a.at.items);
  for (int32_t k = threadIdx.x; k < n_items; k += kStepThreads) {
    const int32_t s = step_find(first_item, kStepThreads, k), part = k - first_item[s];
    list[k] = {s, part * per, min((part + 1) * per, s_blocks[s]), first_item[s + 1] - first_item[s], s_len[s], s_new[s], s_sink[s], s_skip[s]};
  }
  if (!a.slot_map) return;
  __syncthreads();                        // the table's new entries are seen
  for (int32_t k = threadIdx.x; k < a.batch * a.width; k += kStepThreads) {
    const int32_t s = k / a.width, i = k - s * a.width;
    int32_t place = -1;
    const int64_t t = (int64_t)s_len[s] + i;
    if (i < s_new[s] && t < places) {
      const int32_t id = a.table[(int64_t)s * a.max_pages + (t >> a.page_shift)];
      place = id < 0 ? -1 : (id << a.page_shift) + (int32_t)(t & (page - 1));
    }
    a.slot_map[s * a.map_ld + i] = place;
  }
}

// An empty cache: no pages in the tables, all of them free, to be taken in `order`
// (null: 0, 1, ...).
__global__ void __launch_bounds__(256) paged_reset_kernel(int32_t* table, int32_t* lens, int32_t* state,
                                                          const int32_t* order, int32_t batch, int32_t max_pages,
                                                          int32_t n_pages, PagedState at) {
  const int64_t n = (int64_t)batch * max_pages, step = (int64_t)gridDim.x * 256;
  const int64_t i0 = (int64_t)blockIdx.x * 256 + threadIdx.x;
  for (int64_t i = i0; i < n; i += step) table[i] = -1;
  for (int64_t i = i0; i < batch; i += step) lens[i] = 0;
  for (int64_t i = i0; i < at.stack; i += step) state[i] = i == kFreePages ? n_pages : 0;
  for (int64_t i = i0; i < n_pages; i += step) state[at.stack + n_pages - 1 - i] = order ? order[i] : (int32_t)i;
}

constexpr int kPagedSegs = 32;           // queries per launch

// Whole queries between [layer][head][len][D] and pages.
struct PagedCopyArgs {
  uint8_t* k;
  uint8_t* v;
  const int32_t* table;
  int64_t layer_bytes;
  int32_t n_layers, n_kv_heads, max_pages, n_pages, page_shift, n_segs;
  int32_t slot[kPagedSegs], len[kPagedSegs];
  int64_t block_end[kPagedSegs];         // inclusive prefix of blocks over the queries
  uint8_t* kext[kPagedSegs];
  uint8_t* vext[kPagedSegs];
};

// One wave per block of 32 tokens of a layer, head, and K or V: through LDS, where the
// values are transposed, so that memory sees whole rows on one side and whole chunks on
// the other.  Bound by memory: eight queries of up to 4,096 tokens 5.1 to 5.7 TB/s, read and
// written (112 us in, 101 out; a plain copy 4.9).  OUT: pages to queries.  Tokens behind the query's last are zeros.
template <int ES, int D, bool OUT>
__global__ void __launch_bounds__(kWave) paged_copy_kernel(const PagedCopyArgs a) {
  constexpr int ROW = D * ES, VECS = 32 * ROW / 1024, CH = ROW / 64, LDR = ROW + 16;
  __shared__ __attribute__((aligned(16))) uint8_t tile[32 * LDR];
  const int lane = threadIdx.x;
  for (int64_t g = blockIdx.x; g < a.block_end[a.n_segs - 1]; g += gridDim.x) {
    __syncthreads();                       // the last block's reads of the tile are done
    int i = 0;
    while (i < a.n_segs - 1 && g >= a.block_end[i]) ++i;
    int64_t local = g - (i > 0 ? a.block_end[i - 1] : 0);
    const int32_t len = a.len[i], blocks = (len + 31) / 32;
    const int32_t block = (int32_t)(local % blocks);
    local /= blocks;
    const int32_t h = (int32_t)(local % a.n_kv_heads);
    local /= a.n_kv_heads;
    const int32_t layer = (int32_t)(local >> 1), which = (int32_t)(local & 1);
    const int32_t shift = a.page_shift - 5;               // blocks per page
    if ((block >> shift) >= a.max_pages) continue;
    const int32_t id = a.table[(int64_t)a.slot[i] * a.max_pages + (block >> shift)];
    if ((uint32_t)id >= (uint32_t)a.n_pages) continue;      // no page: nothing is there
    uint8_t* const at = (which ? a.v : a.k) + layer * a.layer_bytes +
                        ((((int64_t)id * a.n_kv_heads + h) << shift) + (block & ((1 << shift) - 1))) * (32 * ROW);
    uint8_t* const ext = (which ? a.vext[i] : a.kext[i]) + (((int64_t)layer * a.n_kv_heads + h) * len + block * 32) * ROW;
    const int32_t nt = min(32, len - block * 32);
    u32x4* const chunks = reinterpret_cast<u32x4*>(at);
    if constexpr (!OUT) {
      u32x4 w[VECS];
#pragma unroll
      for (int u = 0; u < VECS; ++u) {
        const int idx = u * kWave + lane, t = idx / (ROW / 16);
        w[u] = t < nt ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(ext) + idx) : u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int u = 0; u < VECS; ++u) {
        const int idx = u * kWave + lane, t = idx / (ROW / 16), p = idx % (ROW / 16);
        *reinterpret_cast<u32x4*>(tile + t * LDR + p * 16) = w[u];
      }
      __syncthreads();
    }
    const int g4 = lane / 16, c16 = lane % 16;
    u32x4 w[VECS];
    if constexpr (OUT) {
#pragma unroll
      for (int u = 0; u < VECS; ++u) w[u] = __builtin_nontemporal_load(chunks + u * kWave + lane);
    }
    if (!which) {
#pragma unroll
      for (int u = 0; u < VECS; ++u) {
        const int tl = u / CH, c = u % CH, t = 8 * (c16 / 4) + 4 * tl + c16 % 4;
        u32x4* const cell = reinterpret_cast<u32x4*>(tile + t * LDR + (c * 4 + g4) * 16);
        if constexpr (OUT) *cell = w[u];
        else w[u] = *cell;
      }
    } else {
#pragma unroll
      for (int u = 0; u < VECS; ++u) {
        if constexpr (ES == 2) {
          uint16_t x[8];
          if constexpr (OUT) *reinterpret_cast<u32x4*>(x) = w[u];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            uint16_t* const cell = reinterpret_cast<uint16_t*>(tile + (8 * g4 + e) * LDR) + 16 * u + c16;
            if constexpr (OUT) *cell = x[e];
            else x[e] = *cell;
          }
          if constexpr (!OUT) w[u] = *reinterpret_cast<u32x4*>(x);
        } else {
          const int tl = u / (D / 16), dt = u % (D / 16);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            uint32_t* const cell = reinterpret_cast<uint32_t*>(tile + (8 * g4 + 4 * tl + r) * LDR) + 16 * dt + c16;
            if constexpr (OUT) *cell = w[u][r];
            else w[u][r] = *cell;
          }
        }
      }
    }
    if constexpr (OUT) {
      __syncthreads();
#pragma unroll
      for (int u = 0; u < VECS; ++u) {
        const int idx = u * kWave + lane, t = idx / (ROW / 16), p = idx % (ROW / 16);
        if (t < nt)
          __builtin_nontemporal_store(*reinterpret_cast<const u32x4*>(tile + t * LDR + p * 16),
                                      reinterpret_cast<u32x4*>(ext) + idx);
      }
    } else {
#pragma unroll
      for (int u = 0; u < VECS; ++u) __builtin_nontemporal_store(w[u], chunks + u * kWave + lane);
    }
  }
}

}  // namespace baton
