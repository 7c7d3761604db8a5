// Host side of the verification of drafted tokens: argument checks and launches.  The
// C ABI is documented in include/baton.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "baton.h"
#include "verify_kernel.hpp"

namespace {

bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

size_t kept_bytes(int32_t batch, int32_t width) {
  return ((size_t)batch * (2 * width - 1) * sizeof(baton::SampleKept) + 255) / 256 * 256;
}

size_t sums_bytes(int32_t batch) { return (size_t)2 * batch * baton::kVerifyParts * sizeof(uint64_t); }

// Pieces of a row of `bytes`-byte elements, at the worst alignment of its first one.
int32_t row_pieces(int32_t vocab, int32_t bytes) {
  const int32_t per = 16 / bytes, vecs = (int32_t)(((int64_t)vocab + 2 * (per - 1)) / per);
  const int32_t each = baton::kVerifyThreads * baton::kVerifyVecs;
  return (vecs + each - 1) / each;
}

template <typename T>
baton_status launch(const baton::VerifyArgs& a, hipStream_t s) {
  const int64_t vec = ((int64_t)a.vocab + 2 * (16 / T::kBytes - 1)) / (16 / T::kBytes);
  int64_t lds = (sizeof(baton::SampleShared) + 15) / 16 * 16 + std::min<int64_t>(vec * 16, baton::kSampleRowBytes);
  if (T::kBytes == 2) lds = std::max<int64_t>(lds, sizeof(baton::ValueShared));
  const int32_t rows = a.batch * a.slot_rows;
  hipLaunchKernelGGL(baton::verify_pieces_kernel<T>, dim3(a.n_pieces, rows), dim3(baton::kVerifyThreads), 0, s, a);
  hipLaunchKernelGGL(baton::verify_rows_kernel<T>, dim3(rows), dim3(baton::kSampleThreads), (uint32_t)lds, s, a);
  hipLaunchKernelGGL(baton::verify_sums_kernel<T>, dim3(a.segs, a.batch), dim3(baton::kVerifyThreads), 0, s, a);
  hipLaunchKernelGGL(baton::verify_draw_kernel<T>, dim3(a.batch), dim3(baton::kVerifyThreads), 0, s, a);
  return hipGetLastError() == hipSuccess ? BATON_OK : BATON_EHIP;
}

}  // namespace

namespace baton {

baton_status verify(const int32_t* taken, int32_t dtype, const void* target, int64_t target_ld, const void* draft,
                    int64_t draft_ld, int32_t batch, int32_t width, int32_t vocab, const int32_t* drafted,
                    const int32_t* n_draft, const float* u_accept, const float* u_token, const float* temperature,
                    const int32_t* top_k, const float* top_p, const float* min_p, int32_t* tokens, int32_t* n_out,
                    void* ws, size_t ws_bytes, hipStream_t stream) {
  const int64_t most_ld = int64_t(1) << 40;
  if (batch < 1 || batch > BATON_MAX_BATCH || width < 1 || width > BATON_PAGED_MAX_WIDTH || vocab < 1 ||
      vocab > (1 << 24) || !target || target_ld < vocab || target_ld > most_ld || !u_token || !tokens || !n_out)
    return BATON_EINVAL;
  if (width > 1 && (!drafted || !u_accept || (draft && (draft_ld < vocab || draft_ld > most_ld)))) return BATON_EINVAL;
  if (dtype != BATON_F32 && dtype != BATON_BF16) return BATON_EDTYPE;
  const uintptr_t es = dtype == BATON_F32 ? 4 : 2;
  if (!aligned(target, es) || !aligned(draft, es) || !aligned(drafted, 4) || !aligned(n_draft, 4) ||
      !aligned(u_accept, 4) || !aligned(u_token, 4) || !aligned(temperature, 4) || !aligned(top_k, 4) ||
      !aligned(top_p, 4) || !aligned(min_p, 4) || !aligned(tokens, 4) || !aligned(n_out, 4))
    return BATON_EINVAL;
  // launches of fewer than 2^32 threads (logits of 256 GiB and more)
  if ((int64_t)batch * (2 * width - 1) * row_pieces(vocab, (int32_t)es) >= (int64_t(1) << 24)) return BATON_EINVAL;
  if (!ws || !aligned(ws, 16) || ws_bytes < baton_verify_workspace_bytes(batch, width, vocab)) return BATON_EINVAL;
  VerifyArgs a;
  std::memset(&a, 0, sizeof(a));
  a.target = static_cast<const uint8_t*>(target);
  a.draft = width > 1 ? static_cast<const uint8_t*>(draft) : nullptr;
  a.target_ld = target_ld;
  a.draft_ld = draft_ld;
  a.batch = batch;
  a.width = width;
  a.vocab = vocab;
  int32_t bits = 0;
  while ((1 << bits) < vocab) ++bits;
  a.shift = std::min(62 - bits, 51);
  // As many segments as fill the GPU: before the first token a workgroup waits for a chain
  // of loads.  64 slots of 128,000: 144 us with half as many, 131 with these and with twice as many.
  const int32_t parts = std::min(kVerifySegs, std::max(1, 1024 / batch)) * kVerifyWaves;
  a.per_part = std::max(((vocab + parts - 1) / parts + 7) / 8 * 8, kWave);   // whole 16-byte vectors
  a.segs = (vocab + kVerifyWaves * a.per_part - 1) / (kVerifyWaves * a.per_part);
  a.drafted = drafted;
  a.n_draft = n_draft;
  a.taken = taken;
  a.u_accept = u_accept;
  a.u_token = u_token;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.tokens = tokens;
  a.n_out = n_out;
  a.kept = static_cast<SampleKept*>(ws);
  a.sums = reinterpret_cast<uint64_t*>(static_cast<char*>(ws) + kept_bytes(batch, width));
  a.pieces = reinterpret_cast<VerifyPiece*>(reinterpret_cast<char*>(a.sums) + sums_bytes(batch));
  a.n_pieces = row_pieces(vocab, (int32_t)es);
  a.slot_rows = a.draft ? 2 * width - 1 : width;
  return dtype == BATON_F32 ? launch<F32Tag>(a, stream) : launch<BF16Tag>(a, stream);
}

}  // namespace baton

extern "C" {

size_t baton_verify_workspace_bytes(int32_t batch, int32_t width, int32_t vocab) {
  if (batch < 1 || batch > BATON_MAX_BATCH || width < 1 || width > BATON_PAGED_MAX_WIDTH || vocab < 1 ||
      vocab > (1 << 24))
    return 0;
  return kept_bytes(batch, width) + sums_bytes(batch) +
         (size_t)batch * (2 * width - 1) * row_pieces(vocab, 4) * sizeof(baton::VerifyPiece);
}

baton_status baton_verify(int32_t dtype, const void* target, int64_t target_ld, const void* draft, int64_t draft_ld,
                          int32_t batch, int32_t width, int32_t vocab, const int32_t* drafted, const int32_t* n_draft,
                          const float* u_accept, const float* u_token, const float* temperature, const int32_t* top_k,
                          const float* top_p, const float* min_p, int32_t* tokens, int32_t* n_out, void* ws,
                          size_t ws_bytes, hipStream_t stream) {
  return baton::verify(nullptr, dtype, target, target_ld, draft, draft_ld, batch, width, vocab, drafted, n_draft,
                       u_accept, u_token, temperature, top_k, top_p, min_p, tokens, n_out, ws, ws_bytes, stream);
}

}  // extern "C"
