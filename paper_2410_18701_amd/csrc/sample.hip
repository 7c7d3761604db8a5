// Host side of sampling: argument checks and the launch.  The C ABI is
// documented in include/baton.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "baton.h"
#include "sample_kernel.hpp"

namespace {

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

template <typename T>
baton_status launch_sample(const baton::SampleArgs& a, int32_t rows, hipStream_t s) {
  // the row's vectors, at the worst alignment of its first element
  const int64_t vec = ((int64_t)a.vocab + 2 * (16 / T::kBytes - 1)) / (16 / T::kBytes);
  const uint32_t lds = (uint32_t)std::min<int64_t>(vec * 16, baton::kSampleRowBytes);
  hipLaunchKernelGGL(baton::sample_kernel<T>, dim3(rows), dim3(baton::kSampleThreads), lds, s, a);
  return hipGetLastError() == hipSuccess ? BATON_OK : BATON_EHIP;
}

}  // namespace

extern "C" {

baton_status baton_sample(int32_t dtype, const void* logits, int64_t ld, int32_t rows, int32_t vocab,
                          const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                          const float* u, int32_t* tokens, hipStream_t stream) {
  // fewer than 2^32 threads: 1024 a row
  if (!logits || !u || !tokens || rows < 1 || rows > (1 << 21) || vocab < 1 || vocab > (1 << 24) || ld < vocab || ld > (int64_t(1) << 40))
    return BATON_EINVAL;
  if (dtype != BATON_F32 && dtype != BATON_BF16) return BATON_EDTYPE;
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == BATON_F32 ? 4 : 2) || !aligned4(temperature) ||
      !aligned4(top_k) || !aligned4(top_p) || !aligned4(min_p) || !aligned4(u) || !aligned4(tokens))
    return BATON_EINVAL;
  baton::SampleArgs a;
  std::memset(&a, 0, sizeof(a));
  a.logits = static_cast<const uint8_t*>(logits);
  a.ld = ld;
  a.vocab = vocab;
  int32_t bits = 0;
  while ((1 << bits) < vocab) ++bits;
  a.shift = std::min(62 - bits, 51);
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.u = u;
  a.tokens = tokens;
  return dtype == BATON_F32 ? launch_sample<baton::F32Tag>(a, rows, stream)
                            : launch_sample<baton::BF16Tag>(a, rows, stream);
}

}  // extern "C"
