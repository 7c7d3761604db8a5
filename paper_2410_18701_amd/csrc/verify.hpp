// The verification of drafted tokens as baton_verify has it (include/baton.h), and for the
// drafts of a paged cache's step: taken, device [batch], the new tokens that the step took
// of each slot, or null.
#pragma once

#include "baton.h"

namespace baton {

baton_status verify(const int32_t* taken, int32_t dtype, const void* target, int64_t target_ld, const void* draft,
                    int64_t draft_ld, int32_t batch, int32_t width, int32_t vocab, const int32_t* drafted,
                    const int32_t* n_draft, const float* u_accept, const float* u_token, const float* temperature,
                    const int32_t* top_k, const float* top_p, const float* min_p, int32_t* tokens, int32_t* n_out,
                    void* ws, size_t ws_bytes, hipStream_t stream);

}  // namespace baton
