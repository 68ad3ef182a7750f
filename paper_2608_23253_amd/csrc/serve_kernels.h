// Launchers of the operators of e2s_serve.h (host side).  Arguments are validated by the
// caller; each launcher only enqueues kernels on `stream`.
#pragma once

#include <hip/hip_runtime.h>

#include "serve_validate.h"

namespace e2s {

hipError_t launch_rotate(const e2s_rotary_shape& s, const e2s_rotary_plan& p,
                         const int32_t* positions, const void* q, const void* k, void* q_out,
                         void* k_out, hipStream_t stream);

hipError_t launch_cache_append(const e2s_cache& c, const e2s_cache_append_shape& s,
                               const int32_t* pages, const int32_t* start, const int32_t* count,
                               const int32_t* src_idx, const void* k, const void* v,
                               hipStream_t stream);

hipError_t launch_cache_attend(const e2s_cache& c, const e2s_cache_attend_shape& s,
                               const int32_t* pages, const int32_t* lengths,
                               const int32_t* q_count, const void* q, void* out,
                               const float* weights_in, float* weights_out, void* workspace,
                               hipStream_t stream);

hipError_t launch_cache_evict(const e2s_cache& c, const e2s_cache_evict_shape& s,
                              const int32_t* pages, const int32_t* lengths, const float* weights,
                              const int32_t* new_pages, int32_t* keep_idx, int32_t* new_len,
                              float* left, hipStream_t stream);

}  // namespace e2s
