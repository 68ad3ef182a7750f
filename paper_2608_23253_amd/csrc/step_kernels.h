// Launchers of the operators of e2s_step.h (host side).  Arguments are validated by the
// caller; each launcher only enqueues kernels on `stream`.
#pragma once

#include <hip/hip_runtime.h>

#include "step_validate.h"

namespace e2s {

// Pairs: of q and of k.
hipError_t launch_norm_rotate(const e2s_norm_rotate_shape& s, const e2s_rotary_plan& p,
                              const int32_t* positions, const void* const (&src)[2],
                              const void* const (&weight)[2], const void* const (&grad)[2],
                              void* const (&dst)[2], void* const (&weight_grad)[2],
                              void* workspace, bool back, hipStream_t stream);

hipError_t launch_cache4_append(const e2s_cache4& c, const e2s_cache_append_shape& s,
                                const int32_t* pages, const int32_t* start, const int32_t* count,
                                const int32_t* src_idx, const void* k, const void* v,
                                hipStream_t stream);

hipError_t launch_cache4_read(const e2s_cache4& c, const e2s_cache4_read_shape& s,
                              const int32_t* pages, const int32_t* start, const int32_t* count,
                              void* k_out, void* v_out, hipStream_t stream);

hipError_t launch_cache4_attend(const e2s_cache4& c, const e2s_cache4_attend_shape& s,
                                const int32_t* pages, const int32_t* lengths,
                                const int32_t* q_count, const void* q, void* out, void* workspace,
                                hipStream_t stream);

}  // namespace e2s
