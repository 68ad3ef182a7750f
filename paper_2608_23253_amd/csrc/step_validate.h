// Host-side argument checks of e2s_step.h.  Pure C++, no HIP: every entry point runs these
// before it touches the runtime, so an invalid call enqueues nothing.
#pragma once

#include "e2s_step.h"
#include "serve_validate.h"

namespace e2s {

// `back`: the gradients' strides count as well.
e2s_status check_norm_rotate(const e2s_norm_rotate_shape* s, const e2s_rotary_plan& p, bool back);
// Workgroups of the backward pass at most: each stores one partial row per weight.  Eight to a
// compute unit fill the device.
constexpr int64_t kNormMostParts = 2048;
size_t norm_rotate_back_bytes(const e2s_norm_rotate_shape& s, const e2s_rotary_plan& p,
                              bool weight_grads);

e2s_status check_cache4(const e2s_cache4* c);
e2s_status check_append4(const e2s_cache4& c, const e2s_cache_append_shape* s);
e2s_status check_read4(const e2s_cache4& c, const e2s_cache4_read_shape* s);
e2s_status check_attend4(const e2s_cache4& c, const e2s_cache4_attend_shape* s);

constexpr int kGroup4 = 32;          // tokens whose values share their bytes
constexpr int kStep4 = 128;          // keys of a wave's step

// How an attention call is cut into workgroups, from its sizes alone.
struct Attend4Plan {
    int64_t rows;        // query rows of one key head: H/Hkv * T, row = t * (H/Hkv) + head
    int64_t row_groups;  // workgroups along the rows, 16 each
    int waves;           // of a workgroup, which part its keys: 1, 2, 4 or 8
    int64_t chunk;       // keys of a workgroup, a multiple of kStep4 * waves
    int64_t splits;      // workgroups along the keys at max_tokens
    size_t max_off, sum_off, part_off, bytes;    // workspace regions
};
Attend4Plan attend4_plan(const e2s_cache4& c, const e2s_cache4_attend_shape& s);

}  // namespace e2s
