// Host-side argument checks of e2s_serve.h.  Pure C++, no HIP: every entry point runs
// these before it touches the runtime, so an invalid call enqueues nothing.
#pragma once

#include <cstddef>
#include <cstdint>

#include "e2s_serve.h"
#include "e2s_validate.h"

namespace e2s {

constexpr int64_t kMaxCachedTokens = 1 << 20;   // per sequence

bool known_dtype(int32_t t);
// Strides of n dimensions of rows of `row` elements of `bytes` each (see the definition).
e2s_status check_strides(const int64_t* st, const int64_t* counts, int n, int64_t row, int least,
                         int64_t align, int bytes);
e2s_status check_table(int64_t batch, int64_t max_pages, int64_t stride);

e2s_status check_rotary_spec(const e2s_rotary_spec* s);
// Frequencies, axes and amplitude of a checked spec.
void fill_rotary_plan(const e2s_rotary_spec& s, e2s_rotary_plan* p);
// A plan as e2s_rotary_plan_init leaves it: counts and axes in range (the kernel indexes
// by them).
e2s_status check_rotary_plan(const e2s_rotary_plan* p);
e2s_status check_rotary_shape(const e2s_rotary_shape* s, const e2s_rotary_plan& p);

e2s_status check_cache(const e2s_cache* c);
e2s_status check_append(const e2s_cache& c, const e2s_cache_append_shape* s);
e2s_status check_attend(const e2s_cache& c, const e2s_cache_attend_shape* s);
e2s_status check_evict(const e2s_cache& c, const e2s_cache_evict_shape* s);

inline int elem_bytes(int dtype) { return dtype == E2S_DTYPE_F32 ? 4 : 2; }

// How an attention call is cut into workgroups, from its sizes alone.
struct AttendPlan {
    int64_t rows;        // query rows of one key head: H/Hkv * T, row = t * (H/Hkv) + head
    bool shared_rows;    // the kernel whose waves part the rows (else: the keys)
    int tiles;           // 16-row tiles of a wave: 1 or 2
    int waves;           // of a workgroup: kAttendWaves or 8
    int64_t row_groups;  // workgroups along the rows
    int64_t chunk;       // keys of a workgroup, a multiple of kAttendStep * waves
    int64_t splits;      // workgroups along the keys at max_tokens
    int64_t logit_stride;             // floats between the rows of the stored logits
    bool lse_kept;       // the rows' sums go to the workspace, for the weights' own launch
    size_t max_off, sum_off, part_off, lse_off, logit_off, bytes;   // workspace regions
};
constexpr int kAttendWaves = 4;
constexpr int kAttendStep = 32;     // keys of a wave's step
constexpr int kWeightKeys = 64;     // keys of a wave that adds up many rows' weights
constexpr int64_t kFewKeys = 1024, kShortKeys = 2048;
AttendPlan attend_plan(const e2s_cache& c, const e2s_cache_attend_shape& s);

}  // namespace e2s
