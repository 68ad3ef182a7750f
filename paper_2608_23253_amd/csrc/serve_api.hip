// extern "C" entry points of e2s_serve.h.  Each call validates every argument on the host
// before it touches the HIP runtime, then enqueues its kernels on the caller's stream.
#include <initializer_list>

#include "e2s_serve.h"
#include "serve_kernels.h"

namespace {

e2s_status from_hip(hipError_t err) { return err == hipSuccess ? E2S_OK : E2S_ERR_LAUNCH; }

#define E2S_TRY(expr)                          \
    do {                                       \
        const e2s_status st_ = (expr);         \
        if (st_ != E2S_OK) return st_;         \
    } while (0)

// A required pointer, aligned to `a` bytes; an optional one.
e2s_status need(const void* p, size_t a) {
    return p ? e2s::check_aligned(p, a) : E2S_ERR_NULL_POINTER;
}
e2s_status optional(const void* p, size_t a) { return p ? e2s::check_aligned(p, a) : E2S_OK; }

// An output in its input's place has the input's strides (where a dimension has more than one
// index): with others it would write what is still to be read.
e2s_status in_place(const void* in, const void* out, const int64_t* is, const int64_t* os,
                    std::initializer_list<int64_t> counts) {
    if (in != out || in == nullptr) return E2S_OK;
    int i = 0;
    for (const int64_t n : counts) {
        if (n > 1 && is[i] != os[i]) return E2S_ERR_BAD_PARAM;
        ++i;
    }
    return E2S_OK;
}

}  // namespace

extern "C" {

int32_t e2s_serve_abi_version(void) { return E2S_SERVE_ABI_VERSION; }

e2s_status e2s_rotary_plan_init(const e2s_rotary_spec* spec, e2s_rotary_plan* plan) {
    E2S_TRY(e2s::check_rotary_spec(spec));
    if (plan == nullptr) return E2S_ERR_NULL_POINTER;
    e2s::fill_rotary_plan(*spec, plan);
    return E2S_OK;
}

e2s_status e2s_rotate_positions(const e2s_rotary_shape* shape, const e2s_rotary_plan* plan,
                                const int32_t* positions, const void* q, const void* k,
                                void* q_out, void* k_out, void* stream) {
    E2S_TRY(e2s::check_rotary_plan(plan));
    E2S_TRY(e2s::check_rotary_shape(shape, *plan));
    if (shape->num_tokens == 0) return E2S_OK;
    const size_t eb = static_cast<size_t>(e2s::elem_bytes(shape->dtype));
    E2S_TRY(need(positions, 4));
    if (shape->q_heads > 0) {
        E2S_TRY(need(q, eb));
        E2S_TRY(need(q_out, eb));
        E2S_TRY(in_place(q, q_out, shape->q_stride, shape->q_out_stride,
                         {shape->batch, shape->q_heads, shape->num_tokens}));
    }
    if (shape->k_heads > 0) {
        E2S_TRY(need(k, eb));
        E2S_TRY(need(k_out, eb));
        E2S_TRY(in_place(k, k_out, shape->k_stride, shape->k_out_stride,
                         {shape->batch, shape->k_heads, shape->num_tokens}));
    }
    // each output is written while the other tensor's rows are still read, or written
    if (shape->q_heads > 0 && shape->k_heads > 0 &&
        (q_out == k_out || q_out == k || k_out == q))
        return E2S_ERR_BAD_PARAM;
    return from_hip(e2s::launch_rotate(*shape, *plan, positions, q, k, q_out, k_out,
                                       static_cast<hipStream_t>(stream)));
}

e2s_status e2s_cache_append(const e2s_cache* cache, const e2s_cache_append_shape* shape,
                            const int32_t* pages, const int32_t* start, const int32_t* count_opt,
                            const int32_t* src_idx_opt, const void* k, const void* v,
                            void* stream) {
    E2S_TRY(e2s::check_cache(cache));
    E2S_TRY(e2s::check_append(*cache, shape));
    if (shape->num_tokens == 0) return E2S_OK;
    if (src_idx_opt == nullptr && shape->src_tokens < shape->num_tokens) return E2S_ERR_BAD_SHAPE;
    E2S_TRY(need(pages, 4));
    E2S_TRY(need(start, 4));
    E2S_TRY(optional(count_opt, 4));
    E2S_TRY(optional(src_idx_opt, 4));
    E2S_TRY(need(k, 16));
    E2S_TRY(need(v, 16));
    return from_hip(e2s::launch_cache_append(*cache, *shape, pages, start, count_opt, src_idx_opt,
                                             k, v, static_cast<hipStream_t>(stream)));
}

e2s_status e2s_cache_attend_workspace_size(const e2s_cache* cache,
                                           const e2s_cache_attend_shape* shape, size_t* bytes) {
    E2S_TRY(e2s::check_cache(cache));
    E2S_TRY(e2s::check_attend(*cache, shape));
    if (bytes == nullptr) return E2S_ERR_NULL_POINTER;
    *bytes = e2s::attend_plan(*cache, *shape).bytes;
    return E2S_OK;
}

e2s_status e2s_cache_attend(const e2s_cache* cache, const e2s_cache_attend_shape* shape,
                            const int32_t* pages, const int32_t* lengths,
                            const int32_t* q_count_opt, const void* q, void* out,
                            const float* weights_in_opt, float* weights_out_opt, void* workspace,
                            size_t workspace_bytes, void* stream) {
    E2S_TRY(e2s::check_cache(cache));
    E2S_TRY(e2s::check_attend(*cache, shape));
    E2S_TRY(need(pages, 4));
    E2S_TRY(need(lengths, 4));
    E2S_TRY(optional(q_count_opt, 4));
    E2S_TRY(need(q, 16));
    E2S_TRY(need(out, 16));
    // weights_out exactly where the shape announced it: its strides and workspace are sized by it
    if ((weights_out_opt != nullptr) != (shape->weights != 0)) return E2S_ERR_BAD_PARAM;
    if (weights_in_opt != nullptr && weights_out_opt == nullptr) return E2S_ERR_BAD_PARAM;
    E2S_TRY(optional(weights_in_opt, 4));
    E2S_TRY(optional(weights_out_opt, 4));
    E2S_TRY(in_place(weights_in_opt, weights_out_opt, shape->weights_in_stride,
                     shape->weights_out_stride, {shape->batch, cache->num_kv_heads}));
    const size_t bytes = e2s::attend_plan(*cache, *shape).bytes;
    if (bytes > 0) E2S_TRY(need(workspace, 256));
    if (workspace_bytes < bytes) return E2S_ERR_WORKSPACE_TOO_SMALL;
    // many rows' weights read the queries again when the outputs are there
    if (out == q) return E2S_ERR_BAD_PARAM;
    return from_hip(e2s::launch_cache_attend(*cache, *shape, pages, lengths, q_count_opt, q, out,
                                             weights_in_opt, weights_out_opt, workspace,
                                             static_cast<hipStream_t>(stream)));
}

e2s_status e2s_cache_evict(const e2s_cache* cache, const e2s_cache_evict_shape* shape,
                           const int32_t* pages, const int32_t* lengths, const float* weights,
                           const int32_t* new_pages, int32_t* keep_idx, int32_t* new_len,
                           float* weights_left_opt, void* stream) {
    E2S_TRY(e2s::check_cache(cache));
    E2S_TRY(e2s::check_evict(*cache, shape));
    E2S_TRY(need(pages, 4));
    E2S_TRY(need(lengths, 4));
    E2S_TRY(need(weights, 4));
    E2S_TRY(need(new_pages, 4));
    E2S_TRY(need(keep_idx, 4));
    E2S_TRY(need(new_len, 4));
    E2S_TRY(optional(weights_left_opt, 4));
    // the same table would move rows within the pages that other workgroups still read
    if (new_pages == pages) return E2S_ERR_BAD_PARAM;
    // the selection reads the weights several times while it writes the kept ones
    if (weights_left_opt == weights) return E2S_ERR_BAD_PARAM;
    // one key head's workgroup writes the new length while others read the old one
    if (new_len == lengths) return E2S_ERR_BAD_PARAM;
    return from_hip(e2s::launch_cache_evict(*cache, *shape, pages, lengths, weights, new_pages,
                                            keep_idx, new_len, weights_left_opt,
                                            static_cast<hipStream_t>(stream)));
}

}  // extern "C"
