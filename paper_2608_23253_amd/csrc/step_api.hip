// extern "C" entry points of e2s_step.h.  Each call validates every argument on the host
// before it touches the HIP runtime, then enqueues its kernels on the caller's stream.
#include "e2s_step.h"
#include "step_kernels.h"

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

}  // namespace

extern "C" {

int32_t e2s_step_abi_version(void) { return E2S_STEP_ABI_VERSION; }

e2s_status e2s_norm_rotate(const e2s_norm_rotate_shape* shape, const e2s_rotary_plan* plan,
                           const int32_t* positions, const void* q, const void* k,
                           const void* q_weight_opt, const void* k_weight_opt, void* q_out,
                           void* k_out, void* stream) {
    E2S_TRY(e2s::check_rotary_plan(plan));
    E2S_TRY(e2s::check_norm_rotate(shape, *plan, false));
    if (shape->num_tokens == 0) return E2S_OK;
    const size_t eb = static_cast<size_t>(e2s::elem_bytes(shape->dtype));
    const size_t wb = static_cast<size_t>(e2s::elem_bytes(shape->weight_dtype));
    E2S_TRY(need(positions, 4));
    const int64_t heads[2] = {shape->q_heads, shape->k_heads};
    const void* const src[2] = {q, k};
    const void* const weight[2] = {q_weight_opt, k_weight_opt};
    const void* const grad[2] = {nullptr, nullptr};
    void* const dst[2] = {q_out, k_out};
    void* const weight_grad[2] = {nullptr, nullptr};
    const int64_t* in[2] = {shape->q_stride, shape->k_stride};
    const int64_t* out[2] = {shape->q_out_stride, shape->k_out_stride};
    for (int w = 0; w < 2; ++w) {
        E2S_TRY(optional(weight[w], wb));
        if (heads[w] == 0) continue;
        E2S_TRY(need(src[w], eb));
        E2S_TRY(need(dst[w], eb));
        // an output in its input's place has its strides (where there is more than one index)
        const int64_t counts[3] = {shape->batch, heads[w], shape->num_tokens};
        for (int i = 0; i < 3; ++i)
            if (src[w] == dst[w] && counts[i] > 1 && in[w][i] != out[w][i])
                return E2S_ERR_BAD_PARAM;
    }
    // each output is written while the other tensor's rows are still read, or written
    if (heads[0] > 0 && heads[1] > 0 && (q_out == k_out || q_out == k || k_out == q))
        return E2S_ERR_BAD_PARAM;
    return from_hip(e2s::launch_norm_rotate(*shape, *plan, positions, src, weight, grad, dst,
                                            weight_grad, nullptr, false,
                                            static_cast<hipStream_t>(stream)));
}

e2s_status e2s_norm_rotate_backward_workspace_size(const e2s_norm_rotate_shape* shape,
                                                   const e2s_rotary_plan* plan,
                                                   int32_t weight_grads, size_t* bytes) {
    E2S_TRY(e2s::check_rotary_plan(plan));
    E2S_TRY(e2s::check_norm_rotate(shape, *plan, true));
    if (weight_grads != 0 && weight_grads != 1) return E2S_ERR_BAD_PARAM;
    if (bytes == nullptr) return E2S_ERR_NULL_POINTER;
    *bytes = e2s::norm_rotate_back_bytes(*shape, *plan, weight_grads != 0);
    return E2S_OK;
}

e2s_status e2s_norm_rotate_backward(const e2s_norm_rotate_shape* shape,
                                    const e2s_rotary_plan* plan, const int32_t* positions,
                                    const void* q, const void* k, const void* q_weight_opt,
                                    const void* k_weight_opt, const void* q_grad,
                                    const void* k_grad, void* q_out, void* k_out,
                                    void* q_weight_grad_opt, void* k_weight_grad_opt,
                                    void* workspace, size_t workspace_bytes, void* stream) {
    E2S_TRY(e2s::check_rotary_plan(plan));
    E2S_TRY(e2s::check_norm_rotate(shape, *plan, true));
    const size_t eb = static_cast<size_t>(e2s::elem_bytes(shape->dtype));
    const size_t wb = static_cast<size_t>(e2s::elem_bytes(shape->weight_dtype));
    const int64_t heads[2] = {shape->q_heads, shape->k_heads};
    const void* const src[2] = {q, k};
    const void* const weight[2] = {q_weight_opt, k_weight_opt};
    const void* const grad[2] = {q_grad, k_grad};
    void* const dst[2] = {q_out, k_out};
    void* const weight_grad[2] = {q_weight_grad_opt, k_weight_grad_opt};
    const void* ins[6];
    const void* outs[4];
    int n_in = 0, n_out = 0;
    for (int w = 0; w < 2; ++w) {
        E2S_TRY(optional(weight[w], wb));
        E2S_TRY(optional(weight_grad[w], wb));
        if (weight[w]) ins[n_in++] = weight[w];
        if (weight_grad[w]) outs[n_out++] = weight_grad[w];
    }
    if (shape->num_tokens > 0) {
        E2S_TRY(need(positions, 4));
        for (int w = 0; w < 2; ++w) {
            if (heads[w] == 0) continue;
            E2S_TRY(need(src[w], eb));
            E2S_TRY(need(grad[w], eb));
            E2S_TRY(need(dst[w], eb));
            ins[n_in++] = src[w];
            ins[n_in++] = grad[w];
            outs[n_out++] = dst[w];
        }
    }
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < n_in; ++j)
            if (outs[i] == ins[j]) return E2S_ERR_BAD_PARAM;
        for (int j = 0; j < i; ++j)
            if (outs[i] == outs[j]) return E2S_ERR_BAD_PARAM;
    }
    const size_t bytes = e2s::norm_rotate_back_bytes(
        *shape, *plan, q_weight_grad_opt != nullptr || k_weight_grad_opt != nullptr);
    if (bytes > 0) E2S_TRY(need(workspace, 256));
    if (workspace_bytes < bytes) return E2S_ERR_WORKSPACE_TOO_SMALL;
    return from_hip(e2s::launch_norm_rotate(*shape, *plan, positions, src, weight, grad, dst,
                                            weight_grad, workspace, true,
                                            static_cast<hipStream_t>(stream)));
}

e2s_status e2s_cache4_append(const e2s_cache4* cache, const e2s_cache_append_shape* shape,
                             const int32_t* pages, const int32_t* start, const int32_t* count_opt,
                             const int32_t* src_idx_opt, const void* k, const void* v,
                             void* stream) {
    E2S_TRY(e2s::check_cache4(cache));
    E2S_TRY(e2s::check_append4(*cache, shape));
    if (shape->num_tokens == 0) return E2S_OK;
    if (src_idx_opt == nullptr && shape->src_tokens < shape->num_tokens) return E2S_ERR_BAD_SHAPE;
    E2S_TRY(need(pages, 4));
    E2S_TRY(need(start, 4));
    E2S_TRY(optional(count_opt, 4));
    E2S_TRY(optional(src_idx_opt, 4));
    E2S_TRY(need(k, 16));
    E2S_TRY(need(v, 16));
    return from_hip(e2s::launch_cache4_append(*cache, *shape, pages, start, count_opt, src_idx_opt,
                                              k, v, static_cast<hipStream_t>(stream)));
}

e2s_status e2s_cache4_read(const e2s_cache4* cache, const e2s_cache4_read_shape* shape,
                           const int32_t* pages, const int32_t* start, const int32_t* count_opt,
                           void* k_out_opt, void* v_out_opt, void* stream) {
    E2S_TRY(e2s::check_cache4(cache));
    E2S_TRY(e2s::check_read4(*cache, shape));
    if (shape->num_tokens == 0) return E2S_OK;
    E2S_TRY(need(pages, 4));
    E2S_TRY(need(start, 4));
    E2S_TRY(optional(count_opt, 4));
    E2S_TRY(optional(k_out_opt, 16));
    E2S_TRY(optional(v_out_opt, 16));
    if (k_out_opt == nullptr && v_out_opt == nullptr) return E2S_ERR_NULL_POINTER;
    if (k_out_opt == v_out_opt) return E2S_ERR_BAD_PARAM;
    return from_hip(e2s::launch_cache4_read(*cache, *shape, pages, start, count_opt, k_out_opt,
                                            v_out_opt, static_cast<hipStream_t>(stream)));
}

e2s_status e2s_cache4_attend_workspace_size(const e2s_cache4* cache,
                                            const e2s_cache4_attend_shape* shape, size_t* bytes) {
    E2S_TRY(e2s::check_cache4(cache));
    E2S_TRY(e2s::check_attend4(*cache, shape));
    if (bytes == nullptr) return E2S_ERR_NULL_POINTER;
    *bytes = e2s::attend4_plan(*cache, *shape).bytes;
    return E2S_OK;
}

e2s_status e2s_cache4_attend(const e2s_cache4* cache, const e2s_cache4_attend_shape* shape,
                             const int32_t* pages, const int32_t* lengths,
                             const int32_t* q_count_opt, const void* q, void* out,
                             void* workspace, size_t workspace_bytes, void* stream) {
    E2S_TRY(e2s::check_cache4(cache));
    E2S_TRY(e2s::check_attend4(*cache, shape));
    E2S_TRY(need(pages, 4));
    E2S_TRY(need(lengths, 4));
    E2S_TRY(optional(q_count_opt, 4));
    E2S_TRY(need(q, 16));
    E2S_TRY(need(out, 16));
    const size_t bytes = e2s::attend4_plan(*cache, *shape).bytes;
    if (bytes > 0) E2S_TRY(need(workspace, 256));
    if (workspace_bytes < bytes) return E2S_ERR_WORKSPACE_TOO_SMALL;
    // other workgroups still read queries when the first outputs are there
    if (out == q) return E2S_ERR_BAD_PARAM;
    return from_hip(e2s::launch_cache4_attend(*cache, *shape, pages, lengths, q_count_opt, q, out,
                                              workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
