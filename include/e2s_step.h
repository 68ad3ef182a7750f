/*
 * e2s_step.h - C ABI of what a layer's step takes beside the operators of e2s_serve.h:
 *
 *   norm_rotate   root-mean-square norms of every head's queries and keys and the rotation
 *                 of their positions in one pass, and the pass back to their gradients
 *   cache4_append, cache4_read, cache4_attend
 *                 a paged key/value cache held in 4 bits: new tokens - all, or the ones
 *                 e2s_prune kept - into it, its values out of it, and softmax attention of
 *                 queries against it
 *
 * The conventions and shape symbols of e2s_serve.h hold: device pointers the caller owns,
 * every argument checked on the host before anything is enqueued, no allocation, no
 * synchronisation, kernels only on `stream`, stateless and reentrant; calls that share a
 * workspace, an output or a written page are ordered by the caller; what lives in device
 * memory is bounded by the kernels.  Strides count elements unless said otherwise; a row
 * (the d elements of one token and head) is contiguous.  An output overlaps neither an
 * input nor another output unless its call says that it may.
 */
#ifndef E2S_STEP_H
#define E2S_STEP_H

#include "e2s_serve.h"

#ifdef __cplusplus
extern "C" {
#endif

#define E2S_STEP_ABI_VERSION 1

/* ---------------------------------------------------------------------------
 * Norms and positions.  For every row x of q and of k:
 *   y = turned(x r * w),  r = 1 / sqrt(mean(x^2) + eps)
 * with w the tensor's weight (d elements, all heads alike; 1 without one) and the rotation,
 * amplitude included, of e2s_rotate_positions.  Everything between the loads and the one
 * rounding of y is in 32 bits (squares too: a row with elements past 1e18 may give zeros),
 * angles as there.
 * ------------------------------------------------------------------------- */
typedef struct {
    int32_t batch;             /* B >= 1                                              */
    int32_t num_tokens;        /* T >= 0 (0: nothing to do); B*T < 2^24               */
    int32_t q_heads, k_heads;  /* >= 0, their sum >= 1; 0: that tensor is absent      */
    int32_t dtype;             /* an e2s_dtype, of the rows                           */
    int32_t weight_dtype;      /* of the weights: dtype, or E2S_DTYPE_F32             */
    float eps;                 /* > 0, finite                                         */
    int32_t reserved;          /* 0                                                   */
    int64_t q_stride[3], k_stride[3];          /* sequence, head, token of q and k     */
    int64_t q_grad_stride[3], k_grad_stride[3];  /* of the outputs' gradients (back only) */
    int64_t q_out_stride[3], k_out_stride[3];  /* of what is written, > 0 where the count
                                                  is above 1                           */
    int64_t pos_stride[3];     /* axis, sequence, token of positions, >= 0             */
} e2s_norm_rotate_shape;

/* q_out, k_out = q, k normed and turned by positions [axes, B, T] int32.  Rows may have any
 * alignment and stride that holds whole elements.  An output may be its input (the same
 * pointer and strides). */
E2S_API e2s_status e2s_norm_rotate(const e2s_norm_rotate_shape* shape, const e2s_rotary_plan* plan,
                                   const int32_t* positions, const void* q, const void* k,
                                   const void* q_weight_opt, const void* k_weight_opt,
                                   void* q_out, void* k_out, void* stream);

/* Bytes of device workspace e2s_norm_rotate_backward needs (host only; 0 where no weight's
 * gradient is asked for). */
E2S_API e2s_status e2s_norm_rotate_backward_workspace_size(const e2s_norm_rotate_shape* shape,
                                                           const e2s_rotary_plan* plan,
                                                           int32_t weight_grads, size_t* bytes);

/* The gradients of q, k (q_out, k_out, by q_out_stride, k_out_stride) and of the weights
 * ([d] of weight_dtype each, or NULL) from those of the outputs, q_grad and k_grad:
 *   g = turned back(grad), q_out = r (g w - x r mean(g w x r)), weight's = sum g x r
 * over all sequences, heads and tokens, in a fixed order and 32 bits.  A weight's gradient
 * without num_tokens or without its tensor's heads is zeros.  Outputs are neither inputs
 * nor one another.  workspace: 256-byte aligned, >= what the size call says for
 * weight_grads = 1 if a weight's gradient is asked for, else NULL. */
E2S_API e2s_status e2s_norm_rotate_backward(const e2s_norm_rotate_shape* shape,
                                            const e2s_rotary_plan* plan, const int32_t* positions,
                                            const void* q, const void* k, const void* q_weight_opt,
                                            const void* k_weight_opt, const void* q_grad,
                                            const void* k_grad, void* q_out, void* k_out,
                                            void* q_weight_grad_opt, void* k_weight_grad_opt,
                                            void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * The 4-bit cache.  Elements have one sign, two exponent and one mantissa bit: 0, 1/2, 1,
 * 3/2, 2, 3, 4 and 6, code 0 to 7, with the sign in bit 3.  Of a token and key head,
 *   the key has a scale for each block of 32 elements: a power of two 2^e, e >= -100, held
 *   as the byte e + 127 (0xFF: NaN), the smallest that holds the block's largest magnitude
 *   (6 * 2^e);
 *   the value has one bfloat16 scale, the smallest >= 2^-100 that holds the row's.
 * A held element is its code's value times the scale; codes are to nearest, ties to the even
 * code.  A block (key) or row (value) that holds a NaN or an infinity has a NaN scale: all
 * of it is NaN.
 *   Codes and scales that a caller writes itself are of these kinds: any code, exponent bytes 27
 * to 253 and 0xFF, value scales of 2^-100 and more or NaN.
 *   Tokens lie in pages as those of the 8-bit cache do.  A page holds, for every key head:
 *   k        [P, d/2]: byte i of a token: elements 2i (low half) and 2i + 1
 *   k_scale  [P/16, 4, d/32, 4]: [n, r, c, u]: block c of token 16 n + 4 u + r
 *   v        [P/32, d, 16]: byte i of [n, j]: element j of tokens 32 n + 2i (low half) and
 *            32 n + 2i + 1
 *   v_scale  [P]
 * the order in which the matrix instructions take them.
 * ------------------------------------------------------------------------- */
typedef struct {
    int32_t num_pages;      /* >= 1                                                   */
    int32_t page_tokens;    /* P: 32, 64 or 128                                       */
    int32_t num_kv_heads;   /* Hkv, 1 .. 128                                          */
    int32_t head_dim;       /* d: 64 or 128                                           */
    int64_t k_page_stride;  /* bytes from page to page, multiples of 16, at least     */
    int64_t v_page_stride;  /* Hkv*P*d/2                                              */
    void* k;                /* [num_pages, Hkv, P, d/2], 16-byte aligned              */
    void* v;                /* [num_pages, Hkv, P/32, d, 16], 16-byte aligned         */
    void* k_scale;          /* [num_pages, Hkv, P * d/32] bytes, 16-byte aligned      */
    void* v_scale;          /* [num_pages, Hkv, P] bfloat16, 16-byte aligned          */
} e2s_cache4;

/* New tokens into the cache, by e2s_cache_append's rules for k, v, pages, start, count_opt and
 * src_idx_opt.  A token's codes and scales do not depend on other tokens; no
 * other token of a page changes.  Neighbouring tokens share bytes: two calls that write
 * tokens of one page are ordered by the caller, and no two sequences of a call write tokens of
 * one page. */
E2S_API e2s_status e2s_cache4_append(const e2s_cache4* cache, const e2s_cache_append_shape* shape,
                                     const int32_t* pages, const int32_t* start,
                                     const int32_t* count_opt, const int32_t* src_idx_opt,
                                     const void* k, const void* v, void* stream);

typedef struct {
    int32_t batch;          /* B >= 1                                                 */
    int32_t num_tokens;     /* T >= 0: tokens per sequence at most                    */
    int32_t dtype;          /* an e2s_dtype, of k_out and v_out                       */
    int32_t max_pages;      /* >= 1                                                   */
    int64_t pages_stride;
    int64_t k_out_stride[3];   /* sequence, head, token; > 0 where the count is above 1 */
    int64_t v_out_stride[3];
} e2s_cache4_read_shape;

/* k_out, v_out [B, Hkv, T, d]: row j < count[b] of sequence b is the held key or value of
 * its token start[b] + j, rounded once to dtype (float32 holds it exactly, up to its range;
 * one past the range, which rounding up to a code can lead to, is an infinity); rows behind them
 * are left as they were.  A token before 0, past max_pages * P or whose page is outside
 * [0, num_pages) reads as zeros.  Base pointers and strides keep rows 16-byte aligned; either
 * output may be NULL. */
E2S_API e2s_status e2s_cache4_read(const e2s_cache4* cache, const e2s_cache4_read_shape* shape,
                                   const int32_t* pages, const int32_t* start,
                                   const int32_t* count_opt, void* k_out_opt, void* v_out_opt,
                                   void* stream);

typedef struct {
    int32_t batch;          /* B >= 1                                                 */
    int32_t num_heads;      /* H, a multiple of Hkv, 1 .. 128                         */
    int32_t num_queries;    /* T >= 1: queries per sequence at most                   */
    int32_t dtype;          /* an e2s_dtype, of q and out                             */
    int32_t max_tokens;     /* 1 .. 2^20: no length is larger (longer ones are cut)   */
    int32_t max_pages;      /* >= 1                                                   */
    int32_t causal;         /* 1: the queries are the sequence's last tokens; 0: every
                               query sees all                                         */
    float scale;            /* logit scale, 0 .. 1e38; 0 selects 1/sqrt(d)            */
    int64_t pages_stride;
    int64_t q_stride[3];    /* sequence, head, query                                  */
    int64_t out_stride[3];  /* > 0 where the count is above 1                         */
} e2s_cache4_attend_shape;

/* Bytes of device workspace e2s_cache4_attend needs (host only; may be 0). */
E2S_API e2s_status e2s_cache4_attend_workspace_size(const e2s_cache4* cache,
                                                    const e2s_cache4_attend_shape* shape,
                                                    size_t* bytes);

/* out = softmax(scale q . k) v over the cached tokens, with q, out, lengths, q_count_opt and
 * `causal` as in e2s_cache_attend: rows of out behind a sequence's queries are left as they
 * were, a query that sees no token gets zeros, a token whose page is outside [0, num_pages)
 * is seen by no query.
 * Logits, maxima, sums and the output accumulate in 32 bits.  A query is held as terms of 4
 * bits each on a scale of its largest element in 32: to 8, 12 or 24 bits of an element
 * (bf16, f16, f32), its own precision, or 2^-15, 2^-19 or 2^-31 of that largest one.  What
 * multiplies the values' codes - a softmax weight times the value's scale - is rounded to 12,
 * 16 or 24 bits, or 2^-19, 2^-23, 2^-31 of the largest among 128 tokens.  Values below 2^116
 * cannot overflow on the way; what adds less than 2^-100 may be lost.  A NaN in a held key
 * or value reaches the queries that see it and no other; a query that holds a NaN or an
 * infinity and sees a token gets NaN.
 * workspace: 256-byte aligned, >= e2s_cache4_attend_workspace_size bytes (NULL if 0). */
E2S_API e2s_status e2s_cache4_attend(const e2s_cache4* cache, const e2s_cache4_attend_shape* shape,
                                     const int32_t* pages, const int32_t* lengths,
                                     const int32_t* q_count_opt, const void* q, void* out,
                                     void* workspace, size_t workspace_bytes, void* stream);

/* E2S_STEP_ABI_VERSION of the built library. */
E2S_API int32_t e2s_step_abi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* E2S_STEP_H */
