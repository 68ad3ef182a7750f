/*
 * e2s_serve.h - C ABI of the operators on either side of the scoring path (e2s.h):
 * what encodes the positions of its queries and keys, where the kept tokens' keys and
 * values go, what attends to them while the model answers, and what shortens them again.
 *
 *   rotate   rotary positions of queries and keys (before the path)
 *   append   new tokens - all, or the ones e2s_prune kept - quantised into a paged
 *            8-bit key/value cache with a scale for each block of tokens and head
 *   attend   softmax attention of queries against the cached tokens, and the weight
 *            that every cached token received
 *   evict    the tokens of largest accumulated weight moved to fewer pages
 *
 * The conventions of e2s.h hold: device pointers the caller owns, every argument
 * checked on the host before anything is enqueued, no allocation, no synchronisation,
 * kernels only on `stream` (so every call can be captured in a graph), stateless and
 * reentrant; calls that share a workspace, an output or a written page are ordered by
 * the caller.  What lives in device memory (page tables, lengths, positions, indices)
 * cannot be checked on the host: the kernels bound every access by it, as stated
 * below, so a bad entry gives wrong or missing values and no fault.
 *
 * Shape symbols: B sequences, H query heads, Hkv key heads (query head h reads key head
 * floor(h*Hkv/H)), T new tokens or queries per sequence, d head_dim, P tokens per page.
 * Strides count elements; a row (the d elements of one token and head) is contiguous.
 * An output overlaps neither an input nor another output unless its call says that it may.
 */
#ifndef E2S_SERVE_H
#define E2S_SERVE_H

#include "e2s.h"

#ifdef __cplusplus
extern "C" {
#endif

#define E2S_SERVE_ABI_VERSION 1

/* ---------------------------------------------------------------------------
 * Rotary positions.  Pair j of the R/2 pairs in a row's first R elements is turned by
 * the angle p * f_j, p the token's position: (x0, x1) -> A (x0 cos - x1 sin,
 * x0 sin + x1 cos).  The other d - R elements are copied.  f_j = base^(-2j/R), scaled
 * for contexts longer than the model was trained on:
 *   LINEAR  f_j / factor
 *   BASE    base * factor^(R/(R-2)) in place of base (R = 2: base)
 *   RAMP    by the turns r_j = original_len * f_j / (2 pi) that a pair makes over the
 *           original context: f_j / factor up to `low` turns, f_j from `high` turns on,
 *           linear in r_j between them.  (Some implementations ramp linearly in the
 *           pair's number j between the pairs of those turns.  A model trained so has other
 *           frequencies in between, which no scaling here gives.)
 * Angles are reduced in 64 bits, so positions up to 2^31 keep the digits of their
 * angle; sine and cosine are those of a 32-bit angle within one turn.
 * ------------------------------------------------------------------------- */
#define E2S_ROTARY_MAX_PAIRS 128

typedef enum { E2S_ROTARY_HALF = 0,          /* pair j: elements j and j + R/2  */
               E2S_ROTARY_INTERLEAVED = 1    /* pair j: elements 2j and 2j + 1  */
} e2s_rotary_layout;

typedef enum { E2S_ROTARY_NONE = 0, E2S_ROTARY_LINEAR = 1, E2S_ROTARY_BASE = 2,
               E2S_ROTARY_RAMP = 3 } e2s_rotary_scaling;

typedef struct {
    int32_t head_dim;      /* d, 2 .. 256                                             */
    int32_t rot_dim;       /* R, even, 2 .. d                                         */
    int32_t layout;        /* an e2s_rotary_layout                                    */
    int32_t scaling;       /* an e2s_rotary_scaling                                   */
    int32_t sections[3];   /* all 0: one position per token; else the number of pairs,
                              in order, that turn by each of three positions (e.g.
                              time, row and column of a visual token); their sum is R/2 */
    int32_t reserved;      /* 0                                                       */
    double amplitude;      /* A, finite, > 0; 0 selects 1 (RAMP: 0.1 ln(factor) + 1)  */
    double base;           /* > 1, finite                                             */
    double factor;         /* >= 1, finite; ignored by NONE                           */
    double original_len;   /* RAMP: > 0, finite                                       */
    double low, high;      /* RAMP: 0 <= low < high, finite, in turns                 */
} e2s_rotary_spec;

/* Filled by e2s_rotary_plan_init; kept by the caller and passed to every call. */
typedef struct {
    int32_t head_dim, rot_dim, layout, axes;   /* axes: 1 or 3 positions per token    */
    float amplitude;
    int32_t reserved;
    uint8_t axis[E2S_ROTARY_MAX_PAIRS];        /* pair j's axis                       */
    double turns[E2S_ROTARY_MAX_PAIRS];        /* f_j / (2 pi): turns per position    */
} e2s_rotary_plan;

/* Host only: checks `spec` and fills `plan`. */
E2S_API e2s_status e2s_rotary_plan_init(const e2s_rotary_spec* spec, e2s_rotary_plan* plan);

typedef struct {
    int32_t batch;             /* B >= 1                                              */
    int32_t num_tokens;        /* T >= 0 (0: nothing to do); B*T < 2^24               */
    int32_t q_heads, k_heads;  /* >= 0, their sum >= 1; 0: that tensor is absent      */
    int32_t dtype;             /* an e2s_dtype                                        */
    int32_t inverse;           /* 1: turns back by -p f_j, still times A: the
                                  transpose, which takes the gradient of the outputs to
                                  that of the inputs                                   */
    int64_t q_stride[3], k_stride[3];          /* sequence, head, token of q and k     */
    int64_t q_out_stride[3], k_out_stride[3];  /* the same of the outputs, > 0 where
                                                  the count is above 1                 */
    int64_t pos_stride[3];     /* axis, sequence, token of positions, >= 0; 0 where
                                  all share one                                        */
} e2s_rotary_shape;

/* q_out, k_out = q, k turned by positions [axes, B, T] int32 (negative ones allowed).
 * Rows may have any alignment and stride that holds whole elements.  An output may be
 * its input (the same pointer and strides) and must not overlap it otherwise. */
E2S_API e2s_status e2s_rotate_positions(const e2s_rotary_shape* shape,
                                        const e2s_rotary_plan* plan, const int32_t* positions,
                                        const void* q, const void* k, void* q_out, void* k_out,
                                        void* stream);

/* ---------------------------------------------------------------------------
 * The 8-bit cache.  A page holds one block of P consecutive tokens of a sequence: for
 * every key head the P keys and the P values as e4m3 bytes (4 exponent and 3 mantissa
 * bits, no infinities, largest value 448), and a scale for the keys and one for the
 * values of that block and head.  A held value is byte * scale.
 *   Scales are powers of two, 2^e with e >= -100 the smallest that holds the block's
 * largest finite value (448 * 2^e).  So a block whose maximum grows as tokens are
 * appended, and rows that eviction regroups into other blocks, are rescaled exactly but
 * for values under 2^-13 of the block's maximum, below e4m3's normal range.  NaN
 * stays NaN; infinities are held as NaN.  Elements from 248 * 2^120 on (3.3e38) are held as
 * 2^128.  A scale that the caller writes has to be a power of two in 2^-100 .. 2^120, too:
 * attention reads its exponent alone.
 *   A sequence's tokens lie in the pages that its row of a page
 * table [B, max_pages] int32 names: token n in page pages[b, n / P], row n % P.  A page
 * belongs to one sequence while it is written.
 * ------------------------------------------------------------------------- */
typedef struct {
    int32_t num_pages;      /* >= 1                                                   */
    int32_t page_tokens;    /* P: 16, 32, 64 or 128                                   */
    int32_t num_kv_heads;   /* Hkv, 1 .. 128                                          */
    int32_t head_dim;       /* d: 64 or 128                                           */
    int64_t k_page_stride;  /* bytes from page to page, multiples of 16, at least     */
    int64_t v_page_stride;  /* Hkv*P*d                                                */
    void* k;                /* [num_pages, Hkv, P, d] e4m3, 16-byte aligned           */
    void* v;
    float* k_scale;         /* [num_pages, Hkv] f32                                   */
    float* v_scale;
} e2s_cache;

typedef struct {
    int32_t batch;          /* B >= 1                                                 */
    int32_t num_tokens;     /* T >= 0: new tokens per sequence at most                */
    int32_t src_tokens;     /* N >= 1: tokens per sequence in k and v (T without
                               src_idx)                                               */
    int32_t dtype;          /* an e2s_dtype, of k and v                               */
    int32_t max_pages;      /* >= 1                                                   */
    int32_t reserved;       /* 0                                                      */
    int64_t pages_stride;   /* between the sequences' rows of the page table          */
    int64_t k_stride[3];    /* sequence, head, token                                  */
    int64_t v_stride[3];
} e2s_cache_append_shape;

/* Token j < count[b] of sequence b becomes its cached token start[b] + j:
 *   k, v      [B, Hkv, N, d]; base pointers and strides keep rows 16-byte aligned
 *   pages     [B, max_pages] int32; start [B] int32: tokens cached before the call
 *   count_opt [B] int32 or NULL (all T), cut to 0 .. T
 *   src_idx_opt [B, T] int32 or NULL: token j is row src_idx[b, j] of k and v (e.g.
 *             e2s_prune's keep_idx), row j without it; an index outside [0, N) appends
 *             zeros
 * Tokens past max_pages * P, tokens whose page is outside [0, num_pages) and sequences
 * of a negative start are not written.  Rows of a page before start[b] keep their values
 * (rescaled where the block's scale grows), rows behind the new tokens their bytes. */
E2S_API e2s_status e2s_cache_append(const e2s_cache* cache, const e2s_cache_append_shape* shape,
                                    const int32_t* pages, const int32_t* start,
                                    const int32_t* count_opt, const int32_t* src_idx_opt,
                                    const void* k, const void* v, void* stream);

typedef struct {
    int32_t batch;          /* B >= 1                                                 */
    int32_t num_heads;      /* H, a multiple of Hkv, 1 .. 128                         */
    int32_t num_queries;    /* T >= 1: queries per sequence at most                   */
    int32_t dtype;          /* an e2s_dtype, of q and out                             */
    int32_t max_tokens;     /* 1 .. 2^20: no length is larger (longer ones are cut)   */
    int32_t max_pages;      /* >= 1                                                   */
    int32_t causal;         /* 1: the queries are the sequence's last tokens; 0: every
                               query sees all                                         */
    int32_t weights;        /* 1: weights_out is given; sizes the workspace           */
    float scale;            /* logit scale, 0 .. 1e38; 0 selects 1/sqrt(d)            */
    int32_t reserved;       /* 0                                                      */
    int64_t pages_stride;
    int64_t q_stride[3];    /* sequence, head, query                                  */
    int64_t out_stride[3];  /* > 0 where the count is above 1                         */
    int64_t weights_in_stride[2], weights_out_stride[2];   /* sequence, head          */
} e2s_cache_attend_shape;

/* Bytes of device workspace e2s_cache_attend needs (host only; may be 0). */
E2S_API e2s_status e2s_cache_attend_workspace_size(const e2s_cache* cache,
                                                   const e2s_cache_attend_shape* shape,
                                                   size_t* bytes);

/* out = softmax(scale q . k) v over the cached tokens.
 *   q, out   [B, H, T, d]; base pointers and strides keep rows 16-byte aligned; out is
 *            not q
 *   lengths  [B] int32: cached tokens, the queries' own among them (cut to 0 ..
 *            min(max_tokens, max_pages * P))
 *   q_count_opt [B] int32 or NULL (all T): sequence b's queries, cut to 0 .. T; rows of
 *            out behind them are left as they were
 * With `causal`, query t of c sees the first len - (c - 1 - t) tokens.  A query that sees
 * none gets zeros.  A token whose page is outside [0, num_pages) is seen by no query.
 *   weights_out_opt [B, Hkv, >= max_tokens] f32 or NULL: for n < len, weights_in[b, h, n]
 *            (0 where weights_in_opt is NULL) plus the softmax weight of token n summed
 *            over the queries and the query heads of key head h, in a fixed order;
 *            entries from len on are left as they were.  It may be weights_in itself,
 *            with its strides.
 * Logits, maxima, sums and the output accumulate in 32 bits; the weights that multiply
 * the values are rounded to 16 bits (bf16 and f16 q) or 24 bits (f32).  The sums are divided
 * by the weights' at the end: values below 2^116 cannot overflow on the way, and what adds
 * less than 2^-110 may be lost.
 * workspace: 256-byte aligned, >= e2s_cache_attend_workspace_size bytes (NULL if 0),
 * contents undefined on return.  A NaN in a held key or value reaches the queries that
 * see it and no other. */
E2S_API e2s_status e2s_cache_attend(const e2s_cache* cache, const e2s_cache_attend_shape* shape,
                                    const int32_t* pages, const int32_t* lengths,
                                    const int32_t* q_count_opt, const void* q, void* out,
                                    const float* weights_in_opt, float* weights_out_opt,
                                    void* workspace, size_t workspace_bytes, void* stream);

typedef struct {
    int32_t batch;              /* B >= 1                                             */
    int32_t max_tokens;         /* 1 .. 2^20, as in e2s_cache_attend_shape            */
    int32_t budget;             /* K >= 1 tokens kept at most, K <= new_max_pages * P */
    int32_t sinks, recent;      /* >= 0, sum <= K: first and last tokens always kept  */
    int32_t max_pages, new_max_pages;   /* >= 1                                       */
    int32_t left_tokens;        /* W >= K: width of weights_left                      */
    int64_t pages_stride, new_pages_stride;
    int64_t weights_stride[2], left_stride[2];   /* sequence, head                    */
} e2s_cache_evict_shape;

/* Every (sequence, key head) keeps min(len, K) of its len tokens: the first `sinks`, the
 * last `recent`, and of the others those of largest weight (equal weights: the earlier
 * token; NaN after all others), in their order.
 *   weights   [B, Hkv, >= max_tokens] f32
 *   keep_idx  [B, Hkv, K] int32 out: the kept tokens, ascending, then -1
 *   new_len   [B] int32 out: min(len, K); not lengths itself
 *   weights_left_opt [B, Hkv, W] f32 out or NULL: the kept tokens' weights, then zeros
 * The kept rows go to the pages of new_pages [B, new_max_pages], which must not be among
 * the sequences' present pages; each new block gets its own scale.  A kept row whose page
 * is outside [0, num_pages) becomes zeros; a new page outside it is not written. */
E2S_API e2s_status e2s_cache_evict(const e2s_cache* cache, const e2s_cache_evict_shape* shape,
                                   const int32_t* pages, const int32_t* lengths,
                                   const float* weights, const int32_t* new_pages,
                                   int32_t* keep_idx, int32_t* new_len, float* weights_left_opt,
                                   void* stream);

/* E2S_SERVE_ABI_VERSION of the built library. */
E2S_API int32_t e2s_serve_abi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* E2S_SERVE_H */
