// Host-side argument checks of e2s_step.h (see step_validate.h).
#include "step_validate.h"

#include <algorithm>
#include <cmath>
#include <limits>

namespace e2s {
namespace {

constexpr double kBig = static_cast<double>(std::numeric_limits<int64_t>::max() / 16);
constexpr int64_t kMaxStride = std::numeric_limits<int64_t>::max() / 64;
constexpr double kItems = 4294967296.0;          // work-items of a launch
constexpr int64_t kSimds = 1024;                 // 256 compute units of 4

#define E2S_TRY_(expr)                         \
    do {                                       \
        const e2s_status st__ = (expr);        \
        if (st__ != E2S_OK) return st__;       \
    } while (0)

}  // namespace

e2s_status check_norm_rotate(const e2s_norm_rotate_shape* s, const e2s_rotary_plan& p, bool back) {
    if (s == nullptr) return E2S_ERR_NULL_POINTER;
    if (s->batch < 1 || s->num_tokens < 0 || s->q_heads < 0 || s->k_heads < 0 ||
        s->q_heads + static_cast<int64_t>(s->k_heads) < 1)
        return E2S_ERR_BAD_SHAPE;
    if (!known_dtype(s->dtype) || s->reserved != 0) return E2S_ERR_BAD_PARAM;
    if (s->weight_dtype != s->dtype && s->weight_dtype != E2S_DTYPE_F32) return E2S_ERR_BAD_PARAM;
    if (!std::isfinite(s->eps) || !(s->eps > 0.0f)) return E2S_ERR_BAD_PARAM;
    // one workgroup of 256 threads takes at least one token of a sequence
    if (static_cast<double>(s->batch) * s->num_tokens >= 16777216.0) return E2S_ERR_UNSUPPORTED;
    if (s->q_heads > 65535 || s->k_heads > 65535) return E2S_ERR_UNSUPPORTED;
    const int eb = elem_bytes(s->dtype);
    const int64_t heads[2] = {s->q_heads, s->k_heads};
    const int64_t* in[2] = {s->q_stride, s->k_stride};
    const int64_t* grad[2] = {s->q_grad_stride, s->k_grad_stride};
    const int64_t* out[2] = {s->q_out_stride, s->k_out_stride};
    for (int w = 0; w < 2; ++w) {
        if (heads[w] == 0) continue;
        const int64_t counts[3] = {s->batch, heads[w], s->num_tokens};
        E2S_TRY_(check_strides(in[w], counts, 3, p.head_dim, 0, 0, eb));
        if (back) E2S_TRY_(check_strides(grad[w], counts, 3, p.head_dim, 0, 0, eb));
        E2S_TRY_(check_strides(out[w], counts, 3, p.head_dim, 1, 0, eb));
    }
    const int64_t counts[3] = {p.axes, s->batch, s->num_tokens};
    return check_strides(s->pos_stride, counts, 3, 1, 0, 0, 4);
}

size_t norm_rotate_back_bytes(const e2s_norm_rotate_shape& s, const e2s_rotary_plan& p,
                              bool weight_grads) {
    if (!weight_grads || s.num_tokens == 0) return 0;
    const int64_t parts =
        std::min<int64_t>(kNormMostParts, static_cast<int64_t>(s.batch) * s.num_tokens);
    return static_cast<size_t>(parts) * 2 * p.head_dim * sizeof(float);
}

e2s_status check_cache4(const e2s_cache4* c) {
    if (c == nullptr) return E2S_ERR_NULL_POINTER;
    if (c->num_pages < 1 || c->num_kv_heads < 1 || c->head_dim < 1 || c->page_tokens < 1)
        return E2S_ERR_BAD_SHAPE;
    if (c->num_kv_heads > kMaxHeads) return E2S_ERR_UNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128) return E2S_ERR_UNSUPPORTED;
    if (c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128)
        return E2S_ERR_UNSUPPORTED;
    const int64_t page = static_cast<int64_t>(c->num_kv_heads) * c->page_tokens * c->head_dim / 2;
    const int64_t strides[2] = {c->k_page_stride, c->v_page_stride};
    for (int64_t st : strides) {
        if (st < page || st > kMaxStride) return E2S_ERR_BAD_SHAPE;
        if (st % 16 != 0) return E2S_ERR_MISALIGNED;
        if (static_cast<double>(st) * c->num_pages > kBig) return E2S_ERR_BAD_SHAPE;
    }
    const void* all[4] = {c->k, c->v, c->k_scale, c->v_scale};
    for (const void* p : all)
        if (p == nullptr) return E2S_ERR_NULL_POINTER;
    for (const void* p : all) E2S_TRY_(check_aligned(p, 16));
    return E2S_OK;
}

e2s_status check_append4(const e2s_cache4& c, const e2s_cache_append_shape* s) {
    if (s == nullptr) return E2S_ERR_NULL_POINTER;
    if (s->batch < 1 || s->num_tokens < 0 || s->src_tokens < 1) return E2S_ERR_BAD_SHAPE;
    if (!known_dtype(s->dtype) || s->reserved != 0) return E2S_ERR_BAD_PARAM;
    if (s->num_tokens > kMaxCachedTokens) return E2S_ERR_UNSUPPORTED;
    E2S_TRY_(check_table(s->batch, s->max_pages, s->pages_stride));
    const int eb = elem_bytes(s->dtype);
    const int64_t counts[3] = {s->batch, c.num_kv_heads, s->src_tokens};
    E2S_TRY_(check_strides(s->k_stride, counts, 3, c.head_dim, 0, 16 / eb, eb));
    E2S_TRY_(check_strides(s->v_stride, counts, 3, c.head_dim, 0, 16 / eb, eb));
    // one workgroup of at most 256 threads per (sequence, head, touched group of 32 tokens)
    const double groups = static_cast<double>(s->num_tokens) / kGroup4 + 2.0;
    if (static_cast<double>(s->batch) * c.num_kv_heads * groups * 256.0 >= kItems)
        return E2S_ERR_UNSUPPORTED;
    return E2S_OK;
}

e2s_status check_read4(const e2s_cache4& c, const e2s_cache4_read_shape* s) {
    if (s == nullptr) return E2S_ERR_NULL_POINTER;
    if (s->batch < 1 || s->num_tokens < 0) return E2S_ERR_BAD_SHAPE;
    if (!known_dtype(s->dtype)) return E2S_ERR_BAD_PARAM;
    if (s->num_tokens > kMaxCachedTokens) return E2S_ERR_UNSUPPORTED;
    E2S_TRY_(check_table(s->batch, s->max_pages, s->pages_stride));
    const int eb = elem_bytes(s->dtype);
    const int64_t counts[3] = {s->batch, c.num_kv_heads, s->num_tokens};
    E2S_TRY_(check_strides(s->k_out_stride, counts, 3, c.head_dim, 1, 16 / eb, eb));
    E2S_TRY_(check_strides(s->v_out_stride, counts, 3, c.head_dim, 1, 16 / eb, eb));
    const double groups = static_cast<double>(s->num_tokens) / kGroup4 + 2.0;
    if (static_cast<double>(s->batch) * c.num_kv_heads * groups * 256.0 >= kItems)
        return E2S_ERR_UNSUPPORTED;
    return E2S_OK;
}

e2s_status check_attend4(const e2s_cache4& c, const e2s_cache4_attend_shape* s) {
    if (s == nullptr) return E2S_ERR_NULL_POINTER;
    if (s->batch < 1 || s->num_heads < 1 || s->num_queries < 1 || s->max_tokens < 1)
        return E2S_ERR_BAD_SHAPE;
    if (s->num_heads % c.num_kv_heads != 0) return E2S_ERR_BAD_SHAPE;
    if (!known_dtype(s->dtype)) return E2S_ERR_BAD_PARAM;
    if (s->causal != 0 && s->causal != 1) return E2S_ERR_BAD_PARAM;
    // (finite in log2 as well, and twice that)
    if (!(s->scale >= 0.0f && s->scale <= std::numeric_limits<float>::max() / 3.0f))
        return E2S_ERR_BAD_PARAM;
    if (s->num_heads > kMaxHeads || s->max_tokens > kMaxCachedTokens ||
        s->num_queries > kMaxCachedTokens)
        return E2S_ERR_UNSUPPORTED;
    E2S_TRY_(check_table(s->batch, s->max_pages, s->pages_stride));
    const int eb = elem_bytes(s->dtype);
    const int64_t counts[3] = {s->batch, s->num_heads, s->num_queries};
    E2S_TRY_(check_strides(s->q_stride, counts, 3, c.head_dim, 0, 16 / eb, eb));
    E2S_TRY_(check_strides(s->out_stride, counts, 3, c.head_dim, 1, 16 / eb, eb));
    // Fewer than 2^24 rows in all, before the plan's products of rows and tokens, which 63
    // bits hold then.
    const double heads = static_cast<double>(s->batch) * c.num_kv_heads;
    const double rows = static_cast<double>(s->num_heads / c.num_kv_heads) * s->num_queries;
    if (heads * rows * 256.0 >= kItems) return E2S_ERR_UNSUPPORTED;
    const Attend4Plan p = attend4_plan(c, *s);
    if (heads * p.row_groups * p.splits * 64 * p.waves >= kItems) return E2S_ERR_UNSUPPORTED;
    if (heads * p.rows * (static_cast<double>(p.splits) * (c.head_dim + 2)) * 4.0 > kBig)
        return E2S_ERR_BAD_SHAPE;
    return E2S_OK;
}

Attend4Plan attend4_plan(const e2s_cache4& c, const e2s_cache4_attend_shape& s) {
    Attend4Plan p{};
    const int64_t B = s.batch, G = c.num_kv_heads, D = c.head_dim;
    p.rows = static_cast<int64_t>(s.num_heads) / G * s.num_queries;
    p.row_groups = (p.rows + 15) / 16;
    const int64_t units = B * G * p.row_groups;
    // The device holds 2048 waves at two to a SIMD.  Times of one query of 7 heads to each of 4
    // key heads, d = 128, bf16, by units and longest length; "even": all sequences as long,
    // "ragged": any length up to it.
    //   Eight waves, which have all keys of a unit, for few short sequences: at 16 x 1100 9.1 us
    // against 9.9 in parts and joined, at 128 x 1100 9.4 and 11.7, at 252 x 2048 16.6 and 18.7; at
    // 64 x 2048 11.3 and 10.1.  Beyond 2048 keys they lose (64 x 4096: 17.1 and 14.3) until the
    // units fill the device (252 x 4096: 25.5 and 30.6); at 256 x 1100 and x 2048 eight would
    // still be ahead (10.8 for 17.2, 16.7 for 19.2).
    //   One wave from 2048 units on: 2048 x 1100 even 51 us, of two waves 55, of four 59; ragged
    // 36, 35, 40; x 4096 even 198, 206, 199; ragged 139, 123, 115.
    //   Between, parts: workgroups of four or two waves, until there are three or four waves to a
    // SIMD, more than fit.  16 units of up to 131072 ragged keys take 35 us with three of four
    // (two 37, four 44, workgroups of two 43), 1344 units (16 sequences of up to 4200 keys and 48
    // queries, ragged counts) 38 with four of two (three 45, workgroups of four 52).  Neither
    // number holds everywhere, as whole steps of 128 keys round a wave's share: at 384 x 4096 even
    // three of four are best (38.6; two 43.7, four 41.6), at 508 x 4096 two of four are (44; three
    // 56), at 1024 x 2048 even two of two (45; four 54) and at 1536 x 4096 two of four (150; four
    // of two 188); at 1024 x 512 ragged four of two take 23, two 12.5, one wave 12.9.  A cut by the
    // lengths that a call has would need neither.
    if (units < 256 && s.max_tokens <= 2048) p.waves = 8;
    else p.waves = units < 512 ? 4 : units < 2048 ? 2 : 1;
    const int64_t unit = static_cast<int64_t>(kStep4) * p.waves;
    int64_t per = s.max_tokens;
    const int64_t waves = (p.waves == 2 ? 4 : 3) * kSimds;
    if (p.waves == 2 || p.waves == 4) per = (s.max_tokens * units * p.waves + waves - 1) / waves;
    p.chunk = (per + unit - 1) / unit * unit;
    p.splits = (s.max_tokens + p.chunk - 1) / p.chunk;
    const size_t all = static_cast<size_t>(B * G * p.rows);
    size_t at = 0;
    auto region = [&](size_t floats) {
        const size_t here = at;
        at += align_up(floats * sizeof(float), 256);
        return here;
    };
    const size_t parts = p.splits > 1 ? static_cast<size_t>(p.splits) : 0;
    p.max_off = region(all * parts);
    p.sum_off = region(all * parts);
    p.part_off = region(all * parts * D);
    p.bytes = at;
    return p;
}

}  // namespace e2s
