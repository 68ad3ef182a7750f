// Host-side argument checks of e2s_serve.h (see serve_validate.h).
#include "serve_validate.h"

#include <algorithm>
#include <cmath>
#include <limits>

namespace e2s {
namespace {

constexpr double kBig = static_cast<double>(std::numeric_limits<int64_t>::max() / 16);
constexpr int64_t kMaxStride = std::numeric_limits<int64_t>::max() / 64;

}  // namespace

bool known_dtype(int32_t t) {
    return t == E2S_DTYPE_F32 || t == E2S_DTYPE_BF16 || t == E2S_DTYPE_F16;
}

// Strides of an input (`least` 0) or of an output (1, asked only where the count is above
// one): within range, whole 16-byte rows where `align` is given (elements per 16 bytes; a
// stride that only index 0 takes may be anything), and the last row's end addressable.
e2s_status check_strides(const int64_t* st, const int64_t* counts, int n, int64_t row, int least,
                         int64_t align, int bytes) {
    double end = static_cast<double>(row);
    for (int i = 0; i < n; ++i) {
        if (st[i] < 0 || st[i] > kMaxStride) return E2S_ERR_BAD_SHAPE;
        if (counts[i] > 1 && st[i] < least) return E2S_ERR_BAD_SHAPE;
        if (align > 0 && counts[i] > 1 && st[i] % align != 0) return E2S_ERR_MISALIGNED;
        if (counts[i] > 1)
            end += static_cast<double>(counts[i] - 1) * static_cast<double>(st[i]);
    }
    return end * bytes > kBig ? E2S_ERR_BAD_SHAPE : E2S_OK;
}

#define E2S_TRY_(expr)                         \
    do {                                       \
        const e2s_status st__ = (expr);        \
        if (st__ != E2S_OK) return st__;       \
    } while (0)

e2s_status check_rotary_spec(const e2s_rotary_spec* s) {
    if (s == nullptr) return E2S_ERR_NULL_POINTER;
    if (s->head_dim < 2 || s->rot_dim < 2 || s->rot_dim % 2 != 0 || s->rot_dim > s->head_dim)
        return E2S_ERR_BAD_SHAPE;
    if (s->head_dim > 2 * E2S_ROTARY_MAX_PAIRS) return E2S_ERR_UNSUPPORTED;
    if (s->layout != E2S_ROTARY_HALF && s->layout != E2S_ROTARY_INTERLEAVED)
        return E2S_ERR_BAD_PARAM;
    if (s->scaling < E2S_ROTARY_NONE || s->scaling > E2S_ROTARY_RAMP) return E2S_ERR_BAD_PARAM;
    if (s->reserved != 0) return E2S_ERR_BAD_PARAM;
    int64_t sum = 0;
    for (int32_t n : s->sections) {
        if (n < 0) return E2S_ERR_BAD_SHAPE;
        sum += n;
    }
    if (sum != 0 && sum != s->rot_dim / 2) return E2S_ERR_BAD_SHAPE;
    if (!std::isfinite(s->amplitude) || s->amplitude < 0.0 ||
        s->amplitude > std::numeric_limits<float>::max())
        return E2S_ERR_BAD_PARAM;
    if (!std::isfinite(s->base) || s->base <= 1.0) return E2S_ERR_BAD_PARAM;
    if (s->scaling != E2S_ROTARY_NONE && (!std::isfinite(s->factor) || s->factor < 1.0))
        return E2S_ERR_BAD_PARAM;
    if (s->scaling == E2S_ROTARY_RAMP) {
        if (!std::isfinite(s->original_len) || s->original_len <= 0.0) return E2S_ERR_BAD_PARAM;
        if (!std::isfinite(s->low) || !std::isfinite(s->high) || s->low < 0.0 || s->high <= s->low)
            return E2S_ERR_BAD_PARAM;
    }
    return E2S_OK;
}

void fill_rotary_plan(const e2s_rotary_spec& s, e2s_rotary_plan* p) {
    const double two_pi = 6.283185307179586476925287;
    const int R = s.rot_dim, pairs = R / 2;
    *p = e2s_rotary_plan{};
    p->head_dim = s.head_dim;
    p->rot_dim = R;
    p->layout = s.layout;
    const bool one = s.sections[0] + s.sections[1] + s.sections[2] == 0;
    p->axes = one ? 1 : 3;
    double base = s.base;
    if (s.scaling == E2S_ROTARY_BASE && R > 2)
        base *= std::pow(s.factor, static_cast<double>(R) / (R - 2));
    for (int j = 0; j < pairs; ++j) {
        double f = std::pow(base, -2.0 * j / R);
        if (s.scaling == E2S_ROTARY_LINEAR) f /= s.factor;
        if (s.scaling == E2S_ROTARY_RAMP) {
            const double r = s.original_len * f / two_pi;
            const double g = std::min(1.0, std::max(0.0, (r - s.low) / (s.high - s.low)));
            f = (1.0 - g) * (f / s.factor) + g * f;
        }
        p->turns[j] = f / two_pi;
        p->axis[j] = one ? 0 : j < s.sections[0] ? 0 : j < s.sections[0] + s.sections[1] ? 1 : 2;
    }
    double a = s.amplitude;
    if (a == 0.0) a = s.scaling == E2S_ROTARY_RAMP ? 0.1 * std::log(s.factor) + 1.0 : 1.0;
    p->amplitude = static_cast<float>(a);
}

e2s_status check_rotary_plan(const e2s_rotary_plan* p) {
    if (p == nullptr) return E2S_ERR_NULL_POINTER;
    if (p->head_dim < 2 || p->head_dim > 2 * E2S_ROTARY_MAX_PAIRS || p->rot_dim < 2 ||
        p->rot_dim % 2 != 0 || p->rot_dim > p->head_dim)
        return E2S_ERR_BAD_SHAPE;
    if (p->layout != E2S_ROTARY_HALF && p->layout != E2S_ROTARY_INTERLEAVED)
        return E2S_ERR_BAD_PARAM;
    if (p->axes != 1 && p->axes != 3) return E2S_ERR_BAD_PARAM;
    for (int j = 0; j < p->rot_dim / 2; ++j)
        if (p->axis[j] >= p->axes) return E2S_ERR_BAD_PARAM;
    return E2S_OK;
}

e2s_status check_rotary_shape(const e2s_rotary_shape* s, const e2s_rotary_plan& p) {
    if (s == nullptr) return E2S_ERR_NULL_POINTER;
    if (s->batch < 1 || s->num_tokens < 0 || s->q_heads < 0 || s->k_heads < 0 ||
        s->q_heads + static_cast<int64_t>(s->k_heads) < 1)
        return E2S_ERR_BAD_SHAPE;
    if (!known_dtype(s->dtype)) return E2S_ERR_BAD_PARAM;
    if (s->inverse != 0 && s->inverse != 1) return E2S_ERR_BAD_PARAM;
    // one workgroup of 256 threads takes at least one token of a sequence
    if (static_cast<double>(s->batch) * s->num_tokens >= 16777216.0) return E2S_ERR_UNSUPPORTED;
    if (s->q_heads > 65535 || s->k_heads > 65535) return E2S_ERR_UNSUPPORTED;
    const int eb = elem_bytes(s->dtype);
    const int64_t qc[3] = {s->batch, s->q_heads, s->num_tokens};
    const int64_t kc[3] = {s->batch, s->k_heads, s->num_tokens};
    const int64_t pc[3] = {p.axes, s->batch, s->num_tokens};
    if (s->q_heads > 0) {
        E2S_TRY_(check_strides(s->q_stride, qc, 3, p.head_dim, 0, 0, eb));
        E2S_TRY_(check_strides(s->q_out_stride, qc, 3, p.head_dim, 1, 0, eb));
    }
    if (s->k_heads > 0) {
        E2S_TRY_(check_strides(s->k_stride, kc, 3, p.head_dim, 0, 0, eb));
        E2S_TRY_(check_strides(s->k_out_stride, kc, 3, p.head_dim, 1, 0, eb));
    }
    return check_strides(s->pos_stride, pc, 3, 1, 0, 0, 4);
}

e2s_status check_cache(const e2s_cache* c) {
    if (c == nullptr) return E2S_ERR_NULL_POINTER;
    if (c->num_pages < 1 || c->num_kv_heads < 1 || c->head_dim < 1 || c->page_tokens < 1)
        return E2S_ERR_BAD_SHAPE;
    if (c->num_kv_heads > kMaxHeads) return E2S_ERR_UNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128) return E2S_ERR_UNSUPPORTED;
    if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 &&
        c->page_tokens != 128)
        return E2S_ERR_UNSUPPORTED;
    const int64_t page = static_cast<int64_t>(c->num_kv_heads) * c->page_tokens * c->head_dim;
    const int64_t strides[2] = {c->k_page_stride, c->v_page_stride};
    for (int64_t st : strides) {
        if (st < page || st > kMaxStride) return E2S_ERR_BAD_SHAPE;
        if (st % 16 != 0) return E2S_ERR_MISALIGNED;
        if (static_cast<double>(st) * c->num_pages > kBig) return E2S_ERR_BAD_SHAPE;
    }
    if (!c->k || !c->v || !c->k_scale || !c->v_scale) return E2S_ERR_NULL_POINTER;
    if (check_aligned(c->k, 16) != E2S_OK || check_aligned(c->v, 16) != E2S_OK ||
        check_aligned(c->k_scale, 4) != E2S_OK || check_aligned(c->v_scale, 4) != E2S_OK)
        return E2S_ERR_MISALIGNED;
    return E2S_OK;
}

e2s_status check_table(int64_t batch, int64_t max_pages, int64_t stride) {
    if (max_pages < 1) return E2S_ERR_BAD_SHAPE;
    const int64_t counts[1] = {batch};
    return check_strides(&stride, counts, 1, max_pages, 0, 0, 4);
}

e2s_status check_append(const e2s_cache& c, const e2s_cache_append_shape* s) {
    if (s == nullptr) return E2S_ERR_NULL_POINTER;
    if (s->batch < 1 || s->num_tokens < 0 || s->src_tokens < 1) return E2S_ERR_BAD_SHAPE;
    if (!known_dtype(s->dtype) || s->reserved != 0) return E2S_ERR_BAD_PARAM;
    if (s->num_tokens > kMaxCachedTokens) return E2S_ERR_UNSUPPORTED;
    E2S_TRY_(check_table(s->batch, s->max_pages, s->pages_stride));
    const int eb = elem_bytes(s->dtype);
    const int64_t counts[3] = {s->batch, c.num_kv_heads, s->src_tokens};
    E2S_TRY_(check_strides(s->k_stride, counts, 3, c.head_dim, 0, 16 / eb, eb));
    E2S_TRY_(check_strides(s->v_stride, counts, 3, c.head_dim, 0, 16 / eb, eb));
    // one workgroup of at most 256 threads per (sequence, head, touched block, keys/values)
    const double blocks = static_cast<double>(s->num_tokens) / c.page_tokens + 2.0;
    if (2.0 * s->batch * c.num_kv_heads * blocks * 256.0 >= 4294967296.0)
        return E2S_ERR_UNSUPPORTED;
    return E2S_OK;
}

e2s_status check_attend(const e2s_cache& c, const e2s_cache_attend_shape* s) {
    if (s == nullptr) return E2S_ERR_NULL_POINTER;
    if (s->batch < 1 || s->num_heads < 1 || s->num_queries < 1 || s->max_tokens < 1)
        return E2S_ERR_BAD_SHAPE;
    if (s->num_heads % c.num_kv_heads != 0) return E2S_ERR_BAD_SHAPE;
    if (!known_dtype(s->dtype) || s->reserved != 0) return E2S_ERR_BAD_PARAM;
    if ((s->causal != 0 && s->causal != 1) || (s->weights != 0 && s->weights != 1))
        return E2S_ERR_BAD_PARAM;
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
    if (s->weights) {
        const int64_t wc[2] = {s->batch, c.num_kv_heads};
        E2S_TRY_(check_strides(s->weights_in_stride, wc, 2, s->max_tokens, 0, 0, 4));
        E2S_TRY_(check_strides(s->weights_out_stride, wc, 2, s->max_tokens, 1, 0, 4));
    }
    // Fewer than 2^24 rows in all (the join has a workgroup to a row), before the plan's
    // products of rows and tokens, which 63 bits hold then.
    const double heads = static_cast<double>(s->batch) * c.num_kv_heads;
    const double rows = static_cast<double>(s->num_heads / c.num_kv_heads) * s->num_queries;
    if (heads * rows * 256.0 >= 4294967296.0) return E2S_ERR_UNSUPPORTED;
    const AttendPlan p = attend_plan(c, *s);
    // every kernel of the call: fewer than 2^32 work-items
    if (heads * p.row_groups * p.splits * 64 * p.waves >= 4294967296.0 ||
        heads * (static_cast<double>(p.rows) + (s->max_tokens + 127) / 128) * 256.0 >= 4294967296.0)
        return E2S_ERR_UNSUPPORTED;
    // and a workspace that 63 bits address
    if (heads * p.rows * (static_cast<double>(p.splits) * (c.head_dim + 2) + p.logit_stride) * 4.0 >
        kBig)
        return E2S_ERR_BAD_SHAPE;
    return E2S_OK;
}

e2s_status check_evict(const e2s_cache& c, const e2s_cache_evict_shape* s) {
    if (s == nullptr) return E2S_ERR_NULL_POINTER;
    if (s->batch < 1 || s->max_tokens < 1 || s->budget < 1 || s->max_pages < 1 ||
        s->new_max_pages < 1)
        return E2S_ERR_BAD_SHAPE;
    if (s->max_tokens > kMaxCachedTokens || s->budget > kMaxCachedTokens)
        return E2S_ERR_UNSUPPORTED;
    if (s->sinks < 0 || s->recent < 0 ||
        static_cast<int64_t>(s->sinks) + s->recent > s->budget)
        return E2S_ERR_BAD_PARAM;
    if (static_cast<int64_t>(s->new_max_pages) * c.page_tokens < s->budget)
        return E2S_ERR_BAD_SHAPE;
    if (s->left_tokens < s->budget) return E2S_ERR_BAD_SHAPE;
    E2S_TRY_(check_table(s->batch, s->max_pages, s->pages_stride));
    E2S_TRY_(check_table(s->batch, s->new_max_pages, s->new_pages_stride));
    const int64_t wc[2] = {s->batch, c.num_kv_heads};
    E2S_TRY_(check_strides(s->weights_stride, wc, 2, s->max_tokens, 0, 0, 4));
    E2S_TRY_(check_strides(s->left_stride, wc, 2, s->left_tokens, 1, 0, 4));
    const double heads = static_cast<double>(s->batch) * c.num_kv_heads;
    const double blocks = static_cast<double>(s->budget) / c.page_tokens + 1.0;
    if (heads * 1024.0 >= 4294967296.0 || 2.0 * heads * blocks * 256.0 >= 4294967296.0)
        return E2S_ERR_UNSUPPORTED;
    return E2S_OK;
}

AttendPlan attend_plan(const e2s_cache& c, const e2s_cache_attend_shape& s) {
    AttendPlan p{};
    const int64_t B = s.batch, G = c.num_kv_heads, D = c.head_dim;
    p.rows = static_cast<int64_t>(s.num_heads) / G * s.num_queries;
    // Up to 32 rows, a workgroup's waves share the rows and part the keys; above, they part
    // the rows (16 or 32 each) and share the keys' operands in LDS.  Two tiles of rows keep a
    // wave that parts the keys busy with products, so from 17 rows on the rows are parted where
    // there are many keys, although half of the waves then have none: 4 queries of 28 heads
    // (4 key heads) against 4 sequences of 16000 keys take 27 us so and 36 us, of 2000 keys 18
    // and 15.
    p.shared_rows = p.rows > 32 || (p.rows > 16 && B * G * s.max_tokens > 131072);
    const int64_t per_tile = p.shared_rows ? 16 * kAttendWaves : 16;
    p.tiles = p.rows <= per_tile ? 1 : 2;
    // 32 rows to a wave halve what is widened and read from LDS per row, where that still
    // gives two workgroups to a compute unit; with queries in two or three parts they do not
    // fit the registers.
    if (p.shared_rows && (s.dtype != E2S_DTYPE_BF16 ||
                          B * G * ((p.rows + 2 * per_tile - 1) / (2 * per_tile)) < 512))
        p.tiles = 1;
    p.row_groups = (p.rows + per_tile * p.tiles - 1) / (per_tile * p.tiles);
    const int64_t units = B * G * p.row_groups;
    // Keys are split until 2048 workgroups fill the device, most of which have nothing to do
    // where sequences are of unequal lengths (16 of 300 to 4200 keys, up to 48 queries of 28
    // heads: 52 us; 1536 workgroups: 63, 2560: 56).  Units of 32 rows to a wave are enough as
    // they are: 4 sequences of 512 queries and 2000 keys, 32 heads take 107 us unsplit, 153
    // with 16 rows to a wave, which are split.
    int64_t per = p.shared_rows && p.tiles == 2 ? s.max_tokens
                                                : (s.max_tokens * units + 2047) / 2048;
    // Short sequences: one workgroup of eight waves has all keys, and nothing is left to join.
    // With few units that pays up to kFewKeys keys.  Captured calls of 4 units, 28 heads at
    // d = 128, take 8.6 us and 8.9 in parts with 768 keys, 9.7 and 9.3 with 1024, 10.8 and 9.8
    // with 1152 (f32 9.7 and 9.5, 11.4 and 10.0, 12.9 and 10.4); of 120 units 10.7 and 12.1 with
    // 1024, 13.0 and 14.3 with 1280; at d = 64 7.9 and 8.4 with 1024, 9.9 and 9.2 with 1536.
    // Calls that the host makes one by one pay for the join's launch: 9.6 and 11.3 with 1024,
    // 12.0 and 11.2 with 1536.  With more units it pays up to kShortKeys (32 of 2000
    // keys, 8 key heads: 25 us and 32; 64 of 1024: 24 and 31), until workgroups of four waves
    // fill the device unsplit (200 of 300 keys: 35 us and 25).
    p.waves = !p.shared_rows && units < 1024 &&
                      s.max_tokens <= (units < 128 ? kFewKeys : kShortKeys)
                  ? 8
                  : kAttendWaves;
    const int64_t unit = kAttendStep * p.waves;
    if (p.waves == 8) {
        per = s.max_tokens;
    } else if (p.shared_rows) {
        per = std::max<int64_t>(per, 4 * unit);
    } else {
        // Parts of fewer than 1024 keys are mostly their own beginning and end: there 1024
        // workgroups are enough (200 sequences of 300 keys: 26 us, 40 in two parts).
        per = std::max<int64_t>(
            per, std::min<int64_t>(1024, (s.max_tokens * units + 1023) / 1024));
        per = std::max<int64_t>(per, 2 * unit);
    }
    p.chunk = (per + unit - 1) / unit * unit;
    p.splits = (s.max_tokens + p.chunk - 1) / p.chunk;
    // Few rows keep their logits (in whole steps) for the tokens' weights; many make them twice.
    p.logit_stride = s.weights && !p.shared_rows ? (s.max_tokens + 63) / 64 * 64 : 0;
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
    // Weights take a launch of their own behind rows shared by several workgroups, and behind
    // a full device, where a workgroup's wait for its last logits would cost more (64
    // sequences of 32 heads: 85 us in one launch, 73 + 7.5 in two).
    p.lse_kept = s.weights && (p.shared_rows || (p.splits == 1 && p.waves == kAttendWaves));
    p.lse_off = region(p.lse_kept ? all : 0);
    p.logit_off = region(all * p.logit_stride);
    p.bytes = at;
    return p;
}

}  // namespace e2s
