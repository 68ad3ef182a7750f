// Prints how an attention call is cut, for tests/test_serve_plan.py: a line of
//   num_pages page_tokens Hkv d  batch heads queries dtype max_tokens causal weights
// on the input gives a line of the plan's numbers.  Then random calls with large sizes
// together, whose plans have to hold together; built with AddressSanitizer and
// UndefinedBehaviorSanitizer.
#include <cinttypes>
#include <cstdio>
#include <random>

#include "serve_validate.h"

namespace {
int failures = 0;
void expect(bool ok, const char* what) {
    if (!ok) {
        std::printf("FAIL: %s\n", what);
        ++failures;
    }
}

e2s_cache cache_of(int32_t pages, int32_t page, int32_t heads, int32_t d) {
    void* p = reinterpret_cast<void*>(uintptr_t{1} << 20);
    float* f = static_cast<float*>(p);
    const int64_t size = static_cast<int64_t>(heads) * page * d;
    return {pages, page, heads, d, size, size, p, p, f, f};
}

e2s_cache_attend_shape shape_of(const e2s_cache& c, int32_t batch, int32_t heads, int32_t queries,
                                int32_t dtype, int32_t max_tokens, int32_t causal, int32_t weights) {
    e2s_cache_attend_shape s{};
    s.batch = batch;
    s.num_heads = heads;
    s.num_queries = queries;
    s.dtype = dtype;
    s.max_tokens = max_tokens;
    s.max_pages = (max_tokens + c.page_tokens - 1) / c.page_tokens;
    s.causal = causal;
    s.weights = weights;
    s.pages_stride = s.max_pages;
    const int64_t rows[3] = {static_cast<int64_t>(heads) * queries * c.head_dim,
                             static_cast<int64_t>(queries) * c.head_dim, c.head_dim};
    for (int i = 0; i < 3; ++i) s.q_stride[i] = s.out_stride[i] = rows[i];
    s.weights_in_stride[0] = s.weights_out_stride[0] =
        static_cast<int64_t>(c.num_kv_heads) * max_tokens;
    s.weights_in_stride[1] = s.weights_out_stride[1] = max_tokens;
    return s;
}

// What the kernels and their launches assume of a plan.
void check_plan(const e2s_cache& c, const e2s_cache_attend_shape& s) {
    using namespace e2s;
    const AttendPlan p = attend_plan(c, s);
    const int64_t heads = static_cast<int64_t>(s.batch) * c.num_kv_heads;
    const double items = 4294967296.0;
    expect(p.rows == static_cast<int64_t>(s.num_heads) / c.num_kv_heads * s.num_queries, "rows");
    expect(p.waves == kAttendWaves || p.waves == 8, "four or eight waves");
    expect(p.tiles == 1 || p.tiles == 2, "one or two tiles of rows");
    const int64_t per = p.shared_rows ? 16 * kAttendWaves * p.tiles : 16 * p.tiles;
    expect(p.row_groups == (p.rows + per - 1) / per, "the row groups cover the rows, each needed");
    expect(p.shared_rows || (p.row_groups == 1 && p.rows <= 32),
           "waves that part the keys share all rows");
    expect(p.chunk % (kAttendStep * p.waves) == 0, "a wave's keys are whole steps");
    expect(p.splits >= 1 && p.splits * p.chunk >= s.max_tokens &&
               (p.splits - 1) * p.chunk < s.max_tokens, "the parts cover the tokens, each needed");
    expect(p.waves == kAttendWaves || (!p.shared_rows && p.splits == 1),
           "eight waves have all keys of their rows");
    expect(!(p.shared_rows && p.tiles == 2) || p.splits == 1, "32 rows a wave are not split");
    expect(!(p.shared_rows && p.tiles == 2) || s.dtype == E2S_DTYPE_BF16,
           "32 rows a wave are bf16's");
    expect(p.lse_kept == (s.weights && (p.shared_rows || (p.splits == 1 && p.waves == kAttendWaves))),
           "sums are kept for the weights' own launch");
    expect((p.logit_stride > 0) == (s.weights && !p.shared_rows), "few rows keep their logits");
    expect(p.logit_stride == 0 ||
               (p.logit_stride % 64 == 0 && p.logit_stride >= s.max_tokens), "whole steps of logits");
    expect(static_cast<double>(heads) * p.row_groups * p.splits * 64 * p.waves < items,
           "the grid's size");
    expect(static_cast<double>(heads) * p.rows * 256.0 < items, "the join's size");
    const int64_t all = heads * p.rows, parts = p.splits > 1 ? p.splits : 0;
    const int64_t need[5] = {all * parts, all * parts, all * parts * c.head_dim,
                             p.lse_kept ? all : 0, all * p.logit_stride};
    const size_t at[6] = {p.max_off, p.sum_off, p.part_off, p.lse_off, p.logit_off, p.bytes};
    for (int i = 0; i < 5; ++i)
        expect(at[i] % 256 == 0 && at[i + 1] - at[i] >= static_cast<size_t>(need[i]) * 4,
               "the workspace's regions hold what is put there");
}
}  // namespace

int main() {
    using namespace e2s;
    int32_t v[11];
    while (std::scanf("%" SCNd32, &v[0]) == 1) {
        for (int i = 1; i < 11; ++i)
            if (std::scanf("%" SCNd32, &v[i]) != 1) return 2;
        const e2s_cache c = cache_of(v[0], v[1], v[2], v[3]);
        const e2s_cache_attend_shape s = shape_of(c, v[4], v[5], v[6], v[7], v[8], v[9], v[10]);
        const int st = check_cache(&c) != E2S_OK ? check_cache(&c) : check_attend(c, &s);
        if (st != E2S_OK) {
            std::printf("plan %d\n", st);
            continue;
        }
        check_plan(c, s);
        const AttendPlan p = attend_plan(c, s);
        std::printf("plan 0 %d %d %d %d %" PRId64 " %" PRId64 " %zu\n", p.shared_rows, p.tiles,
                    p.waves, p.lse_kept, p.splits, p.chunk, p.bytes);
    }
    std::mt19937_64 rng(8);
    auto upto = [&](int64_t most) {      // mostly of any magnitude, now and then the largest
        const int bits = static_cast<int>(rng() % 33);
        const int64_t n = static_cast<int64_t>(rng() % ((uint64_t{1} << bits) + 1)) + 1;
        return static_cast<int32_t>(rng() % 8 == 0 || n > most ? most : n);
    };
    long valid = 0;
    for (int it = 0; it < 400000; ++it) {
        static const int32_t group[] = {1, 2, 3, 7, 8, 16, 32, 128};
        const int32_t kv = upto(128), g = group[rng() % 8];
        const e2s_cache c = cache_of(upto(1 << 20), 16 << (rng() % 4), kv, rng() % 2 ? 64 : 128);
        if (check_cache(&c) != E2S_OK) continue;
        const int32_t heads = kv * g > 128 ? kv : kv * g;
        const e2s_cache_attend_shape s =
            shape_of(c, upto(2147483647), heads, upto(1 << 20), static_cast<int32_t>(rng() % 3),
                     upto(1 << 20), static_cast<int32_t>(rng() % 2),
                     static_cast<int32_t>(rng() % 2));
        if (check_attend(c, &s) != E2S_OK) continue;
        ++valid;
        check_plan(c, s);
    }
    std::printf("%ld valid records; %d failures\n", valid, failures);
    return failures == 0 && valid > 10000 ? 0 : 1;
}
