// Randomized exercise of the host-side checks and plans of e2s_step.h, built with
// AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_step_abi.py: what a check lets
// through has a plan that the kernels can take.
#include <cstdint>
#include <cstdio>
#include <limits>
#include <random>

#include "step_validate.h"

namespace {
std::mt19937_64 rng(7);
int failures = 0;
void expect(bool ok, const char* what) {
    if (!ok) {
        std::printf("FAIL: %s\n", what);
        ++failures;
    }
}
int64_t pick64() {
    static const int64_t edges[] = {0, 1, -1, 2, 8, 16, 32, 64, 128, 2048, 1 << 20, (1 << 20) + 1,
                                    int64_t(1) << 31, std::numeric_limits<int64_t>::max(),
                                    std::numeric_limits<int64_t>::min(),
                                    std::numeric_limits<int64_t>::max() / 64};
    switch (rng() % 3) {
        case 0: return edges[rng() % (sizeof(edges) / sizeof(edges[0]))];
        case 1: return static_cast<int64_t>(rng() % 4096) - 8;
        default: return static_cast<int64_t>(rng());
    }
}
int32_t pick32() { return static_cast<int32_t>(pick64()); }
int32_t upto(int64_t most) {
    const int bits = static_cast<int>(rng() % 33);
    const int64_t n = static_cast<int64_t>(rng() % ((uint64_t{1} << bits) + 1)) + 1;
    return static_cast<int32_t>(rng() % 8 == 0 || n > most ? most : n);
}

void check_plan(const e2s_cache4& c, const e2s_cache4_attend_shape& s) {
    using namespace e2s;
    const Attend4Plan p = attend4_plan(c, s);
    const int64_t heads = static_cast<int64_t>(s.batch) * c.num_kv_heads;
    expect(p.rows == static_cast<int64_t>(s.num_heads) / c.num_kv_heads * s.num_queries, "rows");
    expect(p.waves == 1 || p.waves == 2 || p.waves == 4 || p.waves == 8, "the kernels' waves");
    expect(p.row_groups == (p.rows + 15) / 16, "row groups of 16, each needed");
    expect(p.chunk > 0 && p.chunk % (kStep4 * p.waves) == 0, "whole steps to every wave");
    expect(p.splits >= 1 && p.splits * p.chunk >= s.max_tokens &&
               (p.splits - 1) * p.chunk < s.max_tokens, "the parts cover the tokens, each needed");
    expect(p.splits * p.chunk < (int64_t{1} << 31), "keys that 31 bits number");
    expect(static_cast<double>(heads) * p.row_groups * p.splits * 64 * p.waves < 4294967296.0,
           "the grid's size");
    expect(static_cast<double>(heads) * p.rows * 256.0 < 4294967296.0, "the join's size");
    const int64_t all = heads * p.rows, parts = p.splits > 1 ? p.splits : 0;
    const int64_t need[3] = {all * parts, all * parts, all * parts * c.head_dim};
    const size_t at[4] = {p.max_off, p.sum_off, p.part_off, p.bytes};
    for (int i = 0; i < 3; ++i)
        expect(at[i] % 256 == 0 && at[i + 1] - at[i] >= static_cast<size_t>(need[i]) * 4,
               "the workspace's regions hold what is put there");
}
}  // namespace

int main() {
    using namespace e2s;
    void* p = reinterpret_cast<void*>(uintptr_t{1} << 20);
    long valid = 0;
    for (int it = 0; it < 300000; ++it) {
        // sizes that mostly fit together, of any magnitude
        static const int32_t group[] = {1, 2, 3, 7, 8, 16, 32, 128};
        const int32_t kv = upto(128), g = group[rng() % 8], page = 32 << (rng() % 3);
        const int32_t d = rng() % 2 ? 64 : 128;
        e2s_cache4 c{upto(1 << 20), page, kv, d, int64_t{kv} * page * d / 2,
                     int64_t{kv} * page * d / 2, p, p, p, p};
        if (rng() % 8 == 0) {
            int32_t* f = &c.num_pages;
            f[rng() % 4] = pick32();
            if (rng() % 2) (rng() % 2 ? c.k_page_stride : c.v_page_stride) = pick64();
        }
        if (check_cache4(&c) != E2S_OK) continue;
        const int32_t heads = kv * g > 128 ? kv : kv * g;
        e2s_cache4_attend_shape s{};
        s.batch = upto(2147483647);
        s.num_heads = heads;
        s.num_queries = upto(1 << 20);
        s.dtype = static_cast<int32_t>(rng() % 3);
        s.max_tokens = upto(1 << 20);
        s.max_pages = (s.max_tokens + page - 1) / page;
        s.causal = static_cast<int32_t>(rng() % 2);
        s.pages_stride = s.max_pages;
        const int64_t rows[3] = {int64_t{heads} * s.num_queries * d, int64_t{s.num_queries} * d, d};
        for (int i = 0; i < 3; ++i) s.q_stride[i] = s.out_stride[i] = rows[i];
        if (rng() % 4 == 0) {
            int32_t* f = &s.batch;
            f[rng() % 7] = pick32();
            if (rng() % 2) (rng() % 2 ? s.q_stride : s.out_stride)[rng() % 3] = pick64();
            if (rng() % 4 == 0) s.pages_stride = pick64();
        }
        if (check_attend4(c, &s) == E2S_OK) {
            ++valid;
            check_plan(c, s);
        }
        e2s_cache_append_shape a{upto(1 << 24), upto(1 << 21), upto(1 << 21),
                                 static_cast<int32_t>(rng() % 4), upto(1 << 16), 0, 4,
                                 {int64_t{kv} * d, d, d}, {int64_t{kv} * d, d, d}};
        if (rng() % 2) a.k_stride[rng() % 3] = pick64();
        valid += check_append4(c, &a) == E2S_OK;
        e2s_cache4_read_shape r{upto(1 << 24), upto(1 << 21), static_cast<int32_t>(rng() % 4),
                                upto(1 << 16), 4, {int64_t{kv} * d, d, d}, {int64_t{kv} * d, d, d}};
        if (rng() % 2) r.v_out_stride[rng() % 3] = pick64();
        valid += check_read4(c, &r) == E2S_OK;
        e2s_rotary_plan plan{};
        const e2s_rotary_spec spec{128, 64, 0, 0, {0, 0, 0}, 0, 0.0, 1e4, 1.0, 0.0, 1.0, 32.0};
        fill_rotary_plan(spec, &plan);
        e2s_norm_rotate_shape n{2, 5, 4, 2, 1, 1, 1e-6f, 0, {2560, 640, 128}, {1280, 640, 128},
                                {2560, 640, 128}, {1280, 640, 128}, {2560, 640, 128},
                                {1280, 640, 128}, {0, 5, 1}};
        (&n.batch)[rng() % 6] = pick32();
        n.q_grad_stride[rng() % 3] = pick64();
        if (check_norm_rotate(&n, plan, true) == E2S_OK) {
            ++valid;
            const size_t bytes = norm_rotate_back_bytes(n, plan, true);
            expect(bytes <= kNormMostParts * 2 * 128 * 4 && bytes % 1024 == 0, "partial rows");
            expect(check_norm_rotate(&n, plan, false) == E2S_OK, "what holds back holds forward");
        }
    }
    std::printf("%ld valid records; %d failures\n", valid, failures);
    return failures == 0 && valid > 50000 ? 0 : 1;
}
