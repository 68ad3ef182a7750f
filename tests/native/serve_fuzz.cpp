// Randomized exercise of the host-side argument checks of e2s_serve.h, built with
// AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_serve_abi.py.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <limits>
#include <random>

#include "serve_validate.h"

namespace {
std::mt19937_64 rng(23253);

int64_t pick64() {
    static const int64_t edges[] = {0, 1, -1, 2, 8, 16, 64, 128, 2048, 1 << 20, (1 << 20) + 1,
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
double pickd() {
    static const double edges[] = {0.0, 1.0, -1.0, 1e4, 4096.0, 1e308, 1e-308,
                                   std::numeric_limits<double>::infinity(),
                                   std::numeric_limits<double>::quiet_NaN(), 0.5, 32.0};
    return edges[rng() % (sizeof(edges) / sizeof(edges[0]))];
}
const void* pickp() { return reinterpret_cast<const void*>((rng() % 8) * 8); }

int failures = 0;
void expect(bool ok, const char* what) {
    if (!ok) {
        std::printf("FAIL: %s\n", what);
        ++failures;
    }
}
// One field of a good record replaced, or several.
template <typename F> void vary(int fields, F set) {
    const int n = rng() % 3 == 0 ? 3 : 1;
    for (int i = 0; i < n; ++i) set(static_cast<int>(rng() % fields));
}
}  // namespace

int main() {
    using namespace e2s;
    long valid = 0;
    for (int it = 0; it < 200000; ++it) {
        e2s_rotary_spec sp{128, 64, 0, static_cast<int32_t>(rng() % 4), {0, 0, 0}, 0,
                           0.0, 1e4, 4.0, 4096.0, 1.0, 32.0};
        vary(12, [&](int f) {
            if (f < 8) reinterpret_cast<int32_t*>(&sp)[f] = pick32();
            else {
                double* all[6] = {&sp.amplitude, &sp.base, &sp.factor, &sp.original_len, &sp.low,
                                  &sp.high};
                *all[rng() % 6] = pickd();
            }
        });
        e2s_rotary_plan plan{};
        if (check_rotary_spec(&sp) == E2S_OK) {
            ++valid;
            fill_rotary_plan(sp, &plan);
            expect(check_rotary_plan(&plan) == E2S_OK, "a filled plan is a valid plan");
        } else {
            sp = e2s_rotary_spec{128, 128, 0, 0, {16, 24, 24}, 0, 0.0, 1e4, 1.0, 0.0, 1.0, 32.0};
            fill_rotary_plan(sp, &plan);
            vary(4, [&](int f) { reinterpret_cast<int32_t*>(&plan)[f] = pick32(); });
            plan.axis[rng() % E2S_ROTARY_MAX_PAIRS] = static_cast<uint8_t>(rng() % 5);
        }
        e2s_rotary_shape rs{2, 5, 4, 2, 1, 0, {1280, 320, 64}, {640, 320, 64}, {1280, 320, 64},
                            {640, 320, 64}, {0, 5, 1}};
        vary(21, [&](int f) {
            if (f < 6) reinterpret_cast<int32_t*>(&rs)[f] = pick32();
            else {
                int64_t* all[5] = {rs.q_stride, rs.k_stride, rs.q_out_stride, rs.k_out_stride,
                                   rs.pos_stride};
                all[(f - 6) / 3][(f - 6) % 3] = pick64();
            }
        });
        if (check_rotary_plan(&plan) == E2S_OK) valid += check_rotary_shape(&rs, plan) == E2S_OK;

        void* p = reinterpret_cast<void*>(uintptr_t{1} << 20);
        float* pf = static_cast<float*>(p);
        e2s_cache c{9, 16, 2, 64, 2048, 2048, p, p, pf, pf};
        if (rng() % 4 == 0) {
            vary(6, [&](int f) {
                if (f < 4) reinterpret_cast<int32_t*>(&c)[f] = pick32();
                else (f == 4 ? c.k_page_stride : c.v_page_stride) = pick64();
            });
            if (rng() % 4 == 0) c.k = const_cast<void*>(pickp());
        }
        if (check_cache(&c) != E2S_OK) continue;
        ++valid;
        e2s_cache_append_shape as{3, 5, 5, 1, 4, 0, 4, {640, 320, 64}, {640, 320, 64}};
        vary(13, [&](int f) {
            if (f < 6) reinterpret_cast<int32_t*>(&as)[f] = pick32();
            else if (f == 6) as.pages_stride = pick64();
            else (f < 10 ? as.k_stride[f - 7] : as.v_stride[f - 10]) = pick64();
        });
        valid += check_append(c, &as) == E2S_OK;
        e2s_cache_attend_shape at{3, 4, 2, 1, 100, 7, 1, 1, 0.0f, 0, 7, {512, 128, 64},
                                  {512, 128, 64}, {200, 100}, {200, 100}};
        vary(20, [&](int f) {
            if (f < 8) reinterpret_cast<int32_t*>(&at)[f] = pick32();
            else if (f == 8) at.scale = static_cast<float>(pickd());
            else if (f == 9) at.pages_stride = pick64();
            else if (f < 13) at.q_stride[f - 10] = pick64();
            else if (f < 16) at.out_stride[f - 13] = pick64();
            else if (f < 18) at.weights_in_stride[f - 16] = pick64();
            else at.weights_out_stride[f - 18] = pick64();
        });
        if (check_attend(c, &at) == E2S_OK) {
            ++valid;
            const AttendPlan pl = attend_plan(c, at);
            expect(pl.chunk % (kAttendStep * kAttendWaves) == 0 && pl.splits >= 1 &&
                       pl.splits * pl.chunk >= at.max_tokens &&
                       (pl.splits - 1) * pl.chunk < at.max_tokens,
                   "the parts cover the tokens");
            expect(pl.row_groups * pl.tiles * (pl.shared_rows ? 64 : 16) >= pl.rows, "the row groups cover the rows");
            expect(pl.max_off <= pl.sum_off && pl.sum_off <= pl.part_off &&
                       pl.part_off <= pl.lse_off && pl.lse_off <= pl.logit_off &&
                       pl.logit_off <= pl.bytes,
                   "the workspace's regions follow one another");
        }
        e2s_cache_evict_shape ev{3, 100, 40, 4, 8, 7, 3, 40, 7, 3, {200, 100}, {80, 40}};
        vary(14, [&](int f) {
            if (f < 8) reinterpret_cast<int32_t*>(&ev)[f] = pick32();
            else if (f < 10) (f == 8 ? ev.pages_stride : ev.new_pages_stride) = pick64();
            else (f < 12 ? ev.weights_stride[f - 10] : ev.left_stride[f - 12]) = pick64();
        });
        valid += check_evict(c, &ev) == E2S_OK;
    }
    std::printf("%ld valid records; %d failures\n", valid, failures);
    return failures == 0 ? 0 : 1;
}
