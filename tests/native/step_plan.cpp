// Prints how an attention call over the 4-bit cache is cut, for tests/test_step_plan.py: a line of
//   page_tokens Hkv d  batch heads queries dtype max_tokens causal
// on the input gives a line of the plan's numbers.
#include <cinttypes>
#include <cstdio>

#include "step_validate.h"

int main() {
    using namespace e2s;
    void* p = reinterpret_cast<void*>(uintptr_t{1} << 20);
    int32_t page, kv, d, batch, heads, queries, dtype, max_tokens, causal;
    while (std::scanf("%" SCNd32 "%" SCNd32 "%" SCNd32 "%" SCNd32 "%" SCNd32 "%" SCNd32 "%" SCNd32
                      "%" SCNd32 "%" SCNd32, &page, &kv, &d, &batch, &heads, &queries, &dtype,
                      &max_tokens, &causal) == 9) {
        const int64_t bytes = int64_t{kv} * page * d / 2;
        const e2s_cache4 c{1 << 16, page, kv, d, bytes, bytes, p, p, p, p};
        e2s_cache4_attend_shape s{};
        s.batch = batch;
        s.num_heads = heads;
        s.num_queries = queries;
        s.dtype = dtype;
        s.max_tokens = max_tokens;
        s.max_pages = (max_tokens + page - 1) / page;
        s.causal = causal;
        s.pages_stride = s.max_pages;
        const int64_t rows[3] = {int64_t{heads} * queries * d, int64_t{queries} * d, d};
        for (int i = 0; i < 3; ++i) s.q_stride[i] = s.out_stride[i] = rows[i];
        const int status = check_cache4(&c) != E2S_OK ? -1 : check_attend4(c, &s);
        const Attend4Plan q = attend4_plan(c, s);
        std::printf("plan %d %d %" PRId64 " %" PRId64 " %zu\n", status, q.waves, q.chunk, q.splits,
                    q.bytes);
    }
    return 0;
}
