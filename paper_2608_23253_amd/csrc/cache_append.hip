// New tokens into the 8-bit cache (e2s_cache_append).
//
// One workgroup per (sequence, touched block, key head), keys and values together (they
// share the lookups): it alone writes that block's rows and scales, so nothing is shared and
// the result does not depend on any order.  It holds the block's new rows in registers
// between the two things that need them, the largest magnitude and the conversion, so every
// element is read once: the source's bytes and the copy rate bound it (201 MB in 48 us, 4.2
// TB/s: rows of 256 bytes picked by an index; such a gather without any arithmetic reaches
// 4.9), or, for one token per sequence, the launch (64 sequences: 4.2 us).
//
// The scale is the power of two that the block's largest value asks for (block_scale), and
// never falls while tokens are appended: rows before the new ones are rescaled where it
// grows, an exact step but for subnormal results.
#include "serve_device.h"
#include "serve_kernels.h"

namespace e2s {
namespace {

struct AppendArgs {
    const void* src[2];              // keys, values
    uint8_t* dst[2];
    float* scale[2];
    const int32_t* pages;
    const int32_t* start;
    const int32_t* count;            // or null
    const int32_t* src_idx;          // or null
    int64_t ss[2][3];                // sequence, head, token, in elements
    int64_t page_stride[2];          // bytes
    int64_t pages_stride;
    int T, N, G, P, page_shift, num_pages, max_pages, blocks;
};

// PACKETS packets of 8 elements per thread cover the new keys of a block, and as many its
// new values.
template <typename T, int D, int THREADS, int PACKETS>
__global__ __launch_bounds__(THREADS) void append_kernel(const AppendArgs a) {
    constexpr int kLanes = D / 8;                   // threads of a row
    constexpr int kRows = THREADS / kLanes;         // rows of a pass
    __shared__ float shared[2][THREADS / kWave];
    const uint32_t unit = blockIdx.x;
    const int g = static_cast<int>(unit % static_cast<uint32_t>(a.G));
    const uint32_t ub = unit / static_cast<uint32_t>(a.G);
    const int64_t b = ub / static_cast<uint32_t>(a.blocks);

    const int64_t start = a.start[b];
    const int64_t count = a.count ? min(max(a.count[b], 0), a.T) : a.T;
    const int64_t end = min(start + count, static_cast<int64_t>(a.max_pages) << a.page_shift);
    if (start < 0 || start >= end) return;
    const int64_t blk = (start >> a.page_shift) + ub % static_cast<uint32_t>(a.blocks);
    const int64_t first = blk << a.page_shift;      // the block's first token
    if (first >= end) return;
    const int page = a.pages[b * a.pages_stride + blk];
    if (page < 0 || page >= a.num_pages) return;
    const int r0 = static_cast<int>(max(start - first, int64_t{0}));
    const int r1 = static_cast<int>(min(end - first, static_cast<int64_t>(a.P)));
    const int lane = threadIdx.x % kLanes, sub = threadIdx.x / kLanes;

    Packet<T> x[PACKETS][2];
#pragma unroll
    for (int n = 0; n < PACKETS; ++n) {
        const int r = r0 + n * kRows + sub;
        int64_t from = first + r - start;
        bool live = r < r1;
        if (live && a.src_idx) {
            from = a.src_idx[b * a.T + from];
            live = from >= 0 && from < a.N;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            x[n][k] = Packet<T>{};
            if (live)
                load_packet(x[n][k], static_cast<const T*>(a.src[k]) + b * a.ss[k][0] +
                                         g * a.ss[k][1] + from * a.ss[k][2] + lane * 8);
        }
    }
    const int64_t at = static_cast<int64_t>(page) * a.G + g;
    float had[2], want[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        had[k] = r0 > 0 ? a.scale[k][at] : 0.0f;
        float top = 0.0f;
#pragma unroll
        for (int n = 0; n < PACKETS; ++n) {
            float v[8];
            unpack(x[n][k], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float m = fabsf(v[i]);
                top = fmaxf(top, m < __builtin_huge_valf() ? m : 0.0f);   // finite values only
            }
        }
        top = wave_max(top);
        if ((threadIdx.x & (kWave - 1)) == 0) shared[k][threadIdx.x / kWave] = top;
    }
    __syncthreads();                                // every thread has read the scales
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float top = shared[k][0];
#pragma unroll
        for (int w = 1; w < THREADS / kWave; ++w) top = fmaxf(top, shared[k][w]);
        want[k] = fmaxf(block_scale(top), had[k]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        uint8_t* rows = a.dst[k] + page * a.page_stride[k] +
                        static_cast<int64_t>(g) * (D << a.page_shift);
        if (r0 > 0 && want[k] > had[k]) {
            const float ratio = scale_ratio(had[k], want[k]);
            for (int i = threadIdx.x; i < r0 * (D / 16); i += THREADS) {
                u32x4* to = reinterpret_cast<u32x4*>(rows) + i;
                u32x4 w = *to;
                w.x = rescale_e4m3(w.x, ratio);
                w.y = rescale_e4m3(w.y, ratio);
                w.z = rescale_e4m3(w.z, ratio);
                w.w = rescale_e4m3(w.w, ratio);
                *to = w;
            }
        }
        const float inv = 1.0f / want[k];           // exact: a power of two
#pragma unroll
        for (int n = 0; n < PACKETS; ++n) {
            const int r = r0 + n * kRows + sub;
            if (r >= r1) continue;
            float v[8];
            unpack(x[n][k], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] *= inv;
                if (!(fabsf(v[i]) < __builtin_huge_valf())) v[i] = __builtin_nanf("");
            }
            u32x2 w = {to_e4m3(v[0], v[1], v[2], v[3]), to_e4m3(v[4], v[5], v[6], v[7])};
            *reinterpret_cast<u32x2*>(rows + r * D + lane * 8) = w;
        }
    }
    if (threadIdx.x == 0) {
        a.scale[0][at] = want[0];
        a.scale[1][at] = want[1];
    }
}

template <typename T, int D, int THREADS, int PACKETS>
void launch_k(const AppendArgs& a, int64_t units, hipStream_t st) {
    hipLaunchKernelGGL((append_kernel<T, D, THREADS, PACKETS>),
                       dim3(static_cast<unsigned>(units)), dim3(THREADS), 0, st, a);
}

template <typename T, int D>
hipError_t launch_t(const AppendArgs& a, int64_t B, hipStream_t st) {
    const int64_t units = B * a.blocks * a.G;
    // The most new rows that one block can get decide how many packets a thread holds.  A
    // row is D / 8 threads: one wave is enough for the few tokens of a decoding step.
    const int packets = std::min(a.T, a.P) * (D / 8);
    if (packets <= 64) launch_k<T, D, 64, 1>(a, units, st);
    else if (packets <= 256) launch_k<T, D, 256, 1>(a, units, st);
    else if (packets <= 512) launch_k<T, D, 256, 2>(a, units, st);
    else if (packets <= 1024) launch_k<T, D, 256, 4>(a, units, st);
    else launch_k<T, D, 256, 8>(a, units, st);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_d(const AppendArgs& a, int64_t B, int D, hipStream_t st) {
    return D == 64 ? launch_t<T, 64>(a, B, st) : launch_t<T, 128>(a, B, st);
}

}  // namespace

hipError_t launch_cache_append(const e2s_cache& c, const e2s_cache_append_shape& s,
                               const int32_t* pages, const int32_t* start, const int32_t* count,
                               const int32_t* src_idx, const void* k, const void* v,
                               hipStream_t st) {
    AppendArgs a{};
    a.src[0] = k;
    a.src[1] = v;
    a.dst[0] = static_cast<uint8_t*>(c.k);
    a.dst[1] = static_cast<uint8_t*>(c.v);
    a.scale[0] = c.k_scale;
    a.scale[1] = c.v_scale;
    a.pages = pages;
    a.start = start;
    a.count = count;
    a.src_idx = src_idx;
    for (int i = 0; i < 3; ++i) {
        a.ss[0][i] = s.k_stride[i];
        a.ss[1][i] = s.v_stride[i];
    }
    a.page_stride[0] = c.k_page_stride;
    a.page_stride[1] = c.v_page_stride;
    a.pages_stride = s.pages_stride;
    a.T = s.num_tokens;
    a.N = s.src_tokens;
    a.G = c.num_kv_heads;
    a.P = c.page_tokens;
    a.page_shift = __builtin_ctz(static_cast<unsigned>(c.page_tokens));   // a power of two
    a.num_pages = c.num_pages;
    a.max_pages = s.max_pages;
    // blocks that T tokens can touch, starting anywhere in a block
    a.blocks = (s.num_tokens + c.page_tokens - 2) / c.page_tokens + 1;
    if (s.dtype == E2S_DTYPE_F32) return launch_d<float>(a, s.batch, c.head_dim, st);
    if (s.dtype == E2S_DTYPE_F16) return launch_d<_Float16>(a, s.batch, c.head_dim, st);
    return launch_d<uint16_t>(a, s.batch, c.head_dim, st);
}

}  // namespace e2s
