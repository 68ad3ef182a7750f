// New tokens into the 4-bit cache (e2s_cache4_append), and its values out of it
// (e2s_cache4_read).
//
// One workgroup per (sequence, touched group of 32 tokens, key head), keys and values
// together: it alone writes that group's bytes, so nothing is shared.  A row's 8-element
// packets are neighbouring lanes: a key block of 32 is 4 of them and a value's row all, so
// both maxima are a few DPP steps, and every element is read once.  Key codes are written from
// the lanes that hold them.  Value bytes hold two tokens of one dimension, so value codes
// cross LDS once, and what other tokens of the group hold is merged in.
//
// 128 kept tokens of 64 x 576, 32 heads, bf16 (134 MB picked by an index, 18 MB written): 39 us,
// 3.9 TB/s; 48 with maxima and value codes an element at a time, 22 instructions to an
// element (the vector unit was busy for 45 of them); workgroups of 128 or 512 threads: 50 and 55.
// Read back (134 MB written): 28 us, 5.5 TB/s.  One token of 64 sequences: 4.0 and 3.5 us, the launch.
#include "serve_device.h"
#include "step_kernels.h"

namespace e2s {
namespace {

constexpr float kInf = __builtin_huge_valf();

struct Pool4Args {                   // the cache and the page table, as kernels see them
    uint8_t* k;
    uint8_t* v;
    uint8_t* k_scale;
    uint16_t* v_scale;
    int64_t k_page, v_page;          // bytes
    const int32_t* pages;
    int64_t pages_stride;
    int G, P, page_shift, num_pages, max_pages;
};
struct Append4Args {
    Pool4Args c;
    const void* src[2];              // keys, values
    const int32_t* start;
    const int32_t* count;            // or null
    const int32_t* src_idx;          // or null
    int64_t ss[2][3];                // sequence, head, token, in elements
    int T, N, groups;
};

// The largest magnitude of a packet, an infinity if one of them is or is NaN.  Magnitudes are
// ordered as their bits are, and what is not finite comes last.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t top_half(const u32x4& a) {
    u16x2 m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = __builtin_bit_cast(u16x2, a[i] & 0x7FFF7FFFu);
    const u16x2 t = __builtin_elementwise_max(__builtin_elementwise_max(m[0], m[1]),
                                              __builtin_elementwise_max(m[2], m[3]));
    return max(static_cast<uint32_t>(t.x), static_cast<uint32_t>(t.y));
}
__device__ __forceinline__ float packet_top(const Packet<uint16_t>& p) {
    const uint32_t m = top_half(p.a);
    return m < 0x7F80u ? __uint_as_float(m << 16) : kInf;
}
__device__ __forceinline__ float packet_top(const Packet<_Float16>& p) {
    const uint32_t m = top_half(p.a);
    return m < 0x7C00u ? f16lo(m) : kInf;
}
__device__ __forceinline__ float packet_top(const Packet<float>& p) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m = max(m, __float_as_uint(p.a[i]) & 0x7FFFFFFFu);
        m = max(m, __float_as_uint(p.b[i]) & 0x7FFFFFFFu);
    }
    return m < 0x7F800000u ? __uint_as_float(m) : kInf;
}

__device__ __forceinline__ float quad_max(float v) {
    v = fmaxf(v, dpp<kQuadSwap1>(v));
    return fmaxf(v, dpp<kQuadSwap2>(v));
}

// The group's bytes of a key head: pointers to its first token's.
template <int D>
struct Group4 {
    uint8_t* k;                      // [32, d/2]
    uint8_t* v;                      // [d, 16]
    uint8_t* k_scale;                // [2, 4, d/32, 4]
    uint16_t* v_scale;               // [32]
    __device__ __forceinline__ Group4(const Pool4Args& c, int page, int g, int row) {
        const int64_t at = static_cast<int64_t>(page) * c.G + g;
        const int64_t head = static_cast<int64_t>(g) * (D / 2) << c.page_shift;
        k = c.k + page * c.k_page + head + row * (D / 2);
        v = c.v + page * c.v_page + head + row * (D / 2);
        k_scale = c.k_scale + ((at << c.page_shift) + row) * (D / 32);
        v_scale = c.v_scale + (at << c.page_shift) + row;
    }
};
template <int D>
__device__ __forceinline__ int key_scale_at(int r, int c) {      // r: 0 .. 31
    return (r >> 4) * (D / 2) + ((r & 3) * (D / 32) + c) * 4 + (r >> 2 & 3);
}

// The code (without its sign) of magnitude m at scale s: nearest, ties to the even code.  The
// borders times s, 8 bits at most, are exact.
__device__ __forceinline__ uint32_t value_code(float m, float s) {
    const bool b2 = m >= 1.75f * s;
    const bool b1 = m >= (b2 ? 3.5f : 0.75f) * s;
    const float t = b2 ? (b1 ? 5.0f : 2.5f) : (b1 ? 1.25f : 0.25f);
    return (b2 ? 4u : 0u) | (b1 ? 2u : 0u) | (m > t * s ? 1u : 0u);
}

// The codes of 8 elements at a row's scale s, element 2 i in the low half of byte i.
__device__ __forceinline__ uint32_t key_codes(const float (&e)[8], float s) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e[0], e[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e[2], e[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e[4], e[5], s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, e[6], e[7], s, 3);
}
// The conversion's scale is a power of two, so a value is divided by its own first.  A border
// between codes has 11 bits (3 times the scale's 8), so an element of 8 or 11 bits that is not
// one is 2^-11 of it away at least, and one that is comes out exactly, by a step of Newton's.
// Elements of 24 bits are compared with the borders instead.
template <typename T>
__device__ __forceinline__ uint32_t value_codes(const float (&e)[8], float s) {
    if constexpr (sizeof(T) == 4) {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            w |= (value_code(fabsf(e[i]), s) | (__float_as_uint(e[i]) >> 28 & 8u)) << (4 * i);
        return w;
    } else {
        const float r = 1.0f / s;
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float q = e[i] * r;
            // (a negative zero keeps its sign)
            y[i] = copysignf(__builtin_fmaf(__builtin_fmaf(-q, s, e[i]), r, q), e[i]);
        }
        return key_codes(y, 1.0f);
    }
}

// The smallest bfloat16 s >= 2^-100 with amax <= 6 s, NaN for an infinite amax.  6 s is exact.
__device__ __forceinline__ float value_scale(float amax) {
    uint32_t bits = __float_as_uint(amax / 6.0f) & 0xFFFF0000u;
    if (6.0f * __uint_as_float(bits) < amax) bits += 0x10000u;
    const float s = fmaxf(__uint_as_float(bits), 0x1p-100f);
    return amax < kInf ? s : __builtin_nanf("");
}

// PACKETS packets of 8 elements per thread cover a group's new keys, and as many its values.
template <typename T, int D, int THREADS, int PACKETS>
__global__ __launch_bounds__(THREADS) void append4_kernel(const Append4Args a) {
    constexpr int kLanes = D / 8;                   // threads of a row
    constexpr int kRows = THREADS / kLanes;         // rows of a pass
    constexpr int kPad = D + 4;
    // of the values, a byte each: of 8 elements the even ones, then the odd ones
    __shared__ alignas(8) uint8_t codes[kGroup4 * kPad];
    const uint32_t unit = blockIdx.x;
    const int g = static_cast<int>(unit % static_cast<uint32_t>(a.c.G));
    const uint32_t ub = unit / static_cast<uint32_t>(a.c.G);
    const int64_t b = ub / static_cast<uint32_t>(a.groups);

    const int64_t start = a.start[b];
    const int64_t count = a.count ? min(max(a.count[b], 0), a.T) : a.T;
    const int64_t end = min(start + count, static_cast<int64_t>(a.c.max_pages) << a.c.page_shift);
    if (start < 0 || start >= end) return;
    const int64_t first =
        ((start / kGroup4) + ub % static_cast<uint32_t>(a.groups)) * kGroup4;
    if (first >= end) return;
    const int page = a.c.pages[b * a.c.pages_stride + (first >> a.c.page_shift)];
    if (page < 0 || page >= a.c.num_pages) return;
    const int r0 = static_cast<int>(max(start - first, int64_t{0}));
    const int r1 = static_cast<int>(min(end - first, static_cast<int64_t>(kGroup4)));
    const int lane = threadIdx.x % kLanes, sub = threadIdx.x / kLanes;
    const Group4<D> at(a.c, page, g, static_cast<int>(first) & (a.c.P - 1));

    // Values: thread (4 dimensions, 8 tokens) owns a word of each dimension.
    constexpr int kParts = D, kPer = (kParts + THREADS - 1) / THREADS;
    auto dim_of = [](int part, int j) { return (part >> 3) * 8 + (part >> 2 & 1) + 2 * j; };
    uint32_t mask[kPer], old[kPer][4];
#pragma unroll
    for (int n = 0; n < kPer; ++n) {
        const int part = threadIdx.x + n * THREADS, t8 = (part & 3) * 8;
        const int lo = min(max(r0 - t8, 0), 8), hi = min(max(r1 - t8, 0), 8);
        mask[n] = part < kParts ? static_cast<uint32_t>((1ull << (4 * hi)) - (1ull << (4 * lo)))
                                : 0u;
        if (mask[n] != 0u && mask[n] != ~0u) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                old[n][j] = *reinterpret_cast<const uint32_t*>(at.v + dim_of(part, j) * 16 +
                                                               (part & 3) * 4);
        }
    }
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
#pragma unroll
    for (int n = 0; n < PACKETS; ++n) {
        const int r = r0 + n * kRows + sub;
        float e[2][8], top[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            unpack(x[n][k], e[k]);
            top[k] = quad_max(packet_top(x[n][k]));
        }
        top[1] = fmaxf(top[1], dpp<kRowHalfMirror>(top[1]));
        if (kLanes == 16) top[1] = fmaxf(top[1], dpp<kRowMirror>(top[1]));
        if (r >= r1) continue;                                    // whole rows of lanes
        // keys: the smallest 2^e >= 2^-100 with amax <= 6 * 2^e; 6 = 0.75 * 2^3
        const bool finite = top[0] < kInf;
        const int x2 = __builtin_amdgcn_frexp_expf(finite ? top[0] : 1.0f);
        const float f = __builtin_amdgcn_frexp_mantf(finite ? top[0] : 1.0f);
        int ex = f <= 0.75f ? x2 - 3 : x2 - 2;
        if (top[0] == 0.0f || ex < kLowestScale) ex = kLowestScale;
        const float s = __builtin_ldexpf(1.0f, ex);
        *reinterpret_cast<uint32_t*>(at.k + r * (D / 2) + lane * 4) = key_codes(e[0], s);
        if ((lane & 3) == 0)
            at.k_scale[key_scale_at<D>(r, lane >> 2)] =
                static_cast<uint8_t>(finite ? ex + 127 : 255);
        const float vs = value_scale(top[1]);
        const uint32_t c = value_codes<T>(e[1], vs);
        uint32_t* to = reinterpret_cast<uint32_t*>(codes + r * kPad + lane * 8);
        to[0] = c & 0x0F0F0F0Fu;
        to[1] = c >> 4 & 0x0F0F0F0Fu;
        if (lane == 0) at.v_scale[r] = from_f32<uint16_t>(vs);
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kPer; ++n) {
        if (mask[n] == 0u) continue;
        const int part = threadIdx.x + n * THREADS, t8 = (part & 3) * 8, d4 = (part >> 2) * 4;
        uint32_t y[4];                               // byte j: dimension dim_of(part, j), two tokens
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t* lo = reinterpret_cast<const uint32_t*>(codes + (t8 + 2 * i) * kPad + d4);
            // (tokens that are not new may have left anything there)
            y[i] = (lo[0] & 0x0F0F0F0Fu) | (lo[kPad / 4] & 0x0F0F0F0Fu) << 4;
        }
        // a 4 x 4 transpose of bytes
        const uint32_t a0 = __builtin_amdgcn_perm(y[1], y[0], 0x05010400u);
        const uint32_t a1 = __builtin_amdgcn_perm(y[1], y[0], 0x07030602u);
        const uint32_t b0 = __builtin_amdgcn_perm(y[3], y[2], 0x05010400u);
        const uint32_t b1 = __builtin_amdgcn_perm(y[3], y[2], 0x07030602u);
        uint32_t z[4] = {__builtin_amdgcn_perm(b0, a0, 0x05040100u),
                         __builtin_amdgcn_perm(b0, a0, 0x07060302u),
                         __builtin_amdgcn_perm(b1, a1, 0x05040100u),
                         __builtin_amdgcn_perm(b1, a1, 0x07060302u)};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (mask[n] != ~0u) z[j] = (z[j] & mask[n]) | (old[n][j] & ~mask[n]);
            *reinterpret_cast<uint32_t*>(at.v + dim_of(part, j) * 16 + (part & 3) * 4) = z[j];
        }
    }
}

template <typename T, int D>
hipError_t launch_append(const Append4Args& a, int64_t B, hipStream_t st) {
    const dim3 grid(static_cast<unsigned>(B * a.groups * a.c.G));
    // One wave is enough for the few tokens of a decoding step.
    if (std::min(a.T, kGroup4) * (D / 8) <= 64)
        hipLaunchKernelGGL((append4_kernel<T, D, 64, 1>), grid, dim3(64), 0, st, a);
    else
        hipLaunchKernelGGL((append4_kernel<T, D, 256, D / 64>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

struct Read4Args {
    Pool4Args c;
    void* dst[2];                    // either may be null
    const int32_t* start;
    const int32_t* count;            // or null
    int64_t ds[2][3];
    int T, groups;
};

template <typename T> struct alignas(16) Row8 { T x[8]; };

template <typename T, int D>
__global__ __launch_bounds__(256) void read4_kernel(const Read4Args a) {
    constexpr int kLanes = D / 8, kRows = 256 / kLanes, kPad = 20;
    __shared__ alignas(16) uint8_t held[D * kPad];   // [d][16] bytes of the group's values
    const uint32_t unit = blockIdx.x;
    const int g = static_cast<int>(unit % static_cast<uint32_t>(a.c.G));
    const uint32_t ub = unit / static_cast<uint32_t>(a.c.G);
    const int64_t b = ub / static_cast<uint32_t>(a.groups);
    const int64_t start = a.start[b];
    const int64_t count = a.count ? min(max(a.count[b], 0), a.T) : a.T;
    const int64_t end = start + count;
    const int64_t first = ((start >> 5) + ub % static_cast<uint32_t>(a.groups)) * kGroup4;
    if (first >= end) return;
    int page = -1;
    if (first >= 0 && first < static_cast<int64_t>(a.c.max_pages) << a.c.page_shift)
        page = a.c.pages[b * a.c.pages_stride + (first >> a.c.page_shift)];
    const bool there = page >= 0 && page < a.c.num_pages;
    const Group4<D> at(a.c, there ? page : 0, g,
                       there ? static_cast<int>(first) & (a.c.P - 1) : 0);
    const int r0 = static_cast<int>(max(start - first, int64_t{0}));
    const int r1 = static_cast<int>(min(end - first, static_cast<int64_t>(kGroup4)));
    const int lane = threadIdx.x % kLanes, sub = threadIdx.x / kLanes;
    if (a.dst[1] != nullptr) {
        for (int i = threadIdx.x; i < D; i += 256) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(at.v + i * 16);
            uint32_t* to = reinterpret_cast<uint32_t*>(held + i * kPad);
            to[0] = w.x;
            to[1] = w.y;
            to[2] = w.z;
            to[3] = w.w;
        }
        __syncthreads();
    }
    for (int r = r0 + sub; r < r1; r += kRows) {
        const int64_t row = first + r - start;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (a.dst[k] == nullptr) continue;
            uint32_t w = 0;
            float s;
            if (k == 0) {
                w = *reinterpret_cast<const uint32_t*>(at.k + r * (D / 2) + lane * 4);
                const uint32_t e = at.k_scale[key_scale_at<D>(r, lane >> 2)];
                s = e == 255u ? __builtin_nanf("") : __uint_as_float(e << 23);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    w |= (static_cast<uint32_t>(held[(lane * 8 + i) * kPad + (r >> 1)]) >>
                              (4 * (r & 1)) & 15u) << (4 * i);
                s = to_f32(at.v_scale[r]);
            }
            const f32x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0),
                                __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1),
                                __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2),
                                __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3)};
            Row8<T> y;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                y.x[i] = from_f32<T>(there ? p[i >> 1][i & 1] * s : 0.0f);
            *reinterpret_cast<Row8<T>*>(static_cast<T*>(a.dst[k]) + b * a.ds[k][0] +
                                        g * a.ds[k][1] + row * a.ds[k][2] + lane * 8) = y;
        }
    }
}

template <typename T>
hipError_t launch_read(const Read4Args& a, int64_t B, int D, hipStream_t st) {
    const dim3 grid(static_cast<unsigned>(B * a.groups * a.c.G));
    if (D == 64) hipLaunchKernelGGL((read4_kernel<T, 64>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((read4_kernel<T, 128>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

Pool4Args pool_args(const e2s_cache4& c, const int32_t* pages, int64_t pages_stride,
                    int max_pages) {
    Pool4Args p{};
    p.k = static_cast<uint8_t*>(c.k);
    p.v = static_cast<uint8_t*>(c.v);
    p.k_scale = static_cast<uint8_t*>(c.k_scale);
    p.v_scale = static_cast<uint16_t*>(c.v_scale);
    p.k_page = c.k_page_stride;
    p.v_page = c.v_page_stride;
    p.pages = pages;
    p.pages_stride = pages_stride;
    p.G = c.num_kv_heads;
    p.P = c.page_tokens;
    p.page_shift = __builtin_ctz(static_cast<unsigned>(c.page_tokens));   // a power of two
    p.num_pages = c.num_pages;
    p.max_pages = max_pages;
    return p;
}

// groups that T tokens can touch, starting anywhere in a group
int touched(int T) { return (T + kGroup4 - 2) / kGroup4 + 1; }

}  // namespace

hipError_t launch_cache4_append(const e2s_cache4& c, const e2s_cache_append_shape& s,
                                const int32_t* pages, const int32_t* start, const int32_t* count,
                                const int32_t* src_idx, const void* k, const void* v,
                                hipStream_t st) {
    Append4Args a{};
    a.c = pool_args(c, pages, s.pages_stride, s.max_pages);
    a.src[0] = k;
    a.src[1] = v;
    a.start = start;
    a.count = count;
    a.src_idx = src_idx;
    for (int i = 0; i < 3; ++i) {
        a.ss[0][i] = s.k_stride[i];
        a.ss[1][i] = s.v_stride[i];
    }
    a.T = s.num_tokens;
    a.N = s.src_tokens;
    a.groups = touched(s.num_tokens);
    const int D = c.head_dim;
    const int64_t B = s.batch;
    if (s.dtype == E2S_DTYPE_F32)
        return D == 64 ? launch_append<float, 64>(a, B, st) : launch_append<float, 128>(a, B, st);
    if (s.dtype == E2S_DTYPE_F16)
        return D == 64 ? launch_append<_Float16, 64>(a, B, st)
                       : launch_append<_Float16, 128>(a, B, st);
    return D == 64 ? launch_append<uint16_t, 64>(a, B, st)
                   : launch_append<uint16_t, 128>(a, B, st);
}

hipError_t launch_cache4_read(const e2s_cache4& c, const e2s_cache4_read_shape& s,
                              const int32_t* pages, const int32_t* start, const int32_t* count,
                              void* k_out, void* v_out, hipStream_t st) {
    Read4Args a{};
    a.c = pool_args(c, pages, s.pages_stride, s.max_pages);
    a.dst[0] = k_out;
    a.dst[1] = v_out;
    a.start = start;
    a.count = count;
    for (int i = 0; i < 3; ++i) {
        a.ds[0][i] = s.k_out_stride[i];
        a.ds[1][i] = s.v_out_stride[i];
    }
    a.T = s.num_tokens;
    a.groups = touched(s.num_tokens);
    if (s.dtype == E2S_DTYPE_F32) return launch_read<float>(a, s.batch, c.head_dim, st);
    if (s.dtype == E2S_DTYPE_F16) return launch_read<_Float16>(a, s.batch, c.head_dim, st);
    return launch_read<uint16_t>(a, s.batch, c.head_dim, st);
}

}  // namespace e2s
