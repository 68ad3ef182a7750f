// Attention over the 4-bit cache (e2s_cache4_attend).
//
//   s = scale * q . k over the cached tokens a query sees, p = softmax(s), out = sum p v
//
// The cached bytes go from memory into the matrix instructions as they are: nothing is widened
// and nothing crosses LDS on the way.  A step is 128 keys of a wave's 16 query rows,
//   S^T [16 keys x 16 rows] = K Q^T      8 products of 16 x 16 x 128
//   O^T [16 dims x 16 rows] += V^T P^T   d / 16 products
// with the 4-bit operand on the left and e4m3 terms of the queries, or of the weights, on
// the right.  The instruction takes a power-of-two scale per 32 elements of either operand:
// the keys' own scales on one side, the terms' on the other.  In its layout
//   left    lane (m, g) holds k = 32 g .. 32 g + 31 of row m, and their scale
//   right   lane (n, g) holds k = 16 g .. 16 g + 15 and 64 + 16 g .. 64 + 16 g + 15 of column n,
//           and the scale of k = 32 g .. 32 g + 31
//   result  lane (n, g) holds rows 4 g .. 4 g + 3 of column n.
// Row m = 4 g + r of tile t = 4 f + u is made key 64 f + 16 g + 4 u + r of the step, so that
// a lane's results are the very weights that it holds of the right operand of the second
// product; the page layout puts the 16 bytes and 4 scales of every lane side by side.
//
// A query is the sum of 2, 3 or 6 e4m3 terms (bf16, f16, f32), a weight times its value's scale
// of 3, 4 or 6: each term takes 4 bits off what is left, and its scale is 2^-4 of the last
// one's.  The weights' terms are on a scale of the row's largest among the 128.  With d = 64
// the two halves of a key product's k take two terms of the query at once.
//
// One pass: a running maximum and sum per row; the maximum is raised (and the output rescaled)
// only when a logit passes it by 2^8 in the exponential.  16 rows to a workgroup, whose waves
// part its keys and merge in LDS; keys are split over workgroups where there are few rows, and
// attend4_join_kernel joins the parts.
//
// What bounds it.  A decoding step reads 133 bytes per token and key head (d = 128, of 258 in 8
// bits): 64 sequences of 4096 keys, 32 heads, take 196 us (5.75 TB/s; f16 200, f32 209).  Of 4
// sequences of 60000 to 131072 keys this kernel takes 35 us (4.8 TB/s) and the join 5, of 64 of 130
// to 1200 keys, 32 heads, f16, 46: there the longest wave's steps.
// With many rows neither unit is full: 2 x 1024 queries of 2048 keys, 28 heads, bf16, take 78 to
// 90 us (f16 97, f32 136), 500 to 580 TFLOP/s of the 45 GFLOP that the mask leaves.  Those are
// 44800 steps of 504 vector instructions and 40 matrix products.  By counters the vector unit is at
// work for 54 % of the time and the matrix unit for 28 %; a SIMD has 1.3 waves on average of the
// two that fit (3584 waves of 9 to 16 steps on 2048 places), and a wave alone seldom has products
// and conversions under way at once.  Waves wait 35 % of their time for a turn to issue, 16 % for
// what they read.  Two waves to a SIMD (213 registers) hold a step's keys and values: three
// waves spilled (107 us for 91).  What the
// steps of making it fast gave for the 1024 queries, in us: 155 as first written; 116 with two
// waves to a SIMD; 102 with loops that leave keys and outputs in place; 91 with addresses from
// one lookup a segment and maxima without the compiler's quieting; 89 with the values' loads
// before the logits and the keys' after them.  Logits of the next step beside this one's weights
// (245 registers) gave nothing: 103 for 102.
#include <type_traits>

#include "serve_device.h"
#include "step_kernels.h"

namespace e2s {
namespace {

constexpr int kTile = 16;
constexpr float kInf = __builtin_huge_valf();
constexpr float kRaise = 8.0f;       // log2 by which a logit may pass the maximum
// Outputs are held at 2^-24 of their size, by the values' scale in the products: up to 2^20
// weights (2^kRaise each) times values below 2^116 stay finite.
constexpr int kDown = 24;
constexpr float kDownScale = 1.0f / (1 << kDown);

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

struct Attend4Args {
    const uint8_t* k;
    const uint8_t* v;
    const uint8_t* k_scale;
    const uint16_t* v_scale;
    int64_t k_page, v_page, pages_stride;
    const int32_t* pages;
    const int32_t* lengths;
    const int32_t* q_count;          // or null
    const void* q;
    void* out;
    float* part_max;                 // [B, Hkv, rows, splits], or null with one split
    float* part_sum;
    float* part_out;                 // [B, Hkv, rows, splits, d]
    int64_t chunk;
    int64_t qs[3], os[3];
    int G, group, T, rows, row_groups, splits;
    int P, page_shift, num_pages, max_pages, max_tokens, causal;
    float scale;                     // logit scale times log2(e)
};

__device__ __forceinline__ int length_of(const Attend4Args& a, int64_t b) {
    const int64_t cap = min(static_cast<int64_t>(a.max_pages) << a.page_shift,
                            static_cast<int64_t>(a.max_tokens));
    return static_cast<int>(min(static_cast<int64_t>(max(a.lengths[b], 0)), cap));
}
__device__ __forceinline__ int count_of(const Attend4Args& a, int64_t b) {
    return a.q_count ? min(max(a.q_count[b], 0), a.T) : a.T;
}
// Tokens that query t of `count` sees.
__device__ __forceinline__ int seen_by(const Attend4Args& a, int len, int count, int t) {
    return a.causal ? max(0, len - (count - 1 - t)) : len;
}

template <typename T> struct Terms4;             // e4m3 terms of a query, of a weight
template <> struct Terms4<uint16_t> { static constexpr int q = 2, p = 3; };
template <> struct Terms4<_Float16> { static constexpr int q = 3, p = 4; };
template <> struct Terms4<float> { static constexpr int q = 6, p = 6; };

// The biased exponent of a scale that takes magnitudes up to m, once they are rounded to 4
// bits, to below 4 (and m to 1.9 at least); not under 39, so that the terms' scales stay normal.
// The instruction adds eight neighbouring products with 13 bits below the largest one's
// exponent, and drops what is lower: a 256 beside it costs a 2^-6 all its bits.  On this scale
// nothing is lower: terms are below 4 and multiples of 2^-9, e4m3's smallest step, so products
// are multiples of 2^-10, 13 bits under the largest exponent that they can have, 3.  (One term of
// 4 would cost a row of float32 1e-5.)
__device__ __forceinline__ int term_exponent(float m) {
    return max(static_cast<int>((__float_as_uint(m) + (1u << 19)) >> 23 & 0xFFu), 40) - 1;
}
__device__ __forceinline__ float exponent_scale(int e) { return __int_as_float(e << 23); }

// Four values to a word of e4m3 bytes at a scale; the values become what that leaves of them.
template <bool LAST>
__device__ __forceinline__ int take_term(f32x4& x, float scale) {
    s16x2 w;
    asm volatile("" : "=v"(w));      // any register: both halves are written
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[0], x[1], scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[2], x[3], scale, true);
    const uint32_t bits = __builtin_bit_cast(uint32_t, w);
    if constexpr (!LAST) {
        const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(bits, scale, false);
        const f32x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(bits, scale, true);
        x[0] -= lo.x;
        x[1] -= lo.y;
        x[2] -= hi.x;
        x[3] -= hi.y;
    }
    return static_cast<int>(bits);
}

// a [16 x 128] 4-bit times b [128 x 16] e4m3, scales in byte SA of sa and byte SB of sb.
template <int SA, int SB>
__device__ __forceinline__ f32x4 product(const u32x4& a, const i32x8& b, const f32x4& c, int sa,
                                         int sb) {
    const i32x8 w = {static_cast<int>(a.x), static_cast<int>(a.y), static_cast<int>(a.z),
                     static_cast<int>(a.w), 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, b, c, 4, 0, SA, sa, SB, sb);
}
template <int SB>
__device__ __forceinline__ f32x4 key_product(int u, const u32x4& a, const i32x8& b, const f32x4& c,
                                             int sa, int sb) {
    switch (u) {                                 // a constant where it is unrolled
        case 0: return product<0, SB>(a, b, c, sa, sb);
        case 1: return product<1, SB>(a, b, c, sa, sb);
        case 2: return product<2, SB>(a, b, c, sa, sb);
        default: return product<3, SB>(a, b, c, sa, sb);
    }
}
__device__ __forceinline__ f32x4 key_product(int m, int u, const u32x4& a, const i32x8& b,
                                             const f32x4& c, int sa, int sb) {
    switch (m & 3) {
        case 0: return key_product<0>(u, a, b, c, sa, sb);
        case 1: return key_product<1>(u, a, b, c, sa, sb);
        case 2: return key_product<2>(u, a, b, c, sa, sb);
        default: return key_product<3>(u, a, b, c, sa, sb);
    }
}

__device__ __forceinline__ f32x4 value_product(int i, const u32x4& a, const i32x8& b,
                                               const f32x4& c, int sb) {
    constexpr int kUnit = 127 - kDown;
    switch (i & 3) {
        case 0: return product<0, 0>(a, b, c, kUnit, sb);
        case 1: return product<0, 1>(a, b, c, kUnit, sb);
        case 2: return product<0, 2>(a, b, c, kUnit, sb);
        default: return product<0, 3>(a, b, c, kUnit, sb);
    }
}

// (the compiler would quieten every operand of its own first)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// The maximum over a column's lanes, g = 0 .. 3: rows of 16 lanes change places with their
// neighbours, then halves of the wave.
__device__ __forceinline__ float across_rows(float v) {
    typedef unsigned int u32x2a __attribute__((ext_vector_type(2)));
    u32x2a p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(p.x), __uint_as_float(p.y));
    p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(p.x), __uint_as_float(p.y));
}

template <typename T, int N> struct alignas(N * sizeof(T) < 16 ? N * sizeof(T) : 16) Run4 {
    T x[N];
};

// 16 rows to a workgroup, whose waves part its keys.
template <typename T, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void attend4_kernel(
    const Attend4Args a) {
    constexpr int kQ = Terms4<T>::q, kP = Terms4<T>::p;
    constexpr int kHalves = D == 128 ? 1 : 2;            // terms of a product's k
    constexpr int kQm = (kQ + kHalves - 1) / kHalves;    // key products of a tile
    constexpr int kDims = D / kTile;
    constexpr int kPad = D + 4;
    // the queries' operands; the waves' outputs at the end
    __shared__ union {
        i32x4 q[kQm][2][64];
        float out[WAVES > 1 ? WAVES : 1][kTile][kPad];
    } lds;
    __shared__ float top_of[WAVES][kTile], sum_of[WAVES][kTile];

    uint32_t id = blockIdx.x;
    // (causal: the last rows, which see the most, first)
    const int rg = a.row_groups - 1 - static_cast<int>(id % static_cast<uint32_t>(a.row_groups));
    id /= static_cast<uint32_t>(a.row_groups);
    const int split = static_cast<int>(id % static_cast<uint32_t>(a.splits));
    id /= static_cast<uint32_t>(a.splits);
    const int g = static_cast<int>(id % static_cast<uint32_t>(a.G));
    const int64_t b = id / static_cast<uint32_t>(a.G);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, g4 = lane >> 4;

    const int len = length_of(a, b), count = count_of(a, b);
    const int row0 = rg * kTile;
    const int row_end = min(row0 + kTile, count * a.group);
    if (row0 >= row_end) return;
    // what the first row and the last row see
    const int least = seen_by(a, len, count, row0 / a.group);
    const int most = seen_by(a, len, count, (row_end - 1) / a.group);
    const int64_t key_begin = split * a.chunk;
    if (split > 0 && key_begin >= most) return;
    const int row = row0 + n16;
    const bool live = row < row_end;
    const int at_t = live ? row / a.group : 0, at_h = live ? row - at_t * a.group : 0;
    // rows that do not exist see everything, so that they mask nothing
    const int limit = live ? seen_by(a, len, count, at_t) : a.max_tokens;
    // this wave's keys: an equal share of the steps that the rows see
    const int begin = static_cast<int>(min(key_begin, static_cast<int64_t>(most)));
    const int end_of = static_cast<int>(min(key_begin + a.chunk, static_cast<int64_t>(most)));
    const int share = ((end_of - begin + kStep4 - 1) / kStep4 + WAVES - 1) / WAVES * kStep4;
    const int w0 = min(begin + wave * share, end_of);
    const int w1 = min(w0 + share, end_of);

    // Queries as operands: the first wave lays them out.  Lane (n, g4) holds
    // elements lo .. lo + 15 and hi .. hi + 15 of row n; d = 64: the same twice, of two terms.
    int qs[(kQ + 3) / 4 + 1];                            // scales of the terms, a byte each
    {
        const int lo = 16 * g4, hi = D == 128 ? 64 + 16 * g4 : lo;
        f32x4 x[8];
        const T* src = static_cast<const T*>(a.q) + b * a.qs[0] +
                       (static_cast<int64_t>(g) * a.group + at_h) * a.qs[1] + at_t * a.qs[2];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            Packet<T> p{};
            if (live) load_packet(p, src + (w < 2 ? lo : hi) + (w & 1) * 8);
            float f[8];
            unpack(p, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[2 * w + (i >> 2)][i & 3] = f[i];
        }
        float m[2] = {0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < 8; ++w)
#pragma unroll
            for (int i = 0; i < 4; ++i) m[w >> 2] = fmaxf(m[w >> 2], fabsf(x[w][i]));
        int e[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) e[h] = term_exponent(fmaxf(m[h], __shfl_xor(m[h], 16)));
        // this lane's scale is that of elements 32 g4 .. (d = 64: 32 (g4 & 1) .., term g4 >> 1)
        const int from = n16 + 32 * (g4 & 1);
        const int e_lo = __shfl(e[0], from), e_hi = __shfl(e[1], from);
        const int mine = D == 128 ? (g4 < 2 ? e_lo : e_hi) : e_lo - 4 * (g4 >> 1);
#pragma unroll
        for (int w = 0; w < static_cast<int>(sizeof(qs) / 4); ++w) qs[w] = 0;
#pragma unroll
        for (int i = 0; i < kQm; ++i)
            qs[i >> 2] |= (mine - 4 * kHalves * i) << (8 * (i & 3));
        if (wave == 0) {
#pragma unroll
            for (int i = 0; i < kQm * kHalves; ++i) {
                i32x4 t[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
                if (i < kQ) {
#pragma unroll
                    for (int w = 0; w < 8; ++w) {
                        if (kHalves == 2 && w >= 4) break;
                        const int word =
                            take_term<false>(x[w], exponent_scale(e[w >> 2] - 4 * i));
                        if (w < 4) t[0][w] = word;
                        else t[1][w - 4] = word;
                    }
                }
                if constexpr (kHalves == 1) {
                    lds.q[i][0][lane] = t[0];
                    lds.q[i][1][lane] = t[1];
                } else {
                    lds.q[i >> 1][i & 1][lane] = t[0];
                }
            }
        }
    }
    __syncthreads();

    // Lane l looks up group l (32 keys) of a segment of 64: its page (-1: none), the byte offsets
    // of its keys and its values, and the number of its first token and head among all.  (Groups
    // without a page read the first page's, unused.)
    constexpr int kSegment = 64 * kGroup4;
    struct Segment {
        int page;
        int64_t k, v, token;
    };
    const int64_t head = static_cast<int64_t>(g) * (D / 2) << a.page_shift;
    auto look_up = [&](int seg) {
        Segment w;
        const int key = seg + lane * kGroup4, row = key & (a.P - 1);
        int pg = -1;
        if (key < w1) pg = a.pages[b * a.pages_stride + (key >> a.page_shift)];
        w.page = pg < a.num_pages ? max(pg, -1) : -1;
        const int64_t at = max(w.page, 0);
        w.k = at * a.k_page + head + row * (D / 2);
        w.v = at * a.v_page + head + row * (D / 2);
        w.token = ((at * a.G + g) << a.page_shift) + row;
        return w;
    };
    auto from_lane = [&](int64_t x, int index) {
        const int lo = __builtin_amdgcn_ds_bpermute(index, static_cast<int>(x));
        const int hi = __builtin_amdgcn_ds_bpermute(index, static_cast<int>(x >> 32));
        return static_cast<int64_t>(hi) << 32 | static_cast<uint32_t>(lo);
    };
    // A step's operands, as loaded.
    u32x4 kx[8], vx[kDims], vs[4];
    uint32_t ks[2];
    // lane constants: of its keys' rows, their scales, its value rows, and the values' scales
    const int k_tok = 16 * (n16 >> 2 & 1) + (n16 & 3);
    const int k_block = D == 128 ? g4 : g4 & 1;
    const uint8_t* const k_lane = a.k + k_tok * (D / 2) + k_block * 16;
    const uint8_t* const ks_lane =
        a.k_scale + (n16 >> 2 & 1) * (D / 2) + ((n16 & 3) * (D / 32) + k_block) * 4;
    const uint8_t* const v_lane = a.v + n16 * 16;
    const uint16_t* const vs_lane = a.v_scale + 16 * (g4 & 1);
    // the lane (times 4) of its keys', its values' and its values' scales' first group in a segment
    const int k_from = (n16 >> 3) * 4, v_from = g4 * 4, vs_from = (g4 >> 1) * 4;
    auto fetch_k = [&](const Segment& w, int key) {      // key: of the segment
        const int at = (key >> 5) * 4 + k_from;
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            const uint8_t* p = k_lane + from_lane(w.k, at + 8 * f);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                kx[4 * f + u] = *reinterpret_cast<const u32x4*>(p + u * 2 * D);
            ks[f] = *reinterpret_cast<const uint32_t*>(ks_lane +
                                                       from_lane(w.token, at + 8 * f) * (D / 32));
        }
    };
    auto fetch_v = [&](const Segment& w, int key) {
        const int at = (key >> 5) * 4;
        const uint8_t* p = v_lane + from_lane(w.v, at + v_from);
        const u32x4* s[2];
#pragma unroll
        for (int f = 0; f < 2; ++f)
            s[f] = reinterpret_cast<const u32x4*>(vs_lane +
                                                  from_lane(w.token, at + vs_from + 8 * f));
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            vs[2 * f] = s[f][0];
            vs[2 * f + 1] = s[f][1];
        }
#pragma unroll
        for (int j = 0; j < kDims; ++j) vx[j] = *reinterpret_cast<const u32x4*>(p + j * 256);
    };

    f32x4 o[kDims];
    float top = -kInf, base = 0.0f, sum = 0.0f;  // running maximum; the same, 0 before any
#pragma unroll
    for (int j = 0; j < kDims; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};

    f32x4 s[8];                          // logits before their scale
    // The parts of a step of 128 keys.
    auto read_query = [&](int i) {
        // an index that the compiler cannot know keeps the queries' reads in the loop
        int my = lane;
        asm volatile("" : "+v"(my));
        const i32x4 q0 = lds.q[i][0][my], q1 = lds.q[i][1][my];
        return i32x8{q0.x, q0.y, q0.z, q0.w, q1.x, q1.y, q1.z, q1.w};
    };
    auto logit_term = [&](int i, int t, const i32x8& q, const f32x4& c) {
        return key_product(i, t & 3, kx[t], q, c, static_cast<int>(ks[t >> 2]), qs[i >> 2]);
    };
    // Lane (n, g4): s[4 f + u][r] is key 64 f + 16 g4 + 4 u + r; -inf where it is not seen.
    auto mask = [&](const Segment& w, int seg, int key) {
        int page[2];                             // of the lane's two groups
#pragma unroll
        for (int f = 0; f < 2; ++f)
            page[f] = __builtin_amdgcn_ds_bpermute((key >> 5) * 4 + vs_from + 8 * f, w.page);
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const int end = page[t >> 2] >= 0 ? limit : 0;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (seg + key + 64 * (t >> 2) + 16 * g4 + 4 * (t & 3) + r >= end) s[t][r] = -kInf;
        }
    };
    auto raise = [&]() {
        float mx = -kInf;
#pragma unroll
        for (int i = 0; i < 32; i += 2) mx = max3(mx, s[i >> 2][i & 3], s[i >> 2][(i & 3) + 1]);
        mx *= a.scale;
        if (__ballot(mx > top + kRaise)) {
            // (a whole number: what is taken from the logits is exact)
            mx = ceilf(across_rows(mx));
            const float up = fmaxf(top, mx);
            const float shrink = up == top ? 1.0f : __builtin_amdgcn_exp2f(top - up);
            top = up;
            base = up == -kInf ? 0.0f : up;
            sum *= shrink;
#pragma unroll
            for (int j = 0; j < kDims; ++j) o[j] *= shrink;
        }
    };
    // One step, of key `key` of the segment that starts at seg, with key `ahead` behind it.
    // `whole`: every row sees every key of it.
    auto step = [&](auto whole_tag, const Segment& now, int seg, int key, int ahead) {
        constexpr bool kWhole = decltype(whole_tag)::value;
        fetch_v(now, key);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = kQm - 1; i >= 0; --i) {
            const i32x8 q = read_query(i);
#pragma unroll
            for (int t = 0; t < 8; ++t)
                s[t] = logit_term(i, t, q, i == kQm - 1 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[t]);
        }
        // (the loads take the registers of what they follow, and no others)
        __builtin_amdgcn_sched_barrier(0);
        fetch_k(now, ahead);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!kWhole) mask(now, seg, key);
        raise();
        // logits to weights times their values' scales
        uint32_t pm = 0;                         // the largest: their bits are ordered as they are
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const uint32_t w2[2] = {vs[t >> 1][2 * (t & 1)], vs[t >> 1][2 * (t & 1) + 1]};
            float part[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float x = s[t][r];
                part[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x, a.scale, -base));
                const float f = r & 1 ? bf16hi(w2[r >> 1]) : bf16lo(w2[r >> 1]);
                // (what is not seen may have any scale)
                s[t][r] = !kWhole && x == -kInf ? 0.0f : part[r] * f;
            }
            pm = max(max(pm, __float_as_uint(s[t][0])), __float_as_uint(s[t][1]));
            pm = max(max(pm, __float_as_uint(s[t][2])), __float_as_uint(s[t][3]));
            sum += (part[0] + part[1]) + (part[2] + part[3]);
        }
        __builtin_amdgcn_sched_barrier(0);
        const int e = term_exponent(across_rows(__uint_as_float(pm)));
        int es = 0, es2 = 0;
#pragma unroll
        for (int i = 0; i < kP; ++i) (i < 4 ? es : es2) |= (e - 4 * i) << (8 * (i & 3));
        // A term's products beside the conversion of the next one's words: the vector unit and
        // the matrix unit work side by side where a wave's instructions alternate, which the
        // scheduling fences keep them to.
        i32x8 w[2];
#pragma unroll
        for (int t = 0; t < 8; ++t) w[0][t] = take_term<false>(s[t], exponent_scale(e));
#pragma unroll
        for (int i = 0; i < kP; ++i) {
            const float sc = exponent_scale(e - 4 * (i + 1));
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j < kDims) o[j] = value_product(i, vx[j], w[i & 1], o[j], i < 4 ? es : es2);
                if (i + 1 < kP)
                    w[(i + 1) & 1][j] =
                        i + 2 < kP ? take_term<false>(s[j], sc) : take_term<true>(s[j], sc);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };

    // A segment's steps that every row sees whole, all pages there, come first, by code that
    // masks nothing; the others by code that does.
    for (int seg = w0; seg < w1; seg += kSegment) {
        const Segment now = look_up(seg);
        fetch_k(now, 0);
        const int end = min(w1 - seg, kSegment);
        const bool paged = __ballot(lane * kGroup4 < end && now.page < 0) == 0;
        const int whole_end = paged ? min(end, least - seg) : 0;
        // (behind the last step nothing follows: the same again, unused)
        auto ahead = [&](int key) { return key + kStep4 < end ? key + kStep4 : key; };
        int key = 0;
        for (; key + kStep4 <= whole_end; key += kStep4)
            step(std::true_type{}, now, seg, key, ahead(key));
        for (; key < end; key += kStep4) step(std::false_type{}, now, seg, key, ahead(key));
    }

    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    sum *= kDownScale;
    const int64_t lines = (b * a.G + g) * static_cast<int64_t>(a.rows);
    auto put = [&](int r, int d0, const float (&y)[4], float m, float total) {
        const int the_row = row0 + r;
        if (a.splits == 1) {
            const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
            const int t = the_row / a.group;
            T* to = static_cast<T*>(a.out) + b * a.os[0] +
                    (static_cast<int64_t>(g) * a.group + the_row - t * a.group) * a.os[1] +
                    t * a.os[2] + d0;
            Run4<T, 4> z;
#pragma unroll
            for (int i = 0; i < 4; ++i) z.x[i] = from_f32<T>(y[i] * inv);
            *reinterpret_cast<Run4<T, 4>*>(to) = z;
        } else {
            const int64_t part = (lines + the_row) * a.splits + split;
            *reinterpret_cast<f32x4*>(a.part_out + part * D + d0) = f32x4{y[0], y[1], y[2], y[3]};
            if (d0 == 0) {
                a.part_max[part] = m;
                a.part_sum[part] = total;
            }
        }
    };
    if constexpr (WAVES == 1) {
        // lane (n, g4) holds dimensions 16 j + 4 g4 .. of row n
        if (live) {
#pragma unroll
            for (int j = 0; j < kDims; ++j) {
                const float y[4] = {o[j][0], o[j][1], o[j][2], o[j][3]};
                put(n16, kTile * j + 4 * g4, y, top, sum);
            }
        }
    } else {
        __syncthreads();                         // all have read their last queries
        if (g4 == 0) {
            top_of[wave][n16] = top;
            sum_of[wave][n16] = sum;
        }
        __syncthreads();
        float all = top_of[0][n16];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) all = fmaxf(all, top_of[w][n16]);
        const float f = top == -kInf ? 0.0f : top == all ? 1.0f : __builtin_amdgcn_exp2f(top - all);
#pragma unroll
        for (int j = 0; j < kDims; ++j) {
            const f32x4 y = {o[j][0] * f, o[j][1] * f, o[j][2] * f, o[j][3] * f};
            *reinterpret_cast<f32x4*>(&lds.out[wave][n16][kTile * j + 4 * g4]) = y;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < kTile * D / 4; i += 64 * WAVES) {
            const int r = i / (D / 4), d0 = i % (D / 4) * 4;
            if (row0 + r >= row_end) continue;
            float m = top_of[0][r];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) m = fmaxf(m, top_of[w][r]);
            float total = 0.0f, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                // without a maximum a sum is 0, or NaN, which stays
                const float tw = top_of[w][r];
                total += sum_of[w][r] *
                         (tw == m || tw == -kInf ? 1.0f : __builtin_amdgcn_exp2f(tw - m));
                const f32x4 x = *reinterpret_cast<const f32x4*>(&lds.out[w][r][d0]);
#pragma unroll
                for (int k = 0; k < 4; ++k) y[k] += x[k];
            }
            put(r, d0, y, m, total);
        }
    }
}

// The parts of a row joined, 4 dimensions to a thread, PARTS threads to every 4 dimensions: one
// takes the first of them, and every PARTS-th behind it.  A part is there where its first key is
// seen by the workgroup that wrote it; parts whose keys this row does not see hold a maximum of
// -inf (and zeros, or NaN, which only rows that do not exist make).
template <typename T, int D, int PARTS>
__global__ __launch_bounds__(256) void attend4_join_kernel(const Attend4Args a, uint32_t lines) {
    constexpr int kLanes = D / 4, kLines = 256 / (kLanes * PARTS);
    __shared__ float tops[PARTS > 1 ? PARTS : 1][kLines][kLanes];
    __shared__ float sums[PARTS > 1 ? PARTS : 1][kLines][kLanes];
    __shared__ f32x4 outs[PARTS > 1 ? PARTS : 1][kLines][kLanes];
    const int lane = threadIdx.x % kLanes, part0 = threadIdx.x / kLanes % PARTS;
    const int which = threadIdx.x / (kLanes * PARTS), d0 = lane * 4;
    const uint32_t line = blockIdx.x * kLines + which;
    const uint32_t bg = line < lines ? line / static_cast<uint32_t>(a.rows) : 0;
    const int row = line < lines ? static_cast<int>(line - bg * static_cast<uint32_t>(a.rows)) : 0;
    const int64_t b = bg / static_cast<uint32_t>(a.G);
    const int g = static_cast<int>(bg - static_cast<uint32_t>(b) * a.G);
    const int t = row / a.group;
    const int len = length_of(a, b), count = count_of(a, b);
    const bool live = line < lines && t < count;
    const int chunk = static_cast<int>(a.chunk);
    const int parts = live ? (seen_by(a, len, count, t) + chunk - 1) / chunk : 0;     // <= splits
    const int64_t first = static_cast<int64_t>(line) * a.splits;
    float m = -kInf, total = 0.0f;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = part0; i0 < parts; i0 += 4 * PARTS) {
        f32x4 x[4];
        float pm[4], ps[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {            // loads of four parts under way at once
            const int i = i0 + j * PARTS;
            const int64_t at = first + min(i, parts - 1);
            x[j] = *reinterpret_cast<const f32x4*>(a.part_out + at * D + d0);
            pm[j] = i < parts ? a.part_max[at] : -kInf;
            ps[j] = i < parts ? a.part_sum[at] : 0.0f;
        }
        // (maxima are whole numbers: their distances' powers of two are exact)
        const float up = fmaxf(fmaxf(fmaxf(pm[0], pm[1]), fmaxf(pm[2], pm[3])), m);
        const float old = m == up ? 1.0f : __builtin_amdgcn_exp2f(m - up);
        total *= old;
        y *= old;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (i0 + j * PARTS >= parts) break;
            // without a maximum sum and output are 0, or NaN, which stays
            const float f = pm[j] == up || pm[j] == -kInf ? 1.0f
                                                          : __builtin_amdgcn_exp2f(pm[j] - up);
            total += ps[j] * f;
            y += x[j] * f;
        }
        m = up;
    }
    if constexpr (PARTS > 1) {
        tops[part0][which][lane] = m;
        sums[part0][which][lane] = total;
        outs[part0][which][lane] = y;
        __syncthreads();
        if (part0 > 0) return;
#pragma unroll
        for (int i = 1; i < PARTS; ++i) m = fmaxf(m, tops[i][which][lane]);
        total = 0.0f;
        y = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < PARTS; ++i) {
            const float of = tops[i][which][lane];
            const float f = of == m || of == -kInf ? 1.0f : __builtin_amdgcn_exp2f(of - m);
            total += sums[i][which][lane] * f;
            y += outs[i][which][lane] * f;
        }
    }
    if (!live) return;
    const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
    T* to = static_cast<T*>(a.out) + b * a.os[0] +
            (static_cast<int64_t>(g) * a.group + row - t * a.group) * a.os[1] + t * a.os[2] + d0;
    Run4<T, 4> z;
#pragma unroll
    for (int k = 0; k < 4; ++k) z.x[k] = from_f32<T>(y[k] * inv);
    *reinterpret_cast<Run4<T, 4>*>(to) = z;
}

template <typename T, int D, int PARTS>
void launch_join(const Attend4Args& a, int64_t lines, hipStream_t st) {
    const int per = 256 / (D / 4 * PARTS);
    hipLaunchKernelGGL((attend4_join_kernel<T, D, PARTS>),
                       dim3(static_cast<unsigned>((lines + per - 1) / per)), dim3(256), 0, st, a,
                       static_cast<uint32_t>(lines));
}

template <typename T, int D, int WAVES>
void launch_k(const Attend4Args& a, dim3 grid, hipStream_t st) {
    hipLaunchKernelGGL((attend4_kernel<T, D, WAVES>), grid, dim3(64 * WAVES), 0, st, a);
}

template <typename T, int D>
hipError_t launch_d(const Attend4Args& a, const Attend4Plan& p, int64_t heads, hipStream_t st) {
    const dim3 grid(static_cast<unsigned>(heads * p.row_groups * p.splits));
    switch (p.waves) {
        case 1: launch_k<T, D, 1>(a, grid, st); break;
        case 2: launch_k<T, D, 2>(a, grid, st); break;
        case 4: launch_k<T, D, 4>(a, grid, st); break;
        default: launch_k<T, D, 8>(a, grid, st); break;
    }
    if (p.splits > 8) launch_join<T, D, 8>(a, heads * p.rows, st);
    else if (p.splits > 1) launch_join<T, D, 1>(a, heads * p.rows, st);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_t(const Attend4Args& a, const Attend4Plan& p, int64_t heads, int D,
                    hipStream_t st) {
    return D == 64 ? launch_d<T, 64>(a, p, heads, st) : launch_d<T, 128>(a, p, heads, st);
}

}  // namespace

hipError_t launch_cache4_attend(const e2s_cache4& c, const e2s_cache4_attend_shape& s,
                                const int32_t* pages, const int32_t* lengths,
                                const int32_t* q_count, const void* q, void* out, void* workspace,
                                hipStream_t st) {
    const Attend4Plan p = attend4_plan(c, s);
    Attend4Args a{};
    a.k = static_cast<const uint8_t*>(c.k);
    a.v = static_cast<const uint8_t*>(c.v);
    a.k_scale = static_cast<const uint8_t*>(c.k_scale);
    a.v_scale = static_cast<const uint16_t*>(c.v_scale);
    a.k_page = c.k_page_stride;
    a.v_page = c.v_page_stride;
    a.pages_stride = s.pages_stride;
    a.pages = pages;
    a.lengths = lengths;
    a.q_count = q_count;
    a.q = q;
    a.out = out;
    if (p.splits > 1) {
        uint8_t* w = static_cast<uint8_t*>(workspace);
        a.part_max = reinterpret_cast<float*>(w + p.max_off);
        a.part_sum = reinterpret_cast<float*>(w + p.sum_off);
        a.part_out = reinterpret_cast<float*>(w + p.part_off);
    }
    a.chunk = p.chunk;
    for (int i = 0; i < 3; ++i) {
        a.qs[i] = s.q_stride[i];
        a.os[i] = s.out_stride[i];
    }
    a.G = c.num_kv_heads;
    a.group = s.num_heads / c.num_kv_heads;
    a.T = s.num_queries;
    a.rows = static_cast<int>(p.rows);
    a.row_groups = static_cast<int>(p.row_groups);
    a.splits = static_cast<int>(p.splits);
    a.P = c.page_tokens;
    a.page_shift = __builtin_ctz(static_cast<unsigned>(c.page_tokens));   // a power of two
    a.num_pages = c.num_pages;
    a.max_pages = s.max_pages;
    a.max_tokens = s.max_tokens;
    a.causal = s.causal;
    const float scale =
        s.scale > 0.0f ? s.scale : 1.0f / sqrtf(static_cast<float>(c.head_dim));
    a.scale = scale * 1.44269504088896340736f;
    const int64_t heads = static_cast<int64_t>(s.batch) * c.num_kv_heads;
    if (s.dtype == E2S_DTYPE_F32) return launch_t<float>(a, p, heads, c.head_dim, st);
    if (s.dtype == E2S_DTYPE_F16) return launch_t<_Float16>(a, p, heads, c.head_dim, st);
    return launch_t<uint16_t>(a, p, heads, c.head_dim, st);
}

}  // namespace e2s
