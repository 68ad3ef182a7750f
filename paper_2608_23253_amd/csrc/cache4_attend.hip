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
// only when a logit passes it by 2^8 in the exponential.  Waves take rows of 16, or part the
// keys and merge in LDS; keys are split over workgroups where there are few rows, and
// attend4_join_kernel joins the parts.
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
__device__ __forceinline__ int take_term(float (&x)[4], float scale) {
    s16x2 w = {0, 0};
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

__device__ __forceinline__ float across_rows(float v) {      // the maximum over a column's lanes
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}

// 16 of the cache's bytes; read once: past the caches.
template <bool ONCE>
__device__ __forceinline__ u32x4 load_keys(const uint8_t* p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    else return *reinterpret_cast<const u32x4*>(p);
}

template <typename T, int N> struct alignas(N * sizeof(T) < 16 ? N * sizeof(T) : 16) Run4 {
    T x[N];
};

// WAVES waves, ROW_WAVES of them along the rows (16 each), the others along the keys.
template <typename T, int D, int WAVES, int ROW_WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES == 8 ? 2 : 1) void attend4_kernel(
    const Attend4Args a) {
    constexpr int kQ = Terms4<T>::q, kP = Terms4<T>::p;
    constexpr int kHalves = D == 128 ? 1 : 2;            // terms of a product's k
    constexpr int kQm = (kQ + kHalves - 1) / kHalves;    // key products of a tile
    constexpr int kDims = D / kTile;
    constexpr int kKeyWaves = WAVES / ROW_WAVES;
    constexpr int kPad = D + 4;
    // the queries' operands; the waves' outputs at the end
    __shared__ union {
        i32x4 q[ROW_WAVES][kQm][2][64];
        float out[kKeyWaves > 1 ? WAVES : 1][kTile][kPad];
    } lds;
    __shared__ float top_of[WAVES][kTile], sum_of[WAVES][kTile];

    uint32_t id = blockIdx.x;
    const int rg = static_cast<int>(id % static_cast<uint32_t>(a.row_groups));
    id /= static_cast<uint32_t>(a.row_groups);
    const int split = static_cast<int>(id % static_cast<uint32_t>(a.splits));
    id /= static_cast<uint32_t>(a.splits);
    const int g = static_cast<int>(id % static_cast<uint32_t>(a.G));
    const int64_t b = id / static_cast<uint32_t>(a.G);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row_wave = wave % ROW_WAVES, key_wave = wave / ROW_WAVES;
    const int n16 = lane & 15, g4 = lane >> 4;

    const int len = length_of(a, b), count = count_of(a, b);
    const int group0 = rg * kTile * ROW_WAVES;
    const int group_end = min(group0 + kTile * ROW_WAVES, count * a.group);
    if (group0 >= group_end) return;
    const int64_t key_begin = split * a.chunk;
    if (split > 0 && key_begin >= seen_by(a, len, count, (group_end - 1) / a.group)) return;

    // this wave's rows: what its first row and its last row see
    const int row0 = group0 + row_wave * kTile;
    const int row_end = min(row0 + kTile, group_end);
    const bool any_row = row0 < row_end;
    const int least = any_row ? seen_by(a, len, count, row0 / a.group) : 0;
    const int most = any_row ? seen_by(a, len, count, (row_end - 1) / a.group) : 0;
    const int row = row0 + n16;
    const bool live = row < row_end;
    const int at_t = live ? row / a.group : 0, at_h = live ? row - at_t * a.group : 0;
    // rows that do not exist see everything, so that they mask nothing
    const int limit = live ? seen_by(a, len, count, at_t) : a.max_tokens;
    // and this wave's keys
    const int64_t quarter = a.chunk / kKeyWaves;
    const int64_t wave_begin = key_begin + key_wave * quarter;
    const int w0 = static_cast<int>(min(wave_begin, static_cast<int64_t>(most)));
    const int w1 = static_cast<int>(min(wave_begin + quarter, static_cast<int64_t>(most)));

    // Queries as operands: the first wave of each 16 rows lays them out.  Lane (n, g4) holds
    // elements lo .. lo + 15 and hi .. hi + 15 of row n; d = 64: the same twice, of two terms.
    int qs[(kQ + 3) / 4 + 1];                            // scales of the terms, a byte each
    {
        const int lo = 16 * g4, hi = D == 128 ? 64 + 16 * g4 : lo;
        float x[8][4];
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
        if (key_wave == 0) {
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
                    lds.q[row_wave][i][0][lane] = t[0];
                    lds.q[row_wave][i][1][lane] = t[1];
                } else {
                    lds.q[row_wave][i >> 1][i & 1][lane] = t[0];
                }
            }
        }
    }
    __syncthreads();

    // Lane l looks up the page of group l (32 keys) of a segment of 64.
    constexpr int kSegment = 64 * kGroup4;
    int page = -1;
    auto look_up = [&](int seg) {
        const int key = seg + lane * kGroup4;
        page = -1;
        if (key < w1) page = a.pages[b * a.pages_stride + (key >> a.page_shift)];
        if (page < 0 || page >= a.num_pages) page = -1;
    };
    // A step's operands, as loaded.
    u32x4 kx[8], vx[kDims], vs[4];
    uint32_t ks[2];
    const int page_mask = a.P - 1;
    // lane constants: of its keys' rows, their scales, its value rows, and the values' scales
    const int m16 = n16;
    const int k_tok = 16 * (m16 >> 2 & 1) + (m16 & 3);
    const int k_off = k_tok * (D / 2) + (D == 128 ? g4 : g4 & 1) * 16;
    const int ks_off = (m16 >> 2 & 1) * (D / 2) +
                       ((m16 & 3) * (D / 32) + (D == 128 ? g4 : g4 & 1)) * 4;
    const int v_off = m16 * 16;
    const int vs_off = 16 * (g4 & 1);
    // Of the step's four groups of 32 keys: their pages (-1: none).
    struct Where {
        int key, p0, p1, p2, p3;
    };
    auto where = [&](int key, int seg) {
        const int i = (key - seg) >> 5;
        return Where{key, __builtin_amdgcn_readlane(page, i),
                     __builtin_amdgcn_readlane(page, i + 1),
                     __builtin_amdgcn_readlane(page, i + 2),
                     __builtin_amdgcn_readlane(page, i + 3)};
    };
    // Byte offsets of a group's keys and values (by page stride), and of its tokens among all.
    // (Groups without a page read the first one's, unused.)
    const int64_t head = static_cast<int64_t>(g) * (D / 2) << a.page_shift;
    auto bytes_at = [&](int pg, int key, int64_t stride) {
        return max(pg, 0) * stride + head + (key & page_mask) * (D / 2);
    };
    auto token_at = [&](int pg, int key) {
        return ((static_cast<int64_t>(max(pg, 0)) * a.G + g) << a.page_shift) + (key & page_mask);
    };
    const bool k_odd = (m16 & 8) != 0, v_odd = (g4 & 1) != 0, v_far = (g4 & 2) != 0;
    auto fetch_half = [&](int f, int pa, int pb, int key) {
        const int64_t ka = bytes_at(pa, key, a.k_page), kb = bytes_at(pb, key + 32, a.k_page);
        const int64_t sa = token_at(pa, key) * (D / 32), sb = token_at(pb, key + 32) * (D / 32);
        const uint8_t* p = a.k + (k_odd ? kb : ka) + k_off;
#pragma unroll
        for (int u = 0; u < 4; ++u) kx[4 * f + u] = load_keys<ROW_WAVES == 1>(p + u * 2 * D);
        ks[f] = *reinterpret_cast<const uint32_t*>(a.k_scale + (k_odd ? sb : sa) + ks_off);
    };
    auto fetch_k = [&](const Where& w) {
        fetch_half(0, w.p0, w.p1, w.key);
        fetch_half(1, w.p2, w.p3, w.key + 64);
    };
    auto fetch_v = [&](const Where& w) {
        const int64_t v0 = bytes_at(w.p0, w.key, a.v_page), v1 = bytes_at(w.p1, w.key + 32, a.v_page);
        const int64_t v2 = bytes_at(w.p2, w.key + 64, a.v_page);
        const int64_t v3 = bytes_at(w.p3, w.key + 96, a.v_page);
        const int64_t va = v_odd ? v1 : v0, vb = v_odd ? v3 : v2;
        const uint8_t* p = a.v + (v_far ? vb : va) + v_off;
#pragma unroll
        for (int j = 0; j < kDims; ++j) vx[j] = load_keys<ROW_WAVES == 1>(p + j * 256);
        const int64_t s0 = token_at(w.p0, w.key), s1 = token_at(w.p1, w.key + 32);
        const int64_t s2 = token_at(w.p2, w.key + 64), s3 = token_at(w.p3, w.key + 96);
        const u32x4* sa = reinterpret_cast<const u32x4*>(a.v_scale + (v_far ? s1 : s0) + vs_off);
        const u32x4* sb = reinterpret_cast<const u32x4*>(a.v_scale + (v_far ? s3 : s2) + vs_off);
        vs[0] = sa[0];
        vs[1] = sa[1];
        vs[2] = sb[0];
        vs[3] = sb[1];
    };

    f32x4 o[kDims];
    float top = -kInf, base = 0.0f, sum = 0.0f;  // running maximum; the same, 0 before any
#pragma unroll
    for (int j = 0; j < kDims; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};

    // One step of 128 keys.  `whole`: every row sees every key of it.
    auto step = [&](auto whole_tag, int key, const Where& now, const Where& next) {
        constexpr bool kWhole = decltype(whole_tag)::value;
        // an index that the compiler cannot know keeps the queries' reads in the loop
        int my = lane;
        asm volatile("" : "+v"(my));
        f32x4 s[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = kQm - 1; i >= 0; --i) {
            const i32x4 q0 = lds.q[row_wave][i][0][my], q1 = lds.q[row_wave][i][1][my];
            const i32x8 q = {q0.x, q0.y, q0.z, q0.w, q1.x, q1.y, q1.z, q1.w};
#pragma unroll
            for (int t = 0; t < 8; ++t)
                s[t] = key_product(i, t & 3, kx[t], q, s[t], static_cast<int>(ks[t >> 2]),
                                   qs[i >> 2]);
        }
        fetch_k(next);
        // Logits to weights.  Lane (n, g4): s[4 f + u][r] is key 64 f + 16 g4 + 4 u + r.
        float y[8][4];
        float mx = -kInf;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const bool there = t < 4 ? (v_far ? now.p1 : now.p0) >= 0 : (v_far ? now.p3 : now.p2) >= 0;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                y[t][r] = s[t][r];
                if constexpr (!kWhole) {
                    const int kk = key + 64 * (t >> 2) + 16 * g4 + 4 * (t & 3) + r;
                    if (!there || kk >= limit) y[t][r] = -kInf;
                }
                mx = fmaxf(mx, y[t][r]);
            }
        }
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
        float pm = 0.0f;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const uint32_t w2[2] = {vs[t >> 1][2 * (t & 1)], vs[t >> 1][2 * (t & 1) + 1]};
            float part[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bool masked = !kWhole && y[t][r] == -kInf;
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(y[t][r], a.scale, -base));
                part[r] = p;
                const float f = r & 1 ? bf16hi(w2[r >> 1]) : bf16lo(w2[r >> 1]);
                y[t][r] = masked ? 0.0f : p * f;
                pm = fmaxf(pm, y[t][r]);
            }
            sum += (part[0] + part[1]) + (part[2] + part[3]);
        }
        pm = across_rows(pm);
        const int e = term_exponent(pm);
        int es = 0, es2 = 0;
#pragma unroll
        for (int i = 0; i < kP; ++i) (i < 4 ? es : es2) |= (e - 4 * i) << (8 * (i & 3));
#pragma unroll
        for (int i = 0; i < kP; ++i) {
            const float sc = exponent_scale(e - 4 * i);
            i32x8 w;
#pragma unroll
            for (int t = 0; t < 8; ++t)
                w[t] = i + 1 < kP ? take_term<false>(y[t], sc) : take_term<true>(y[t], sc);
#pragma unroll
            for (int j = 0; j < kDims; ++j)
                o[j] = value_product(i, vx[j], w, o[j], i < 4 ? es : es2);
        }
        fetch_v(next);
    };

    if (w0 < w1) {
        look_up(w0);
        Where now = where(w0, w0);
        fetch_k(now);
        fetch_v(now);
        int seg = w0;
        for (int key = w0; key < w1; key += kStep4) {
            int ahead = key + kStep4;
            if (ahead >= w1) ahead = key;            // nothing follows: the same again, unused
            if (ahead - seg >= kSegment) {
                seg = ahead;
                look_up(seg);
            }
            const Where next = where(ahead, seg);
            const bool paged = (now.p0 | now.p1 | now.p2 | now.p3) >= 0;
            if (paged && key + kStep4 <= least) step(std::true_type{}, key, now, next);
            else step(std::false_type{}, key, now, next);
            now = next;
        }
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
    if constexpr (kKeyWaves == 1) {
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
        float all = top_of[row_wave][n16];
#pragma unroll
        for (int w = 1; w < kKeyWaves; ++w) all = fmaxf(all, top_of[row_wave + w * ROW_WAVES][n16]);
        const float f = top == -kInf ? 0.0f : top == all ? 1.0f : __builtin_amdgcn_exp2f(top - all);
#pragma unroll
        for (int j = 0; j < kDims; ++j) {
            const f32x4 y = {o[j][0] * f, o[j][1] * f, o[j][2] * f, o[j][3] * f};
            *reinterpret_cast<f32x4*>(&lds.out[wave][n16][kTile * j + 4 * g4]) = y;
        }
        __syncthreads();
        // the key waves of 16 rows share what is left
        for (int i = key_wave * 64 + lane; i < kTile * D / 4; i += 64 * kKeyWaves) {
            const int r = i / (D / 4), d0 = i % (D / 4) * 4;
            if (row0 + r >= row_end) continue;
            float m = top_of[row_wave][r];
#pragma unroll
            for (int w = 1; w < kKeyWaves; ++w) m = fmaxf(m, top_of[row_wave + w * ROW_WAVES][r]);
            float total = 0.0f, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kKeyWaves; ++w) {
                const int from = row_wave + w * ROW_WAVES;
                // without a maximum a sum is 0, or NaN, which stays
                const float tw = top_of[from][r];
                total += sum_of[from][r] *
                         (tw == m || tw == -kInf ? 1.0f : __builtin_amdgcn_exp2f(tw - m));
                const f32x4 x = *reinterpret_cast<const f32x4*>(&lds.out[from][r][d0]);
#pragma unroll
                for (int k = 0; k < 4; ++k) y[k] += x[k];
            }
            put(r, d0, y, m, total);
        }
    }
}

// The parts of a row joined, 4 dimensions to a thread.  A part is there where its first key is
// seen by the workgroup that wrote it; parts whose keys this row does not see hold a maximum
// of -inf (and zeros, or NaN, which only rows that do not exist make).
template <typename T, int D>
__global__ __launch_bounds__(256) void attend4_join_kernel(const Attend4Args a, uint32_t lines) {
    constexpr int kLanes = D / 4;
    const uint32_t line = blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
    if (line >= lines) return;
    const int d0 = static_cast<int>(threadIdx.x % kLanes) * 4;
    const uint32_t bg = line / static_cast<uint32_t>(a.rows);
    const int row = static_cast<int>(line - bg * static_cast<uint32_t>(a.rows));
    const int64_t b = bg / static_cast<uint32_t>(a.G);
    const int g = static_cast<int>(bg - static_cast<uint32_t>(b) * a.G);
    const int t = row / a.group;
    const int len = length_of(a, b), count = count_of(a, b);
    if (t >= count) return;
    const int64_t sees = seen_by(a, len, count, t);
    const int parts = static_cast<int>((sees + a.chunk - 1) / a.chunk);
    const int64_t first = static_cast<int64_t>(line) * a.splits;
    float m = -kInf;
    for (int i = 0; i < parts; ++i) m = fmaxf(m, a.part_max[first + i]);
    float total = 0.0f, y[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < parts; i0 += 4) {
        f32x4 x[4];
        float pm[4], ps[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {            // loads of four parts under way at once
            const int64_t at = first + min(i0 + j, parts - 1);
            x[j] = *reinterpret_cast<const f32x4*>(a.part_out + at * D + d0);
            pm[j] = a.part_max[at];
            ps[j] = a.part_sum[at];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (i0 + j >= parts) break;
            const float f =
                pm[j] == m || pm[j] == -kInf ? 1.0f : __builtin_amdgcn_exp2f(pm[j] - m);
            total += ps[j] * f;
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] += x[j][k] * f;
        }
    }
    const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
    T* to = static_cast<T*>(a.out) + b * a.os[0] +
            (static_cast<int64_t>(g) * a.group + row - t * a.group) * a.os[1] + t * a.os[2] + d0;
    Run4<T, 4> z;
#pragma unroll
    for (int k = 0; k < 4; ++k) z.x[k] = from_f32<T>(y[k] * inv);
    *reinterpret_cast<Run4<T, 4>*>(to) = z;
}

template <typename T, int D>
hipError_t launch_d(const Attend4Args& a, const Attend4Plan& p, int64_t heads, hipStream_t st) {
    const dim3 grid(static_cast<unsigned>(heads * p.row_groups * p.splits));
    if (p.waves == 8)
        hipLaunchKernelGGL((attend4_kernel<T, D, 8, 1>), grid, dim3(512), 0, st, a);
    else if (p.row_waves == 1)
        hipLaunchKernelGGL((attend4_kernel<T, D, 4, 1>), grid, dim3(256), 0, st, a);
    else if (p.row_waves == 2)
        hipLaunchKernelGGL((attend4_kernel<T, D, 4, 2>), grid, dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((attend4_kernel<T, D, 4, 4>), grid, dim3(256), 0, st, a);
    if (p.splits > 1) {
        const int64_t lines = heads * p.rows;
        const int per = 256 / (D / 4);
        hipLaunchKernelGGL((attend4_join_kernel<T, D>),
                           dim3(static_cast<unsigned>((lines + per - 1) / per)), dim3(256), 0, st,
                           a, static_cast<uint32_t>(lines));
    }
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
