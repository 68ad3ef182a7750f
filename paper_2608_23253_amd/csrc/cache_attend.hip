// Attention over the 8-bit cache (e2s_cache_attend).
//
//   s = scale * q . k over the cached tokens a query sees, p = softmax(s), out = sum p v,
// and, where asked for, the weight sum over queries and grouped heads of p per token.
//
// A decoding step reads 2 d bytes per token and key head and makes 4 d products per query
// with them: memory bounds it, so the design reads every cached byte once, whole rows at a
// time, straight into registers.  The query heads of one key head are the rows of one
// matrix product (16 rows to a tile; short tiles waste matrix time, of which there is
// plenty), and products run transposed on the matrix cores:
//   S^T [16 keys x 16 rows] = K Q^T        O^T [d x 16 rows] += V^T P^T
// In this form a lane holds the logits of ONE row (n = lane & 15) for keys 4 g + r
// (g = lane >> 4), which is exactly the operand layout that P^T needs - the order in which
// a product sums its keys is free - so the weights go from one product to the next without
// leaving their lane.  The values' operand needs 8 keys of one dimension per lane: a lane
// reads its 8 keys' bytes of d / 16 neighbouring dimensions and byte-permutes pairs of
// keys together.  e4m3 bytes become bf16 exactly, with the block's power-of-two scale
// applied by the conversion.
//
// One pass: a running maximum and sum per row.  The maximum is raised (and the output
// rescaled) only when a logit passes it by 2^8 in the exponential: weights then stay below
// 256, within float32's and bf16's range, and the cross-lane reduction is rare.
//
// Four waves take neighbouring runs of a workgroup's keys and merge through LDS; the keys
// of a sequence are split over workgroups when there are too few (sequence, head) pairs to
// fill the device, and attend_join_kernel joins the parts.
#include "serve_device.h"
#include "serve_kernels.h"

namespace e2s {
namespace {

constexpr int kThreads = 64 * kAttendWaves;
constexpr int kTile = 16;                      // keys and rows of a product tile
constexpr float kInf = __builtin_huge_valf();
constexpr float kRaise = 8.0f;                 // log2 by which a logit may pass the maximum


typedef __bf16 bf16x8s __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4s __attribute__((ext_vector_type(4)));

struct AttendArgs {
    const uint8_t* k;
    const uint8_t* v;
    const float* k_scale;
    const float* v_scale;
    int64_t k_page, v_page, pages_stride;
    const int32_t* pages;
    const int32_t* lengths;
    const int32_t* q_count;          // or null
    const void* q;
    void* out;
    const float* w_in;               // or null
    float* w_out;                    // or null
    float* part_max;                 // [B, Hkv, rows, splits], or null with one split
    float* part_sum;
    float* part_out;                 // [B, Hkv, rows, splits, d]
    float* lse;                      // [B, Hkv, rows]: log2 of a row's sum, or null
    float* logits;                   // [B, Hkv, rows, logit_stride] in log2, or null
    int64_t logit_stride, chunk;
    int64_t qs[3], os[3], wi[2], wo[2];
    int G, group, T, rows, row_groups, splits;
    int P, num_pages, max_pages, max_tokens, causal;
    float scale;                     // logit scale times log2(e)
};

__device__ __forceinline__ int attend_length(const AttendArgs& a, int64_t b) {
    const int64_t cap = min(static_cast<int64_t>(a.max_pages) * a.P,
                            static_cast<int64_t>(a.max_tokens));
    return static_cast<int>(min(static_cast<int64_t>(max(a.lengths[b], 0)), cap));
}
__device__ __forceinline__ int attend_count(const AttendArgs& a, int64_t b) {
    return a.q_count ? min(max(a.q_count[b], 0), a.T) : a.T;
}
// Tokens that query t of `count` sees.
__device__ __forceinline__ int seen_by(const AttendArgs& a, int len, int count, int t) {
    return a.causal ? max(0, len - (count - 1 - t)) : len;
}

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// Terms of a float as a sum of bf16 values: 8, 16 or 24 bits.
template <int TERMS>
__device__ __forceinline__ void split_bf16(float x, __bf16* out) {
#pragma unroll
    for (int i = 0; i < TERMS; ++i) {
        out[i] = static_cast<__bf16>(x);
        x -= static_cast<float>(out[i]);
    }
}

template <typename T, int N>             // neighbouring elements, stored at once
struct alignas(N * sizeof(T) < 16 ? N * sizeof(T) : 16) Run { T x[N]; };

template <typename T> struct Terms;      // bf16 terms that hold a query's element exactly
template <> struct Terms<uint16_t> { static constexpr int n = 1; };
template <> struct Terms<_Float16> { static constexpr int n = 2; };
template <> struct Terms<float> { static constexpr int n = 3; };

__device__ __forceinline__ uint32_t pack_bf16(uint32_t w, float scale, bool high) {
    const bf16x2s r = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true)
                           : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    return __builtin_bit_cast(uint32_t, r);
}
// 8 consecutive bytes (two words) to an operand of 8 bf16.
__device__ __forceinline__ bf16x8s widen8(uint32_t a, uint32_t b, float scale) {
    u32x4s r = {pack_bf16(a, scale, false), pack_bf16(a, scale, true), pack_bf16(b, scale, false),
                pack_bf16(b, scale, true)};
    return __builtin_bit_cast(bf16x8s, r);
}
// Words whose bytes are 0x80 where w has a NaN (0x7F or 0xFF).
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
    return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
}

// The bytes of 32 keys that a wave holds: its part of two 16-key tiles.
template <int D>
struct Step {
    u32x4 k[2][D / 64];                  // tile, half of the row
    uint32_t v[8][D / 64];               // key (4 of each tile), words of its D / 16 bytes
};

template <typename T, int D, int TILES>
__global__ __launch_bounds__(kThreads) void attend_kernel(const AttendArgs a) {
    constexpr int kTerms = Terms<T>::n;
    constexpr int kHalves = D / 64;
    constexpr int kDims = D / 16;                // dimensions of a lane's values
    constexpr int kPad = D + 4;
    __shared__ float merge[kAttendWaves][kTile][kPad];
    __shared__ float top_of[kAttendWaves][TILES * kTile], sum_of[kAttendWaves][TILES * kTile];

    int64_t id = blockIdx.x;
    const int rg = static_cast<int>(id % a.row_groups);
    id /= a.row_groups;
    const int split = static_cast<int>(id % a.splits);
    id /= a.splits;
    const int g = static_cast<int>(id % a.G);
    const int64_t b = id / a.G;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n16 = lane & 15, g4 = lane >> 4;

    const int len = attend_length(a, b), count = attend_count(a, b);
    const int row0 = rg * TILES * kTile;
    const int row_end = min(row0 + TILES * kTile, count * a.group);
    if (row0 >= row_end) return;
    // what the workgroup's first row and last row see: every row sees between them
    const int least = seen_by(a, len, count, row0 / a.group);
    const int most = seen_by(a, len, count, (row_end - 1) / a.group);
    const int64_t key_begin = split * a.chunk;
    if (split > 0 && key_begin >= most) return;

    // queries as operand columns: lane (n, g4) holds row n's elements 64 h + 16 g4 + 8 s + i
    bf16x8s q[TILES][kTerms][2 * kHalves];
    int limit[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const int row = row0 + t * kTile + n16;
        const bool live = row < row_end;
        const int at = live ? row / a.group : 0;
        // rows that do not exist see everything, so that they mask nothing
        limit[t] = live ? seen_by(a, len, count, at) : a.max_tokens;
        const T* src = static_cast<const T*>(a.q) + b * a.qs[0] +
                       (g * a.group + (live ? row - at * a.group : 0)) * a.qs[1] + at * a.qs[2];
#pragma unroll
        for (int s = 0; s < 2 * kHalves; ++s) {
            Packet<T> p{};
            if (live) load_packet(p, src + (s >> 1) * 64 + g4 * 16 + (s & 1) * 8);
            float x[8];
            unpack(p, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                __bf16 w[kTerms];
                split_bf16<kTerms>(x[i], w);
#pragma unroll
                for (int m = 0; m < kTerms; ++m) q[t][m][s][i] = w[m];
            }
        }
    }

    f32x4 o[TILES][kDims];
    float top[TILES], base[TILES], sum[TILES];   // running maximum; the same, 0 before any
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
#pragma unroll
        for (int j = 0; j < kDims; ++j) o[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        top[t] = -kInf;
        base[t] = 0.0f;
        sum[t] = 0.0f;
    }

    // this wave's keys
    const int64_t quarter = a.chunk / kAttendWaves;
    const int w0 = static_cast<int>(min(key_begin + wave * quarter, static_cast<int64_t>(most)));
    const int w1 = static_cast<int>(min(key_begin + (wave + 1) * quarter,
                                        static_cast<int64_t>(most)));
    const uint32_t k_lane = static_cast<uint32_t>(n16 * D + g4 * 16);
    const uint32_t v_lane = static_cast<uint32_t>(4 * g4 * D + n16 * kDims);
    const int64_t head = static_cast<int64_t>(g) * a.P * D;

    for (int seg = w0; seg < w1; seg += 64 * kTile) {
        // lane l looks up tile l of the next 64: its page, or -1, and the block's scales
        const int mine = seg + lane * kTile;
        int page = -1;
        if (mine < w1) page = a.pages[b * a.pages_stride + mine / a.P];
        if (page < 0 || page >= a.num_pages) page = -1;
        const int64_t at = static_cast<int64_t>(max(page, 0)) * a.G + g;
        // (without a page: any finite scale, the scale at hand may not have been written)
        const float ks = page < 0 ? 1.0f : a.k_scale[at], vs = page < 0 ? 1.0f : a.v_scale[at];
        const int seg_end = min(w1, seg + 64 * kTile);

        auto fetch = [&](int key, Step<D>& x) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int i = (key - seg) / kTile + t;
                const int pg = max(__builtin_amdgcn_readlane(page, i), 0);
                const int64_t row = head + static_cast<int64_t>((key + t * kTile) % a.P) * D;
                const uint8_t* kp = a.k + pg * a.k_page + row;
                const uint8_t* vp = a.v + pg * a.v_page + row;
#pragma unroll
                for (int h = 0; h < kHalves; ++h)
                    x.k[t][h] = __builtin_nontemporal_load(
                        reinterpret_cast<const u32x4*>(kp + k_lane + h * 64));
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint8_t* p = vp + v_lane + r * D;
                    if constexpr (kHalves == 2) {
                        const u32x2 w = __builtin_nontemporal_load(
                            reinterpret_cast<const u32x2*>(p));
                        x.v[4 * t + r][0] = w.x;
                        x.v[4 * t + r][kHalves - 1] = w.y;
                    } else {
                        x.v[4 * t + r][0] = __builtin_nontemporal_load(
                            reinterpret_cast<const uint32_t*>(p));
                    }
                }
            }
        };

        Step<D> cur, next;
        fetch(seg, cur);
        for (int key = seg; key < seg_end; key += kAttendStep) {
            if (key + kAttendStep < seg_end) fetch(key + kAttendStep, next);
            const int i0 = (key - seg) / kTile;
            const int pg0 = __builtin_amdgcn_readlane(page, i0);
            const int pg1 = __builtin_amdgcn_readlane(page, i0 + 1);
            const float ks0 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(ks), i0));
            const float ks1 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(ks), i0 + 1));
            const float vs0 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(vs), i0));
            const float vs1 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(vs), i0 + 1));

            // S^T of both tiles
            f32x4 s[TILES][2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const float sc = t ? ks1 : ks0;
                bf16x8s kf[2 * kHalves];
#pragma unroll
                for (int h = 0; h < kHalves; ++h) {
                    kf[2 * h] = widen8(cur.k[t][h].x, cur.k[t][h].y, sc);
                    kf[2 * h + 1] = widen8(cur.k[t][h].z, cur.k[t][h].w, sc);
                }
#pragma unroll
                for (int u = 0; u < TILES; ++u) {
                    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int m = kTerms - 1; m >= 0; --m)
#pragma unroll
                        for (int e = 0; e < 2 * kHalves; ++e)
                            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[e], q[u][m][e], acc,
                                                                          0, 0, 0);
                    s[u][t] = acc;
                }
            }
            // keys that some row does not see: beyond `least`, or without a page
            const bool whole = key + kAttendStep <= least && pg0 >= 0 && pg1 >= 0;
            bool lost = false;                   // a NaN among the values of a masked step
            if (!whole) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int kk = key + (i >> 2) * kTile + 4 * g4 + (i & 3);
                    const bool there = kk < most && ((i >> 2) ? pg1 : pg0) >= 0;
#pragma unroll
                    for (int h = 0; h < kHalves; ++h) {
                        // what no row sees may hold anything: 0 * NaN must not reach the sum
                        if (!there) cur.v[i][h] = 0u;
                        lost = lost || nan_bytes(cur.v[i][h]) != 0u;
                    }
                }
                lost = __ballot(lost) != 0;
            }
#pragma unroll
            for (int u = 0; u < TILES; ++u) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = s[u][i >> 2][i & 3] * a.scale;
                if (!whole) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int kk = key + (i >> 2) * kTile + 4 * g4 + (i & 3);
                        if (kk >= limit[u] || ((i >> 2) ? pg1 : pg0) < 0)
                            x[i] = -kInf;
                    }
                }
                if (a.logits) {
                    const int row = row0 + u * kTile + n16;
                    if (row < row_end) {
                        float* to = a.logits +
                                    ((b * a.G + g) * static_cast<int64_t>(a.rows) + row) *
                                        a.logit_stride + key + 4 * g4;
                        *reinterpret_cast<f32x4*>(to) = f32x4{x[0], x[1], x[2], x[3]};
                        *reinterpret_cast<f32x4*>(to + kTile) = f32x4{x[4], x[5], x[6], x[7]};
                    }
                }
                float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                                 fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
                if (__ballot(mx > top[u] + kRaise)) {
                    mx = fmaxf(mx, __shfl_xor(mx, 16));
                    mx = fmaxf(mx, __shfl_xor(mx, 32));
                    const float up = fmaxf(top[u], mx);
                    const float shrink = up == top[u] ? 1.0f : exp2_hw(top[u] - up);
                    top[u] = up;
                    base[u] = up == -kInf ? 0.0f : up;
                    sum[u] *= shrink;
#pragma unroll
                    for (int j = 0; j < kDims; ++j) o[u][j] *= shrink;
                }
                float p[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] = exp2_hw(x[i] - base[u]);
                sum[u] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
#pragma unroll
                for (int i = 0; i < 8; ++i) s[u][i >> 2][i & 3] = p[i];
            }
            // weights as operand columns, in kTerms parts
            bf16x8s pf[TILES][kTerms];
#pragma unroll
            for (int u = 0; u < TILES; ++u)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    __bf16 w[kTerms];
                    split_bf16<kTerms>(s[u][i >> 2][i & 3], w);
#pragma unroll
                    for (int m = 0; m < kTerms; ++m) pf[u][m][i] = w[m];
                }
            // O^T: 4 dimensions of each word, keys paired by byte permutation
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                u32x4s vf[4];
#pragma unroll
                for (int pr = 0; pr < 4; ++pr) {
                    uint32_t wa = cur.v[2 * pr][h], wb = cur.v[2 * pr + 1][h];
                    if (lost) {                  // NaN bytes to 0 here, counted below
                        wa &= ~((nan_bytes(wa) >> 7) * 0xFFu);
                        wb &= ~((nan_bytes(wb) >> 7) * 0xFFu);
                    }
                    const uint32_t lo = __builtin_amdgcn_perm(wb, wa, 0x05010400u);
                    const uint32_t hi = __builtin_amdgcn_perm(wb, wa, 0x07030602u);
                    const float sc = pr < 2 ? vs0 : vs1;
                    vf[0][pr] = pack_bf16(lo, sc, false);
                    vf[1][pr] = pack_bf16(lo, sc, true);
                    vf[2][pr] = pack_bf16(hi, sc, false);
                    vf[3][pr] = pack_bf16(hi, sc, true);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int u = 0; u < TILES; ++u)
#pragma unroll
                        for (int m = kTerms - 1; m >= 0; --m)
                            o[u][4 * h + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                __builtin_bit_cast(bf16x8s, vf[j]), pf[u][m], o[u][4 * h + j], 0,
                                0, 0);
            }
            if (lost) {
                // A NaN value reaches the rows that see its key, and no other: count, per
                // dimension and row, the seen keys that hold one.
                bf16x8s seen[TILES];
#pragma unroll
                for (int u = 0; u < TILES; ++u)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int kk = key + (i >> 2) * kTile + 4 * g4 + (i & 3);
                        seen[u][i] = static_cast<__bf16>(kk < limit[u] ? 1.0f : 0.0f);
                    }
#pragma unroll
                for (int j = 0; j < kDims; ++j) {
                    bf16x8s bad;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        bad[i] = static_cast<__bf16>(
                            (nan_bytes(cur.v[i][j / 4]) >> (8 * (j % 4) + 7)) & 1u ? 1.0f : 0.0f);
#pragma unroll
                    for (int u = 0; u < TILES; ++u) {
                        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
                        const f32x4 hits =
                            __builtin_amdgcn_mfma_f32_16x16x32_bf16(bad, seen[u], zero, 0, 0, 0);
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (hits[r] > 0.0f) o[u][j][r] = __builtin_nanf("");
                    }
                }
            }
            cur = next;
        }
    }

    // merge the four waves, a 16-row tile at a time
#pragma unroll
    for (int u = 0; u < TILES; ++u) {
        sum[u] += __shfl_xor(sum[u], 16);
        sum[u] += __shfl_xor(sum[u], 32);
        if (g4 == 0) {
            top_of[wave][u * kTile + n16] = top[u];
            sum_of[wave][u * kTile + n16] = sum[u];
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < TILES; ++u) {
        float all = top_of[0][u * kTile + n16];
#pragma unroll
        for (int w = 1; w < kAttendWaves; ++w) all = fmaxf(all, top_of[w][u * kTile + n16]);
        const float f = top[u] == -kInf ? 0.0f
                        : top[u] == all                  ? 1.0f
                                                         : exp2_hw(top[u] - all);
        // lane (n, g4) holds dimensions (4 g4 + r) * kDims + j of row n
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < kDims; ++j)
                merge[wave][n16][(4 * g4 + r) * kDims + j] = o[u][j][r] * f;
        __syncthreads();
        constexpr int kPer = kTile * D / kThreads;       // dimensions per thread: 4 or 8
        const int r = threadIdx.x / (D / kPer), d0 = threadIdx.x % (D / kPer) * kPer;
        const int row = row0 + u * kTile + r;
        if (row < row_end) {
            float m = top_of[0][u * kTile + r];
#pragma unroll
            for (int w = 1; w < kAttendWaves; ++w) m = fmaxf(m, top_of[w][u * kTile + r]);
            float total = 0.0f;
#pragma unroll
            for (int w = 0; w < kAttendWaves; ++w) {
                // without a maximum a sum is 0, or NaN, which stays
                const float tw = top_of[w][u * kTile + r];
                total += sum_of[w][u * kTile + r] *
                         (tw == m || tw == -kInf ? 1.0f : exp2_hw(tw - m));
            }
            float y[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                y[i] = merge[0][r][d0 + i];
#pragma unroll
                for (int w = 1; w < kAttendWaves; ++w) y[i] += merge[w][r][d0 + i];
            }
            const int64_t line = (b * a.G + g) * static_cast<int64_t>(a.rows) + row;
            if (a.splits == 1) {
                const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
                const int t = row / a.group;
                T* to = static_cast<T*>(a.out) + b * a.os[0] +
                        (g * a.group + row - t * a.group) * a.os[1] + t * a.os[2] + d0;
                Run<T, kPer> z;
#pragma unroll
                for (int i = 0; i < kPer; ++i) z.x[i] = from_f32<T>(y[i] * inv);
                *reinterpret_cast<Run<T, kPer>*>(to) = z;
                if (a.lse && d0 == 0)
                    a.lse[line] = total > 0.0f || total != total ? m + __log2f(total)
                                                                 : -kInf;
            } else {
                const int64_t part = line * a.splits + split;
                Run<float, kPer> z;
#pragma unroll
                for (int i = 0; i < kPer; ++i) z.x[i] = y[i];
                *reinterpret_cast<Run<float, kPer>*>(a.part_out + part * D + d0) = z;
                if (d0 == 0) {
                    a.part_max[part] = m;
                    a.part_sum[part] = total;
                }
            }
        }
        __syncthreads();
    }
}

// Joins the parts of a row: one workgroup per (sequence, key head, row).  A part is there
// where its first key is seen by the workgroup that wrote it; parts whose keys this row
// does not see hold a maximum of -inf.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void attend_join_kernel(const AttendArgs a) {
    __shared__ float merge[kAttendWaves][D];
    __shared__ float sums[kAttendWaves];
    const int64_t line = blockIdx.x;
    const int64_t bg = line / a.rows;
    const int row = static_cast<int>(line - bg * a.rows);
    const int64_t b = bg / a.G;
    const int g = static_cast<int>(bg - b * a.G);
    const int len = attend_length(a, b), count = attend_count(a, b);
    const int t = row / a.group;
    if (t >= count) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int limit = seen_by(a, len, count, t);
    const int parts = static_cast<int>((limit + a.chunk - 1) / a.chunk);   // <= splits
    constexpr int kPer = D / 64;
    float m = -kInf;
    for (int i = lane; i < parts; i += 64) m = fmaxf(m, a.part_max[line * a.splits + i]);
    m = wave_max(m);
    float total = 0.0f, y[kPer] = {};
#pragma unroll 4
    for (int i = wave; i < parts; i += kAttendWaves) {
        const int64_t part = line * a.splits + i;
        const float pm = a.part_max[part];      // -inf: the part holds zeros, or NaN
        const float f = pm == -kInf ? 1.0f : exp2_hw(pm - m);
        total += a.part_sum[part] * f;
#pragma unroll
        for (int k = 0; k < kPer; ++k) y[k] += a.part_out[part * D + lane * kPer + k] * f;
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) merge[wave][lane * kPer + k] = y[k];
    if (lane == 0) sums[wave] = total;
    __syncthreads();
    total = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
    if (threadIdx.x < D) {
        const int d = threadIdx.x;
        const float z = (merge[0][d] + merge[1][d]) + (merge[2][d] + merge[3][d]);
        T* to = static_cast<T*>(a.out) + b * a.os[0] +
                (g * a.group + row - t * a.group) * a.os[1] + t * a.os[2];
        to[d] = from_f32<T>(z * inv);
    }
    if (a.lse && threadIdx.x == 0)
        a.lse[line] = total > 0.0f || total != total ? m + __log2f(total)
                                                     : -kInf;
}

// The weight that every token received: sum over the rows of exp2(logit - lse), from the
// stored logits, rows in order.  One thread takes four neighbouring tokens.
__global__ __launch_bounds__(kThreads) void attend_weights_kernel(const AttendArgs a, int blocks) {
    const int64_t bg = blockIdx.x / blocks;
    const int64_t b = bg / a.G;
    const int g = static_cast<int>(bg - b * a.G);
    const int n0 = (static_cast<int>(blockIdx.x - bg * blocks) * kThreads +
                    static_cast<int>(threadIdx.x)) * 4;
    const int len = attend_length(a, b), count = attend_count(a, b);
    if (n0 >= len) return;
    float w[4] = {0.f, 0.f, 0.f, 0.f};
    const int rows = count * a.group;
    for (int row = 0; row < rows; ++row) {
        const int limit = seen_by(a, len, count, row / a.group);
        if (n0 >= limit) continue;
        const int64_t line = bg * a.rows + row;
        const float l = a.lse[line];
        if (l == -kInf) continue;
        const f32x4 x = *reinterpret_cast<const f32x4*>(a.logits + line * a.logit_stride + n0);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] += n0 + i < limit ? exp2_hw(x[i] - l) : 0.0f;
    }
    const float* in = a.w_in ? a.w_in + b * a.wi[0] + g * a.wi[1] : nullptr;
    float* out = a.w_out + b * a.wo[0] + g * a.wo[1];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n0 + i < len) out[n0 + i] = in ? in[n0 + i] + w[i] : w[i];
}

template <typename T, int D>
hipError_t launch_t(const AttendArgs& a, const AttendPlan& p, int64_t B, hipStream_t st) {
    const dim3 grid(static_cast<unsigned>(B * a.G * a.splits * a.row_groups));
    if (p.tiles == 1)
        hipLaunchKernelGGL((attend_kernel<T, D, 1>), grid, dim3(kThreads), 0, st, a);
    else
        hipLaunchKernelGGL((attend_kernel<T, D, 2>), grid, dim3(kThreads), 0, st, a);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    if (a.splits > 1) {
        hipLaunchKernelGGL((attend_join_kernel<T, D>), dim3(static_cast<unsigned>(B * a.G * a.rows)),
                           dim3(kThreads), 0, st, a);
        err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    if (a.w_out) {
        const int blocks = (a.max_tokens + 4 * kThreads - 1) / (4 * kThreads);
        hipLaunchKernelGGL(attend_weights_kernel, dim3(static_cast<unsigned>(B * a.G * blocks)),
                           dim3(kThreads), 0, st, a, blocks);
        err = hipGetLastError();
    }
    return err;
}

template <typename T>
hipError_t launch_d(const AttendArgs& a, const AttendPlan& p, int64_t B, int D, hipStream_t st) {
    return D == 64 ? launch_t<T, 64>(a, p, B, st) : launch_t<T, 128>(a, p, B, st);
}

}  // namespace

hipError_t launch_cache_attend(const e2s_cache& c, const e2s_cache_attend_shape& s,
                               const int32_t* pages, const int32_t* lengths,
                               const int32_t* q_count, const void* q, void* out,
                               const float* weights_in, float* weights_out, void* workspace,
                               hipStream_t st) {
    const AttendPlan p = attend_plan(c, s);
    char* ws = static_cast<char*>(workspace);
    AttendArgs a{};
    a.k = static_cast<const uint8_t*>(c.k);
    a.v = static_cast<const uint8_t*>(c.v);
    a.k_scale = c.k_scale;
    a.v_scale = c.v_scale;
    a.k_page = c.k_page_stride;
    a.v_page = c.v_page_stride;
    a.pages_stride = s.pages_stride;
    a.pages = pages;
    a.lengths = lengths;
    a.q_count = q_count;
    a.q = q;
    a.out = out;
    a.w_in = weights_in;
    a.w_out = weights_out;
    if (p.splits > 1) {
        a.part_max = reinterpret_cast<float*>(ws + p.max_off);
        a.part_sum = reinterpret_cast<float*>(ws + p.sum_off);
        a.part_out = reinterpret_cast<float*>(ws + p.part_off);
    }
    if (weights_out) {
        a.lse = reinterpret_cast<float*>(ws + p.lse_off);
        a.logits = reinterpret_cast<float*>(ws + p.logit_off);
    }
    a.logit_stride = p.logit_stride;
    a.chunk = p.chunk;
    for (int i = 0; i < 3; ++i) {
        a.qs[i] = s.q_stride[i];
        a.os[i] = s.out_stride[i];
    }
    for (int i = 0; i < 2; ++i) {
        a.wi[i] = s.weights_in_stride[i];
        a.wo[i] = s.weights_out_stride[i];
    }
    a.G = c.num_kv_heads;
    a.group = s.num_heads / c.num_kv_heads;
    a.T = s.num_queries;
    a.rows = static_cast<int>(p.rows);
    a.row_groups = static_cast<int>(p.row_groups);
    a.splits = static_cast<int>(p.splits);
    a.P = c.page_tokens;
    a.num_pages = c.num_pages;
    a.max_pages = s.max_pages;
    a.max_tokens = s.max_tokens;
    a.causal = s.causal;
    const double scale = s.scale != 0.0f ? s.scale : 1.0 / std::sqrt(static_cast<double>(c.head_dim));
    a.scale = static_cast<float>(scale * 1.4426950408889634);
    if (s.dtype == E2S_DTYPE_F32) return launch_d<float>(a, p, s.batch, c.head_dim, st);
    if (s.dtype == E2S_DTYPE_F16) return launch_d<_Float16>(a, p, s.batch, c.head_dim, st);
    return launch_d<uint16_t>(a, p, s.batch, c.head_dim, st);
}

}  // namespace e2s
