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
// Weights are rounded to two bf16 terms (16 bits; three, 24 bits, for float32 queries): one
// term's 2^-9 would be as large as the output's own rounding where many weights are alike.
// Queries are split into as many terms as hold them exactly.
//
// Few rows (attend_kernel): the waves take neighbouring runs of a workgroup's keys and merge
// through LDS; the keys of a sequence are split over workgroups when there are too few
// (sequence, head) pairs to fill the device.  4 sequences of 60000 to 131072 keys, 28 heads to
// 4 (322 MB): 57 us, 5.7 TB/s of the 6.8 that a plain read of as much reaches; 64 sequences of
// 130 to 1200 keys, 32 heads, f16, the logits kept (378 MB): 74 us.  Without their loads
// the same steps take 35 and 47 us: instruction issue (some 280 vector and 125 scalar
// instructions to 32 keys) and memory share the time.
//
// Many rows (attend_rows_kernel): the waves take 16 or 32 rows each, widen the keys' and
// values' operands once for all into LDS, and wait for each other twice a step.  2 sequences
// of 2048 queries and keys, 28 heads, bf16: 145 us, 415 TFLOP/s of the 60 GFLOP that the mask
// leaves, 620 counting the second term's products (f16, two query terms and 16 rows a wave: 188
// us); 16 ragged ones of up to 48 queries and 4200 keys: 47 us before the join, where few
// workgroups remain to hide a step's latencies (registers leave three waves a SIMD; all
// operands read ahead from LDS, two waves a SIMD: 60).
//
// attend_finish_kernel joins the parts (21504 rows of up to 5: 6 us) and adds up few rows'
// weights, attend_weights_kernel does where that is a launch of its own, and
// attend_rows_weights_kernel adds up many rows'.
#include <type_traits>

#include "serve_device.h"
#include "serve_kernels.h"

namespace e2s {
namespace {

constexpr int kThreads = 64 * kAttendWaves;
constexpr int kTile = 16;                      // keys and rows of a product tile
constexpr float kInf = __builtin_huge_valf();
constexpr float kRaise = 8.0f;                 // log2 by which a logit may pass the maximum

// Keys are widened at half their size and values at 2^-16 of it, exactly: the largest held
// value, 2^128, is finite so, and so is a sum of values below 2^116 under 2^20 weights of up to
// 2^kRaise.  The logits' scale and the division by the weights' sum give it back.
constexpr int kKeyDown = 1, kValueDown = 16;
constexpr float kKeySize = 1.0f / (1 << kKeyDown), kValueUp = 1 << kValueDown;

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
    int P, page_shift, num_pages, max_pages, max_tokens, causal;
    float scale;                     // logit scale times log2(e), of halved keys
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

// Bits 0, 8, 16 and 24 side by side.
__device__ __forceinline__ uint32_t gather_bits(uint32_t n) {
    return (n & 1u) | (n >> 7 & 2u) | (n >> 14 & 4u) | (n >> 21 & 8u);
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
// What the wave's lanes wrote to LDS before is what they read after, and the other way round:
// the hardware keeps a wave's accesses in order, this keeps the compiler's.
__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
template <typename V>
__device__ __forceinline__ V load_stream(const uint8_t* p) {
    return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
}
// A lane's scale at 2^-DOWN of its size: a power of two's exponent, on scalars (in the vector
// unit, behind the lookup, it showed: 9.50 us for 9.43 with one sequence).
template <int DOWN>
__device__ __forceinline__ float lane_scale(float x, int lane) {
    const int bits = __builtin_amdgcn_readlane(__float_as_int(x), lane);
    return __int_as_float(max(bits - (DOWN << 23), 0));
}
// Words whose bytes are 0x80 where w has a NaN (0x7F or 0xFF).
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
    return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
}

// Logits (before their positive scale, -inf where masked) to weights against a row's running
// maximum, which is raised - with the sum and the output so far - where a logit passes it by
// more than kRaise.  The four lanes of a row hold N of its logits each, and part of its sum.
template <int N, int DIMS>
__device__ __forceinline__ void weigh(float (&y)[N], float scale, float& top, float& base,
                                      float& sum, f32x4 (&o)[DIMS]) {
    float mx = fmaxf(y[0], y[1]);
#pragma unroll
    for (int i = 2; i < N; i += 2) mx = fmaxf(mx, fmaxf(y[i], y[i + 1]));
    mx *= scale;
    if (__ballot(mx > top + kRaise)) {
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float up = fmaxf(top, mx);
        const float shrink = up == top ? 1.0f : exp2_hw(top - up);
        top = up;
        base = up == -kInf ? 0.0f : up;
        sum *= shrink;
#pragma unroll
        for (int j = 0; j < DIMS; ++j) o[j] *= shrink;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = exp2_hw(__builtin_fmaf(y[i], scale, -base));
#pragma unroll
    for (int i = 0; i < N; i += 8)
        sum += ((y[i] + y[i + 1]) + (y[i + 2] + y[i + 3])) +
               ((y[i + 4] + y[i + 5]) + (y[i + 6] + y[i + 7]));
}

// The weight that tokens n0 .. n0 + 3, n0 + step .. received: the sum over the rows, in
// order, of exp2(logit - lse), from the stored logits.  lse: per row, -inf where it sees none.
__device__ __forceinline__ void token_weights(const AttendArgs& a, int64_t b, int g,
                                              const float* lse, int len, int count, int n0,
                                              int step) {
    constexpr int kBatch = 4;                    // rows whose loads are under way at once
    const int64_t bg = b * a.G + g;
    const int rows = count * a.group;
    const float* in = a.w_in ? a.w_in + b * a.wi[0] + g * a.wi[1] : nullptr;
    float* out = a.w_out + b * a.wo[0] + g * a.wo[1];
    for (; n0 < len; n0 += step) {
        float w[4] = {0.f, 0.f, 0.f, 0.f};
        int t = 0, h = 0;                        // of the row whose weight is added next
        for (int row0 = 0; row0 < rows; row0 += kBatch) {
            // what a row does not see was not written, and is read but not used
            f32x4 x[kBatch];
            float l[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const int row = min(row0 + j, rows - 1);
                l[j] = lse[row];
                x[j] = *reinterpret_cast<const f32x4*>(
                    a.logits + (bg * a.rows + row) * a.logit_stride + n0);
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                if (row0 + j >= rows) break;
                const int limit = l[j] == -kInf ? 0 : seen_by(a, len, count, t);
                if (++h == a.group) {
                    h = 0;
                    ++t;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    // (-inf: no page, so no weight, also of a row whose sum is NaN)
                    w[i] += n0 + i < limit && x[j][i] != -kInf ? exp2_hw(x[j][i] - l[j]) : 0.0f;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n0 + i < len) out[n0 + i] = in ? in[n0 + i] + w[i] : w[i];
    }
}

// The permutation of a row's 16-byte chunks in LDS.
template <int D>
__device__ __forceinline__ int swizzle(int row) {
    return D == 128 ? row & 7 : (row >> 1) & 3;
}

// A wave's part of 32 keys, as loaded.
template <int D>
struct Step {
    u32x4 k[D / 32];                     // 1 KB each of the keys' rows in order
    uint32_t v[8][D / 64];               // key (4 of each tile), words of its D / 16 bytes
};

template <typename T, int D, int TILES, int WAVES>
__global__ __launch_bounds__(64 * WAVES, TILES == 1 ? 4 : 2) void attend_kernel(
    const AttendArgs a) {
    constexpr int kTerms = Terms<T>::n;
    constexpr int kParts = kTerms < 2 ? 2 : kTerms;      // bf16 terms of a softmax weight
    constexpr int kHalves = D / 64;
    constexpr int kDims = D / 16;                // dimensions of a lane's values
    constexpr int kPad = D + 4;
    constexpr int kFrags = TILES * kTerms * 2 * kHalves;     // operands of the queries
    // the queries' operands, in the order lanes read them; the waves' outputs at the end
    __shared__ union {
        struct {
            bf16x8s q[kFrags][64];
            u32x4 k[WAVES][kAttendStep * D / 16];
        } in;
        float out[WAVES][kTile][kPad];
    } lds;
    __shared__ float top_of[WAVES][TILES * kTile], sum_of[WAVES][TILES * kTile];

    __shared__ float lse_of[TILES * kTile];

    uint32_t id = blockIdx.x;
    const int split = static_cast<int>(id % static_cast<uint32_t>(a.splits));
    id /= static_cast<uint32_t>(a.splits);
    const int g = static_cast<int>(id % static_cast<uint32_t>(a.G));
    const int64_t b = id / static_cast<uint32_t>(a.G);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, g4 = lane >> 4;

    // Lane l looks up tile l of 64: its page, or -1, and the block's scales (without a page
    // any finite scale: the one at hand may not have been written).  The first lookup does
    // not wait for the length.
    const int64_t key_begin = split * a.chunk, quarter = a.chunk / WAVES;
    const int64_t cap = static_cast<int64_t>(a.max_pages) << a.page_shift;
    const int64_t wave_begin = key_begin + wave * quarter;
    auto page_at = [&](int64_t key, int64_t end) {
        return key < end ? a.pages[b * a.pages_stride + (key >> a.page_shift)] : -1;
    };
    int page = page_at(wave_begin + lane * kTile, min(wave_begin + quarter, cap));

    const int len = attend_length(a, b), count = attend_count(a, b);
    constexpr int row0 = 0;
    const int row_end = count * a.group;
    if (row_end == 0) {                          // no query: no weight is added
        if (WAVES == 8 && a.w_out)
            token_weights(a, b, g, lse_of, len, 0, static_cast<int>(threadIdx.x) * 4, 256 * WAVES);
        return;
    }
    // what the first row and the last row see: every row sees between them
    const int least = seen_by(a, len, count, 0);
    const int most = seen_by(a, len, count, count - 1);
    if (split > 0 && key_begin >= most) return;

    // this wave's keys
    const int w0 = static_cast<int>(min(wave_begin, static_cast<int64_t>(most)));
    const int w1 = static_cast<int>(min(wave_begin + quarter, static_cast<int64_t>(most)));
    const int64_t head = static_cast<int64_t>(g) * (D << a.page_shift);
    const int page_mask = (1 << a.page_shift) - 1;
    float ks = 1.0f, vs = 1.0f;
    auto look_up = [&](int seg) {
        if (seg + lane * kTile >= w1 || page >= a.num_pages || page < 0) page = -1;
        ks = vs = 1.0f;
        if (page >= 0) {
            const int64_t at = static_cast<int64_t>(page) * a.G + g;
            ks = a.k_scale[at];
            vs = a.v_scale[at];
        }
    };
    // Every address is a uniform base and a lane's constant offset.
    const uint32_t k_lane = static_cast<uint32_t>(lane * 16);
    const uint32_t v_lane = static_cast<uint32_t>(4 * g4 * D + n16 * kDims);
    Step<D> x;
    auto row_of = [&](int key, int t) { return head + ((key + t * kTile) & page_mask) * D; };
    // The next step's loads are issued unconditionally, so that a wait counts on them; where
    // there is no next step (`live` 0) all lanes read the cache's first bytes.
    auto fetch_k = [&](int key, int seg, uint32_t live) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int i = ((key - seg) >> 4) + t;
            const int64_t pg = max(__builtin_amdgcn_readlane(page, i), 0);
            const uint8_t* p = a.k + (live ? pg * a.k_page + row_of(key, t) : 0);
            const uint32_t at = live ? k_lane : 0;
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
                x.k[t * kHalves + h] = load_stream<u32x4>(p + at + h * 1024);
        }
    };
    auto fetch_v = [&](int key, int seg, uint32_t live) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int i = ((key - seg) >> 4) + t;
            const int64_t pg = max(__builtin_amdgcn_readlane(page, i), 0);
            const uint8_t* p = a.v + (live ? pg * a.v_page + row_of(key, t) : 0);
            const uint32_t at = live ? v_lane : 0;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if constexpr (kHalves == 2) {
                    const u32x2 w = load_stream<u32x2>(p + at + r * D);
                    x.v[4 * t + r][0] = w.x;
                    x.v[4 * t + r][kHalves - 1] = w.y;
                } else {
                    x.v[4 * t + r][0] = load_stream<uint32_t>(p + at + r * D);
                }
            }
        }
    };
    if (w0 < w1) {
        look_up(w0);
        fetch_k(w0, w0, 1);
        fetch_v(w0, w0, 1);
    }

    // Queries as operand columns: lane (n, g4) of an operand holds row n's elements
    // 64 h + 16 g4 + 8 s + i.  They lie in LDS - in registers they would cost 16 to 48 of
    // the 128 that leave room for four workgroups on a compute unit - and are read once a
    // step; each thread lays out operands of its own lane.
    int limit[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const int row = row0 + t * kTile + n16;
        // rows that do not exist see everything, so that they mask nothing
        limit[t] = row < row_end ? seen_by(a, len, count, row / a.group) : a.max_tokens;
    }
    for (int e = wave; e < TILES * 2 * kHalves; e += WAVES) {
        const int t = e / (2 * kHalves), s = e - t * (2 * kHalves);
        const int row = row0 + t * kTile + n16;
        const int at = row / a.group;
        Packet<T> p{};
        if (row < row_end)
            load_packet(p, static_cast<const T*>(a.q) + b * a.qs[0] +
                               (g * a.group + row - at * a.group) * a.qs[1] + at * a.qs[2] +
                               (s >> 1) * 64 + g4 * 16 + (s & 1) * 8);
        float f[8];
        unpack(p, f);
        bf16x8s w[kTerms];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            __bf16 part[kTerms];
            split_bf16<kTerms>(f[i], part);
#pragma unroll
            for (int m = 0; m < kTerms; ++m) w[m][i] = part[m];
        }
#pragma unroll
        for (int m = 0; m < kTerms; ++m) lds.in.q[(t * kTerms + m) * 2 * kHalves + s][lane] = w[m];
    }
    __syncthreads();

    f32x4 o[TILES][kDims];
    float top[TILES], base[TILES], sum[TILES];   // running maximum; the same, 0 before any
    uint32_t poison[TILES];                      // bit 8 r + j: o[.][j][r] is NaN
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        poison[t] = 0u;
#pragma unroll
        for (int j = 0; j < kDims; ++j) o[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        top[t] = -kInf;
        base[t] = 0.0f;
        sum[t] = 0.0f;
    }

    // One step of 32 keys.  `whole`: every row sees every key of it.
    auto step = [&](auto whole_tag, int key, int seg, int end) {
        constexpr bool kWhole = decltype(whole_tag)::value;
        const int i0 = (key - seg) >> 4;
        const float ks0 = lane_scale<kKeyDown>(ks, i0);
        const float ks1 = lane_scale<kKeyDown>(ks, i0 + 1);
        const float vs0 = lane_scale<kValueDown>(vs, i0);
        const float vs1 = lane_scale<kValueDown>(vs, i0 + 1);
        int end0 = 0, end1 = 0;                  // first key of a tile that no page holds
        if constexpr (!kWhole) {
            end0 = __builtin_amdgcn_readlane(page, i0) >= 0 ? most : key;
            end1 = __builtin_amdgcn_readlane(page, i0 + 1) >= 0 ? most : key;
        }

        // The keys' rows go through the wave's own part of LDS into operand order (16 bytes
        // of one row per lane, 16 rows side by side).  A row's 16-byte chunks are permuted by
        // its number, so that neighbouring rows' equal chunks lie in different banks.  A
        // wave's LDS accesses keep their order, so nothing waits.
        constexpr int kChunks = D / 16;
        u32x4* const mine = lds.in.k[wave];
#pragma unroll
        for (int j = 0; j < 2 * kHalves; ++j) {
            const int r = (j * 64 + lane) / kChunks, c = lane % kChunks;
            mine[r * kChunks + (c ^ swizzle<D>(r))] = x.k[j];
        }
        wave_order();
        // an index that the compiler cannot know keeps the reads of the queries in the loop,
        // and their registers free
        int my = lane;
        asm volatile("" : "+v"(my));
        f32x4 s[TILES][2];
#pragma unroll
        for (int u = 0; u < TILES; ++u)
#pragma unroll
            for (int t = 0; t < 2; ++t) s[u][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
            u32x4 w[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int r = t * kTile + n16;
                w[t] = mine[r * kChunks + ((4 * h + g4) ^ swizzle<D>(r))];
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                bf16x8s kf[2];
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    kf[t] = e ? widen8(w[t].z, w[t].w, t ? ks1 : ks0)
                              : widen8(w[t].x, w[t].y, t ? ks1 : ks0);
#pragma unroll
                for (int u = 0; u < TILES; ++u)
#pragma unroll
                    for (int m = kTerms - 1; m >= 0; --m) {
                        const bf16x8s qf = lds.in.q[(u * kTerms + m) * 2 * kHalves + 2 * h + e][my];
#pragma unroll
                        for (int t = 0; t < 2; ++t)
                            s[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t], qf, s[u][t],
                                                                              0, 0, 0);
                    }
            }
        }
        wave_order();
        const uint32_t live = key + kAttendStep < end;
        const int next = live ? key + kAttendStep : key;
        fetch_k(next, seg, live);

        if constexpr (!kWhole) {
            // What no row sees may hold anything, and 0 * NaN must not reach the sums.  A NaN
            // that only some rows see is taken out too and noted for those rows.
            uint32_t nans[2] = {0u, 0u};         // 8 bits per key, a tile's four keys a word
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int kk = key + (i >> 2) * kTile + 4 * g4 + (i & 3);
                const bool there = kk < ((i >> 2) ? end1 : end0);
#pragma unroll
                for (int h = 0; h < kHalves; ++h) {
                    const uint32_t w = there ? x.v[i][h] : 0u;
                    const uint32_t n = nan_bytes(w) >> 7;
                    nans[i >> 2] |= gather_bits(n) << (8 * (i & 3) + 4 * h);
                    x.v[i][h] = w & ~(n * 0xFFu);
                }
            }
            if (__ballot((nans[0] | nans[1]) != 0u)) {
                // lane (m, g) holds the bits of keys 4 g .. and dimensions m * kDims ..
#pragma unroll
                for (int i = 0; i < 8; ++i) {
#pragma unroll 1
                    for (int from = 0; from < 4; ++from) {
                        const int kk = key + (i >> 2) * kTile + 4 * from + (i & 3);
                        uint32_t bits = 0;
#pragma unroll 1
                        for (int r = 0; r < 4; ++r)
                            bits |= (static_cast<uint32_t>(
                                         __shfl(static_cast<int>(nans[i >> 2]),
                                                from * kTile + 4 * g4 + r)) >> (8 * (i & 3)) &
                                     0xFFu) << (8 * r);
#pragma unroll
                        for (int u = 0; u < TILES; ++u)
                            if (kk < limit[u]) poison[u] |= bits;
                    }
                }
            }
        }
        bf16x8s pf[TILES][kParts];               // weights as operand columns, in parts
#pragma unroll
        for (int u = 0; u < TILES; ++u) {
            float y[8];                          // logits before their scale
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = s[u][i >> 2][i & 3];
            if constexpr (!kWhole) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int kk = key + (i >> 2) * kTile + 4 * g4 + (i & 3);
                    if (kk >= min(limit[u], (i >> 2) ? end1 : end0)) y[i] = -kInf;
                }
            }
            if (a.logits) {
                // a uniform base and a lane's offset, which is not worth a register
                const int row = row0 + u * kTile + (my & 15);
                float* to = a.logits +
                            ((b * a.G + g) * static_cast<int64_t>(a.rows) + row0 + u * kTile) *
                                a.logit_stride + key;
                const uint32_t at = static_cast<uint32_t>(my & 15) *
                                        static_cast<uint32_t>(a.logit_stride) + (my >> 4) * 4;
                if (row < row_end) {
                    *reinterpret_cast<f32x4*>(to + at) =
                        f32x4{y[0] * a.scale, y[1] * a.scale, y[2] * a.scale, y[3] * a.scale};
                    *reinterpret_cast<f32x4*>(to + at + kTile) =
                        f32x4{y[4] * a.scale, y[5] * a.scale, y[6] * a.scale, y[7] * a.scale};
                }
            }
            weigh<8, kDims>(y, a.scale, top[u], base[u], sum[u], o[u]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                __bf16 w[kParts];
                split_bf16<kParts>(y[i], w);
#pragma unroll
                for (int m = 0; m < kParts; ++m) pf[u][m][i] = w[m];
            }
        }
        // O^T: 4 dimensions of each word, keys paired by byte permutation
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
            u32x4s vf[4];
#pragma unroll
            for (int pr = 0; pr < 4; ++pr) {
                const uint32_t wa = x.v[2 * pr][h], wb = x.v[2 * pr + 1][h];
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
                    for (int m = kParts - 1; m >= 0; --m)
                        o[u][4 * h + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8s, vf[j]), pf[u][m], o[u][4 * h + j], 0, 0,
                            0);
        }
        fetch_v(next, seg, live);
    };

    for (int seg = w0; seg < w1; seg += 64 * kTile) {
        const int seg_end = min(w1, seg + 64 * kTile);
        if (seg > w0) {
            page = page_at(seg + lane * kTile, w1);
            look_up(seg);
            fetch_k(seg, seg, 1);
            fetch_v(seg, seg, 1);
        }
        // steps that every row sees whole: before `least`, if all of the segment's pages exist
        const bool paged = __ballot(seg + lane * kTile < seg_end && page < 0) == 0;
        const int whole_end = paged ? min(seg_end, least) : seg;
        int key = seg;
        for (; key + kAttendStep <= whole_end; key += kAttendStep)
            step(std::true_type{}, key, seg, seg_end);
        for (; key < seg_end; key += kAttendStep)
            step(std::false_type{}, key, seg, seg_end);
    }

    // merge the four waves, a 16-row tile at a time (all have read their last queries)
    __syncthreads();
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
        for (int w = 1; w < WAVES; ++w) all = fmaxf(all, top_of[w][u * kTile + n16]);
        const float f = top[u] == -kInf ? 0.0f : top[u] == all ? 1.0f : exp2_hw(top[u] - all);
        // lane (n, g4) holds dimensions (4 g4 + r) * kDims + j of row n
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < kDims; ++j)
                lds.out[wave][n16][(4 * g4 + r) * kDims + j] =
                    poison[u] >> (8 * r + j) & 1u ? __builtin_nanf("") : o[u][j][r] * f;
        __syncthreads();
        constexpr int kPer = kTile * D / (64 * WAVES);   // dimensions per thread: 2 to 8
        const int r = threadIdx.x / (D / kPer), d0 = threadIdx.x % (D / kPer) * kPer;
        const int row = row0 + u * kTile + r;
        if (row < row_end) {
            float m = top_of[0][u * kTile + r];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) m = fmaxf(m, top_of[w][u * kTile + r]);
            float total = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                // without a maximum a sum is 0, or NaN, which stays
                const float tw = top_of[w][u * kTile + r];
                total += sum_of[w][u * kTile + r] *
                         (tw == m || tw == -kInf ? 1.0f : exp2_hw(tw - m));
            }
            float y[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                y[i] = lds.out[0][r][d0 + i];
#pragma unroll
                for (int w = 1; w < WAVES; ++w) y[i] += lds.out[w][r][d0 + i];
            }
            const int64_t line = (b * a.G + g) * static_cast<int64_t>(a.rows) + row;
            if (WAVES == 8 || a.splits == 1) {           // eight waves: never split
                const float inv = total > 0.0f || total != total ? kValueUp / total : 0.0f;
                const int t = row / a.group;
                T* to = static_cast<T*>(a.out) + b * a.os[0] +
                        (g * a.group + row - t * a.group) * a.os[1] + t * a.os[2] + d0;
                Run<T, kPer> z;
#pragma unroll
                for (int i = 0; i < kPer; ++i) z.x[i] = from_f32<T>(y[i] * inv);
                *reinterpret_cast<Run<T, kPer>*>(to) = z;
                if (d0 == 0) {
                    const float l = total > 0.0f || total != total ? m + __log2f(total) : -kInf;
                    lse_of[u * kTile + r] = l;
                    if (a.lse) a.lse[line] = l;
                }
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
    // A call of few workgroups that see every token turns its logits into weights itself:
    // they were stored by other waves of the same workgroup, before the barriers above.
    if (WAVES == 8 && a.w_out)
        token_weights(a, b, g, lse_of, len, count, static_cast<int>(threadIdx.x) * 4, 256 * WAVES);
}

// Many rows per key head (a run of queries): attend_rows_kernel.  Here the products count,
// and every row needs the same widened keys and values, so a workgroup widens 64 keys at a
// time into LDS, in the order in which operands are read, and its four waves take 16 * TILES
// rows each over all keys.  Wave w widens 16-key tile w: page and scales are uniform to it.
// One buffer of 33 KB, so that four workgroups of 16-row waves share a compute unit and one
// multiplies while another widens or waits: a wave's step is a chain of dependent products,
// maxima and exponentials that leaves most of its issue slots to others.
constexpr int kRowStep = 64;

template <int D>
struct RowsShared {
    // operand e of tile t, operand j of 32 keys; a key operand's lanes are permuted by its
    // 16-byte chunk, so that the chunks of one row, written together, lie in different banks
    bf16x8s k[4][D / 32][64];
    u32x2 v[2][D / 16][64][2];           // two halves: 8 bytes of each 16-key tile
    alignas(16) uint8_t nan[4][kTile][16];   // per key, a bit per dimension: masked steps only
    int state[4];                        // of each tile: kNoPage, kLost
};
constexpr int kNoPage = 1, kLost = 2;    // kLost: a NaN among the values (masked steps)

template <typename T, int D, int TILES>
__global__ __launch_bounds__(kThreads, TILES == 1 && Terms<T>::n == 1 ? 3 : 2) void attend_rows_kernel(const AttendArgs a) {
    constexpr int kTerms = Terms<T>::n;
    constexpr int kParts = kTerms < 2 ? 2 : kTerms;
    constexpr int kHalves = D / 64;
    constexpr int kDims = D / 16;
    constexpr int kSteps = 2 * kHalves;          // operands along a row
    constexpr int kChunks = D / 16;
    __shared__ RowsShared<D> lds;

    uint32_t id = blockIdx.x;
    const int rg = static_cast<int>(id % static_cast<uint32_t>(a.row_groups));
    id /= static_cast<uint32_t>(a.row_groups);
    const int split = static_cast<int>(id % static_cast<uint32_t>(a.splits));
    id /= static_cast<uint32_t>(a.splits);
    const int g = static_cast<int>(id % static_cast<uint32_t>(a.G));
    const int64_t b = id / static_cast<uint32_t>(a.G);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, g4 = lane >> 4;

    const int len = attend_length(a, b), count = attend_count(a, b);
    const int group0 = rg * TILES * kTile * kAttendWaves;
    const int group_end = min(group0 + TILES * kTile * kAttendWaves, count * a.group);
    if (group0 >= group_end) return;
    const int least = seen_by(a, len, count, group0 / a.group);
    const int most = seen_by(a, len, count, (group_end - 1) / a.group);
    const int64_t key_begin = split * a.chunk;
    if (split > 0 && key_begin >= most) return;
    const int k0 = static_cast<int>(key_begin);
    const int k1 = static_cast<int>(min(key_begin + a.chunk, static_cast<int64_t>(most)));

    // this wave's rows
    const int row0 = group0 + wave * TILES * kTile;
    const int row_end = min(row0 + TILES * kTile, group_end);
    int limit[TILES];
    bf16x8s q[TILES][kTerms][kSteps];
#pragma unroll
    for (int u = 0; u < TILES; ++u) {
        const int row = row0 + u * kTile + n16;
        const bool live = row < row_end;
        const int at = live ? row / a.group : 0;
        limit[u] = live ? seen_by(a, len, count, at) : a.max_tokens;
        const T* src = static_cast<const T*>(a.q) + b * a.qs[0] +
                       (g * a.group + (live ? row - at * a.group : 0)) * a.qs[1] + at * a.qs[2];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            Packet<T> p{};
            if (live) load_packet(p, src + (s >> 1) * 64 + g4 * 16 + (s & 1) * 8);
            float f[8];
            unpack(p, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                __bf16 w[kTerms];
                split_bf16<kTerms>(f[i], w);
#pragma unroll
                for (int m = 0; m < kTerms; ++m) q[u][m][s][i] = w[m];
            }
        }
    }
    f32x4 o[TILES][kDims];
    float top[TILES], base[TILES], sum[TILES];
    uint32_t poison[TILES];                      // bit 8 r + j: o[.][j][r] is NaN
#pragma unroll
    for (int u = 0; u < TILES; ++u) {
        poison[u] = 0u;
#pragma unroll
        for (int j = 0; j < kDims; ++j) o[u][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        top[u] = -kInf;
        base[u] = 0.0f;
        sum[u] = 0.0f;
    }

    // Lane l looks up this wave's tile of the l-th of 64 steps.
    const int64_t head = static_cast<int64_t>(g) * (D << a.page_shift);
    const int page_mask = (1 << a.page_shift) - 1;
    int page = -1;
    float ks = 1.0f, vs = 1.0f;
    auto look_up = [&](int seg) {
        const int mine = seg + lane * kRowStep + wave * kTile;
        page = -1;
        if (mine < k1) page = a.pages[b * a.pages_stride + (mine >> a.page_shift)];
        if (page >= a.num_pages || page < 0) page = -1;
        ks = vs = 1.0f;
        if (page >= 0) {
            const int64_t at = static_cast<int64_t>(page) * a.G + g;
            ks = a.k_scale[at];
            vs = a.v_scale[at];
        }
    };
    // A step's bytes of this wave's tile, loaded a step ahead.
    struct Raw {
        u32x4 k[kHalves];                // 1 KB each of the tile's rows in order
        uint32_t v[4][kHalves];          // keys 4 g4 + r, dimensions n16 * kDims ..
        int page;
        float ks, vs;
    };
    auto fetch = [&](int step, Raw& x) {
        const int i = step & 63;         // within the segment looked up
        x.page = __builtin_amdgcn_readlane(page, i);
        x.ks = lane_scale<kKeyDown>(ks, i);
        x.vs = lane_scale<kValueDown>(vs, i);
        const int64_t pg = max(x.page, 0);
        const int64_t row = head + ((k0 + step * kRowStep + wave * kTile) & page_mask) * D;
        const uint8_t* kp = a.k + pg * a.k_page + row;
        const uint8_t* vp = a.v + pg * a.v_page + row;
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
            x.k[h] = *reinterpret_cast<const u32x4*>(kp + lane * 16 + h * 1024);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint8_t* p = vp + (4 * g4 + r) * D + n16 * kDims;
            if constexpr (kHalves == 2) {
                const u32x2 w = *reinterpret_cast<const u32x2*>(p);
                x.v[r][0] = w.x;
                x.v[r][kHalves - 1] = w.y;
            } else {
                x.v[r][0] = *reinterpret_cast<const uint32_t*>(p);
            }
        }
    };
    const int steps = k1 > k0 ? (k1 - k0 + kRowStep - 1) / kRowStep : 0;
    // The step behind the last, and tiles without a page, load from page 0, unused.
    Raw x;
    look_up(k0);
    fetch(0, x);
#pragma unroll 1
    for (int st = 0; st < steps; ++st) {
        const int key = k0 + st * kRowStep;
        __syncthreads();                         // all have read the step before
        // widen this wave's tile
        {
            const int pg = x.page;
            const float ksc = x.ks, vsc = x.vs;
            bool bad = false;
            if (key + kRowStep > least || pg < 0) {
                // what no row sees may hold anything; a NaN that some row sees is set apart
                const int there = pg < 0 ? key : most;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const bool in = key + wave * kTile + 4 * g4 + r < there;
                    uint32_t bits = 0;
#pragma unroll
                    for (int h = 0; h < kHalves; ++h) {
                        uint32_t w = in ? x.v[r][h] : 0u;
                        const uint32_t n = nan_bytes(w) >> 7;
                        bits |= gather_bits(n) << (4 * h);
                        x.v[r][h] = w & ~(n * 0xFFu);
                    }
                    lds.nan[wave][4 * g4 + r][n16] = static_cast<uint8_t>(bits);
                    bad = bad || bits != 0;
                }
            }
            const uint64_t any = __ballot(bad);
            if (lane == 0) lds.state[wave] = (pg < 0 ? kNoPage : 0) | (any != 0 ? kLost : 0);
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                // lane's 16 bytes: row r, chunk c = 4 e' + g' holds operands 2 e', 2 e' + 1
                const int r = (h * 64 + lane) / kChunks, c = lane % kChunks;
                const int slot = (c & 3) * kTile + (r ^ c);
                lds.k[wave][2 * (c >> 2)][slot] = widen8(x.k[h].x, x.k[h].y, ksc);
                lds.k[wave][2 * (c >> 2) + 1][slot] = widen8(x.k[h].z, x.k[h].w, ksc);
            }
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                uint32_t lo[2], hi[2];
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    lo[p] = __builtin_amdgcn_perm(x.v[2 * p + 1][h], x.v[2 * p][h], 0x05010400u);
                    hi[p] = __builtin_amdgcn_perm(x.v[2 * p + 1][h], x.v[2 * p][h], 0x07030602u);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    u32x2 w = {pack_bf16(j < 2 ? lo[0] : hi[0], vsc, j & 1),
                               pack_bf16(j < 2 ? lo[1] : hi[1], vsc, j & 1)};
                    lds.v[wave >> 1][4 * h + j][lane][wave & 1] = w;
                }
            }
        }
        if (((st + 1) & 63) == 0) look_up(key + kRowStep);
        fetch(st + 1, x);
        __syncthreads();
        if (row0 >= row_end) continue;
        int any = 0, there[4];                   // first key of a tile that no page holds
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int state = __builtin_amdgcn_readfirstlane(lds.state[t]);
            there[t] = state & kNoPage ? key : most;
            any |= state;
        }
        const bool whole = key + kRowStep <= least && any == 0;
        const bool lost = (any & kLost) != 0;
        // Operands are read from LDS a group ahead of the products that take them; the
        // scheduling fences keep the compiler from sinking the reads to their use, where each
        // would be waited for alone.
        auto key_operands = [&](int t, bf16x8s (&kf)[kSteps]) {
#pragma unroll
            for (int e = 0; e < kSteps; ++e)
                kf[e] = lds.k[t][e][g4 * kTile + (n16 ^ (4 * (e >> 1) + g4))];
        };
        constexpr int kGroup = 4;
        auto value_operands = [&](int i, bf16x8s (&vf)[kGroup]) {
#pragma unroll
            for (int j = 0; j < kGroup; ++j)
                vf[j] = *reinterpret_cast<const bf16x8s*>(
                    &lds.v[i / kHalves][kGroup * (i % kHalves) + j][lane][0]);
        };
        f32x4 s[TILES][4];
        bf16x8s kf[2][kSteps], vf[2][kGroup];
        key_operands(0, kf[0]);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (t < 3) key_operands(t + 1, kf[(t + 1) & 1]);
            else value_operands(0, vf[0]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < TILES; ++u) s[u][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < kSteps; ++e)
#pragma unroll
                for (int u = 0; u < TILES; ++u)
#pragma unroll
                    for (int m = kTerms - 1; m >= 0; --m)
                        s[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t & 1][e], q[u][m][e],
                                                                          s[u][t], 0, 0, 0);
        }
        bf16x8s pf[TILES][2][kParts];
#pragma unroll
        for (int u = 0; u < TILES; ++u) {
            float y[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = s[u][i >> 2][i & 3];
            if (!whole) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int kk = key + (i >> 2) * kTile + 4 * g4 + (i & 3);
                    if (kk >= min(limit[u], there[i >> 2])) y[i] = -kInf;
                }
            }
            weigh<16, kDims>(y, a.scale, top[u], base[u], sum[u], o[u]);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                __bf16 w[kParts];
                split_bf16<kParts>(y[i], w);
#pragma unroll
                for (int m = 0; m < kParts; ++m) pf[u][i >> 3][m][i & 7] = w[m];
            }
        }
#pragma unroll
        for (int i = 0; i < 2 * kHalves; ++i) {
            if (i + 1 < 2 * kHalves) value_operands(i + 1, vf[(i + 1) & 1]);
            __builtin_amdgcn_sched_barrier(0);
            const int h = i / kHalves, j0 = kGroup * (i % kHalves);
#pragma unroll
            for (int m = kParts - 1; m >= 0; --m)
#pragma unroll
                for (int j = 0; j < kGroup; ++j)
#pragma unroll
                    for (int u = 0; u < TILES; ++u)
                        o[u][j0 + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            vf[i & 1][j], pf[u][h][m], o[u][j0 + j], 0, 0, 0);
        }
        if (lost) {
            // a NaN value reaches the rows that see its key, and no other
#pragma unroll 1
            for (int i = 0; i < kRowStep; ++i) {
                const uint32_t bits =
                    *reinterpret_cast<const uint32_t*>(&lds.nan[i >> 4][i & 15][4 * g4]);
                if ((lds.state[i >> 4] & kLost) == 0) continue;    // (not written)
#pragma unroll
                for (int u = 0; u < TILES; ++u)
                    if (key + i < limit[u]) poison[u] |= bits;
            }
        }
    }

    // each wave has its rows' whole sums: lane (n, g4) holds dimensions (4 g4 + r) kDims + j
#pragma unroll
    for (int u = 0; u < TILES; ++u) {
        const int row = row0 + u * kTile + n16;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < kDims; ++j)
                if (poison[u] >> (8 * r + j) & 1u) o[u][j][r] = __builtin_nanf("");
        float total = sum[u];
        total += __shfl_xor(total, 16);
        total += __shfl_xor(total, 32);
        if (row >= row_end) continue;
        const int64_t line = (b * a.G + g) * static_cast<int64_t>(a.rows) + row;
        if (TILES == 2 || a.splits == 1) {           // 32 rows a wave: never split
            const float inv = total > 0.0f || total != total ? kValueUp / total : 0.0f;
            const int t = row / a.group;
            T* to = static_cast<T*>(a.out) + b * a.os[0] +
                    (g * a.group + row - t * a.group) * a.os[1] + t * a.os[2] + 4 * g4 * kDims;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                Run<T, kDims> z;
#pragma unroll
                for (int j = 0; j < kDims; ++j) z.x[j] = from_f32<T>(o[u][j][r] * inv);
                *reinterpret_cast<Run<T, kDims>*>(to + r * kDims) = z;
            }
            if (a.lse && g4 == 0)
                a.lse[line] = total > 0.0f || total != total ? top[u] + __log2f(total) : -kInf;
        } else {
            const int64_t part = line * a.splits + split;
            float* to = a.part_out + part * D + 4 * g4 * kDims;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                Run<float, kDims> z;
#pragma unroll
                for (int j = 0; j < kDims; ++j) z.x[j] = o[u][j][r];
                *reinterpret_cast<Run<float, kDims>*>(to + r * kDims) = z;
            }
            if (g4 == 0) {
                a.part_max[part] = top[u];
                a.part_sum[part] = total;
            }
        }
    }
}

// The parts of a row that were written: a part is there where its first key is seen by the
// workgroup that wrote it; parts whose keys this row does not see hold a maximum of -inf (and
// zeros, or NaN).
struct JoinRow {
    int64_t b, first;                            // sequence; the row's first part
    int g, head, t, parts;
    bool live;
};
__device__ __forceinline__ JoinRow join_row(const AttendArgs& a, uint32_t line, uint32_t lines) {
    JoinRow r;
    const uint32_t bg = line < lines ? line / static_cast<uint32_t>(a.rows) : 0;
    const uint32_t row = line - bg * static_cast<uint32_t>(a.rows);
    r.b = bg / static_cast<uint32_t>(a.G);
    r.g = static_cast<int>(bg - static_cast<uint32_t>(r.b) * a.G);
    r.t = static_cast<int>(row / static_cast<uint32_t>(a.group));
    r.head = r.g * a.group + static_cast<int>(row) - r.t * a.group;
    const int len = attend_length(a, r.b), count = attend_count(a, r.b);
    r.live = line < lines && r.t < count;
    const int chunk = static_cast<int>(a.chunk);
    r.parts = r.live ? (seen_by(a, len, count, r.t) + chunk - 1) / chunk : 0;   // <= splits
    r.first = static_cast<int64_t>(line) * a.splits;
    return r;
}

template <typename T, int N>
__device__ __forceinline__ void join_out(const AttendArgs& a, const JoinRow& r, uint32_t line,
                                         int dim, float m, float total, const float (&y)[N]) {
    const float inv = total > 0.0f || total != total ? kValueUp / total : 0.0f;
    T* to = static_cast<T*>(a.out) + r.b * a.os[0] + r.head * a.os[1] + r.t * a.os[2] + dim;
    Run<T, N> z;
#pragma unroll
    for (int k = 0; k < N; ++k) z.x[k] = from_f32<T>(y[k] * inv);
    *reinterpret_cast<Run<T, N>*>(to) = z;
    if (a.lse && dim == 0)
        a.lse[line] = total > 0.0f || total != total ? m + __log2f(total) : -kInf;
}

// Joins few parts (<= kFewParts), four dimensions to a thread: every thread reads the maxima
// and sums of its row itself, so all that it needs is under way at once.
constexpr int kFewParts = 8;
template <typename T, int D>
__device__ __forceinline__ void join_few(const AttendArgs& a, uint32_t block, uint32_t lines) {
    constexpr int kLanes = D / 4, kBatch = 4;
    const uint32_t line = block * (kThreads / kLanes) + threadIdx.x / kLanes;   // < 2^24 + 16
    const int dim = static_cast<int>(threadIdx.x) % kLanes * 4;
    const JoinRow r = join_row(a, line, lines);
    if (!r.live) return;
    float m = -kInf, total = 0.0f, y[4] = {};
    for (int i0 = 0; i0 < r.parts; i0 += kBatch) {
        float pm[kBatch], ps[kBatch];
        f32x4 v[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int64_t part = r.first + min(i0 + j, r.parts - 1);
            pm[j] = a.part_max[part];
            ps[j] = a.part_sum[part];
            v[j] = *reinterpret_cast<const f32x4*>(a.part_out + part * D + dim);
        }
        float up = m;
#pragma unroll
        for (int j = 0; j < kBatch; ++j) up = fmaxf(up, pm[j]);
        const float shrink = up == m ? 1.0f : exp2_hw(m - up);
        m = up;
        total *= shrink;
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] *= shrink;
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (i0 + j >= r.parts) break;
            const float f = pm[j] == -kInf ? 1.0f : exp2_hw(pm[j] - up);
            total += ps[j] * f;
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] += v[j][k] * f;
        }
    }
    join_out<T>(a, r, line, dim, m, total, y);
}

// Joins many parts, a workgroup to a row: a lane has the maximum and sum of one of 64 parts,
// and the waves share the outputs, each reading kBatch at a time.
template <typename T, int D>
__device__ __forceinline__ void join_many(const AttendArgs& a, uint32_t line, uint32_t lines) {
    constexpr int kPer = D / 64, kBatch = 8;
    __shared__ float merge[kAttendWaves][D];
    __shared__ float sums[kAttendWaves];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const JoinRow r = join_row(a, line, lines);
    if (!r.live) return;                         // all threads
    float m = -kInf, total = 0.0f, y[kPer] = {};
    for (int seg = 0; seg < r.parts; seg += 64) {
        const int here = min(r.parts - seg, 64);
        const float pm = lane < here ? a.part_max[r.first + seg + lane] : -kInf;
        const float ps = lane < here ? a.part_sum[r.first + seg + lane] : 0.0f;
        const float up = fmaxf(m, wave_max(pm));
        const float shrink = up == m ? 1.0f : exp2_hw(m - up);
        m = up;
        total *= shrink;
#pragma unroll
        for (int k = 0; k < kPer; ++k) y[k] *= shrink;
        const float f = pm == -kInf ? 1.0f : exp2_hw(pm - up);
        const float sf = ps * f;
        for (int i0 = wave; i0 < here; i0 += kAttendWaves * kBatch) {
            float v[kBatch][kPer];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const int i = min(i0 + j * kAttendWaves, here - 1);
                const float* from = a.part_out + (r.first + seg + i) * D + lane * kPer;
#pragma unroll
                for (int k = 0; k < kPer; ++k) v[j][k] = from[k];
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const int i = i0 + j * kAttendWaves;
                if (i >= here) break;
                const float fi = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), i));
                total += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sf), i));
#pragma unroll
                for (int k = 0; k < kPer; ++k) y[k] += v[j][k] * fi;
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) merge[wave][lane * kPer + k] = y[k];
    if (lane == 0) sums[wave] = total;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < kAttendWaves; ++w) {
        total += sums[w];
#pragma unroll
        for (int k = 0; k < kPer; ++k) y[k] += merge[w][lane * kPer + k];
    }
    join_out<T>(a, r, line, lane * kPer, m, total, y);
}

// log2 of the sums of up to kFewRows rows, from their parts, into LDS: a wave to a row.
constexpr int kFewRows = 32;
__device__ __forceinline__ void sums_of_parts(const AttendArgs& a, int64_t bg, int len, int count,
                                              float* lse) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int row = wave; row < count * a.group; row += kAttendWaves) {
        const int limit = seen_by(a, len, count, row / a.group);
        const int parts = static_cast<int>((limit + a.chunk - 1) / a.chunk);
        const int64_t first = (bg * a.rows + row) * a.splits;
        float m = -kInf;
        for (int i = lane; i < parts; i += 64) m = fmaxf(m, a.part_max[first + i]);
        m = wave_max(m);
        float total = 0.0f;
        for (int i = lane; i < parts; i += 64) {
            const float pm = a.part_max[first + i];
            total += a.part_sum[first + i] * (pm == -kInf ? 1.0f : exp2_hw(pm - m));
        }
        total = wave_sum(total);
        if (lane == 0) lse[row] = total > 0.0f || total != total ? m + __log2f(total) : -kInf;
    }
    __syncthreads();
}

// What is left after the parts: the rows' joins (the first `joins` workgroups) and, where
// weights are wanted and the rows are few, the tokens' weights (`blocks` workgroups to a
// (sequence, key head), four neighbouring tokens to a thread).
template <typename T, int D, bool MANY>
__global__ __launch_bounds__(kThreads) void attend_finish_kernel(const AttendArgs a, uint32_t lines,
                                                                 uint32_t joins, uint32_t blocks) {
    if (blockIdx.x < joins) {
        if constexpr (MANY) join_many<T, D>(a, blockIdx.x, lines);
        else join_few<T, D>(a, blockIdx.x, lines);
        return;
    }
    __shared__ float lse[kFewRows];
    const uint32_t id = blockIdx.x - joins;
    const uint32_t bg = id / blocks;
    const int64_t b = bg / static_cast<uint32_t>(a.G);
    const int n0 = static_cast<int>(id % blocks) * 4 * kThreads;
    const int len = attend_length(a, b), count = attend_count(a, b);
    if (n0 >= len) return;
    sums_of_parts(a, bg, len, count, lse);
    token_weights(a, b, static_cast<int>(bg - b * a.G), lse, len, count,
                  n0 + static_cast<int>(threadIdx.x) * 4, a.max_tokens);
}

// The tokens' weights from few rows whose sums lie in the workspace.
__global__ __launch_bounds__(kThreads) void attend_weights_kernel(const AttendArgs a,
                                                                  uint32_t blocks) {
    const uint32_t bg = blockIdx.x / blocks;
    const int64_t b = bg / static_cast<uint32_t>(a.G);
    const int n0 = (static_cast<int>(blockIdx.x % blocks) * kThreads +
                    static_cast<int>(threadIdx.x)) * 4;
    token_weights(a, b, static_cast<int>(bg - b * a.G), a.lse + static_cast<int64_t>(bg) * a.rows,
                  attend_length(a, b), attend_count(a, b), n0, a.max_tokens);
}

// The tokens' weights from many rows, whose sums lie in the workspace: the logits are made a
// second time, since through memory they would cost 8 bytes per row and key (16 sequences of
// up to 48 queries and 4200 keys, 28 heads: 183 us for the call, 82 so, 51 without weights).
// A wave holds the operands of its 64 keys and walks over the rows, 16 at a time (32 keys: 93
// us, 16: 110); a lane adds up what its row of each tile gives 16 keys, and the 16 lanes of a
// key are summed at the end.  Reading and widening the queries and the exponentials bound it.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void attend_rows_weights_kernel(const AttendArgs a,
                                                                       uint32_t blocks) {
    constexpr int kTerms = Terms<T>::n, kSteps = D / 32, kTiles = kWeightKeys / kTile;
    const uint32_t bg = blockIdx.x / blocks;
    const int64_t b = bg / static_cast<uint32_t>(a.G);
    const int g = static_cast<int>(bg - static_cast<uint32_t>(b) * a.G);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, g4 = lane >> 4;
    const int key0 =
        (static_cast<int>(blockIdx.x % blocks) * kAttendWaves + wave) * kWeightKeys;
    const int len = attend_length(a, b), count = attend_count(a, b);
    if (key0 >= len) return;

    const int64_t head = static_cast<int64_t>(g) * (D << a.page_shift);
    bf16x8s kf[kTiles][kSteps];
    bool there[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const int key = key0 + t * kTile;
        int page = -1;
        if (key < len) page = a.pages[b * a.pages_stride + (key >> a.page_shift)];
        there[t] = page >= 0 && page < a.num_pages;
        const int64_t pg = there[t] ? page : 0;
        const float ks = there[t] ? kKeySize * a.k_scale[pg * a.G + g] : 1.0f;
        const uint8_t* p = a.k + pg * a.k_page + head +
                           ((key & ((1 << a.page_shift) - 1)) + n16) * D + g4 * 16;
#pragma unroll
        for (int h = 0; h < kSteps / 2; ++h) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(p + h * 64);
            kf[t][2 * h] = widen8(w.x, w.y, ks);
            kf[t][2 * h + 1] = widen8(w.z, w.w, ks);
        }
    }

    // the first row that sees key0
    const int rows = count * a.group;
    const int first = a.causal ? max(0, key0 - len + count) * a.group / kTile * kTile : 0;
    const float* lse = a.lse + static_cast<int64_t>(bg) * a.rows;
    struct Tile {
        Packet<T> q[kSteps];
        float l;
        int limit;
    };
    auto load = [&](int r0, Tile& x) {           // rows behind the last: it again, seeing nothing
        const int row = min(r0 + n16, rows - 1), at = row / a.group;
        x.limit = r0 + n16 < rows ? seen_by(a, len, count, at) : 0;
        x.l = lse[row];
        const T* src = static_cast<const T*>(a.q) + b * a.qs[0] +
                       (g * a.group + row - at * a.group) * a.qs[1] + at * a.qs[2];
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
            x.q[s] = *reinterpret_cast<const Packet<T>*>(src + (s >> 1) * 64 + g4 * 16 +
                                                         (s & 1) * 8);
    };
    float w[kTiles][4] = {};
    if (first < rows) {
        Tile next;
        load(first, next);
#pragma unroll 1
        for (int r0 = first; r0 < rows; r0 += kTile) {
            const Tile x = next;
            load(r0 + kTile, next);
            f32x4 s[kTiles];
#pragma unroll
            for (int t = 0; t < kTiles; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < kSteps; ++e) {
                bf16x8s qf[kTerms];
                if constexpr (kTerms == 1) {
                    qf[0] = __builtin_bit_cast(bf16x8s, x.q[e]);
                } else {
                    float f[8];
                    unpack(x.q[e], f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        __bf16 part[kTerms];
                        split_bf16<kTerms>(f[i], part);
#pragma unroll
                        for (int m = 0; m < kTerms; ++m) qf[m][i] = part[m];
                    }
                }
#pragma unroll
                for (int m = kTerms - 1; m >= 0; --m)
#pragma unroll
                    for (int t = 0; t < kTiles; ++t)
                        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t][e], qf[m], s[t], 0,
                                                                       0, 0);
            }
            const int limit = x.l == -kInf ? 0 : x.limit;
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    w[t][r] += key0 + t * kTile + 4 * g4 + r < limit
                                   ? exp2_hw(__builtin_fmaf(s[t][r], a.scale, -x.l))
                                   : 0.0f;
        }
    }
    const float* in = a.w_in ? a.w_in + b * a.wi[0] + g * a.wi[1] : nullptr;
    float* out = a.w_out + b * a.wo[0] + g * a.wo[1];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float y = w[t][r];
#pragma unroll
            for (int o = 1; o < kTile; o <<= 1) y += __shfl_xor(y, o);
            const int key = key0 + t * kTile + 4 * g4 + r;
            if (!there[t]) y = 0.0f;
            if (n16 == 0 && key < len) out[key] = in ? in[key] + y : y;
        }
}

template <typename T, int D>
hipError_t launch_t(const AttendArgs& a, const AttendPlan& p, int64_t B, hipStream_t st) {
    const dim3 grid(static_cast<unsigned>(B * a.G * a.splits * a.row_groups)), block(kThreads);
    if (p.shared_rows) {
        if constexpr (Terms<T>::n == 1) {
            if (p.tiles == 2)
                hipLaunchKernelGGL((attend_rows_kernel<T, D, 2>), grid, block, 0, st, a);
        }
        if (p.tiles == 1)
            hipLaunchKernelGGL((attend_rows_kernel<T, D, 1>), grid, block, 0, st, a);
    } else if (p.waves == 8) {
        if (p.tiles == 1)
            hipLaunchKernelGGL((attend_kernel<T, D, 1, 8>), grid, dim3(512), 0, st, a);
        else
            hipLaunchKernelGGL((attend_kernel<T, D, 2, 8>), grid, dim3(512), 0, st, a);
    } else {
        if (p.tiles == 1)
            hipLaunchKernelGGL((attend_kernel<T, D, 1, 4>), grid, block, 0, st, a);
        else
            hipLaunchKernelGGL((attend_kernel<T, D, 2, 4>), grid, block, 0, st, a);
    }
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    const uint32_t lines = static_cast<uint32_t>(B * a.G * a.rows);
    const uint32_t blocks = static_cast<uint32_t>((a.max_tokens + 4 * kThreads - 1) /
                                                  (4 * kThreads));
    if (a.splits > 1) {
        // the weights of few rows in the same launch
        const uint32_t more =
            a.w_out && !p.lse_kept ? static_cast<uint32_t>(B * a.G) * blocks : 0u;
        if (a.splits > kFewParts) {
            const uint32_t joins = lines;
            hipLaunchKernelGGL((attend_finish_kernel<T, D, true>), dim3(joins + more),
                               block, 0, st, a, lines, joins, blocks);
        } else {
            const uint32_t per = kThreads / (D / 4), joins = (lines + per - 1) / per;
            hipLaunchKernelGGL((attend_finish_kernel<T, D, false>), dim3(joins + more), block, 0, st,
                               a, lines, joins, blocks);
        }
        err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    if (a.w_out && p.shared_rows) {
        constexpr int kKeys = kWeightKeys * kAttendWaves;
        const uint32_t per = static_cast<uint32_t>((a.max_tokens + kKeys - 1) / kKeys);
        hipLaunchKernelGGL((attend_rows_weights_kernel<T, D>),
                           dim3(static_cast<unsigned>(B * a.G) * per), block, 0, st, a, per);
        err = hipGetLastError();
    } else if (a.w_out && p.lse_kept) {
        hipLaunchKernelGGL(attend_weights_kernel,
                           dim3(static_cast<unsigned>(B * a.G) * blocks), block, 0, st, a, blocks);
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
        if (p.lse_kept) a.lse = reinterpret_cast<float*>(ws + p.lse_off);
        if (p.logit_stride > 0) a.logits = reinterpret_cast<float*>(ws + p.logit_off);
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
    a.page_shift = __builtin_ctz(static_cast<unsigned>(c.page_tokens));   // a power of two
    a.num_pages = c.num_pages;
    a.max_pages = s.max_pages;
    a.max_tokens = s.max_tokens;
    a.causal = s.causal;
    const double scale = s.scale != 0.0f ? s.scale : 1.0 / std::sqrt(static_cast<double>(c.head_dim));
    // one rounding for both factors: every logit is off by at most 2^-24 of itself by it, which
    // f32 queries show where logits are large (a weight by 2^-24 of its logit's distance from
    // the maximum); a second factor would cost an operation per logit
    a.scale = static_cast<float>(scale * 1.4426950408889634 / kKeySize);
    if (s.dtype == E2S_DTYPE_F32) return launch_d<float>(a, p, s.batch, c.head_dim, st);
    if (s.dtype == E2S_DTYPE_F16) return launch_d<_Float16>(a, p, s.batch, c.head_dim, st);
    return launch_d<uint16_t>(a, p, s.batch, c.head_dim, st);
}

}  // namespace e2s
