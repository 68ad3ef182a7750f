// Norms of every head's queries and keys with the rotation of their positions
// (e2s_norm_rotate), and the pass back (e2s_norm_rotate_backward).
//
//   y = turned(x r w),  r = 1 / sqrt(mean(x^2) + eps)
//   back: g = turned back(grad), u = g w, dx = r (u - x r mean(u x r)), dw = sum g x r
//
// Streams: forward reads and writes every element once, back reads two and writes one, so what
// bounds both is a copy: of 1 GiB 5.8 TB/s, 6.3 with non-temporal loads and stores.  As in the
// rotation alone, a workgroup takes a run of TT tokens of one sequence for all heads: cosines and
// sines of the run go to LDS once, and a thread keeps those of its pairs in registers while it
// walks over the heads.  A unit is two chunks of W elements of a row that turn together (see
// rotary.hip), so the rotation stays in a lane; the units of a row are neighbouring lanes, LPR (a
// power of two) of them, which add the squares up across the row by DPP: no LDS and no second look
// at the row.
//
// Each thread's next rows are under way while it turns the present ones, its first ones while
// cosines and sines are made: 1.07 GB forward (32768 tokens of 64 heads, bf16) take 198 us, 5.4
// TB/s, 249 us without; 336 MB 67 us; back, 503 MB take 105 to 114 us, 4.4 to 4.8 TB/s, 145
// without.  Float32 of few heads is further off: 76 MB (5331 tokens of 14 heads) take 20.5 us, 3.7
// TB/s, where a thread has one or two rows behind a table of angles in 64 bits.  Back keeps to 168
// registers, three waves to a SIMD (174 as the compiler chose, two waves: 125 us; 128 with spills:
// 196).
//
// The weights' gradients: a thread owns its unit's columns of every row it walks over, a
// workgroup joins its threads' in LDS and stores one partial row per tensor, and a second
// launch adds the partial rows up in order.  Back, a workgroup takes several runs, so that
// at most kNormMostParts partial rows exist.
#include "serve_device.h"
#include "step_kernels.h"

namespace e2s {
namespace {

constexpr int kThreads = 256;

struct NormArgs {
    e2s_rotary_plan plan;
    const int32_t* pos;
    const void* src[2];
    const void* grad[2];
    const void* weight[2];
    void* dst[2];
    float* part;                     // [workgroups, 2, d], or null
    int64_t ss[2][3], gs[2][3], ds[2][3];
    int64_t ps[3];
    int heads[2];
    int T, tiles, TT;                // tokens; runs per sequence; tokens per run
    int units, turning, lpr;         // units of a row, of which turned; lanes of a row
    int64_t runs;                    // B * tiles
    bool weight_f32;
    float eps, inv_d, sign;
};

template <typename T, int W> struct alignas(sizeof(T) * W) NormChunk { T x[W]; };

template <bool STREAM, typename C>
__device__ __forceinline__ C get_chunk(const void* p) {
    if constexpr (STREAM)
        return __builtin_bit_cast(C, __builtin_nontemporal_load(static_cast<const u32x4*>(p)));
    else
        return *static_cast<const C*>(p);
}
template <bool STREAM, typename C>
__device__ __forceinline__ void put_chunk(void* p, const C& c) {
    if constexpr (STREAM)
        __builtin_nontemporal_store(__builtin_bit_cast(u32x4, c), static_cast<u32x4*>(p));
    else
        *static_cast<C*>(p) = c;
}

// The sum over the lpr (4 .. 64) lanes of a row, the same bits in each.
__device__ __forceinline__ float row_sum(float v, int lpr) {
    v += dpp<kQuadSwap1>(v);
    v += dpp<kQuadSwap2>(v);
    if (lpr > 4) v += dpp<kRowHalfMirror>(v);
    if (lpr > 8) v += dpp<kRowMirror>(v);
    if (lpr > 16) v += __shfl_xor(v, 16);
    if (lpr > 32) v += __shfl_xor(v, 32);
    return v;
}

// (x0, x1) -> (x0 c - x1 s, x0 s + x1 c) over the W pairs of a unit's 2 W elements.
template <int W, bool HALF>
__device__ __forceinline__ void turn_unit(float (&v)[2 * W], const f32x2 (&cs)[W]) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
        float& a = v[HALF ? i : 2 * i];
        float& b = v[HALF ? W + i : 2 * i + 1];
        const float p = a, q = b;
        a = p * cs[i].x - q * cs[i].y;
        b = p * cs[i].y + q * cs[i].x;
    }
}

// What a thread knows of a unit: where its chunks are, and which of them exist.
struct Unit {
    int o0, o1;
    bool live, turn, second;
};
template <int W, bool HALF>
__device__ __forceinline__ Unit unit_of(const NormArgs& a, int u) {
    Unit n;
    n.live = u < a.units;
    n.turn = u < a.turning;
    n.second = n.live;
    if (n.turn) {
        n.o0 = HALF ? u * W : 2 * u * W;
        n.o1 = HALF ? n.o0 + a.plan.rot_dim / 2 : n.o0 + W;
    } else {
        n.o0 = a.plan.rot_dim + 2 * (u - a.turning) * W;
        n.o1 = n.o0 + W;
        n.second = n.live && n.o1 < a.plan.head_dim;
    }
    return n;
}

// Cosine and sine of nt tokens' pairs.
__device__ __forceinline__ void fill_table(const NormArgs& a, f32x2* table, int64_t b, int t0,
                                           int nt) {
    const int pairs = a.plan.rot_dim / 2;
    for (int i = threadIdx.x; i < nt * pairs; i += kThreads) {
        const int t = i / pairs, j = i - t * pairs;
        const int32_t p = a.pos[a.plan.axis[j] * a.ps[0] + b * a.ps[1] + (t0 + t) * a.ps[2]];
        double turns = static_cast<double>(p) * a.plan.turns[j];
        turns -= rint(turns);
        float s, c;
        sincospif(static_cast<float>(2.0 * turns), &s, &c);
        table[i] = f32x2{a.plan.amplitude * c, a.sign * a.plan.amplitude * s};
    }
}

template <typename T>
__device__ __forceinline__ float weight_at(const NormArgs& a, int w, int j) {
    if (a.weight[w] == nullptr) return 1.0f;
    if (a.weight_f32) return static_cast<const float*>(a.weight[w])[j];
    return to_f32(static_cast<const T*>(a.weight[w])[j]);
}

template <typename T, int W, int NU, bool STREAM>
struct RowIo {
    using C = NormChunk<T, W>;
    C c0[NU], c1[NU];
    __device__ __forceinline__ void load(const T* row, const Unit (&n)[NU]) {
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            c0[i] = C{};
            c1[i] = C{};
            if (n[i].live) c0[i] = get_chunk<STREAM, C>(row + n[i].o0);
            if (n[i].second) c1[i] = get_chunk<STREAM, C>(row + n[i].o1);
        }
    }
    __device__ __forceinline__ void values(int i, float (&v)[2 * W]) const {
#pragma unroll
        for (int e = 0; e < W; ++e) {
            v[e] = to_f32(c0[i].x[e]);
            v[W + e] = to_f32(c1[i].x[e]);
        }
    }
    static __device__ __forceinline__ void store(T* row, const Unit& n, const float (&v)[2 * W]) {
        C x, y;
#pragma unroll
        for (int e = 0; e < W; ++e) {
            x.x[e] = from_f32<T>(v[e]);
            y.x[e] = from_f32<T>(v[W + e]);
        }
        if (n.live) put_chunk<STREAM>(row + n.o0, x);
        if (n.second) put_chunk<STREAM>(row + n.o1, y);
    }
};

template <int W>
__device__ __forceinline__ void unit_weights(const float* w, const Unit& n, float (&v)[2 * W]) {
#pragma unroll
    for (int e = 0; e < W; ++e) {
        v[e] = n.live ? w[n.o0 + e] : 0.0f;
        v[W + e] = n.second ? w[n.o1 + e] : 0.0f;
    }
}

constexpr int kAtOnce = 2;           // rows of a batch per thread; the next batch is under way

template <typename T, int W, int NU, bool HALF, bool STREAM>
__global__ __launch_bounds__(kThreads) void norm_rotate_kernel(const NormArgs a) {
    __shared__ f32x2 table[kThreads * (W > 2 ? W : 2)];
    alignas(16) __shared__ float weights[2][2 * E2S_ROTARY_MAX_PAIRS];
    const int pairs = a.plan.rot_dim / 2;
    const int64_t b = blockIdx.x / static_cast<uint32_t>(a.tiles);
    const int t0 = static_cast<int>(blockIdx.x - b * a.tiles) * a.TT;
    const int nt = min(a.TT, a.T - t0);
    const int u = threadIdx.x & (a.lpr - 1), rest = threadIdx.x / a.lpr;
    const int t = rest % a.TT, lane = rest / a.TT;
    const int lanes = kThreads / (a.lpr * a.TT);
    const bool some = lane < lanes && t < nt;    // whole rows of lanes
    Unit n[NU];
#pragma unroll
    for (int i = 0; i < NU; ++i) n[i] = unit_of<W, HALF>(a, u + i * a.lpr);
    const int Hq = a.heads[0], H = some ? Hq + a.heads[1] : 0;
    using Rows = RowIo<T, W, NU, STREAM>;
    Rows x[kAtOnce];
    auto load = [&](int h0) {
#pragma unroll
        for (int m = 0; m < kAtOnce; ++m) {
            const int h = h0 + m * lanes;
            if (h >= H) break;
            const int w = h >= Hq;
            x[m].load(static_cast<const T*>(a.src[w]) + b * a.ss[w][0] +
                          (h - (w ? Hq : 0)) * a.ss[w][1] + (t0 + t) * a.ss[w][2], n);
        }
    };
    // The first rows are under way while cosines and sines are made.
    load(lane);
    fill_table(a, table, b, t0, nt);
    for (int i = threadIdx.x; i < 2 * a.plan.head_dim; i += kThreads) {
        const int w = i >= a.plan.head_dim, j = i - w * a.plan.head_dim;
        weights[w][j] = weight_at<T>(a, w, j);
    }
    __syncthreads();
    f32x2 cs[NU][W];
#pragma unroll
    for (int i = 0; i < NU; ++i)
#pragma unroll
        for (int e = 0; e < W; ++e)
            cs[i][e] = some && n[i].turn ? table[t * pairs + (u + i * a.lpr) * W + e]
                                         : f32x2{1.0f, 0.0f};
    for (int h0 = lane; h0 < H; h0 += lanes * kAtOnce) {
        Rows now[kAtOnce];
#pragma unroll
        for (int m = 0; m < kAtOnce; ++m) now[m] = x[m];
        load(h0 + lanes * kAtOnce);
#pragma unroll
        for (int m = 0; m < kAtOnce; ++m) {
            const int h = h0 + m * lanes;
            if (h >= H) break;
            const int w = h >= Hq;
            T* row = static_cast<T*>(a.dst[w]) + b * a.ds[w][0] +
                     (h - (w ? Hq : 0)) * a.ds[w][1] + (t0 + t) * a.ds[w][2];
            float v[NU][2 * W], sq = 0.0f;
#pragma unroll
            for (int i = 0; i < NU; ++i) {
                now[m].values(i, v[i]);
#pragma unroll
                for (int e = 0; e < 2 * W; ++e) sq = __builtin_fmaf(v[i][e], v[i][e], sq);
            }
            sq = row_sum(sq, a.lpr);
            const float r = 1.0f / sqrtf(__builtin_fmaf(sq, a.inv_d, a.eps));
#pragma unroll
            for (int i = 0; i < NU; ++i) {
                float f[2 * W];
                unit_weights<W>(weights[w], n[i], f);
#pragma unroll
                for (int e = 0; e < 2 * W; ++e) v[i][e] = v[i][e] * r * f[e];
                if (n[i].turn) turn_unit<W, HALF>(v[i], cs[i]);
                Rows::store(row, n[i], v[i]);
            }
        }
    }
}

// Back.  One tensor after the other, so that a thread has one set of column sums.
template <typename T, int W, int NU, bool HALF, bool STREAM>
__global__ __launch_bounds__(kThreads, 3) void norm_rotate_back_kernel(const NormArgs a) {
    constexpr int kCols = 2 * W * NU;
    union Shared {
        f32x2 table[kThreads * (W > 2 ? W : 2)];
        float sums[kThreads][kCols + 1];
    };
    __shared__ Shared lds;
    __shared__ float weights[2][2 * E2S_ROTARY_MAX_PAIRS];
    const int pairs = a.plan.rot_dim / 2, D = a.plan.head_dim;
    for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
        const int w = i >= D, j = i - w * D;
        weights[w][j] = weight_at<T>(a, w, j);
    }
    const int u = threadIdx.x & (a.lpr - 1), rest = threadIdx.x / a.lpr;
    const int t = rest % a.TT, lane = rest / a.TT;
    const int lanes = kThreads / (a.lpr * a.TT);
    Unit n[NU];
#pragma unroll
    for (int i = 0; i < NU; ++i) n[i] = unit_of<W, HALF>(a, u + i * a.lpr);
    float sums[2][NU][2 * W];
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int i = 0; i < NU; ++i)
#pragma unroll
            for (int e = 0; e < 2 * W; ++e) sums[w][i][e] = 0.0f;

    using Rows = RowIo<T, W, NU, STREAM>;
    for (int64_t run = blockIdx.x; run < a.runs; run += gridDim.x) {
        const int64_t b = run / a.tiles;
        const int t0 = static_cast<int>(run - b * a.tiles) * a.TT;
        const int nt = min(a.TT, a.T - t0);
        const bool some = lane < lanes && t < nt;
        Rows x, g;
        auto load = [&](int w, int h) {
            if (!some || h >= a.heads[w]) return;
            x.load(static_cast<const T*>(a.src[w]) + b * a.ss[w][0] + (t0 + t) * a.ss[w][2] +
                       h * a.ss[w][1], n);
            g.load(static_cast<const T*>(a.grad[w]) + b * a.gs[w][0] + (t0 + t) * a.gs[w][2] +
                       h * a.gs[w][1], n);
        };
        __syncthreads();                         // the run before has been read
        load(0, lane);                           // under way while cosines and sines are made
        fill_table(a, lds.table, b, t0, nt);
        __syncthreads();
        f32x2 cs[NU][W];
#pragma unroll
        for (int i = 0; i < NU; ++i)
#pragma unroll
            for (int e = 0; e < W; ++e)
                cs[i][e] = some && n[i].turn ? lds.table[t * pairs + (u + i * a.lpr) * W + e]
                                             : f32x2{1.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            T* dst = static_cast<T*>(a.dst[w]) + b * a.ds[w][0] + (t0 + t) * a.ds[w][2];
            if (w == 1) load(1, lane);
            for (int h = lane; some && h < a.heads[w]; h += lanes) {
                float v[NU][2 * W], f[NU][2 * W], sq = 0.0f, dot = 0.0f;
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    x.values(i, v[i]);
                    g.values(i, f[i]);
                }
                load(w, h + lanes);              // the next row
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    float wt[2 * W];
                    unit_weights<W>(weights[w], n[i], wt);
                    if (n[i].turn) turn_unit<W, HALF>(f[i], cs[i]);
#pragma unroll
                    for (int e = 0; e < 2 * W; ++e) {
                        sq = __builtin_fmaf(v[i][e], v[i][e], sq);
                        dot = __builtin_fmaf(f[i][e] * wt[e], v[i][e], dot);
                    }
                }
                sq = row_sum(sq, a.lpr);
                dot = row_sum(dot, a.lpr);
                const float r = 1.0f / sqrtf(__builtin_fmaf(sq, a.inv_d, a.eps));
                const float mean = dot * r * a.inv_d;            // of u x r
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    float wt[2 * W], y[2 * W];
                    unit_weights<W>(weights[w], n[i], wt);
#pragma unroll
                    for (int e = 0; e < 2 * W; ++e) {
                        const float unit = v[i][e] * r;
                        sums[w][i][e] = __builtin_fmaf(f[i][e], unit, sums[w][i][e]);
                        y[e] = r * (f[i][e] * wt[e] - unit * mean);
                    }
                    Rows::store(dst + h * a.ds[w][1], n[i], y);
                }
            }
        }
    }
    if (a.part == nullptr) return;
    // this workgroup's partial rows: its threads' column sums in order
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NU; ++i)
#pragma unroll
            for (int e = 0; e < 2 * W; ++e)
                lds.sums[threadIdx.x][i * 2 * W + e] = sums[w][i][e];
        __syncthreads();
        for (int c = threadIdx.x; c < a.lpr * kCols; c += kThreads) {
            const int uu = c / kCols, col = c - uu * kCols;
            const Unit m = unit_of<W, HALF>(a, uu + col / (2 * W) * a.lpr);
            const int e = col % (2 * W);
            if (!(e < W ? m.live : m.second)) continue;
            float total = 0.0f;
            for (int k = uu; k < kThreads; k += a.lpr) total += lds.sums[k][col];
            a.part[(static_cast<int64_t>(blockIdx.x) * 2 + w) * D +
                   (e < W ? m.o0 + e : m.o1 + e - W)] = total;
        }
    }
}

// The partial rows added up: 16 columns of a tensor to a workgroup, 64 threads to a column.
constexpr int kSumThreads = 1024, kSumCols = 16;
template <typename T>
__global__ __launch_bounds__(kSumThreads) void norm_weights_kernel(const float* part, int parts,
                                                                   int D, T* dq, T* dk) {
    constexpr int kLanes = kSumThreads / kSumCols;
    __shared__ float all[kLanes][kSumCols + 1];
    const int col = threadIdx.x % kSumCols, k = threadIdx.x / kSumCols;
    const int w = blockIdx.y, j = blockIdx.x * kSumCols + col;
    T* out = w ? dk : dq;
    if (out == nullptr) return;
    float total = 0.0f;
    if (j < D) {
        int p = k;
        for (; p + 7 * kLanes < parts; p += 8 * kLanes) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                x[i] = part[(static_cast<int64_t>(p + i * kLanes) * 2 + w) * D + j];
            total += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
        }
        for (; p < parts; p += kLanes) total += part[(static_cast<int64_t>(p) * 2 + w) * D + j];
    }
    all[k][col] = total;
    __syncthreads();
    if (k < 8) {
        total = 0.0f;
#pragma unroll
        for (int i = 0; i < kLanes / 8; ++i) total += all[k + 8 * i][col];
    }
    __syncthreads();
    if (k < 8) all[k][col] = total;
    __syncthreads();
    if (k == 0 && j < D) {
        total = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) total += all[i][col];
        out[j] = from_f32<T>(total);
    }
}

// Elements per chunk: the widest of 16 bytes' worth down to 1 that divides R/2 and d - R and
// that every pointer and stride is aligned to.
int norm_chunk(const NormArgs& a, int64_t B, int eb) {
    for (int w = 16 / eb; w > 1; w /= 2) {
        if ((a.plan.rot_dim / 2) % w != 0 || (a.plan.head_dim - a.plan.rot_dim) % w != 0) continue;
        bool fits = true;
        for (int i = 0; i < 2; ++i) {
            if (a.heads[i] == 0) continue;
            for (const void* p : {a.src[i], a.grad[i], static_cast<const void*>(a.dst[i])})
                fits = fits && reinterpret_cast<uintptr_t>(p) % (w * eb) == 0;
            const int64_t counts[3] = {B, a.heads[i], a.T};
            for (int k = 0; k < 3; ++k)          // (a stride that only index 0 takes: any)
                fits = fits && (counts[k] == 1 || (a.ss[i][k] % w == 0 && a.gs[i][k] % w == 0 &&
                                                   a.ds[i][k] % w == 0));
        }
        if (fits) return w;
    }
    return 1;
}

template <typename T, int W, bool HALF, bool STREAM>
void launch_h(const NormArgs& a, bool back, unsigned groups, hipStream_t st) {
    constexpr int NU = W == 1 ? 2 : 1;           // up to 128 units, 64 lanes
    if (back)
        hipLaunchKernelGGL((norm_rotate_back_kernel<T, W, NU, HALF, STREAM>), dim3(groups),
                           dim3(kThreads), 0, st, a);
    else
        hipLaunchKernelGGL((norm_rotate_kernel<T, W, NU, HALF, STREAM>), dim3(groups),
                           dim3(kThreads), 0, st, a);
}

template <typename T, int W>
hipError_t launch_w(NormArgs& a, int64_t B, bool back, void* dq, void* dk, hipStream_t st) {
    a.turning = a.plan.rot_dim / 2 / W;
    a.units = a.turning + (a.plan.head_dim - a.plan.rot_dim + 2 * W - 1) / (2 * W);
    a.lpr = 4;
    while (a.lpr < 64 && a.lpr < a.units) a.lpr *= 2;
    // Tokens per workgroup: as in the rotation, as many as its threads hold one unit each of,
    // but no fewer than 2048 workgroups where the tokens allow it.
    const int64_t most = kThreads / a.lpr;
    a.TT = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(most, B * a.T / 2048)));
    a.tiles = (a.T + a.TT - 1) / a.TT;
    a.runs = B * a.tiles;
    const unsigned groups =
        static_cast<unsigned>(back ? std::min<int64_t>(a.runs, kNormMostParts) : a.runs);
    const bool half = a.plan.layout == E2S_ROTARY_HALF;
    // What does not fit the last-level cache passes it by, as in the rotation.
    const double moved = (back ? 3.0 : 2.0) * B * a.T * (a.heads[0] + a.heads[1]) *
                         a.plan.head_dim * sizeof(T);
    if (sizeof(T) * W == 16 && moved > 268435456.0) {
        if (half) launch_h<T, W, true, sizeof(T) * W == 16>(a, back, groups, st);
        else launch_h<T, W, false, sizeof(T) * W == 16>(a, back, groups, st);
    } else {
        if (half) launch_h<T, W, true, false>(a, back, groups, st);
        else launch_h<T, W, false, false>(a, back, groups, st);
    }
    if (a.part != nullptr) {
        const dim3 grid((a.plan.head_dim + kSumCols - 1) / kSumCols, 2);
        if (a.weight_f32)
            hipLaunchKernelGGL((norm_weights_kernel<float>), grid, dim3(kSumThreads), 0, st, a.part,
                               static_cast<int>(groups), a.plan.head_dim, static_cast<float*>(dq),
                               static_cast<float*>(dk));
        else
            hipLaunchKernelGGL((norm_weights_kernel<T>), grid, dim3(kSumThreads), 0, st, a.part,
                               static_cast<int>(groups), a.plan.head_dim, static_cast<T*>(dq),
                               static_cast<T*>(dk));
    }
    return hipGetLastError();
}

template <typename T, int MAX>
hipError_t launch_t(NormArgs& a, int w, int64_t B, bool back, void* dq, void* dk,
                    hipStream_t st) {
    if constexpr (MAX == 8)
        if (w == 8) return launch_w<T, 8>(a, B, back, dq, dk, st);
    if (w >= 4) return launch_w<T, 4>(a, B, back, dq, dk, st);
    if (w == 2) return launch_w<T, 2>(a, B, back, dq, dk, st);
    return launch_w<T, 1>(a, B, back, dq, dk, st);
}

__global__ void zero_weights_kernel(uint8_t* dq, uint8_t* dk, int bytes) {
    uint8_t* out = blockIdx.x ? dk : dq;
    for (int i = threadIdx.x; out != nullptr && i < bytes; i += blockDim.x) out[i] = 0;
}

}  // namespace

hipError_t launch_norm_rotate(const e2s_norm_rotate_shape& s, const e2s_rotary_plan& p,
                              const int32_t* positions, const void* const (&src)[2],
                              const void* const (&weight)[2], const void* const (&grad)[2],
                              void* const (&dst)[2], void* const (&weight_grad)[2],
                              void* workspace, bool back, hipStream_t st) {
    const bool want = back && (weight_grad[0] != nullptr || weight_grad[1] != nullptr);
    if (s.num_tokens == 0) {
        if (!want) return hipSuccess;
        hipLaunchKernelGGL(zero_weights_kernel, dim3(2), dim3(256), 0, st,
                           static_cast<uint8_t*>(weight_grad[0]),
                           static_cast<uint8_t*>(weight_grad[1]),
                           p.head_dim * elem_bytes(s.weight_dtype));
        return hipGetLastError();
    }
    NormArgs a{};
    a.plan = p;
    a.pos = positions;
    a.heads[0] = s.q_heads;
    a.heads[1] = s.k_heads;
    for (int w = 0; w < 2; ++w) {
        const bool there = a.heads[w] > 0;
        a.src[w] = there ? src[w] : nullptr;
        a.grad[w] = there ? grad[w] : nullptr;
        a.dst[w] = there ? dst[w] : nullptr;
        a.weight[w] = weight[w];
    }
    for (int i = 0; i < 3; ++i) {
        a.ss[0][i] = s.q_stride[i];
        a.ss[1][i] = s.k_stride[i];
        a.gs[0][i] = back ? s.q_grad_stride[i] : 0;
        a.gs[1][i] = back ? s.k_grad_stride[i] : 0;
        a.ds[0][i] = s.q_out_stride[i];
        a.ds[1][i] = s.k_out_stride[i];
        a.ps[i] = s.pos_stride[i];
    }
    a.T = s.num_tokens;
    a.weight_f32 = s.weight_dtype == E2S_DTYPE_F32;
    a.eps = s.eps;
    a.inv_d = 1.0f / static_cast<float>(p.head_dim);
    a.sign = back ? -1.0f : 1.0f;
    a.part = want ? static_cast<float*>(workspace) : nullptr;
    const int w = norm_chunk(a, s.batch, elem_bytes(s.dtype));
    void *dq = weight_grad[0], *dk = weight_grad[1];
    if (s.dtype == E2S_DTYPE_F32) return launch_t<float, 4>(a, w, s.batch, back, dq, dk, st);
    if (s.dtype == E2S_DTYPE_F16) return launch_t<_Float16, 8>(a, w, s.batch, back, dq, dk, st);
    return launch_t<uint16_t, 8>(a, w, s.batch, back, dq, dk, st);
}

}  // namespace e2s
