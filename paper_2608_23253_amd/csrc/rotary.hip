// Rotary positions (e2s_rotate_positions): pair j of a row's first R elements turned by
// p * f_j.
//
// A stream: every element is read and written once, with 3 operations, so the copy rate
// bounds it: 1.07 GB of bf16 take 205 us, 5.2 TB/s (a copy of as much 4.95), 76 MB of float32
// 14.5 us, most of them from the last-level cache; one token's heads 3.6 us.  Sine and cosine depend on the token and the pair alone, not on the head, so
// a workgroup takes a run of TT tokens of one sequence for all heads of q and k: its
// threads first compute the TT * R/2 pairs (cos, sin) into LDS - the angle as turns,
// p * f_j / (2 pi), in float64, of which only the fraction matters, rounded to float32 (at most
// pi 2^-25 of an angle within half a turn; float32 rows are 4.7e-8 off on the whole, 3.6e-8 with
// sine and cosine of float64 angles) - and then each keeps
// its pairs' values in registers while it walks over the heads.
//
// A unit is two chunks of W elements of a row: the first and second members of W pairs
// (half layout), W pairs in order (interleaved), or 2W elements to copy behind R.  W is the
// widest of 16 bytes' worth of elements down to 1 that divides R/2 and d - R and that every
// pointer and stride is aligned to.
#include "serve_device.h"
#include "serve_kernels.h"

namespace e2s {
namespace {

constexpr int kThreads = 256;
constexpr int kHeadsAtOnce = 4;      // heads in flight per thread

struct RotateArgs {
    e2s_rotary_plan plan;
    const int32_t* pos;
    const void* src[2];
    void* dst[2];
    int64_t ss[2][3], ds[2][3];      // sequence, head, token, in elements
    int64_t ps[3];
    int T, Hq, H;                    // tokens, heads of q, heads of q and k
    int tiles, TT;                   // token runs per sequence, tokens per run
    int units, turning;              // units of a row, of which turned
    float sign;
};

template <typename T, int W> struct alignas(sizeof(T) * W) Chunk { T x[W]; };

// STREAM (16-byte chunks): past the caches.
template <bool STREAM, typename C>
__device__ __forceinline__ C load_chunk(const void* p) {
    if constexpr (STREAM)
        return __builtin_bit_cast(C, __builtin_nontemporal_load(static_cast<const u32x4*>(p)));
    else
        return *static_cast<const C*>(p);
}
template <bool STREAM, typename C>
__device__ __forceinline__ void store_chunk(void* p, const C& c) {
    if constexpr (STREAM)
        __builtin_nontemporal_store(__builtin_bit_cast(u32x4, c), static_cast<u32x4*>(p));
    else
        *static_cast<C*>(p) = c;
}

template <typename T, int W, bool HALF, bool STREAM>
__global__ __launch_bounds__(kThreads) void rotate_kernel(const RotateArgs a) {
    __shared__ f32x2 table[kThreads * 8];     // TT * R/2 <= (256 / units) * 8 * units
    const int pairs = a.plan.rot_dim / 2;
    const int64_t b = blockIdx.x / a.tiles;
    const int t0 = static_cast<int>(blockIdx.x - b * a.tiles) * a.TT;
    const int nt = min(a.TT, a.T - t0);
    for (int i = threadIdx.x; i < nt * pairs; i += kThreads) {
        const int t = i / pairs, j = i - t * pairs;
        const int32_t p = a.pos[a.plan.axis[j] * a.ps[0] + b * a.ps[1] + (t0 + t) * a.ps[2]];
        double turns = static_cast<double>(p) * a.plan.turns[j];
        turns -= rint(turns);
        float s, c;
        sincospif(static_cast<float>(2.0 * turns), &s, &c);
        f32x2 v = {a.plan.amplitude * c, a.sign * a.plan.amplitude * s};
        table[i] = v;
    }
    __syncthreads();
    const int u = threadIdx.x % a.units;
    const int rest = threadIdx.x / a.units;
    const int t = rest % a.TT, lane = rest / a.TT;
    const int lanes = kThreads / (a.units * a.TT);
    if (lane >= lanes || t >= nt) return;

    const bool turn = u < a.turning;
    f32x2 cs[W];
    int o0, o1;                       // element offsets of the unit's chunks
    bool second = true;
    if (turn) {
        o0 = HALF ? u * W : 2 * u * W;
        o1 = HALF ? o0 + pairs : o0 + W;
#pragma unroll
        for (int i = 0; i < W; ++i) cs[i] = table[t * pairs + u * W + i];
    } else {
        o0 = a.plan.rot_dim + 2 * (u - a.turning) * W;
        o1 = o0 + W;
        second = o1 < a.plan.head_dim;
    }
    using C = Chunk<T, W>;
    for (int h0 = lane; h0 < a.H; h0 += lanes * kHeadsAtOnce) {
        C x0[kHeadsAtOnce], x1[kHeadsAtOnce];
#pragma unroll
        for (int n = 0; n < kHeadsAtOnce; ++n) {
            const int h = h0 + n * lanes;
            if (h >= a.H) break;
            const int w = h >= a.Hq;
            const T* row = static_cast<const T*>(a.src[w]) + b * a.ss[w][0] +
                           (h - (w ? a.Hq : 0)) * a.ss[w][1] + (t0 + t) * a.ss[w][2];
            x0[n] = load_chunk<STREAM, C>(row + o0);
            if (second) x1[n] = load_chunk<STREAM, C>(row + o1);
        }
#pragma unroll
        for (int n = 0; n < kHeadsAtOnce; ++n) {
            const int h = h0 + n * lanes;
            if (h >= a.H) break;
            const int w = h >= a.Hq;
            T* row = static_cast<T*>(a.dst[w]) + b * a.ds[w][0] +
                     (h - (w ? a.Hq : 0)) * a.ds[w][1] + (t0 + t) * a.ds[w][2];
            C y0 = x0[n], y1 = x1[n];
            if (turn) {
                if constexpr (HALF) {
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        const float p = to_f32(x0[n].x[i]), q = to_f32(x1[n].x[i]);
                        y0.x[i] = from_f32<T>(p * cs[i].x - q * cs[i].y);
                        y1.x[i] = from_f32<T>(p * cs[i].y + q * cs[i].x);
                    }
                } else {
                    // pair i: elements 2i and 2i + 1 of the two chunks in a row
                    T in[2 * W], out[2 * W];
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        in[i] = x0[n].x[i];
                        in[W + i] = x1[n].x[i];
                    }
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        const float p = to_f32(in[2 * i]), q = to_f32(in[2 * i + 1]);
                        out[2 * i] = from_f32<T>(p * cs[i].x - q * cs[i].y);
                        out[2 * i + 1] = from_f32<T>(p * cs[i].y + q * cs[i].x);
                    }
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        y0.x[i] = out[i];
                        y1.x[i] = out[W + i];
                    }
                }
            }
            store_chunk<STREAM>(row + o0, y0);
            if (second) store_chunk<STREAM>(row + o1, y1);
        }
    }
}

// Elements per chunk: see the head of this file.
int chunk_width(const RotateArgs& a, int eb) {
    for (int w = 16 / eb; w > 1; w /= 2) {
        if ((a.plan.rot_dim / 2) % w != 0 || (a.plan.head_dim - a.plan.rot_dim) % w != 0) continue;
        bool fits = true;
        for (int i = 0; i < 2; ++i) {
            if (a.src[i] == nullptr) continue;
            fits = fits && reinterpret_cast<uintptr_t>(a.src[i]) % (w * eb) == 0 &&
                   reinterpret_cast<uintptr_t>(a.dst[i]) % (w * eb) == 0;
            for (int k = 0; k < 3; ++k) fits = fits && a.ss[i][k] % w == 0 && a.ds[i][k] % w == 0;
        }
        if (fits) return w;
    }
    return 1;
}

template <typename T, int W, bool HALF, bool STREAM>
void launch_k(const RotateArgs& a, dim3 grid, hipStream_t st) {
    hipLaunchKernelGGL((rotate_kernel<T, W, HALF, STREAM>), grid, dim3(kThreads), 0, st, a);
}

template <typename T, int W>
hipError_t launch_w(RotateArgs& a, int64_t B, hipStream_t st) {
    a.turning = a.plan.rot_dim / 2 / W;
    a.units = a.turning + (a.plan.head_dim - a.plan.rot_dim + 2 * W - 1) / (2 * W);
    // Tokens per workgroup: as many as its threads hold one unit each of, but fewer where
    // that would leave fewer than 2048 workgroups (8 per compute unit): then the threads
    // share the heads instead.  4096 tokens of 32 heads take 14.2 us so, 15.8 for 512
    // workgroups, 15.3 for 8192; 16384 tokens 48, 57 and 45.
    const int64_t most = kThreads / a.units;
    a.TT = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(most, B * a.T / 2048)));
    a.tiles = (a.T + a.TT - 1) / a.TT;
    const dim3 grid(static_cast<unsigned>(B * a.tiles));
    // What does not fit the 256 MiB last-level cache passes it by: 1 GB of reads and writes
    // take 209 us so and 224 us through the caches, 76 MB 21 us and 15 us.
    const double moved = 2.0 * B * a.T * a.H * a.plan.head_dim * sizeof(T);
    const bool half = a.plan.layout == E2S_ROTARY_HALF;
    if (sizeof(T) * W == 16 && moved > 268435456.0) {
        if (half) launch_k<T, W, true, sizeof(T) * W == 16>(a, grid, st);
        else launch_k<T, W, false, sizeof(T) * W == 16>(a, grid, st);
    } else {
        if (half) launch_k<T, W, true, false>(a, grid, st);
        else launch_k<T, W, false, false>(a, grid, st);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const e2s_rotary_shape& s, const e2s_rotary_plan& p,
                         const int32_t* positions, const void* q, const void* k, void* q_out,
                         void* k_out, hipStream_t st) {
    RotateArgs a{};
    a.plan = p;
    a.pos = positions;
    a.src[0] = s.q_heads > 0 ? q : nullptr;
    a.src[1] = s.k_heads > 0 ? k : nullptr;
    a.dst[0] = q_out;
    a.dst[1] = k_out;
    for (int i = 0; i < 3; ++i) {
        a.ss[0][i] = s.q_stride[i];
        a.ss[1][i] = s.k_stride[i];
        a.ds[0][i] = s.q_out_stride[i];
        a.ds[1][i] = s.k_out_stride[i];
        a.ps[i] = s.pos_stride[i];
    }
    a.T = s.num_tokens;
    a.Hq = s.q_heads;
    a.H = s.q_heads + s.k_heads;
    a.sign = s.inverse ? -1.0f : 1.0f;
    const int w = chunk_width(a, elem_bytes(s.dtype));
    const int64_t B = s.batch;
    if (s.dtype == E2S_DTYPE_F32) {
        if (w == 4) return launch_w<float, 4>(a, B, st);
        if (w == 2) return launch_w<float, 2>(a, B, st);
        return launch_w<float, 1>(a, B, st);
    }
    if (s.dtype == E2S_DTYPE_F16) {
        if (w == 8) return launch_w<_Float16, 8>(a, B, st);
        if (w == 4) return launch_w<_Float16, 4>(a, B, st);
        if (w == 2) return launch_w<_Float16, 2>(a, B, st);
        return launch_w<_Float16, 1>(a, B, st);
    }
    if (w == 8) return launch_w<uint16_t, 8>(a, B, st);
    if (w == 4) return launch_w<uint16_t, 4>(a, B, st);
    if (w == 2) return launch_w<uint16_t, 2>(a, B, st);
    return launch_w<uint16_t, 1>(a, B, st);
}

}  // namespace e2s
