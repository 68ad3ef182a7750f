// Eviction by accumulated attention weight (e2s_cache_evict), in two launches.
//
// evict_select_kernel, one workgroup per (sequence, key head): the tokens between the
// first `sinks` and the last `recent` are ranked by a 32-bit key that orders floats as
// integers (larger weight, larger key; NaN lowest), and the want-th largest key is found
// digit by digit (11, 11 and 10 bits) from a histogram in LDS, until all tokens that share
// the digits found so far stay.  Tokens above it stay, and
// of those equal to it the first ones; counts per wave and a scan over the waves place the
// kept tokens in ascending order.  All decisions are on integers, so nothing depends on
// the order of the atomic increments.  Latency bounds it: a thread loads its keys (up to 16)
// at once and keeps them in registers for all passes where the sequences fit one segment of
// 1024 x 16 tokens (256 of up to 16000 tokens: 18.7 us, 32 when every pass read them); longer
// ones are read again, a segment at a time, in every pass.  One histogram is enough: 4, 8 or
// 16 copies for neighbouring lanes took 21.8, 23.2 and 27.7 us where one took 21.7.
//
// evict_move_kernel, one workgroup per (sequence, key head, new block), keys and values
// together (they share the lookups of indices and pages): gathers the block's kept rows,
// takes their largest magnitude to the block's scale, and writes them rescaled by the ratio
// of two powers of two.  It moves each kept byte once, and the copy rate bounds it: 280 MB
// read and written, a row of 128 bytes here and there, take 47 to 56 us, 5.0 to 6.0 TB/s
// (one block of keys or of values per workgroup: 63).
#include "serve_device.h"
#include "serve_kernels.h"

namespace e2s {
namespace {

constexpr int kBins = 2048;

// Maxima of held values are compared 2^-16 of their size: float32 has the largest, 2^128, and
// the smallest, 2^-109, so (exact products of 4 bits and a power of two).
constexpr int kDownBits = 16;
constexpr float kDown = 1.0f / (1 << kDownBits);

struct EvictArgs {
    const int32_t* pages;
    const int32_t* lengths;
    const float* weights;
    const int32_t* new_pages;
    int32_t* keep;
    int32_t* new_len;
    float* left;                     // or null
    const uint8_t* src[2];
    uint8_t* dst[2];
    float* scale[2];
    int64_t page_stride[2];
    int64_t pages_stride, new_pages_stride;
    int64_t ws[2], ls[2];
    int G, P, page_shift, K, W, sinks, recent, max_tokens, max_pages, num_pages, blocks;
};

__device__ __forceinline__ int evict_length(const EvictArgs& a, int64_t b) {
    const int64_t cap = min(static_cast<int64_t>(a.max_pages) * a.P,
                            static_cast<int64_t>(a.max_tokens));
    return static_cast<int>(min(static_cast<int64_t>(max(a.lengths[b], 0)), cap));
}

// Larger weight, larger key; -0 as 0; NaN below everything.
__device__ __forceinline__ uint32_t rank_key(float w) {
    return w != w ? 0u : ordered_bits(w + 0.0f);
}

// How many of the lanes before this one a ballot names.
__device__ __forceinline__ uint32_t lanes_below(uint64_t ballot) {
    return __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(ballot >> 32),
                                     __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(ballot), 0u));
}

template <int THREADS, int PER>          // PER tokens per thread and segment
__global__ __launch_bounds__(THREADS) void evict_select_kernel(const EvictArgs a) {
    constexpr int kSelWaves = THREADS / kWave;
    constexpr int kOwn = kBins / THREADS;        // bins of a thread
    __shared__ uint32_t hist[kBins];
    __shared__ uint32_t sums[kSelWaves];
    __shared__ uint32_t ties[kSelWaves];
    __shared__ uint32_t found[3];             // digit, still wanted, of how many
    constexpr int kSegment = THREADS * PER;
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int64_t b = blockIdx.x / a.G;
    const int g = static_cast<int>(blockIdx.x - b * a.G);
    const int n = evict_length(a, b);
    const int kept = min(n, a.K);
    const float* w = a.weights + b * a.ws[0] + g * a.ws[1];
    int32_t* keep = a.keep + (b * a.G + g) * static_cast<int64_t>(a.K);
    float* left = a.left ? a.left + b * a.ls[0] + g * a.ls[1] : nullptr;
    if (g == 0 && tid == 0) a.new_len[b] = kept;
    for (int j = kept + tid; j < a.K; j += THREADS) keep[j] = -1;
    if (left)
        for (int j = kept + tid; j < a.W; j += THREADS) left[j] = 0.0f;
    if (n <= a.K) {
        for (int j = tid; j < n; j += THREADS) {
            keep[j] = j;
            if (left) left[j] = w[j];
        }
        return;
    }
    // sinks + recent <= K < n: the ends do not meet, and m0 < m1
    const int m0 = a.sinks, m1 = n - a.recent;
    // A wave holds PER runs of 64 neighbouring tokens of a segment, one after the other.
    float x[PER];
    uint32_t key[PER];
    auto token = [&](int seg, int j) { return seg + (wave * PER + j) * kWave + lane; };
    auto load = [&](int seg) {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int i = token(seg, j);
            x[j] = i < n ? w[i] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < PER; ++j) key[j] = rank_key(x[j]);
    };
    const uint32_t between = static_cast<uint32_t>(m1 - m0);
    auto ranked = [&](int i) { return static_cast<uint32_t>(i - m0) < between; };
    const bool once = n <= kSegment;
    if (once) load(0);
    uint32_t want = static_cast<uint32_t>(a.K - a.sinks - a.recent);
    // keys above `limit` stay, and of the keys equal to it the first `want`
    uint32_t limit = 0xFFFFFFFFu;
    if (want > 0) {
        limit = 0;
        uint32_t known = 0;                            // mask of the digits found
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            const uint32_t mask = pass == 2 ? 1023u : 2047u;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) hist[tid + i * THREADS] = 0;
            __syncthreads();
            for (int seg = 0; seg < n; seg += kSegment) {
                if (!once) load(seg);
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    if (ranked(token(seg, j)) && (key[j] & known) == limit)
                        atomicAdd(&hist[(key[j] >> shift) & mask], 1u);
                }
            }
            __syncthreads();
            // thread t owns the kOwn bins below 2048 - kOwn t: sums from the top
            uint32_t own[kOwn], all = 0;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                own[i] = hist[kBins - 1 - kOwn * tid - i];
                all += own[i];
            }
            uint32_t run = all;
            for (int o = 1; o < kWave; o <<= 1) {
                const uint32_t v = __shfl_up(run, o);
                if (lane >= o) run += v;
            }
            if (lane == kWave - 1) sums[wave] = run;
            __syncthreads();
            uint32_t above = run - all;
#pragma unroll
            for (int v = 0; v < kSelWaves; ++v) above += v < wave ? sums[v] : 0u;
            // the digit at which the count from the top reaches `want`
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                if (above < want && above + own[i] >= want) {
                    found[0] = static_cast<uint32_t>(kBins - 1 - kOwn * tid - i);
                    found[1] = want - above;
                    found[2] = own[i];
                }
                above += own[i];
            }
            __syncthreads();
            limit |= found[0] << shift;
            want = found[1];
            known |= mask << shift;
            if (found[2] == want && limit > 0) {       // all that share the digits stay
                --limit;
                want = 0;
                break;
            }
        }
    }
    // Per segment: every wave counts its tokens that stay and its ties, then places them.
    uint32_t more = 0, same = 0;                       // of the segments before
    for (int seg = 0; seg < n; seg += kSegment) {
        if (!once) load(seg);
        bool up[PER], equal[PER];
        uint32_t up_here = 0, tie_here = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int i = token(seg, j);
            const bool inner = ranked(i);
            up[j] = i < n && (!inner || key[j] > limit);
            equal[j] = inner && key[j] == limit;
            up_here += __popcll(__ballot(up[j]));
            tie_here += __popcll(__ballot(equal[j]));
        }
        __syncthreads();                               // sums and ties are free
        if (lane == 0) {
            sums[wave] = up_here;
            ties[wave] = tie_here;
        }
        __syncthreads();
        uint32_t before = same, slot0 = more;
#pragma unroll
        for (int v = 0; v < kSelWaves; ++v) {
            slot0 += v < wave ? sums[v] : 0u;
            before += v < wave ? ties[v] : 0u;
            more += sums[v];
            same += ties[v];
        }
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const uint64_t ups = __ballot(up[j]), ties_here = __ballot(equal[j]);
            const uint32_t tie = before + lanes_below(ties_here);
            if (up[j] || (equal[j] && tie < want)) {   // K tokens in all, so slot < K
                const uint32_t slot = slot0 + lanes_below(ups) + min(tie, want);
                keep[slot] = token(seg, j);
                if (left) left[slot] = x[j];
            }
            slot0 += __popcll(ups);
            before += __popcll(ties_here);
        }
    }
}

// PACKETS packets of 16 bytes per thread cover a block of keys, and as many its values.
template <int D, int THREADS, int PACKETS>
__global__ __launch_bounds__(THREADS) void evict_move_kernel(const EvictArgs a) {
    constexpr int kLanes = D / 16;
    __shared__ float shared[2][THREADS / kWave];
    const uint32_t unit = blockIdx.x;
    const int g = static_cast<int>(unit % static_cast<uint32_t>(a.G));
    const uint32_t ub = unit / static_cast<uint32_t>(a.G);
    const int64_t b = ub / static_cast<uint32_t>(a.blocks);
    const int blk = static_cast<int>(ub % static_cast<uint32_t>(a.blocks));
    const int kept = min(evict_length(a, b), a.K);
    const int first = blk << a.page_shift;
    if (first >= kept) return;
    const int page = a.new_pages[b * a.new_pages_stride + blk];
    if (page < 0 || page >= a.num_pages) return;
    const int rows = min(kept - first, a.P);
    const int32_t* keep = a.keep + (b * a.G + g) * static_cast<int64_t>(a.K) + first;
    const int64_t head = static_cast<int64_t>(g) * (D << a.page_shift);

    u32x4 x[PACKETS][2];
    float from[PACKETS][2];
    int idx[PACKETS], src[PACKETS];
#pragma unroll
    for (int p = 0; p < PACKETS; ++p) {
        const int r = (p * THREADS + static_cast<int>(threadIdx.x)) / kLanes;
        idx[p] = r < rows ? keep[r] : -1;           // < length <= max_pages * P
    }
#pragma unroll
    for (int p = 0; p < PACKETS; ++p) {
        src[p] = idx[p] >= 0 ? a.pages[b * a.pages_stride + (idx[p] >> a.page_shift)] : -1;
        if (src[p] >= a.num_pages) src[p] = -1;
    }
#pragma unroll
    for (int p = 0; p < PACKETS; ++p)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            x[p][k] = u32x4{0u, 0u, 0u, 0u};
            from[p][k] = 1.0f;
            if (src[p] < 0) continue;
            from[p][k] = a.scale[k][static_cast<int64_t>(src[p]) * a.G + g];
            const int row = idx[p] & (a.P - 1);
            const int c = static_cast<int>(threadIdx.x) % kLanes;
            x[p][k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(
                a.src[k] + src[p] * a.page_stride[k] + head + row * D + c * 16));
        }
    float to[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float top = 0.0f;
#pragma unroll
        for (int p = 0; p < PACKETS; ++p) {
            const uint32_t word[4] = {x[p][k].x, x[p][k].y, x[p][k].z, x[p][k].w};
            float most = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v[4];
                from_e4m3(word[i], v);
#pragma unroll
                for (int e = 0; e < 4; ++e) most = fmaxf(most, fabsf(v[e]));   // skips NaN
            }
            top = fmaxf(top, most * (from[p][k] * kDown));
        }
        top = wave_max(top);
        if ((threadIdx.x & (kWave - 1)) == 0) shared[k][threadIdx.x / kWave] = top;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float top = shared[k][0];
#pragma unroll
        for (int v = 1; v < THREADS / kWave; ++v) top = fmaxf(top, shared[k][v]);
        to[k] = block_scale<kDownBits>(top);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        uint8_t* out = a.dst[k] + page * a.page_stride[k] + head;
#pragma unroll
        for (int p = 0; p < PACKETS; ++p) {
            const int i = p * THREADS + static_cast<int>(threadIdx.x);
            if (i / kLanes >= rows) continue;
            u32x4 w = x[p][k];
            if (from[p][k] != to[k]) {
                const float ratio = scale_ratio(from[p][k], to[k]);
                w.x = rescale_e4m3(w.x, ratio);
                w.y = rescale_e4m3(w.y, ratio);
                w.z = rescale_e4m3(w.z, ratio);
                w.w = rescale_e4m3(w.w, ratio);
            }
            *(reinterpret_cast<u32x4*>(out) + i) = w;
        }
    }
    if (threadIdx.x == 0) {
        const int64_t at = static_cast<int64_t>(page) * a.G + g;
        a.scale[0][at] = to[0];
        a.scale[1][at] = to[1];
    }
}

template <int D, int THREADS, int PACKETS>
void launch_move_k(const EvictArgs& a, int64_t B, hipStream_t st) {
    hipLaunchKernelGGL((evict_move_kernel<D, THREADS, PACKETS>),
                       dim3(static_cast<unsigned>(B * a.blocks * a.G)), dim3(THREADS), 0, st,
                       a);
}

template <int D>
void launch_move(const EvictArgs& a, int64_t B, hipStream_t st) {
    const int packets = a.P * (D / 16);             // 64 .. 1024
    if (packets <= 64) launch_move_k<D, 64, 1>(a, B, st);
    else if (packets <= 256) launch_move_k<D, 256, 1>(a, B, st);
    else if (packets <= 512) launch_move_k<D, 256, 2>(a, B, st);
    else launch_move_k<D, 256, 4>(a, B, st);
}

}  // namespace

hipError_t launch_cache_evict(const e2s_cache& c, const e2s_cache_evict_shape& s,
                              const int32_t* pages, const int32_t* lengths, const float* weights,
                              const int32_t* new_pages, int32_t* keep_idx, int32_t* new_len,
                              float* left, hipStream_t st) {
    EvictArgs a{};
    a.pages = pages;
    a.lengths = lengths;
    a.weights = weights;
    a.new_pages = new_pages;
    a.keep = keep_idx;
    a.new_len = new_len;
    a.left = left;
    a.src[0] = a.dst[0] = static_cast<uint8_t*>(c.k);
    a.src[1] = a.dst[1] = static_cast<uint8_t*>(c.v);
    a.scale[0] = c.k_scale;
    a.scale[1] = c.v_scale;
    a.page_stride[0] = c.k_page_stride;
    a.page_stride[1] = c.v_page_stride;
    a.pages_stride = s.pages_stride;
    a.new_pages_stride = s.new_pages_stride;
    for (int i = 0; i < 2; ++i) {
        a.ws[i] = s.weights_stride[i];
        a.ls[i] = s.left_stride[i];
    }
    a.G = c.num_kv_heads;
    a.P = c.page_tokens;
    a.page_shift = __builtin_ctz(static_cast<unsigned>(c.page_tokens));   // a power of two
    a.K = s.budget;
    a.W = s.left_tokens;
    a.sinks = s.sinks;
    a.recent = s.recent;
    a.max_tokens = s.max_tokens;
    a.max_pages = s.max_pages;
    a.num_pages = c.num_pages;
    a.blocks = (s.budget + c.page_tokens - 1) / c.page_tokens;
    const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(s.batch) * a.G));
    // Small workgroups have short barriers and more of them fit a compute unit; all of a
    // sequence's keys have to fit their registers.  640 tokens: 9.4 us for the call, 11.0 with
    // 1024 threads; 64 sequences and 32 heads of 105 tokens 16 and 44, of 4000 tokens 122 with
    // 512 threads, 119 with 256 x 16 keys and 153 with 1024; one of 4000 tokens 11.3, 12.9, 13.0.
    if (s.max_tokens <= 1024)
        hipLaunchKernelGGL((evict_select_kernel<256, 4>), grid, dim3(256), 0, st, a);
    else if (s.max_tokens <= 4096)
        hipLaunchKernelGGL((evict_select_kernel<512, 8>), grid, dim3(512), 0, st, a);
    else
        hipLaunchKernelGGL((evict_select_kernel<1024, 16>), grid, dim3(1024), 0, st, a);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    if (c.head_dim == 64) launch_move<64>(a, s.batch, st);
    else launch_move<128>(a, s.batch, st);
    return hipGetLastError();
}

}  // namespace e2s
