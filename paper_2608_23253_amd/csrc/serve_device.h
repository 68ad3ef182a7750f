// Device helpers of the operators of e2s_serve.h.
#pragma once

#include "e2s_device.h"

namespace e2s {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2s __attribute__((ext_vector_type(2)));

// Element types as in e2s_device.h: uint16_t holds bfloat16 bits.
__device__ __forceinline__ float to_f32(uint16_t x) {
    return __uint_as_float(static_cast<uint32_t>(x) << 16);
}
__device__ __forceinline__ float to_f32(_Float16 x) { return static_cast<float>(x); }
__device__ __forceinline__ float to_f32(float x) { return x; }

template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ uint16_t from_f32<uint16_t>(float x) {
    return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
}
template <> __device__ __forceinline__ _Float16 from_f32<_Float16>(float x) {
    return static_cast<_Float16>(x);
}
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }

// ---------------------------------------------------------------------------
// The cache's e4m3 bytes and their power-of-two scales.
// ---------------------------------------------------------------------------
constexpr int kLowestScale = -100;      // exponent of the smallest scale

// The smallest 2^e, e >= kLowestScale, with amax * 2^SHIFT <= 448 * 2^e.  amax = f * 2^x with
// f in [1/2, 1), and 448 = 0.875 * 2^9.
template <int SHIFT = 0>
__device__ __forceinline__ float block_scale(float amax) {
    const int x = __builtin_amdgcn_frexp_expf(amax) + SHIFT;
    const float f = __builtin_amdgcn_frexp_mantf(amax);
    int e = f <= 0.875f ? x - 9 : x - 8;
    if (amax == 0.0f || e < kLowestScale) e = kLowestScale;
    return __builtin_ldexpf(1.0f, e);
}

// Four values, at most 448 in magnitude or NaN, to e4m3 bytes (to nearest, ties to even).
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
    uint32_t w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ void from_e4m3(uint32_t w, float* x) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    x[0] = lo.x;
    x[1] = lo.y;
    x[2] = hi.x;
    x[3] = hi.y;
}

// Four bytes times `ratio`, a ratio of two scales that keeps every value within 448.
__device__ __forceinline__ uint32_t rescale_e4m3(uint32_t w, float ratio) {
    float x[4];
    from_e4m3(w, x);
    return to_e4m3(x[0] * ratio, x[1] * ratio, x[2] * ratio, x[3] * ratio);
}

// The ratio by which bytes at scale `from` become bytes at scale `to`.  Where `from` is
// far above `to`, the block's values at `from` can only be zeros (its maximum fits 448 of
// `to`), which an infinite ratio would turn into NaN.
__device__ __forceinline__ float scale_ratio(float from, float to) {
    return fminf(from / to, 1048576.0f);
}

}  // namespace e2s
