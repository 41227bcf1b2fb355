// Shared by the 8-bit operators: values of either storage type read at any alignment of their own, magnitudes as bits, int8 steps.
#pragma once
#include "device_utils.h"

namespace tabed {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// Magnitudes are compared as the bits of their absolute value: the order is the same, and a NaN or an infinity comes out as
// the largest instead of being passed over.
constexpr uint32_t kInfBits = 0x7f800000u;
__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v) { return (uint32_t)dpp_i32<CTRL>((int)v); }
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
    v = max(v, dpp_u32<kDppXor1>(v));
    v = max(v, dpp_u32<kDppXor2>(v));
    v = max(v, dpp_u32<kDppHalfMirror>(v));
    v = max(v, dpp_u32<kDppMirror>(v));
    auto at = [&](int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); };
    return max(max(at(0), at(16)), max(at(32), at(48)));
}

// The scale of a row or block whose largest magnitude is `bits`: 1/127 of it; 0 (all zeros) below 2^-100, where reciprocals
// would leave fp32's range; NaN if some value is not finite, so that whatever reads the row shows it.
constexpr float kTiny = 7.888609052210118e-31f;        // 2^-100
__device__ __forceinline__ float scale_of(uint32_t bits) {
    const float most = __builtin_bit_cast(float, bits);
    return bits >= kInfBits ? __builtin_nanf("") : most >= kTiny ? most / 127.f : 0.f;
}
__device__ __forceinline__ int to_step(float steps) {          // of a finite value
    return (int)rintf(fminf(fmaxf(steps, -127.f), 127.f));
}
// round(x / scale), the division as fp32 rounds it, for |x| of at most 127 scale.  A product with the reciprocal (inv) is off by less than 1.6e-5 steps: only
// where one comes that near to the middle between two steps is the division made (a dozen instructions each: half of the time of appending a prompt).
template <int N>
__device__ __forceinline__ void steps_of(const float (&x)[N], float scale, float inv, int (&s)[N]) {
    float far = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float t = x[e] * inv, r = rintf(t);
        far = fmaxf(far, fabsf(t - r));
        s[e] = (int)r;
    }
    if (__any(far > 0.5f - 2e-5f)) {
#pragma unroll
        for (int e = 0; e < N; ++e) s[e] = (int)rintf(x[e] / scale);
    }
}
__device__ __forceinline__ uint32_t pack_i8(int a, int b, int c, int d) {
    return (uint32_t)(a & 255) | (uint32_t)(b & 255) << 8 | (uint32_t)(c & 255) << 16 | (uint32_t)d << 24;
}

// N consecutive values as fp32.  The vector loads need no more than the values' own alignment.
typedef uint32_t u32x4_e2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_e4 __attribute__((ext_vector_type(4), aligned(4)));
template <int N, bool BF16>
__device__ __forceinline__ void load_values(const void* base, int64_t at, float (&x)[N]) {
    static_assert(N % 8 == 0, "pieces of 8");
    if constexpr (BF16) {
        const uint16_t* p = static_cast<const uint16_t*>(base) + at;
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            const u32x4_e2 w = *reinterpret_cast<const u32x4_e2*>(p + 8 * i);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                x[8 * i + 2 * q] = __builtin_bit_cast(float, w[q] << 16);
                x[8 * i + 2 * q + 1] = __builtin_bit_cast(float, w[q] & 0xffff0000u);
            }
        }
    } else {
        const float* p = static_cast<const float*>(base) + at;
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const f32x4_any w = *reinterpret_cast<const f32x4_any*>(p + 4 * i);
#pragma unroll
            for (int q = 0; q < 4; ++q) x[4 * i + q] = w[q];
        }
    }
}
template <bool BF16>
__device__ __forceinline__ float load_value(const void* base, int64_t at) {
    if constexpr (BF16) return __builtin_bit_cast(float, (uint32_t)static_cast<const uint16_t*>(base)[at] << 16);
    else return static_cast<const float*>(base)[at];
}

}  // namespace tabed
