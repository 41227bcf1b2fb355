// What the kernels of the draft body and of the attention over trees share: bf16 conversions, vector types, reductions across a wave's groups of 16 lanes.
#pragma once
#include <hip/hip_bf16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tabed {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4b;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4b;

__device__ __forceinline__ uint16_t f32_to_bf16_bits(float f) {            // round to nearest even
    return __builtin_bit_cast(uint16_t, (__bf16)f);
}

__device__ __forceinline__ uint2 pack_bf16x4(float a, float b, float c, float d) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2)),      // one instruction a pair
                      __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{c, d}, bf16x2)));
}

// v combined with the v of the lane 16, or 32, away.  (The results are copied out first: a bit cast of an element of the
// returned vector reads element 0.)
template <typename F>
__device__ __forceinline__ float with_lane16(float v, F f) {
    const uint32_t x = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    const uint32_t r0 = r[0], r1 = r[1];
    return f(__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1));
}
template <typename F>
__device__ __forceinline__ float with_lane32(float v, F f) {
    const uint32_t x = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    const uint32_t r0 = r[0], r1 = r[1];
    return f(__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1));
}
__device__ __forceinline__ float add_lanes16_32(float v) {
    auto add = [](float p, float q) { return p + q; };
    return with_lane32(with_lane16(v, add), add);
}
__device__ __forceinline__ float max_lanes16_32(float v) {
    auto larger = [](float p, float q) { return fmaxf(p, q); };
    return with_lane32(with_lane16(v, larger), larger);
}

}  // namespace tabed
