// The code of one low-bit head state, as kv_quant.hip describes it, for the kernels that make such codes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hbl {

__device__ __forceinline__ float as_f(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t as_u(float f) { return __builtin_bit_cast(uint32_t, f); }

constexpr float kMagic = 12582912.0f;   // 1.5 * 2^23: adding it rounds to an integer (nearest-even)

template <int BITS>
__device__ __forceinline__ float kv_gain(float gamma, float eps) {
    return (float)((1 << (BITS - 1)) - 1) / (gamma + eps);
}
template <int BITS>
__device__ __forceinline__ float kv_scale(float gamma) {
    return gamma / (float)((1 << (BITS - 1)) - 1);
}
// t + (1.5*2^23 + half): the fp32 adder rounds to nearest even and leaves code + half in the low mantissa bits
template <int BITS>
__device__ __forceinline__ void kv_codes8(const float* h, float gain, uint32_t* u) {
    constexpr int half = 1 << (BITS - 1);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        u[i] = as_u(__builtin_amdgcn_fmed3f(h[i] * gain, -(float)half, (float)(half - 1)) + (kMagic + (float)half)) & 0xFFu;
}

__device__ __forceinline__ uint4 pack_bf16x8(const float* v) {   // round to nearest even
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){v[2 * i], v[2 * i + 1]}, bf16x2));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

}  // namespace hbl
