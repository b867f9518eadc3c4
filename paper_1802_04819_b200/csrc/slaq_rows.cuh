// Rows of logits: element types, the order of their values, reductions of a block.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>
#include <stdint.h>

namespace slaq {

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float as_float(__half x) { return __half2float(x); }
template <class E> __device__ __forceinline__ E from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// 2^x to 2 ulp, 0 from -126 down
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// max that is NaN as soon as one operand is
__device__ __forceinline__ float max_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// Unsigned integers in the order of the values, -0 equal to +0, NaN above everything.  No value maps to 0.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
// .. and with the position: of equal values the one further to the left is the larger
__device__ __forceinline__ unsigned long long key_of(float x, uint32_t i) {
    return (unsigned long long)order_of(x) << 32 | (0xFFFFFFFFu - i);
}
__device__ __forceinline__ uint32_t position_of(unsigned long long key) { return 0xFFFFFFFFu - (uint32_t)key; }

constexpr float kLog2E = 1.4426950408889634f;

}  // namespace slaq
