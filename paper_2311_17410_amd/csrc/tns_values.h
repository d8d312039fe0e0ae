// Values of the training operators as they lie in memory (fp32 or bf16) and as they are computed with (fp32), and the two
// functions of the recurrence's gate.  Included by .hip files only.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace tns {
namespace {

struct bf16 { uint16_t bits; };

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(bf16 v) { return __uint_as_float((uint32_t)v.bits << 16); }
template <typename T> __device__ __forceinline__ T as_value(float v);
template <> __device__ __forceinline__ float as_value<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 as_value<bf16>(float v) { return __builtin_bit_cast(bf16, (__bf16)v); }      // to nearest, ties to even

constexpr float kLog2e = 1.44269504088896340736f;

// z = sigmoid(u) and 1 - z, each with an error of some units in its last place: with E = exp(-u), z = 1 / (1 + E) and
// 1 - z = E z, which is 1 from E = 2^24 on (and would be infinity times 0 in the end).
__device__ __forceinline__ void gate_of(float u, float& z, float& rest) {
    const float a = u * -kLog2e, e = __builtin_amdgcn_exp2f(a);
    z = __builtin_amdgcn_rcpf(1.0f + e);
    rest = a > 64.0f ? 1.0f : e * z;                 // (a NaN stays)
}

// Time between two events: never negative, never NaN, never infinite (so that a decay of 0 times it is 0).
__device__ __forceinline__ float gap_of(float t, float before) { return fminf(fmaxf(t - before, 0.0f), 3.402823466e+38f); }

}  // namespace
}  // namespace tns
