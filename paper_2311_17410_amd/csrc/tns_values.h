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

// z = sigmoid(u) and 1 - z: with E = exp(-u), z = 1 / (1 + E) and 1 - z = E z, which is 1 from E = 2^64 on (and would be infinity times 0
// in the end).  The exponent is rounded to 32 bits before it is raised, so E and whichever of the two is small have a relative error of
// (1.5 |u| + 6) 2^-24 at most: 14 half units in the last place at |u| = 5, where z is 0.007, 126 at 80, where it is 2e-35.  This is a choice.
// What the rounding leaves out can be put back (two more products, a sum and a select, three half units everywhere; the decay's likewise), but
// these kernels issue vector instructions nearly as fast as memory feeds them: 0.79 M rows of 256 bf16 channels, states 219 -> 227 us and
// gradients 394 -> 425 (with the decay's 251 and 471), 0.80 M of 172 fp32, gradients 607 -> 613 (621).  An absolute error of z is 2^-22 at most.
__device__ __forceinline__ void gate_of(float u, float& z, float& rest) {
    const float a = u * -kLog2e, e = __builtin_amdgcn_exp2f(a);
    z = __builtin_amdgcn_rcpf(1.0f + e);
    rest = a > 64.0f ? 1.0f : e * z;                 // (a NaN stays)
}

// Time between two events: never negative, never NaN, never infinite (so that a decay of 0 times it is 0).
__device__ __forceinline__ float gap_of(float t, float before) { return fminf(fmaxf(t - before, 0.0f), 3.402823466e+38f); }

}  // namespace
}  // namespace tns
