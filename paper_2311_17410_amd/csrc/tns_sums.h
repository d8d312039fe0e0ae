// Sums and maxima over the lanes of a wave and the waves of a workgroup, in fp32.  Included by .hip files only; called by whole waves.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace tns {
namespace {

// Sums over lanes as vector instructions (a shuffle through the LDS unit is some sixty cycles).  Lanes that have the same sum read each
// other's in mirrored order, so all of them add the same two values and get the same bits.
template <int CTRL>
__device__ __forceinline__ float moved_lane(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true)); }

struct Add {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
    static constexpr float none = 0.0f;
};
struct Max {                            // (a NaN loses: it shows in the sums)
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
    static constexpr float none = -__builtin_inff();
};

template <int BY, typename Op>
__device__ __forceinline__ float with_neighbour(float v, const Op& op) {      // the value of the other BY lanes of 2 BY
    if constexpr (BY == 1) return op(v, moved_lane<0xB1>(v));                 // quad_perm 1, 0, 3, 2
    else if constexpr (BY == 2) return op(v, moved_lane<0x4E>(v));            // quad_perm 2, 3, 0, 1
    else if constexpr (BY == 4) return op(v, moved_lane<0x141>(v));           // row_half_mirror
    else if constexpr (BY == 8) return op(v, moved_lane<0x140>(v));           // row_mirror
    else if constexpr (BY == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
}
// Over each n lanes side by side, n a power of two that is the same for the wave.
template <typename Op>
__device__ __forceinline__ float over_lanes(float v, int n, const Op& op) {
    if (n > 1) v = with_neighbour<1>(v, op);
    if (n > 2) v = with_neighbour<2>(v, op);
    if (n > 4) v = with_neighbour<4>(v, op);
    if (n > 8) v = with_neighbour<8>(v, op);
    if (n > 16) v = with_neighbour<16>(v, op);
    if (n > 32) v = with_neighbour<32>(v, op);
    return v;
}
// The value of the lane BY below in a row of sixteen, going round.
template <int BY>
__device__ __forceinline__ float row_turned(float v) { return moved_lane<0x120 + BY>(v); }
// Over the lanes of a row of sixteen that have the same number modulo n: from half a row down, so that what is turned has the turn's period.
template <typename Op>
__device__ __forceinline__ float over_row_strided(float v, int n, const Op& op) {
    if (n <= 8) v = op(v, row_turned<8>(v));
    if (n <= 4) v = op(v, row_turned<4>(v));
    if (n <= 2) v = op(v, row_turned<2>(v));
    if (n <= 1) v = op(v, row_turned<1>(v));
    return v;
}
// Over the lanes that have the same number modulo n.
template <typename Op>
__device__ __forceinline__ float over_strided(float v, int n, const Op& op) {
    v = over_row_strided(v, n, op);
    if (n <= 16) v = with_neighbour<16>(v, op);
    if (n <= 32) v = with_neighbour<32>(v, op);
    return v;
}
// Two sums for the price of one: over the lanes 16 (32) apart, `a` for those in even rows (the lower half), `b` for the others.
template <int BY>
__device__ __forceinline__ float add_either(float a, float b) {
    static_assert(BY == 16 || BY == 32);
    if constexpr (BY == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
}

}  // namespace
}  // namespace tns
