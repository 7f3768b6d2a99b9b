// Sums over groups of neighbouring lanes, in every one of them, by data-parallel
// moves: a sixth of what shuffles through LDS take.  The order is the same in
// every run.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace edb {
namespace lanes {

template <int MOVE>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, MOVE, 0xf, 0xf, false);
}
template <int MOVE>
__device__ __forceinline__ int32_t moved(int32_t v) {
    return (int32_t)moved<MOVE>((uint32_t)v);
}
template <int MOVE>
__device__ __forceinline__ float moved(float v) {
    return __builtin_bit_cast(float, moved<MOVE>(__builtin_bit_cast(uint32_t, v)));
}
template <int MOVE>
__device__ __forceinline__ double moved(double v) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)moved<MOVE>((uint32_t)u) | (uint64_t)moved<MOVE>((uint32_t)(u >> 32)) << 32);
}

// The sum of both rows of 16 lanes, or of both halves of the wave.
template <bool HALVES>
__device__ __forceinline__ void both(uint32_t v, uint32_t& a, uint32_t& b) {
    const auto p = HALVES ? __builtin_amdgcn_permlane32_swap(v, v, false, false) : __builtin_amdgcn_permlane16_swap(v, v, false, false);
    a = (uint32_t)p[0];
    b = (uint32_t)p[1];
}
template <bool HALVES, class T>
__device__ __forceinline__ T across(T v) {
    uint32_t a[sizeof(T) / 4], b[sizeof(T) / 4];
    if constexpr (sizeof(T) == 4) {
        both<HALVES>(__builtin_bit_cast(uint32_t, v), a[0], b[0]);
        return __builtin_bit_cast(T, a[0]) + __builtin_bit_cast(T, b[0]);
    } else {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        both<HALVES>((uint32_t)u, a[0], b[0]);
        both<HALVES>((uint32_t)(u >> 32), a[1], b[1]);
        return __builtin_bit_cast(T, (uint64_t)a[0] | (uint64_t)a[1] << 32) + __builtin_bit_cast(T, (uint64_t)b[0] | (uint64_t)b[1] << 32);
    }
}

// Over LANES (2, 4 .. 64) lanes.  Below a full wave only groups that are active
// whole take part.
template <int LANES, class T>
__device__ __forceinline__ T sum(T v) {
    if constexpr (LANES >= 2) v += moved<0xb1>(v);     // lane ^ 1
    if constexpr (LANES >= 4) v += moved<0x4e>(v);     // lane ^ 2
    if constexpr (LANES >= 8) v += moved<0x141>(v);    // the other four of eight
    if constexpr (LANES >= 16) v += moved<0x128>(v);   // lane ^ 8
    if constexpr (LANES >= 32) v = across<false>(v);
    if constexpr (LANES >= 64) v = across<true>(v);
    return v;
}

}  // namespace lanes
}  // namespace edb
