// Scales of groups of channels as the kernels read them.
#pragma once

#include "qlinear_device.h"

namespace qconv {

// The group of a row's n-th 32 channels.
__device__ __forceinline__ int group_of(const GroupArg &g, int n) { return (int)((uint32_t)n * g.per32 >> 20); }

// A scale's bits, and what they stand for.
template <int GS>
__device__ __forceinline__ uint32_t load_scale(const GroupArg &g, int64_t at) {
    if constexpr (GS == 4) return static_cast<const uint32_t *>(g.scale)[at];
    else return static_cast<const uint16_t *>(g.scale)[at];
}
template <int GS>
__device__ __forceinline__ float scale_value(const GroupArg &g, uint32_t bits) {
    if constexpr (GS == 4) return __builtin_bit_cast(float, bits);
    // (both forms, one of them of zero: a branch would part the loads around it)
    const uint32_t b = g.bf16 ? bits : 0u, f = g.bf16 ? 0u : bits;
    return __builtin_bit_cast(float, b << 16 | __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, (uint16_t)f)));
}

}  // namespace qconv
