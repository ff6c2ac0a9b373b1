// Values that are not finite under a causal mask.  The weights of keys behind a query are 0, and 0 times an infinite value or a
// NaN is NaN: such values leave the product, and the queries that see them get them as a summand.
#pragma once

#include "fd_types.h"

namespace fd {

// Values that are not finite: counted in a product of their own, in which an infinite one is 1, one of the other sign 64
// and a NaN 4096 (of 32 keys the counts do not meet).
template <class T> __device__ __forceinline__ u32x4_t not_finite(u32x4_t v)
{
    u32x4_t x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float f[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const unsigned h = v[i] >> (16 * k) & 0xffffu, size = h & 0x7fffu;
            f[k] = size < T::kInfinity ? 0.f : size > T::kInfinity ? 4096.f : h == size ? 1.f : 64.f;
        }
        x[i] = T::pack(f[0], f[1]);
    }
    return x;
}
template <class T> __device__ __forceinline__ u32x4_t finite(u32x4_t v)          // 0 in their place
{
    u32x4_t x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned low = (v[i] & 0x7fffu) < T::kInfinity ? v[i] & 0xffffu : 0u;
        const unsigned high = (v[i] >> 16 & 0x7fffu) < T::kInfinity ? v[i] & 0xffff0000u : 0u;
        x[i] = low | high;
    }
    return x;
}
// What counts stand for as a summand.
__device__ __forceinline__ float summand(float counts)
{
    const unsigned n = (unsigned)counts;
    return (n >= 4096 ? __builtin_nanf("") : 0.f) + (n & 63 ? INFINITY : 0.f) - (n & 4032 ? INFINITY : 0.f);
}

}  // namespace fd
