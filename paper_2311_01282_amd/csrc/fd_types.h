// fp16 and bf16 as the kernels of the smaller caches take them: conversions and matrix instructions by type.
#pragma once

#include "fd_internal.h"

namespace fd {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));

struct F16 {
    static constexpr float kSmallest = 0x1p-14f;           // normal number
    static constexpr unsigned kInfinity = 0x7c00u;         // bits
    // log2 of a softmax weight at its reference.  Numbers below 2^-25 round to 0.  With a reference of 1 that loses the
    // weights of keys 17.4 and more below the largest logit: of 16384 such keys 5e-4 of the sum.  With 2^7 it loses those
    // below 2^-32 of it, and weights of 2^8 times the reference's are still numbers.
    static constexpr float kLift = 7.f;
    static __device__ __forceinline__ float lo(unsigned w) { return (float)__builtin_bit_cast(f16x2_t, w).x; }
    static __device__ __forceinline__ float hi(unsigned w) { return (float)__builtin_bit_cast(f16x2_t, w).y; }
    static __device__ __forceinline__ unsigned short bits(float x)
    {
        const _Float16 h = (_Float16)x;
        return __builtin_bit_cast(unsigned short, h);
    }
    static __device__ __forceinline__ unsigned pack(float a, float b)
    {
        f16x2_t h;
        h.x = (_Float16)a;
        h.y = (_Float16)b;
        return __builtin_bit_cast(unsigned, h);
    }
    static __device__ __forceinline__ f32x4_t mfma(u32x4_t a, u32x4_t b, f32x4_t c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
    }
};
struct BF16 {
    static constexpr float kSmallest = 0x1p-126f;
    static constexpr unsigned kInfinity = 0x7f80u;
    static constexpr float kLift = 0.f;
    static __device__ __forceinline__ float lo(unsigned w) { return __builtin_bit_cast(float, w << 16); }
    static __device__ __forceinline__ float hi(unsigned w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
    static __device__ __forceinline__ unsigned short bits(float x)
    {
        const __bf16 h = (__bf16)x;
        return __builtin_bit_cast(unsigned short, h);
    }
    static __device__ __forceinline__ unsigned pack(float a, float b)
    {
        bf16x2_t h;
        h.x = (__bf16)a;
        h.y = (__bf16)b;
        return __builtin_bit_cast(unsigned, h);
    }
    static __device__ __forceinline__ f32x4_t mfma(u32x4_t a, u32x4_t b, f32x4_t c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    }
};

}  // namespace fd
