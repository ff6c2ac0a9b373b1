// What the kernels over the paged cache of 16 or 8 bits share: rows of the cache as operands of the matrix instructions.
//
// A block is 32 keys of a KV head, key0 .. key0 + 31.  Lanes (16 x 16 x 32): n = lane % 16, g = lane / 16.
//   scores   S^T[key][query] = K . Q^T: A = K, B = Q^T.  Row 4 g + r of key tile t is key 8 g + 4 t + r of the block, so that
//            lane (n, g) holds keys 8 g .. 8 g + 7 of query n: the B operand of
//   output   O^T[d][query] = V^T . P^T: A = V^T.  Row i of element tile dt is element 8 i + dt, so that lane (n, g) of the
//            operand takes elements 8 n .. 8 n + 7 of its eight keys, a piece of a row each.
// In 8 bits a row is c_d 2^e, and what the conversion makes of a code and the scale is the value itself: the cache's rows come
// from rows of the type, whose exponents leave the four significant bits room.
#pragma once

#include "fd_chunk.h"
#include "fd_cache.h"
#include "fd_finite.h"

namespace fd {

typedef __attribute__((address_space(4))) const int32_t *scalar_i32;      // read through the scalar cache

// Eight codes as numbers of the type.
template <class T> __device__ __forceinline__ u32x4_t from_codes(unsigned w0, unsigned w1, float scale)
{
    if constexpr (std::is_same<T, F16>::value)
        return u32x4_t{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, scale, false)),
                       __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, scale, true)),
                       __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, scale, false)),
                       __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, scale, true))};
    else
        return u32x4_t{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false)),
                       __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true)),
                       __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false)),
                       __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true))};
}
__device__ __forceinline__ float scale_of(unsigned byte) { return __builtin_bit_cast(float, byte << 23); }

// Where a block's rows are: the first of keys 0 .. 15 in the pool, and of 16 .. 31, which may lie in another page.
struct BlockRows {
    size_t low, high;
};
// The pages of a block of a sequence whose last key is `last`: keys behind it are read from the last 16 that hold one.
struct BlockPages {
    int low, high;
};
__device__ __forceinline__ BlockPages block_pages(scalar_i32 table, int shift, int key0, int last)
{
    return BlockPages{table[min(key0, last) >> shift], table[min(key0 + 16, last) >> shift]};
}
__device__ __forceinline__ size_t page_row(const KvPool &pool, int hkv, int entry, int key)
{
    const int page = min(max(entry, 0), pool.n_pages - 1);
    return (((size_t)page * pool.Hkv + hkv) << pool.page_shift) + (key & ((1 << pool.page_shift) - 1));
}
__device__ __forceinline__ BlockRows block_rows(const KvPool &pool, int hkv, const BlockPages &pages, int key0, int last)
{
    return BlockRows{page_row(pool, hkv, pages.low, min(key0, last & ~15)), page_row(pool, hkv, pages.high, min(key0 + 16, last & ~15))};
}

// The rows of a block in a wavefront's registers, as they lie in the cache; k8: of 8 bits.
template <class T, bool k8> struct Keys {
    u32x4_t x[2][k8 ? 2 : 4];
    u32x2_t scales;                                 // of keys 8 (n / 4) .. + 7
    __device__ __forceinline__ void load(const KvPool &pool, BlockRows at, int lane)
    {
        const int n = lane & 15, g = lane >> 4;
        // key 8 (n / 4) + 4 t + n % 4 of the block
        const size_t first = (n < 8 ? at.low : at.high) + 8 * ((n >> 2) & 1);
        constexpr int kRow = k8 ? kHeadDim : 2 * kHeadDim;
        const unsigned char *from = pool.k + first * kRow + (n & 3) * kRow + 16 * g;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < (k8 ? 2 : 4); ++i)
                x[t][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(from + 4 * t * kRow + 64 * i));
        if constexpr (k8) scales = *reinterpret_cast<const u32x2_t *>(pool.k_scales + first);
    }
    // operand kb of tile t
    __device__ __forceinline__ u32x4_t operand(int t, int kb, int lane) const
    {
        if constexpr (k8) {
            const unsigned byte = scales[t] >> (8 * (lane & 3)) & 255u;
            const u32x4_t w = x[t][kb >> 1];
            return kb & 1 ? from_codes<T>(w[2], w[3], scale_of(byte)) : from_codes<T>(w[0], w[1], scale_of(byte));
        } else {
            return x[t][kb];
        }
    }
    // the element of a query that lane (., g) of operand kb begins with
    static __device__ __forceinline__ int element(int kb, int g) { return k8 ? 64 * (kb >> 1) + 16 * g + 8 * (kb & 1) : 32 * kb + 8 * g; }
};

template <class T, bool k8> struct Values {
    u32x4_t x[k8 ? 4 : 8];                          // elements 8 n .. + 7 of key 8 g + j; of 8 bits: of two keys
    u32x2_t scales;
    __device__ __forceinline__ void load(const KvPool &pool, BlockRows at, int lane)
    {
        const int n = lane & 15, g = lane >> 4;
        const size_t first = (g < 2 ? at.low : at.high) + 8 * (g & 1);
        constexpr int kRow = k8 ? kHeadDim : 2 * kHeadDim;
        const unsigned char *from = pool.v + first * kRow + (k8 ? 8 : 16) * n;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (k8) {
                const u32x2_t y = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t *>(from + j * kRow));
                x[j >> 1][2 * (j & 1)] = y[0];
                x[j >> 1][2 * (j & 1) + 1] = y[1];
            } else {
                x[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(from + j * kRow));
            }
        }
        if constexpr (k8) scales = *reinterpret_cast<const u32x2_t *>(pool.v_scales + first);
    }
    // Rows without a key may hold anything: keys from 8 g + live on become 0.
    __device__ __forceinline__ void keep(int live)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if constexpr (k8) {
                x[j >> 1][2 * (j & 1)] = j < live ? x[j >> 1][2 * (j & 1)] : 0u;
                x[j >> 1][2 * (j & 1) + 1] = j < live ? x[j >> 1][2 * (j & 1) + 1] : 0u;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) x[j][i] = j < live ? x[j][i] : 0u;
            }
        if constexpr (k8)                                       // (0 times the infinity of byte 255 is none)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int bytes = min(max(live - 4 * i, 0), 4);
                scales[i] &= bytes == 4 ? ~0u : (1u << (8 * bytes)) - 1u;
            }
    }
    // element tiles 2 w and 2 w + 1 of the operand, w = 0 .. 3: pairs of keys, by their low and high halves
    __device__ __forceinline__ void operands(u32x4_t (&a)[8]) const
    {
        u32x4_t y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (k8) y[j] = from_codes<T>(x[j >> 1][2 * (j & 1)], x[j >> 1][2 * (j & 1) + 1], scale_of(scales[j >> 2] >> (8 * (j & 3)) & 255u));
            else y[j] = x[j];
        }
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned even = y[2 * i][w], odd = y[2 * i + 1][w];
                a[2 * w][i] = __builtin_amdgcn_perm(odd, even, 0x05040100u);
                a[2 * w + 1][i] = __builtin_amdgcn_perm(odd, even, 0x07060302u);
            }
    }
};

// Whether a wavefront's operand holds an infinite value or a NaN.
template <class T, int N> __device__ __forceinline__ bool any_not_finite(const u32x4_t (&a)[N])
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 top = {0, 0};
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned w = a[k][i] & 0x7fff7fffu;
            top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, w));
        }
    return __any(max((unsigned)top.x, (unsigned)top.y) >= T::kInfinity);
}

// The reference of a query's weights follows its maximum only where that has grown by more than this (in units of log2):
// the sums are brought to another reference a few times a row instead of at every new maximum.
constexpr float kKvSlack = 8.f;

// A query's running softmax over blocks, lane (n, g) of query n: the reference of the weights, in units of log2 and T::kLift below
// the logit it was taken from; this lane's part of their sum; O^T, element 32 g + 8 r + dt in acc[dt][r].
template <class T> struct Softmax {
    float ref, sum;
    f32x4_t acc[8];
    __device__ __forceinline__ void clear()
    {
        ref = -INFINITY;
        sum = 0.f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    // A block's two steps; z: this lane's eight logits, in units of log2.  The reference first: it multiplies the sums, by 0 where they had
    // none, and a summand of infinity has to come after that.
    __device__ __forceinline__ void refer(const float (&z)[8])
    {
        float top = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
        top = columns_max(top) - T::kLift;
        if (__any(top > ref + kKvSlack)) {                     // (also where there is no reference yet)
            const float to = fmaxf(ref, top), f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ref - to);
            sum *= f;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) acc[dt] *= f;
            ref = to;
        }
    }
    // odd: there may be values in `a` that are not finite
    __device__ __forceinline__ void weigh(const float (&z)[8], u32x4_t (&a)[8], bool odd)
    {
        const float from = ref == -INFINITY ? 0.f : ref;
        u32x4_t hi, lo;                                        // the weights as the sum of two numbers of the type
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a0 = __builtin_amdgcn_exp2f(z[2 * i] - from), a1 = __builtin_amdgcn_exp2f(z[2 * i + 1] - from);
            sum += a0 + a1;
            const unsigned h = T::pack(a0, a1);
            hi[i] = h;
            lo[i] = T::pack(a0 - T::lo(h), a1 - T::hi(h));
        }
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[dt] = T::mfma(a[dt], hi, acc[dt]);
        if (odd)                                               // (a small part may be 0 or negative: the large one's product tells)
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) a[dt] = finite<T>(a[dt]);
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[dt] = T::mfma(a[dt], lo, acc[dt]);
    }
};

// A wavefront's blocks of 32 keys, every fourth from key0 on and below `end`, for up to 16 rows (of query heads or of tokens, lane
// (n, .) row n) that share a KV head.  Nothing of the cache passes through LDS.  kMasks: a row sees the keys up to `position`, where
// positions differ by less than 16: only a wavefront's last block has keys that not all see.
// pages: of the first block.
template <class T, bool k8, bool kMasks>
__device__ __forceinline__ void walk_keys(const KvPool &pool, int hkv, scalar_i32 table, BlockPages pages, int key0, int end, int position,
                                          const u32x4_t (&q)[4], float c1, int lane, Softmax<T> &state)
{
    constexpr int kNext = 4 * 32;
    const int g = lane >> 4, last = end - 1;
    Keys<T, k8> keys;
    Values<T, k8> values;
    // A block, and the loads of the next where there is one.  (Loads that a branch may have left out would be waited for as if they had
    // not been: all of them, at every wait.)
    auto block = [&](auto has_next, auto ends_here) {
        constexpr bool kLoads = decltype(has_next)::value, kTail = decltype(ends_here)::value;
        const int next = key0 + kNext;
        f32x4_t s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) s[t] = T::mfma(keys.operand(t, kb, lane), q[kb], s[t]);
        }
        // (the next rows take the registers of those that have been used)
        __builtin_amdgcn_sched_barrier(0);
        BlockRows at;
        if constexpr (kLoads) {
            at = block_rows(pool, hkv, pages, next, last);
            keys.load(pool, at, lane);
        }
        __builtin_amdgcn_sched_barrier(0);
        float z[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = s[j >> 2][j & 3] * c1;
        const int live = end - key0 - 8 * g, own = kMasks ? min(position + 1 - key0 - 8 * g, live) : live;      // keys from 8 g on
        if constexpr (kTail) {
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = j < own ? z[j] : -INFINITY;
            values.keep(live);
        }
        u32x4_t a[8];
        values.operands(a);
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) asm volatile("" : "+v"(a[dt]));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (kLoads) {
            values.load(pool, at, lane);
            pages = block_pages(table, pool.page_shift, next + kNext, last);
        }
        // (no code of 8 bits is infinite, and NaN stay what they are)
        const bool odd = (!k8 || (kMasks && kTail)) && any_not_finite<T>(a);
        state.refer(z);
        if constexpr (kMasks && kTail)
            if (odd) {
                // keys behind a row have the weight 0: what they hold must not reach it, be it infinite
                u32x4_t seen;
#pragma unroll
                for (int j = 0; j < 8; j += 2) seen[j >> 1] = T::pack(j < own ? 1.f : 0.f, j + 1 < own ? 1.f : 0.f);
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) {
                    const f32x4_t counts = T::mfma(not_finite<T>(a[dt]), seen, f32x4_t{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                    for (int r = 0; r < 4; ++r) state.acc[dt][r] += summand(counts[r]);
                    a[dt] = finite<T>(a[dt]);
                }
            }
        state.weigh(z, a, odd);
    };
    const std::true_type yes;
    const std::false_type no;
    if (key0 < end) {
        const BlockRows at = block_rows(pool, hkv, pages, key0, last);
        keys.load(pool, at, lane);
        values.load(pool, at, lane);
        pages = block_pages(table, pool.page_shift, key0 + kNext, last);
#pragma unroll 1
        for (; key0 + kNext < end; key0 += kNext) block(yes, no);
        block(no, yes);
    }
}

// The sums of a workgroup's four wavefronts, and one row of all of them: lane l has elements 2 l and 2 l + 1.
constexpr int kSumRow = kHeadDim + 4;            // (rows start in different banks)
struct WaveSums {
    alignas(16) float rows[4][16][kSumRow];
    float m[4][16], l[4][16];
    // (to be followed by a barrier)
    template <class T> __device__ __forceinline__ void put(const Softmax<T> &state, int wave, int lane, int rows_used)
    {
        const int n = lane & 15, g = lane >> 4;
        float sum = rows_sum(state.sum, state.sum);
        sum = halves_sum(sum, sum);
        if (n >= rows_used) return;
        if (g == 0) {
            m[wave][n] = state.ref;
            l[wave][n] = sum;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<f32x4_t *>(&rows[wave][n][32 * g + 8 * r + 4 * h]) =
                    f32x4_t{state.acc[4 * h][r], state.acc[4 * h + 1][r], state.acc[4 * h + 2][r], state.acc[4 * h + 3][r]};
    }
    __device__ __forceinline__ void row(int n, int lane, float &a0, float &a1, float &top, float &sum) const
    {
        top = -INFINITY;
        a0 = a1 = sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, m[w][n]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float mw = m[w][n];
            // a wavefront without keys has m = -inf and zeros; one whose logits are all -inf or NaN has NaN, and keeps it
            const float f = mw == top ? 1.f : __builtin_amdgcn_exp2f(mw - top);
            const float2 x = *reinterpret_cast<const float2 *>(&rows[w][n][2 * lane]);
            a0 = __builtin_fmaf(x.x, f, a0);
            a1 = __builtin_fmaf(x.y, f, a1);
            sum = __builtin_fmaf(l[w][n], f, sum);
        }
    }
};

}  // namespace fd
