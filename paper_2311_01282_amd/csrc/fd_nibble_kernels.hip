// The 4-bit cache: rows into it, rows out of it, and the decode attention over it.
//
// A group of 32, 64 or 128 neighbouring elements of a row (128 elements of a token and KV head) shares a scale s and a
// lowest value l of the cache's type; an element is l + s c, c = 0 .. 15.  Codes: 64 bytes a row, lower half of a byte
// first, V in order, K with its 16 words of eight elements transposed as a 4 x 4 matrix (elements 32 t + 8 c .. + 7 in word
// 4 c + t): a lane of the matrix instruction that multiplies K then finds its 16 bytes, one word for each of the four steps
// over a row, side by side, and a step covers one group of 32.  Scales: all s of a row, then all l.
#include "fd_chunk.h"
#include "fd_cache.h"
#include "fd_types.h"

namespace fd {

namespace {

// ---- rows in and out ----
// A row is read, coded and written within eight lanes, 16 elements to a lane; with eight elements to a lane the places and
// the two divisions of a group cost as much as the codes (16001 tokens x 8 heads, fp16: 26.8 us so, 18.6 with 16).  The
// arithmetic is in fp32: the differences and the division are rounded once each.  What bounds the coding is its vector
// instructions, some 16 an element with all else, next to memory (91 MB).  Reading back is bound by memory (84 MB): the
// rows leave past the caches (18.8 us without, 17.5 so).

template <class F> __device__ __forceinline__ float group_reduce(float x, int lanes, F f)
{
    x = f(x, dpp_swap<0xB1>(x));
    if (lanes > 2) x = f(x, dpp_swap<0x4E>(x));
    if (lanes > 4) x = f(x, dpp_swap<0x141>(x));
    return x;
}

struct RowPlace {
    size_t row;                 // of the pool: (page, head, token in page)
    int token, head;
    bool is_v, live;
};

// Row r of the call: K and V rows of a token's heads, one after the other.  (32 bits: a division of 64 is a hundred instructions.)
__device__ __forceinline__ RowPlace row_place(const NibblePool &pool, const int32_t *slots, int n_tokens, unsigned r)
{
    RowPlace at;
    const unsigned per = 2 * pool.Hkv, token = r / per, rest = r - token * per;
    at.is_v = rest >= (unsigned)pool.Hkv;
    at.head = at.is_v ? rest - pool.Hkv : rest;
    at.token = (int)token;
    at.live = token < (unsigned)n_tokens;
    const int slot = at.live ? slots[token] : -1;
    at.live = slot >= 0 && (slot >> pool.page_shift) < pool.n_pages;         // anything else: padding, left alone
    const int page = at.live ? slot >> pool.page_shift : 0;
    at.row = (((size_t)page * pool.Hkv + at.head) << pool.page_shift) + (at.live ? slot & ((1 << pool.page_shift) - 1) : 0);
    return at;
}

template <class T> __global__ __launch_bounds__(256) void nibble_write_kernel(NibblePool pool, TokenRows rows)
{
    const unsigned row = blockIdx.x * 32 + (threadIdx.x >> 3);
    const int j = threadIdx.x & 7;                                          // 16 elements from 16 j: words 2 j and 2 j + 1
    const RowPlace at = row_place(pool, rows.slots, rows.n_tokens, row);
    if (!at.live) return;                                                   // (whole rows of 8 lanes)
    const uint16_t *token = at.is_v ? rows.v + at.token * rows.v_stride : rows.k + at.token * rows.k_stride;
    const u32x4_t *src = reinterpret_cast<const u32x4_t *>(token + at.head * kHeadDim + 16 * j);
    const u32x4_t x[2] = {src[0], src[1]};
    float f[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned w = x[i >> 2][i & 3];
        f[2 * i] = T::lo(w);
        f[2 * i + 1] = T::hi(w);
    }
    float lo = f[0], hi = f[0];                                             // NaN where an element is
#pragma unroll
    for (int i = 1; i < 16; ++i) {
        lo = __builtin_elementwise_minimum(lo, f[i]);
        hi = __builtin_elementwise_maximum(hi, f[i]);
    }
    const int lanes = 8 / pool.NG;
    lo = group_reduce(lo, lanes, [](float a, float b) { return __builtin_elementwise_minimum(a, b); });
    hi = group_reduce(hi, lanes, [](float a, float b) { return __builtin_elementwise_maximum(a, b); });
    // The scale as it is stored is the one that the codes are taken against.  Quotients are those of fp32 division: with r
    // = 1 / s rounded, q = t r and one correction, q + r (t - q s), give the correctly rounded t / s (Markstein) where
    // nothing leaves the range of normal numbers; where it might, divisions do.  (With a division for each element the call
    // was bounded by them: 16001 tokens x 8 heads 35 us, 26.8 so, eight elements to a lane.)  A scale that is a normal
    // number is off by 2^-8 of itself at most, so that no quotient passes 15.5 and has to be limited.
    const float span = hi - lo;
    const bool ordinary = (span >= 15.5f * T::kSmallest && span < 0x1p100f) || span == 0.f;
    constexpr float kFifteenth = 1.f / 15.f;
    float fifteenth = span * kFifteenth;
    fifteenth = __builtin_fmaf(__builtin_fmaf(-fifteenth, 15.f, span), kFifteenth, fifteenth);
    if (!__all(ordinary)) fifteenth = span / 15.f;
    unsigned short s_bits = T::bits(fifteenth), l_bits = T::bits(lo);
    const float s = T::lo(s_bits), inv = 1.f / s;
    float quarter[4] = {0.f, 0.f, 0.f, 0.f};                                // four codes each: whole numbers below 2^16
    auto put = [&](int i, float c) { quarter[i >> 2] = __builtin_fmaf(quarter[i >> 2], 16.f, c); };
    if (__all(ordinary)) {
#pragma unroll
        for (int i = 15; i >= 0; --i) {
            const float t = f[i] - lo, q = t * inv;
            put(i, __builtin_rintf(__builtin_fmaf(__builtin_fmaf(-q, s, t), inv, q)));
        }
    } else {
#pragma unroll
        for (int i = 15; i >= 0; --i) put(i, fminf(__builtin_rintf((f[i] - lo) / s), 15.f));       // (t is not negative)
    }
    const bool odd = !(span < INFINITY);                                    // an infinite element, a NaN or such a range
    unsigned word[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        word[i] = (unsigned)quarter[2 * i] | ((unsigned)quarter[2 * i + 1] << 16);
        if (odd || !(s > 0.f)) word[i] = 0;                                 // (what was put together is NaN, then)
    }
    if (odd) s_bits = l_bits = 0x7fff;                               // NaN in both types: the group reads as NaN
    unsigned *codes = reinterpret_cast<unsigned *>((at.is_v ? pool.v_codes : pool.k_codes) + at.row * 64);
    const int place = at.is_v ? 2 * j : 8 * (j & 1) + (j >> 1), apart = at.is_v ? 1 : 4;
    codes[place] = word[0];
    codes[place + apart] = word[1];
    uint16_t *scales = (at.is_v ? pool.v_scales : pool.k_scales) + at.row * (2 * pool.NG);
    const int g = j / lanes;
    if (j % lanes == 0) scales[g] = s_bits;
    else if (j % lanes == 1) scales[pool.NG + g] = l_bits;
}

template <class T> __global__ __launch_bounds__(256) void nibble_read_kernel(NibblePool pool, TokenRows rows)
{
    const unsigned row = blockIdx.x * 32 + (threadIdx.x >> 3);
    // elements from 8 j and from 64 + 8 j: stores of eight lanes lie side by side
    const int j = threadIdx.x & 7;
    const RowPlace at = row_place(pool, rows.slots, rows.n_tokens, row);
    if (!at.live) return;
    const unsigned *codes = reinterpret_cast<const unsigned *>((at.is_v ? pool.v_codes : pool.k_codes) + at.row * 64);
    const int place = at.is_v ? j : 4 * (j & 3) + (j >> 2), apart = at.is_v ? 8 : 2;
    const unsigned word[2] = {codes[place], codes[place + apart]};
    const uint16_t *scales = (at.is_v ? pool.v_scales : pool.k_scales) + at.row * (2 * pool.NG);
    uint16_t *token = at.is_v ? rows.v + at.token * rows.v_stride : rows.k + at.token * rows.k_stride;
    u32x4_t *dst = reinterpret_cast<u32x4_t *>(token + at.head * kHeadDim) + j;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const int g = (j + 8 * w) * pool.NG >> 4;
        const float s = T::lo(scales[g]), l = T::lo(scales[pool.NG + g]);
        // bytes, of which a conversion takes any
        const unsigned even = word[w] & 0x0f0f0f0fu, odd = (word[w] >> 4) & 0x0f0f0f0fu;
        u32x4_t x;
        // s c is exact in fp32: one rounding there, one to the type
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[i] = T::pack(__builtin_fmaf(s, (float)((even >> (8 * i)) & 255), l), __builtin_fmaf(s, (float)((odd >> (8 * i)) & 255), l));
        __builtin_nontemporal_store(x, dst + 8 * w);
    }
}

// ---- attention ----
//
// One query token a sequence over the coded rows, synchronized softmax with a running maximum.  The codes go to the matrix
// cores as the numbers 16 + c, exact in both types, without touching the scales: of an element l + s c the product with a
// query is
//     sum_d q_d (l_g + s_g c_d) = sum_g s_g (sum_{d in g} q_d c_d) + l_g (sum_{d in g} q_d),
// four matrix instructions a row, one a group of 32, and a multiply-add with s and one with l a group; the 16 is taken off
// in the term with l.  Of the output
//     sum_j p_j (l_jg + s_jg c_jd) = sum_j (p_j s_jg) (16 + c_jd) + sum_j p_j (l_jg - 16 s_jg),
// the weights p s of a group as the operand, in two numbers of bf16 whatever the cache's type (hi + lo: 16 significant
// bits; one alone would add an error as large as the output's rounding), the last sum in fp32.  Of fp16 they would be 22
// bits where p s is large, but nothing below 2^-25, and the two sums then disagree by up to 31 times that a key, however
// small the values are (16384 keys, logits of deviation 3, values of 0.01: 2 % of the output; 4e-6 so).
//
// Lanes (16 x 16 x 32): n = lane % 16, c = lane / 16.  Scores of 16 query heads (rows) and 16 keys (columns): the lane of a
// key has its scales in registers.  Query head h of a tile sits in row 4 (h % 4) + h / 4, so that R = ceil(heads / 4) of a
// lane's four rows are in use.
// The weights pass through LDS (a wavefront's own), where lane n then finds row n; V's codes pass through LDS too, and the
// transposing read of 4-bit elements gives lane n the codes of element n of 16 keys: two operands of eight.
// A wavefront takes 64 keys at a time, four tiles of 16, every fourth such block of its workgroup's chunk; the four are
// joined at the end.  (Workgroups of one wavefront, with a chunk and a partial result each, did 32 x 64/8 heads x 4096 keys
// in 38.5 us at their best chunk, these then 35.4.)  Of the 64, operand u of lanes c takes keys of two tiles, 2 (c / 2) and
// the next, 8 (c % 2) + 4 u .. + 3 of each: what a lane has of the two tiles then lies side by side (expand's pairs).
// What bounds it: vector instructions, 60 % of the issue slots (16 x 32 heads x up to 4096 keys, fp16: 50 us, 4.3 TB/s; 32
// x 64/8 heads x 4096, bf16: 34 us, 4.5), which do not run under the other wavefront's matrix instructions (18 %).
constexpr int kBlock = 64;                       // keys of a wavefront step
constexpr int kJoinWorkgroups = 512;             // of a launch that joins its rows itself
constexpr int kJoinInPlace = 16;                 // chunks of a row that the launch itself can join
// bytes of a row of weights: 64 of two bytes, and 16 so that rows start in different banks
constexpr int kRowStride = 144;

// The reference of a row's weights follows its maximum only where that has grown by more than this (in units of log2): see
// the latent rows' kernel.
// (32 x 64/8 heads x 4096 keys, bf16: 1 % less than with 2.)
constexpr float kSlack = 8.f;
template <class T> struct Magic;                 // 16 + c: c in the low bits above the last ones of the mantissa of 16
template <> struct Magic<F16> {
    static constexpr unsigned kSixteen = 0x4c004c00u, kMask = 0x03c003c0u;
    static constexpr int kShift = 6;
};
template <> struct Magic<BF16> {
    static constexpr unsigned kSixteen = 0x41804180u, kMask = 0x00780078u;
    static constexpr int kShift = 3;
};

// Eight codes of a word as an operand: pairs (0, 4), (1, 5), (2, 6), (3, 7).  sixteen: Magic::kSixteen in a register the
// compiler cannot see through, which keeps "and" and "or" one instruction (of two constants only one can be other than a
// register).
template <class T> __device__ __forceinline__ u32x4_t expand(unsigned w, unsigned sixteen)
{
    constexpr int k = Magic<T>::kShift;
    u32x4_t x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned y = 4 * i <= k ? w << (k - 4 * i) : w >> (4 * i - k);
        x[i] = (y & Magic<T>::kMask) | sixteen;
    }
    return x;
}

// Two numbers as the sum of two of bf16 each, neighbours in a word.  They are rounded (ties away from 0) by an addition to
// their bits and cut off by a byte permutation: the conversion instruction takes several times as long as either (16 x 32
// heads x up to 4096 keys, fp16: 52.9 us with it, 49.8 so; 32 x 64/8 heads x 4096, bf16: 35.9, 33.9).  Some NaN become
// other numbers in this; the sum in fp32 of the same key and group has them too and keeps them.
struct TwoParts {
    unsigned hi, lo;
};
__device__ __forceinline__ unsigned as_u32(float x) { return __builtin_bit_cast(unsigned, x); }
__device__ __forceinline__ TwoParts two_parts(float a, float b)
{
    constexpr unsigned kHalf = 0x8000u, kHigh = 0xffff0000u, kHighHalves = 0x07060302u;
    const unsigned ra = as_u32(a) + kHalf, rb = as_u32(b) + kHalf;
    const unsigned la = as_u32(a - as_f32(ra & kHigh)) + kHalf, lb = as_u32(b - as_f32(rb & kHigh)) + kHalf;
    return TwoParts{__builtin_amdgcn_perm(rb, ra, kHighHalves), __builtin_amdgcn_perm(lb, la, kHighHalves)};
}

template <int R> struct NibbleLds {
    union {
        struct {
            alignas(16) unsigned char v[4][2][kBlock * 64];            // of this step and of the next
            // weights of a group, two groups in turn: hi and lo parts; row 4 c + r in place R c + r
            alignas(16) unsigned char w[4][2][2][4 * R * kRowStride];
        };
        float rows[4][4 * R][kHeadDim];                                // at the end: the wavefronts' sums
    };
    float m[4][4 * R], l[4][4 * R];
    int last;
};
// Loads into LDS, 1 KiB at lds_1k.  In assembly: of those that the compiler knows it would wait before every transposing
// read.  They are older than the loads of K's codes of the same step, and loads arrive in order: once K's codes are there,
// so are they.
// (That the scalar registers of an address have settled: tests/test_wait_states_host.py.)
__device__ __forceinline__ void load_to_lds(const unsigned char *base, int voff, unsigned lds_1k)
{
    const unsigned long long at = reinterpret_cast<unsigned long long>(base);
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(lds_1k), "v"(voff), "s"(at) : "memory");
}

template <class T> __device__ __forceinline__ float scale_at(const unsigned *w, int i)
{
    return (i & 1) ? T::hi(w[i >> 1]) : T::lo(w[i >> 1]);
}

__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); __builtin_amdgcn_wave_barrier(); }

typedef __attribute__((address_space(4))) const int32_t *scalar_i32;      // read through the scalar cache

template <class T, int NG, int R> __global__ __launch_bounds__(256, 2) void nibble_attn_kernel(NibbleProblem p)
{
    __shared__ NibbleLds<R> lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, c = lane >> 4;
    const int chunk = blockIdx.x % p.nc, group = blockIdx.x / p.nc;
    int unit = group;
    const int tile = unit % p.tiles;
    unit /= p.tiles;
    const int hkv = unit % p.pool.Hkv, b = unit / p.pool.Hkv;
    const int start = chunk * p.C, shift = p.pool.page_shift, mask = (1 << shift) - 1;
    const scalar_i32 table = (scalar_i32)(uintptr_t)(p.table + (size_t)b * p.width);
    const int len = min(max(((scalar_i32)(uintptr_t)p.seq_lens)[b], 0), p.Smax);
    const int end = min(len, start + p.C);
    const int heads = min(p.G - 16 * tile, 16), head0 = hkv * p.G + 16 * tile;      // query heads of this tile
    if (start >= end) {
        // a sequence without keys: zero rows, by the first chunk (other chunks without keys leave nothing)
        if (chunk == 0)
            for (int i = tid; i < heads * kHeadDim / 2; i += 256)
                reinterpret_cast<unsigned *>(p.out + ((size_t)b * p.Hq + head0) * kHeadDim)[i] = 0u;
        return;
    }
    constexpr int SW = NG;                         // 32-bit words of a row's scales
    u32x4_t kc[4];
    unsigned ks[4][SW], vs[4][SW];
    // pages of the four tiles from key0 (of the last tile with a key, for those behind it)
    const int last_tile = (end - 1) & ~15;
    int page[4];
    auto load_pages = [&](int key0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) page[i] = table[min(key0 + 16 * i, last_tile) >> shift];
    };
    size_t row[4];                                 // of the pool: the tiles' first
    auto find_rows = [&](int key0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int pg = min(max(page[i], 0), p.pool.n_pages - 1);
            row[i] = (((size_t)pg * p.pool.Hkv + hkv) << shift) + (min(key0 + 16 * i, last_tile) & mask);
        }
    };
    // (a uniform base and a 32-bit offset of the lane)
    auto load_codes = [&](const unsigned char *base, u32x4_t (&x)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(base + row[i] * 64 + (unsigned)(64 * n + 16 * c)));
    };
    auto load_scales = [&](const uint16_t *base, unsigned (&w)[4][SW]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned char *at = reinterpret_cast<const unsigned char *>(base) + row[i] * (4 * SW) + (unsigned)(4 * SW * n);
            if constexpr (NG == 4) {
                const u32x4_t x = *reinterpret_cast<const u32x4_t *>(at);
                w[i][0] = x[0]; w[i][1] = x[1]; w[i][2] = x[2]; w[i][3] = x[3];
            } else if constexpr (NG == 2) {
                const u32x2_t x = *reinterpret_cast<const u32x2_t *>(at);
                w[i][0] = x[0]; w[i][1] = x[1];
            } else {
                w[i][0] = *reinterpret_cast<const unsigned *>(at);
            }
        }
    };
    // V's codes in LDS: row of key k of tile i at 64 (16 i + k), its 16-byte piece x in place x ^ (2 (i % 2) + (k / 4) % 2)
    const int v_lane = 64 * (lane >> 2) + 16 * ((lane & 3) ^ ((lane >> 4) & 1));
    const unsigned v_lds = __builtin_amdgcn_readfirstlane(
        (unsigned)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char *)lds.v[wave][0]));
    auto load_v = [&](int buffer) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            load_to_lds(p.pool.v_codes + row[i] * 64, v_lane ^ ((i & 1) << 5), v_lds + buffer * (kBlock * 64) + 1024 * i);
    };
    int key0 = start + kBlock * wave, buffer = 0;
    if (key0 < end) {
        load_pages(key0);
        find_rows(key0);
        load_v(0);
        load_codes(p.pool.k_codes, kc);
        load_scales(p.pool.k_scales, ks);
        load_scales(p.pool.v_scales, vs);
        load_pages(key0 + 4 * kBlock);
    }

    // the query rows: A operand, elements 32 t + 8 c .. + 7 of row n in the order of the expanded codes
    u32x4_t qa[4];
    float qs[4];
    {
        const int head = 4 * (n & 3) + (n >> 2);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            u32x4_t x = {0u, 0u, 0u, 0u};
            if (head < heads) x = *reinterpret_cast<const u32x4_t *>(p.q + ((size_t)b * p.Hq + head0 + head) * kHeadDim + 32 * t + 8 * c);
            const unsigned x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
            qs[t] = ((T::lo(x0) + T::hi(x0)) + (T::lo(x1) + T::hi(x1))) + ((T::lo(x2) + T::hi(x2)) + (T::lo(x3) + T::hi(x3)));
            qs[t] += __shfl_xor(qs[t], 16);
            qs[t] += __shfl_xor(qs[t], 32);
            qa[t] = u32x4_t{__builtin_amdgcn_perm(x2, x0, 0x05040100u), __builtin_amdgcn_perm(x2, x0, 0x07060302u),
                            __builtin_amdgcn_perm(x3, x1, 0x05040100u), __builtin_amdgcn_perm(x3, x1, 0x07060302u)};
        }
    }
    // sums of the query over a group, for this lane's rows 4 c + r
    float qsum[NG][R];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        float s = 0.f;
#pragma unroll
        for (int t = 0; t < 4 / NG; ++t) s += qs[g * (4 / NG) + t];
#pragma unroll
        for (int r = 0; r < R; ++r) qsum[g][r] = __shfl(s, 4 * c + r);
    }

    const float c1 = p.scale * kLog2e;
    float m[R], l[R], low[R][NG];
    f32x4_t acc[8];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.f;
#pragma unroll
        for (int g = 0; g < NG; ++g) low[r][g] = 0.f;
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) acc[dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    unsigned sixteen, sixteen_v;                   // of K, whose products are with queries of type T, and of V
    asm("v_mov_b32 %0, %1" : "=v"(sixteen) : "i"(Magic<T>::kSixteen));
    asm("v_mov_b32 %0, %1" : "=v"(sixteen_v) : "i"(Magic<BF16>::kSixteen));

    unsigned char *w_at = lds.w[wave][0][0];
    // from a hi part to its lo part, from a group to the next
    constexpr int kLo = 4 * R * kRowStride, kTurn = 2 * kLo;
    const int w_row = (R * (n >> 2) + min(n & 3, R - 1)) * kRowStride;      // of row n (of rows that no head sits in: another's)
    // this lane's row for the transposing reads of V's codes
    const int v_tile = 2 * (c >> 1) + ((n >> 2) & 1), v_key = 8 * (c & 1) + 4 * (n >> 3) + (n & 3);
    const unsigned char *v_row = lds.v[wave][0] + (16 * v_tile + v_key) * 64;
    const int v_turn = 2 * (v_tile & 1) + ((v_key >> 2) & 1);

    for (; key0 < end; key0 += 4 * kBlock, buffer ^= 1) {
        const int next = key0 + 4 * kBlock;
        // Scores, in units of log2.  The matrix instructions of a tile run while the codes of the next are expanded (left
        // to itself the compiler takes one register after the other through expand, product and sum, and waits in between).
        float z[4][R];
        {
            u32x4_t e[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) e[t] = expand<T>(kc[0][t], sixteen);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x4_t a[NG];
                u32x4_t en[4];
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    a[t * NG / 4] = T::mfma(qa[t], e[t], t % (4 / NG) == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : a[t * NG / 4]);
                if (i < 3)
#pragma unroll
                    for (int t = 0; t < 4; ++t) en[t] = expand<T>(kc[i + 1][t], sixteen);
                float s[NG], lw[NG];
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    s[g] = scale_at<T>(ks[i], g);
                    lw[g] = __builtin_fmaf(-16.f, s[g], scale_at<T>(ks[i], NG + g));
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);         // a matrix instruction ...
                    __builtin_amdgcn_sched_group_barrier(0x002, 9, 0);         // ... and vector instructions behind it
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    float x = lw[0] * qsum[0][r], y = s[0] * a[0][r];
#pragma unroll
                    for (int g = 1; g < NG; ++g) {
                        x = __builtin_fmaf(lw[g], qsum[g][r], x);
                        y = __builtin_fmaf(s[g], a[g][r], y);
                    }
                    z[i][r] = (x + y) * c1;
                }
                if (i < 3)
#pragma unroll
                    for (int t = 0; t < 4; ++t) e[t] = en[t];
            }
        }
        if (key0 + kBlock > end) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool live = key0 + 16 * i + n < end;
#pragma unroll
                for (int r = 0; r < R; ++r) z[i][r] = live ? z[i][r] : -INFINITY;
                // of keys that are not there: may be anything
#pragma unroll
                for (int k = 0; k < SW; ++k) vs[i][k] = live ? vs[i][k] : 0u;
            }
        }
        asm volatile("" ::: "memory");                                                 // K's codes have been used: V's are there
        // ... and what was read of the step before has arrived
        __builtin_amdgcn_s_waitcnt(0xc07f);
        if (next < end) {                                                              // under way during the rest of the step
            find_rows(next);
            load_v(buffer ^ 1);
            load_codes(p.pool.k_codes, kc);
            load_scales(p.pool.k_scales, ks);
        }
        // the running maximum; what was summed is brought to it where it grew
        bool grew = false;
        float top[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            top[r] = row16_max(fmaxf(fmaxf(z[0][r], z[1][r]), fmaxf(z[2][r], z[3][r])));
            grew |= top[r] > m[r] + kSlack;
        }
        if (__any(grew)) {                                                             // (also where there is no reference yet)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float to = fmaxf(m[r], top[r]), f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[r] - to);
                l[r] *= f;
#pragma unroll
                for (int g = 0; g < NG; ++g) low[r][g] *= f;
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) acc[dt][r] *= f;
                m[r] = to;
            }
        }
        // weights
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float ref = m[r] == -INFINITY ? 0.f : m[r];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = __builtin_amdgcn_exp2f(z[i][r] - ref);
                l[r] += e;
                z[i][r] = e;
            }
        }
        auto put_weights = [&](int g) {
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                const float s0 = scale_at<T>(vs[i], g), s1 = scale_at<T>(vs[i + 1], g);
                const float l0 = __builtin_fmaf(-16.f, s0, scale_at<T>(vs[i], NG + g));
                const float l1 = __builtin_fmaf(-16.f, s1, scale_at<T>(vs[i + 1], NG + g));
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    low[r][g] = __builtin_fmaf(z[i][r], l0, low[r][g]);
                    low[r][g] = __builtin_fmaf(z[i + 1][r], l1, low[r][g]);
                    const TwoParts w = two_parts(z[i][r] * s0, z[i + 1][r] * s1);
                    unsigned char *at = w_at + (g & 1) * kTurn + (R * c + r) * kRowStride + 32 * i + 4 * n;
                    *reinterpret_cast<unsigned *>(at) = w.hi;
                    *reinterpret_cast<unsigned *>(at + kLo) = w.lo;
                }
            }
        };
        typedef int i32x2 __attribute__((ext_vector_type(2)));
        typedef __attribute__((address_space(3))) i32x2 *lds_i32x2;
        // 16 elements from 16 dt of this lane's row: lane n receives element n of the 16 rows
        auto read_v = [&](int dt) {
            const unsigned char *at = v_row + buffer * (kBlock * 64) + (((dt >> 1) ^ v_turn) << 4) + ((dt & 1) << 3);
            return __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2)at);
        };
        i32x2 vc[2][2];                                                                // of elements 32 pr .. + 31, two in turn
        vc[0][0] = read_v(0);
        vc[0][1] = read_v(1);
        put_weights(0);
        u32x4_t e[2][2];
#pragma unroll
        for (int d = 0; d < 2; ++d)
#pragma unroll
            for (int u = 0; u < 2; ++u) e[d][u] = expand<BF16>((unsigned)vc[0][d][u], sixteen_v);
        u32x4_t ah[2], al[2];
#pragma unroll
        for (int pr = 0; pr < 4; ++pr) {
            const int g = pr * NG / 4;
            if (pr % (4 / NG) == 0) {
                wave_fence();
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const unsigned char *at = w_at + (g & 1) * kTurn + w_row + 32 * c + 16 * u;
                    ah[u] = *reinterpret_cast<const u32x4_t *>(at);
                    al[u] = *reinterpret_cast<const u32x4_t *>(at + kLo);
                }
                if (g + 1 < NG) put_weights(g + 1);
                if (g == NG - 1 && next < end) {
                    load_scales(p.pool.v_scales, vs);
                    load_pages(next + 4 * kBlock);
                }
            }
            if (pr < 3) {
                vc[(pr + 1) & 1][0] = read_v(2 * pr + 2);
                vc[(pr + 1) & 1][1] = read_v(2 * pr + 3);
            }
            __builtin_amdgcn_sched_barrier(0);
            u32x4_t en[2][2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int d = 0; d < 2; ++d) acc[2 * pr + d] = BF16::mfma(ah[u], e[d][u], acc[2 * pr + d]);
#pragma unroll
                for (int d = 0; d < 2; ++d) acc[2 * pr + d] = BF16::mfma(al[u], e[d][u], acc[2 * pr + d]);
            }
            if (pr < 3) {
#pragma unroll
                for (int d = 0; d < 2; ++d)
#pragma unroll
                    for (int u = 0; u < 2; ++u) en[d][u] = expand<BF16>((unsigned)vc[(pr + 1) & 1][d][u], sixteen_v);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int d = 0; d < 2; ++d)
#pragma unroll
                for (int u = 0; u < 2; ++u) e[d][u] = en[d][u];
        }
        wave_fence();
    }

    // the four wavefronts' sums: lane (n, c) holds element 16 dt + n of rows 4 c + r
    __syncthreads();                                                       // (the weights' place becomes the sums')
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float ls = row16_sum(l[r]);
        float lw[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) lw[g] = row16_sum(low[r][g]);
        if (n == 0) {
            lds.m[wave][R * c + r] = m[r];
            lds.l[wave][R * c + r] = ls;
        }
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) lds.rows[wave][R * c + r][16 * dt + n] = acc[dt][r] + lw[dt * NG / 8];
    }
    __syncthreads();
    const int chunks = (len + p.C - 1) / p.C;                              // of this sequence
    for (int h = wave; h < heads; h += 4) {
        const int row = R * (h & 3) + (h >> 2);
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, lds.m[w][row]);
        float a0 = 0.f, a1 = 0.f, sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float mw = lds.m[w][row];
            // a wavefront without keys has m = -inf and zeros; one whose logits are all -inf or NaN has NaN, and keeps it
            const float f = mw == top ? 1.f : __builtin_amdgcn_exp2f(mw - top);
            const float2 x = *reinterpret_cast<const float2 *>(&lds.rows[w][row][2 * lane]);
            a0 = __builtin_fmaf(x.x, f, a0);
            a1 = __builtin_fmaf(x.y, f, a1);
            sum = __builtin_fmaf(lds.l[w][row], f, sum);
        }
        const size_t out_row = (size_t)b * p.Hq + head0 + h;
        if (chunks == 1) {
            const float inv = 1.f / sum;
            reinterpret_cast<unsigned *>(p.out + out_row * kHeadDim)[lane] = T::pack(a0 * inv, a1 * inv);
        } else {
            const size_t slot = out_row * p.nc + chunk;
            float *num = p.num + slot * kHeadDim + 2 * lane, *ml = reinterpret_cast<float *>(p.ml + slot);
            // past the caches: a workgroup on another XCD may join the row
            if (p.counters) {
                store_coherent2(num, a0, a1);
                if (lane == 0) store_coherent2(ml, top, sum);
            } else {
                *reinterpret_cast<float2 *>(num) = float2{a0, a1};
                if (lane == 0) *reinterpret_cast<float2 *>(ml) = float2{top, sum};
            }
        }
    }
    if (!p.counters || chunks == 1) return;
    // The workgroup of the group's last chunk to arrive joins its rows: a round trip to memory for the stores, one for the
    // counter, one for the partial results.
    wait_stores_performed();
    __syncthreads();
    if (tid == 0) {
        const int arrived = __hip_atomic_fetch_add(p.counters + group, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        lds.last = arrived == chunks - 1;
        if (arrived == chunks - 1) store_coherent(p.counters + group, 0);          // ready for the next call
    }
    __syncthreads();
    if (!lds.last) return;
    for (int h = wave; h < heads; h += 4) {
        const size_t out_row = (size_t)b * p.Hq + head0 + h, slot = out_row * p.nc;
        // chunk i's reference and denominator in lane i of every 16; all partial vectors under way before the first is used
        unsigned long long x[kJoinInPlace];
        const unsigned long long s = load_coherent(reinterpret_cast<const unsigned long long *>(p.ml + slot + min(n, chunks - 1)));
#pragma unroll
        for (int i = 0; i < kJoinInPlace; ++i)
            x[i] = load_coherent(reinterpret_cast<const unsigned long long *>(p.num + (slot + min(i, chunks - 1)) * kHeadDim) + lane);
        const float mi = n < chunks ? as_f32((unsigned)s) : -INFINITY, top = row16_max(mi);
        const float f = n >= chunks ? 0.f : mi == top ? 1.f : __builtin_amdgcn_exp2f(mi - top);
        const float sum = row16_sum(n < chunks ? as_f32((unsigned)(s >> 32)) * f : 0.f);
        float a0 = 0.f, a1 = 0.f;
        each16(std::make_integer_sequence<int, kJoinInPlace>{}, [&](auto of) {
            constexpr int i = decltype(of)::value;
            if (i < chunks) {
                const float fi = row16_lane<i>(f);
                a0 = __builtin_fmaf(as_f32((unsigned)x[i]), fi, a0);
                a1 = __builtin_fmaf(as_f32((unsigned)(x[i] >> 32)), fi, a1);
            }
        });
        const float inv = 1.f / sum;
        reinterpret_cast<unsigned *>(p.out + out_row * kHeadDim)[lane] = T::pack(a0 * inv, a1 * inv);
    }
}

// ---- the join of rows that several workgroups share ----
// A workgroup a row, of several slices that take every kSlices-th eight of the partial vectors.  Its length is that of its
// loads, so as many as can be are asked for together:
// first the references and denominators of 64 chunks, then, with their factors in LDS, eight vectors of a slice at a time.
constexpr int kJoinWindow = 64;
template <class T, int DIM, int kSlices> __global__ __launch_bounds__(DIM / 2 * kSlices) void join_kernel(JoinProblem p)
{
    constexpr int kLanes = DIM / 2;
    __shared__ float factor[kJoinWindow];
    __shared__ float2 sums[kSlices][kLanes];
    const int row = blockIdx.x, b = row / p.H, tid = threadIdx.x, lane = tid & 63, slice = tid / kLanes, at = tid % kLanes;
    const int len = min(max(p.seq_lens[b], 0), p.Smax), nb = (len + p.C - 1) / p.C;
    if (nb <= 1) return;                                        // done by the launch before
    const float2 *ml = p.ml + (size_t)row * p.nc;
    const float *num = p.num + (size_t)row * p.nc * DIM + 2 * at;
    float top = -INFINITY, a0 = 0.f, a1 = 0.f, sum = 0.f;
    for (int w0 = 0; w0 < nb; w0 += kJoinWindow) {
        const int count = min(nb - w0, kJoinWindow);
        float2 s = {-INFINITY, 0.f};
        if (lane < count) s = ml[w0 + lane];
        const float t = columns_max(row16_max(s.x));
        if (t > top) {                                          // (uniform) what the windows before left, to the new reference
            const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - t);
            a0 *= f;
            a1 *= f;
            sum *= f;
            top = t;
        }
        const float f = s.x == top ? 1.f : __builtin_amdgcn_exp2f(s.x - top);
        float d = lane < count ? s.y * f : 0.f;
        d = row16_sum(d);
        d = rows_sum(d, d);
        sum += halves_sum(d, d);
        __syncthreads();                                        // (the factors of the window before are out of use)
        if (tid < kJoinWindow) factor[tid] = f;
        __syncthreads();
        for (int i = 8 * slice; i < count; i += 8 * kSlices) {
            float2 x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                x[k] = i + k < count ? *reinterpret_cast<const float2 *>(num + (size_t)(w0 + i + k) * DIM) : float2{0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (i + k < count) {
                    a0 = __builtin_fmaf(x[k].x, factor[i + k], a0);
                    a1 = __builtin_fmaf(x[k].y, factor[i + k], a1);
                }
        }
    }
    sums[slice][at] = float2{a0, a1};
    __syncthreads();
    if (slice) return;
#pragma unroll
    for (int i = 1; i < kSlices; ++i) {
        a0 += sums[i][at].x;
        a1 += sums[i][at].y;
    }
    const float inv = 1.f / sum;
    reinterpret_cast<unsigned *>(p.out + (size_t)row * DIM)[at] = T::pack(a0 * inv, a1 * inv);
}

template <class T, int NG> hipError_t attn_rows(const NibbleProblem &p, hipStream_t s)
{
    const dim3 grid((unsigned)((long long)p.B * p.pool.Hkv * p.tiles * p.nc)), block(256);
    const int rows = p.G > 8 ? 4 : p.G > 4 ? 2 : 1;
    if (rows == 4) return launch(nibble_attn_kernel<T, NG, 4>, grid, block, s, p);
    if (rows == 2) return launch(nibble_attn_kernel<T, NG, 2>, grid, block, s, p);
    return launch(nibble_attn_kernel<T, NG, 1>, grid, block, s, p);
}
template <class T> hipError_t attn_groups(const NibbleProblem &p, hipStream_t s)
{
    return p.pool.NG == 4 ? attn_rows<T, 4>(p, s) : p.pool.NG == 2 ? attn_rows<T, 2>(p, s) : attn_rows<T, 1>(p, s);
}

}  // namespace

hipError_t launch_nibble_write(const NibblePool &pool, const TokenRows &rows, hipStream_t s)
{
    const dim3 grid((unsigned)(((long long)rows.n_tokens * 2 * pool.Hkv + 31) / 32));
    return launch(pool.dtype == kF16 ? nibble_write_kernel<F16> : nibble_write_kernel<BF16>, grid, dim3(256), s, pool, rows);
}
hipError_t launch_nibble_read(const NibblePool &pool, const TokenRows &rows, hipStream_t s)
{
    const dim3 grid((unsigned)(((long long)rows.n_tokens * 2 * pool.Hkv + 31) / 32));
    return launch(pool.dtype == kF16 ? nibble_read_kernel<F16> : nibble_read_kernel<BF16>, grid, dim3(256), s, pool, rows);
}
template <class T, int DIM> static hipError_t join(const JoinProblem &p, hipStream_t s)
{
    const dim3 grid((unsigned)p.rows);
    // (of up to eight vectors a row every slice but one would be idle: 128 x 128 latent rows of two 83 us, with two slices 97)
    if (p.nc > 8) return launch(join_kernel<T, DIM, 1024 / DIM>, grid, dim3(512), s, p);
    return launch(join_kernel<T, DIM, 1>, grid, dim3(DIM / 2), s, p);
}
hipError_t launch_join(const JoinProblem &p, hipStream_t s)
{
    if (p.dim == kHeadDim) return p.dtype == kF16 ? join<F16, kHeadDim>(p, s) : join<BF16, kHeadDim>(p, s);
    return p.dtype == kF16 ? join<F16, kLatent>(p, s) : join<BF16, kLatent>(p, s);
}
hipError_t launch_nibble_attn(const NibbleProblem &p_, hipStream_t s)
{
    NibbleProblem p = p_;
    // A workgroup that joins a unit's rows keeps the others of its compute unit waiting less than a second launch costs
    // while there are few.
    if (p.nc > kJoinInPlace || (long long)p.B * p.pool.Hkv * p.tiles * p.nc > kJoinWorkgroups) p.counters = nullptr;
    const hipError_t e = p.pool.dtype == kF16 ? attn_groups<F16>(p, s) : attn_groups<BF16>(p, s);
    if (e != hipSuccess || p.nc == 1 || p.counters) return e;
    JoinProblem j{p.num, p.ml, p.seq_lens, p.out, p.B * p.Hq, p.Hq, p.C, p.nc, p.Smax, kHeadDim, p.pool.dtype};
    return launch_join(j, s);
}

}  // namespace fd
