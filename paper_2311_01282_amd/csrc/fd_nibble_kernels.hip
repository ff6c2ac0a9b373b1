// The 4-bit cache: rows into it, rows out of it, and the decode attention over it.
//
// A group of 32, 64 or 128 neighbouring elements of a row (128 elements of a token and KV head) shares a scale s and a lowest value l
// of the cache's type; an element is l + s c, c = 0 .. 15.  Codes: 64 bytes a row, lower half of a byte first, V in order, K with its
// 16 words of eight elements transposed as a 4 x 4 matrix (elements 32 t + 8 c .. + 7 in word 4 c + t): a lane of the matrix
// instruction that multiplies K then finds its 16 bytes, one word for each of the four steps over a row, side by side, and a step
// covers one group of 32.  Scales: all s of a row, then all l.
#include "fd_chunk.h"
#include "fd_cache.h"
#include "fd_types.h"

namespace fd {

namespace {

// ---- rows in and out ----
// 16 lanes to a row, eight elements (16 bytes, one word of codes) to a lane: a row is read, coded and written within a DPP row.  The
// arithmetic is in fp32: the differences and the division are rounded once each.  What bounds both calls is memory.

template <class F> __device__ __forceinline__ float group_reduce(float x, int lanes, F f)
{
    x = f(x, dpp_swap<0xB1>(x));
    x = f(x, dpp_swap<0x4E>(x));
    if (lanes > 4) x = f(x, dpp_swap<0x141>(x));
    if (lanes > 8) x = f(x, dpp_swap<0x140>(x));
    return x;
}

struct RowPlace {
    size_t row;                 // of the pool: (page, head, token in page)
    int token, head;
    bool is_v, live;
};

// Row r of the call: K and V rows of a token's heads, one after the other.
__device__ __forceinline__ RowPlace row_place(const NibblePool &pool, const int32_t *slots, int n_tokens, long long r)
{
    RowPlace at;
    const int per = 2 * pool.Hkv;
    const long long token = r / per;
    const int rest = (int)(r - token * per);
    at.is_v = rest >= pool.Hkv;
    at.head = at.is_v ? rest - pool.Hkv : rest;
    at.token = (int)token;
    at.live = token < n_tokens;
    const int slot = at.live ? slots[token] : -1;
    at.live = slot >= 0 && (slot >> pool.page_shift) < pool.n_pages;         // anything else: padding, left alone
    const int page = at.live ? slot >> pool.page_shift : 0;
    at.row = (((size_t)page * pool.Hkv + at.head) << pool.page_shift) + (at.live ? slot & ((1 << pool.page_shift) - 1) : 0);
    return at;
}

template <class T> __global__ __launch_bounds__(256) void nibble_write_kernel(NibblePool pool, NibbleRows rows)
{
    const long long r = ((long long)blockIdx.x * 256 + threadIdx.x) >> 4;
    const int j = threadIdx.x & 15;                                         // eight elements from 8 j
    const RowPlace at = row_place(pool, rows.slots, rows.n_tokens, r);
    if (!at.live) return;                                                   // (whole rows of 16 lanes)
    const uint16_t *src = (at.is_v ? rows.v + at.token * rows.v_stride : rows.k + at.token * rows.k_stride) + at.head * kHeadDim + 8 * j;
    const u32x4_t x = *reinterpret_cast<const u32x4_t *>(src);
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned w = x[i];
        f[2 * i] = T::lo(w);
        f[2 * i + 1] = T::hi(w);
    }
    float lo = f[0], hi = f[0], odd = 0.f;                                  // odd: NaN where an element is infinite or NaN
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo = fminf(lo, f[i]);
        hi = fmaxf(hi, f[i]);
        odd += f[i] - f[i];
    }
    const int lanes = 16 / pool.NG;
    lo = group_reduce(lo, lanes, [](float a, float b) { return fminf(a, b); });
    hi = group_reduce(hi, lanes, [](float a, float b) { return fmaxf(a, b); });
    odd = group_reduce(odd, lanes, [](float a, float b) { return a + b; });
    // the scale as it is stored is the one that the codes are taken against
    unsigned short s_bits = T::bits((hi - lo) / 15.f), l_bits = T::bits(lo);
    const float s = T::lo(s_bits);
    unsigned word = 0;
    if (odd == 0.f && s > 0.f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = fminf(fmaxf(__builtin_rintf((f[i] - lo) / s), 0.f), 15.f);
            word |= (unsigned)c << (4 * i);
        }
    }
    if (odd != 0.f) s_bits = l_bits = 0x7fff;                               // NaN in both types: the group reads as NaN
    unsigned char *codes = (at.is_v ? pool.v_codes : pool.k_codes) + at.row * 64;
    const int place = at.is_v ? j : 4 * (j & 3) + (j >> 2);
    *reinterpret_cast<unsigned *>(codes + 4 * place) = word;
    uint16_t *scales = (at.is_v ? pool.v_scales : pool.k_scales) + at.row * (2 * pool.NG);
    const int g = j / lanes;
    if (j % lanes == 0) scales[g] = s_bits;
    else if (j % lanes == 1) scales[pool.NG + g] = l_bits;
}

template <class T> __global__ __launch_bounds__(256) void nibble_read_kernel(NibblePool pool, NibbleRows rows)
{
    const long long r = ((long long)blockIdx.x * 256 + threadIdx.x) >> 4;
    const int j = threadIdx.x & 15;
    const RowPlace at = row_place(pool, rows.slots, rows.n_tokens, r);
    if (!at.live) return;
    const unsigned char *codes = (at.is_v ? pool.v_codes : pool.k_codes) + at.row * 64;
    const unsigned word = *reinterpret_cast<const unsigned *>(codes + 4 * (at.is_v ? j : 4 * (j & 3) + (j >> 2)));
    const uint16_t *scales = (at.is_v ? pool.v_scales : pool.k_scales) + at.row * (2 * pool.NG);
    const int g = j / (16 / pool.NG);
    const float s = T::lo(scales[g]), l = T::lo(scales[pool.NG + g]);
    u32x4_t x;
#pragma unroll
    for (int i = 0; i < 4; ++i)                                             // s c is exact in fp32: one rounding there, one to the type
        x[i] = T::pack(__builtin_fmaf(s, (float)((word >> (8 * i)) & 15), l), __builtin_fmaf(s, (float)((word >> (8 * i + 4)) & 15), l));
    uint16_t *dst = (at.is_v ? rows.v + at.token * rows.v_stride : rows.k + at.token * rows.k_stride) + at.head * kHeadDim + 8 * j;
    *reinterpret_cast<u32x4_t *>(dst) = x;
}

// ---- attention ----
//
// One query token a sequence over the coded rows, synchronized softmax with a running maximum.  The codes go to the matrix cores as the
// numbers 16 + c, exact in both types, without touching the scales: of an element l + s c the product with a query is
//     sum_d q_d (l_g + s_g c_d) = sum_g s_g (sum_{d in g} q_d c_d) + l_g (sum_{d in g} q_d),
// four matrix instructions a row, one a group of 32, and a multiply-add with s and one with l a group; the 16 is taken off in the accumulator the
// instruction starts from.  Of the output
//     sum_j p_j (l_jg + s_jg c_jd) = sum_j (p_j s_jg) (16 + c_jd) + sum_j p_j (l_jg - 16 s_jg),
// the weights p s of a group as the operand, in two parts of the type (hi + lo: 16 significant bits in bf16, 22 in fp16; one part alone
// would add an error as large as the output's rounding), the last sum in fp32.
//
// Lanes (16 x 16 x 32): n = lane % 16, c = lane / 16.  Scores of 16 query heads (rows) and 16 keys (columns): the lane of a key has its
// scales in registers.  Query head h of a tile sits in row 4 (h % 4) + h / 4, so that R = ceil(heads / 4) of a lane's four rows are in use.
// The weights pass through LDS (a wavefront's own), where lane n then finds row n; V's codes pass through LDS too, and the transposing
// read of 4-bit elements gives lane n the codes of element n of 16 keys: two operands of eight keys.
// A wavefront takes 64 keys at a time, every fourth such block of its workgroup's chunk; the four are joined at the end.
constexpr int kBlock = 64;                       // keys of a wavefront step
constexpr int kRowStride = 144;                  // bytes of a row of weights: 64 of two bytes, and 16 so that rows start in different banks
constexpr int kMaxPages = 1026;                  // table entries of a chunk (16384 keys in pages of 16)

template <class T> struct Magic;                 // 16 + c: c in the low bits above the last ones of the mantissa of 16
template <> struct Magic<F16> { static constexpr unsigned kSixteen = 0x4c004c00u, kMask = 0x03c003c0u; static constexpr int kShift = 6; };
template <> struct Magic<BF16> { static constexpr unsigned kSixteen = 0x41804180u, kMask = 0x00780078u; static constexpr int kShift = 3; };

// Eight codes of a word as an operand: pairs (0, 4), (1, 5), (2, 6), (3, 7).
template <class T> __device__ __forceinline__ u32x4_t expand(unsigned w)
{
    constexpr int k = Magic<T>::kShift;
    u32x4_t x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned y = 4 * i <= k ? w << (k - 4 * i) : w >> (4 * i - k);
        x[i] = (y & Magic<T>::kMask) | Magic<T>::kSixteen;
    }
    return x;
}

struct NibbleLds {
    union {
        struct {
            alignas(16) unsigned char v[4][kBlock * 64];
            alignas(16) unsigned char w[4][2][16 * kRowStride];       // weights, hi and lo parts
        };
        float rows[4][16][kHeadDim];                                  // at the end: the wavefronts' sums
    };
    float m[4][16], l[4][16];
    int pages[kMaxPages];
};

template <class T> __device__ __forceinline__ float scale_at(const unsigned *w, int i) { return (i & 1) ? T::hi(w[i >> 1]) : T::lo(w[i >> 1]); }

__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); __builtin_amdgcn_wave_barrier(); }

template <class T, int NG, int R> __global__ __launch_bounds__(256, 2) void nibble_attn_kernel(NibbleProblem p)
{
    __shared__ NibbleLds lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, c = lane >> 4;
    const int chunk = blockIdx.x % p.nc;
    int unit = blockIdx.x / p.nc;
    const int tile = unit % p.tiles;
    unit /= p.tiles;
    const int hkv = unit % p.pool.Hkv, b = unit / p.pool.Hkv;
    const int len = min(max(p.seq_lens[b], 0), p.Smax);
    const int start = chunk * p.C, end = min(len, start + p.C);
    const int heads = min(p.G - 16 * tile, 16), head0 = hkv * p.G + 16 * tile;      // query heads of this tile
    if (start >= end) {
        // a sequence without keys: zero rows, by the first chunk (chunks without keys leave nothing: the join knows the lengths)
        if (p.nc == 1)
            for (int i = tid; i < heads * kHeadDim / 2; i += 256) reinterpret_cast<unsigned *>(p.out + ((size_t)b * p.Hq + head0) * kHeadDim)[i] = 0u;
        return;
    }
    const int shift = p.pool.page_shift, mask = (1 << shift) - 1, first_page = start >> shift;
    const int used = ((end - 1) >> shift) - first_page + 1;
    for (int i = tid; i < used; i += 256) lds.pages[i] = min(max(p.table[(size_t)b * p.width + first_page + i], 0), p.pool.n_pages - 1);

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
    float qsum[NG][4];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        float s = 0.f;
#pragma unroll
        for (int t = 0; t < 4 / NG; ++t) s += qs[g * (4 / NG) + t];
#pragma unroll
        for (int r = 0; r < 4; ++r) qsum[g][r] = __shfl(s, 4 * c + r);
    }
    __syncthreads();

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

    constexpr int SW = NG;                         // 32-bit words of a row's scales
    u32x4_t kc[4], vc[4];
    unsigned ks[4][SW], vs[4][SW];
    // row 0 of the 16 keys from key0 (those behind the last key: of the last 16 that hold one)
    auto row_of = [&](int key0) -> size_t {
        const int k0 = min(key0, (end - 1) & ~15);
        const int page = __builtin_amdgcn_readfirstlane(lds.pages[(k0 >> shift) - first_page]);
        return (((size_t)page * p.pool.Hkv + hkv) << shift) + (k0 & mask);
    };
    auto load_scales = [&](const uint16_t *base, size_t row, unsigned (&w)[SW]) {
        const unsigned *at = reinterpret_cast<const unsigned *>(base) + (row + n) * SW;
        if constexpr (NG == 4) {
            const u32x4_t x = *reinterpret_cast<const u32x4_t *>(at);
            w[0] = x[0]; w[1] = x[1]; w[2] = x[2]; w[3] = x[3];
        } else if constexpr (NG == 2) {
            const u32x2_t x = *reinterpret_cast<const u32x2_t *>(at);
            w[0] = x[0]; w[1] = x[1];
        } else {
            w[0] = *at;
        }
    };
    auto load_block = [&](int key0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const size_t row = row_of(key0 + 16 * i);
            kc[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p.pool.k_codes + row * 64) + 4 * n + c);
            vc[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p.pool.v_codes + row * 64) + 4 * n + c);
            load_scales(p.pool.k_scales, row, ks[i]);
            load_scales(p.pool.v_scales, row, vs[i]);
        }
    };
    unsigned char *v_at = lds.v[wave], *w_hi = lds.w[wave][0], *w_lo = lds.w[wave][1];

    for (int key0 = start + kBlock * wave; key0 < end; key0 += 4 * kBlock) {
        load_block(key0);
        // scores, in units of log2
        float z[4][R];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[R];
#pragma unroll
            for (int r = 0; r < R; ++r) x[r] = 0.f;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                f32x4_t a = {-16.f * qsum[g][0], -16.f * qsum[g][1], -16.f * qsum[g][2], -16.f * qsum[g][3]};
#pragma unroll
                for (int t = 0; t < 4 / NG; ++t) a = T::mfma(qa[g * (4 / NG) + t], expand<T>(kc[i][g * (4 / NG) + t]), a);
                const float s = scale_at<T>(ks[i], g), lw = scale_at<T>(ks[i], NG + g);
#pragma unroll
                for (int r = 0; r < R; ++r) x[r] = __builtin_fmaf(s, a[r], __builtin_fmaf(lw, qsum[g][r], x[r]));
            }
            const bool live = key0 + 16 * i + n < end;
#pragma unroll
            for (int r = 0; r < R; ++r) z[i][r] = live ? x[r] * c1 : -INFINITY;
            // V's scales of keys that are not there may be anything
#pragma unroll
            for (int k = 0; k < SW; ++k) vs[i][k] = live ? vs[i][k] : 0u;
        }
        // V's codes into LDS: row of key k at 64 k, its 16-byte piece x in place x ^ ((k >> 2) & 3), with the halves of the odd 16 keys swapped
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u32x4_t x = (i & 1) ? u32x4_t{vc[i][2], vc[i][3], vc[i][0], vc[i][1]} : vc[i];
            *reinterpret_cast<u32x4_t *>(v_at + (16 * i + n) * 64 + ((c ^ ((n >> 2) & 3)) << 4)) = x;
        }
        // the running maximum; what was summed is brought to it where it grew
        bool grew = false;
        float mn[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float top = row16_max(fmaxf(fmaxf(z[0][r], z[1][r]), fmaxf(z[2][r], z[3][r])));
            mn[r] = fmaxf(m[r], top);
            grew |= mn[r] > m[r];
        }
        if (__any(grew)) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float f = mn[r] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[r] - mn[r]);
                l[r] *= f;
#pragma unroll
                for (int g = 0; g < NG; ++g) low[r][g] *= f;
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) acc[dt][r] *= f;
                m[r] = mn[r];
            }
        }
        // weights
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float e = __builtin_amdgcn_exp2f(z[i][r] - (m[r] == -INFINITY ? 0.f : m[r]));
                l[r] += e;
                z[i][r] = e;
            }
        const int slot = ((n >> 3) << 3) + ((n & 3) << 1) + ((n >> 2) & 1);           // of a key in its run of 16: as expand orders the codes
#pragma unroll
        for (int g = 0; g < NG; ++g) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float s = scale_at<T>(vs[i], g), lw = __builtin_fmaf(-16.f, s, scale_at<T>(vs[i], NG + g));
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    low[r][g] = __builtin_fmaf(z[i][r], lw, low[r][g]);
                    const float w = z[i][r] * s;
                    const unsigned short h = T::bits(w);
                    const unsigned short d = T::bits(w - T::lo(h));
                    const int at = (4 * c + r) * kRowStride + 32 * i + 2 * slot;
                    *reinterpret_cast<unsigned short *>(w_hi + at) = h;
                    *reinterpret_cast<unsigned short *>(w_lo + at) = d;
                }
            }
            wave_fence();
            // keys 16 c + 8 u .. + 7 of row n
            u32x4_t ah[2], al[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                ah[u] = *reinterpret_cast<const u32x4_t *>(w_hi + n * kRowStride + 32 * c + 16 * u);
                al[u] = *reinterpret_cast<const u32x4_t *>(w_lo + n * kRowStride + 32 * c + 16 * u);
            }
#pragma unroll
            for (int d = 0; d < 8 / NG; ++d) {
                const int dt = g * (8 / NG) + d;
                typedef int i32x2 __attribute__((ext_vector_type(2)));
                typedef __attribute__((address_space(3))) i32x2 *lds_i32x2;
                // 16 elements from 16 dt of key 16 c + n: lane n receives element n of the 16 keys
                unsigned char *at = v_at + (16 * c + n) * 64 + (((dt >> 1) ^ ((n >> 2) & 3)) << 4) + (((dt & 1) ^ (c & 1)) << 3);
                const i32x2 x = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2)at);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const u32x4_t vb = expand<T>((unsigned)x[u]);
                    acc[dt] = T::mfma(ah[u], vb, acc[dt]);
                    acc[dt] = T::mfma(al[u], vb, acc[dt]);
                }
            }
            wave_fence();
        }
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
            lds.m[wave][4 * c + r] = m[r];
            lds.l[wave][4 * c + r] = ls;
        }
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) lds.rows[wave][4 * c + r][16 * dt + n] = acc[dt][r] + lw[dt * NG / 8];
    }
    __syncthreads();
    for (int i = tid; i < heads * (kHeadDim / 2); i += 256) {
        const int h = i >> 6, d = (i & 63) * 2, row = 4 * (h & 3) + (h >> 2);
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, lds.m[w][row]);
        float a0 = 0.f, a1 = 0.f, sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float mw = lds.m[w][row];
            // a wavefront without keys has m = -inf and zeros; one whose logits are all -inf or NaN has NaN, and keeps it
            const float f = mw == top ? 1.f : __builtin_amdgcn_exp2f(mw - top);
            const float2 x = *reinterpret_cast<const float2 *>(&lds.rows[w][row][d]);
            a0 = __builtin_fmaf(x.x, f, a0);
            a1 = __builtin_fmaf(x.y, f, a1);
            sum = __builtin_fmaf(lds.l[w][row], f, sum);
        }
        const size_t out_row = (size_t)b * p.Hq + head0 + h;
        if (p.nc == 1) {
            const float inv = 1.f / sum;
            *reinterpret_cast<unsigned *>(p.out + out_row * kHeadDim + d) = T::pack(a0 * inv, a1 * inv);
        } else {
            *reinterpret_cast<float2 *>(p.num + (out_row * p.nc + chunk) * kHeadDim + d) = float2{a0, a1};
            if (d == 0) p.ml[out_row * p.nc + chunk] = float2{top, sum};
        }
    }
}

// ---- the join of rows that several workgroups share ----
// A workgroup a row.  Its length is that of its loads, so all of them are asked for together: first the references and denominators of 64 chunks, then, with
// their factors in LDS, eight partial vectors at a time.
constexpr int kJoinWindow = 64;
template <class T, int DIM> __global__ __launch_bounds__(DIM / 2) void join_kernel(JoinProblem p)
{
    __shared__ float factor[kJoinWindow];
    const int row = blockIdx.x, b = row / p.H, tid = threadIdx.x, lane = tid & 63;
    const int len = min(max(p.seq_lens[b], 0), p.Smax), nb = (len + p.C - 1) / p.C;
    unsigned *out = reinterpret_cast<unsigned *>(p.out + (size_t)row * DIM) + tid;
    if (nb == 0) { *out = 0u; return; }
    const float2 *ml = p.ml + (size_t)row * p.nc;
    const float *num = p.num + (size_t)row * p.nc * DIM + 2 * tid;
    float top = -INFINITY, a0 = 0.f, a1 = 0.f, sum = 0.f;
    for (int w0 = 0; w0 < nb; w0 += kJoinWindow) {
        const int count = min(nb - w0, kJoinWindow);
        float2 s = {-INFINITY, 0.f};
        if (lane < count) s = ml[w0 + lane];
        float t = columns_max(row16_max(s.x));
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
        for (int i = 0; i < count; i += 8) {
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
    const float inv = 1.f / sum;
    *out = T::pack(a0 * inv, a1 * inv);
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

hipError_t launch_nibble_write(const NibblePool &pool, const NibbleRows &rows, hipStream_t s)
{
    const dim3 grid((unsigned)(((long long)rows.n_tokens * 2 * pool.Hkv + 15) / 16));
    return pool.dtype == kF16 ? launch(nibble_write_kernel<F16>, grid, dim3(256), s, pool, rows) : launch(nibble_write_kernel<BF16>, grid, dim3(256), s, pool, rows);
}
hipError_t launch_nibble_read(const NibblePool &pool, const NibbleRows &rows, hipStream_t s)
{
    const dim3 grid((unsigned)(((long long)rows.n_tokens * 2 * pool.Hkv + 15) / 16));
    return pool.dtype == kF16 ? launch(nibble_read_kernel<F16>, grid, dim3(256), s, pool, rows) : launch(nibble_read_kernel<BF16>, grid, dim3(256), s, pool, rows);
}
hipError_t launch_join(const JoinProblem &p, hipStream_t s)
{
    const dim3 grid((unsigned)p.rows), block((unsigned)p.dim / 2);
    if (p.dim == kHeadDim)
        return p.dtype == kF16 ? launch(join_kernel<F16, kHeadDim>, grid, block, s, p) : launch(join_kernel<BF16, kHeadDim>, grid, block, s, p);
    return p.dtype == kF16 ? launch(join_kernel<F16, 512>, grid, block, s, p) : launch(join_kernel<BF16, 512>, grid, block, s, p);
}
hipError_t launch_nibble_attn(const NibbleProblem &p, hipStream_t s)
{
    const hipError_t e = p.pool.dtype == kF16 ? attn_groups<F16>(p, s) : attn_groups<BF16>(p, s);
    if (e != hipSuccess || p.nc == 1) return e;
    JoinProblem j{p.num, p.ml, p.seq_lens, p.out, p.B * p.Hq, p.Hq, p.C, p.nc, p.Smax, kHeadDim, p.pool.dtype};
    return launch_join(j, s);
}

}  // namespace fd
