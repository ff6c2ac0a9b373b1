// Latent attention over a paged cache: one row of 576 elements a token -- 512 that stand for the keys and values of all
// heads, 64 rotary ones that all heads share -- and queries that the caller has taken into the latent space (the absorbed
// form):
//     x_j = scale (q_latent . c_j + q_rope . r_j),   out = sum_j softmax(x)_j c_j.
// Every head reads the same rows, as keys and as values: a row is fetched once for up to 128 heads.
#include "fd_chunk.h"
#include "fd_cache.h"
#include "fd_types.h"

namespace fd {

namespace {

// ---- rows into the cache: 72 pieces of 16 bytes a row, 64 of the latent part and 8 of the rotary one ----
constexpr int kPieces = kLatentRow / 8, kWriteTokens = 4;      // tokens of a workgroup: a thread a piece
__global__ __launch_bounds__(kPieces * kWriteTokens)
void latent_write_kernel(LatentPool pool, const uint16_t *latent, long long latent_stride, const uint16_t *rope,
                         long long rope_stride, int n_tokens, const int32_t *slots)
{
    const int i = threadIdx.x / kPieces, piece = threadIdx.x - i * kPieces, token = blockIdx.x * kWriteTokens + i;
    if (token >= n_tokens) return;
    const int slot = slots[token];
    const uint16_t *from = piece < kLatent / 8 ? latent + token * latent_stride + 8 * piece
                                               : rope + token * rope_stride + (8 * piece - kLatent);
    const u32x4_t x = *reinterpret_cast<const u32x4_t *>(from);
    if (slot < 0 || (slot >> pool.page_shift) >= pool.n_pages) return;      // padding
    *reinterpret_cast<u32x4_t *>(pool.rows + (size_t)slot * kLatentRow + 8 * piece) = x;
}

// ---- attention ----
//
// Matrix-core mapping (16 x 16 x 32; lane = (n, g) = (lane % 16, lane / 16)):
//   scores   S^T[key][head] = C . Q^T: A = 16 rows of the tile in LDS, B = Q^T in registers for the whole kernel (18
//            operands).  Row 4 g + r of key block t is key 8 g + 4 t + r of the tile, so that the two blocks leave lane (n,
//            g) holding keys 8 g .. 8 g + 7 of head n: the B operand of
//   output   O^T[d][head] = C^T . P^T: A = the same rows, turned round by the transposing LDS read.  32 tiles of 16 elements.
// The weights enter as the sum of two numbers of the type (hi + lo), since one alone adds an error as large as the output's
// rounding, and the second half of the instructions is hidden behind memory; of more than 64 heads, where the matrix cores
// are the bound, as one, and their sum is that of the rounded ones (64 x 128 heads x 4096 keys: 106 us with two, 93 with
// one).
// A wavefront owns 16 heads: 72 registers of queries and 128 of sums.  A workgroup of NW wavefronts takes 16 NH heads of a
// sequence and a chunk of its keys, TPW tiles of 32 at a time, which all its wavefronts fetch straight into LDS while they
// work on those before.  Where there are fewer heads than wavefronts, DS = NW / NH of them share 16 heads: of the scores
// each forms a part (one of the two key blocks, of four wavefronts every other operand of one) and finds the others' in
// LDS, then all form the weights, and each adds up its part of the elements (all scores by each: 1 x 16 heads x 2048 keys
// 10.9 us, 8.9 so).
// What bounds it, of 256 sequences x 1024 keys in one chunk each: memory for 16 and 32 heads (52 and 58 us, 5.8 and 5.2
// TB/s), waits within a tile for 64 and 128 (74 and 92 us; of 128 heads matrix instructions fill 43 % of the cycles, LDS 42
// %).
constexpr int kTile = 32;
// The reference of a head's weights follows its maximum only where that has grown by more than this (in units of log2):
// weights are at most 2^8 times the reference's then, and the sums, 128 registers of a wavefront, are brought to another
// reference once or twice a chunk; of 16 heads some maximum grows in most tiles.
constexpr float kSlack = 8.f;
constexpr int kRowBytes = kLatentRow * 2;                      // in the cache
constexpr int kCBytes = kLatent * 2, kRBytes = kRope * 2;      // in LDS the two parts of a row lie apart

// Steps in LDS: one in work, one under way.  Two workgroups of up to 64 heads fit a compute unit, which covers the loads
// better than one with four steps: 16 x 64 heads x 2000 keys 30.1 / 31.7 us, 64 x 16 x 1000 25.3 / 26.9; in long launches
// it is the other way round, 64 x 64 x 4000 88.7 / 86.6.
constexpr int kSteps = 2;
template <int NW, int DS, int TPW> struct LatentLds {
    alignas(256) unsigned char c[kSteps * TPW][kTile * kCBytes];      // piece x (16 bytes) of row r in place x ^ c_key(r)
    alignas(256) unsigned char r[kSteps * TPW][kTile * kRBytes];      // ... x ^ r_key(r)
    alignas(256) f32x4_t x[NW / DS][DS][DS == 1 ? 1 : 64];               // parts of the scores of 16 heads
};
// A cycle of the 16-byte operand reads holds every n once, from two neighbouring g: with these keys the 16 pieces lie in 16
// different places modulo 256 bytes.  The transposing reads take 32 bytes of eight rows at a time, 8 g + 4 h + (0 .. 3) of
// two neighbouring g: in eight different places.  Rows r and r + 4 have the same keys.
__device__ __forceinline__ constexpr int c_key(int r) { return ((r & 1) << 1) | (((r >> 1) & 1) << 2) | (((r >> 3) & 1) << 3); }
__device__ __forceinline__ constexpr int r_key(int r) { return (((r >> 3) & 1) << 1) | (((r >> 1) & 1) << 2); }

// (in assembly: of loads into LDS that the compiler knows it would wait before every transposing read)
__device__ __forceinline__ void load_to_lds(u32x4_t rs, int voff, int soff, unsigned lds_1k)
{
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"{m0}"(lds_1k), "v"(voff), "s"(rs), "s"(soff) : "memory");
}
__device__ __forceinline__ unsigned lds_address(const void *p)
{
    return __builtin_amdgcn_readfirstlane(
        (unsigned)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const unsigned char *)p));
}
__device__ __forceinline__ void wait_fetches() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void tile_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);                        // this wavefront's LDS reads have arrived
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t *lds_s16x4;
typedef __attribute__((address_space(3))) const u32x4_t *lds_u32x4;
typedef __attribute__((address_space(4))) const int32_t *scalar_i32;      // read through the scalar cache

template <class T, int NW, int DS, int TPW> __global__ __launch_bounds__(64 * NW, 2) void latent_decode_kernel(LatentProblem p)
{
    // (a step's tiles are taken together: their weights wait for one maximum, their reads run ahead over both -- 256
    // sequences of 1024 keys, 128 heads: 101 us one by one, 97 so, 92 with the scaling in the exponents' multiply-adds and
    // the sum of weights on the matrix cores)
    constexpr int NH = NW / DS, kDt = 32 / DS;                 // groups of 16 heads; tiles of 16 elements of a wavefront
    constexpr bool kTwoParts = NW < 8;                         // of a weight
    constexpr int kKeys = TPW * kTile, kRows = 8;              // keys of a step; rows that a wavefront fetches, all of one page
    static_assert(kKeys == NW * kRows && kSteps == 2);
    // of the scores, of a wavefront
    constexpr int kParts = DS == 4 ? 2 : 1, kBlocks = DS == 1 ? 2 : 1, kOperands = 18 / kParts;
    __shared__ LatentLds<NW, DS, TPW> lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    // workgroups that read the same rows lie on one XCD (index modulo 8), one after the other
    const int tiles = (p.H + 16 * NH - 1) / (16 * NH), units = p.B * p.nc;
    const int unit = (blockIdx.x / (8 * tiles)) * 8 + blockIdx.x % 8;
    const int head0 = (blockIdx.x / 8 % tiles) * (16 * NH) + 16 * (wave % NH), d0 = wave / NH * (16 * kDt);
    if (unit >= units) return;
    const int chunk = unit % p.nc, b = unit / p.nc;
    const int start = chunk * p.C, shift = p.pool.page_shift, mask = (1 << shift) - 1;
    const scalar_i32 table = (scalar_i32)(uintptr_t)(p.table + (size_t)b * p.width);
    // page of this wavefront's rows in step s (of the last entry, behind the table)
    auto page_of = [&](int s) { return table[min((start + s * kKeys + wave * kRows) >> shift, p.width - 1)]; };
    int page = page_of(0);
    const int len = min(max(((scalar_i32)(uintptr_t)p.seq_lens)[b], 0), p.Smax);
    const int end = min(len, start + p.C);
    const int heads = min(p.H - head0, 16);                    // of this wavefront; may be 0 or less: it only fetches
    if (start >= end) {
        if (chunk == 0)                                        // no keys at all: zero rows
            for (int h = wave / NH; h < heads; h += DS)
                reinterpret_cast<u32x4_t *>(p.out + ((size_t)b * p.H + head0 + h) * kLatent)[lane] = u32x4_t{0u, 0u, 0u, 0u};
        return;
    }

    // Fetches: 1 KiB an instruction, the latent part of a row, or the rotary parts of eight; what lies behind the last key
    // arrives as zeros.
    const int steps = (end - start + kKeys - 1) / kKeys;
    const unsigned lds_c = lds_address(lds.c[0]), lds_r = lds_address(lds.r[0]);
    auto fetch = [&](int s) {
        int l0 = lane;
        asm volatile("" : "+v"(l0));    // (offsets are formed anew each time: there are no registers to keep them in)
        const unsigned to_c = lds_c + s % kSteps * (kKeys * kCBytes) + wave * (kRows * kCBytes);
        const unsigned to_r = lds_r + s % kSteps * (kKeys * kRBytes) + wave * (kRows * kRBytes);
        const int key0 = start + s * kKeys + wave * kRows;
        const int left = min(max(end - key0, 0), kRows);
        const int pg = min(max(page, 0), p.pool.n_pages - 1);
        const unsigned long long at =
            reinterpret_cast<unsigned long long>(p.pool.rows) + (((size_t)pg << shift) + (key0 & mask)) * kRowBytes;
        const u32x4_t rs = {(unsigned)__builtin_amdgcn_readfirstlane((unsigned)at),
                            (unsigned)__builtin_amdgcn_readfirstlane((unsigned)(at >> 32)) & 0xffffu,
                            (unsigned)__builtin_amdgcn_readfirstlane(left * kRowBytes), 0x00027000u};
        const int odd = wave & 1;                              // (bit 3 of the row, which is in the keys)
#pragma unroll
        for (int i = 0; i < kRows; ++i) load_to_lds(rs, (l0 ^ c_key(i) ^ (odd << 3)) << 4, i * kRowBytes, to_c + i * kCBytes);
        const int r = l0 >> 3;
        load_to_lds(rs, r * kRowBytes + kCBytes + (((l0 & 7) ^ r_key(r) ^ (odd << 1)) << 4), 0, to_r);
        page = page_of(s + 1);
    };
    fetch(0);

    // this wavefront's part of the scores: key block t (or both), operands kParts i + odd
    const int part = DS == 1 ? 0 : wave / NH, odd = part / 2;
    u32x4_t q[kOperands];
#pragma unroll
    for (int i = 0; i < kOperands; ++i) {
        q[i] = u32x4_t{0u, 0u, 0u, 0u};
        if (n < heads) {
            const size_t row = (size_t)b * p.H + head0 + n;
            const int kb = kParts * i + odd;
            q[i] = *reinterpret_cast<const u32x4_t *>(kParts * i < 16 ? p.q_latent + row * kLatent + 32 * kb + 8 * g
                                                                      : p.q_rope + row * kRope + 32 * (kb - 16) + 8 * g);
        }
        q[i] ^= p.scale < 0.f ? 0x80008000u : 0u;               // (the largest product is then the largest logit)
    }
    f32x4_t acc[kDt];
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt) acc[dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    // of rounded weights, in every element (C^T of ones); else of this lane's, in l
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
    const unsigned one2 = T::pack(1.f, 1.f);
    // (not 0: of a masked score it has to leave -inf; the smallest number, of other scores nothing)
    const float c1 = fmaxf(fabsf(p.scale) * kLog2e, 0x1p-149f);
    // this lane's operand reads: piece 4 kb + g of row k_row; 32 bytes from element 16 dt of row v_row.  Pieces within 256
    // bytes differ by an exclusive or.
    const int k_row = 8 * (n >> 2) + (n & 3), v_row = 8 * g + (n >> 2);
    const int k_first = k_row + (DS == 1 ? 0 : 4 * (part & 1));
    const unsigned k_at = k_first * kCBytes + ((g ^ c_key(k_row)) << 4 ^ odd << 6);
    const unsigned kr_at = k_first * kRBytes + ((g ^ r_key(k_row)) << 4 ^ odd << 6);
    const unsigned v_at = v_row * kCBytes + (((n >> 1) & 1) << 4) + ((n & 1) << 3) + (c_key(v_row) << 4);

    // the queries, and with them step 0 (the compiler, which does not count the fetches, would wait within the loop)
    __builtin_amdgcn_s_waitcnt(0x0f70);

    for (int s = 0; s < steps; ++s) {
        wait_fetches();                                        // step s
        tile_barrier();                                        // ... for every wavefront, all of which are through with step s - 1
        fetch(s + 1);                                          // (behind the last step: nothing)
        if (heads <= 0) continue;
        const unsigned tile_c = lds_c + s % kSteps * (kKeys * kCBytes), tile_r = lds_r + s % kSteps * (kKeys * kRBytes);
        f32x4_t sc[TPW][2];
        {
            const unsigned kc = tile_c + k_at, kr = tile_r + kr_at;
            auto read = [&](int op) {                          // of tile op / kOperands / kBlocks
                const int i = op / (kOperands * kBlocks), t = op % kBlocks, kb = op / kBlocks % kOperands * kParts;
                const unsigned x = kb < 16 ? (kc ^ ((kb & 3) << 6)) + ((kb >> 2) << 8) + t * 4 * kCBytes + i * (kTile * kCBytes)
                                           : (kr ^ ((kb & 1) << 6)) + t * 4 * kRBytes + i * (kTile * kRBytes);
                return *(lds_u32x4)(uintptr_t)x;
            };
            // reads run kAhead operands ahead of the instructions that use them
            constexpr int kOps = TPW * kOperands * kBlocks, kAhead = 3;
            u32x4_t a[kAhead + 2];
#pragma unroll
            for (int i = 0; i < TPW; ++i) sc[i][0] = sc[i][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int op = 0; op < kAhead; ++op) a[op] = read(op);
#pragma unroll
            for (int op = 0; op < kOps; op += kBlocks) {
#pragma unroll
                for (int t = 0; t < kBlocks; ++t)
                    if (op + t + kAhead < kOps) a[(op + t + kAhead) % (kAhead + 2)] = read(op + t + kAhead);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int t = 0; t < kBlocks; ++t) {
                    // (of one block: two chains)
                    const int i = op / (kOperands * kBlocks), at = op / kBlocks % kOperands, to = kBlocks == 1 ? at & 1 : t;
                    sc[i][to] = T::mfma(a[(op + t) % (kAhead + 2)], q[at], sc[i][to]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if constexpr (DS > 1) {                                // the wavefronts of 16 heads exchange their parts
            static_assert(TPW == 1);
            lds.x[wave % NH][part][lane] = sc[0][0] + sc[0][1];
            tile_barrier();
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                sc[0][t] = lds.x[wave % NH][t][lane];
                if constexpr (DS == 4) sc[0][t] += lds.x[wave % NH][t + 2][lane];
            }
        }
        const unsigned vc = tile_c + v_at + 2 * d0;
        // the output's operands: two tiles of elements, each of all tiles of keys, and on
        auto read = [&](int op) {
            const int dt = op / (2 * TPW) * 2 + op % 2, i = op / 2 % TPW;
            const unsigned x = (vc ^ ((dt & 7) << 5)) + ((dt >> 3) << 8) + i * (kTile * kCBytes);
            const s16x4_t u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)x);
            const s16x4_t w = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(x + 4 * kCBytes));
            return __builtin_bit_cast(u32x4_t, __builtin_shufflevector(u, w, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        constexpr int kOps = TPW * kDt, kAhead = 4;
        u32x4_t a[kAhead + 2];
#pragma unroll
        for (int op = 0; op < kAhead; ++op) a[op] = read(op);
        __builtin_amdgcn_sched_barrier(0);

        const int left = end - (start + s * kKeys);            // keys from the step's first
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < TPW; ++i) {
            if (left < kKeys) {
#pragma unroll
                for (int j = 0; j < 8; ++j) sc[i][j >> 2][j & 3] = kTile * i + 8 * g + j < left ? sc[i][j >> 2][j & 3] : -INFINITY;
            }
            // (of a NaN or not: of one the output is NaN anyway)
#pragma unroll
            for (int j = 0; j < 8; ++j) top = __builtin_elementwise_maximum(top, sc[i][j >> 2][j & 3]);
        }
        top = columns_max(top) * c1;
        if (__any(top > m + kSlack)) {                         // (also where there is no reference yet)
            const float to = fmaxf(m, top), f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
            l *= f;
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[r] *= f;
#pragma unroll
            for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[dt][r] *= f;
            m = to;
        }
        const float ref = (m == -INFINITY ? 0.f : m) - T::kLift;
        u32x4_t hi[TPW], lo[TPW];
#pragma unroll
        for (int i = 0; i < TPW; ++i)
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i][j >> 2][j & 3], c1, -ref));
                const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i][j >> 2][(j & 3) + 1], c1, -ref));
                const unsigned h = T::pack(e0, e1);
                hi[i][j >> 1] = h;
                if constexpr (kTwoParts) {
                    l += e0 + e1;
                    lo[i][j >> 1] = T::pack(e0 - T::lo(h), e1 - T::hi(h));
                }
            }
        if constexpr (!kTwoParts)
#pragma unroll
            for (int i = 0; i < TPW; ++i) sum = T::mfma(u32x4_t{one2, one2, one2, one2}, hi[i], sum);
#pragma unroll
        for (int op = 0; op < kOps; op += 2) {
            const int dt = op / (2 * TPW) * 2, i = op / 2 % TPW;
#pragma unroll
            for (int d = 0; d < 2; ++d)
                if (op + d + kAhead < kOps) a[(op + d + kAhead) % (kAhead + 2)] = read(op + d + kAhead);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int d = 0; d < 2; ++d) acc[dt + d] = T::mfma(a[(op + d) % (kAhead + 2)], hi[i], acc[dt + d]);
            if constexpr (kTwoParts)
#pragma unroll
                for (int d = 0; d < 2; ++d) acc[dt + d] = T::mfma(a[(op + d) % (kAhead + 2)], lo[i], acc[dt + d]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    wait_fetches();                                            // (nothing may land in LDS after the workgroup's end)
    if (n >= heads) return;
    if constexpr (kTwoParts) {
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
    } else {
        l = sum[0];
    }
    const size_t row = (size_t)b * p.H + head0 + n;
    if (len <= p.C) {                                          // the only chunk with keys
        const float inv = 1.f / l;
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt)
            *reinterpret_cast<u32x2_t *>(p.out + row * kLatent + d0 + 16 * dt + 4 * g) =
                u32x2_t{T::pack(acc[dt][0] * inv, acc[dt][1] * inv), T::pack(acc[dt][2] * inv, acc[dt][3] * inv)};
    } else {
        float *num = p.num + (row * p.nc + chunk) * kLatent;
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt) *reinterpret_cast<f32x4_t *>(num + d0 + 16 * dt + 4 * g) = acc[dt];
        if (g == 0 && d0 == 0) p.ml[row * p.nc + chunk] = float2{m, l};
    }
}

template <class T, int NW, int DS, int TPW> hipError_t decode(const LatentProblem &p, hipStream_t s)
{
    constexpr int heads = 16 * NW / DS;
    const long long tiles = (p.H + heads - 1) / heads, units = (long long)p.B * p.nc;
    return launch(latent_decode_kernel<T, NW, DS, TPW>, dim3((unsigned)((units + 7) / 8 * 8 * tiles)), dim3(64 * NW), s, p);
}
template <class T> hipError_t decode_heads(const LatentProblem &p, hipStream_t s)
{
    if (p.H > 64) return decode<T, 8, 1, 2>(p, s);
    if (p.H > 32) return decode<T, 4, 1, 1>(p, s);
    return p.H > 16 ? decode<T, 4, 2, 1>(p, s) : decode<T, 4, 4, 1>(p, s);
}

}  // namespace

hipError_t launch_latent_write(const LatentPool &pool, const uint16_t *latent, long long latent_stride, const uint16_t *rope,
                               long long rope_stride, int n_tokens, const int32_t *slots, hipStream_t s)
{
    const dim3 grid((unsigned)((n_tokens + kWriteTokens - 1) / kWriteTokens));
    return launch(latent_write_kernel, grid, dim3(kPieces * kWriteTokens), s, pool, latent, latent_stride, rope, rope_stride,
                  n_tokens, slots);
}
hipError_t launch_latent_decode(const LatentProblem &p, hipStream_t s)
{
    const hipError_t e = p.pool.dtype == kF16 ? decode_heads<F16>(p, s) : decode_heads<BF16>(p, s);
    if (e != hipSuccess || p.nc == 1) return e;
    JoinProblem j{p.num, p.ml, p.seq_lens, p.out, p.B * p.H, p.H, p.C, p.nc, p.Smax, kLatent, p.pool.dtype};
    return launch_join(j, s);
}

}  // namespace fd
