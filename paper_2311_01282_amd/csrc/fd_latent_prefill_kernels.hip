// Prompts with latent attention in the expanded form: every head has keys of 128 elements and 64 rotary ones that all heads
// share, values of 128, and token i attends to tokens 0 .. i.  Operands lie token by token, as projections leave them.
//
// Mapping as in the prompt kernel of the equal-sized heads (16 x 16 x 32; lane = (n, g) = (lane % 16, lane / 16)): a
// workgroup owns 128 queries of a head, a wavefront 32 of them in two blocks of 16;
//   scores   S^T[key][query] = K . Q^T: A = 16 keys of the tile in LDS, B = Q^T in registers.  Row 4 g + r of key block t
//            is key 8 g + 4 t + r of the 32 of a step, so that lane (n, g) holds keys 8 g .. 8 g + 7 of query n: the B
//            operand of
//   output   O^T[d][query] = V^T . P^T: A = V^T by the transposing LDS read.
// Where a launch has few workgroups, a workgroup is two such halves that take every other step and join their sums at the
// end (kHalves).
// Softmax with a running maximum per query; the weights are of the type (one rounding, as large as the output's own), their
// sum is that of the rounded ones, in fp32.
// The matrix cores bound long prompts, at the clock that power leaves them: 64 heads x 4001 tokens 331 .. 373 us, 0.88 ..
// 0.99 PFLOP/s of what the mask leaves, matrix instructions in 53 % of the cycles; short ones the length of a tile's walk.
#include <utility>

#include "fd_chunk.h"
#include "fd_cache.h"
#include "fd_finite.h"

namespace fd {

namespace {

constexpr int kNope = 128, kQueryDim = kNope + kRope, kStep = 32, kTileQ = 128, kRingK = 4, kRingV = 3;
// The reference of a query's weights follows its maximum only where that has grown by more than this (in units of log2):
// weights are then at most 2^8 times the reference's, and the sums are brought to another reference a few times a row
// instead of at every new maximum.
constexpr float kSlack = 8.f;

struct PromptLds {
    alignas(256) unsigned char k[kRingK][kStep * kNope * 2];    // piece x (16 bytes) of row r in place x ^ k_place(r)
    alignas(256) unsigned char r[kRingK][kStep * kRope * 2];    // ... x ^ r_place(r)
    alignas(256) unsigned char v[kRingV][kStep * kNope * 2];    // 32-byte unit x of row r in place x ^ v_unit(r)
};
// With these the 16-byte operand reads, whose cycles hold every n once from two neighbouring g, and the transposing reads,
// which take 32 bytes of rows 8 g + 4 h + (0 .. 3) of two neighbouring g at a time, have no bank conflicts.
__device__ __forceinline__ int k_place(int r) { return (r & 3) | (((r >> 3) & 3) << 2); }
__device__ __forceinline__ int r_place(int r) { return 2 * ((r >> 3) & 1) + 4 * ((r >> 1) & 1); }
__device__ __forceinline__ int v_unit(int r) { return (r & 3) | (((r >> 3) & 1) << 2); }

__device__ __forceinline__ unsigned lds_address(const void *p)
{
    return __builtin_amdgcn_readfirstlane(
        (unsigned)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const unsigned char *)p));
}
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t *lds_s16x4;
typedef __attribute__((address_space(3))) u32x4_t *lds_u32x4;
// (In assembly: of loads into LDS that the compiler knows it would wait before every transposing read.  That the window's scalar
// registers have settled, five states behind a vector instruction, is as the code around it comes out; tests/test_wait_states_host.py
// follows them through the assembly.)
__device__ __forceinline__ void load_to_lds(u32x4_t rs, int voff, int soff, unsigned lds_1k)
{
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"{m0}"(lds_1k), "v"(voff), "s"(rs), "s"(soff) : "memory");
}
template <class F, int... I> __device__ __forceinline__ void slots(std::integer_sequence<int, I...>, F f)
{
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N> __device__ __forceinline__ void wait_fetches() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void tile_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ u32x4_t window(const void *base, long long bytes)
{
    const unsigned long long at = reinterpret_cast<unsigned long long>(base);
    return u32x4_t{(unsigned)__builtin_amdgcn_readfirstlane((unsigned)at),
                   (unsigned)__builtin_amdgcn_readfirstlane((unsigned)(at >> 32)) & 0xffffu,
                   (unsigned)__builtin_amdgcn_readfirstlane((unsigned)bytes), 0x00027000u};
}

template <class T, int kHalves> __global__ __launch_bounds__(256 * kHalves, 2) void latent_prefill_kernel(LatentPromptProblem p)
{
    __shared__ union { PromptLds ring[kHalves]; f32x4_t sums[4][18][64]; } both;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6) & 3, n = lane & 15, g = lane >> 4;
    const int half = kHalves == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 8);      // takes the steps half, half + kHalves, ...
    PromptLds &lds = both.ring[half];
    // The longest walks first.  An XCD (index modulo 8) takes neighbouring heads, all tiles of a head on one: its keys and
    // values are read into one L2 only.  (Heads dealt out to the XCDs in turn measured the same.)
    const int pairs = p.B * p.H, per = (pairs + 7) / 8, tiles = (p.Smax + kTileQ - 1) / kTileQ;
    const int at = blockIdx.x % (8 * per), pair = at % 8 * per + at / 8, i0 = (tiles - 1 - blockIdx.x / (8 * per)) * kTileQ;
    if (pair >= pairs) return;
    const int b = pair / p.H, h = pair % p.H;
    const int S = min(max(p.seq_lens[b], 0), p.Smax);
    const int w0 = i0 + 32 * wave;
    uint16_t *out = p.out + ((size_t)b * p.Smax * p.H + h) * kNope;
    const size_t out_stride = (size_t)p.H * kNope;
    if (i0 >= S) {                                             // rows past the prompt: zeros
        for (int i = i0 + (tid >> 4); i < min(i0 + kTileQ, p.Smax); i += 16 * kHalves)
            *reinterpret_cast<u32x4_t *>(out + i * out_stride + 8 * (tid & 15)) = u32x4_t{0u, 0u, 0u, 0u};
        return;
    }
    // this half's steps, of the workgroup (the first half has as many or one more) and of the wavefront, whose last step of
    // all is the one with masks
    const int steps = ((min(i0 + kTileQ, S) - 1) / kStep + kHalves) / kHalves;
    const int all = w0 < S ? (min(w0 + 32, S) - 1) / kStep + 1 : 0, mine = (all - half + kHalves - 1) / kHalves;

    const unsigned lds_k = lds_address(lds.k[0]), lds_r = lds_address(lds.r[0]), lds_v = lds_address(lds.v[0]);
    u32x4_t q[2][6];
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        int row = w0 + 16 * qb + n;
        asm volatile("" : "+v"(row));                          // (nothing of these addresses is kept for the output's)
#pragma unroll
        for (int kb = 0; kb < 6; ++kb) {
            q[qb][kb] = u32x4_t{0u, 0u, 0u, 0u};
            const uint16_t *from = p.q + (((size_t)b * p.Smax + row) * p.H + h) * kQueryDim + 32 * kb + 8 * g;
            if (row < S) q[qb][kb] = *reinterpret_cast<const u32x4_t *>(from);
            q[qb][kb] ^= p.scale < 0.f ? 0x80008000u : 0u;     // (the largest product is then the largest logit)
        }
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);                        // the queries have arrived: what is counted from here on are fetches

    // A wavefront's five of the 20 KiB of a step: rows 8 wave .. + 7 of the keys and of the values, four rows an
    // instruction, of the rotary parts all eight.
    // (The places of rows r and r + 4 are the same: the second instruction is the first, four rows on.)
    const int row_bytes = p.H * (2 * kNope * 2), rope_bytes = (int)(p.rope_stride * 2);
    int koff, voff, roff;
    {
        const int r = 8 * wave + (lane >> 4), x = lane & 15, rr = 8 * wave + (lane >> 3);
        koff = r * row_bytes + ((x ^ k_place(r)) << 4);
        voff = r * row_bytes + ((x ^ (v_unit(r) << 1)) << 4);
        roff = rr * rope_bytes + (((lane & 7) ^ r_place(rr)) << 4);
    }
    // The fetches walk along the rows: a place in memory, the rows left from there, a place in the ring.  Rows without keys
    // arrive as zeros.
    struct Walk { const unsigned char *from; int left; unsigned to; };
    const unsigned char *kv = reinterpret_cast<const unsigned char *>(p.kv) + ((size_t)b * p.Smax * p.H + h) * (2 * kNope * 2);
    const int skip = half * kStep;
    Walk wk = {kv + (size_t)skip * row_bytes, S - skip, 0u}, wv = {kv + (size_t)skip * row_bytes + kNope * 2, S - skip, 0u};
    const unsigned char *rope_from = reinterpret_cast<const unsigned char *>(p.rope) + ((size_t)b * p.Smax + skip) * rope_bytes;
    auto bytes_of = [&](int left, int stride, int row) {
        const int rows = min(left, kStep);
        return rows > 0 ? (rows - 1) * stride + row : 0;
    };
    auto fetch_k = [&] {
        const u32x4_t rk = window(wk.from, bytes_of(wk.left, row_bytes, kNope * 2));
#pragma unroll
        for (int k = 0; k < 2; ++k) load_to_lds(rk, koff, 4 * k * row_bytes, lds_k + wk.to * (kStep * kNope * 2) + (2 * wave + k) * 1024);
        wk.from += (size_t)kHalves * kStep * row_bytes;
    };
    auto fetch_r = [&] {                                       // behind fetch_k
        const u32x4_t rr = window(rope_from, bytes_of(wk.left, rope_bytes, kRope * 2));
        load_to_lds(rr, roff, 0, lds_r + wk.to * (kStep * kRope * 2) + wave * 1024);
        rope_from += (size_t)kHalves * kStep * rope_bytes;
        wk.left -= kHalves * kStep;
        wk.to = wk.to == kRingK - 1 ? 0 : wk.to + 1;
    };
    auto fetch_v = [&] {
        const u32x4_t rv = window(wv.from, bytes_of(wv.left, row_bytes, kNope * 2));
#pragma unroll
        for (int k = 0; k < 2; ++k) load_to_lds(rv, voff, 4 * k * row_bytes, lds_v + wv.to * (kStep * kNope * 2) + (2 * wave + k) * 1024);
        wv.from += (size_t)kHalves * kStep * row_bytes;
        wv.left -= kHalves * kStep;
        wv.to = wv.to == kRingV - 1 ? 0 : wv.to + 1;
    };
    // Entering step s, K of s + 2 and V of s have landed; the step fetches K of s + 4 and V of s + 2, whose places were
    // last read in step s - 1 or before.
    for (int i = 0; i < kRingK; ++i) {
        fetch_k();
        fetch_r();
        if (i >= kRingK - 2) fetch_v();
    }

    f32x4_t acc[8][2], sum[2];                                 // sum: of the rounded weights, in every element (V^T of ones)
    // of the weights, in units of log2: T::kLift below the logit it was taken from
    float ref[2] = {0.f, 0.f};
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        sum[qb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[dt][qb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const unsigned one2 = T::pack(1.f, 1.f);
    const float c1 = fabsf(p.scale) * kLog2e;
    // This lane's operand reads: piece 4 kb + g of row k_row (+ 4 t: the same places), 32 bytes from element 16 dt of row
    // v_row.  Those of a row differ by an exclusive or with a constant.
    const int k_row = 8 * (n >> 2) + (n & 3), v_row = 8 * g + (n >> 2);
    const unsigned k_at = k_row * (kNope * 2) + ((g ^ k_place(k_row)) << 4), r_at = k_row * (kRope * 2) + ((g ^ r_place(k_row)) << 4);
    const unsigned v_at = v_row * (kNope * 2) + (v_unit(v_row) << 5) + ((n & 3) << 3);

    // operand op = 2 kb + t of a step's scores: 16 keys
    auto read_k = [&](unsigned kk, unsigned rr, int op) {
        const int kb = op >> 1, t = op & 1;
        return *(lds_u32x4)(uintptr_t)(kb < 4 ? (kk ^ (kb << 6)) + 4 * t * (kNope * 2) : (rr ^ ((kb - 4) << 6)) + 4 * t * (kRope * 2));
    };
    auto read_v = [&](unsigned vv, int dt) {
        const unsigned at = vv ^ (dt << 5);
        const s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)at);
        const s16x4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(at + 4 * kNope * 2));
        return __builtin_bit_cast(u32x4_t, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};

    // Step s from its scores sc[key block][query block], and the scores of step s + 1, which do not depend on it, in their
    // place.  Vector instructions of one wavefront do not run under the matrix instructions of the other of its SIMD, but
    // within a wavefront two or three independent ones do under each: so the two are woven by hand, a matrix instruction
    // and what runs under it to a slot.  24 slots of scores hide the logits, their maxima and the first query block's
    // exponentials, 18 of V^T P^T the second's.
    unsigned k_next = 1, v_now = 0;
    u32x4_t first[4];
    auto step = [&](auto last_step, int s, f32x4_t (&sc)[2][2]) {
        constexpr bool kLast = decltype(last_step)::value;
        // places of K of s + 1 (whose first four operands are there already), of K of s + 2, of V of s
        unsigned kk = lds_k + k_next * (kStep * kNope * 2) + k_at, rr = lds_r + k_next * (kStep * kRope * 2) + r_at;
        unsigned vv = lds_v + v_now * (kStep * kNope * 2) + v_at;
        k_next = k_next == kRingK - 1 ? 0 : k_next + 1;
        v_now = v_now == kRingV - 1 ? 0 : v_now + 1;
        unsigned k2 = lds_k + k_next * (kStep * kNope * 2) + k_at;
        asm("" : "+v"(kk), "+v"(rr), "+v"(vv), "+v"(k2));      // (or addresses of every place are kept in registers of their own)
        // key 8 g + j of the step is visible to query 16 qb + n of the wavefront where j - 16 qb <= own
        const int own = kHalves == 1 || (all - 1) % kHalves == half ? n - 8 * g : kStep;
        float z[2][8], top[2];
        f32x4_t scn[2][2];
        u32x4_t a[12], av[8], w[2];
        const u32x4_t none_of = {0u, 0u, 0u, 0u};
        f32x4_t any[2] = {zero, zero};                         // V^T times 0: NaN where a value is not finite
#pragma unroll
        for (int op = 0; op < 4; ++op) a[op] = first[op];
        auto score_slot = [&](auto mi) {
            constexpr int mm = decltype(mi)::value, op = mm >> 1, kb = op >> 1, t = op & 1, qb = mm & 1;
            scn[t][qb] = T::mfma(a[op], q[qb][kb], kb == 0 ? zero : scn[t][qb]);
            if constexpr (qb == 0 && op + 4 < 12) a[op + 4] = read_k(kk, rr, op + 4);
        };
        __builtin_amdgcn_sched_barrier(0);
        slots(std::make_integer_sequence<int, 12>{}, [&](auto mi) {
            constexpr int mm = decltype(mi)::value;
            if constexpr (!kLast) score_slot(mi);
            if constexpr (kLast && mm < 8) av[mm] = read_v(vv, mm);      // (early: see `any`)
            if constexpr (mm == 1) fetch_k();
            if constexpr (mm == 3) fetch_r();
            if constexpr (mm == 5) fetch_v();
            if constexpr (mm < 8) {                            // two logits a slot, against the reference so far
                constexpr int qb = mm >> 2, j = 2 * (mm & 3);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float x = __builtin_fmaf(sc[j >> 2][qb][(j & 3) + i], c1, -ref[qb]);
                    z[qb][j + i] = !kLast || j + i - 16 * qb <= own ? x : -INFINITY;
                }
            }
            if constexpr (mm >= 4 && mm < 10) {                // maxima, two slots behind the logits
                constexpr int qb = mm >= 8, i = qb ? mm - 8 : mm - 4;
                if constexpr (qb == 0) {
                    if constexpr (i == 0) top[0] = fmaxf(fmaxf(z[0][0], z[0][1]), z[0][2]);
                    if constexpr (i == 1) top[0] = fmaxf(fmaxf(top[0], z[0][3]), z[0][4]);
                    if constexpr (i == 2) top[0] = fmaxf(fmaxf(top[0], z[0][5]), z[0][6]);
                    if constexpr (i == 3) top[0] = fmaxf(top[0], z[0][7]);
                } else {
                    if constexpr (i == 0) top[1] = fmaxf(fmaxf(fmaxf(fmaxf(z[1][0], z[1][1]), z[1][2]), z[1][3]), z[1][4]);
                    if constexpr (i == 1) top[1] = fmaxf(fmaxf(fmaxf(top[1], z[1][5]), z[1][6]), z[1][7]);
                }
            }
            if constexpr (mm == 9) top[0] = columns_max(top[0]);
            if constexpr (mm == 11) top[1] = columns_max(top[1]);
            __builtin_amdgcn_sched_barrier(0);
        });
        // Relative to the reference, which a query whose logits have all been -inf does not have yet: none of its weights
        // is above 0, and any number becomes it.
        const bool none[2] = {sum[0][0] == 0.f, sum[1][0] == 0.f};
        constexpr float kMost = kSlack + T::kLift;
        if (__any((top[0] > (none[0] ? -INFINITY : kMost)) | (top[1] > (none[1] ? -INFINITY : kMost)))) {
#pragma unroll
            for (int qb = 0; qb < 2; ++qb) {
                float d = none[qb] ? top[qb] - T::kLift : fmaxf(top[qb] - T::kLift, 0.f);
                d = d == -INFINITY ? 0.f : d;
                const float f = none[qb] ? 1.f : __builtin_amdgcn_exp2f(-d);
                ref[qb] += d;
#pragma unroll
                for (int j = 0; j < 8; ++j) z[qb][j] -= d;
                if (s > 0)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        sum[qb][r] *= f;
#pragma unroll
                        for (int dt = 0; dt < 8; ++dt) acc[dt][qb][r] *= f;
                    }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        slots(std::make_integer_sequence<int, 12>{}, [&](auto mi) {
            constexpr int mm = decltype(mi)::value;
            if constexpr (!kLast) score_slot(std::integral_constant<int, mm + 12>{});
            if constexpr (!kLast && mm >= 2 && mm < 10) av[mm - 2] = read_v(vv, mm - 2);
            if constexpr (kLast && mm < 8) any[mm & 1] = T::mfma(av[mm], none_of, any[mm & 1]);
            if constexpr (mm < 8) {
                z[0][mm] = __builtin_amdgcn_exp2f(z[0][mm]);
                if constexpr (mm & 1) w[0][mm >> 1] = T::pack(z[0][mm - 1], z[0][mm]);
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        // In the step with masks the weights of keys behind a query are 0, and 0 times an infinite value or a NaN is NaN:
        // such values leave the product, and the queries that see them get them as a summand.  (In the steps before all
        // keys are seen.)
        if constexpr (kLast) {
            const float all_of = (any[0][0] + any[0][1]) + (any[0][2] + any[0][3]) + (any[1][0] + any[1][1]) + (any[1][2] + any[1][3]);
            if (__any(all_of != 0.f)) {
                u32x4_t seen[2];
#pragma unroll
                for (int qb = 0; qb < 2; ++qb)
#pragma unroll
                    for (int j = 0; j < 8; j += 2)
                        seen[qb][j >> 1] = T::pack(j - 16 * qb <= own ? 1.f : 0.f, j + 1 - 16 * qb <= own ? 1.f : 0.f);
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) {
                    const u32x4_t counted = not_finite<T>(av[dt]);
#pragma unroll
                    for (int qb = 0; qb < 2; ++qb) {
                        const f32x4_t counts = T::mfma(counted, seen[qb], zero);
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[dt][qb][r] += summand(counts[r]);
                    }
                    av[dt] = finite<T>(av[dt]);
                }
            }
        }
        const u32x4_t ones = {one2, one2, one2, one2};
        slots(std::make_integer_sequence<int, 9>{}, [&](auto mi) {
            constexpr int mm = decltype(mi)::value;
            if constexpr (mm == 0) sum[0] = T::mfma(ones, w[0], sum[0]);
            else acc[mm - 1][0] = T::mfma(av[mm - 1], w[0], acc[mm - 1][0]);
            if constexpr (mm < 8) {
                z[1][mm] = __builtin_amdgcn_exp2f(z[1][mm]);
                if constexpr (mm & 1) w[1][mm >> 1] = T::pack(z[1][mm - 1], z[1][mm]);
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        slots(std::make_integer_sequence<int, 9>{}, [&](auto mi) {
            constexpr int mm = decltype(mi)::value;
            if constexpr (mm == 0) sum[1] = T::mfma(ones, w[1], sum[1]);
            else acc[mm - 1][1] = T::mfma(av[mm - 1], w[1], acc[mm - 1][1]);
            if constexpr (!kLast && mm < 8) {
                constexpr int t = mm >> 2, qb = (mm >> 1) & 1, r = 2 * (mm & 1);
                sc[t][qb][r] = scn[t][qb][r];
                sc[t][qb][r + 1] = scn[t][qb][r + 1];
                if constexpr (mm >= 1 && mm < 5) first[mm - 1] = read_k(k2, 0u, mm - 1);
            }
            __builtin_amdgcn_sched_barrier(0);
        });
    };

    f32x4_t scA[2][2];
    wait_fetches<10>();                                        // K of steps 0 and 1
    tile_barrier();
    if (mine > 0) {
        unsigned kk = lds_k + k_at, rr = lds_r + r_at, k1 = lds_k + kStep * kNope * 2 + k_at;
        asm("" : "+v"(kk), "+v"(rr), "+v"(k1));
#pragma unroll
        for (int op = 0; op < 12; ++op) {
            const u32x4_t a = read_k(kk, rr, op);
#pragma unroll
            for (int qb = 0; qb < 2; ++qb) scA[op & 1][qb] = T::mfma(a, q[qb][op >> 1], op < 2 ? zero : scA[op & 1][qb]);
        }
#pragma unroll
        for (int op = 0; op < 4; ++op) first[op] = read_k(k1, 0u, op);
    }
    auto enter = [&] {
        wait_fetches<5>();                                     // K of s + 2 and V of s; what step s - 1 fetched is under way
        tile_barrier();
    };
    int s = 0;
#pragma unroll 1
    for (; s < mine - 1; ++s) {
        enter();
        step(std::false_type{}, s, scA);
    }
    if (mine > 0) {
        enter();
        step(std::true_type{}, s, scA);
        ++s;
    }
    for (; s < steps; ++s) {                                   // the steps that only later wavefronts have
        enter();
        fetch_k();
        fetch_r();
        fetch_v();
    }
    wait_fetches<0>();                                         // nothing may land in LDS after the workgroup has ended
    if constexpr (kHalves == 2) {                              // the second half's sums to the first, in the rings' place
        tile_barrier();
        auto reference = [&](int qb) { return sum[qb][0] == 0.f ? -INFINITY : ref[qb]; };      // (-inf: none, as in step)
        if (half == 1) {
#pragma unroll
            for (int qb = 0; qb < 2; ++qb) {
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) both.sums[wave][8 * qb + dt][lane] = acc[dt][qb];
                both.sums[wave][16 + qb][lane] = f32x4_t{sum[qb][0], reference(qb), 0.f, 0.f};
            }
        }
        tile_barrier();
        if (half == 1) return;
        if (all > 1)                                           // (of one step the second half has none)
#pragma unroll
            for (int qb = 0; qb < 2; ++qb) {
                const f32x4_t x = both.sums[wave][16 + qb][lane];
                const float own = reference(qb), top = fmaxf(own, x[1]);
                const float f0 = __builtin_amdgcn_exp2f(own - top), f1 = __builtin_amdgcn_exp2f(x[1] - top);
                sum[qb][0] = sum[qb][0] * f0 + x[0] * f1;
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) {
                    const f32x4_t y = both.sums[wave][8 * qb + dt][lane];
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[dt][qb][r] = acc[dt][qb][r] * f0 + y[r] * f1;
                }
            }
    }
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        const int row = w0 + 16 * qb + n;
        const float inv = row < S ? 1.f / sum[qb][0] : 0.f;
        if (row >= p.Smax) continue;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
            const f32x4_t a = acc[dt][qb];
            *reinterpret_cast<u32x2_t *>(out + row * out_stride + 16 * dt + 4 * g) =
                row < S ? u32x2_t{T::pack(a[0] * inv, a[1] * inv), T::pack(a[2] * inv, a[3] * inv)} : u32x2_t{0u, 0u};
        }
    }
}

template <class T> hipError_t prefill(const LatentPromptProblem &p, hipStream_t s)
{
    const long long workgroups = ((long long)p.B * p.H + 7) / 8 * 8 * ((p.Smax + kTileQ - 1) / kTileQ);
    const dim3 grid((unsigned)workgroups);
    // A wavefront alone on its SIMD takes 0.75 us a step, two 1.05 together: launches that leave the second place empty
    // give it to a second half of the workgroup, unless they are so short that joining the halves costs as much (with
    // halves / without, us: 1 x 16 heads x 2000 tokens 42.6 / 54.0, 1 x 8 x 4000 75.2 / 100.0, 1 x 32 x 500 18.3 / 19.6, 3
    // x 16 x 150 .. 1000 31.3 / 32.9, 4 x 16 x 200 .. 400 17.0 / 17.2, 1 x 16 x 128 11.2 / 10.0, 32 x 16 x 100 22.5 / 16.3,
    // 1 x 64 x 2000 117 / 107).
    if (workgroups <= kComputeUnits * 3 / 2 && p.Smax > 2 * kTileQ)
        return launch(latent_prefill_kernel<T, 2>, grid, dim3(512), s, p);
    return launch(latent_prefill_kernel<T, 1>, grid, dim3(256), s, p);
}

}  // namespace

hipError_t launch_latent_prefill(const LatentPromptProblem &p, hipStream_t s)
{
    return p.dtype == kF16 ? prefill<F16>(p, s) : prefill<BF16>(p, s);
}

}  // namespace fd
