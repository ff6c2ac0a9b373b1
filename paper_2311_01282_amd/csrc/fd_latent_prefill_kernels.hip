// Prompts with latent attention in the expanded form: every head has keys of 128 elements and 64 rotary ones that all heads share, values of 128, and token
// i attends to tokens 0 .. i.  Operands lie token by token, as projections leave them.
//
// Mapping as in the prompt kernel of the equal-sized heads (16 x 16 x 32; lane = (n, g) = (lane % 16, lane / 16)): a workgroup owns 128 queries of a head, a
// wavefront 32 of them in two blocks of 16;
//   scores   S^T[key][query] = K . Q^T: A = 16 keys of the tile in LDS, B = Q^T in registers.  Row 4 g + r of key block t is key 8 g + 4 t + r of the 32 of a step, so
//            that lane (n, g) holds keys 8 g .. 8 g + 7 of query n: the B operand of
//   output   O^T[d][query] = V^T . P^T: A = V^T by the transposing LDS read.
// Softmax with a running maximum per query; the weights are of the type (one rounding, as large as the output's own), their sum is that of the
// rounded ones, in fp32.
#include "fd_chunk.h"
#include "fd_cache.h"
#include "fd_types.h"

namespace fd {

namespace {

constexpr int kNope = 128, kQueryDim = kNope + kRope, kStep = 32, kTileQ = 128, kRing = 3;
// The reference of a query's weights follows its maximum only where that has grown by more than this (in units of log2): weights are then at
// most 2^8, and the sums are brought to another reference a few times a row instead of at every new maximum.
constexpr float kSlack = 8.f;

struct PromptLds {
    alignas(16) unsigned char k[kRing][kStep * kNope * 2];      // piece x (16 bytes) of row r in place x ^ key(r)
    alignas(16) unsigned char r[kRing][kStep * kRope * 2];      // ... x ^ swizzle(r)
    alignas(16) unsigned char v[kRing][kStep * kNope * 2];      // 32-byte unit x of row r in place x ^ v_unit(r)
};
// With these the 16-byte operand reads, whose cycles hold every n once from two neighbouring g, and the transposing reads, which take 32 bytes of
// rows 8 g + 4 h + (0 .. 3) of two neighbouring g at a time, have no bank conflicts.
__device__ __forceinline__ int k_place(int r) { return (r & 3) | (((r >> 3) & 3) << 2); }
__device__ __forceinline__ int r_place(int r) { return 2 * ((r >> 3) & 1) + 4 * ((r >> 1) & 1); }
__device__ __forceinline__ int v_unit(int r) { return (r & 3) | (((r >> 3) & 1) << 2); }

__device__ __forceinline__ void load_to_lds(u32x4_t rs, int voff, const unsigned char *lds_1k)
{
    const unsigned at = __builtin_amdgcn_readfirstlane((unsigned)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const unsigned char *)lds_1k));
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(at), "v"(voff), "s"(rs) : "memory");
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
    return u32x4_t{(unsigned)__builtin_amdgcn_readfirstlane((unsigned)at), (unsigned)__builtin_amdgcn_readfirstlane((unsigned)(at >> 32)) & 0xffffu,
                   (unsigned)__builtin_amdgcn_readfirstlane((unsigned)bytes), 0x00027000u};
}

template <class T> __global__ __launch_bounds__(256, 2) void latent_prefill_kernel(LatentPromptProblem p)
{
    __shared__ PromptLds lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const int pairs = p.B * p.H, tiles = (p.Smax + kTileQ - 1) / kTileQ;
    const int pair = blockIdx.x % pairs, i0 = (tiles - 1 - blockIdx.x / pairs) * kTileQ;      // the longest walks first
    const int b = pair / p.H, h = pair % p.H;
    const int S = min(max(p.seq_lens[b], 0), p.Smax);
    const int w0 = i0 + 32 * wave;
    uint16_t *out = p.out + ((size_t)b * p.Smax * p.H + h) * kNope;
    const size_t out_stride = (size_t)p.H * kNope;
    if (i0 >= S) {                                             // rows past the prompt: zeros
        for (int i = i0 + (tid >> 4); i < min(i0 + kTileQ, p.Smax); i += 16)
            *reinterpret_cast<u32x4_t *>(out + i * out_stride + 8 * (tid & 15)) = u32x4_t{0u, 0u, 0u, 0u};
        return;
    }
    const int steps = (min(i0 + kTileQ, S) - 1) / kStep + 1;
    const int mine = w0 < S ? (min(w0 + 32, S) - 1) / kStep + 1 : 0;

    u32x4_t q[2][6];
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        const int row = w0 + 16 * qb + n;
#pragma unroll
        for (int kb = 0; kb < 6; ++kb) {
            q[qb][kb] = u32x4_t{0u, 0u, 0u, 0u};
            if (row < S) q[qb][kb] = *reinterpret_cast<const u32x4_t *>(p.q + (((size_t)b * p.Smax + row) * p.H + h) * kQueryDim + 32 * kb + 8 * g);
        }
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);                        // the queries have arrived: what is counted from here on are fetches

    // A wavefront's five of the 20 KiB of a step: rows 8 wave .. + 7 of the keys and of the values, four rows an instruction, of the rotary parts all eight
    const int row_bytes = p.H * (2 * kNope * 2), rope_bytes = (int)(p.rope_stride * 2);
    int koff[2], voff[2], roff;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int r = 8 * wave + 4 * k + (lane >> 4), x = lane & 15;
        koff[k] = r * row_bytes + ((x ^ k_place(r)) << 4);
        voff[k] = r * row_bytes + ((x ^ (v_unit(r) << 1)) << 4);
    }
    {
        const int r = 8 * wave + (lane >> 3), x = lane & 7;
        roff = r * rope_bytes + ((x ^ r_place(r)) << 4);
    }
    const unsigned char *kv = reinterpret_cast<const unsigned char *>(p.kv) + ((size_t)b * p.Smax * p.H + h) * (2 * kNope * 2);
    const unsigned char *rp = reinterpret_cast<const unsigned char *>(p.rope) + (size_t)b * p.Smax * rope_bytes;
    auto fetch = [&](int s) {
        const int left = min(max(S - s * kStep, 0), kStep), at = s % kRing;          // rows without keys arrive as zeros
        const long long bytes = left > 0 ? (long long)(left - 1) * row_bytes + kNope * 2 : 0;
        const unsigned char *base = kv + (size_t)s * kStep * row_bytes;
        const u32x4_t rk = window(base, bytes), rv = window(base + kNope * 2, bytes);
        const u32x4_t rr = window(rp + (size_t)s * kStep * rope_bytes, left > 0 ? (long long)(left - 1) * rope_bytes + kRope * 2 : 0);
#pragma unroll
        for (int k = 0; k < 2; ++k) load_to_lds(rk, koff[k], lds.k[at] + (2 * wave + k) * 1024);
        load_to_lds(rr, roff, lds.r[at] + wave * 1024);
#pragma unroll
        for (int k = 0; k < 2; ++k) load_to_lds(rv, voff[k], lds.v[at] + (2 * wave + k) * 1024);
    };
    fetch(0);
    fetch(1);

    f32x4_t acc[8][2];
    float m[2], l[2];
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        m[qb] = -INFINITY;
        l[qb] = 0.f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[dt][qb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const float c1 = p.scale * kLog2e;
    const int k_row = 8 * (n >> 2) + (n & 3);                  // (+ 4 t: the same places)
    const int v_row = 8 * g + (n >> 2);

    for (int s = 0; s < steps; ++s) {
        wait_fetches<5>();                                     // step s; s + 1 is under way
        tile_barrier();
        fetch(s + 2);
        if (s >= mine) continue;
        const int slot = s % kRing;
        f32x4_t sc[2][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int qb = 0; qb < 2; ++qb) sc[qb][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kb = 0; kb < 6; ++kb) {
                const unsigned char *at = kb < 4 ? lds.k[slot] + (k_row + 4 * t) * (kNope * 2) + (((4 * kb + g) ^ k_place(k_row)) << 4)
                                                 : lds.r[slot] + (k_row + 4 * t) * (kRope * 2) + (((4 * (kb - 4) + g) ^ r_place(k_row)) << 4);
                const u32x4_t a = *reinterpret_cast<const u32x4_t *>(at);
#pragma unroll
                for (int qb = 0; qb < 2; ++qb) sc[qb][t] = T::mfma(a, q[qb][kb], sc[qb][t]);
            }
        }
        const bool last = s == mine - 1;
        u32x4_t w[2];
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
            float z[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                z[j] = sc[qb][j >> 2][j & 3] * c1;
                if (last && s * kStep + 8 * g + j > w0 + 16 * qb + n) z[j] = -INFINITY;
            }
            float top = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
            top = columns_max(top);
            if (__any(top > m[qb] + kSlack)) {                 // (also where there is no reference yet)
                const float to = fmaxf(top, m[qb]), f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[qb] - to);
                l[qb] *= f;
#pragma unroll
                for (int dt = 0; dt < 8; ++dt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[dt][qb][r] *= f;
                m[qb] = to;
            }
            const float ref = m[qb] == -INFINITY ? 0.f : m[qb];
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const unsigned x = T::pack(__builtin_amdgcn_exp2f(z[j] - ref), __builtin_amdgcn_exp2f(z[j + 1] - ref));
                l[qb] += T::lo(x) + T::hi(x);
                w[qb][j >> 1] = x;
            }
        }
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;
            unsigned char *at = lds.v[slot] + v_row * (kNope * 2) + ((dt ^ v_unit(v_row)) << 5) + ((n & 3) << 3);
            const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)at);
            const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at + 4 * kNope * 2));
            const u32x4_t a = __builtin_bit_cast(u32x4_t, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int qb = 0; qb < 2; ++qb) acc[dt][qb] = T::mfma(a, w[qb], acc[dt][qb]);
        }
    }
    wait_fetches<0>();                                         // nothing may land in LDS after the workgroup has ended
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
        const int row = w0 + 16 * qb + n;
        float sum = l[qb];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        const float inv = row < S ? 1.f / sum : 0.f;
        if (row >= p.Smax) continue;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
            const f32x4_t a = acc[dt][qb];
            *reinterpret_cast<u32x2_t *>(out + row * out_stride + 16 * dt + 4 * g) =
                row < S ? u32x2_t{T::pack(a[0] * inv, a[1] * inv), T::pack(a[2] * inv, a[3] * inv)} : u32x2_t{0u, 0u};
        }
    }
}

}  // namespace

hipError_t launch_latent_prefill(const LatentPromptProblem &p, hipStream_t s)
{
    const dim3 grid((unsigned)((long long)p.B * p.H * ((p.Smax + kTileQ - 1) / kTileQ)));
    return p.dtype == kF16 ? launch(latent_prefill_kernel<F16>, grid, dim3(256), s, p) : launch(latent_prefill_kernel<BF16>, grid, dim3(256), s, p);
}

}  // namespace fd
