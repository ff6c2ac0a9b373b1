// Latent attention over a paged cache: one row of 576 elements a token -- 512 that stand for the keys and values of all heads, 64 rotary ones
// that all heads share -- and queries that the caller has taken into the latent space (the absorbed form):
//     x_j = scale (q_latent . c_j + q_rope . r_j),   out = sum_j softmax(x)_j c_j.
// Every head reads the same rows, as keys and as values: a row is fetched once for 64 heads.
#include "fd_chunk.h"
#include "fd_cache.h"
#include "fd_types.h"

namespace fd {

namespace {

// ---- rows into the cache: 72 pieces of 16 bytes a row, 64 of the latent part and 8 of the rotary one ----
__global__ __launch_bounds__(256) void latent_write_kernel(LatentPool pool, const uint16_t *latent, long long latent_stride, const uint16_t *rope,
                                                           long long rope_stride, int n_tokens, const int32_t *slots)
{
    constexpr int kPieces = kLatentRow / 8;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long token = i / kPieces;
    const int piece = (int)(i - token * kPieces);
    if (token >= n_tokens) return;
    const int slot = slots[token];
    if (slot < 0 || (slot >> pool.page_shift) >= pool.n_pages) return;      // padding
    const uint16_t *src = piece < kLatent / 8 ? latent + token * latent_stride + 8 * piece : rope + token * rope_stride + (8 * piece - kLatent);
    *reinterpret_cast<u32x4_t *>(pool.rows + (size_t)slot * kLatentRow + 8 * piece) = *reinterpret_cast<const u32x4_t *>(src);
}

// ---- attention ----
//
// Matrix-core mapping (16 x 16 x 32; lane = (n, g) = (lane % 16, lane / 16)):
//   scores   S^T[key][head] = C . Q^T: A = 16 rows of the tile in LDS, B = Q^T in registers for the whole kernel (18 operands).  Row 4 g + r of key
//            block t is key 8 g + 4 t + r of the tile, so that the two blocks leave lane (n, g) holding keys 8 g .. 8 g + 7 of head n: the B operand of
//   output   O^T[d][head] = C^T . P^T: A = the same rows, turned round by the transposing LDS read.  32 tiles of 16 elements.
// The weights enter as the sum of two numbers of the type (hi + lo): one alone adds an error as large as the output's rounding.
// A workgroup takes 64 heads of a sequence (a wavefront 16) and a chunk of its keys, 32 at a time: tiles of 32 rows, fetched straight into LDS by all four
// wavefronts, in a ring of four.
constexpr int kTile = 32, kRing = 4;
constexpr int kRowBytes = kLatentRow * 2;                      // 1152 = 72 pieces of 16 bytes
constexpr int kLatentTileBytes = kTile * kRowBytes;            // 36 KiB
constexpr int kChunkPages = 1026;

struct LatentLds {
    alignas(16) unsigned char rows[kRing][kLatentTileBytes];
    int pages[kChunkPages];
};

// Piece x of row r lies in piece x ^ swizzle(r) of the row.  A cycle of the 16-byte operand reads holds every n once, from two neighbouring g;
// with rows 128 bytes apart modulo 256 the 16 pieces then lie in 16 different places modulo 256 bytes.  The transposing reads take 32 bytes of eight
// rows at a time, 8 g + 4 h + (0 .. 3) of two neighbouring g, in eight different places.
__device__ __forceinline__ int swizzle(int r) { return 2 * ((r >> 3) & 1) + 4 * ((r >> 1) & 1); }

__device__ __forceinline__ void load_to_lds(u32x4_t rs, int voff, const unsigned char *lds_1k)
{
    const unsigned at = __builtin_amdgcn_readfirstlane((unsigned)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const unsigned char *)lds_1k));
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(at), "v"(voff), "s"(rs) : "memory");
}
template <int N> __device__ __forceinline__ void wait_fetches() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void tile_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);                        // this wavefront's LDS reads have arrived
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <class T> __global__ __launch_bounds__(256, 1) void latent_decode_kernel(LatentProblem p)
{
    __shared__ LatentLds lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    // workgroups that read the same rows lie on one XCD (index modulo 8), one after the other
    const int tiles = (p.H + 63) / 64, units = p.B * p.nc;
    const int unit = (blockIdx.x / (8 * tiles)) * 8 + blockIdx.x % 8, head0 = (blockIdx.x / 8 % tiles) * 64 + 16 * wave;
    if (unit >= units) return;
    const int chunk = unit % p.nc, b = unit / p.nc;
    const int len = min(max(p.seq_lens[b], 0), p.Smax);
    const int start = chunk * p.C, end = min(len, start + p.C);
    const int heads = min(p.H - head0, 16);                    // of this wavefront; may be 0 or less: it only fetches
    if (start >= end) {
        if (p.nc == 1)                                         // no keys at all: zero rows
            for (int h = 0; h < heads; ++h)
                reinterpret_cast<u32x4_t *>(p.out + ((size_t)b * p.H + head0 + h) * kLatent)[lane] = u32x4_t{0u, 0u, 0u, 0u};
        return;
    }
    const int shift = p.pool.page_shift, mask = (1 << shift) - 1, first_page = start >> shift;
    const int used = ((end - 1) >> shift) - first_page + 1;
    for (int i = tid; i < used; i += 256) lds.pages[i] = min(max(p.table[(size_t)b * p.width + first_page + i], 0), p.pool.n_pages - 1);

    u32x4_t q[18];
#pragma unroll
    for (int kb = 0; kb < 18; ++kb) {
        q[kb] = u32x4_t{0u, 0u, 0u, 0u};
        if (n < heads) {
            const size_t row = (size_t)b * p.H + head0 + n;
            q[kb] = *reinterpret_cast<const u32x4_t *>(kb < 16 ? p.q_latent + row * kLatent + 32 * kb + 8 * g : p.q_rope + row * kRope + 32 * (kb - 16) + 8 * g);
        }
    }
    __syncthreads();                                           // the pages; and every load so far has arrived
    __builtin_amdgcn_s_waitcnt(0x0f70);

    // Fetches: instruction k of 18 fills KiB k of 16 rows' 18 KiB.  576 pieces are 8 rows: instruction k + 9 is k, 8 rows further.  Wavefronts 0 and 1
    // fetch rows 0 .. 15 of a tile, 2 and 3 the others.
    int voff[9];
#pragma unroll
    for (int k = 0; k < 9; ++k) {
        const int u = 64 * k + lane + 576 * (wave & 1), r = u / 72, x = u % 72;
        voff[k] = r * kRowBytes + ((x ^ swizzle(r)) << 4);
    }
    const int steps = (end - start + kTile - 1) / kTile;
    auto fetch = [&](int s) {
        const int key0 = start + s * kTile + 16 * (wave >> 1);
        const int left = min(max(end - key0, 0), 16);          // rows with keys: the others arrive as zeros
        const int k0 = left > 0 ? key0 : start;
        const int page = __builtin_amdgcn_readfirstlane(lds.pages[(k0 >> shift) - first_page]);
        const unsigned long long at = reinterpret_cast<unsigned long long>(p.pool.rows) + (((size_t)page << shift) + (k0 & mask)) * kRowBytes;
        const u32x4_t rs = {(unsigned)__builtin_amdgcn_readfirstlane((unsigned)at), __builtin_amdgcn_readfirstlane((unsigned)(at >> 32)) & 0xffffu,
                            (unsigned)__builtin_amdgcn_readfirstlane(left * kRowBytes), 0x00027000u};
        const unsigned char *to = lds.rows[s % kRing] + wave * 9 * 1024;
#pragma unroll
        for (int k = 0; k < 9; ++k) load_to_lds(rs, voff[k], to + k * 1024);
    };
    fetch(0);
    fetch(1);
    fetch(2);

    f32x4_t acc[32];
#pragma unroll
    for (int dt = 0; dt < 32; ++dt) acc[dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    const float c1 = p.scale * kLog2e;
    const int k_row = 8 * (n >> 2) + (n & 3), k_swz = swizzle(k_row);
    const int v_row = 8 * g + (n >> 2), v_swz = swizzle(v_row);

    for (int s = 0; s < steps; ++s) {
        wait_fetches<18>();                                    // tile s; s + 1 and s + 2 are under way
        tile_barrier();                                        // ... and every wavefront is through with tile s - 1
        fetch(s + 3);
        if (heads > 0) {
            unsigned char *rows = lds.rows[s % kRing];
            f32x4_t sc[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                sc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kb = 0; kb < 18; ++kb) {
                    const u32x4_t a = *reinterpret_cast<const u32x4_t *>(rows + (k_row + 4 * t) * kRowBytes + (((4 * kb + g) ^ k_swz) << 4));
                    sc[t] = T::mfma(a, q[kb], sc[t]);
                }
            }
            float z[8];
            const int left = end - (start + s * kTile) - 8 * g;
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = j < left ? sc[j >> 2][j & 3] * c1 : -INFINITY;
            float top = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
            top = fmaxf(m, columns_max(top));
            if (__any(top > m)) {
                const float f = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - top);
                l *= f;
#pragma unroll
                for (int dt = 0; dt < 32; ++dt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[dt][r] *= f;
                m = top;
            }
            const float ref = m == -INFINITY ? 0.f : m;
            u32x4_t hi, lo;
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float e0 = __builtin_amdgcn_exp2f(z[j] - ref), e1 = __builtin_amdgcn_exp2f(z[j + 1] - ref);
                l += e0 + e1;
                const unsigned h = T::pack(e0, e1);
                hi[j >> 1] = h;
                lo[j >> 1] = T::pack(e0 - T::lo(h), e1 - T::hi(h));
            }
#pragma unroll
            for (int dt = 0; dt < 32; ++dt) {
                typedef short s16x4 __attribute__((ext_vector_type(4)));
                typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;
                unsigned char *at = rows + v_row * kRowBytes + (((2 * dt + ((n >> 1) & 1)) ^ v_swz) << 4) + ((n & 1) << 3);
                const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)at);
                const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at + 4 * kRowBytes));
                const u32x4_t a = __builtin_bit_cast(u32x4_t, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
                acc[dt] = T::mfma(a, hi, acc[dt]);
                acc[dt] = T::mfma(a, lo, acc[dt]);
            }
        }
    }
    wait_fetches<0>();                                         // nothing may land in LDS after the workgroup has ended
    if (n >= heads) return;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    const size_t row = (size_t)b * p.H + head0 + n;
    if (p.nc == 1) {
        const float inv = 1.f / l;
#pragma unroll
        for (int dt = 0; dt < 32; ++dt)
            *reinterpret_cast<u32x2_t *>(p.out + row * kLatent + 16 * dt + 4 * g) =
                u32x2_t{T::pack(acc[dt][0] * inv, acc[dt][1] * inv), T::pack(acc[dt][2] * inv, acc[dt][3] * inv)};
    } else {
        float *num = p.num + (row * p.nc + chunk) * kLatent;
#pragma unroll
        for (int dt = 0; dt < 32; ++dt) *reinterpret_cast<f32x4_t *>(num + 16 * dt + 4 * g) = acc[dt];
        if (g == 0) p.ml[row * p.nc + chunk] = float2{m, l};
    }
}

}  // namespace

hipError_t launch_latent_write(const LatentPool &pool, const uint16_t *latent, long long latent_stride, const uint16_t *rope,
                               long long rope_stride, int n_tokens, const int32_t *slots, hipStream_t s)
{
    const dim3 grid((unsigned)(((long long)n_tokens * (kLatentRow / 8) + 255) / 256));
    return launch(latent_write_kernel, grid, dim3(256), s, pool, latent, latent_stride, rope, rope_stride, n_tokens, slots);
}
hipError_t launch_latent_decode(const LatentProblem &p, hipStream_t s)
{
    const long long tiles = (p.H + 63) / 64, units = (long long)p.B * p.nc;
    const dim3 grid((unsigned)((units + 7) / 8 * 8 * tiles));
    const hipError_t e = p.pool.dtype == kF16 ? launch(latent_decode_kernel<F16>, grid, dim3(256), s, p) : launch(latent_decode_kernel<BF16>, grid, dim3(256), s, p);
    if (e != hipSuccess || p.nc == 1) return e;
    JoinProblem j{p.num, p.ml, p.seq_lens, p.out, p.B * p.H, p.H, p.C, p.nc, p.Smax, kLatent, p.pool.dtype};
    return launch_join(j, s);
}

}  // namespace fd
