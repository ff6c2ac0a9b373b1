// Attention of a step's new tokens over the paged cache: sequences one behind the other, each token over its sequence's keys up to
// its own position.
//
// A row is a (token, query head) pair; the G query heads that share a KV head go together, rows r = G i + j of head j of the
// sequence's new token i, so that a tile of neighbouring rows reads the same keys whatever G is and however few tokens there are.
// A wavefront owns 16 rows and walks along the keys in blocks of 32 (fd_kv.h).
#include "fd_kv.h"

namespace fd {

namespace {

constexpr int kTileRows = 64;                    // of a workgroup: four wavefronts

// The sequence and the place of a tile of the launch: sequences in order, a sequence's tiles from its last to its first.
struct TilePlace {
    int b, tile, first, tokens;                  // b < 0: there is none; the sequence's first token and their number
};
__device__ __forceinline__ int tiles_of(int tokens, int G) { return (int)(((long long)tokens * G + kTileRows - 1) / kTileRows); }
__device__ __forceinline__ TilePlace find_tile(const KvPromptProblem &p, int at, int lane)
{
    int before = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int b = b0 + lane;
        int first = 0, tokens = 0;
        if (b < p.B) {
            first = min(max(p.starts[b], 0), p.n_tokens);
            tokens = max(min(max(p.starts[b + 1], 0), p.n_tokens) - first, 0);
        }
        const int tiles = tiles_of(tokens, p.G), upto = before + lanes_scan(tiles);
        const unsigned long long past = __ballot(upto > at);
        if (past) {
            const int l = __builtin_ctzll(past);
            const int end = __builtin_amdgcn_readlane(upto, l);
            return TilePlace{b0 + l, end - 1 - at, __builtin_amdgcn_readlane(first, l), __builtin_amdgcn_readlane(tokens, l)};
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return TilePlace{-1, 0, 0, 0};
}

template <class T, bool k8> __global__ __launch_bounds__(256, 2) void kv_prefill_kernel(KvPromptProblem p)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    const int hkv = blockIdx.x % p.pool.Hkv;
    const TilePlace at = find_tile(p, blockIdx.x / p.pool.Hkv, lane);
    if (at.b < 0) return;
    const int rows = at.tokens * p.G, row0 = at.tile * kTileRows + 16 * wave;       // of the sequence
    if (row0 >= rows) return;
    const int len = min(max(p.seq_lens[at.b], 0), p.Smax);
    const int row = row0 + n, token = row / p.G, head = hkv * p.G + row % p.G;
    const bool live = row < rows;
    const int position = len - at.tokens + token;              // below 0: nothing to attend to
    const int end = min(len, len - at.tokens + (min(row0 + 15, rows - 1)) / p.G + 1);      // keys of the 16 rows
    const int first_position = len - at.tokens + row0 / p.G;
    const size_t q_row = (size_t)(at.first + token);
    u32x4_t q[4];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
        q[kb] = u32x4_t{0u, 0u, 0u, 0u};
        if (live) q[kb] = *reinterpret_cast<const u32x4_t *>(p.q + q_row * p.q_stride + (size_t)head * kHeadDim + Keys<T, k8>::element(kb, g));
    }
    const scalar_i32 table = (scalar_i32)(uintptr_t)(p.table + (size_t)at.b * p.width);
    const float c1 = p.scale * kLog2e;
    Softmax<T> state;
    state.clear();
    const int last = end - 1;
    for (int key0 = 0; key0 < end; key0 += 32) {
        Keys<T, k8> keys;
        Values<T, k8> values;
        const BlockRows rows_at = block_rows(p.pool, hkv, block_pages(table, p.pool.page_shift, key0, last), key0, last);
        keys.load(p.pool, rows_at, lane);
        values.load(p.pool, rows_at, lane);
        f32x4_t s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) s[t] = T::mfma(keys.operand(t, kb, lane), q[kb], s[t]);
        }
        float z[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = key0 + 8 * g + j <= position ? s[j >> 2][j & 3] * c1 : -INFINITY;
        if (key0 + 32 > end) values.keep(end - key0 - 8 * g);
        u32x4_t a[8];
        values.operands(a);
        const bool odd = any_not_finite<T>(a);
        if (odd && key0 + 31 > first_position) {
            // keys behind a query have the weight 0: what they hold must not reach it, be it infinite
            u32x4_t seen;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                seen[i] = T::pack(key0 + 8 * g + 2 * i <= position ? 1.f : 0.f, key0 + 8 * g + 2 * i + 1 <= position ? 1.f : 0.f);
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) {
                const f32x4_t counts = T::mfma(not_finite<T>(a[dt]), seen, f32x4_t{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                for (int r = 0; r < 4; ++r) state.acc[dt][r] += summand(counts[r]);
                a[dt] = finite<T>(a[dt]);
            }
        }
        state.block(z, a, odd);
    }
    float sum = rows_sum(state.sum, state.sum);
    sum = halves_sum(sum, sum);
    if (!live) return;
    const float inv = position >= 0 ? 1.f / sum : 0.f;
    uint16_t *out = p.out + (q_row * p.Hq + head) * kHeadDim + 32 * g;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        u32x4_t x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = position >= 0 ? T::pack(state.acc[2 * i][r] * inv, state.acc[2 * i + 1][r] * inv) : 0u;
        *reinterpret_cast<u32x4_t *>(out + 8 * r) = x;
    }
}

}  // namespace

hipError_t launch_kv_prefill(const KvPromptProblem &p, hipStream_t s)
{
    // (no sequence leaves more than one tile unfilled)
    const long long tiles = (long long)p.n_tokens * p.G / kTileRows + p.B;
    const dim3 grid((unsigned)(tiles * p.pool.Hkv));
    if (p.pool.store == kE4m3)
        return p.pool.dtype == kF16 ? launch(kv_prefill_kernel<F16, true>, grid, dim3(256), s, p) : launch(kv_prefill_kernel<BF16, true>, grid, dim3(256), s, p);
    return p.pool.dtype == kF16 ? launch(kv_prefill_kernel<F16, false>, grid, dim3(256), s, p) : launch(kv_prefill_kernel<BF16, false>, grid, dim3(256), s, p);
}

}  // namespace fd
