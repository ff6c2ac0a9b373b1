// Internal declarations of the calls around the smaller paged caches: page tables, the 4-bit cache, the cache of latent rows.
#pragma once

#include "fd_internal.h"

namespace fd {

enum { kF16 = 0, kBf16 = 1 };                      // fd_dtype

// fd_page_kernels.hip
struct PageProblem {
    const int32_t *cached, *fresh;                 // [batch] tokens in the cache, tokens to come
    const int32_t *free_pages, *n_free;
    int32_t *table, *seq_lens, *starts, *slots, *n_left;
    int batch, page_shift, n_pages, width, max_tokens;
};
hipError_t launch_page_tables(const PageProblem &p, hipStream_t s);

// fd_nibble_kernels.hip
struct NibblePool {
    unsigned char *k_codes, *v_codes;              // [n_pages, Hkv, page, 64]
    uint16_t *k_scales, *v_scales;                 // [n_pages, Hkv, page, 2, NG]
    int n_pages, page_shift, Hkv, NG, dtype;       // NG groups to a row: 4, 2 or 1
};
struct NibbleRows {
    uint16_t *k, *v;                               // [n_tokens, Hkv, 128], token strides of their own
    long long k_stride, v_stride;                  // elements
    const int32_t *slots;
    int n_tokens;
};
hipError_t launch_nibble_write(const NibblePool &pool, const NibbleRows &rows, hipStream_t s);
hipError_t launch_nibble_read(const NibblePool &pool, const NibbleRows &rows, hipStream_t s);

struct NibbleProblem {
    NibblePool pool;
    const uint16_t *q;                             // [B, Hq, 128]
    const int32_t *seq_lens, *table;
    uint16_t *out;
    float *num;                                    // workspace: [B, Hq, nc, 128] sum e^{x-m} v
    float2 *ml;                                    // [B, Hq, nc] (m, l), m the reference of the weights times log2 e
    // [B, Hkv, tiles] chunks that have arrived, zero between calls; null: the join is a launch of its own
    int32_t *counters;
    int B, Hq, G, tiles, C, nc, Smax, width;       // tiles: of 16 query heads of a KV head
    float scale;
};
hipError_t launch_nibble_attn(const NibbleProblem &p, hipStream_t s);

// fd_latent_kernels.hip
constexpr int kLatent = 512, kRope = 64, kLatentRow = kLatent + kRope;
struct LatentPool {
    uint16_t *rows;                                // [n_pages, page, 576]
    int n_pages, page_shift, dtype;
};
hipError_t launch_latent_write(const LatentPool &pool, const uint16_t *latent, long long latent_stride, const uint16_t *rope,
                               long long rope_stride, int n_tokens, const int32_t *slots, hipStream_t s);
struct LatentProblem {
    LatentPool pool;
    const uint16_t *q_latent, *q_rope;             // [B, H, 512], [B, H, 64]
    const int32_t *seq_lens, *table;
    uint16_t *out;                                 // [B, H, 512]
    float *num;                                    // workspace: [B, H, nc, 512]
    float2 *ml;                                    // [B, H, nc]
    int B, H, C, nc, Smax, width;
    float scale;
};
hipError_t launch_latent_decode(const LatentProblem &p, hipStream_t s);

// fd_latent_prefill_kernels.hip
struct LatentPromptProblem {
    const uint16_t *q;                             // [B, Smax, H, 192]
    const uint16_t *kv;                            // [B, Smax, H, 256]: key, value
    const uint16_t *rope;                          // [B, Smax, 64], token stride of its own
    long long rope_stride;
    const int32_t *seq_lens;
    uint16_t *out;                                 // [B, Smax, H, 128]
    int B, H, Smax, dtype;
    float scale;
};
hipError_t launch_latent_prefill(const LatentPromptProblem &p, hipStream_t s);

// Splits of a row between workgroups, joined by a launch of its own: out = sum_c 2^{m_c - M} num_c / sum_c 2^{m_c - M} l_c over the
// chunks that hold a key, of rows with two or more of them.  rows: [B, H] output rows of `dim` elements.
struct JoinProblem {
    const float *num;
    const float2 *ml;
    const int32_t *seq_lens;
    uint16_t *out;
    int rows, H, C, nc, Smax, dim, dtype;
};
hipError_t launch_join(const JoinProblem &p, hipStream_t s);

}  // namespace fd
