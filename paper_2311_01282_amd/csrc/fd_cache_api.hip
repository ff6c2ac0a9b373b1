// C-ABI entry points around the smaller paged caches: argument checks, workspace carving, launches.
#include "../../include/fdattn.h"
#include "fd_cache.h"

#include <cmath>

namespace {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline bool off(const void *p, size_t to) { return ((uintptr_t)p % to) != 0; }
inline bool is_page_size(int32_t page_size) { return page_size >= 16 && (page_size & (page_size - 1)) == 0; }

constexpr long long kMostThreads = 1ll << 32;      // of a launch

#define FD_TRY(expr) do { if ((expr) != hipSuccess) return FD_ERR_HIP; } while (0)

// Device arrays of a call, to see whether two share a byte.
struct Array {
    const void *at;
    long long bytes;
};
inline bool meet(const Array &a, const Array &b)
{
    const uintptr_t x = (uintptr_t)a.at, y = (uintptr_t)b.at;
    return a.bytes > 0 && b.bytes > 0 && (x < y ? y - x < (uintptr_t)a.bytes : x - y < (uintptr_t)b.bytes);
}

// A pool's pages: a power of two of rows each, and slots that fit 31 bits.
fd_status check_pages(int32_t n_pages, int32_t page_size, int *shift)
{
    if (!is_page_size(page_size) || n_pages < 1 || (long long)n_pages * page_size >= (1ll << 31)) return FD_ERR_SHAPE;
    *shift = __builtin_ctz((unsigned)page_size);
    return FD_OK;
}
inline bool known_type(int32_t dtype) { return dtype == FD_F16 || dtype == FD_BF16; }

fd_status nibble_pool(const fd_nibble_pool *pool, fd::NibblePool *out)
{
    if (!pool) return FD_ERR_NULL;
    if (!pool->k_codes || !pool->k_scales || !pool->v_codes || !pool->v_scales) return FD_ERR_NULL;
    fd::NibblePool o{};
    const fd_status st = check_pages(pool->n_pages, pool->page_size, &o.page_shift);
    if (st != FD_OK) return st;
    if (pool->n_kv_heads < 1 || pool->head_dim < 1) return FD_ERR_SHAPE;
    if (off(pool->k_codes, 16) || off(pool->k_scales, 16) || off(pool->v_codes, 16) || off(pool->v_scales, 16)) return FD_ERR_SHAPE;
    if (pool->head_dim != fd::kHeadDim || pool->n_kv_heads > 65535 || !known_type(pool->dtype) ||
        (pool->group != 32 && pool->group != 64 && pool->group != 128))
        return FD_ERR_UNSUPPORTED;
    o.k_codes = static_cast<unsigned char *>(pool->k_codes);
    o.v_codes = static_cast<unsigned char *>(pool->v_codes);
    o.k_scales = static_cast<uint16_t *>(pool->k_scales);
    o.v_scales = static_cast<uint16_t *>(pool->v_scales);
    o.n_pages = pool->n_pages;
    o.Hkv = pool->n_kv_heads;
    o.NG = fd::kHeadDim / pool->group;
    o.dtype = pool->dtype;
    *out = o;
    return FD_OK;
}

fd_status nibble_rows(const fd_nibble_pool *pool, const void *k, int64_t k_stride, const void *v, int64_t v_stride, int32_t n_tokens,
                   const int32_t *slot_map, fd::NibblePool *P, fd::NibbleRows *R)
{
    const fd_status st = nibble_pool(pool, P);
    if (st != FD_OK) return st;
    if (!k || !v || !slot_map) return FD_ERR_NULL;
    const long long width = (long long)P->Hkv * fd::kHeadDim;
    if (n_tokens < 0 || off(k, 16) || off(v, 16) || off(slot_map, 4) || k_stride < width || v_stride < width || k_stride % 8 != 0 ||
        v_stride % 8 != 0)
        return FD_ERR_SHAPE;
    if ((long long)n_tokens * 2 * P->Hkv >= kMostThreads / 16) return FD_ERR_UNSUPPORTED;
    *R = fd::NibbleRows{const_cast<uint16_t *>(static_cast<const uint16_t *>(k)),
                        const_cast<uint16_t *>(static_cast<const uint16_t *>(v)), k_stride, v_stride, slot_map, n_tokens};
    return FD_OK;
}

fd_status latent_pool(const fd_latent_pool *pool, fd::LatentPool *out)
{
    if (!pool || !pool->rows) return FD_ERR_NULL;
    fd::LatentPool o{};
    const fd_status st = check_pages(pool->n_pages, pool->page_size, &o.page_shift);
    if (st != FD_OK) return st;
    if (off(pool->rows, 16) || pool->latent_dim < 1 || pool->rope_dim < 1) return FD_ERR_SHAPE;
    if (pool->latent_dim != fd::kLatent || pool->rope_dim != fd::kRope || !known_type(pool->dtype)) return FD_ERR_UNSUPPORTED;
    o.rows = static_cast<uint16_t *>(pool->rows);
    o.n_pages = pool->n_pages;
    o.dtype = pool->dtype;
    *out = o;
    return FD_OK;
}

// A row is cut into chunks, one workgroup each, whose sums meet in the workspace.  It begins with arrival counters, a fixed
// number of them, so that they stay where they are whatever the shape.
constexpr int kCounters = 4096;
struct Split {
    long long rows, nc;
    size_t num, ml, total;
};
fd_status check_shape(const fd_shape *sh, int head_dim)
{
    if (!sh) return FD_ERR_NULL;
    if (sh->batch < 0 || sh->n_q_heads <= 0 || sh->n_kv_heads <= 0 || sh->head_dim <= 0 || sh->max_seq <= 0) return FD_ERR_SHAPE;
    if (sh->n_q_heads % sh->n_kv_heads != 0 || !std::isfinite(sh->scale)) return FD_ERR_SHAPE;
    if (sh->head_dim != head_dim || sh->max_seq > (1 << 30)) return FD_ERR_UNSUPPORTED;      // (a chunk's end fits 31 bits)
    return FD_OK;
}
fd_status split(const fd_shape *sh, int head_dim, int dim, int unit, Split *S)
{
    const fd_status st = check_shape(sh, head_dim);
    if (st != FD_OK) return st;
    if (sh->chunk <= 0) return FD_ERR_SHAPE;
    if (sh->chunk % unit != 0 || sh->chunk > 16384) return FD_ERR_UNSUPPORTED;
    S->rows = (long long)sh->batch * sh->n_q_heads;
    S->nc = ((long long)sh->max_seq + sh->chunk - 1) / sh->chunk;
    // (no more workgroups than these, of 512 threads at most)
    if (S->rows * S->nc > kMostThreads / 512) return FD_ERR_UNSUPPORTED;
    const size_t slots = (size_t)(S->rows * S->nc);
    S->num = align_up(kCounters * sizeof(int32_t));
    S->ml = align_up(S->num + (S->nc == 1 ? 0 : slots * dim * sizeof(float)));
    S->total = align_up(S->ml + (S->nc == 1 ? 0 : slots * sizeof(float2)));
    return FD_OK;
}
inline bool bad_ws(fd_workspace ws, const Split &S) { return !ws.ptr || off(ws.ptr, kAlign) || ws.bytes < S.total; }

fd_status nibble_split(const fd_shape *sh, Split *S) { return split(sh, fd::kHeadDim, fd::kHeadDim, 64, S); }
fd_status latent_split(const fd_shape *sh, Split *S)
{
    const fd_status st = split(sh, fd::kLatentRow, fd::kLatent, 64, S);
    if (st != FD_OK) return st;
    return sh->n_kv_heads == 1 ? FD_OK : FD_ERR_UNSUPPORTED;
}

// Keys of a chunk, a multiple of `unit`, so that `units` rows of max_seq keys make about `want` workgroups of at least
// `least` keys.
int32_t chunk_for(int32_t max_seq, long long units, long long want, int32_t least, int32_t unit)
{
    long long nc = units > 0 ? want / units : 1;
    const long long most = ((long long)max_seq + least - 1) / least;
    if (nc > most) nc = most;
    if (nc < 1) nc = 1;
    long long chunk = ((long long)max_seq + nc - 1) / nc;
    chunk = (chunk + unit - 1) / unit * unit;
    return (int32_t)(chunk > 16384 ? 16384 : chunk);
}

}  // namespace

extern "C" {

fd_status fd_page_tables(int32_t batch, int32_t page_size, int32_t n_pages, int32_t pages_per_seq, int32_t max_tokens,
                         const int32_t *cached_lens, const int32_t *new_lens, const int32_t *free_pages, const int32_t *n_free,
                         int32_t *block_table, int32_t *seq_lens, int32_t *token_starts, int32_t *slot_map, int32_t *n_left,
                         void *stream)
{
    fd::PageProblem p{};
    const fd_status st = check_pages(n_pages, page_size, &p.page_shift);
    if (st != FD_OK) return st;
    if (batch < 0 || pages_per_seq < 1 || max_tokens < 0 || (long long)pages_per_seq * page_size >= (1ll << 31)) return FD_ERR_SHAPE;
    if (max_tokens > (1 << 30) || batch > (1 << 30)) return FD_ERR_UNSUPPORTED;
    if (!cached_lens || !new_lens || !free_pages || !n_free || !block_table || !seq_lens || !token_starts || !slot_map || !n_left)
        return FD_ERR_NULL;
    // Workgroups read the inputs and the table at any time while others write: an output that shares memory with another
    // array would be read as such.
    const long long one = sizeof(int32_t), b = batch * one;
    const Array all[] = {{cached_lens, b}, {new_lens, b}, {free_pages, n_pages * one}, {n_free, one},
                         {block_table, b * pages_per_seq}, {seq_lens, b}, {token_starts, b + one}, {slot_map, max_tokens * one},
                         {n_left, one}};
    constexpr int kInputs = 4, kArrays = 9;
    for (const Array &x : all)
        if (off(x.at, 4)) return FD_ERR_SHAPE;
    for (int i = kInputs; i < kArrays; ++i)
        for (int j = 0; j < i; ++j)
            if (meet(all[i], all[j])) return FD_ERR_SHAPE;
    p.cached = cached_lens; p.fresh = new_lens; p.free_pages = free_pages; p.n_free = n_free;
    p.table = block_table; p.seq_lens = seq_lens; p.starts = token_starts; p.slots = slot_map; p.n_left = n_left;
    p.batch = batch; p.n_pages = n_pages; p.width = pages_per_seq; p.max_tokens = max_tokens;
    FD_TRY(fd::launch_page_tables(p, static_cast<hipStream_t>(stream)));
    return FD_OK;
}

fd_status fd_nibble_write(const fd_nibble_pool *pool, const void *k, int64_t k_stride, const void *v, int64_t v_stride, int32_t n_tokens,
                       const int32_t *slot_map, void *stream)
{
    fd::NibblePool P;
    fd::NibbleRows R;
    const fd_status st = nibble_rows(pool, k, k_stride, v, v_stride, n_tokens, slot_map, &P, &R);
    if (st != FD_OK) return st;
    if (n_tokens == 0) return FD_OK;
    FD_TRY(fd::launch_nibble_write(P, R, static_cast<hipStream_t>(stream)));
    return FD_OK;
}

fd_status fd_nibble_read(const fd_nibble_pool *pool, const int32_t *slot_map, int32_t n_tokens, void *k, int64_t k_stride, void *v,
                      int64_t v_stride, void *stream)
{
    fd::NibblePool P;
    fd::NibbleRows R;
    const fd_status st = nibble_rows(pool, k, k_stride, v, v_stride, n_tokens, slot_map, &P, &R);
    if (st != FD_OK) return st;
    if (n_tokens == 0) return FD_OK;
    FD_TRY(fd::launch_nibble_read(P, R, static_cast<hipStream_t>(stream)));
    return FD_OK;
}

fd_status fd_cache_workspace_init(fd_workspace ws, void *stream)
{
    if (!ws.ptr || off(ws.ptr, kAlign) || ws.bytes < kCounters * sizeof(int32_t)) return FD_ERR_WORKSPACE;
    FD_TRY(fd::launch_clear_tickets(static_cast<int32_t *>(ws.ptr), kCounters, static_cast<hipStream_t>(stream)));
    return FD_OK;
}

size_t fd_nibble_workspace_bytes(const fd_shape *shape)
{
    Split S;
    return nibble_split(shape, &S) == FD_OK ? S.total : 0;
}

int32_t fd_nibble_pick_chunk(const fd_shape *shape)
{
    if (check_shape(shape, fd::kHeadDim) != FD_OK) return 0;
    const long long units = (long long)shape->batch * shape->n_kv_heads * ((shape->n_q_heads / shape->n_kv_heads + 15) / 16);
    // Two workgroups fit a compute unit, and a launch of one round of them is the fastest there is, ragged or not: a
    // workgroup's beginning and end cost as much as three blocks of its four wavefronts.  Up to there 1024 keys are the
    // best length where they fill the chip once, otherwise what does, down to a block a wavefront.
    // (Whole call, chunks of 256 / 512 / 1024 / 2048 / 4096 keys, the choice marked: 16 x 32 heads x 2000 44 / 37.7 / 33.7
    // / *30.2, 64 x 32/8 x 4000 95 / 72 / 64 / 60 / *56.4, 32 x 32/8 x 2000 33.5 / 27.4 / *22.9 / 23.3, 1 x 32 x 8192 21.7
    // / 16.7 / *15.9 / 21.8 / 35.6, 8 x 32/8 x 4000 17.8 / 14.4 / *14.0 / 18.2 / 26.7, 4 x 64/8 x 2000 *11.3 / 12.9 /
    // 17.0.)
    const long long chip = fd::kComputeUnits, rows = units > 0 ? units : 1;
    for (int32_t c : {1024, 512, 256}) {
        const long long w = rows * (((long long)shape->max_seq + c - 1) / c);
        if (w <= 2 * chip && (w >= chip || c == 256)) return c;
    }
    return chunk_for(shape->max_seq, rows, 2 * chip, 256, 256);
}

fd_status fd_decode_attn_nibble(const fd_shape *shape, const fd_nibble_pool *pool, const void *q, const int32_t *block_table,
                             const int32_t *seq_lens, void *out, fd_workspace ws, void *stream)
{
    Split S;
    fd_status st = nibble_split(shape, &S);
    if (st != FD_OK) return st;
    fd::NibbleProblem p{};
    st = nibble_pool(pool, &p.pool);
    if (st != FD_OK) return st;
    if (!q || !block_table || !seq_lens || !out) return FD_ERR_NULL;
    if (off(q, 16) || off(out, 16) || off(block_table, 4) || off(seq_lens, 4)) return FD_ERR_SHAPE;
    if (pool->n_kv_heads != shape->n_kv_heads || shape->max_seq % pool->page_size != 0) return FD_ERR_SHAPE;
    if (bad_ws(ws, S)) return FD_ERR_WORKSPACE;
    if (shape->batch == 0) return FD_OK;
    p.q = static_cast<const uint16_t *>(q);
    p.seq_lens = seq_lens;
    p.table = block_table;
    p.out = static_cast<uint16_t *>(out);
    p.num = reinterpret_cast<float *>(static_cast<char *>(ws.ptr) + S.num);
    p.ml = reinterpret_cast<float2 *>(static_cast<char *>(ws.ptr) + S.ml);
    p.B = shape->batch; p.Hq = shape->n_q_heads; p.G = shape->n_q_heads / shape->n_kv_heads; p.tiles = (p.G + 15) / 16;
    if ((long long)p.B * shape->n_kv_heads * p.tiles <= kCounters) p.counters = static_cast<int32_t *>(ws.ptr);
    p.C = shape->chunk; p.nc = (int)S.nc; p.Smax = shape->max_seq; p.width = shape->max_seq / pool->page_size;
    p.scale = shape->scale;
    FD_TRY(fd::launch_nibble_attn(p, static_cast<hipStream_t>(stream)));
    return FD_OK;
}

fd_status fd_latent_write(const fd_latent_pool *pool, const void *latent, int64_t latent_stride, const void *rope, int64_t rope_stride,
                          int32_t n_tokens, const int32_t *slot_map, void *stream)
{
    fd::LatentPool P;
    const fd_status st = latent_pool(pool, &P);
    if (st != FD_OK) return st;
    if (!latent || !rope || !slot_map) return FD_ERR_NULL;
    if (n_tokens < 0 || off(latent, 16) || off(rope, 16) || off(slot_map, 4) || latent_stride < fd::kLatent || rope_stride < fd::kRope ||
        latent_stride % 8 != 0 || rope_stride % 8 != 0)
        return FD_ERR_SHAPE;
    if (n_tokens > (1 << 25)) return FD_ERR_UNSUPPORTED;                    // (72 threads each)
    if (n_tokens == 0) return FD_OK;
    FD_TRY(fd::launch_latent_write(P, static_cast<const uint16_t *>(latent), latent_stride, static_cast<const uint16_t *>(rope),
                                   rope_stride, n_tokens, slot_map, static_cast<hipStream_t>(stream)));
    return FD_OK;
}

size_t fd_latent_workspace_bytes(const fd_shape *shape)
{
    Split S;
    return latent_split(shape, &S) == FD_OK ? S.total : 0;
}

int32_t fd_latent_pick_chunk(const fd_shape *shape)
{
    if (check_shape(shape, fd::kLatentRow) != FD_OK || shape->n_kv_heads != 1) return 0;
    // A chunk of c keys takes c / 32 tiles of about 1 us (1.4 of 64 heads, 1.5 of 128), and every workgroup leaves 2 KiB of
    // sums a head, written and read again: about 0.07 us for 128 heads.  The sum of the two is least near sqrt(k units
    // max_seq) keys; a row of many pieces takes its join 0.07 us for each, which adds sqrt(2.2 max_seq); and more than one
    // workgroup a compute unit gains nothing.  A row that would be cut into little goes in one piece, without the join's
    // launch.
    // (Whole call, chunks of 64 / 128 / 256 / 512 / 1024 keys: 8 x 128 heads x 4000 77 / 46 / 41.7 / 51 / 73 us, 1 x 16 x
    // 30000 50 / 33 / 27.4 / 31 / 45, 64 x 64 x 4000 - / - / 124 / 99 / 89, 128 x 16 x 300 29 / 26 / 25.5 / 19.5.)
    const double units = (double)shape->batch * ((shape->n_q_heads + 127) / 128), S = shape->max_seq;
    const double k = shape->n_q_heads > 64 ? 1.5 : shape->n_q_heads / 76.0;
    const double c = std::fmax(std::fmax(units * S / fd::kComputeUnits, std::sqrt(k * units * S)), std::sqrt(2.2 * S));
    long long nc = (long long)(S / c);
    if (nc < 2 || S * (1.0 - 1.0 / (double)nc) < 192.0) nc = 1;
    const long long chunk = (((long long)shape->max_seq + nc - 1) / nc + 63) / 64 * 64;
    return (int32_t)(chunk > 16384 ? 16384 : chunk);
}

fd_status fd_latent_decode_attn(const fd_shape *shape, const fd_latent_pool *pool, const void *q_latent, const void *q_rope,
                                const int32_t *block_table, const int32_t *seq_lens, void *out, fd_workspace ws, void *stream)
{
    Split S;
    fd_status st = latent_split(shape, &S);
    if (st != FD_OK) return st;
    fd::LatentProblem p{};
    st = latent_pool(pool, &p.pool);
    if (st != FD_OK) return st;
    if (!q_latent || !q_rope || !block_table || !seq_lens || !out) return FD_ERR_NULL;
    if (off(q_latent, 16) || off(q_rope, 16) || off(out, 16) || off(block_table, 4) || off(seq_lens, 4)) return FD_ERR_SHAPE;
    if (shape->max_seq % pool->page_size != 0) return FD_ERR_SHAPE;
    if (bad_ws(ws, S)) return FD_ERR_WORKSPACE;
    if (shape->batch == 0) return FD_OK;
    p.q_latent = static_cast<const uint16_t *>(q_latent);
    p.q_rope = static_cast<const uint16_t *>(q_rope);
    p.seq_lens = seq_lens;
    p.table = block_table;
    p.out = static_cast<uint16_t *>(out);
    p.num = reinterpret_cast<float *>(static_cast<char *>(ws.ptr) + S.num);
    p.ml = reinterpret_cast<float2 *>(static_cast<char *>(ws.ptr) + S.ml);
    p.B = shape->batch; p.H = shape->n_q_heads; p.C = shape->chunk; p.nc = (int)S.nc; p.Smax = shape->max_seq;
    p.width = shape->max_seq / pool->page_size;
    p.scale = shape->scale;
    FD_TRY(fd::launch_latent_decode(p, static_cast<hipStream_t>(stream)));
    return FD_OK;
}

fd_status fd_latent_prefill_attn(const fd_shape *shape, int32_t dtype, const void *q, const void *kv, const void *rope,
                                 int64_t rope_stride, const int32_t *seq_lens, void *out, void *stream)
{
    const fd_status st = check_shape(shape, 128 + fd::kRope);
    if (st != FD_OK) return st;
    if (shape->n_kv_heads != shape->n_q_heads || shape->n_q_heads > 65535 || !known_type(dtype)) return FD_ERR_UNSUPPORTED;
    const long long pairs = (long long)shape->batch * shape->n_q_heads, tiles = ((long long)shape->max_seq + 127) / 128;
    // (the launch has as many workgroups, of 256 threads, for each of the eight XCDs)
    if (pairs * tiles > kMostThreads / 512 || (pairs + 7) / 8 * 8 * tiles >= kMostThreads / 256) return FD_ERR_UNSUPPORTED;
    if (!q || !kv || !rope || !seq_lens || !out) return FD_ERR_NULL;
    if (off(q, 16) || off(kv, 16) || off(rope, 16) || off(out, 16) || off(seq_lens, 4)) return FD_ERR_SHAPE;
    if (rope_stride < fd::kRope || rope_stride % 8 != 0 || rope_stride > (1 << 24)) return FD_ERR_SHAPE;
    if (shape->batch == 0) return FD_OK;
    fd::LatentPromptProblem p{};
    p.q = static_cast<const uint16_t *>(q);
    p.kv = static_cast<const uint16_t *>(kv);
    p.rope = static_cast<const uint16_t *>(rope);
    p.rope_stride = rope_stride;
    p.seq_lens = seq_lens;
    p.out = static_cast<uint16_t *>(out);
    p.B = shape->batch; p.H = shape->n_q_heads; p.Smax = shape->max_seq; p.dtype = dtype;
    p.scale = shape->scale;
    FD_TRY(fd::launch_latent_prefill(p, static_cast<hipStream_t>(stream)));
    return FD_OK;
}

}  // extern "C"
