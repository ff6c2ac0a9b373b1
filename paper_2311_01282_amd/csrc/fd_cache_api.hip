// C-ABI entry points around the smaller paged caches: argument checks, workspace carving, launches.
#include "../../include/fdattn.h"
#include "fd_cache.h"

#include <algorithm>
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

// K and V rows of a call's tokens, as the caller has them.
fd_status token_rows(int Hkv, const void *k, int64_t k_stride, const void *v, int64_t v_stride, int32_t n_tokens, const int32_t *slot_map,
                     fd::TokenRows *R)
{
    if (!k || !v || !slot_map) return FD_ERR_NULL;
    const long long width = (long long)Hkv * fd::kHeadDim;
    if (n_tokens < 0 || off(k, 16) || off(v, 16) || off(slot_map, 4) || k_stride < width || v_stride < width || k_stride % 8 != 0 ||
        v_stride % 8 != 0)
        return FD_ERR_SHAPE;
    if ((long long)n_tokens * 2 * Hkv >= kMostThreads / 16) return FD_ERR_UNSUPPORTED;
    *R = fd::TokenRows{const_cast<uint16_t *>(static_cast<const uint16_t *>(k)),
                        const_cast<uint16_t *>(static_cast<const uint16_t *>(v)), k_stride, v_stride, slot_map, n_tokens};
    return FD_OK;
}
fd_status nibble_rows(const fd_nibble_pool *pool, const void *k, int64_t k_stride, const void *v, int64_t v_stride, int32_t n_tokens,
                   const int32_t *slot_map, fd::NibblePool *P, fd::TokenRows *R)
{
    const fd_status st = nibble_pool(pool, P);
    if (st != FD_OK) return st;
    return token_rows(P->Hkv, k, k_stride, v, v_stride, n_tokens, slot_map, R);
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

fd_status kv_pool(const fd_kv_pool *pool, fd::KvPool *out)
{
    if (!pool || !pool->k || !pool->v) return FD_ERR_NULL;
    const bool coded = pool->store == FD_E4M3;
    if (coded && (!pool->k_scales || !pool->v_scales)) return FD_ERR_NULL;
    fd::KvPool o{};
    const fd_status st = check_pages(pool->n_pages, pool->page_size, &o.page_shift);
    if (st != FD_OK) return st;
    if (pool->n_kv_heads < 1 || pool->head_dim < 1) return FD_ERR_SHAPE;
    if (off(pool->k, 16) || off(pool->v, 16) || (coded && (off(pool->k_scales, 16) || off(pool->v_scales, 16)))) return FD_ERR_SHAPE;
    if (pool->head_dim != fd::kHeadDim || pool->n_kv_heads > 65535 || !known_type(pool->dtype) || (!coded && pool->store != pool->dtype))
        return FD_ERR_UNSUPPORTED;
    o.k = static_cast<unsigned char *>(pool->k);
    o.v = static_cast<unsigned char *>(pool->v);
    o.k_scales = static_cast<uint8_t *>(pool->k_scales);
    o.v_scales = static_cast<uint8_t *>(pool->v_scales);
    o.n_pages = pool->n_pages;
    o.Hkv = pool->n_kv_heads;
    o.store = pool->store;
    o.dtype = pool->dtype;
    *out = o;
    return FD_OK;
}
fd_status kv_rows(const fd_kv_pool *pool, const void *k, int64_t k_stride, const void *v, int64_t v_stride, int32_t n_tokens,
                  const int32_t *slot_map, fd::KvPool *P, fd::TokenRows *R)
{
    const fd_status st = kv_pool(pool, P);
    if (st != FD_OK) return st;
    return token_rows(P->Hkv, k, k_stride, v, v_stride, n_tokens, slot_map, R);
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

fd_status kv_split(const fd_shape *sh, Split *S) { return split(sh, fd::kHeadDim, fd::kHeadDim, 64, S); }

// The packed tokens: tiles of 128 (token, query head) rows of a KV head, of which no sequence leaves more than one unfilled.  A sequence of
// t tiles and L keys is cut into ceil(L / (chunk t)) pieces, so that it has at most t + L / chunk (tile, piece) units; a unit that is
// not its rows' only one leaves their sums in the workspace.
fd_status prompt_split(const fd_shape *sh, int32_t n_tokens, long long *units, Split *S)
{
    const fd_status st = check_shape(sh, fd::kHeadDim);
    if (st != FD_OK) return st;
    if (sh->chunk <= 0 || n_tokens < 0) return FD_ERR_SHAPE;
    const long long tiles = (long long)n_tokens * (sh->n_q_heads / sh->n_kv_heads) / 128 + sh->batch;
    *units = tiles + (sh->chunk < sh->max_seq ? (long long)sh->batch * (sh->max_seq / sh->chunk) : 0);
    if (*units > kMostThreads / 512 || *units * sh->n_kv_heads > kMostThreads / 512) return FD_ERR_UNSUPPORTED;
    // (the launch that joins pieces has a token's 16 heads a workgroup)
    if (sh->chunk < sh->max_seq && (n_tokens > kMostThreads / 512 || sh->n_q_heads > 16 * 65535)) return FD_ERR_UNSUPPORTED;
    const size_t slots = sh->chunk < sh->max_seq ? (size_t)(*units * sh->n_kv_heads * 128) : 0;
    S->num = align_up(kCounters * sizeof(int32_t));
    S->ml = align_up(S->num + slots * fd::kHeadDim * sizeof(float));
    S->total = align_up(S->ml + slots * sizeof(float2));
    return FD_OK;
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
    fd::TokenRows R;
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
    fd::TokenRows R;
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

fd_status fd_kv_write(const fd_kv_pool *pool, const void *k, int64_t k_stride, const void *v, int64_t v_stride, int32_t n_tokens,
                      const int32_t *slot_map, void *stream)
{
    fd::KvPool P;
    fd::TokenRows R;
    const fd_status st = kv_rows(pool, k, k_stride, v, v_stride, n_tokens, slot_map, &P, &R);
    if (st != FD_OK) return st;
    if (n_tokens == 0) return FD_OK;
    FD_TRY(fd::launch_kv_write(P, R, static_cast<hipStream_t>(stream)));
    return FD_OK;
}

fd_status fd_kv_read(const fd_kv_pool *pool, const int32_t *slot_map, int32_t n_tokens, void *k, int64_t k_stride, void *v,
                     int64_t v_stride, void *stream)
{
    fd::KvPool P;
    fd::TokenRows R;
    const fd_status st = kv_rows(pool, k, k_stride, v, v_stride, n_tokens, slot_map, &P, &R);
    if (st != FD_OK) return st;
    if (n_tokens == 0) return FD_OK;
    FD_TRY(fd::launch_kv_read(P, R, static_cast<hipStream_t>(stream)));
    return FD_OK;
}

size_t fd_kv_workspace_bytes(const fd_shape *shape)
{
    Split S;
    return kv_split(shape, &S) == FD_OK ? S.total : 0;
}

int32_t fd_kv_pick_chunk(const fd_shape *shape)
{
    if (check_shape(shape, fd::kHeadDim) != FD_OK) return 0;
    const long long units = (long long)shape->batch * shape->n_kv_heads * ((shape->n_q_heads / shape->n_kv_heads + 15) / 16);
    // A workgroup draws what its compute unit can take (four wavefronts, a block each under way), and costs three round trips to memory
    // before its first keys arrive.  So whole rows, which the launch sorts by length, where they fill the chip and are short enough not to
    // outlast the others; where chunks of 512 keys would fill it more than once and the launch makes pieces by the sequences' lengths, no
    // more of a sequence than it has chunks, those; otherwise one workgroup a compute unit, in chunks of 256 keys at least and 2048 at most.
    // (Whole call, us, chunks of 256 / 512 / 1024 / 2048 / 4096 keys, the choice marked: 32 x 64/8 heads x 4096, 8 bits 51 / 51 / 51 / 51 /
    // *44, 16 x 32 x 512 .. 4096, 8 bits 65 / 65 / 65 / 70 / *56, 64 x 32/8 x 500 .. 4000, 16 bits 115 / 112 / 111 / 109 / *93, 12 x 32/8 x
    // 5000 .. 20001, 16 bits 103 / *102 / 102 / 102 / 105, 4 x 32/8 x 1000 .. 30000, 16 bits 33 / *33 / 33 / 38 / 64, 1 x 32 x 8192, 8 bits 19 /
    // 16.3 / *15.7 / 23 / 37, 4 x 64/8 x 2000, 8 bits *9.5 / 11.2 / 14.6 / 15.5.)
    const long long S = shape->max_seq, chip = fd::kComputeUnits;
    if (units >= chip && S <= 4096) return chunk_for(shape->max_seq, 1, 1, 256, 64);
    if (shape->batch > 1 && shape->batch <= 64 && units <= 2 * chip && units * ((S + 511) / 512) > chip) {
        // (at most 128 chunks a row, and their sums, 520 bytes for each head, 128 MiB)
        const long long slots = (128ll << 20) / (520ll * shape->batch * shape->n_q_heads), nc = std::max(std::min(slots, 128ll), 1ll);
        return (int32_t)std::min<long long>(std::max<long long>(512, ((S + nc - 1) / nc + 63) / 64 * 64), 16384);
    }
    const long long nc = std::max(units > 0 ? chip / units : 1, (S + 2047) / 2048);
    int32_t chunk = chunk_for(shape->max_seq, 1, nc, 256, 64);
    // (longer where there would be more of them than a launch may have)
    const long long rows = (long long)shape->batch * shape->n_q_heads;
    while (chunk < 16384 && rows * ((S + chunk - 1) / chunk) > kMostThreads / 512) chunk = std::min(2 * chunk, 16384);
    return chunk;
}

fd_status fd_kv_decode_attn(const fd_shape *shape, const fd_kv_pool *pool, const void *q, const int32_t *block_table, const int32_t *seq_lens,
                            void *out, fd_workspace ws, void *stream)
{
    Split S;
    fd_status st = kv_split(shape, &S);
    if (st != FD_OK) return st;
    fd::KvProblem p{};
    st = kv_pool(pool, &p.pool);
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
    FD_TRY(fd::launch_kv_decode(p, static_cast<hipStream_t>(stream)));
    return FD_OK;
}

size_t fd_kv_prefill_workspace_bytes(const fd_shape *shape, int32_t n_tokens)
{
    Split S;
    long long units;
    return prompt_split(shape, n_tokens, &units, &S) == FD_OK ? S.total : 0;
}

int32_t fd_kv_prefill_pick_chunk(const fd_shape *shape, int32_t n_tokens)
{
    if (check_shape(shape, fd::kHeadDim) != FD_OK || n_tokens < 0) return 0;
    if (shape->batch == 0 || n_tokens == 0) return shape->max_seq;
    const long long B = shape->batch, Hkv = shape->n_kv_heads, S = shape->max_seq;
    const long long tiles = (long long)n_tokens * (shape->n_q_heads / shape->n_kv_heads) / 128, whole = std::max(tiles, std::min<long long>(B, n_tokens));
    const bool single = tiles < B;
    long long chunk = S;
    if (single) {
        // Sequences of few rows are bound by memory and cut into one workgroup a compute unit, of 768 keys at least; where there are as
        // many units without that, only walks that would outlast the others are cut.
        if (whole * Hkv >= fd::kComputeUnits * 5 / 4)
            chunk = S <= 4096 ? S : 2048;
        else if (S > 1024)
            chunk = std::min<long long>(std::max((whole * Hkv * S + 2 * fd::kComputeUnits - 1) / (2 * fd::kComputeUnits), 768ll), 2048);
    } else {
        // Prompts, us in n pieces.  A step of 32 keys takes 0.62 alone on a compute unit and 1.05 beside another workgroup, of which longer
        // units have less the shorter the others are; sums of pieces, 520 bytes a row, are written and read again, by a launch more.
        // (Uncut / as picked / in the pieces that measured best: 512 tokens over 30000, 64/8 heads, 8 bits 645 / 533 / 533, 256 over 30000,
        // 32/8 533 / 141 / 141, 100 over 8000, 64/8 147 / 52 / 48, 8 x 64 over 2000 .. 4000, 32/8 76 / 53 / 52, 64 over 1000, 32/8 25 / 19 / 19,
        // 4000 of 8 heads that share one 77 / 58 / 58, 5000 of 4 heads 93 / 49 / 49, 2500 over 20000, 32/8 1005 / 905 / 896; not cut: 1200, 32/8
        // 29, in two 33, 1600 over 3000 109, in two 128, 16000 2039, in two 2145.)
        const double chip = fd::kComputeUnits, W = (double)(whole * Hkv), steps = S / 32.0, rows = (double)n_tokens * shape->n_q_heads;
        const double f = 1.0 - std::fmin((double)n_tokens / (double)(2 * B * S), 0.5);      // keys of a row on the average, of S
        double least = 0.0;
        long long pieces = 1;
        for (long long n = 1; n <= 64; ++n) {
            const double some = f + (1.0 - f) / n, units = W * n * some, even = f / some;   // units with keys; their mean length, of the longest
            // (half-full last rounds cost the more the more alike the units are: 0 where they go down to nothing)
            const double alike = std::fmax(2.0 * even - 1.0, 0.0), rounds = units / (2.0 * chip);
            const double step = units <= chip ? 0.62 : rounds <= 1.0 ? 0.62 + 0.43 * alike : std::fmax(0.525 * (2.0 * rounds * even + alike), 0.62);
            double t = steps / n * step;
            if (n > 1) t += 5.0 + 8.0 * std::fmax(rounds - 1.0, 0.0) + units * rows / W * 1040.0 / 5e6;
            if (n == 1 || t < least) {
                least = t;
                pieces = n;
            }
        }
        const long long each = std::max<long long>(tiles / B, 1);
        if (pieces > 1) chunk = (S + pieces * each - 1) / (pieces * each);
    }
    // ... and no workspace of more than 256 MiB
    fd_shape cut = *shape;
    for (;; chunk *= 2) {
        if (chunk >= S) return shape->max_seq;
        cut.chunk = (int32_t)chunk;
        const size_t bytes = fd_kv_prefill_workspace_bytes(&cut, n_tokens);
        if (bytes > 0 && bytes <= (256u << 20)) return cut.chunk;
    }
}

fd_status fd_kv_prefill_attn(const fd_shape *shape, const fd_kv_pool *pool, const void *q, int64_t q_stride, int32_t n_tokens,
                             const int32_t *token_starts, const int32_t *block_table, const int32_t *seq_lens, void *out, fd_workspace ws,
                             void *stream)
{
    Split S;
    long long units;
    fd_status st = prompt_split(shape, n_tokens, &units, &S);
    if (st != FD_OK) return st;
    fd::KvPromptProblem p{};
    st = kv_pool(pool, &p.pool);
    if (st != FD_OK) return st;
    if (!q || !token_starts || !block_table || !seq_lens || !out) return FD_ERR_NULL;
    if (off(q, 16) || off(out, 16) || off(token_starts, 4) || off(block_table, 4) || off(seq_lens, 4)) return FD_ERR_SHAPE;
    if (q_stride < (int64_t)shape->n_q_heads * fd::kHeadDim || q_stride % 8 != 0) return FD_ERR_SHAPE;
    if (pool->n_kv_heads != shape->n_kv_heads || shape->max_seq % pool->page_size != 0) return FD_ERR_SHAPE;
    if (bad_ws(ws, S)) return FD_ERR_WORKSPACE;
    if (shape->batch == 0 || n_tokens == 0) return FD_OK;
    p.q = static_cast<const uint16_t *>(q);
    p.q_stride = q_stride;
    p.starts = token_starts;
    p.seq_lens = seq_lens;
    p.table = block_table;
    p.out = static_cast<uint16_t *>(out);
    p.num = reinterpret_cast<float *>(static_cast<char *>(ws.ptr) + S.num);
    p.ml = reinterpret_cast<float2 *>(static_cast<char *>(ws.ptr) + S.ml);
    p.B = shape->batch; p.Hq = shape->n_q_heads; p.G = shape->n_q_heads / shape->n_kv_heads; p.n_tokens = n_tokens;
    p.units = (int)units;
    p.C = shape->chunk; p.Smax = shape->max_seq; p.width = shape->max_seq / pool->page_size;
    p.scale = shape->scale;
    FD_TRY(fd::launch_kv_prefill(p, static_cast<hipStream_t>(stream)));
    return FD_OK;
}

}  // extern "C"
