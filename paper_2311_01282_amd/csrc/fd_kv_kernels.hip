// The paged cache of 16 or 8 bits: rows into it, rows out of it, and decode attention over it.
//
// In 8 bits a row (128 elements of a token and KV head) is c_d 2^e: e the smallest whole number with max |x| <= 448 2^e, c_d
// e4m3.  The scale is a power of two, so that a value is a number of the type (four significant bits) and needs no rounding
// on the way back; what an arbitrary scale could gain, less than a factor of two of the range, is not precision: e4m3 has that down
// to 2^-6 of its 448.
#include "fd_kv.h"

namespace fd {

namespace {

// ---- rows in and out ----
// A row is read, coded and written within eight lanes: 16 elements a lane, from 8 j and from 64 + 8 j, so that eight lanes' loads
// and stores lie side by side.  Memory bounds it: 16001 tokens of 8 heads in 8 bits, 99 MB each way, go in in 19.0 us and out in 16.0 (5.2
// and 6.2 TB/s; a large copy reaches 5.1).

struct KvPlace {
    size_t row;                 // of the pool: (page, head, token in page)
    int token, head;
    bool is_v, live;
};

// Row r of the call: K and V rows of a token's heads, one after the other.  (32 bits: a division of 64 is a hundred instructions.)
__device__ __forceinline__ KvPlace kv_place(const KvPool &pool, const TokenRows &rows, unsigned r)
{
    KvPlace at;
    const unsigned per = 2 * pool.Hkv, token = r / per, rest = r - token * per;
    at.is_v = rest >= (unsigned)pool.Hkv;
    at.head = at.is_v ? rest - pool.Hkv : rest;
    at.token = (int)token;
    at.live = token < (unsigned)rows.n_tokens;
    const int slot = at.live ? rows.slots[token] : -1;
    at.live = slot >= 0 && (slot >> pool.page_shift) < pool.n_pages;         // anything else: padding, left alone
    const int page = at.live ? slot >> pool.page_shift : 0;
    at.row = (((size_t)page * pool.Hkv + at.head) << pool.page_shift) + (at.live ? slot & ((1 << pool.page_shift) - 1) : 0);
    return at;
}

__device__ __forceinline__ unsigned lanes8_max(unsigned x)
{
    auto swap = [](unsigned y, auto control) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)y, decltype(control)::value, 0xf, 0xf, true); };
    x = max(x, swap(x, std::integral_constant<int, 0xB1>{}));
    x = max(x, swap(x, std::integral_constant<int, 0x4E>{}));
    return max(x, swap(x, std::integral_constant<int, 0x141>{}));
}

template <class T, bool k8> __global__ __launch_bounds__(256) void kv_write_kernel(KvPool pool, TokenRows rows)
{
    const KvPlace at = kv_place(pool, rows, blockIdx.x * 32 + (threadIdx.x >> 3));
    const int j = threadIdx.x & 7;
    if (!at.live) return;                                                   // (whole rows of 8 lanes)
    const uint16_t *token = at.is_v ? rows.v + at.token * rows.v_stride : rows.k + at.token * rows.k_stride;
    const u32x4_t *src = reinterpret_cast<const u32x4_t *>(token + at.head * kHeadDim) + j;
    const u32x4_t x[2] = {src[0], src[8]};
    unsigned char *to = at.is_v ? pool.v : pool.k;
    if constexpr (!k8) {
        u32x4_t *dst = reinterpret_cast<u32x4_t *>(to + at.row * (2 * kHeadDim)) + j;
        dst[0] = x[0];
        dst[8] = x[1];
    } else {
        // The largest magnitude, as bits of the type: infinity and NaN are the largest of all.
        unsigned top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const unsigned w = x[i >> 2][i & 3] & 0x7fff7fffu;
            top = max(top, max(w & 0xffffu, w >> 16));
        }
        top = lanes8_max(top);
        const bool odd = top >= T::kInfinity;
        // max <= 1.75 2^8 2^e: the exponent of max, less 8, one more where its mantissa is above 1.75
        const int e = max((int)((__builtin_bit_cast(unsigned, T::lo(top)) + 0x1fffffu) >> 23) - 127 - 8, kLowestExponent);
        const float by = __builtin_bit_cast(float, (unsigned)(127 - e) << 23);
        // (exact, or below what any code stands for)  Where 256 2^e is beyond the type the largest code is 240.
        const float most = e >= T::kLastExponent ? 240.f : 448.f;
        unsigned *codes = reinterpret_cast<unsigned *>(to + at.row * kHeadDim) + 2 * j;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            unsigned c[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const unsigned w0 = x[h][2 * i], w1 = x[h][2 * i + 1];
                auto in = [&](float f) { return __builtin_amdgcn_fmed3f(f * by, -most, most); };
                int y = __builtin_amdgcn_cvt_pk_fp8_f32(in(T::lo(w0)), in(T::hi(w0)), 0, false);
                y = __builtin_amdgcn_cvt_pk_fp8_f32(in(T::lo(w1)), in(T::hi(w1)), y, true);
                c[i] = odd ? 0x7f7f7f7fu : (unsigned)y;                     // NaN
            }
            *reinterpret_cast<u32x2_t *>(codes + 16 * h) = u32x2_t{c[0], c[1]};
        }
        if (j == 0) (at.is_v ? pool.v_scales : pool.k_scales)[at.row] = odd ? 255 : (uint8_t)(e + 127);
    }
}

template <class T, bool k8> __global__ __launch_bounds__(256) void kv_read_kernel(KvPool pool, TokenRows rows)
{
    const KvPlace at = kv_place(pool, rows, blockIdx.x * 32 + (threadIdx.x >> 3));
    const int j = threadIdx.x & 7;
    if (!at.live) return;
    const unsigned char *from = at.is_v ? pool.v : pool.k;
    uint16_t *token = at.is_v ? rows.v + at.token * rows.v_stride : rows.k + at.token * rows.k_stride;
    u32x4_t *dst = reinterpret_cast<u32x4_t *>(token + at.head * kHeadDim) + j;
    u32x4_t x[2];
    if constexpr (k8) {
        const float s = scale_of((at.is_v ? pool.v_scales : pool.k_scales)[at.row]);
        const u32x2_t *codes = reinterpret_cast<const u32x2_t *>(from + at.row * kHeadDim) + j;
        const u32x2_t c[2] = {codes[0], codes[8]};
#pragma unroll
        for (int h = 0; h < 2; ++h) x[h] = from_codes<T>(c[h][0], c[h][1], s);
    } else {
        const u32x4_t *src = reinterpret_cast<const u32x4_t *>(from + at.row * (2 * kHeadDim)) + j;
        x[0] = src[0];
        x[1] = src[8];
    }
    __builtin_nontemporal_store(x[0], dst);
    __builtin_nontemporal_store(x[1], dst + 8);
}

// ---- decode attention ----
// A workgroup takes a chunk of a sequence's keys for up to 16 query heads that share a KV head, a wavefront every fourth block of
// it; nothing of the cache passes through LDS.  The wavefronts' sums are joined at the end, those of chunks by the
// workgroup that arrives last or by a launch of its own.
// Memory bounds it, at 6.5 TB/s for rows in this order: 32 sequences of 4096 keys, 64/8 heads, 8 bits, take 44.9 us (6.05 TB/s), 16 of 512
// .. 4096, 32 heads, 56.1 (6.1), 12 of 5000 .. 20001, 32/8 heads, 16 bits, 102.1 (5.95).  One sequence of 1024 keys takes 7.4: the
// launch, three round trips before the first keys, the hand-over.
constexpr int kBlock = 32;
constexpr int kJoinWorkgroups = 512;             // of a launch that joins its rows itself
constexpr int kJoinInPlace = 16;                 // chunks of a row that the launch itself can join
// Launches of more chunks than this are cut by the sequences' own lengths instead, where there are 2 to 64 of them and no more than 512
// groups: chunks of a number are many short ones where lengths differ, and a workgroup that begins while others run leaves its half of a
// compute unit's loads idle for three round trips.  (us, in chunks of the best number and so: 12 x 32/8 heads x 5000 .. 20001 112.5 / 102.1,
// 8 x 32/8 x 1000 .. 30000 112 / 83, 30 x 8/1 x 1000 .. 20000 37 / 31.8, 16 x 32/8 x 2000 .. 16000, 8 bits 69.5 / 54.6, 64 x 32/8 x 1000 ..
// 16000 392 / 376; of one length 2 x 30000 41.0 / 41.6, 8 x 8000 42.9 / 44.1, 24 x 8192 124 / 132.)
constexpr int kSharesFrom = 256;
constexpr int kMostSequences = 64;               // a lane each
constexpr int kMostShared = 1 << 26;             // max_seq (see pieces_of)
struct DecodeLds {
    WaveSums sums;
    int last;
};

// The group that takes place `at` where the longest sequences come first (of at most 64; of equal ones the first).  Of launches that
// give a compute unit two workgroups the first 256 go in reverse: the longest of the others join the shortest of them.
__device__ __forceinline__ int by_length(const KvProblem &p, int at, int per, int lane)
{
    if (at < kComputeUnits) at = min(kComputeUnits, p.B * per) - 1 - at;
    const int len = lane < p.B ? min(max(p.seq_lens[lane], 0), p.Smax) : -1;
    int rank = 0;
    for (int i = 0; i < p.B; ++i) {
        const int other = __builtin_amdgcn_readlane(len, i);
        rank += (other > len) | ((other == len) & (i < lane));
    }
    const unsigned long long it = __ballot(lane < p.B && rank == at / per);
    return (int)__builtin_ctzll(it) * per + at % per;
}

// ceil(n / by), n + by < 2^21: the quotient of n + by - 1/2 stays 1 / (2 by) away from whole numbers, which no rounding bridges.
__device__ __forceinline__ int pieces_of(int n, int by, float inv_by) { return (int)(((float)(n + by) - 0.5f) * inv_by); }

// Piece `at` of the sequences (of at most 64).  A piece's most keys are as few, a multiple of 128 and at least p.C, as leave no more than
// p.shares pieces, two workgroups a compute unit; or half as many, one each, where those are no longer than kOne times the others' two (1
// and 1.05 measure the same; with 1.15 16 x 32/8 heads x 2000 .. 16000, 8 bits, take 58 us for 55).  Each sequence is then cut into equal ones,
// which may be shorter than p.C; as many as with the most keys each, so that their number is ceil(length / p.C) at most, and their
// indexes stay below p.nc, the places that a row has for its sums.
struct Piece {
    int b, index, keys;                          // b < 0: there is none
};
__device__ __forceinline__ Piece find_piece(const KvProblem &p, int at, int lane)
{
    constexpr int kUnit = 128;
    constexpr float kOne = 1.05f;
    const int len = lane < p.B ? min(max(p.seq_lens[lane], 0), p.Smax) : 0, units = (len + kUnit - 1) / kUnit;
    const int total = __builtin_amdgcn_readlane(lanes_scan(units), 63);
    // Of n units at most n / k + 1 pieces of k: enough of most units each.  32 lengths from the least to that one in the lanes, for
    // half as many pieces and for all.
    const int room = lane < 32 ? p.shares >> 1 : p.shares;
    const int least = max((p.C + kUnit - 1) / kUnit, (total + room - 1) / room);
    const int most = max(least, (total + room - p.B - 1) / (room - p.B));
    const int mine = least + ((most - least) * (lane & 31) + 30) / 31;
    const float inv = 1.f / (float)mine;
    int count = 0;
    for (int b = 0; b < p.B; ++b) count += max(pieces_of(__builtin_amdgcn_readlane(units, b), mine, inv), 1);
    const unsigned long long fits = __ballot(count <= room);
    const int one = __builtin_ctz((unsigned)fits | 1u << 31), two = 32 + __builtin_ctz((unsigned)(fits >> 32) | 1u << 31);
    const float ahead = 2.f * kOne * (float)__builtin_amdgcn_readlane(mine, two);
    const int chosen = (float)__builtin_amdgcn_readlane(mine, one) <= ahead ? one : two;
    const int size = __builtin_amdgcn_readlane(mine, chosen);
    const float by = as_f32((unsigned)__builtin_amdgcn_readlane(__builtin_bit_cast(int, inv), chosen));
    // (a sequence without keys has a piece too; as many, but equal ones)
    const int pieces = lane < p.B ? max(pieces_of(units, size, by), 1) : 0, before = lanes_scan(pieces) - pieces;
    const int keys = kUnit * max(pieces_of(units, max(pieces, 1), 1.f / (float)max(pieces, 1)), 1);
    const unsigned long long it = __ballot(before <= at && at < before + pieces);
    if (!it) return Piece{-1, 0, 0};
    const int b = __builtin_ctzll(it);
    return Piece{b, at - __builtin_amdgcn_readlane(before, b), __builtin_amdgcn_readlane(keys, b)};
}

template <class T, bool k8> __global__ __launch_bounds__(256, 2) void kv_decode_kernel(KvProblem p)
{
    __shared__ DecodeLds lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
    // The first chunk of every row, then the second: every XCD (index modulo 8) has as many of a chunk, which the short rows do not
    // have, as of another.
    const int groups = p.B * p.pool.Hkv * p.tiles, per = p.pool.Hkv * p.tiles;
    int group, chunk, keys = p.C;
    if (p.shares) {
        const Piece at = find_piece(p, blockIdx.x / per, lane);
        if (at.b < 0) return;
        group = at.b * per + blockIdx.x % per;
        chunk = at.index;
        keys = at.keys;
    } else {
        chunk = blockIdx.x / groups;
        group = blockIdx.x % groups;
        if (p.by_length) group = __builtin_amdgcn_readfirstlane(by_length(p, group, per, lane));
    }
    int unit = group;
    const int tile = unit % p.tiles;
    unit /= p.tiles;
    const int hkv = unit % p.pool.Hkv, b = unit / p.pool.Hkv;
    const int start = chunk * keys;
    const int heads = min(p.G - 16 * tile, 16), head0 = hkv * p.G + 16 * tile;      // query heads of this tile
    // Everything that does not depend on the length is under way before it: the queries (which are first in the order of arrival, so that
    // no wait for them is one for keys) and the pages of the first block.
    u32x4_t q[4];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)                             // (columns without a head repeat the last)
        q[kb] = *reinterpret_cast<const u32x4_t *>(p.q + ((size_t)b * p.Hq + head0 + min(n, heads - 1)) * kHeadDim + Keys<T, k8>::element(kb, g));
    asm volatile("" ::: "memory");
    const scalar_i32 table = (scalar_i32)(uintptr_t)(p.table + (size_t)b * p.width);
    int key0 = start + kBlock * wave;
    BlockPages pages = block_pages(table, p.pool.page_shift, key0, p.Smax - 1);
    const int len = min(max(((scalar_i32)(uintptr_t)p.seq_lens)[b], 0), p.Smax);
    const int end = min(len, start + keys);
    if (start >= end) {
        // a sequence without keys: zero rows, by the first chunk (other chunks without keys leave nothing)
        if (chunk == 0)
            for (int i = tid; i < heads * kHeadDim / 2; i += 256)
                reinterpret_cast<unsigned *>(p.out + ((size_t)b * p.Hq + head0) * kHeadDim)[i] = 0u;
        return;
    }
    Softmax<T> state;
    state.clear();
    walk_keys<T, k8, false>(p.pool, hkv, table, pages, key0, end, 0, q, p.scale * kLog2e, lane, state);
    lds.sums.put(state, wave, lane, heads);
    __syncthreads();
    const int chunks = (len + keys - 1) / keys;                            // of this sequence
    for (int h = wave; h < heads; h += 4) {
        float a0, a1, top, sum;
        lds.sums.row(h, lane, a0, a1, top, sum);
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
        // 16 chunks at a time, chunk i's reference and denominator in lane i of every 16; all their partial vectors under way before
        // the first is used
        float top = -INFINITY, a0 = 0.f, a1 = 0.f, sum = 0.f;
        for (int w0 = 0; w0 < chunks; w0 += kJoinInPlace) {
            const int count = min(chunks - w0, kJoinInPlace);
            unsigned long long x[kJoinInPlace];
            const unsigned long long s = load_coherent(reinterpret_cast<const unsigned long long *>(p.ml + slot + w0 + min(n, count - 1)));
#pragma unroll
            for (int i = 0; i < kJoinInPlace; ++i)
                x[i] = load_coherent(reinterpret_cast<const unsigned long long *>(p.num + (slot + w0 + min(i, count - 1)) * kHeadDim) + lane);
            const float mi = n < count ? as_f32((unsigned)s) : -INFINITY, most = row16_max(mi);
            if (most > top) {                                  // (uniform) what the chunks before left, to the new reference
                const float by = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - most);
                a0 *= by;
                a1 *= by;
                sum *= by;
                top = most;
            }
            const float f = n >= count ? 0.f : mi == top ? 1.f : __builtin_amdgcn_exp2f(mi - top);
            sum += row16_sum(n < count ? as_f32((unsigned)(s >> 32)) * f : 0.f);
            each16(std::make_integer_sequence<int, kJoinInPlace>{}, [&](auto of) {
                constexpr int i = decltype(of)::value;
                if (i < count) {
                    const float fi = row16_lane<i>(f);
                    a0 = __builtin_fmaf(as_f32((unsigned)x[i]), fi, a0);
                    a1 = __builtin_fmaf(as_f32((unsigned)(x[i] >> 32)), fi, a1);
                }
            });
        }
        const float inv = 1.f / sum;
        reinterpret_cast<unsigned *>(p.out + out_row * kHeadDim)[lane] = T::pack(a0 * inv, a1 * inv);
    }
}

template <class F> auto by_type(const KvPool &pool, F f)
{
    const std::true_type yes;
    const std::false_type no;
    if (pool.store == kE4m3) return pool.dtype == kF16 ? f(F16{}, yes) : f(BF16{}, yes);
    return pool.dtype == kF16 ? f(F16{}, no) : f(BF16{}, no);
}
dim3 rows_grid(const KvPool &pool, const TokenRows &rows) { return dim3((unsigned)(((long long)rows.n_tokens * 2 * pool.Hkv + 31) / 32)); }

}  // namespace

hipError_t launch_kv_write(const KvPool &pool, const TokenRows &rows, hipStream_t s)
{
    return by_type(pool, [&](auto type, auto k8) {
        return launch(kv_write_kernel<decltype(type), decltype(k8)::value>, rows_grid(pool, rows), dim3(256), s, pool, rows);
    });
}
hipError_t launch_kv_read(const KvPool &pool, const TokenRows &rows, hipStream_t s)
{
    return by_type(pool, [&](auto type, auto k8) {
        return launch(kv_read_kernel<decltype(type), decltype(k8)::value>, rows_grid(pool, rows), dim3(256), s, pool, rows);
    });
}
hipError_t launch_kv_decode(const KvProblem &p_, hipStream_t s)
{
    KvProblem p = p_;
    const long long per = (long long)p.pool.Hkv * p.tiles, groups = p.B * per;
    long long workgroups = groups * p.nc;
    if (p.nc > 1 && workgroups > kSharesFrom && p.B > 1 && p.B <= kMostSequences && groups <= kJoinWorkgroups && p.Smax <= kMostShared) {
        // a round of two workgroups a compute unit, or as many rounds as give a sequence four pieces
        p.shares = (int)((4 * groups + kJoinWorkgroups - 1) / kJoinWorkgroups * kJoinWorkgroups / per);
        workgroups = p.shares * per;
    } else if (p.nc > kJoinInPlace || workgroups > kJoinWorkgroups) {
        p.counters = nullptr;
    }
    p.by_length = p.nc == 1 && p.B > 1 && p.B <= kMostSequences && workgroups > kComputeUnits;
    const hipError_t e = by_type(p.pool, [&](auto type, auto k8) {
        return launch(kv_decode_kernel<decltype(type), decltype(k8)::value>, dim3((unsigned)workgroups), dim3(256), s, p);
    });
    if (e != hipSuccess || p.nc == 1 || p.counters) return e;
    JoinProblem j{p.num, p.ml, p.seq_lens, p.out, p.B * p.Hq, p.Hq, p.C, p.nc, p.Smax, kHeadDim, p.pool.dtype};
    return launch_join(j, s);
}

}  // namespace fd
