// Attention of a step's new tokens over the paged cache: sequences one behind the other, each token over its sequence's keys up to
// its own position.
//
// A row is a (token, query head) pair; the G query heads that share a KV head go together, rows r = G i + j of head j of the
// sequence's new token i, so that a tile of neighbouring rows reads the same keys whatever G is and however few tokens there are.
// A workgroup owns a tile of 128 rows, a wavefront 32 of them, and walks along the keys in steps of 32, which pass through LDS.
// Lanes (32 x 32 x 16): c = lane % 32, h = lane / 32;
//   scores   S^T[key][row] = K . Q^T: A = the 32 keys of a step in LDS, B = Q^T in registers.  Row 8 j + 4 h + i of the result
//            is key 16 (j / 2) + 8 h + 4 (j % 2) + i, so that lane (c, h) holds of row c the keys 16 m + 8 h + 0 .. 7: the B
//            operands m = 0, 1 of
//   output   O^T[d][row] = V^T . P^T: A = V^T by the transposing LDS read.
// Softmax with a running maximum per row; the weights are of the type (one rounding, as large as the output's own), their sum
// is that of the rounded ones, in fp32.
//
// What bounds it: 512 operations for each (row, key), of which a plain product of 8192^3 reaches 1.34 (fp16) and 1.40 (bf16) PFLOP/s, and
// in long calls the power that they draw: one prompt of 8001 tokens, 32/8 heads, bf16, takes 506 us (1.04 PFLOP/s), with queries
// and keys of zeros 399 (1.31).  So products of 32 x 32, whose operands serve twice as many rows or keys as those of 16 x 16 (a wavefront
// reads 16 KiB of LDS for 0.5 MFLOP), rows in lanes, so that a softmax needs one exchange, of two lanes, and two workgroups a compute
// unit, one with products while the other has exponentials.  A step takes 1.05 us (both), one workgroup alone 0.62.  Outside its loop a
// workgroup takes 8 us: 2 until it knows its sequence, 3 to 4 until the page table, the first rows and the queries have arrived one
// after the other, 2 for the output; five prompts of 150 to 2000 tokens, 32 heads, fp16, take 103 us for 51 of products.
// Rows of 8 bits are converted once a workgroup, a vector instruction an element: 700 .. 3000 tokens over up to 1500, 32/4 heads, bf16, take
// 244 us (0.90 PFLOP/s), 512 over 30000, 64/8, fp16, 533 (0.95).
#include <utility>

#include "fd_kv.h"

namespace fd {

namespace {

constexpr int kTileRows = 128, kStep = 32, kRingK = 4, kRingV = 3, kRowBytes = 2 * kHeadDim, kStepBytes = kStep * kRowBytes;

typedef float f32x16_t __attribute__((ext_vector_type(16)));
template <class T> __device__ __forceinline__ f32x16_t mfma32(u32x4_t a, u32x4_t b, f32x16_t c)
{
    if constexpr (std::is_same<T, F16>::value)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
// sum += a + b of two numbers of the type
template <class T> __device__ __forceinline__ float add_pair(unsigned pair, float sum)
{
    if constexpr (std::is_same<T, F16>::value)
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2_t, pair), __builtin_bit_cast(f16x2_t, 0x3c003c00u), sum, false);
    else
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pair), __builtin_bit_cast(bf16x2_t, 0x3f803f80u), sum, false);
}
// the larger of the two halves' values, in both
__device__ __forceinline__ float halves_max(float a)
{
    const unsigned u = __builtin_bit_cast(unsigned, a);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned x = r[0], y = r[1];
    return fmaxf(as_f32(x), as_f32(y));
}

// The places of 16-byte piece x of row r of a step's keys, x ^ k_place(r), and of its 32-byte unit x of the values, x ^ v_unit(r):
// the 16 rows that 16 neighbouring lanes read lie in places of their own, and so do the eight units of the two neighbouring
// groups of 16 lanes that a transposing read takes at a time, rows 4 i .. 4 i + 3 of two units.
__device__ __forceinline__ int k_place(int r) { return (r & 3) | ((r >> 3) & 1) << 2 | ((r >> 2) & 1) << 3; }
__device__ __forceinline__ int v_unit(int r) { return 2 * (r & 3); }

struct PromptLds {
    alignas(256) unsigned char k[kRingK][kStepBytes];
    alignas(256) unsigned char v[kRingV][kStepBytes];
};

__device__ __forceinline__ unsigned lds_address(const void *p)
{
    return __builtin_amdgcn_readfirstlane(
        (unsigned)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const unsigned char *)p));
}
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t *lds_s16x4;
typedef __attribute__((address_space(3))) u32x4_t *lds_u32x4;
// (In assembly: of loads into LDS that the compiler knows it would wait before every transposing read.  A scalar register that a
// vector instruction has written is read by a load five states later at the earliest; the compiler sees to that in its own code
// only.)
__device__ __forceinline__ void load_to_lds(u32x4_t rs, int voff, unsigned lds_1k)
{
    asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(lds_1k), "v"(voff), "s"(rs) : "memory");
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
__device__ __forceinline__ u32x4_t window(const void *base, int bytes)
{
    const unsigned long long at = reinterpret_cast<unsigned long long>(base);
    return u32x4_t{(unsigned)__builtin_amdgcn_readfirstlane((unsigned)at),
                   (unsigned)__builtin_amdgcn_readfirstlane((unsigned)(at >> 32)) & 0xffffu,
                   (unsigned)__builtin_amdgcn_readfirstlane((unsigned)bytes), 0x00027000u};
}

constexpr int kFewRows = 16;
// Units of work of a KV head: a sequence of t tiles is cut into pieces of p.C t keys (rounded up to 64), as fewer tiles need more pieces
// to fill the chip; piece by piece, a piece's tiles from the last to the first.  Sequences of up to 64 go from the longest to the
// shortest (of equal ones the first), of more in their order; those of few rows count half: a key takes them 16 ns, others 33 (31 single
// tokens beside a prompt of 1492, 32/8 heads: 140 us by the number of keys alone, 127 so).
struct Sequence {
    int b, first, tokens, len;                   // its first new token, their number, its keys
    int tiles, piece, units, before;             // keys of a piece; its units, and those of the sequences in front
};
__device__ __forceinline__ Sequence lane_sequence(const Sequence &x, int lane)
{
    auto of = [&](int v) { return __builtin_amdgcn_readlane(v, lane); };
    return Sequence{of(x.b), of(x.first), of(x.tokens), of(x.len), of(x.tiles), of(x.piece), of(x.units), of(x.before)};
}
// The sequences of 64 lanes, in that order, behind `before` units of others.
__device__ __forceinline__ Sequence load_sequences(const KvPromptProblem &p, int b0, int before, int lane)
{
    Sequence x{b0 + lane, 0, 0, -1, 0, 64, 0, 0};
    if (x.b < p.B) {
        x.first = min(max(p.starts[x.b], 0), p.n_tokens);
        x.tokens = max(min(max(p.starts[x.b + 1], 0), p.n_tokens) - x.first, 0);
        x.len = min(max(p.seq_lens[x.b], 0), p.Smax);
    }
    if (p.B <= 64) {
        const int cost = x.tokens * p.G <= kFewRows ? x.len >> 1 : x.len;      // (of lanes without a sequence -1)
        int rank = lane;
        for (int i = 0; i < p.B; ++i) {
            const int other = __builtin_amdgcn_readlane(cost, i);
            rank += (int)(i > lane && other > cost) - (int)(i < lane && other < cost);
        }
        // (a permutation: lanes without a sequence are the last before and after)
        x.b = __builtin_amdgcn_ds_permute(rank << 2, x.b);
        x.first = __builtin_amdgcn_ds_permute(rank << 2, x.first);
        x.tokens = __builtin_amdgcn_ds_permute(rank << 2, x.tokens);
        x.len = __builtin_amdgcn_ds_permute(rank << 2, x.len);
    }
    x.tiles = (x.tokens * p.G + kTileRows - 1) / kTileRows;
    // (in 32 bits: beyond Smax, which is 2^30 at most, a piece is the whole sequence)
    const unsigned most = (unsigned)(p.Smax + 63) & ~63u;
    x.piece = (int)most;
    x.units = x.tiles;
    if (p.C < p.Smax && x.len > 0 && x.tiles > 0) {        // in pieces of one length, as many as those of p.C t keys (64 or more)
        const int piece = (int)min(__umulhi((unsigned)p.C, (unsigned)x.tiles) ? most : min((unsigned)p.C * (unsigned)x.tiles, most) + 63, most) & ~63;
        const int n = (x.len + piece - 1) / piece;
        x.piece = ((x.len + n - 1) / n + 63) & ~63;
        x.units = x.tiles * ((x.len + x.piece - 1) / x.piece);
    }
    x.before = before + lanes_scan(x.units) - x.units;
    return x;
}
// The first sequence in that order for which `is` holds; b < 0: none.
template <class F> __device__ __forceinline__ Sequence find_sequence(const KvPromptProblem &p, int lane, F is)
{
    int before = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const Sequence x = load_sequences(p, b0, before, lane);
        const unsigned long long found = __ballot(is(x));
        if (found) return lane_sequence(x, __builtin_ctzll(found));
        before = __builtin_amdgcn_readlane(x.before + x.units, 63);
    }
    return Sequence{-1, 0, 0, 0, 0, 64, 0, 0};
}
// A window of memory that loads the compiler knows of go through: 0 behind it.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void *base, int bytes)
{
    const unsigned long long at = reinterpret_cast<unsigned long long>(base);
    const unsigned low = __builtin_amdgcn_readfirstlane((unsigned)at), high = __builtin_amdgcn_readfirstlane((unsigned)(at >> 32));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>((unsigned long long)high << 32 | low), 0,
                                             __builtin_amdgcn_readfirstlane(bytes), 0x00027000);
}

// A piece of a sequence of up to 16 rows, single tokens among them: what bounds it is memory, and the four wavefronts share its keys,
// which pass from the cache into registers.
template <class T, bool k8>
__device__ __forceinline__ void few_rows(const KvPromptProblem &p, const Sequence &at, int chunk, int hkv, WaveSums &sums, int lane, int wave)
{
    const int n = lane & 15, g = lane >> 4, rows = at.tokens * p.G, ahead = at.len - at.tokens, begin = chunk * at.piece;
    const int row = min(n, rows - 1), position = ahead + row / p.G, end = min(at.len, begin + at.piece);
    const uint16_t *from = p.q + (size_t)(at.first + row / p.G) * p.q_stride + (size_t)(hkv * p.G + row % p.G) * kHeadDim;
    u32x4_t q[4];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) q[kb] = *reinterpret_cast<const u32x4_t *>(from + Keys<T, k8>::element(kb, g));
    asm volatile("" ::: "memory");
    const scalar_i32 table = (scalar_i32)(uintptr_t)(p.table + (size_t)at.b * p.width);
    const int key0 = begin + 32 * wave;
    Softmax<T> state;
    state.clear();
    const BlockPages pages = block_pages(table, p.pool.page_shift, min(key0, max(end - 1, 0)), max(end - 1, 0));
    walk_keys<T, k8, true>(p.pool, hkv, table, pages, key0, end, position, q, p.scale * kLog2e, lane, state);
    sums.put(state, wave, lane, rows);
    __syncthreads();
    for (int r = wave; r < rows; r += 4) {
        float a0, a1, top, sum;
        sums.row(r, lane, a0, a1, top, sum);
        const int seen = ahead + r / p.G + 1, chunks = (seen + at.piece - 1) / at.piece;     // (of rows without keys: none)
        if (chunks <= 1) {
            if (chunk > 0) continue;
            const float inv = 1.f / sum;
            const size_t out_row = (size_t)(at.first + r / p.G) * p.Hq + hkv * p.G + r % p.G;
            reinterpret_cast<unsigned *>(p.out + out_row * kHeadDim)[lane] = seen > 0 ? T::pack(a0 * inv, a1 * inv) : 0u;
        } else if (chunk < chunks && at.before + at.units <= p.units) {
            const size_t slot = ((size_t)(at.before + chunk) * p.pool.Hkv + hkv) * kTileRows + r;
            *reinterpret_cast<float2 *>(p.num + slot * kHeadDim + 2 * lane) = float2{a0, a1};
            if (lane == 0) p.ml[slot] = float2{top, sum};
        }
    }
}

template <class T, bool k8> __global__ __launch_bounds__(256, 2) void kv_prefill_kernel(KvPromptProblem p)
{
    __shared__ union { PromptLds lds; WaveSums sums; } both;
    PromptLds &lds = both.lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, h = lane >> 5;
    // Of launches that give no compute unit more than two workgroups the first one each go in reverse: the longest of the others join the
    // shortest of them.  (2000 tokens, 32/8 heads 54.4 -> 50.5 us, 1500 over 500 52.8 -> 47.5, 300 and 800, 64/8 24.8 -> 21.6.)
    const int hkv = blockIdx.x % p.pool.Hkv, turn = blockIdx.x / p.pool.Hkv, alone = kComputeUnits / p.pool.Hkv;
    const int unit = gridDim.x <= 2 * kComputeUnits && gridDim.x > kComputeUnits && turn < alone ? alone - 1 - turn : turn;
    const Sequence at = find_sequence(p, lane, [&](const Sequence &x) { return unit < x.before + x.units; });
    if (at.b < 0) return;
    const int index = unit - at.before;
    if (at.tokens * p.G <= kFewRows) {
        few_rows<T, k8>(p, at, index, hkv, both.sums, lane, wave);
        return;
    }
    const int chunk = index / at.tiles, tile = at.tiles - 1 - index % at.tiles;
    const int rows = at.tokens * p.G, row0 = tile * kTileRows + 32 * wave;          // of the sequence
    const int len = at.len, ahead = len - at.tokens;          // position of new token 0
    const int begin = chunk * at.piece, limit = min(len, begin + at.piece);
    auto keys_upto = [&](int row) { return min(ahead + row / p.G + 1, limit) - begin; };      // of the chunk, that a row sees
    const int tile_keys = keys_upto(min(tile * kTileRows + kTileRows, rows) - 1);
    if (tile_keys <= 0 && chunk > 0) return;
    const int row = min(row0 + c, rows - 1), token = row / p.G, head = hkv * p.G + row % p.G, position = ahead + token;
    const bool live = row0 + c < rows;
    const size_t out_row = (size_t)(at.first + token) * p.Hq + head;
    uint16_t *out = p.out + out_row * kHeadDim + 4 * h;
    if (tile_keys <= 0) {                                      // (in the first chunk only) no row of the tile sees a key
        if (live)
#pragma unroll
            for (int i = 0; i < 16; ++i) *reinterpret_cast<u32x2_t *>(out + 8 * i) = u32x2_t{0u, 0u};
        return;
    }
    // steps of the workgroup, of the wavefront, and those of it in which every row sees every key
    const int steps = (tile_keys + kStep - 1) / kStep;
    const int mine = row0 < rows ? max(keys_upto(min(row0 + 32, rows) - 1) + kStep - 1, 0) / kStep : 0;
    const int full = row0 < rows ? max(keys_upto(row0), 0) / kStep : 0;

    const unsigned lds_k = lds_address(lds.k[0]), lds_v = lds_address(lds.v[0]);

    // A wavefront fetches rows 8 wave .. + 7 of a step's keys and values, four rows an instruction: they share a page.  Rows
    // without keys arrive as zeros.
    const scalar_i32 table = (scalar_i32)(uintptr_t)(p.table + (size_t)at.b * p.width);
    const int key_mine = begin + 8 * wave, last = begin + tile_keys - 1, shift = p.pool.page_shift;
    auto page_entry = [&](int s) { return table[min(key_mine + kStep * s, last) >> shift]; };
    auto row_place = [&](int entry, int s) {                   // the row of the pool
        const int page = min(max(entry, 0), p.pool.n_pages - 1);
        return (((size_t)page * p.pool.Hkv + hkv) << shift) + ((key_mine + kStep * s) & ((1 << shift) - 1));
    };
    auto rows_of = [&](int s) { return min(max(last + 1 - key_mine - kStep * s, 0), 8); };
    unsigned k_to = 0, v_to = 0;                               // places in the rings
    auto next_k = [&] { k_to = k_to == kRingK - 1 ? 0 : k_to + 1; };
    auto next_v = [&] { v_to = v_to == kRingV - 1 ? 0 : v_to + 1; };
    // 16 bits: straight into LDS, four rows an instruction
    int koff[2], voff[2];
    // 8 bits: through registers, 16 codes a lane, and into LDS as numbers of the type
    u32x4_t codes_k, codes_v;
    unsigned byte_k, byte_v;
    if constexpr (!k8) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = 8 * wave + 4 * i + (lane >> 4), x = lane & 15;
            koff[i] = (4 * i + (lane >> 4)) * kRowBytes + ((x ^ k_place(r)) << 4);
            voff[i] = (4 * i + (lane >> 4)) * kRowBytes + ((x ^ (v_unit(r) << 1)) << 4);
        }
    } else {
        const int r = 8 * wave + (lane >> 3), x = 2 * (lane & 7);
        koff[0] = r * kRowBytes + ((x ^ k_place(r)) << 4);
        koff[1] = r * kRowBytes + (((x + 1) ^ k_place(r)) << 4);
        voff[0] = r * kRowBytes + ((x ^ (v_unit(r) << 1)) << 4);
        voff[1] = voff[0] + 16;
    }
    auto fetch_k = [&](size_t place, int n) {
        if constexpr (!k8) {
            const u32x4_t r = window(p.pool.k + place * kRowBytes, n * kRowBytes);
#pragma unroll
            for (int i = 0; i < 2; ++i) load_to_lds(r, koff[i], lds_k + k_to * kStepBytes + (2 * wave + i) * 1024);
            next_k();
        } else {
            codes_k = __builtin_amdgcn_raw_buffer_load_b128(buffer(p.pool.k + place * kHeadDim, n * kHeadDim), lane * 16, 0, 0);
            byte_k = __builtin_amdgcn_raw_buffer_load_b8(buffer(p.pool.k_scales + place, n), lane >> 3, 0, 0);
        }
    };
    auto fetch_v = [&](size_t place, int n) {
        if constexpr (!k8) {
            const u32x4_t r = window(p.pool.v + place * kRowBytes, n * kRowBytes);
#pragma unroll
            for (int i = 0; i < 2; ++i) load_to_lds(r, voff[i], lds_v + v_to * kStepBytes + (2 * wave + i) * 1024);
            next_v();
        } else {
            codes_v = __builtin_amdgcn_raw_buffer_load_b128(buffer(p.pool.v + place * kHeadDim, n * kHeadDim), lane * 16, 0, 0);
            byte_v = __builtin_amdgcn_raw_buffer_load_b8(buffer(p.pool.v_scales + place, n), lane >> 3, 0, 0);
        }
    };
    auto put = [&](unsigned at, const int (&off)[2], u32x4_t codes, unsigned byte) {
        const float by = scale_of(byte);
        *(lds_u32x4)(uintptr_t)(at + off[0]) = from_codes<T>(codes[0], codes[1], by);
        *(lds_u32x4)(uintptr_t)(at + off[1]) = from_codes<T>(codes[2], codes[3], by);
    };
    auto put_k = [&] {
        put(lds_k + k_to * kStepBytes, koff, codes_k, byte_k);
        next_k();
    };
    auto put_v = [&] {
        put(lds_v + v_to * kStepBytes, voff, codes_v, byte_v);
        next_v();
    };
    // Entering step s, K of s + 2 and V of s are in LDS.  16 bits: the step fetches K of s + 4 and V of s + 2, whose places were
    // last read in step s - 1 or before.  8 bits: it puts those there, fetched by the step before, and fetches K of s + 5 and
    // V of s + 3.
    constexpr int kAhead = k8 ? 1 : 0;
    size_t place[3];                                           // of steps s + 2 + kAhead .. s + 4 + kAhead
    int entry;                                                 // of the last of these
    {
        // (one round trip for all of them)
        int entries[5 + kAhead];
        size_t first[4 + kAhead];
#pragma unroll
        for (int i = 0; i < 5 + kAhead; ++i) entries[i] = page_entry(i);
        asm volatile("" ::"s"(entries[0]), "s"(entries[1]), "s"(entries[2]), "s"(entries[3]), "s"(entries[4]), "s"(entries[4 + kAhead]));
#pragma unroll
        for (int i = 0; i < 4 + kAhead; ++i) first[i] = row_place(entries[i], i);
        if constexpr (!k8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                fetch_k(first[i], rows_of(i));
                if (i >= 2) fetch_v(first[i - 2], rows_of(i - 2));
            }
        } else {
            // (all of them under way before the first is put in its place)
            u32x4_t k[4], v[2];
            unsigned kb[4], vb[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                fetch_k(first[i], rows_of(i));
                k[i] = codes_k;
                kb[i] = byte_k;
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                fetch_v(first[i], rows_of(i));
                v[i] = codes_v;
                vb[i] = byte_v;
            }
            fetch_k(first[4], rows_of(4));
            fetch_v(first[2], rows_of(2));
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 4; ++i) put(lds_k + i * kStepBytes, koff, k[i], kb[i]);
#pragma unroll
            for (int i = 0; i < 2; ++i) put(lds_v + i * kStepBytes, voff, v[i], vb[i]);
            v_to = 2;                                          // (and k_to 0 again)
        }
        place[0] = first[2 + kAhead];
        place[1] = first[3 + kAhead];
        entry = entries[4 + kAhead];
    }
    // (behind the first fetches, and waited for with them)
    u32x4_t q[8];
    {
        const uint16_t *from = p.q + (size_t)(at.first + token) * p.q_stride + (size_t)head * kHeadDim + 8 * h;
#pragma unroll
        for (int kb = 0; kb < 8; ++kb) q[kb] = *reinterpret_cast<const u32x4_t *>(from + 16 * kb);
    }

    f32x16_t acc[4];
    float sum = 0.f;                                           // of this lane's rounded weights
    // The reference of the weights, in units of log2, is T::kLift below the logit it was taken from; it follows the maximum only
    // where that has grown by kKvSlack.  threshold: what a logit relative to it has to pass; -inf until there is one.
    constexpr float kMost = kKvSlack + T::kLift;
    float ref = 0.f, threshold = -INFINITY;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[dt][r] = 0.f;
    const float c1 = p.scale * kLog2e;
    const int k_row = (c & 19) | (c & 4) << 1 | (c & 8) >> 1;  // the key whose row of the operand is c
    const unsigned k_at = k_row * kRowBytes + ((h ^ k_place(k_row)) << 4);
    const int v_row = 8 * h + ((lane >> 2) & 3);
    const unsigned v_at = v_row * kRowBytes + ((((lane >> 4) & 1) ^ v_unit(v_row)) << 5) + ((lane & 3) << 3);
    auto read_k = [&](unsigned kk, int kb) { return *(lds_u32x4)(uintptr_t)(kk ^ (kb << 5)); };
    auto read_v = [&](unsigned vv, int m, int dt) {
        const unsigned from = (vv ^ (dt << 6)) + 16 * m * kRowBytes;
        const s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)from);
        const s16x4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(from + 4 * kRowBytes));
        return __builtin_bit_cast(u32x4_t, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    f32x16_t zero;
#pragma unroll
    for (int r = 0; r < 16; ++r) zero[r] = 0.f;

    // Logits z[8 m + i] of keys 16 m + 8 h + i of a step, relative to the reference, and their maximum.
    float z[16], top = 0.f;
    unsigned k_next = 1, v_now = 0;
    u32x4_t first[4];                                          // the first operands of the next step's keys
    f32x16_t scn;
    // own: of a step s, key 16 m + 8 h + i is visible to the lane's row where 16 m + i <= own
    auto own_of = [&](int s) { return position - begin - kStep * s - 8 * h; };

    auto next_places = [&] {
        place[0] = place[1];
        place[1] = place[2];
    };

    // Step s from its logits, and the scores and logits of step s + 1, which do not depend on it.  Matrix instructions and what
    // runs under them are woven by hand, 16 slots of one matrix instruction: eight of scores, eight of V^T P^T.
    auto step = [&](auto with_masks, int s) {
        constexpr bool kMasks = decltype(with_masks)::value;
        unsigned kk = lds_k + k_next * kStepBytes + k_at, vv = lds_v + v_now * kStepBytes + v_at;
        k_next = k_next == kRingK - 1 ? 0 : k_next + 1;
        v_now = v_now == kRingV - 1 ? 0 : v_now + 1;
        unsigned k2 = lds_k + k_next * kStepBytes + k_at;
        asm("" : "+v"(kk), "+v"(vv), "+v"(k2));                // (or addresses of every place are kept in registers of their own)
        // A row whose logits have all been -inf has no reference yet: any number becomes it.
        if (__any(top > threshold)) {
            const bool none = threshold == -INFINITY;
            float d = none ? top - T::kLift : fmaxf(top - T::kLift, 0.f);
            d = d == -INFINITY ? 0.f : d;
            const float f = none ? 1.f : __builtin_amdgcn_exp2f(-d);
            if (top > -INFINITY) threshold = kMost;
            ref += d;
            sum *= f;
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] -= d;
            if (s > 0)
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) acc[dt] *= f;
        }
        u32x4_t a[8], av[2][4], w[2];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = first[i];
        auto weight = [&](auto ii) {                           // the i-th, and of every second the pair
            constexpr int i = decltype(ii)::value;
            z[i] = __builtin_amdgcn_exp2f(z[i]);
            if constexpr (i & 1) {
                w[i >> 3][(i >> 1) & 3] = T::pack(z[i - 1], z[i]);
                sum = add_pair<T>(w[i >> 3][(i >> 1) & 3], sum);
            }
        };
        __builtin_amdgcn_sched_barrier(0);
        slots(std::make_integer_sequence<int, 8>{}, [&](auto mi) {
            constexpr int mm = decltype(mi)::value;
            scn = mfma32<T>(a[mm], q[mm], mm == 0 ? zero : scn);
            if constexpr (mm < 4) a[mm + 4] = read_k(kk, mm + 4);
            if constexpr (!k8 && mm == 0) fetch_k(place[2], rows_of(s + 4));
            if constexpr (!k8 && mm == 2) fetch_v(place[0], rows_of(s + 2));
            av[mm >> 2][mm & 3] = read_v(vv, mm >> 2, mm & 3);
            weight(std::integral_constant<int, mm>{});
            if constexpr (mm >= 6) weight(std::integral_constant<int, mm + 2>{});
            __builtin_amdgcn_sched_barrier(0);
        });
        // In a step with masks the weights of keys behind a row are 0, and 0 times an infinite value or a NaN is NaN: such values
        // leave the product, and the rows that see them get them as a summand.
        if constexpr (kMasks) {
            if (s >= full && (any_not_finite<T>(av[0]) || any_not_finite<T>(av[1]))) {
                const int own = own_of(s);
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    u32x4_t seen;
#pragma unroll
                    for (int i = 0; i < 8; i += 2) seen[i >> 1] = T::pack(16 * m + i <= own ? 1.f : 0.f, 16 * m + i + 1 <= own ? 1.f : 0.f);
#pragma unroll
                    for (int dt = 0; dt < 4; ++dt) {
                        __builtin_amdgcn_sched_barrier(0);     // (one after the other: rare, and registers are scarce)
                        const f32x16_t counts = mfma32<T>(not_finite<T>(av[m][dt]), seen, zero);
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[dt][r] += summand(counts[r]);
                        av[m][dt] = finite<T>(av[m][dt]);
                    }
                }
            }
        }
        slots(std::make_integer_sequence<int, 4>{}, [&](auto mi) {
            constexpr int mm = decltype(mi)::value;
            acc[mm] = mfma32<T>(av[0][mm], w[0], acc[mm]);
            first[mm] = read_k(k2, mm);
            if constexpr (mm == 0) entry = page_entry(s + 5 + kAhead);
            if constexpr (mm < 3) {
                weight(std::integral_constant<int, 10 + 2 * mm>{});
                weight(std::integral_constant<int, 11 + 2 * mm>{});
            }
            if constexpr (k8 && mm == 2) put_k();
            if constexpr (k8 && mm == 3) put_v();
            __builtin_amdgcn_sched_barrier(0);
        });
        const int own = kMasks ? own_of(s + 1) : 0;
        slots(std::make_integer_sequence<int, 4>{}, [&](auto mi) {
            constexpr int mm = decltype(mi)::value;
            acc[mm] = mfma32<T>(av[1][mm], w[1], acc[mm]);
            if constexpr (k8 && mm == 0) fetch_k(place[2], rows_of(s + 5));
            if constexpr (k8 && mm == 1) fetch_v(place[0], rows_of(s + 3));
#pragma unroll
            for (int i = 4 * mm; i < 4 * mm + 4; ++i) {
                z[i] = __builtin_fmaf(scn[i], c1, -ref);
                if constexpr (kMasks) z[i] = i + 8 * (i >> 3) <= own ? z[i] : -INFINITY;
            }
            if constexpr (mm == 0) top = fmaxf(fmaxf(z[0], z[1]), z[2]);
            if constexpr (mm == 1) top = fmaxf(fmaxf(fmaxf(fmaxf(top, z[3]), z[4]), z[5]), z[6]);
            if constexpr (mm == 2) top = fmaxf(fmaxf(fmaxf(fmaxf(top, z[7]), z[8]), z[9]), z[10]);
            if constexpr (mm == 3) {
                top = fmaxf(fmaxf(fmaxf(fmaxf(top, z[11]), z[12]), z[13]), z[14]);
                top = halves_max(fmaxf(top, z[15]));
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        next_places();
    };

    if constexpr (!k8) __builtin_amdgcn_s_waitcnt(0x0f70);     // everything: the queries are the last; from here on fetches are counted
    tile_barrier();
    if (mine > 0) {
        unsigned kk = lds_k + k_at, k1 = kk + kStepBytes;
        asm("" : "+v"(kk), "+v"(k1));
        u32x4_t a[8];
#pragma unroll
        for (int kb = 0; kb < 8; ++kb) a[kb] = read_k(kk, kb);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kb = 0; kb < 8; ++kb) scn = mfma32<T>(a[kb], q[kb], kb == 0 ? zero : scn);
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) first[kb] = read_k(k1, kb);
        const int own = own_of(0);
        top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            z[i] = scn[i] * c1;
            z[i] = i + 8 * (i >> 3) <= own ? z[i] : -INFINITY;
            top = fmaxf(top, z[i]);
        }
        top = halves_max(top);
    }
    auto enter = [&](int s) {
        if constexpr (!k8) wait_fetches<4>();                  // K of s + 2 and V of s; what step s - 1 fetched is under way
        tile_barrier();
        place[2] = row_place(entry, s + 4 + kAhead);
    };
    int s = 0;
#pragma unroll 1
    for (; s < full - 1; ++s) {
        enter(s);
        step(std::false_type{}, s);
    }
#pragma unroll 1
    for (; s < mine; ++s) {
        enter(s);
        step(std::true_type{}, s);
    }
    for (; s < steps; ++s) {                                   // the steps that only other wavefronts have
        enter(s);
        if constexpr (k8) {
            put_k();
            put_v();
        }
        fetch_k(place[2], rows_of(s + 4 + kAhead));
        fetch_v(place[0], rows_of(s + 2 + kAhead));
        next_places();
        entry = page_entry(s + 5 + kAhead);
    }
    wait_fetches<0>();                                         // nothing may land in LDS after the workgroup has ended
    sum = halves_sum(sum, sum);
    if (!live) return;
    const int chunks = (position + at.piece) / at.piece;       // that hold a key of the row
    if (chunks <= 1) {
        if (chunk > 0) return;
        const bool some = position >= 0;
        const float inv = 1.f / sum;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                u32x2_t x = {T::pack(acc[dt][4 * j] * inv, acc[dt][4 * j + 1] * inv), T::pack(acc[dt][4 * j + 2] * inv, acc[dt][4 * j + 3] * inv)};
                if (!some) x = u32x2_t{0u, 0u};
                *reinterpret_cast<u32x2_t *>(out + 32 * dt + 8 * j) = x;
            }
    } else if (chunk < chunks && at.before + at.units <= p.units) {        // (sequences that overlap may have more than there is room for)
        const size_t slot = ((size_t)(at.before + index) * p.pool.Hkv + hkv) * kTileRows + 32 * wave + c;
        float *num = p.num + slot * kHeadDim + 4 * h;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<f32x4_t *>(num + 32 * dt + 8 * j) = f32x4_t{acc[dt][4 * j], acc[dt][4 * j + 1], acc[dt][4 * j + 2], acc[dt][4 * j + 3]};
        if (h == 0) p.ml[slot] = float2{threshold == -INFINITY ? -INFINITY : ref, sum};
    }
}

// Rows that several workgroups share: out = sum_c 2^{m_c - M} num_c / sum_c 2^{m_c - M} l_c.  A workgroup takes 16 heads of a token, a
// wavefront four of them, so that the loads of all are under way together.  (By tiles of a unit instead 8 x 64 tokens over 2000 .. 4000,
// 32/8 heads, took 60 us for 52.5.)
constexpr int kJoinHeads = 16;
template <class T> __global__ __launch_bounds__(256) void kv_prefill_join_kernel(KvPromptProblem p)
{
    constexpr int kRows = 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), token = blockIdx.x;
    const int head = kJoinHeads * blockIdx.y + kRows * wave;
    if (head >= p.Hq) return;
    const Sequence at = find_sequence(p, lane, [&](const Sequence &x) { return x.first <= token && token < x.first + x.tokens; });
    // (of no sequence; not cut; or of sequences that overlap, see above)
    if (at.b < 0 || at.units == at.tiles || at.before < 0 || at.before + at.units > p.units) return;
    const int chunks = (at.len - at.tokens + token - at.first + at.piece) / at.piece;
    if (chunks <= 1) return;                                   // done by the launch before
    const size_t next = (size_t)at.tiles * p.pool.Hkv * kTileRows;             // slots from a piece to the next
    const float2 *ml[kRows];
    const float *num[kRows];
    float top[kRows], a0[kRows], a1[kRows], sum[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int of = min(head + r, p.Hq - 1), hkv = of / p.G, row = (token - at.first) * p.G + of % p.G;
        const int unit = at.before + at.tiles - 1 - row / kTileRows;           // its tile's in the first piece
        const size_t slot = ((size_t)unit * p.pool.Hkv + hkv) * kTileRows + row % kTileRows;
        ml[r] = p.ml + slot;
        num[r] = p.num + slot * kHeadDim + 2 * lane;
        top[r] = -INFINITY;
        a0[r] = a1[r] = sum[r] = 0.f;
    }
    // 64 pieces at a time, their factors in the lanes; two partial vectors of each row under way, the first before the factors
    for (int w0 = 0; w0 < chunks; w0 += 64) {
        const int count = min(chunks - w0, 64);
        float2 s[kRows], x[2][kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) s[r] = ml[r][(w0 + min(lane, count - 1)) * next];
        auto load = [&](int i) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int r = 0; r < kRows; ++r)
                    x[k][r] = *reinterpret_cast<const float2 *>(num[r] + (w0 + min(i + k, count - 1)) * next * kHeadDim);
        };
        load(0);
        float f[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const float m = lane < count ? s[r].x : -INFINITY, t = columns_max(row16_max(m));
            if (t > top[r]) {                                  // (uniform) what the pieces before left, to the new reference
                const float by = top[r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top[r] - t);
                a0[r] *= by;
                a1[r] *= by;
                sum[r] *= by;
                top[r] = t;
            }
            f[r] = m == top[r] ? 1.f : __builtin_amdgcn_exp2f(m - top[r]);
            float d = row16_sum(lane < count ? s[r].y * f[r] : 0.f);
            d = rows_sum(d, d);
            sum[r] += halves_sum(d, d);
        }
        for (int i = 0; i < count; i += 2) {
            if (i > 0) load(i);
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    if (i + k >= count) continue;
                    const float by = as_f32((unsigned)__builtin_amdgcn_readlane(__builtin_bit_cast(int, f[r]), i + k));
                    a0[r] = __builtin_fmaf(x[k][r].x, by, a0[r]);
                    a1[r] = __builtin_fmaf(x[k][r].y, by, a1[r]);
                }
        }
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const float inv = 1.f / sum[r];
        if (head + r < p.Hq)
            reinterpret_cast<unsigned *>(p.out + ((size_t)token * p.Hq + head + r) * kHeadDim)[lane] = T::pack(a0[r] * inv, a1[r] * inv);
    }
}

}  // namespace

hipError_t launch_kv_prefill(const KvPromptProblem &p, hipStream_t s)
{
    const dim3 grid((unsigned)((long long)p.units * p.pool.Hkv));
    const bool f16 = p.pool.dtype == kF16;
    const hipError_t e = p.pool.store == kE4m3 ? launch(f16 ? kv_prefill_kernel<F16, true> : kv_prefill_kernel<BF16, true>, grid, dim3(256), s, p)
                                               : launch(f16 ? kv_prefill_kernel<F16, false> : kv_prefill_kernel<BF16, false>, grid, dim3(256), s, p);
    if (e != hipSuccess || p.C >= p.Smax) return e;
    return launch(f16 ? kv_prefill_join_kernel<F16> : kv_prefill_join_kernel<BF16>, dim3(p.n_tokens, (p.Hq + kJoinHeads - 1) / kJoinHeads), dim3(256), s, p);
}

}  // namespace fd
