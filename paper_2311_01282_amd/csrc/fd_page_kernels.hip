// Page tables and slot maps from request lengths, in one launch.
//
// Request b holds ceil(c / P) pages for its c cached tokens and needs ceil((c + n) / P) with its n new ones; the difference
// is taken from the end of the free list, in the order of the requests, so that request b's share starts where the needs of
// those before it add up to: a prefix sum.  A token's place follows from another prefix sum (whose token it is) and the
// table.
//
// Every workgroup forms both prefix sums itself, over all requests, and then serves its own 1024 tokens: a token looks its
// request up among the starts in LDS and takes its page from the table if the request held it before, and straight from the
// free list if it is fresh (another workgroup may be the one to write that entry).  Each fresh page has a first token,
// which writes the table's entry.  What bounds it is latency (8 requests 4.0 us, 300 prompts of 600000 tokens 8.2): a scan
// by one workgroup followed by a launch that fills would pay a second launch.
#include "fd_cache.h"

namespace fd {

namespace {

constexpr int kThreads = 512, kItems = 4, kWindow = kThreads * kItems;      // requests scanned at a time
constexpr int kTokens = 2;                                                  // tokens of a thread

struct PageLds {
    int start[kWindow];         // first token of a request, at most max_tokens
    int offset[kWindow];        // pages taken before it; -1: not served
    int cached[kWindow];
    unsigned tokens[kThreads / 64], pages[kThreads / 64];
    int taken[kThreads / 64];
};

// Sums of tokens and of pages end at kMany, which is more than there may be of either (max_tokens <= 2^30, fewer pages):
// sums that end somewhere add in any order as sums do.
constexpr unsigned kMany = (1u << 30) + 1;
__device__ __forceinline__ unsigned add(unsigned a, unsigned b) { return min(a + b, kMany); }
template <int kControl, int kRows> __device__ __forceinline__ unsigned add_dpp(unsigned x)
{
    return add(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, kControl, kRows, 0xf, false));
}
// sum of x over the lanes up to this one
__device__ __forceinline__ unsigned prefix(unsigned x)
{
    x = add_dpp<0x111, 0xf>(x);                                             // from 1, 2, 4 and 8 lanes before, within a row of 16
    x = add_dpp<0x112, 0xf>(x);
    x = add_dpp<0x114, 0xf>(x);
    x = add_dpp<0x118, 0xf>(x);
    x = add_dpp<0x142, 0xa>(x);                                             // the sum of row 0 to row 1 and of 2 to 3
    return add_dpp<0x143, 0xc>(x);                                          // of rows 0 and 1 to 2 and 3
}

__global__ __launch_bounds__(kThreads) void page_tables_kernel(PageProblem p)
{
    __shared__ PageLds lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int P = 1 << p.page_shift;
    const int room = p.width << p.page_shift;
    auto pages = [&](unsigned len) { return (int)((len + P - 1) >> p.page_shift); };
    const int n_free = min(max(*p.n_free, 0), p.n_pages);
    const int t0 = blockIdx.x * (kThreads * kTokens) + tid;                 // this thread's tokens: t0 + i kThreads
    unsigned tokens_before = 0, pages_before = 0;                           // of the windows before this one
    int taken = 0;
    int slot[kTokens];
#pragma unroll
    for (int i = 0; i < kTokens; ++i) slot[i] = -1;

    for (int w0 = 0; w0 < p.batch; w0 += kWindow) {
        const int count = min(p.batch - w0, kWindow);
        int c[kItems], n[kItems];
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int b = w0 + tid * kItems + i;
            c[i] = n[i] = 0;
            if (b < p.batch) {
                c[i] = min(max(p.cached[b], 0), room);
                n[i] = max(p.fresh[b], 0);
            }
        }
        unsigned tok = 0;
#pragma unroll
        for (int i = 0; i < kItems; ++i) tok = add(tok, n[i]);
        // (without this lane's)
        const unsigned run = prefix(tok), before = (unsigned)__builtin_amdgcn_update_dpp(0, (int)run, 0x138, 0xf, 0xf, false);
        if (lane == 63) lds.tokens[wave] = run;
        __syncthreads();
        unsigned start = tokens_before, all = tokens_before;
        for (int w = 0; w < kThreads / 64; ++w) {
            if (w < wave) start = add(start, lds.tokens[w]);
            all = add(all, lds.tokens[w]);
        }
        start = add(start, before);
        // what a request needs, where it has room for its tokens in the table and in the slot map
        int need[kItems];
        unsigned pg = 0, at = start;
        bool fits[kItems];
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            at = add(at, n[i]);
            const unsigned len = (unsigned)c[i] + (unsigned)n[i];
            fits[i] = len <= (unsigned)room && at <= (unsigned)p.max_tokens;
            need[i] = fits[i] ? pages(len) - pages(c[i]) : 0;
            pg = add(pg, need[i]);
        }
        const unsigned prun = prefix(pg), pbefore = (unsigned)__builtin_amdgcn_update_dpp(0, (int)prun, 0x138, 0xf, 0xf, false);
        if (lane == 63) lds.pages[wave] = prun;
        __syncthreads();
        unsigned off = pages_before, pages_all = pages_before;
        for (int w = 0; w < kThreads / 64; ++w) {
            if (w < wave) off = add(off, lds.pages[w]);
            pages_all = add(pages_all, lds.pages[w]);
        }
        off = add(off, pbefore);
        at = start;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int r = tid * kItems + i, b = w0 + r;
            const unsigned upto = add(off, need[i]);
            const bool listed = upto <= (unsigned)n_free, served = fits[i] && (need[i] == 0 || listed);
            // (grows along the requests of a thread, and from window to window)
            if (listed) taken = (int)upto;
            if (b < p.batch) {
                const int s = (int)min(at, (unsigned)p.max_tokens);
                lds.start[r] = s;
                lds.cached[r] = c[i];
                // (beyond the list only where nothing is needed)
                lds.offset[r] = served ? (int)min(off, (unsigned)n_free) : -1;
                if ((b / kWindow + r / 64) % gridDim.x == blockIdx.x) {     // the workgroups share these out by 64 requests
                    p.starts[b] = s;
                    p.seq_lens[b] = served ? c[i] + n[i] : c[i];
                }
            }
            at = add(at, n[i]);
            off = upto;
        }
        __syncthreads();
        // tokens of this window's requests
        const int end = (int)min(all, (unsigned)p.max_tokens), first = (int)min(tokens_before, (unsigned)p.max_tokens);
        // where the token's page stands; null: no slot from this window
        const int32_t *from[kTokens];
        int32_t *to[kTokens];                                               // the table's entry, of a fresh page's first token
        int in_page[kTokens], page[kTokens];
#pragma unroll
        for (int i = 0; i < kTokens; ++i) {
            const int t = t0 + i * kThreads;
            from[i] = nullptr;
            to[i] = nullptr;
            if (t < first || t >= end) continue;
            int lo = 0, hi = count;                                         // the last request that starts at or before t
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (lds.start[mid] <= t) lo = mid; else hi = mid;
            }
            if (lds.offset[lo] < 0) continue;
            const int b = w0 + lo;
            const int cached = lds.cached[lo];
            const int pos = cached + t - lds.start[lo];
            const int held = pages(cached), j = pos >> p.page_shift;
            int32_t *entry = p.table + (size_t)b * p.width + j;
            in_page[i] = pos & (P - 1);
            from[i] = j < held ? entry : p.free_pages + (n_free - 1 - (lds.offset[lo] + j - held));
            if (j >= held && in_page[i] == 0) to[i] = entry;
        }
        // (all before the first store, which they might otherwise have to wait for)
#pragma unroll
        for (int i = 0; i < kTokens; ++i)
            if (from[i]) page[i] = *from[i];
#pragma unroll
        for (int i = 0; i < kTokens; ++i) {
            if (!from[i]) continue;
            if (to[i]) *to[i] = page[i];
            if ((unsigned)page[i] < (unsigned)p.n_pages) slot[i] = (page[i] << p.page_shift) + in_page[i];
        }
        tokens_before = all;
        pages_before = pages_all;
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kTokens; ++i) {
        const int t = t0 + i * kThreads;
        if (t < p.max_tokens) p.slots[t] = slot[i];
    }
    if (blockIdx.x == 0) {
        // pages taken: the largest running need that the list could serve
#pragma unroll
        for (int d = 1; d < 64; d *= 2) taken = max(taken, __shfl_xor(taken, d));
        if (lane == 0) lds.taken[wave] = taken;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kThreads / 64; ++w) taken = max(taken, lds.taken[w]);
            *p.n_left = n_free - taken;
            p.starts[p.batch] = (int)min(tokens_before, (unsigned)p.max_tokens);
        }
    }
}

}  // namespace

hipError_t launch_page_tables(const PageProblem &p, hipStream_t s)
{
    const int per = kThreads * kTokens;
    const int grid = p.max_tokens > 0 ? (p.max_tokens - 1) / per + 1 : 1;
    return launch(page_tables_kernel, dim3(grid), dim3(kThreads), s, p);
}

}  // namespace fd
