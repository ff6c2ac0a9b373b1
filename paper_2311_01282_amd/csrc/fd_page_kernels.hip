// Page tables and slot maps from request lengths, in one launch.
//
// Request b holds ceil(c / P) pages for its c cached tokens and needs ceil((c + n) / P) with its n new ones; the difference is
// taken from the end of the free list, in the order of the requests, so that request b's share starts where the needs of those
// before it add up to: a prefix sum.  A token's place follows from another prefix sum (whose token it is) and the table.
//
// Every workgroup forms both prefix sums itself, over all requests, and then serves its own 1024 tokens: a token looks its
// request up among the starts in LDS and takes its page from the table if the request held it before, and straight from the free list
// if it is fresh (another workgroup may be the one to write that entry).  Each fresh page has a first token, which writes the
// table's entry.  What bounds it is latency: a scan by one workgroup followed by a launch that fills would pay a second launch.
#include <type_traits>

#include "fd_cache.h"

namespace fd {

namespace {

constexpr int kThreads = 512, kItems = 4, kWindow = kThreads * kItems;      // requests scanned at a time
constexpr int kTokens = 2;                                                  // tokens of a thread

struct PageLds {
    int start[kWindow];         // first token of a request, at most max_tokens
    int offset[kWindow];        // pages taken before it; -1: not served
    int cached[kWindow];
    long long tokens[kThreads / 64], pages[kThreads / 64];
    long long taken[kThreads / 64];
};

__device__ __forceinline__ long long shift_up(long long x, int d, int lane)
{
    const long long y = __shfl_up(x, d);
    return lane >= d ? y : 0;
}

__global__ __launch_bounds__(kThreads) void page_tables_kernel(PageProblem p)
{
    __shared__ PageLds lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int P = 1 << p.page_shift;
    const long long room = (long long)p.width << p.page_shift;
    const int n_free = min(max(*p.n_free, 0), p.n_pages);
    const int t0 = blockIdx.x * (kThreads * kTokens) + tid;                 // this thread's tokens: t0 + i kThreads
    long long tokens_before = 0, pages_before = 0, taken = 0;               // of the windows before this one
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
                c[i] = (int)min((long long)max(p.cached[b], 0), room);
                n[i] = max(p.fresh[b], 0);
            }
        }
        long long tok = 0;
#pragma unroll
        for (int i = 0; i < kItems; ++i) tok += n[i];
        long long run = tok;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) run += shift_up(run, d, lane);
        if (lane == 63) lds.tokens[wave] = run;
        __syncthreads();
        long long start = tokens_before + run - tok, all = tokens_before;
        for (int w = 0; w < kThreads / 64; ++w) {
            if (w < wave) start += lds.tokens[w];
            all += lds.tokens[w];
        }
        // what a request needs, where it has room for its tokens in the table and in the slot map
        int need[kItems];
        long long pg = 0, at = start;
        bool fits[kItems];
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            at += n[i];
            fits[i] = c[i] + (long long)n[i] <= room && at <= p.max_tokens;
            need[i] = fits[i] ? (int)((c[i] + (long long)n[i] + P - 1) >> p.page_shift) - (int)(((long long)c[i] + P - 1) >> p.page_shift) : 0;
            pg += need[i];
        }
        long long prun = pg;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) prun += shift_up(prun, d, lane);
        if (lane == 63) lds.pages[wave] = prun;
        __syncthreads();
        long long off = pages_before + prun - pg, pages_all = pages_before;
        for (int w = 0; w < kThreads / 64; ++w) {
            if (w < wave) off += lds.pages[w];
            pages_all += lds.pages[w];
        }
        at = start;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int r = tid * kItems + i, b = w0 + r;
            const bool served = fits[i] && (need[i] == 0 || off + need[i] <= n_free);
            if (off + need[i] <= n_free) taken = off + need[i];             // (grows along the requests of a thread, and from window to window)
            if (b < p.batch) {
                const int s = (int)min(at, (long long)p.max_tokens);
                lds.start[r] = s;
                lds.cached[r] = c[i];
                lds.offset[r] = served ? (int)min(off, (long long)n_free) : -1;     // (beyond the list only where nothing is needed)
                if ((b / kWindow + r / 64) % gridDim.x == blockIdx.x) {     // the workgroups share these out by 64 requests
                    p.starts[b] = s;
                    p.seq_lens[b] = served ? c[i] + n[i] : c[i];
                }
            }
            at += n[i];
            off += need[i];
        }
        __syncthreads();
        // tokens of this window's requests
        const long long end = min(all, (long long)p.max_tokens);
#pragma unroll
        for (int i = 0; i < kTokens; ++i) {
            const int t = t0 + i * kThreads;
            if (t < tokens_before || t >= end) continue;
            int lo = 0, hi = count;                                         // the last request that starts at or before t
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (lds.start[mid] <= t) lo = mid; else hi = mid;
            }
            if (lds.offset[lo] < 0) continue;
            const int b = w0 + lo;
            const int cached = lds.cached[lo];
            const int pos = cached + t - lds.start[lo];
            const int held = (int)(((long long)cached + P - 1) >> p.page_shift), j = pos >> p.page_shift;
            int32_t *entry = p.table + (size_t)b * p.width + j;
            int page;
            if (j < held) page = *entry;
            else {
                page = p.free_pages[n_free - 1 - (lds.offset[lo] + j - held)];
                if ((pos & (P - 1)) == 0) *entry = page;
            }
            if ((unsigned)page < (unsigned)p.n_pages) slot[i] = (page << p.page_shift) + (pos & (P - 1));
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
        for (int d = 1; d < 64; d *= 2) taken = max(taken, (long long)__shfl_xor(taken, d));
        if (lane == 0) lds.taken[wave] = taken;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kThreads / 64; ++w) taken = max(taken, lds.taken[w]);
            *p.n_left = n_free - (int)taken;
            p.starts[p.batch] = (int)min(tokens_before, (long long)p.max_tokens);
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
