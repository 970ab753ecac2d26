// The plan of a step: exclusive prefix sums over the requests of their new
// tokens and of the pages these need, then per page the table entry and per
// token its request, position, slot and ancestors.
//
// One launch: every workgroup repeats the scan over the R <= 4096 requests
// (8 bytes each, from L2) into LDS and then takes its share of the pages and
// tokens, finding their requests by binary search.  A token's page comes from
// the table where it was there before and from the free list where this call
// hands it out, so no workgroup reads what another one writes.
//
// Ancestors: a workgroup's tokens and the 63 before them hold every ancestor
// of a tree of at most 64, so their parents are staged in LDS and each thread
// walks up from its token.
#include "step.h"

namespace sbvr {

constexpr int PLAN_THREADS = 256;

__device__ __forceinline__ long long page_count(long long tokens, int shift)
{
    return (tokens + (1ll << shift) - 1) >> shift;
}

// pages of request r's cached tokens (within the table) and pages it takes now
__device__ __forceinline__ void request_pages(long long ctx, long long n, const PlanArgs &a, long long &have,
                                              long long &need)
{
    have = min(page_count(ctx, a.page_shift), (long long)a.max_pages);
    need = max(min(page_count(ctx + n, a.page_shift), (long long)a.max_pages) - have, 0ll);
}

__global__ void __launch_bounds__(PLAN_THREADS) plan_kernel(PlanArgs a)
{
    __shared__ int start[SBVR_REQUESTS_MAX + 1];       // tokens before request r, at most T
    __shared__ int first_page[SBVR_REQUESTS_MAX + 1];  // pages taken before request r
    __shared__ long long scratch[2 * PLAN_THREADS / 64];
    __shared__ int parent[PLAN_THREADS + SBVR_TREE_MAX];

    const int per = (a.R + PLAN_THREADS - 1) / PLAN_THREADS;
    const int r0 = min((int)threadIdx.x * per, a.R), r1 = min(r0 + per, a.R);
    long long tokens = 0, pages = 0, total_tokens, total_pages;
    for (int r = r0; r < r1; ++r) {
        const long long ctx = max(a.context_lens[r], 0), n = max(a.new_lens[r], 0);
        long long have, need;
        request_pages(ctx, n, a, have, need);
        tokens += n;
        pages += need;
    }
    scan_pair<PLAN_THREADS>(tokens, pages, total_tokens, total_pages, scratch);
    for (int r = r0; r < r1; ++r) {
        const long long ctx = max(a.context_lens[r], 0), n = max(a.new_lens[r], 0);
        long long have, need;
        request_pages(ctx, n, a, have, need);
        start[r] = (int)min(tokens, (long long)a.T);
        first_page[r] = (int)min(pages, 0x7fffffffll);
        if (blockIdx.x == 0)
            a.query_start[r] = start[r];
        tokens += n;
        pages += need;
    }
    const int n_tokens = (int)min(total_tokens, (long long)a.T);
    const int n_pages = (int)min(total_pages, 0x7fffffffll);
    if (threadIdx.x == 0) {
        start[a.R] = n_tokens;
        first_page[a.R] = n_pages;
        if (blockIdx.x == 0) {
            a.query_start[a.R] = n_tokens;
            a.used[0] = n_pages;
            a.used[1] = (int)min(total_tokens, 0x7fffffffll);
        }
    }
    __syncthreads();

    const long long step = (long long)gridDim.x * PLAN_THREADS;
    for (long long p = (long long)blockIdx.x * PLAN_THREADS + threadIdx.x; p < n_pages; p += step) {
        const int r = owner_of(first_page, a.R, (int)p);
        long long have, need;
        request_pages(max(a.context_lens[r], 0), 0, a, have, need);
        a.page_table[r * a.table_stride + have + (p - first_page[r])] = p < a.n_free ? a.free_pages[p] : -1;
    }

    for (long long t0 = (long long)blockIdx.x * PLAN_THREADS; t0 < a.T; t0 += step) {
        if (a.parents) {
            __syncthreads();
            for (int i = threadIdx.x; i < PLAN_THREADS + SBVR_TREE_MAX - 1; i += PLAN_THREADS) {
                const long long t = t0 - (SBVR_TREE_MAX - 1) + i;
                parent[i] = t >= 0 && t < n_tokens ? a.parents[t] : -1;
            }
            __syncthreads();
        }
        const long long t = t0 + threadIdx.x;
        if (t >= a.T)
            continue;
        if (t >= n_tokens) {
            a.token_request[t] = -1;
            a.positions[t] = 0;
            a.slots[t] = -1;
            a.tree_mask[t] = 0;
            continue;
        }
        const int r = owner_of(start, a.R, (int)t);
        const int j = (int)t - start[r];
        const long long ctx = max(a.context_lens[r], 0);
        long long have, need;
        request_pages(ctx, 0, a, have, need);
        const long long at = ctx + j, e = at >> a.page_shift;
        int page = -1;
        if (e < have) {
            page = a.page_table[r * a.table_stride + e];
        } else if (e < a.max_pages) {
            const long long n = first_page[r] + (e - have);
            page = n < a.n_free ? a.free_pages[n] : -1;
        }
        int depth = j;
        uint64_t mask = 0;
        if (a.new_lens[r] <= SBVR_TREE_MAX) {
            if (a.parents) {
                mask = 1ull << j;
                depth = 0;
                for (int up = j;;) {
                    const int p = parent[threadIdx.x + SBVR_TREE_MAX - 1 - (j - up)];
                    if (p < 0 || p >= up)
                        break;
                    up = p;
                    mask |= 1ull << up;
                    ++depth;
                }
            } else {
                mask = ~0ull >> (63 - j);
            }
        }
        a.token_request[t] = r;
        a.positions[t] = (int)(ctx + depth);
        a.slots[t] = page < 0 ? -1 : ((long long)page << a.page_shift) + (at & ((1 << a.page_shift) - 1));
        a.tree_mask[t] = mask;
    }
}

int launch_plan(const PlanArgs &a, hipStream_t stream)
{
    // one workgroup for 256 tokens or pages, whichever are more; a few hundred
    // at most, since each repeats the scan
    const long long pages = (long long)a.R + (a.T >> a.page_shift);
    const long long items = a.T > pages ? a.T : pages;
    long long grid = (items + PLAN_THREADS - 1) / PLAN_THREADS;
    if (grid > 512)
        grid = 512;
    if (grid < 1)
        grid = 1;
    PlanArgs args = a;
    void *argv[] = {&args};
    return launch_kernel((const void *)plan_kernel, dim3((unsigned)grid), dim3(PLAN_THREADS), 0, stream, argv);
}

}  // namespace sbvr
