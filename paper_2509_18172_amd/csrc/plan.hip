// The plan of a step: exclusive prefix sums over the requests of their new
// tokens and of the pages these need, then per page the table entry and per
// token its request, position, slot and ancestors.
//
// One launch: every workgroup repeats the scan over the R <= 4096 requests
// (8 bytes each, from L2) into LDS and then takes its share of the pages and
// tokens.  Sums saturate at 2^32 - 1 (addition that saturates is still
// associative; what lies past T tokens or 2^31 pages is cut anyway), so the scan
// is 32-bit.  Past 256 requests the workgroups have 1024 threads: fewer of them
// repeat the scan, with four requests a thread.  A wavefront finds the requests
// of its first and last token by comparing 64 starts at a time, and each lane
// its own between the two.  A token's page comes from the table where it was
// there before and from the free list where this call hands it out, so no
// workgroup reads what another one writes.
//
// Ancestors: a workgroup's tokens and the 63 before them hold every ancestor
// of a tree of at most 64, so their parents are staged in LDS and each thread
// walks up from its token.
//
// Measured in a graph: one request of one token 3.9 us, of which an empty launch
// is 2.1 and the rest the chain of the scan; 4096 requests with trees of up to 64
// (197 thousand tokens, 5.7 MB in and out) 10.7 us, where a copy of as many bytes takes
// 1.1.  It is one workgroup's chain -- loads, scan, LDS, a search per page, then two
// per wavefront of tokens: 4096 requests of one token, five workgroups, take 9.4.
#include "step.h"

namespace sbvr {

struct RequestPages {
    int have, need;  // pages of the cached tokens (within the table), pages taken now
};

__device__ __forceinline__ long long page_count(long long tokens, int shift)
{
    return (tokens + (1ll << shift) - 1) >> shift;
}

__device__ __forceinline__ RequestPages request_pages(int ctx, int n, const PlanArgs &a)
{
    const int have = (int)min(page_count(ctx, a.page_shift), (long long)a.max_pages);
    return {have, max((int)min(page_count((long long)ctx + n, a.page_shift), (long long)a.max_pages) - have, 0)};
}

__device__ __forceinline__ uint32_t add_sat(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }

// Inclusive scan over a wavefront's lanes with saturating sums.
__device__ __forceinline__ uint32_t scan_sat(uint32_t v)
{
    v = add_sat(v, __builtin_amdgcn_update_dpp(0u, v, 0x111, 0xf, 0xf, false));  // row_shr 1, 2, 4, 8
    v = add_sat(v, __builtin_amdgcn_update_dpp(0u, v, 0x112, 0xf, 0xf, false));
    v = add_sat(v, __builtin_amdgcn_update_dpp(0u, v, 0x114, 0xf, 0xf, false));
    v = add_sat(v, __builtin_amdgcn_update_dpp(0u, v, 0x118, 0xf, 0xf, false));
    v = add_sat(v, __builtin_amdgcn_update_dpp(0u, v, 0x142, 0xa, 0xf, false));  // row_bcast 15, 31
    v = add_sat(v, __builtin_amdgcn_update_dpp(0u, v, 0x143, 0xc, 0xf, false));
    return v;
}

// The last i of the ascending LDS array start[0 .. n] with start[i] <= v, for a
// v < start[n] that is the same in every lane.
__device__ __forceinline__ int owner_of_uniform(const int *start, int n, int v)
{
    const int lane = threadIdx.x & 63;
    int lo = 0;
    if (n > 64) {
        const int step = (n + 63) / 64, at = lane * step;
        lo = (63 - __builtin_clzll(__ballot(at < n && start[min(at, n)] <= v))) * step;
        n = min(n - lo, step);
    }
    return lo + 63 - __builtin_clzll(__ballot(lane < n && start[lo + min(lane, n)] <= v));
}

// PER: requests per thread of the scan.
template <int THREADS, int PER>
__global__ void __launch_bounds__(THREADS) plan_kernel(PlanArgs a)
{
    constexpr int WAVES = THREADS / 64, MAX_R = THREADS * PER;
    __shared__ int start[MAX_R + 1];       // tokens before request r, at most T
    __shared__ int first_page[MAX_R + 1];  // pages taken before request r
    __shared__ uint32_t wave_tokens[WAVES], wave_pages[WAVES];
    __shared__ int parent[THREADS + SBVR_TREE_MAX];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

    uint32_t n[PER], need[PER], tokens = 0, pages = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int r = threadIdx.x * PER + i;
        const int ctx = r < a.R ? max(a.context_lens[r], 0) : 0;
        n[i] = r < a.R ? max(a.new_lens[r], 0) : 0;
        need[i] = r < a.R ? request_pages(ctx, n[i], a).need : 0;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        tokens = add_sat(tokens, n[i]);
        pages = add_sat(pages, need[i]);
    }
    const uint32_t scan_t = scan_sat(tokens), scan_p = scan_sat(pages);
    if (lane == 63) {
        wave_tokens[wave] = scan_t;
        wave_pages[wave] = scan_p;
    }
    __syncthreads();
    uint32_t t0 = __builtin_amdgcn_update_dpp(0u, scan_t, 0x138, 0xf, 0xf, false);  // wave_shr 1: exclusive
    uint32_t p0 = __builtin_amdgcn_update_dpp(0u, scan_p, 0x138, 0xf, 0xf, false);
    uint32_t all_tokens = 0, all_pages = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w == wave) {
            t0 = add_sat(t0, all_tokens);
            p0 = add_sat(p0, all_pages);
        }
        all_tokens = add_sat(all_tokens, wave_tokens[w]);
        all_pages = add_sat(all_pages, wave_pages[w]);
    }
    const int n_tokens = (int)min(all_tokens, (uint32_t)a.T), n_pages = (int)min(all_pages, 0x7fffffffu);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int r = threadIdx.x * PER + i;
        if (r <= a.R) {
            start[r] = (int)min(t0, (uint32_t)a.T);
            first_page[r] = (int)min(p0, 0x7fffffffu);
            if (blockIdx.x == 0)
                a.query_start[r] = start[r];
        }
        t0 = add_sat(t0, n[i]);
        p0 = add_sat(p0, need[i]);
    }
    if (threadIdx.x == 0) {
        start[a.R] = n_tokens;
        first_page[a.R] = n_pages;
        if (blockIdx.x == 0) {
            a.query_start[a.R] = n_tokens;
            a.used[0] = n_pages;
            a.used[1] = (int)min(all_tokens, 0x7fffffffu);
        }
    }
    __syncthreads();

    const long long step = (long long)gridDim.x * THREADS;
    for (long long p = (long long)blockIdx.x * THREADS + threadIdx.x; p < n_pages; p += step) {
        const int r = owner_of(first_page, a.R, (int)p);
        const int have = request_pages(max(a.context_lens[r], 0), 0, a).have;
        a.page_table[r * a.table_stride + have + (p - first_page[r])] = p < a.n_free ? a.free_pages[p] : -1;
    }

    for (long long b0 = (long long)blockIdx.x * THREADS; b0 < a.T; b0 += step) {
        if (a.parents) {
            __syncthreads();
            for (int i = threadIdx.x; i < THREADS + SBVR_TREE_MAX - 1; i += THREADS) {
                const long long t = b0 - (SBVR_TREE_MAX - 1) + i;
                parent[i] = t >= 0 && t < n_tokens ? a.parents[t] : -1;
            }
            __syncthreads();
        }
        const long long w0 = b0 + 64 * wave, t = w0 + lane;
        if (t < a.T && t >= n_tokens) {
            a.token_request[t] = -1;
            a.positions[t] = 0;
            a.slots[t] = -1;
            a.tree_mask[t] = 0;
        }
        if (w0 >= n_tokens)
            continue;
        const int r_first = owner_of_uniform(start, a.R, (int)w0);
        const int r_last = owner_of_uniform(start, a.R, (int)min(w0 + 63, (long long)n_tokens - 1));
        if (t >= n_tokens)
            continue;
        const int r = r_first + owner_of(start + r_first, r_last - r_first + 1, (int)t);
        const int j = (int)t - start[r], new_len = a.new_lens[r];
        const int ctx = max(a.context_lens[r], 0), have = request_pages(ctx, 0, a).have;
        const long long at = (long long)ctx + j, e = at >> a.page_shift;
        int page = -1;
        if (e < have) {
            page = a.page_table[r * a.table_stride + e];
        } else if (e < a.max_pages) {
            const long long k = first_page[r] + (e - have);
            page = k < a.n_free ? a.free_pages[k] : -1;
        }
        int depth = j;
        uint64_t mask = 0;
        if (new_len <= SBVR_TREE_MAX) {
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
        a.positions[t] = (int)(ctx + (long long)depth);
        a.slots[t] = page < 0 ? -1 : ((long long)page << a.page_shift) + (at & ((1 << a.page_shift) - 1));
        a.tree_mask[t] = mask;
    }
}

template <int THREADS, int PER>
int run_plan(const PlanArgs &a, hipStream_t stream)
{
    // one workgroup for THREADS tokens or pages, whichever are more; as many
    // as the chip holds at most, since each repeats the scan
    const long long pages = (long long)a.R + (a.T >> a.page_shift);
    const long long items = a.T > pages ? a.T : pages;
    long long grid = (items + THREADS - 1) / THREADS;
    if (grid > 512 * 256 / THREADS * 2)
        grid = 512 * 256 / THREADS * 2;
    if (grid < 1)
        grid = 1;
    PlanArgs args = a;
    void *argv[] = {&args};
    return launch_kernel((const void *)plan_kernel<THREADS, PER>, dim3((unsigned)grid), dim3(THREADS), 0, stream, argv);
}

int launch_plan(const PlanArgs &a, hipStream_t stream)
{
    static_assert(1024 * 4 == SBVR_REQUESTS_MAX, "four requests a thread");
    // 256 requests of eight tokens: 5.6 us with 256 threads, 7.1 with 1024; 512:
    // 9.2 us with 256 threads of 16 requests, 7.3 with 1024 of four; 4096 of 64:
    // 27 and 11.
    return a.R <= 256 ? run_plan<256, 1>(a, stream) : run_plan<1024, 4>(a, stream);
}

}  // namespace sbvr
