// Pages that sequences share: which are used and free, the fork of rows with a
// copy of the page that they cannot share, moving pages together, and the copies.
//
// Tables are a few megabytes at most, and their operators chains of latencies: what
// counts is how few launches and dependent loads they take.  Where every workgroup
// needs the same sums (pages before its own, rows before its own) each one repeats
// them, so that none waits for another.  The copies are memory-bound, in one launch
// for the keys and values of all layers.
#include "step.h"

namespace sbvr {

__device__ __forceinline__ int entries_in_use(int length, const PageTable &t)
{
    const long long n = ((long long)max(length, 0) + (1 << t.page_shift) - 1) >> t.page_shift;
    return (int)min(n, (long long)t.max_pages);
}

// Sum of v over the workgroup's threads before this one, and over all of them.
template <int THREADS>
__device__ __forceinline__ int sum_before(int v, int &all, int *scratch)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int up = v;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int other = __shfl_up(up, m);
        up += lane >= m ? other : 0;
    }
    __syncthreads();
    if (lane == 63)
        scratch[wave] = up;
    __syncthreads();
    int before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        before += w < wave ? scratch[w] : 0;
        all += scratch[w];
    }
    return before + up - v;
}

// ---------------------------------------------------------------------------
// use of pages
// ---------------------------------------------------------------------------

constexpr int PAGE_THREADS = 1024;

// Words of marks, a bit per page; the launches below read whole ones.
__host__ __device__ constexpr int mark_words(int n_pages) { return (n_pages + 31) / 32; }

__global__ void __launch_bounds__(256) clear_kernel(uint32_t *p, int n, uint32_t *q, int m)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n)
        p[i] = 0;
    if (i < m)
        q[i] = 0;
}

// A wavefront per 256 entries of a row: marks their pages, and counts them where
// refs is given.
__global__ void __launch_bounds__(256) mark_kernel(PageTable t, int n_pages, uint32_t *marks, int32_t *refs, int pieces)
{
    const long long items = (long long)t.R * pieces;
    for (long long item = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); item < items; item += (long long)gridDim.x * 4) {
        const int r = (int)(item / pieces), e0 = (int)(item % pieces) * 256 + (threadIdx.x & 63);
        const int used = entries_in_use(t.context_lens[r], t);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int e = e0 + 64 * u;
            const int page = e < used ? t.page_table[r * t.table_stride + e] : -1;
            if (page >= 0 && page < n_pages) {
                if (!refs || atomicAdd(&refs[page], 1) == 0)
                    atomicOr(&marks[page >> 5], 1u << (page & 31));
            }
        }
    }
}

// Pages marked before `page`, by the whole workgroup.
__device__ __forceinline__ int marked_before(const uint32_t *marks, int page, int *scratch)
{
    int n = 0, all;
    for (int w = threadIdx.x; w < page / 32; w += PAGE_THREADS)
        n += __popc(marks[w]);
    if (threadIdx.x == 0 && (page & 31))
        n += __popc(marks[page / 32] & ((1u << (page & 31)) - 1));
    sum_before<PAGE_THREADS>(n, all, scratch);
    return all;
}

// The free pages in order, a word of marks a thread.
__global__ void __launch_bounds__(PAGE_THREADS) free_kernel(UsageArgs a)
{
    __shared__ int scratch[PAGE_THREADS / 64];
    const int words = mark_words(a.n_pages), first = blockIdx.x * PAGE_THREADS;
    const int before = marked_before(a.marks, min(first * 32, a.n_pages), scratch);
    const int total = marked_before(a.marks, a.n_pages, scratch);
    const int w = first + (int)threadIdx.x, p0 = w * 32;
    const uint32_t mark = w < words ? a.marks[w] : ~0u;
    int here;
    int used = before + sum_before<PAGE_THREADS>(w < words ? __popc(mark) : 0, here, scratch);
    for (int i = 0; i < 32 && p0 + i < a.n_pages; ++i) {
        const int p = p0 + i;
        if ((mark >> i) & 1)
            ++used;
        else
            a.free_pages[p - used] = p;
        if (p >= a.n_pages - total)
            a.free_pages[p] = -1;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.counts[0] = a.n_pages - total;
        a.counts[1] = total;
    }
}

size_t usage_workspace_bytes(int n_pages) { return ((size_t)mark_words(n_pages) * 4 + 15) / 16 * 16; }

namespace {

// workgroups of a launch whose items may be more than a grid can be
unsigned capped(long long n) { return (unsigned)(n < (1 << 20) ? n : 1 << 20); }

int run_mark(const PageTable &t, int n_pages, uint32_t *marks, int32_t *refs, hipStream_t stream)
{
    int words = mark_words(n_pages), n = refs ? n_pages : 0;
    uint32_t *counts = (uint32_t *)refs;
    void *clear[] = {&marks, &words, &counts, &n};
    const int most = n > words ? n : words;
    int st = launch_kernel((const void *)clear_kernel, dim3((most + 255) / 256), dim3(256), 0, stream, clear);
    if (st != SBVR_OK || t.R == 0)
        return st;
    PageTable table = t;
    int pieces = (t.max_pages + 255) / 256;
    const long long items = (long long)t.R * pieces;
    void *mark[] = {&table, &n_pages, &marks, &refs, &pieces};
    return launch_kernel((const void *)mark_kernel, dim3(capped((items + 3) / 4)), dim3(256), 0, stream, mark);
}

int mark_groups(int n_pages) { return (mark_words(n_pages) + PAGE_THREADS - 1) / PAGE_THREADS; }

}  // namespace

int launch_usage(const UsageArgs &a, hipStream_t stream)
{
    const int st = run_mark(a.t, a.n_pages, a.marks, a.refs, stream);
    if (st != SBVR_OK)
        return st;
    UsageArgs args = a;
    void *argv[] = {&args};
    return launch_kernel((const void *)free_kernel, dim3(mark_groups(a.n_pages)), dim3(PAGE_THREADS), 0, stream, argv);
}

// ---------------------------------------------------------------------------
// fork
// ---------------------------------------------------------------------------

// Every workgroup finds which rows need a page, and how many do before each; then
// it writes its share of the rows.
template <int THREADS, int PER>
__global__ void __launch_bounds__(THREADS) fork_kernel(ForkArgs a)
{
    constexpr int MOST = THREADS * PER;
    __shared__ int first_child[MOST], parent_row[MOST], page_of[MOST], scratch[THREADS / 64];
    const PageTable &t = a.t;
    const int tid = threadIdx.x, page_size = 1 << t.page_shift;
    for (int i = tid; i < t.R; i += THREADS)
        first_child[i] = 0x7fffffff;
    __syncthreads();
    int parent[PER], length[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int i = tid * PER + k;
        const int p = i < a.rows_out ? a.parents[i] : -1;
        parent[k] = p >= 0 && p < a.group_in ? i / a.group_out * a.group_in + p : -1;
        if (parent[k] >= 0)
            atomicMin(&first_child[parent[k]], i);
        if (i < a.rows_out)
            parent_row[i] = parent[k];
    }
    __syncthreads();
    int need[PER], source[PER], own = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int i = tid * PER + k, p = parent[k];
        length[k] = p >= 0 ? max(t.context_lens[p], 0) : 0;
        const int full = length[k] >> t.page_shift;
        source[k] = p >= 0 && (length[k] & (page_size - 1)) && full < t.max_pages && first_child[max(p, 0)] != i
                        ? t.page_table[p * t.table_stride + full]
                        : -1;
        need[k] = source[k] >= 0;
        own += need[k];
    }
    int all;
    long long at = sum_before<THREADS>(own, all, scratch);
    at += a.taken ? max(uniform_load(a.taken), 0) : 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int i = tid * PER + k;
        int page = -1;
        if (need[k]) {
            page = at < a.n_free ? a.free_pages[at] : -1;
            ++at;
        }
        if (i < a.rows_out) {
            page_of[i] = need[k] ? max(page, -1) : -2;  // -2: the parent's own
            if (blockIdx.x == 0) {
                a.out_lens[i] = length[k];
                a.src[i] = page >= 0 ? source[k] : -1;
                a.dst[i] = max(page, -1);
                a.tokens[i] = page >= 0 ? length[k] & (page_size - 1) : 0;
            }
        }
    }
    if (blockIdx.x == 0 && tid == 0)
        a.used[0] = all;
    __syncthreads();
    const int pieces = (t.max_pages + THREADS - 1) / THREADS;
    const long long items = (long long)a.rows_out * pieces;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const int i = (int)(item / pieces), e = (int)(item % pieces) * THREADS + tid;
        const int p = parent_row[i];
        if (e >= t.max_pages)
            continue;
        int page = -1;
        if (p >= 0) {
            const int len = max(uniform_load(t.context_lens + p), 0);
            if (e < entries_in_use(len, t))
                page = page_of[i] != -2 && e == len >> t.page_shift ? page_of[i] : t.page_table[p * t.table_stride + e];
        }
        a.out_table[i * a.out_stride + e] = page;
    }
}

int launch_fork(const ForkArgs &a, hipStream_t stream)
{
    static_assert(1024 * 4 == SBVR_REQUESTS_MAX, "four rows a thread");
    ForkArgs args = a;
    void *argv[] = {&args};
    const int rows = a.rows_out > a.t.R ? a.rows_out : a.t.R, threads = rows <= 256 ? 256 : 1024;
    const long long items = (long long)a.rows_out * ((a.t.max_pages + threads - 1) / threads);
    const int most = 256 * 1024 / threads;
    const unsigned grid = items < 1 ? 1 : items < most ? (unsigned)items : most;
    return rows <= 256 ? launch_kernel((const void *)fork_kernel<256, 1>, dim3(grid), dim3(256), 0, stream, argv)
                       : launch_kernel((const void *)fork_kernel<1024, 4>, dim3(grid), dim3(1024), 0, stream, argv);
}

// ---------------------------------------------------------------------------
// compaction
// ---------------------------------------------------------------------------

// The k-th free page below the number of used ones is dst[k], the k-th used page from
// there on src[k]; number[p] = k for the latter.
__global__ void __launch_bounds__(PAGE_THREADS) moves_kernel(CompactArgs a)
{
    __shared__ int scratch[PAGE_THREADS / 64];
    const int words = mark_words(a.n_pages), first = blockIdx.x * PAGE_THREADS;
    const int total = marked_before(a.marks, a.n_pages, scratch);
    const int low = marked_before(a.marks, total, scratch);  // those that stay
    const int before = marked_before(a.marks, min(first * 32, a.n_pages), scratch);
    const int w = first + (int)threadIdx.x, p0 = w * 32;
    const uint32_t mark = w < words ? a.marks[w] : 0;
    int here;
    int used = before + sum_before<PAGE_THREADS>(__popc(mark), here, scratch);
    const int moved = total - low, lists = a.n_pages / 2;
    for (int i = 0; i < 32 && p0 + i < a.n_pages; ++i) {
        const int p = p0 + i;
        const bool in_use = (mark >> i) & 1;
        if (in_use && p >= total) {
            a.number[p] = used - low;
            a.src[used - low] = p;
        } else if (!in_use && p < total) {
            a.dst[p - used] = p;
        }
        used += in_use;
        if (p >= moved && p < lists)
            a.src[p] = a.dst[p] = -1;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.counts[0] = total;
        a.counts[1] = moved;
    }
}

__global__ void __launch_bounds__(256) renumber_kernel(CompactArgs a, int pieces)
{
    const PageTable &t = a.t;
    const long long items = (long long)t.R * pieces;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const int r = (int)(item / pieces), e = (int)(item % pieces) * 256 + threadIdx.x;
        if (e >= t.max_pages)
            continue;
        int page = e < entries_in_use(t.context_lens[r], t) ? t.page_table[r * t.table_stride + e] : -1;
        if (page < 0 || page >= a.n_pages)
            page = -1;
        else if (page >= a.counts[0])
            page = a.dst[a.number[page]];
        a.out_table[r * a.out_stride + e] = page;
    }
}

size_t compact_workspace_bytes(int n_pages) { return usage_workspace_bytes(n_pages) + (size_t)n_pages * sizeof(int32_t); }

int launch_compact(const CompactArgs &a, hipStream_t stream)
{
    int st = run_mark(a.t, a.n_pages, a.marks, nullptr, stream);
    if (st != SBVR_OK)
        return st;
    CompactArgs args = a;
    void *moves[] = {&args};
    st = launch_kernel((const void *)moves_kernel, dim3(mark_groups(a.n_pages)), dim3(PAGE_THREADS), 0, stream, moves);
    if (st != SBVR_OK || a.t.R == 0)
        return st;
    int pieces = (a.t.max_pages + 255) / 256;
    void *renumber[] = {&args, &pieces};
    return launch_kernel((const void *)renumber_kernel, dim3(capped((long long)a.t.R * pieces)), dim3(256), 0, stream,
                         renumber);
}

// ---------------------------------------------------------------------------
// copies
// ---------------------------------------------------------------------------

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr int COPY_THREADS = 256, COPY_UNROLL = 4, COPY_CACHES = 64;

struct CopyArgs {
    sbvr_kv_cache c;  // without addresses
    int n, page_shift, chunk;
    const int32_t *src, *dst, *tokens;
    void *kv[COPY_CACHES][2];
};

// A workgroup takes `chunk` tokens of a page, in one cache's keys or values: X lanes
// for a token's pieces by Y tokens, as in the cache write.
__global__ void __launch_bounds__(COPY_THREADS) page_copy_kernel(CopyArgs a)
{
    const int layer = blockIdx.z >> 1, is_v = blockIdx.z & 1, first = blockIdx.y * a.chunk;
    const int64_t page_stride = is_v ? a.c.v_page_stride : a.c.k_page_stride;
    const int64_t token_stride = is_v ? a.c.v_token_stride : a.c.k_token_stride;
    const int64_t head_stride = is_v ? a.c.v_head_stride : a.c.k_head_stride;
    const int per_head = a.c.head_dim / 8, Y = blockDim.y;
    uint16_t *base = (uint16_t *)a.kv[layer][is_v];
    for (long long i = blockIdx.x; i < a.n; i += gridDim.x) {
        const int src = uniform_load(a.src + i), dst = uniform_load(a.dst + i);
        int last = min(a.tokens ? uniform_load(a.tokens + i) : 1 << a.page_shift, 1 << a.page_shift);
        last = min(last, first + a.chunk);
        if (src < 0 || dst < 0 || src >= a.c.n_pages || dst >= a.c.n_pages || first >= last)
            continue;
        for (int c = threadIdx.x; c < a.c.kv_heads * per_head; c += blockDim.x) {
            const int64_t at = c / per_head * head_stride + c % per_head * 8;
            const uint16_t *from = base + src * page_stride + at;
            uint16_t *to = base + dst * page_stride + at;
            for (int t0 = first + threadIdx.y; t0 < last; t0 += Y * COPY_UNROLL) {
                v4u v[COPY_UNROLL];
#pragma unroll
                for (int u = 0; u < COPY_UNROLL; ++u)
                    v[u] = *(const v4u *)(from + min(t0 + u * Y, last - 1) * token_stride);
#pragma unroll
                for (int u = 0; u < COPY_UNROLL; ++u)
                    if (t0 + u * Y < last)
                        *(v4u *)(to + (t0 + u * Y) * token_stride) = v[u];
            }
        }
    }
}

int launch_page_copy(const sbvr_kv_cache *caches, int n_caches, int n, const int32_t *src, const int32_t *dst,
                     const int32_t *tokens, hipStream_t stream)
{
    const sbvr_kv_cache &c = caches[0];
    CopyArgs a = {};
    a.c = c;
    a.c.k = a.c.v = nullptr;
    a.n = n;
    a.page_shift = __builtin_ctz(c.page_size);
    a.src = src;
    a.dst = dst;
    a.tokens = tokens;
    int x = 1;
    while (x < c.kv_heads * (c.head_dim / 8) && x < COPY_THREADS)
        x *= 2;
    const int y = COPY_THREADS / x;
    a.chunk = y * COPY_UNROLL < c.page_size ? y * COPY_UNROLL : c.page_size;
    for (int first = 0; first < n_caches; first += COPY_CACHES) {
        const int count = n_caches - first < COPY_CACHES ? n_caches - first : COPY_CACHES;
        for (int i = 0; i < count; ++i) {
            a.kv[i][0] = caches[first + i].k;
            a.kv[i][1] = caches[first + i].v;
        }
        void *argv[] = {&a};
        const int chunks = (c.page_size + a.chunk - 1) / a.chunk, most = (1 << 23) / (chunks * 2 * count);
        const dim3 grid(n < most ? n : most, chunks, 2 * count);
        const int st = launch_kernel((const void *)page_copy_kernel, grid, dim3(x, y), 0, stream, argv);
        if (st != SBVR_OK)
            return st;
    }
    return SBVR_OK;
}

}  // namespace sbvr
