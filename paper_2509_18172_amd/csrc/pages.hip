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

// Inclusive scan over a wavefront's lanes: row shifts by 1, 2, 4 and 8, and the rows'
// last lanes to the rows behind.
__device__ __forceinline__ int scan_of_wave(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
    return v;
}

// Sum of v over the workgroup's threads before this one, and over all of them.
template <int THREADS>
__device__ __forceinline__ int sum_before(int v, int &all, int *scratch)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, up = scan_of_wave(v);
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

constexpr int PAGE_THREADS = 1024, PAGE_WAVES = PAGE_THREADS / 64;

__device__ __forceinline__ int lanes_before(uint64_t mask)
{
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// Calls f(page) for every entry in use, and f(-1) beside, of one of `splits` parts, by
// a workgroup of PAGE_THREADS.  The rows' entries are chunks of 64, numbered over all
// rows, and shared out evenly: sixteen a wavefront are in flight, whose rows its lanes
// find together.  start: R + 1 numbers of LDS; meanwhile(): what is done while the
// lengths are loaded, ready for f behind a barrier.
template <typename M, typename F>
__device__ __forceinline__ void each_page(const PageTable &t, int split, int splits, int *start, int *scratch, M meanwhile, F f)
{
    constexpr int PER = SBVR_REQUESTS_MAX / PAGE_THREADS, FLIGHT = 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int chunks[PER], own = 0, all;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int r = threadIdx.x * PER + i;
        chunks[i] = r < t.R ? (entries_in_use(t.context_lens[r], t) + 63) >> 6 : 0;
    }
    meanwhile();
#pragma unroll
    for (int i = 0; i < PER; ++i)
        own += chunks[i];
    int before = sum_before<PAGE_THREADS>(own, all, scratch);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int r = threadIdx.x * PER + i;
        if (r < t.R)
            start[r] = before;
        before += chunks[i];
    }
    if (threadIdx.x == 0)
        start[t.R] = all;
    __syncthreads();
    // while one batch is used the next one is on its way
    const int step = splits * PAGE_WAVES * FLIGHT;
    int a[FLIGHT], b[FLIGHT];
    auto fetch = [&](int c0, int (&page)[FLIGHT]) {
        const int c = c0 + lane % FLIGHT, row = owner_of(start, t.R, min(c, all - 1)), entry = (c - start[row]) * 64;
        const int left = c < all ? entries_in_use(t.context_lens[row], t) - entry : 0;
        const uint64_t at = (uint64_t)(t.page_table + row * t.table_stride + entry);
#pragma unroll
        for (int u = 0; u < FLIGHT; ++u) {
            const int n = __builtin_amdgcn_readlane(left, u);
            const uint32_t low = __builtin_amdgcn_readlane((uint32_t)at, u);
            const uint32_t high = __builtin_amdgcn_readlane((uint32_t)(at >> 32), u);
            const int32_t *entries = (const int32_t *)((uint64_t)high << 32 | low);
            page[u] = lane < n ? entries[lane] : -1;
        }
    };
    auto use = [&](const int (&page)[FLIGHT]) {
#pragma unroll
        for (int u = 0; u < FLIGHT; ++u)
            f(page[u]);
    };
    int c0 = (split * PAGE_WAVES + wave) * FLIGHT;
    if (c0 < all)
        fetch(c0, a);
    for (; c0 < all; c0 += 2 * step) {
        if (c0 + step < all)
            fetch(c0 + step, b);
        use(a);
        if (c0 + 2 * step < all)
            fetch(c0 + 2 * step, a);
        if (c0 + step < all)
            use(b);
    }
}

// A workgroup owns USAGE_PAGES pages, whose counts it holds in LDS: it goes through
// the entries in use and counts its own.  (Counting in memory, by atomic additions
// that cross the chip's L2s, took 40 us for 262144 entries.)  Few pages and entries:
// that is all, and the workgroup makes the list of free pages too.  Many entries are
// split over several workgroups, whose counts a second launch adds up; the list of
// many pages is made by a last launch, where each workgroup adds up the used pages
// before its own.
constexpr int USAGE_PAGES = 11264, SHARE = USAGE_PAGES / PAGE_WAVES;  // SHARE: pages of a wavefront, or of a later launch's workgroup
// A part has USAGE_CHUNKS chunks or more: splitting pays from 32768 entries on (of
// 11264 pages, 12.0 us either way; 16384 entries 9.8 us whole, 11.9 in two parts;
// 65536 of 65536 pages 17.9 whole, 12.6 in four).  1024 rows of 8192 tokens (524288
// entries): 16.9 us, 77.9 whole, of which the table's 2 MB are the least.
constexpr int USAGE_CHUNKS = 256, USAGE_SPLITS = 16, USAGE_GROUPS = 256;

// The list of free pages for the pages first .. first + n, by one wavefront; `used`
// of the lower ones are, and `total` of all.
__device__ __forceinline__ void list_free(const UsageArgs &a, const int *count, int first, int n, int used, int total)
{
    const int lane = threadIdx.x & 63;
    for (int i = 0; i < n; i += 64) {
        const bool in = i + lane < n;
        const bool here = in && count[min(i + lane, n - 1)] > 0;
        const uint64_t marks = __ballot(here);
        const int p = first + i + lane;
        if (in && !here)
            a.free_pages[p - (used + lanes_before(marks))] = p;
        if (in && p >= a.n_pages - total)
            a.free_pages[p] = -1;
        used += __popcll(marks);
    }
}

__device__ __forceinline__ int count_used(const int *count, int n)
{
    const int lane = threadIdx.x & 63;
    int used = 0;
    for (int i = 0; i < n; i += 64)
        used += __popcll(__ballot(i + lane < n && count[min(i + lane, n - 1)] > 0));
    return used;
}

__global__ void __launch_bounds__(PAGE_THREADS) usage_kernel(UsageArgs a)
{
    __shared__ int count[USAGE_PAGES], start[SBVR_REQUESTS_MAX + 1], used_by_wave[PAGE_WAVES];
    const int first = blockIdx.x * USAGE_PAGES, n = min(USAGE_PAGES, a.n_pages - first);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool alone = gridDim.x == 1 && gridDim.y == 1;
    auto clear = [&] {
        for (int i = threadIdx.x; i < n; i += PAGE_THREADS)
            count[i] = 0;
    };
    each_page(a.t, blockIdx.y, gridDim.y, start, used_by_wave, clear, [&](int page) {
        const uint32_t own = (uint32_t)page - (uint32_t)first;
        if (own < (uint32_t)n)
            atomicAdd(&count[own], 1);
    });
    __syncthreads();
    int32_t *out = (gridDim.y > 1 ? a.partial + (long long)blockIdx.y * a.n_pages : a.refs) + first;
    for (int i = threadIdx.x; i < n; i += PAGE_THREADS)
        out[i] = count[i];
    if (gridDim.y > 1)
        return;
    // alone: the wavefronts share the pages evenly
    const int share = alone ? (n + PAGE_THREADS - 1) / PAGE_THREADS * 64 : SHARE;
    const int i0 = min(wave * share, n), m = min(share, n - i0);
    const int used = count_used(count + i0, m);
    if (!alone) {
        if (lane == 0 && m > 0)
            a.used[blockIdx.x * PAGE_WAVES + wave] = used;
        return;
    }
    if (lane == 0)
        used_by_wave[wave] = used;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < PAGE_WAVES; ++w) {
        before += w < wave ? used_by_wave[w] : 0;
        all += used_by_wave[w];
    }
    list_free(a, count + i0, i0, m, before, all);
    if (threadIdx.x == 0) {
        a.counts[0] = a.n_pages - all;
        a.counts[1] = all;
    }
}

// A share's counts added up over the splits.
__global__ void __launch_bounds__(256) add_kernel(UsageArgs a, int splits)
{
    __shared__ int scratch[4];
    const int first = blockIdx.x * SHARE, n = min(SHARE, a.n_pages - first);
    int used = 0, all;
#pragma unroll
    for (int k = 0; k < (SHARE + 255) / 256; ++k) {
        const int i = k * 256 + threadIdx.x;
        int sum = 0, part[USAGE_SPLITS];
#pragma unroll
        for (int s = 0; s < USAGE_SPLITS; ++s)
            part[s] = i < n && s < splits ? a.partial[(long long)s * a.n_pages + first + i] : 0;
#pragma unroll
        for (int s = 0; s < USAGE_SPLITS; ++s)
            sum += part[s];
        if (i < n)
            a.refs[first + i] = sum;
        used += sum > 0;
    }
    sum_before<256>(used, all, scratch);
    if (threadIdx.x == 0)
        a.used[blockIdx.x] = all;
}

// The free pages of a share.
__global__ void __launch_bounds__(256) free_kernel(UsageArgs a)
{
    __shared__ int scratch[4], used_by_wave[4];
    const int first = blockIdx.x * SHARE, n = min(SHARE, a.n_pages - first), shares = gridDim.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int i0 = min(wave * (SHARE / 4), n), m = min(SHARE / 4, n - i0);
    const int used = count_used(a.refs + first + i0, m);
    if (lane == 0)
        used_by_wave[wave] = used;
    int before = 0, all = 0, sum;
    for (int w = threadIdx.x; w < shares; w += 256) {
        const int u = a.used[w];
        all += u;
        before += w < (int)blockIdx.x ? u : 0;
    }
    sum_before<256>(all, sum, scratch);
    all = sum;
    sum_before<256>(before, sum, scratch);
    before = sum;
    for (int w = 0; w < wave; ++w)
        before += used_by_wave[w];
    list_free(a, a.refs + first + i0, first + i0, m, before, all);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.counts[0] = a.n_pages - all;
        a.counts[1] = all;
    }
}

namespace {

struct UsageShape {
    int owners, splits, shares;
};

UsageShape usage_shape(int R, int max_pages, int n_pages)
{
    UsageShape s;
    s.owners = (n_pages + USAGE_PAGES - 1) / USAGE_PAGES;
    s.shares = (n_pages + SHARE - 1) / SHARE;
    const long long chunks = (long long)R * ((max_pages + 63) / 64);
    s.splits = chunks < 2 * USAGE_CHUNKS ? 1 : chunks < USAGE_SPLITS * USAGE_CHUNKS ? (int)(chunks / USAGE_CHUNKS) : USAGE_SPLITS;
    if (s.splits * s.owners > USAGE_GROUPS)
        s.splits = USAGE_GROUPS / s.owners > 1 ? USAGE_GROUPS / s.owners : 1;
    return s;
}

size_t used_bytes(const UsageShape &s) { return ((size_t)s.shares * sizeof(int32_t) + 15) / 16 * 16; }

}  // namespace

size_t usage_workspace_bytes(int R, int max_pages, int n_pages)
{
    const UsageShape s = usage_shape(R, max_pages, n_pages);
    return used_bytes(s) + (s.splits > 1 ? (size_t)s.splits * n_pages * sizeof(int32_t) : 0);
}

int launch_usage(const UsageArgs &a, hipStream_t stream)
{
    const UsageShape s = usage_shape(a.t.R, a.t.max_pages, a.n_pages);
    UsageArgs args = a;
    args.partial = (int32_t *)((char *)a.used + used_bytes(s));
    int splits = s.splits;
    void *argv[] = {&args, &splits};
    int st = launch_kernel((const void *)usage_kernel, dim3(s.owners, s.splits), dim3(PAGE_THREADS), 0, stream, argv);
    if (st != SBVR_OK || (s.owners == 1 && s.splits == 1))
        return st;
    if (s.splits > 1 &&
        (st = launch_kernel((const void *)add_kernel, dim3(s.shares), dim3(256), 0, stream, argv)) != SBVR_OK)
        return st;
    return launch_kernel((const void *)free_kernel, dim3(s.shares), dim3(256), 0, stream, argv);
}

// ---------------------------------------------------------------------------
// fork
// ---------------------------------------------------------------------------

// Every workgroup finds which rows need a page, and how many do before each; then
// it writes its share of the rows.  A chain of latencies -- parents and free pages,
// lengths, table, scan, table again: 4 rows of 63 pages with their copies 5.6 us in
// two launches of which an empty one is 2.1.
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
    // as few rows a thread as can be: 512 rows of 40 pages take 4.3 us with one, 5.8 with
    // four (256 threads of four: 5.3), 1000 rows of 1024 pages 6.5 and 7.8
    const void *kernel = rows <= 256    ? (const void *)fork_kernel<256, 1>
                         : rows <= 1024 ? (const void *)fork_kernel<1024, 1>
                                        : (const void *)fork_kernel<1024, 4>;
    return launch_kernel(kernel, dim3(grid), dim3(threads), 0, stream, argv);
}

// ---------------------------------------------------------------------------
// compaction
// ---------------------------------------------------------------------------

// Words of marks, a bit per page.
__host__ __device__ constexpr int mark_words(int n_pages) { return (n_pages + 31) / 32; }

// The new number of an entry's page: the used pages that stay keep theirs.
__device__ __forceinline__ int renumbered(const CompactArgs &a, int page, int used)
{
    if (page < 0 || page >= a.n_pages)
        return -1;
    return page < used ? page : a.dst[a.number[page]];
}

// (A wavefront per 64 entries of a row; at most 4096 rows of 2^22.)
__device__ __forceinline__ void renumber_entries(const CompactArgs &a, int used, int first, int step)
{
    const PageTable &t = a.t;
    const int pieces = (t.max_pages + 63) / 64, items = t.R * pieces;
    for (int item = first; item < items; item += step) {
        const int r = item / pieces, e = (item - r * pieces) * 64 + (threadIdx.x & 63);
        if (e >= t.max_pages)
            continue;
        const int page = e < entries_in_use(t.context_lens[r], t) ? t.page_table[r * t.table_stride + e] : -1;
        a.out_table[r * a.out_stride + e] = renumbered(a, page, used);
    }
}

// Few pages and entries: one workgroup marks the used pages in LDS, finds the moves
// -- the k-th free page below the number of used ones is dst[k], the k-th used page
// from there on src[k], and number[p] = k for that -- and, if `whole`, rewrites the
// tables too.  Measured: 1024 entries 6.2 us whole, 7.5 with a second launch for the
// tables; 4096 9.9 and 9.5; 16384 25.3 and 16.4.  131072 entries 55 us in two launches,
// 58 with the marks in memory; 262144 73 and 64; 1048576 193 and 115.
constexpr int COMPACT_WHOLE = 2048, COMPACT_ENTRIES = 131072;
constexpr int COMPACT_PAGES = 131072;  // whose marks, and their sums, LDS holds

__global__ void __launch_bounds__(PAGE_THREADS) compact_kernel(CompactArgs a, int whole)
{
    __shared__ uint32_t marks[COMPACT_PAGES / 32];
    __shared__ int used_before[COMPACT_PAGES / 32];  // of each word
    __shared__ int start[SBVR_REQUESTS_MAX + 1];
    __shared__ int scratch[PAGE_WAVES], stays;
    const int tid = threadIdx.x, words = mark_words(a.n_pages), lists = a.n_pages / 2;
    auto clear = [&] {
        for (int w = tid; w < words; w += PAGE_THREADS)
            marks[w] = 0;
    };
    each_page(a.t, 0, 1, start, scratch, clear, [&](int page) {
        if ((uint32_t)page < (uint32_t)a.n_pages)
            atomicOr(&marks[page >> 5], 1u << (page & 31));
    });
    __syncthreads();
    constexpr int PER = COMPACT_PAGES / 32 / PAGE_THREADS;
    int own = 0, total;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        own += tid * PER + i < words ? __popc(marks[tid * PER + i]) : 0;
    int before = sum_before<PAGE_THREADS>(own, total, scratch);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int w = tid * PER + i;
        if (w < words) {
            used_before[w] = before;
            if (w == total >> 5)
                stays = before + __popc(marks[w] & ((1u << (total & 31)) - 1));
            before += __popc(marks[w]);
        }
    }
    if (tid == 0 && total == 32 * words)
        stays = total;
    __syncthreads();
    const int moved = total - stays;
    for (int p = tid; p < a.n_pages; p += PAGE_THREADS) {
        const uint32_t mark = marks[p >> 5];
        const int used = used_before[p >> 5] + __popc(mark & ((1u << (p & 31)) - 1));
        const bool in_use = (mark >> (p & 31)) & 1;
        if (in_use && p >= total) {
            a.number[p] = used - stays;
            a.src[used - stays] = p;
        } else if (!in_use && p < total) {
            a.dst[p - used] = p;
        }
        if (p >= moved && p < lists)
            a.src[p] = a.dst[p] = -1;
    }
    if (tid == 0) {
        a.counts[0] = total;
        a.counts[1] = moved;
    }
    if (whole) {
        __syncthreads();
        renumber_entries(a, total, tid >> 6, PAGE_WAVES);
    }
}

// Many: the same in launches of many workgroups, with the marks in memory.
__global__ void __launch_bounds__(256) clear_kernel(uint32_t *marks, int words)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < words)
        marks[i] = 0;
}

__global__ void __launch_bounds__(256) mark_kernel(CompactArgs a)
{
    const PageTable &t = a.t;
    const int pieces = (t.max_pages + 255) / 256;
    const long long items = (long long)t.R * pieces;
    for (long long item = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); item < items; item += (long long)gridDim.x * 4) {
        const int r = (int)(item / pieces), e0 = (int)(item % pieces) * 256 + (threadIdx.x & 63);
        const int used = entries_in_use(t.context_lens[r], t);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int e = e0 + 64 * u;
            const int page = e < used ? t.page_table[r * t.table_stride + e] : -1;
            if (page >= 0 && page < a.n_pages)
                atomicOr(&a.marks[page >> 5], 1u << (page & 31));
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

__global__ void __launch_bounds__(PAGE_THREADS) moves_kernel(CompactArgs a)
{
    __shared__ int scratch[PAGE_WAVES];
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

__global__ void __launch_bounds__(256) renumber_kernel(CompactArgs a)
{
    renumber_entries(a, a.counts[0], blockIdx.x * 4 + (threadIdx.x >> 6), gridDim.x * 4);
}

size_t compact_workspace_bytes(int n_pages)
{
    return ((size_t)mark_words(n_pages) * sizeof(uint32_t) + 15) / 16 * 16 + (size_t)n_pages * sizeof(int32_t);
}

namespace {

// workgroups of a launch whose items may be more than a grid can be
unsigned capped(long long n) { return (unsigned)(n < (1 << 20) ? n : 1 << 20); }

}  // namespace

int launch_compact(const CompactArgs &a, hipStream_t stream)
{
    CompactArgs args = a;
    args.number = (int32_t *)((char *)a.marks + ((size_t)mark_words(a.n_pages) * sizeof(uint32_t) + 15) / 16 * 16);
    void *argv[] = {&args};
    const long long entries = (long long)a.t.R * a.t.max_pages;
    int st;
    if (a.n_pages <= COMPACT_PAGES && entries <= COMPACT_ENTRIES) {
        int whole = entries <= COMPACT_WHOLE;
        void *one[] = {&args, &whole};
        st = launch_kernel((const void *)compact_kernel, dim3(1), dim3(PAGE_THREADS), 0, stream, one);
        if (st != SBVR_OK || whole)
            return st;
    } else {
        int words = mark_words(a.n_pages);
        void *clear[] = {&args.marks, &words};
        st = launch_kernel((const void *)clear_kernel, dim3((words + 255) / 256), dim3(256), 0, stream, clear);
        if (st == SBVR_OK && a.t.R)
            st = launch_kernel((const void *)mark_kernel, dim3(capped(((long long)a.t.R * ((a.t.max_pages + 255) / 256) + 3) / 4)),
                               dim3(256), 0, stream, argv);
        if (st == SBVR_OK)
            st = launch_kernel((const void *)moves_kernel, dim3((words + PAGE_THREADS - 1) / PAGE_THREADS),
                               dim3(PAGE_THREADS), 0, stream, argv);
        if (st != SBVR_OK || a.t.R == 0)
            return st;
    }
    return launch_kernel((const void *)renumber_kernel, dim3(capped(((long long)a.t.R * ((a.t.max_pages + 63) / 64) + 3) / 4)),
                         dim3(256), 0, stream, argv);
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
// for a token's pieces by Y tokens, as in the cache write.  Stores go past the caches
// (484 MB of forked pages in 8 layers: 126 us with the fork, 130 through them); loads do not (copies
// that fit in the caches 12.8 us, 13.8 past them).  256 rows of 4096 tokens compacted in
// two layers, 3.0 GB: 606 us together, 4.95 TB/s -- what a plain copy reaches.
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
                        __builtin_nontemporal_store(v[u], (v4u *)(to + (t0 + u * Y) * token_stride));
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
