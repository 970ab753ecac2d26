// Shared by the operators between the products of a step (plan, cache write,
// attention, norms, logits, rotation, beams, pages): element types, launch
// parameters and a search.
#pragma once

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <type_traits>

#include "launch.h"
#include "sbvr.h"

namespace sbvr {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// a 16-byte or 8-byte piece of a row of 16-bit elements
template <int N>
struct alignas(2 * N) Halves {
    uint32_t w[N / 2];
};

// N elements, at any alignment of T: one or two 16-byte accesses, which the
// hardware takes at any address
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Loose {
    T e[N];
};

// its words, loaded and stored as whole vectors (a struct may be taken apart by
// elements, and a branch's result then is, with a wait for it)
template <typename T>
using Words = uint32_t __attribute__((ext_vector_type(2 * sizeof(T))));
template <typename T>
using LooseWords = uint32_t __attribute__((ext_vector_type(2 * sizeof(T)), aligned(sizeof(T))));

template <typename T>
__device__ __forceinline__ Words<T> load_words(const T *p)
{
    return *(const LooseWords<T> *)p;
}

template <typename T>
__device__ __forceinline__ Words<T> to_words(const Loose<T, 8> &r)
{
    Words<T> w;
    __builtin_memcpy(&w, &r, sizeof(w));
    return w;
}

template <typename T>
__device__ __forceinline__ Loose<T, 8> from_words(const Words<T> &w)
{
    Loose<T, 8> r;
    __builtin_memcpy(&r, &w, sizeof(r));
    return r;
}

template <typename T>
__device__ __forceinline__ void store_words(T *p, const Words<T> &w)
{
    *(LooseWords<T> *)p = w;
}

// A value whose address is the same in every lane and that the kernel that reads it
// does not write (an earlier one may have: a kernel's start drops what the scalar
// cache holds), read on the scalar side: a vector load would take a lane's worth of
// work per wavefront and have its wait among those of the data.
template <typename T>
__device__ __forceinline__ T uniform_load(const T *p)
{
    return *(const __attribute__((address_space(4))) T *)p;
}

struct PlanArgs {
    int R, T, page_shift, n_free, max_pages;
    const int32_t *context_lens, *new_lens, *free_pages, *parents;
    int32_t *page_table;
    int64_t table_stride;
    int32_t *query_start, *token_request, *positions;
    int64_t *slots;
    uint64_t *tree_mask;
    int32_t *used;
};

struct AttnArgs {
    sbvr_kv_cache kv;
    int R, T, heads, max_pages, max_new;
    // the most of a request's new tokens that are computed where not all of them
    // are: max_new, or 0 if every row of the output is to be written
    int cut;
    const void *q;
    int64_t q_token_stride, q_head_stride;
    const int32_t *page_table;
    int64_t table_stride;
    const int32_t *context_lens, *query_start;
    const uint64_t *tree_mask;
    float scale;
    void *out;
    void *workspace;
    int by_item;  // set by the launcher: joins are numbered by item
    int joins;    // and the number of joins
};

struct NormArgs {
    int T, H;
    const void *x, *y, *post, *gate, *pre;
    void *x_out, *h_out;
    int64_t x_stride, y_stride, gate_stride, x_out_stride, h_stride;
    float scale, eps;
};

// sbvr_rotary and sbvr_rotary_write: v and slots are given for the latter.
struct RotaryArgs {
    sbvr_rotary_args r;
    sbvr_kv_cache kv;
    const void *v;
    int64_t v_token_stride, v_head_stride;
    const int64_t *slots;
};

struct PageTable {
    int R, page_shift, max_pages;
    const int32_t *context_lens, *page_table;
    int64_t table_stride;
};

struct UsageArgs {
    PageTable t;
    int n_pages;
    int32_t *refs, *free_pages, *counts;
    int32_t *used;     // the workspace: used pages of each share of the pages, and behind
    int32_t *partial;  // them, set by the launcher, counts by splits of the rows
};

struct ForkArgs {
    PageTable t;  // R: old rows
    int rows_out, group_in, group_out, n_free;
    const int32_t *parents, *free_pages, *taken;
    int32_t *out_table;
    int64_t out_stride;
    int32_t *out_lens, *src, *dst, *tokens, *used;
};

struct CompactArgs {
    PageTable t;
    int n_pages;
    int32_t *out_table;
    int64_t out_stride;
    int32_t *src, *dst, *counts;
    uint32_t *marks;  // the workspace: a bit per page, and behind them, set by the
    int32_t *number;  // launcher, the number of the move of a page that moves
};

int launch_plan(const PlanArgs &a, hipStream_t stream);
int launch_cache_write(const sbvr_kv_cache &c, int T, const void *k, int64_t k_token_stride, int64_t k_head_stride,
                       const void *v, int64_t v_token_stride, int64_t v_head_stride, const int64_t *slots,
                       hipStream_t stream);
size_t attn_workspace_bytes(int R, int max_new, int heads, int kv_heads, int head_dim);
int launch_attn(const AttnArgs &a, hipStream_t stream);
int launch_norm(const NormArgs &a, int dtype, int x_dtype, hipStream_t stream);
int launch_logits(const sbvr_logits_args &a, hipStream_t stream);
int launch_rotary(const RotaryArgs &a, hipStream_t stream);
size_t beam_workspace_bytes(int R, int B, int V, int n, int n_end);
int launch_beam(const sbvr_beam_args &a, void *workspace, hipStream_t stream);
size_t usage_workspace_bytes(int R, int max_pages, int n_pages);
int launch_usage(const UsageArgs &a, hipStream_t stream);
int launch_fork(const ForkArgs &a, hipStream_t stream);
size_t compact_workspace_bytes(int n_pages);
int launch_compact(const CompactArgs &a, hipStream_t stream);
int launch_page_copy(const sbvr_kv_cache *caches, int n_caches, int n, const int32_t *src, const int32_t *dst,
                     const int32_t *tokens, hipStream_t stream);

// i / d for 0 <= i < 2^24
__device__ __forceinline__ int small_div(int i, int d, float inverse)
{
    int q = (int)((float)i * inverse);
    q -= q * d > i;
    q += (q + 1) * d <= i;
    return q;
}

// The last index i of the ascending start[0 .. n] with start[i] <= v, for
// start[0] <= v < start[n]: the owner of item v, empty owners skipped.
template <typename I>
__device__ __forceinline__ int owner_of(const I *start, int n, I v)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= v)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

}  // namespace sbvr
