// Shared by the operators between the products of a step (plan, cache write,
// attention, norms, logits): element types, launch parameters and a search.
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

// A value whose address is the same in every lane and that no kernel of these
// operators writes, read on the scalar side: a vector load would take a lane's
// worth of work per wavefront and have its wait among those of the data.
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

int launch_plan(const PlanArgs &a, hipStream_t stream);
int launch_cache_write(const sbvr_kv_cache &c, int T, const void *k, int64_t k_token_stride, int64_t k_head_stride,
                       const void *v, int64_t v_token_stride, int64_t v_head_stride, const int64_t *slots,
                       hipStream_t stream);
size_t attn_workspace_bytes(int R, int max_new, int heads, int kv_heads, int head_dim);
int launch_attn(const AttnArgs &a, hipStream_t stream);
int launch_norm(const NormArgs &a, int dtype, int x_dtype, hipStream_t stream);
int launch_logits(const sbvr_logits_args &a, hipStream_t stream);

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
