// C ABI of the operators between the products of a step (include/sbvr.h):
// argument validation on the host, then dispatch to the kernel launchers.  A
// rejected call enqueues nothing and touches no output.
#include <math.h>
#include <stdint.h>

#include "sbvr.h"
#include "step.h"

using namespace sbvr;

namespace {

bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

constexpr int64_t STRIDE_MAX = (int64_t)1 << 40;  // elements: products with any index stay in 64 bits

bool stride_ok(int64_t s) { return s >= 0 && s <= STRIDE_MAX; }

bool piece_stride_ok(int64_t s) { return stride_ok(s) && s % 8 == 0; }

int check_page_size(int page_size)
{
    return page_size >= 16 && page_size <= SBVR_PAGE_MAX && (page_size & (page_size - 1)) == 0 ? SBVR_OK
                                                                                             : SBVR_E_INVALID_ARG;
}

int check_cache(const sbvr_kv_cache *c)
{
    if (!c || !c->k || !c->v || c->n_pages < 1 || c->kv_heads < 1 || c->head_dim < 8 || c->head_dim % 8 != 0 ||
        (c->dtype != SBVR_F16 && c->dtype != SBVR_BF16))
        return SBVR_E_INVALID_ARG;
    const int64_t strides[] = {c->k_page_stride, c->k_token_stride, c->k_head_stride,
                               c->v_page_stride, c->v_token_stride, c->v_head_stride};
    for (int64_t s : strides)
        if (!piece_stride_ok(s))
            return SBVR_E_INVALID_ARG;
    if (check_page_size(c->page_size) != SBVR_OK)
        return SBVR_E_INVALID_ARG;
    if (c->head_dim > 128 || c->kv_heads > 4096)
        return SBVR_E_UNSUPPORTED;
    // the kernels' byte offsets within a page are 32-bit
    if ((c->k_token_stride | c->v_token_stride) > (1ll << 30) / c->page_size)
        return SBVR_E_UNSUPPORTED;
    if (!aligned(c->k, 16) || !aligned(c->v, 16))
        return SBVR_E_ALIGNMENT;
    return SBVR_OK;
}

int check_attn_shape(int R, int max_new, int heads, int kv_heads, int head_dim)
{
    if (R < 1 || max_new < 1 || max_new > SBVR_TREE_MAX || kv_heads < 1 || heads < kv_heads ||
        heads % kv_heads != 0 || head_dim < 8 || head_dim % 8 != 0)
        return SBVR_E_INVALID_ARG;
    if (R > SBVR_REQUESTS_MAX || heads > 4096 || head_dim > 128)
        return SBVR_E_UNSUPPORTED;
    return SBVR_OK;
}

int tree_attention(bool whole, const sbvr_kv_cache *cache, int R, int T, int heads, const void *q,
                   int64_t q_token_stride, int64_t q_head_stride, const int32_t *page_table, int max_pages,
                   int64_t table_stride, const int32_t *context_lens, const int32_t *query_start,
                   const uint64_t *tree_mask, int max_new, float scale, void *out, void *workspace, size_t ws_bytes,
                   hipStream_t stream)
{
    int st = check_cache(cache);
    if (st != SBVR_OK)
        return st;
    if ((st = check_attn_shape(R, max_new, heads, cache->kv_heads, cache->head_dim)) != SBVR_OK)
        return st;
    if (T < 0 || max_pages < 1 || table_stride < max_pages || !stride_ok(table_stride) ||
        !piece_stride_ok(q_token_stride) || !piece_stride_ok(q_head_stride) || !isfinite(scale))
        return SBVR_E_INVALID_ARG;
    if (T == 0)
        return SBVR_OK;
    if (!q || !page_table || !context_lens || !query_start || !tree_mask || !out)
        return SBVR_E_INVALID_ARG;
    const size_t need = attn_workspace_bytes(R, max_new, heads, cache->kv_heads, cache->head_dim);
    if (ws_bytes < need || (need && !workspace))
        return SBVR_E_WORKSPACE;
    if (!aligned(q, 16) || !aligned(page_table, 4) || !aligned(context_lens, 4) || !aligned(query_start, 4) ||
        !aligned(tree_mask, 8) || !aligned(out, 16) || (need && !aligned(workspace, 16)))
        return SBVR_E_ALIGNMENT;
    const AttnArgs a{*cache, R, T, heads, max_pages, max_new, whole ? 0 : max_new, q, q_token_stride, q_head_stride,
                     page_table, table_stride, context_lens, query_start, tree_mask, scale, out, workspace, 0, 0};
    return launch_attn(a, stream);
}

}  // namespace

extern "C" {

int sbvr_batch_plan(int R, int T, int page_size, const int32_t *context_lens, const int32_t *new_lens,
                    const int32_t *free_pages, int n_free, const int32_t *parents, int32_t *page_table,
                    int max_pages, int64_t table_stride, int32_t *query_start, int32_t *token_request,
                    int32_t *positions, int64_t *slots, uint64_t *tree_mask, int32_t *used, hipStream_t stream)
{
    if (R < 1 || T < 0 || n_free < 0 || max_pages < 1 || table_stride < max_pages || !stride_ok(table_stride) ||
        check_page_size(page_size) != SBVR_OK)
        return SBVR_E_INVALID_ARG;
    if (!context_lens || !new_lens || (n_free && !free_pages) || !page_table || !query_start || !used)
        return SBVR_E_INVALID_ARG;
    if (T && (!token_request || !positions || !slots || !tree_mask))
        return SBVR_E_INVALID_ARG;
    if (R > SBVR_REQUESTS_MAX)
        return SBVR_E_UNSUPPORTED;
    if (!aligned(context_lens, 4) || !aligned(new_lens, 4) || !aligned(free_pages, 4) || !aligned(parents, 4) ||
        !aligned(page_table, 4) || !aligned(query_start, 4) || !aligned(token_request, 4) || !aligned(positions, 4) ||
        !aligned(slots, 8) || !aligned(tree_mask, 8) || !aligned(used, 4))
        return SBVR_E_ALIGNMENT;
    const PlanArgs a{R, T, __builtin_ctz(page_size), n_free, max_pages, context_lens, new_lens, free_pages, parents,
                     page_table, table_stride, query_start, token_request, positions, slots, tree_mask, used};
    return launch_plan(a, stream);
}

int sbvr_cache_write(const sbvr_kv_cache *cache, int T, const void *k, int64_t k_token_stride, int64_t k_head_stride,
                     const void *v, int64_t v_token_stride, int64_t v_head_stride, const int64_t *slots,
                     hipStream_t stream)
{
    const int st = check_cache(cache);
    if (st != SBVR_OK)
        return st;
    if (T < 0 || !piece_stride_ok(k_token_stride) || !piece_stride_ok(k_head_stride) ||
        !piece_stride_ok(v_token_stride) || !piece_stride_ok(v_head_stride))
        return SBVR_E_INVALID_ARG;
    if (T == 0)
        return SBVR_OK;
    if (!k || !v || !slots)
        return SBVR_E_INVALID_ARG;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8))
        return SBVR_E_ALIGNMENT;
    return launch_cache_write(*cache, T, k, k_token_stride, k_head_stride, v, v_token_stride, v_head_stride, slots,
                              stream);
}

size_t sbvr_tree_attention_workspace_bytes(int R, int max_new, int heads, int kv_heads, int head_dim)
{
    return check_attn_shape(R, max_new, heads, kv_heads, head_dim) == SBVR_OK
               ? attn_workspace_bytes(R, max_new, heads, kv_heads, head_dim)
               : 0;
}

int sbvr_tree_attention(const sbvr_kv_cache *cache, int R, int T, int heads, const void *q, int64_t q_token_stride,
                        int64_t q_head_stride, const int32_t *page_table, int max_pages, int64_t table_stride,
                        const int32_t *context_lens, const int32_t *query_start, const uint64_t *tree_mask,
                        int max_new, float scale, void *out, void *workspace, size_t ws_bytes, hipStream_t stream)
{
    return tree_attention(false, cache, R, T, heads, q, q_token_stride, q_head_stride, page_table, max_pages,
                          table_stride, context_lens, query_start, tree_mask, max_new, scale, out, workspace, ws_bytes,
                          stream);
}

int sbvr_tree_attention_whole(const sbvr_kv_cache *cache, int R, int T, int heads, const void *q,
                              int64_t q_token_stride, int64_t q_head_stride, const int32_t *page_table, int max_pages,
                              int64_t table_stride, const int32_t *context_lens, const int32_t *query_start,
                              const uint64_t *tree_mask, int max_new, float scale, void *out, void *workspace,
                              size_t ws_bytes, hipStream_t stream)
{
    return tree_attention(true, cache, R, T, heads, q, q_token_stride, q_head_stride, page_table, max_pages,
                          table_stride, context_lens, query_start, tree_mask, max_new, scale, out, workspace, ws_bytes,
                          stream);
}

int sbvr_residual_norm(int T, int H, int dtype, int x_dtype, const void *x, int64_t x_stride, const void *y,
                       int64_t y_stride, const void *post_weight, const void *gate, int64_t gate_stride, float scale,
                       const void *pre_weight, float eps, void *x_out, int64_t x_out_stride, void *h_out,
                       int64_t h_stride, hipStream_t stream)
{
    if (T < 0 || H < 1 || (dtype != SBVR_F16 && dtype != SBVR_BF16) || (x_dtype != dtype && x_dtype != SBVR_F32) ||
        !(eps >= 0.f) || !isfinite(eps) || !isfinite(scale))
        return SBVR_E_INVALID_ARG;
    const int64_t strides[] = {x_stride, y ? y_stride : 0, gate ? gate_stride : 0, x_out ? x_out_stride : 0,
                               h_out ? h_stride : 0};
    for (int64_t s : strides)
        if (!stride_ok(s))
            return SBVR_E_INVALID_ARG;
    if (T > 1 && ((x_out && x_out_stride < H) || (h_out && h_stride < H)))  // rows would overlap
        return SBVR_E_INVALID_ARG;
    if (H > SBVR_NORM_MAX_WIDTH)
        return SBVR_E_UNSUPPORTED;
    if (T == 0)
        return SBVR_OK;
    if (!x || (!x_out && !h_out) || (h_out && !pre_weight))
        return SBVR_E_INVALID_ARG;
    if (T > 1 && x_out == x && x_out_stride != x_stride)  // rows would be written before they are read
        return SBVR_E_INVALID_ARG;
    const size_t xa = x_dtype == SBVR_F32 ? 4 : 2;
    if (!aligned(x, xa) || !aligned(x_out, xa) || !aligned(y, 2) || !aligned(post_weight, 2) || !aligned(gate, 2) ||
        !aligned(pre_weight, 2) || !aligned(h_out, 2))
        return SBVR_E_ALIGNMENT;
    const NormArgs a{T, H, x, y, y ? post_weight : nullptr, y ? gate : nullptr, h_out ? pre_weight : nullptr, x_out,
                     h_out, strides[0], strides[1], y ? strides[2] : 0, strides[3], strides[4], scale, eps};
    return launch_norm(a, dtype, x_dtype, stream);
}

int sbvr_adjust_logits(const sbvr_logits_args *a, hipStream_t stream)
{
    if (!a || a->R < 1 || a->T < 0 || a->V < 1 || a->dtype < SBVR_F16 || a->dtype > SBVR_F32 ||
        (a->out_dtype != a->dtype && a->out_dtype != SBVR_F32) || !stride_ok(a->logits_stride) ||
        !stride_ok(a->out_stride) || (a->T > 1 && a->out_stride < a->V))
        return SBVR_E_INVALID_ARG;
    if (a->T > (1 << 16) - 1 || a->V > (1 << 30))
        return SBVR_E_UNSUPPORTED;
    if (a->T == 0)  // (an empty list may have no address: the checks of what goes together are for rows)
        return SBVR_OK;
    if (a->history && !a->history_start)
        return SBVR_E_INVALID_ARG;
    if (a->bias_tokens && (!a->bias_start || !a->bias_values))
        return SBVR_E_INVALID_ARG;
    if (a->grammar && (a->grammar_count < 1 || !stride_ok(a->grammar_stride) ||
                       a->grammar_stride < ((int64_t)a->V + 31) / 32))
        return SBVR_E_INVALID_ARG;
    const int drafts = (a->draft_tokens != nullptr) + (a->query_start != nullptr) + (a->tree_mask != nullptr);
    if (drafts != 0 && drafts != 3)
        return SBVR_E_INVALID_ARG;
    if (!a->logits || !a->out)
        return SBVR_E_INVALID_ARG;
    const size_t ia = a->dtype == SBVR_F32 ? 4 : 2, oa = a->out_dtype == SBVR_F32 ? 4 : 2;
    const void *words[] = {a->token_request, a->history, a->history_start, a->prompt_lens, a->repetition,
                           a->frequency, a->presence, a->temperature, a->bias_tokens, a->bias_start, a->bias_values,
                           a->grammar, a->grammar_rows, a->draft_tokens, a->query_start};
    for (const void *p : words)
        if (!aligned(p, 4))
            return SBVR_E_ALIGNMENT;
    if (!aligned(a->logits, ia) || !aligned(a->out, oa) || !aligned(a->tree_mask, 8))
        return SBVR_E_ALIGNMENT;
    // elements would be written before they are read
    if (a->out == a->logits && (a->out_dtype != a->dtype || (a->T > 1 && a->out_stride != a->logits_stride)))
        return SBVR_E_INVALID_ARG;
    return launch_logits(*a, stream);
}

}  // extern "C"
