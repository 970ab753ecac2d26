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

// A [T][heads][head_dim] tensor that is read.
int check_heads(const void *p, int64_t token_stride, int64_t head_stride)
{
    if (!piece_stride_ok(token_stride) || !piece_stride_ok(head_stride))
        return SBVR_E_INVALID_ARG;
    return !p ? SBVR_E_INVALID_ARG : !aligned(p, 16) ? SBVR_E_ALIGNMENT : SBVR_OK;
}

// One that is written, in place where it is `in`: its rows must not overlap.
int check_heads_out(const void *p, int64_t token_stride, int64_t head_stride, int T, int heads, int head_dim,
                    const void *in, int64_t in_token_stride, int64_t in_head_stride)
{
    const int st = check_heads(p, token_stride, head_stride);
    if (st != SBVR_OK)
        return st;
    const int64_t token = T > 1 ? token_stride : head_dim, head = heads > 1 ? head_stride : head_dim;
    const __int128 row = (__int128)(heads - 1) * head + head_dim, column = (__int128)(T - 1) * token + head_dim;
    if (token < head_dim || head < head_dim || (T > 1 && heads > 1 && token < row && head < column))
        return SBVR_E_INVALID_ARG;
    if (p == in && ((T > 1 && token_stride != in_token_stride) || (heads > 1 && head_stride != in_head_stride)))
        return SBVR_E_INVALID_ARG;
    return SBVR_OK;
}

// cache: what the keys are written to, or NULL
int check_rotary(const sbvr_rotary_args *a, const sbvr_kv_cache *cache)
{
    if (!a || a->T < 0 || a->heads < 0 || a->kv_heads < 0 || a->heads + (int64_t)a->kv_heads < 1 || a->head_dim < 8 ||
        a->head_dim % 8 != 0 || a->pairs < 1 || a->pairs > a->head_dim / 2 || a->axes < 1 || a->dtype < SBVR_F16 ||
        a->dtype > SBVR_F32 || (a->interleaved & ~1) || (a->inverse & ~1) || !stride_ok(a->position_stride) ||
        (a->axes > 1 && a->position_stride != 0 && a->position_stride < a->T))
        return SBVR_E_INVALID_ARG;
    if (cache && (a->kv_heads != cache->kv_heads || a->head_dim != cache->head_dim || a->dtype != cache->dtype || a->k_out))
        return SBVR_E_INVALID_ARG;
    if (a->heads > 4096 || a->kv_heads > 4096 || a->head_dim > SBVR_ROTARY_DIM_MAX)
        return SBVR_E_UNSUPPORTED;
    if (a->T == 0)
        return SBVR_OK;
    if (!a->positions || !a->frequencies)
        return SBVR_E_INVALID_ARG;
    int st = SBVR_OK;
    if (a->heads && (st = check_heads(a->q, a->q_token_stride, a->q_head_stride)) != SBVR_OK)
        return st;
    if (a->heads && (st = check_heads_out(a->q_out, a->q_out_token_stride, a->q_out_head_stride, a->T, a->heads,
                                          a->head_dim, a->q, a->q_token_stride, a->q_head_stride)) != SBVR_OK)
        return st;
    if (a->kv_heads && (st = check_heads(a->k, a->k_token_stride, a->k_head_stride)) != SBVR_OK)
        return st;
    if (a->kv_heads && !cache &&
        (st = check_heads_out(a->k_out, a->k_out_token_stride, a->k_out_head_stride, a->T, a->kv_heads, a->head_dim, a->k,
                              a->k_token_stride, a->k_head_stride)) != SBVR_OK)
        return st;
    if (!aligned(a->positions, 4) || !aligned(a->frequencies, 4) || !aligned(a->pair_axis, 4))
        return SBVR_E_ALIGNMENT;
    return SBVR_OK;
}

int check_beam_shape(int R, int B, int V, int n, int n_end)
{
    if (R < 0 || B < 1 || V < 1 || n < 1 || n_end < 0)
        return SBVR_E_INVALID_ARG;
    if (B > SBVR_BEAMS_MAX || V > (1 << 30) || (int64_t)n + n_end > SBVR_BEAM_KEEP_MAX || (int64_t)R * B > (1 << 16) - 1)
        return SBVR_E_UNSUPPORTED;
    return SBVR_OK;
}

int check_table_shape(int R, int max_pages, int64_t table_stride, int page_size)
{
    if (R < 0 || max_pages < 1 || table_stride < max_pages || !stride_ok(table_stride) ||
        check_page_size(page_size) != SBVR_OK)
        return SBVR_E_INVALID_ARG;
    return R > SBVR_REQUESTS_MAX || max_pages > SBVR_POOL_MAX ? SBVR_E_UNSUPPORTED : SBVR_OK;
}

int check_pool(int n_pages)
{
    return n_pages < 1 ? SBVR_E_INVALID_ARG : n_pages > SBVR_POOL_MAX ? SBVR_E_UNSUPPORTED : SBVR_OK;
}

bool alike(const sbvr_kv_cache &a, const sbvr_kv_cache &b)
{
    return a.k_page_stride == b.k_page_stride && a.k_token_stride == b.k_token_stride &&
           a.k_head_stride == b.k_head_stride && a.v_page_stride == b.v_page_stride &&
           a.v_token_stride == b.v_token_stride && a.v_head_stride == b.v_head_stride && a.n_pages == b.n_pages &&
           a.page_size == b.page_size && a.kv_heads == b.kv_heads && a.head_dim == b.head_dim && a.dtype == b.dtype;
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

int sbvr_rotary(const sbvr_rotary_args *a, hipStream_t stream)
{
    const int st = check_rotary(a, nullptr);
    if (st != SBVR_OK || a->T == 0)
        return st;
    RotaryArgs args = {};
    args.r = *a;
    return launch_rotary(args, stream);
}

int sbvr_rotary_write(const sbvr_rotary_args *a, const sbvr_kv_cache *cache, const void *v, int64_t v_token_stride,
                      int64_t v_head_stride, const int64_t *slots, hipStream_t stream)
{
    int st = check_cache(cache);
    if (st != SBVR_OK || (st = check_rotary(a, cache)) != SBVR_OK)
        return st;
    if (a->T == 0)
        return SBVR_OK;
    if ((st = check_heads(v, v_token_stride, v_head_stride)) != SBVR_OK)
        return st;
    if (!slots)
        return SBVR_E_INVALID_ARG;
    if (!aligned(slots, 8))
        return SBVR_E_ALIGNMENT;
    return launch_rotary(RotaryArgs{*a, *cache, v, v_token_stride, v_head_stride, slots}, stream);
}

size_t sbvr_beam_select_workspace_bytes(int R, int B, int V, int n, int n_end)
{
    return check_beam_shape(R, B, V, n, n_end) == SBVR_OK ? beam_workspace_bytes(R, B, V, n, n_end) : 0;
}

int sbvr_beam_select(const sbvr_beam_args *a, void *workspace, size_t ws_bytes, hipStream_t stream)
{
    if (!a || a->dtype < SBVR_F16 || a->dtype > SBVR_F32 || !stride_ok(a->logits_stride))
        return SBVR_E_INVALID_ARG;
    const int st = check_beam_shape(a->R, a->B, a->V, a->n, a->n_end);
    if (st != SBVR_OK || a->R == 0)
        return st;
    if (!a->logits || !a->scores || !a->tokens || !a->parents || !a->scores_out || !a->ended || !a->ended_tokens ||
        (a->n_end && !a->end_tokens))
        return SBVR_E_INVALID_ARG;
    if (ws_bytes < beam_workspace_bytes(a->R, a->B, a->V, a->n, a->n_end) || !workspace)
        return SBVR_E_WORKSPACE;
    const void *words[] = {a->scores, a->end_tokens, a->tokens, a->parents, a->scores_out, a->ended, a->ended_tokens};
    for (const void *p : words)
        if (!aligned(p, 4))
            return SBVR_E_ALIGNMENT;
    if (!aligned(a->logits, a->dtype == SBVR_F32 ? 4 : 2) || !aligned(workspace, 16))
        return SBVR_E_ALIGNMENT;
    if (a->scores_out == a->scores && a->n != a->B)  // in place, one request's would lie on another's
        return SBVR_E_INVALID_ARG;
    return launch_beam(*a, workspace, stream);
}

size_t sbvr_page_usage_workspace_bytes(int R, int max_pages, int n_pages)
{
    return check_table_shape(R, max_pages, max_pages, 16) == SBVR_OK && check_pool(n_pages) == SBVR_OK
               ? usage_workspace_bytes(R, max_pages, n_pages)
               : 0;
}

int sbvr_page_usage(int R, int page_size, int n_pages, const int32_t *context_lens, const int32_t *page_table,
                    int max_pages, int64_t table_stride, int32_t *refs, int32_t *free_pages, int32_t *counts,
                    void *workspace, size_t ws_bytes, hipStream_t stream)
{
    int st = check_table_shape(R, max_pages, table_stride, page_size);
    if (st != SBVR_OK || (st = check_pool(n_pages)) != SBVR_OK)
        return st;
    if ((R && (!context_lens || !page_table)) || !refs || !free_pages || !counts)
        return SBVR_E_INVALID_ARG;
    if (ws_bytes < usage_workspace_bytes(R, max_pages, n_pages) || !workspace)
        return SBVR_E_WORKSPACE;
    if (!aligned(context_lens, 4) || !aligned(page_table, 4) || !aligned(refs, 4) || !aligned(free_pages, 4) ||
        !aligned(counts, 4) || !aligned(workspace, 16))
        return SBVR_E_ALIGNMENT;
    const PageTable t{R, __builtin_ctz(page_size), max_pages, context_lens, page_table, table_stride};
    return launch_usage(UsageArgs{t, n_pages, refs, free_pages, counts, (int32_t *)workspace, nullptr}, stream);
}

int sbvr_page_fork(int groups, int rows_in, int rows_out, int page_size, const int32_t *context_lens,
                   const int32_t *page_table, int max_pages, int64_t table_stride, const int32_t *parents,
                   const int32_t *free_pages, int n_free, const int32_t *taken, int32_t *out_table,
                   int64_t out_stride, int32_t *out_lens, int32_t *src, int32_t *dst, int32_t *tokens, int32_t *used,
                   hipStream_t stream)
{
    if (groups < 0 || rows_in < 0 || rows_out < 0 || n_free < 0 || (groups == 0 && (rows_in || rows_out)))
        return SBVR_E_INVALID_ARG;
    groups = groups > 0 ? groups : 1;  // no groups: no rows
    if (rows_in % groups || rows_out % groups)
        return SBVR_E_INVALID_ARG;
    int st = check_table_shape(rows_in, max_pages, table_stride, page_size);
    if (st != SBVR_OK || (st = check_table_shape(rows_out, max_pages, out_stride, page_size)) != SBVR_OK)
        return st;
    if ((rows_in && (!context_lens || !page_table)) || (n_free && !free_pages) || !used ||
        (rows_out && (!parents || !out_table || !out_lens || !src || !dst || !tokens)))
        return SBVR_E_INVALID_ARG;
    const void *words[] = {context_lens, page_table, parents, free_pages, taken, out_table, out_lens, src, dst, tokens,
                           used};
    for (const void *p : words)
        if (!aligned(p, 4))
            return SBVR_E_ALIGNMENT;
    // one workgroup writes the lengths and lists while others read what they come from
    const void *read[] = {rows_in ? context_lens : nullptr, rows_in ? page_table : nullptr, rows_out ? parents : nullptr,
                          n_free ? free_pages : nullptr, taken};
    const void *written[] = {out_table, out_lens, src, dst, tokens};
    for (const void *p : read) {
        if (p && p == used)
            return SBVR_E_INVALID_ARG;
        for (const void *q : written)
            if (p && p == q && rows_out)
                return SBVR_E_INVALID_ARG;
    }
    const PageTable t{rows_in, __builtin_ctz(page_size), max_pages, context_lens, page_table, table_stride};
    const ForkArgs a{t, rows_out, rows_in / groups, rows_out / groups > 0 ? rows_out / groups : 1, n_free, parents,
                     free_pages, taken, out_table, out_stride, out_lens, src, dst, tokens, used};
    return launch_fork(a, stream);
}

size_t sbvr_page_compact_workspace_bytes(int R, int max_pages, int n_pages)
{
    return check_table_shape(R, max_pages, max_pages, 16) == SBVR_OK && check_pool(n_pages) == SBVR_OK
               ? compact_workspace_bytes(n_pages)
               : 0;
}

int sbvr_page_compact(int R, int page_size, int n_pages, const int32_t *context_lens, const int32_t *page_table,
                      int max_pages, int64_t table_stride, int32_t *out_table, int64_t out_stride, int32_t *src,
                      int32_t *dst, int32_t *counts, void *workspace, size_t ws_bytes, hipStream_t stream)
{
    int st = check_table_shape(R, max_pages, table_stride, page_size);
    if (st != SBVR_OK || (st = check_table_shape(R, max_pages, out_stride, page_size)) != SBVR_OK ||
        (st = check_pool(n_pages)) != SBVR_OK)
        return st;
    if ((R && (!context_lens || !page_table || !out_table)) || (n_pages > 1 && (!src || !dst)) || !counts ||
        (R > 1 && out_table == page_table && out_stride != table_stride))
        return SBVR_E_INVALID_ARG;
    if (ws_bytes < compact_workspace_bytes(n_pages) || !workspace)
        return SBVR_E_WORKSPACE;
    const void *words[] = {context_lens, page_table, out_table, src, dst, counts};
    for (const void *p : words)
        if (!aligned(p, 4))
            return SBVR_E_ALIGNMENT;
    if (!aligned(workspace, 16))
        return SBVR_E_ALIGNMENT;
    const PageTable t{R, __builtin_ctz(page_size), max_pages, context_lens, page_table, table_stride};
    return launch_compact(CompactArgs{t, n_pages, out_table, out_stride, src, dst, counts, (uint32_t *)workspace, nullptr},
                          stream);
}

int sbvr_page_copy(const sbvr_kv_cache *caches, int n_caches, int n, const int32_t *src, const int32_t *dst,
                   const int32_t *tokens, hipStream_t stream)
{
    if (!caches || n_caches < 1 || n < 0)
        return SBVR_E_INVALID_ARG;
    for (int i = 0; i < n_caches; ++i) {
        const int st = check_cache(&caches[i]);
        if (st != SBVR_OK)
            return st;
        if (!alike(caches[0], caches[i]))
            return SBVR_E_INVALID_ARG;
    }
    if (n == 0)
        return SBVR_OK;
    if (!src || !dst)
        return SBVR_E_INVALID_ARG;
    if (!aligned(src, 4) || !aligned(dst, 4) || !aligned(tokens, 4))
        return SBVR_E_ALIGNMENT;
    return launch_page_copy(caches, n_caches, n, src, dst, tokens, stream);
}

}  // extern "C"
