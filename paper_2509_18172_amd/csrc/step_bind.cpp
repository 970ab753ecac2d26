// The tensor helpers of the operators between the products of a step: argument
// checks, outputs and workspaces, and the C call (include/sbvr.h).  They are
// native because a step makes hundreds of these calls and each is a few
// microseconds on the GPU: from Python, over ctypes, a residual_norm took 10.7
// us of the host, a batch_plan 14.6.  The library's functions are handed over as
// addresses by the package, which has loaded it.
#include <c10/core/StreamGuard.h>
#include <torch/extension.h>

#include <string>

#include "sbvr.h"

namespace {

using at::Tensor;
using Maybe = std::optional<Tensor>;

struct Api {
    decltype(&sbvr_batch_plan) batch_plan;
    decltype(&sbvr_cache_write) cache_write;
    decltype(&sbvr_tree_attention_workspace_bytes) workspace_bytes;
    decltype(&sbvr_tree_attention) tree_attention;
    decltype(&sbvr_tree_attention_whole) tree_attention_whole;
    decltype(&sbvr_residual_norm) residual_norm;
    decltype(&sbvr_adjust_logits) adjust_logits;
    decltype(&sbvr_rotary) rotary;
    decltype(&sbvr_rotary_write) rotary_write;
    decltype(&sbvr_beam_select_workspace_bytes) beam_workspace_bytes;
    decltype(&sbvr_beam_select) beam_select;
    decltype(&sbvr_page_usage_workspace_bytes) usage_workspace_bytes;
    decltype(&sbvr_page_usage) page_usage;
    decltype(&sbvr_page_fork) page_fork;
    decltype(&sbvr_page_compact_workspace_bytes) compact_workspace_bytes;
    decltype(&sbvr_page_compact) page_compact;
    decltype(&sbvr_page_copy) page_copy;
} api;

// SBVRError, torch's query of a device's current stream and its change of the
// current device (which returns the one before); never released, as the
// interpreter may be gone before this module's statics are
py::handle status_error, current_stream, exchange_device;

[[noreturn]] void refuse(const std::string &what)
{
    PyErr_SetString(PyExc_AssertionError, what.c_str());
    throw py::error_already_set();
}

void require(bool ok, const char *what)
{
    if (!ok)
        refuse(what);
}

void check(int status, const char *call)
{
    if (status != SBVR_OK) {
        PyErr_SetObject(status_error.ptr(), py::make_tuple(status, call).ptr());
        throw py::error_already_set();
    }
}

// The GPU of a call's tensors as the current one, as long as the call lasts, and
// the stream of the call.  A default stream's handle is 0 on every GPU, and the
// runtime takes that for the current one's.  A given stream is torch's current one
// meanwhile, so that outputs and workspaces come from its memory: what another
// stream has just freed may still be in use there.
class Scope {
  public:
    Scope(const at::Device &device, const py::object &stream)
        : now(device.index()), before(exchange_device(now).cast<int>())
    {
        try {
            if (stream.is_none()) {
                raw = (hipStream_t)current_stream(now).cast<uintptr_t>();
            } else {
                const int index = stream.attr("device_index").cast<int>();
                require(index == now, "stream must be one of the tensors' GPU");
                raw = (hipStream_t)stream.attr("cuda_stream").cast<uintptr_t>();
                current.reset_stream(c10::Stream::unpack3(stream.attr("stream_id").cast<c10::StreamId>(),
                                                          (c10::DeviceIndex)index,
                                                          (c10::DeviceType)stream.attr("device_type").cast<int>()));
            }
        } catch (...) {
            leave();
            throw;
        }
    }
    ~Scope() { leave(); }
    Scope(const Scope &) = delete;
    Scope &operator=(const Scope &) = delete;
    hipStream_t stream() const { return raw; }

  private:
    void leave() noexcept
    {
        current.reset();
        if (before == now)
            return;
        try {
            exchange_device(before);
        } catch (py::error_already_set &e) {
            e.discard_as_unraisable("the current GPU");
        }
    }

    int now, before;
    hipStream_t raw;
    c10::OptionalStreamGuard current;
};

int dtype_of(const Tensor &t)
{
    switch (t.scalar_type()) {
    case at::kHalf: return SBVR_F16;
    case at::kBFloat16: return SBVR_BF16;
    case at::kFloat: return SBVR_F32;
    default: return -1;
    }
}

Tensor empty(at::IntArrayRef shape, at::ScalarType type, const at::Device &device)
{
    return at::empty(shape, at::TensorOptions().dtype(type).device(device));
}

std::string text(at::ScalarType type, at::IntArrayRef shape, const at::Device &device)
{
    std::string s = std::string(at::toString(type)) + " [";
    for (size_t i = 0; i < shape.size(); ++i)
        s += (i ? ", " : "") + std::to_string(shape[i]);
    return s + "] on " + device.str();
}

// The pointer of a contiguous tensor of one type and shape.
template <typename P = void>
P *dense(const Tensor &t, at::ScalarType type, at::IntArrayRef shape, const at::Device &device, const char *what)
{
    if (t.scalar_type() != type || t.sizes() != shape || !t.is_contiguous() || t.device() != device)
        refuse(std::string(what) + " must be a contiguous tensor " + text(type, shape, device));
    return (P *)t.data_ptr();
}

template <typename P = void>
P *dense(const Maybe &t, at::ScalarType type, at::IntArrayRef shape, const at::Device &device, const char *what)
{
    return t ? dense<P>(*t, type, shape, device, what) : nullptr;
}

// The same for a list: one dimension of any length.
template <typename P>
P *list(const Maybe &t, at::ScalarType type, const at::Device &device, const char *what)
{
    if (!t)
        return nullptr;
    require(t->dim() == 1, (std::string(what) + " must have one dimension").c_str());
    return dense<P>(*t, type, {t->size(0)}, device, what);
}

// The pointer and row stride of a 2-D tensor with contiguous rows.
struct RowsOf {
    void *p = nullptr;
    int64_t stride = 0;
};

RowsOf rows(const Tensor &t, at::ScalarType type, int64_t n, int64_t width, const at::Device &device, const char *what)
{
    if (t.scalar_type() != type || t.dim() != 2 || t.size(0) != n || t.size(1) != width || t.device() != device ||
        (t.stride(1) != 1 && width != 1))
        refuse(std::string(what) + " must be a tensor of contiguous rows, " + text(type, {n, width}, device));
    return {t.data_ptr(), t.stride(0)};
}

// The stride of rows that the library must find whole, one after the other: what
// the tensor says, which the library refuses where the rows overlap (an expanded
// view has 0).  A single row's means nothing, and torch may report a smaller one.
int64_t whole_rows(const Tensor &t, const RowsOf &r)
{
    return t.size(0) > 1 ? r.stride : std::max(r.stride, t.size(1));
}

int narrow(int64_t v, const char *what)
{
    require(v >= INT32_MIN && v <= INT32_MAX, what);
    return (int)v;
}

struct Table {
    int32_t *p;
    int pages;
    int64_t stride;
};

Table table_of(const Tensor &t, int64_t R, const at::Device &device)
{
    require(t.dim() == 2, "page_table must have two dimensions");
    const RowsOf r = rows(t, at::kInt, R, t.size(1), device, "page_table");
    return {(int32_t *)r.p, narrow(t.size(1), "page_table is too wide"), whole_rows(t, r)};
}

sbvr_kv_cache cache_of(const Tensor &k, const Tensor &v)
{
    require(k.dim() == 4 && k.sizes() == v.sizes() && k.scalar_type() == v.scalar_type() && k.is_cuda() &&
                k.device() == v.device(),
            "k and v must be alike, [pages][page_size][kv_heads][head_dim], on a GPU");
    require(k.stride(3) == 1 && v.stride(3) == 1, "a head's elements must be contiguous");
    return {k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), k.stride(2), v.stride(0), v.stride(1), v.stride(2),
            narrow(k.size(0), "too many pages"), narrow(k.size(1), "page_size is too large"),
            narrow(k.size(2), "too many heads"), narrow(k.size(3), "head_dim is too large"), dtype_of(k)};
}

// A [tokens][heads][head_dim] tensor that goes with a cache.
const void *heads_of(const Tensor &t, int64_t heads, const Tensor &k, const char *what)
{
    if (t.dim() != 3 || t.size(1) != heads || t.size(2) != k.size(3) || t.stride(2) != 1 ||
        t.scalar_type() != k.scalar_type() || t.device() != k.device())
        refuse(std::string(what) + " must have contiguous heads and be " +
               text(k.scalar_type(), {t.dim() ? t.size(0) : 0, heads, k.size(3)}, k.device()));
    return t.data_ptr();
}

py::tuple batch_plan(const Tensor &context_lens, const Tensor &new_lens, const Tensor &free_pages,
                     const Tensor &page_table, int64_t page_size, int64_t n_tokens, const Maybe &parents,
                     const std::optional<std::vector<Tensor>> &out, const py::object &stream)
{
    require(context_lens.is_cuda() && context_lens.dim() == 1, "context_lens must be a list on a GPU");
    const at::Device device = context_lens.device();
    const Scope scope(device, stream);
    const int64_t R = context_lens.size(0), T = n_tokens;
    const Table table = table_of(page_table, R, device);
    require(T >= 0, "n_tokens must not be negative");
    const auto i32 = at::kInt, i64 = at::kLong;
    std::vector<Tensor> o = out ? *out
                                : std::vector<Tensor>{empty({R + 1}, i32, device), empty({T}, i32, device),
                                                      empty({T}, i32, device), empty({T}, i64, device),
                                                      empty({T}, i64, device), empty({2}, i32, device)};
    check(api.batch_plan(narrow(R, "too many requests"), narrow(T, "too many tokens"),
                         narrow(page_size, "page_size is too large"),
                         dense<int32_t>(context_lens, i32, {R}, device, "context_lens"),
                         dense<int32_t>(new_lens, i32, {R}, device, "new_lens"),
                         list<int32_t>(free_pages, i32, device, "free_pages"),
                         narrow(free_pages.size(0), "too many pages"),
                         dense<int32_t>(parents, i32, {T}, device, "parents"), table.p, table.pages, table.stride,
                         dense<int32_t>(o[0], i32, {R + 1}, device, "query_start"),
                         dense<int32_t>(o[1], i32, {T}, device, "token_request"),
                         dense<int32_t>(o[2], i32, {T}, device, "positions"),
                         dense<int64_t>(o[3], i64, {T}, device, "slots"),
                         dense<uint64_t>(o[4], i64, {T}, device, "tree_mask"),
                         dense<int32_t>(o[5], i32, {2}, device, "used"), scope.stream()),
          "sbvr_batch_plan");
    return py::make_tuple(o[0], o[1], o[2], o[3], o[4], o[5]);
}

void cache_write(const Tensor &k_cache, const Tensor &v_cache, const Tensor &k, const Tensor &v, const Tensor &slots,
                 const py::object &stream)
{
    const sbvr_kv_cache cache = cache_of(k_cache, v_cache);
    const at::Device device = k_cache.device();
    const Scope scope(device, stream);
    const void *kp = heads_of(k, cache.kv_heads, k_cache, "k"), *vp = heads_of(v, cache.kv_heads, k_cache, "v");
    const int64_t T = k.size(0);
    require(v.size(0) == T, "k and v must have the same tokens");
    check(api.cache_write(&cache, narrow(T, "too many tokens"), kp, k.stride(0), k.stride(1), vp, v.stride(0),
                          v.stride(1), dense<int64_t>(slots, at::kLong, {T}, device, "slots"), scope.stream()),
          "sbvr_cache_write");
}

Tensor tree_attention(const Tensor &q, const Tensor &k_cache, const Tensor &v_cache, const Tensor &page_table,
                      const Tensor &context_lens, const Tensor &query_start, const Tensor &tree_mask, int64_t max_new,
                      std::optional<double> scale, const Maybe &out, const Maybe &workspace, const py::object &stream)
{
    const sbvr_kv_cache cache = cache_of(k_cache, v_cache);
    const at::Device device = k_cache.device();
    const Scope scope(device, stream);
    require(q.dim() == 3 && context_lens.dim() == 1, "q must have three dimensions, context_lens one");
    const int64_t T = q.size(0), H = q.size(1), D = q.size(2), R = context_lens.size(0);
    const void *qp = heads_of(q, H, k_cache, "q");
    const Table table = table_of(page_table, R, device);
    const int r = narrow(R, "too many requests"), h = narrow(H, "too many heads"), n = narrow(max_new, "max_new");
    Tensor o = out ? *out : empty({T, H, D}, q.scalar_type(), device);
    void *op = dense(o, q.scalar_type(), {T, H, D}, device, "out");
    const size_t need = api.workspace_bytes(r, n, h, cache.kv_heads, cache.head_dim);
    Tensor ws;
    if (workspace) {
        list<void>(workspace, at::kByte, device, "workspace");
        ws = *workspace;
    } else if (need) {
        ws = empty({(int64_t)need}, at::kByte, device);
    }
    // a new output has no content that rows could keep
    const auto call = out ? api.tree_attention : api.tree_attention_whole;
    check(call(&cache, r, narrow(T, "too many tokens"), h, qp, q.stride(0), q.stride(1), table.p, table.pages,
               table.stride, dense<int32_t>(context_lens, at::kInt, {R}, device, "context_lens"),
               dense<int32_t>(query_start, at::kInt, {R + 1}, device, "query_start"),
               dense<uint64_t>(tree_mask, at::kLong, {T}, device, "tree_mask"), n,
               scale ? (float)*scale : 1.f / std::sqrt((float)D), op, ws.defined() ? ws.data_ptr() : nullptr,
               ws.defined() ? (size_t)ws.numel() : 0, scope.stream()),
          "sbvr_tree_attention");
    return o;
}

py::tuple residual_norm(const Tensor &x, const Maybe &y, const Maybe &post_weight, const Maybe &gate, double scale,
                        const Maybe &pre_weight, double eps, const Maybe &x_out, const Maybe &h_out,
                        const py::object &stream)
{
    require(x.dim() == 2 && x.is_cuda() && dtype_of(x) >= 0, "x must be a GPU tensor [tokens][width] of fp16, bf16 or fp32");
    const at::Device device = x.device();
    const Scope scope(device, stream);
    const int64_t T = x.size(0), H = x.size(1);
    const at::ScalarType xt = x.scalar_type(), type = (y ? *y : pre_weight ? *pre_weight : x).scalar_type();
    const RowsOf xr = rows(x, xt, T, H, device, "x");
    RowsOf yr, gr, xo, hr;
    Tensor x2, h;
    if (y) {
        yr = rows(*y, type, T, H, device, "y");
        if (gate && gate->dim() == 1)
            gr = {dense(*gate, type, {H}, device, "gate"), 0};
        else if (gate)
            gr = rows(*gate, type, T, H, device, "gate");
        x2 = x_out ? *x_out : empty({T, H}, xt, device);
        xo = rows(x2, xt, T, H, device, "x_out");
    } else {
        require(!post_weight && !gate && !x_out, "post_weight, gate and x_out need a y");
        require(pre_weight.has_value(), "nothing to compute: neither y nor pre_weight");
        x2 = x;
    }
    if (pre_weight) {
        h = h_out ? *h_out : empty({T, H}, type, device);
        hr = rows(h, type, T, H, device, "h_out");
    } else {
        require(!h_out, "an h needs a pre_weight");
    }
    Tensor typed = y ? *y : pre_weight ? *pre_weight : x;
    check(api.residual_norm(narrow(T, "too many tokens"), narrow(H, "too wide"), dtype_of(typed), dtype_of(x), xr.p,
                            xr.stride, yr.p, yr.stride, dense(post_weight, type, {H}, device, "post_weight"), gr.p,
                            gr.stride, (float)scale, dense(pre_weight, type, {H}, device, "pre_weight"), (float)eps, xo.p,
                            xo.stride, hr.p, hr.stride, scope.stream()),
          "sbvr_residual_norm");
    if (!h.defined())
        return py::make_tuple(x2, py::none());
    return py::make_tuple(x2, h);
}

Tensor adjust_logits(const Tensor &logits, const Maybe &history, const Maybe &history_start, const Maybe &prompt_lens,
                     const Maybe &repetition, const Maybe &frequency, const Maybe &presence, const Maybe &temperature,
                     const Maybe &bias_tokens, const Maybe &bias_values, const Maybe &bias_start, const Maybe &grammar,
                     const Maybe &grammar_rows, const Maybe &token_request, const Maybe &query_start,
                     const Maybe &tree_mask, const Maybe &draft_tokens, std::optional<int64_t> n_requests,
                     const Maybe &out, std::optional<at::ScalarType> out_dtype, const py::object &stream)
{
    require(logits.dim() == 2 && logits.is_cuda() && dtype_of(logits) >= 0,
            "logits must be a GPU tensor [rows][vocabulary] of fp16, bf16 or fp32");
    const at::Device device = logits.device();
    const Scope scope(device, stream);
    const int64_t T = logits.size(0), V = logits.size(1);
    require(!history == !history_start, "history and history_start go together");
    require(!bias_tokens == !bias_start && !bias_tokens == !bias_values, "the three bias tensors go together");
    int64_t R = std::max<int64_t>(T, 1);  // no rows: a request all the same
    if (n_requests) {
        R = *n_requests;
    } else {
        const Maybe *per_request[] = {&prompt_lens, &repetition, &frequency, &presence, &temperature};
        const Maybe *starts[] = {&history_start, &bias_start, &query_start};
        for (const Maybe *m : starts)
            if (*m && (*m)->dim() == 1)
                R = (*m)->size(0) - 1;
        for (const Maybe *m : per_request)
            if (*m && (*m)->dim() == 1)
                R = (*m)->size(0);
    }
    Tensor o = out ? *out : empty({T, V}, out_dtype.value_or(logits.scalar_type()), device);
    require(!out_dtype || o.scalar_type() == *out_dtype, "out must be of out_dtype");
    const RowsOf in = rows(logits, logits.scalar_type(), T, V, device, "logits");
    const RowsOf to = rows(o, o.scalar_type(), T, V, device, "out");
    RowsOf g;
    int64_t masks = 0;
    if (grammar) {
        require(grammar->dim() == 2, "grammar must have two dimensions");
        masks = grammar->size(0);
        g = rows(*grammar, at::kInt, masks, (V + 31) / 32, device, "grammar");
        g.stride = whole_rows(*grammar, g);
    }
    const auto i32 = at::kInt, f32 = at::kFloat;
    const int64_t n_bias = bias_tokens && bias_tokens->dim() == 1 ? bias_tokens->size(0) : 0;
    sbvr_logits_args a = {};
    a.R = narrow(R, "too many requests");
    a.T = narrow(T, "too many rows");
    a.V = narrow(V, "the vocabulary is too large");
    a.dtype = dtype_of(logits);
    a.out_dtype = dtype_of(o);
    a.logits = in.p;
    a.logits_stride = in.stride;
    a.out = to.p;
    a.out_stride = to.stride;
    a.token_request = dense<int32_t>(token_request, i32, {T}, device, "token_request");
    a.history = list<int32_t>(history, i32, device, "history");
    a.history_start = dense<int32_t>(history_start, i32, {R + 1}, device, "history_start");
    a.prompt_lens = dense<int32_t>(prompt_lens, i32, {R}, device, "prompt_lens");
    a.repetition = dense<float>(repetition, f32, {R}, device, "repetition");
    a.frequency = dense<float>(frequency, f32, {R}, device, "frequency");
    a.presence = dense<float>(presence, f32, {R}, device, "presence");
    a.temperature = dense<float>(temperature, f32, {R}, device, "temperature");
    a.bias_tokens = dense<int32_t>(bias_tokens, i32, {n_bias}, device, "bias_tokens");
    a.bias_start = dense<int32_t>(bias_start, i32, {R + 1}, device, "bias_start");
    a.bias_values = dense<float>(bias_values, f32, {n_bias}, device, "bias_values");
    a.grammar = (const uint32_t *)g.p;
    a.grammar_stride = g.stride;
    a.grammar_rows = dense<int32_t>(grammar_rows, i32, {T}, device, "grammar_rows");
    a.grammar_count = narrow(masks, "too many masks");
    a.draft_tokens = dense<int32_t>(draft_tokens, i32, {T}, device, "draft_tokens");
    a.query_start = dense<int32_t>(query_start, i32, {R + 1}, device, "query_start");
    a.tree_mask = dense<uint64_t>(tree_mask, at::kLong, {T}, device, "tree_mask");
    check(api.adjust_logits(&a, scope.stream()), "sbvr_adjust_logits");
    return o;
}

// A [tokens][heads][head_dim] tensor of a type, with contiguous heads.
struct HeadsOf {
    void *p = nullptr;
    int64_t token_stride = 0, head_stride = 0;
};

HeadsOf heads_like(const Tensor &t, const Tensor &model, const char *what)
{
    if (t.dim() != 3 || t.sizes() != model.sizes() || t.stride(2) != 1 || t.scalar_type() != model.scalar_type() ||
        t.device() != model.device())
        refuse(std::string(what) + " must have contiguous heads and be " +
               text(model.scalar_type(), model.sizes(), model.device()));
    return {t.data_ptr(), t.stride(0), t.stride(1)};
}

// What rotary and rotary_write have in common: everything but the outputs.
sbvr_rotary_args rotary_args(const Maybe &q, const Maybe &k, const Tensor &positions, const Tensor &frequencies,
                             const Maybe &axes, bool interleaved, bool inverse, const at::Device &device)
{
    const Tensor &x = q ? *q : *k;
    require(x.dim() == 3 && dtype_of(x) >= 0, "q and k must be [tokens][heads][head_dim] of fp16, bf16 or fp32");
    require(!q || !k || (k->dim() == 3 && k->size(0) == q->size(0) && k->size(2) == q->size(2) &&
                         k->scalar_type() == q->scalar_type()),
            "q and k must have the same tokens, head_dim and type");
    const int64_t T = x.size(0);
    sbvr_rotary_args a = {};
    a.T = narrow(T, "too many tokens");
    a.head_dim = narrow(x.size(2), "head_dim is too large");
    a.dtype = dtype_of(x);
    a.interleaved = interleaved;
    a.inverse = inverse;
    if (q) {
        const HeadsOf h = heads_like(*q, *q, "q");
        a.heads = narrow(q->size(1), "too many heads");
        a.q = h.p;
        a.q_token_stride = h.token_stride;
        a.q_head_stride = h.head_stride;
    }
    if (k) {
        const HeadsOf h = heads_like(*k, *k, "k");
        a.kv_heads = narrow(k->size(1), "too many heads");
        a.k = h.p;
        a.k_token_stride = h.token_stride;
        a.k_head_stride = h.head_stride;
        require(k->device() == device, "q and k must be on one GPU");
    }
    require(positions.dim() == 1 || positions.dim() == 2, "positions must be [tokens] or [axes][tokens]");
    if (positions.dim() == 1) {
        a.axes = 1;
        a.positions = dense<int32_t>(positions, at::kInt, {T}, device, "positions");
        a.position_stride = T;
    } else {
        const RowsOf r = rows(positions, at::kInt, positions.size(0), T, device, "positions");
        a.axes = narrow(positions.size(0), "too many axes");
        a.positions = (const int32_t *)r.p;
        a.position_stride = whole_rows(positions, r);
    }
    require(frequencies.dim() == 1, "frequencies must have one dimension");
    const int64_t n = frequencies.size(0);
    a.pairs = narrow(n, "too many frequencies");
    a.frequencies = dense<float>(frequencies, at::kFloat, {n}, device, "frequencies");
    a.pair_axis = dense<int32_t>(axes, at::kInt, {n}, device, "axes");
    return a;
}

Tensor rotated(const Tensor &x, const Maybe &out)
{
    return out ? *out : empty(x.sizes(), x.scalar_type(), x.device());
}

py::tuple rotary(const Maybe &q, const Maybe &k, const Tensor &positions, const Tensor &frequencies, const Maybe &axes,
                 bool interleaved, bool inverse, const Maybe &q_out, const Maybe &k_out, const py::object &stream)
{
    require(q || k, "neither q nor k");
    require((q || !q_out) && (k || !k_out), "an output needs its input");
    const at::Device device = (q ? *q : *k).device();
    require(device.is_cuda(), "q and k must be on a GPU");
    const Scope scope(device, stream);
    sbvr_rotary_args a = rotary_args(q, k, positions, frequencies, axes, interleaved, inverse, device);
    Tensor qo, ko;
    if (q) {
        qo = rotated(*q, q_out);
        const HeadsOf h = heads_like(qo, *q, "q_out");
        a.q_out = h.p;
        a.q_out_token_stride = h.token_stride;
        a.q_out_head_stride = h.head_stride;
    }
    if (k) {
        ko = rotated(*k, k_out);
        const HeadsOf h = heads_like(ko, *k, "k_out");
        a.k_out = h.p;
        a.k_out_token_stride = h.token_stride;
        a.k_out_head_stride = h.head_stride;
    }
    check(api.rotary(&a, scope.stream()), "sbvr_rotary");
    return py::make_tuple(q ? py::cast(qo) : py::none(), k ? py::cast(ko) : py::none());
}

py::object rotary_write(const Maybe &q, const Tensor &k_cache, const Tensor &v_cache, const Tensor &k, const Tensor &v,
                        const Tensor &slots, const Tensor &positions, const Tensor &frequencies, const Maybe &axes,
                        bool interleaved, bool inverse, const Maybe &q_out, const py::object &stream)
{
    const sbvr_kv_cache cache = cache_of(k_cache, v_cache);
    const at::Device device = k_cache.device();
    const Scope scope(device, stream);
    require(q || !q_out, "an output needs its input");
    heads_of(k, cache.kv_heads, k_cache, "k");
    const void *vp = heads_of(v, cache.kv_heads, k_cache, "v");
    require(v.size(0) == k.size(0), "k and v must have the same tokens");
    require(!q || q->device() == device, "q must be on the cache's GPU");
    sbvr_rotary_args a = rotary_args(q, k, positions, frequencies, axes, interleaved, inverse, device);
    Tensor qo;
    if (q) {
        qo = rotated(*q, q_out);
        const HeadsOf h = heads_like(qo, *q, "q_out");
        a.q_out = h.p;
        a.q_out_token_stride = h.token_stride;
        a.q_out_head_stride = h.head_stride;
    }
    check(api.rotary_write(&a, &cache, vp, v.stride(0), v.stride(1),
                           dense<int64_t>(slots, at::kLong, {k.size(0)}, device, "slots"), scope.stream()),
          "sbvr_rotary_write");
    return q ? py::cast(qo) : py::none();
}

// A given workspace, or a new one.
Tensor workspace_of(const Maybe &given, size_t need, const at::Device &device)
{
    if (given) {
        list<void>(given, at::kByte, device, "workspace");
        return *given;
    }
    return empty({(int64_t)need}, at::kByte, device);
}

py::tuple beam_select(const Tensor &logits, const Tensor &scores, std::optional<int64_t> n, const Maybe &end_tokens,
                      const std::optional<std::vector<Tensor>> &out, const Maybe &workspace, const py::object &stream)
{
    require(logits.dim() == 2 && logits.is_cuda() && dtype_of(logits) >= 0,
            "logits must be a GPU tensor [requests * beams][vocabulary] of fp16, bf16 or fp32");
    require(scores.dim() == 2, "scores must be [requests][beams]");
    const at::Device device = logits.device();
    const Scope scope(device, stream);
    const int64_t R = scores.size(0), B = scores.size(1), V = logits.size(1), N = n.value_or(B);
    const RowsOf in = rows(logits, logits.scalar_type(), R * B, V, device, "logits");
    const auto i32 = at::kInt, f32 = at::kFloat;
    require(N >= 0, "n must not be negative");
    std::vector<Tensor> o = out ? *out
                                : std::vector<Tensor>{empty({R, N}, i32, device), empty({R, N}, i32, device),
                                                      empty({R, N}, f32, device), empty({R, B}, f32, device),
                                                      empty({R, B}, i32, device)};
    sbvr_beam_args a = {};
    a.R = narrow(R, "too many requests");
    a.B = narrow(B, "too many beams");
    a.V = narrow(V, "the vocabulary is too large");
    a.n = narrow(N, "n is too large");
    a.dtype = dtype_of(logits);
    a.logits = in.p;
    a.logits_stride = in.stride;
    a.scores = dense<float>(scores, f32, {R, B}, device, "scores");
    a.end_tokens = list<int32_t>(end_tokens, i32, device, "end_tokens");
    a.n_end = end_tokens ? narrow(end_tokens->size(0), "too many end tokens") : 0;
    a.tokens = dense<int32_t>(o[0], i32, {R, N}, device, "tokens");
    a.parents = dense<int32_t>(o[1], i32, {R, N}, device, "parents");
    a.scores_out = dense<float>(o[2], f32, {R, N}, device, "scores of the output");
    a.ended = dense<float>(o[3], f32, {R, B}, device, "ended");
    a.ended_tokens = dense<int32_t>(o[4], i32, {R, B}, device, "ended_tokens");
    const Tensor ws = workspace_of(workspace, api.beam_workspace_bytes(a.R, a.B, a.V, a.n, a.n_end), device);
    check(api.beam_select(&a, ws.data_ptr(), (size_t)ws.numel(), scope.stream()), "sbvr_beam_select");
    return py::make_tuple(o[0], o[1], o[2], o[3], o[4]);
}

py::tuple page_usage(const Tensor &context_lens, const Tensor &page_table, int64_t page_size, int64_t n_pages,
                     const std::optional<std::vector<Tensor>> &out, const Maybe &workspace, const py::object &stream)
{
    require(context_lens.is_cuda() && context_lens.dim() == 1, "context_lens must be a list on a GPU");
    const at::Device device = context_lens.device();
    const Scope scope(device, stream);
    const int64_t R = context_lens.size(0);
    const Table table = table_of(page_table, R, device);
    require(n_pages >= 0, "n_pages must not be negative");
    const auto i32 = at::kInt;
    const int r = narrow(R, "too many rows"), pages = narrow(n_pages, "too many pages");
    std::vector<Tensor> o = out ? *out
                                : std::vector<Tensor>{empty({n_pages}, i32, device), empty({n_pages}, i32, device),
                                                      empty({2}, i32, device)};
    const Tensor ws = workspace_of(workspace, api.usage_workspace_bytes(r, table.pages, pages), device);
    check(api.page_usage(r, narrow(page_size, "page_size is too large"), pages,
                         dense<int32_t>(context_lens, i32, {R}, device, "context_lens"), table.p, table.pages,
                         table.stride, dense<int32_t>(o[0], i32, {n_pages}, device, "refs"),
                         dense<int32_t>(o[1], i32, {n_pages}, device, "free_pages"),
                         dense<int32_t>(o[2], i32, {2}, device, "counts"), ws.data_ptr(), (size_t)ws.numel(),
                         scope.stream()),
          "sbvr_page_usage");
    return py::make_tuple(o[0], o[1], o[2]);
}

py::tuple page_fork(const Tensor &context_lens, const Tensor &page_table, const Tensor &parents, int64_t page_size,
                    const Tensor &free_pages, const Maybe &taken, const std::optional<std::vector<Tensor>> &out,
                    const py::object &stream)
{
    require(context_lens.is_cuda() && context_lens.dim() == 1, "context_lens must be a list on a GPU");
    require(parents.dim() == 2, "parents must be [groups][rows of a group]");
    const at::Device device = context_lens.device();
    const Scope scope(device, stream);
    const int64_t G = parents.size(0), N = G * parents.size(1), R = context_lens.size(0);
    const Table table = table_of(page_table, R, device);
    const auto i32 = at::kInt;
    std::vector<Tensor> o = out ? *out
                                : std::vector<Tensor>{empty({N, table.pages}, i32, device), empty({N}, i32, device),
                                                      empty({N}, i32, device), empty({N}, i32, device),
                                                      empty({N}, i32, device), empty({1}, i32, device)};
    const RowsOf to = rows(o[0], i32, N, table.pages, device, "the new page_table");
    const int32_t *first = list<int32_t>(taken, i32, device, "taken");
    require(!taken || taken->size(0) >= 1, "taken must have an element");
    check(api.page_fork(narrow(G, "too many groups"), narrow(R, "too many rows"), narrow(N, "too many rows"),
                        narrow(page_size, "page_size is too large"),
                        dense<int32_t>(context_lens, i32, {R}, device, "context_lens"), table.p, table.pages,
                        table.stride, dense<int32_t>(parents, i32, parents.sizes(), device, "parents"),
                        list<int32_t>(free_pages, i32, device, "free_pages"),
                        narrow(free_pages.size(0), "too many pages"), first, (int32_t *)to.p, whole_rows(o[0], to),
                        dense<int32_t>(o[1], i32, {N}, device, "the new context_lens"),
                        dense<int32_t>(o[2], i32, {N}, device, "src"), dense<int32_t>(o[3], i32, {N}, device, "dst"),
                        dense<int32_t>(o[4], i32, {N}, device, "tokens"), dense<int32_t>(o[5], i32, {1}, device, "used"),
                        scope.stream()),
          "sbvr_page_fork");
    return py::make_tuple(o[0], o[1], o[2], o[3], o[4], o[5]);
}

py::tuple page_compact(const Tensor &context_lens, const Tensor &page_table, int64_t page_size, int64_t n_pages,
                       const std::optional<std::vector<Tensor>> &out, const Maybe &workspace, const py::object &stream)
{
    require(context_lens.is_cuda() && context_lens.dim() == 1, "context_lens must be a list on a GPU");
    const at::Device device = context_lens.device();
    const Scope scope(device, stream);
    const int64_t R = context_lens.size(0), moves = n_pages / 2;
    const Table table = table_of(page_table, R, device);
    require(n_pages >= 0, "n_pages must not be negative");
    const auto i32 = at::kInt;
    const int r = narrow(R, "too many rows"), pages = narrow(n_pages, "too many pages");
    std::vector<Tensor> o = out ? *out
                                : std::vector<Tensor>{empty({R, table.pages}, i32, device), empty({moves}, i32, device),
                                                      empty({moves}, i32, device), empty({2}, i32, device)};
    const RowsOf to = rows(o[0], i32, R, table.pages, device, "the new page_table");
    const Tensor ws = workspace_of(workspace, api.compact_workspace_bytes(r, table.pages, pages), device);
    check(api.page_compact(r, narrow(page_size, "page_size is too large"), pages,
                           dense<int32_t>(context_lens, i32, {R}, device, "context_lens"), table.p, table.pages,
                           table.stride, (int32_t *)to.p, whole_rows(o[0], to),
                           dense<int32_t>(o[1], i32, {moves}, device, "src"),
                           dense<int32_t>(o[2], i32, {moves}, device, "dst"),
                           dense<int32_t>(o[3], i32, {2}, device, "counts"), ws.data_ptr(), (size_t)ws.numel(),
                           scope.stream()),
          "sbvr_page_compact");
    return py::make_tuple(o[0], o[1], o[2], o[3]);
}

void page_copy(const std::vector<Tensor> &k_caches, const std::vector<Tensor> &v_caches, const Tensor &src,
               const Tensor &dst, const Maybe &tokens, const py::object &stream)
{
    require(!k_caches.empty() && k_caches.size() == v_caches.size(), "no caches");
    std::vector<sbvr_kv_cache> caches;
    for (size_t i = 0; i < k_caches.size(); ++i) {
        caches.push_back(cache_of(k_caches[i], v_caches[i]));
        require(k_caches[i].device() == k_caches[0].device(), "the caches must be on one GPU");
    }
    const at::Device device = k_caches[0].device();
    const Scope scope(device, stream);
    require(src.dim() == 1, "src must be a list");
    const int64_t n = src.size(0);
    check(api.page_copy(caches.data(), narrow((int64_t)caches.size(), "too many caches"), narrow(n, "too many copies"),
                        dense<int32_t>(src, at::kInt, {n}, device, "src"),
                        dense<int32_t>(dst, at::kInt, {n}, device, "dst"),
                        dense<int32_t>(tokens, at::kInt, {n}, device, "tokens"), scope.stream()),
          "sbvr_page_copy");
}

// The library's functions by name, the class of its errors, torch's query of a
// device's current stream and its change of the current device.
void connect(const std::map<std::string, uintptr_t> &address, const py::object &error, const py::object &stream,
             const py::object &device)
{
    api.batch_plan = (decltype(api.batch_plan))address.at("sbvr_batch_plan");
    api.cache_write = (decltype(api.cache_write))address.at("sbvr_cache_write");
    api.workspace_bytes = (decltype(api.workspace_bytes))address.at("sbvr_tree_attention_workspace_bytes");
    api.tree_attention = (decltype(api.tree_attention))address.at("sbvr_tree_attention");
    api.tree_attention_whole =
        (decltype(api.tree_attention_whole))address.at("sbvr_tree_attention_whole");
    api.residual_norm = (decltype(api.residual_norm))address.at("sbvr_residual_norm");
    api.adjust_logits = (decltype(api.adjust_logits))address.at("sbvr_adjust_logits");
    api.rotary = (decltype(api.rotary))address.at("sbvr_rotary");
    api.rotary_write = (decltype(api.rotary_write))address.at("sbvr_rotary_write");
    api.beam_workspace_bytes = (decltype(api.beam_workspace_bytes))address.at("sbvr_beam_select_workspace_bytes");
    api.beam_select = (decltype(api.beam_select))address.at("sbvr_beam_select");
    api.usage_workspace_bytes = (decltype(api.usage_workspace_bytes))address.at("sbvr_page_usage_workspace_bytes");
    api.page_usage = (decltype(api.page_usage))address.at("sbvr_page_usage");
    api.page_fork = (decltype(api.page_fork))address.at("sbvr_page_fork");
    api.compact_workspace_bytes =
        (decltype(api.compact_workspace_bytes))address.at("sbvr_page_compact_workspace_bytes");
    api.page_compact = (decltype(api.page_compact))address.at("sbvr_page_compact");
    api.page_copy = (decltype(api.page_copy))address.at("sbvr_page_copy");
    status_error = error;
    status_error.inc_ref();
    current_stream = stream;
    current_stream.inc_ref();
    exchange_device = device;
    exchange_device.inc_ref();
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m)
{
    m.def("connect", &connect);
    m.def("batch_plan", &batch_plan);
    m.def("cache_write", &cache_write);
    m.def("tree_attention", &tree_attention);
    m.def("residual_norm", &residual_norm);
    m.def("adjust_logits", &adjust_logits);
    m.def("rotary", &rotary);
    m.def("rotary_write", &rotary_write);
    m.def("beam_select", &beam_select);
    m.def("page_usage", &page_usage);
    m.def("page_fork", &page_fork);
    m.def("page_compact", &page_compact);
    m.def("page_copy", &page_copy);
}
