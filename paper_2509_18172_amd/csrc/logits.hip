// Adjustment of logits before sampling: penalties for tokens that occurred,
// biases, temperature and a grammar's mask, one pass over the logits.
//
// A workgroup takes a tile of the vocabulary for one row.  It counts the row's
// history (prompt, generated tokens, drafted path) and finds the biases that
// fall in the tile with integer LDS atomics -- sums and maxima, so their order
// does not matter -- and then streams the tile once, memory-bound.  The history
// is short against the vocabulary, and its re-reading by a row's tiles comes
// from L2.
#include "step.h"

namespace sbvr {

constexpr uint32_t IN_PROMPT = 1u << 31;  // beside the count of generated tokens

// N elements, at any alignment of T
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Loose {
    T e[N];
};

// f(i, ids[i]) for i0 <= i < i1 over a workgroup, AHEAD pieces of four a thread
// at a time; past the end f gets the id -1.
template <int THREADS, int AHEAD, typename F>
__device__ __forceinline__ void each_id(const int32_t *ids, int i0, int i1, F f)
{
    constexpr int STEP = 4 * THREADS;
    for (int base = i0; base < i1; base += AHEAD * STEP) {
        Loose<int32_t, 4> p[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int i = base + k * STEP + 4 * (int)threadIdx.x;
            if (i + 4 <= i1)
                p[k] = *(const Loose<int32_t, 4> *)(ids + i);
            else
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    p[k].e[e] = i + e < i1 ? ids[i + e] : -1;
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                f(base + k * STEP + 4 * (int)threadIdx.x + e, p[k].e[e]);
    }
}

template <typename T, typename O, int TILE, int THREADS>
__global__ void __launch_bounds__(THREADS) logits_kernel(sbvr_logits_args a)
{
    constexpr int PIECES = TILE / (8 * THREADS);
    __shared__ __attribute__((aligned(16))) uint32_t count[TILE];
    __shared__ __attribute__((aligned(16))) uint32_t bias_at[TILE];  // 1 + index of the token's last bias, 0: none
    const long long t = blockIdx.y;
    const int v0 = blockIdx.x * TILE, n = min(TILE, a.V - v0);
    const T *in = (const T *)a.logits + t * a.logits_stride + v0;
    O *out = (O *)a.out + t * a.out_stride + v0;
    const int r = a.token_request ? a.token_request[t] : (int)t;
    Loose<T, 8> l[PIECES];
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
        const int i = (k * THREADS + (int)threadIdx.x) * 8;
        if (i + 8 <= n)
            l[k] = *(const Loose<T, 8> *)(in + i);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e)
                l[k].e[e] = i + e < n ? in[i + e] : (T)0.f;
    }

    // everything of the row that a later load depends on is asked for now
    const bool adjust = r >= 0 && r < a.R;
    const bool counted = adjust && (a.history || a.draft_tokens), biased = adjust && a.bias_tokens;
    const int row = adjust ? r : 0;
    const int h0 = a.history ? a.history_start[row] : 0, h1 = a.history ? a.history_start[row + 1] : 0;
    const int b0 = a.bias_tokens ? a.bias_start[row] : 0, b1 = a.bias_tokens ? a.bias_start[row + 1] : 0;
    const int prompt = a.prompt_lens ? a.prompt_lens[row] : 0;
    const uint64_t path = a.draft_tokens ? a.tree_mask[t] : 0;
    const long long node = a.draft_tokens ? (long long)a.query_start[row] + threadIdx.x : 0;
    const int g = a.grammar && a.grammar_rows ? a.grammar_rows[t] : (int)t;
    const float rep = adjust && a.repetition ? a.repetition[row] : 1.f;
    const float freq = adjust && a.frequency ? a.frequency[row] : 0.f;
    const float pres = adjust && a.presence ? a.presence[row] : 0.f;
    const float temp = adjust && a.temperature ? a.temperature[row] : 1.f;
    uint32_t allowed[PIECES];
    const bool constrained = adjust && a.grammar && g >= 0 && g < a.grammar_count;
    const uint8_t *grammar = (const uint8_t *)(a.grammar + (constrained ? g : 0) * a.grammar_stride) + v0 / 8;
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
        const int i = (k * THREADS + (int)threadIdx.x) * 8;
        allowed[k] = constrained && i < n ? grammar[i / 8] : 0xffu;
    }

    if (counted || biased) {
#pragma unroll
        for (int k = 0; k < TILE / 4 / THREADS; ++k) {
            const int i = 4 * (k * THREADS + (int)threadIdx.x);
            *(uint4 *)&count[i] = uint4{0, 0, 0, 0};
            *(uint4 *)&bias_at[i] = uint4{0, 0, 0, 0};
        }
        __syncthreads();
        // An id below v0 or negative is a large d (v0 is at most 2^30), as is the
        // -1 past the end.
        if (counted) {
            each_id<THREADS, 4>(a.history, h0, h1, [&](int i, int id) {
                const uint32_t d = (uint32_t)(id - v0);
                if (d < (uint32_t)n) {
                    if (i - h0 < prompt)
                        atomicOr(&count[d], IN_PROMPT);
                    else
                        atomicAdd(&count[d], 1u);
                }
            });
            if (threadIdx.x < SBVR_TREE_MAX && ((path >> threadIdx.x) & 1) && node >= 0 && node < a.T) {
                const uint32_t d = (uint32_t)(a.draft_tokens[node] - v0);
                if (d < (uint32_t)n)
                    atomicAdd(&count[d], 1u);
            }
        }
        if (biased)
            each_id<THREADS, 1>(a.bias_tokens, b0, b1, [&](int i, int id) {
                const uint32_t d = (uint32_t)(id - v0);
                if (d < (uint32_t)n)
                    atomicMax(&bias_at[d], (uint32_t)(i - b0) + 1u);
            });
        __syncthreads();
    }

    const float inv_rep = 1.f / rep, inv_temp = temp > 0.f ? 1.f / temp : 1.f;
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
        const int i = (k * THREADS + (int)threadIdx.x) * 8;
        if (i >= n)
            continue;
        uint32_t c[8] = {}, b[8] = {}, any_c = 0, any_b = 0;
        if (counted) {
            *(uint4 *)&c[0] = *(const uint4 *)&count[i];
            *(uint4 *)&c[4] = *(const uint4 *)&count[i + 4];
        }
        if (biased) {
            *(uint4 *)&b[0] = *(const uint4 *)&bias_at[i];
            *(uint4 *)&b[4] = *(const uint4 *)&bias_at[i + 4];
        }
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = (float)l[k].e[e];
            any_c |= c[e];
            any_b |= b[e];
        }
        if (any_c) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t times = c[e] & ~IN_PROMPT;
                const float y = x[e] * (x[e] > 0.f ? inv_rep : rep) - (freq * (float)times + (times ? pres : 0.f));
                x[e] = c[e] ? y : x[e];
            }
        }
        if (any_b) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (b[e])
                    x[e] += a.bias_values[b0 + (int)b[e] - 1];
        }
        Loose<O, 8> o;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            o.e[e] = (O)((allowed[k] >> e) & 1 ? x[e] * inv_temp : -INFINITY);
        if (i + 8 <= n)
            *(Loose<O, 8> *)(out + i) = o;
        else
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (i + e < n)
                    out[i + e] = o.e[e];
    }
}

template <typename T, typename O, int TILE, int THREADS>
int run_logits(const sbvr_logits_args &a, hipStream_t stream)
{
    sbvr_logits_args args = a;
    void *argv[] = {&args};
    return launch_kernel((const void *)logits_kernel<T, O, TILE, THREADS>, dim3((a.V + TILE - 1) / TILE, a.T),
                         dim3(THREADS), 0, stream, argv);
}

template <typename T, typename O>
int go_logits(const sbvr_logits_args &a, hipStream_t stream)
{
    // large tiles read the history less often; small ones where those would not
    // fill the chip twice
    if ((long long)a.T * ((a.V + 8191) / 8192) >= 512)
        return run_logits<T, O, 8192, 512>(a, stream);
    return run_logits<T, O, 2048, 256>(a, stream);
}

int launch_logits(const sbvr_logits_args &a, hipStream_t stream)
{
    const bool f32 = a.out_dtype == SBVR_F32;
    switch (a.dtype) {
    case SBVR_F16: return f32 ? go_logits<f16_t, float>(a, stream) : go_logits<f16_t, f16_t>(a, stream);
    case SBVR_BF16: return f32 ? go_logits<bf16_t, float>(a, stream) : go_logits<bf16_t, bf16_t>(a, stream);
    default: return go_logits<float, float>(a, stream);
    }
}

}  // namespace sbvr
