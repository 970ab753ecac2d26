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

constexpr int LOGITS_THREADS = 256;
constexpr uint32_t IN_PROMPT = 1u << 31;  // beside the count of generated tokens

// 8 elements, at any alignment of T
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Loose8 {
    T e[8];
};

template <typename T, typename O, int TILE>
__global__ void __launch_bounds__(LOGITS_THREADS) logits_kernel(sbvr_logits_args a)
{
    __shared__ uint32_t count[TILE];
    __shared__ uint32_t bias_at[TILE];  // 1 + index of the last bias of the token, 0: none
    const long long t = blockIdx.y;
    const int v0 = blockIdx.x * TILE, n = min(TILE, a.V - v0);
    const int r = a.token_request ? a.token_request[t] : (int)t;
    const bool adjust = r >= 0 && r < a.R;
    const bool counted = adjust && (a.history || a.draft_tokens), biased = adjust && a.bias_tokens;

    if (counted || biased) {
        for (int i = threadIdx.x; i < TILE; i += LOGITS_THREADS) {
            count[i] = 0;
            bias_at[i] = 0;
        }
        __syncthreads();
        if (counted && a.history) {
            const int h0 = a.history_start[r], h1 = a.history_start[r + 1];
            const int prompt = a.prompt_lens ? a.prompt_lens[r] : 0;
            for (int i = h0 + threadIdx.x; i < h1; i += LOGITS_THREADS) {
                const uint32_t d = (uint32_t)(a.history[i] - v0);
                if (d < (uint32_t)n) {
                    if (i - h0 < prompt)
                        atomicOr(&count[d], IN_PROMPT);
                    else
                        atomicAdd(&count[d], 1u);
                }
            }
        }
        if (counted && a.draft_tokens && threadIdx.x < SBVR_TREE_MAX && ((a.tree_mask[t] >> threadIdx.x) & 1)) {
            const long long node = (long long)a.query_start[r] + threadIdx.x;
            if (node >= 0 && node < a.T) {
                const uint32_t d = (uint32_t)(a.draft_tokens[node] - v0);
                if (d < (uint32_t)n)
                    atomicAdd(&count[d], 1u);
            }
        }
        if (biased) {
            const int b0 = a.bias_start[r], b1 = a.bias_start[r + 1];
            for (int i = b0 + threadIdx.x; i < b1; i += LOGITS_THREADS) {
                const uint32_t d = (uint32_t)(a.bias_tokens[i] - v0);
                if (d < (uint32_t)n)
                    atomicMax(&bias_at[d], (uint32_t)(i - b0) + 1u);
            }
        }
        __syncthreads();
    }

    const float rep = adjust && a.repetition ? a.repetition[r] : 1.f;
    const float freq = adjust && a.frequency ? a.frequency[r] : 0.f;
    const float pres = adjust && a.presence ? a.presence[r] : 0.f;
    const float temp = adjust && a.temperature ? a.temperature[r] : 1.f;
    const float inv_temp = temp > 0.f ? 1.f / temp : 1.f;
    const float *bias = biased ? a.bias_values + a.bias_start[r] : nullptr;
    const uint8_t *grammar = nullptr;
    if (adjust && a.grammar) {
        const int g = a.grammar_rows ? a.grammar_rows[t] : (int)t;
        if (g >= 0 && g < a.grammar_count)
            grammar = (const uint8_t *)(a.grammar + g * a.grammar_stride) + v0 / 8;
    }
    const T *in = (const T *)a.logits + t * a.logits_stride + v0;
    O *out = (O *)a.out + t * a.out_stride + v0;

    auto one = [&](float l, int i) {
        if (counted) {
            const uint32_t c = count[i];
            if (c) {
                l = l > 0.f ? l / rep : l * rep;
                const uint32_t times = c & ~IN_PROMPT;
                l -= freq * (float)times + (times ? pres : 0.f);
            }
        }
        if (biased) {
            const uint32_t b = bias_at[i];
            if (b)
                l += bias[b - 1];
        }
        return l * inv_temp;
    };
    for (int i = threadIdx.x * 8; i < n; i += LOGITS_THREADS * 8) {
        const uint32_t allowed = grammar ? grammar[i / 8] : 0xffu;
        if (i + 8 <= n) {
            const Loose8<T> l = *(const Loose8<T> *)(in + i);
            Loose8<O> o;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                o.e[e] = (O)((allowed >> e) & 1 ? one((float)l.e[e], i + e) : -INFINITY);
            *(Loose8<O> *)(out + i) = o;
        } else {
            for (int e = 0; e < n - i; ++e)
                out[i + e] = (O)((allowed >> e) & 1 ? one((float)in[i + e], i + e) : -INFINITY);
        }
    }
}

template <typename T, typename O>
int go_logits(const sbvr_logits_args &a, hipStream_t stream)
{
    sbvr_logits_args args = a;
    void *argv[] = {&args};
    constexpr int TILE = 4096;
    return launch_kernel((const void *)logits_kernel<T, O, TILE>, dim3((a.V + TILE - 1) / TILE, a.T),
                         dim3(LOGITS_THREADS), 0, stream, argv);
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
