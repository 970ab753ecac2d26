// Adjustment of logits before sampling: penalties for tokens that occurred,
// biases, temperature and a grammar's mask, one pass over the logits.
//
// A workgroup takes tiles of the vocabulary for one row, one after the other.
// For each it counts the row's history (prompt, generated tokens, drafted path)
// and finds the biases that fall in the tile with integer LDS atomics -- sums,
// ors and maxima, so their order does not matter -- and then streams the tile
// once, memory-bound; a thread clears the entries that it has used.  What a row
// needs is loaded once, 4096 tokens of the history stay in registers from tile to
// tile (a longer one is read again, from L2), and a tile's logits are loaded while
// the one before is stored.  (With a workgroup per tile the chain of loads before
// the counting bound the kernel: 256 rows of 131072 took 63 us.)
//
// Measured in a graph, binary16 to binary32: 256 rows of 131072 with histories of
// 4000 50 us, 4.0 TB/s read and written (a copy of as many bytes 41 us; the rest is
// the counting, between whose barriers nothing is stored); one row of 50001 5.5 us,
// the latency of its chain: row, history, counts, logits.
#include "step.h"

namespace sbvr {

constexpr uint32_t IN_PROMPT = 1u << 31;  // beside the count of generated tokens

// ids[i0 ..] of a thread: K pieces of four, -1 past i1.
template <int THREADS, int K>
__device__ __forceinline__ void load_ids(const int32_t *ids, int i0, int i1, Loose<int32_t, 4> (&p)[K])
{
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = i0 + 4 * (k * THREADS + (int)threadIdx.x);
        if (i + 4 <= i1)
            p[k] = *(const Loose<int32_t, 4> *)(ids + i);
        else
#pragma unroll
            for (int e = 0; e < 4; ++e)
                p[k].e[e] = i + e < i1 ? ids[i + e] : -1;
    }
}

template <int THREADS, int K, typename F>
__device__ __forceinline__ void each_id(const Loose<int32_t, 4> (&p)[K], int i0, F f)
{
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            f(i0 + 4 * (k * THREADS + (int)threadIdx.x) + e, p[k].e[e]);
}

// tiles of 8 THREADS tokens, `per` of them a workgroup
template <typename T, typename O, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 1024 ? 2 : 1) logits_kernel(sbvr_logits_args a, int per)
{
    constexpr int TILE = 8 * THREADS, HELD = 1024 / THREADS, STEP = 4 * THREADS * HELD;
    __shared__ __attribute__((aligned(16))) uint32_t count[TILE];
    __shared__ __attribute__((aligned(16))) uint32_t bias_at[TILE];  // 1 + index of the token's last bias, 0: none
    const long long t = blockIdx.y;
    const int first = blockIdx.x * per * TILE, last = (int)min((long long)first + (long long)per * TILE, (long long)a.V);
    const int i = 8 * (int)threadIdx.x;
    const T *in = (const T *)a.logits + t * a.logits_stride;
    O *out = (O *)a.out + t * a.out_stride;
    const int r = a.token_request ? uniform_load(a.token_request + t) : (int)t;
    const bool adjust = r >= 0 && r < a.R;
    const bool counted = adjust && (a.history || a.draft_tokens), biased = adjust && a.bias_tokens;
    const int row = adjust ? r : 0;
    const int h0 = a.history ? uniform_load(a.history_start + row) : 0;
    const int h1 = a.history && adjust ? uniform_load(a.history_start + row + 1) : h0;
    const int b0 = a.bias_tokens ? uniform_load(a.bias_start + row) : 0;
    const int b1 = biased ? uniform_load(a.bias_start + row + 1) : b0;
    const int prompt = a.prompt_lens ? uniform_load(a.prompt_lens + row) : 0;
    const uint64_t path = a.draft_tokens && adjust ? uniform_load(a.tree_mask + t) : 0;
    const long long node = a.draft_tokens ? (long long)uniform_load(a.query_start + row) + threadIdx.x : 0;
    const int g = a.grammar && a.grammar_rows ? uniform_load(a.grammar_rows + t) : (int)t;
    const float rep = adjust && a.repetition ? uniform_load(a.repetition + row) : 1.f;
    const float freq = adjust && a.frequency ? uniform_load(a.frequency + row) : 0.f;
    const float pres = adjust && a.presence ? uniform_load(a.presence + row) : 0.f;
    const float temp = adjust && a.temperature ? uniform_load(a.temperature + row) : 1.f;
    const float inv_rep = 1.f / rep, inv_temp = temp > 0.f ? 1.f / temp : 1.f;
    const bool constrained = adjust && a.grammar && g >= 0 && g < a.grammar_count;
    const uint8_t *grammar = constrained ? (const uint8_t *)(a.grammar + g * a.grammar_stride) : nullptr;
    // A tile is loaded without a branch, so that the compiler counts what it
    // waits for: a piece that would pass the row's end is moved back to end with
    // it, and its elements are moved to their places later (a byte of the row is
    // loaded for a grammar that is not there).
    const bool wide = a.V >= 8;
    Words<T> coming = {};
    uint32_t coming_allowed = 0;
    auto load = [&](int v) {
        coming = load_words(in + min(v + i, a.V - 8));
        coming_allowed = *(grammar ? grammar + min(v + i, a.V - 1) / 8 : (const uint8_t *)in);
    };
    if (wide)
        load(first);

    Loose<int32_t, 4> history[HELD], biases[1];
    int drafted = -1;
    if (counted) {
        load_ids<THREADS>(a.history, h0, h1, history);
        if (threadIdx.x < SBVR_TREE_MAX && ((path >> threadIdx.x) & 1) && node >= 0 && node < a.T)
            drafted = a.draft_tokens[node];
    }
    if (biased)
        load_ids<THREADS>(a.bias_tokens, b0, b1, biases);
    if (counted || biased) {
        *(uint4 *)&count[i] = *(uint4 *)&count[i + 4] = uint4{0, 0, 0, 0};
        *(uint4 *)&bias_at[i] = *(uint4 *)&bias_at[i + 4] = uint4{0, 0, 0, 0};
        __syncthreads();
    }

    // (waits for the ids here, so that no tile does)
    if (counted)
        each_id<THREADS>(history, 0, [](int, int id) { asm volatile("" ::"v"(id)); });
    if (biased)
        each_id<THREADS>(biases, 0, [](int, int id) { asm volatile("" ::"v"(id)); });
    for (int v0 = first; v0 < last; v0 += TILE) {
        const int n = min(TILE, last - v0);
        // An id below v0 or negative is a large d (v0 is at most 2^30), as is the
        // -1 past the end.
        if (counted) {
            auto occurs = [&](int k, int id) {
                const uint32_t d = (uint32_t)(id - v0);
                if (d < (uint32_t)n) {
                    if (k - h0 < prompt)
                        atomicOr(&count[d], IN_PROMPT);
                    else
                        atomicAdd(&count[d], 1u);
                }
            };
            each_id<THREADS>(history, h0, occurs);
            for (int k = h0 + STEP; k < h1; k += STEP) {
                Loose<int32_t, 4> more[HELD];
                load_ids<THREADS>(a.history, k, h1, more);
                each_id<THREADS>(more, k, occurs);
            }
            const uint32_t d = (uint32_t)(drafted - v0);
            if (d < (uint32_t)n)
                atomicAdd(&count[d], 1u);
        }
        if (biased) {
            auto bias = [&](int k, int id) {
                const uint32_t d = (uint32_t)(id - v0);
                if (d < (uint32_t)n)
                    atomicMax(&bias_at[d], (uint32_t)(k - b0) + 1u);
            };
            each_id<THREADS>(biases, b0, bias);
            for (int k = b0 + 4 * THREADS; k < b1; k += 4 * THREADS) {
                Loose<int32_t, 4> more[1];
                load_ids<THREADS>(a.bias_tokens, k, b1, more);
                each_id<THREADS>(more, k, bias);
            }
        }
        if (counted || biased)
            __syncthreads();
        if (!wide) {
            Loose<T, 8> l;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                l.e[e] = in[v0 + (i + e < n ? i + e : 0)];
            coming = to_words(l);
            coming_allowed = grammar ? grammar[(v0 + (i < n ? i : 0)) / 8] : 0;
            asm volatile("" : "+v"(coming), "+v"(coming_allowed));  // waited for here
        }
        float x[8];
        const uint32_t allowed = grammar ? coming_allowed : 0xffu;
        {
            const Loose<T, 8> l = from_words<T>(coming);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = (float)l.e[e];
        }
        if (n < TILE && wide) {
            const int back = v0 + i - min(v0 + i, a.V - 8);
#pragma unroll
            for (int by = 4; by; by /= 2)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[e] = back & by ? x[min(e + by, 7)] : x[e];
        }
        if (wide)
            load(v0 + TILE);

        if (counted || biased) {
            uint32_t c[8], b[8], any_c = 0, any_b = 0;
            *(uint4 *)&c[0] = *(const uint4 *)&count[i];
            *(uint4 *)&c[4] = *(const uint4 *)&count[i + 4];
            *(uint4 *)&b[0] = *(const uint4 *)&bias_at[i];
            *(uint4 *)&b[4] = *(const uint4 *)&bias_at[i + 4];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                any_c |= c[e];
                any_b |= b[e];
            }
            if (any_c) {
                *(uint4 *)&count[i] = *(uint4 *)&count[i + 4] = uint4{0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t times = c[e] & ~IN_PROMPT;
                    const float y = x[e] * (x[e] > 0.f ? inv_rep : rep) - (freq * (float)times + (times ? pres : 0.f));
                    x[e] = c[e] ? y : x[e];
                }
            }
            if (any_b) {
                *(uint4 *)&bias_at[i] = *(uint4 *)&bias_at[i + 4] = uint4{0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (b[e])
                        x[e] += a.bias_values[b0 + (int)b[e] - 1];
            }
        }
        Loose<O, 8> o;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            o.e[e] = (O)((allowed >> e) & 1 ? x[e] * inv_temp : -INFINITY);
        if (i + 8 <= n)
            store_words(out + v0 + i, to_words(o));
        else
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (i + e < n)
                    out[v0 + i + e] = o.e[e];
        if (counted || biased)
            __syncthreads();
    }
}

template <typename T, typename O, int THREADS>
int run_logits(const sbvr_logits_args &a, int per, hipStream_t stream)
{
    constexpr int TILE = 8 * THREADS;
    sbvr_logits_args args = a;
    void *argv[] = {&args, &per};
    const int tiles = (a.V + TILE - 1) / TILE;
    return launch_kernel((const void *)logits_kernel<T, O, THREADS>, dim3((tiles + per - 1) / per, a.T), dim3(THREADS), 0,
                         stream, argv);
}

template <typename T, typename O>
int go_logits(const sbvr_logits_args &a, hipStream_t stream)
{
    // Large tiles and several of them a workgroup, as far as the 512 workgroups
    // that the chip holds have work; small tiles where there is less.  Large and
    // small: 160 rows of 32000 (640 tiles) 22.5 and 17.7 us, 192 rows (768) 21.0 and
    // 20.3, 256 rows (1024) 22.0 and 24.8, 64 rows of 131072 (1024) 18.6 and 22.0.
    const int tiles = (a.V + 8191) / 8192;
    const long long all = (long long)a.T * tiles;
    if (all <= 768)
        return run_logits<T, O, 256>(a, 1, stream);
    const int ranges = (int)((tiles * 512ll + all - 1) / all);  // of a row
    return run_logits<T, O, 1024>(a, (tiles + ranges - 1) / ranges, stream);
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
