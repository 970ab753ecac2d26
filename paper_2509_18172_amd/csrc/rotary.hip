// Rotation of queries and keys by their positions, and the same with the cache
// write: (a, b) -> (a cos - b sin, b cos + a sin) for the pairs of every head.
//
// Memory-bound for many tokens, a latency for few.  A workgroup takes the work of
// some tokens, or a part of one's: pieces of eight pairs of a head (two loads and
// two stores of 16 bytes), and pieces of sixteen elements that are only copied (what
// lies behind the pairs, and the values).  The sine and cosine of a pair are the
// same in all heads, so they are computed once a workgroup, into LDS.  The angle's
// turn is taken in binary64: a binary32 product of position 100000 and a frequency
// is off by 4e-3, and one in 64 bits costs a few instructions a pair.
//
// Where the last piece would not be whole it is moved back to end with the pairs (or
// the head), and some elements are computed and written twice, alike (8192 tokens of
// 40 heads of 128 with 37 pairs: 41 us, 105 by elements).  In place that would turn
// them twice, so it is done by elements there (36 pairs of 80 elements 32 us, 21 out
// of place).  No piece is loaded by a lane that another lane stores, so the outputs
// may be the inputs.
//
// Measured: 16384 tokens of 72 heads of 128, three axes, 604 MB in 110 us (5.5 TB/s, above
// what a plain copy of 2 GiB reaches: 5.0); 8192 tokens with the cache write, 335 MB
// in 69 us (4.9); one token 3.0 us, of which an empty launch is 2.1.
#include "step.h"

namespace sbvr {

constexpr int ROTARY_THREADS = 256;
// As a cosine: a pair of no axis, whose elements are copied (cosine 1 and sine 0 would
// make NaN of one beside an infinity).
constexpr float STILL = 2.f;

struct RotaryShape {
    int turned, per_head, valued;  // pieces of a head that are turned, all of it, and of its values
    int units;                   // pieces of a token
    int split, tokens;           // pieces and tokens of a workgroup (split < units: one token)
    int width;                   // pairs rounded up to pieces
};

// The two elements of a pair turned: spelt out and in binary32, so that they are
// rounded alike however a piece is taken (the compiler would round some of them
// straight to 16 bits).
__device__ __forceinline__ float in_binary32(float v)
{
    asm("" : "+v"(v));
    return v;
}
__device__ __forceinline__ float turned_first(float a, float b, float c, float s)
{
    return in_binary32(__builtin_fmaf(a, c, -(b * s)));
}
__device__ __forceinline__ float turned_second(float a, float b, float c, float s)
{
    return in_binary32(__builtin_fmaf(b, c, a * s));
}

// T: element type; EVEN: every piece is whole (pairs a multiple of 8); WRITE: keys
// and values go into the cache; AXES: pairs have axes, or none (8192 tokens of 40 heads
// of 128 with 37 pairs, in the caches: 28.7 us, 30.1 if the kernel looks for pairs of no
// axis all the same; with three axes 29.2).
template <typename T, bool EVEN, bool WRITE, bool AXES>
__global__ void __launch_bounds__(ROTARY_THREADS) rotary_kernel(RotaryArgs args, RotaryShape s, int page_shift)
{
    extern __shared__ __attribute__((aligned(16))) float turn[];  // cosines, then sines, of [tokens][width]
    const sbvr_rotary_args &a = args.r;
    __shared__ int some_still;  // (the same for all tokens)
    if (AXES && threadIdx.x == 0)
        some_still = 0;
    const int n = a.pairs, heads = a.heads + a.kv_heads;
    float *cosine = turn, *sine = turn + s.tokens * s.width;
    for (long long t0 = (long long)blockIdx.x * s.tokens; t0 < a.T; t0 += (long long)gridDim.x * s.tokens) {
        const int tokens = (int)min((long long)s.tokens, a.T - t0);
        __syncthreads();
        for (int i = threadIdx.x; i < tokens * s.width; i += ROTARY_THREADS) {
            const int t = small_div(i, s.width, 1.f / (float)s.width), p = min(i - t * s.width, n - 1);
            const int axis = AXES ? a.pair_axis[p] : 0;
            const bool turns = !AXES || (axis >= 0 && axis < a.axes);
            const int position = a.positions[(turns ? axis : 0) * a.position_stride + t0 + t];
            double angle = (double)position * (double)a.frequencies[p] * 0.15915494309189535;  // in turns
            angle -= rint(angle);
            float c = STILL, sn = 0.f;
            if (turns)
                sincospif(2.f * (float)angle, &sn, &c);
            else
                some_still = 1;
            cosine[i] = c;
            sine[i] = a.inverse ? -sn : sn;
        }
        __syncthreads();
        const bool still = AXES && __builtin_amdgcn_readfirstlane(some_still);

        const int first = blockIdx.y * s.split, last = min(first + s.split, tokens * s.units);
        for (int i = first + (int)threadIdx.x; i < last; i += ROTARY_THREADS) {
            const int dt = small_div(i, s.units, 1.f / (float)s.units);
            const long long t = t0 + dt;
            int j = i - dt * s.units;
            // which head, and which piece of it: the pieces of a head lie together
            const bool value = WRITE && j >= heads * s.per_head;
            j -= value ? heads * s.per_head : 0;
            const int per = value ? s.valued : s.per_head;
            int head = small_div(j, per, 1.f / (float)per), piece = j - head * per;
            const bool turns = !value && piece < s.turned;
            piece -= turns || value ? 0 : s.turned;
            const bool key = value || head >= a.heads;
            head -= !value && key ? a.heads : 0;
            const T *in = value ? (const T *)args.v + t * args.v_token_stride + head * args.v_head_stride
                          : key ? (const T *)a.k + t * a.k_token_stride + head * a.k_head_stride
                                : (const T *)a.q + t * a.q_token_stride + head * a.q_head_stride;
            T *out;
            bool keep = true;
            if (WRITE && key) {
                const sbvr_kv_cache &c = args.kv;
                const long long slot = args.slots[t];
                keep = slot >= 0 && slot < (long long)c.n_pages << page_shift;
                const long long at = slot & ((1 << page_shift) - 1);
                out = value ? (T *)c.v + (slot >> page_shift) * c.v_page_stride + at * c.v_token_stride + head * c.v_head_stride
                            : (T *)c.k + (slot >> page_shift) * c.k_page_stride + at * c.k_token_stride + head * c.k_head_stride;
            } else {
                out = key ? (T *)a.k_out + t * a.k_out_token_stride + head * a.k_out_head_stride
                          : (T *)a.q_out + t * a.q_out_token_stride + head * a.q_out_head_stride;
            }
            const bool in_place = out == in;
            // what is copied in place stays; both kinds load and store two pieces
            if (!keep || (in_place && !turns))
                continue;
            const int base = value ? 0 : 2 * n, end = a.head_dim;
            const int p0 = !turns ? 0 : EVEN || 8 * piece + 8 <= n || n < 8 || in_place ? 8 * piece : n - 8;
            const int at = base + 16 * piece + 16 > end && end - base >= 16 ? end - 16 : base + 16 * piece;
            const float *c = cosine + dt * s.width + p0, *sn = sine + dt * s.width + p0;
            if (turns ? EVEN || p0 + 8 <= n : at + 16 <= end) {
                const int a0 = !turns ? at : a.interleaved ? 2 * p0 : p0;
                const int b0 = !turns ? at + 8 : a.interleaved ? 2 * p0 + 8 : n + p0;
                const Words<T> wx = load_words(in + a0), wy = load_words(in + b0);
                const Loose<T, 8> x = from_words<T>(wx), y = from_words<T>(wy);
                Loose<T, 8> xo, yo;
                if (a.interleaved) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float u = (float)x.e[2 * e], v = (float)x.e[2 * e + 1];
                        xo.e[2 * e] = (T)turned_first(u, v, c[e], sn[e]);
                        xo.e[2 * e + 1] = (T)turned_second(u, v, c[e], sn[e]);
                        const float w = (float)y.e[2 * e], z = (float)y.e[2 * e + 1];
                        yo.e[2 * e] = (T)turned_first(w, z, c[e + 4], sn[e + 4]);
                        yo.e[2 * e + 1] = (T)turned_second(w, z, c[e + 4], sn[e + 4]);
                    }
                    if (still)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            xo.e[e] = c[e / 2] == STILL ? x.e[e] : xo.e[e];
                            yo.e[e] = c[e / 2 + 4] == STILL ? y.e[e] : yo.e[e];
                        }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float u = (float)x.e[e], v = (float)y.e[e];
                        xo.e[e] = (T)turned_first(u, v, c[e], sn[e]);
                        yo.e[e] = (T)turned_second(u, v, c[e], sn[e]);
                    }
                    if (still)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            xo.e[e] = c[e] == STILL ? x.e[e] : xo.e[e];
                            yo.e[e] = c[e] == STILL ? y.e[e] : yo.e[e];
                        }
                }
                store_words(out + a0, turns ? to_words(xo) : wx);
                store_words(out + b0, turns ? to_words(yo) : wy);
            } else if (turns) {
                for (int p = p0; p < min(p0 + 8, n); ++p) {
                    const int ia = a.interleaved ? 2 * p : p, ib = a.interleaved ? 2 * p + 1 : n + p;
                    const T u = in[ia], v = in[ib];
                    const bool turn_it = !AXES || c[p - p0] != STILL;
                    out[ia] = turn_it ? (T)turned_first((float)u, (float)v, c[p - p0], sn[p - p0]) : u;
                    out[ib] = turn_it ? (T)turned_second((float)u, (float)v, c[p - p0], sn[p - p0]) : v;
                }
            } else {
                int e = at;
                for (; e + 8 <= end; e += 8)
                    store_words(out + e, load_words(in + e));
                for (; e < end; ++e)
                    out[e] = in[e];
            }
        }
    }
}

template <typename T, bool WRITE>
int run_rotary(const RotaryArgs &a, hipStream_t stream)
{
    const sbvr_rotary_args &r = a.r;
    RotaryShape s;
    s.turned = (r.pairs + 7) / 8;
    s.per_head = s.turned + (r.head_dim - 2 * r.pairs + 15) / 16;
    s.valued = (r.head_dim + 15) / 16;
    s.width = 8 * s.turned;
    s.units = (r.heads + r.kv_heads) * s.per_head + (WRITE ? r.kv_heads * s.valued : 0);
    // four pieces a thread where there are many tokens, one where there are few (tokens
    // of 40 heads of 128: 64 take 3.2 us, with four 5.1; 16384 take 64 us, with one 68)
    const int target = (long long)r.T * s.units > 1024ll * ROTARY_THREADS ? 4 * ROTARY_THREADS : ROTARY_THREADS;
    s.tokens = s.units > target ? 1 : target / s.units;
    const int fit = (int)(SBVR_MAX_DYN_LDS / 4 / (2 * sizeof(float) * s.width));
    if (s.tokens > fit)
        s.tokens = fit;
    s.split = s.tokens > 1 || s.units <= target ? s.tokens * s.units : target;
    const int splits = (s.tokens * s.units + s.split - 1) / s.split;
    const long long groups = (r.T + (long long)s.tokens - 1) / s.tokens, most = (1 << 22) / splits;
    const dim3 grid((unsigned)(groups < most ? groups : most), splits);
    RotaryArgs args = a;
    int page_shift = WRITE ? __builtin_ctz(a.kv.page_size) : 0;
    void *argv[] = {&args, &s, &page_shift};
    const void *kernel = r.pairs % 8 == 0 ? (r.pair_axis ? (const void *)rotary_kernel<T, true, WRITE, true>
                                                         : (const void *)rotary_kernel<T, true, WRITE, false>)
                                          : (r.pair_axis ? (const void *)rotary_kernel<T, false, WRITE, true>
                                                         : (const void *)rotary_kernel<T, false, WRITE, false>);
    return launch_kernel(kernel, grid, dim3(ROTARY_THREADS), 2 * sizeof(float) * s.tokens * s.width, stream, argv);
}

int launch_rotary(const RotaryArgs &a, hipStream_t stream)
{
    switch (a.r.dtype) {
    case SBVR_F16: return a.slots ? run_rotary<f16_t, true>(a, stream) : run_rotary<f16_t, false>(a, stream);
    case SBVR_BF16: return a.slots ? run_rotary<bf16_t, true>(a, stream) : run_rotary<bf16_t, false>(a, stream);
    default: return run_rotary<float, false>(a, stream);
    }
}

}  // namespace sbvr
