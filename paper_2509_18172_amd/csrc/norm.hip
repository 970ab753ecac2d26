// The norms around a block with its gate and residual scale: z = rms(y) * w,
// x' = x + scale * gate * z, h = rms(x') * w', one pass over the rows.
//
// A row is held by THREADS threads, in registers, CH pieces of eight elements
// each, so x, y and the gate are read once and x' and h written once; the two
// means are sums in a fixed order.  Every load is sent off at the start, without
// a branch, so that one latency covers them; the first reduction and the second
// follow.  Up to 512 elements a wavefront has a row of its own, four to a
// workgroup, and no barrier.  Memory-bound for many tokens.
//
// Measured in a graph: 4096 rows of 8192 in bfloat16 with both norms and a gate
// 67.5 us, 5.0 TB/s read and written, the rate of a large copy (4.94); 4096 rows of
// 1024 10 us and 2048 14.4 us (4.7 TB/s); one row of 4096 3.9 us, of which an empty
// launch is 2.1 and the rest two latencies and two reductions.
//
// Above 16384 elements a thread has four pieces, and some of the row does not fit
// the 128 registers that 1024 threads leave each: 20 to 100 bytes a lane go to
// scratch.  512 rows of 16384 24.5 us (4.1 TB/s), of 32768 60.1 us (3.4) with a binary32
// stream and 34 us (3.9 to 4.0) with a 16-bit one.  Widths that are no multiple of 8
// load and store at any address: 1000 rows of 5003 16.4 to 18.2 us, of 5000 14.6.
//
// Rows need no alignment beyond their elements'.  A piece that would pass the
// row's end is moved back to end with it: of its elements the first ones belong
// to the piece before and are neither summed nor stored.
#include "step.h"

namespace sbvr {

enum Tail { EVEN, ODD, SHORT };  // H a multiple of 8; any other from 8 on; below 8

// where a thread's piece lies: from `at`, its own elements from `own` on (8: none)
struct Piece {
    int at, own;
};

template <Tail TAIL>
__device__ __forceinline__ Piece piece_at(int i, int H)
{
    if constexpr (TAIL == SHORT)
        return {0, i == 0 ? 0 : 8};
    const int at = min(i, H - 8);
    return {at, min(i - at, 8)};
}

template <Tail TAIL, typename T>
__device__ __forceinline__ Loose<T, 8> load8(const T *row, Piece p, int H)
{
    if constexpr (TAIL != SHORT)
        return from_words<T>(load_words(row + p.at));
    Loose<T, 8> r;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        r.e[e] = row[min(e, H - 1)];
    return r;
}

// whether element e of the piece is the thread's own
template <Tail TAIL>
__device__ __forceinline__ bool owns(Piece p, int e, int H)
{
    return TAIL == EVEN ? p.own == 0 : TAIL == ODD ? e >= p.own : e >= p.own && e < H;
}

template <Tail TAIL, typename T>
__device__ __forceinline__ void store8(T *row, Piece p, int H, const float (&v)[8])
{
    Loose<T, 8> r;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        r.e[e] = (T)v[e];
    if (TAIL != SHORT && p.own == 0)
        store_words(row + p.at, to_words(r));
    else if (TAIL != EVEN)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (owns<TAIL>(p, e, H))
                row[p.at + e] = r.e[e];
}

template <int THREADS>
__device__ __forceinline__ float row_sum(float v, float *scratch)
{
#pragma unroll
    for (int s = 32; s; s >>= 1)
        v += __shfl_xor(v, s);
    if constexpr (THREADS == 64)
        return v;
    if ((threadIdx.x & 63) == 0)
        scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w)
        t += scratch[w];
    return t;
}

constexpr int rows_of(int threads) { return threads == 64 ? 4 : 1; }  // rows of a workgroup

// A: type of y, gate, weights, h; X: type of the residual stream.
template <typename A, typename X, int CH, int THREADS, Tail TAIL>
__global__ void __launch_bounds__(THREADS *rows_of(THREADS)) norm_kernel(NormArgs a)
{
    __shared__ float scratch[2][THREADS / 64];
    const int lane = threadIdx.x % THREADS;
    const long long t = (long long)blockIdx.x * rows_of(THREADS) + threadIdx.x / THREADS;
    if (t >= a.T)  // only where a wavefront has a row of its own
        return;
    // an operand that is not given is read from x's row all the same (x is no
    // shorter) and not used
    const X *x = (const X *)a.x + t * a.x_stride;
    const A *y = a.y ? (const A *)a.y + t * a.y_stride : (const A *)x;
    const A *gate = a.gate ? (const A *)a.gate + t * a.gate_stride : (const A *)x;
    const A *post = a.post ? (const A *)a.post : (const A *)x, *pre = a.h_out ? (const A *)a.pre : (const A *)x;

    Piece p[CH];
    Loose<X, 8> xr[CH];
    Loose<A, 8> yr[CH], postr[CH], gater[CH], prer[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        p[c] = piece_at<TAIL>((c * THREADS + lane) * 8, a.H);
        xr[c] = load8<TAIL>(x, p[c], a.H);
        yr[c] = load8<TAIL>(y, p[c], a.H);
        postr[c] = load8<TAIL>(post, p[c], a.H);
        gater[c] = load8<TAIL>(gate, p[c], a.H);
        prer[c] = load8<TAIL>(pre, p[c], a.H);
    }
    float xv[CH][8], sum = 0.f;
    if (a.y && a.post) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = (float)yr[c].e[e];
                sum += owns<TAIL>(p[c], e, a.H) ? v * v : 0.f;
            }
        sum = row_sum<THREADS>(sum, scratch[0]);
    }
    const float inv_y = 1.f / sqrtf(sum / (float)a.H + a.eps);
    sum = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float z = (float)yr[c].e[e];
            if (a.post)
                z = z * inv_y * (float)postr[c].e[e];
            if (a.gate)
                z *= (float)gater[c].e[e];
            xv[c][e] = (float)xr[c].e[e] + (a.y ? a.scale * z : 0.f);
            sum += owns<TAIL>(p[c], e, a.H) ? xv[c][e] * xv[c][e] : 0.f;
        }
        if (a.x_out)
            store8<TAIL>((X *)a.x_out + t * a.x_out_stride, p[c], a.H, xv[c]);
    }
    if (!a.h_out)
        return;
    const float inv = 1.f / sqrtf(row_sum<THREADS>(sum, scratch[1]) / (float)a.H + a.eps);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        float h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            h[e] = xv[c][e] * inv * (float)prer[c].e[e];
        store8<TAIL>((A *)a.h_out + t * a.h_stride, p[c], a.H, h);
    }
}

template <typename A, typename X, int CH, int THREADS>
int go(const NormArgs &a, hipStream_t stream)
{
    constexpr int ROWS = rows_of(THREADS);
    NormArgs args = a;
    void *argv[] = {&args};
    const void *kernel = a.H < 8        ? (const void *)norm_kernel<A, X, 1, 64, SHORT>
                         : a.H % 8 == 0 ? (const void *)norm_kernel<A, X, CH, THREADS, EVEN>
                                        : (const void *)norm_kernel<A, X, CH, THREADS, ODD>;
    return launch_kernel(kernel, dim3((unsigned)((a.T + (long long)ROWS - 1) / ROWS)), dim3(THREADS * ROWS), 0, stream,
                         argv);
}

template <typename A, typename X>
int dispatch(const NormArgs &a, hipStream_t stream)
{
    // One piece a thread as far as a workgroup's threads go: with two pieces for
    // half the threads one row of 4096 takes 4.6 us instead of 4.2, 4096 rows of
    // 1024 11.7 instead of 11.0, of 4096 38.0 instead of 36.5 (binary32 stream); four
    // pieces are slower again.
    if (a.H <= 64 * 8)
        return go<A, X, 1, 64>(a, stream);
    if (a.H <= 128 * 8)
        return go<A, X, 1, 128>(a, stream);
    if (a.H <= 256 * 8)
        return go<A, X, 1, 256>(a, stream);
    if (a.H <= 512 * 8)
        return go<A, X, 1, 512>(a, stream);
    if (a.H <= 1024 * 8)
        return go<A, X, 1, 1024>(a, stream);
    if (a.H <= 2048 * 8)
        return go<A, X, 2, 1024>(a, stream);
    return go<A, X, 4, 1024>(a, stream);
}

int launch_norm(const NormArgs &a, int dtype, int x_dtype, hipStream_t stream)
{
    if (dtype == SBVR_F16)
        return x_dtype == SBVR_F32 ? dispatch<f16_t, float>(a, stream) : dispatch<f16_t, f16_t>(a, stream);
    return x_dtype == SBVR_F32 ? dispatch<bf16_t, float>(a, stream) : dispatch<bf16_t, bf16_t>(a, stream);
}

}  // namespace sbvr
