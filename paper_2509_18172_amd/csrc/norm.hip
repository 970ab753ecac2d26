// The norms around a block with its gate and residual scale: z = rms(y) * w,
// x' = x + scale * gate * z, h = rms(x') * w', one pass over the rows.
//
// A row is held in registers by the threads of one workgroup (a piece of VEC
// elements each, CH times), so x, y and the gate are read once and x' and h
// written once; the two means are sums over the workgroup in a fixed order.
// Memory-bound for many tokens, bound by its two reductions' latency for few.
#include "step.h"

namespace sbvr {

template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
    T e[N];
};

template <typename T>
__device__ __forceinline__ float widen(T v)
{
    return (float)v;
}

template <int THREADS>
__device__ __forceinline__ float block_sum(float v, float *scratch)
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

// A: type of y, gate, weights, h; X: type of the residual stream.
template <typename A, typename X, int VEC, int CH, int THREADS>
__global__ void __launch_bounds__(THREADS) norm_kernel(NormArgs a)
{
    __shared__ float scratch[2][THREADS / 64];
    const long long t = blockIdx.x;
    const A *y = (const A *)a.y + t * a.y_stride;
    const A *gate = (const A *)a.gate + t * a.gate_stride;
    const X *x = (const X *)a.x + t * a.x_stride;
    const A *post = (const A *)a.post, *pre = (const A *)a.pre;

    float xv[CH][VEC], yv[CH][VEC];
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int i = (c * THREADS + (int)threadIdx.x) * VEC;
        Vec<X, VEC> xr = {};
        Vec<A, VEC> yr = {};
        if (i < a.H) {
            xr = *(const Vec<X, VEC> *)(x + i);
            if (a.y)
                yr = *(const Vec<A, VEC> *)(y + i);
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            xv[c][e] = widen(xr.e[e]);
            yv[c][e] = widen(yr.e[e]);
            sum += yv[c][e] * yv[c][e];
        }
    }
    if (a.y) {
        float inv = 1.f;
        if (a.post)
            inv = 1.f / sqrtf(block_sum<THREADS>(sum, scratch[0]) / (float)a.H + a.eps);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int i = (c * THREADS + (int)threadIdx.x) * VEC;
            if (i < a.H) {
                Vec<A, VEC> w = {}, g = {};
                if (a.post)
                    w = *(const Vec<A, VEC> *)(post + i);
                if (a.gate)
                    g = *(const Vec<A, VEC> *)(gate + i);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    float z = yv[c][e];
                    if (a.post)
                        z = z * inv * widen(w.e[e]);
                    if (a.gate)
                        z *= widen(g.e[e]);
                    xv[c][e] += a.scale * z;
                }
            }
        }
    }
    sum = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int i = (c * THREADS + (int)threadIdx.x) * VEC;
        Vec<X, VEC> o;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            o.e[e] = (X)xv[c][e];
            sum += xv[c][e] * xv[c][e];
        }
        if (a.x_out && i < a.H)
            *(Vec<X, VEC> *)((X *)a.x_out + t * a.x_out_stride + i) = o;
    }
    if (!a.h_out)
        return;
    const float inv = 1.f / sqrtf(block_sum<THREADS>(sum, scratch[1]) / (float)a.H + a.eps);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int i = (c * THREADS + (int)threadIdx.x) * VEC;
        if (i < a.H) {
            const Vec<A, VEC> w = *(const Vec<A, VEC> *)(pre + i);
            Vec<A, VEC> o;
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                o.e[e] = (A)(xv[c][e] * inv * widen(w.e[e]));
            *(Vec<A, VEC> *)((A *)a.h_out + t * a.h_stride + i) = o;
        }
    }
}

template <typename A, typename X, int VEC, int CH, int THREADS>
int go(const NormArgs &a, hipStream_t stream)
{
    NormArgs args = a;
    void *argv[] = {&args};
    return launch_kernel((const void *)norm_kernel<A, X, VEC, CH, THREADS>, dim3((unsigned)a.T), dim3(THREADS), 0,
                         stream, argv);
}

template <typename A, typename X>
int dispatch(const NormArgs &a, hipStream_t stream)
{
    // 16 bytes a lane where every row of 16-bit elements starts on them (the
    // residual stream's rows then start on 16 or 32)
    const uintptr_t at = (uintptr_t)a.x | (uintptr_t)a.y | (uintptr_t)a.post | (uintptr_t)a.gate |
                         (uintptr_t)a.pre | (uintptr_t)a.x_out | (uintptr_t)a.h_out;
    const int64_t strides = a.x_stride | a.y_stride | a.gate_stride | a.x_out_stride | a.h_stride | (int64_t)a.H;
    if (at % 32 == 0 && strides % 8 == 0) {
        if (a.H <= 512 * 8)
            return go<A, X, 8, 1, 512>(a, stream);
        if (a.H <= 1024 * 8)
            return go<A, X, 8, 1, 1024>(a, stream);
        return go<A, X, 8, 4, 1024>(a, stream);
    }
    if (a.H <= 256 * 8)
        return go<A, X, 1, 8, 256>(a, stream);
    if (a.H <= 1024 * 8)
        return go<A, X, 1, 8, 1024>(a, stream);
    return go<A, X, 1, 32, 1024>(a, stream);
}

int launch_norm(const NormArgs &a, int dtype, int x_dtype, hipStream_t stream)
{
    if (dtype == SBVR_F16)
        return x_dtype == SBVR_F32 ? dispatch<f16_t, float>(a, stream) : dispatch<f16_t, f16_t>(a, stream);
    return x_dtype == SBVR_F32 ? dispatch<bf16_t, float>(a, stream) : dispatch<bf16_t, bf16_t>(a, stream);
}

}  // namespace sbvr
