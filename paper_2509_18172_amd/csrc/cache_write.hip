// A step's keys and values into their slots of the paged cache: a copy of
// 2 * kv_heads * head_dim elements per token, memory-bound, 16 bytes a lane.
//
// A workgroup is X lanes (the 16-byte pieces of a token's keys and values, so
// a lane works out its head and offset once) by Y tokens; four tokens a lane
// are in flight (with eight, eight tokens take 4.0 us instead of 3.5 and 16384
// no less; two are within 1 % of four).
//
// Measured in a graph, eight key/value heads of 128 elements: 16384 tokens 27.0
// us, 4.97 TB/s read and written, which is the rate of a large copy (4.94); eight
// tokens 3.0 us, of which an empty launch is 2.1.
#include "step.h"

namespace sbvr {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr int WRITE_THREADS = 256, WRITE_UNROLL = 4;

struct WriteArgs {
    sbvr_kv_cache c;
    int T, page_shift;
    const uint16_t *k, *v;
    int64_t k_token_stride, k_head_stride, v_token_stride, v_head_stride;
    const int64_t *slots;
};

__global__ void __launch_bounds__(WRITE_THREADS) cache_write_kernel(WriteArgs a)
{
    const int per_head = a.c.head_dim / 8, half = a.c.kv_heads * per_head;
    const int Y = blockDim.y;
    const long long n_slots = (long long)a.c.n_pages << a.page_shift;
    const int in_page = (1 << a.page_shift) - 1;
    const long long t0 = (long long)blockIdx.x * Y * WRITE_UNROLL + threadIdx.y;
    for (int c = threadIdx.x; c < 2 * half; c += blockDim.x) {
        const bool is_v = c >= half;
        const int piece = is_v ? c - half : c, head = piece / per_head, off = (piece % per_head) * 8;
        const uint16_t *src = is_v ? a.v + head * a.v_head_stride + off : a.k + head * a.k_head_stride + off;
        const int64_t src_stride = is_v ? a.v_token_stride : a.k_token_stride;
        uint16_t *dst = (uint16_t *)(is_v ? a.c.v : a.c.k) + off + head * (is_v ? a.c.v_head_stride : a.c.k_head_stride);
        const int64_t page_stride = is_v ? a.c.v_page_stride : a.c.k_page_stride;
        const int64_t token_stride = is_v ? a.c.v_token_stride : a.c.k_token_stride;
        v4u val[WRITE_UNROLL];
        long long slot[WRITE_UNROLL];
#pragma unroll
        for (int u = 0; u < WRITE_UNROLL; ++u) {
            const long long t = t0 + u * Y;
            const long long at = min(t, (long long)a.T - 1);  // no branch around the loads
            slot[u] = t < a.T ? a.slots[at] : -1;
            val[u] = *(const v4u *)(src + at * src_stride);
        }
#pragma unroll
        for (int u = 0; u < WRITE_UNROLL; ++u)
            if (slot[u] >= 0 && slot[u] < n_slots)
                *(v4u *)(dst + (slot[u] >> a.page_shift) * page_stride + (slot[u] & in_page) * token_stride) = val[u];
    }
}

int launch_cache_write(const sbvr_kv_cache &c, int T, const void *k, int64_t k_token_stride, int64_t k_head_stride,
                       const void *v, int64_t v_token_stride, int64_t v_head_stride, const int64_t *slots,
                       hipStream_t stream)
{
    WriteArgs a{c, T, __builtin_ctz(c.page_size), (const uint16_t *)k, (const uint16_t *)v,
                k_token_stride, k_head_stride, v_token_stride, v_head_stride, slots};
    int x = 1;
    while (x < 2 * c.kv_heads * (c.head_dim / 8) && x < WRITE_THREADS)
        x *= 2;
    const int y = WRITE_THREADS / x;
    const long long grid = ((long long)T + (long long)y * WRITE_UNROLL - 1) / ((long long)y * WRITE_UNROLL);
    void *argv[] = {&a};
    return launch_kernel((const void *)cache_write_kernel, dim3((unsigned)grid), dim3(x, y), 0, stream, argv);
}

}  // namespace sbvr
