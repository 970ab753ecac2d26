// Attention of a step's tokens over a paged key/value cache (tree attention).
//
// The rows of a key/value head are the request's new tokens times the query
// heads that share it; up to 16 NT of them are one item.  Everything is
// computed transposed, on v_mfma_f32_16x16x32: S^T = K Q^T gives a lane four
// positions of one row, so a row's maximum and sum are mostly within lanes,
// and exp(S^T) is, unmoved, the operand of O^T = V^T P^T: its slot e of lane
// group g = lane / 16 stands for position 4g + e (e < 4) and 16 + 4g + e - 4
// of the 32-position tile, and the V operand is laid out the same way.
//   K: lane (c = lane % 16, g) holds position c, elements 32 s + 8 g .. + 7.
//   V: lane (c, g) holds elements DV c .. DV c + DV - 1 (DV = DP / 16) of its
//      eight positions; row c of operand q is element DV c + q, picked from
//      the eight rows with byte permutes.
// head_dim below DP: lanes past the end read piece 0 instead; their Q is zero
// and their outputs are not stored.
//
// A request's last positions are the step's own tokens, which a row sees as
// its tree mask says; tiles that reach into them, or into pages outside the
// cache, are masked, others are not.  What a masked slot holds must not
// matter: scores are replaced, values past the end are zeroed, and values
// that some rows see and others do not are added apart where they are not
// finite.
#include "step.h"

namespace sbvr {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef f16_t v8h __attribute__((ext_vector_type(8)));
typedef bf16_t v8b __attribute__((ext_vector_type(8)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr int ATTN_WAVES = 4, ATTN_THREADS = 64 * ATTN_WAVES;
constexpr int TILE = 32;               // positions per wavefront and step
constexpr float NO_SCORE = -1.0e30f;   // running maximum before any score

template <bool BF>
__device__ __forceinline__ v4f mfma(v4u a, v4u b, v4f c)
{
    if constexpr (BF)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0,
                                                       0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0,
                                                      0);
}

// two binary32 values rounded to nearest even and packed
template <bool BF>
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    typedef float v2f __attribute__((ext_vector_type(2)));
    typedef f16_t v2h __attribute__((ext_vector_type(2)));
    typedef bf16_t v2b __attribute__((ext_vector_type(2)));
    const v2f v = {lo, hi};
    if constexpr (BF)
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, v2b));
    else
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, v2h));
}

template <bool BF>
__device__ __forceinline__ float unpack(uint32_t w, int hi)
{
    const uint32_t h = hi ? w >> 16 : w & 0xffffu;
    if constexpr (BF)
        return __builtin_bit_cast(float, h << 16);
    else
        return (float)__builtin_bit_cast(f16_t, (uint16_t)h);
}

// true where one of the two 16-bit values is an infinity or NaN
template <bool BF>
__device__ __forceinline__ bool not_finite(uint32_t w)
{
    constexpr uint32_t E = BF ? 0x7f80u : 0x7c00u;
    return (w & E) == E || (w & (E << 16)) == (E << 16);
}

__device__ __forceinline__ float max4(float v)  // over the four lane groups
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}

// one request's part of the step
struct Request {
    int ctx, n, first;  // cached tokens, new tokens, its first token
};

__device__ __forceinline__ Request request_of(const AttnArgs &a, int r)
{
    Request q;
    const int s0 = min(max(a.query_start[r], 0), a.T), s1 = min(max(a.query_start[r + 1], s0), a.T);
    const long long room = min((long long)a.max_pages * a.kv.page_size, 0x7fffff00ll);
    q.first = s0;
    q.n = min(s1 - s0, a.max_new);
    q.ctx = (int)min((long long)max(a.context_lens[r], 0), room);
    q.n = (int)min((long long)q.n, room - q.ctx);
    return q;
}

// DP: padded head size, DS: 32-element steps of it that hold elements, NT:
// 16-row tiles per item, BF: bfloat16.
template <int DP, int DS, int NT, bool BF>
__global__ void __launch_bounds__(ATTN_THREADS) attn_kernel(AttnArgs a)
{
    constexpr int DV = DP / 16, ROWS = 16 * NT;
    __shared__ float lds_o[ATTN_WAVES][ROWS][DP + 4];
    __shared__ float lds_m[ATTN_WAVES][ROWS], lds_l[ATTN_WAVES][ROWS];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = lane & 15, g = lane >> 4;
    const int group = a.heads / a.kv.kv_heads;
    const int r = blockIdx.x, kvh = blockIdx.y, row0 = blockIdx.z * ROWS;
    const Request rq = request_of(a, r);
    const int rows = rq.n * group;
    if (row0 >= rows)
        return;
    const int D = a.kv.head_dim, pieces = D / 8;
    const int page_shift = __builtin_ctz(a.kv.page_size);
    const int end = rq.ctx + rq.n;

    // Q operands and masks of this lane's rows
    v4u qf[NT][DS];
    uint64_t mask[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int row = row0 + 16 * nt + c;
        const bool ok = row < rows;
        const int tok = rq.first + (ok ? row / group : 0), head = kvh * group + (ok ? row % group : 0);
        const uint16_t *q = (const uint16_t *)a.q + tok * a.q_token_stride + head * a.q_head_stride;
        mask[nt] = ok ? a.tree_mask[tok] : 0;
#pragma unroll
        for (int s = 0; s < DS; ++s) {
            const int piece = 4 * s + g;
            qf[nt][s] = ok && piece < pieces ? *(const v4u *)(q + 8 * piece) : v4u{0, 0, 0, 0};
        }
    }

    v4f acc[NT][DV];
    float m[NT], l[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m[nt] = NO_SCORE;
        l[nt] = 0.f;
#pragma unroll
        for (int q = 0; q < DV; ++q)
            acc[nt][q] = v4f{0.f, 0.f, 0.f, 0.f};
    }
    const float scale2 = a.scale * 1.4426950408889634f;  // exponentials as powers of two
    const int32_t *table = a.page_table + r * a.table_stride;
    const uint16_t *kb = (const uint16_t *)a.kv.k + kvh * a.kv.k_head_stride;
    const uint16_t *vb = (const uint16_t *)a.kv.v + kvh * a.kv.v_head_stride;
    const int v_off = DV * c < D ? DV * c : 0;

    for (int p0 = wave * TILE; p0 < end; p0 += ATTN_WAVES * TILE) {
        // the pages of the tile's two halves (a page holds whole halves)
        const uint16_t *kp[2], *vp[2];
        bool page_ok[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int p = p0 + 16 * h;
            const int page = p < end ? table[p >> page_shift] : -1;
            page_ok[h] = page >= 0 && page < a.kv.n_pages;
            const long long at = page_ok[h] ? page : 0;
            const int off = p & (a.kv.page_size - 1);
            kp[h] = kb + at * a.kv.k_page_stride + off * a.kv.k_token_stride;
            vp[h] = vb + at * a.kv.v_page_stride + off * a.kv.v_token_stride;
        }
        v4u kf[2][DS];
        uint32_t vr[8][DV / 2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int s = 0; s < DS; ++s) {
                const int piece = 4 * s + g < pieces ? 4 * s + g : 0;
                kf[h][s] = *(const v4u *)(kp[h] + c * a.kv.k_token_stride + 8 * piece);
            }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const Halves<DV> v = *(const Halves<DV> *)(vp[e / 4] + (4 * g + e % 4) * a.kv.v_token_stride + v_off);
#pragma unroll
            for (int i = 0; i < DV / 2; ++i)
                vr[e][i] = v.w[i];
        }

        v4f s[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                s[nt][h] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int d = 0; d < DS; ++d)
                    s[nt][h] = mfma<BF>(kf[h][d], qf[nt][d], s[nt][h]);
                s[nt][h] *= scale2;
            }

        const bool masked = p0 + TILE > rq.ctx || !page_ok[0] || !page_ok[1];
        bool odd_values = false;
        if (masked) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int p = p0 + 16 * (e / 4) + 4 * g + e % 4, j = p - rq.ctx;
                const bool there = p < end && page_ok[e / 4];
                bool odd = false;
#pragma unroll
                for (int i = 0; i < DV / 2; ++i) {
                    if (!there)
                        vr[e][i] = 0;
                    odd |= not_finite<BF>(vr[e][i]);
                }
                odd_values |= odd && j >= 0;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const bool seen = there && (j < 0 || ((mask[nt] >> (j & 63)) & 1));
                    if (!seen)
                        s[nt][e / 4][e % 4] = -INFINITY;
                }
            }
            odd_values = __ballot(odd_values) != 0;
        }

        v4u pf[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float x[8], top = NO_SCORE;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = s[nt][e / 4][e % 4];
                top = fmaxf(top, x[e]);
            }
            top = fmaxf(max4(top), m[nt]);
            const float keep = exp2f(m[nt] - top);
            m[nt] = top;
            l[nt] *= keep;
#pragma unroll
            for (int q = 0; q < DV; ++q)
                acc[nt][q] *= keep;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = exp2f(x[e] - top);
                l[nt] += x[e];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                pf[nt][i] = pack2<BF>(x[2 * i], x[2 * i + 1]);
        }

        if (odd_values) {
            // some of the step's own values are not finite: their products are
            // added one by one to the rows that see them, and 0 stands in
            // their place below
            for (int e = 0; e < 8; ++e)
                for (int gg = 0; gg < 4; ++gg) {
                    const int p = p0 + 16 * (e / 4) + 4 * gg + e % 4, j = p - rq.ctx;
                    if (p >= end || j < 0 || !page_ok[e / 4])
                        continue;
                    const uint16_t *v = (e / 4 ? vp[1] : vp[0]) + (4 * gg + e % 4) * a.kv.v_token_stride;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const uint32_t w = e / 2 == 0 ? pf[nt][0] : e / 2 == 1 ? pf[nt][1] : e / 2 == 2 ? pf[nt][2]
                                                                                                      : pf[nt][3];
                        const float weight = unpack<BF>(__shfl(w, 16 * gg + c), e & 1);
                        const bool seen = (mask[nt] >> j) & 1;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int d = DV * (4 * g + i);
                            if (d >= D)
                                continue;
#pragma unroll
                            for (int q = 0; q < DV; ++q) {
                                const uint32_t bits = v[d + q];
                                if (seen && not_finite<BF>(bits))
                                    acc[nt][q][i] += weight * unpack<BF>(bits, 0);
                            }
                        }
                    }
                }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (p0 + 16 * (e / 4) + 4 * g + e % 4 < rq.ctx)
                    continue;
#pragma unroll
                for (int i = 0; i < DV / 2; ++i) {
                    if (not_finite<BF>(vr[e][i] & 0xffffu))
                        vr[e][i] &= 0xffff0000u;
                    if (not_finite<BF>(vr[e][i] >> 16))
                        vr[e][i] &= 0xffffu;
                }
            }
        }

#pragma unroll
        for (int q = 0; q < DV; ++q) {
            v4u vf;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                vf[i] = __builtin_amdgcn_perm(vr[2 * i + 1][q / 2], vr[2 * i][q / 2], q & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                acc[nt][q] = mfma<BF>(vf, pf[nt], acc[nt][q]);
        }
    }

    // the wavefronts' parts meet in LDS
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        l[nt] += __shfl_xor(l[nt], 16);
        l[nt] += __shfl_xor(l[nt], 32);
        if (g == 0) {
            lds_m[wave][16 * nt + c] = m[nt];
            lds_l[wave][16 * nt + c] = l[nt];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int q = 0; q < DV; ++q)
                lds_o[wave][16 * nt + c][DV * (4 * g + i) + q] = acc[nt][q][i];
    }
    __syncthreads();
    for (int row = wave; row < min(ROWS, rows - row0); row += ATTN_WAVES) {
        float top = NO_SCORE;
#pragma unroll
        for (int w = 0; w < ATTN_WAVES; ++w)
            top = fmaxf(top, lds_m[w][row]);
        float f[ATTN_WAVES], total = 0.f;
#pragma unroll
        for (int w = 0; w < ATTN_WAVES; ++w) {
            f[w] = exp2f(lds_m[w][row] - top);
            total += f[w] * lds_l[w][row];
        }
        const float inv = total > 0.f ? 1.f / total : total == 0.f ? 0.f : total;
        const int tok = rq.first + (row0 + row) / group, head = kvh * group + (row0 + row) % group;
        uint16_t *out = (uint16_t *)a.out + ((long long)tok * a.heads + head) * D;
        for (int d = 2 * lane; d < D; d += 128) {
            float o0 = 0.f, o1 = 0.f;
#pragma unroll
            for (int w = 0; w < ATTN_WAVES; ++w) {
                o0 += f[w] * lds_o[w][row][d];
                o1 += f[w] * lds_o[w][row][d + 1];
            }
            *(uint32_t *)(out + d) = pack2<BF>(o0 * inv, o1 * inv);
        }
    }
}

template <int DP, int DS, int NT, bool BF>
int go_attn(const AttnArgs &a, hipStream_t stream)
{
    AttnArgs args = a;
    void *argv[] = {&args};
    const int rows = a.max_new * (a.heads / a.kv.kv_heads);
    return launch_kernel((const void *)attn_kernel<DP, DS, NT, BF>,
                         dim3(a.R, a.kv.kv_heads, (rows + 16 * NT - 1) / (16 * NT)), dim3(ATTN_THREADS), 0, stream,
                         argv);
}

template <int DP, int DS>
int by_type(const AttnArgs &a, hipStream_t stream)
{
    return a.kv.dtype == SBVR_BF16 ? go_attn<DP, DS, 1, true>(a, stream) : go_attn<DP, DS, 1, false>(a, stream);
}

size_t attn_workspace_bytes(int, int, int, int, int) { return 0; }

int launch_attn(const AttnArgs &a, hipStream_t stream)
{
    if (a.kv.head_dim <= 64)
        return by_type<64, 2>(a, stream);
    if (a.kv.head_dim <= 96)
        return by_type<128, 3>(a, stream);
    return by_type<128, 4>(a, stream);
}

}  // namespace sbvr
