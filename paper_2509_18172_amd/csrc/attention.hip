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
// Work: the cached positions of all items, in units of one step of a
// workgroup, are one line that is cut into (up to) SPLITS equal ranges,
// whatever the requests' lengths; a workgroup runs the segments of items in its range.  An
// item within one range is finished there; of an item that a cut divides,
// every workgroup leaves its unnormalised sums, and a second kernel joins
// them.  Which workgroup has what follows from the lengths alone.
//
// Loads: K's registers are refilled for the next step as soon as the scores
// are formed and V's as soon as the products are, so each is in flight while
// the other is used.
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
constexpr int UNIT = ATTN_WAVES * TILE;  // positions per workgroup and step
constexpr int SPLITS = 512;            // ranges: two workgroups a CU
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

// Where the items lie on the line of units: request r's kv_heads * row blocks
// items one after the other, each of the request's units.
struct Line {
    long long total;
    int per;  // requests per thread of the scan
};

struct Item {
    int r, kvh, block;
    Request rq;
    long long start;  // first unit
    int units;
};

__device__ __forceinline__ int item_units(const Request &q) { return (q.ctx + q.n + UNIT - 1) / UNIT; }

template <int ROWS>
__device__ __forceinline__ int row_blocks(const AttnArgs &a, const Request &q)
{
    return (q.n * (a.heads / a.kv.kv_heads) + ROWS - 1) / ROWS;
}

// chunk[i]: units before the requests of thread i (chunk[THREADS]: all).
template <int ROWS, int THREADS>
__device__ __forceinline__ Line lay_out(const AttnArgs &a, long long *chunk, long long *scratch)
{
    Line line;
    line.per = (a.R + THREADS - 1) / THREADS;
    long long units = 0, none = 0, zero;
    const int r0 = threadIdx.x * line.per, r1 = min(r0 + line.per, a.R);
    for (int r = r0; r < r1; ++r) {
        const Request q = request_of(a, r);
        units += (long long)item_units(q) * row_blocks<ROWS>(a, q) * a.kv.kv_heads;
    }
    scan_pair<THREADS>(units, none, line.total, zero, scratch);
    chunk[threadIdx.x] = units;
    if (threadIdx.x == 0)
        chunk[THREADS] = line.total;
    __syncthreads();
    return line;
}

// The item that holds unit u of the line.
template <int ROWS, int THREADS>
__device__ __forceinline__ Item item_at(const AttnArgs &a, const Line &line, const long long *chunk, long long u)
{
    const int i = owner_of(chunk, THREADS, u);
    long long base = chunk[i];
    Item it;
    for (it.r = i * line.per;; ++it.r) {
        it.rq = request_of(a, it.r);
        it.units = item_units(it.rq);
        const int blocks = row_blocks<ROWS>(a, it.rq);
        const long long all = (long long)it.units * blocks * a.kv.kv_heads;
        if (u < base + all) {
            const long long k = (u - base) / it.units;
            it.start = base + k * it.units;
            it.kvh = (int)(k / blocks);
            it.block = (int)(k % blocks);
            return it;
        }
        base += all;
    }
}

// The line's ranges, none empty: their number, where range i starts, and the
// range that holds unit u.
__device__ __forceinline__ int ranges(long long total) { return (int)min(total, (long long)SPLITS); }
__device__ __forceinline__ long long cut(long long total, int i)
{
    return total <= SPLITS ? i : total * i / SPLITS;
}
__device__ __forceinline__ int range_of(long long total, long long u)
{
    return total <= SPLITS ? (int)u : (int)(((u + 1) * SPLITS - 1) / total);
}

// Partial sums of a divided item in the workspace: the range's own slot 2 i for
// its first segment, 2 i + 1 for another (only its last can be divided too).
template <int ROWS, int DP>
struct Part {
    float o[ROWS][DP];
    float m[ROWS], l[ROWS];
};

__device__ __forceinline__ uint16_t *out_row(const AttnArgs &a, const Item &it, int row, int group)
{
    const int tok = it.rq.first + row / group, head = it.kvh * group + row % group;
    return (uint16_t *)a.out + ((long long)tok * a.heads + head) * a.kv.head_dim;
}

__device__ __forceinline__ float inverse(float total)  // 0 for a row that saw nothing; NaN stays
{
    return total == 0.f ? 0.f : 1.f / total;
}

// DP: padded head size, DS: 32-element steps of it that hold elements, NT:
// 16-row tiles per item, BF: bfloat16.
template <int DP, int DS, int NT, bool BF>
__global__ void __launch_bounds__(ATTN_THREADS, 2) attn_kernel(AttnArgs a)
{
    constexpr int DV = DP / 16, ROWS = 16 * NT;
    __shared__ float lds_o[ATTN_WAVES][ROWS][DP + 4];
    __shared__ float lds_m[ATTN_WAVES][ROWS], lds_l[ATTN_WAVES][ROWS];
    __shared__ long long chunk[ATTN_THREADS + 1], scratch[2 * ATTN_WAVES];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = lane & 15, g = lane >> 4;
    const int group = a.heads / a.kv.kv_heads;
    const int D = a.kv.head_dim, pieces = D / 8;
    const int page_shift = __builtin_ctz(a.kv.page_size);
    const Line line = lay_out<ROWS, ATTN_THREADS>(a, chunk, scratch);
    if ((int)blockIdx.x >= ranges(line.total))
        return;
    const long long u0 = cut(line.total, blockIdx.x), u1 = cut(line.total, blockIdx.x + 1);

    for (long long u = u0; u < u1;) {
    const Item it = item_at<ROWS, ATTN_THREADS>(a, line, chunk, u);
    const Request &rq = it.rq;
    const int row0 = it.block * ROWS, rows = min(rq.n * group - row0, ROWS);
    const int end = rq.ctx + rq.n;
    const long long stop = min(u1, it.start + it.units);
    const bool whole = u == it.start && stop == it.start + it.units;
    const int first = (int)(u - it.start) * UNIT + wave * TILE, last = min((int)(stop - it.start) * UNIT, end);

    // Q operands and masks of this lane's rows
    v4u qf[NT][DS];
    uint64_t mask[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const bool ok = 16 * nt + c < rows;
        const int row = ok ? row0 + 16 * nt + c : row0;
        const int tok = rq.first + row / group, head = it.kvh * group + row % group;
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
    const int32_t *table = a.page_table + it.r * a.table_stride;
    const uint16_t *kb = (const uint16_t *)a.kv.k + it.kvh * a.kv.k_head_stride;
    const uint16_t *vb = (const uint16_t *)a.kv.v + it.kvh * a.kv.v_head_stride;
    const int v_off = DV * c < D ? DV * c : 0;

    // The pages of a tile's two halves (a page holds whole halves); -1: past the
    // end or outside the cache, read from page 0 and masked.
    auto pages_of = [&](int p0, int *page) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int p = __builtin_amdgcn_readfirstlane(p0 + 16 * h);
            const int id = p < end ? table[p >> page_shift] : -1;
            page[h] = __builtin_amdgcn_readfirstlane(id < a.kv.n_pages ? max(id, -1) : -1);
        }
    };
    v4u kf[2][DS];
    uint32_t vr[8][DV / 2];
    // every load is a uniform address (page, half, position) plus the lane's
    // 32-bit byte offset
    const uint32_t k_step = 2 * (uint32_t)a.kv.k_token_stride, v_step = 2 * (uint32_t)a.kv.v_token_stride;
    const uint32_t k_lane = c * k_step, v_lane = 4 * g * v_step + 2 * v_off;
    auto at_page = [&](const void *base, int page, int p, int64_t page_stride, uint32_t step) {
        const uint32_t off = (uint32_t)p & (a.kv.page_size - 1);
        return (const char *)base + 2 * (long long)max(page, 0) * page_stride + (uint64_t)off * step;
    };
    auto load_k = [&](int p0, const int *page) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const char *kp = at_page(kb, page[h], p0 + 16 * h, a.kv.k_page_stride, k_step);
#pragma unroll
            for (int s = 0; s < DS; ++s) {
                const uint32_t piece = 4 * s + 3 < pieces || 4 * s + g < pieces ? 4 * s + g : 0;
                kf[h][s] = *(const v4u *)(kp + (uint64_t)(k_lane + 16 * piece));
            }
        }
    };
    auto load_v = [&](int p0, const int *page) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const char *vp = at_page(vb, page[h], p0 + 16 * h, a.kv.v_page_stride, v_step);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const Halves<DV> v = *(const Halves<DV> *)(vp + (uint64_t)(e * v_step) + (uint64_t)v_lane);
#pragma unroll
                for (int i = 0; i < DV / 2; ++i)
                    vr[4 * h + e][i] = v.w[i];
            }
        }
    };

    int page[2], next[2];
    if (first < last) {
        pages_of(first, page);
        load_k(first, page);
        load_v(first, page);
    }
    for (int p0 = first; p0 < last; p0 += UNIT) {
        const bool page_ok[2] = {page[0] >= 0, page[1] >= 0};
        const bool more = p0 + UNIT < last;
        if (more)
            pages_of(p0 + UNIT, next);

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

        if (more)
            load_k(p0 + UNIT, next);

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
#pragma unroll 1
            for (int e = 0; e < 8; ++e)
#pragma unroll 1
                for (int gg = 0; gg < 4; ++gg) {
                    const int p = p0 + 16 * (e / 4) + 4 * gg + e % 4, j = p - rq.ctx;
                    if (p >= end || j < 0 || !page_ok[e / 4])
                        continue;
                    const uint16_t *v = (const uint16_t *)(at_page(vb, page[e / 4], p0 + 16 * (e / 4), a.kv.v_page_stride,
                                                                     v_step) +
                                                             (uint64_t)((4 * gg + e % 4) * v_step));
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
        if (more) {
            load_v(p0 + UNIT, next);
            page[0] = next[0];
            page[1] = next[1];
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
    Part<ROWS, DP> &part = ((Part<ROWS, DP> *)a.workspace)[2 * blockIdx.x + (u != u0)];
    for (int row = wave; row < rows; row += ATTN_WAVES) {
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
        if (!whole && lane == 0) {
            part.m[row] = top;
            part.l[row] = total;
        }
        const float inv = inverse(total);
        uint16_t *out = out_row(a, it, row0 + row, group);
        for (int d = 2 * lane; d < D; d += 128) {
            float o0 = 0.f, o1 = 0.f;
#pragma unroll
            for (int w = 0; w < ATTN_WAVES; ++w) {
                o0 += f[w] * lds_o[w][row][d];
                o1 += f[w] * lds_o[w][row][d + 1];
            }
            if (whole)
                *(uint32_t *)(out + d) = pack2<BF>(o0 * inv, o1 * inv);
            else
                *(float2 *)&part.o[row][d] = make_float2(o0, o1);
        }
    }
    __syncthreads();
    u = stop;
    }
}

constexpr int JOIN_ROWS = 4, JOIN_WAVES = 4, JOIN_THREADS = 64 * JOIN_WAVES;

// Joins the parts of a divided item: workgroup (i, y) takes rows JOIN_ROWS y ..
// of the item that cut i + 1 divides first.  Wavefront w first works out the
// factors of row w's parts, a part a lane; then the wavefronts share the parts
// of all rows among them, so that many loads are in flight, and meet in LDS.
template <int DP, int NT, bool BF>
__global__ void __launch_bounds__(JOIN_THREADS) attn_join_kernel(AttnArgs a)
{
    constexpr int ROWS = 16 * NT;
    static_assert(JOIN_ROWS == JOIN_WAVES && ROWS % JOIN_ROWS == 0, "a row's factors per wavefront");
    __shared__ long long chunk[JOIN_THREADS + 1], scratch[2 * JOIN_WAVES];
    __shared__ float factor[SPLITS][JOIN_ROWS], total[JOIN_ROWS];
    __shared__ float2 sum[JOIN_WAVES][JOIN_ROWS][64];
    const Line line = lay_out<ROWS, JOIN_THREADS>(a, chunk, scratch);
    if ((int)blockIdx.x + 1 >= ranges(line.total))
        return;
    const long long u = cut(line.total, blockIdx.x + 1);
    const Item it = item_at<ROWS, JOIN_THREADS>(a, line, chunk, u);
    if (u == it.start || cut(line.total, blockIdx.x) > it.start)
        return;
    const int group = a.heads / a.kv.kv_heads, row0 = it.block * ROWS + blockIdx.y * JOIN_ROWS;
    const int rows = min(it.rq.n * group - row0, JOIN_ROWS);
    if (rows <= 0)
        return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int w0 = range_of(line.total, it.start), n = range_of(line.total, it.start + it.units - 1) - w0 + 1;
    // the first part is its range's second segment unless it starts with it
    const Part<ROWS, DP> *parts = (const Part<ROWS, DP> *)a.workspace + 2 * w0;
    const int second = cut(line.total, w0) < it.start;
    auto part = [&](int k) -> const Part<ROWS, DP> & { return parts[k ? 2 * k : second]; };

    const int row = blockIdx.y * JOIN_ROWS + wave;
    if (wave < rows) {
        float m[SPLITS / 64], top = NO_SCORE, t = 0.f;
#pragma unroll
        for (int i = 0; i < SPLITS / 64; ++i) {
            m[i] = 64 * i + lane < n ? part(64 * i + lane).m[row] : NO_SCORE;
            top = fmaxf(top, m[i]);
        }
#pragma unroll
        for (int s = 32; s; s >>= 1)
            top = fmaxf(top, __shfl_xor(top, s));
#pragma unroll
        for (int i = 0; i < SPLITS / 64; ++i) {
            const int k = 64 * i + lane;
            if (k < n) {
                const float f = exp2f(m[i] - top);
                factor[k][wave] = f;
                t += f * part(k).l[row];
            }
        }
#pragma unroll
        for (int s = 32; s; s >>= 1)
            t += __shfl_xor(t, s);
        if (lane == 0)
            total[wave] = t;
    }
    __syncthreads();

    const int D = a.kv.head_dim, d = 2 * lane < D ? 2 * lane : 0;
    float2 o[JOIN_ROWS] = {};
#pragma unroll 4
    for (int k = wave; k < n; k += JOIN_WAVES) {
        const Part<ROWS, DP> &p = part(k);
#pragma unroll
        for (int r = 0; r < JOIN_ROWS; ++r) {
            const int rr = min(r, rows - 1);
            const float2 v = *(const float2 *)&p.o[blockIdx.y * JOIN_ROWS + rr][d];
            o[r].x += factor[k][rr] * v.x;
            o[r].y += factor[k][rr] * v.y;
        }
    }
#pragma unroll
    for (int r = 0; r < JOIN_ROWS; ++r)
        sum[wave][r][lane] = o[r];
    __syncthreads();
    if (wave < rows && 2 * lane < D) {
        float2 v = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < JOIN_WAVES; ++w) {
            v.x += sum[w][wave][lane].x;
            v.y += sum[w][wave][lane].y;
        }
        const float inv = inverse(total[wave]);
        *(uint32_t *)(out_row(a, it, row0 + wave, group) + 2 * lane) = pack2<BF>(v.x * inv, v.y * inv);
    }
}

template <int DP, int DS, int NT, bool BF>
int go_attn(const AttnArgs &a, hipStream_t stream)
{
    AttnArgs args = a;
    void *argv[] = {&args};
    const int st = launch_kernel((const void *)attn_kernel<DP, DS, NT, BF>, dim3(SPLITS), dim3(ATTN_THREADS), 0, stream,
                                 argv);
    if (st != SBVR_OK)
        return st;
    const int rows = min(a.max_new * (a.heads / a.kv.kv_heads), 16 * NT);
    return launch_kernel((const void *)attn_join_kernel<DP, NT, BF>,
                         dim3(SPLITS - 1, (rows + JOIN_ROWS - 1) / JOIN_ROWS), dim3(JOIN_THREADS), 0, stream, argv);
}

// rows per item: as many as the call can have, up to 32
int row_tiles(int max_new, int heads, int kv_heads) { return max_new * (heads / kv_heads) <= 16 ? 1 : 2; }

template <int DP, int DS>
int by_type(const AttnArgs &a, hipStream_t stream)
{
    const bool bf = a.kv.dtype == SBVR_BF16;
    if (row_tiles(a.max_new, a.heads, a.kv.kv_heads) == 1)
        return bf ? go_attn<DP, DS, 1, true>(a, stream) : go_attn<DP, DS, 1, false>(a, stream);
    return bf ? go_attn<DP, DS, 2, true>(a, stream) : go_attn<DP, DS, 2, false>(a, stream);
}

size_t attn_workspace_bytes(int, int max_new, int heads, int kv_heads, int head_dim)
{
    const bool narrow = head_dim <= 64;
    if (row_tiles(max_new, heads, kv_heads) == 1)
        return 2 * SPLITS * (narrow ? sizeof(Part<16, 64>) : sizeof(Part<16, 128>));
    return 2 * SPLITS * (narrow ? sizeof(Part<32, 64>) : sizeof(Part<32, 128>));
}

int launch_attn(const AttnArgs &a, hipStream_t stream)
{
    if (a.kv.head_dim <= 64)
        return by_type<64, 2>(a, stream);
    if (a.kv.head_dim <= 96)
        return by_type<128, 3>(a, stream);
    return by_type<128, 4>(a, stream);
}

}  // namespace sbvr
