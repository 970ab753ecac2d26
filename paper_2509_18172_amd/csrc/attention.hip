// Attention of a step's tokens over a paged key/value cache (tree attention).
//
// The rows of a key/value head are the request's new tokens times the query
// heads that share it; a block of them is one item.  Everything is computed
// transposed, on v_mfma_f32_16x16x32: S^T = K Q^T gives a lane four positions
// of one row, so a row's maximum and sum are mostly within lanes, and
// exp(S^T) is, unmoved, the operand of O^T = V^T P^T: its slot e of lane group
// g = lane / 16 stands for position 4g + e (e < 4) and 16 + 4g + e - 4 of a
// 32-position tile, and the V operand is laid out the same way.
//   K: lane (c = lane % 16, g) holds position c, elements 32 s + 8 g .. + 7.
//   V: lane (c, g) holds elements DV c .. DV c + DV - 1 (DV = DP / 16) of its
//      eight positions; row c of operand q is element DV c + q, picked from
//      the eight rows with byte permutes.
// head_dim below DP: lanes past the end read piece 0 instead; their Q is zero
// and their outputs are not stored.
//
// Two kernels, by the rows of an item:
//   attn_rows_kernel (up to 32 rows): memory-bound.  Each wavefront streams
//     tiles of its own straight into operand registers; K's registers are
//     refilled for the next tile as soon as the scores are formed and V's as
//     soon as the products are, so each is in flight while the other is used.
//     The four wavefronts' sums meet in LDS at the end.
//   attn_block_kernel (up to 128 rows): each wavefront has 16 or 32 rows of its
//     own and all four share the tiles, which go through LDS once for all of
//     them, one tile ahead; pieces are stored permuted so that both operands'
//     reads are free of bank conflicts.
//
// Work: the cached positions of all items, in units of one step of a
// workgroup, are one line that is cut into (up to) SPLITS equal ranges,
// whatever the requests' lengths; a workgroup runs the segments of items in
// its range.  An item within one range is finished there; of an item that a
// cut divides, every workgroup leaves its unnormalised sums, and a second
// kernel joins them.  Which workgroup has what follows from the lengths alone.
//
// A row's running maximum is moved only when a score passes it by 2^GAP: the
// weights then stay within the 16-bit types' range, sums and products are
// binary32, and most tiles need neither the maximum over lanes nor the
// rescaling of the sums.
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
constexpr int TILE = 32;              // positions of one score / product step
constexpr int SPLITS = 512;           // ranges: two workgroups a CU
constexpr float NO_SCORE = -1.0e30f;  // running maximum before any score
constexpr float GAP = 8.f;            // binary exponent by which weights may exceed 1
constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

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

// ---------------------------------------------------------------------------
// the line of work
// ---------------------------------------------------------------------------

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
struct Item {
    int r, kvh, block;
    Request rq;
    long long start;  // first unit
    int units;
};

template <int ROWS>
__device__ __forceinline__ int row_blocks(const AttnArgs &a, const Request &q)
{
    return (q.n * (a.heads / a.kv.kv_heads) + ROWS - 1) / ROWS;
}

// Up to 64 requests: a lane each, in every wavefront by itself.  More: each
// thread sums up a run of them, the workgroup scans the runs.
template <int ROWS, int UNIT>
struct Line {
    long long total;
    const AttnArgs &a;
    const long long *runs;  // LDS [ATTN_THREADS + 1]; unused up to 64 requests
    int per;
    Request mine;
    long long before;

    __device__ static long long units_of(const AttnArgs &a, const Request &q)
    {
        return (long long)((q.ctx + q.n + UNIT - 1) / UNIT) * row_blocks<ROWS>(a, q) * a.kv.kv_heads;
    }

    __device__ Line(const AttnArgs &a_, long long *lds, long long *scratch) : a(a_), runs(lds)
    {
        if (a.R <= 64) {
            const int lane = threadIdx.x & 63;
            mine = request_of(a, min(lane, a.R - 1));
            const long long own = lane < a.R ? units_of(a, mine) : 0;
            long long sum = own;
#pragma unroll
            for (int s = 1; s < 64; s <<= 1) {
                const long long p = __shfl_up(sum, s);
                if (lane >= s)
                    sum += p;
            }
            before = sum - own;
            total = __shfl(sum, 63);
            return;
        }
        per = (a.R + ATTN_THREADS - 1) / ATTN_THREADS;
        long long units = 0, none = 0, zero;
        const int r0 = threadIdx.x * per, r1 = min(r0 + per, a.R);
        for (int r = r0; r < r1; ++r)
            units += units_of(a, request_of(a, r));
        scan_pair<ATTN_THREADS>(units, none, total, zero, scratch);
        lds[threadIdx.x] = units;
        if (threadIdx.x == 0)
            lds[ATTN_THREADS] = total;
        __syncthreads();
    }

    // the item that holds unit u (the same in every lane)
    __device__ Item item_at(long long u) const
    {
        Item it;
        long long base;
        if (a.R <= 64) {
            it.r = 63 - __builtin_clzll(__ballot((threadIdx.x & 63) < (unsigned)a.R && before <= u));
            it.rq.ctx = __builtin_amdgcn_readlane(mine.ctx, it.r);
            it.rq.n = __builtin_amdgcn_readlane(mine.n, it.r);
            it.rq.first = __builtin_amdgcn_readlane(mine.first, it.r);
            base = (long long)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(before >> 32), it.r) << 32) |
                               (uint32_t)__builtin_amdgcn_readlane((int)before, it.r));
        } else {
            const int i = owner_of(runs, ATTN_THREADS, u);
            base = runs[i];
            for (it.r = i * per;; ++it.r) {
                it.rq = request_of(a, it.r);
                const long long all = units_of(a, it.rq);
                if (u < base + all || it.r + 1 >= a.R)
                    break;
                base += all;
            }
            it.r = __builtin_amdgcn_readfirstlane(it.r);
            it.rq.ctx = __builtin_amdgcn_readfirstlane(it.rq.ctx);
            it.rq.n = __builtin_amdgcn_readfirstlane(it.rq.n);
            it.rq.first = __builtin_amdgcn_readfirstlane(it.rq.first);
        }
        it.units = (it.rq.ctx + it.rq.n + UNIT - 1) / UNIT;
        const int blocks = row_blocks<ROWS>(a, it.rq);
        const uint32_t k = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)(u - base) / (uint32_t)it.units));
        it.start = base + (long long)k * it.units;
        it.kvh = k / blocks;
        it.block = k % blocks;
        return it;
    }
};

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

// The workspace: what the join of cut i has to do (parts 0: nothing; the first
// cut that divides an item does it), then the parts -- the range's own part
// 2 i for its first segment, 2 i + 1 for another (only its last can be divided
// too).
struct Join {
    int parts, range, second;  // parts of the item, the first one's range and whether it is its second
    int rows, row0, first, kvh;
    int unused;
};

template <int ROWS, int DP>
struct Part {
    float o[ROWS][DP];
    float m[ROWS], l[ROWS];
};

template <int ROWS, int DP>
struct Workspace {
    Join join[SPLITS];
    Part<ROWS, DP> part[2 * SPLITS];
};

// Start of a workgroup's segment: its item, its positions, and, at the range's
// start, the join that its cut asks for.
template <int ROWS, int UNIT>
__device__ __forceinline__ Item open_segment(const Line<ROWS, UNIT> &line, long long u, long long u0, Join *join,
                                             const AttnArgs &a)
{
    const Item it = line.item_at(u);
    if (u == u0 && threadIdx.x == 0) {
        Join j = {};
        const int i = blockIdx.x;
        if (i > 0 && u > it.start && cut(line.total, i - 1) <= it.start) {
            j.range = range_of(line.total, it.start);
            j.parts = range_of(line.total, it.start + it.units - 1) - j.range + 1;
            j.second = cut(line.total, j.range) < it.start;
            j.row0 = it.block * ROWS;
            j.rows = min(it.rq.n * (a.heads / a.kv.kv_heads) - j.row0, ROWS);
            j.first = it.rq.first;
            j.kvh = it.kvh;
        }
        join[i] = j;
    }
    return it;
}

__device__ __forceinline__ uint16_t *out_row(const AttnArgs &a, int first, int kvh, int row, int group)
{
    const int tok = first + row / group, head = kvh * group + row % group;
    return (uint16_t *)a.out + ((long long)tok * a.heads + head) * a.kv.head_dim;
}

__device__ __forceinline__ float inverse(float total)  // 0 for a row that saw nothing; NaN stays
{
    return total == 0.f ? 0.f : 1.f / total;
}

// ---------------------------------------------------------------------------
// one tile
// ---------------------------------------------------------------------------

// A wavefront's 16 NT rows, c of each sixteen in lanes (c, *).
template <int DP, int DS, int NT, bool BF>
struct Rows {
    static constexpr int DV = DP / 16;
    v4u q[NT][DS];
    uint64_t mask[NT];
    v4f acc[NT][DV];
    float m[NT], l[NT];
    float scale2;

    // rows row0 .. row0 + rows - 1 of the item; the scale's sign goes into Q,
    // and a scale of zero too, so that masked scores stay -infinity
    __device__ __forceinline__ void open(const AttnArgs &a, const Item &it, int row0, int rows, int group)
    {
        const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4, pieces = a.kv.head_dim / 8;
        const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u, keep = a.scale == 0.f ? 0u : ~0u;
        scale2 = a.scale == 0.f ? 1.f : fabsf(a.scale) * LOG2E;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const bool ok = 16 * nt + c < rows;
            const int row = ok ? row0 + 16 * nt + c : row0;
            const int tok = it.rq.first + row / group, head = it.kvh * group + row % group;
            const uint16_t *p = (const uint16_t *)a.q + tok * a.q_token_stride + head * a.q_head_stride;
            mask[nt] = ok ? a.tree_mask[tok] : 0;
#pragma unroll
            for (int s = 0; s < DS; ++s) {
                const int piece = 4 * s + g;
                q[nt][s] = v4u{0, 0, 0, 0};
                if (ok && piece < pieces)
                    q[nt][s] = (*(const v4u *)(p + 8 * piece) ^ flip) & keep;
            }
            m[nt] = NO_SCORE;
            l[nt] = 0.f;
#pragma unroll
            for (int i = 0; i < DV; ++i)
                acc[nt][i] = v4f{0.f, 0.f, 0.f, 0.f};
        }
    }

    __device__ __forceinline__ void scores(const v4u (&k)[2][DS], v4f (&s)[NT][2])
    {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                s[nt][h] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int d = 0; d < DS; ++d)
                    s[nt][h] = mfma<BF>(k[h][d], q[nt][d], s[nt][h]);
            }
    }

    // Masks the tile at p0: scores of what a row does not see, and the values
    // of positions that are not there.  True where values of the step's own
    // tokens are not finite (the same in every lane).
    __device__ __forceinline__ bool hide(int p0, bool ok0, bool ok1, const Request &rq, v4f (&s)[NT][2],
                                         uint32_t (&v)[8][DV / 2])
    {
        const int g = (threadIdx.x & 63) >> 4;
        bool odd_values = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int p = p0 + 16 * (e / 4) + 4 * g + e % 4, j = p - rq.ctx;
            const bool there = j < rq.n && (e / 4 ? ok1 : ok0);
            bool odd = false;
#pragma unroll
            for (int i = 0; i < DV / 2; ++i) {
                if (!there)
                    v[e][i] = 0;
                odd |= not_finite<BF>(v[e][i]);
            }
            odd_values |= odd && j >= 0;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const bool seen = there && (j < 0 || ((mask[nt] >> (j & 63)) & 1));
                if (!seen)
                    s[nt][e / 4][e % 4] = -INFINITY;
            }
        }
        return __ballot(odd_values) != 0;
    }

    // weights of the tile, as the products' operand
    __device__ __forceinline__ void weights(const v4f (&s)[NT][2], v4u (&pf)[NT])
    {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float top = fmaxf(fmaxf(fmaxf(s[nt][0][0], s[nt][0][1]), fmaxf(s[nt][0][2], s[nt][0][3])),
                              fmaxf(fmaxf(s[nt][1][0], s[nt][1][1]), fmaxf(s[nt][1][2], s[nt][1][3])));
            top *= scale2;
            if (__ballot(top > m[nt] + GAP)) {
                top = fmaxf(max4(top), m[nt]);
                const float keep = fast_exp2(m[nt] - top);
                m[nt] = top;
                l[nt] *= keep;
#pragma unroll
                for (int i = 0; i < DV; ++i)
                    acc[nt][i] *= keep;
            }
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = fast_exp2(fmaf(s[nt][e / 4][e % 4], scale2, -m[nt]));
            l[nt] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
            for (int i = 0; i < 4; ++i)
                pf[nt][i] = pack2<BF>(x[2 * i], x[2 * i + 1]);
        }
    }

    // Values of the step's own tokens that are not finite: their products are
    // added one by one to the rows that see them, and 0 stands in their place
    // in the operand.  value(p): position p's values.
    template <typename F>
    __device__ __forceinline__ void odd_products(int p0, bool ok0, bool ok1, const AttnArgs &a, const Request &rq,
                                                 const v4u (&pf)[NT], uint32_t (&v)[8][DV / 2], F value)
    {
        const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
#pragma unroll 1
        for (int e = 0; e < 8; ++e)
#pragma unroll 1
            for (int gg = 0; gg < 4; ++gg) {
                const int p = p0 + 16 * (e / 4) + 4 * gg + e % 4, j = p - rq.ctx;
                if (j >= rq.n || j < 0 || !(e / 4 ? ok1 : ok0))
                    continue;
                const uint16_t *row = value(p);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint32_t w = e / 2 == 0   ? pf[nt][0]
                                       : e / 2 == 1 ? pf[nt][1]
                                       : e / 2 == 2 ? pf[nt][2]
                                                    : pf[nt][3];
                    const float weight = unpack<BF>(__shfl(w, 16 * gg + c), e & 1);
                    const bool seen = (mask[nt] >> j) & 1;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int d = DV * (4 * g + i);
                        if (d >= a.kv.head_dim)
                            continue;
                        const Halves<DV> piece = *(const Halves<DV> *)(row + d);
#pragma unroll
                        for (int q = 0; q < DV; ++q) {
                            const uint32_t bits = q & 1 ? piece.w[q / 2] >> 16 : piece.w[q / 2] & 0xffffu;
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
                if (not_finite<BF>(v[e][i] & 0xffffu))
                    v[e][i] &= 0xffff0000u;
                if (not_finite<BF>(v[e][i] >> 16))
                    v[e][i] &= 0xffffu;
            }
        }
    }

    __device__ __forceinline__ void products(const v4u (&pf)[NT], const uint32_t (&v)[8][DV / 2])
    {
#pragma unroll
        for (int i = 0; i < DV; ++i) {
            v4u vf;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                vf[e] = __builtin_amdgcn_perm(v[2 * e + 1][i / 2], v[2 * e][i / 2], i & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                acc[nt][i] = mfma<BF>(vf, pf[nt], acc[nt][i]);
        }
    }

    __device__ __forceinline__ float row_sum(int nt) const
    {
        float t = l[nt] + __shfl_xor(l[nt], 16);
        return t + __shfl_xor(t, 32);
    }
};

// Uniform address of position p of a page plus a 32-bit lane offset is what
// every load uses.
__device__ __forceinline__ const char *at_page(const void *base, int page, int p, int page_size, int64_t page_stride,
                                               uint32_t step)
{
    const uint32_t off = (uint32_t)p & (page_size - 1);
    return (const char *)base + 2 * (long long)max(page, 0) * page_stride + (uint64_t)off * step;
}

// The page of the sixteen positions at p (a page holds whole sixteens); -1:
// past the end or outside the cache, read from page 0 and masked.
__device__ __forceinline__ int page_at(const AttnArgs &a, const int32_t *table, int p, int end, int page_shift)
{
    p = __builtin_amdgcn_readfirstlane(p);
    const int id = p < end ? table[p >> page_shift] : -1;
    return __builtin_amdgcn_readfirstlane(id < a.kv.n_pages ? max(id, -1) : -1);
}

// ---------------------------------------------------------------------------
// items of few rows
// ---------------------------------------------------------------------------

// DP: padded head size, DS: 32-element steps of it that hold elements, NT:
// 16-row tiles per item, BF: bfloat16.
template <int DP, int DS, int NT, bool BF>
__global__ void __launch_bounds__(ATTN_THREADS, 2) attn_rows_kernel(AttnArgs a)
{
    constexpr int DV = DP / 16, ROWS = 16 * NT, UNIT = ATTN_WAVES * TILE;
    __shared__ float lds_o[ATTN_WAVES][ROWS][DP + 4];
    __shared__ float lds_m[ATTN_WAVES][ROWS], lds_l[ATTN_WAVES][ROWS];
    __shared__ long long runs[ATTN_THREADS + 1], scratch[2 * ATTN_WAVES];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int group = a.heads / a.kv.kv_heads;
    const int D = a.kv.head_dim, pieces = D / 8;
    const int page_shift = __builtin_ctz(a.kv.page_size);
    Workspace<ROWS, DP> &ws = *(Workspace<ROWS, DP> *)a.workspace;
    const Line<ROWS, UNIT> line(a, runs, scratch);
    if ((int)blockIdx.x >= ranges(line.total)) {
        if (threadIdx.x == 0)
            ws.join[blockIdx.x].parts = 0;
        return;
    }
    const long long u0 = cut(line.total, blockIdx.x), u1 = cut(line.total, blockIdx.x + 1);
    const uint32_t k_step = 2 * (uint32_t)a.kv.k_token_stride, v_step = 2 * (uint32_t)a.kv.v_token_stride;
    const uint32_t k_lane = c * k_step, v_lane = 4 * g * v_step + 2 * (DV * c < D ? DV * c : 0);

    for (long long u = u0; u < u1;) {
        const Item it = open_segment(line, u, u0, ws.join, a);
        const Request &rq = it.rq;
        const int row0 = it.block * ROWS, rows = min(rq.n * group - row0, ROWS), end = rq.ctx + rq.n;
        const long long stop = min(u1, it.start + it.units);
        const bool whole = u == it.start && stop == it.start + it.units;
        const int first = (int)(u - it.start) * UNIT + wave * TILE, last = min((int)(stop - it.start) * UNIT, end);
        const int32_t *table = a.page_table + it.r * a.table_stride;
        const uint16_t *kb = (const uint16_t *)a.kv.k + it.kvh * a.kv.k_head_stride;
        const uint16_t *vb = (const uint16_t *)a.kv.v + it.kvh * a.kv.v_head_stride;

        v4u kf[2][DS];
        uint32_t vr[8][DV / 2];
        auto load_k = [&](int p0, const int *page) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const char *kp = at_page(kb, page[h], p0 + 16 * h, a.kv.page_size, a.kv.k_page_stride, k_step);
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
                const char *vp = at_page(vb, page[h], p0 + 16 * h, a.kv.page_size, a.kv.v_page_stride, v_step);
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
        auto pages_of = [&](int p0, int *id) {
            id[0] = page_at(a, table, p0, end, page_shift);
            id[1] = page_at(a, table, p0 + 16, end, page_shift);
        };
        if (first < last) {
            pages_of(first, page);
            load_k(first, page);
            load_v(first, page);
        }
        Rows<DP, DS, NT, BF> row;
        row.open(a, it, row0, rows, group);
        for (int p0 = first; p0 < last; p0 += UNIT) {
            const bool more = p0 + UNIT < last;
            if (more)
                pages_of(p0 + UNIT, next);
            v4f s[NT][2];
            row.scores(kf, s);
            if (more)
                load_k(p0 + UNIT, next);
            bool odd = false;
            if (p0 + TILE > rq.ctx || (page[0] | page[1]) < 0)
                odd = row.hide(p0, page[0] >= 0, page[1] >= 0, rq, s, vr);
            v4u pf[NT];
            row.weights(s, pf);
            if (odd)
                row.odd_products(p0, page[0] >= 0, page[1] >= 0, a, rq, pf, vr, [&](int p) {
                    const int id = p - p0 < 16 ? page[0] : page[1];
                    return (const uint16_t *)at_page(vb, id, p, a.kv.page_size, a.kv.v_page_stride, v_step);
                });
            row.products(pf, vr);
            if (more) {
                load_v(p0 + UNIT, next);
                page[0] = next[0];
                page[1] = next[1];
            }
        }

        // the wavefronts' parts meet in LDS
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float l = row.row_sum(nt);
            if (g == 0) {
                lds_m[wave][16 * nt + c] = row.m[nt];
                lds_l[wave][16 * nt + c] = l;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int q = 0; q < DV; ++q)
                    lds_o[wave][16 * nt + c][DV * (4 * g + i) + q] = row.acc[nt][q][i];
        }
        __syncthreads();
        Part<ROWS, DP> &part = ws.part[2 * blockIdx.x + (u != u0)];
        for (int i = wave; i < rows; i += ATTN_WAVES) {
            float top = NO_SCORE;
#pragma unroll
            for (int w = 0; w < ATTN_WAVES; ++w)
                top = fmaxf(top, lds_m[w][i]);
            float f[ATTN_WAVES], total = 0.f;
#pragma unroll
            for (int w = 0; w < ATTN_WAVES; ++w) {
                f[w] = fast_exp2(lds_m[w][i] - top);
                total += f[w] * lds_l[w][i];
            }
            if (!whole && lane == 0) {
                part.m[i] = top;
                part.l[i] = total;
            }
            const float inv = inverse(total);
            if (2 * lane < D) {
                float o0 = 0.f, o1 = 0.f;
#pragma unroll
                for (int w = 0; w < ATTN_WAVES; ++w) {
                    o0 += f[w] * lds_o[w][i][2 * lane];
                    o1 += f[w] * lds_o[w][i][2 * lane + 1];
                }
                if (whole)
                    *(uint32_t *)(out_row(a, rq.first, it.kvh, row0 + i, group) + 2 * lane) =
                        pack2<BF>(o0 * inv, o1 * inv);
                else
                    *(float2 *)&part.o[i][2 * lane] = make_float2(o0, o1);
            }
        }
        __syncthreads();
        u = stop;
    }
}

// ---------------------------------------------------------------------------
// items of many rows
// ---------------------------------------------------------------------------

template <int DP, int DS, int NT, bool BF>
__global__ void __launch_bounds__(ATTN_THREADS, 2) attn_block_kernel(AttnArgs a)
{
    constexpr int DV = DP / 16, WROWS = 16 * NT, ROWS = WROWS * ATTN_WAVES, UNIT = 64;
    constexpr int PIECES = DP / 8;         // 16-byte pieces of a stored row
    constexpr int LOADS = UNIT * PIECES / ATTN_THREADS;  // per thread, of keys and of values
    constexpr int LOAD_ROWS = 64 / PIECES; // rows that one load of a wavefront covers
    __shared__ v4u tile[2][2][UNIT][PIECES];  // [buffer][keys, values][position][piece, permuted]
    __shared__ long long runs[ATTN_THREADS + 1], scratch[2 * ATTN_WAVES];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int group = a.heads / a.kv.kv_heads;
    const int D = a.kv.head_dim, pieces = D / 8;
    const int page_shift = __builtin_ctz(a.kv.page_size);
    Workspace<ROWS, DP> &ws = *(Workspace<ROWS, DP> *)a.workspace;
    const Line<ROWS, UNIT> line(a, runs, scratch);
    if ((int)blockIdx.x >= ranges(line.total)) {
        if (threadIdx.x == 0)
            ws.join[blockIdx.x].parts = 0;
        return;
    }
    const long long u0 = cut(line.total, blockIdx.x), u1 = cut(line.total, blockIdx.x + 1);
    const uint32_t k_step = 2 * (uint32_t)a.kv.k_token_stride, v_step = 2 * (uint32_t)a.kv.v_token_stride;

    // Piece j of stored row r lies at j ^ swap(r): sixteen lanes that read one
    // piece of sixteen rows, or the pieces of one row, meet all banks once.
    auto swap = [](int r) { return PIECES == 16 ? r & 15 : (r >> 1) & 7; };

    // Wavefront w brings in positions 16 w .. 16 w + 15 of a unit, LOAD_ROWS a
    // load; lane -> (row of the load, piece).
    const int load_row = lane / PIECES, load_piece = lane % PIECES;
    const int from = load_piece < pieces ? load_piece : 0;
    const uint32_t k_lane = load_row * k_step + 16 * from, v_lane = load_row * v_step + 16 * from;

    for (long long u = u0; u < u1;) {
        const Item it = open_segment(line, u, u0, ws.join, a);
        const Request &rq = it.rq;
        const int row0 = it.block * ROWS + wave * WROWS, rows = min(max(rq.n * group - row0, 0), WROWS);
        const int end = rq.ctx + rq.n;
        const long long stop = min(u1, it.start + it.units);
        const bool whole = u == it.start && stop == it.start + it.units;
        const int first = (int)(u - it.start) * UNIT, last = min((int)(stop - it.start) * UNIT, end);
        const int32_t *table = a.page_table + it.r * a.table_stride;
        const uint16_t *kb = (const uint16_t *)a.kv.k + it.kvh * a.kv.k_head_stride;
        const uint16_t *vb = (const uint16_t *)a.kv.v + it.kvh * a.kv.v_head_stride;

        v4u kin[LOADS], vin[LOADS];
        // brings in the unit at p0 and says which of its four sixteens are there
        auto load = [&](int p0) {
            int ok = 0, mine = -1;
#pragma unroll
            for (int w = 0; w < ATTN_WAVES; ++w) {
                const int id = page_at(a, table, p0 + 16 * w, end, page_shift);
                ok |= (id >= 0) << w;
                mine = w == wave ? id : mine;
            }
            const char *kp = at_page(kb, mine, p0 + 16 * wave, a.kv.page_size, a.kv.k_page_stride, k_step);
            const char *vp = at_page(vb, mine, p0 + 16 * wave, a.kv.page_size, a.kv.v_page_stride, v_step);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                kin[i] = *(const v4u *)(kp + (uint64_t)(i * LOAD_ROWS * k_step) + (uint64_t)k_lane);
                vin[i] = *(const v4u *)(vp + (uint64_t)(i * LOAD_ROWS * v_step) + (uint64_t)v_lane);
            }
            return ok;
        };
        auto store = [&](int buffer) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int r = 16 * wave + i * LOAD_ROWS + load_row;
                tile[buffer][0][r][load_piece ^ swap(r)] = kin[i];
                tile[buffer][1][r][load_piece ^ swap(r)] = vin[i];
            }
        };

        int there = load(first), coming = 0;
        Rows<DP, DS, NT, BF> row;
        row.open(a, it, rows ? row0 : it.block * ROWS, rows, group);
        store(0);
        if (first + UNIT < last)
            coming = load(first + UNIT);
        __syncthreads();
        int buffer = 0;
        for (int p0 = first; p0 < last; p0 += UNIT) {
#pragma unroll 1
            for (int t = 0; t < UNIT / TILE; ++t) {
                const int pt = p0 + t * TILE;
                if (pt >= end || rows == 0)
                    continue;
                v4u kf[2][DS];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int s = 0; s < DS; ++s) {
                        const int r = t * TILE + 16 * h + c;
                        kf[h][s] = tile[buffer][0][r][(4 * s + g) ^ swap(r)];
                    }
                v4f s[NT][2];
                row.scores(kf, s);
                uint32_t vr[8][DV / 2];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int r = t * TILE + 16 * (e / 4) + 4 * g + e % 4;
                    const char *p = (const char *)tile[buffer][1][r];
                    const Halves<DV> v = *(const Halves<DV> *)(p + 16 * ((DV * c / 8) ^ swap(r)) + 2 * (DV * c % 8));
#pragma unroll
                    for (int i = 0; i < DV / 2; ++i)
                        vr[e][i] = v.w[i];
                }
                const bool ok0 = (there >> (2 * t)) & 1, ok1 = (there >> (2 * t + 1)) & 1;
                bool odd = false;
                if (pt + TILE > rq.ctx || !ok0 || !ok1)
                    odd = row.hide(pt, ok0, ok1, rq, s, vr);
                v4u pf[NT];
                row.weights(s, pf);
                if (odd)
                    row.odd_products(pt, ok0, ok1, a, rq, pf, vr, [&](int p) {
                        return (const uint16_t *)at_page(vb, table[p >> page_shift], p, a.kv.page_size,
                                                         a.kv.v_page_stride, v_step);
                    });
                row.products(pf, vr);
            }
            if (p0 + UNIT < last) {
                // the other buffer was last read before the barrier at the end
                // of the step before
                store(buffer ^ 1);
                there = coming;
                if (p0 + 2 * UNIT < last)
                    coming = load(p0 + 2 * UNIT);
            }
            buffer ^= 1;
            __syncthreads();
        }

        Part<ROWS, DP> &part = ws.part[2 * blockIdx.x + (u != u0)];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float total = row.row_sum(nt), inv = inverse(total);
            const int i = 16 * nt + c;
            if (i >= rows)
                continue;
            if (!whole && g == 0) {
                part.m[wave * WROWS + i] = row.m[nt];
                part.l[wave * WROWS + i] = total;
            }
            uint16_t *out = out_row(a, rq.first, it.kvh, row0 + i, group);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int d = DV * (4 * g + j);
                if (d >= D)
                    continue;
                if (whole) {
                    Halves<DV> o;
#pragma unroll
                    for (int q = 0; q < DV; q += 2)
                        o.w[q / 2] = pack2<BF>(row.acc[nt][q][j] * inv, row.acc[nt][q + 1][j] * inv);
                    *(Halves<DV> *)(out + d) = o;
                } else {
#pragma unroll
                    for (int q = 0; q < DV; q += 4)
                        *(v4f *)&part.o[wave * WROWS + i][d + q] = v4f{row.acc[nt][q][j], row.acc[nt][q + 1][j],
                                                                       row.acc[nt][q + 2][j], row.acc[nt][q + 3][j]};
                }
            }
        }
        u = stop;
    }
}

// ---------------------------------------------------------------------------
// the join
// ---------------------------------------------------------------------------

constexpr int JOIN_ROWS = 4, JOIN_WAVES = 4, JOIN_THREADS = 64 * JOIN_WAVES, JOIN_GROUPS = 8;

// Joins the parts of a divided item: workgroup (i, y) takes rows JOIN_ROWS y ..
// (and on, JOIN_GROUPS apart) of the item that cut i + 1 divides first.
// Wavefront w first works out the factors of row w's parts, a part a lane;
// then the wavefronts share the parts of all rows among them, so that many
// loads are in flight, and meet in LDS.
template <int DP, int ROWS, bool BF>
__global__ void __launch_bounds__(JOIN_THREADS) attn_join_kernel(AttnArgs a)
{
    static_assert(JOIN_ROWS == JOIN_WAVES && ROWS % JOIN_ROWS == 0, "a row's factors per wavefront");
    __shared__ float factor[SPLITS][JOIN_ROWS], total[JOIN_ROWS];
    __shared__ float2 sum[JOIN_WAVES][JOIN_ROWS][64];
    const Workspace<ROWS, DP> &ws = *(const Workspace<ROWS, DP> *)a.workspace;
    const Join j = ws.join[blockIdx.x + 1];
    if (j.parts == 0)
        return;
    const int group = a.heads / a.kv.kv_heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = j.parts;
    const Part<ROWS, DP> *parts = ws.part + 2 * j.range;
    auto part = [&](int k) -> const Part<ROWS, DP> & { return parts[k ? 2 * k : j.second]; };
    const int D = a.kv.head_dim, d = 2 * lane < D ? 2 * lane : 0;

    for (int i0 = blockIdx.y * JOIN_ROWS; i0 < j.rows; i0 += JOIN_GROUPS * JOIN_ROWS) {
        const int rows = min(j.rows - i0, JOIN_ROWS);
        if (wave < rows) {
            float top = NO_SCORE, t = 0.f;
            for (int k = lane; k < n; k += 64)
                top = fmaxf(top, part(k).m[i0 + wave]);
#pragma unroll
            for (int s = 32; s; s >>= 1)
                top = fmaxf(top, __shfl_xor(top, s));
            for (int k = lane; k < n; k += 64) {
                const float f = fast_exp2(part(k).m[i0 + wave] - top);
                factor[k][wave] = f;
                t += f * part(k).l[i0 + wave];
            }
#pragma unroll
            for (int s = 32; s; s >>= 1)
                t += __shfl_xor(t, s);
            if (lane == 0)
                total[wave] = t;
        }
        __syncthreads();

        float2 o[JOIN_ROWS] = {};
#pragma unroll 4
        for (int k = wave; k < n; k += JOIN_WAVES) {
            const Part<ROWS, DP> &p = part(k);
#pragma unroll
            for (int r = 0; r < JOIN_ROWS; ++r) {
                const int rr = min(r, rows - 1);
                const float2 v = *(const float2 *)&p.o[i0 + rr][d];
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
            *(uint32_t *)(out_row(a, j.first, j.kvh, j.row0 + i0 + wave, group) + 2 * lane) =
                pack2<BF>(v.x * inv, v.y * inv);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// launch
// ---------------------------------------------------------------------------

// How a call's items are run: rows of an item by the most rows that a request
// has per key/value head.
enum Shape { ROWS16, ROWS32, ROWS64, ROWS128 };

Shape shape_of(int max_new, int heads, int kv_heads)
{
    const int rows = max_new * (heads / kv_heads);
    return rows <= 16 ? ROWS16 : rows <= 32 ? ROWS32 : rows <= 64 ? ROWS64 : ROWS128;
}

int item_rows(Shape s) { return 16 << (int)s; }

template <int DP, int ROWS, bool BF>
int run_attn(const void *kernel, const AttnArgs &a, hipStream_t stream)
{
    AttnArgs args = a;
    void *argv[] = {&args};
    const int st = launch_kernel(kernel, dim3(SPLITS), dim3(ATTN_THREADS), 0, stream, argv);
    if (st != SBVR_OK)
        return st;
    const int groups = (min(a.max_new * (a.heads / a.kv.kv_heads), ROWS) + JOIN_ROWS - 1) / JOIN_ROWS;
    return launch_kernel((const void *)attn_join_kernel<DP, ROWS, BF>, dim3(SPLITS - 1, min(groups, JOIN_GROUPS)),
                         dim3(JOIN_THREADS), 0, stream, argv);
}

template <int DP, int DS, bool BF>
int by_shape(const AttnArgs &a, hipStream_t stream)
{
    switch (shape_of(a.max_new, a.heads, a.kv.kv_heads)) {
    case ROWS16: return run_attn<DP, 16, BF>((const void *)attn_rows_kernel<DP, DS, 1, BF>, a, stream);
    case ROWS32: return run_attn<DP, 32, BF>((const void *)attn_rows_kernel<DP, DS, 2, BF>, a, stream);
    case ROWS64: return run_attn<DP, 64, BF>((const void *)attn_block_kernel<DP, DS, 1, BF>, a, stream);
    default: return run_attn<DP, 128, BF>((const void *)attn_block_kernel<DP, DS, 2, BF>, a, stream);
    }
}

template <int DP, int DS>
int by_type(const AttnArgs &a, hipStream_t stream)
{
    return a.kv.dtype == SBVR_BF16 ? by_shape<DP, DS, true>(a, stream) : by_shape<DP, DS, false>(a, stream);
}

size_t attn_workspace_bytes(int, int max_new, int heads, int kv_heads, int head_dim)
{
    const size_t rows = item_rows(shape_of(max_new, heads, kv_heads)), dp = head_dim <= 64 ? 64 : 128;
    static_assert(sizeof(Workspace<16, 64>) == SPLITS * (sizeof(Join) + 2 * 4 * 16 * (64 + 2)), "no padding");
    return SPLITS * (sizeof(Join) + 2 * 4 * rows * (dp + 2));
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
