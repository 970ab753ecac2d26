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
//   V: row c of operand q is element DV c + q (DV = DP / 16) of the lane's eight
//      positions, picked from the eight rows with byte permutes, or 16 q + c,
//      where LDS hands it out transposed.
// head_dim below 32 DS (PAD): lanes past the end read piece 0 instead; their Q and
// K are zero (both: 0 times an infinity of the key is NaN) and their outputs are
// not stored.  Kernels of their own, since heads that need it not would pay for it:
// 64 ragged single tokens up to 2047 positions, 64 wide, 34.8 us and with a test of
// the size in the loop 41.8; 80 wide 51.4 without the zeros and 51.9 with them.
//
// Two kernels, by the rows of an item:
//   attn_rows_kernel (up to 16 rows): memory-bound.  Each wavefront streams
//     tiles of its own straight into operand registers; K's registers are
//     refilled for the next tile as soon as the scores are formed and V's as
//     soon as the products are, so each is in flight while the other is used.
//     The four wavefronts' sums meet in LDS at the end.
//   attn_block_kernel (up to 64 or 128 rows): each wavefront has 16 or 32 rows of
//     its own and all four share the tiles, which go straight into LDS, three of
//     32 positions ahead (seven where a head has 64 elements); pieces lie permuted
//     so that sixteen lanes' reads of an operand meet every bank once.  (The
//     counters call a third of the LDS cycles conflicts all the same; which
//     accesses have them has not been found.)
// What only one block of rows reads is loaded past the caches: 64 trees of 16 at
// 8192 positions take 359 us so and 404 otherwise.
// Measured, four query heads on each of eight key/value heads of 128 elements,
// binary16, pages token by token: 64 requests of one token at 8192 positions 345 to
// 358 us (6.1 TB/s; pages head by head 334 to 337, 6.4), one request at 4096 13.6 to
// 14.5 us, of which the join is 3.9; 64 trees of eight 361 us, of 16 345 to 366 (5.9 to
// 6.1 TB/s), of 32 (128 rows) 441 to 465 us, 600 TFLOP/s; 64 trees of 32 at 2048 131 to
// 133 us and as two blocks of 64 rows 217.  A plain read of as many bytes takes 317
// us.  With 128 rows the time follows the clock, which falls under this load: four
// trees of 16 with eight rows a token at 131072 positions, 30 runs, 388 us at 2.18 GHz to
// 483 at 1.75, the same cycles.  Within a wavefront a tile's scores, weights and
// products follow one another, with two wavefronts a SIMD and a barrier a tile; no
// pipe is near full (matrix cores 34 %, vector work 40 %, LDS 24 % of the cycles).
//
// Work: the cached positions of all items, in units of one step of a workgroup,
// are one line that is cut into (up to) SPLITS (as many workgroups as the chip
// holds) equal ranges, whatever the requests' lengths; a workgroup runs the
// segments of items in its range.  An item within one range is finished there; of
// an item that a cut divides, every workgroup leaves its unnormalised sums, and a
// second kernel joins them.  Which workgroup has what follows from the lengths
// alone.
//
// A row's running maximum is moved only when a score passes it by 2^GAP: most
// tiles then need neither the maximum over lanes nor the rescaling of the sums,
// which are binary32.  The weights are rounded to the cache's type, once: the
// matrix cores take both factors of a product in one type, a second product for
// the rest would be half of the matrix work again, and a weight's relative error
// (2^-8 or 2^-11 at most) is that of the values, which are stored so.  The sum of
// weights takes the rounded ones, so that a row of equal values keeps them.  So
// that small weights are not lost in binary16, whose numbers end at 2^-24, the
// maximum itself has the weight 2^LIFT there: a small weight is off by 2^-32 of
// the largest one at most, and 131072 of them together by 2^-15.
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
constexpr int CUS = 256;
constexpr float NO_SCORE = -3.0e38f;  // running maximum before any score
constexpr int GAP = 8;                // binary exponent by which a weight may exceed the running maximum's
constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// binary exponent of the running maximum's weight; 2^(LIFT + GAP) is a number of
// the type
template <bool BF>
constexpr int LIFT = BF ? 0 : 7;

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

// Sixteen lanes' 8-byte pieces of LDS are four rows of sixteen 16-bit elements
// (lane i: row i / 4, elements 4 (i % 4) ..), and lane i gets element i of the
// four rows: at each of four addresses and HALF bytes past it.  They are waited
// for here.  (The compiler lets its own transposing reads wait for every load
// into LDS that is on its way.)
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
template <int HALF>
__device__ __forceinline__ void read_transposed(const uint32_t (&at)[4], v4u (&v)[4])
{
    v2u lo[4], hi[4];
    asm volatile("ds_read_b64_tr_b16 %0, %8\n\t"
                 "ds_read_b64_tr_b16 %4, %8 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %1, %9\n\t"
                 "ds_read_b64_tr_b16 %5, %9 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %2, %10\n\t"
                 "ds_read_b64_tr_b16 %6, %10 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %3, %11\n\t"
                 "ds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(lo[0]), "=&v"(lo[1]), "=&v"(lo[2]), "=&v"(lo[3]), "=&v"(hi[0]), "=&v"(hi[1]), "=&v"(hi[2]),
                   "=&v"(hi[3])
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(HALF)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[i] = v4u{lo[i][0], lo[i][1], hi[i][0], hi[i][1]};
}

// true where one of the two 16-bit values is an infinity or NaN
template <bool BF>
__device__ __forceinline__ bool not_finite(uint32_t w)
{
    constexpr uint32_t E = BF ? 0x7f80u : 0x7c00u;
    return ((w & E) == E) | ((w & (E << 16)) == (E << 16));
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
    q.n = s1 - s0 <= a.max_new ? s1 - s0 : a.cut;
    q.ctx = (int)min((long long)max(a.context_lens[r], 0), room);
    q.n = q.n <= room - q.ctx ? q.n : min((int)(room - q.ctx), a.cut);
    return q;
}

// Where the items lie on the line of units: request r's kv_heads * row blocks
// items one after the other, each of the request's units.  The line has fewer
// than 2^31 units (checked by the launcher).  Where the line is long enough that
// no range is all of them, an item has `lead` empty units before its own, which
// stand for the time that it takes to begin and end one: a workgroup whose range
// has many short items gets fewer of them.  (64 ragged requests of up to 2047
// positions: one token each, heads 64 wide, 40.7 us without and 37.8 with one;
// eight tokens 73.8 and 67.0; trees of 32 119 us without, 107 with one, 93 with
// three.)
struct Item {
    int r, kvh, block;
    Request rq;
    int start, units, lead;  // first unit, number of units, the empty ones among them
};

template <int ROWS>
__device__ __forceinline__ int row_blocks(const AttnArgs &a, const Request &q)
{
    return (q.n * (a.heads / a.kv.kv_heads) + ROWS - 1) / ROWS;
}

// Inclusive prefix sum over a wavefront's lanes.
__device__ __forceinline__ int wave_scan(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast 15, 31
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
    return v;
}

// Up to 64 requests: a lane each, in every wavefront by itself.  More: each
// lane has a run of requests, in every wavefront again.
template <int ROWS, int UNIT, int SPLITS>
struct Line {
    static constexpr int LEAD = ROWS == 128 ? 3 : 1;
    const AttnArgs &a;
    int total, per, before, lead;
    Request mine;  // per == 1: the lane's request

    __device__ static int items_of(const AttnArgs &a, const Request &q)
    {
        return row_blocks<ROWS>(a, q) * a.kv.kv_heads;
    }
    __device__ static int units_of(const AttnArgs &a, const Request &q, int lead)
    {
        return ((q.ctx + q.n + UNIT - 1) / UNIT + lead) * items_of(a, q);
    }

    __device__ explicit Line(const AttnArgs &a_) : a(a_)
    {
        const int lane = threadIdx.x & 63;
        per = (a.R + 63) / 64;
        const int r0 = lane * per, r1 = min(r0 + per, a.R);
        mine = request_of(a, min(r0, a.R - 1));
        int own = r0 < a.R ? units_of(a, mine, 0) : 0, items = r0 < a.R ? items_of(a, mine) : 0;
        for (int r = r0 + 1; r < r1; ++r) {
            const Request q = request_of(a, r);
            own += units_of(a, q, 0);
            items += items_of(a, q);
        }
        const int sum = wave_scan(own), sum_items = wave_scan(items);
        total = __builtin_amdgcn_readlane(sum, 63);
        lead = total >= (LEAD + 1) * SPLITS ? LEAD : 0;
        before = sum - own + lead * (sum_items - items);
        total += lead * __builtin_amdgcn_readlane(sum_items, 63);
    }

    // the item that holds unit u (the same in every lane)
    __device__ Item item_at(int u) const
    {
        Item it;
        const int lane = threadIdx.x & 63;
        const int run = 63 - __builtin_clzll(__ballot(lane * per < a.R && before <= u));
        int base = __builtin_amdgcn_readlane(before, run), at = run;
        it.r = run;
        Request q = mine;
        if (per > 1) {
            // the run's requests, a lane each
            it.r = run * per;
            const int n = min(per, a.R - it.r);
            q = request_of(a, it.r + min(lane, n - 1));
            const int own = lane < n ? units_of(a, q, lead) : 0, sum = wave_scan(own);
            at = 63 - __builtin_clzll(__ballot(lane < n && base + sum - own <= u));
            base += __builtin_amdgcn_readlane(sum - own, at);
            it.r += at;
        }
        it.rq.ctx = __builtin_amdgcn_readlane(q.ctx, at);
        it.rq.n = __builtin_amdgcn_readlane(q.n, at);
        it.rq.first = __builtin_amdgcn_readlane(q.first, at);
        it.lead = lead;
        it.units = (it.rq.ctx + it.rq.n + UNIT - 1) / UNIT + lead;
        const uint32_t blocks = row_blocks<ROWS>(a, it.rq);
        const uint32_t k = __builtin_amdgcn_readfirstlane((uint32_t)(u - base) / (uint32_t)it.units);
        it.start = base + (int)k * it.units;
        it.kvh = __builtin_amdgcn_readfirstlane(k / blocks);
        it.block = (int)k - it.kvh * (int)blocks;
        return it;
    }
};

// The line's ranges, none empty: their number, where range i starts, and the
// range that holds unit u.  The first `more` ranges have one unit more.
template <int SPLITS>
struct Cuts {
    uint32_t total, each, more;
    __device__ explicit Cuts(int t) : total(t), each((uint32_t)t / SPLITS), more((uint32_t)t % SPLITS) {}
    __device__ __forceinline__ int ranges() const { return min((int)total, SPLITS); }
    __device__ __forceinline__ int start(uint32_t i) const { return (int)(each * i + min(i, more)); }
    __device__ __forceinline__ int holder(uint32_t u) const
    {
        const uint32_t longer = more * (each + 1);
        return (int)(u < longer ? u / (each + 1) : more + (u - longer) / each);
    }
};

// The workspace: the joins of divided items, then the parts -- range i's own
// part 2 i for its first segment, 2 i + 1 for another (only its last can be
// divided too).  A join is written by the range in which its item begins: as
// entry i by range i (at most one divided item begins in a range), or, where the
// call has few items (a.by_item), as the item's entry, by number.
struct Join {
    int parts, range, second;  // parts (0: nothing to do), the first one's range and whether it is its second
    int rows, row0, first, kvh;
    int unused;
};

template <int ROWS, int DP>
struct Part {
    float o[ROWS][DP];
    float m[ROWS], l[ROWS];
};

template <int ROWS, int DP, int SPLITS>
struct Workspace {
    Join join[SPLITS];
    Part<ROWS, DP> part[2 * SPLITS];
};

template <int ROWS>
__device__ __forceinline__ int most_blocks(const AttnArgs &a)
{
    return (a.max_new * (a.heads / a.kv.kv_heads) + ROWS - 1) / ROWS;
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

// A wavefront's 16 NT rows, c of each sixteen in lanes (c, *).  Output element
// i of operand row 4 g + i of product q is element d(q, i) of the head: DV (4 g
// + i) + q, or, where the values came transposed out of LDS, 16 q + 4 g + i.
template <int DP, int DS, bool PAD, int NT, bool BF, bool TRANSPOSED>
struct Rows {
    static constexpr int DV = DP / 16;
    v4u q[NT][DS];
    uint64_t mask[NT];
    v4f acc[NT][DV], sum[NT];  // sum: every element is the lane's row's sum of weights
    float m[NT];  // the running maximum, in binary exponents, less LIFT
    float scale2;

    // Rows row0 .. row0 + rows - 1 of the item: begin() sends the loads off,
    // without a branch (past the end, a piece that is there is read), and
    // finish() drops what is past the end.
    __device__ __forceinline__ void begin(const AttnArgs &a, const Item &it, int row0, int rows, int group)
    {
        const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4, pieces = a.kv.head_dim / 8;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = 16 * nt + c < rows ? row0 + 16 * nt + c : row0;
            const int tok = it.rq.first + row / group, head = it.kvh * group + row % group;
            const uint16_t *p = (const uint16_t *)a.q + tok * a.q_token_stride + head * a.q_head_stride;
            mask[nt] = a.tree_mask[tok];
#pragma unroll
            for (int s = 0; s < DS; ++s)
                q[nt][s] = *(const v4u *)(p + 8 * (4 * s + g < pieces ? 4 * s + g : 0));
        }
    }

    // The scale's sign goes into Q, and a scale of zero too, so that masked
    // scores stay -infinity.
    __device__ __forceinline__ void finish(const AttnArgs &a, int rows)
    {
        const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4, pieces = a.kv.head_dim / 8;
        const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u, keep = a.scale == 0.f ? 0u : ~0u;
        scale2 = a.scale == 0.f ? 1.f : fabsf(a.scale) * LOG2E;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const bool ok = 16 * nt + c < rows;
            mask[nt] = ok ? mask[nt] : 0;
#pragma unroll
            for (int s = 0; s < DS; ++s)
                q[nt][s] = (q[nt][s] ^ flip) & (ok && 4 * s + g < pieces ? keep : 0u);
            m[nt] = NO_SCORE;
            sum[nt] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < DV; ++i)
                acc[nt][i] = v4f{0.f, 0.f, 0.f, 0.f};
        }
    }

    __device__ __forceinline__ void scores(v4u (&k)[2][DS], int pieces, v4f (&s)[NT][2])
    {
        if constexpr (PAD) {
            const int g = (threadIdx.x & 63) >> 4;
            // (of more than two steps all but the last are whole)
#pragma unroll
            for (int d = DS > 2 ? DS - 1 : 0; d < DS; ++d) {
                const uint32_t keep = 4 * d + g < pieces ? ~0u : 0u;
                k[0][d] &= keep;
                k[1][d] &= keep;
            }
        }
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

    // hides the scores of the tile at p0 that a row does not see
    __device__ __forceinline__ void hide(int p0, bool ok0, bool ok1, const Request &rq, v4f (&s)[NT][2])
    {
        const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int j = p0 + 16 * (e / 4) + 4 * g + e % 4 - rq.ctx;
            const bool there = (j < rq.n) & (e / 4 ? ok1 : ok0);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const bool seen = there & ((j < 0) | (((mask[nt] >> (j & 63)) & 1) != 0));
                s[nt][e / 4][e % 4] = seen ? s[nt][e / 4][e % 4] : -INFINITY;
            }
        }
    }

    __device__ __forceinline__ void form(const v4f (&s)[2], float top, v4u &pf)
    {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = fast_exp2(fmaf(s[e / 4][e % 4], scale2, -top));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            pf[i] = pack2<BF>(x[2 * i], x[2 * i + 1]);
    }

    // Weights of the tile, as the products' operand.  They are formed with the
    // maximum so far; only where one exceeds 2^(LIFT + GAP) (compared as integers,
    // two at a time: they are not negative) is the maximum moved and the tile done
    // again.
    __device__ __forceinline__ void weights(const v4f (&s)[NT][2], v4u (&pf)[NT])
    {
        typedef uint16_t v2s __attribute__((ext_vector_type(2)));
        // 2^(LIFT + GAP), twice
        constexpr uint32_t LIMIT = 0x10001u * (BF ? (127 + LIFT<BF> + GAP) << 7 : (15 + LIFT<BF> + GAP) << 10);
        const v2s limit = __builtin_bit_cast(v2s, LIMIT);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            form(s[nt], m[nt], pf[nt]);
            v2s most = limit;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                most = __builtin_elementwise_max(most, __builtin_bit_cast(v2s, (uint32_t)pf[nt][i]));
            if (__ballot(__builtin_bit_cast(uint32_t, most) != LIMIT)) {
                float top = fmaxf(fmaxf(fmaxf(s[nt][0][0], s[nt][0][1]), fmaxf(s[nt][0][2], s[nt][0][3])),
                                  fmaxf(fmaxf(s[nt][1][0], s[nt][1][1]), fmaxf(s[nt][1][2], s[nt][1][3])));
                top = fmaxf(max4(top * scale2) - LIFT<BF>, m[nt]);
                const float keep = fast_exp2(m[nt] - top);
                m[nt] = top;
                sum[nt] *= keep;
#pragma unroll
                for (int i = 0; i < DV; ++i)
                    acc[nt][i] *= keep;
                form(s[nt], top, pf[nt]);
            }
        }
    }

    // The values of positions that are not there become 0.  True where values
    // of the step's own tokens are not finite (the same in every lane).
    __device__ __forceinline__ bool hide_values(int p0, bool ok0, bool ok1, const Request &rq, v4u (&v)[DV])
    {
        const int g = (threadIdx.x & 63) >> 4;
        bool odd = false;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint32_t there = 0, own = 0;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int e = 2 * w + k, j = p0 + 16 * (e / 4) + 4 * g + e % 4 - rq.ctx;
                const uint32_t half = k ? 0xffff0000u : 0xffffu;
                there |= (j < rq.n) & (e / 4 ? ok1 : ok0) ? half : 0;
                own |= j >= 0 ? half : 0;
            }
#pragma unroll
            for (int i = 0; i < DV; ++i) {
                v[i][w] &= there;
                odd |= not_finite<BF>(v[i][w] & own);
            }
        }
        return __ballot(odd) != 0;
    }

    // Values of the step's own tokens that are not finite: their products are
    // added one by one to the rows that see them, and 0 stands in their place
    // in the operand.  value(p): position p's values.
    template <typename F>
    __device__ __forceinline__ void odd_products(int p0, bool ok0, bool ok1, const AttnArgs &a, const Request &rq,
                                                 const v4u (&pf)[NT], v4u (&v)[DV], F value)
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
                    auto term = [&](uint32_t bits) {
                        return seen & not_finite<BF>(bits) ? weight * unpack<BF>(bits, 0) : 0.f;
                    };
                    if constexpr (TRANSPOSED) {
#pragma unroll
                        for (int i = 0; i < DV; ++i) {
                            if (16 * i + 4 * g >= a.kv.head_dim)
                                continue;
                            const Halves<4> piece = *(const Halves<4> *)(row + 16 * i + 4 * g);
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                acc[nt][i][k] += term(k & 1 ? piece.w[k / 2] >> 16 : piece.w[k / 2] & 0xffffu);
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            if (DV * (4 * g + k) >= a.kv.head_dim)
                                continue;
                            const Halves<DV> piece = *(const Halves<DV> *)(row + DV * (4 * g + k));
#pragma unroll
                            for (int i = 0; i < DV; ++i)
                                acc[nt][i][k] += term(i & 1 ? piece.w[i / 2] >> 16 : piece.w[i / 2] & 0xffffu);
                        }
                    }
                }
            }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (p0 + 16 * (e / 4) + 4 * g + e % 4 < rq.ctx)
                continue;
            const uint32_t half = e & 1 ? 0xffff0000u : 0xffffu;
#pragma unroll
            for (int i = 0; i < DV; ++i)
                if (not_finite<BF>(v[i][e / 2] & half))
                    v[i][e / 2] &= ~half;
        }
    }

    __device__ __forceinline__ void products(const v4u (&pf)[NT], const v4u (&v)[DV])
    {
        constexpr uint32_t ONE = BF ? 0x3f803f80u : 0x3c003c00u;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
            sum[nt] = mfma<BF>(v4u{ONE, ONE, ONE, ONE}, pf[nt], sum[nt]);
#pragma unroll
        for (int i = 0; i < DV; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                acc[nt][i] = mfma<BF>(v[i], pf[nt], acc[nt][i]);
    }
};

// Uniform address of position p of a page plus a 32-bit lane offset is what
// every load uses.  The offset is made opaque where it is used, or the compiler
// widens it outside of the loop and adds 64-bit addresses per lane and load.
__device__ __forceinline__ uint64_t lane_offset(uint32_t off)
{
    asm volatile("" : "+v"(off));
    return off;
}

// Keeps loads that were written before it from being moved behind it: towards
// their use, where they would no longer run under the work in between.
__device__ __forceinline__ void issue_loads() { asm volatile("" ::: "memory"); }

__device__ __forceinline__ const char *at_page(const void *base, int page, int p, int page_size, int64_t page_stride,
                                               uint32_t step)
{
    const uint32_t off = (uint32_t)p & (page_size - 1);
    return (const char *)base + 2 * (long long)max(page, 0) * page_stride + (uint64_t)off * step;
}

// The page of the sixteen positions at p (a page holds whole sixteens); -1:
// past the end or outside the cache, read from page 0 and masked.
__device__ __forceinline__ int table_entry(const int32_t *table, int p, int end, int page_shift)
{
    return uniform_load(table + (min(__builtin_amdgcn_readfirstlane(p), end - 1) >> page_shift));
}

__device__ __forceinline__ int page_of(const AttnArgs &a, int entry, int p, int end)
{
    return p < end && entry < a.kv.n_pages ? max(entry, -1) : -1;
}

__device__ __forceinline__ int page_at(const AttnArgs &a, const int32_t *table, int p, int end, int page_shift)
{
    return page_of(a, table_entry(table, p, end, page_shift), p, end);
}

// A workgroup's part [u, stop) of an item: the item's rows from row0 on, the
// positions first .. last - 1 of its end, and where its pages and its head lie.
struct Segment {
    Item it;
    int u, stop, row0, rows, first, last, end;
    const int32_t *table;
    const uint16_t *k, *v;
};

template <int ROWS, int UNIT, int SPLITS>
__device__ __forceinline__ Segment segment_at(const Line<ROWS, UNIT, SPLITS> &line, const AttnArgs &a, int u, int u1)
{
    Segment s;
    s.it = line.item_at(u);
    s.u = u;
    s.stop = min(u1, s.it.start + s.it.units);
    s.row0 = s.it.block * ROWS;
    s.rows = min(s.it.rq.n * (a.heads / a.kv.kv_heads) - s.row0, ROWS);
    s.end = s.it.rq.ctx + s.it.rq.n;
    s.first = max(u - s.it.start - s.it.lead, 0) * UNIT;
    s.last = min((s.stop - s.it.start - s.it.lead) * UNIT, s.end);
    s.table = a.page_table + s.it.r * a.table_stride;
    s.k = (const uint16_t *)a.kv.k + s.it.kvh * a.kv.k_head_stride;
    s.v = (const uint16_t *)a.kv.v + s.it.kvh * a.kv.v_head_stride;
    return s;
}

// (a range may start among an item's empty units)
__device__ __forceinline__ bool begins_item(const Segment &s) { return s.u <= s.it.start + s.it.lead; }

__device__ __forceinline__ bool is_whole(const Segment &s)
{
    return begins_item(s) && s.stop == s.it.start + s.it.units;
}

// whether the range has another item's positions
__device__ __forceinline__ bool more_after(const Segment &s, int u1) { return s.stop + s.it.lead < u1; }

// End of a workgroup's segment (called by one thread).
template <int ROWS, int SPLITS>
__device__ __forceinline__ void note_join(const AttnArgs &a, const Cuts<SPLITS> &cuts, const Segment &s, int u0, int u1,
                                          Join *join)
{
    const Item &it = s.it;
    const bool begins = begins_item(s), divided = begins && s.stop < it.start + it.units;
    if (a.by_item ? !begins : more_after(s, u1))
        return;
    Join j = {};
    if (divided) {
        j.range = blockIdx.x;
        j.parts = cuts.holder(it.start + it.units - 1) - j.range + 1;
        j.second = s.u != u0;
        j.row0 = s.row0;
        j.rows = s.rows;
        j.first = it.rq.first;
        j.kvh = it.kvh;
    }
    join[a.by_item ? (it.r * a.kv.kv_heads + it.kvh) * most_blocks<ROWS>(a) + it.block : blockIdx.x] = j;
}

// ---------------------------------------------------------------------------
// items of few rows
// ---------------------------------------------------------------------------

// DP: padded head size, DS: 32-element steps of it that hold elements, PAD: the
// last of them are not whole, BF: bfloat16, WGS: workgroups a CU.
template <int DP, int DS, bool PAD, bool BF, int WGS>
__global__ void __launch_bounds__(ATTN_THREADS, WGS) attn_rows_kernel(AttnArgs a)
{
    constexpr int NT = 1, DV = DP / 16, ROWS = 16 * NT, UNIT = ATTN_WAVES * TILE, SPLITS = WGS * CUS;
    __shared__ float lds_o[ATTN_WAVES][ROWS][DP + 4];
    __shared__ float lds_m[ATTN_WAVES][ROWS], lds_l[ATTN_WAVES][ROWS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int group = a.heads / a.kv.kv_heads;
    const int D = a.kv.head_dim, pieces = D / 8;
    const int page_shift = __builtin_ctz(a.kv.page_size);
    Workspace<ROWS, DP, SPLITS> &ws = *(Workspace<ROWS, DP, SPLITS> *)a.workspace;
    const Line<ROWS, UNIT, SPLITS> line(a);
    const Cuts<SPLITS> cuts(line.total);
    if ((int)blockIdx.x >= cuts.ranges()) {
        if (!a.by_item && threadIdx.x == 0)
            ws.join[blockIdx.x].parts = 0;
        return;
    }
    const int u0 = cuts.start(blockIdx.x), u1 = cuts.start(blockIdx.x + 1);
    const uint32_t k_step = 2 * (uint32_t)a.kv.k_token_stride, v_step = 2 * (uint32_t)a.kv.v_token_stride;
    const uint32_t k_lane = c * k_step, v_lane = 4 * g * v_step + 2 * (DV * c < D ? DV * c : 0);

    v4u kf[2][DS];
    uint32_t vr[8][DV / 2];
    // (used: ~0; 0 where the tile is not used: every lane loads the first one's)
    auto load_k = [&](const Segment &sg, int p0, const int *page, uint32_t used) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const char *kp = at_page(sg.k, page[h], p0 + 16 * h, a.kv.page_size, a.kv.k_page_stride, k_step);
#pragma unroll
            for (int s = 0; s < DS; ++s) {
                const uint32_t piece = 4 * s + 3 < pieces || 4 * s + g < pieces ? 4 * s + g : 0;
                kf[h][s] = *(const v4u *)(kp + lane_offset((k_lane + 16 * piece) & used));
            }
        }
        issue_loads();
    };
    auto load_v = [&](const Segment &sg, int p0, const int *page, uint32_t used) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const char *vp = at_page(sg.v, page[h], p0 + 16 * h, a.kv.page_size, a.kv.v_page_stride, v_step);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // read once: the caches need not keep it (a load of keys takes
                // half a cache line, and its other half is still to come)
                typedef uint32_t part_t __attribute__((ext_vector_type(DV / 2)));
                const part_t v =
                    __builtin_nontemporal_load((const part_t *)(vp + (uint64_t)(e * v_step) + lane_offset(v_lane & used)));
#pragma unroll
                for (int i = 0; i < DV / 2; ++i)
                    vr[4 * h + e][i] = v[i];
            }
        }
        issue_loads();
    };
    int page[2], next[2], after[2];
    auto pages_of = [&](const Segment &sg, int p0, int *id) {
        id[0] = page_at(a, sg.table, p0, sg.end, page_shift);
        id[1] = page_at(a, sg.table, p0 + 16, sg.end, page_shift);
    };
    // a tile past the segment's end is the one before it once more
    auto next_tile = [](const Segment &sg, int p0) { return p0 + UNIT < sg.last ? p0 + UNIT : p0; };
    Rows<DP, DS, PAD, NT, BF, false> row;
    // sends off a segment's first loads
    auto open = [&](int u) {
        const Segment sg = segment_at(line, a, u, u1);
        row.begin(a, sg.it, sg.row0, sg.rows, group);
        // (a wavefront without a tile loads one too)
        const int start = min(sg.first + wave * TILE, (sg.last - 1) & ~(TILE - 1));
        const uint32_t used = start == sg.first + wave * TILE ? ~0u : 0u;
        pages_of(sg, start, page);
        pages_of(sg, next_tile(sg, start), next);
        load_k(sg, start, page, used);
        load_v(sg, start, page, used);
        return sg;
    };

    Segment seg = open(u0);
    for (;;) {
        const Request &rq = seg.it.rq;
        row.finish(a, seg.rows);
        for (int p0 = seg.first + wave * TILE; p0 < seg.last; p0 += UNIT) {
            // no branch around the loads, so that their counters stay exact: a
            // little of the last tile is loaded once more and not used
            const int pn = next_tile(seg, p0);
            const uint32_t used = pn != p0 ? ~0u : 0u;
            pages_of(seg, next_tile(seg, pn), after);
            v4f s[NT][2];
            row.scores(kf, pieces, s);
            load_k(seg, pn, next, used);
            const bool masked = p0 + TILE > rq.ctx || (page[0] | page[1]) < 0;
            if (masked)
                row.hide(p0, page[0] >= 0, page[1] >= 0, rq, s);
            v4u pf[NT];
            row.weights(s, pf);
            // operand i of the values: element DV c + i of the lane's eight rows
            v4u vf[DV];
#pragma unroll
            for (int i = 0; i < DV; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    vf[i][e] = __builtin_amdgcn_perm(vr[2 * e + 1][i / 2], vr[2 * e][i / 2],
                                                     i & 1 ? 0x07060302u : 0x05040100u);
            if (__builtin_expect(masked && row.hide_values(p0, page[0] >= 0, page[1] >= 0, rq, vf), 0))
                row.odd_products(p0, page[0] >= 0, page[1] >= 0, a, rq, pf, vf, [&](int p) {
                    const int id = p - p0 < 16 ? page[0] : page[1];
                    return (const uint16_t *)at_page(seg.v, id, p, a.kv.page_size, a.kv.v_page_stride, v_step);
                });
            row.products(pf, vf);
            load_v(seg, pn, next, used);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                page[h] = next[h];
                next[h] = after[h];
            }
        }

        // the wavefronts' parts meet in LDS, under the next segment's first loads
        const Segment done = seg;
        const bool more = more_after(done, u1), whole = is_whole(done);
        if (more)
            seg = open(done.stop);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (g == 0) {
                lds_m[wave][16 * nt + c] = row.m[nt];
                lds_l[wave][16 * nt + c] = row.sum[nt][0];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int q = 0; q < DV; ++q)
                    lds_o[wave][16 * nt + c][DV * (4 * g + i) + q] = row.acc[nt][q][i];
        }
        __syncthreads();
        if (threadIdx.x == 0)
            note_join<ROWS>(a, cuts, done, u0, u1, ws.join);
        Part<ROWS, DP> &part = ws.part[2 * blockIdx.x + (done.u != u0)];
        for (int i = wave; i < done.rows; i += ATTN_WAVES) {
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
                    *(uint32_t *)(out_row(a, done.it.rq.first, done.it.kvh, done.row0 + i, group) + 2 * lane) =
                        pack2<BF>(o0 * inv, o1 * inv);
                else
                    *(float2 *)&part.o[i][2 * lane] = make_float2(o0, o1);
            }
        }
        if (!more)
            break;
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// items of many rows
// ---------------------------------------------------------------------------

// One load of 1 KiB into LDS: every lane's 16 bytes at its `src` to dst + 16 lane.
// It is complete when the wavefront's vector-memory count says so.  ONCE: the
// caches need not keep it.
template <bool ONCE>
__device__ __forceinline__ void load_to_lds(const char *src, v4u *dst)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src,
                                     (__attribute__((address_space(3))) void *)dst, 16, 0, ONCE ? 2 : 0);
}

// Waits until the wavefront has read what it reads of LDS and its loads into LDS
// are complete but for those of the `younger` last tiles, or of the MOST last.
template <int MOST, int LOADS>
__device__ __forceinline__ void wait_tiles(int younger)
{
    if constexpr (MOST > 0)
        if (younger < MOST)
            return wait_tiles<MOST - 1, LOADS>(younger);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(MOST *LOADS) : "memory");
}

// NT: 16-row tiles per wavefront; the others as above.
template <int DP, int DS, bool PAD, int NT, bool BF, int WGS>
__global__ void __launch_bounds__(ATTN_THREADS, WGS) attn_block_kernel(AttnArgs a)
{
    constexpr int DV = DP / 16, WROWS = 16 * NT, ROWS = WROWS * ATTN_WAVES, UNIT = 64, SPLITS = WGS * CUS;
    constexpr int PIECES = DP / 8;               // 16-byte pieces of a stored row
    constexpr int STAGES = 64 / PIECES;          // tiles of 32 positions in LDS: 64 KiB
    constexpr int AHEAD = STAGES - 1;            // of them on their way or waiting
    constexpr int WAVE_ROWS = TILE / ATTN_WAVES; // positions of a tile that a wavefront brings in
    constexpr int LOAD_ROWS = 64 / PIECES;       // of them in one load
    constexpr int LOADS = WAVE_ROWS / LOAD_ROWS; // loads, of keys and of values
    // [stage][keys, values][position][piece, permuted]; aligned, since offsets are
    // put together by exclusive or
    __shared__ __attribute__((aligned(1024))) v4u tile[STAGES][2][TILE][PIECES];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int group = a.heads / a.kv.kv_heads;
    const int D = a.kv.head_dim, pieces = D / 8;
    const int page_shift = __builtin_ctz(a.kv.page_size);
    Workspace<ROWS, DP, SPLITS> &ws = *(Workspace<ROWS, DP, SPLITS> *)a.workspace;
    const Line<ROWS, UNIT, SPLITS> line(a);
    const Cuts<SPLITS> cuts(line.total);
    if ((int)blockIdx.x >= cuts.ranges()) {
        if (!a.by_item && threadIdx.x == 0)
            ws.join[blockIdx.x].parts = 0;
        return;
    }
    const int u0 = cuts.start(blockIdx.x), u1 = cuts.start(blockIdx.x + 1);
    const uint32_t k_step = 2 * (uint32_t)a.kv.k_token_stride, v_step = 2 * (uint32_t)a.kv.v_token_stride;

    // Piece j of stored row r lies at j ^ swap(r): sixteen lanes that read one
    // piece of sixteen rows, or the pieces of one row, meet all banks once.
    auto swap = [](int r) { return PIECES == 16 ? r & 15 : (r >> 1) & 7; };

    // Wavefront w brings in positions 8 w .. 8 w + 7 of a tile, straight into LDS:
    // a load's lanes lie one after the other there, so a lane takes the piece that
    // belongs to its place.
    uint32_t k_lane[LOADS], v_lane[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int r = i * LOAD_ROWS + lane / PIECES, piece = (lane % PIECES) ^ swap(wave * WAVE_ROWS + r);
        const int from = piece < pieces ? piece : 0;
        k_lane[i] = r * k_step + 16 * from;
        v_lane[i] = r * v_step + 16 * from;
    }

    // Where lane (c, g) reads its operands in a stored tile: keys, piece 4 s + g
    // of row c (and 16 + c); values, transposed, elements 16 i + 4 (c % 4) .. of
    // row 4 g + c / 4 (and 16 + that) -- row and swap are the same for both
    // halves, and s and i only move the piece.
    constexpr int ROW_BYTES = 16 * PIECES;
    const int v_row = 4 * g + c / 4;
    const uint32_t k_read = c * ROW_BYTES + 16 * (g ^ swap(c));
    const uint32_t v_read = v_row * ROW_BYTES + 16 * (((c & 3) >> 1) ^ swap(v_row)) + 8 * (c & 1);

    int ids[2 * AHEAD];  // table entries of the sixteens that are brought in next
    uint32_t there = 0;  // two bits a stage: which of its sixteens are there
    auto pages_of = [&](const Segment &sg, int p0, int *id) {
        id[0] = table_entry(sg.table, p0, sg.end, page_shift);
        id[1] = table_entry(sg.table, p0 + 16, sg.end, page_shift);
    };
    // brings in the tile at p0
    auto load = [&](const Segment &sg, int p0, const int *entry, int stage) {
        const int id[2] = {page_of(a, entry[0], p0, sg.end), page_of(a, entry[1], p0 + 16, sg.end)};
        const int mine = wave < ATTN_WAVES / 2 ? id[0] : id[1], p = p0 + wave * WAVE_ROWS;
        const char *kp = at_page(sg.k, mine, p, a.kv.page_size, a.kv.k_page_stride, k_step);
        const char *vp = at_page(sg.v, mine, p, a.kv.page_size, a.kv.v_page_stride, v_step);
        v4u(*const to)[TILE][PIECES] = tile[stage];
        if (NT == 1 || sg.it.rq.n * group <= ROWS) {  // no other block of rows reads it too
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                load_to_lds<true>(kp + lane_offset(k_lane[i]), to[0][wave * WAVE_ROWS + i * LOAD_ROWS]);
                load_to_lds<true>(vp + lane_offset(v_lane[i]), to[1][wave * WAVE_ROWS + i * LOAD_ROWS]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                load_to_lds<false>(kp + lane_offset(k_lane[i]), to[0][wave * WAVE_ROWS + i * LOAD_ROWS]);
                load_to_lds<false>(vp + lane_offset(v_lane[i]), to[1][wave * WAVE_ROWS + i * LOAD_ROWS]);
            }
        }
        issue_loads();
        there = (there & ~(3u << (2 * stage))) | ((id[0] >= 0 ? 1u : 0u) | (id[1] >= 0 ? 2u : 0u)) << (2 * stage);
    };
    Rows<DP, DS, PAD, NT, BF, true> row;
    // the wavefront's own rows of a segment's
    auto my_rows = [&](const Segment &sg) { return min(max(sg.rows - wave * WROWS, 0), WROWS); };
    auto tiles_of = [](const Segment &sg) { return (sg.last - sg.first + TILE - 1) / TILE; };
    // sends off a segment's first loads, its first tile to `stage`
    auto open = [&](int u, int stage) {
        const Segment sg = segment_at(line, a, u, u1);
        row.begin(a, sg.it, sg.row0 + (my_rows(sg) ? wave * WROWS : 0), my_rows(sg), group);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            pages_of(sg, sg.first + k * TILE, &ids[2 * k]);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (k < tiles_of(sg))
                load(sg, sg.first + k * TILE, &ids[2 * k], (stage + k) % STAGES);
        pages_of(sg, sg.first + AHEAD * TILE, ids);
        return sg;
    };

    int stage = 0;
    Segment seg = open(u0, 0);
    for (;;) {
        const Request &rq = seg.it.rq;
        const int rows = my_rows(seg), tiles = tiles_of(seg);
        row.finish(a, rows);
        for (int k = 0; k < tiles; ++k) {
            // This tile is there and the one before it is read, in every
            // wavefront: the next loads take its place.
            wait_tiles<STAGES - 2, 2 * LOADS>(tiles - 1 - k);
            __builtin_amdgcn_s_barrier();
            issue_loads();
            const int pt = seg.first + k * TILE, at = stage;
            if (k + AHEAD < tiles) {
                load(seg, pt + AHEAD * TILE, ids, (stage + AHEAD) % STAGES);
                pages_of(seg, pt + (AHEAD + 1) * TILE, ids);
            }
            stage = (stage + 1) % STAGES;
            if (rows) {
                const char *keys = (const char *)tile[at][0];
                const uint32_t values = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)tile[at][1];
                v4u kf[2][DS];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int s = 0; s < DS; ++s)
                        kf[h][s] = *(const v4u *)(keys + 16 * h * ROW_BYTES + (k_read ^ (64 * s)));
                v4f s[NT][2];
                row.scores(kf, pieces, s);
                v4u vf[DV];
#pragma unroll
                for (int i = 0; i < DV; i += 4) {
                    const uint32_t v_at = values + v_read;
                    const uint32_t from[4] = {v_at ^ (32 * i), v_at ^ (32 * (i + 1)), v_at ^ (32 * (i + 2)),
                                              v_at ^ (32 * (i + 3))};
                    read_transposed<16 * ROW_BYTES>(from, *(v4u(*)[4]) & vf[i]);
                }
                const bool ok0 = (there >> (2 * at)) & 1, ok1 = (there >> (2 * at + 1)) & 1;
                const bool masked = pt + TILE > rq.ctx || !ok0 || !ok1;
                if (masked)
                    row.hide(pt, ok0, ok1, rq, s);
                v4u pf[NT];
                row.weights(s, pf);
                if (__builtin_expect(masked && row.hide_values(pt, ok0, ok1, rq, vf), 0))
                    row.odd_products(pt, ok0, ok1, a, rq, pf, vf, [&](int p) {
                        return (const uint16_t *)at_page(seg.v, seg.table[p >> page_shift], p, a.kv.page_size,
                                                         a.kv.v_page_stride, v_step);
                    });
                row.products(pf, vf);
            }
        }

        // the segment's results leave under the next one's first loads
        const Segment done = seg;
        const bool more = more_after(done, u1), whole = is_whole(done);
        if (more)
            seg = open(done.stop, stage);
        if (threadIdx.x == 0)
            note_join<ROWS>(a, cuts, done, u0, u1, ws.join);
        Part<ROWS, DP> &part = ws.part[2 * blockIdx.x + (done.u != u0)];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float total = row.sum[nt][0], inv = inverse(total);
            const int i = 16 * nt + c;
            if (i >= rows)
                continue;
            if (!whole && g == 0) {
                part.m[wave * WROWS + i] = row.m[nt];
                part.l[wave * WROWS + i] = total;
            }
            uint16_t *out = out_row(a, done.it.rq.first, done.it.kvh, done.row0 + wave * WROWS + i, group);
#pragma unroll
            for (int q = 0; q < DV; ++q) {
                const int d = 16 * q + 4 * g;
                if (d >= D)
                    continue;
                const v4f o = row.acc[nt][q];
                if (whole)
                    *(Halves<4> *)(out + d) = Halves<4>{pack2<BF>(o[0] * inv, o[1] * inv),
                                                        pack2<BF>(o[2] * inv, o[3] * inv)};
                else
                    *(v4f *)&part.o[wave * WROWS + i][d] = o;
            }
        }
        if (!more)
            break;
    }
}

// ---------------------------------------------------------------------------
// the join
// ---------------------------------------------------------------------------

constexpr int JOIN_WAVES = 4, JOIN_THREADS = 64 * JOIN_WAVES;

// The rows that no item has, of the tokens that workgroup `part` of `parts` takes,
// a wavefront each in turn: 0 where the token is of no request, NaN where its
// request is not wholly computed.  Beside the joins: one token at 4096 positions
// takes 14.5 us so and 14.1 without, eight trees of eight at 8192 42.7 and 42.4, where
// clearing the output first would be a launch more (2.1 us).
template <bool BF>
__device__ __forceinline__ void fill_rows(const AttnArgs &a, int part, int parts)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int pieces = a.heads * (a.kv.head_dim / 8);
    for (long long t = (long long)part * JOIN_WAVES + wave; t < a.T; t += (long long)parts * JOIN_WAVES) {
        // the last request that starts at or before t, 64 starts at a time
        int r = 0, n = a.R;
        uint64_t below = 1;
        if (n > 64) {
            const int step = (n + 63) / 64, at = lane * step;
            below = __ballot(at < n && a.query_start[min(at, n)] <= t);
            r = below ? (63 - __builtin_clzll(below)) * step : 0;
            n = min(n - r, step);
        }
        below = below ? __ballot(lane < n && a.query_start[r + min(lane, n)] <= t) : 0;
        uint32_t value = 0;
        if (below) {
            r += 63 - __builtin_clzll(below);
            const Request q = request_of(a, r);
            if (t - q.first < q.n)
                continue;
            if (t < a.query_start[r + 1])
                value = BF ? 0x7fc07fc0u : 0x7e007e00u;
        }
        v4u *row = (v4u *)a.out + t * pieces;
        for (int i = lane; i < pieces; i += 64)
            row[i] = v4u{value, value, value, value};
    }
}

// Joins the parts of a divided item (join i of workgroup (i, y)).  Few rows in
// all: a workgroup has one row, its wavefronts share the parts and meet in LDS --
// a CU brings in no more than some ten bytes a cycle of other XCDs' results, so
// the rows are spread.  Many rows: a wavefront has four rows of its own.  The
// first parts' sums are loaded together with the maxima, so that one latency
// covers both.
template <int DP, int ROWS, bool BF, int SPLITS, bool SPREAD>
__global__ void __launch_bounds__(JOIN_THREADS) attn_join_kernel(AttnArgs a)
{
    constexpr int JR = SPREAD ? 1 : 4, STEP = SPREAD ? JOIN_WAVES : 1;  // rows and parts of a wavefront's turn
    constexpr int JOIN_AHEAD = SPREAD ? 8 : 4;
    static_assert(ROWS % (4 * JOIN_WAVES) == 0, "whole row groups");
    typedef float vrows __attribute__((ext_vector_type(JR)));
    __shared__ float2 meet[JOIN_WAVES][64];
    const Workspace<ROWS, DP, SPLITS> &ws = *(const Workspace<ROWS, DP, SPLITS> *)a.workspace;
    if (__builtin_expect((int)blockIdx.x >= a.joins, 0)) {
        fill_rows<BF>(a, (blockIdx.x - a.joins) * gridDim.y + blockIdx.y, (gridDim.x - a.joins) * gridDim.y);
        return;
    }
    const Join j = ws.join[blockIdx.x];
    if (a.by_item) {
        // no range begins an item that has no units
        const int blocks = most_blocks<ROWS>(a);
        const Request q = request_of(a, blockIdx.x / blocks / a.kv.kv_heads);
        if ((int)(blockIdx.x % blocks) >= row_blocks<ROWS>(a, q))
            return;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i0 = SPREAD ? blockIdx.y : (blockIdx.y * JOIN_WAVES + wave) * JR, turn = SPREAD ? wave : 0, n = j.parts;
    if (n == 0 || i0 >= j.rows)  // (the same for the workgroup where it meets)
        return;
    const Part<ROWS, DP> *parts = ws.part + 2 * j.range;
    auto part = [&](int k) -> const Part<ROWS, DP> & { return parts[k ? 2 * k : j.second]; };
    const int D = a.kv.head_dim, d = 2 * lane < D ? 2 * lane : 0;

    // (rows past the item's are in the workspace too, and not used)
    float2 ahead[JOIN_AHEAD][JR];
#pragma unroll
    for (int k = 0; k < JOIN_AHEAD; ++k)
#pragma unroll
        for (int r = 0; r < JR; ++r)
            ahead[k][r] = turn + k * STEP < n ? *(const float2 *)&part(turn + k * STEP).o[i0 + r][d]
                                              : make_float2(0.f, 0.f);
    vrows m0 = NO_SCORE, l0 = 0.f;  // of the first 64 parts
    if (lane < n) {
        m0 = *(const vrows *)&part(lane).m[i0];
        l0 = *(const vrows *)&part(lane).l[i0];
    }
    vrows top = m0;
    for (int k = lane + 64; k < n; k += 64) {
        const vrows m = *(const vrows *)&part(k).m[i0];
#pragma unroll
        for (int r = 0; r < JR; ++r)
            top[r] = fmaxf(top[r], m[r]);
    }
#pragma unroll
    for (int s = 32; s; s >>= 1)
#pragma unroll
        for (int r = 0; r < JR; ++r)
            top[r] = fmaxf(top[r], __shfl_xor(top[r], s));
    vrows total = 0.f;
    float2 o[JR] = {};
    for (int k0 = 0; k0 < n; k0 += 64) {
        // factors of 64 parts, a part a lane
        vrows f = 0.f;
        if (k0 + lane < n) {
            const vrows m = k0 ? *(const vrows *)&part(k0 + lane).m[i0] : m0;
            const vrows l = k0 ? *(const vrows *)&part(k0 + lane).l[i0] : l0;
#pragma unroll
            for (int r = 0; r < JR; ++r) {
                f[r] = fast_exp2(m[r] - top[r]);
                total[r] += f[r] * l[r];
            }
        }
        auto factor = [&](int r, int k) {
            return __builtin_bit_cast(float,
                                      __builtin_amdgcn_readlane(__builtin_bit_cast(int, (float)f[r]), k - k0));
        };
        const int k1 = min(n, k0 + 64);
        int k = k0 + turn;
        if (k0 == 0) {
#pragma unroll
            for (int i = 0; i < JOIN_AHEAD; ++i, k += STEP)
                if (k < k1)
#pragma unroll
                    for (int r = 0; r < JR; ++r) {
                        const float w = factor(r, k);
                        o[r].x += w * ahead[i][r].x;
                        o[r].y += w * ahead[i][r].y;
                    }
        }
#pragma unroll 4
        for (; k < k1; k += STEP)
#pragma unroll
            for (int r = 0; r < JR; ++r) {
                const float w = factor(r, k);
                const float2 v = *(const float2 *)&part(k).o[i0 + r][d];
                o[r].x += w * v.x;
                o[r].y += w * v.y;
            }
    }
#pragma unroll
    for (int s = 32; s; s >>= 1)
#pragma unroll
        for (int r = 0; r < JR; ++r)
            total[r] += __shfl_xor(total[r], s);
    if constexpr (SPREAD) {
        meet[wave][lane] = o[0];
        __syncthreads();
        if (wave != 0)
            return;
#pragma unroll
        for (int w = 1; w < JOIN_WAVES; ++w) {
            o[0].x += meet[w][lane].x;
            o[0].y += meet[w][lane].y;
        }
    }
    if (2 * lane >= D)
        return;
    const int group = a.heads / a.kv.kv_heads;
#pragma unroll
    for (int r = 0; r < JR; ++r)
        if (i0 + r < j.rows) {
            const float inv = inverse(total[r]);
            *(uint32_t *)(out_row(a, j.first, j.kvh, j.row0 + i0 + r, group) + 2 * lane) =
                pack2<BF>(o[r].x * inv, o[r].y * inv);
        }
}

// ---------------------------------------------------------------------------
// launch
// ---------------------------------------------------------------------------

// How a call's items are run: rows of an item by the most rows that a request
// has per key/value head.  Up to 16 rows by the rows kernel, as against the block
// kernel with 64: one request at 4096 positions 13.6 and 15.6 us, 64 requests up to
// 2047 with heads of 64 32.4 and 40.0; but with heads of 128 that fill the chip the
// block kernel is a little better, 64 at 8192 345 to 358 and 340 (pages head by head
// 334 and 352), 64 up to 2047 59.8 to 62 and 58.3, 512 up to 400 111 and 105.  The rule
// goes by rows alone.
enum Shape { ROWS16, ROWS64, ROWS128 };

Shape shape_of(int max_new, int heads, int kv_heads)
{
    const int rows = max_new * (heads / kv_heads);
    return rows <= 16 ? ROWS16 : rows <= 64 ? ROWS64 : ROWS128;
}

// Workgroups a CU, by registers.  Narrow heads of few rows need few: four finished
// 64 requests of up to 2047 positions, 64 wide, in 41 us and two in 45 when this
// was chosen; at 8192 positions, where starting up counts less, 199 and 192 us.
// Up to 64 rows of 128 elements with one (and seven tiles ahead), two and three (two
// tiles ahead): 64 trees of 16 at 8192 positions 479, 345 and 426 us, 16 trees 136,
// 114 and 122, one tree 25.6, 26.8 and 31.6.
constexpr int wgs_of(Shape s, int dp) { return s == ROWS16 && dp == 64 ? 4 : 2; }

// Rows up to which a join has a workgroup for each.  With that and with a
// wavefront for four rows: one request at 4096 positions, 32 rows in all, 14.3 and
// 23.0 us; four trees of 16 at 8192, 2048 rows, 43.1 and 46.7; eight, 4096 rows,
// 76.6 and 72.3; 16, 8192 rows, 131 and 124.
constexpr int JOIN_MOST = 2048;

template <int DP, int ROWS, bool BF, int WGS>
int run_attn(const void *kernel, const AttnArgs &a, hipStream_t stream)
{
    constexpr int SPLITS = WGS * CUS;
    AttnArgs args = a;
    const int rows = a.max_new * (a.heads / a.kv.kv_heads), blocks = (rows + ROWS - 1) / ROWS;
    const long long items = (long long)a.R * a.kv.kv_heads * blocks;
    // units of 64 positions at least, on a line numbered in 32 bits
    if (((long long)a.max_pages * a.kv.page_size / 64 + 5) * items >= (1ll << 31))
        return SBVR_E_UNSUPPORTED;
    args.by_item = items < SPLITS;
    void *argv[] = {&args};
    const int st = launch_kernel(kernel, dim3(SPLITS), dim3(ATTN_THREADS), 0, stream, argv);
    if (st != SBVR_OK)
        return st;
    const int joins = args.by_item ? (int)items : SPLITS - 1, most = min(rows, ROWS);  // the last range divides nothing
    const bool spread = (long long)joins * most <= JOIN_MOST;
    const int y = spread ? most : (most + 15) / 16;
    // workgroups that look after the rows of no item: one for four tokens, up to the chip's fill
    const int fill = a.cut == 0 ? (min(a.T / JOIN_WAVES + 1, 4 * CUS) + y - 1) / y : 0;
    args.joins = joins;
    return launch_kernel(spread ? (const void *)attn_join_kernel<DP, ROWS, BF, SPLITS, true>
                                : (const void *)attn_join_kernel<DP, ROWS, BF, SPLITS, false>,
                         dim3(joins + fill, y), dim3(JOIN_THREADS), 0, stream, argv);
}

template <int DP, int DS, bool PAD, bool BF>
int by_shape(const AttnArgs &a, hipStream_t stream)
{
    constexpr int W = wgs_of(ROWS16, DP), V = wgs_of(ROWS128, DP);
    switch (shape_of(a.max_new, a.heads, a.kv.kv_heads)) {
    case ROWS16: return run_attn<DP, 16, BF, W>((const void *)attn_rows_kernel<DP, DS, PAD, BF, W>, a, stream);
    case ROWS64: return run_attn<DP, 64, BF, V>((const void *)attn_block_kernel<DP, DS, PAD, 1, BF, V>, a, stream);
    default: return run_attn<DP, 128, BF, V>((const void *)attn_block_kernel<DP, DS, PAD, 2, BF, V>, a, stream);
    }
}

template <int DP, int DS>
int by_type(const AttnArgs &a, hipStream_t stream)
{
    const bool bf = a.kv.dtype == SBVR_BF16;
    if (a.kv.head_dim == 32 * DS)
        return bf ? by_shape<DP, DS, false, true>(a, stream) : by_shape<DP, DS, false, false>(a, stream);
    return bf ? by_shape<DP, DS, true, true>(a, stream) : by_shape<DP, DS, true, false>(a, stream);
}

template <int DP>
size_t workspace_of(Shape s)
{
    switch (s) {
    case ROWS16: return sizeof(Workspace<16, DP, wgs_of(ROWS16, DP) * CUS>);
    case ROWS64: return sizeof(Workspace<64, DP, wgs_of(ROWS64, DP) * CUS>);
    default: return sizeof(Workspace<128, DP, wgs_of(ROWS128, DP) * CUS>);
    }
}

size_t attn_workspace_bytes(int, int max_new, int heads, int kv_heads, int head_dim)
{
    const Shape s = shape_of(max_new, heads, kv_heads);
    return head_dim <= 64 ? workspace_of<64>(s) : workspace_of<128>(s);
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
