// The selection of a beam search: per request the best continuations of its beams
// over the vocabulary, and the beams that end.
//
// Two launches.  The first reads the logits once: a row is cut into parts, one a
// workgroup, which goes through its part in tiles held in registers and leaves the
// part's sum of exponentials and its `keep` = n + n_end best logits (no beam can have
// more continuations among the chosen ones, and an end that counts is among the n
// best).  The second joins a request's parts.
//
// What a tile adds to the best so far: each four lanes' largest logit is a group's, 64
// groups in all, and the keep-th largest of these is a value that at least `keep`
// logits reach, so what is below it cannot be chosen.  What is left -- hardly more
// than `keep` -- goes into a list, whose entries are ranked by counting the better
// ones; a longer list, as of a tile that is hardly filled, is first thinned out the
// same way.  A logit is compared with its place: key = (logit, ~token) as one
// number, so equal logits are ordered and keys are all different.  Where so many are
// alike that the list does not hold them, those above the value go into it and of the
// equal ones the `keep` first.
//
// Sums: exp(l - r) = 2^(l log2 e - c), one rounding for the exponent; r = c / log2 e
// is what the sum refers to, so c's own rounding costs nothing.  (The rounding of
// log2 e is 1.4e-8 of the exponent; between a request's beams nearly all of that
// cancels.)  Binary32 within a lane and a tile, binary64 between lanes, tiles and
// parts: two continuations' order may hang on the last bits.
//
// Memory-bound for many rows: 245 rows of 131072 in binary32 (128 MB, 20 to 21 us of a
// plain read) take 31 us, in binary16 26; of that 3 to 5 are the join, the rest above
// the read the beginning of the workgroups and, in binary16, the exponentials.  Few
// rows are a chain of latencies: four rows of 50001 8.8 us, an empty launch 2.1.
#include "step.h"

namespace sbvr {

// BEAM_ENTRIES: of a request's parts together, which the join holds in registers and,
// if need be, in LDS
constexpr int BEAM_THREADS = 256, BEAM_WAVES = BEAM_THREADS / 64, BEAM_ENTRIES = 2816;
static_assert(BEAM_ENTRIES < 4096, "places have 12 bits");
constexpr int BEAM_RANKED = 2 * BEAM_THREADS, BEAM_LIST = 2048 + SBVR_BEAM_KEEP_MAX;  // logits to be ranked, and to be thinned out before
constexpr float LOG2E = 1.44269502f, LARGEST = 3.402823466e38f;

struct PartSum {
    double sum, reference;  // of exp(logit - reference); reference -infinity: the part has no logit
};

struct BeamShape {
    int parts, tiles, keep;  // parts of a row, tiles of a part, entries of a part
};

// Numbers in the order of the logits, 0 below that of every logit.
__device__ __forceinline__ uint32_t ordered(float v)
{
    const uint32_t u = __float_as_uint(v);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t ordered(double v)
{
    const uint64_t u = __double_as_longlong(v);
    return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }

constexpr uint64_t END_ENTRY = 1ull << 31;  // cleared in an entry whose token is an end (tokens have 30 bits)

// (+infinity as the largest number, and -0 as 0)
__device__ __forceinline__ uint64_t key_of(float v, int token)
{
    return (uint64_t)ordered(fminf(v, LARGEST) + 0.f) << 32 | (uint32_t)~token;
}

template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float dpp(float v, float out)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(out), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double dpp(double v, double out)
{
    const uint64_t u = __double_as_longlong(v), o = __double_as_longlong(out);
    const uint32_t low = __builtin_amdgcn_update_dpp((uint32_t)o, (uint32_t)u, CTRL, ROWS, 0xf, false);
    const uint32_t high = __builtin_amdgcn_update_dpp((uint32_t)(o >> 32), (uint32_t)(u >> 32), CTRL, ROWS, 0xf, false);
    return __longlong_as_double((uint64_t)high << 32 | low);
}

// A wavefront's sum, in its last lane, and its maximum, in all.  (Row shifts by 1,
// 2, 4 and 8, and the rows' last lanes to the rows behind.)
__device__ __forceinline__ double sum_to_last(double v)
{
    v += dpp<0x111>(v, 0.);
    v += dpp<0x112>(v, 0.);
    v += dpp<0x114>(v, 0.);
    v += dpp<0x118>(v, 0.);
    v += dpp<0x142, 0xa>(v, 0.);
    v += dpp<0x143, 0xc>(v, 0.);
    return v;
}
__device__ __forceinline__ float max_of_wave(float v)
{
    v = fmaxf(v, dpp<0x111>(v, -INFINITY));
    v = fmaxf(v, dpp<0x112>(v, -INFINITY));
    v = fmaxf(v, dpp<0x114>(v, -INFINITY));
    v = fmaxf(v, dpp<0x118>(v, -INFINITY));
    v = fmaxf(v, dpp<0x142, 0xa>(v, -INFINITY));
    v = fmaxf(v, dpp<0x143, 0xc>(v, -INFINITY));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// exp(x) for x <= 0 and log(x) for a normal x, to 2^-36: the join is a chain of such
// steps, and the sums are no better.  (Taylor's series to the 9th power behind the
// powers of 2: the next term is 7e-12; log m = 2 artanh((m - 1) / (m + 1)) for m
// between the roots of 1/2 and 2, to the 13th power: 5e-13.)
__device__ __forceinline__ double exp_of(double x)
{
    x = fmax(x, -700.);
    const double k = rint(x * 1.4426950408889634), r = fma(-k, 0.6931471805599453, x);
    double p = 1. / 362880;
    p = fma(p, r, 1. / 40320);
    p = fma(p, r, 1. / 5040);
    p = fma(p, r, 1. / 720);
    p = fma(p, r, 1. / 120);
    p = fma(p, r, 1. / 24);
    p = fma(p, r, 1. / 6);
    p = fma(p, r, 1. / 2);
    p = fma(p, r, 1.);
    p = fma(p, r, 1.);
    return ldexp(p, (int)k);
}
__device__ __forceinline__ double log_of(double x)
{
    int e = __builtin_amdgcn_frexp_exp(x);
    double m = __builtin_amdgcn_frexp_mant(x);
    const bool low = m < 0.7071067811865476;
    m = low ? 2. * m : m;
    e -= low;
    const double d = m + 1.;
    double inverse = __builtin_amdgcn_rcp(d);
    inverse = fma(fma(-d, inverse, 1.), inverse, inverse);
    inverse = fma(fma(-d, inverse, 1.), inverse, inverse);
    const double z = (m - 1.) * inverse, q = z * z;
    double p = 2. / 13;
    p = fma(p, q, 2. / 11);
    p = fma(p, q, 2. / 9);
    p = fma(p, q, 2. / 7);
    p = fma(p, q, 2. / 5);
    p = fma(p, q, 2. / 3);
    p = fma(p, q, 2.);
    return fma((double)e, 0.6931471805599453, p * z);
}

// The `keep` largest of the c > keep different numbers in list, to kept, in no order:
// bit by bit the largest number that `keep` of them reach.  counts: 65 numbers.
template <typename F>
__device__ __forceinline__ void largest(F number, int c, int keep, uint64_t *kept, int *counts)
{
    const int lane = threadIdx.x & 63;
    __syncthreads();
    if (threadIdx.x < 65)
        counts[threadIdx.x] = 0;
    __syncthreads();
    uint64_t least = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t candidate = least | 1ull << bit;
        int reach = 0;
        for (int i = threadIdx.x; i < (c + 63) / 64 * 64; i += BEAM_THREADS)
            reach += __popcll(__ballot(i < c && number(min(i, c - 1)) >= candidate));
        if (lane == 0 && reach)
            atomicAdd(&counts[bit], reach);
        __syncthreads();
        if (counts[bit] >= keep)
            least = candidate;
        if (counts[bit] == keep)
            break;
    }
    for (int i = threadIdx.x; i < c; i += BEAM_THREADS) {
        const uint64_t v = number(i);
        if (v && v >= least)
            kept[atomicAdd(&counts[64], 1)] = v;
    }
    __syncthreads();
}

// The keep-th largest of the lanes' numbers, to the bits from `last` up.
__device__ __forceinline__ uint32_t reached_by(uint32_t number, int keep, int last)
{
    uint32_t least = 0;
#pragma unroll
    for (int bit = 31; bit >= last; --bit) {
        const uint32_t candidate = least | 1u << bit;
        least = __popcll(__ballot(number >= candidate)) >= keep ? candidate : least;
    }
    return least;
}

// Thins out the c different keys of list to those whose value a quarter of `keep`
// threads of each wavefront reach, and returns how many are left.
__device__ __forceinline__ int thin_out(uint64_t *list, int c, int keep, uint32_t *least_of, int *count)
{
    const int tid = threadIdx.x;
    uint32_t mine = 0, least = ~0u;
    for (int i = tid; i < c; i += BEAM_THREADS)
        mine = max(mine, (uint32_t)(list[i] >> 32));
    mine = reached_by(mine, (keep + BEAM_WAVES - 1) / BEAM_WAVES, 0);
    __syncthreads();
    if ((tid & 63) == 0)
        least_of[tid >> 6] = mine;
    if (tid == 0)
        *count = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < BEAM_WAVES; ++w)
        least = min(least, least_of[w]);
    // (what is written lies in what all threads have read)
    for (int i0 = 0; i0 < c; i0 += BEAM_THREADS) {
        const uint64_t key = i0 + tid < c ? list[i0 + tid] : 0;
        __syncthreads();
        if (key && (uint32_t)(key >> 32) >= least)
            list[atomicAdd(count, 1)] = key;
        __syncthreads();
    }
    return *count;
}

// CH: pieces of eight logits a thread holds of a tile.
// Six wavefronts a SIMD: 256 rows of 131072 in binary16 take 26.2 us with the 80
// registers that this leaves, 27.5 with five and 82 (seven: 42, with spills).
template <typename T, int CH>
__global__ void __launch_bounds__(BEAM_THREADS, 6) beam_part_kernel(sbvr_beam_args a, BeamShape s, PartSum *sums, uint64_t *entries)
{
    constexpr int TILE = 8 * CH * BEAM_THREADS, WAVES = BEAM_WAVES;
    __shared__ uint64_t list[BEAM_LIST], kept[SBVR_BEAM_KEEP_MAX];  // the best so far, and what may be better
    __shared__ float group[2][64];
    __shared__ int count, counts[65], ends[SBVR_BEAM_KEEP_MAX], equal_before[WAVES];
    __shared__ uint32_t least_of[BEAM_WAVES];
    __shared__ double wave_sum[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, row = blockIdx.x / s.parts, part = blockIdx.x % s.parts;
    if (!isfinite(uniform_load(a.scores + row)))
        return;  // the join knows
    const T *in = (const T *)a.logits + row * a.logits_stride;

    if (tid < a.n_end)
        ends[tid] = a.end_tokens[tid];
    double total = 0., reference = -INFINITY;
    float top = -INFINITY, offset = 0.f;
    uint32_t floor = ordered(-LARGEST);  // what a logit has to reach: more than the keep-th best so far
    int have = 0;
    const int first_tile = part * s.tiles;
    for (int tile = first_tile; tile < first_tile + s.tiles && (long long)tile * TILE < a.V; ++tile) {
        float x[CH][8];
        // a piece that would pass the row's end is moved back to end with it; its
        // first elements belong to the piece before
        const int v0 = tile * TILE + tid * 8;
        auto at = [&](int c) { return max(min(v0 + c * 8 * BEAM_THREADS, a.V - 8), 0); };
        if (a.V >= 8) {
            Words<T> w[CH];
#pragma unroll
            for (int c = 0; c < CH; ++c)
                w[c] = load_words(in + at(c));
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const Loose<T, 8> l = from_words<T>(w[c]);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[c][e] = (float)l.e[e];
            }
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[c][e] = (float)in[min(e, a.V - 1)];
        }
        if ((tile + 1ll) * TILE > a.V)  // the row's last tile
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[c][e] = at(c) + e >= v0 + c * 8 * BEAM_THREADS && at(c) + e < a.V ? x[c][e] : -INFINITY;
        float piece_top[CH], best = -INFINITY;  // (NaN is passed over)
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            piece_top[c] = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                piece_top[c] = fmaxf(piece_top[c], x[c][e]);
            best = fmaxf(best, piece_top[c]);
        }
        float in_group = fmaxf(best, dpp<0xb1>(best, best));         // lanes 1 0 3 2
        in_group = fmaxf(in_group, dpp<0x4e>(in_group, in_group));  // lanes 2 3 0 1
        float *groups = group[tile & 1];
        if ((tid & 3) == 0)
            groups[tid >> 2] = in_group;
        // many to keep: the 64 groups' maxima are no close bound, the lanes' of each
        // wavefront are (128 rows of 131072 in binary16: 64 kept 68.3 us, by the groups
        // 70.4; 48 34.0 both ways; 32 29.4 by the groups, 30.1)
        const bool many = s.keep > 32;
        if (many) {
            const uint32_t reached = reached_by(ordered(best), (s.keep + WAVES - 1) / WAVES, 16);
            if (lane == 0)
                least_of[tid >> 6] = reached;
        }
        if (tid == 0)
            count = have;
        __syncthreads();

        const float mine = groups[lane];
        float tile_top = max_of_wave(mine);
        uint32_t least = ~0u;
        if (many)
#pragma unroll
            for (int w = 0; w < WAVES; ++w)
                least = min(least, least_of[w]);
        else
            least = reached_by(ordered(mine), s.keep, 16);
        float least_value = fminf(unordered(max(least, floor)), LARGEST);
        if (tile_top > -INFINITY) {  // the same for all
            tile_top = fminf(tile_top, LARGEST);
            // differences instead where c is so large that 2 to its rounding is (2^-25 of
            // c: 0.04 at a million); the largest so far, whose c this tile takes, decides
            const bool huge = fabsf(fmaxf(tile_top, top)) > 1e6f;
            if (tile_top > top) {
                const double now = huge ? (double)tile_top : (double)(tile_top * LOG2E) * (1. / (double)LOG2E);
                total *= exp_of(reference - now);  // (0 before the first)
                reference = now;
                offset = tile_top * LOG2E;
                top = tile_top;
            }
            float sum = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    sum += __builtin_amdgcn_exp2f(__builtin_fmaf(x[c][e], LOG2E, -offset));
            if (huge || sum != sum || sum > LARGEST) {
                sum = 0.f;
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float l = x[c][e] == x[c][e] ? fminf(x[c][e], LARGEST) : -INFINITY;
                        sum += __builtin_amdgcn_exp2f(huge ? (l - top) * LOG2E : __builtin_fmaf(l, LOG2E, -offset));
                    }
            }
            total += (double)sum;

#pragma unroll
            for (int c = 0; c < CH; ++c)
                if (piece_top[c] >= least_value)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (x[c][e] >= least_value) {
                            const int k = atomicAdd(&count, 1);
                            if (k < BEAM_LIST)
                                list[k] = key_of(x[c][e], at(c) + e);
                        }
        }
        __syncthreads();
        int c = count;
        const bool more = c > have;
        const uint64_t *from = list;
        if (c > BEAM_LIST) {
            // too many alike: the value to the last bit, those above it, and the first
            // of those that have it
            least = reached_by(ordered(mine), s.keep, 0);
            least_value = fminf(unordered(max(least, floor)), LARGEST);
            __syncthreads();
            if (tid == 0)
                count = have;
            __syncthreads();
            int equal = 0;  // of the pieces before, in all threads
#pragma unroll 1
            for (int i = 0; i < CH; ++i) {
                // (read again: held until here, they cost every tile registers)
                const int v = tile * TILE + (i * BEAM_THREADS + tid) * 8;
                float l[8];
                int own = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    l[e] = v + e < a.V ? (float)in[min(v + e, a.V - 1)] : -INFINITY;
                    l[e] = l[e] == l[e] ? fminf(l[e], LARGEST) : -INFINITY;
                    own += l[e] == least_value;
                    if (l[e] > least_value) {
                        const int k = atomicAdd(&count, 1);
                        if (k < BEAM_LIST)
                            list[k] = key_of(l[e], v + e);
                    }
                }
                int up = own;  // with the lanes before
#pragma unroll
                for (int m = 1; m < 64; m <<= 1) {
                    const int other = __shfl_up(up, m);
                    up += lane >= m ? other : 0;
                }
                __syncthreads();
                if (lane == 63)
                    equal_before[tid >> 6] = up;
                __syncthreads();
                int place = equal + up - own;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    place += w < tid >> 6 ? equal_before[w] : 0;
                    equal += equal_before[w];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (l[e] == least_value && place++ < s.keep) {
                        const int k = atomicAdd(&count, 1);
                        if (k < BEAM_LIST)
                            list[k] = key_of(l[e], v + e);
                    }
            }
            __syncthreads();
            c = count;
        }
        if (c > BEAM_LIST) {
            // even so, as in a tile whose best lie together: from the logits in memory
            const int first = tile * TILE, n = min(TILE, a.V - first);
            largest([&](int i) -> uint64_t {
                if (i < have)
                    return list[i];
                const float l = (float)in[first + i - have];
                return l > -INFINITY ? key_of(l, first + i - have) : 0;
            }, n + have, s.keep, kept, counts);
            from = kept;
            c = s.keep;
        } else if (c > BEAM_THREADS) {
            c = thin_out(list, c, s.keep, least_of, &count);
        }
        if (from == list && c > BEAM_RANKED) {
            largest([&](int i) { return list[i]; }, c, s.keep, kept, counts);
            from = kept;
            c = s.keep;
        }
        if (more) {
            uint64_t key[BEAM_RANKED / BEAM_THREADS];
            int better[BEAM_RANKED / BEAM_THREADS] = {};
#pragma unroll
            for (int i = 0; i < BEAM_RANKED / BEAM_THREADS; ++i) {
                key[i] = 0;
                if (i * BEAM_THREADS + tid < c) {
                    key[i] = from[i * BEAM_THREADS + tid];
#pragma unroll 8
                    for (int j = 0; j < c; ++j)
                        better[i] += from[j] > key[i];
                }
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < BEAM_RANKED / BEAM_THREADS; ++i)
                if (key[i] && better[i] < s.keep)
                    list[better[i]] = key[i];
            have = min(c, s.keep);
            __syncthreads();
            if (have == s.keep)
                floor = (uint32_t)(list[s.keep - 1] >> 32) + 1;
        }
    }
    if (tid < s.keep) {
        uint64_t entry = tid < have ? list[tid] : 0;
        for (int e = 0; e < a.n_end; ++e)
            if (entry && ends[e] == (int)~(uint32_t)entry)
                entry &= ~END_ENTRY;  // (once: then the token is another)
        entries[(long long)blockIdx.x * s.keep + tid] = entry;
    }
    total = sum_to_last(total);
    if (lane == 63)
        wave_sum[tid >> 6] = total;
    __syncthreads();
    if (tid == 0) {
        total = 0.;
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
            total += wave_sum[w];
        sums[blockIdx.x] = PartSum{total, reference};
    }
}

// Candidates to be ranked by counting, without thinning out (77 steps, some 15 us) before:
// of 8 equal rows of 131072 and n = 4 there are 512, whose ranking alone made it 66 us
// instead of 40; n = 16 394 instead of 53.
constexpr int JOIN_RANKED = 256;

// Of equal scores the lower beam is the better, in a beam the higher logit -- a score of
// -1e30 has no room for them --, and of equal logits the lower place: entries are in the
// order of beam, part and rank, and those of a part in that of their keys.  So the place
// decides unless two of a beam have one score and different logits, which the next number
// behind the lower one's logit shows: it then has that score too.
struct Candidate {
    double score;
    int place;  // number of the entry
};
__device__ __forceinline__ bool better_than(const Candidate &a, const Candidate &b)
{
    return (a.score > b.score) | ((a.score == b.score) & (a.place < b.place));  // (no branch: LDS reads stay in flight)
}
// The whole order of equal scores as one number of 49 bits, more than 0.
constexpr int ORDER_BITS = 49;
__device__ __forceinline__ uint64_t order_of(uint32_t logit, int beam, int place)
{
    return (uint64_t)(SBVR_BEAMS_MAX - 1 - beam) << 44 | (uint64_t)logit << 12 | (uint64_t)(4095 - place);
}

// One request.  A chain of latencies: the entries are loaded beside the sums.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) beam_join_kernel(sbvr_beam_args a, BeamShape s, const PartSum *sums,
                                                            const uint64_t *entries)
{
    constexpr int PER = THREADS == 1024 ? (BEAM_ENTRIES + 1023) / 1024 : 4, WAVES = THREADS / 64;
    constexpr uint32_t END = 1u << 31;
    extern __shared__ double list_score[];  // and behind them, each entry's place, beam and whether it is an end, its token and logit
    __shared__ double add[SBVR_BEAMS_MAX], beam_reference[SBVR_BEAMS_MAX];
    __shared__ __attribute__((aligned(16))) uint32_t group[256];
    __shared__ int rank[256], count, hides;  // hides: a score may be that of another logit of its beam too
    __shared__ float score_out[SBVR_BEAM_KEEP_MAX], ended[SBVR_BEAMS_MAX];
    __shared__ int token_out[SBVR_BEAM_KEEP_MAX], parent_out[SBVR_BEAM_KEEP_MAX], ended_token[SBVR_BEAMS_MAX];
    const int tid = threadIdx.x, lane = tid & 63, per_beam = s.parts * s.keep, all = a.B * per_beam;
    const long long request = blockIdx.x;
    uint32_t *list_what = (uint32_t *)(list_score + all), *list_token = list_what + all, *list_logit = list_token + all;
    entries += request * all;
    sums += request * a.B * s.parts;

    uint64_t key[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i)
        key[i] = entries[min(i * THREADS + tid, all - 1)];
    // what a beam's logits, less the reference of its sum, are added to: its score
    // without the sum's logarithm
    for (int b = tid >> 6; b < a.B; b += WAVES) {
        const float base = a.scores[request * a.B + b];
        PartSum first = {0., -INFINITY};
        if (lane < s.parts)
            first = sums[b * s.parts + lane];  // (of a beam that is none not written, and not used)
        double value = -INFINITY, reference = -INFINITY;
        if (isfinite(base)) {
            float top = (float)first.reference;
            for (int p = lane + 64; p < s.parts; p += 64)
                top = fmaxf(top, (float)sums[b * s.parts + p].reference);
            top = max_of_wave(top);
            if (top > -INFINITY) {
                reference = top;
                double sum = first.sum * exp_of(first.reference - reference);  // (0 for a part without logits)
                for (int p = lane + 64; p < s.parts; p += 64) {
                    const PartSum q = sums[b * s.parts + p];
                    sum += q.sum * exp_of(q.reference - reference);
                }
                value = (double)base - log_of(sum_to_last(sum));
            }
        }
        if (lane == 63) {
            add[b] = value;
            beam_reference[b] = reference;
        }
    }
    if (tid < 256)
        rank[tid] = group[tid] = 0;
    if (tid < 64) {
        score_out[tid] = -INFINITY;
        token_out[tid] = parent_out[tid] = -1;
    }
    if (tid < SBVR_BEAMS_MAX) {
        ended[tid] = -INFINITY;
        ended_token[tid] = -1;
    }
    if (tid == 0)
        count = hides = 0;
    __syncthreads();

    // As in a tile: the n-th largest of 64 groups' best scores that go on (256 where n
    // is large), here rounded to binary32, which keeps their order, leaves hardly more
    // than the n best.
    float mine = -INFINITY;
    double score[PER];
    int beam[PER];
    bool same_as_next = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int place = i * THREADS + tid;
        beam[i] = small_div(min(place, all - 1), per_beam, 1.f / (float)per_beam);
        // (the score of a beam that is none is -infinity)
        const double value = add[beam[i]] + ((double)unordered((uint32_t)(key[i] >> 32)) - beam_reference[beam[i]]);
        const double next = add[beam[i]] + ((double)unordered((uint32_t)(key[i] >> 32) + 1) - beam_reference[beam[i]]);
        score[i] = (place < all) & (key[i] != 0) & (add[beam[i]] > -INFINITY) ? value : -INFINITY;
        same_as_next |= (next == score[i]) & (score[i] > -INFINITY);
        mine = fmaxf(mine, key[i] & END_ENTRY ? (float)score[i] : -INFINITY);
    }
    // A group is every 64th or 256th thread: neighbours are of one list, in order.
    // (16 requests of 8 beams of 131072: n = 8 takes 18.5 us, with 256 groups 20.6; 14
    // 19.0 and 20.2; 16 21.2 so, with 64 groups 26.6.)
    const int groups = a.n >= 16 ? 256 : 64, slot = tid & (groups - 1), share = groups * groups / THREADS;
    if (mine > -INFINITY)
        atomicMax(&group[slot], ordered(mine));
    __syncthreads();
    const uint32_t number = group[slot];
    int above = 0;
#pragma unroll 4
    for (int j = tid / groups * share; j < (tid / groups + 1) * share; j += 4) {
        const uint4 g = *(const uint4 *)&group[j];
        above += (g.x > number) + (g.y > number) + (g.z > number) + (g.w > number);
    }
    if (above)
        atomicAdd(&rank[slot], above);
    __syncthreads();
    float least = INFINITY;
    for (int g = lane; g < groups; g += 64)
        if (rank[g] < a.n)
            least = fminf(least, group[g] ? unordered(group[g]) : -INFINITY);
    least = -max_of_wave(-least);
    int listed[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i)
        listed[i] = (score[i] > -INFINITY) & ((float)score[i] >= least);
    auto list_them = [&] {
        int mine_listed = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            mine_listed += listed[i];
        if (mine_listed) {
            int k = atomicAdd(&count, mine_listed);
            if (same_as_next)
                hides = 1;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (listed[i]) {
                    list_score[k] = score[i];
                    list_what[k] = (uint32_t)beam[i] << 16 | (i * THREADS + tid) | (key[i] & END_ENTRY ? 0 : END);
                    list_logit[k] = (uint32_t)(key[i] >> 32);
                    list_token[k++] = ~(uint32_t)(key[i] | END_ENTRY);
                }
        }
        __syncthreads();
        return count;
    };
    int c = list_them();
    if (c > JOIN_RANKED) {
        // Equal or nearly so: only what is no worse than the n-th best that goes on, found
        // bit by bit -- its score, and of those that have it the places that are left, or,
        // where their logits are not all alike, the orders.  Each step counts in a word of
        // its own.
        __syncthreads();
        if (tid < 256)
            group[tid] = 0;
        if (tid == 0)
            count = 0;
        __syncthreads();
        auto reach = [&](int word, auto in) {
            int mine = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                mine += __popcll(__ballot(listed[i] && (key[i] & END_ENTRY) && in(i)));
            if (lane == 0 && mine)
                atomicAdd(&group[word], (uint32_t)mine);
            __syncthreads();
            return (int)group[word];
        };
        uint64_t bound = 0;
        for (int bit = 63; bit >= 0; --bit) {
            const uint64_t candidate = bound | 1ull << bit;
            bound = reach(bit, [&](int i) { return ordered(score[i]) >= candidate; }) >= a.n ? candidate : bound;
        }
        const int equal = a.n - reach(64, [&](int i) { return ordered(score[i]) > bound; });
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (listed[i] && ordered(score[i]) == bound)
                group[65] = (uint32_t)(key[i] >> 32);  // any one's
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (listed[i] && ordered(score[i]) == bound && group[65] != (uint32_t)(key[i] >> 32))
                group[66] = 1;
        __syncthreads();
        int places = 0;  // as many as still leave `equal` of them, or fewer
        uint64_t last = 0;
        if (!group[66]) {
            for (int bit = 11; bit >= 0; --bit) {
                const int candidate = places | 1 << bit;
                const int n = reach(67 + bit, [&](int i) { return ordered(score[i]) == bound && i * THREADS + tid < candidate; });
                places = n <= equal ? candidate : places;
            }
        } else {
            places = 4096;
            for (int bit = ORDER_BITS - 1; bit >= 0; --bit) {
                const uint64_t candidate = last | 1ull << bit;
                const int n = reach(67 + bit, [&](int i) {
                    return ordered(score[i]) == bound &&
                           order_of((uint32_t)(key[i] >> 32), beam[i], i * THREADS + tid) >= candidate;
                });
                last = n >= equal ? candidate : last;
            }
        }
#pragma unroll
        for (int i = 0; i < PER; ++i)
            listed[i] &= (ordered(score[i]) > bound) |
                         ((ordered(score[i]) == bound) & (i * THREADS + tid < places) &
                          (order_of((uint32_t)(key[i] >> 32), beam[i], i * THREADS + tid) >= last));
        c = list_them();
    }
    for (int i = tid; i < c; i += THREADS) {
        const uint32_t w = list_what[i];
        const Candidate me = {list_score[i], (int)(w & 0xffff)};
        const uint32_t beam = (w >> 16) & 0x7fff;
        int better = 0, going = 0, same = 0;  // all, those that go on, and ends of the beam
        if (!hides) {
#pragma unroll 4
            for (int j = 0; j < c; ++j) {
                const uint32_t u = list_what[j];
                const int b = better_than(Candidate{list_score[j], (int)(u & 0xffff)}, me), end = u >> 31;
                better += b;
                going += b & ~end;
                same += b & end & (int)(((u >> 16) & 0x7fff) == beam);
            }
        } else {
            const uint64_t order = order_of(list_logit[i], beam, me.place);
            for (int j = 0; j < c; ++j) {
                const uint32_t u = list_what[j], of = (u >> 16) & 0x7fff;
                const int b = (list_score[j] > me.score) |
                              ((list_score[j] == me.score) & (order_of(list_logit[j], of, u & 0xffff) > order));
                const int end = u >> 31;
                better += b;
                going += b & ~end;
                same += b & end & (int)(of == beam);
            }
        }
        if (!(w & END)) {
            if (going < a.n) {
                token_out[going] = (int)list_token[i];
                parent_out[going] = beam;
                score_out[going] = (float)me.score;
            }
        } else if (better < a.n && same == 0) {
            ended[beam] = (float)me.score;
            ended_token[beam] = (int)list_token[i];
        }
    }
    __syncthreads();
    if (tid < a.n) {
        a.tokens[request * a.n + tid] = token_out[tid];
        a.parents[request * a.n + tid] = parent_out[tid];
        a.scores_out[request * a.n + tid] = score_out[tid];
    }
    if (tid < a.B) {
        a.ended[request * a.B + tid] = ended[tid];
        a.ended_tokens[request * a.B + tid] = ended_token[tid];
    }
}

namespace {

// pieces of a thread: large tiles unless the rows have too few of them for half of the chip
// (binary16, 8 beams: 8 rows of 131072 take 10.5 us with four, 12.2 with one; 256 rows 26
// and 47; 16 of 32000 10.7 and 10.1).  Where BEAM_ENTRIES leaves fewer parts than that a
// part has several tiles (8 rows of 131072, 64 continuations: 32 workgroups, 65 us).
int beam_pieces(long long rows, int V)
{
    return rows * ((V + 8191ll) / 8192) >= 128 ? 4 : 1;
}

BeamShape beam_shape(int R, int B, int V, int n, int n_end)
{
    BeamShape s;
    const int tile = 8 * BEAM_THREADS * beam_pieces((long long)R * B, V);
    const int tiles = (V + tile - 1) / tile;
    s.keep = n + n_end;
    // (and no more workgroups than a grid can have)
    const int rows = R * B > 0 ? R * B : 1, wide = (1 << 20) / rows;
    int most = BEAM_ENTRIES / (B * s.keep);
    if (most > wide)
        most = wide;
    s.parts = tiles < most ? tiles : most;
    s.tiles = (tiles + s.parts - 1) / s.parts;
    s.parts = (tiles + s.tiles - 1) / s.tiles;
    return s;
}

size_t sums_bytes(int R, int B, const BeamShape &s) { return (size_t)R * B * s.parts * sizeof(PartSum); }

template <typename T, int CH>
int run_parts(const sbvr_beam_args &a, const BeamShape &s, PartSum *sums, uint64_t *entries, hipStream_t stream)
{
    sbvr_beam_args args = a;
    BeamShape shape = s;
    void *argv[] = {&args, &shape, &sums, &entries};
    return launch_kernel((const void *)beam_part_kernel<T, CH>, dim3((unsigned)(a.R * a.B * s.parts)), dim3(BEAM_THREADS), 0,
                         stream, argv);
}

}  // namespace

size_t beam_workspace_bytes(int R, int B, int V, int n, int n_end)
{
    const BeamShape s = beam_shape(R, B, V, n, n_end);
    return sums_bytes(R, B, s) + (size_t)R * B * s.parts * s.keep * sizeof(uint64_t);
}

int launch_beam(const sbvr_beam_args &a, void *workspace, hipStream_t stream)
{
    const BeamShape s = beam_shape(a.R, a.B, a.V, a.n, a.n_end);
    PartSum *sums = (PartSum *)workspace;
    uint64_t *entries = (uint64_t *)((char *)workspace + sums_bytes(a.R, a.B, s));
    const bool large = beam_pieces((long long)a.R * a.B, a.V) == 4;
    int st;
    switch (a.dtype) {
    case SBVR_F16: st = large ? run_parts<f16_t, 4>(a, s, sums, entries, stream) : run_parts<f16_t, 1>(a, s, sums, entries, stream); break;
    case SBVR_BF16: st = large ? run_parts<bf16_t, 4>(a, s, sums, entries, stream) : run_parts<bf16_t, 1>(a, s, sums, entries, stream); break;
    default: st = large ? run_parts<float, 4>(a, s, sums, entries, stream) : run_parts<float, 1>(a, s, sums, entries, stream); break;
    }
    if (st != SBVR_OK)
        return st;
    sbvr_beam_args args = a;
    BeamShape shape = s;
    const PartSum *sums_in = sums;
    const uint64_t *entries_in = entries;
    void *argv[] = {&args, &shape, &sums_in, &entries_in};
    const int all = a.B * s.parts * s.keep;
    const size_t lds = (size_t)all * (sizeof(double) + 3 * sizeof(uint32_t));
    return all <= 1024 ? launch_kernel((const void *)beam_join_kernel<256>, dim3(a.R), dim3(256), lds, stream, argv)
                       : launch_kernel((const void *)beam_join_kernel<1024>, dim3(a.R), dim3(1024), lds, stream, argv);
}

}  // namespace sbvr
