// The selection of a beam search: per request the best continuations of its beams
// over the vocabulary, and the beams that end.
//
// Two launches.  The first reads the logits once: a row is cut into parts, one a
// workgroup, which goes through its part in tiles held in registers and leaves the
// part's largest logit, its sum of exponentials, and its `keep` = n + n_end best
// logits (no beam can have more continuations among the chosen ones, and an end
// that counts is among the n best).  The second joins a request's parts.
//
// What a tile adds to the best so far: each four lanes' best logit is a group's, 64
// groups in all, and the keep-th best of the groups is a value that at least `keep`
// logits reach, so what is below it cannot be chosen.  What is left -- hardly more
// than `keep` -- goes into a list, whose entries are ranked by counting the better
// ones.  A logit is compared with its place: key = (logit, ~token) as one number, so
// equal logits are ordered, keys are all different, and lists have a bound: the
// logits of `keep` groups.
//
// Sums: exp(l - max) = 2^((l - max) log2 e), with log2 e in two parts, since its
// rounding would show in every term alike; binary32 within a lane and a tile,
// binary64 between lanes, tiles and parts.  Two continuations' order may hang on the
// last bits of these sums.
#include "step.h"

namespace sbvr {

constexpr int BEAM_THREADS = 256, BEAM_ENTRIES = 4096;  // of a request's parts together
constexpr float LARGEST = 3.402823466e38f;
constexpr float LOG2E_HIGH = 1.44269502162933349609375f, LOG2E_LOW = 1.92596299112661746887e-8f;

struct PartSum {
    double sum;  // of exp(logit - top)
    float top;   // -infinity: the part has no logit
    float unused;
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
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }

__device__ __forceinline__ uint64_t key_of(float v, int token) { return (uint64_t)ordered(v) << 32 | (uint32_t)~token; }

__device__ __forceinline__ uint64_t shuffle_xor(uint64_t v, int mask)
{
    return (uint64_t)__shfl_xor((uint32_t)(v >> 32), mask) << 32 | __shfl_xor((uint32_t)v, mask);
}

// The `keep` largest of the c > keep different numbers in list, to kept, in no order.
__device__ void largest(const uint64_t *list, int c, int keep, uint64_t *kept, int *counts)
{
    const int lane = threadIdx.x & 63;
    __syncthreads();
    if (threadIdx.x < 65)
        counts[threadIdx.x] = 0;
    __syncthreads();
    uint64_t least = 0;  // bit by bit the largest number that `keep` of them reach
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t candidate = least | 1ull << bit;
        int reach = 0;
        for (int i = threadIdx.x; i < (c + 63) / 64 * 64; i += BEAM_THREADS)
            reach += __popcll(__ballot(i < c && list[min(i, c - 1)] >= candidate));
        if (lane == 0 && reach)
            atomicAdd(&counts[bit], reach);
        __syncthreads();
        if (counts[bit] >= keep)
            least = candidate;
    }
    for (int i = threadIdx.x; i < c; i += BEAM_THREADS)
        if (list[i] >= least)
            kept[atomicAdd(&counts[64], 1)] = list[i];
    __syncthreads();
}

// CH: pieces of eight logits a thread holds of a tile.
template <typename T, int CH>
__global__ void __launch_bounds__(BEAM_THREADS) beam_part_kernel(sbvr_beam_args a, BeamShape s, PartSum *sums, uint64_t *entries)
{
    constexpr int TILE = 8 * CH * BEAM_THREADS;
    extern __shared__ uint64_t list[];  // keep entries of the tiles before, and the logits of keep groups
    __shared__ uint64_t group[64], kept[SBVR_BEAM_KEEP_MAX], least_key;
    __shared__ int rank[64], count, counts[65];
    __shared__ float tile_top;
    __shared__ double lane_sum[BEAM_THREADS / 64];
    const int tid = threadIdx.x, row = blockIdx.x / s.parts, part = blockIdx.x % s.parts;
    if (!isfinite(uniform_load(a.scores + row)))
        return;  // the join knows
    const T *in = (const T *)a.logits + row * a.logits_stride;

    float top = -INFINITY;
    uint64_t floor_key = 1;  // the keep-th best so far
    int have = 0;
    double total = 0.;
    const int first_tile = part * s.tiles;
    for (int tile = first_tile; tile < first_tile + s.tiles && (long long)tile * TILE < a.V; ++tile) {
        float x[CH][8];
        int at[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int v = tile * TILE + (c * BEAM_THREADS + tid) * 8;
            Loose<T, 8> l;
            at[c] = max(min(v, a.V - 8), 0);
            if (a.V >= 8)
                l = from_words<T>(load_words(in + at[c]));
            else
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    l.e[e] = in[min(e, a.V - 1)];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[c][e] = at[c] + e >= v && at[c] + e < a.V ? (float)l.e[e] : -INFINITY;
        }
        float best = -INFINITY;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                best = fmaxf(best, x[c][e]);
        int token = 0;
#pragma unroll
        for (int c = CH - 1; c >= 0; --c)
#pragma unroll
            for (int e = 7; e >= 0; --e)
                token = x[c][e] == best ? at[c] + e : token;
        uint64_t mine = best > -INFINITY ? key_of(fminf(best, LARGEST), token) : 0;
        mine = max(mine, shuffle_xor(mine, 1));
        mine = max(mine, shuffle_xor(mine, 2));
        if ((tid & 3) == 0)
            group[tid >> 2] = mine;
        if (tid < 64)
            rank[tid] = 0;
        if (tid == 0) {
            least_key = 1;
            tile_top = -INFINITY;
            count = have;
        }
        __syncthreads();
        {
            const uint64_t g = group[tid & 63];
            int better = 0;
#pragma unroll
            for (int j = 0; j < 16; ++j)
                better += group[(tid >> 6) * 16 + j] > g;
            if (better)
                atomicAdd(&rank[tid & 63], better);
        }
        __syncthreads();
        if (tid < 64 && group[tid]) {
            if (rank[tid] == s.keep - 1)
                least_key = group[tid];
            if (rank[tid] == 0)
                tile_top = unordered((uint32_t)(group[tid] >> 32));
        }
        __syncthreads();
        if (tile_top > -INFINITY) {  // the same for all
            // NaN is passed over by the maxima above and the comparisons below, and
            // would show in the sum only; +infinity counts as the largest number
            auto clean = [&] {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[c][e] = x[c][e] == x[c][e] ? fminf(x[c][e], LARGEST) : -INFINITY;
            };
            if (tile_top >= LARGEST)
                clean();
            const float new_top = fmaxf(top, tile_top);
            total *= top > -INFINITY ? exp((double)top - (double)new_top) : 0.;
            top = new_top;
            auto exponentials = [&] {
                float sum = 0.f;
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float d = x[c][e] - top;
                        sum += __builtin_amdgcn_exp2f(__builtin_fmaf(d, LOG2E_HIGH, d * LOG2E_LOW));
                    }
                return sum;
            };
            float sum = exponentials();
            if (sum != sum) {
                clean();
                sum = exponentials();
            }
            total += (double)sum;
            const uint64_t least = max(least_key, floor_key);
            const float least_value = least > 1 ? unordered((uint32_t)(least >> 32)) : -INFINITY;
            if (mine >= least)  // something in the four lanes
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (x[c][e] > -INFINITY && x[c][e] >= least_value) {
                            const uint64_t key = key_of(x[c][e], at[c] + e);
                            if (key >= least)
                                list[atomicAdd(&count, 1)] = key;
                        }
        }
        __syncthreads();
        int c = count;
        if (c > have) {
            const uint64_t *from = list;
            if (c > BEAM_THREADS) {
                largest(list, c, s.keep, kept, counts);
                from = kept;
                c = s.keep;
            }
            const uint64_t key = tid < c ? from[tid] : 0;
            int better = 0;
            for (int j = 0; j < c; ++j)
                better += from[j] > key;
            __syncthreads();
            if (tid < c && better < s.keep)
                list[better] = key;
            have = min(c, s.keep);
            __syncthreads();
            if (have == s.keep)
                floor_key = list[s.keep - 1];
        }
    }
#pragma unroll
    for (int m = 32; m; m >>= 1)
        total += __shfl_xor(total, m);
    if ((tid & 63) == 0)
        lane_sum[tid >> 6] = total;
    __syncthreads();
    if (tid == 0) {
        total = 0.;
#pragma unroll
        for (int w = 0; w < BEAM_THREADS / 64; ++w)
            total += lane_sum[w];
        sums[blockIdx.x] = PartSum{total, top, 0.f};
    }
    if (tid < s.keep)
        entries[(long long)blockIdx.x * s.keep + tid] = tid < have ? list[tid] : 0;
}

struct Candidate {
    double score;
    int place;  // number of the entry; of equal scores the lower place is better
};
__device__ __forceinline__ bool better_than(const Candidate &a, const Candidate &b)
{
    return a.score > b.score || (a.score == b.score && a.place < b.place);
}

// One request.  Entries are in the order of beam, part and rank, so of those with
// equal scores the lower place has the lower beam, or token.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) beam_join_kernel(sbvr_beam_args a, BeamShape s, const PartSum *sums,
                                                            const uint64_t *entries)
{
    constexpr int PER = THREADS == 1024 ? BEAM_ENTRIES / 1024 : 4, WAVES = THREADS / 64;
    constexpr uint32_t END = 1u << 31;
    extern __shared__ double list_score[];  // and behind them, each entry's place, beam and whether it is an end
    __shared__ double add[SBVR_BEAMS_MAX];
    __shared__ float beam_top[SBVR_BEAMS_MAX];
    __shared__ Candidate group[64], least;
    __shared__ int rank[64], count;
    __shared__ float score_out[SBVR_BEAM_KEEP_MAX], ended[SBVR_BEAMS_MAX];
    __shared__ int token_out[SBVR_BEAM_KEEP_MAX], parent_out[SBVR_BEAM_KEEP_MAX], ended_token[SBVR_BEAMS_MAX];
    const int tid = threadIdx.x, lane = tid & 63, per_beam = s.parts * s.keep, all = a.B * per_beam;
    const long long request = blockIdx.x;
    uint32_t *list_what = (uint32_t *)(list_score + all);
    entries += request * all;
    sums += request * a.B * s.parts;

    // what a beam's logits, less the largest, are added to: its score without the
    // logarithm of its sum
    for (int b = tid >> 6; b < a.B; b += WAVES) {
        const float base = a.scores[request * a.B + b];
        double value = -INFINITY;
        float top = -INFINITY;
        if (isfinite(base)) {
            for (int p = lane; p < s.parts; p += 64)
                top = fmaxf(top, sums[b * s.parts + p].top);
#pragma unroll
            for (int m = 32; m; m >>= 1)
                top = fmaxf(top, __shfl_xor(top, m));
            if (top > -INFINITY) {
                double sum = 0.;
                for (int p = lane; p < s.parts; p += 64) {
                    const PartSum q = sums[b * s.parts + p];
                    if (q.top > -INFINITY)
                        sum += q.sum * exp((double)q.top - (double)top);
                }
#pragma unroll
                for (int m = 32; m; m >>= 1)
                    sum += __shfl_xor(sum, m);
                value = (double)base - log(sum);
            }
        }
        if (lane == 0) {
            add[b] = value;
            beam_top[b] = top;
        }
    }
    if (tid < 64) {
        rank[tid] = 0;
        score_out[tid] = -INFINITY;
        token_out[tid] = parent_out[tid] = -1;
    }
    if (tid < SBVR_BEAMS_MAX) {
        ended[tid] = -INFINITY;
        ended_token[tid] = -1;
    }
    if (tid == 0) {
        least = {-INFINITY, 0};
        count = 0;
    }
    __syncthreads();

    Candidate mine = {-INFINITY, BEAM_ENTRIES};  // the thread's best that goes on
    double score[PER];
    uint32_t what[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int place = i * THREADS + tid;
        const uint64_t key = place < all ? entries[place] : 0;
        const int beam = place < all ? place / per_beam : 0;
        score[i] = -INFINITY;
        what[i] = (uint32_t)beam << 16 | place;
        if (key && add[beam] > -INFINITY) {
            score[i] = add[beam] + ((double)unordered((uint32_t)(key >> 32)) - (double)beam_top[beam]);
            const int token = (int)~(uint32_t)key;
            bool end = false;
            for (int e = 0; e < a.n_end; ++e)
                end |= uniform_load(a.end_tokens + e) == token;
            const Candidate c = {score[i], place};
            if (end)
                what[i] |= END;
            else if (better_than(c, mine))
                mine = c;
        }
    }
#pragma unroll
    for (int m = 1; m < WAVES; m <<= 1) {
        const Candidate other = {__shfl_xor(mine.score, m), __shfl_xor(mine.place, m)};
        if (better_than(other, mine))
            mine = other;
    }
    if (tid % WAVES == 0)
        group[tid / WAVES] = mine;
    __syncthreads();
    {
        const Candidate g = group[lane];
        int better = 0;
#pragma unroll
        for (int j = 0; j < 64 / WAVES; ++j)
            better += better_than(group[(tid >> 6) * (64 / WAVES) + j], g);
        if (better)
            atomicAdd(&rank[lane], better);
    }
    __syncthreads();
    // what is worse than the n-th best group has n better ones that go on
    if (tid < 64 && group[tid].score > -INFINITY && rank[tid] == a.n - 1)
        least = group[tid];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (score[i] > -INFINITY && !better_than(least, Candidate{score[i], (int)(what[i] & 0xffff)})) {
            const int k = atomicAdd(&count, 1);
            list_score[k] = score[i];
            list_what[k] = what[i];
        }
    __syncthreads();
    const int c = count;
    for (int i = tid; i < c; i += THREADS) {
        const uint32_t w = list_what[i];
        const Candidate me = {list_score[i], (int)(w & 0xffff)};
        const int beam = (w >> 16) & 0x7fff;
        int better = 0, going = 0, same = 0;  // all, those that go on, and ends of the beam
        for (int j = 0; j < c; ++j) {
            const uint32_t u = list_what[j];
            const bool b = better_than(Candidate{list_score[j], (int)(u & 0xffff)}, me);
            better += b;
            going += b && !(u & END);
            same += b && (u & END) && ((u >> 16) & 0x7fff) == beam;
        }
        const int token = (int)~(uint32_t)entries[me.place];
        if (!(w & END)) {
            if (going < a.n) {
                token_out[going] = token;
                parent_out[going] = beam;
                score_out[going] = (float)me.score;
            }
        } else if (better < a.n && same == 0) {
            ended[beam] = (float)me.score;
            ended_token[beam] = token;
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

// pieces of a thread: large tiles where their workgroups fill the chip, and their
// lists fit
int beam_pieces(long long rows, int V, int keep)
{
    return keep <= 32 && rows * ((V + 8191ll) / 8192) >= 512 ? 4 : 1;
}

BeamShape beam_shape(int R, int B, int V, int n, int n_end)
{
    BeamShape s;
    const int tile = 8 * BEAM_THREADS * beam_pieces((long long)R * B, V, n + n_end);
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
    // the entries kept, and all logits of as many groups of four lanes (at most a tile's)
    const size_t held = (size_t)s.keep * 4 * 8 * CH, list = s.keep + held;
    return launch_kernel((const void *)beam_part_kernel<T, CH>, dim3((unsigned)(a.R * a.B * s.parts)), dim3(BEAM_THREADS),
                         list * sizeof(uint64_t), stream, argv);
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
    const bool large = beam_pieces((long long)a.R * a.B, a.V, s.keep) == 4;
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
    const size_t lds = (size_t)all * (sizeof(double) + sizeof(uint32_t));
    return all <= 1024 ? launch_kernel((const void *)beam_join_kernel<256>, dim3(a.R), dim3(256), lds, stream, argv)
                       : launch_kernel((const void *)beam_join_kernel<1024>, dim3(a.R), dim3(1024), lds, stream, argv);
}

}  // namespace sbvr
