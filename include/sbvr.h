/*
 * sbvr.h -- C ABI of the MI355X (gfx950) SBVR GEMV library.
 *
 * SBVR (Summation of BitVector Representation; Bang et al., Sec. 4.1) stores
 * each group of 128 consecutive weights along the inner-product dimension as
 * k bitvectors ("planes") plus k coefficients, so that every decoded weight is
 * a subset sum of its group's coefficients:
 *
 *     w_hat[o][128 g + j] = sum_{i<k} c[o][g][i] * b[o][g][i][j]      (Sec. 4.1)
 *
 * and the GEMV is computed directly on that representation (Sec. 4.4):
 *
 *     y[o] = sum_g sum_i c[o][g][i] * (sum_{j : b[o][g][i][j] = 1} x[128 g + j])
 *
 * Activations x and outputs y are IEEE binary16; accumulation is binary32;
 * y is rounded to binary16 to nearest-even.
 *
 * CANONICAL FORMAT (host-independent, what an encoder writes):
 *   planes  uint32_t [O][G][k][4], G = I / 128.  Bit t (LSB = 0) of word w is
 *           element j = 32 w + t of the group.  Plane i pairs with coefficient
 *           i.  (The paper stores bitvectors "partitioned into 32-bit
 *           integers" in one contiguous tensor, Sec. 4.4.)
 *   coeffs  uint16_t [O][G][k], binary16 bit patterns of c[o][g][i].  The
 *           per-(row, group, plane) coefficient tensor holds the values the
 *           paper's coefficient cache + index (Sec. 4.4) decode to; that
 *           format itself has its own entry points below.
 *
 * DEVICE FORMAT: an opaque, padded repacking of the canonical tensors that
 * the GEMV kernels stream with 128-bit coalesced loads.  It is produced by
 * sbvr_pack and inverted bit-exactly by sbvr_unpack; its size comes from the
 * two size queries.  Its layout is private to the library and may change.
 *
 * CONVENTIONS for every entry point:
 *   - O (out_features) >= 1; I (in_features) >= 128 and a multiple of 128;
 *     1 <= k <= 4 planes; 1 <= B <= 8 activation vectors.
 *   - Pointers named *_dev, x, y, X, Y, planes_canon and coeffs_canon are
 *     device pointers (HIP global memory) owned by the caller.  The library
 *     never allocates, frees or synchronises; work is enqueued on `stream`
 *     (0 = the null stream) and completes asynchronously.  Every call is
 *     safe to capture in a HIP graph.
 *   - Alignment: planes_dev, coeffs_dev, planes_canon, x and X 16 bytes;
 *     coeffs_canon, y and Y 2 bytes.
 *   - On any error nothing is enqueued and no output is written.  No call
 *     aborts, throws or prints.
 *   - Inputs are assumed finite.  Calls on one stream are ordered; calls that
 *     run concurrently on different streams must not share an output buffer.
 */
#ifndef SBVR_H
#define SBVR_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Status codes.  Every entry point returns one of these. */
enum sbvr_status {
    SBVR_OK = 0,
    SBVR_E_INVALID_ARG = -1, /* null pointer, bad shape, B out of range */
    SBVR_E_UNSUPPORTED = -2, /* valid SBVR parameters this build does not run (k > 4) */
    SBVR_E_WORKSPACE = -3,   /* workspace smaller than sbvr_workspace_bytes */
    SBVR_E_ALIGNMENT = -4,   /* a pointer violates the alignment above */
    SBVR_E_HIP = -5          /* the HIP runtime reported a launch error */
};

/* Human-readable name of a status code; never NULL, static storage. */
const char *sbvr_status_string(int status);

/* Library ABI version (major * 100 + minor); 1.01 adds sbvr_decompress,
 * 1.02 sbvr_gemv_a8, 1.03 the coefficient-cache format entry points,
 * 1.04 sbvr_encode and sbvr_decompress_indexed, 1.05 sbvr_gemm_prefill,
 * 1.06 sbvr_gemv_grouped and sbvr_gemv_grouped_a8, 1.07 sbvr_encode_cached,
 * 1.08 the operators between the products of a step: sbvr_batch_plan,
 * sbvr_cache_write, sbvr_tree_attention, sbvr_residual_norm,
 * sbvr_adjust_logits, 1.09 sbvr_tree_attention_whole. */
int sbvr_version(void);

/*
 * Size queries (pure host functions, no HIP calls).  Bytes the caller must
 * provide for the device planes / device coefficients of an O x I matrix
 * with k planes (the k bitvectors and k coefficients per 128-weight group of
 * Sec. 4.1, stored as in Sec. 4.4, plus the device layout's zero padding of
 * the last row tile and the last 512-element block); 0 if the arguments are
 * invalid.
 */
size_t sbvr_packed_plane_bytes(int O, int I, int k);
size_t sbvr_packed_coeff_bytes(int O, int I, int k);

/*
 * Workspace a GEMV call needs, in bytes (0 means none: pass workspace = NULL
 * and ws_bytes = 0).  The inner-product sum of Sec. 4.4 is split over the
 * wavefronts of one workgroup and reduced there, so the current kernels need
 * no global workspace.
 */
size_t sbvr_workspace_bytes(int O, int I, int k, int B);

/*
 * Repack canonical SBVR tensors into the device format (the storage of
 * Sec. 4.4, laid out for the GEMV kernels).
 *   planes_canon  uint32 [O][G][k][4], coeffs_canon uint16 [O][G][k]: input.
 *   planes_dev    >= sbvr_packed_plane_bytes(O, I, k) bytes: output.
 *   coeffs_dev    >= sbvr_packed_coeff_bytes(O, I, k) bytes: output.
 * Every byte of both outputs is written (padding with zeros).  Inputs and
 * outputs must not overlap.
 */
int sbvr_pack(int O, int I, int k, const uint32_t *planes_canon, const uint16_t *coeffs_canon,
              void *planes_dev, void *coeffs_dev, hipStream_t stream);

/*
 * Inverse of sbvr_pack: recover the canonical tensors (the bitvectors and
 * coefficients of Sec. 4.1 in the storage order of Sec. 4.4), bit for bit,
 * from the device format.  Same shapes and ownership as sbvr_pack with the
 * roles of input and output exchanged.
 */
int sbvr_unpack(int O, int I, int k, const void *planes_dev, const void *coeffs_dev,
                uint32_t *planes_canon, uint16_t *coeffs_canon, hipStream_t stream);

/*
 * Batch-1 SBVR GEMV (Sec. 4.4 with binary16 activations):
 *     y[o] = fp16_rne( sum_g sum_i c[o][g][i] * sum_j b[o][g][i][j] x[128 g + j] )
 *   planes_dev, coeffs_dev  device-format weights from sbvr_pack.
 *   x  binary16 [I] (input);  y  binary16 [O] (output, every element written).
 *   workspace / ws_bytes    see sbvr_workspace_bytes (may be NULL / 0).
 * x must not overlap y.
 */
int sbvr_gemv(int O, int I, int k, const void *planes_dev, const void *coeffs_dev,
              const uint16_t *x, uint16_t *y, void *workspace, size_t ws_bytes,
              hipStream_t stream);

/*
 * Small-batch SBVR GEMM: the GEMV of Sec. 4.4 applied to each of the B
 * activation vectors X[b][0..I) (the paper's kernel handles one token per
 * decode step; a batch of B tokens multiplies the same SBVR weights B times),
 *     Y[b][o] = fp16_rne( sum_g sum_i c[o][g][i] * sum_j b[o][g][i][j] X[b][128 g + j] ),
 * with the weights read from memory once for all B.
 *   X  binary16 [B][I] row-major (input);  Y  binary16 [B][O] row-major
 *   (output, every element written).  1 <= B <= 8.  workspace / ws_bytes as
 *   sbvr_gemv.  X must not overlap Y.
 */
int sbvr_gemm_small_batch(int O, int I, int k, const void *planes_dev, const void *coeffs_dev,
                          const uint16_t *X, uint16_t *Y, int B, void *workspace,
                          size_t ws_bytes, hipStream_t stream);

/*
 * The W4A8 decode GEMV (Sec. 4.3 and 4.4 with 8-bit SBVR activations): x is
 * converted online, per 128-element group g, to an 8-bit code with Eq. 12's
 * two's-complement coefficients {-128 s_g, s_g, 2 s_g, ..., 64 s_g}:
 *     s_g = max_j abs(x[128 g + j]) / 127,  q_j = rne(x_j / s_g) in [-127, 127]
 * (binary32, correctly rounded division; a zero group has s_g = 0, q = 0),
 * and
 *     y[o] = fp16_rne( sum_g s_g sum_i c[o][g][i] * sum_j b[o][g][i][j] q_j ).
 * Arguments as sbvr_gemv (x binary16 [I], y binary16 [O]).
 */
int sbvr_gemv_a8(int O, int I, int k, const void *planes_dev, const void *coeffs_dev,
                 const uint16_t *x, uint16_t *y, void *workspace, size_t ws_bytes,
                 hipStream_t stream);

/* Most GEMVs one sbvr_gemv_grouped call takes. */
#define SBVR_GEMV_GROUP_MAX 4

/*
 * Grouped batch-1 GEMV: n independent GEMVs of Sec. 4.4 (each exactly the
 * sbvr_gemv of its arguments, bit for bit) enqueued as ONE kernel launch, for
 * the projections of a decode step that run back to back -- e.g. q, k and v,
 * or gate and up, each with its own packed weights -- so that a captured
 * decode step (the paper runs it under a CUDA graph, Sec. 5.2) pays one
 * launch instead of n.
 *   n                 1 <= n <= SBVR_GEMV_GROUP_MAX.
 *   O                 host array [n]: out_features of member i.
 *   I, k              shared by every member.
 *   planes_dev, coeffs_dev, x, y
 *                     host arrays [n] of device pointers, member i's
 *                     device-format weights (sbvr_pack of O[i] x I, k),
 *                     binary16 x[i] [I] (input) and y[i] [O[i]] (output,
 *                     every element written).  Same alignment as sbvr_gemv.
 *   workspace / ws_bytes  as sbvr_gemv (may be NULL / 0).
 * The host arrays are read during the call only.  Members may share an x;
 * no y may overlap another member's y or any x.  Every member is validated
 * as sbvr_gemv would validate it before anything is enqueued; the first
 * failing member's status is returned.
 */
int sbvr_gemv_grouped(int n, const int *O, int I, int k, const void *const *planes_dev,
                      const void *const *coeffs_dev, const uint16_t *const *x, uint16_t *const *y,
                      void *workspace, size_t ws_bytes, hipStream_t stream);

/*
 * The same grouping for the W4A8 decode GEMV: n independent sbvr_gemv_a8
 * calls (Sec. 4.3 and 4.4 with 8-bit SBVR activations, each member bit for
 * bit its own sbvr_gemv_a8) as one kernel launch.  Arguments, ownership and
 * errors as sbvr_gemv_grouped.
 */
int sbvr_gemv_grouped_a8(int n, const int *O, int I, int k, const void *const *planes_dev,
                         const void *const *coeffs_dev, const uint16_t *const *x, uint16_t *const *y,
                         void *workspace, size_t ws_bytes, hipStream_t stream);

/*
 * Prefill GEMM on SBVR weights (the prefill design of Sec. 5.1: the weights
 * are decompressed to binary16 and multiplied on the matrix cores), for a
 * prompt of T tokens, without writing the decompressed matrix to memory:
 *     Y[t][o] = fp16_rne( sum_j X[t][j] * fp16_rne(w_hat[o][j]) ),
 * where fp16_rne(w_hat[o][j]) is the correctly rounded subset sum of
 * Sec. 4.1 (the value sbvr_decompress writes); binary32 accumulation.
 *   planes_dev, coeffs_dev  device-format weights from sbvr_pack.
 *   X  binary16 [T][I] row-major (input, 16-byte aligned);
 *   Y  binary16 [T][O] row-major (output, every element written).
 *   1 <= T <= 2^22 (larger: SBVR_E_UNSUPPORTED).  X must not overlap Y.
 *   The summation order is fixed for given (O, I, k, T), so repeated calls
 *   give identical bits; it follows the launch shape, which depends on T.
 */
int sbvr_gemm_prefill(int O, int I, int k, const void *planes_dev, const void *coeffs_dev, const uint16_t *X,
                      uint16_t *Y, int T, hipStream_t stream);

/*
 * COEFFICIENT-CACHE FORMAT (Sec. 4.4): the coefficients are stored once per
 * distinct coefficient set in a cache, and each (row, group) names the set
 * its k bitvectors use:
 *   planes  uint32_t [O][G][k][4] as in the canonical format;
 *   index   uint16_t [O][G]: coefficient-set index of (row o, group g);
 *   table   uint16_t [n_sets][k]: binary16 coefficient sets, 1 <= n_sets <= 65536;
 *     c[o][g][i] = table[index[o][g]][i].
 * Per weight this stores 2 bytes per group instead of 2k (k = 4: 4.125
 * instead of 4.5 bits per weight) plus the table.  An index >= n_sets is a
 * caller error; the GEMV then reads zero coefficients for that group (the
 * table is read through a bounds-checked path), nothing faults.
 */

/* Device bytes of the index blocks of an O x I matrix with k planes, and of
 * a table of n_sets coefficient sets (8 bytes per set); 0 if invalid. */
size_t sbvr_packed_index_bytes(int O, int I, int k);
size_t sbvr_packed_table_bytes(int n_sets, int k);

/*
 * Repack the coefficient-cache format into its device format.
 *   planes_canon uint32 [O][G][k][4], index_canon uint16 [O][G],
 *   table_canon uint16 [n_sets][k]: inputs (device memory; planes_canon
 *   16-byte aligned, the others 2).
 *   planes_dev (sbvr_packed_plane_bytes), index_dev
 *   (sbvr_packed_index_bytes), table_dev (sbvr_packed_table_bytes): outputs,
 *   16-byte aligned, every byte written.  Inputs and outputs must not overlap.
 */
int sbvr_pack_indexed(int O, int I, int k, int n_sets, const uint32_t *planes_canon,
                      const uint16_t *index_canon, const uint16_t *table_canon, void *planes_dev,
                      void *index_dev, void *table_dev, hipStream_t stream);

/* Inverse of sbvr_pack_indexed, bit for bit (roles of inputs and outputs
 * exchanged). */
int sbvr_unpack_indexed(int O, int I, int k, int n_sets, const void *planes_dev, const void *index_dev,
                        const void *table_dev, uint32_t *planes_canon, uint16_t *index_canon,
                        uint16_t *table_canon, hipStream_t stream);

/*
 * Batch-1 GEMV on the coefficient-cache format (Sec. 4.4):
 *     y[o] = fp16_rne( sum_g sum_i table[index[o][g]][i] * sum_j b[o][g][i][j] x[128 g + j] )
 * i.e. sbvr_gemv with the gathered coefficients.  planes_dev, index_dev,
 * table_dev from sbvr_pack_indexed; x, y, workspace as sbvr_gemv.
 */
int sbvr_gemv_indexed(int O, int I, int k, int n_sets, const void *planes_dev, const void *index_dev,
                      const void *table_dev, const uint16_t *x, uint16_t *y, void *workspace,
                      size_t ws_bytes, hipStream_t stream);

/*
 * The same with SBVR-8 activations (the conversion of sbvr_gemv_a8): the
 * paper's decode configuration, W4A8 with a coefficient cache (Sec. 4.3-4.4).
 */
int sbvr_gemv_indexed_a8(int O, int I, int k, int n_sets, const void *planes_dev, const void *index_dev,
                         const void *table_dev, const uint16_t *x, uint16_t *y, void *workspace,
                         size_t ws_bytes, hipStream_t stream);

/*
 * Decompression for the prefill path: the decoded matrix as binary16,
 *     W[o][128 g + j] = fp16_rne( sum_i c[o][g][i] * b[o][g][i][j] )
 * (the subset-sum decoding of Sec. 4.1, computed exactly and rounded once),
 * for a dense matrix-core GEMM over many tokens.
 *   planes_dev, coeffs_dev  device-format weights from sbvr_pack.
 *   W  binary16 [O][I] row-major (output, every element written), 16-byte
 *      aligned; must not overlap the inputs.
 */
int sbvr_decompress(int O, int I, int k, const void *planes_dev, const void *coeffs_dev, uint16_t *W,
                    hipStream_t stream);

/*
 * Prefill decompression of the coefficient-cache format: as sbvr_decompress
 * with c[o][g][i] = table[index[o][g]][i] (zero for an index >= n_sets).
 * planes_dev, index_dev, table_dev from sbvr_pack_indexed; W as for
 * sbvr_decompress.
 */
int sbvr_decompress_indexed(int O, int I, int k, int n_sets, const void *planes_dev, const void *index_dev,
                            const void *table_dev, uint16_t *W, hipStream_t stream);

#define SBVR_ENCODE_MAX_ENTRIES 65536

/*
 * SBVR encoding on the GPU (Algorithm 1 and the bitvector assignment of
 * Sec. 4.2): every 128-weight group of W takes, from the (r, s, b) grid of
 * Eqs. 4-11 with |R1| = n_ratio1, |R2| = n_ratio2, N_scale = n_scale and
 * N_bias = n_bias entries, the binary16 coefficient set with the smallest
 * mean squared error of nearest-subset-sum reconstruction (first such entry
 * in (r, s, b) order), and each weight the bit pattern of its nearest subset
 * sum (lowest pattern index on ties).  normalise = 1 divides the geometric
 * series of Eq. 4 by sum_i abs(r)^i (the span-normalised reading), 0 takes
 * Eq. 4 literally.  Groups with no admissible entry (s <= 0 or a non-finite
 * coefficient everywhere) get (fp16(mean), 0, ...).  All arithmetic is
 * binary64 in a fixed order, so the output is deterministic and reproducible
 * bit for bit by a CPU implementation of the same definition.
 *   W             float32 [O][I] row-major, device, 4-byte aligned; finite.
 *   planes_canon  uint32 [O][G][k][4] canonical planes (output, 16-byte aligned).
 *   coeffs_canon  uint16 [O][G][k] binary16 coefficients (output).
 *   mse           binary64 [O][G] (output, 8-byte aligned) or NULL.
 * At most SBVR_ENCODE_MAX_ENTRIES grid entries ((n_ratio1 + n_ratio2) *
 * n_scale * n_bias); more is SBVR_E_UNSUPPORTED.
 */
int sbvr_encode(int O, int I, int k, const float *W, int n_ratio1, int n_ratio2, int n_scale, int n_bias,
                int normalise, uint32_t *planes_canon, uint16_t *coeffs_canon, double *mse,
                hipStream_t stream);

#define SBVR_ENCODE_CACHE_MAX 64

/*
 * The encoder with the cache of Sec. 4.2 (last paragraph and its footnote):
 * before the full search, a group tries the coefficient sets that the search
 * chose for earlier groups, and keeps one if its error is below the moving
 * average of the quantization error; groups that hit share their set with an
 * earlier group, which also shrinks the coefficient cache of the indexed
 * format (sbvr_pack_indexed).  Each row of W is encoded on its own, its
 * groups in index order:
 *   - the cache holds the coefficient sets the full search chose for the
 *     row's last cache_slots searched groups (the oldest is replaced first;
 *     the (fp16(mean), 0, ...) fallback is not cached);
 *   - every held set is scored on the group with the search's MSE; the
 *     smallest (the oldest set among equal ones) is taken, with each weight's
 *     nearest-subset-sum pattern, if it is strictly below the mean MSE of
 *     the row's earlier groups (binary64 sum in group order over their count);
 *   - otherwise the group runs the search of sbvr_encode, and its set enters
 *     the cache.
 * The first group of a row always searches; cache_slots = 0 gives exactly
 * sbvr_encode's output.  Arguments as sbvr_encode, plus
 *   cache_slots  0 .. SBVR_ENCODE_CACHE_MAX (else SBVR_E_INVALID_ARG).
 *   hits         uint8 [O][G] (output): 1 where the group took a cached set,
 *                0 where it searched; or NULL.
 * Rows are independent (one wavefront each), a row's groups sequential.
 */
int sbvr_encode_cached(int O, int I, int k, const float *W, int n_ratio1, int n_ratio2, int n_scale, int n_bias,
                       int normalise, int cache_slots, uint32_t *planes_canon, uint16_t *coeffs_canon,
                       double *mse, uint8_t *hits, hipStream_t stream);

/*
 * OPERATORS BETWEEN THE PRODUCTS OF A STEP.  A step takes R requests; request
 * r has context_lens[r] tokens in a paged key/value cache and brings
 * new_lens[r] more: one (plain decoding), a tree of drafted tokens to verify,
 * or a prompt chunk.  The step's tokens are numbered request by request;
 * token t of request r is its j-th new token, j = t - query_start[r], and its
 * key and value have position context_lens[r] + j of the request.
 *
 * Pages: position p of request r lies in page page_table[r][p / page_size] at
 * offset p % page_size; its slot number is page * page_size + offset.
 *   page_size  a power of two, 16 .. SBVR_PAGE_MAX.
 *
 * Trees: a tree has at most SBVR_TREE_MAX tokens; parents[t] is the index j
 * of token t's parent within its request (smaller than its own; anything else
 * makes it a root), and tree_mask[t] has bit j set where token t sees the
 * request's j-th new token.
 *
 * The conventions above hold for these entry points too, with these alignments:
 * keys, values, queries, attention outputs and the cache 16 bytes, int64 /
 * uint64 arrays 8, int32 / uint32 / binary32 arrays 4, 16-bit arrays 2.
 * Zero tokens is a valid step: nothing is enqueued and no pointer is read.
 */
enum sbvr_dtype {
    SBVR_F16 = 0,  /* IEEE binary16 */
    SBVR_BF16 = 1, /* bfloat16 */
    SBVR_F32 = 2   /* IEEE binary32 */
};

#define SBVR_REQUESTS_MAX 4096
#define SBVR_TREE_MAX 64
#define SBVR_PAGE_MAX 4096

/*
 * The plan of a step: pages for the new tokens, and what the other operators
 * need per token.
 *   R, T          1 <= R <= SBVR_REQUESTS_MAX requests; room for T >= 0 tokens
 *                 in the outputs per token.
 *   context_lens, new_lens   int32 [R] (a negative length counts as 0).
 *   free_pages    int32 [n_free]: unused pages, taken in order.
 *   parents       int32 [T] (above), or NULL: each token's parent is the one
 *                 before it.  Requests of more than SBVR_TREE_MAX new tokens are
 *                 such chains in any case, and have tree_mask 0.
 *   page_table    int32 [R][table_stride], max_pages used (in and out).  The
 *                 ceil(context_lens[r] / page_size) entries of the cached tokens
 *                 are read; the entries of the pages that the new tokens need
 *                 beyond them are written: request by request, then by position,
 *                 from free_pages in order, -1 once that is used up.  A request
 *                 takes no pages beyond max_pages.  No other entry is touched.
 *   query_start   int32 [R + 1] (output): tokens before request r, at most T;
 *                 the last one is the number of tokens.
 *   token_request int32 [T] (output): the token's request; -1 past the last token.
 *   positions     int32 [T] (output): context_lens[r] + the number of the
 *                 token's proper ancestors; 0 past the last token.
 *   slots         int64 [T] (output): the token's slot; -1 where it has no page
 *                 and past the last token.
 *   tree_mask     uint64 [T] (output): the token's ancestors, itself included;
 *                 0 past the last token.
 *   used          int32 [2] (output): pages taken (more than n_free: the free
 *                 pages did not suffice), and new tokens (more than T: the last
 *                 ones were left out).
 * Inputs and outputs must not overlap.
 */
int sbvr_batch_plan(int R, int T, int page_size, const int32_t *context_lens, const int32_t *new_lens,
                    const int32_t *free_pages, int n_free, const int32_t *parents, int32_t *page_table,
                    int max_pages, int64_t table_stride, int32_t *query_start, int32_t *token_request,
                    int32_t *positions, int64_t *slots, uint64_t *tree_mask, int32_t *used, hipStream_t stream);

/*
 * A paged key/value cache: element (page, offset, head, d) of the keys is at
 * k + page * k_page_stride + offset * k_token_stride + head * k_head_stride + d
 * (strides in elements, multiples of 8, not negative), values likewise.
 *   dtype     SBVR_F16 or SBVR_BF16.
 *   head_dim  a multiple of 8, 8 .. 128 (larger: SBVR_E_UNSUPPORTED).
 * Token strides are at most 2^30 / page_size (else SBVR_E_UNSUPPORTED).
 * The struct is read during the call only.
 */
typedef struct sbvr_kv_cache {
    void *k, *v;
    int64_t k_page_stride, k_token_stride, k_head_stride;
    int64_t v_page_stride, v_token_stride, v_head_stride;
    int32_t n_pages, page_size, kv_heads, head_dim, dtype;
} sbvr_kv_cache;

/*
 * Write a step's keys and values into the cache: token t's at slots[t]; a
 * token whose slot is negative or past the cache is skipped.  Two tokens must
 * not share a slot.
 *   k, v   [T][kv_heads][head_dim] of the cache's dtype, with the given token
 *          and head strides (elements, multiples of 8, not negative).
 *   slots  int64 [T].
 */
int sbvr_cache_write(const sbvr_kv_cache *cache, int T, const void *k, int64_t k_token_stride,
                     int64_t k_head_stride, const void *v, int64_t v_token_stride, int64_t v_head_stride,
                     const int64_t *slots, hipStream_t stream);

/*
 * Attention of a step's tokens over the cache, which already holds their own
 * keys and values (sbvr_cache_write).  Token t of request r sees all
 * context_lens[r] cached tokens, and of its request's new tokens those whose
 * bit is set in tree_mask[t]; head h reads key/value head
 * h / (heads / kv_heads).
 *     out[t][h] = sum_p w_p v_p / sum_p w_p,  w_p = exp(scale q[t][h] . k_p - max)
 * over the positions p that t sees; a token that sees none gets 0.  Scores,
 * exponentials' sums and products are accumulated in binary32; the weights
 * are rounded to the cache's type for the product with the values (in binary16
 * by 2^-32 of a row's largest weight where they are small); the output is
 * rounded once.  What lies in a slot that a token does not see has no
 * effect on it, NaN and infinities included.
 *   q            [T][heads][head_dim] of the cache's dtype, with strides as
 *                sbvr_cache_write's inputs; heads a multiple of kv_heads.
 *   page_table   int32 [R][table_stride], max_pages used.  A request is cut to
 *                max_pages * page_size tokens; the positions of a page outside
 *                0 .. n_pages - 1 are not seen.
 *   context_lens int32 [R]; query_start int32 [R + 1] ascending, at most T;
 *   tree_mask    uint64 [T].  1 <= R <= SBVR_REQUESTS_MAX.
 *   max_new      1 .. SBVR_TREE_MAX: no request brings more new tokens than
 *                this (the rest of a longer one is left out).
 *                With B = max_new * heads / kv_heads / 128 rounded up,
 *                R * kv_heads * B * (max_pages * page_size / 64 + 5) of 2^31 or
 *                more: SBVR_E_UNSUPPORTED.
 *   out          [T][heads][head_dim] contiguous; rows past query_start[R] are
 *                left as they are.  Must not overlap the inputs.
 *   workspace    sbvr_tree_attention_workspace_bytes, 16-byte aligned; its
 *                content needs no preparation and is not kept.
 */
size_t sbvr_tree_attention_workspace_bytes(int R, int max_new, int heads, int kv_heads, int head_dim);
int sbvr_tree_attention(const sbvr_kv_cache *cache, int R, int T, int heads, const void *q, int64_t q_token_stride,
                        int64_t q_head_stride, const int32_t *page_table, int max_pages, int64_t table_stride,
                        const int32_t *context_lens, const int32_t *query_start, const uint64_t *tree_mask,
                        int max_new, float scale, void *out, void *workspace, size_t ws_bytes, hipStream_t stream);

/*
 * The same, with every row of out written.  A request that sbvr_tree_attention
 * would cut, because it brings more new tokens than max_new or has more tokens
 * than max_pages * page_size, is not computed in part: all its rows are NaN.
 * (A prompt chunk of more than SBVR_TREE_MAX tokens, for which sbvr_batch_plan
 * has no masks, is such a request: it goes in several steps.)  Rows of no request,
 * past query_start[R] or before query_start[0], are 0.
 */
int sbvr_tree_attention_whole(const sbvr_kv_cache *cache, int R, int T, int heads, const void *q,
                              int64_t q_token_stride, int64_t q_head_stride, const int32_t *page_table, int max_pages,
                              int64_t table_stride, const int32_t *context_lens, const int32_t *query_start,
                              const uint64_t *tree_mask, int max_new, float scale, void *out, void *workspace,
                              size_t ws_bytes, hipStream_t stream);

#define SBVR_NORM_MAX_WIDTH 32768

/*
 * The norms around a block, with its gate and residual scale, in one pass:
 *     z = y * rsqrt(mean(y^2) + eps) * post_weight     (post_weight NULL: z = y)
 *     x' = x + scale * gate * z                        (gate NULL: 1; y NULL: x' = x)
 *     h = x' * rsqrt(mean(x'^2) + eps) * pre_weight
 * per token, in binary32, each output rounded once (h from the unrounded x').
 *   T, H     T >= 0 tokens of 1 <= H <= SBVR_NORM_MAX_WIDTH elements (more:
 *            SBVR_E_UNSUPPORTED).
 *   dtype    of y, gate, the weights and h: SBVR_F16 or SBVR_BF16.
 *   x_dtype  of x and x_out (the residual stream): dtype or SBVR_F32.
 *   x, y, gate, x_out, h_out   [T][H] with the given row strides in elements;
 *            gate_stride 0 is one gate for all tokens, [H]; output rows must not
 *            overlap.
 *   x_out    may be x itself (same stride), or NULL: not wanted.
 *   h_out    NULL: not wanted (and pre_weight is not read; else it must be given).
 * Apart from x_out = x, inputs and outputs must not overlap.
 */
int sbvr_residual_norm(int T, int H, int dtype, int x_dtype, const void *x, int64_t x_stride, const void *y,
                       int64_t y_stride, const void *post_weight, const void *gate, int64_t gate_stride, float scale,
                       const void *pre_weight, float eps, void *x_out, int64_t x_out_stride, void *h_out,
                       int64_t h_stride, hipStream_t stream);

/*
 * Adjustment of logits before sampling.  Row t belongs to request r =
 * token_request[t] (NULL: r = t); for token v of the vocabulary, with c the
 * number of times v occurs among the request's generated tokens and on t's
 * drafted path, and "seen" where c > 0 or v occurs in the request's prompt:
 *     l = logits[t][v]
 *     seen:   l = l > 0 ? l / repetition[r] : l * repetition[r]
 *     l = l - frequency[r] * c - presence[r] * (c > 0)
 *     l = l + bias(r, v)
 *     l = l / temperature[r]            (temperature <= 0: unchanged)
 *     grammar bit v of the row is 0:  l = -infinity
 * in binary32, rounded once to the output type.
 *   logits  [T][V] of dtype, row stride logits_stride elements; out [T][V] of
 *           out_dtype (dtype or SBVR_F32), row stride out_stride; out may be
 *           logits itself where the types and strides agree.  Rows whose request
 *           is outside 0 .. R - 1 are converted, not adjusted.
 *   history int32, request r's tokens at history_start[r] .. history_start[r + 1]
 *           (int32 [R + 1], ascending), the first prompt_lens[r] (int32 [R], NULL:
 *           0) of them its prompt, the others generated; NULL: none.
 *   repetition, frequency, presence, temperature  binary32 [R], or NULL: 1, 0, 0, 1.
 *   bias_tokens, bias_values  int32 and binary32, request r's at bias_start[r] ..
 *           bias_start[r + 1] (int32 [R + 1]); of several entries for a token the
 *           last one counts; NULL: none.
 *   grammar uint32 [grammar_count][grammar_stride]: bit v % 32 of word v / 32 is 1
 *           where v is allowed; grammar_rows int32 [T] names each row's mask
 *           (outside 0 .. grammar_count - 1: unconstrained; NULL: row t has mask t);
 *           grammar NULL: none.
 *   draft_tokens int32 [T], tree_mask uint64 [T], query_start int32 [R + 1]: token
 *           t's drafted path is the tokens of its tree_mask, numbered within the
 *           request from query_start[r]; all three or none (NULL).
 * Token ids outside 0 .. V - 1 are ignored.  At most 65535 rows and 2^30 tokens
 * in the vocabulary (more: SBVR_E_UNSUPPORTED).  The struct is read during the call.
 */
typedef struct sbvr_logits_args {
    int32_t R, T, V, dtype, out_dtype;
    const void *logits;
    int64_t logits_stride;
    void *out;
    int64_t out_stride;
    const int32_t *token_request;
    const int32_t *history, *history_start, *prompt_lens;
    const float *repetition, *frequency, *presence, *temperature;
    const int32_t *bias_tokens, *bias_start;
    const float *bias_values;
    const uint32_t *grammar;
    int64_t grammar_stride;
    const int32_t *grammar_rows;
    int32_t grammar_count;
    const int32_t *draft_tokens, *query_start;
    const uint64_t *tree_mask;
} sbvr_logits_args;

int sbvr_adjust_logits(const sbvr_logits_args *args, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* SBVR_H */
