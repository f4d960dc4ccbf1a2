/*
 * lpq.h - low-precision (int8) brute-force k-nearest-neighbour search on one
 * AMD Instinct MI355X (gfx950).  C ABI of liblpq.so.
 *
 * The library implements the exhaustive-search hot path of "Low-Precision
 * Quantization for Efficient Nearest Neighbor Search": a feature-wise clamped linear
 * quantizer learned from the corpus (Section 3.2, Equation 1; Sections 4.1, 4.2)
 * maps items and queries into a low-precision integer domain, the distance function
 * is evaluated on the integers (phi : Z^d x Z^d -> Z, Section 3.1), and the k nearest
 * items of every query are returned (problem statement, Section 1).
 *
 * General conventions
 *   - "dev" pointers are DEVICE pointers of the current HIP device, owned by the
 *     caller (e.g. storage of a torch tensor); "host" pointers are host memory.
 *     Matrices are row-major; `ld` is the row stride in ELEMENTS (ld >= d).
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  Calls
 *     only enqueue work on it and do not synchronise unless stated otherwise.
 *   - Every function returning int returns LPQ_OK (0) or an error code below; on
 *     error no output buffer has been written by the failing call and
 *     lpq_last_error() describes the failure.  No C++ exception crosses the ABI.
 *   - The library owns only its opaque handle types.  A handle may be used from
 *     one thread at a time.
 *   - Item ids are 0-based row numbers in the order the items were added.
 */
#ifndef LPQ_H
#define LPQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct lpq_quantizer lpq_quantizer;
typedef struct lpq_index lpq_index;
typedef struct lpq_kv lpq_kv;

enum {
    LPQ_OK = 0,
    LPQ_EINVAL = 1,     /* null pointer, d < 1, bits outside 1..8, ld < d, k < 1, unknown enum */
    LPQ_ERANGE = 2,     /* k > n, n >= 2^31, d beyond the int32 bound, capacity or workspace too small */
    LPQ_ENOMEM = 3,     /* device or host allocation failed */
    LPQ_EDEVICE = 4,    /* a HIP call failed */
    LPQ_ENONFINITE = 5, /* calibration data held a NaN or an infinity */
    LPQ_ESTATE = 6      /* encode before calibrate/set_params, search on an empty index */
};

/* How the range [S_b, S_e] and the offset k of Equation 1 are learned.
 *   MINMAX  S_b = min, S_e = max, k = (min + max) / 2: the observed range (Section 1,
 *           the value range the data actually occupies).
 *   ABSMAX  S_b = -A, S_e = +A, k = 0 with A the absolute maximum observed in the
 *           dimension (Section 4.2).
 *   GAUSS   S_b = mu - c sigma, S_e = mu + c sigma, k = mu, with the maximum-likelihood
 *           (1/n) estimates of a normal law per dimension; the paper uses c = 1
 *           (Section 3.2).
 *   QUANTILE  the observed range with outliers discarded (Section 4.2 leaves the technique
 *           open; here a two-sided quantile clip): of the values of the dimension sorted
 *           ascending, S_b is the one of rank floor(p (n-1)) and S_e the one of rank
 *           ceil((1-p)(n-1)) (ranks from 0), k = (S_b + S_e) / 2; p = 0 is MINMAX.  Exact
 *           order statistics (radix selection), not estimates. */
enum { LPQ_CALIB_MINMAX = 0, LPQ_CALIB_ABSMAX = 1, LPQ_CALIB_GAUSS = 2, LPQ_CALIB_QUANTILE = 3 };

/* PER_FEATURE: constants per dimension (the superscripts i of Equation 1).
 * GLOBAL: one set of constants from all n*d values, for all dimensions (Section 4.1).
 * SHARED_WIDTH: an offset per dimension and one scale for all of them - a reading of the end of
 *   Section 3.2, which asks for extra per-dimension constants (scale as well as offset) when the
 *   dimensions differ much.  The PER_FEATURE constants are learned first; then every range keeps its centre
 *   (S_b + S_e) / 2 and takes the half-width of the widest range, H = max_i (S_e - S_b) / 2
 *   (binary64 on the binary32 constants): S_b = fl32(centre - H), S_e = fl32(centre + H),
 *   k unchanged.  One code step then has the same length in every dimension, so L2SQ on codes
 *   weighs all dimensions alike (PER_FEATURE turns it into a weighted distance) while offsets
 *   between dimensions cost no code range (as they do under GLOBAL). */
enum { LPQ_SCOPE_PER_FEATURE = 0, LPQ_SCOPE_GLOBAL = 1, LPQ_SCOPE_SHARED_WIDTH = 2 };

/* L2SQ: sum_i (a_i - b_i)^2 on codes, smaller = nearer.
 * IP:   sum_i a_i b_i on codes, LARGER = nearer (maximum inner product search, Section
 *       3.1).  Angular search = IP on vectors the caller normalised to unit length. */
enum { LPQ_METRIC_L2SQ = 0, LPQ_METRIC_IP = 1 };

/* ------------------------------------------------------------------ quantizer ---- */

/* New quantizer for d-dimensional vectors and bit-width B = bits (1..8); codes lie in
 * [-2^(B-1), 2^(B-1)] and are stored one per int8 (at B = 8 the value +128 of the upper
 * clamp is stored as 127).  *out is written on success only. */
int lpq_quantizer_create(lpq_quantizer **out, int d, int bits);
void lpq_quantizer_destroy(lpq_quantizer *q);

/* Learn the constants from n >= 1 vectors x_dev[n][ld] (fp32, device).  sigma_mult is c
 * above (GAUSS; must be > 0) or the clipped fraction p per side (QUANTILE; 0 <= p < 0.5).
 * Statistics are exact for MINMAX/ABSMAX/QUANTILE; GAUSS sums in
 * fp64 (two passes: mean, then centred second moment).  This call SYNCHRONISES `stream`
 * before returning, because its status depends on the data: LPQ_ENONFINITE if a NaN or
 * an infinity was seen (the quantizer then keeps its previous state). */
int lpq_quantizer_calibrate(lpq_quantizer *q, const float *x_dev, int64_t n, int64_t ld,
                            int mode, int scope, float sigma_mult, void *stream);

/* Set / read the constants directly (host arrays of d floats each; `m` may be NULL).
 * m_i = fl32(2^B / (S_e_i - S_b_i)) is derived in fp64; a feature with S_e <= S_b gets
 * m = 0 and encodes to 0 everywhere.  Both calls synchronise the device. */
int lpq_quantizer_set_params(lpq_quantizer *q, const float *k, const float *s_b, const float *s_e);
int lpq_quantizer_get_params(const lpq_quantizer *q, float *k, float *s_b, float *s_e, float *m);

/* Equation 1 on n vectors: codes_dev[j][i] for i < d (row stride ld_codes >= d bytes;
 * bytes i >= d of a row are not touched), and, if norms_dev is not NULL, norms_dev[j] =
 * sum_i code^2 (int32).  Per value, in IEEE binary32 without fused multiply-add:
 * NaN -> 0; x < S_b -> -2^(B-1); x > S_e -> +2^(B-1); otherwise floor((x - k) * m). */
int lpq_encode(const lpq_quantizer *q, const float *x_dev, int64_t n, int64_t ld,
               int8_t *codes_dev, int64_t ld_codes, int32_t *norms_dev, void *stream);

/* ---------------------------------------------------------------------- index ---- */

/* Flat index for up to `capacity` items (1 <= capacity < 2^31).  The index takes a copy
 * of the quantizer's constants (later changes to q do not affect it) and allocates, with
 * hipMalloc, the int8 codes (rows zero padded to 64, 96, 128, 192, 256, 384, 512, 768, 1024 or
 * 1536 bytes, beyond 1536 features to a multiple of 128 bytes) and the integer norms.
 * d <= 32 768 keeps every integer distance inside int32. */
int lpq_index_create(lpq_index **out, const lpq_quantizer *q, int64_t capacity);

/* The same index with two codes per byte, for quantizers of B <= 4 bits (the memory saving
 * that Section 1 names as the first gain of a compact representation, taken below one byte per
 * feature; Section 3.1 asks for the lowest precision that keeps relative positions):
 * code c is stored as the nibble c + 8, feature 2j in the low and 2j + 1 in the high half
 * of byte j, rows padded with code 0 to 64, 96, 128, 192 or 256 features.  A nibble holds
 * -8 .. 7, so at B = 4 the top code +8 is stored as 7, for items and for queries alike (the
 * way +128 becomes 127 at B = 8); distances and norms are those of the stored codes.
 * Searches (lpq_search, lpq_search_i8) unpack in registers and give bit-identical results to
 * an unpacked index holding the same saturated codes; they take k <= 128.  Up to 128 queries run
 * the scan once per 64 queries (the small batches whose time is the corpus read: half the bytes);
 * larger batches take one scan over all queries at about the speed of an unpacked index.
 * lpq_index_data returns the packed rows (*ld_codes = bytes per row); lpq_gather_dist_i8
 * saturates the query codes the same way.  LPQ_EINVAL: B > 4; LPQ_ERANGE: d > 256. */
int lpq_index_create_packed(lpq_index **out, const lpq_quantizer *q, int64_t capacity);
void lpq_index_destroy(lpq_index *idx);

/* Append n items: fp32 vectors (encoded with the index's quantizer, Equation 1) or codes
 * produced earlier by lpq_encode with the same constants (row stride ld bytes).  Item ids are
 * the positions in add order.  Results never depend on the order of the items, but large-batch
 * search time does when near neighbours sit in adjacent rows (a corpus stored cluster by cluster:
 * up to ~2x slower, see lpq_search_overflow_stats); adding the items in shuffled order avoids it. */
int lpq_index_add_f32(lpq_index *idx, const float *x_dev, int64_t n, int64_t ld, void *stream);
int lpq_index_add_i8(lpq_index *idx, const int8_t *codes_dev, int64_t n, int64_t ld, void *stream);
int64_t lpq_index_size(const lpq_index *idx);  /* items added so far; -1 for NULL */

/* Read-only view of the index storage (device pointers owned by the index, valid until it
 * is destroyed): codes [size][*ld_codes] int8 and norms [size] int32.  Any may be NULL. */
int lpq_index_data(const lpq_index *idx, const int8_t **codes_dev, int64_t *ld_codes,
                   const int32_t **norms_dev);

/* --------------------------------------------------------------------- search ---- */

/* Bytes of device workspace lpq_search / lpq_search_i8 need for nq queries and k results
 * (0 on invalid arguments).  The workspace needs 256-byte alignment.  It grows with the batch and
 * with k (1M x 128: 10 000 queries 247 MB at k = 10, 299 at k = 100; about 4 GB for 100 000 queries on long
 * rows): where that is too much, search a batch in parts. */
size_t lpq_search_workspace_bytes(const lpq_index *idx, int64_t nq, int k, int metric);

/* k nearest items of each of nq queries q_dev[nq][ld] (fp32; encoded with the index's
 * quantizer exactly like the items).  Outputs, row i = query i, best first:
 *   ids_dev [nq][k] int32 item ids;
 *   dist_dev[nq][k] int32: L2SQ the full integer distance sum (cq - cx)^2, ascending;
 *                          IP the integer inner product, descending.
 * Equal distances are ordered by ascending id, so the result is unique.
 * 1 <= k <= min(size, 1024).  nq = 0 is a no-op.  Asynchronous on `stream`.
 * Every shape returns the same exact result; speed differs: an index of any number of features is
 * searched on the matrix cores for every k and batch size once it holds enough items for a
 * threshold sample (64 k of them, at most half of the items); smaller indexes go through a plain
 * dot-product kernel (about two orders of magnitude slower per contraction). */
int lpq_search(const lpq_index *idx, const float *q_dev, int64_t nq, int64_t ld, int k,
               int metric, int32_t *ids_dev, int32_t *dist_dev, void *workspace_dev,
               size_t workspace_bytes, void *stream);

/* lpq_search for callers that cannot allocate device memory or pass a workspace: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, results
 * and errors as lpq_search, but the intermediates (query codes, group maxima, candidate lists or
 * regions, counters) live in a device array that is part of the library: LPQ_STATIC_WORKSPACE_BYTES
 * on every GPU the library is used on, held until the process ends.  The call allocates nothing
 * (no hipMalloc / hipFree, no allocating library routine) and is kernel launches only, after one
 * hipGetSymbolAddress per device on the first call there.  A search whose plan needs more than
 * LPQ_STATIC_WORKSPACE_BYTES (lpq_search_workspace_bytes tells) takes a slower one that needs less; if
 * that does not fit either the call returns LPQ_ERANGE and launches nothing: it is meant for small
 * batches (1M x 128: the usual plan fits up to 256 queries at k = 10, 219 at k = 100).  All calls on one GPU share the array, which keeps the previous call's contents (every
 * counter in it is cleared by the kernels that precede its use): calls that overlap on one GPU -
 * different streams, or different threads - race; serialise them on one stream. */
#define LPQ_STATIC_WORKSPACE_BYTES (64u << 20)
int lpq_search_static(const lpq_index *idx, const float *q_dev, int64_t nq, int64_t ld, int k,
                      int metric, int32_t *ids_dev, int32_t *dist_dev, void *stream);

/* Same, for queries that are already codes (int8, row stride ld bytes). */
int lpq_search_i8(const lpq_index *idx, const int8_t *qcodes_dev, int64_t nq, int64_t ld, int k,
                  int metric, int32_t *ids_dev, int32_t *dist_dev, void *workspace_dev,
                  size_t workspace_bytes, void *stream);

/* Exact search on the original fp32 vectors (the reference set S_E of the recall
 * definition, Section 5.3): x_dev[n][ldx], q_dev[nq][ldq], fp32 arithmetic (the squared
 * distance is summed directly as (q - x)^2, never through norms).  dist_dev [nq][k] fp32,
 * L2SQ ascending / IP descending, ties to the lower id.  1 <= k <= min(n, 1024).  A workgroup keeps
 * a query vector and its candidate buffer in 64 KB of LDS, which bounds d: at most 15 328 features
 * for k <= 256, 12 256 for k = 1024 (in between: (65 408 - 8 c) / 4 rounded down to a multiple of 4,
 * c = the power of two >= max(2 k, k + 256)); beyond that LPQ_ERANGE, and the workspace query
 * returns 0.  Batches are searched in parts of as many queries as about 256 MB of workspace hold. */
size_t lpq_search_f32_workspace_bytes(int64_t n, int64_t nq, int d, int k);
int lpq_search_f32(const float *x_dev, int64_t n, int64_t ldx, const float *q_dev, int64_t nq,
                   int64_t ldq, int d, int k, int metric, int32_t *ids_dev, float *dist_dev,
                   void *workspace_dev, size_t workspace_bytes, void *stream);

/* ------------------------------------------------------------ candidate lists ---- */

/* Integer distances between each query and the items its id list names: the distance
 * routine that Section 5.2 swaps into graph indexes, phi(Q(q), Q(x_id)), as one batched
 * call.  qcodes_dev int8 [nq][ld] are codes of the index's quantizer (lpq_encode), ld >= d;
 * ids_dev int32 [nq][m]; dist_dev int32 [nq][m] receives sum (cq - cx)^2 (L2SQ) or
 * sum cq cx (IP).  An id outside [0, size) means "no item" and gives INT32_MAX (L2SQ) /
 * INT32_MIN (IP).  On a packed index the distances are those of the stored (saturated) codes
 * and of the query codes saturated to -8 .. 7.  All buffers are the caller's device memory;
 * asynchronous on stream.
 * LPQ_EINVAL: null argument, m < 1, ld < d, unknown metric; LPQ_ESTATE: empty index. */
int lpq_gather_dist_i8(const lpq_index *idx, const int8_t *qcodes_dev, int64_t nq, int64_t ld,
                       const int32_t *ids_dev, int m, int metric, int32_t *dist_dev, void *stream);

/* Second stage on the original vectors, recovering the recall that quantization costs
 * (the 2-6 % of Section 5.3): for each query the exact distance (binary64 sums) to each of
 * its kc candidates cand_ids_dev [nq][kc] (e.g. the ids of an int8 search with k' > k),
 * the k best sorted by (distance, id): ids_dev int32 [nq][k], dist_dev fp32 [nq][k]
 * (L2SQ ascending / IP descending).  Candidate ids outside [0, n) are skipped; if fewer
 * than k remain the row is completed with id -1 and distance +inf (L2SQ) / -inf (IP).
 * 1 <= kc <= 4096, k >= 1.  Asynchronous on stream; no workspace.
 * LPQ_EINVAL: null argument, d < 1, ldx/ldq < d, kc or k < 1, unknown metric; LPQ_ERANGE:
 * kc > 4096. */
int lpq_rerank_f32(const float *x_dev, int64_t n, int64_t ldx, const float *q_dev, int64_t nq,
                   int64_t ldq, int d, const int32_t *cand_ids_dev, int kc, int k, int metric,
                   int32_t *ids_dev, float *dist_dev, void *stream);

/* ------------------------------------------------------------- key-value cache ---- */

/* The maximum-inner-product search a language model makes for every token it generates, over keys that
 * grow by one per step: keys and values of the tokens so far, held as codes of Equation 1 in pages of a
 * pool, and the attention that reads them.  One lpq_kv is the cache of one layer: `heads` key-value heads
 * of D = d / heads features (feature h D + i of the quantizers is feature i of head h).
 *
 * Storage is the caller's device memory, 256-byte aligned, and must outlive the handle:
 *   k_dev, v_dev  [pages][heads][page][row bytes] codes: one byte each, rows padded to 64, 128, 192 or 256
 *                 features with code 0; packed: two 4-bit codes per byte as in lpq_index_create_packed
 *                 (stored + 8, feature 2j in the low half of byte j, +8 stored as 7)
 *   bounds_dev    [pages][heads][2][padded features] int8: the smallest and the largest key code of each feature
 *                 over the page's tokens
 * It need not be cleared.  A sequence's token at position p lies in row p % page of page table[p / page] of
 * its row of a table (int32, device, ld_table apart, table_pages columns).  Every call checks table entries:
 * one outside [0, pages) means that there is no page there (what would go there is dropped, what would be
 * read there does not exist).  A position at or beyond table_pages * page has no page.
 *
 * A code c reads back as x^ = k + (c + 1/2) s with s = fl32(1 / m), each operation rounded to binary32 (a
 * feature without a range reads back as k).  Types of rows and queries: */
enum { LPQ_TYPE_F32 = 0, LPQ_TYPE_F16 = 1, LPQ_TYPE_BF16 = 2 };

/* Bytes of k_dev and of v_dev (each) and of bounds_dev; *row_features receives the padded features of a row.
 * Any output may be null.  head_dim 1..256; page 16, 32, 64, 128 or 256 tokens.
 * LPQ_EINVAL: heads, head_dim or pages < 1, another page size; LPQ_ERANGE: head_dim > 256, pages >= 2^31. */
int lpq_kv_storage_bytes(int heads, int head_dim, int page, int64_t pages, int packed, size_t *codes, size_t *bounds,
                         int *row_features);

/* The cache of the quantizers' constants (copied; both of the same d, a multiple of heads; packed: of at most
 * 4 bits).  Synchronises the device.  Errors as above; LPQ_ESTATE: a quantizer without constants. */
int lpq_kv_create(lpq_kv **out, const lpq_quantizer *keys, const lpq_quantizer *values, int heads, int page,
                  int64_t pages, int packed, void *k_dev, void *v_dev, void *bounds_dev);
void lpq_kv_destroy(lpq_kv *kv);

/* Encodes n new rows of keys and values, k_dev / v_dev [n][heads][D] of `type` (strides in elements, the features
 * of a head contiguous), and stores them: row starts_dev[b] + i goes to position first_dev[b] + i of sequence b
 * (starts_dev int32 [nseq + 1], ascending; null: one row per sequence, n = nseq).  Rows at negative positions and rows
 * of no sequence, ahead of starts_dev[0] or from starts_dev[nseq] on, are dropped.  Bounds of the pages touched become
 * those of their tokens up to the last one written, so that a sequence may be cut back and written on.  No page may be
 * touched twice by one call.
 * Asynchronous on stream.  n = 0 is a no-op.
 * LPQ_EINVAL: null argument, n or nseq < 0, strides that overlap (of rows that are written, by lpq_kv_read), unknown type,
 * starts_dev null and n != nseq, rows but no sequence;
 * LPQ_ERANGE: nseq * heads or table_pages * page too large. */
int lpq_kv_write(const lpq_kv *kv, const void *k_dev, int64_t ldk_token, int64_t ldk_head, const void *v_dev,
                 int64_t ldv_token, int64_t ldv_head, int type, int64_t n, int64_t nseq, const int32_t *first_dev,
                 const int32_t *starts_dev, const int32_t *table_dev, int64_t ld_table, int64_t table_pages,
                 void *stream);

/* lpq_kv_write of keys that are turned by the angles of their positions first (values are not), and with them the
 * queries of the same tokens.  cos_dev, sin_dev float [angles][rotated / 2], ld_angles apart: row p belongs to position p.  The
 * first `rotated` features of a head are turned in pairs, (i, i + rotated / 2) or, interleaved != 0, (2 i, 2 i + 1), the others not:
 *   a' = fl(fl(a cos) - fl(b sin)),  b' = fl(fl(b cos) + fl(a sin))   in binary32,
 * and the keys encoded from that, without a rounding to their type between.  A row's position is the one that it is written to, or
 * positions_dev[row] (int32 [n], null: none given), as for drafted tokens that share a depth in a tree.
 * q_dev null, or n rows [n][q_heads][D] numbered as the keys, of the same type: out_dev receives them turned, rounded to
 * the type; q_heads a multiple of heads.  out_dev may be q_dev with its strides (turned in place); else the two must not overlap, and out_dev
 * never overlaps the keys, the values or the angles.
 * Rows at positions below 0 and rows of no sequence are not turned (queries come out as they are; keys as in lpq_kv_write); at positions beyond the table's
 * the turned features are NaN (which a key's code holds as 0).
 * Errors as lpq_kv_write; LPQ_EINVAL: rotated odd, below 2 or above D, angles < 1, ld_angles < rotated / 2, queries without an
 * output, q_heads not a multiple of heads, strides of the output that overlap, an output that begins where the keys or the values do, or where the
 * queries do with other strides; LPQ_ERANGE: angles >= 2^31, q_heads > 65536. */
int lpq_kv_write_rotated(const lpq_kv *kv, const void *k_dev, int64_t ldk_token, int64_t ldk_head, const void *v_dev,
                         int64_t ldv_token, int64_t ldv_head, int type, int64_t n, int64_t nseq,
                         const int32_t *first_dev, const int32_t *starts_dev, const int32_t *table_dev, int64_t ld_table,
                         int64_t table_pages, const float *cos_dev, const float *sin_dev, int64_t ld_angles,
                         int64_t angles, int rotated, int interleaved, const int32_t *positions_dev, const void *q_dev,
                         int64_t ldq_token, int64_t ldq_head, int q_heads, void *out_dev, int64_t ldo_token,
                         int64_t ldo_head, void *stream);

/* The way back: rows of the same numbering receive x^ of their position, rounded to `type`; positions without a
 * page and rows of no sequence give zeros.  Errors as above. */
int lpq_kv_read(const lpq_kv *kv, void *k_dev, int64_t ldk_token, int64_t ldk_head, void *v_dev, int64_t ldv_token,
                int64_t ldv_head, int type, int64_t n, int64_t nseq, const int32_t *first_dev,
                const int32_t *starts_dev, const int32_t *table_dev, int64_t ld_table, int64_t table_pages,
                void *stream);

/* Queries of the calls below: q_dev [nseq][new_tokens][q_heads][D] of `type`, strides in elements; q_heads a multiple
 * of heads, query heads h G .. h G + G - 1 share key-value head h (G = q_heads / heads).  lengths_dev int32 [nseq]:
 * tokens of each sequence, the new ones included: new token i sees positions <= length - new_tokens + i.
 * A call takes new_tokens * q_heads <= 65536, nseq * new_tokens * q_heads and nseq * heads <= 2^22, and table_pages * page < 2^31 (else
 * LPQ_ERANGE); longer prompts go through attention in parts, each with the length up to its end.
 *
 * Which pages can hold large inner products.  Over the R = new_tokens * G rows of a key-value head, in binary32:
 * q' = q s, A = max |q'|, z = rint(q' * (127 / A)) (what is not finite counts as 0; A <= 1e-30: all 0);
 *   score(page) = sum_i [ (sum_r max(z_ri, 0)) hi_i + (sum_r min(z_ri, 0)) lo_i ],
 * an upper bound, summed over the rows, of the integer product with any token of the page.  pages_dev
 * [nseq][heads][n_select] receives the numbers (columns of the table) of the first keep_first and the last keep_last of
 * a sequence's pages and of those with the largest scores, ties to the lower number, ascending; -1 behind them where
 * there are fewer.  Integers throughout: the result is unique.  Workspace: 256-byte aligned (0 bytes for small tables).
 * LPQ_EINVAL: null argument, n_select < 1, keep_first or keep_last < 0 or more than n_select together, q_heads not a
 * multiple of heads; LPQ_ERANGE: new_tokens * G > 128, workspace too small, sizes as above. */
size_t lpq_kv_select_workspace_bytes(const lpq_kv *kv, int64_t nseq, int64_t table_pages);
int lpq_kv_select(const lpq_kv *kv, const void *q_dev, int64_t ldq_seq, int64_t ldq_token, int64_t ldq_head, int type,
                  int64_t nseq, int new_tokens, int q_heads, const int32_t *lengths_dev, const int32_t *table_dev,
                  int64_t ld_table, int64_t table_pages, int n_select, int keep_first, int keep_last, int32_t *pages_dev,
                  void *workspace_dev, size_t workspace_bytes, void *stream);

/* Attention: out_dev (as q_dev, strides of its own) = sum_j p_j y^_j over the tokens j a row sees, p = softmax(scale
 * q . x^_j), x^ and y^ keys and values as they read back.  chosen_dev null: all pages (n_select is not used); else
 * int32 [nseq][heads][n_select] pages as lpq_kv_select gives them, in any order (an entry outside [0, table_pages) is
 * none; a page named twice counts twice).  lse_dev: null, or float [nseq][new_tokens][q_heads], the logarithm of the sum of
 * exp(scale q . x^_j), with which attention over other tokens can be joined.  A row that sees no token gives
 * zeros and -inf, whatever it holds; else a row of queries that holds a NaN or an infinity gives NaN.  Scores are exact
 * sums of a query rounded to 16 bits (float16: 24, float32: 32) of its largest q s; weights are rounded to fp16
 * (float32: to 22 bits); sums are in 32 bits.
 * The order of all sums is fixed: equal calls give equal bits.
 * The workspace (256-byte aligned) holds the parts a long sequence is split into.
 * LPQ_EINVAL: null argument, new_tokens < 1, q_heads not a multiple of heads, strides that overlap, unknown type,
 * n_select < 1 with chosen_dev, scale not finite; LPQ_ERANGE: workspace too small, sizes as above. */
size_t lpq_kv_attend_workspace_bytes(const lpq_kv *kv, int64_t nseq, int new_tokens, int q_heads, int64_t table_pages,
                                     int n_select);
int lpq_kv_attend(const lpq_kv *kv, const void *q_dev, int64_t ldq_seq, int64_t ldq_token, int64_t ldq_head, int type,
                  int64_t nseq, int new_tokens, int q_heads, float scale, const int32_t *lengths_dev,
                  const int32_t *table_dev, int64_t ld_table, int64_t table_pages, const int32_t *chosen_dev,
                  int n_select, void *out_dev, int64_t ldo_seq, int64_t ldo_token, int64_t ldo_head, float *lse_dev,
                  void *workspace_dev, size_t workspace_bytes, void *stream);

/* The same where new tokens see less.  One of
 *   window > 0   a token at position p sees the positions j <= p with j > p - window, and those with j < sinks (the window
 *                counts the token itself; window 0: none, and then no sinks);
 *   tree_dev     not null: drafted tokens that do not follow one another.  A new token sees every position ahead of the
 *                new ones (below length - new_tokens), and of the new ones those that its row of tree_dev [nseq][new_tokens]
 *                [new_tokens] names (bytes, 0: not seen; the last axis contiguous, strides of the others in bytes, 0 where a
 *                mask is shared): itself and its ancestors, as a rule.  A row that names nothing sees the tokens ahead
 *                only.  New tokens whose own position is below 0 see nothing, as in lpq_kv_attend;
 * or neither: lpq_kv_attend.  Of chosen pages, the tokens that are seen.  Only pages that a row sees something of are read (chosen pages:
 * all of them).
 * A row's result does not depend on what is stored at positions that it does not see, and on the rows beside it only within the roundings of its
 * weights (where their common maximum stood).
 * LPQ_EINVAL beside what is named above: window or sinks below 0, sinks without a window, window and tree, strides of the
 * tree below 0 or beyond 2^40; LPQ_ERANGE: a tree of more than 4096 new tokens. */
size_t lpq_kv_attend_masked_workspace_bytes(const lpq_kv *kv, int64_t nseq, int new_tokens, int q_heads,
                                            int64_t table_pages, int n_select, int64_t window, int sinks, int tree);
int lpq_kv_attend_masked(const lpq_kv *kv, const void *q_dev, int64_t ldq_seq, int64_t ldq_token, int64_t ldq_head,
                         int type, int64_t nseq, int new_tokens, int q_heads, float scale, const int32_t *lengths_dev,
                         const int32_t *table_dev, int64_t ld_table, int64_t table_pages, const int32_t *chosen_dev,
                         int n_select, int64_t window, int sinks, const uint8_t *tree_dev, int64_t ldt_seq,
                         int64_t ldt_token, void *out_dev, int64_t ldo_seq, int64_t ldo_token, int64_t ldo_head,
                         float *lse_dev, void *workspace_dev, size_t workspace_bytes, void *stream);

/* ------------------------------------------------- linear layers on 8-bit codes ---- */

/* Rows of a model's type as codes of their own scale, and their products.  Of a row x of d values and A = max |x|:
 *   code = rint(fl(x * fl(127 / A))),  scale = fl(A / 127)   in binary32, to nearest even (A below 2^-100: x and A times 2^60 first,
 * exactly); a row of zeros has the scale 0.  A row that holds an infinity or a NaN has the codes 0 and the scale NaN, and all its
 * products are NaN.
 *
 * Codes are kept in blocks of 16 rows x 64 features, the shape in which the matrix instructions take them: row i, feature k is byte
 * ((i / 16) B + k / 64) 1024 + (k % 64 / 16) 256 + (i % 16) 16 + k % 16, with B = 2 ceil(d / 128) blocks to a row.
 * lpq_row_codes_bytes: what n rows take, the last block's rows behind n included (0: out of range).
 * lpq_encode_rows: x_dev [n][d] of `type`, rows ldx elements apart, to codes and scales_dev float [n].  Features from d to the end of the last
 * block are set to 0; rows of it behind n are not touched.
 * lpq_matmul_i8: out[i][c] = (sum_k a[i][k] b[c][k]) * a_scale[i] * b_scale[c] + bias[c] for m rows and n channels.  Sums are exact in 32 bits; then
 * each step is rounded to binary32: the sum itself (beyond 2^24), its products with the scales in this order, the sum with the bias; and the result to
 * `type`.  No scale makes a product leave binary32's range on the way.  bias_dev float [n] or null; rows of the output ldo elements apart.
 * Codes are -127 .. 127 as lpq_encode_rows leaves them: features behind d are read and must be 0 in a or in b; what rows behind m or n hold does
 * not matter.  One set of codes can go through several products.
 * lpq_linear8: both for rows x_dev [m][d] of `type`, which the output has too.  Rows x_dev may overlap (ldx 0: one row n times).  A row's results do not depend on the rows beside it.
 * Codes: 256-byte aligned.  Workspace: 256-byte aligned, for the one call (null where 0 bytes are needed); one that
 * was captured into a graph belongs to the graph.  Output and workspace must not overlap the inputs.
 * LPQ_EINVAL: null argument, negative size, unknown type, strides below 0, beyond 2^40 elements or with which
 * outputs overlap, misaligned codes or workspace;
 * LPQ_ERANGE: d > 131072 (its sums would not fit 32 bits), more than 2^25 rows or channels, more than 2^22 tiles of 128 rows x 128
 * channels, too small a workspace. */
size_t lpq_row_codes_bytes(int64_t n, int d);
int lpq_encode_rows(const void *x_dev, int64_t ldx, int type, int64_t n, int d, int8_t *codes_dev, float *scales_dev, void *stream);
size_t lpq_matmul_i8_workspace_bytes(int64_t m, int64_t n, int d);
int lpq_matmul_i8(const int8_t *a_dev, const float *a_scales_dev, int64_t m, const int8_t *b_dev, const float *b_scales_dev, int64_t n, int d,
                  const float *bias_dev, void *out_dev, int64_t ldo, int type, void *workspace_dev, size_t workspace_bytes, void *stream);
size_t lpq_linear8_workspace_bytes(int64_t m, int64_t n, int d);
int lpq_linear8(const void *x_dev, int64_t ldx, int type, int64_t m, const int8_t *codes_dev, const float *scales_dev, int64_t n,
                int d, const float *bias_dev, void *out_dev, int64_t ldo, void *workspace_dev, size_t workspace_bytes,
                void *stream);

/* ---------------------------------------------------------------- diagnostics ---- */

/* Process-wide tuning knobs for measurements; 0 restores the built-in choice.
 *   LPQ_TUNE_PATH        1 = generic dot-product kernel, 2 = matrix-core kernels (built-in
 *                        choice of variant), 3 = the collecting matrix-core variant for every
 *                        k it takes, 4 = matrix-core kernels without the
 *                        collecting variant
 *   LPQ_TUNE_SPLITS      number of corpus splits per query tile in the main pass
 *   LPQ_TUNE_SEED_ROWS   rows of the threshold-seeding pass (0 = built-in choice,
 *                        -1 = no seeding pass)
 *   LPQ_TUNE_DRY_RUN     timing ablations of the matrix-core kernel whose results are meaningless
 *                        (1 never collects a candidate, 2 no workgroup barrier, 3 no corpus
 *                        copies, 4 neither, 5 candidates detected but not queued, 6 queued but
 *                        not processed, 7 every copy reads the first two stages of its split, which
 *                        stay in L2).  Compiled only into builds made with -DLPQ_ABLATION
 *                        (python -m paper_2110_08919_amd.build --ablation writes
 *                        liblpq_ablation.so); the shipped library has none of these branches
 *                        and rejects a non-zero value with LPQ_EINVAL.
 *   LPQ_TUNE_WORK_ORDER  how workgroups of the matrix-core kernel are dealt to (split, query tile)
 *                        pairs: 0 built-in, 1 each XCD takes whole splits, 2 each XCD takes whole
 *                        query tiles, 3 plain block order
 *   LPQ_TUNE_WAVE_QUERIES queries per wave of the collecting variant: 64 or 128 (0 = built-in)
 *   LPQ_TUNE_REGION_CAP  candidates a region of the collecting variant holds (0 = built-in); a tiny
 *                        value makes most queries overflow and go through the exact redo paths
 * Results never depend on PATH, SPLITS, SEED_ROWS, WORK_ORDER, WAVE_QUERIES or REGION_CAP.
 * The knobs are atomics: setting one while other threads search is not a data race; a search
 * reads each knob at some moment of its planning, so set them before the searches they are for
 * (lpq_search_workspace_bytes and the lpq_search that uses its answer must see the same values). */
enum { LPQ_TUNE_PATH = 0, LPQ_TUNE_SPLITS = 1, LPQ_TUNE_SEED_ROWS = 2, LPQ_TUNE_DRY_RUN = 3, LPQ_TUNE_WORK_ORDER = 4,
       LPQ_TUNE_WAVE_QUERIES = 5, LPQ_TUNE_REGION_CAP = 6, LPQ_TUNE_COUNT_ = 7 };
int lpq_set_tuning(int key, int64_t value);

/* Kernel timing for benchmarks.  While enabled, every launch of the contraction/top-k
 * kernel of lpq_search* (LPQ_PROFILE_SCAN) and of its threshold-seeding pass
 * (LPQ_PROFILE_SEED) is bracketed by a pair of HIP events on the launch stream.
 * lpq_profile_read synchronises those events and returns the number of bracketed
 * launches and their summed duration in milliseconds since the last enable;
 * lpq_profile_read_kind does the same for one kind of launch. */
enum { LPQ_PROFILE_SCAN = 0, LPQ_PROFILE_SEED = 1 };
int lpq_profile_enable(int on);
int lpq_profile_read(int64_t *launches, double *total_ms);
int lpq_profile_read_kind(int kind, int64_t *launches, double *total_ms);

/* How lpq_search would run a search, computed on the host without any device or index: the plan
 * for nq queries and k results on an index of n_items items of d features at `bits` bits (packed:
 * two codes per byte).  For capacity planning (out[16] is what lpq_search_workspace_bytes would
 * return less its 256 bytes of alignment slack) and for checking the planner itself.  out receives
 * LPQ_PLAN_INFO_COUNT values:
 *   [0] kernel family (0 generic dot-product kernel, 1 matrix-core with lists in LDS, 2 matrix-core
 *       with lists in registers, 3 matrix-core collecting scan)   [1] row-split workgroups (0/1)
 *   [2] waves of a row-split workgroup   [3] queries per wave of the collecting scan
 *   [4] query rows the workspace holds (padded)   [5] rows of the threshold-seeding pass (0 = none)
 *   [6] corpus splits of the seeding pass   [7] corpus splits of the main scan   [8] segments per split
 *   and [9] group maxima per query of the seeding pass   [10] candidate regions per query and
 *   [11] their capacity (collecting scan)   [12] splits of the generic redo   [13] splits of the
 *   register-list redo   [14] further rounds of the collecting scan   [15] lists merged per workgroup
 *   in a first merge pass (0 = one pass)   [16] workspace bytes   [17] offset of the per-tile plan
 *   inside the workspace (packed index; else 0)
 *   [18..33] byte offsets of the plan's buffers in the order they are laid out (0 = not used), [34]
 *   their end.  Every offset is a multiple of 256 and the used ones never decrease.  (A packed
 *   index is searched in tiles of 64 queries unless one collecting scan takes the whole batch: the
 *   values then describe the plan of a full tile, [4], [16] and [17] the whole workspace.)
 * Where lpq_search_maxima_info reports groups, the search goes by group maxima: [1], [2], [4] and
 * [16..34] are of that search, [0], [3] and [5..15] of the one with lists or regions that it takes
 * the place of, which runs as soon as a tuning key asks for another kernel, split, sample or region.
 * LPQ_EINVAL / LPQ_ERANGE as for lpq_quantizer_create, lpq_index_create and lpq_search. */
#define LPQ_PLAN_INFO_COUNT 35
int lpq_search_plan_info(int d, int bits, int packed, int64_t n_items, int64_t nq, int k, int64_t *out,
                         int out_count);
/* Whether such a search goes by group maxima (small batches: one scan of all rows that keeps the largest score of
 * each group of rows, and one kernel that scores the groups again which reach the k-th largest; no sample, lists,
 * regions or redo), and how.  out receives LPQ_MAXIMA_INFO_COUNT values, all 0 where it does not:
 *   [0] groups per query   [1] corpus splits   [2] segments per split   [3] waves of a workgroup of the scan
 *   [4] rows of a stage   [5] threads of a workgroup of the last kernel, and how many of them search for a query
 *   [6] usually and [7] where many groups reach the bound.   Of a packed index: of a full tile of 64 queries.
 * Errors as above. */
#define LPQ_MAXIMA_INFO_COUNT 8
int lpq_search_maxima_info(int d, int bits, int packed, int64_t n_items, int64_t nq, int k, int64_t *out,
                           int out_count);

/* Attainable-rate probes (benchmarks only): what this GPU sustains on the two resources that
 * bound lpq_search, measured by kernels that do nothing else, so that a roofline fraction quoted
 * against a published peak can be read next to what the part reaches in practice.  Both calls
 * allocate a small device buffer, time with events on `stream` and synchronise it.
 *   lpq_probe_mfma_i8: a register-resident loop of the int8 matrix instruction the search uses
 *     (the contraction of Section 3.1's phi on codes), `iters` x 8 instructions per wave, four
 *     waves per workgroup, two workgroups per CU.  The operand registers are filled from
 *     operands_dev[operand_bytes] (device memory, 16-byte aligned; null = all-zero operands): the
 *     sustained rate depends on how many operand bits toggle, so pass the bytes of interest
 *     (random bytes, or the codes of an index).  *tops = 1e12 integer operations per second.
 *   lpq_probe_scan_core: the inner loop of the batched scan and nothing else - per 32 rows and 128
 *     queries of a wave sixteen matrix instructions with the filter epilogue (maximum of the 16
 *     accumulators of a lane, threshold compare, branch) and the row operands and accumulator seeds
 *     read from LDS - without corpus copies, barriers or candidates; `stages` x 64 instructions
 *     per wave.  LDS ring and query registers are filled from operands_dev as above.  *tops as
 *     above: the ceiling of that loop on this GPU for such operand bits.
 *   lpq_probe_stream: reads bytes (rounded down to a multiple of 4096) of src_dev `reps` times,
 *     mode 0 through the asynchronous global->LDS copies of the scan kernels, mode 1 through
 *     16-byte register loads.  *gbps = 1e9 bytes per second.
 * LPQ_EINVAL: null output, iters or stages outside 1..10 000 000, misaligned or too small a buffer,
 * unknown mode, reps outside 1..10 000. */
int lpq_probe_mfma_i8(const void *operands_dev, size_t operand_bytes, int iters, double *tops, void *stream);
int lpq_probe_scan_core(const void *operands_dev, size_t operand_bytes, int stages, double *tops, void *stream);
int lpq_probe_stream(const void *src_dev, size_t bytes, int mode, int reps, double *gbps, void *stream);

/* How lpq_matmul_i8 goes about a product: [0] tokens and [1] channels of a workgroup, [2] parts that the features are dealt out in (0: few
 * rows, whose weights go past LDS), [3] 1 where lpq_linear8 makes the codes in the same launch.  Needs no device.  LPQ_EINVAL /
 * LPQ_ERANGE as lpq_matmul_i8; out_count < LPQ_LINEAR8_INFO_COUNT. */
#define LPQ_LINEAR8_INFO_COUNT 4
int lpq_linear8_plan_info(int64_t m, int64_t n, int d, int64_t *out, int out_count);

/* Diagnostics of the collecting variant: after a search with the same (idx, nq, k, metric) and
 * workspace has finished, the number of queries whose candidates did not fit and that were
 * searched again (0 when the search did not use the collecting variant) and the
 * largest number of candidates any region received in the last round of the scan.  Of a small batch
 * that was searched by group maxima: the queries that more groups of rows tie for than are all
 * scored again, and the most candidates one of the last workgroups kept.  Synchronises the device. */
int lpq_search_overflow_stats(const lpq_index *idx, int64_t nq, int k, int metric, const void *workspace_dev,
                              int64_t *redone_queries, int64_t *max_region_fill);

/* Where the plan has further rounds (for k > 16, and on rows of more than 256 bytes) such queries are not
 * searched again exactly at once (but for a few of a large batch with k <= 32): the scan runs again (up to two more rounds) over the query tiles that
 * hold one, with bounds taken from the candidates the round before did collect, and only queries that
 * overflow every time go through the generic kernel.  *left_queries = their number after the last search
 * (0 when the plan has no further rounds or they did not run).  Same arguments and synchronisation as above. */
int lpq_search_overflow_left(const lpq_index *idx, int64_t nq, int k, int metric, const void *workspace_dev,
                             int64_t *left_queries);

/* Message of the last error on the calling thread ("" if none). */
const char *lpq_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* LPQ_H */
