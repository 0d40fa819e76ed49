/*
 * archer_ops.h -- single-kernel entry points and timing of the Archer library.
 *
 * archer_op_gemm, archer_op_attention and archer_op_attention_noalloc run one kernel of the
 * decoding path exactly as the model path launches it (same kernels, same tile and split
 * choices for the same shapes), on caller-provided device buffers.  They exist so that the
 * kernels can be checked element by element at full model sizes and timed in
 * isolation.  The calls of the 4-bit and 8-bit paged prompt caches, of pages that sequences
 * share and of sampling are operators of their own, for programs that hold prompts
 * so and draw tokens: the decoding path keeps its fp16 cache and its greedy decision and
 * runs none of them.  Conventions as in archer.h: device pointers, caller-owned
 * memory, asynchronous on the given stream, host-side argument checks.
 */
#ifndef ARCHER_OPS_H
#define ARCHER_OPS_H

#include "archer.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Y = A W^T (a projection of the transformer layer; the alpha_l work of
 * Eq. theory-cost).  A: [M][K], W: [N][K], both of element type dtype,
 * row-major; Y: fp32 [M][N].  M >= 1; N and K multiples of 64.
 * A_lo (bf16 only, may be NULL): low part of a two-term activation, so that
 * A + A_lo carries about 16 significant bits; the product is then
 * (A + A_lo) W^T, as in every projection of the bf16 model path. */
archer_status archer_op_gemm(int32_t dtype, int32_t M, int32_t N, int32_t K, const void *A,
                             const void *A_lo, const void *W, float *Y, void *hip_stream);

/* The tiles that a projection of the model path takes, as text (host only, no
 * GPU is touched): class k_class (ARCHER_K_GEMM_QKV, _O, _GATEUP, _DOWN or
 * _HEAD; a full pass chooses like a cached one of as many rows) over `rows`
 * rows in a context of this bf16 model and these limits, weights in `layout`,
 * activations of the default precision; stats: the LM head also writes the
 * decision statistics.  One part per launch, "<rows> rows [staged |wide ]<BM>x<BN>"
 * with ", <S> slices" or ", <S> folded slices" where K is split, joined by
 * "; ".  For checking that a shape reaches the kernel it is meant to. */
archer_status archer_op_projection_tiles(const archer_model_cfg *cfg, const archer_limits *lim, int32_t layout,
                                         int32_t k_class, int32_t rows, int32_t stats, char *text, size_t bytes);

/* Non-causal attention of one sequence over two key segments, the anchored
 * attention of Eq. archer-attention: every query of head h attends to the nk1
 * keys of segment 1 followed by the nk2 keys of segment 2 of key/value head
 * h / (Hq / Hkv), scale 1 / sqrt(hd).  Q, K and V are fp16 for ARCHER_BF16
 * (as the bf16 model path stores them) and fp32 for ARCHER_FP32; O has the
 * element type dtype (bf16 / fp32).
 *   Q   [Hq][Mq][hd]                    O  [Mq][Hq hd]
 *   K1  [Hkv][ld1][hd]   Vt1 [Hkv][hd][ld1]   (segment 1, keys 0..nk1-1)
 *   K2  [Hkv][ld2][hd]   Vt2 [Hkv][hd][ld2]   (segment 2, keys 0..nk2-1)
 * V is stored transposed (Vt[h][d][key]).  ld1, ld2 multiples of 64,
 * nk1 <= ld1, nk2 <= ld2, head_dim 64 or 128.  Keys are read in tiles of
 * 64, so segment 1 must be readable up to nk1 rounded up to 64 (the values
 * there are ignored).
 * workspace: device scratch of archer_op_attention_ws_bytes(...) bytes,
 * 256-byte aligned (split-KV partial results; none is needed, and NULL is
 * accepted, when the key count gives one split).  Calls sharing a workspace
 * must not overlap. */
size_t archer_op_attention_ws_bytes(int32_t dtype, int32_t Mq, int32_t Hq, int32_t hd, int32_t nk);
archer_status archer_op_attention(int32_t dtype, int32_t Mq, int32_t Hq, int32_t Hkv, int32_t hd,
                                  const void *Q, const void *K1, const void *Vt1, int32_t nk1,
                                  int32_t ld1, const void *K2, const void *Vt2, int32_t nk2,
                                  int32_t ld2, void *O, void *workspace, size_t ws_bytes,
                                  void *hip_stream);

/* archer_op_attention for callers that cannot allocate device memory (code
 * under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc): the same kernels, launch configuration and results, with the
 * split-KV partials in a fixed scratch array that the library holds in each
 * device's memory (64 MiB per device, for the life of the process) instead
 * of a caller workspace.  Arguments as archer_op_attention without the
 * workspace; hip_stream must belong to the calling thread's current device.
 * Allocates nothing: ARCHER_E_SHAPE (before any launch) when the shape's
 * split-KV partials, archer_op_attention_ws_bytes, exceed 64 MiB.  All calls
 * on one device share its array: calls that overlap in time on one device
 * (other streams, other threads) race, and must be serialised by the caller.
 * The array is fully rewritten before it is read in every call, so nothing
 * carries over from the previous call. */
archer_status archer_op_attention_noalloc(int32_t dtype, int32_t Mq, int32_t Hq, int32_t Hkv, int32_t hd,
                                          const void *Q, const void *K1, const void *Vt1, int32_t nk1,
                                          int32_t ld1, const void *K2, const void *Vt2, int32_t nk2,
                                          int32_t ld2, void *O, void *hip_stream);

/* ---- 4-bit paged prompt cache -------------------------------------------------
 * One layer's keys and values in e2m1 (sign, two exponent bits, one mantissa
 * bit: 0, .5, 1, 1.5, 2, 3, 4, 6) with one power-of-two scale per 32
 * dimensions: 136 instead of 512 bytes per token and head of 128 dimensions.
 * Tokens live in pages of page_size tokens; a slot is
 * page * page_size + position in the page, and a sequence's row of a block
 * table lists its pages in order.  The table of a read or an attention may list a
 * page in several rows; a plan's may not (archer_cache4_plan).
 *
 * data: device, 16-byte aligned, archer_cache4_bytes bytes, caller-owned.
 * [n_pages][n_kv_heads] blocks of page_size * (head_dim + head_dim / 16) bytes:
 *   keys    [page_size][head_dim / 2]             byte j: dimensions 2j (low nibble), 2j + 1
 *   values  [page_size / 8][16][8][head_dim / 32] unit u: dimensions u head_dim / 16 ..
 *   key scales, then value scales [page_size / 8][head_dim / 32][8]   exponent + 127
 * page_size 32, 64, 128 or 256; head_dim 64 or 128; n_pages * page_size < 2^31. */
typedef struct {
  void *data;
  int32_t n_pages, page_size, n_kv_heads, head_dim;
} archer_cache4;

/* Bytes of the cache's data (0 and last_error for a bad shape; data is not read). */
size_t archer_cache4_bytes(const archer_cache4 *cache);

/* Block tables, free pages and the slots of new rows for requests whose
 * lengths change from len_old[b] to len_new[b] (device int32 [batch]; batch <=
 * 4096): a request that grows takes pages, one that shrinks (rollback, or 0:
 * finished) gives its last ones back.  One call, no synchronisation.
 *   table       [batch][max_pages], in place: entries below ceil(len_old / page_size)
 *               are the request's pages; the taken ones are appended, all others
 *               (those given back too) stay as they are
 *   free_pages  [n_pages], in place: a ring of the free pages
 *   pool_in     [2]: index of the ring's first free page, number of free pages
 *   pool_out    [2]: the same after the call; must not alias pool_in
 *   row_off     [batch + 1]: prefix sums of the rows added, max(len_new - len_old, 0)
 *   slot_map    [slot_rows]: the slot of every added row, request by request, then -1
 *   status      [1]: 0, or why nothing was changed (pool_out = pool_in, row_off 0,
 *               slot_map -1): 1 too few free pages, 2 a length is negative or beyond
 *               max_pages, 3 more than slot_rows rows, 4 the pool is inconsistent
 * A plan counts no references: every page that it is to take, keep or give back must be the
 * page of one request, once, and not be free.  A page shared by several sequences
 * belongs to one of them here; the others list it in tables of their own, and its owner
 * must not shrink below it while they do (it would be handed out again).  This
 * is not checked.
 * Pages are taken from the ring's front in request order and given back behind
 * its end, those of this call for later ones.  Called again with the same
 * arguments it gives the same results.  The arrays must not overlap. */
archer_status archer_cache4_plan(int32_t batch, const int32_t *len_old, const int32_t *len_new,
                                 int32_t page_size, int32_t n_pages, int32_t max_pages, int32_t *table,
                                 int32_t *free_pages, const int32_t *pool_in, int32_t *pool_out,
                                 int32_t *row_off, int32_t *slot_map, int32_t slot_rows, int32_t *status,
                                 void *hip_stream);

/* Store rows of keys and values (fp16 for ARCHER_BF16, fp32 for ARCHER_FP32) in
 * the slots slot_map[row]; rows whose slot is outside the cache (-1) are
 * skipped.  Slots of one call must be distinct (of rows that share one, an
 * unspecified mixture is stored); rows >= 0.  Element (head, row, d) is at
 * K[head k_head + row k_row + d] and V[head v_head + row v_row + d v_dim] (strides in
 * elements, any sign), with v_dim = 1 or v_row = 1: the prompt cache's
 * transposed values are stored as they lie (else ARCHER_E_UNSUPPORTED; of a single row
 * any v_dim will do).
 * Per 32 dimensions the scale is 2^e, e the least integer with max |x| <= 7 * 2^e,
 * clamped to [-23, 13]; elements are rounded to the nearest e2m1 value of
 * x / 2^e, ties to the even code, and saturate at 6 * 2^e (49152 at most).  Every
 * stored element is exact in fp16.  A NaN makes its 32 elements NaN. */
archer_status archer_cache4_write(int32_t dtype, const archer_cache4 *cache, int32_t rows, const void *K,
                                  int64_t k_head, int64_t k_row, const void *V, int64_t v_head,
                                  int64_t v_row, int64_t v_dim, const int32_t *slot_map, void *hip_stream);

/* The stored elements of the slots slot_map[row], as fp16 (ARCHER_BF16) or
 * fp32 (ARCHER_FP32): K and V [n_kv_heads][rows][head_dim], 16-byte aligned.
 * Rows whose slot is outside the cache become zeros.  Slots may repeat. */
archer_status archer_cache4_read(int32_t dtype, const archer_cache4 *cache, int32_t rows,
                                 const int32_t *slot_map, void *K, void *V, void *hip_stream);

/* The anchored attention with the cached segment in 4 bits, for a batch: row i of
 * sequence b attends to the sequence's cached keys, positions 0 ..
 * cached_len[b] - 1 through row b of the block table, and, where K2 is given, to the
 * sequence's fresh keys; no other mask, scale 1 / sqrt(hd).  Types and heads
 * as archer_op_attention (hd and Hkv are the cache's).
 *   Q          [Hq][batch G][hd]: G query rows per sequence
 *   O          [batch G][Hq hd]: a row without any key gives zeros, one whose scores are all -infinity NaN
 *   table      device int32 [batch][max_pages]; the keys of an entry outside
 *              [0, n_pages) are left out
 *   cached_len device int32 [batch], >= 0; no more than max_cached (host; sizes the
 *              launch: of more than 32768 it has every sequence's keys looked at for a split,
 *              which short ones pay for) and max_pages * page_size keys are read
 *   K2, Vt2    [Hkv][ld2][hd], [Hkv][hd][ld2], or both NULL: sequence b's fresh keys
 *              are rows b fresh_stride .. + resp_len[b] - 1; ld2 and fresh_stride multiples of
 *              8, fresh_stride >= G, batch fresh_stride <= ld2
 *   resp_len   device int32 [batch] in [0, G], or NULL (G each): the sequence's
 *              query rows and fresh keys; rows of O from resp_len[b] on stay as they are
 * A single token per sequence is G = 1, its key stored beforehand (K2 NULL) or
 * fresh.  Q, K2, Vt2 and O 16-byte aligned.  workspace: device scratch of
 * archer_op_attention_cache4_ws_bytes bytes, 256-byte aligned (NULL if that is
 * 0); calls sharing a workspace must not overlap.  A row's result does not depend on
 * the other sequences' data, but, to rounding, on batch, G, max_cached and the batch's
 * lengths, which choose the kernel and the split of the keys.  fp16: probabilities are
 * rounded to fp16, and where batch and G are large the queries to 2^-18 of the largest of
 * 32 elements, which is less than the fp32 sums of the scores may be off by. */
size_t archer_op_attention_cache4_ws_bytes(int32_t dtype, int32_t batch, int32_t G, int32_t Hq, int32_t Hkv,
                                           int32_t hd, int32_t max_cached, int32_t fresh);
archer_status archer_op_attention_cache4(int32_t dtype, const archer_cache4 *cache, int32_t batch, int32_t G,
                                         int32_t Hq, const void *Q, const int32_t *table, int32_t max_pages,
                                         const int32_t *cached_len, int32_t max_cached, const void *K2,
                                         const void *Vt2, int32_t ld2, int32_t fresh_stride,
                                         const int32_t *resp_len, void *O, void *workspace, size_t ws_bytes,
                                         void *hip_stream);

/* ---- 8-bit paged prompt cache -------------------------------------------------
 * One layer's keys and values in e4m3 (sign, four exponent bits, three mantissa bits, at
 * most 448) with one power-of-two scale per block of 32 tokens and head, for its keys and for its
 * values: 256 bytes per token and head of 128 dimensions, and 16 a page.  Pages, slots and
 * block tables as for the 4-bit cache: plans are archer_cache4_plan's or, for pages that
 * sequences share, archer_pages_plan's.
 *
 * data: device, 16-byte aligned, archer_cache8_bytes bytes, caller-owned.
 * [n_pages][n_kv_heads] blocks of page_size * 2 * head_dim + 16 bytes:
 *   keys    [page_size][head_dim]
 *   values  [page_size / 8][head_dim / 32][16][2][8]   dimension u head_dim / 16 + 2 i + s of
 *           token t of an 8-token block is at [i][u][s][t]
 *   scales  [page_size / 32][2]   exponent + 127 of a block's keys, of its values; then unused
 * page_size 32, 64, 128 or 256; head_dim 64 or 128; n_pages * page_size < 2^31. */
typedef struct {
  void *data;
  int32_t n_pages, page_size, n_kv_heads, head_dim;
} archer_cache8;

/* Bytes of the cache's data (0 and last_error for a bad shape; data is not read). */
size_t archer_cache8_bytes(const archer_cache8 *cache);

/* Store rows of keys and values (fp16 for ARCHER_BF16, fp32 for ARCHER_FP32): rows row_off[b] ..
 * row_off[b + 1] - 1 become the tokens from position start[b] on of sequence b, b < batch, whose
 * pages row b of the block table lists.  A sequence ends with the last row stored: of later tokens
 * in that row's block nothing is kept.
 *   table    device int32 [batch][max_pages]; tokens of an entry outside [0, n_pages), or beyond
 *            the row of the table, are not stored.  A page that is stored to is one sequence's.
 *   start    device int32 [batch], >= 0
 *   row_off  device int32 [batch + 1], rising; rows beyond `rows` (host; sizes the launch) are not stored
 * Element (head, row, d) is at K[head k_head + row k_row + d] and V[head v_head + row v_row + d
 * v_dim] (strides in elements, any sign), with v_dim = 1 or v_row = 1 (else ARCHER_E_UNSUPPORTED; of a
 * single row any v_dim will do).
 * A block's scale is 2^e, e the least integer with max |x| <= 448 * 2^e over its new rows, clamped
 * to [-15, 7]; elements are rounded to the nearest e4m3 value of x / 2^e, ties to the even code, and
 * saturate at 448 * 2^e (57344 at most).  Where a block holds earlier tokens of the sequence e
 * is no less than theirs, and they are rounded once more in the new scale (exact but for elements
 * below 2^-6 * 2^e, less than 2^-13 of the block's largest).  Every stored element is exact in fp16.
 * A NaN stays one. */
archer_status archer_cache8_write(int32_t dtype, const archer_cache8 *cache, int32_t batch, const int32_t *table,
                                  int32_t max_pages, const int32_t *start, const int32_t *row_off, int32_t rows,
                                  const void *K, int64_t k_head, int64_t k_row, const void *V, int64_t v_head,
                                  int64_t v_row, int64_t v_dim, void *hip_stream);

/* The stored elements of the slots slot_map[row], as archer_cache4_read. */
archer_status archer_cache8_read(int32_t dtype, const archer_cache8 *cache, int32_t rows,
                                 const int32_t *slot_map, void *K, void *V, void *hip_stream);

/* archer_op_attention_cache4 over the 8-bit cache: the same arguments, limits and results of rows
 * without keys.  What blocks without a token of the sequence hold does not matter.  fp16:
 * probabilities are rounded to fp16, and nothing else is but the output. */
size_t archer_op_attention_cache8_ws_bytes(int32_t dtype, int32_t batch, int32_t G, int32_t Hq, int32_t Hkv,
                                           int32_t hd, int32_t max_cached, int32_t fresh);
archer_status archer_op_attention_cache8(int32_t dtype, const archer_cache8 *cache, int32_t batch, int32_t G,
                                         int32_t Hq, const void *Q, const int32_t *table, int32_t max_pages,
                                         const int32_t *cached_len, int32_t max_cached, const void *K2,
                                         const void *Vt2, int32_t ld2, int32_t fresh_stride,
                                         const int32_t *resp_len, void *O, void *workspace, size_t ws_bytes,
                                         void *hip_stream);

/* ---- pages that several sequences share ----------------------------------------
 * Block tables, the ring of free pages and slots as in archer_cache4_plan, with a count
 * refs[p] of the table rows that hold page p (device int32 [n_pages]; 0: free): samples of
 * one prompt list its pages, and only what a sample writes is its own.  For any cache
 * of pages (archer_cache4, archer_cache8): one call serves every layer's.  No call
 * synchronises.  Every row holds a page at most once, and counts and tables agree with
 * each other; of that no more is checked than keeps the calls inside their arrays.
 * In-and-out pairs (refs_in, refs_out; table_in, table_out) may be the same array: then
 * the call changes it in place; otherwise they must not overlap, and the call
 * may be repeated with the same result.  Other arrays must not overlap.
 *
 * archer_pages_fork: row dst[i] of the table gets the pages of the first len[i] tokens of row
 * src[i], i < n <= 4096, each page one holder more.  Rows dst held nothing before
 * (archer_pages_plan frees a row); the rest of them stays as it is.
 *   table   [n_rows][max_pages], n_rows <= 65536
 *   status  [1]: 0, or 2 and nothing changed (refs_out = refs_in): a row outside the table, a
 *           length beyond max_pages, a dst twice, or a dst that is a src */
archer_status archer_pages_fork(int32_t n, const int32_t *src, const int32_t *dst, const int32_t *len,
                                int32_t page_size, int32_t n_pages, int32_t n_rows, int32_t max_pages,
                                int32_t *table, const int32_t *refs_in, int32_t *refs_out, int32_t *status,
                                void *hip_stream);

/* archer_cache4_plan for rows that share pages: rows go from len_old[b] to len_new[b] tokens
 * (batch <= 4096), with len_new 0 to the end of their request.
 *   - A row that shrinks drops its last pages, each one holder less.  Those without a holder
 *     left go behind the ring's end, in the order of the last row that drops them.
 *   - A row that grows from inside its last page (len_old no multiple of page_size) writes to
 *     it.  While others hold that page, after this call's drops, the row takes one of its own,
 *     and the page has to be copied to it (archer_pages_copy) before the row's new tokens are
 *     stored.  Where all of a page's holders write, the last of them keeps it.
 *   - Pages are taken from the ring's front in row order, a row's copy first; each has one holder.
 *   pool_in, pool_out, row_off, slot_map, status   as in archer_cache4_plan; slots are those after
 *             the copies.  Status 4 also where a page that is dropped or written to is none of the
 *             pool's.  Of a status other than 0: nothing changed, copies -1.
 *   copy_src, copy_dst [batch]: the page that row b's copy is made of and the new one, or -1
 *   workspace  device scratch of archer_pages_plan_ws_bytes bytes (0 for a bad shape), 256-byte aligned */
size_t archer_pages_plan_ws_bytes(int32_t batch, int32_t n_pages);
archer_status archer_pages_plan(int32_t batch, const int32_t *len_old, const int32_t *len_new, int32_t page_size,
                                int32_t n_pages, int32_t max_pages, const int32_t *table_in, int32_t *table_out,
                                int32_t *free_pages, const int32_t *pool_in, int32_t *pool_out,
                                const int32_t *refs_in, int32_t *refs_out, int32_t *row_off, int32_t *slot_map,
                                int32_t slot_rows, int32_t *copy_src, int32_t *copy_dst, int32_t *status,
                                void *workspace, size_t ws_bytes, void *hip_stream);

/* Moves the pages in use to the front of the pool, so that its end can be given away: with U
 * pages in use, those from U on, in rising order, move to the free ones below U, in
 * rising order.  The tables are rewritten at once; the pages' bytes move with
 * archer_pages_copy(move_src, move_dst, moves), before they are next read.
 *   table     [batch][max_pages]; a row's pages are those of its first len[b] tokens (clamped
 *             to [0, max_pages * page_size]), the other entries stay as they are
 *   free_pages [n_pages], pool_out [2]: the new ring: pages U .. n_pages - 1, then -1; 0 and their number
 *   move_src, move_dst [n_pages / 2]: the moves, then -1; moves [1]: their number
 *   workspace  device scratch of archer_pages_compact_ws_bytes bytes, 256-byte aligned */
size_t archer_pages_compact_ws_bytes(int32_t n_pages);
archer_status archer_pages_compact(int32_t batch, const int32_t *len, int32_t page_size, int32_t n_pages,
                                   int32_t max_pages, const int32_t *table_in, int32_t *table_out,
                                   const int32_t *refs_in, int32_t *refs_out, int32_t *free_pages,
                                   int32_t *pool_out, int32_t *move_src, int32_t *move_dst, int32_t *moves,
                                   void *workspace, size_t ws_bytes, void *hip_stream);

/* Copies page src[i] to page dst[i], i < n (and < *count, device int32, where count is not NULL),
 * in each of n_planes pools (one per layer) plane_stride bytes apart, of n_pages pages of
 * page_bytes bytes, a multiple of 16 (a cache's bytes / n_pages); data 16-byte aligned.  Pairs with
 * an entry outside [0, n_pages) are passed over.  No page may be a dst twice, or both a src and a dst. */
archer_status archer_pages_copy(int64_t page_bytes, int32_t n_pages, int32_t n_planes, int64_t plane_stride,
                                void *data, int32_t n, const int32_t *src, const int32_t *dst,
                                const int32_t *count, void *hip_stream);

/* ---- sampling --------------------------------------------------------------------
 * A token for each row of logits, from given random numbers: what archer_decide's unmasking
 * takes greedily (xhat, and its log-probability) drawn instead.
 *   logits  [rows][vocab] of type dtype (ARCHER_FP32, as a forward gives them, ARCHER_BF16 or
 *           ARCHER_FP16), rows row_stride elements apart (any); vocab <= 524288
 *   exclude a token that is never drawn (MASK), or -1
 *   u       device float [rows], in [0, 1)
 *   temperature, top_k, top_p, min_p   device float, int32, float, float [rows], or NULL: 1, and off
 *   token   device int32 [rows]
 *   logp    device float [rows], or NULL: log-probability of the token in what it was drawn from
 * With z = logit / temperature, w = exp(z - max z) and the tokens ordered by falling logit, equal
 * ones by rising index:
 *   S1  the first top_k tokens (top_k < 1: all)
 *   S2  the shortest prefix of S1 whose weight is at least top_p of S1's (top_p >= 1: S1; <= 0: one token)
 *   S3  the tokens with w >= min_p (min_p <= 0: all)
 * kept are the tokens of S2 that are in S3, and the first token of the order always; the token
 * drawn is the first one by index at which the sum of the kept weights up to it exceeds u times all of
 * it (with rounding at u near 1: the last one of any weight).  A temperature that is not
 * positive takes the first token of the order, with logp 0.  Weights are off by 2^-44 of themselves or
 * 2^-49 of the largest one at most and summed in 64 bits, by fixed orders: a row's result does not depend
 * on the other rows or on the run, but a sum as near as that to a border may fall on either side of it.  A
 * token whose z is more than 33 below the largest may count as one without weight (2^19 of them
 * together: 2^-28.6 of the row's).  Infinite logits share the weight; -infinity has none, every finite
 * value has one, the lowest too.  A row without a token (all -infinity or excluded): token -1, logp
 * -infinity; a row with a NaN: token -1, logp NaN.
 *   workspace  device scratch of archer_op_sample_ws_bytes bytes (0 for a bad shape; 0.3 MB a row, of 1024 rows
 *              at most), 256-byte aligned; nothing in it is kept for another call */
size_t archer_op_sample_ws_bytes(int32_t dtype, int32_t rows, int32_t vocab);
archer_status archer_op_sample(int32_t dtype, int32_t rows, int32_t vocab, const void *logits, int64_t row_stride,
                               int32_t exclude, const float *u, const float *temperature, const int32_t *top_k,
                               const float *top_p, const float *min_p, int32_t *token, float *logp,
                               void *workspace, size_t ws_bytes, void *hip_stream);

/* Kernel classes for timing.  The projection classes _QKV, _O, _GATEUP and
 * _DOWN are the launches of CachedForward passes (M = G per sequence); their
 * _FULL twins are the same projections in FullForward (refresh) passes
 * (M = P_b + G per sequence).  The LM head runs on the response rows in both
 * passes and has one class. */
enum {
  ARCHER_K_EMBED = 0, ARCHER_K_NORM = 1, ARCHER_K_GEMM_QKV = 2,
  ARCHER_K_ATTN = 3 /* attention of CachedForward passes (with its split-KV merge) */,
  ARCHER_K_ATTN_FULL = 4 /* attention of FullForward (refresh) passes */,
  ARCHER_K_GEMM_O = 5, ARCHER_K_GEMM_GATEUP = 6,
  ARCHER_K_GEMM_DOWN = 7, ARCHER_K_GEMM_HEAD = 8, ARCHER_K_DECIDE = 9,
  ARCHER_K_GEMM_QKV_FULL = 10, ARCHER_K_GEMM_O_FULL = 11, ARCHER_K_GEMM_GATEUP_FULL = 12,
  ARCHER_K_GEMM_DOWN_FULL = 13,
  ARCHER_K_COUNT = 14
};

/* Start recording HIP events around launches of the classes in class_mask
 * (bit c = class c) made by this context: the 1st, (every+1)-th, (2 every+1)-th
 * ... launch of each class (every >= 1; 1 = every launch).  Each event pair
 * idles the GPU for a few microseconds, so a stride keeps the measurement from
 * slowing what it measures.  Stops and clears any earlier recording;
 * ARCHER_E_ARG if every < 1. */
archer_status archer_timing_begin(archer_ctx *ctx, uint32_t class_mask, int32_t every);

/* Synchronise, stop recording and return, per class c < ARCHER_K_COUNT:
 * launches[c] (recorded launches), total_ms[c] (sum of their event-bracketed
 * durations) and the algorithmic bytes[c] and flops[c] of those launches
 * (minimum HBM traffic: operands read once and results written once).  Any
 * output may be NULL. */
archer_status archer_timing_end(archer_ctx *ctx, int64_t *launches, double *total_ms,
                                double *bytes, double *flops);

/* Read-only copies of context state, for checking it against a reference
 * (none of these changes the state).  dst: device, caller-owned, >= the
 * stated size in bytes; copies are enqueued on the context's stream.
 *   ARCHER_READ_LOGITS    fp32 [B][G][V]: the logits the session's decoder reads
 *                         (those of the last forward of archer_decode or a session).
 *   ARCHER_READ_HIDDEN    fp32 [n][d]: the final normalised hidden state (the LM
 *                         head's input) of the response rows of the most recent
 *                         forward pass, n = G x (sequences in that pass), in
 *                         ascending sequence order.  bf16 models hold it as a
 *                         two-term pair; the copy is hi + lo (exact in fp32).
 *   ARCHER_READ_RESIDUAL  fp32 [n][d]: the residual stream after the last layer
 *                         for the same rows.
 *   ARCHER_READ_PROMPT_K  [Hkv][P_b][hd] of the cache's element type (fp16 for
 *                         ARCHER_BF16 models, fp32 for ARCHER_FP32): the cached
 *   ARCHER_READ_PROMPT_V  post-RoPE prompt K / prompt V of layer `layer`,
 *                         sequence `seq` -- C_p of Eq. app-cached (App. "Formal
 *                         Analysis"), one layer of it.
 * layer and seq are ignored where they do not apply.  ARCHER_E_STATE before
 * the first forward (or for a sequence without a cache), ARCHER_E_ARG for a
 * short dst or an unknown `what`. */
enum {
  ARCHER_READ_LOGITS = 0, ARCHER_READ_HIDDEN = 1, ARCHER_READ_RESIDUAL = 2,
  ARCHER_READ_PROMPT_K = 3, ARCHER_READ_PROMPT_V = 4
};
archer_status archer_read_state(archer_ctx *ctx, int32_t what, int32_t layer, int32_t seq, void *dst,
                                size_t bytes);

/* Precision of the activation operand of each projection class (bf16 models).
 * By default every projection multiplies a two-term bf16 activation
 * (hi + lo, about 16 significant bits; two MFMAs per fragment), except the
 * gate/up projection of a model with gateup_fp16 (single fp16).  A set bit
 * ARCHER_K_GEMM_QKV, _O, _GATEUP, _DOWN or _HEAD in class_mask makes that
 * class's producer store and its GEMM read the single bf16 rounding hi = bf16(v)
 * instead (half the MFMA work of that projection).  Applies to forwards
 * enqueued after the call.  ARCHER_E_ARG for other bits, ARCHER_E_UNSUPPORTED
 * for a nonzero mask on an fp32 model and for _GATEUP on a model with
 * gateup_fp16 (whose gate/up operands are single fp16 values already). */
archer_status archer_set_single_term(archer_ctx *ctx, uint32_t class_mask);

#ifdef __cplusplus
}
#endif
#endif /* ARCHER_OPS_H */
