/*
 * treespark_kv.h -- the target's 4-bit key-value cache around the draft tree
 * (C ABI, same library and conventions as treespark.h).
 *
 * A round of speculative decoding has the target verify a tree of rows per
 * request in one pass (§3.2 item 3).  In that pass every layer needs a place
 * for each row's key and value, writes them there, and attends over the
 * request's context and the row's ancestors; after ts_verify the accepted
 * path's rows stay and the others go:
 *   ts_kv_plan       pages for each request's rows, block tables and slots
 *   ts_kv_append     keys and values into the cache, in 4 bits
 *   ts_kv_attention  attention over context and tree under ts_tree_mask's mask
 *   ts_kv_accept     the accepted path's rows moved behind the context
 *   ts_kv_read       rows of the cache back as numbers
 *
 * Positions.  A request's cache holds its tokens at positions 0, 1, ...:
 * len[q] tokens of context, then the rows of this round: row i (node i of the
 * tree, the root first) at position len[q] + i.  Position t lies in block
 * t / page_size of the request's block table, at offset t % page_size of that
 * page.  A slot is page * page_size + offset.
 * n[q] counts rows as ts_tree does: nodes without the root, so n[q] + 1 rows;
 * n[q] < 0 means no rows (a request that sits this round out) and
 * n[q] >= cap is read as cap - 1.  len[q] < 0 is read as 0.
 * A prompt is a chain: rows 0..n of it, without a mask.
 *
 * Format.  The cache is bytes: a block per (layer, page, kv head) at
 *   pages + layer * layer_stride + page * page_stride
 *         + head * ts_kv_block_bytes(page_size, head_dim)
 * and in it, for a page of P tokens and D values a head,
 *   key codes [P][D/2], key scales [P][D/32], value codes [P][D/2], value scales [P][D/32].
 * Codes are E2M1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives by bit 3):
 * element d of a token in byte d / 2, the low half for even d.  A scale byte s
 * covers 32 elements and stands for 2^(s - 127).  Key scale 255 makes its 32
 * keys not-a-number; a value scale of 255 reads as zero values, and attention
 * reads value scales 253 and 254, which ts_kv_append never writes, as 252.
 */
#ifndef TREESPARK_KV_H
#define TREESPARK_KV_H

#include "treespark.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A cache (pages: DEVICE memory, 16-byte aligned; strides in bytes, multiples
 * of 16, in either nesting order of layers and pages).  page_size is one of 16,
 * 32, 64, 128, 256, head_dim one of 64, 128, 256; num_pages * page_size < 2^31. */
typedef struct {
  void* pages;
  int64_t layer_stride, page_stride;
  int32_t layers, num_pages, page_size, heads, head_dim;
} ts_kv_cache;

/* Largest number of rows per request without a mask (with one: TS_MAX_CAP). */
#define TS_KV_MAX_CAP (1 << 20)

/* Bytes of one (layer, page, head) block: page_size * head_dim * 17 / 16 (0 for
 * sizes that ts_kv_cache does not allow). */
size_t ts_kv_block_bytes(int32_t page_size, int32_t head_dim);

/*
 * ts_kv_plan: the pages, block tables and slots of a round, from the requests'
 * lengths, on the GPU.  Request q needs ceil((len[q] + n[q] + 1) / page_size)
 * pages (ceil(len[q] / page_size) for n[q] < 0; with len[q] = 0 too, a request
 * gives all its pages back).
 *   1. Pages that a request holds beyond its need go back on the free stack:
 *      its table's last blocks, so that the first of them, of the first
 *      request, comes to lie on top.  Their table entries become -1.
 *   2. Requests in the order of q take the pages they lack from the top of the
 *      stack, each all of them or none: a request whose lack, with what those
 *      before it lack, exceeds the stack gets none.  So does one that needs more
 *      than max_blocks (whose lack does not count for the others).
 * Giving back at once what was just taken restores the stack.
 *   len [R], n [R]: DEVICE inputs;
 *   free_pages [num_pages], free_count [1], held [R] (pages each request
 *       holds), table [R][max_blocks]: DEVICE, read and updated;
 *   slot [R][cap] (may be NULL): DEVICE output, fully written: the slot of row
 *       i, -1 for rows past the request's;
 *   granted [R]: DEVICE output: n[q] (at most cap - 1), or -1 where n[q] < 0 or
 *       the request got no pages, which then keeps what it held.
 * Start a pool with free_count = num_pages, the page ids in free_pages, held
 * all 0 and table all -1.  Counts outside their range are read as the nearest
 * in it, and a page id outside [0, num_pages) gives slot -1.  len, n and the
 * other arrays must not overlap.  Asynchronous on `stream`.  Host checks: null
 * pointers, 0 <= R <= 65536, 1 <= cap <= TS_KV_MAX_CAP, page_size, num_pages
 * >= 1 with num_pages * page_size < 2^31, max_blocks >= 1 with R * max_blocks +
 * num_pages, R * cap < 2^31 and max_blocks * page_size <= 2^30.
 */
int32_t ts_kv_plan(const int32_t* len, const int32_t* n, int32_t R, int32_t cap, int32_t page_size,
                   int32_t num_pages, int32_t max_blocks, int32_t* free_pages, int32_t* free_count,
                   int32_t* held, int32_t* table, int32_t* slot, int32_t* granted, void* stream);

/*
 * ts_kv_append: write rows' keys and values into a layer of the cache.  k and
 * v are DEVICE [rows][heads][head_dim] of dtype (ts_dtype), k_stride and
 * v_stride elements from a row to the next (so that both may lie in one
 * projection's output), 16-byte aligned with strides of whole 16 bytes.
 * slot [rows] (DEVICE, ts_kv_plan's): rows with a slot outside [0, num_pages *
 * page_size) are skipped and not read; no two rows may have the same slot
 * (which row's bytes stay is then open).
 * Of each 32 values with largest magnitude m the scale is the least power of
 * two 2^(s-127) with m <= 7 * 2^(s-127), s in [2, 252], so that no value is
 * further off than half the format's widest step; the codes are the nearest
 * values (ties to the even code), at most 6 scales.  Where a key or a value of
 * a (row, head) holds a NaN or an infinity, all its key scales are 255 and its
 * values zero: rows that attend to it give NaN, others are not touched by it.
 * Asynchronous on `stream`.  Host checks: the cache, null pointers, layer,
 * dtype, rows >= 0 with rows * heads * head_dim <= 2^34, strides, alignment.
 */
int32_t ts_kv_append(const ts_kv_cache* cache, int32_t layer, const void* k, const void* v, int32_t dtype,
                     int64_t k_stride, int64_t v_stride, const int32_t* slot, int32_t rows, void* stream);

/*
 * ts_kv_read: rows of the cache back as numbers, for `layers` layers from
 * `layer` on: k, v (either may be NULL) DEVICE [layers][rows][heads][head_dim]
 * of dtype, 16-byte aligned, exact in both dtypes.  Rows with a slot outside
 * [0, num_pages * page_size) are left as they were.  Asynchronous on `stream`.
 * Host checks as ts_kv_append's.
 */
int32_t ts_kv_read(const ts_kv_cache* cache, int32_t layer, int32_t layers, const int32_t* slot, int32_t rows,
                   void* k, void* v, int32_t dtype, void* stream);

/* Bytes of device workspace ts_kv_attention needs (0 for sizes it refuses): a
 * partial result per workgroup that the device can hold at a time, whatever
 * the lengths. */
size_t ts_kv_attention_workspace_size(const ts_kv_cache* cache, int32_t R, int32_t cap, int32_t q_heads,
                                      int32_t dtype);

/*
 * ts_kv_attention: for every request q, row i <= n[q] and query head a,
 *   out = sum_t w_t V_t / sum_t w_t,  w_t = exp(scale * <Q, K_t> - max),
 * over the positions t that row i sees: the context t < len[q] and, of this
 * round's rows, t = len[q] + j with bit j of row i of the mask set, or with j <= i
 * where mask is NULL (a chain: plain decoding, a prompt).  The tokens, K and V
 * are those of kv head a / (q_heads / heads).  A row that sees nothing gets 0
 * and log-sum-exp -inf.
 *   q: DEVICE [R][cap][q_heads][head_dim] of dtype, q_stride elements from a
 *      row to the next, 16-byte aligned, rows of whole 16 bytes;
 *   len, n [R], table [R][max_blocks]: DEVICE (n: ts_kv_plan's granted).  A
 *      position whose block lies past max_blocks or whose page id is outside
 *      [0, num_pages) reads as not-a-number; nothing outside is read;
 *   mask: DEVICE [R][cap][ts_tree_mask_words(cap)] as ts_tree_mask writes it
 *      (bits past row n[q] do not count), or NULL;
 *   scale: below 2^127 in magnitude (usually head_dim^-0.5).  <Q, K_t> is an fp32
 *      number and so is the score: what passes 2^128 is infinite (or, where sums
 *      of both signs pass it, not-a-number).  A score of -inf has weight 0, and a row
 *      of no other sees nothing; one of +inf makes its row not-a-number;
 *   out: DEVICE [R][cap][q_heads][head_dim] of dtype, 16-byte aligned; lse (may
 *      be NULL): DEVICE float [R][cap][q_heads], log sum_t exp(scale <Q, K_t>).
 *      Rows past n[q] of both are left as they were.  Neither may overlap an
 *      input.
 * Scores, softmax statistics and sums are held in fp32; weights are taken against a
 * maximum that may lag by 2^12, so values near 2^116 over the number of tokens can
 * overflow their sum.  With TS_F32 nothing is
 * rounded below that.  With TS_BF16
 *   - a query's elements are held to 2^-18 of its head's largest, and the matrix unit
 *     that multiplies 4-bit keys cuts off what is small beside the largest of eight
 *     neighbouring products, less than 7 * 2^-17 of that: a score is off by at most
 *     scale * (2^-14 sum |Q| |K_t| + 2^-18 max |Q| sum |K_t|), usually far less;
 *   - a weight w_t is rounded to bf16 before it multiplies a value, and out is
 *     divided by the sum of the rounded weights; lse is that of the unrounded ones.
 * A call's result does not depend on what else the device runs: the same call on
 * the same device gives the same bits.  Asynchronous on `stream`; workspace: DEVICE, 16-byte
 * aligned, of at least ts_kv_attention_workspace_size bytes, not shared by
 * calls that may overlap.
 * Host checks: the cache, null pointers, layer, dtype, q_heads a multiple of
 * heads and at most 256 times them, 0 <= R <= 65536, 1 <= cap <= TS_MAX_CAP
 * (TS_KV_MAX_CAP without a mask), R * cap * q_heads < 2^31, max_blocks, strides,
 * alignment, scale, out not q, workspace.
 */
int32_t ts_kv_attention(const ts_kv_cache* cache, int32_t layer, const void* q, int32_t dtype, int64_t q_stride,
                        int32_t q_heads, const int32_t* len, const int32_t* n, int32_t R, int32_t cap,
                        const int32_t* table, int32_t max_blocks, const uint32_t* mask, float scale, void* out,
                        float* lse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * ts_kv_accept: keep the accepted path of ts_verify.  In every layer and head
 * of the cache the key and value of row path_nodes[q][j] move to position
 * len[q] + 1 + j, for j < path_len[q]; the root's row already lies at len[q].
 * new_len[q] = len[q] + 1 + path_len[q] is the request's context of the next
 * round (which starts with the bonus token as its root); ts_kv_plan then takes
 * back the pages it no longer needs.
 *   len, n [R], table [R][max_blocks], path_nodes [R][TS_MAX_D], path_len [R]:
 *      DEVICE (ts_verify's results, copied to the device); new_len [R]: DEVICE
 *      output, none of the inputs.
 * n[q] < 0 or path_len[q] < 0: the request keeps len[q].  A path stops before a
 * node that is not larger than the one before it, larger than n[q], or whose
 * place lies in no page; path_len[q] > TS_MAX_D is read as TS_MAX_D.
 * Asynchronous on `stream`.  Host checks: the cache, null pointers, 0 <= R <=
 * 65536, max_blocks, new_len.
 */
int32_t ts_kv_accept(const ts_kv_cache* cache, const int32_t* len, const int32_t* n, int32_t R,
                     const int32_t* table, int32_t max_blocks, const int32_t* path_nodes,
                     const int32_t* path_len, int32_t* new_len, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* TREESPARK_KV_H */
