/*
 * mstar_cache.h - operators on paged KV caches beside those of mstar_attn.h:
 * a cache held in 4 bits (rows stored, attended, read back) and block tables
 * built on the GPU.  Plans, streams, errors and the sticky device error word
 * are those of mstar_attn.h.
 *
 * The 4-bit cache.  A pool (K or V) is uint8 [num_pages][Hkv][17 * head_dim / 2],
 * 16-byte aligned; a record holds the 16 keys of one page and KV head: 8 *
 * head_dim bytes of codes, then head_dim / 2 scale bytes.
 *
 *   value  = magnitude * 2^(b - 127), negative if bit 3 of the code is set, with
 *            magnitude 0, 0.5, 1, 1.5, 2, 3, 4, 6 by bits 0-2 of the code and
 *            b the scale byte of the key's 32 dims [32 j, 32 j + 32)
 *   K codes  [4][16 keys][head_dim / 8] bytes: piece g of a key holds its dims
 *            [g * head_dim / 4, (g + 1) * head_dim / 4)
 *   V codes  [4 key groups][16][4 keys][head_dim / 32] bytes: piece n of a key
 *            holds its dims [n * head_dim / 16, (n + 1) * head_dim / 16); key t
 *            is key t % 4 of group t / 4
 *   scales   [head_dim / 32][16 keys] bytes
 *
 * with two codes a byte, the lower dim in bits 0-3.  (These are the element
 * and scale formats of OCP microscaling FP4, blocks of 32 along head_dim; the
 * order is that in which a wave's lanes take a page as matrix operands.)
 * Stored rows are rounded as follows: b - 127 is the smallest e with
 * max |x| <= 7 * 2^e over the 32 dims, within [-125, 125]; a code is the nearest
 * one, ties to the even code, so that no value between 2^-126 and 7 * 2^125 is
 * off by more than half a step.  Larger values and infinities take the largest
 * magnitude, NaN is stored as 0, and an infinity or NaN also sets
 * MSTAR_DEVERR_NONFINITE in the plan's error word: attended pages hold finite
 * values only, whatever keys a row may not see.  Scale bytes above 252 (never
 * stored) read as unspecified values.  Attention takes less than can be stored:
 * see mstar_kv4_fwd.
 */
#ifndef MSTAR_CACHE_H
#define MSTAR_CACHE_H

#include "mstar_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Another bit of the sticky device error word (mstar_attn_check). */
#define MSTAR_DEVERR_NONFINITE 2 /* a new key or value was infinite or NaN */

/* Bytes of a record (one page and KV head of a K or V pool) of the 4-bit cache. */
#define MSTAR_KV4_RECORD_BYTES(head_dim) (17 * (head_dim) / 2)

/* mstar_kv_append for a 4-bit cache: the plan's new rows k_new / v_new
 * ([total_q][Hkv][head_dim] bf16, the row numbering of q) are rounded to 4 bits
 * and written to their places in the 4-bit pools k_pages / v_pages.  No other
 * key's codes or scales are written.  Pages, targets outside the pool, stream and
 * capture as for mstar_kv_append; if two new rows target one slot, which they must
 * not, its values are finite and otherwise unspecified (the codes of one may meet
 * the scales of the other).  Errors: INVALID_ARG
 * (null or misaligned pointer, host-only plan, the plan's device is not the
 * current one), UNSUPPORTED (a plan of the fp32 dtype), HIP. */
int mstar_kv4_append(const mstar_plan_t* plan, const void* k_new, const void* v_new, const int32_t* block_table,
                     void* k_pages, void* v_pages, hipStream_t stream);

/* mstar_attn_fwd over a 4-bit cache: the same plan (of the bf16 dtype, cascades
 * included), masks, q, out, lse, workspace, streams and capture, with k_pages /
 * v_pages 4-bit pools.  out and lse are the attention over the values that the
 * cache stands for; scores, softmax statistics and sums are fp32, the
 * probabilities enter the value product in bf16.  That holds for rows whose
 * scores q . k are finite in fp32 and which see values of V up to 2^64 in
 * magnitude, at any length.  Weights are sums of powers relative to an earlier
 * maximum, divided out at the end: with larger values they may overflow, and out
 * of a row that sees one is unspecified (so is that of a row that sees a stored
 * infinity, of largest magnitude).  Rows that do not see it are not touched by
 * it.  Errors as mstar_attn_fwd, plus UNSUPPORTED (a plan of the fp32 dtype) and
 * INVALID_ARG (the plan's device is not the current one). */
int mstar_kv4_fwd(const mstar_plan_t* plan, const void* q, const void* k_pages, const void* v_pages,
                  const int32_t* block_table, void* out, float* lse, void* workspace, size_t workspace_bytes,
                  hipStream_t stream);

/* mstar_attn_fwd_noalloc over a 4-bit cache: the partials go to the library's
 * static device array, which all such calls on a GPU (and those of
 * mstar_attn_fwd_noalloc) share, so that no two of them may overlap in time. */
int mstar_kv4_fwd_noalloc(const mstar_plan_t* plan, const void* q, const void* k_pages, const void* v_pages,
                          const int32_t* block_table, void* out, float* lse, hipStream_t stream);

/* Pages of a 4-bit cache back as 16-bit ones: page page_ids[i] (device memory,
 * int32) of the pools k_pages / v_pages goes to k_out / v_out [i][16][Hkv][head_dim]
 * in bf16, exactly (every stored value is a bf16 value).  A page index outside
 * [0, num_pages) gives a page of zeros.  For contexts that move to a 16-bit pool,
 * or whose rows are read outside attention.  num_ids may be 0.  Enqueued on
 * `stream` with no allocation and no host synchronisation; may be captured.
 * Errors: INVALID_ARG (null or misaligned pointer, counts below 0 or, for heads
 * and pages, below 1), UNSUPPORTED (head_dim), HIP. */
int mstar_kv4_unpack(int32_t num_kv_heads, int32_t head_dim, int32_t num_pages, const void* k_pages,
                     const void* v_pages, const int32_t* page_ids, int32_t num_ids, void* k_out, void* v_out,
                     hipStream_t stream);

/* Pages that the plan's new rows start: the sum over requests of
 * ceil(kv_len / 16) - ceil((kv_len - q_len) / 16).  0 for a NULL plan. */
int64_t mstar_block_tables_pages(const mstar_plan_t* plan);

/* The step's block tables and slot map on the GPU (any plan dtype): every
 * request's new rows that start a page take one from free_pages (device memory,
 * int32 page indices), the plan's requests in order and each one's pages in
 * order (free_pages[0 .. mstar_block_tables_pages(plan)) in all), which is written
 * to the request's entry (position / 16) of block_table ([num_seqs][max_blocks_per_seq] int32).  No
 * other entry is written: those of cached positions are the caller's.  slots, if
 * not NULL, is [total_q] int64: the entry of every new row becomes its flat slot,
 * page * 16 + position % 16 (entries of rows of no request are left as they
 * are).  A page outside [0, num_pages), taken or found in the table, gives slot
 * -1 and sets MSTAR_DEVERR_PAGE_RANGE; one that was taken is entered as -1.
 * Enqueued on `stream` with no allocation and no host synchronisation; may be
 * captured.  mstar_kv_append, mstar_kv4_append and the attention calls on the
 * same stream afterwards see the table.  Errors: INVALID_ARG (null pointer,
 * fewer free pages than the plan needs, host-only plan, the plan's device is not
 * the current one), HIP. */
int mstar_block_tables(const mstar_plan_t* plan, const int32_t* free_pages, int64_t num_free, int32_t* block_table,
                       int64_t* slots, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* MSTAR_CACHE_H */
