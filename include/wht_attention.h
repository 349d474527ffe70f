/*
 * wht_attention.h -- serving attention that feeds the Walsh-Hadamard head mixing of wht_affine.h.
 *
 * The head mixing takes the concatenated head outputs [T x (Hq*D)] of an attention block.  In serving these
 * come from queries that attend to a paged cache of keys and values; this header has the three operators
 * around that cache:
 *
 *   wht_kv_append      rotates new queries and keys by their positions and writes keys and values into the
 *                      cache; keeps, if asked, a small summary of each page's keys
 *   wht_attn_prefix    attention of a batch whose sequences share a prefix (computed once for all of them)
 *                      and go on with pages of their own
 *   wht_attn_select    attention of each query to the few pages that a whole-number score over the pages'
 *                      summaries selects for it
 *
 * Conventions
 *   - Tensor pointers are DEVICE pointers owned by the caller, 16-byte aligned.  Calls enqueue work on
 *     `stream` (a cudaStream_t as void*, NULL = default stream) and return without synchronising; they never
 *     allocate.  Status codes, wht_affine_last_cuda_error() and wht_affine_status_string() are those of
 *     wht_affine.h; no exception crosses this boundary and no kernel traps.
 *   - Storage types: WHT_F32 (queries, keys, values, caches, outputs float32) or WHT_BF16 (all bfloat16).
 *     Scores, softmax statistics and sums are fp32 whatever the type.  On bf16 tensors the softmax weights
 *     enter the product with the values as two bf16 terms (16 significant bits; the tensor core takes both operands
 *     in one type), as one (8 bits, the softmax sum taken of the same terms) where 33 and more rows of a key head share a prefix
 *     of 256 and more keys and that product is what the time goes to; on fp32 tensors both products take each operand as
 *     two terms, about 21 significant bits.
 *   - Caches: k_cache, v_cache [num_pages x Hkv x page x D], contiguous.  page in {16, 32, 64, 128}; D in
 *     {64, 96, 128}; Hq = G*Hkv query heads, head h reading key head h / G, G <= 64.
 *   - Slots, page numbers, lengths and query offsets are read on the device.  A page number or slot outside
 *     the cache, or a position outside the table, is never used as an address: nothing is written for such a slot, page 0
 *     is read for such a page, positions, lengths and offsets are clamped, and the device status word is set;
 *     wht_attn_device_status() then reports WHT_ERR_DEVICE_INDEX, and the call's outputs are invalid.
 *   - Lengths being on the device, the division of the work goes by table_width: with a table much wider than its sequences
 *     a call is right but can take several times as long as with one that is as wide as the longest of them.
 *   - Rows that see no key (a length of zero) get zeros.  So do rows of tokens that no sequence covers (before q_start[0], from q_start[B]
 *     on); these are reported like an index out of range, and their entries of pages_out are -1.
 *   - Cache entries that a row does not see (beyond a sequence's length, at the places of later tokens) never
 *     reach its result, whatever they hold (NaN and infinities included).  An infinity among the values that it does see
 *     may come out as NaN, in that channel.
 *   - In a -DWHT_DEBUG build these calls run as they do otherwise, without guarded buffers.
 */
#ifndef WHT_ATTENTION_H_
#define WHT_ATTENTION_H_

#include "wht_affine.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Append with the position rotation.
 *   k, v     [T x Hkv x D], q [T x Hq x D] or NULL: element strides *_stride_t between tokens and *_stride_h
 *            between heads (multiples of 16 bytes where there are several; channels contiguous), so slices of a fused projection serve as they are.
 *   q_out    [T x Hq x D] contiguous; may be q itself if that is contiguous; NULL exactly when q is NULL.
 *   slots    [T] int64: page * page_size + place in the page; negative = the token is padding, its keys and
 *            values are dropped (its query is still rotated; without q its position is not looked at).
 *   positions[T] int32, cos_table, sin_table [max_pos x rot/2] float32.  rot: how many leading channels turn,
 *            a multiple of 16 up to D; 0 = none (positions and tables may be NULL).  Channel pairs are (i, i + rot/2), or
 *            (2i, 2i + 1) with interleaved = 1.  Each product and each sum is rounded to fp32 on its own and the
 *            result once to the storage type: the cache does not depend on how a compiler contracts them.
 *   summary  [num_pages x Hkv x 2 x D] int8 or NULL: per page, head and channel the least (index 0) and the largest
 *            (index 1) value of c(k) over the page's tokens, c(k) = clamp(rint(k * summary_scale[head]), -127, 127)
 *            of the stored key.  A token at place 0 starts its page's summary anew, others join the one
 *            that is there.  With a summary, tokens that go to one page in one call stand next to each other, in
 *            ascending order of their slots (as they do in any prompt or step); no two tokens share a slot.
 */
int wht_kv_append(const void* k, int64_t k_stride_t, int64_t k_stride_h,
                  const void* v, int64_t v_stride_t, int64_t v_stride_h,
                  const void* q, int64_t q_stride_t, int64_t q_stride_h, void* q_out,
                  const int64_t* slots, const int32_t* positions, const float* cos_table, const float* sin_table,
                  void* k_cache, void* v_cache, int8_t* summary, const float* summary_scale,
                  int64_t T, int32_t Hq, int32_t Hkv, int32_t D, int32_t rot, int32_t interleaved, int64_t max_pos,
                  int64_t num_pages, int32_t page, int dtype, void* stream);

/*
 * Attention behind a shared prefix.  Token t of sequence b sees all prefix_len prefix keys and the keys
 * 0 .. (kv_lens[b] - n_b + i) of its own pages, where it is the i-th of the sequence's n_b tokens in this call (its own
 * keys have been appended before):   out[t, h] = sum_j softmax_j(scale * q[t, h] . k_j) v_j.
 *   q [T x Hq x D] with strides as above; out [T x Hq x D] contiguous (rows of the head mixing).
 *   prefix_pages [ceil(prefix_len / page)] int32 (may be NULL when prefix_len == 0).
 *   page_table   [B x table_width] int32: a sequence's own pages in order (at most 2^31 - 256 keys; entries beyond its length are
 *                not looked at); kv_lens [B] int32: its own keys.  B >= 1 where T > 0.
 *   q_start      [B + 1] int32: sequence b's tokens are q_start[b] .. q_start[b+1]-1, at most max_q_len of them;
 *                NULL = one token per sequence (T == B).
 *   workspace    at least wht_attn_prefix_workspace_bytes(...) bytes of device memory, 16-byte aligned.
 * The prefix is read once for the whole batch: every row of the batch that shares a key head is a row of one product.
 */
int wht_attn_prefix(const void* q, int64_t q_stride_t, int64_t q_stride_h, const void* k_cache, const void* v_cache,
                    const int32_t* prefix_pages, int64_t prefix_len, const int32_t* page_table, int32_t table_width,
                    const int32_t* kv_lens, const int32_t* q_start, void* out,
                    int64_t T, int32_t B, int32_t max_q_len, int32_t Hq, int32_t Hkv, int32_t D,
                    int64_t num_pages, int32_t page, float scale, int dtype,
                    void* workspace, size_t workspace_bytes, void* stream);
size_t wht_attn_prefix_workspace_bytes(int64_t prefix_len, int32_t table_width, int64_t T, int32_t B, int32_t max_q_len,
                                       int32_t Hq, int32_t Hkv, int32_t D, int32_t page, int dtype);

/*
 * Attention over selected pages.  A token at place p of its sequence (places as above, no prefix) always reads its own
 * page p / page, and before it the select - 1 pages of the highest score, ties to the lowest page:
 *     q8[h, :] = rint(q[h, :] * (127 * (1 / max |q|))),  the maximum over the G heads of a key head; reciprocal and products
 *                each rounded to fp32; 0 where the maximum is below 1e-30
 *     score    = sum over the G heads and the channels of max(q8 * summary_min, q8 * summary_max)
 * -- an upper bound of what any key of the page can score, in whole numbers, so that the selection does not depend on
 * the order of a sum.  The G heads of a key head read the same pages.  Keys after p are not seen.
 *   select       pages per query and key head, 1 .. 1024.
 *   table_width  up to 49152 (a row's scores are picked from in shared memory).
 *   pages_out    [T x Hkv x select] int32: the pages read (index in the sequence), ascending, then -1.
 *   workspace    at least wht_attn_select_workspace_bytes(...) bytes.
 */
int wht_attn_select(const void* q, int64_t q_stride_t, int64_t q_stride_h, const void* k_cache, const void* v_cache,
                    const int8_t* summary, const int32_t* page_table, int32_t table_width, const int32_t* kv_lens,
                    const int32_t* q_start, int32_t select, void* out, int32_t* pages_out,
                    int64_t T, int32_t B, int32_t max_q_len, int32_t Hq, int32_t Hkv, int32_t D,
                    int64_t num_pages, int32_t page, float scale, int dtype,
                    void* workspace, size_t workspace_bytes, void* stream);
size_t wht_attn_select_workspace_bytes(int32_t table_width, int32_t select, int64_t T, int32_t B, int32_t max_q_len,
                                       int32_t Hq, int32_t Hkv, int32_t D, int32_t page, int dtype);

/*
 * Synchronises with the current device and reports what the kernels of this header recorded since the last query:
 * WHT_ERR_DEVICE_INDEX (a page number, slot, position or length out of range), WHT_ERR_DEVICE_WAIT (a bounded wait
 * expired; never expected), else WHT_OK.  Clears the record (what another thread's call records meanwhile may go with it).
 */
int wht_attn_device_status(void);

#ifdef __cplusplus
}
#endif
#endif /* WHT_ATTENTION_H_ */
