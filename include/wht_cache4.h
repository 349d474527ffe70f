/*
 * wht_cache4.h -- serving attention over a paged cache held in 4 bits.
 *
 * Beside the caches of wht_attention.h, which hold keys and values in the tensors' type: a cache of about a quarter of their
 * size, the attention that reads it, and the eviction of the keys that have received the least weight.
 *
 *   wht_kv_append4       rotates new queries and keys by their positions, quantises keys and values and writes them
 *   wht_kv_read4         the rows that the cache holds at given slots
 *   wht_attn_paged4      attention of each sequence's tokens to its own pages; if asked, the weight that each key receives
 *   wht_kv_evict4        moves what is to stay of each sequence into pages of its own
 *
 * A row x of D channels (of one key head: a key after its rotation, or a value) is held as
 *     lo = bf16(min x),  step = bf16((max x - lo) * fl(1/15)),  code_i = clamp(rint((x_i - lo) * fl(1/step)), 0, 15)
 * and stands for lo + step * code_i; a step below 2^-100 counts as 0 and makes all codes 0.  Every operation is fp32,
 * rounded on its own, so that the cache is a function of the inputs alone.  A channel is held to half a step or to 2^-8 of |min x| (lo is a bf16 number), whichever
 * is more: rows whose offset is far above their spread keep little of it.  A row that holds a NaN or an infinity, or whose spread
 * passes fp32, stands for NaN.
 *
 * Conventions are those of wht_attention.h (device pointers, 16-byte aligned; streams; status codes; D in {64, 96, 128}, pages of 16, 32, 64 or
 * 128 keys, up to 64 query heads per key head), and wht_attn_device_status() covers these kernels too.
 *   - cache: [num_pages x Hkv x page / 16 x (16 D + 128)] bytes, contiguous: per 16 keys the codes of the keys, the codes of the
 *     values, and for each key step and lo of the key, step and lo of the value (bf16).  The order of the codes is the library's own
 *     (csrc/cache4_common.cuh states it).  It has no storage type: queries and outputs of a call are WHT_F32 or WHT_BF16.
 *     Fresh memory may hold anything.
 *   - Scores, softmax statistics and the weights' sums are fp32, long sums in pieces.  Products are summed by the tensor core, which truncates as it adds: those of a score over its
 *     channels, to about 20 bits; those of the output over 1024 keys at most (4096 in the tcgen05 kernel), whose sums are then added in fp32 with rounding.  Queries enter the product as fp16 numbers shifted by a power of two per row: bf16 ones
 *     keep all bits but those below 2^-33 of the row's largest, fp32 ones are two terms (22 bits).  The softmax weights, times the values' steps and a power
 *     of two per row, enter the second product as one fp16 term (11 bits) where the output is bf16 and as two (22 bits) where it is fp32.
 *     Queries of 2^116 and more (divided by the scale, where that is above 1) may come out as NaN.  Long prompts of bf16 queries over long contexts take a
 *     tcgen05 kernel, by sizes that the host knows; there queries enter as they are, and the weights as one fp16 term.
 *   - The work is divided by the lengths themselves, so that a table wider than its sequences costs the attention of single tokens and short prompts nothing but its
 *     memory.  The width counts in three places: the received weight is written (and zeros behind the lengths) over all of it, in pieces whose size follows it; the workspace for its
 *     scores grows with it; and for bf16 prompts of more than 16 rows a sequence and key head the choice of kernel takes the tables as full, so that short contexts in
 *     wide tables go to the tcgen05 kernel although the other one is faster, and the last bits of a result depend on the table's width.
 */
#ifndef WHT_CACHE4_H_
#define WHT_CACHE4_H_

#include "wht_attention.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Append: the arguments are those of wht_kv_append (strides, slots, positions, tables), without summaries.  No two tokens of a call share a slot. */
int wht_kv_append4(const void* k, int64_t k_stride_t, int64_t k_stride_h,
                   const void* v, int64_t v_stride_t, int64_t v_stride_h,
                   const void* q, int64_t q_stride_t, int64_t q_stride_h, void* q_out,
                   const int64_t* slots, const int32_t* positions, const float* cos_table, const float* sin_table,
                   void* cache, int64_t T, int32_t Hq, int32_t Hkv, int32_t D, int32_t rot, int32_t interleaved, int64_t max_pos,
                   int64_t num_pages, int32_t page, int dtype, void* stream);

/* k_out, v_out [n x Hkv x D] of `dtype`: lo + step * code of the rows at slots [n] (fp32: product and sum rounded; bf16: rounded once); zeros where a slot is
 * negative. */
int wht_kv_read4(const void* cache, const int64_t* slots, void* k_out, void* v_out, int64_t n, int32_t Hkv, int32_t D,
                 int64_t num_pages, int32_t page, int dtype, void* stream);

/*
 * Attention: token t of sequence b sees the keys 0 .. (kv_lens[b] - n_b + i), the i-th of the sequence's n_b tokens in this call.  Arguments as for
 * wht_attn_prefix without a prefix.
 *   weights      [B x Hkv x table_width * page] float32 or NULL: what each key has received so far (NULL: nothing).
 *   weights_out  the same shape, or NULL: weights + the softmax weights of this call's tokens and the query heads of the key
 *                head, summed; 0 from kv_lens[b] on.  May be `weights` itself.  Sums have one order: results repeat bit for bit.
 *                Queries may be read again for it, after `out` has been written: `out` does not overlap them.
 *   workspace    at least wht_attn_paged4_workspace_bytes(...) bytes; weigh: whether weights_out is given (the scores of up to 8 rows a sequence and key head
 *                are then kept for it, in 1 GiB at most; beyond that they are taken again).  It holds nothing between calls; calls that may run at the same time
 *                need one each.
 * Lengths, offsets and tables are read by several kernels of a call: they must not change before it has ended.
 */
int wht_attn_paged4(const void* q, int64_t q_stride_t, int64_t q_stride_h, const void* cache,
                    const int32_t* page_table, int32_t table_width, const int32_t* kv_lens, const int32_t* q_start, void* out,
                    const float* weights, float* weights_out,
                    int64_t T, int32_t B, int32_t max_q_len, int32_t Hq, int32_t Hkv, int32_t D,
                    int64_t num_pages, int32_t page, float scale, int dtype, void* workspace, size_t workspace_bytes, void* stream);
size_t wht_attn_paged4_workspace_bytes(int32_t table_width, int64_t T, int32_t B, int32_t max_q_len, int32_t Hq, int32_t Hkv,
                                       int32_t D, int32_t page, int dtype, int32_t weigh);

/*
 * Eviction: of each sequence's n = kv_lens[b] keys, min(n, budget) stay per key head: the first keep_first, the last keep_last, and of
 * those between the ones of the largest weight, ties to the lowest key (a NaN counts as the least weight, -0 as 0).  They move, in their order, into
 * the pages of out_table [B x out_width], which no sequence of the call reads: its own pages are left as they are, and so are the rows of the new
 * pages behind the last key moved.
 *   weights      [B x Hkv x table_width * page]; table_width * page up to 2^30.
 *   weights_out  [B x Hkv x out_width * page]: the weights of what stays, then zeros.
 *   lens_out [B] int32: min(n, budget); kept [B x Hkv x budget] int32: which keys stayed, ascending, then -1.
 *   budget >= 1, keep_first + keep_last <= budget <= out_width * page.
 */
int wht_kv_evict4(void* cache, const int32_t* page_table, int32_t table_width, const int32_t* kv_lens, const float* weights,
                  const int32_t* out_table, int32_t out_width, int32_t* lens_out, float* weights_out, int32_t* kept,
                  int32_t B, int32_t Hkv, int32_t D, int64_t num_pages, int32_t page,
                  int32_t budget, int32_t keep_first, int32_t keep_last, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* WHT_CACHE4_H_ */
