/*
 * b200kv -- an INT8 key/value cache for transformer inference on one NVIDIA B200
 * (sm_100a), and attention over it.  Part of libb200gemm.so; return codes,
 * streams, threads and the device status word are those of b200gemm.h.
 *
 * Cache.  Pages of `page_size` tokens.  K and V are int8 arrays
 *     [num_pages][kv_heads][page_size][head_dim]
 * and each (page, head) has one FP32 scale for K and one for V ([num_pages][kv_heads]):
 * the value of a code is code * scale.  The caller owns all four arrays and
 * hands pages to sequences through a block table, int32 [batch][table_stride]:
 * entry (b, j) is the page that holds tokens [j * page_size, (j+1) * page_size) of
 * sequence b.  Entries beyond a sequence's length are never read, nor by attention those of
 * pages that lie in front of every query's window.  Different
 * sequences may share pages that neither of them writes.
 *
 * Batches are ragged: sequence b has the rows cu[b] .. cu[b+1]-1 of a packed
 * [tokens][heads][head_dim] array (cu: int32 [batch+1], device memory, starting
 * at 0, not decreasing); zero rows are allowed.
 *
 * page_size: 16, 32, 64 or 128.  head_dim: 64, 128 or 256.  Positions and lengths
 * are 32-bit, addresses inside the cache 64-bit.  Code, scale and table arrays
 * 16-, 4- and 4-byte aligned; FP16 inputs and outputs 16-byte aligned with strides that
 * are multiples of 8 elements.
 *
 * Lengths, counts and table entries are read on the device.  An entry outside
 * [0, num_pages), a length that the table cannot hold, or a row outside the packed
 * arrays is not followed: nothing outside the arrays is read or written, the status
 * word (gemm_last_device_status, gemm_read_device_status) reads 6 afterwards, and what
 * the call gives for that sequence is undefined.  The library knows how many rows the packed
 * arrays have from the entry points' forms ..._rows, whose last argument before the
 * stream is that number; the forms without it take cu at its word: the caller
 * vouches that cu[batch] rows are there.
 */
#ifndef B200KV_H_
#define B200KV_H_

#include "b200gemm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct kv_cache_s8 {
  int8_t* k;
  int8_t* v;
  float* k_scale;
  float* v_scale;
  int num_pages;
  int kv_heads;
  int page_size;
  int head_dim;
} kv_cache_s8_t;

/*
 * Writes new tokens: row cu[b] + i of K and V becomes token past[b] + i of
 * sequence b, quantised with its page's scale.  Per page and head, with s0 the scale of
 * the tokens the page already held (positions below past[b]; a page that held none starts
 * afresh),
 *     s = max(s0, max |x| / 127) over the new tokens x of the page,
 *     code(x) = rint(x * (1 / s)),   older codes q -> rint(q * (s0 * (1 / s)))
 * in FP32, ties to even; s = 0 (all zeros) gives codes 0.  Values that are not
 * finite make their page's scale, and so every value read from it, not finite.
 * K, V: binary16, element (row, head, d) at row * token_stride + head * head_stride + d.
 * max_new: an upper bound of the tokens any sequence adds (sequences with more are cut
 * there, status 6).
 */
int kv_append_s8(const kv_cache_s8_t* cache, int batch, const int* cu, const int* past,
                 const int* block_table, int table_stride, int max_new, const void* K,
                 const void* V, long long token_stride, long long head_stride,
                 gemm_stream_t stream);
int kv_append_s8_rows(const kv_cache_s8_t* cache, int batch, const int* cu, const int* past,
                      const int* block_table, int table_stride, int max_new, const void* K,
                      const void* V, long long token_stride, long long head_stride, int rows,
                      gemm_stream_t stream);

/*
 * Reads tokens first[b] .. first[b] + (cu[b+1] - cu[b]) - 1 of each sequence back as
 * binary16: K and V are packed dense [tokens][kv_heads][head_dim] arrays, rows by cu.
 * Either may be NULL.  max_read: as max_new above.
 */
int kv_read_s8(const kv_cache_s8_t* cache, int batch, const int* cu, const int* first,
               const int* block_table, int table_stride, int max_read, void* K, void* V,
               gemm_stream_t stream);
int kv_read_s8_rows(const kv_cache_s8_t* cache, int batch, const int* cu, const int* first,
                    const int* block_table, int table_stride, int max_read, void* K, void* V,
                    int rows, gemm_stream_t stream);

/*
 * Attention over the cache.  Sequence b has kv_len[b] tokens in the cache and
 * n = cu[b+1] - cu[b] query rows, which are its LAST n tokens: query i stands at position
 * kv_len[b] - n + i and sees the tokens up to and including that position, with
 * window > 0 only the last `window` of them (itself included).  Query head h reads
 * KV head h / (q_heads / kv_heads).
 *     out = sum_t softmax_t(softmax_scale * q . k_t) v_t
 * A query that sees nothing (position below 0) gives zeros, one that sees a page whose
 * scale is not finite or below 0 (which no append leaves), or that holds a NaN or an infinity
 * itself, NaN; pages that it does not see leave it alone, whatever they hold.
 * Q, out: binary16, element (row, head, d) at row * token_stride + head * head_dim + d for
 * out, row * q_token_stride + head * q_head_stride + d for Q.  max_q: an upper bound of n
 * over the batch (rows beyond it are not computed, status 6).
 * Scores, softmax statistics and sums are FP32.  The tensor cores' sums of weighted values cut
 * off what does not fit, up to 2^-27 of the sum a token: 16384 tokens at most (1.2e-4), or for
 * sequences of few rows (below) up to a quarter of the sequence.  Two operands have fewer bits:
 *   - the softmax weights (times their page's value scale) are rounded to binary16 for the
 *     product with the codes, which are exact there: by 2^-11 of themselves, or up to 2^-32 of
 *     the row's largest where they are below 2^-21 of it;
 *   - sequences of up to 32 rows (n * q_heads / kv_heads; 16 for head_dim 256) are scored on
 *     the integer codes, with each row of Q in fixed point of 16 bits under one scale: a
 *     value is off by up to max|q| / 64516 of its row, a score by up to softmax_scale *
 *     sum|k| times that.  Longer ones take Q as it is.
 * So what a token gets depends, within these bounds, on how many come with it.
 * GEMM_ERR_TOO_LARGE: batch * kv_heads * (tokens a row of the table can name / 16 + 13) of
 * 2^30 or more, or max_q * q_heads / kv_heads near 2^31.
 * Work of long sequences is split over CTAs and joined in a fixed order: results
 * do not vary from run to run.  The library keeps grow-only scratch per stream for
 * that, as for gemm_s4; gemm_release_workspaces frees it.
 */
int kv_attention_s8(const kv_cache_s8_t* cache, int batch, const int* cu, const int* kv_len,
                    const int* block_table, int table_stride, int max_q, int q_heads,
                    const void* Q, long long q_token_stride, long long q_head_stride,
                    float softmax_scale, int window, void* out, long long out_token_stride,
                    gemm_stream_t stream);
int kv_attention_s8_rows(const kv_cache_s8_t* cache, int batch, const int* cu, const int* kv_len,
                         const int* block_table, int table_stride, int max_q, int q_heads,
                         const void* Q, long long q_token_stride, long long q_head_stride,
                         float softmax_scale, int window, void* out, long long out_token_stride,
                         int rows, gemm_stream_t stream);

/*
 * The same cache in 4 bits: half the bytes, and a scale and an offset for every token and head, so that
 * writing never touches older tokens and a token is held the same whichever call brings it.
 * K and V are uint8 arrays [num_pages][kv_heads][page_size][head_dim / 2], code d of a token in bits
 * [4 (d & 1), 4 (d & 1) + 4) of byte d >> 1; k_scale and v_scale are pairs of binary16 (scale, offset),
 * [num_pages][kv_heads][page_size][2], 16-byte aligned like the codes.  The value of a code is
 * offset + code * scale, within binary16's range; scales of either sign are read (none below 0 is
 * written).  Pages, tables, batches and what is done about bad ones are as above.
 */
typedef struct kv_cache_u4 {
  uint8_t* k;
  uint8_t* v;
  void* k_scale;
  void* v_scale;
  int num_pages;
  int kv_heads;
  int page_size;
  int head_dim;
} kv_cache_u4_t;

/*
 * Writes new tokens, as kv_append_s8_rows does.  Per token and head, over its head_dim values x,
 *     offset = min x,   scale = (max x - min x) / 15 rounded to binary16,
 *     code(x) = min(rint((x - offset) * (1 / scale)), 15),
 * in FP32, ties to even; scale = 0 gives codes 0.  (Where offset + 15 scale would pass the largest binary16, scale is
 * the next smaller one.)  A row of values with a NaN or an infinity has a NaN for its scale.
 */
int kv_append_u4(const kv_cache_u4_t* cache, int batch, const int* cu, const int* past,
                 const int* block_table, int table_stride, int max_new, const void* K,
                 const void* V, long long token_stride, long long head_stride, int rows,
                 gemm_stream_t stream);

/* Reads tokens back as binary16, as kv_read_s8_rows does. */
int kv_read_u4(const kv_cache_u4_t* cache, int batch, const int* cu, const int* first,
               const int* block_table, int table_stride, int max_read, void* K, void* V, int rows,
               gemm_stream_t stream);

/*
 * Attention over it, as kv_attention_s8_rows; q_heads / kv_heads: up to 128.  A query that sees a token whose scale
 * or offset (of K or of V) is not finite gives NaN, as does one that holds a NaN or an infinity itself; tokens that it
 * does not see leave it alone.
 * Scores, softmax statistics and sums are FP32.  The tensor cores' sums cut off what does not fit, up to 2^-27 of the
 * sum a token, and take 16384 tokens at most (1.2e-4), or for sequences of few rows up to a quarter of the sequence; longer
 * ones go on from their parts, which out holds while the call runs: it overlaps no input.  Operands with fewer bits:
 *   - the softmax weights, as for kv_attention_s8 (in sequences of few rows times their token's value scale);
 *   - sequences of up to 16 rows (n * q_heads / kv_heads) are scored on the integer codes, with Q in fixed point of 16 bits as
 *     there: a value is off by up to max|q| / 64516 of its row.  Longer ones take Q as it is;
 *   - values are exact in sequences of few rows (codes, and a sum of offsets in FP32), and within 2^-22 of themselves in
 *     longer ones, as two binary16.
 * So what a token gets depends, within these bounds, on how many come with it.
 * GEMM_ERR_TOO_LARGE: batch * kv_heads * (tokens a row of the table can name / 32 + 9) of 2^30 or more (/ 16 for head_dim 256),
 * or max_q * q_heads / kv_heads near 2^31.
 */
int kv_attention_u4(const kv_cache_u4_t* cache, int batch, const int* cu, const int* kv_len,
                    const int* block_table, int table_stride, int max_q, int q_heads,
                    const void* Q, long long q_token_stride, long long q_head_stride,
                    float softmax_scale, int window, void* out, long long out_token_stride,
                    int rows, gemm_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* B200KV_H_ */
