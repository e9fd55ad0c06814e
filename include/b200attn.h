/*
 * b200attn -- what stands between a transformer's projections and its cache, on one NVIDIA B200
 * (sm_100a): rotary positions, and attention of prompts over their own binary16 keys and values.
 * Part of libb200gemm.so; return codes, streams, threads and the device status word are those of
 * b200gemm.h, packed ragged batches those of b200kv.h.
 *
 * All tensors of values are binary16, 16-byte aligned, with strides (in elements) that are multiples of 8:
 * element (row, head, d) at row * token_stride + head * head_stride + d.
 */
#ifndef B200ATTN_H_
#define B200ATTN_H_

#include "b200gemm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rows of `heads` heads each that are read at x and written at y.  y is x itself, with the same strides, or
 * does not overlap it. */
typedef struct rotary_rows {
  const void* x;
  void* y;
  int heads;
  long long x_token_stride, x_head_stride;
  long long y_token_stride, y_head_stride;
} rotary_rows_t;

enum { ROTARY_HALVES = 0, ROTARY_NEIGHBOURS = 1 };

/*
 * Rotary positions of one to four axes (text: one; images: height, width; video: time, height, width).
 * Frequency i, 0 <= i < rotary_dim / 2, turns the pair
 *     (a, b) = (i, i + rotary_dim / 2)   ROTARY_HALVES,   (2i, 2i + 1)   ROTARY_NEIGHBOURS
 * of every head by angle = positions[axis(i)][token] * inv_freq[i]:
 *     y_a = x_a cos(angle) - x_b sin(angle),   y_b = x_b cos(angle) + x_a sin(angle).
 * The first sections[0] frequencies belong to axis 0, the next sections[1] to axis 1 and so on; they
 * sum to rotary_dim / 2.  Values from rotary_dim on are passed on.
 * positions: int32 [axes] rows of `tokens` entries, axis_stride entries apart, any 32-bit value; inv_freq: FP32
 * [rotary_dim / 2]; both in device memory.  sections: host memory (axes = 1: may be NULL).
 * rotary_dim: a multiple of 16 up to head_dim; head_dim: a multiple of 8 up to 1024.
 * q, k: either may be NULL.  Angles are exact to 5e-7 at any position, the rest is FP32, rounded once.
 */
int rotary_fp16(int tokens, int head_dim, int rotary_dim, int pairs, const rotary_rows_t* q,
                const rotary_rows_t* k, const int* positions, int axes, long long axis_stride,
                const int* sections, const float* inv_freq, gemm_stream_t stream);

/*
 * Attention of packed sequences over themselves: sequence b has the rows cu[b] .. cu[b+1]-1 of Q, K, V and
 * out (cu: int32 [batch + 1], device memory, starting at 0, not decreasing; zero rows are allowed).  Query head h
 * reads KV head h / (q_heads / kv_heads).
 *     out_i = sum_t softmax_t(softmax_scale * q_i . k_t) v_t
 * over the tokens t of the same sequence; causal = 1: those with t <= i, and with window > 0 the last `window` of
 * them only (i itself included); causal = 0: all (window must be 0).
 * head_dim: 64, 128 or 256; q_heads / kv_heads: up to 128.  max_len: an upper bound of the rows of a
 * sequence, rows: of the packed arrays; rows beyond either are not computed, status 6.  Rows behind the last
 * sequence are left as they are.  K and V have one common pair of strides; heads of a row of out are dense.
 * Scores, softmax statistics and sums are FP32; the softmax weights are rounded to binary16 for the product with V,
 * by 2^-11 of themselves (2^-32 of the row's largest where they are below 2^-21 of it).  The tensor cores' sums cut off what
 * does not fit, up to 2^-27 of the sum a token; a sum takes 16384 tokens at most (1.2e-4), and longer ones go on from its parts.
 * out, which holds such parts while the call runs, overlaps no input.
 * A token that a query does not see leaves it alone, whatever it holds, to the last bit; one that it sees counts as the formula
 * has it, NaN and infinities included (but an infinite value with a weight below 2^-32 of the row's largest may give a NaN).
 */
int attention_fp16(int batch, const int* cu, int max_len, int rows, int q_heads, int kv_heads,
                   int head_dim, const void* Q, long long q_token_stride, long long q_head_stride,
                   const void* K, const void* V, long long kv_token_stride, long long kv_head_stride,
                   float softmax_scale, int causal, int window, void* out,
                   long long out_token_stride, gemm_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* B200ATTN_H_ */
