/* libswz, attention layers: norm and rotation of queries and keys, attention over packed prompts with its gradient, and attention
 * over a cache of keys and values held in 4 bits.  Same library, conventions and status codes as swz.h: plain pointers and sizes, DEVICE
 * pointers unless said otherwise, asynchronous on `stream`, no allocation, no synchronisation, and on an error that is
 * returned nothing was written.
 *
 * Queries, keys, values and what is made of them are bfloat16; statistics, sums and gradients of weights are kept in 32 bits and
 * everything else is rounded once, to nearest even, when it is stored (the places where 32-bit values are rounded on the way to a matrix
 * instruction are said).  head_dim is 64 or 128.  A tensor of heads is given as a pointer with the distance, in elements, from one
 * token to the next and from one head to the next: multiples of 8 (a pointer is 16-byte aligned), the dimensions of a head being dense.
 * q_heads is a multiple of k_heads: query head h looks at key head h / (q_heads / k_heads).
 *
 * Sequences are packed: sequence b owns tokens cu[b] .. cu[b+1] - 1 of the tensor, cu being sequences + 1 rising int32 on the
 * device.  Empty sequences are allowed.  What stands in cu, in positions, lengths or block tables is not known to the
 * host: kernels keep every access inside the tensors whatever they hold.  Tokens that no sequence owns are not written.
 */
#ifndef SWZ_ATTENTION_H
#define SWZ_ATTENTION_H

#include "swz.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  void* data;      /* bfloat16, 16-byte aligned */
  int64_t token;   /* elements from one token to the next, a multiple of 8 */
  int64_t head;    /* elements from one head to the next, a multiple of 8 */
} swz_heads;

/* z = R(position) (x / sqrt(mean(x^2) + eps) * weight) for every head of q and of k, one pass over both.
 *   R turns pairs of the first `rotary_dim` dimensions by the angles whose cosines and sines stand in row `position` of the tables: pair i is
 *   (i, i + rotary_dim / 2), or (2 i, 2 i + 1) where interleaved is not 0.  The other dimensions are not turned.
 *   q_out, k_out may be q, k themselves (the same pointer and distances), else they must not overlap them.
 *   A token whose position is not in 0 .. table_rows - 1 gets NaN. */
typedef struct {
  swz_heads q, k, q_out, k_out;
  const void *q_weight, *k_weight;   /* head_dim bfloat16 each, 16-byte aligned */
  const float *cos, *sin;            /* table_rows x rotary_dim / 2, dense, 16-byte aligned */
  const int32_t* positions;          /* one for each token */
  int64_t tokens;
  int32_t q_heads, k_heads, head_dim;
  int32_t rotary_dim;                /* a multiple of 16, 16 .. head_dim */
  int32_t interleaved;
  int64_t table_rows;
  float eps;                         /* >= 0 */
} swz_norm_args;

/* Errors (all functions here): INVALID_ARG (null pointer, a size or count < 0, heads or sequences < 1, heads not a multiple of one
 * another, eps < 0 or a scale that is not finite and > 0), UNSUPPORTED (head_dim, rotary_dim, page size, alignment, distances), OVERFLOW (tokens >= 2^31, for attention tokens or a table's positions > 2^31 - 4096, or a
 * launch of 2^32 threads or more), HIP.  No tokens at all: SWZ_OK, and gradients of weights are 0. */
int swz_qk_norm_rope(const swz_norm_args* args, hipStream_t stream);

/* The gradient of swz_qk_norm_rope.  args->q, k and the tables as in the forward call; q_out, k_out hold the gradients of its
 * outputs (read), dq, dk receive those of q and k (may be q_out, k_out themselves), dq_weight, dk_weight (head_dim 32-bit floats each, 16-byte aligned) those of the weights, whole:
 * sums over all tokens and heads, in an order that depends on the sizes and the device alone.
 *   workspace : swz_qk_norm_rope_backward_workspace(args) bytes, 16-byte aligned, needed until the call has run. */
int64_t swz_qk_norm_rope_backward_workspace(const swz_norm_args* args);
int swz_qk_norm_rope_backward(const swz_norm_args* args, const swz_heads* dq, const swz_heads* dk, float* dq_weight, float* dk_weight,
                              void* workspace, int64_t workspace_bytes, hipStream_t stream);

/* out = softmax(scale q k^T) v for every sequence and head, and lse = log(sum(exp(scale q k^T))).
 *   causal not 0: the last query of a sequence looks at all its keys, each query before at one key fewer; with fewer keys than queries the
 *   first queries look at nothing.  A query that looks at nothing gets out = 0, lse = -inf.
 *   The weights are rounded to bfloat16 for their product with v, their sum is not.  Infinities and NaN in keys and values that a query does not look
 *   at do not reach its output.   The distances of tokens of q, k, v (and dout below) are less than 2^28 elements. */
typedef struct {
  swz_heads q, k, v, out;
  float* lse;                        /* q_heads x total_q, dense */
  const int32_t *cu_q, *cu_k;        /* sequences + 1 each; the same pointer where queries and keys belong to the same tokens */
  int64_t total_q, total_k;
  int32_t sequences, q_heads, k_heads, head_dim;
  int32_t causal;
  float scale;
} swz_attention_args;

/*   workspace : swz_attention_workspace(args) bytes, 16-byte aligned; may be null where that is 0 (it is not where few queries look at many keys, which are then
 *   cut among workgroups and joined by a second launch). */
int64_t swz_attention_workspace(const swz_attention_args* args);
int swz_attention(const swz_attention_args* args, void* workspace, int64_t workspace_bytes, hipStream_t stream);

/* The gradient of swz_attention: args as in the forward call, with its out and lse (read).
 *   dout : gradient of out.   dq, dk, dv : receive those of q, k, v, for all tokens of the sequences (must not overlap anything that is read).
 *   Weights and their gradients are rounded to bfloat16 for the products.  No atomics: the bits do not depend on the run.
 *   workspace : swz_attention_backward_workspace(args) bytes, 16-byte aligned; may be null where that is 0. */
int64_t swz_attention_backward_workspace(const swz_attention_args* args);
int swz_attention_backward(const swz_attention_args* args, const swz_heads* dout, const swz_heads* dq, const swz_heads* dk, const swz_heads* dv,
                           void* workspace, int64_t workspace_bytes, hipStream_t stream);

/* A cache of keys and values in pages.  64 values of a head (a group) share a step and a low: value = low + step * n, n in 0..15.
 *   low = the smallest value, step = (largest - low) / 15 rounded to bfloat16, n = (value - low) / step rounded to nearest even.  A group whose range is
 *   not finite (infinities or NaN in it, or values too far apart) is held as NaN.
 *   k_words  : pages x k_heads x page_tokens x head_dim / 8 words of 32 bits: word head_dim / 32 * g + s of a key holds its dimensions 32 s + 8 g .. + 7.
 *   v_words  : pages x k_heads x page_tokens / 8 x head_dim words: 8 tokens of one dimension each.
 *   Number 2 i + h of a word's eight stands in its bits 4 (i + 4 h) .. + 3.
 *   k_scales, v_scales : pages x k_heads x page_tokens x head_dim / 64 x (step, low), bfloat16.
 *   All dense, 16-byte aligned.  page_tokens is a power of two, 32 or more. */
typedef struct {
  int32_t *k_words, *v_words;
  void *k_scales, *v_scales;
  int64_t pages;
  int32_t page_tokens, k_heads, head_dim;
} swz_cache4;

/* Writes the tokens of k and v into the cache: token i of sequence b becomes position before[b] + i of the sequence.
 *   block_table : sequences x table_width int32, the page of positions page_tokens * j .. of sequence b at [b][j].  Positions past the table's width and
 *   entries that name no page of the cache are not written.  A page must belong to one sequence of a call. */
int swz_cache4_append(const swz_cache4* cache, const swz_heads* k, const swz_heads* v, int64_t tokens, const int32_t* cu, const int32_t* before,
                      const int32_t* block_table, int32_t table_width, int32_t sequences, hipStream_t stream);

/* Reads positions first[b] .. of every sequence back as bfloat16, cu[b+1] - cu[b] of them, into k and v.  Positions past the table's width and
 * entries that name no page read as NaN. */
int swz_cache4_read(const swz_cache4* cache, const swz_heads* k, const swz_heads* v, int64_t tokens, const int32_t* cu, const int32_t* first,
                    const int32_t* block_table, int32_t table_width, int32_t sequences, hipStream_t stream);

/* Attention of one token of each sequence over the first lengths[b] positions of the cache, its own among them.  A sequence of length 0 gets 0; one longer
 * than its table is cut to it; pages that the cache has not give NaN.
 *   q, out : sequences tokens of q_heads heads.   max_length : the longest length, or more (0: the table's); it decides how many waves share the work, no
 *   more: longer lengths are right too, and slower.
 *   The weights times the steps of v are rounded to bfloat16 for their product with v's numbers.
 *   workspace : swz_cache4_attention_workspace(...) bytes, 16-byte aligned; may be null where that is 0 (it is where the longest length is short). */
int64_t swz_cache4_attention_workspace(const swz_cache4* cache, int32_t sequences, int32_t q_heads, int32_t table_width, int32_t max_length);
int swz_cache4_attention(const swz_cache4* cache, const swz_heads* q, const swz_heads* out, const int32_t* lengths, const int32_t* block_table,
                         int32_t table_width, int32_t sequences, int32_t q_heads, int32_t max_length, float scale, void* workspace, int64_t workspace_bytes,
                         hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* SWZ_ATTENTION_H */
