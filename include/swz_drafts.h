/* libswz, a step with drafted tokens: a cache of keys and values in bfloat16, appending to it with the rotation on the way, attention of the
 * drafted tokens of every sequence over it, the verification of the drafts, and the accepted path kept in the cache.  Same library, conventions and status
 * codes as swz.h and swz_attention.h: plain pointers and sizes, DEVICE pointers unless said otherwise, asynchronous on `stream`, no allocation, no
 * synchronisation, and on an error that is returned nothing was written.
 *
 * A step has a block of tokens for every sequence: the last token that stands, whose keys and values are not in the cache yet (the root), and drafts.  The
 * drafts are a chain, each after the one before it, or a tree: a token's parent stands before it in the block.  Blocks are packed: sequence b owns tokens
 * cu[b] .. cu[b+1] - 1, cu being sequences + 1 rising int32 on the device.  What stands in cu, positions, lengths, block tables, trees, paths and
 * tokens is not known to the host: kernels keep every access inside the tensors whatever they hold.  Tokens that no sequence owns are not written. */
#ifndef SWZ_DRAFTS_H
#define SWZ_DRAFTS_H

#include "swz_attention.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A cache of keys and values in pages, bfloat16: k, v : pages x k_heads x page_tokens x head_dim, dense, 16-byte aligned.  page_tokens is a power of two, 16 or more;
 * head_dim 64 or 128.
 *   block_table (all functions) : sequences x table_width int32, the page of positions page_tokens * j .. of sequence b at [b][j].  A page that is written must belong to one
 *   sequence of a call. */
typedef struct {
  void *k, *v;
  int64_t pages;
  int32_t page_tokens, k_heads, head_dim;
} swz_cache16;

/* Writes the tokens of k and v into the cache, token i of sequence b as position before[b] + i, the keys turned on the way; and q, turned alike, to q_out.
 *   cos, sin : table_rows x rotary_dim / 2 floats, dense, 16-byte aligned: pairs of the first `rotary_dim` dimensions are turned by the angles of a row, (a, b) becoming
 *   (a cos - b sin, b cos + a sin); pair i is (i, i + rotary_dim / 2), or (2 i, 2 i + 1) where interleaved is not 0.  32-bit arithmetic, rounded once.  cos null: nothing is turned, and there is
 *   no q.
 *   positions : a row for each token; null: the token's place in its sequence, before[b] + i.  A row that the tables have not gives NaN in the dimensions that are turned.
 *   q.data null: no queries (q_heads is not read).  q_out may be q itself (the same pointer and distances), else it must not overlap anything.
 *   Positions past the table's width, entries that name no page of the cache and sequences whose before is negative are not written to the cache.
 * Errors (all functions here): INVALID_ARG (null pointer, a size or count < 0, heads or sequences < 1, heads not a multiple of one another, a scale that is not finite and > 0, too small a
 * workspace), UNSUPPORTED (head_dim, rotary_dim, page size, element size, alignment, distances), OVERFLOW (counts that do not fit 32-bit indices, a table of more than 2^31 - 4096 positions, a launch
 * of 2^32 threads or more), HIP.  No tokens at all: SWZ_OK. */
typedef struct {
  swz_heads q, k, v, q_out;
  const float *cos, *sin;
  const int32_t *positions, *cu, *before, *block_table;
  int64_t tokens, table_rows;
  int32_t sequences, table_width, q_heads;
  int32_t rotary_dim;                /* a multiple of 16, 16 .. head_dim */
  int32_t interleaved;
} swz_append16_args;

int swz_cache16_append(const swz_cache16* cache, const swz_append16_args* args, hipStream_t stream);

/* out = softmax(scale q k^T) v of every token and query head over the first lengths[b] positions of its sequence in the cache, of which the last ones are the block's own tokens, appended
 * before: token j of n is position lengths[b] - n + j.  A token looks at all positions before the block, and
 *   tree null     : at the block's tokens up to itself (a chain, or the next piece of a prompt, of any length; every token costs the sequence's whole length, where swz_attention leaves out what is
 *                   behind a token: a prompt of 8192 tokens by itself takes three times as long as there);
 *   tree not null : at token j of its block where bit j of the token's 64-bit mask is set; at those from the 65th on none looks.
 * A token that looks at nothing gets 0, and so does one whose scores are all minus infinity, if the values are finite (0 times another one is NaN).  A length is cut to the table's positions; pages that the cache has not give NaN to what looks at them.  Infinities and NaN in keys and
 * values that a token does not look at do not reach its output.  The weights are rounded to bfloat16 for their product with v, their sum is not.
 *   q, out : `tokens` tokens of q_heads heads, query head h looking at key head h / (q_heads / k_heads).
 *   max_length : the longest length, or more (0: the table's); it decides how many workgroups share the work, no more: longer lengths are right too, and slower.
 *   workspace : swz_cache16_attention_workspace(...) bytes, 16-byte aligned; may be null where that is 0. */
typedef struct {
  swz_heads q, out;
  const int32_t *cu, *lengths, *block_table;
  const int64_t* tree;
  int64_t tokens;
  int32_t sequences, table_width, q_heads, max_length;
  float scale;
} swz_attention16_args;

int64_t swz_cache16_attention_workspace(const swz_cache16* cache, const swz_attention16_args* args);
int swz_cache16_attention(const swz_cache16* cache, const swz_attention16_args* args, void* workspace, int64_t workspace_bytes, hipStream_t stream);

/* Which drafts stand, and the token after them, from given random numbers: what is emitted has the target's distribution.
 *   target : for each token of the blocks the target's probabilities of what follows it: rows of `vocab` values, `target_pitch` elements apart, bfloat16 (elem_bytes 2) or float (4), aligned to
 *            their size.  They need not add up to 1; values below 0 count as 0.
 *   draft  : the probabilities that the token's children were drawn from (independently, with replacement), laid out alike with draft_pitch; or null: children are points, chosen by any rule.
 *   parents: the place in its block of each token's parent, less than its own (the root's is not read); null: the one before it.
 *   tokens, uniforms : what each node proposes, and a number of [0, 1) for each; the root's is the new token's.
 * From the root on, the children of the current node are tested in their order; the first that passes becomes the current node.  P is the target's row of the current node, at first.
 *   draft not null: child c, of token x, passes if uniforms[c] * Q(x) < P(x).  If it does not, P becomes max(P - Q, 0) / its sum (or stays, if that sum is not above 0).
 *   draft null    : it passes if P(x) > 0 and P(x) > uniforms[c] * M, M being 1 at first.  If it does not, M loses P(x), and P(x) becomes 0.
 * A comparison with NaN is false: a child of such a probability fails, and so do all those after it under the same node where children are points, as M is NaN then.
 * Where no child passes, the new token is the first x where P(0) + .. + P(x) > uniforms[root] * sum(P), or the last x of P(x) > 0 where none is; -1 if sum(P) is no finite number above 0.
 * All in 64-bit arithmetic.  A token outside the vocabulary, one whose parent does not stand before it, and those of a block from the 65th on are not tested.  The order of the sums depends on
 * the sizes alone.
 *   accepted : receives the number of drafts that stand, for each sequence.   token : the new token (-1 also for a block of no tokens).
 *   path     : receives, in the place of the block's tokens, the places of the root and of the drafts that stand, in order, then -1.
 *   workspace: swz_verify_drafts_workspace(args) bytes, 16-byte aligned. */
typedef struct {
  const void *target, *draft;
  int64_t target_pitch, draft_pitch, vocab, total;      /* total: tokens of all blocks; vocab below 2^30 */
  const int32_t *tokens, *parents, *cu;
  const float* uniforms;
  int32_t *accepted, *path, *token;
  int32_t sequences, elem_bytes;
} swz_verify_args;

int64_t swz_verify_drafts_workspace(const swz_verify_args* args);
int swz_verify_drafts(const swz_verify_args* args, void* workspace, int64_t workspace_bytes, hipStream_t stream);

/* Keeps the accepted path: position before[b] + path[cu[b] + i] of sequence b moves to before[b] + i, i = 1 .. accepted[b].  The path rises, as that of swz_verify_drafts does.  Entries that name no
 * token of the block and positions without a page are left out.   tokens : of all blocks. */
int swz_cache16_keep(const swz_cache16* cache, const int32_t* cu, const int32_t* before, const int32_t* path, const int32_t* accepted, int64_t tokens, const int32_t* block_table,
                     int32_t table_width, int32_t sequences, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* SWZ_DRAFTS_H */
