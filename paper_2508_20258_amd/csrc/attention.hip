// libswz: C-ABI entry points of attention layers (declared in include/swz_attention.h).  Host side: argument checks, the split of the
// work, launches.  Nothing here allocates device memory or synchronises.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/swz_attention.h"
#include "attention_backward_kernel.h"
#include "attention_kernel.h"
#include "cache4_kernel.h"
#include "host_checks.h"
#include "launch.h"
#include "pid_decode.h"
#include "qk_norm_kernel.h"

namespace {

using namespace swz::host;
using swz::DeviceFacts;
using swz::launch;
using swz::query_device;

constexpr int64_t kRowDistance = (int64_t)1 << 28;      // less than this from one token to the next, where tiles of tokens are loaded (RowLoader)

// XCDs that the workgroups are dealt to; 1 (their order as it is) where the device does not say.
int xcds() {
  DeviceFacts f;
  return query_device(&f) == SWZ_OK && f.num_xcd > 0 ? f.num_xcd : 1;
}

// ---------------------------------------------------------------- norm and rotation

int check_norm(const swz_norm_args* a) {
  if (a == nullptr || a->q_weight == nullptr || a->k_weight == nullptr || a->cos == nullptr || a->sin == nullptr || a->positions == nullptr) return SWZ_ERR_INVALID_ARG;
  if (a->tokens < 0 || a->q_heads < 1 || a->k_heads < 1 || a->table_rows < 0 || !(a->eps >= 0.f)) return SWZ_ERR_INVALID_ARG;
  const int st = check_heads(a->q, a->k, a->q_out, a->k_out);
  if (st != SWZ_OK) return st;
  if (!head_dim_ok(a->head_dim) || a->rotary_dim < 16 || a->rotary_dim > a->head_dim || a->rotary_dim % 16 != 0) return SWZ_ERR_UNSUPPORTED;
  if (!aligned(a->q_weight, 16) || !aligned(a->k_weight, 16) || !aligned(a->cos, 16) || !aligned(a->sin, 16) || !aligned(a->positions, 4)) return SWZ_ERR_UNSUPPORTED;
  if (a->q_heads > 65536 || a->k_heads > 65536 || a->table_rows >= kTokens) return SWZ_ERR_OVERFLOW;
  if (a->tokens >= kTokens || a->tokens * a->q_heads >= kTokens || a->tokens * a->k_heads >= kTokens) return SWZ_ERR_OVERFLOW;
  return SWZ_OK;
}

swz::NormSide norm_side(const swz_heads& x, const swz_heads& z, const void* weight, int heads, int64_t tokens) {
  const int blocks = swz::norm_blocks(heads);
  return {device_heads(x), device_heads(z), {}, static_cast<const uint16_t*>(weight), heads, blocks, (int)(tokens * blocks)};
}
swz::NormArgs norm_args(const swz_norm_args& a) {
  swz::NormArgs n{};
  n.q = norm_side(a.q, a.q_out, a.q_weight, a.q_heads, a.tokens);
  n.k = norm_side(a.k, a.k_out, a.k_weight, a.k_heads, a.tokens);
  n.cos = a.cos, n.sin = a.sin, n.positions = a.positions;
  n.rotary = a.rotary_dim, n.table_rows = (int)a.table_rows, n.eps = a.eps;
  return n;
}
// Of the backward pass: as many as have items, at most four to a compute unit.
int norm_backward_workgroups(const swz::NormArgs& n, int head_dim) {
  const int most = 4 * compute_units(), some = swz::norm_workgroups(n.q.items > n.k.items ? n.q.items : n.k.items, head_dim);
  return some < 1 ? 1 : some < most ? some : most;
}

// ---------------------------------------------------------------- prompts

int check_prompt(const swz_attention_args* a) {
  if (a == nullptr || a->lse == nullptr || a->cu_q == nullptr || a->cu_k == nullptr) return SWZ_ERR_INVALID_ARG;
  if (a->total_q < 0 || a->total_k < 0 || a->sequences < 1 || a->q_heads < 1 || a->k_heads < 1 || a->q_heads % a->k_heads != 0) return SWZ_ERR_INVALID_ARG;
  if (!(a->scale > 0.f) || !isfinite(a->scale)) return SWZ_ERR_INVALID_ARG;
  const int st = check_heads(a->q, a->k, a->v, a->out);
  if (st != SWZ_OK) return st;
  if (a->q.token >= kRowDistance || a->k.token >= kRowDistance || a->v.token >= kRowDistance) return SWZ_ERR_UNSUPPORTED;
  if (!head_dim_ok(a->head_dim) || !aligned(a->lse, 4) || !aligned(a->cu_q, 4) || !aligned(a->cu_k, 4)) return SWZ_ERR_UNSUPPORTED;
  return a->total_q > kMostKeys || a->total_k > kMostKeys ? SWZ_ERR_OVERFLOW : SWZ_OK;
}

swz::PromptArgs prompt_args(const swz_attention_args& a) {
  swz::PromptArgs p{};
  p.q = device_heads(a.q), p.k = device_heads(a.k), p.v = device_heads(a.v), p.out = device_heads(a.out);
  p.lse = a.lse, p.cu_q = a.cu_q, p.cu_k = a.cu_k;
  p.total_q = (int)a.total_q, p.total_k = (int)a.total_k, p.sequences = a.sequences;
  p.q_heads = a.q_heads, p.k_heads = a.k_heads, p.num_xcd = xcds(), p.sets = swz::prompt_sets(a.k_heads, p.num_xcd), p.scale = a.scale;
  return p;
}

// Workgroups for tiles of `rows` tokens (see find_slot) and `heads` heads; the launch refuses what is too many threads.
int64_t slots_of(int64_t total, int sequences, int rows, int per = 1) { return total / rows + (int64_t)per * sequences; }

// The launch of a kernel over prompts: `slots` turns, of `splits` workgroups each, for each of `group` parts of a key head's query heads.
template <auto KERNEL, class Args>
int launch_prompt(Args& args, swz::PromptArgs& p, int64_t slots, int splits, int group, int threads, hipStream_t stream) {
  const int64_t workgroups = slots * splits < kTokens ? swz::prompt_workgroups(slots * splits, p.k_heads, group, p.num_xcd) : kTokens;
  if (workgroups >= kTokens) return SWZ_ERR_OVERFLOW;
  p.slots = (int)slots;
  p.splits = splits;
  return launch(KERNEL, dim3((unsigned)workgroups), dim3((unsigned)threads), 0, stream, args);
}
bool too_many_threads(int64_t slots, int heads_k, int group, int num_xcd, int threads) {
  return slots >= kTokens || swz::prompt_workgroups(slots, heads_k, group, num_xcd) * threads > swz::kLaunchThreads;
}

// Waves of a workgroup that share its tiles, 32 rows each (8 instead of 4: 0.7% less time at 32768 tokens, more at short ones).  As many of them as the sharing of key heads
// allows have the same rows of another query head: a tile is then loaded once for all of them, and short sequences fill their workgroups.  Causal, 32 heads of 128 sharing 8,
// with four query heads together and with the 128 rows of one: 32 sequences of 16 tokens 6.6 us and 11.8, of 200 37.6 and 44.8, of 512 124 and 139, one of 8192 499 and 501.
constexpr int kPromptWaves = 4;
int heads_together(const swz_attention_args& a) {
  const int group = a.q_heads / a.k_heads;
  return group % 4 == 0 ? 4 : group % 2 == 0 ? 2 : 1;
}
template <class F>
int for_heads_together(int heads, F&& f) {
  return heads == 4 ? f(std::integral_constant<int, 4>{}) : heads == 2 ? f(std::integral_constant<int, 2>{}) : f(std::integral_constant<int, 1>{});
}

// Forward: into how many pieces the keys of a row are cut.
int forward_splits(const swz_attention_args& a) {
  const int64_t cus = compute_units();
  const int heads = heads_together(a), group = a.q_heads / a.k_heads;
  const int64_t few = swz::prompt_workgroups(slots_of(a.total_q, 1, 32 * kPromptWaves / heads), a.k_heads, group / heads, xcds());       // workgroups, if the sequences were one
  const int64_t tiles = a.total_k / a.sequences / swz::kPromptKeys;                                      // of an average sequence
  if (few >= cus || tiles < 16) return 1;
  const int64_t splits = 2 * cus / few < tiles / 8 ? 2 * cus / few : tiles / 8;
  return (int)(splits < 32 ? splits : 32);
}
int64_t forward_floats(const swz_attention_args& a, int splits) { return splits == 1 ? 0 : (int64_t)splits * a.total_q * a.q_heads * (a.head_dim + 2); }

template <int D>
struct DkvShape {
  static constexpr int kKeyWaves = D == 128 ? 4 : 2, kParts = 2;
  static constexpr int kKeys = 32 * kKeyWaves, kThreads = 64 * kKeyWaves * kParts;
};

// How many workgroups share the queries of a tile of keys and leave their sums to another kernel.  Where tiles and key heads give no more workgroups than one for each compute unit (two of
// 256 threads: a compute unit holds one of 512, or three of 256), as many as give two (four) to each, or one for every eight rounds of the
// queries of an average sequence, if that is fewer, as writing and reading the sums takes about as long as ten rounds; at most 16.  8 query heads of one key head, 4096 causal tokens, the
// whole gradient: 928 us whole, 268 with 15 splits; 32 heads of 8, 2048 tokens: 312 whole, 210 with 3; 16 of 2, 2007 tokens of four sequences: 263 whole, 103 with 7, 113 with 15.
int dkv_splits(const swz_attention_args& a) {
  auto splits = [&](auto shape) {
    using K = decltype(shape);
    const int64_t room = (K::kThreads == 512 ? 2 : 4) * (int64_t)compute_units() / (slots_of(a.total_k, 1, K::kKeys) * a.k_heads);
    const int64_t rounds = (a.total_q / a.sequences / swz::kBackRows + 1) * (a.q_heads / a.k_heads) / K::kParts, most = room < rounds / 8 ? room : rounds / 8;
    return (int)(most < 1 ? 1 : most < 16 ? most : 16);
  };
  return a.head_dim == 128 ? splits(DkvShape<128>{}) : splits(DkvShape<64>{});
}
// Statistics of queries, then the splits' sums.
int64_t backward_floats(const swz_attention_args& a, int splits) {
  const int64_t stats = (2 * a.total_q * a.q_heads + 3) / 4 * 4;
  return stats + (splits == 1 ? 0 : (int64_t)splits * a.total_k * a.k_heads * 2 * a.head_dim);
}

// ---------------------------------------------------------------- the cache

int check_cache(const swz_cache4* c) {
  if (c == nullptr || c->k_words == nullptr || c->v_words == nullptr || c->k_scales == nullptr || c->v_scales == nullptr || c->pages < 1 || c->k_heads < 1) return SWZ_ERR_INVALID_ARG;
  if (!head_dim_ok(c->head_dim) || c->page_tokens < 32 || (c->page_tokens & (c->page_tokens - 1)) != 0) return SWZ_ERR_UNSUPPORTED;
  if (!aligned(c->k_words, 16) || !aligned(c->v_words, 16) || !aligned(c->k_scales, 16) || !aligned(c->v_scales, 16)) return SWZ_ERR_UNSUPPORTED;
  return c->pages >= kTokens ? SWZ_ERR_OVERFLOW : SWZ_OK;
}

swz::CacheArgs cache_args(const swz_cache4& c, const int32_t* table, int table_width) {
  swz::CacheArgs a{};
  a.k_words = reinterpret_cast<uint32_t*>(c.k_words), a.v_words = reinterpret_cast<uint32_t*>(c.v_words);
  a.k_scales = static_cast<uint32_t*>(c.k_scales), a.v_scales = static_cast<uint32_t*>(c.v_scales);
  a.table = table, a.pages = c.pages, a.page_shift = __builtin_ctz((unsigned)c.page_tokens), a.k_heads = c.k_heads, a.table_width = table_width;
  return a;
}

template <bool READ>
int store_or_read(const swz_cache4* cache, const swz_heads* k, const swz_heads* v, int64_t tokens, const int32_t* cu, const int32_t* before, const int32_t* table,
                  int32_t table_width, int32_t sequences, hipStream_t stream) {
  int st = check_cache(cache);
  if (st != SWZ_OK) return st;
  if (k == nullptr || v == nullptr || cu == nullptr || before == nullptr || table == nullptr || tokens < 0 || sequences < 1 || table_width < 1) return SWZ_ERR_INVALID_ARG;
  if (tokens == 0) return SWZ_OK;
  st = check_heads(*k, *v);
  if (st != SWZ_OK) return st;
  if (!aligned(cu, 4) || !aligned(before, 4) || !aligned(table, 4)) return SWZ_ERR_UNSUPPORTED;
  if (tokens >= kTokens) return SWZ_ERR_OVERFLOW;
  return for_head_dim(cache->head_dim, [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    swz::StoreArgs a{};
    a.c = cache_args(*cache, table, table_width);
    a.k = device_heads(*k), a.v = device_heads(*v);
    a.cu = cu, a.before = before, a.total = (int)tokens, a.sequences = sequences;
    a.head_blocks = (cache->k_heads + swz::StoreShape<D>::kHeads - 1) / swz::StoreShape<D>::kHeads;
    auto kernel = READ ? swz::cache4_read_kernel<D> : swz::cache4_append_kernel<D>;
    // a workgroup for every block of heads where that does not fill the chip twice over, else one for all of them
    const int64_t slots = slots_of(tokens, sequences, 8, 2);
    a.splits = slots * a.head_blocks <= 4 * (int64_t)compute_units() ? a.head_blocks : 1;
    if (slots * a.splits >= kTokens) return (int)SWZ_ERR_OVERFLOW;
    return launch(kernel, dim3((unsigned)(slots * a.splits)), dim3(256), 0, stream, a);
  });
}

// A decoding step: waves that share the steps of a key head (of each block of 16 of its query heads), rows that a product has for queries.
struct DecodePlan {
  int columns, rows, shares;         // shares 0: a workgroup for each sequence and key head
};
DecodePlan decode_plan(const swz_cache4& c, int sequences, int q_heads, int table_width, int max_length) {
  const int group = q_heads / c.k_heads, columns = (group + 15) / 16, rows = group <= 4 ? 4 : group <= 8 ? 8 : 16;
  const int64_t cut = (int64_t)table_width * c.page_tokens, longest = max_length > 0 && max_length < cut ? max_length : cut;
  // Few tokens: one launch, a workgroup of 8 waves for each sequence and key head, not waves that share all steps and a second launch that joins them.  4 heads of 128 for each of 8 key
  // heads: 16 sequences of 256 tokens 8.1 us and 10.8, of 1000 11.5 and 15.0, of 2000 18.3 and 19.8, of 4000 28.8 and 26.0; one of 1000 10.8 and 10.9, of 2000 15.1 and 12.5; 64 of
  // 1000 25.8 and 25.7.  16 heads of one key head, 8 of 1000: 13.6 and 12.9.  Heads of 64: 8 of 2000 10.1 and 13.5, of 4000 18.4 and 17.1.  The rule goes by the length alone; where the two
  // cross also depends on sequences and heads, and of these it takes the slower one for 16 of 2000 and for the 16 heads of one key head, by 5 and 8 %.
  if (longest * c.head_dim <= 1 << 17) return {columns, rows, 0};
  // as many as run together; fewer where there are fewer steps
  const int64_t together = (int64_t)compute_units() * 4 * (c.head_dim == 64 ? 3 : rows >= 8 ? 2 : 3) / ((int64_t)c.k_heads * columns);
  const int64_t steps = (longest + swz::kDecodeStep - 1) / swz::kDecodeStep * sequences;
  return {columns, rows, (int)(together < 1 ? 1 : steps < together ? steps : together)};
}

int check_decode(const swz_cache4* c, int sequences, int q_heads, int table_width, int max_length) {
  const int st = check_cache(c);
  if (st != SWZ_OK) return st;
  if (sequences < 1 || q_heads < 1 || q_heads % c->k_heads != 0 || table_width < 1 || max_length < 0) return SWZ_ERR_INVALID_ARG;
  if ((int64_t)table_width * c->page_tokens > kMostKeys || (int64_t)sequences * q_heads >= kTokens) return SWZ_ERR_OVERFLOW;
  return SWZ_OK;
}

// The parts' sums, their statistics, and where they are.
int64_t decode_parts(const swz_cache4& c, const DecodePlan& p) { return (int64_t)p.shares * c.k_heads * p.columns * 2 * p.rows; }
int64_t decode_bytes(const swz_cache4& c, const DecodePlan& p, int sequences) { return p.shares == 0 ? 0 : 4 * decode_parts(c, p) * (c.head_dim + 2) + (int64_t)8 * sequences * c.k_heads * p.columns; }

}  // namespace

extern "C" {

int swz_qk_norm_rope(const swz_norm_args* args, hipStream_t stream) {
  const int st = check_norm(args);
  if (st != SWZ_OK || args->tokens == 0) return st;
  swz::NormArgs n = norm_args(*args);
  return for_head_dim(args->head_dim, [&](auto dim) {
    return for_flag(args->interleaved != 0, [&](auto interleaved) {
      constexpr int D = decltype(dim)::value;
      n.workgroups_q = swz::norm_workgroups(n.q.items, D);
      return launch(swz::qk_norm_kernel<D, decltype(interleaved)::value>, dim3((unsigned)(n.workgroups_q + swz::norm_workgroups(n.k.items, D))), dim3(swz::kNormThreads), 0, stream, n);
    });
  });
}

int64_t swz_qk_norm_rope_backward_workspace(const swz_norm_args* args) {
  const int st = check_norm(args);
  return st != SWZ_OK ? st : (int64_t)norm_backward_workgroups(norm_args(*args), args->head_dim) * 2 * args->head_dim * 4;
}

int swz_qk_norm_rope_backward(const swz_norm_args* args, const swz_heads* dq, const swz_heads* dk, float* dq_weight, float* dk_weight,
                              void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  int st = check_norm(args);
  if (st != SWZ_OK) return st;
  if (dq == nullptr || dk == nullptr || dq_weight == nullptr || dk_weight == nullptr || workspace == nullptr) return SWZ_ERR_INVALID_ARG;
  st = check_heads(*dq, *dk);
  if (st != SWZ_OK) return st;
  if (!aligned(dq_weight, 16) || !aligned(dk_weight, 16) || !aligned(workspace, 16)) return SWZ_ERR_UNSUPPORTED;
  if (workspace_bytes < swz_qk_norm_rope_backward_workspace(args)) return SWZ_ERR_INVALID_ARG;
  swz::NormArgs n = norm_args(*args);
  n.q.dx = device_heads(*dq), n.k.dx = device_heads(*dk);
  n.partial = static_cast<float*>(workspace);
  const int blocks = norm_backward_workgroups(n, args->head_dim);
  st = for_head_dim(args->head_dim, [&](auto dim) {
    return for_flag(args->interleaved != 0, [&](auto interleaved) {
      return launch(swz::qk_norm_backward_kernel<decltype(dim)::value, decltype(interleaved)::value>, dim3((unsigned)blocks), dim3(swz::kNormThreads), 0, stream, n);
    });
  });
  if (st != SWZ_OK) return st;
  return launch(swz::norm_weights_kernel, dim3((unsigned)(2 * args->head_dim / 4)), dim3(256), 0, stream, n.partial, blocks, args->head_dim, dq_weight, dk_weight);
}

int64_t swz_attention_workspace(const swz_attention_args* args) {
  const int st = check_prompt(args);
  return st != SWZ_OK ? st : 4 * forward_floats(*args, forward_splits(*args));
}

int swz_attention(const swz_attention_args* args, void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  const int st = check_prompt(args);
  if (st != SWZ_OK || args->total_q == 0) return st;
  const int splits = forward_splits(*args);
  const int64_t floats = forward_floats(*args, splits);
  if (floats > 0 && (workspace == nullptr || workspace_bytes < 4 * floats)) return SWZ_ERR_INVALID_ARG;
  if (!aligned(workspace, 16)) return SWZ_ERR_UNSUPPORTED;
  swz::PromptArgs p = prompt_args(*args);
  p.part_sums = static_cast<float*>(workspace);
  p.part_stats = p.part_sums + (floats > 0 ? floats / (args->head_dim + 2) * args->head_dim : 0);
  const int64_t join_slots = slots_of(args->total_q, args->sequences, swz::kJoinRows);
  if (splits > 1 && too_many_threads(join_slots, args->q_heads, 1, p.num_xcd, 64 * swz::kJoinRows)) return SWZ_ERR_OVERFLOW;
  return for_head_dim(args->head_dim, [&](auto dim) {
    return for_flag(args->causal != 0, [&](auto causal) {
      constexpr int D = decltype(dim)::value;
      constexpr bool kCausal = decltype(causal)::value;
      const int status = for_heads_together(heads_together(*args), [&](auto heads) {
        constexpr int H = decltype(heads)::value;
        return launch_prompt<swz::attention_kernel<D, kPromptWaves, H, kCausal>>(p, p, slots_of(args->total_q, args->sequences, 32 * kPromptWaves / H), splits, args->q_heads / args->k_heads / H,
                                                                                 64 * kPromptWaves, stream);
      });
      if (status != SWZ_OK || splits == 1) return status;
      p.sets = swz::prompt_sets(args->q_heads, p.num_xcd);
      p.slots = (int)join_slots;
      return launch(swz::attention_join_kernel<D>, dim3((unsigned)swz::prompt_workgroups(join_slots, args->q_heads, 1, p.num_xcd)), dim3(64 * swz::kJoinRows), 0, stream, p);
    });
  });
}

int64_t swz_attention_backward_workspace(const swz_attention_args* args) {
  const int st = check_prompt(args);
  return st != SWZ_OK ? st : 4 * backward_floats(*args, dkv_splits(*args));
}

int swz_attention_backward(const swz_attention_args* args, const swz_heads* dout, const swz_heads* dq, const swz_heads* dk, const swz_heads* dv,
                           void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  int st = check_prompt(args);
  if (st != SWZ_OK) return st;
  if (dout == nullptr || dq == nullptr || dk == nullptr || dv == nullptr) return SWZ_ERR_INVALID_ARG;
  st = check_heads(*dout, *dq, *dk, *dv);
  if (st != SWZ_OK) return st;
  if (!aligned(workspace, 16) || dout->token >= kRowDistance) return SWZ_ERR_UNSUPPORTED;
  const int64_t bytes = swz_attention_backward_workspace(args);
  if (bytes > 0 && (workspace == nullptr || workspace_bytes < bytes)) return SWZ_ERR_INVALID_ARG;
  swz::PromptBackArgs p{};
  p.f = prompt_args(*args);
  p.dout = device_heads(*dout), p.dq = device_heads(*dq), p.dk = device_heads(*dk), p.dv = device_heads(*dv);
  p.log_sums = static_cast<float*>(workspace);
  p.deltas = p.log_sums + args->total_q * args->q_heads;
  const int splits = dkv_splits(*args);
  p.f.part_sums = p.log_sums + backward_floats(*args, 1);
  return for_head_dim(args->head_dim, [&](auto dim) {
    return for_flag(args->causal != 0, [&](auto causal) {
      constexpr int D = decltype(dim)::value;
      constexpr bool kCausal = decltype(causal)::value;
      using K = DkvShape<D>;
      const int heads = heads_together(*args);
      const int64_t q_slots = slots_of(args->total_q, args->sequences, 32 * kPromptWaves / heads), k_slots = slots_of(args->total_k, args->sequences, K::kKeys);
      const int64_t sum_slots = slots_of(args->total_k, args->sequences, swz::SumShape<D>::kKeys);
      const int group = args->q_heads / args->k_heads / heads;
      if (too_many_threads(q_slots, args->k_heads, group, p.f.num_xcd, 64 * kPromptWaves) || too_many_threads(k_slots * splits, args->k_heads, 1, p.f.num_xcd, K::kThreads) ||
          (splits > 1 && too_many_threads(sum_slots, args->k_heads, 1, p.f.num_xcd, swz::kSumThreads))) {
        return (int)SWZ_ERR_OVERFLOW;
      }
      int status = SWZ_OK;
      if (args->total_q > 0) {
        status = for_heads_together(heads, [&](auto together) {
          return launch_prompt<swz::attention_dq_kernel<D, kPromptWaves, decltype(together)::value, kCausal>>(p, p.f, q_slots, 1, group, 64 * kPromptWaves, stream);
        });
      }
      if (status != SWZ_OK || args->total_k == 0) return status;
      status = launch_prompt<swz::attention_dkv_kernel<D, K::kKeyWaves, K::kParts, kCausal>>(p, p.f, k_slots, splits, 1, K::kThreads, stream);
      if (status != SWZ_OK || splits == 1) return status;
      p.f.slots = (int)sum_slots;
      return launch(swz::attention_dkv_sum_kernel<D>, dim3((unsigned)swz::prompt_workgroups(sum_slots, args->k_heads, 1, p.f.num_xcd)), dim3(swz::kSumThreads), 0, stream, p);
    });
  });
}

int swz_cache4_append(const swz_cache4* cache, const swz_heads* k, const swz_heads* v, int64_t tokens, const int32_t* cu, const int32_t* before,
                      const int32_t* block_table, int32_t table_width, int32_t sequences, hipStream_t stream) {
  return store_or_read<false>(cache, k, v, tokens, cu, before, block_table, table_width, sequences, stream);
}

int swz_cache4_read(const swz_cache4* cache, const swz_heads* k, const swz_heads* v, int64_t tokens, const int32_t* cu, const int32_t* first,
                    const int32_t* block_table, int32_t table_width, int32_t sequences, hipStream_t stream) {
  return store_or_read<true>(cache, k, v, tokens, cu, first, block_table, table_width, sequences, stream);
}

int64_t swz_cache4_attention_workspace(const swz_cache4* cache, int32_t sequences, int32_t q_heads, int32_t table_width, int32_t max_length) {
  const int st = check_decode(cache, sequences, q_heads, table_width, max_length);
  if (st != SWZ_OK) return st;
  return decode_bytes(*cache, decode_plan(*cache, sequences, q_heads, table_width, max_length), sequences);
}

int swz_cache4_attention(const swz_cache4* cache, const swz_heads* q, const swz_heads* out, const int32_t* lengths, const int32_t* block_table,
                         int32_t table_width, int32_t sequences, int32_t q_heads, int32_t max_length, float scale, void* workspace, int64_t workspace_bytes,
                         hipStream_t stream) {
  int st = check_decode(cache, sequences, q_heads, table_width, max_length);
  if (st != SWZ_OK) return st;
  if (q == nullptr || out == nullptr || lengths == nullptr || block_table == nullptr || !(scale > 0.f) || !isfinite(scale)) return SWZ_ERR_INVALID_ARG;
  st = check_heads(*q, *out);
  if (st != SWZ_OK) return st;
  const DecodePlan p = decode_plan(*cache, sequences, q_heads, table_width, max_length);
  const int64_t bytes = decode_bytes(*cache, p, sequences);
  if (bytes > 0 && (workspace == nullptr || workspace_bytes < bytes)) return SWZ_ERR_INVALID_ARG;
  if (!aligned(lengths, 4) || !aligned(block_table, 4) || !aligned(workspace, 16)) return SWZ_ERR_UNSUPPORTED;
  swz::DecodeArgs a{};
  a.c = cache_args(*cache, block_table, table_width);
  a.q = device_heads(*q), a.out = device_heads(*out);
  a.lengths = lengths, a.sequences = sequences, a.q_heads = q_heads;
  a.columns = p.columns, a.shares = p.shares, a.scale = scale;
  a.sums = static_cast<float*>(workspace);
  a.stats = a.sums + decode_parts(*cache, p) * cache->head_dim;
  a.parts = reinterpret_cast<int2*>(a.stats + decode_parts(*cache, p) * 2);
  return for_head_dim(cache->head_dim, [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    const int64_t heads = (int64_t)cache->k_heads * p.columns, waves = p.shares * heads;
    if (2 * waves >= kTokens || sequences * heads >= kTokens || (int64_t)sequences * q_heads * 64 * swz::kJoinWaves > swz::kLaunchThreads || sequences * heads * 64 * swz::kOwnWaves > swz::kLaunchThreads) {
      return (int)SWZ_ERR_OVERFLOW;
    }
    if (p.shares == 0) {
      auto kernel = p.rows == 4 ? swz::cache4_attention_kernel<D, 4, true> : p.rows == 8 ? swz::cache4_attention_kernel<D, 8, true> : swz::cache4_attention_kernel<D, 16, true>;
      return launch(kernel, dim3((unsigned)(sequences * heads)), dim3(64 * swz::kOwnWaves), 0, stream, a);
    }
    const dim3 grid((unsigned)((waves + swz::kDecodeWaves - 1) / swz::kDecodeWaves)), block(64 * swz::kDecodeWaves);
    auto kernel = p.rows == 4 ? swz::cache4_attention_kernel<D, 4, false> : p.rows == 8 ? swz::cache4_attention_kernel<D, 8, false> : swz::cache4_attention_kernel<D, 16, false>;
    const int status = launch(kernel, grid, block, 0, stream, a);
    if (status != SWZ_OK) return status;
    return launch(swz::cache4_join_kernel<D>, dim3((unsigned)((int64_t)sequences * q_heads)), dim3(64 * swz::kJoinWaves), 0, stream, a, p.rows);
  });
}

}  // extern "C"
