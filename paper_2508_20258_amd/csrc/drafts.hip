// libswz: C-ABI entry points of a step with drafted tokens (declared in include/swz_drafts.h).  Host side: argument checks, the split of the
// work, launches.  Nothing here allocates device memory or synchronises.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/swz_drafts.h"
#include "cache16_kernel.h"
#include "draft_attention_kernel.h"
#include "host_checks.h"
#include "verify_kernel.h"

namespace {

using namespace swz::host;
using swz::launch;

constexpr int64_t kCacheBytes = (int64_t)256 << 20;          // the memory-side cache: what is more is not found there again

int check_cache(const swz_cache16* c) {
  if (c == nullptr || c->k == nullptr || c->v == nullptr || c->pages < 1 || c->k_heads < 1) return SWZ_ERR_INVALID_ARG;
  if (!head_dim_ok(c->head_dim) || c->page_tokens < 16 || (c->page_tokens & (c->page_tokens - 1)) != 0 || !aligned(c->k, 16) || !aligned(c->v, 16)) return SWZ_ERR_UNSUPPORTED;
  return c->pages >= kTokens || c->k_heads > kMostHeads ? SWZ_ERR_OVERFLOW : SWZ_OK;
}

int check_blocks(const int32_t* cu, const int32_t* table, int64_t tokens, int32_t sequences, int32_t table_width) {
  if (cu == nullptr || table == nullptr || tokens < 0 || sequences < 1 || table_width < 1) return SWZ_ERR_INVALID_ARG;
  if (!aligned(cu, 4) || !aligned(table, 4)) return SWZ_ERR_UNSUPPORTED;
  return tokens > kMostKeys ? SWZ_ERR_OVERFLOW : SWZ_OK;
}

// Positions are 32-bit numbers in the kernels, whatever starts and lengths the device has: those of a table have to be.
bool too_many_positions(const swz_cache16& c, int32_t table_width) { return (int64_t)table_width * c.page_tokens > kMostKeys; }

swz::PageTable page_table(const swz_cache16& c, const int32_t* table, int table_width) {
  return {table, c.pages, __builtin_ctz((unsigned)c.page_tokens), c.k_heads, table_width};
}

int check_append(const swz_cache16* cache, const swz_append16_args* a) {
  int st = check_cache(cache);
  if (st != SWZ_OK) return st;
  if (a == nullptr || a->before == nullptr) return SWZ_ERR_INVALID_ARG;
  st = check_blocks(a->cu, a->block_table, a->tokens, a->sequences, a->table_width);
  if (st != SWZ_OK) return st;
  const bool turned = a->cos != nullptr, queries = a->q.data != nullptr;
  if ((a->sin != nullptr) != turned || (queries && !turned) || (queries && a->q_heads < 1) || (turned && a->table_rows < 0)) return SWZ_ERR_INVALID_ARG;
  if (a->tokens == 0) return SWZ_OK;
  st = check_heads(a->k, a->v);
  if (st != SWZ_OK) return st;
  if (queries && (st = check_heads(a->q, a->q_out)) != SWZ_OK) return st;
  if (!aligned(a->before, 4) || !aligned(a->positions, 4) || !aligned(a->cos, 16) || !aligned(a->sin, 16)) return SWZ_ERR_UNSUPPORTED;
  if (turned && (a->rotary_dim < 16 || a->rotary_dim > cache->head_dim || a->rotary_dim % 16 != 0)) return SWZ_ERR_UNSUPPORTED;
  return too_many_positions(*cache, a->table_width) || (queries && a->q_heads > kMostHeads) ? SWZ_ERR_OVERFLOW : SWZ_OK;
}

// ---------------------------------------------------------------- attention

int check_attention(const swz_cache16* cache, const swz_attention16_args* a) {
  int st = check_cache(cache);
  if (st != SWZ_OK) return st;
  if (a == nullptr || a->lengths == nullptr) return SWZ_ERR_INVALID_ARG;
  st = check_blocks(a->cu, a->block_table, a->tokens, a->sequences, a->table_width);
  if (st == SWZ_ERR_INVALID_ARG) return st;
  if (a->q_heads < 1 || a->q_heads % cache->k_heads != 0 || a->max_length < 0 || !(a->scale > 0.f) || !isfinite(a->scale)) return SWZ_ERR_INVALID_ARG;
  if (st != SWZ_OK) return st;
  if (!aligned(a->lengths, 4) || !aligned(a->tree, 8)) return SWZ_ERR_UNSUPPORTED;
  if (a->q_heads > kMostHeads || too_many_positions(*cache, a->table_width) || a->tokens * a->q_heads >= kTokens) return SWZ_ERR_OVERFLOW;
  return SWZ_OK;
}

struct AttentionPlan {
  int rows, shares;                  // of a tile; shares 0: a workgroup for each tile of rows and key head
  int64_t items;                     // tiles of rows, at most
  bool once;                         // an average block is one tile of rows
  int join_groups;
};

// f(integral_constant<int, D>, integral_constant<int, ROWS>)
template <class F>
auto for_shape(int d, int rows, F&& f) {
  return for_head_dim(d, [&](auto dim) {
    return rows == 32 ? f(dim, std::integral_constant<int, 32>{}) : rows == 64 ? f(dim, std::integral_constant<int, 64>{}) : f(dim, std::integral_constant<int, 128>{});
  });
}

// Rows of a tile.  32 heads of 128 sharing 8, us in tiles of 32, 64 and 128 rows: blocks of 32 rows, 32 sequences of 3000 positions 71, 74 and 91; of 64 rows 135, 74 and 88; of 192 381, 225 and 122.  Blocks of 128, 32 sequences
// of 512 to 8192 positions: 138 in tiles of 64, 96 in tiles of 128 (as two tiles of a block read its positions at different times; at the same time, in 32 sequences of 3000, 89 and 92).  Few positions are soon read
// again: blocks of 192 rows, 4 sequences of 500 positions 13, 14 and 17.  Heads of 64, 32 sequences of 3000: 32 rows 41, 39 and 51; 64 rows 46, 41 and 50; 128 rows 88, 47 and 52; 192 rows 133, 93 and 70, the slower one being taken for 65
// to 128 rows, by a tenth; and so it is for 32 rows in many sequences (heads of 128, 64 of 2000: 93, 84 and 99).  The average is of all blocks: one of 512 tokens over 4096 positions beside 64 single tokens over 2000 193, 134 and 151 (64 taken), one of 2048 over 8192 beside them 983, 465 and 435 (128 taken); heads of 64,
// sharing in twos, 64, 66 and 82 (32 taken), 217, 170 and 176 (128 taken).
int tile_rows(int64_t rows, int64_t longest) { return rows <= 32 ? 32 : rows <= 64 || longest <= 1024 ? 64 : 128; }

// A workgroup for each tile of rows and key head, or the steps of all of them dealt evenly and the parts joined.  The latter takes another launch and the parts' traffic, 6 us and theirs, the former as long as the longest tile, of
// about 2.7 us for 256 positions (4.2 with 128 rows); lengths are taken to be 0.6 of the longest on average.  Single tokens of 32 heads of 128 sharing 8, the one and the other: 16 sequences of 256 positions 8.8 us and 12.0,
// of 1024 21.0 and 21.7, of 2048 34.7 and 30.5; one of 512 11.4 and 13.7, of 1024 16.6 and 15.1, of 4096 49 and 18.  Blocks of 128 rows: 16 of 1024 28 and 41, one 25 and 16.
// Heads of 64, by the same figures: 16 sequences of 512 9.5 and 12.0, of 1024 13.0 and 15.4 (where the rule takes the latter, as for one, 12.5 and 10.8), of 2048 22 and 19; 64 of 1024 25.0 and 27.5, of 4096 89 and 88.
// A tile of rows whose parts are joined by one workgroup, or (of each 32 rows) by 8, each looking for the tile by itself.  Blocks of 1 and 8 tokens, both kinds of heads, us with the one and the other: where a tile has 5.3 parts
// 26.3 and 25.4, 7 parts 12.8 and 11.4 to 15.8 and 15.8, 4 parts 31.2 and 31.4 to 56.5 and 57.5, 2 parts 50.5 and 51.6 to 97.4 and 103.4.
AttentionPlan attention_plan(const swz_cache16& c, const swz_attention16_args& a) {
  const int64_t group = a.q_heads / c.k_heads, rows = (a.tokens + a.sequences - 1) / a.sequences * group;          // of an average block
  const int64_t cut = (int64_t)a.table_width * c.page_tokens, longest = a.max_length > 0 && a.max_length < cut ? a.max_length : cut;
  AttentionPlan p{};
  p.rows = tile_rows(rows, longest);
  p.once = rows <= p.rows;
  p.join_groups = 1;
  for_shape(c.head_dim, p.rows, [&](auto dim, auto of_tile) {
    using S = swz::DraftShape<decltype(dim)::value, decltype(of_tile)::value>;
    p.items = a.tokens * group / p.rows + a.sequences;
    const int64_t room = (int64_t)compute_units() * S::kPerCu, steps = (longest + S::kStep - 1) / S::kStep + S::kSwitch;
    const int64_t tiles = (a.tokens * group + p.rows - 1) / p.rows > a.sequences ? (a.tokens * group + p.rows - 1) / p.rows : a.sequences;       // about as many as there are
    const int64_t shares = room / c.k_heads < 1 ? 1 : room / c.k_heads < tiles * steps ? room / c.k_heads : tiles * steps;
    const double whole = (p.rows == 128 ? 4.2 : 2.7) / 256 * longest, filled = (double)tiles * c.k_heads / room;
    const double parts = (double)shares * c.k_heads * p.rows * c.head_dim * 4 * 2 / 5e6;
    if (whole * (filled > 1 ? filled : 1) <= 0.6 * whole * filled + 6 + parts) return 0;
    p.shares = (int)shares;
    p.join_groups = p.shares > 4 * tiles ? 8 : 1;          // by the parts of a tile of rows, about
    return 0;
  });
  return p;
}
// Steps of all tiles of rows fit 32 bits, whatever the lengths.
bool too_many_steps(const swz_cache16& c, const swz_attention16_args& a, const AttentionPlan& p) {
  const int64_t steps = ((int64_t)a.table_width * c.page_tokens + swz::kDraftKeys - 1) / swz::kDraftKeys + 8;       // and what a tile of rows counts more
  return p.items >= kTokens || steps * p.items >= kTokens;
}
int64_t attention_places(const swz_cache16& c, const AttentionPlan& p) { return (int64_t)p.shares * c.k_heads * 2 * p.rows; }
int64_t attention_bytes(const swz_cache16& c, const AttentionPlan& p) { return p.shares == 0 ? 0 : 4 * attention_places(c, p) * (c.head_dim + 2) + 8 * p.items * c.k_heads; }

// ---------------------------------------------------------------- verification

int check_verify(const swz_verify_args* a) {
  if (a == nullptr || a->target == nullptr || a->tokens == nullptr || a->cu == nullptr || a->uniforms == nullptr || a->accepted == nullptr || a->path == nullptr || a->token == nullptr) return SWZ_ERR_INVALID_ARG;
  if (a->vocab < 1 || a->total < 0 || a->sequences < 1 || a->target_pitch < a->vocab || (a->draft != nullptr && a->draft_pitch < a->vocab)) return SWZ_ERR_INVALID_ARG;
  if ((a->elem_bytes != 2 && a->elem_bytes != 4) || !aligned(a->target, a->elem_bytes) || !aligned(a->draft, a->elem_bytes)) return SWZ_ERR_UNSUPPORTED;
  if (!aligned(a->tokens, 4) || !aligned(a->cu, 4) || !aligned(a->uniforms, 4) || !aligned(a->accepted, 4) || !aligned(a->path, 4) || !aligned(a->token, 4) || !aligned(a->parents, 4)) return SWZ_ERR_UNSUPPORTED;
  if (a->vocab >= (1 << 30) || a->total >= kTokens || a->target_pitch >= kTokens || (a->draft != nullptr && a->draft_pitch >= kTokens)) return SWZ_ERR_OVERFLOW;
  const int64_t pieces = (a->vocab + swz::kPieceValues - 1) / swz::kPieceValues;
  return pieces * a->sequences * swz::kVerifyThreads > swz::kLaunchThreads || (int64_t)a->sequences * swz::kWalkThreads > swz::kLaunchThreads ? SWZ_ERR_OVERFLOW : SWZ_OK;
}
int verify_pieces(const swz_verify_args& a) { return (int)((a.vocab + swz::kPieceValues - 1) / swz::kPieceValues); }

template <class T, bool DRAWN>
int launch_verify(const swz::VerifyArgs& v, hipStream_t stream) {
  const dim3 block(swz::kVerifyThreads), grid((unsigned)((int64_t)v.sequences * v.pieces));
  int st;
  if (DRAWN && v.parents != nullptr) {
    st = launch(swz::verify_walk_kernel<T>, dim3((unsigned)v.sequences), dim3(swz::kWalkThreads), 0, stream, v);
    if (st == SWZ_OK) st = launch(swz::verify_sums_kernel<T, true, true>, grid, block, 0, stream, v);
  } else {
    st = launch(swz::verify_sums_kernel<T, DRAWN, false>, grid, block, 0, stream, v);
  }
  return st != SWZ_OK ? st : launch(swz::verify_token_kernel<T, DRAWN>, dim3((unsigned)v.sequences), block, 0, stream, v);
}

}  // namespace

extern "C" {

int swz_cache16_append(const swz_cache16* cache, const swz_append16_args* args, hipStream_t stream) {
  const int st = check_append(cache, args);
  if (st != SWZ_OK || args->tokens == 0) return st;
  swz::Append16Args a{};
  a.c = page_table(*cache, args->block_table, args->table_width);
  a.k_pages = static_cast<uint16_t*>(cache->k), a.v_pages = static_cast<uint16_t*>(cache->v);
  a.k = device_heads(args->k), a.v = device_heads(args->v);
  if (args->q.data != nullptr) a.q = device_heads(args->q), a.q_out = device_heads(args->q_out), a.q_heads = args->q_heads;
  a.cos = args->cos, a.sin = args->sin, a.positions = args->positions, a.cu = args->cu, a.before = args->before;
  a.table_rows = args->table_rows, a.total = (int)args->tokens, a.sequences = args->sequences, a.rotary = args->cos != nullptr ? args->rotary_dim : 0;
  return for_head_dim(cache->head_dim, [&](auto dim) {
    return for_flag(args->interleaved != 0, [&](auto interleaved) {
      constexpr int D = decltype(dim)::value, kHeads = 1024 / D, kWaves = swz::kAppendThreads / 64;
      const int blocks = (a.q_heads + 2 * a.c.k_heads + kHeads - 1) / kHeads;
      a.splits = args->tokens * blocks <= 32 * (int64_t)compute_units() ? blocks : 1;
      const int64_t workgroups = (args->tokens * a.splits + kWaves - 1) / kWaves;
      if (workgroups >= kTokens) return (int)SWZ_ERR_OVERFLOW;
      constexpr bool kInterleaved = decltype(interleaved)::value;
      const bool stream_out = args->tokens * (a.q_heads + 2 * a.c.k_heads) * D * 4 > kCacheBytes;
      return launch(stream_out ? swz::cache16_append_kernel<D, kInterleaved, true> : swz::cache16_append_kernel<D, kInterleaved, false>, dim3((unsigned)workgroups), dim3(swz::kAppendThreads), 0, stream, a);
    });
  });
}

int64_t swz_cache16_attention_workspace(const swz_cache16* cache, const swz_attention16_args* args) {
  const int st = check_attention(cache, args);
  if (st != SWZ_OK) return st;
  const AttentionPlan p = attention_plan(*cache, *args);
  return too_many_steps(*cache, *args, p) ? SWZ_ERR_OVERFLOW : attention_bytes(*cache, p);
}

int swz_cache16_attention(const swz_cache16* cache, const swz_attention16_args* args, void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  int st = check_attention(cache, args);
  if (st != SWZ_OK || args->tokens == 0) return st;
  st = check_heads(args->q, args->out);
  if (st != SWZ_OK) return st;
  const AttentionPlan p = attention_plan(*cache, *args);
  if (too_many_steps(*cache, *args, p)) return SWZ_ERR_OVERFLOW;
  const int64_t bytes = attention_bytes(*cache, p);
  if (bytes > 0 && (workspace == nullptr || workspace_bytes < bytes)) return SWZ_ERR_INVALID_ARG;
  if (!aligned(workspace, 16)) return SWZ_ERR_UNSUPPORTED;
  swz::DraftArgs a{};
  a.c = page_table(*cache, args->block_table, args->table_width);
  a.k_pages = static_cast<const uint16_t*>(cache->k), a.v_pages = static_cast<const uint16_t*>(cache->v);
  a.q = device_heads(args->q), a.out = device_heads(args->out);
  a.cu = args->cu, a.lengths = args->lengths, a.tree = reinterpret_cast<const uint64_t*>(args->tree);
  a.sums = static_cast<float*>(workspace);
  a.stats = a.sums + attention_places(*cache, p) * cache->head_dim;
  a.parts = reinterpret_cast<int2*>(a.stats + attention_places(*cache, p) * 2);
  a.total = (int)args->tokens, a.sequences = args->sequences, a.q_heads = args->q_heads, a.items = (int)p.items, a.shares = p.shares, a.scale = args->scale;
  const int64_t workgroups = (p.shares == 0 ? p.items : p.shares) * cache->k_heads, joins = p.shares == 0 ? 0 : p.items * (p.rows / 32) * p.join_groups * cache->k_heads;
  if (workgroups * 256 > swz::kLaunchThreads || joins * 256 > swz::kLaunchThreads) return SWZ_ERR_OVERFLOW;
  return for_shape(cache->head_dim, p.rows, [&](auto dim, auto rows) {
    constexpr int D = decltype(dim)::value, ROWS = decltype(rows)::value;
    auto kernel = [&] {
      if constexpr (ROWS == 32) return swz::draft_attention_kernel<D>;
      else return p.once ? swz::draft_attention_wide_kernel<D, ROWS, true> : swz::draft_attention_wide_kernel<D, ROWS, false>;
    }();
    const int status = launch(kernel, dim3((unsigned)workgroups), dim3(64 * swz::kDraftWaves), 0, stream, a);
    if (status != SWZ_OK || p.shares == 0) return status;
    return launch(p.join_groups > 1 ? swz::draft_join_kernel<D, ROWS, 8> : swz::draft_join_kernel<D, ROWS, 1>, dim3((unsigned)joins), dim3(256), 0, stream, a);
  });
}

int64_t swz_verify_drafts_workspace(const swz_verify_args* args) {
  const int st = check_verify(args);
  return st != SWZ_OK ? st : args->sequences * ((int64_t)sizeof(swz::VerifyState) + 16 * (int64_t)verify_pieces(*args));
}

int swz_verify_drafts(const swz_verify_args* args, void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  const int st = check_verify(args);
  if (st != SWZ_OK) return st;
  if (workspace == nullptr || workspace_bytes < swz_verify_drafts_workspace(args)) return SWZ_ERR_INVALID_ARG;
  if (!aligned(workspace, 16)) return SWZ_ERR_UNSUPPORTED;
  swz::VerifyArgs v{};
  v.target = args->target, v.draft = args->draft, v.target_pitch = args->target_pitch, v.draft_pitch = args->draft_pitch;
  v.tokens = args->tokens, v.parents = args->parents, v.cu = args->cu, v.uniforms = args->uniforms;
  v.accepted = args->accepted, v.path = args->path, v.token = args->token;
  v.total = (int)args->total, v.sequences = args->sequences, v.vocab = (int)args->vocab, v.pieces = verify_pieces(*args);
  v.states = static_cast<swz::VerifyState*>(workspace);
  v.sums = reinterpret_cast<double*>(v.states + args->sequences);
  return for_flag(args->draft != nullptr, [&](auto drawn) {
    constexpr bool kDrawn = decltype(drawn)::value;
    return args->elem_bytes == 4 ? launch_verify<float, kDrawn>(v, stream) : launch_verify<uint16_t, kDrawn>(v, stream);
  });
}

int swz_cache16_keep(const swz_cache16* cache, const int32_t* cu, const int32_t* before, const int32_t* path, const int32_t* accepted, int64_t tokens, const int32_t* block_table,
                     int32_t table_width, int32_t sequences, hipStream_t stream) {
  int st = check_cache(cache);
  if (st != SWZ_OK) return st;
  if (before == nullptr || path == nullptr || accepted == nullptr) return SWZ_ERR_INVALID_ARG;
  st = check_blocks(cu, block_table, tokens, sequences, table_width);
  if (st != SWZ_OK || tokens == 0) return st;
  if (!aligned(before, 4) || !aligned(path, 4) || !aligned(accepted, 4)) return SWZ_ERR_UNSUPPORTED;
  if (too_many_positions(*cache, table_width)) return SWZ_ERR_OVERFLOW;
  swz::Keep16Args a{};
  a.c = page_table(*cache, block_table, table_width);
  a.k_pages = static_cast<uint16_t*>(cache->k), a.v_pages = static_cast<uint16_t*>(cache->v);
  a.cu = cu, a.before = before, a.path = path, a.accepted = accepted, a.total = (int)tokens, a.sequences = sequences;
  const int64_t items = (int64_t)cache->k_heads * 2 * (cache->head_dim / 8);
  a.blocks = (int)((items + swz::kKeepThreads - 1) / swz::kKeepThreads);
  if ((int64_t)sequences * a.blocks >= kTokens) return SWZ_ERR_OVERFLOW;
  return for_head_dim(cache->head_dim, [&](auto dim) {
    return launch(swz::cache16_keep_kernel<decltype(dim)::value>, dim3((unsigned)(sequences * a.blocks)), dim3(swz::kKeepThreads), 0, stream, a);
  });
}

}  // extern "C"
