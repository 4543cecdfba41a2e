// Attention of the drafted tokens of every sequence over a cache of pages in bfloat16: out = softmax(scale q k^T) v, a token looking at all positions before its block and at those of its block's tokens
// that a mask of 64 bits names, or (no masks) at those up to its own.
//
// The query heads of a key head look at the same keys, so a row is a token of one query head and the rows of a block are n * group.  Scores come as S^T = k q^T and out^T += v^T P^T, as for prompts
// (attention_tiles.h): a lane has 32 scores of one row.  Two kernels, by the rows of a tile:
// 32 or 64 (draft_attention_kernel): the four waves of a workgroup take every fourth tile of 64 keys each, for all the rows.  A wave has a tile of keys and one of values in LDS for itself and waits for nothing but
// its own loads, the next keys being fetched when the scores are done and the next values when those are used up; the four join what they have in LDS.
// 128 (draft_attention_wide_kernel): the waves have 32 rows each and share tiles, two of each, as for prompts: the scores of the next tile beside the weights and values of this one.
//
// The steps of all tiles of rows, in the sequences' order, are dealt evenly to the workgroups that a key head has, whatever the lengths: of `shares`, workgroup i has steps total * i / shares and up.  What it has
// of a tile of rows goes to `out` where that is all of it, else into one of two places of its own (the first it works on, or the last), and draft_join_kernel joins them.
#pragma once

#include "attention_kernel.h"
#include "paged.h"

namespace swz {

struct DraftArgs {
  PageTable c;
  const uint16_t *k_pages, *v_pages;
  Heads q, out;
  const int32_t *cu, *lengths;
  const uint64_t* tree;              // null: causal
  float *sums, *stats;               // places x rows x D, and x 2 (maximum, sum)
  int2* parts;                       // tiles of rows x key heads: place of the first part, share of the last (-1: one workgroup had all)
  int total, sequences, q_heads;
  int items;                         // tiles of rows that `parts` has room for, as many as there are
  int shares;                        // 0: a workgroup for each tile of rows and key head
  float scale;
};

constexpr int kDraftKeys = 64, kDraftWaves = 4;

// ROWS: 32 and 64, or 128 for the kernel whose waves share tiles.
template <int D, int ROWS>
struct DraftShape {
  static constexpr bool kWide = ROWS == 128;
  static constexpr int kStep = kDraftKeys * (kWide ? 1 : kDraftWaves);
  static constexpr int kTileBytes = kDraftKeys * 2 * D, kLdsBytes = 4 * kTileBytes * (kWide ? 1 : 2);
  static constexpr int kJoinPitch = D + 4;                  // floats of a row in LDS when waves join
  static constexpr int kPerCu = kWide || D == 64 ? 2 : 1;   // workgroups of a compute unit
};

// A tile of rows of a sequence.
struct DraftItem {
  int sequence, tile;
  Span tokens;
  int length;
};
__device__ __forceinline__ int draft_length(const DraftArgs& a, int sequence) {
  return (int)min((int64_t)max(a.lengths[sequence], 0), (int64_t)a.c.table_width << a.c.page_shift);
}

// Sum of x over this lane and those before it, at most 2^32 - 1: rising whatever is summed, where cu is not as it should be.
__device__ __forceinline__ uint32_t rising_sum(uint32_t x) {
  auto add = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
    x = __builtin_elementwise_add_sat(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
  };
  add(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});       // row_shr:1, 2, 4, 8
  add(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
  add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});       // row_bcast:15, to rows 1 and 3
  add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});       // row_bcast:31, to rows 2 and 3
  return x;
}
// Of sums over the lanes up to each: the last one, and the one before a lane.
__device__ __forceinline__ int64_t last_sum(uint32_t sum) { return (uint32_t)__builtin_amdgcn_readlane((int)sum, 63); }
__device__ __forceinline__ int64_t sum_up_to(uint32_t sum, int lane) { return lane == 0 ? 0 : (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)sum, lane - 1); }

// f(first sequence, tiles and steps of a tile of the lane's sequence) for 64 sequences at a time, until it says false.
template <int ROWS, int STEP, class F>
__device__ __forceinline__ void over_blocks(const DraftArgs& a, int group, F&& f) {
  for (int first = 0; first < a.sequences; first += 64) {
    const int b = first + (int)(threadIdx.x & 63);
    int tiles = 0, steps = 0;
    if (b < a.sequences) {
      const Span t = span_of(a.cu[b], a.cu[b + 1], a.total);
      tiles = (t.length * group + ROWS - 1) / ROWS;
      steps = (draft_length(a, b) + STEP - 1) / STEP;
    }
    if (!f(first, tiles, steps)) return;
  }
}
__device__ __forceinline__ DraftItem draft_item(const DraftArgs& a, int sequence, int tile) {
  return {sequence, tile, sequence_span(a.cu, sequence, a.total), __builtin_amdgcn_readfirstlane(draft_length(a, sequence))};
}

// The lowest c bits.
__device__ __forceinline__ uint64_t low_bits(int c) { return c >= 64 ? ~0ull : c <= 0 ? 0ull : (1ull << c) - 1; }
__device__ __forceinline__ uint64_t shift_up(uint64_t x, int by) { return by >= 64 || by <= -64 ? 0ull : by >= 0 ? x << by : x >> -by; }

__device__ const u32x4 kNanChunk = {0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};

// 64 positions of a head from their pages into LDS, 16 rows at a time (a page has 16 or more): those past the length are zeros, those without a page NaN.
template <int D>
struct PageLoader {
  static constexpr int kChunks = D / 8, kRows = 64 / kChunks, kLoads = 16 / kRows;          // of 16 rows
  const PageTable& c;
  int k_head, length, lane;
  uint32_t lane_part;

  __device__ __forceinline__ PageLoader(const PageTable& c_, int k_head_, int length_, int lane_) : c(c_), k_head(k_head_), length(length_), lane(lane_) {
    const int r = lane / kChunks;
    lane_part = (uint32_t)(r * 2 * D) + (uint32_t)(((lane % kChunks) ^ tile_key<D>(r)) << 4);
  }
  // position: of the first of 16, less than 2^31; page: theirs
  __device__ __forceinline__ void operator()(const uint16_t* pages, int64_t position, int page, uint32_t lds) const {
    const uint16_t* base = pages + c.token_at(max(page, 0), k_head, (int)position) * D;
    if (page >= 0 && position + 16 <= length) {
      const uint64_t at = reinterpret_cast<uint64_t>(base);
      const uint64_t uniform = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) load_to_lds_base_off(reinterpret_cast<const void*>(uniform), (uint32_t)(i * kRows * 2 * D) + (lane_part ^ key_of(i)), lds + (uint32_t)(i * 1024));
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        uint32_t l = (uint32_t)lane;
        keep(l);                     // or what this needs, once or twice for a sequence, has registers all along
        const int r = i * kRows + (int)l / kChunks;
        const unsigned char* at = reinterpret_cast<const unsigned char*>(base) + (uint32_t)(r * 2 * D) + ((l % kChunks ^ (uint32_t)tile_key<D>(r)) << 4);
        if (page < 0) at = reinterpret_cast<const unsigned char*>(&kNanChunk);
        if (position + r >= length) at = reinterpret_cast<const unsigned char*>(&kZeroChunk);
        load_to_lds(at, lds + (uint32_t)(i * 1024));
      }
    }
  }
  static __device__ __forceinline__ uint32_t key_of(int i) { return (uint32_t)(tile_key<D>(i * kRows) << 4); }
};

// The positions of a tile of which a value is no finite number.
template <int D>
__device__ __forceinline__ uint64_t odd_positions(const unsigned char* tile, int lane) {
  constexpr int kChunks = D / 8, kRows = 64 / kChunks;
  uint32_t l = (uint32_t)lane;
  keep(l);
  uint64_t odd = 0;
#pragma unroll 1
  for (int i = 0; i < kDraftKeys / kRows; ++i) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(tile + i * 1024 + l * 16);
    bool mine = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) mine |= (x[e] & 0x7f80u) == 0x7f80u || (x[e] & 0x7f800000u) == 0x7f800000u;
    const uint64_t found = __ballot(mine);
    if (found == 0) continue;
#pragma unroll
    for (int r = 0; r < kRows; ++r) odd |= (found >> (r * kChunks) & ((1ull << kChunks) - 1)) != 0 ? 1ull << (i * kRows + r) : 0ull;
  }
  return odd;
}

// o += p x for a tile that rows look at in part.  A product carries 0 times an infinity into rows that do not look at it: positions with values that are no finite numbers are left out of it, and then
// taken one at a time, by a product of their own that only the rows keep that look at them.
template <int D>
__device__ __forceinline__ void add_seen(f32x16 (&o)[D / 32], const u32x4 (&p)[4], const unsigned char* tile, uint32_t lds, uint64_t seen, int lane) {
  const uint64_t odd = odd_positions<D>(tile, lane);
  uint32_t l = (uint32_t)lane;
  keep(l);
  const uint32_t column = column_address<D>(lds, (int)l);
  // of 16 positions, those that `bits` names: element e of lane half h is 8 (e / 4) + 4 h + e % 4
  auto only = [&](bf16x8 f, uint32_t bits) __attribute__((always_inline)) {
    u32x4 w = __builtin_bit_cast(u32x4, f);
    bits >>= 4 * (l >> 5);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int at = 8 * (e / 2) + 2 * (e % 2);
      w[e] &= (bits >> at & 1u ? 0xffffu : 0u) | (bits >> (at + 1) & 1u ? 0xffff0000u : 0u);
    }
    return __builtin_bit_cast(bf16x8, w);
  };
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      o[i] = mfma32(only(read_columns<D>(column, k, i), (uint32_t)(~odd >> (16 * k)) & 0xffffu), __builtin_bit_cast(bf16x8, p[k]), o[i]);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll 1
  for (uint64_t rest = odd; rest != 0; rest &= rest - 1) {
    const int at = __ffsll((unsigned long long)rest) - 1, k = at >> 4;
    const bool looks = seen >> at & 1;
    u32x4 w = p[0];
#pragma unroll
    for (int e = 1; e < 4; ++e) w = k == e ? p[e] : w;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const f32x16 with = mfma32(only(read_columns<D>(column + (uint32_t)(k * 32 * D), 0, i), 1u << (at & 15)), __builtin_bit_cast(bf16x8, w), o[i]);
#pragma unroll
      for (int r = 0; r < 16; ++r) o[i][r] = looks ? with[r] : o[i][r];
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// The rows of a wave: 32 of a tile.
struct DraftRows {
  int token, head;                   // the lane's row (past the last one: that)
  bool real;
  uint64_t mask;
  __device__ __forceinline__ DraftRows(const DraftArgs& a, const DraftItem& item, int row, int k_head, int group) {
    const int rows = item.tokens.length * group, at = min(row, rows - 1);
    token = at / group;
    head = k_head * group + at - token * group;
    real = row < rows;
    mask = a.tree != nullptr ? a.tree[item.tokens.first + token] : 0;
  }
  // The positions of a tile that the row looks at.
  __device__ __forceinline__ uint64_t seen(const DraftArgs& a, const DraftItem& item, int tile) const {
    const int first = tile * kDraftKeys, base = item.length - item.tokens.length;
    const uint64_t seen = a.tree != nullptr ? low_bits(base - first) | shift_up(mask, base - first) : low_bits(base + token + 1 - first);
    return seen & low_bits(item.length - first);
  }
};

// What a wave has of its rows: sums of weighted values, the maximum of scores times c, and this half's sum of weights.
template <int D>
struct DraftSums {
  f32x16 o[D / 32];
  float top, sum;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = f32x16{};
    top = -FLT_MAX;
    sum = 0.f;
  }
  // Scores that are as high as `high` (of this half) are to come.
  __device__ __forceinline__ void raise(float high, float c) {
    high = across_halves(high, [](float y, float z) { return fmaxf(y, z); }) * c;
    if (!__any(high > top + kLazyRise)) return;
    const float now = fmaxf(top, high), less = __builtin_amdgcn_exp2f(top - now);
    sum *= less;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] *= less;
    top = now;
  }
  // Scores of a tile to weights, rounded for the product.
  __device__ __forceinline__ void weigh(f32x16 (&x)[2], float c, u32x4 (&p)[4]) {
    float high = x[0][0];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) high = fmaxf(high, x[b][r]);
    raise(high, c);
    float sums[2] = {sum, 0.f};
#pragma unroll
    for (int m = 0; m < 16; ++m) {
      const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[m / 8][m % 8 * 2], c, -top)), w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[m / 8][m % 8 * 2 + 1], c, -top));
      sums[0] += w0;
      sums[1] += w1;
      p[m / 4][m % 4] = pack_bf16(w0, w1);
    }
    sum = sums[0] + sums[1];
  }
};
// Scores of positions that a row does not look at.
__device__ __forceinline__ void hide(f32x16 (&x)[2], uint64_t seen, int h) {
  const uint64_t mine = seen >> (4 * h);
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const uint32_t bits = (uint32_t)(mine >> (32 * b));
#pragma unroll
    for (int r = 0; r < 16; ++r) x[b][r] = bits & (1u << (8 * (r / 4) + r % 4)) ? x[b][r] : -INFINITY;
  }
}

// The pages of the tiles that a wave will take, EVERY tiles apart: lane l has number l of them, `bits` (a power of two) a tile.
template <int EVERY>
struct PagesAhead {
  const PageTable& c;
  int sequence, length, lane, bits, pages, entry;
  __device__ __forceinline__ PagesAhead(const PageTable& c_, const DraftItem& item, int lane_) : c(c_), sequence(item.sequence), length(item.length), lane(lane_), bits(max(0, 6 - c_.page_shift)), pages(0), entry(0) {}
  __device__ __forceinline__ void look_up(int tile) {
    const int64_t position = ((int64_t)tile + (int64_t)(lane >> bits) * EVERY) * kDraftKeys + ((lane & ((1 << bits) - 1)) << c.page_shift);
    pages = position < length ? c.page_of(sequence, (int)position) : -1;
    entry = 0;
  }
  __device__ __forceinline__ void advance(int tile) {        // to `tile`, the one after that of `entry`
    if (++entry == 64 >> bits) look_up(tile);
  }
  // Of position `place` of a tile, `ahead` tiles after that of `entry`.
  __device__ __forceinline__ int operator()(int place) const { return __builtin_amdgcn_readlane(pages, (entry << bits) + (place >> c.page_shift)); }
};

// Deals the steps of all tiles of rows to workgroups: calls process(item, from, to, all, place) for each tile of rows of which steps from .. to - 1, of `all`, are this workgroup's; a part of one
// goes to `place`.
template <int D, int ROWS, class F>
__device__ __forceinline__ void deal(const DraftArgs& a, int share, int k_head, int group, F&& process) {
  constexpr int kStep = DraftShape<D, ROWS>::kStep;
  const int heads = a.c.k_heads;
  // `before` steps are those of the tiles before the sequence's, `items` the tiles
  int64_t my_start = 0, my_end = 0, before = 0, items = 0;
  int sequence = -1;
  if (a.shares == 0) {
    int tile = 0;
    over_blocks<ROWS, kStep>(a, group, [&](int first, int tiles, int) {
      const uint32_t sum = rising_sum((uint32_t)tiles);
      const uint64_t found = __ballot(share < items + sum);
      if (found == 0) {
        items += last_sum(sum);
        return true;
      }
      const int s = __ffsll((unsigned long long)found) - 1;
      sequence = first + s;
      items += sum_up_to(sum, s);
      tile = (int)(share - items);
      return false;
    });
    if (sequence < 0) return;
    const DraftItem item = draft_item(a, sequence, tile);
    const int all = (item.length + kStep - 1) / kStep;
    my_start = (int64_t)tile * all;
    my_end = my_start + all;
    if (all == 0) {                                          // rows that look at nothing
      const int rows = item.tokens.length * group;
      for (int i = (int)threadIdx.x; i < ROWS * (D / 8); i += 64 * kDraftWaves) {
        const int row = tile * ROWS + i / (D / 8);
        if (row < rows) *reinterpret_cast<u32x4*>(a.out.at(item.tokens.first + row / group, k_head * group + row % group) + i % (D / 8) * 8) = u32x4{};
      }
      return;
    }
  } else {
    int64_t total = 0;
    over_blocks<ROWS, kStep>(a, group, [&](int, int tiles, int steps) {
      total += last_sum(rising_sum((uint32_t)tiles * (uint32_t)steps));
      return true;
    });
    const int shares = (int)min((int64_t)a.shares, total);
    if (share >= shares) return;
    my_start = total * share / shares;
    my_end = total * (share + 1) / shares;
    over_blocks<ROWS, kStep>(a, group, [&](int first, int tiles, int steps) {
      const uint32_t sum = rising_sum((uint32_t)tiles * (uint32_t)steps), count = rising_sum((uint32_t)tiles);
      const uint64_t found = __ballot(my_start < before + sum);
      if (found == 0) {
        before += last_sum(sum);
        items += last_sum(count);
        return true;
      }
      const int s = __ffsll((unsigned long long)found) - 1;
      sequence = first + s;
      before += sum_up_to(sum, s);
      items += sum_up_to(count, s);
      return false;
    });
    if (sequence < 0) return;
  }
  for (int64_t step = my_start; step < my_end && sequence < a.sequences; ++sequence) {
    DraftItem item = draft_item(a, sequence, 0);
    const int tiles = (item.tokens.length * group + ROWS - 1) / ROWS, all = (item.length + kStep - 1) / kStep;
    for (item.tile = all > 0 ? (int)((step - before) / all) : tiles; item.tile < tiles && step < my_end; ++item.tile) {
      const int from = (int)(step - before - (int64_t)item.tile * all), count = (int)min((int64_t)(all - from), my_end - step);
      const int place = (share * heads + k_head) * 2 + (step == my_start ? 0 : 1);
      process(item, from, from + count, all, place);
      if (a.shares != 0 && threadIdx.x == 0 && items + item.tile < a.items) {
        int2* part = a.parts + (items + item.tile) * heads + k_head;
        if (from == 0) part->x = place;
        if (from + count == all) part->y = from == 0 ? -1 : share;
      }
      step += count;
    }
    items += tiles;
    before += (int64_t)tiles * all;
  }
}

template <int D, int ROWS>
__global__ void __launch_bounds__(64 * kDraftWaves, (DraftShape<D, ROWS>::kPerCu)) draft_attention_kernel(DraftArgs a) {
  using S = DraftShape<D, ROWS>;
  constexpr int kParts = D / 32, kSteps = D / 16, kTileLoads = S::kTileBytes / 1024, kBlocks = ROWS / 32;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S::kLdsBytes];
  __shared__ float wave_stats[kDraftWaves][32][2];
  const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  unsigned char *const k_tile = smem + 2 * wave * S::kTileBytes, *const v_tile = k_tile + S::kTileBytes;
  const uint32_t k_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)k_tile, v_lds = k_lds + (uint32_t)S::kTileBytes;
  const int heads = a.c.k_heads, group = a.q_heads / heads, share = (int)blockIdx.x / heads, k_head = (int)blockIdx.x - share * heads;
  const float c = a.scale * kLog2E;

  deal<D, ROWS>(a, share, k_head, group, [&](const DraftItem& item, int from, int to, int all, int place) {
    const int rows = item.tokens.length * group, first_row = item.tile * ROWS;
    bf16x8 qf[kBlocks][kSteps];
    DraftSums<D> sums[kBlocks];
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) {
      const DraftRows r(a, item, first_row + 32 * i + (lane & 31), k_head, group);
      load_fragments<D>(qf[i], a.q.at(item.tokens.first + r.token, r.head), lane);
      sums[i].clear();
    }
    const int end = min(to * kDraftWaves, (item.length + kDraftKeys - 1) / kDraftKeys);
    const int whole = min(item.length - item.tokens.length, item.length) / kDraftKeys;      // tiles that all rows look at whole (none where the block is longer than the sequence)
    int t = from * kDraftWaves + wave;
    const PageLoader<D> loader(a.c, k_head, item.length, lane);
    PagesAhead<kDraftWaves> pages(a.c, item, lane);
    auto fetch = [&](const uint16_t* from_pages, int tile, uint32_t lds) {
#pragma unroll
      for (int i = 0; i < 4; ++i) loader(from_pages, (int64_t)tile * kDraftKeys + 16 * i, pages(16 * i), lds + (uint32_t)(16 * i * 2 * D));
    };
    if (t < end) {
      pages.look_up(t);
      fetch(a.k_pages, t, k_lds);
      fetch(a.v_pages, t, v_lds);
    }
    auto take = [&](auto is_masked) __attribute__((always_inline)) {
      constexpr bool masked = decltype(is_masked)::value;
      const int then = t + kDraftWaves;
      const bool more = then < end;
      f32x16 x[kBlocks][2];
      u32x4 p[kBlocks][4];
      __builtin_amdgcn_sched_barrier(0);
      wait_vmcnt<kTileLoads>();                              // the keys have landed, the values may be on their way
      __builtin_amdgcn_sched_barrier(0);
      const uint32_t k_lane = row_address<D>(k_lds, lane);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int j = 0; j < kBlocks; ++j) x[j][b] = f32x16{};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          const bf16x8 f = read_rows<D>(k_lane, b, i);
#pragma unroll
          for (int j = 0; j < kBlocks; ++j) x[j][b] = mfma32(f, qf[j][i], x[j][b]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      wait_vmcnt_lgkmcnt<63, 0>();
      __builtin_amdgcn_sched_barrier(0);
      if (more) {
        pages.advance(then);
        fetch(a.k_pages, then, k_lds);
      }
      uint64_t seen[kBlocks];
#pragma unroll
      for (int j = 0; j < kBlocks; ++j) {
        if constexpr (masked) {
          seen[j] = DraftRows(a, item, first_row + 32 * j + (lane & 31), k_head, group).seen(a, item, t);
          hide(x[j], seen[j], h);
        }
        sums[j].weigh(x[j], c, p[j]);
      }
      __builtin_amdgcn_sched_barrier(0);
      if (more) wait_vmcnt<kTileLoads>();
      else wait_vmcnt<0>();
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (masked) {
#pragma unroll
        for (int j = 0; j < kBlocks; ++j) add_seen<D>(sums[j].o, p[j], v_tile, v_lds, seen[j], lane);
      } else {
        const uint32_t v_lane = column_address<D>(v_lds, lane);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int i = 0; i < kParts; ++i) {
            const bf16x8 f = read_columns<D>(v_lane, k, i);
#pragma unroll
            for (int j = 0; j < kBlocks; ++j) sums[j].o[i] = mfma32(f, __builtin_bit_cast(bf16x8, p[j][k]), sums[j].o[i]);
          }
      }
      __builtin_amdgcn_sched_barrier(0);
      wait_vmcnt_lgkmcnt<63, 0>();
      __builtin_amdgcn_sched_barrier(0);
      if (more) fetch(a.v_pages, then, v_lds);
      t = then;
    };
    while (t < min(whole, end)) take(std::false_type{});
    while (t < end) take(std::true_type{});

    // 32 rows at a time: every wave's into its own tiles, then a row by 8 threads
    const bool entire = from == 0 && to == all;
#pragma unroll
    for (int j = 0; j < kBlocks; ++j) {
      const float sum = across_halves(sums[j].sum, [](float y, float z) { return y + z; });
      float* mine = reinterpret_cast<float*>(k_tile) + (lane & 31) * S::kJoinPitch;
#pragma unroll
      for (int i = 0; i < kParts; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 4) *reinterpret_cast<f32x4*>(mine + 32 * i + 2 * r + 4 * h) = f32x4{sums[j].o[i][r], sums[j].o[i][r + 1], sums[j].o[i][r + 2], sums[j].o[i][r + 3]};
      if (h == 0) wave_stats[wave][lane & 31][0] = sums[j].top, wave_stats[wave][lane & 31][1] = sum;
      __syncthreads();
      const int r = (int)threadIdx.x / 8, d = (int)threadIdx.x % 8 * (D / 8), its = first_row + 32 * j + r;
      if (its < rows) {
        float factor[kDraftWaves], high = -FLT_MAX, total = 0.f;
#pragma unroll
        for (int w = 0; w < kDraftWaves; ++w) high = fmaxf(high, wave_stats[w][r][0]);
#pragma unroll
        for (int w = 0; w < kDraftWaves; ++w) {
          factor[w] = __builtin_amdgcn_exp2f(wave_stats[w][r][0] - high);
          total = __builtin_fmaf(wave_stats[w][r][1], factor[w], total);
        }
        const float f = !entire ? 1.f : total == 0.f ? 0.f : 1.f / total;
        float y[D / 8];
#pragma unroll
        for (int e = 0; e < D / 8; ++e) {
          y[e] = 0.f;
#pragma unroll
          for (int w = 0; w < kDraftWaves; ++w) y[e] = __builtin_fmaf(reinterpret_cast<const float*>(smem + 2 * w * S::kTileBytes)[r * S::kJoinPitch + d + e], factor[w], y[e]);
          y[e] *= f;
        }
        if (entire) {
          uint16_t* to_row = a.out.at(item.tokens.first + its / group, k_head * group + its % group) + d;
#pragma unroll
          for (int e = 0; e < D / 8; e += 8) {
            float z[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = y[e + i];
            *reinterpret_cast<u32x4*>(to_row + e) = pack8(z);
          }
        } else {
          const int64_t at = (int64_t)place * ROWS + 32 * j + r;
#pragma unroll
          for (int e = 0; e < D / 8; e += 4) *reinterpret_cast<f32x4*>(a.sums + at * D + d + e) = f32x4{y[e], y[e + 1], y[e + 2], y[e + 3]};
          if (d == 0) *reinterpret_cast<float2*>(a.stats + 2 * at) = float2{high, total};
        }
      }
      __syncthreads();
    }
  });
}

template <int D>
__global__ void __launch_bounds__(64 * kDraftWaves, 2) draft_attention_wide_kernel(DraftArgs a) {
  constexpr int ROWS = 128;
  using S = DraftShape<D, ROWS>;
  constexpr int kParts = D / 32, kSteps = D / 16;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S::kLdsBytes];
  const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const int heads = a.c.k_heads, group = a.q_heads / heads, share = (int)blockIdx.x / heads, k_head = (int)blockIdx.x - share * heads;
  const float c = a.scale * kLog2E;

  deal<D, ROWS>(a, share, k_head, group, [&](const DraftItem& item, int from, int to, int all, int place) {
    const DraftRows row(a, item, item.tile * ROWS + wave * 32 + (lane & 31), k_head, group);
    bf16x8 qf[kSteps];
    load_fragments<D>(qf, a.q.at(item.tokens.first + row.token, row.head), lane);
    DraftSums<D> sums;
    sums.clear();
    const int whole = min(item.length - item.tokens.length, item.length) / kDraftKeys;
    const PageLoader<D> loader(a.c, k_head, item.length, lane);
    PagesAhead<1> k_page(a.c, item, lane), v_page(a.c, item, lane);
    // this wave's quarter of a tile
    auto fetch = [&](const uint16_t* from_pages, const PagesAhead<1>& pages, int tile, int slot) {
      loader(from_pages, (int64_t)tile * kDraftKeys + 16 * wave, pages(16 * wave), lds + (uint32_t)(slot * S::kTileBytes + 16 * wave * 2 * D));
    };
    auto fetch_k = [&](int t) { fetch(a.k_pages, k_page, t, (t - from) & 1); };
    auto fetch_v = [&](int t) { fetch(a.v_pages, v_page, t, 2 + ((t - from) & 1)); };
    // keys of a tile are fetched two tiles ahead, values one
    k_page.look_up(from);
    v_page.look_up(from);
    fetch_k(from);
    fetch_v(from);
    if (from + 1 < to) {
      k_page.advance(from + 1);
      fetch_k(from + 1);
    }
    auto turn = [&](int t) {
      publish();
      if (t + 2 < to) {
        k_page.advance(t + 2);
        fetch_k(t + 2);
      }
      if (t + 1 < to) {
        v_page.advance(t + 1);
        fetch_v(t + 1);
      }
    };
    f32x16 x[2];
    auto score = [&](int t) __attribute__((always_inline)) {
      const uint32_t k_lane = row_address<D>(lds + (uint32_t)(((t - from) & 1) * S::kTileBytes), lane);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        x[b] = f32x16{};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) x[b] = mfma32(read_rows<D>(k_lane, b, i), qf[i], x[b]);
      }
    };
    publish();
    score(from);
    auto take = [&](int t, auto is_masked) __attribute__((always_inline)) {
      constexpr bool masked = decltype(is_masked)::value;
      turn(t);
      uint64_t seen = 0;
      if constexpr (masked) {
        seen = row.seen(a, item, t);
        hide(x, seen, h);
      }
      if (!masked || __any(seen != 0)) {
        u32x4 p[4];
        sums.weigh(x, c, p);
        const int slot = 2 + ((t - from) & 1);
        if constexpr (masked) {
          add_seen<D>(sums.o, p, smem + slot * S::kTileBytes, lds + (uint32_t)(slot * S::kTileBytes), seen, lane);
        } else {
          const uint32_t v_lane = column_address<D>(lds + (uint32_t)(slot * S::kTileBytes), lane);
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < kParts; ++i) sums.o[i] = mfma32(read_columns<D>(v_lane, k, i), __builtin_bit_cast(bf16x8, p[k]), sums.o[i]);
        }
      }
      if (t + 1 < to) score(t + 1);
    };
    int t = from;
    for (; t < min(whole, to); ++t) take(t, std::false_type{});
    for (; t < to; ++t) take(t, std::true_type{});
    publish();                                               // the tiles have been read

    const float sum = across_halves(sums.sum, [](float y, float z) { return y + z; });
    if (from == 0 && to == all) {
      store_columns<D>(sums.o, sum == 0.f ? 0.f : 1.f / sum, a.out.at(item.tokens.first + row.token, row.head), row.real, lane);
    } else if (row.real) {
      const int64_t at = (int64_t)place * ROWS + wave * 32 + (lane & 31);
      if (h == 0) *reinterpret_cast<float2*>(a.stats + 2 * at) = float2{sums.top, sum};
#pragma unroll
      for (int i = 0; i < kParts; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 4) *reinterpret_cast<f32x4*>(a.sums + at * D + 32 * i + 2 * r + 4 * h) = f32x4{sums.o[i][r], sums.o[i][r + 1], sums.o[i][r + 2], sums.o[i][r + 3]};
    }
  });
}

// What several workgroups have of a row joined, a wave for each token and query head, D / 64 dimensions a lane; and zeros for sequences without positions.
template <int D, int ROWS>
__global__ void __launch_bounds__(256) draft_join_kernel(DraftArgs a) {
  constexpr int kPer = D / 64;
  typedef __attribute__((ext_vector_type(kPer))) float vec;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int64_t id = (int64_t)blockIdx.x * 4 + wave;
  const int token = (int)(id / a.q_heads), head = (int)(id - (int64_t)token * a.q_heads);
  if (token >= a.total) return;
  const int heads = a.c.k_heads, group = a.q_heads / heads, k_head = head / group;
  int64_t items = 0;
  int sequence = -1, first_token = 0;
  for (int first = 0; first < a.sequences && sequence < 0; first += 64) {
    const int b = first + lane;
    Span t = {0, 0};
    if (b < a.sequences) t = span_of(a.cu[b], a.cu[b + 1], a.total);
    const int tiles = (t.length * group + ROWS - 1) / ROWS;
    const uint32_t sum = rising_sum((uint32_t)tiles);
    const uint64_t found = __ballot(t.first <= token && token < t.first + t.length);
    if (found == 0) {
      items += last_sum(sum);
      continue;
    }
    const int s = __ffsll((unsigned long long)found) - 1;
    sequence = first + s;
    items += sum_up_to(sum, s);
    first_token = __builtin_amdgcn_readlane(t.first, s);
  }
  if (sequence < 0) return;
  uint16_t* to = a.out.at(token, head) + lane * kPer;
  if (__builtin_amdgcn_readfirstlane(draft_length(a, sequence)) == 0) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) to[i] = 0;
    return;
  }
  const int row = (token - first_token) * group + head - k_head * group;
  const int64_t item = items + row / ROWS;
  if (item >= a.items) return;                               // (not where cu rises)
  const int2 parts = a.parts[item * heads + k_head];
  const int last = __builtin_amdgcn_readfirstlane(parts.y);
  if (last < 0) return;                                      // one workgroup had all of it
  const int first_part = __builtin_amdgcn_readfirstlane(parts.x), first = first_part / 2 / heads;
  if (last >= a.shares || first_part < 0 || first > last) return;
  auto place = [&](int share) { return (int64_t)(share == first ? first_part : (share * heads + k_head) * 2) * ROWS + row % ROWS; };
  float top = -FLT_MAX, sum = 0.f;
  vec o = 0.f;
  // 64 parts at a time, a lane each for their statistics
  for (int from = first; from <= last; from += 64) {
    float2 x = {-FLT_MAX, 0.f};
    if (from + lane <= last) x = *reinterpret_cast<const float2*>(a.stats + 2 * place(from + lane));
    const float now = fmaxf(top, over_wave(x.x, [](float y, float z) { return fmaxf(y, z); })), less = __builtin_amdgcn_exp2f(top - now);
    const float weight = __builtin_amdgcn_exp2f(x.x - now);
    sum = sum * less + over_wave(x.y * weight, [](float y, float z) { return y + z; });
    o *= less;
    top = now;
    const int count = min(64, last - from + 1);
    for (int p = 0; p < count; ++p) o += *reinterpret_cast<const vec*>(a.sums + place(from + p) * D + lane * kPer) * __int_as_float(__builtin_amdgcn_readlane(__float_as_int(weight), p));
  }
  const float f = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int i = 0; i < kPer; ++i) to[i] = __builtin_bit_cast(uint16_t, (__bf16)(o[i] * f));
}

}  // namespace swz
