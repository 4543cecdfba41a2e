// Attention of the drafted tokens of every sequence over a cache of pages in bfloat16: out = softmax(scale q k^T) v, a token looking at all positions before its block and at those of its block's tokens
// that a mask of 64 bits names, or (no masks) at those up to its own.
//
// The query heads of a key head look at the same keys, so a row is a token of one query head and the rows of a block are n * group.  Scores come as S^T = k q^T and out^T += v^T P^T, as for prompts
// (attention_tiles.h).  A step over the keys is a tile of 64.  Two kernels, by the rows of a tile:
// 32 (draft_attention_kernel): the four waves of a workgroup take every fourth tile of keys each.  A wave has a tile of keys and one of values in LDS for itself and waits for nothing but its own loads, the next
// keys being fetched when the scores are done and the next values when those are used up; the four join what they have in LDS.
// 64 or 128 (draft_attention_wide_kernel): the waves have 32 rows each, or 32 rows and half of the keys, and share tiles, two of each: the scores of the next tile beside the weights and values of this one, in
// slots of one product, as for prompts (attention_kernel.h).
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

constexpr int kDraftKeys = 64, kDraftWaves = 4;        // keys of a tile; waves of a workgroup

template <int D, int ROWS>
struct DraftShape {
  static constexpr bool kWide = ROWS > 32;
  static constexpr int kStep = kDraftKeys * (kWide ? 1 : kDraftWaves);       // keys that the workgroup takes at a time
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

// Positions of a head from their pages into LDS, 16 rows at a time (a page has 16 or more): those from `length` on are zeros, those without a page NaN.
// STREAM: they are read once.
template <int D, bool STREAM>
struct PageLoader {
  static constexpr int kChunks = D / 8, kRows = 64 / kChunks, kLoads = 16 / kRows;          // of 16 rows
  const PageTable& c;
  int k_head, length, lane;
  uint32_t lane_part;

  __device__ __forceinline__ PageLoader(const PageTable& c_, int k_head_, int length_, int lane_) : c(c_), k_head(k_head_), length(length_), lane(lane_) {
    const int r = lane / kChunks;
    lane_part = (uint32_t)(r * 2 * D) + (uint32_t)(((lane % kChunks) ^ tile_key<D>(r)) << 4);
  }
  // Where 16 positions are: elements from the start of the pages, -1 where they have no page.
  __device__ __forceinline__ int64_t place(int64_t position, int page) const { return page < 0 ? -1 : c.token_at(page, k_head, (int)position) * D; }
  __device__ __forceinline__ void operator()(const uint16_t* pages, int64_t position, int64_t place, uint32_t lds) const {
    if (place >= 0 && position + 16 <= length) {
      const uint64_t at = reinterpret_cast<uint64_t>(pages + place);
      const uint64_t uniform = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const uint32_t off = (uint32_t)(i * kRows * 2 * D) + (lane_part ^ key_of(i)), to = lds + (uint32_t)(i * 1024);
        if constexpr (STREAM) stream_to_lds(reinterpret_cast<const void*>(uniform), off, to);
        else load_to_lds_base_off(reinterpret_cast<const void*>(uniform), off, to);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        uint32_t l = (uint32_t)lane;
        keep(l);                     // or what this needs, once or twice for a sequence, has registers all along
        const int r = i * kRows + (int)l / kChunks;
        const unsigned char* at = reinterpret_cast<const unsigned char*>(pages + max(place, (int64_t)0)) + (uint32_t)(r * 2 * D) + ((l % kChunks ^ (uint32_t)tile_key<D>(r)) << 4);
        if (place < 0) at = reinterpret_cast<const unsigned char*>(&kNanChunk);
        if (position + r >= length) at = reinterpret_cast<const unsigned char*>(&kZeroChunk);
        load_to_lds(at, lds + (uint32_t)(i * 1024));
      }
    }
  }
  static __device__ __forceinline__ uint32_t key_of(int i) { return (uint32_t)(tile_key<D>(i * kRows) << 4); }
};

// Of 32 NB positions, those of which a value is no finite number.
template <int D, int NB>
__device__ __forceinline__ uint64_t odd_positions(const unsigned char* tile, int lane) {
  constexpr int kChunks = D / 8, kRows = 64 / kChunks;
  uint32_t l = (uint32_t)lane;
  keep(l);
  uint64_t odd = 0;
#pragma unroll 1
  for (int i = 0; i < 32 * NB / kRows; ++i) {
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

// o += p x for 32 NB positions that rows look at in part.  A product carries 0 times an infinity into rows that do not look at it: positions with values that are no finite numbers are left out of it, and
// then taken one at a time, by a product of their own that only the rows keep that look at them.
template <int D, int NB>
__device__ __forceinline__ void add_seen(f32x16 (&o)[D / 32], const u32x4 (&p)[2 * NB], const unsigned char* tile, uint32_t lds, uint64_t seen, int lane) {
  const uint64_t odd = odd_positions<D, NB>(tile, lane);
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
  for (int k = 0; k < 2 * NB; ++k)
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
    for (int j = 1; j < 2 * NB; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = k == j ? p[j][e] : w[e];
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
  // Scores of 32 NB positions to weights, rounded for the product.
  template <int NB>
  __device__ __forceinline__ void weigh(f32x16 (&x)[NB], float c, u32x4 (&p)[2 * NB]) {
    float high[2] = {x[0][0], x[0][1]};
#pragma unroll
    for (int r = 2; r < 16 * NB; ++r) high[r % 2] = fmaxf(high[r % 2], x[r / 16][r % 16]);
    raise(fmaxf(high[0], high[1]), c);
    float sums[2] = {sum, 0.f};
#pragma unroll
    for (int m = 0; m < 8 * NB; ++m) {
      const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[m / 8][m % 8 * 2], c, -top)), w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[m / 8][m % 8 * 2 + 1], c, -top));
      sums[0] += w0;
      sums[1] += w1;
      p[m / 4][m % 4] = pack_bf16(w0, w1);
    }
    sum = sums[0] + sums[1];
  }
};
// Scores of positions that a row does not look at.
template <int NB>
__device__ __forceinline__ void hide(f32x16 (&x)[NB], uint64_t seen, int h) {
  const uint64_t mine = seen >> (4 * h);
#pragma unroll
  for (int b = 0; b < NB; ++b) {
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
  // Of position `place` of the tile.
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

template <int D>
__global__ void __launch_bounds__(64 * kDraftWaves, (DraftShape<D, 32>::kPerCu)) draft_attention_kernel(DraftArgs a) {
  constexpr int ROWS = 32;
  using S = DraftShape<D, ROWS>;
  constexpr int kParts = D / 32, kSteps = D / 16, kTileLoads = S::kTileBytes / 1024;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S::kLdsBytes];
  __shared__ float wave_stats[kDraftWaves][ROWS][2];
  const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  unsigned char *const k_tile = smem + 2 * wave * S::kTileBytes, *const v_tile = k_tile + S::kTileBytes;
  const uint32_t k_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)k_tile, v_lds = k_lds + (uint32_t)S::kTileBytes;
  const int heads = a.c.k_heads, group = a.q_heads / heads, share = (int)blockIdx.x / heads, k_head = (int)blockIdx.x - share * heads;
  const float c = a.scale * kLog2E;

  deal<D, ROWS>(a, share, k_head, group, [&](const DraftItem& item, int from, int to, int all, int place) {
    const int rows = item.tokens.length * group, first_row = item.tile * ROWS;
    const int end = min(to * kDraftWaves, (item.length + kDraftKeys - 1) / kDraftKeys);
    const int whole = min(min(item.length - item.tokens.length, item.length) / kDraftKeys, end);      // tiles that all rows look at whole (none where the block is longer than the sequence)
    int t = from * kDraftWaves + wave;
    const PageLoader<D, true> loader(a.c, k_head, item.length, lane);
    PagesAhead<kDraftWaves> pages(a.c, item, lane);
    int64_t places[4];
    auto fetch = [&](const uint16_t* from_pages, int tile, uint32_t lds) {
#pragma unroll
      for (int i = 0; i < 4; ++i) loader(from_pages, (int64_t)tile * kDraftKeys + 16 * i, places[i], lds + (uint32_t)(16 * i * 2 * D));
    };
    auto fetch_keys = [&](int tile) {                        // and note where the values are
#pragma unroll
      for (int i = 0; i < 4; ++i) places[i] = loader.place((int64_t)tile * kDraftKeys + 16 * i, pages(16 * i));
      fetch(a.k_pages, tile, k_lds);
    };
    if (t < end) {
      pages.look_up(t);
      fetch_keys(t);
      fetch(a.v_pages, t, v_lds);
    }
    const DraftRows row(a, item, first_row + (lane & 31), k_head, group);
    bf16x8 qf[kSteps];
    load_fragments<D>(qf, a.q.at(item.tokens.first + row.token, row.head), lane);
    DraftSums<D> sums;
    sums.clear();
    auto take = [&](auto is_masked) __attribute__((always_inline)) {
      constexpr bool masked = decltype(is_masked)::value;
      const int then = t + kDraftWaves;
      const bool more = then < end;
      f32x16 x[2];
      u32x4 p[4];
      __builtin_amdgcn_sched_barrier(0);
      wait_vmcnt<kTileLoads>();                              // the keys have landed, the values may be on their way
      __builtin_amdgcn_sched_barrier(0);
      const uint32_t k_lane = row_address<D>(k_lds, lane);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        x[b] = f32x16{};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) x[b] = mfma32(read_rows<D>(k_lane, b, i), qf[i], x[b]);
      }
      __builtin_amdgcn_sched_barrier(0);
      wait_vmcnt_lgkmcnt<63, 0>();
      __builtin_amdgcn_sched_barrier(0);
      if (more) {
        pages.advance(then);
        fetch_keys(then);
      }
      uint64_t seen = 0;
      if constexpr (masked) {
        seen = row.seen(a, item, t);
        hide(x, seen, h);
      }
      sums.weigh(x, c, p);
      __builtin_amdgcn_sched_barrier(0);
      if (more) wait_vmcnt<kTileLoads>();
      else wait_vmcnt<0>();
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (masked) {
        add_seen<D, 2>(sums.o, p, v_tile, v_lds, seen, lane);
      } else {
        const uint32_t v_lane = column_address<D>(v_lds, lane);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int i = 0; i < kParts; ++i) sums.o[i] = mfma32(read_columns<D>(v_lane, k, i), __builtin_bit_cast(bf16x8, p[k]), sums.o[i]);
      }
      __builtin_amdgcn_sched_barrier(0);
      wait_vmcnt_lgkmcnt<63, 0>();
      __builtin_amdgcn_sched_barrier(0);
      if (more) fetch(a.v_pages, then, v_lds);
      t = then;
    };
    while (t < whole) take(std::false_type{});
    while (t < end) take(std::true_type{});

    // every wave's sums into its own tiles, then a row by 8 threads
    const float sum = across_halves(sums.sum, [](float y, float z) { return y + z; });
    float* mine = reinterpret_cast<float*>(k_tile) + (lane & 31) * S::kJoinPitch;
#pragma unroll
    for (int i = 0; i < kParts; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += 4) *reinterpret_cast<f32x4*>(mine + 32 * i + 2 * r + 4 * h) = f32x4{sums.o[i][r], sums.o[i][r + 1], sums.o[i][r + 2], sums.o[i][r + 3]};
    if (h == 0) wave_stats[wave][lane & 31][0] = sums.top, wave_stats[wave][lane & 31][1] = sum;
    __syncthreads();
    const int r = (int)threadIdx.x / 8, d = (int)threadIdx.x % 8 * (D / 8), its = first_row + r;
    if (its < rows) {
      float factor[kDraftWaves], high = -FLT_MAX, total = 0.f;
#pragma unroll
      for (int w = 0; w < kDraftWaves; ++w) high = fmaxf(high, wave_stats[w][r][0]);
#pragma unroll
      for (int w = 0; w < kDraftWaves; ++w) {
        factor[w] = __builtin_amdgcn_exp2f(wave_stats[w][r][0] - high);
        total = __builtin_fmaf(wave_stats[w][r][1], factor[w], total);
      }
      const bool entire = from == 0 && to == all;
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
        const int64_t at = (int64_t)place * ROWS + r;
#pragma unroll
        for (int e = 0; e < D / 8; e += 4) *reinterpret_cast<f32x4*>(a.sums + at * D + d + e) = f32x4{y[e], y[e + 1], y[e + 2], y[e + 3]};
        if (d == 0) *reinterpret_cast<float2*>(a.stats + 2 * at) = float2{high, total};
      }
    }
    __syncthreads();
  });
}

// Pairs of weights taken before a slot, if all `pairs` of them are by slot `last`.
constexpr int pairs_before(int slot, int pairs, int last) { return slot >= last ? pairs : (slot * pairs + last - 1) / last; }

// STREAM: most blocks are one tile of rows, so that keys and values are read once.
template <int D, int ROWS, bool STREAM>
__global__ void __launch_bounds__(64 * kDraftWaves, 2) draft_attention_wide_kernel(DraftArgs a) {
  using S = DraftShape<D, ROWS>;
  constexpr int kParts = D / 32, kSteps = D / 16, kBlocks = ROWS / 64, kRowWaves = ROWS / 32;     // a wave has 32 kBlocks of a tile's keys
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S::kLdsBytes];
  const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), row_wave = wave % kRowWaves, part = wave / kRowWaves;
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem, mine = (uint32_t)(part * 64 * D);      // of a tile: the wave's keys
  const int heads = a.c.k_heads, group = a.q_heads / heads, share = (int)blockIdx.x / heads, k_head = (int)blockIdx.x - share * heads;
  const float c = a.scale * kLog2E;

  deal<D, ROWS>(a, share, k_head, group, [&](const DraftItem& item, int from, int to, int all, int place) {
    const int whole = min(min(item.length - item.tokens.length, item.length) / kDraftKeys, to);
    const PageLoader<D, STREAM> loader(a.c, k_head, item.length, lane);
    PagesAhead<1> pages(a.c, item, lane);
    // The keys of tile t are in slot (t - from) & 1, the values in 2 + that; a wave fetches a quarter of a tile.  Keys are fetched two tiles ahead, values one, from the places that the keys had.
    int64_t key_place = 0, value_place = 0;
    auto fetch_k = [&](int t) {
      value_place = key_place;
      key_place = loader.place((int64_t)t * kDraftKeys + 16 * wave, pages(16 * wave));
      pages.advance(t + 1);
      loader(a.k_pages, (int64_t)t * kDraftKeys + 16 * wave, key_place, lds + (uint32_t)(((t - from) & 1) * S::kTileBytes + 16 * wave * 2 * D));
    };
    auto fetch_v = [&](int t, int64_t at) { loader(a.v_pages, (int64_t)t * kDraftKeys + 16 * wave, at, lds + (uint32_t)((2 + ((t - from) & 1)) * S::kTileBytes + 16 * wave * 2 * D)); };
    pages.look_up(from);
    fetch_k(from);
    fetch_v(from, key_place);
    if (from + 1 < to) fetch_k(from + 1);
    auto turn = [&](int t) __attribute__((always_inline)) {
      publish();
      if (t + 2 < to) {
        fetch_k(t + 2);
        fetch_v(t + 1, value_place);
      } else if (t + 1 < to) {
        fetch_v(t + 1, key_place);
      }
    };
    const DraftRows row(a, item, item.tile * ROWS + row_wave * 32 + (lane & 31), k_head, group);
    bf16x8 qf[kSteps];
    load_fragments<D>(qf, a.q.at(item.tokens.first + row.token, row.head), lane);
    DraftSums<D> sums;
    sums.clear();
    f32x16 x[kBlocks], other[kBlocks];
    auto score = [&](int t) __attribute__((always_inline)) {
      const uint32_t k_lane = row_address<D>(lds + mine + (uint32_t)(((t - from) & 1) * S::kTileBytes), lane);
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        x[b] = f32x16{};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) x[b] = mfma32(read_rows<D>(k_lane, b, i), qf[i], x[b]);
      }
    };
    // One tile that all rows look at whole, and the scores of the next one, another such: kSlots products with the vector unit's share of the work in each, in a fixed order.  The weights come in pairs, all of them by
    // slot kLast, so that each is there before the products that take it.
    constexpr int kScoreSlots = kBlocks * kSteps, kSlots = kScoreSlots + 2 * kBlocks * kParts, kPairs = 8 * kBlocks, kLast = kBlocks == 2 ? kSlots * 7 / 8 : kSlots * 3 / 4;
    uint32_t k_at[kSteps], v_at[kParts][2];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) keep(k_at[i] = row_address<D>(lds + mine, lane) ^ (uint32_t)(i << 5));
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      keep(v_at[i][0] = column_address<D>(lds + mine, lane) ^ (uint32_t)(i << 6));
      keep(v_at[i][1] = (column_address<D>(lds + mine, lane) ^ (uint32_t)(i << 6) ^ 32u) + 16u * D);
    }
    auto tile_pass = [&](f32x16 (&now)[kBlocks], f32x16 (&then)[kBlocks], auto parity) __attribute__((always_inline)) {
      constexpr int PARITY = decltype(parity)::value;
      constexpr uint32_t kKeysAt = (uint32_t)((PARITY ? 0 : 1) * S::kTileBytes), kValuesAt = (uint32_t)((2 + PARITY) * S::kTileBytes);
      auto read = [&](auto slot) __attribute__((always_inline)) {
        constexpr int i = decltype(slot)::value, v = i - kScoreSlots;
        if constexpr (i < kScoreSlots) return read_rows_at<D>(k_at[i % kSteps], kKeysAt + (uint32_t)(i / kSteps * 64 * D));
        else return read_columns_at<D>(v_at[v % kParts][0], v_at[v % kParts][1], kValuesAt + (uint32_t)(v / kParts * 32 * D));
      };
      u32x4 p[2 * kBlocks];
      constexpr int kAhead = 2, kRing = kAhead + 1;          // reads on their way
      bf16x8 f[kRing];
      for_each_index([&](auto slot) __attribute__((always_inline)) { f[decltype(slot)::value] = read(slot); }, std::make_integer_sequence<int, kAhead>{});
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) then[b] = f32x16{};
      float weights[2] = {sums.sum, 0.f}, high[2] = {-INFINITY, -INFINITY};
      now[0][0] = __builtin_fmaf(now[0][0], c, -sums.top);
      now[0][1] = __builtin_fmaf(now[0][1], c, -sums.top);
      __builtin_amdgcn_sched_barrier(0);
      for_each_index([&](auto slot) __attribute__((always_inline)) {
        constexpr int i = decltype(slot)::value, v = i - kScoreSlots;
        if constexpr (i + kAhead < kSlots) f[(i + kAhead) % kRing] = read(std::integral_constant<int, i + kAhead>{});
        if constexpr (i < kScoreSlots) then[i / kSteps] = mfma32(f[i % kRing], qf[i % kSteps], then[i / kSteps]);
        else sums.o[v % kParts] = mfma32(f[i % kRing], __builtin_bit_cast(bf16x8, p[v / kParts]), sums.o[v % kParts]);
        constexpr int kTaken = pairs_before(i, kPairs, kLast), kThen = pairs_before(i + 1, kPairs, kLast);
        static_assert(i < kScoreSlots || kTaken >= (v / kParts + 1) * 4, "weights are there before they are used");
#pragma unroll
        for (int n = kTaken; n < kThen; ++n) {
          const int b = n / 8, r = n % 8 * 2, m = n + 1;
          if (m < kPairs) {
            now[m / 8][m % 8 * 2] = __builtin_fmaf(now[m / 8][m % 8 * 2], c, -sums.top);
            now[m / 8][m % 8 * 2 + 1] = __builtin_fmaf(now[m / 8][m % 8 * 2 + 1], c, -sums.top);
          }
          const float w0 = __builtin_amdgcn_exp2f(now[b][r]), w1 = __builtin_amdgcn_exp2f(now[b][r + 1]);
          weights[0] += w0;
          weights[1] += w1;
          p[n / 4][n % 4] = pack_bf16(w0, w1);
        }
        if constexpr (i >= kScoreSlots) {
          constexpr int kValueSlots = kSlots - kScoreSlots;
#pragma unroll
          for (int e = v * 16 * kBlocks / kValueSlots; e < (v + 1) * 16 * kBlocks / kValueSlots; e += 2)
            high[e / 2 % 2] = __builtin_elementwise_maximum(high[e / 2 % 2], __builtin_elementwise_maximum(then[e / 16][e % 16], then[e / 16][e % 16 + 1]));
        }
        __builtin_amdgcn_sched_barrier(0);
      }, std::make_integer_sequence<int, kSlots>{});
      sums.sum = weights[0] + weights[1];
      sums.raise(fmaxf(high[0], high[1]), c);
    };
    // A tile after the other, the scores of tile t being there.
    auto take = [&](int t, auto is_masked) __attribute__((always_inline)) {
      constexpr bool masked = decltype(is_masked)::value;
      turn(t);
      const uint32_t values = mine + (uint32_t)((2 + ((t - from) & 1)) * S::kTileBytes);
      u32x4 p[2 * kBlocks];
      if constexpr (masked) {
        const uint64_t seen = row.seen(a, item, t) >> (32 * part) & (~0ull >> (64 - 32 * kBlocks));
        hide(x, seen, h);
        if (__any(seen != 0)) {
          sums.weigh(x, c, p);
          add_seen<D, kBlocks>(sums.o, p, smem + values, lds + values, seen, lane);
        }
      } else {
        sums.weigh(x, c, p);
        const uint32_t v_lane = column_address<D>(lds + values, lane);
#pragma unroll
        for (int k = 0; k < 2 * kBlocks; ++k)
#pragma unroll
          for (int i = 0; i < kParts; ++i) sums.o[i] = mfma32(read_columns<D>(v_lane, k, i), __builtin_bit_cast(bf16x8, p[k]), sums.o[i]);
      }
      if (t + 1 < to) score(t + 1);
    };
    publish();
    score(from);
    int t = from;
    if (t + 2 < whole) {
      float high = x[0][0];
#pragma unroll
      for (int r = 1; r < 16 * kBlocks; ++r) high = fmaxf(high, x[r / 16][r % 16]);
      sums.raise(high, c);
      for (; t + 2 < whole; t += 2) {
        turn(t);
        tile_pass(x, other, std::integral_constant<int, 0>{});
        turn(t + 1);
        tile_pass(other, x, std::integral_constant<int, 1>{});
      }
    }
    for (; t < whole; ++t) take(t, std::false_type{});
    for (; t < to; ++t) take(t, std::true_type{});
    publish();                                               // the tiles have been read

    sums.sum = across_halves(sums.sum, [](float y, float z) { return y + z; });
    if constexpr (kRowWaves < kDraftWaves) {
      // the other half of the keys
      float* its = reinterpret_cast<float*>(smem) + (row_wave * 32 + (lane & 31)) * S::kJoinPitch;
      float* its_stats = reinterpret_cast<float*>(smem) + ROWS * S::kJoinPitch + 2 * (row_wave * 32 + (lane & 31));
      if (part == 1) {
#pragma unroll
        for (int i = 0; i < kParts; ++i)
#pragma unroll
          for (int r = 0; r < 16; r += 4) *reinterpret_cast<f32x4*>(its + 32 * i + 2 * r + 4 * h) = f32x4{sums.o[i][r], sums.o[i][r + 1], sums.o[i][r + 2], sums.o[i][r + 3]};
        if (h == 0) its_stats[0] = sums.top, its_stats[1] = sums.sum;
      }
      __syncthreads();
      if (part == 0) {
        const float high = fmaxf(sums.top, its_stats[0]), f = __builtin_amdgcn_exp2f(sums.top - high), g = __builtin_amdgcn_exp2f(its_stats[0] - high);
        sums.top = high;
        sums.sum = __builtin_fmaf(its_stats[1], g, sums.sum * f);
#pragma unroll
        for (int i = 0; i < kParts; ++i)
#pragma unroll
          for (int r = 0; r < 16; r += 4) {
            const f32x4 y = *reinterpret_cast<const f32x4*>(its + 32 * i + 2 * r + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) sums.o[i][r + e] = __builtin_fmaf(y[e], g, sums.o[i][r + e] * f);
          }
      }
    }
    if (part == 0) {
      if (from == 0 && to == all) {
        store_columns<D>(sums.o, sums.sum == 0.f ? 0.f : 1.f / sums.sum, a.out.at(item.tokens.first + row.token, row.head), row.real, lane);
      } else if (row.real) {
        const int64_t at = (int64_t)place * ROWS + row_wave * 32 + (lane & 31);
        if (h == 0) *reinterpret_cast<float2*>(a.stats + 2 * at) = float2{sums.top, sums.sum};
#pragma unroll
        for (int i = 0; i < kParts; ++i)
#pragma unroll
          for (int r = 0; r < 16; r += 4) *reinterpret_cast<f32x4*>(a.sums + at * D + 32 * i + 2 * r + 4 * h) = f32x4{sums.o[i][r], sums.o[i][r + 1], sums.o[i][r + 2], sums.o[i][r + 3]};
      }
    }
    if constexpr (kRowWaves < kDraftWaves) __syncthreads();
  });
}

// What several workgroups have of a tile of rows joined, a workgroup for each 32 of its rows and key head, 8 threads a row; and zeros for sequences without positions.
template <int D, int ROWS>
__global__ void __launch_bounds__(256) draft_join_kernel(DraftArgs a) {
  constexpr int kStep = DraftShape<D, ROWS>::kStep, kPer = D / 8;
  const int heads = a.c.k_heads, group = a.q_heads / heads, id = (int)blockIdx.x / heads, k_head = (int)blockIdx.x - id * heads, slot = id / (ROWS / 32), block = id - slot * (ROWS / 32);
  int64_t items = 0;
  int sequence = -1, tile = 0;
  over_blocks<ROWS, kStep>(a, group, [&](int first, int tiles, int) {
    const uint32_t sum = rising_sum((uint32_t)tiles);
    const uint64_t found = __ballot(slot < items + sum);
    if (found == 0) {
      items += last_sum(sum);
      return true;
    }
    const int s = __ffsll((unsigned long long)found) - 1;
    sequence = first + s;
    tile = (int)(slot - items - sum_up_to(sum, s));
    return false;
  });
  if (sequence < 0) return;
  const DraftItem item = draft_item(a, sequence, tile);
  const int in_tile = block * 32 + (int)threadIdx.x / 8, row = tile * ROWS + in_tile, d = (int)threadIdx.x % 8 * kPer;
  if (row >= item.tokens.length * group) return;
  uint16_t* to = a.out.at(item.tokens.first + row / group, k_head * group + row % group) + d;
  int last = -1, first_part = 0;
  if (item.length > 0) {
    const int2 parts = a.parts[(int64_t)slot * heads + k_head];
    last = __builtin_amdgcn_readfirstlane(parts.y);
    if (last < 0) return;                                    // one workgroup had all of it
    first_part = __builtin_amdgcn_readfirstlane(parts.x);
  }
  const int first = first_part / 2 / heads;
  if (last >= a.shares || first_part < 0) return;            // (not where cu rises)
  float top = -FLT_MAX, sum = 0.f, o[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) o[e] = 0.f;
  for (int share = first; share <= last; ++share) {
    const int64_t at = (int64_t)(share == first ? first_part : (share * heads + k_head) * 2) * ROWS + in_tile;
    const float2 x = *reinterpret_cast<const float2*>(a.stats + 2 * at);
    const float now = fmaxf(top, x.x), less = __builtin_amdgcn_exp2f(top - now), more = __builtin_amdgcn_exp2f(x.x - now);
    sum = __builtin_fmaf(x.y, more, sum * less);
#pragma unroll
    for (int e = 0; e < kPer; e += 4) {
      const f32x4 y = *reinterpret_cast<const f32x4*>(a.sums + at * D + d + e);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[e + i] = __builtin_fmaf(y[i], more, o[e + i] * less);
    }
    top = now;
  }
  const float f = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int e = 0; e < kPer; e += 8) {
    float z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = o[e + i] * f;
    *reinterpret_cast<u32x4*>(to + e) = pack8(z);
  }
}

}  // namespace swz
