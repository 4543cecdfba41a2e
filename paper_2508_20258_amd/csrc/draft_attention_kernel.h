// Attention of the drafted tokens of every sequence over a cache of pages in bfloat16: out = softmax(scale q k^T) v, a token looking at all positions before its block and at those of its block's tokens
// that a mask of 64 bits names, or (no masks) at those up to its own.  One pass over the positions: with m the maximum so far, out and the sum of weights are kept times exp(-m), and scaled where m rises.
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
//
// What bounds it: the cache's bytes up to about 250 rows of a block (4 D bytes and 4 D operations a row for each position and key head, at 6.4 TB/s and 1600 TFLOP/s), products beyond.  With 32 query heads of 128:
// 64 single tokens, sharing 8 key heads, over 151000 positions in all (620 MB) 98 us, 6.3 TB/s, and 4.6 for the join; one over 131072 positions (537 MB) 84 us, 6.4 TB/s, and 5.  32 blocks of 32 tokens over 94000
// positions (388 MB) 87 us, 4.4 TB/s, and 11: the parts of 512 workgroups, 45 MB, are written and read beside it.  A block of 64 tokens, sharing 4 key heads, over 131072 positions, 137 GFLOP, 142 to 144 us and 8.3,
// 0.96 PFLOP/s: the matrix units work for 54 % of the cycles, the vector unit for 47 %, at 1.76 GHz.
//
// The next piece of a prompt is a block as any other: every tile of its rows takes all positions of the sequence, those of the block's own tokens in the slower masked way, though a chain's first rows look at few of those.
// With 32 heads of 128 sharing 8: 8192 tokens by themselves 1580 us (the causal products alone are 343 at 1604 TFLOP/s, and attention_kernel takes 511), 2048 over 16384 positions 562 (321), 512 over 8192 101 (42).
//
// Loads go straight to LDS.  Streaming ones, where positions are read once: 64 single tokens 105 us, with regular ones 121.  More tiles on their way in LDS, or fewer bytes a wave and more waves, changed
// nothing: 5.8 TB/s was what regular loads reach in a kernel that does nothing else.
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
  static constexpr int kSwitch = kWide ? 2 : 1;             // see deal
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

// 64 sequences, a lane each: their tokens, their lengths.
struct DraftWindow {
  int first;                         // sequence of lane 0
  Span tokens;
  int length;
  __device__ __forceinline__ void load(const DraftArgs& a, int from) {
    first = from;
    const int b = from + (int)(threadIdx.x & 63);
    tokens = {0, 0};
    length = 0;
    if (b < a.sequences) {
      tokens = span_of(a.cu[b], a.cu[b + 1], a.total);
      length = draft_length(a, b);
    }
  }
  __device__ __forceinline__ DraftItem item(int sequence, int tile) const {
    const int lane = sequence - first;
    return {sequence, tile, {__builtin_amdgcn_readlane(tokens.first, lane), __builtin_amdgcn_readlane(tokens.length, lane)}, __builtin_amdgcn_readlane(length, lane)};
  }
};
// The window that holds f's sequence: f(window) for one after the other, until it says false.  (One window is loaded once.)
template <class F>
__device__ __forceinline__ void over_windows(const DraftArgs& a, DraftWindow& w, F&& f) {
  for (int first = 0; first < a.sequences; first += 64) {
    if (w.first != first) w.load(a, first);
    if (!f()) return;
  }
}

// The lowest c bits.
__device__ __forceinline__ uint64_t low_bits(int c) { return c >= 64 ? ~0ull : c <= 0 ? 0ull : (1ull << c) - 1; }
__device__ __forceinline__ uint64_t shift_up(uint64_t x, int by) { return by >= 64 || by <= -64 ? 0ull : by >= 0 ? x << by : x >> -by; }

__device__ const u32x4 kNanChunk = {0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};

// Positions of a head from their pages into LDS: GROUPS times 16, as a page has 16 or more.  page(i): of the i-th 16.  Positions from `length` on are zeros, those without a page NaN.  STREAM: they are read once.
template <int D, int GROUPS, bool STREAM, class F>
__device__ __forceinline__ void load_positions(const PageTable& c, const uint16_t* pages, int k_head, int64_t position, int length, uint32_t lds, F&& page) {
  constexpr int kChunks = D / 8, kRows = 64 / kChunks, kLoads = 16 / kRows;          // rows of an instruction; instructions of 16 rows
  constexpr int kUnroll = GROUPS == 1 ? 1 : kLoads;          // where a wave has the one group, the kernel has no room for more of the rarer path
  uint32_t l = threadIdx.x & 63;
  const uint32_t part = (l / kChunks) * (uint32_t)(2 * D) + (((l % kChunks) ^ (uint32_t)tile_key<D>((int)l / kChunks)) << 4);
#pragma unroll 1
  for (int i = 0; i < GROUPS; ++i) {
    const int its = page(i);
    const int64_t from = position + 16 * i;
    if (its >= 0 && from + 16 <= length) {
      const uint64_t at = reinterpret_cast<uint64_t>(pages + c.token_at(its, k_head, (int)from) * D);
      const uint64_t uniform = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const uint32_t off = (uint32_t)(j * kRows * 2 * D) + (part ^ (uint32_t)(tile_key<D>(j * kRows) << 4)), to = lds + (uint32_t)(i * 32 * D + j * 1024);
        if constexpr (STREAM) stream_to_lds(reinterpret_cast<const void*>(uniform), off, to);
        else load_to_lds_base_off(reinterpret_cast<const void*>(uniform), off, to);
      }
    } else {
      keep(l);                       // or what this needs, once or twice for a sequence, has registers all along
      const unsigned char* real = reinterpret_cast<const unsigned char*>(its < 0 ? reinterpret_cast<const uint16_t*>(&kNanChunk) : pages + c.token_at(its, k_head, (int)from) * D);
#pragma unroll kUnroll
      for (int j = 0; j < kLoads; ++j) {
        const int r = j * kRows + (int)l / kChunks;
        const uint32_t off = its < 0 ? 0u : (uint32_t)(r * 2 * D) + ((l % kChunks ^ (uint32_t)tile_key<D>(r)) << 4);
        load_to_lds(from + r < length ? real + off : reinterpret_cast<const unsigned char*>(&kZeroChunk), lds + (uint32_t)(i * 32 * D + j * 1024));
      }
    }
  }
}

// Whether any value of a tile is no finite number: whose exponent is all ones.
template <int D>
__device__ __forceinline__ bool any_odd(const unsigned char* tile, int lane) {
  typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
  uint32_t l = (uint32_t)lane;
  keep(l);                           // or what this needs, once or twice for a sequence, has registers all along
  u16x2 high[2] = {0, 0};
#pragma unroll 1
  for (int i = 0; i < kDraftKeys * 2 * D / 1024; i += 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(tile + (i + j) * 1024 + l * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) high[e % 2] = __builtin_elementwise_max(high[e % 2], __builtin_bit_cast(u16x2, x[e] & 0x7fff7fffu));
    }
  }
  const u16x2 m = __builtin_elementwise_max(high[0], high[1]);
  return __any(m[0] >= 0x7f80 || m[1] >= 0x7f80);
}

// o += p x for 32 NB positions.
template <int D, int NB>
__device__ __forceinline__ void add_values(f32x16 (&o)[D / 32], const u32x4 (&p)[2 * NB], uint32_t lds, int lane) {
  const uint32_t column = column_address<D>(lds, lane);
#pragma unroll
  for (int k = 0; k < 2 * NB; ++k)
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = mfma32(read_columns<D>(column, k, i), __builtin_bit_cast(bf16x8, p[k]), o[i]);
}

// A product carries 0 times an infinity into rows that do not look at it.  So the positions of a tile that have values that are no finite numbers are taken one at a time, by a product of their own that only those rows
// keep that look at them (of the wave's 32 NB positions from 32 `part` NB on), and are zeros in the tile then.  sync(): of the waves that share the tile.
template <int D, int NB, class F>
__device__ __forceinline__ void take_odd(f32x16 (&o)[D / 32], const u32x4 (&p)[2 * NB], unsigned char* tile, uint32_t lds, int part, uint64_t seen, int lane, F&& sync) {
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
#pragma unroll
    for (int r = 0; r < kRows; ++r) odd |= (found >> (r * kChunks) & ((1ull << kChunks) - 1)) != 0 ? 1ull << (i * kRows + r) : 0ull;
  }
  const uint32_t column = column_address<D>(lds + (uint32_t)(part * NB * 64 * D), (int)l);
#pragma unroll 1
  for (uint64_t rest = odd >> (32 * NB * part) & (~0ull >> (64 - 32 * NB)); rest != 0; rest &= rest - 1) {
    const int at = __ffsll((unsigned long long)rest) - 1, k = at >> 4;
    u32x4 w = p[0];
#pragma unroll
    for (int j = 1; j < 2 * NB; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = k == j ? p[j][e] : w[e];
    // element e of lane half h is position 16 k + 8 (e / 4) + 4 h + e % 4
    const int place = at & 15, word = place >> 3 << 1 | (place >> 1 & 1);
    const uint32_t keeps = (place >> 2 & 1) == (int)(l >> 5) ? (place & 1 ? 0xffff0000u : 0xffffu) : 0u;
    const bool looks = seen >> at & 1;
#pragma unroll 1
    for (int i = 0; i < D / 32; ++i) {
      u32x4 f = __builtin_bit_cast(u32x4, read_columns<D>((column ^ (uint32_t)(i << 6)) + (uint32_t)(k * 32 * D), 0, 0));
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] &= e == word ? keeps : 0u;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        if (j != i) continue;
        const f32x16 with = mfma32(__builtin_bit_cast(bf16x8, f), __builtin_bit_cast(bf16x8, w), o[j]);
#pragma unroll
        for (int r = 0; r < 16; ++r) o[j][r] = looks ? with[r] : o[j][r];
      }
    }
  }
  sync();
#pragma unroll 1
  for (uint64_t rest = odd; rest != 0; rest &= rest - 1)
    if (l < (uint32_t)kChunks) *reinterpret_cast<u32x4*>(tile + (__ffsll((unsigned long long)rest) - 1) * 2 * D + l * 16) = u32x4{};
  sync();
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
  // Scores of 32 NB positions to weights, rounded to bfloat16 for the product: 2^-8 of a weight at most, as likely up as down; the sum is of the weights before.  With values of bfloat16 and an output that is
  // rounded to it the error against 64 bits is 0.0023 where 32-bit weights leave 0.0017; they would take two products for one.
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
__device__ __forceinline__ int page_bits(const PageTable& c) { return max(0, 6 - c.page_shift); }
template <int EVERY>
__device__ __forceinline__ int look_up_pages(const PageTable& c, const DraftItem& item, int tile) {
  const int lane = threadIdx.x & 63, bits = page_bits(c);
  const int64_t position = ((int64_t)tile + (int64_t)(lane >> bits) * EVERY) * kDraftKeys + ((lane & ((1 << bits) - 1)) << c.page_shift);
  return position < item.length ? c.page_of(item.sequence, (int)position) : -1;
}
// Of position `place` of the entry-th of those tiles.
__device__ __forceinline__ int page_at(const PageTable& c, int pages, int entry, int place) { return __builtin_amdgcn_readlane(pages, (entry << page_bits(c)) + (place >> c.page_shift)); }

// What a workgroup does after a tile of rows: the next one, its steps from 0 to `to`, and its pages, which look_up() finds.
struct DraftNext {
  bool there;
  DraftItem item;
  int to, pages;
};

// Deals the steps of all tiles of rows to workgroups: calls process(item, from, to, all, place, pages, next, look_up_next) for each tile of rows of which steps from .. to - 1, of `all`, are this workgroup's; a part of
// one goes to `place`.  pages: what look_up(item, from) gave, and look_up_next() looks up next.pages: process calls it when it has no more urgent loads.  A workgroup that goes on to another tile of rows loses the
// time of about kSwitch steps; tiles of rows count as so many steps more.
template <int D, int ROWS, class L, class F>
__device__ __forceinline__ void deal(const DraftArgs& a, int share, int k_head, int group, L&& look_up, F&& process) {
  constexpr int kStep = DraftShape<D, ROWS>::kStep;
  const int heads = a.c.k_heads, kSwitch = a.shares == 0 ? 0 : DraftShape<D, ROWS>::kSwitch;
  auto tiles_of = [&](int tokens) { return (tokens * group + ROWS - 1) / ROWS; };
  auto steps_of = [&](int length) { return length == 0 ? 0 : (length + kStep - 1) / kStep + kSwitch; };
  // `before` steps are those of the tiles before the sequence's, `items` the tiles
  int64_t my_start = 0, my_end = 0, before = 0, items = 0;
  int sequence = -1;
  DraftWindow w;
  w.first = -1;
  if (a.shares == 0) {
    int tile = 0;
    over_windows(a, w, [&] {
      const int tiles = tiles_of(w.tokens.length);
      const uint32_t sum = rising_sum((uint32_t)tiles);
      const uint64_t found = __ballot(share < items + sum);
      if (found == 0) {
        items += last_sum(sum);
        return true;
      }
      const int s = __ffsll((unsigned long long)found) - 1;
      sequence = w.first + s;
      items += sum_up_to(sum, s);
      tile = (int)(share - items);
      return false;
    });
    if (sequence < 0) return;
    const DraftItem item = w.item(sequence, tile);
    const int all = steps_of(item.length);
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
    over_windows(a, w, [&] {
      total += last_sum(rising_sum((uint32_t)tiles_of(w.tokens.length) * (uint32_t)steps_of(w.length)));
      return true;
    });
    const int shares = (int)min((int64_t)a.shares, total);
    if (share >= shares) return;
    my_start = total * share / shares;
    my_end = total * (share + 1) / shares;
    over_windows(a, w, [&] {
      const int tiles = tiles_of(w.tokens.length);
      const uint32_t sum = rising_sum((uint32_t)tiles * (uint32_t)steps_of(w.length)), count = rising_sum((uint32_t)tiles);
      const uint64_t found = __ballot(my_start < before + sum);
      if (found == 0) {
        before += last_sum(sum);
        items += last_sum(count);
        return true;
      }
      const int s = __ffsll((unsigned long long)found) - 1;
      sequence = w.first + s;
      before += sum_up_to(sum, s);
      items += sum_up_to(count, s);
      return false;
    });
    if (sequence < 0) return;
  }
  // the first tile of rows with steps of this workgroup's, then those after it
  DraftItem item = w.item(sequence, 0);
  int all = steps_of(item.length);
  item.tile = (int)((my_start - before) / all);
  int pages = 0;
  bool looked_up = false;
  for (int64_t step = my_start;;) {
    const int64_t at = step - before - (int64_t)item.tile * all, count = min((int64_t)all - at, my_end - step);
    const int from = max((int)at - kSwitch, 0), to = max((int)(at + count) - kSwitch, 0);
    step += count;
    DraftItem then = item;
    int64_t then_before = before, then_items = items;
    if (step < my_end && ++then.tile == tiles_of(item.tokens.length)) {
      // the next sequence that has rows and positions
      do {
        then_items += tiles_of(then.tokens.length);
        then_before += (int64_t)tiles_of(then.tokens.length) * steps_of(then.length);
        const int next = then.sequence + 1;
        if (next >= a.sequences) {
          my_end = step;
          break;
        }
        if (next - w.first >= 64) w.load(a, next & ~63);
        then = w.item(next, 0);
      } while (then.tokens.length == 0 || then.length == 0);
    }
    const bool more = step < my_end;
    if (from < to) {
      const int place = (share * heads + k_head) * 2 + (step - count == my_start ? 0 : 1), real = all - kSwitch;
      if (!looked_up) pages = look_up(item, from);
      DraftNext next = {more, then, more ? (int)min((int64_t)steps_of(then.length), my_end - step) - kSwitch : 0, 0};
      next.there = next.to > 0;
      process(item, from, to, real, place, pages, next, [&] {
        if (next.there) next.pages = look_up(then, 0);
      });
      pages = next.pages;
      looked_up = true;
      if (a.shares != 0 && threadIdx.x == 0 && items + item.tile < a.items) {
        int2* part = a.parts + (items + item.tile) * heads + k_head;
        if (from == 0) part->x = place;
        if (to == real) part->y = from == 0 ? -1 : share;
      }
    }
    if (!more) return;
    item = then;
    before = then_before;
    items = then_items;
    all = steps_of(item.length);
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

  auto look_up = [&](const DraftItem& item, int from) { return look_up_pages<kDraftWaves>(a.c, item, from * kDraftWaves + wave); };
  bool fetched = false;              // the first keys are on their way
  deal<D, ROWS>(a, share, k_head, group, look_up, [&](const DraftItem& item, int from, int to, int all, int place, int pages, DraftNext& next, auto&& look_up_next) {
    const int rows = item.tokens.length * group, first_row = item.tile * ROWS;
    const int end = min(to * kDraftWaves, (item.length + kDraftKeys - 1) / kDraftKeys);
    const int whole = min(min(item.length - item.tokens.length, item.length) / kDraftKeys, end);      // tiles that all rows look at whole (none where the block is longer than the sequence)
    int t = from * kDraftWaves + wave, entry = 0;            // the wave's tile, and which of `pages` is its
    auto fetch = [&](const uint16_t* from_pages, int length, int tile, int pages, int entry, uint32_t lds) {
      load_positions<D, 4, true>(a.c, from_pages, k_head, (int64_t)tile * kDraftKeys, length, lds, [&](int i) { return page_at(a.c, pages, entry, 16 * i); });
    };
    // the keys after those of tile t: of the next tile, or the first of the next tile of rows; whether there are any
    auto fetch_more = [&] {
      const int then = t + kDraftWaves;
      const bool more = then < end;
      if (more && ++entry == 64 >> page_bits(a.c)) {
        pages = look_up_pages<kDraftWaves>(a.c, item, then);
        entry = 0;
      }
      if (!more) fetched = next.there && wave < min(next.to * kDraftWaves, (next.item.length + kDraftKeys - 1) / kDraftKeys);
      if (more || fetched) fetch(a.k_pages, more ? item.length : next.item.length, more ? then : wave, more ? pages : next.pages, more ? entry : 0, k_lds);
      return more || fetched;
    };
    if (t < end) {
      if (!fetched) fetch(a.k_pages, item.length, t, pages, 0, k_lds);
      fetch(a.v_pages, item.length, t, pages, 0, v_lds);
    }
    fetched = false;
    const DraftRows row(a, item, first_row + (lane & 31), k_head, group);
    bf16x8 qf[kSteps];
    load_fragments<D>(qf, a.q.at(item.tokens.first + row.token, row.head), lane);
    look_up_next();
    DraftSums<D> sums;
    sums.clear();
    auto take = [&](auto is_masked) __attribute__((always_inline)) {
      constexpr bool masked = decltype(is_masked)::value;
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
      const bool behind = fetch_more();                      // a tile of keys is on its way behind the values
      uint64_t seen = 0;
      if constexpr (masked) {
        seen = row.seen(a, item, t);
        hide(x, seen, h);
      }
      sums.weigh(x, c, p);
      __builtin_amdgcn_sched_barrier(0);
      if (behind) wait_vmcnt<kTileLoads>();
      else wait_vmcnt<0>();
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (masked) {
        if (__builtin_expect(any_odd<D>(v_tile, lane), 0)) take_odd<D, 2>(sums.o, p, v_tile, v_lds, 0, seen, lane, [] { wait_vmcnt_lgkmcnt<63, 0>(); });
      }
      add_values<D, 2>(sums.o, p, v_lds, lane);
      __builtin_amdgcn_sched_barrier(0);
      wait_vmcnt_lgkmcnt<63, 0>();
      __builtin_amdgcn_sched_barrier(0);
      if (t + kDraftWaves < end) fetch(a.v_pages, item.length, t + kDraftWaves, pages, entry, v_lds);
      t += kDraftWaves;
    };
    if (t >= end) fetch_more();
    while (t < whole) take(std::false_type{});
    while (t < end) take(std::true_type{});

    // Every wave's sums into its tile of values, then a row by 8 threads.  Four dimensions, c, of row r are in slot c ^ r of the row: 32 rows' are spread over all banks.
    const float sum = across_halves(sums.sum, [](float y, float z) { return y + z; });
    auto slot = [](int row, int dims) { return row * D + (dims / 4 ^ row % (D / 4)) * 4; };
    float* mine = reinterpret_cast<float*>(v_tile);
#pragma unroll
    for (int i = 0; i < kParts; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += 4) *reinterpret_cast<f32x4*>(mine + slot(lane & 31, 32 * i + 2 * r + 4 * h)) = f32x4{sums.o[i][r], sums.o[i][r + 1], sums.o[i][r + 2], sums.o[i][r + 3]};
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
      for (int e = 0; e < D / 8; e += 4) {
        f32x4 z = f32x4{};
#pragma unroll
        for (int w = 0; w < kDraftWaves; ++w) z += *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(smem + (2 * w + 1) * S::kTileBytes) + slot(r, d + e)) * factor[w];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[e + i] = z[i] * f;
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

// Where the waves of wide tiles leave their sums of 32 rows, from row `at` of all places on: as they have them, a lane's four dimensions of `chunk` beside the next lane's, which are another row's (row by row, 16 bytes
// of 64 rows with a store: 148 us for 144 with a block of 64 tokens over 131072 positions).
template <int D>
__device__ __forceinline__ f32x4* wide_sums(const DraftArgs& a, int64_t at, int chunk, int lane) { return reinterpret_cast<f32x4*>(a.sums + at * D + (chunk * 64 + lane) * 4); }

// Pairs of weights taken before a slot, if all `pairs` of them are by slot `last`.
constexpr int pairs_before(int slot, int pairs, int last) { return slot >= last ? pairs : (slot * pairs + last - 1) / last; }

// STREAM: most blocks are one tile of rows, so that keys and values are read once.
template <int D, int ROWS, bool STREAM>
__global__ void __launch_bounds__(64 * kDraftWaves, 2) draft_attention_wide_kernel(DraftArgs a) {
  using S = DraftShape<D, ROWS>;
  constexpr int kParts = D / 32, kSteps = D / 16, kBlocks = ROWS / 64, kRowWaves = ROWS / 32;     // a wave has 32 kBlocks of a tile's keys
  constexpr bool kFollow = kRowWaves == kDraftWaves;         // LDS is tiles alone
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S::kLdsBytes];
  const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), row_wave = wave % kRowWaves, part = wave / kRowWaves;
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem, mine = (uint32_t)(part * 64 * D);      // of a tile: the wave's keys
  const int heads = a.c.k_heads, group = a.q_heads / heads, share = (int)blockIdx.x / heads, k_head = (int)blockIdx.x - share * heads;
  const float c = a.scale * kLog2E;

  auto look_up = [&](const DraftItem& item, int from) { return look_up_pages<1>(a.c, item, from); };
  // Tiles of all tiles of rows are numbered on: the keys of number n are in slot n & 1, the values in 2 + that.
  int number = 0;
  bool fetched = false;              // the first keys and values and the second keys are on their way
  int key_page = 0, value_page = 0;  // of the last keys that were fetched, and of those before them
  deal<D, ROWS>(a, share, k_head, group, look_up, [&](const DraftItem& item, int from, int to, int all, int place, int pages, DraftNext& next, auto&& look_up_next) {
    const int whole = min(min(item.length - item.tokens.length, item.length) / kDraftKeys, to);
    const int first_number = number;
    number += to - from;
    auto slot_of = [&](int t) { return first_number + t - from & 1; };
    // A wave fetches a quarter of a tile.  Keys are fetched two tiles ahead, values one, from the pages that the keys had; towards the end those of the next tile of rows.
    const bool follow = kFollow && next.there && next.to >= 2 && to - from >= 2;
    int entry = 0;                                           // of `pages`: that of the keys to come
    auto fetch_k = [&](bool mine, int t, int slot) {
      const int length = mine ? item.length : next.item.length;
      value_page = key_page;
      key_page = page_at(a.c, mine ? pages : next.pages, mine ? entry : t, 16 * wave);
      if (mine && ++entry == 64 >> page_bits(a.c)) {
        pages = look_up_pages<1>(a.c, item, t + 1);
        entry = 0;
      }
      load_positions<D, 1, STREAM>(a.c, a.k_pages, k_head, (int64_t)t * kDraftKeys + 16 * wave, length, lds + (uint32_t)(slot * S::kTileBytes + 16 * wave * 2 * D), [&](int) { return key_page; });
    };
    auto fetch_v = [&](bool mine, int t, int page, int slot) {
      load_positions<D, 1, STREAM>(a.c, a.v_pages, k_head, (int64_t)t * kDraftKeys + 16 * wave, mine ? item.length : next.item.length,
                                   lds + (uint32_t)((2 + slot) * S::kTileBytes + 16 * wave * 2 * D), [&](int) { return page; });
    };
    if (!fetched) {
      fetch_k(true, from, slot_of(from));
      fetch_v(true, from, key_page, slot_of(from));
      if (from + 1 < to) fetch_k(true, from + 1, slot_of(from + 1));
    } else {
      entry = 2;                                             // (a table of 64 has the pages of 16 tiles or more)
    }
    fetched = follow;
    auto turn = [&](int t) __attribute__((always_inline)) {
      publish();
      const bool k_mine = t + 2 < to, v_mine = t + 1 < to;
      if (k_mine || follow) fetch_k(k_mine, k_mine ? t + 2 : t + 2 - to, slot_of(t));
      if (v_mine || follow) fetch_v(v_mine, v_mine ? t + 1 : 0, k_mine || follow ? value_page : key_page, slot_of(t + 1));
    };
    const DraftRows row(a, item, item.tile * ROWS + row_wave * 32 + (lane & 31), k_head, group);
    bf16x8 qf[kSteps];
    load_fragments<D>(qf, a.q.at(item.tokens.first + row.token, row.head), lane);
    look_up_next();
    DraftSums<D> sums;
    sums.clear();
    f32x16 x[kBlocks], other[kBlocks];
    auto score = [&](int t) __attribute__((always_inline)) {
      const uint32_t k_lane = row_address<D>(lds + mine + (uint32_t)(slot_of(t) * S::kTileBytes), lane);
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
      const uint32_t values = (uint32_t)((2 + slot_of(t)) * S::kTileBytes);
      u32x4 p[2 * kBlocks];
      if constexpr (masked) {
        const uint64_t seen = row.seen(a, item, t) >> (32 * part) & (~0ull >> (64 - 32 * kBlocks));
        hide(x, seen, h);
        sums.weigh(x, c, p);
        if (__builtin_expect(any_odd<D>(smem + values, lane), 0))
          take_odd<D, kBlocks>(sums.o, p, smem + values, lds + values, part, seen, lane, [] {
            wait_vmcnt_lgkmcnt<63, 0>();
            block_barrier();
          });
      } else {
        sums.weigh(x, c, p);
      }
      add_values<D, kBlocks>(sums.o, p, lds + values + mine, lane);
      if (t + 1 < to) score(t + 1);
    };
    publish();
    score(from);
    int t = from;
    if (t + 3 < whole && slot_of(t) == 1) take(t++, std::false_type{});
    if (t + 2 < whole && slot_of(t) == 0) {
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
    if constexpr (!kFollow) publish();                       // the tiles have been read
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
          for (int r = 0; r < 16; r += 4) *wide_sums<D>(a, at - (lane & 31), 4 * i + r / 4, lane) = f32x4{sums.o[i][r], sums.o[i][r + 1], sums.o[i][r + 2], sums.o[i][r + 3]};
      }
    }
    if constexpr (kRowWaves < kDraftWaves) __syncthreads();
  });
}

// What several workgroups have of a tile of rows joined, and zeros for sequences without positions: GROUPS workgroups for each 32 of its rows and key head.  Tiles of 32 rows: a workgroup has 32 / GROUPS rows, 8 threads
// a row and GROUPS of them for its parts.  Wide ones: a lane has a row, and four dimensions of each of its chunks of 8; a workgroup has 1 / GROUPS of the chunks, and a wave a quarter of those, or (GROUPS 8) of the parts.
template <int D, int ROWS, int GROUPS>
__global__ void __launch_bounds__(256) draft_join_kernel(DraftArgs a) {
  constexpr bool kWide = ROWS > 32, kSplit = GROUPS > 1;
  constexpr int kPer = kWide && kSplit ? D / 16 : D / 8, kRows = kWide ? 32 : 32 / GROUPS, kParts = !kSplit ? 1 : kWide ? 4 : GROUPS;       // numbers of a thread; rows of a workgroup; parts that it takes at a time
  constexpr int kJoined = !kSplit ? 1 : kWide ? 256 : 32, kJoinedPitch = kWide ? kPer + 4 : D + 4;
  __shared__ __attribute__((aligned(16))) float joined[kJoined][kJoinedPitch];
  const int heads = a.c.k_heads, group = a.q_heads / heads, id = (int)blockIdx.x / heads, k_head = (int)blockIdx.x - id * heads, slot = id / (ROWS / 32 * GROUPS), block = id - slot * (ROWS / 32 * GROUPS);
  int64_t items = 0;
  int sequence = -1, tile = 0;
  DraftWindow w;
  w.first = -1;
  over_windows(a, w, [&] {
    const uint32_t sum = rising_sum((uint32_t)(w.tokens.length * group + ROWS - 1) / ROWS);
    const uint64_t found = __ballot(slot < items + sum);
    if (found == 0) {
      items += last_sum(sum);
      return true;
    }
    const int s = __ffsll((unsigned long long)found) - 1;
    sequence = w.first + s;
    tile = (int)(slot - items - sum_up_to(sum, s));
    return false;
  });
  if (sequence < 0) return;
  const DraftItem item = w.item(sequence, tile);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), mine = kWide ? (int)threadIdx.x : (int)threadIdx.x / 8, part = kWide ? (kSplit ? wave : 0) : mine / kRows;
  const int first_row = kWide ? block / GROUPS * 32 : block * kRows, in_tile = first_row + (kWide ? lane & 31 : mine % kRows), row = tile * ROWS + in_tile;
  const int chunk = kSplit ? block % GROUPS * (kPer / 4) : wave * (kPer / 4), d = kWide ? 8 * chunk + 4 * (lane >> 5) : (int)threadIdx.x % 8 * kPer;
  if (tile * ROWS + first_row >= item.tokens.length * group) return;
  const bool real = row < item.tokens.length * group;
  uint16_t* to = a.out.at(item.tokens.first + (real ? row : 0) / group, k_head * group + (real ? row : 0) % group) + d;
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
  auto add = [&](float its_top, float its_sum, const f32x4 (&y)[kPer / 4]) {
    const float now = fmaxf(top, its_top), less = __builtin_amdgcn_exp2f(top - now), more = __builtin_amdgcn_exp2f(its_top - now);
    sum = __builtin_fmaf(its_sum, more, sum * less);
#pragma unroll
    for (int e = 0; e < kPer; ++e) o[e] = __builtin_fmaf(y[e / 4][e % 4], more, o[e] * less);
    top = now;
  };
#pragma unroll 2
  for (int share = first + part; share <= last; share += kParts) {
    const int64_t at = (int64_t)(share == first ? first_part : (share * heads + k_head) * 2) * ROWS + in_tile;
    const float2 x = *reinterpret_cast<const float2*>(a.stats + 2 * at);
    f32x4 y[kPer / 4];
#pragma unroll
    for (int e = 0; e < kPer / 4; ++e) y[e] = kWide ? *wide_sums<D>(a, at - (lane & 31), chunk + e, lane) : *reinterpret_cast<const f32x4*>(a.sums + at * D + d + 4 * e);
    if (real) add(x.x, x.y, y);
  }
  if constexpr (kSplit) {
    constexpr int kStats = kJoinedPitch - 4;
    const int at = kWide ? 0 : d;
    if (part > 0) {
#pragma unroll
      for (int e = 0; e < kPer; e += 4) *reinterpret_cast<f32x4*>(&joined[mine][at + e]) = f32x4{o[e], o[e + 1], o[e + 2], o[e + 3]};
      if (at == 0) joined[mine][kStats] = top, joined[mine][kStats + 1] = sum;
    }
    __syncthreads();
    if (part > 0) return;
    for (int p = 1; p < kParts; ++p) {
      const float* its = joined[mine + p * (kWide ? 64 : kRows)];
      f32x4 y[kPer / 4];
#pragma unroll
      for (int e = 0; e < kPer / 4; ++e) y[e] = *reinterpret_cast<const f32x4*>(its + at + 4 * e);
      add(its[kStats], its[kStats + 1], y);
    }
  }
  if (!real) return;
  const float f = sum == 0.f ? 0.f : 1.f / sum;
  if constexpr (kWide) {
    typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
    if constexpr (kPer == 4) {
      *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16(o[0] * f, o[1] * f), pack_bf16(o[2] * f, o[3] * f)};
    } else {
      // the halves trade registers so that each lane has a whole chunk, the first or the second of two
#pragma unroll
      for (int e = 0; e < kPer; e += 8) {
        const auto x = __builtin_amdgcn_permlane32_swap(pack_bf16(o[e] * f, o[e + 1] * f), pack_bf16(o[e + 4] * f, o[e + 5] * f), false, false);
        const auto y = __builtin_amdgcn_permlane32_swap(pack_bf16(o[e + 2] * f, o[e + 3] * f), pack_bf16(o[e + 6] * f, o[e + 7] * f), false, false);
        *reinterpret_cast<u32x4*>(to + 2 * e + 4 * (lane >> 5)) = u32x4{x[0], y[0], x[1], y[1]};
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < kPer; e += 8) {
      float z[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = o[e + i] * f;
      *reinterpret_cast<u32x4*>(to + e) = pack8(z);
    }
  }
}

}  // namespace swz
