// Attention of the drafted tokens of every sequence over a cache of pages in bfloat16: out = softmax(scale q k^T) v, a token looking at all positions before its block and at those of its block's tokens
// that a mask of 64 bits names, or (no masks) at those up to its own.
//
// The query heads of a key head look at the same keys, so a row is a token of one query head and the rows of a block are n * group.  A workgroup has a tile of 32 * RW rows, RW waves with 32 rows each
// and 4 / RW groups of waves that take every (4 / RW)th tile of 64 keys.  Scores come as S^T = k q^T and out^T += v^T P^T, as for prompts (attention_tiles.h): a lane has 32 scores of one row.
// RW = 1: each wave has a tile of keys and one of values in LDS for itself and waits for nothing but its own loads, the next keys being fetched when the scores are done and the next values when those are
// used up; the four join what they have in LDS.  RW = 4: the waves share tiles, two of each, the next ones load while these are used.
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

template <int D, int RW>
struct DraftShape {
  static constexpr int kRows = 32 * RW, kGroups = kDraftWaves / RW, kStep = kDraftKeys * kGroups;
  static constexpr int kTileBytes = kDraftKeys * 2 * D, kLdsBytes = 4 * kTileBytes * (RW == 1 ? 2 : 1);
  static constexpr int kJoinPitch = D + 4;                  // floats of a row in LDS when groups join
  static constexpr int kPerCu = RW == 1 && D == 128 ? 1 : 2;          // workgroups of a compute unit
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
        const unsigned char* at = reinterpret_cast<const unsigned char*>(base) + (uint32_t)(i * kRows * 2 * D) + (lane_part ^ key_of(i));
        if (page < 0) at = reinterpret_cast<const unsigned char*>(&kNanChunk);
        if (position + i * kRows + lane / kChunks >= length) at = reinterpret_cast<const unsigned char*>(&kZeroChunk);
        load_to_lds(at, lds + (uint32_t)(i * 1024));
      }
    }
  }
  static __device__ __forceinline__ uint32_t key_of(int i) { return (uint32_t)(tile_key<D>(i * kRows) << 4); }
};

// Whether any of a tile's values is no finite number.
template <int D>
__device__ __forceinline__ bool odd_tile(const unsigned char* tile, int lane) {
  uint32_t odd = 0;
#pragma unroll 4
  for (int i = 0; i < kDraftKeys * 2 * D / 1024; ++i) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(tile + i * 1024 + lane * 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) odd |= (uint32_t)((x[e] & 0x7f80u) == 0x7f80u) | (uint32_t)((x[e] & 0x7f800000u) == 0x7f800000u);
  }
  return __any(odd != 0);
}

// o += p x for the rows of a tile that the lane's bits name, one at a time: a product would carry 0 times an infinity into the others.
template <int D>
__device__ __forceinline__ void add_seen_rows(f32x16 (&o)[D / 32], const u32x4 (&p)[4], const unsigned char* tile, uint64_t seen, int lane) {
#pragma unroll 1
  for (int row = 0; row < kDraftKeys; ++row) {
    uint32_t l = (uint32_t)lane;
    keep(l);                         // or the loop has registers for its addresses, which are the kernel's
    const int h = (int)l >> 5;
    // row 16 j + 8 a + 4 h + e is number 4 a + e of operand j in lane half h
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) word = j == row >> 4 && e == 2 * (row >> 3 & 1) + (row >> 1 & 1) ? p[j][e] : word;
    const float mine = (row >> 2 & 1) == h ? __uint_as_float(row & 1 ? word & 0xffff0000u : word << 16) : 0.f;
    const float w = across_halves(mine, [](float x, float y) { return x + y; });
    const bool looks = seen >> row & 1;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int part = 0; part < 4; ++part) {
        typedef __attribute__((ext_vector_type(4))) uint16_t u16x4;
        const int d = 32 * i + 8 * part + 4 * h;
        const u16x4 x = *reinterpret_cast<const u16x4*>(tile + row * 2 * D + (((d >> 3) ^ tile_key<D>(row)) << 4) + (d & 7) * 2);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][4 * part + e] += looks ? w * __uint_as_float((uint32_t)x[e] << 16) : 0.f;
        __builtin_amdgcn_sched_barrier(0);
      }
  }
}

template <int D, int RW>
__global__ void __launch_bounds__(64 * kDraftWaves, (DraftShape<D, RW>::kPerCu)) draft_attention_kernel(DraftArgs a) {
  using S = DraftShape<D, RW>;
  constexpr int kParts = D / 32, kSteps = D / 16, kTileLoads = S::kTileBytes / 1024;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S::kLdsBytes];
  __shared__ float group_stats[S::kGroups][32][2];
  const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int row_wave = wave % RW, key_group = wave / RW;
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const int heads = a.c.k_heads, group = a.q_heads / heads;
  const int share = (int)blockIdx.x / heads, k_head = (int)blockIdx.x - share * heads;
  const float c = a.scale * kLog2E;
  const int page_bits = max(0, 6 - a.c.page_shift);          // pages of a tile, as a power of two

  // steps [from, to) of a tile of rows, of `all`; place: where a part goes
  auto process = [&](const DraftItem item, int from, int to, int all, int place) {
    const int n = item.tokens.length, rows = n * group, base = item.length - n;
    const int row = item.tile * S::kRows + row_wave * 32 + (lane & 31), real_row = min(row, rows - 1), token = real_row / group, head = k_head * group + real_row % group;
    const uint64_t mask = a.tree != nullptr ? a.tree[item.tokens.first + token] : 0;
    bf16x8 qf[kSteps];
    load_fragments<D>(qf, a.q.at(item.tokens.first + token, head), lane);
    f32x16 o[kParts], x[2];
#pragma unroll
    for (int i = 0; i < kParts; ++i) o[i] = f32x16{};
    float top = -FLT_MAX, sum = 0.f;                         // of scores times c; this lane's half of the sum

    const int end = min(to * S::kGroups, (item.length + kDraftKeys - 1) / kDraftKeys);
    int t = from * S::kGroups + key_group;
    const PageLoader<D> loader(a.c, k_head, item.length, lane);
    // pages of the tiles to come: lane l has number l of those that the wave takes, page_bits a tile
    int pages = 0, entry = 0;
    auto look_up = [&](int tile) {
      const int64_t position = ((int64_t)tile + (int64_t)(lane >> page_bits) * S::kGroups) * kDraftKeys + ((lane & ((1 << page_bits) - 1)) << a.c.page_shift);
      pages = position < item.length ? a.c.page_of(item.sequence, (int)position) : -1;
      entry = 0;
    };
    auto next_entry = [&](int tile) {
      if (++entry == 64 >> page_bits) look_up(tile);
    };
    auto fetch = [&](const uint16_t* from_pages, int tile, int slot) {
#pragma unroll
      for (int i = 0; i < 4 / RW; ++i) {
        const int r = RW == 1 ? 16 * i : 16 * row_wave;
        const int page = __builtin_amdgcn_readlane(pages, (entry << page_bits) + (r >> a.c.page_shift));
        loader(from_pages, (int64_t)tile * kDraftKeys + r, page, lds + (uint32_t)(slot * S::kTileBytes + r * 2 * D));
      }
    };
    auto score = [&](uint32_t tile) __attribute__((always_inline)) {
      const uint32_t k_lane = row_address<D>(tile, lane);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        x[b] = f32x16{};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) x[b] = mfma32(read_rows<D>(k_lane, b, i), qf[i], x[b]);
      }
    };
    // positions of tile `t` that the lane's row looks at
    auto seen_of = [&](int tile) {
      const int first = tile * kDraftKeys;
      const uint64_t seen = a.tree != nullptr ? low_bits(base - first) | shift_up(mask, base - first) : low_bits(base + token + 1 - first);
      return seen & low_bits(item.length - first);
    };
    u32x4 p[4];
    auto weigh = [&](bool masked, uint64_t seen) __attribute__((always_inline)) {
      if (masked) {
        const uint64_t mine = seen >> (4 * h);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const uint32_t bits = (uint32_t)(mine >> (32 * b));
#pragma unroll
          for (int r = 0; r < 16; ++r) x[b][r] = bits & (1u << (8 * (r / 4) + r % 4)) ? x[b][r] : -INFINITY;
        }
      }
      float high = x[0][0];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) high = fmaxf(high, x[b][r]);
      high = across_halves(high, [](float y, float z) { return fmaxf(y, z); }) * c;
      if (__any(high > top + kLazyRise)) {
        const float now = fmaxf(top, high), less = __builtin_amdgcn_exp2f(top - now);
        sum *= less;
#pragma unroll
        for (int i = 0; i < kParts; ++i) o[i] *= less;
        top = now;
      }
      float sums[2] = {sum, 0.f};
#pragma unroll
      for (int m = 0; m < 16; ++m) {
        const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[m / 8][m % 8 * 2], c, -top)), w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[m / 8][m % 8 * 2 + 1], c, -top));
        sums[0] += w0;
        sums[1] += w1;
        p[m / 4][m % 4] = pack_bf16(w0, w1);
      }
      sum = sums[0] + sums[1];
    };
    auto add = [&](int slot, bool masked, uint64_t seen) __attribute__((always_inline)) {
      if (masked && __builtin_expect(odd_tile<D>(smem + slot * S::kTileBytes, lane), 0)) {
        add_seen_rows<D>(o, p, smem + slot * S::kTileBytes, seen, lane);
        return;
      }
      const uint32_t v_lane = column_address<D>(lds + (uint32_t)(slot * S::kTileBytes), lane);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < kParts; ++i) o[i] = mfma32(read_columns<D>(v_lane, j, i), __builtin_bit_cast(bf16x8, p[j]), o[i]);
    };
    const int whole = min(base, item.length) / kDraftKeys;   // tiles that all rows look at whole (none where base < 0)

    if constexpr (RW == 1) {
      const int k_slot = 2 * wave, v_slot = 2 * wave + 1;
      if (t < end) {
        look_up(t);
        fetch(a.k_pages, t, k_slot);
        fetch(a.v_pages, t, v_slot);
      }
      while (t < end) {
        const int then = t + S::kGroups;
        const bool more = then < end, masked = t >= whole;
        const uint64_t seen = masked ? seen_of(t) : 0;
        __builtin_amdgcn_sched_barrier(0);
        wait_vmcnt<kTileLoads>();                            // the keys have landed, the values may be on their way
        __builtin_amdgcn_sched_barrier(0);
        score(lds + (uint32_t)(k_slot * S::kTileBytes));
        __builtin_amdgcn_sched_barrier(0);
        wait_vmcnt_lgkmcnt<63, 0>();
        __builtin_amdgcn_sched_barrier(0);
        if (more) {
          next_entry(then);
          fetch(a.k_pages, then, k_slot);
        }
        weigh(masked, seen);
        __builtin_amdgcn_sched_barrier(0);
        if (more) wait_vmcnt<kTileLoads>();
        else wait_vmcnt<0>();
        __builtin_amdgcn_sched_barrier(0);
        add(v_slot, masked, seen);
        __builtin_amdgcn_sched_barrier(0);
        wait_vmcnt_lgkmcnt<63, 0>();
        __builtin_amdgcn_sched_barrier(0);
        if (more) fetch(a.v_pages, then, v_slot);
        t = then;
      }
    } else {
      int turn = 0;
      if (t < end) {
        look_up(t);
        fetch(a.k_pages, t, 0);
        fetch(a.v_pages, t, 2);
      }
      for (; t < end; ++t, turn ^= 1) {
        publish();
        if (t + 1 < end) {
          next_entry(t + 1);
          fetch(a.k_pages, t + 1, turn ^ 1);
          fetch(a.v_pages, t + 1, 2 + (turn ^ 1));
        }
        const bool masked = t >= whole;
        const uint64_t seen = masked ? seen_of(t) : 0;
        if (masked && !__any(seen != 0)) continue;
        score(lds + (uint32_t)(turn * S::kTileBytes));
        weigh(masked, seen);
        add(2 + turn, masked, seen);
      }
      publish();
    }

    sum = across_halves(sum, [](float y, float z) { return y + z; });
    const bool entire = from == 0 && to == all;
    if constexpr (RW == 1) {
      // every wave's rows into its own tiles, then a row by 8 threads
      float* mine = reinterpret_cast<float*>(smem + 2 * wave * S::kTileBytes) + (lane & 31) * S::kJoinPitch;
#pragma unroll
      for (int i = 0; i < kParts; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 4) *reinterpret_cast<f32x4*>(mine + 32 * i + 2 * r + 4 * h) = f32x4{o[i][r], o[i][r + 1], o[i][r + 2], o[i][r + 3]};
      if (h == 0) group_stats[wave][lane & 31][0] = top, group_stats[wave][lane & 31][1] = sum;
      __syncthreads();
      const int r = (int)threadIdx.x / 8, d = (int)threadIdx.x % 8 * (D / 8), its = item.tile * S::kRows + r;
      if (its < rows) {
        float factor[kDraftWaves], high = -FLT_MAX, total = 0.f;
#pragma unroll
        for (int w = 0; w < kDraftWaves; ++w) high = fmaxf(high, group_stats[w][r][0]);
#pragma unroll
        for (int w = 0; w < kDraftWaves; ++w) {
          factor[w] = __builtin_amdgcn_exp2f(group_stats[w][r][0] - high);
          total = __builtin_fmaf(group_stats[w][r][1], factor[w], total);
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
          const int64_t at = (int64_t)place * S::kRows + r;
#pragma unroll
          for (int e = 0; e < D / 8; e += 4) *reinterpret_cast<f32x4*>(a.sums + at * D + d + e) = f32x4{y[e], y[e + 1], y[e + 2], y[e + 3]};
          if (d == 0) *reinterpret_cast<float2*>(a.stats + 2 * at) = float2{high, total};
        }
      }
      __syncthreads();
    } else if (entire) {
      store_columns<D>(o, sum == 0.f ? 0.f : 1.f / sum, a.out.at(item.tokens.first + token, head), row < rows, lane);
    } else if (row < rows) {
      const int64_t at = (int64_t)place * S::kRows + row_wave * 32 + (lane & 31);
      if (h == 0) *reinterpret_cast<float2*>(a.stats + 2 * at) = float2{top, sum};
#pragma unroll
      for (int i = 0; i < kParts; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 4) *reinterpret_cast<f32x4*>(a.sums + at * D + 32 * i + 2 * r + 4 * h) = f32x4{o[i][r], o[i][r + 1], o[i][r + 2], o[i][r + 3]};
    }
  };

  // the steps that are this workgroup's, and of which tile of rows: `before` steps are those of the tiles before the sequence's, `items` the tiles
  int64_t my_start = 0, my_end = 0, before = 0, items = 0;
  int sequence = -1;
  if (a.shares == 0) {
    int tile = 0;
    over_blocks<S::kRows, S::kStep>(a, group, [&](int first, int tiles, int) {
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
    const int all = (item.length + S::kStep - 1) / S::kStep;
    my_start = (int64_t)tile * all;
    my_end = my_start + all;
    if (all == 0) {                                          // rows that look at nothing
      const int rows = item.tokens.length * group;
      for (int i = (int)threadIdx.x; i < S::kRows * (D / 8); i += 64 * kDraftWaves) {
        const int row = tile * S::kRows + i / (D / 8);
        if (row < rows) *reinterpret_cast<u32x4*>(a.out.at(item.tokens.first + row / group, k_head * group + row % group) + i % (D / 8) * 8) = u32x4{};
      }
      return;
    }
  } else {
    int64_t total = 0;
    over_blocks<S::kRows, S::kStep>(a, group, [&](int, int tiles, int steps) {
      total += last_sum(rising_sum((uint32_t)tiles * (uint32_t)steps));
      return true;
    });
    const int shares = (int)min((int64_t)a.shares, total);
    if (share >= shares) return;
    my_start = total * share / shares;
    my_end = total * (share + 1) / shares;
    over_blocks<S::kRows, S::kStep>(a, group, [&](int first, int tiles, int steps) {
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
    const int tiles = (item.tokens.length * group + S::kRows - 1) / S::kRows, all = (item.length + S::kStep - 1) / S::kStep;
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

// What several workgroups have of a row joined, a wave for each token and query head, D / 64 dimensions a lane; and zeros for sequences without positions.
template <int D, int RW>
__global__ void __launch_bounds__(256) draft_join_kernel(DraftArgs a) {
  using S = DraftShape<D, RW>;
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
    const int tiles = (t.length * group + S::kRows - 1) / S::kRows;
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
  const int64_t item = items + row / S::kRows;
  if (item >= a.items) return;                               // (not where cu rises)
  const int2 parts = a.parts[item * heads + k_head];
  const int last = __builtin_amdgcn_readfirstlane(parts.y);
  if (last < 0) return;                                      // one workgroup had all of it
  const int first_part = __builtin_amdgcn_readfirstlane(parts.x), first = first_part / 2 / heads;
  if (last >= a.shares || first_part < 0 || first > last) return;
  auto place = [&](int share) { return (int64_t)(share == first ? first_part : (share * heads + k_head) * 2) * S::kRows + row % S::kRows; };
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
