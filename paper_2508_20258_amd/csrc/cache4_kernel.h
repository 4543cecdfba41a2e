// A cache of keys and values in 4 bits: writing it, reading it back, attention of single tokens over it.
//
// 64 values of a head share a step and a low, bfloat16 both: 36 bytes instead of 128.  16478 tokens of 8 heads of 128 (68 MB of keys and values, 19 MB of cache): writing 19 us, bound by the
// vector unit (93 %: four instructions a value for its number alone, then words of eight tokens through LDS), reading 16.3 us, 5.3 TB/s.
// Attention: the cache is read once, by all query heads of a key head together.  64 sequences of 512 to 8192 tokens, 32 heads of 128 sharing 8 (176 MB): 34 us, 5.1 TB/s, and
// 6.6 for the join, call after call on the same cache; among other work, which leaves none of it in the memory-side cache, 51 us in all.
#pragma once

#include "qk_norm_kernel.h"

namespace swz {

struct CacheArgs {
  uint32_t *k_words, *v_words, *k_scales, *v_scales;       // a scale: step in the low half, low in the high half
  const int32_t* table;
  int64_t pages;
  int page_shift, k_heads, table_width;
  // The page of a position, or -1.
  __device__ __forceinline__ int page_of(int sequence, int position) const {
    const int j = position >> page_shift;
    if (j >= table_width) return -1;
    const int page = table[(int64_t)sequence * table_width + j];
    return page >= 0 && page < pages ? page : -1;
  }
  // Tokens of a head before this one in the cache.
  __device__ __forceinline__ int64_t token_at(int page, int head, int position) const {
    return (((int64_t)page * k_heads + head) << page_shift) + (position & ((1 << page_shift) - 1));
  }
};

// Bits of a word that hold number e.
__device__ __forceinline__ int number_shift(int e) { return 4 * ((e >> 1) + 4 * (e & 1)); }

// op over 8 neighbouring lanes.
template <class Op>
__device__ __forceinline__ float over8(float x, Op op) {
  auto dpp = [](float v, auto ctrl) __attribute__((always_inline)) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false));
  };
  x = op(x, dpp(x, std::integral_constant<int, 0xB1>{}));
  x = op(x, dpp(x, std::integral_constant<int, 0x4E>{}));
  return op(x, dpp(x, std::integral_constant<int, 0x141>{}));
}

// Step and low (as a scale word) and the numbers (whole, as floats) of a group, 8 values in each of 8 lanes.  The number is that of the rounded quotient of x - low and step.  A product
// with 1 / step, corrected by its residual, is that quotient: what is left of the error is 2^-45 of it, and a quotient of 24 bits by 8 is no nearer than 2^-33 to a boundary of
// rounding.  A division instead is twice the instructions, and the vector unit is the bound.  Infinities, NaN and steps below the normal range come out as NaN and are
// divided.
__device__ __forceinline__ uint32_t quantise8(const u32x4& v, float (&number)[8]) {
  float x[8];
  unpack8(v, x);
  // (minimum, maximum: those that keep a NaN, which is found below; fminf and fmaxf would quiet every value first)
  auto lower = [](float a, float b) { return __builtin_elementwise_minimum(a, b); };
  auto higher = [](float a, float b) { return __builtin_elementwise_maximum(a, b); };
  float low = lower(x[0], x[1]), high = higher(x[0], x[1]);
#pragma unroll
  for (int e = 2; e < 8; e += 2) {
    low = lower(low, lower(x[e], x[e + 1]));
    high = higher(high, higher(x[e], x[e + 1]));
  }
  low = over8(low, lower);
  high = over8(high, higher);
  const float range = high - low;
  // range / 15 the same way: for all 2^23 fractions it is the rounded quotient, and a residual is exact as long as the step is a normal number
  const float fifteenth = range * (1.f / 15.f);
  uint32_t scale = pack_bf16(__builtin_fmaf(__builtin_fmaf(-fifteenth, 15.f, range), 1.f / 15.f, fifteenth), low);
  float step = __uint_as_float(scale << 16);
  const float inverse = step > 0.f ? __builtin_amdgcn_rcpf(step) : 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float above = x[e] - low, quotient = above * inverse;
    number[e] = rintf(__builtin_fmaf(__builtin_fmaf(-quotient, step, above), inverse, quotient));
  }
  const float all = ((number[0] + number[1]) + (number[2] + number[3])) + ((number[4] + number[5]) + (number[6] + number[7]));
  if (!__any(!(all >= 0.f))) return scale;
  float odd = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) odd += x[e] * 0.f;             // NaN where an entry is no finite number
  odd = over8(odd, [](float a, float b) { return a + b; });
  const bool bad = odd != 0.f || !(range < INFINITY);
  scale = pack_bf16(range / 15.f, low);
  step = __uint_as_float(scale << 16);
#pragma unroll
  for (int e = 0; e < 8; ++e) number[e] = !bad && step > 0.f ? fminf(rintf((x[e] - low) / step), 15.f) : 0.f;
  return bad ? 0x7fc07fc0u : scale;                          // NaN, NaN
}

struct StoreArgs {
  CacheArgs c;
  Heads k, v;
  const int32_t *cu, *before;
  int total, sequences, head_blocks, splits;         // workgroup i of `splits` for a word takes head blocks i, i + splits, ..
};

// Eight neighbouring positions of a sequence (a word of values) a workgroup, 256 / D heads at a time: finding the place takes four loads one after another, longer than the
// loads of the heads, which are then on their way a turn ahead.  The slots of a sequence start at its tokens / 8 + 2 * b,
// as its positions start anywhere in a word.
template <int D>
struct StoreShape {
  static constexpr int kLanes = D / 8, kHeads = 32 / kLanes;
};

struct StorePlace {
  int sequence, position, token, from, to, page;            // of the first of 8 positions: token of the call, and which of the 8 are real
};
__device__ __forceinline__ StorePlace store_place(const StoreArgs& a, int slot) {
  const SlotPlace s = find_slot<2>(a.cu, a.sequences, a.total, 8, slot);
  const Span t = sequence_span(a.cu, s.sequence, a.total);
  const int before = __builtin_amdgcn_readfirstlane(a.before[s.sequence]);
  StorePlace p;
  p.sequence = s.sequence;
  p.from = p.to = 0;
  if (before < 0 || s.tile < 0 || before > 0x7fffffff - t.length) return p;
  const int64_t position = (int64_t)((before >> 3) + s.tile) * 8, end = (int64_t)before + t.length;
  if (position >= end) return p;
  p.position = (int)position;
  p.token = t.first + (p.position - before);
  p.from = max(0, before - p.position);
  p.to = (int)min((int64_t)8, end - position);
  p.page = a.c.page_of(s.sequence, p.position);
  return p;
}

template <int D>
__global__ void __launch_bounds__(256) cache4_append_kernel(StoreArgs a) {
  using S = StoreShape<D>;
  __shared__ __attribute__((aligned(16))) unsigned char numbers[2][S::kHeads][8][D];
  const int slot = (int)blockIdx.x / a.splits, split = (int)blockIdx.x - slot * a.splits;
  const StorePlace p = store_place(a, slot);
  if (p.from >= p.to || p.page < 0) return;
  const int lane = (int)threadIdx.x % S::kLanes, place = ((int)threadIdx.x / S::kLanes) % 8, mine = (int)threadIdx.x / (8 * S::kLanes);
  const int d = (int)threadIdx.x % D, h = (int)threadIdx.x / D;
  const bool token = place >= p.from && place < p.to;
  uint32_t mask = 0;                                         // numbers of a word that are written
#pragma unroll
  for (int i = 0; i < 8; ++i) mask |= i >= p.from && i < p.to ? 15u << number_shift(i) : 0u;
  u32x4 k = u32x4{}, v = u32x4{};
  auto load = [&](int block) {
    const int head = block * S::kHeads + mine;
    if (!token || head >= a.c.k_heads) return;
    k = *reinterpret_cast<const u32x4*>(a.k.at(p.token + place, head) + lane * 8);
    v = *reinterpret_cast<const u32x4*>(a.v.at(p.token + place, head) + lane * 8);
  };
  load(split);
  for (int block = split, turn = 0; block < a.head_blocks; block += a.splits, turn ^= 1) {
    const int head = block * S::kHeads + mine;
    const bool real = token && head < a.c.k_heads;
    const int64_t at = a.c.token_at(p.page, min(head, a.c.k_heads - 1), p.position + place);
    const u32x4 keys = k, values = v;
    if (block + a.splits < a.head_blocks) load(block + a.splits);
    float n[8];
    uint32_t scale = quantise8(keys, n);
    if (real) {
      // number 2 i + h in bits 4 (i + 4 h)
      const float even = __builtin_fmaf(__builtin_fmaf(n[6], 16.f, n[4]), 256.f, __builtin_fmaf(n[2], 16.f, n[0]));
      const float odd = __builtin_fmaf(__builtin_fmaf(n[7], 16.f, n[5]), 256.f, __builtin_fmaf(n[3], 16.f, n[1]));
      a.c.k_words[at * (D / 8) + (D / 32) * (lane & 3) + (lane >> 2)] = (uint32_t)odd << 16 | (uint32_t)even;
      if ((lane & 7) == 0) a.c.k_scales[at * (D / 64) + (lane >> 3)] = scale;
    }
    scale = quantise8(values, n);
    if (real && (lane & 7) == 0) a.c.v_scales[at * (D / 64) + (lane >> 3)] = scale;
    u32x2 bytes = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) bytes[e / 4] |= (uint32_t)n[e] << (8 * (e % 4));
    *reinterpret_cast<u32x2*>(&numbers[turn][mine][place][lane * 8]) = bytes;
    __syncthreads();
    if (block * S::kHeads + h < a.c.k_heads) {
      uint32_t word = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) word |= (uint32_t)numbers[turn][h][i][d] << number_shift(i);
      word &= mask;
      uint32_t* to = a.c.v_words + (a.c.token_at(p.page, block * S::kHeads + h, p.position) >> 3) * D + d;
      if (mask != 0xffffffffu) word |= *to & ~mask;          // tokens that were there before
      *to = word;
    }
  }
}

template <int D>
__global__ void __launch_bounds__(256) cache4_read_kernel(StoreArgs a) {
  using S = StoreShape<D>;
  __shared__ __attribute__((aligned(16))) uint16_t values[2][S::kHeads][8][D];
  const int slot = (int)blockIdx.x / a.splits, split = (int)blockIdx.x - slot * a.splits;
  const StorePlace p = store_place(a, slot);
  if (p.from >= p.to) return;
  const int lane = (int)threadIdx.x % S::kLanes, place = ((int)threadIdx.x / S::kLanes) % 8, mine = (int)threadIdx.x / (8 * S::kLanes);
  const int d = (int)threadIdx.x % D, h = (int)threadIdx.x / D;
  const bool token = place >= p.from && place < p.to;
  auto value = [](uint32_t scale, uint32_t n) { return __builtin_fmaf(__uint_as_float(scale << 16), (float)n, __uint_as_float(scale & 0xffff0000u)); };
  constexpr uint32_t kNan = 0x7fc07fc0u;
  uint32_t k_word = 0, k_scale = kNan, v_word = 0, v_scale[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v_scale[i] = kNan;
  auto load = [&](int block) {
    if (p.page < 0) return;
    const int head = block * S::kHeads + mine, v_head = block * S::kHeads + h;
    if (token && head < a.c.k_heads) {
      const int64_t at = a.c.token_at(p.page, head, p.position + place);
      k_word = a.c.k_words[at * (D / 8) + (D / 32) * (lane & 3) + (lane >> 2)];
      k_scale = a.c.k_scales[at * (D / 64) + (lane >> 3)];
    }
    if (v_head < a.c.k_heads) {
      const int64_t at = a.c.token_at(p.page, v_head, p.position);
      v_word = a.c.v_words[(at >> 3) * D + d];
#pragma unroll
      for (int i = 0; i < 8; ++i) v_scale[i] = a.c.v_scales[(at + i) * (D / 64) + d / 64];
    }
  };
  load(split);
  for (int block = split, turn = 0; block < a.head_blocks; block += a.splits, turn ^= 1) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = value(k_scale, k_word >> number_shift(i) & 15u);
      values[turn][h][i][d] = __builtin_bit_cast(uint16_t, (__bf16)value(v_scale[i], v_word >> number_shift(i) & 15u));
    }
    if (block + a.splits < a.head_blocks) load(block + a.splits);
    const int head = block * S::kHeads + mine;
    const bool real = token && head < a.c.k_heads;
    if (real) *reinterpret_cast<u32x4*>(a.k.at(p.token + place, head) + lane * 8) = pack8(x);
    __syncthreads();
    if (real) *reinterpret_cast<u32x4*>(a.v.at(p.token + place, head) + lane * 8) = *reinterpret_cast<const u32x4*>(&values[turn][mine][place][lane * 8]);
  }
}

// ---------------------------------------------------------------- attention of one token of each sequence
//
// A wave takes 64 tokens of a key head at a time.  Scores: queries (A, rows) times keys (B, columns), a product for 16 tokens and 32 dimensions.  A matrix instruction has room
// for 16 queries, a key head has often 4: the queries then stand in all four groups of 4 rows, and lanes 16 g .. + 15 keep what they have of tokens 16 g .. + 15, so that
// each lane has one token and all that is done for a weight (scales, exponential, sums) is done once.  R rows: 4, 8 or 16, 64 R / 64 weights a lane.
// The weights go through LDS to the layout in which the product with the values takes them: values (A, rows are dimensions) times weights (B, columns are queries).
//
// Numbers n of a word become bfloat16 128 + n (0x4300 | n, two an instruction); products of scores start from -128 sum(q), and what the values' 136 adds is taken off with
// the rounded weights themselves.
//
// The steps of all sequences, in their order, are dealt evenly to the waves that a key head has, whatever the lengths: of `shares` waves, wave i has steps
// total * i / shares and up.  All key heads are dealt alike and neighbouring waves have neighbouring heads, whose tokens are neighbours in a page.  What a wave has of a sequence goes to
// `out` where that is all of it, else into one of two places of its own (the first sequence it works on, or the last), and cache4_join_kernel joins them.  Waves share nothing, and wait for
// nothing but their own loads; the loads of the next step's keys are issued when this one's are used up, and so for the values.
struct DecodeArgs {
  CacheArgs c;
  Heads q, out;
  const int32_t* lengths;
  float *sums, *stats;               // shares x heads x 2 x R x D, and x 2 (maximum, sum)
  int2* parts;                       // sequences x heads: place of the first part, share of the last
  int sequences, q_heads, columns;   // columns: blocks of 16 query heads of a key head, each a head of its own here
  int shares;
  float scale;
};

constexpr int kDecodeStep = 64, kDecodeWaves = 4, kOwnWaves = 8;

__device__ __forceinline__ int cached_length(const DecodeArgs& a, int sequence) {
  return (int)min((int64_t)max(a.lengths[sequence], 0), (int64_t)a.c.table_width << a.c.page_shift);
}
__device__ __forceinline__ int steps_of(int length) { return (length + kDecodeStep - 1) / kDecodeStep; }
// f(first sequence, steps of the lane's sequence, steps of the lane's and those before it) for 64 sequences at a time, until it says false.
template <class F>
__device__ __forceinline__ void over_sequences(const DecodeArgs& a, F&& f) {
  for (int first = 0; first < a.sequences; first += 64) {
    const int b = first + (int)(threadIdx.x & 63), n = b < a.sequences ? steps_of(cached_length(a, b)) : 0;
    if (!f(first, n, sum_before(n))) return;
  }
}

// The instruction takes no two constants, so they are kept in registers.
struct Numbers {
  uint32_t mask = 0x000f000fu, one = 0x43004300u;
  __device__ __forceinline__ Numbers() { asm volatile("" : "+s"(mask), "+v"(one)); }
  __device__ __forceinline__ bf16x8 operator()(uint32_t w) const {
    u32x4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = ((w >> (4 * i)) & mask) | one;
    return __builtin_bit_cast(bf16x8, x);
  }
};

__device__ __forceinline__ float scale_step(uint32_t s) { return __uint_as_float(s << 16); }
__device__ __forceinline__ float scale_low(uint32_t s) { return __uint_as_float(s & 0xffff0000u); }

// op over the four lanes l, l ^ 16, l ^ 32, l ^ 48.
template <class Op>
__device__ __forceinline__ float over_rows(float x, Op op) {
  const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return across_halves(op(__uint_as_float(s[0]), __uint_as_float(s[1])), op);
}
// op over the lanes that hold one query's weights: those of a row of 16, and of the rows R / 4 apart.
template <int R, class Op>
__device__ __forceinline__ float over_tokens(float x, Op op) {
  auto dpp = [](float v, auto ctrl) __attribute__((always_inline)) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false));
  };
  x = op(x, dpp(x, std::integral_constant<int, 0xB1>{}));        // quad_perm [1,0,3,2]
  x = op(x, dpp(x, std::integral_constant<int, 0x4E>{}));        // quad_perm [2,3,0,1]
  x = op(x, dpp(x, std::integral_constant<int, 0x141>{}));       // row_half_mirror
  x = op(x, dpp(x, std::integral_constant<int, 0x140>{}));       // row_mirror
  if constexpr (R == 4) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = op(__uint_as_float(s[0]), __uint_as_float(s[1]));
  }
  if constexpr (R <= 8) x = across_halves(x, op);
  return x;
}

// OWN: a workgroup of kOwnWaves for each sequence and key head instead, whose waves share its steps and join what they have in LDS.
template <int D, int R, bool OWN>
__global__ void __launch_bounds__(64 * (OWN ? kOwnWaves : kDecodeWaves), D == 128 && R >= 8 ? 2 : 3) cache4_attention_kernel(DecodeArgs a) {
  constexpr int kGroups = D / 64, kSteps = D / 32;
  constexpr int kQuads = R / 4, kSets = R / 4, kBlocks = 16 / R;      // row groups that a query's four rows take part in; sets of 4 weights a lane; blocks of 16 tokens of a set
  constexpr int kWaves = OWN ? kOwnWaves : kDecodeWaves;
  __shared__ __attribute__((aligned(16))) uint16_t weights[kWaves][kGroups][kDecodeStep][R];
  __shared__ __attribute__((aligned(16))) float own_sums[OWN ? kWaves : 1][OWN ? R : 1][D], own_stats[OWN ? kWaves : 1][OWN ? R : 1][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int heads = a.c.k_heads * a.columns, group = a.q_heads / a.c.k_heads;
  const int id = OWN ? (int)blockIdx.x : (int)blockIdx.x * kDecodeWaves + wave, share = id / heads, pair = id - share * heads;
  int sequence = 0;
  int64_t before = 0, my_start = 0, my_end = 0;              // before: steps of the sequences before it
  if constexpr (OWN) {
    sequence = share;
    const int all = steps_of(__builtin_amdgcn_readfirstlane(cached_length(a, sequence)));
    my_start = (int64_t)all * wave / kWaves;
    my_end = (int64_t)all * (wave + 1) / kWaves;
    if (lane < R) own_stats[wave][lane][0] = -FLT_MAX, own_stats[wave][lane][1] = 0.f;
  } else {
    int64_t total = 0;
    over_sequences(a, [&](int, int, int sum) {
      total += __builtin_amdgcn_readlane(sum, 63);
      return true;
    });
    const int shares = (int)min((int64_t)a.shares, total);
    if (share >= shares) return;
    my_start = total * share / shares;
    my_end = total * (share + 1) / shares;
    over_sequences(a, [&](int first, int n, int sum) {
      const uint64_t found = __ballot(my_start < before + sum);
      if (found == 0) {
        before += __builtin_amdgcn_readlane(sum, 63);
        return true;
      }
      const int s = __ffsll((unsigned long long)found) - 1;
      sequence = first + s;
      before += __builtin_amdgcn_readlane(sum - n, s);
      return false;
    });
  }
  const int k_head = pair / a.columns, column = pair - k_head * a.columns;
  const int head0 = k_head * group + column * 16, queries = min(16, group - column * 16);

  typedef __attribute__((ext_vector_type(kSteps))) uint32_t k_vec;
  typedef __attribute__((ext_vector_type(kGroups))) uint32_t scale_vec;
  typedef __attribute__((address_space(3))) s16x4* tr_ptr;
  const Numbers numbers;
  const float c = a.scale * kLog2E;
  const uint32_t weights_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)&weights[wave][0][0][0];
  // transposing reads: 4 tokens of a row each; columns from R on are what they may be, nothing reads them
  const uint32_t read_at = weights_at + (uint32_t)((8 * g + (n >> 2)) * 2 * R + (n & 3) % kQuads * 8);
  auto token_of = [&](int u) { return 16 * (u * kBlocks + g / kQuads) + n; };            // of a step: the lane's in set u
  // of what the lanes hold for their queries (4 (g mod kQuads) + r): that of query n
  auto of_query = [&](const float (&x)[4]) __attribute__((always_inline)) {
    float mine = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float f = __int_as_float(__builtin_amdgcn_ds_bpermute(n / 4 % kQuads * 64, __float_as_int(x[r])));
      mine = (n & 3) == r ? f : mine;
    }
    return mine;
  };

  for (int64_t step = my_start; step < my_end; ++sequence) {
    const int length = __builtin_amdgcn_readfirstlane(cached_length(a, sequence)), all = steps_of(length);
    if (all == 0) continue;
    const int from = (int)(step - before), count = (int)min((int64_t)(all - from), my_end - step);
    const int begin = from * kDecodeStep, end = min(length, (from + count) * kDecodeStep);

    // queries, in all groups of R rows, and -128 times their sums over a group of dimensions: of the lane's four, 4 (g mod kQuads) + r
    bf16x8 q[kSteps];
    f32x4 start[kGroups];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      q[s] = bf16x8{};
      if (n % R < queries) q[s] = *reinterpret_cast<const bf16x8*>(a.q.at(sequence, head0 + n % R) + 32 * s + 8 * g);
    }

    // keys and values of a step; pages have 32 tokens and more: one for each half of it, looked up a step ahead
    int page[2], next_page[2];
    int64_t at[2];
    k_vec k[4];
    u32x4 v[2][kGroups];
    scale_vec ks[kSets], vs[kSets];
    auto look_up = [&](int t) __attribute__((always_inline)) {
#pragma unroll
      for (int half = 0; half < 2; ++half) next_page[half] = t + 32 * half < end ? a.c.page_of(sequence, t + 32 * half) : 0;
    };
    auto scale_place = [&](int u) {
      const int token = token_of(u);
      return ((token < 32 ? at[0] : at[1]) + (token & 31)) * kGroups;
    };
    auto load_keys = [&](int t) __attribute__((always_inline)) {       // of step t and what places its values; page stays that of the step before
#pragma unroll
      for (int half = 0; half < 2; ++half) at[half] = a.c.token_at(max(next_page[half], 0), k_head, t + 32 * half);
#pragma unroll
      for (int b = 0; b < 4; ++b) k[b] = *reinterpret_cast<const k_vec*>(a.c.k_words + (at[b / 2] + 16 * (b & 1) + n) * (D / 8) + kSteps * g);
#pragma unroll
      for (int u = 0; u < kSets; ++u) ks[u] = *reinterpret_cast<const scale_vec*>(a.c.k_scales + scale_place(u));
    };
    auto load_values = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < kSets; ++u) vs[u] = *reinterpret_cast<const scale_vec*>(a.c.v_scales + scale_place(u));
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < kGroups; ++i) v[half][i] = *reinterpret_cast<const u32x4*>(a.c.v_words + ((at[half] >> 3) + g) * D + 64 * i + 4 * n);
    };
    look_up(begin);
    load_keys(begin);
    load_values();
    page[0] = next_page[0];
    page[1] = next_page[1];
    look_up(begin + kDecodeStep);

#pragma unroll
    for (int j = 0; j < kGroups; ++j) {
      float mine = 0.f;                                      // of query n % R
#pragma unroll
      for (int s = 2 * j; s < 2 * j + 2; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) mine += (float)q[s][e];
      mine = -128.f * over_rows(mine, [](float x, float y) { return x + y; });
#pragma unroll
      for (int r = 0; r < 4; ++r) start[j][r] = __int_as_float(__builtin_amdgcn_ds_bpermute((4 * (g % kQuads) + r) * 4, __float_as_int(mine)));
    }
    f32x4 o[kGroups][4];
    float mids[kGroups][4], top[4], sum[4];                  // of the lane's queries; sums over the lane's tokens
#pragma unroll
    for (int i = 0; i < kGroups; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i][j] = f32x4{}, mids[i][j] = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) top[r] = -FLT_MAX, sum[r] = 0.f;

    for (int t = begin; t < end; t += kDecodeStep) {
      float x[kSets][4];
#pragma unroll
      for (int u = 0; u < kSets; ++u) {
        f32x4 y[2][kGroups], s[kGroups];
        auto take = [&](int p) __attribute__((always_inline)) {        // of block p, by the lanes that keep it
#pragma unroll
          for (int i = 0; i < kGroups; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[i][r] = p == 0 || g / kQuads == p ? y[p % 2][i][r] : s[i][r];
        };
#pragma unroll
        for (int p = 0; p < kBlocks; ++p) {
#pragma unroll
          for (int i = 0; i < kGroups; ++i) {
            y[p % 2][i] = start[i];
#pragma unroll
            for (int w = 2 * i; w < 2 * i + 2; ++w) y[p % 2][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[w], numbers(k[u * kBlocks + p][w]), y[p % 2][i], 0, 0, 0);
          }
          if (p > 0) take(p - 1);
          __builtin_amdgcn_sched_barrier(0);                // or all words are taken apart at once, and registers run out
        }
        take(kBlocks - 1);
        const int token = token_of(u);
        if (t + 32 * (token / 32) < end && (token < 32 ? page[0] : page[1]) < 0) ks[u][0] = 0x7fc07fc0u;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[u][r] = 0.f;
#pragma unroll
          for (int i = 0; i < kGroups; ++i) x[u][r] = __builtin_fmaf(scale_step(ks[u][i]), s[i][r], __builtin_fmaf(scale_low(ks[u][i]) * (-1.f / 128), start[i][r], x[u][r]));
          x[u][r] *= c;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      const bool more = t + kDecodeStep < end;
      if (more) load_keys(t + kDecodeStep);
      if (!more && t + kDecodeStep > end) {
#pragma unroll
        for (int u = 0; u < kSets; ++u) {
          const bool real = t + token_of(u) < end;
#pragma unroll
          for (int i = 0; i < kGroups; ++i) vs[u][i] = real ? vs[u][i] : 0u;
#pragma unroll
          for (int r = 0; r < 4; ++r) x[u][r] = real ? x[u][r] : -INFINITY;
        }
      }
      bool higher = false;
#pragma unroll
      for (int u = 0; u < kSets; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) higher |= x[u][r] > top[r] + kLazyRise;
      if (__any(higher)) {
        float less[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float high = x[0][r];
#pragma unroll
          for (int u = 1; u < kSets; ++u) high = fmaxf(high, x[u][r]);
          const float now = fmaxf(top[r], over_tokens<R>(high, [](float y, float z) { return fmaxf(y, z); }));
          less[r] = __builtin_amdgcn_exp2f(top[r] - now);
          top[r] = now;
          sum[r] *= less[r];
#pragma unroll
          for (int i = 0; i < kGroups; ++i) mids[i][r] *= less[r];
        }
        const float mine = of_query(less);
#pragma unroll
        for (int i = 0; i < kGroups; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) o[i][j] *= mine;
      }
      // value = mid + step (n - 8): the rounding of a weight times step then costs in proportion to the value, not to the range of its group
#pragma unroll
      for (int u = 0; u < kSets; ++u) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[u][r] = __builtin_amdgcn_exp2f(x[u][r] - top[r]);
          sum[r] += x[u][r];
        }
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
          const float size = scale_step(vs[u][i]), mid = __builtin_fmaf(size, 8.f, scale_low(vs[u][i]));
#pragma unroll
          for (int r = 0; r < 4; ++r) mids[i][r] = __builtin_fmaf(x[u][r], mid, mids[i][r]);
          const u32x2 w = {pack_bf16(x[u][0] * size, x[u][1] * size), pack_bf16(x[u][2] * size, x[u][3] * size)};
          *reinterpret_cast<u32x2*>(&weights[wave][i][token_of(u)][4 * (g % kQuads)]) = w;
#pragma unroll
          for (int r = 0; r < 4; ++r) mids[i][r] = __builtin_fmaf(-136.f, r % 2 == 0 ? __uint_as_float(w[r / 2] << 16) : __uint_as_float(w[r / 2] & 0xffff0000u), mids[i][r]);
        }
      }
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
          const uint32_t w_at = read_at + (uint32_t)((i * kDecodeStep + 32 * half) * 2 * R);
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(uintptr_t)w_at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(uintptr_t)(w_at + 8 * R));
          const bf16x8 p = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            o[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(numbers(v[half][i][j]), p, o[i][j], 0, 0, 0);
            if (j % 2 == 1) __builtin_amdgcn_sched_barrier(0);
          }
        }
      if (more) {
        load_values();
        page[0] = next_page[0];
        page[1] = next_page[1];
        look_up(t + 2 * kDecodeStep);
      }
    }

#pragma unroll
    for (int r = 0; r < 4; ++r) {
      sum[r] = over_tokens<R>(sum[r], [](float x, float y) { return x + y; });
#pragma unroll
      for (int i = 0; i < kGroups; ++i) mids[i][r] = over_tokens<R>(mids[i][r], [](float x, float y) { return x + y; });
    }
    const float my_sum = of_query(sum), my_top = of_query(top);
    const bool whole = !OWN && count == all;
    const float f = !whole ? 1.f : my_sum == 0.f ? 0.f : 1.f / my_sum;
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const float mid = of_query(mids[i]);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][j][e] = (o[i][j][e] + mid) * f;
    }
    // query n's dimensions 64 i + 16 g + 4 e + j
    if (n < queries) {
      if (whole) {
#pragma unroll
        for (int i = 0; i < kGroups; ++i)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            float y[8];
#pragma unroll
            for (int z = 0; z < 8; ++z) y[z] = o[i][z % 4][2 * half + z / 4];
            *reinterpret_cast<u32x4*>(a.out.at(sequence, head0 + n) + 64 * i + 16 * g + 8 * half) = pack8(y);
          }
      } else if constexpr (OWN) {
#pragma unroll
        for (int i = 0; i < kGroups; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) *reinterpret_cast<f32x4*>(&own_sums[wave][n][64 * i + 16 * g + 4 * e]) = f32x4{o[i][0][e], o[i][1][e], o[i][2][e], o[i][3][e]};
        if (g == 0) own_stats[wave][n][0] = my_top, own_stats[wave][n][1] = my_sum;
      } else {
        const int part = id * 2 + (step == my_start ? 0 : 1);
        const int64_t to = (int64_t)part * R + n;
#pragma unroll
        for (int i = 0; i < kGroups; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<f32x4*>(a.sums + to * D + 64 * i + 16 * g + 4 * e) = f32x4{o[i][0][e], o[i][1][e], o[i][2][e], o[i][3][e]};
        if (g == 0) *reinterpret_cast<float2*>(a.stats + to * 2) = float2{my_top, my_sum};
        if (lane == 0 && from == 0) a.parts[sequence * heads + pair].x = part;
      }
    }
    if (!OWN && lane == 0 && from + count == all) a.parts[sequence * heads + pair].y = whole ? -1 : share;
    step += count;
    before += all;
  }
  if constexpr (OWN) {
    __syncthreads();
    for (int i = (int)threadIdx.x; i < queries * (D / 2); i += 64 * kWaves) {
      const int query = i / (D / 2), d = i % (D / 2) * 2;
      float top = -FLT_MAX, sum = 0.f, x = 0.f, y = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, own_stats[w][query][0]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float its = own_stats[w][query][1], f = __builtin_amdgcn_exp2f(own_stats[w][query][0] - top);
        if (its == 0.f) continue;                            // no steps, and nothing written
        sum = __builtin_fmaf(its, f, sum);
        x = __builtin_fmaf(own_sums[w][query][d], f, x);
        y = __builtin_fmaf(own_sums[w][query][d + 1], f, y);
      }
      const float f = sum == 0.f ? 0.f : 1.f / sum;
      *reinterpret_cast<uint32_t*>(a.out.at(share, head0 + query) + d) = pack_bf16(x * f, y * f);
    }
  }
}

// What several waves have of a sequence's key head joined, a workgroup for each query head; and zeros for sequences without tokens.
constexpr int kJoinWaves = 4;
template <int D>
__global__ void __launch_bounds__(64 * kJoinWaves) cache4_join_kernel(DecodeArgs a, int rows) {
  constexpr int kPer = D / 64;
  typedef __attribute__((ext_vector_type(kPer))) float vec;
  __shared__ float joined[kJoinWaves][D], joined_stats[kJoinWaves][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int sequence = (int)blockIdx.x / a.q_heads, head = (int)blockIdx.x - sequence * a.q_heads;
  const int heads = a.c.k_heads * a.columns, group = a.q_heads / a.c.k_heads, k_head = head / group, member = head - k_head * group;
  uint16_t* to = a.out.at(sequence, head) + lane * kPer;
  const int pair = k_head * a.columns + member / 16;
  const int2 parts = a.parts[sequence * heads + pair];
  if (__builtin_amdgcn_readfirstlane(cached_length(a, sequence)) == 0) {
    if (wave == 0)
#pragma unroll
      for (int i = 0; i < kPer; ++i) to[i] = 0;
    return;
  }
  const int last = __builtin_amdgcn_readfirstlane(parts.y);
  if (last < 0) return;                                     // one wave had all of it
  const int first_part = __builtin_amdgcn_readfirstlane(parts.x), first = first_part / 2 / heads;
  auto place = [&](int share) { return (int64_t)(share == first ? first_part : (share * heads + pair) * 2) * rows + member % 16; };
  float top = -FLT_MAX, sum = 0.f;
  vec o = 0.f;
  // 64 of a wave's parts at a time, a lane each for their statistics
  for (int from = first + wave; from <= last; from += 64 * kJoinWaves) {
    const int mine = from + lane * kJoinWaves;
    float2 x = {-FLT_MAX, 0.f};
    if (mine <= last) x = *reinterpret_cast<const float2*>(a.stats + 2 * place(mine));
    const float now = fmaxf(top, over_wave(x.x, [](float y, float z) { return fmaxf(y, z); })), less = __builtin_amdgcn_exp2f(top - now);
    const float weight = __builtin_amdgcn_exp2f(x.x - now);
    sum = sum * less + over_wave(x.y * weight, [](float y, float z) { return y + z; });
    o *= less;
    top = now;
    const int parts = min(64, (last - from) / kJoinWaves + 1);
#pragma unroll 4
    for (int p = 0; p < parts; ++p)
      o += *reinterpret_cast<const vec*>(a.sums + place(from + p * kJoinWaves) * D + lane * kPer) * __int_as_float(__builtin_amdgcn_readlane(__float_as_int(weight), p));
  }
  *reinterpret_cast<vec*>(&joined[wave][lane * kPer]) = o;
  if (lane == 0) joined_stats[wave][0] = top, joined_stats[wave][1] = sum;
  __syncthreads();
  if (wave > 0) return;
  float highest = -FLT_MAX, total = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinWaves; ++w) highest = fmaxf(highest, joined_stats[w][0]);
  o = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinWaves; ++w) {
    const float f = __builtin_amdgcn_exp2f(joined_stats[w][0] - highest);
    total += joined_stats[w][1] * f;
    o += *reinterpret_cast<const vec*>(&joined[w][lane * kPer]) * f;
  }
  const float f = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
  for (int i = 0; i < kPer; ++i) to[i] = __builtin_bit_cast(uint16_t, (__bf16)(o[i] * f));
}

}  // namespace swz
