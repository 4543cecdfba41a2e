// A cache of keys and values in 4 bits: writing it, reading it back, attention of single tokens over it.
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

// Step and low (as a scale word) and the numbers of a group, 8 values in each of 8 lanes.
__device__ __forceinline__ uint32_t quantise8(const u32x4& v, uint32_t (&number)[8]) {
  float x[8];
  unpack8(v, x);
  float low = x[0], high = x[0], odd = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    low = fminf(low, x[e]);
    high = fmaxf(high, x[e]);
    odd += x[e] * 0.f;                                       // NaN where an entry is no finite number
  }
  low = over8(low, [](float a, float b) { return fminf(a, b); });
  high = over8(high, [](float a, float b) { return fmaxf(a, b); });
  odd = over8(odd, [](float a, float b) { return a + b; });
  const float range = high - low;
  if (odd != 0.f || !(range < INFINITY)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) number[e] = 0;
    return 0x7fc07fc0u;                                      // NaN, NaN
  }
  const uint32_t scale = pack_bf16(range / 15.f, low);
  const float step = __uint_as_float(scale << 16);
#pragma unroll
  for (int e = 0; e < 8; ++e) number[e] = step > 0.f ? (uint32_t)fminf(rintf((x[e] - low) / step), 15.f) : 0u;
  return scale;
}

struct StoreArgs {
  CacheArgs c;
  Heads k, v;
  const int32_t *cu, *before;
  int total, sequences, head_blocks;
};

// Eight neighbouring positions of a sequence (a word of values) and 2048 / D heads a workgroup.  The slots of a sequence start at its tokens / 8 + 2 * b,
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
  __shared__ __attribute__((aligned(16))) unsigned char numbers[S::kHeads][8][D];
  const int slot = (int)blockIdx.x / a.head_blocks, head0 = ((int)blockIdx.x - slot * a.head_blocks) * S::kHeads;
  const StorePlace p = store_place(a, slot);
  if (p.from >= p.to || p.page < 0) return;
  const int lane = (int)threadIdx.x % S::kLanes, e = ((int)threadIdx.x / S::kLanes) % 8, mine = (int)threadIdx.x / (8 * S::kLanes), head = head0 + mine;
  const bool real = head < a.c.k_heads && e >= p.from && e < p.to;
  u32x4 k = u32x4{}, v = u32x4{};
  if (real) {
    k = *reinterpret_cast<const u32x4*>(a.k.at(p.token + e, head) + lane * 8);
    v = *reinterpret_cast<const u32x4*>(a.v.at(p.token + e, head) + lane * 8);
  }
  const int64_t at = a.c.token_at(p.page, min(head, a.c.k_heads - 1), p.position + e);
  uint32_t n[8];
  uint32_t scale = quantise8(k, n);
  if (real) {
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) word |= n[i] << number_shift(i);
    a.c.k_words[at * (D / 8) + (D / 32) * (lane & 3) + (lane >> 2)] = word;
    if ((lane & 7) == 0) a.c.k_scales[at * (D / 64) + (lane >> 3)] = scale;
  }
  scale = quantise8(v, n);
  if (real && (lane & 7) == 0) a.c.v_scales[at * (D / 64) + (lane >> 3)] = scale;
  *reinterpret_cast<u32x2*>(&numbers[mine][e][lane * 8]) =
      u32x2{n[0] | n[1] << 8 | n[2] << 16 | n[3] << 24, n[4] | n[5] << 8 | n[6] << 16 | n[7] << 24};
  __syncthreads();
  const int d = (int)threadIdx.x % D, h = (int)threadIdx.x / D;
  if (head0 + h >= a.c.k_heads) return;
  uint32_t word = 0, mask = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i >= p.from && i < p.to) {
      word |= (uint32_t)numbers[h][i][d] << number_shift(i);
      mask |= 15u << number_shift(i);
    }
  uint32_t* to = a.c.v_words + (a.c.token_at(p.page, head0 + h, p.position) >> 3) * D + d;
  if (mask != 0xffffffffu) word |= *to & ~mask;              // tokens that were there before
  *to = word;
}

template <int D>
__global__ void __launch_bounds__(256) cache4_read_kernel(StoreArgs a) {
  using S = StoreShape<D>;
  __shared__ __attribute__((aligned(16))) uint16_t values[S::kHeads][8][D];
  const int slot = (int)blockIdx.x / a.head_blocks, head0 = ((int)blockIdx.x - slot * a.head_blocks) * S::kHeads;
  const StorePlace p = store_place(a, slot);
  if (p.from >= p.to) return;
  const int lane = (int)threadIdx.x % S::kLanes, e = ((int)threadIdx.x / S::kLanes) % 8, mine = (int)threadIdx.x / (8 * S::kLanes), head = head0 + mine;
  const bool real = head < a.c.k_heads && e >= p.from && e < p.to;
  auto value = [](uint32_t scale, uint32_t n) { return __builtin_fmaf(__uint_as_float(scale << 16), (float)n, __uint_as_float(scale & 0xffff0000u)); };
  if (real) {
    uint32_t word = 0, scale = 0x7fc07fc0u;
    if (p.page >= 0) {
      const int64_t at = a.c.token_at(p.page, head, p.position + e);
      word = a.c.k_words[at * (D / 8) + (D / 32) * (lane & 3) + (lane >> 2)];
      scale = a.c.k_scales[at * (D / 64) + (lane >> 3)];
    }
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = value(scale, word >> number_shift(i) & 15u);
    *reinterpret_cast<u32x4*>(a.k.at(p.token + e, head) + lane * 8) = pack8(x);
  }
  const int d = (int)threadIdx.x % D, h = (int)threadIdx.x / D;
  if (head0 + h < a.c.k_heads) {
    const int64_t at = p.page < 0 ? 0 : a.c.token_at(p.page, head0 + h, p.position);
    const uint32_t word = p.page < 0 ? 0u : a.c.v_words[(at >> 3) * D + d];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t scale = p.page < 0 ? 0x7fc07fc0u : a.c.v_scales[(at + i) * (D / 64) + d / 64];
      values[h][i][d] = __builtin_bit_cast(uint16_t, (__bf16)value(scale, word >> number_shift(i) & 15u));
    }
  }
  __syncthreads();
  if (real) *reinterpret_cast<u32x4*>(a.v.at(p.token + e, head) + lane * 8) = *reinterpret_cast<const u32x4*>(&values[mine][e][lane * 8]);
}

// ---------------------------------------------------------------- attention of one token of each sequence

struct DecodeArgs {
  CacheArgs c;
  Heads q, out;
  const int32_t* lengths;
  float *sums, *stats;               // of the parts of a sequence: sequences x q_heads x parts x D, and x 2 (maximum, sum)
  int sequences, q_heads, columns;   // columns: blocks of 16 query heads of a key head
  int parts, part_tokens;
  float scale;
};

// Numbers n of a word as bfloat16 128 + n, which is 0x4300 | n: a pair of them an instruction.
__device__ __forceinline__ bf16x8 numbers_128(uint32_t w) {
  u32x4 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = ((w >> (4 * i)) & 0x000f000fu) | 0x43004300u;
  return __builtin_bit_cast(bf16x8, x);
}

__device__ __forceinline__ float scale_step(uint32_t s) { return __uint_as_float(s << 16); }
__device__ __forceinline__ float scale_low(uint32_t s) { return __uint_as_float(s & 0xffff0000u); }

// op over the four lanes l, l ^ 16, l ^ 32, l ^ 48.
template <class Op>
__device__ __forceinline__ float over_rows(float x, Op op) {
  const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return across_halves(op(__uint_as_float(s[0]), __uint_as_float(s[1])), op);
}

// What 32 tokens of a head are in the cache, as the lanes of a wave take them (lane 16 g + m).
template <int D>
struct Raw {
  uint32_t k[2][D / 32];             // token 8 (m / 4) + 4 b + m % 4, words D / 32 * g ..
  u32x4 v[D / 64];                   // tokens 8 g .. + 7, dimensions 64 i + 4 m .. + 3
  uint32_t ks[8][D / 64], vs[8][D / 64];   // scales of tokens 8 g .. + 7
};

template <int D>
__device__ __forceinline__ void load_raw(Raw<D>& r, const CacheArgs& c, int page, int head, int position, int lane) {
  const int m = lane & 15, g = lane >> 4;
  const int64_t at = c.token_at(page, head, position);
  typedef __attribute__((ext_vector_type(D / 32))) uint32_t k_vec;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const k_vec w = *reinterpret_cast<const k_vec*>(c.k_words + (at + 8 * (m >> 2) + 4 * b + (m & 3)) * (D / 8) + (D / 32) * g);
#pragma unroll
    for (int s = 0; s < D / 32; ++s) r.k[b][s] = w[s];
  }
#pragma unroll
  for (int i = 0; i < D / 64; ++i) r.v[i] = *reinterpret_cast<const u32x4*>(c.v_words + ((at >> 3) + g) * D + 64 * i + 4 * m);
#pragma unroll
  for (int i = 0; i < 2 * (D / 64); ++i) {
    const u32x4 k = *reinterpret_cast<const u32x4*>(c.k_scales + (at + 8 * g) * (D / 64) + 4 * i), v = *reinterpret_cast<const u32x4*>(c.v_scales + (at + 8 * g) * (D / 64) + 4 * i);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      r.ks[(4 * i + e) / (D / 64)][(4 * i + e) % (D / 64)] = k[e];
      r.vs[(4 * i + e) / (D / 64)][(4 * i + e) % (D / 64)] = v[e];
    }
  }
}

template <int D, int NW>
__global__ void __launch_bounds__(NW * 64) cache4_attention_kernel(DecodeArgs a) {
  constexpr int kGroups = D / 64, kSteps = D / 32;
  __shared__ f32x4 merge[NW / 2][4 * kGroups][64];
  __shared__ float merge_stats[NW / 2][2][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  int rest = (int)blockIdx.x;
  const int column = rest % a.columns;
  rest /= a.columns;
  const int k_head = rest % a.c.k_heads;
  rest /= a.c.k_heads;
  const int sequence = rest % a.sequences, part = rest / a.sequences;
  const int group = a.q_heads / a.c.k_heads, head = k_head * group + column * 16 + n;
  const bool real = column * 16 + n < group;
  const int length = (int)min((int64_t)max(__builtin_amdgcn_readfirstlane(a.lengths[sequence]), 0), (int64_t)a.c.table_width << a.c.page_shift);
  const int begin = part * a.part_tokens, end = (int)min((int64_t)length, (int64_t)begin + a.part_tokens);
  if (part > 0 && begin >= length) return;

  bf16x8 q[kSteps];
  float q_sum[kGroups];
#pragma unroll
  for (int j = 0; j < kGroups; ++j) q_sum[j] = 0.f;
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    q[s] = bf16x8{};
    if (real) q[s] = *reinterpret_cast<const bf16x8*>(a.q.at(sequence, head) + 32 * s + 8 * g);
#pragma unroll
    for (int e = 0; e < 8; ++e) q_sum[s / 2] += (float)q[s][e];
  }
#pragma unroll
  for (int j = 0; j < kGroups; ++j) q_sum[j] = over_rows(q_sum[j], [](float x, float y) { return x + y; });

  const float c = a.scale * kLog2E;
  const u32x4 minus_136 = {0xc308c308u, 0xc308c308u, 0xc308c308u, 0xc308c308u};
  f32x4 o[kGroups][4], shift[kGroups];
  float mids[kGroups], top = -FLT_MAX, sum = 0.f;
#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    mids[i] = 0.f;
    shift[i] = f32x4{};
#pragma unroll
    for (int j = 0; j < 4; ++j) o[i][j] = f32x4{};
  }

  for (int t = begin + 32 * wave; t < end; t += 32 * NW) {
    const int page = a.c.page_of(sequence, t);
    Raw<D> r;
    load_raw<D>(r, a.c, page < 0 ? 0 : page, k_head, t, lane);
    if (page < 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) r.ks[e][0] = 0x7fc07fc0u;
    }
    if (t + 32 > end) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int i = 0; i < kGroups; ++i) r.vs[e][i] = t + 8 * g + e < end ? r.vs[e][i] : 0u;
    }
    float x[8];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        f32x4 s = f32x4{};
#pragma unroll
        for (int u = 2 * i; u < 2 * i + 2; ++u) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(numbers_128(r.k[b][u]), q[u], s, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t w = r.ks[4 * b + e][i];
          const float part_score = __builtin_fmaf(scale_step(w), __builtin_fmaf(q_sum[i], -128.f, s[e]), scale_low(w) * q_sum[i]);
          x[4 * b + e] = i == 0 ? part_score : x[4 * b + e] + part_score;
        }
      }
    }
    if (t + 32 > end) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = t + 8 * g + e < end ? x[e] : -INFINITY;
    }
    float high = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) high = fmaxf(high, x[e]);
    high = over_rows(high, [](float y, float z) { return fmaxf(y, z); }) * c;
    if (__any(high > top + kLazyRise)) {
      const float now = fmaxf(top, high), less = __builtin_amdgcn_exp2f(top - now);
      sum *= less;
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        mids[i] *= less;
        shift[i] *= less;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[i][j] *= less;
      }
      top = now;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], c, -top));
      sum += x[e];
    }
    // value = mid + step (n - 8): the rounding of a weight times step then costs in proportion to the value, not to the range of its group
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = pack_bf16(x[2 * e] * scale_step(r.vs[2 * e][i]), x[2 * e + 1] * scale_step(r.vs[2 * e + 1][i]));
      const bf16x8 p = __builtin_bit_cast(bf16x8, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) mids[i] = __builtin_fmaf(x[e], __builtin_fmaf(scale_step(r.vs[e][i]), 8.f, scale_low(r.vs[e][i])), mids[i]);
      shift[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, minus_136), p, shift[i], 0, 0, 0);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(numbers_128(r.v[i][j]), p, o[i][j], 0, 0, 0);
    }
  }

#pragma unroll
  for (int i = 0; i < kGroups; ++i) {
    mids[i] = over_rows(mids[i], [](float x, float y) { return x + y; });
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][j][e] += shift[i][e] + mids[i];
  }
  sum = over_rows(sum, [](float x, float y) { return x + y; });

  // the waves in halves: the upper one's sums go to the lower one
#pragma unroll
  for (int half = NW / 2; half > 0; half /= 2) {
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int i = 0; i < kGroups; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) merge[wave - half][4 * i + j][lane] = o[i][j];
      merge_stats[wave - half][0][lane] = top;
      merge_stats[wave - half][1][lane] = sum;
    }
    __syncthreads();
    if (wave < half) {
      const float their_top = merge_stats[wave][0][lane], now = fmaxf(top, their_top);
      const float mine = __builtin_amdgcn_exp2f(top - now), theirs = __builtin_amdgcn_exp2f(their_top - now);
      sum = sum * mine + merge_stats[wave][1][lane] * theirs;
#pragma unroll
      for (int i = 0; i < kGroups; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[i][j] = o[i][j] * mine + merge[wave][4 * i + j][lane] * theirs;
      top = now;
    }
    __syncthreads();
  }
  if (wave > 0 || !real) return;
  // query n's dimensions 64 i + 16 g + 4 e + j
  if (a.parts == 1) {
    const float f = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int i = 0; i < kGroups; ++i)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float y[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) y[x] = o[i][x % 4][2 * half + x / 4] * f;
        *reinterpret_cast<u32x4*>(a.out.at(sequence, head) + 64 * i + 16 * g + 8 * half) = pack8(y);
      }
  } else {
    const int64_t at = ((int64_t)sequence * a.q_heads + head) * a.parts + part;
#pragma unroll
    for (int i = 0; i < kGroups; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<f32x4*>(a.sums + at * D + 64 * i + 16 * g + 4 * e) = f32x4{o[i][0][e], o[i][1][e], o[i][2][e], o[i][3][e]};
    if (g == 0) {
      a.stats[at * 2] = top;
      a.stats[at * 2 + 1] = sum;
    }
  }
}

// The parts of a sequence joined, a wave for each query head.
template <int D>
__global__ void __launch_bounds__(256) cache4_join_kernel(DecodeArgs a) {
  constexpr int kPer = D / 64;
  typedef __attribute__((ext_vector_type(kPer))) float vec;
  const int lane = threadIdx.x & 63, id = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  if (id >= a.sequences * a.q_heads) return;
  const int sequence = id / a.q_heads, head = id - sequence * a.q_heads;
  const int length = (int)min((int64_t)max(__builtin_amdgcn_readfirstlane(a.lengths[sequence]), 0), (int64_t)a.c.table_width << a.c.page_shift);
  const int parts = (int)min((int64_t)a.parts, ((int64_t)length + a.part_tokens - 1) / a.part_tokens);
  const float* stats = a.stats + (int64_t)id * a.parts * 2;
  const float* sums = a.sums + (int64_t)id * a.parts * D + lane * kPer;
  float top = -FLT_MAX;
  for (int p = 0; p < parts; ++p) top = fmaxf(top, stats[2 * p]);
  float total = 0.f;
  vec o = 0.f;
#pragma unroll 4
  for (int p = 0; p < parts; ++p) {
    const float f = __builtin_amdgcn_exp2f(stats[2 * p] - top);
    total += stats[2 * p + 1] * f;
    o += *reinterpret_cast<const vec*>(sums + (int64_t)p * D) * f;
  }
  const float f = total == 0.f ? 0.f : 1.f / total;
  uint16_t* to = a.out.at(sequence, head) + lane * kPer;
#pragma unroll
  for (int i = 0; i < kPer; ++i) to[i] = __builtin_bit_cast(uint16_t, (__bf16)(o[i] * f));
}

}  // namespace swz
