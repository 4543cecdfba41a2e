// Attention over packed prompts, forward: out = softmax(scale q k^T) v.
//
// One pass over the keys, 64 at a time, with the row's maximum m so far and its sum l of exp(score - m) in 32 bits: where m rises, what has been summed is scaled by
// exp(m before - m).  It rises only by 8 powers of two or more (a smaller one costs no precision, as weights up to 2^8 are as exact as those up to 1), so that the rescaling is rare.
// Scores come as S^T = k q^T: a lane has 32 scores of one query, whose maximum and sum need one exchange between the halves of the wave, and its weights, rounded, are the operand of
// out^T += v^T P^T where they are.  The rounding of weights to bfloat16 (the instruction takes nothing else for bfloat16 values) costs 0.0021 relative error against 0.0016 of
// rounding the result alone; their sum is taken before it.
//
// A wave has 32 rows, a workgroup four waves that share tiles of keys and values in LDS, two of each: the next ones load while these are used.  Two or three workgroups to a compute unit.
// With heads of 128 the bound is power: 1.55 to 1.66 GHz under this kernel, the matrix units busy for 71 % of it and the vector unit for 59 % (the exponentials).  32768 causal tokens,
// 16 heads of 128 sharing 4: 3.72 ms, 1183 TFLOP/s, one call after another (4.0 ms where there are 5 ms between them); 8192, 32 heads sharing 8: 487 us, 1129.  With heads of 64 a product has
// half the work for the same exponentials: 8192, 32 heads of 64 sharing 8: 290 us, 947 TFLOP/s; five pieces of 1 to 2048 queries over 200 to 10000 keys 160 us, 800, the vector unit busy for
// 70 %.  Short prompts are bound by the latency of their loads, one after another: places, then queries and keys, then values.  50 sequences of 1 to 512 tokens, 32 heads of 128 sharing 8: 40 us.
#pragma once

#include "attention_tiles.h"

namespace swz {

constexpr int kPromptKeys = 64;        // keys of a tile
constexpr float kLazyRise = 8.f;       // a maximum that rises by less than 2^8 does not rescale what has been summed

template <int D, int QW, int HW = 1>
struct PromptShape {                   // a workgroup: QW waves of 32 rows each, of HW query heads of a key head
  static constexpr int kRows = 32 * QW / HW;
  static constexpr int kTileBytes = kPromptKeys * 2 * D, kLdsBytes = 4 * kTileBytes;      // two tiles of keys, two of values
};

// o += p x for rows `from` .. `to` (the lane's own) of ROWS of a tile, one at a time; p as the product with the tile's columns takes it.
template <int D, int ROWS>
__device__ __forceinline__ void add_by_row(f32x16 (&o)[D / 32], const u32x4 (&p)[ROWS / 16], const unsigned char* tile, int from, int to, int lane) {
#pragma unroll 1
  for (int row = 0; row < ROWS; ++row) {
    uint32_t l = (uint32_t)lane;
    keep(l);                         // or the loop has registers for its addresses, which are the kernel's
    const int h = (int)l >> 5;
    // row 16 j + 8 a + 4 h + e is number 4 a + e of operand j in lane half h
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < ROWS / 16; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) word = j == row >> 4 && e == 2 * (row >> 3 & 1) + (row >> 1 & 1) ? p[j][e] : word;
    const float mine = (row >> 2 & 1) == h ? __uint_as_float(row & 1 ? word & 0xffff0000u : word << 16) : 0.f;
    const float w = across_halves(mine, [](float x, float y) { return x + y; });
    const bool seen = row >= from && row <= to;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int part = 0; part < 4; ++part) {
        typedef __attribute__((ext_vector_type(4))) uint16_t u16x4;
        const int d = 32 * i + 8 * part + 4 * h;
        const u16x4 x = *reinterpret_cast<const u16x4*>(tile + row * 2 * D + (((d >> 3) ^ tile_key<D>(row)) << 4) + (d & 7) * 2);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][4 * part + e] += seen ? w * __uint_as_float((uint32_t)x[e] << 16) : 0.f;
        __builtin_amdgcn_sched_barrier(0);                  // few registers at a time: this path is rare
      }
  }
}

// 0, or NaN where one of the sums is no finite number.
template <int N>
__device__ __forceinline__ float odd_sums(const f32x16 (&x)[N], float odd = 0.f) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) odd = __builtin_fmaf(x[i][r], 0.f, odd);
  return odd;
}
// Whether x is true in any of the workgroup's WAVES waves.  Takes the start of LDS, which no wave reads any more.
template <int WAVES>
__device__ __forceinline__ bool any_wave(bool x, unsigned char* smem, int wave, int lane) {
  publish();
  uint32_t* flags = reinterpret_cast<uint32_t*>(smem);
  if (lane == 0) flags[wave] = x;
  publish();
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) any |= flags[i];
  publish();
  return __builtin_amdgcn_readfirstlane((int)any) != 0;
}

template <int D, int QW, int HW, bool CAUSAL>
__global__ void __launch_bounds__(64 * QW, D == 64 ? 3 : 2) attention_kernel(PromptArgs a) {
  using S = PromptShape<D, QW, HW>;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S::kLdsBytes];
  const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;

  const int group = a.q_heads / a.k_heads;
  const PromptPiece piece = prompt_piece((int)blockIdx.x, a.slots * a.splits, a.k_heads, group / HW, a.num_xcd, a.sets);
  if (piece.turn < 0) return;
  const int k_head = piece.k_head, head = k_head * group + piece.member * HW + wave % HW, split = a.splits == 1 ? 0 : piece.turn % a.splits;
  const TurnPlace place = find_turn(a.cu_q, a.total_q, a.cu_k, a.total_k, a.sequences, S::kRows, a.splits == 1 ? piece.turn : piece.turn / a.splits);
  const Span q = place.mine, k = place.other;
  const int first = ((q.length + S::kRows - 1) / S::kRows - 1 - place.tile) * S::kRows;      // a sequence's last rows look at the most keys
  if (place.tile < 0 || first < 0) return;

  const int row0 = first + wave / HW * 32, row = row0 + (lane & 31);
  const int ahead = k.length - q.length;                    // causal: query i looks at keys 0 .. i + ahead
  auto keys_of = [&](int last_row) { return CAUSAL ? clamp_to(last_row + ahead + 1, 0, k.length) : k.length; };
  const int keys = keys_of(min(first + S::kRows, q.length) - 1);              // of any row of the workgroup,
  const int wave_keys = row0 < q.length ? keys_of(min(row0 + 32, q.length) - 1) : 0, all_keys = keys_of(row0);   // any and every row of the wave
  const int last_key = keys_of(row) - 1;
  // with splits, this workgroup's share of the tiles: `per` of them from `before` on
  const int every = (keys + kPromptKeys - 1) / kPromptKeys, per = a.splits == 1 ? every : (every + a.splits - 1) / a.splits, before = split * per;
  auto my_tiles = [&](int n) { return clamp_to(n - before, 0, per); };       // of the first n
  const int tiles = my_tiles(every), wave_tiles = my_tiles((wave_keys + kPromptKeys - 1) / kPromptKeys);
  auto first_key = [&](int t) { return (before + t) * kPromptKeys; };

  const RowLoader<D, kPromptKeys, QW> load_k(a.k.at(k.first, k_head), a.k.token, k.length, wave, lane), load_v(a.v.at(k.first, k_head), a.v.token, k.length, wave, lane);
  auto fetch_k = [&](int t) { load_k(first_key(t), lds + (uint32_t)((t & 1) * S::kTileBytes)); };
  auto fetch_v = [&](int t) { load_v(first_key(t), lds + (uint32_t)((2 + (t & 1)) * S::kTileBytes)); };
  if (tiles > 0) fetch_k(0), fetch_v(0);
  if (tiles > 1) fetch_k(1);

  bf16x8 qf[D / 16];
  load_fragments<D>(qf, a.q.at(q.first + min(row, q.length - 1), head), lane);
  f32x16 o[D / 32], s[2], next[2];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = f32x16{};
  const float c = a.scale * kLog2E;
  float top = -FLT_MAX, sum = 0.f;                          // of scores times c; this lane's half of the sum

  auto score = [&](f32x16 (&x)[2], int t) __attribute__((always_inline)) {
    const uint32_t k_lane = row_address<D>(lds + (uint32_t)((t & 1) * S::kTileBytes), lane);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      x[b] = f32x16{};
#pragma unroll
      for (int i = 0; i < D / 16; ++i) x[b] = mfma32(read_rows<D>(k_lane, b, i), qf[i], x[b]);
    }
  };
  auto mask = [&](f32x16 (&x)[2], int t) __attribute__((always_inline)) {
    if (first_key(t) + kPromptKeys <= all_keys) return;
    const int last = last_key - first_key(t) - 4 * h;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[b][r] = 32 * b + 8 * (r / 4) + r % 4 <= last ? x[b][r] : -INFINITY;
  };
  auto highest = [&](const f32x16 (&x)[2]) __attribute__((always_inline)) {
    float high = x[0][0];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) high = fmaxf(high, x[b][r]);
    return high;
  };
  auto raise = [&](float high) __attribute__((always_inline)) {
    high = across_halves(high, [](float x, float y) { return fmaxf(x, y); }) * c;
    if (!__any(high > top + kLazyRise)) return;
    const float now = fmaxf(top, high), less = __builtin_amdgcn_exp2f(top - now);
    sum *= less;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] *= less;
    top = now;
  };
  // A tile of scores has 32 weights a lane: 16 pairs, each two exponentials, sums and one rounding.
  constexpr int kSteps = D / 16, kParts = D / 32, kScoreSlots = 2 * kSteps, kSlots = kScoreSlots + 4 * kParts;
  uint32_t k_at[kSteps], v_at[kParts][2];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) keep(k_at[i] = row_address<D>(lds, lane) ^ (uint32_t)(i << 5));
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    keep(v_at[i][0] = column_address<D>(lds, lane) ^ (uint32_t)(i << 6));
    keep(v_at[i][1] = (column_address<D>(lds, lane) ^ (uint32_t)(i << 6) ^ 32u) + 16u * D);
  }
  // One tile: kSlots products, first the next tile's scores (MORE: there is one), then the values, weighted.  The vector unit has about as much to do as the
  // matrix unit, so every slot gets its share of it, in a fixed order (the compiler would move all reads ahead of all products): pair n of weights by slot
  // 7 n / 128 of all, which is before the products with its 16 keys, and in the slots of the values the next tile's maximum.
  // PARITY: of the tile's number, -1 where it is not a constant (t says).
  auto tile_pass = [&](f32x16 (&now)[2], f32x16 (&then)[2], int t, auto parity, auto more, auto masked) __attribute__((always_inline)) {
    constexpr bool MORE = decltype(more)::value, MASKED = decltype(masked)::value;
    constexpr int PARITY = decltype(parity)::value, kFirst = MORE ? 0 : kScoreSlots;
    const uint32_t keys_at = (uint32_t)(((PARITY < 0 ? t : PARITY) & 1 ? 0 : 1) * S::kTileBytes), values_at = (uint32_t)((2 + ((PARITY < 0 ? t : PARITY) & 1)) * S::kTileBytes);
    auto read = [&](auto slot) __attribute__((always_inline)) {
      constexpr int i = decltype(slot)::value, v = i - kScoreSlots;
      if constexpr (i < kScoreSlots) return read_rows_at<D>(k_at[i % kSteps], keys_at + (uint32_t)(i / kSteps * 64 * D));
      else return read_columns_at<D>(v_at[v % kParts][0], v_at[v % kParts][1], values_at + (uint32_t)(v / kParts * 32 * D));
    };
    u32x4 p[4];
    constexpr int kAhead = 2, kRing = kAhead + 1;            // reads on their way
    bf16x8 f[kRing];
    for_each_index([&](auto slot) __attribute__((always_inline)) {
      constexpr int i = kFirst + decltype(slot)::value;
      f[i % kRing] = read(std::integral_constant<int, i>{});
    }, std::make_integer_sequence<int, kAhead>{});
    if constexpr (MORE) then[0] = then[1] = f32x16{};
    float sums[2] = {sum, 0.f}, high[2] = {-INFINITY, -INFINITY};
    now[0][0] = __builtin_fmaf(now[0][0], c, -top);
    now[0][1] = __builtin_fmaf(now[0][1], c, -top);
    __builtin_amdgcn_sched_barrier(0);
    for_each_index([&](auto slot) __attribute__((always_inline)) {
      constexpr int i = kFirst + decltype(slot)::value, v = i - kScoreSlots;
      if constexpr (i + kAhead < kSlots) f[(i + kAhead) % kRing] = read(std::integral_constant<int, i + kAhead>{});
      if constexpr (i < kScoreSlots) then[i / kSteps] = mfma32(f[i % kRing], qf[i % kSteps], then[i / kSteps]);
      if constexpr (MORE && i >= kScoreSlots) o[v % kParts] = mfma32(f[i % kRing], __builtin_bit_cast(bf16x8, p[v / kParts]), o[v % kParts]);
      constexpr auto kPairs = [](int before) constexpr {                // pairs taken before a slot
        if (MORE) return before >= kSlots ? 16 : before <= 0 ? 0 : (before * 128 + 7 * kSlots - 1) / (7 * kSlots) < 16 ? (before * 128 + 7 * kSlots - 1) / (7 * kSlots) : 16;
        const int w = before - kScoreSlots;
        return w <= 0 ? 0 : w < kParts ? 8 : w < 2 * kParts ? 12 : 16;
      };
#pragma unroll
      for (int n = kPairs(i); n < kPairs(i + 1); ++n) {
        const int b = n / 8, r = n % 8 * 2, m = n + 1;
        if (m < 16) {
          now[m / 8][m % 8 * 2] = __builtin_fmaf(now[m / 8][m % 8 * 2], c, -top);
          now[m / 8][m % 8 * 2 + 1] = __builtin_fmaf(now[m / 8][m % 8 * 2 + 1], c, -top);
        }
        const float w0 = __builtin_amdgcn_exp2f(now[b][r]), w1 = __builtin_amdgcn_exp2f(now[b][r + 1]);
        sums[0] += w0;
        sums[1] += w1;
        p[n / 4][n % 4] = pack_bf16(w0, w1);
      }
      if constexpr (!MORE) o[v % kParts] = mfma32(f[i % kRing], __builtin_bit_cast(bf16x8, p[v / kParts]), o[v % kParts]);
      if constexpr (MASKED && i == kScoreSlots - 1) mask(then, t + 1);
      if constexpr (MORE && i >= kScoreSlots) {
#pragma unroll
        for (int e = v * 32 / (4 * kParts); e < (v + 1) * 32 / (4 * kParts); e += 2)
          high[e / 2 % 2] = __builtin_elementwise_maximum(high[e / 2 % 2], __builtin_elementwise_maximum(then[e / 16][e % 16], then[e / 16][e % 16 + 1]));
      }
      __builtin_amdgcn_sched_barrier(0);
    }, std::make_integer_sequence<int, kSlots - kFirst>{});
    sum = sums[0] + sums[1];
    return fmaxf(high[0], high[1]);
  };
  constexpr std::integral_constant<int, 0> kEven{};
  constexpr std::integral_constant<int, 1> kOdd{};
  constexpr std::integral_constant<int, -1> kEither{};

  // The scores of the first tile; then, tile by tile, this one's weights and values beside the scores of the next.  Two sets of scores take turns.
  auto turn = [&](int t) __attribute__((always_inline)) {
    publish();
    if (t + 2 < tiles) fetch_k(t + 2);
    if (t + 1 < tiles) fetch_v(t + 1);
  };
  publish();
  if (wave_tiles > 0) {
    score(s, 0);
    mask(s, 0);
    raise(highest(s));
  }
  const int whole = min(my_tiles(all_keys / kPromptKeys), wave_tiles);          // tiles without a mask
  int t = 0;
  for (; t + 2 < whole; t += 2) {
    turn(t);
    raise(tile_pass(s, next, t, kEven, std::true_type{}, std::false_type{}));
    turn(t + 1);
    raise(tile_pass(next, s, t + 1, kOdd, std::true_type{}, std::false_type{}));
  }
  for (; t + 1 < wave_tiles; ++t) {
    turn(t);
    raise(tile_pass(s, next, t, kEither, std::true_type{}, std::true_type{}));
    s[0] = next[0];
    s[1] = next[1];
  }
  if (t < wave_tiles) {
    turn(t);
    tile_pass(s, next, t, kEither, std::false_type{}, std::false_type{});
    ++t;
  }
  for (; t < tiles; ++t) turn(t);

  // A weight of 0 times an infinity or NaN is NaN: where a value that only some rows of a tile look at is no finite number, the products carry it into the others.
  // The result shows it, and the tiles are then taken a second time, the masked ones key by key.
  if constexpr (CAUSAL) {
    const bool mine = __any(odd_sums(o) != 0.f);            // (the other waves keep what they have)
    if (__builtin_expect(any_wave<QW>(mine, smem, wave, lane), 0)) {
      if (tiles > 0) fetch_k(0), fetch_v(0);
      if (mine) {
        top = -FLT_MAX;
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < kParts; ++i) o[i] = f32x16{};
      }
      for (t = 0; t < tiles; ++t) {
        publish();
        if (t + 1 < tiles) fetch_k(t + 1), fetch_v(t + 1);
        if (!mine || t >= wave_tiles) continue;
        score(s, t);
        mask(s, t);
        raise(highest(s));
        u32x4 p[4];
#pragma unroll
        for (int n = 0; n < 16; ++n) {
          const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n / 8][n % 8 * 2], c, -top)), w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n / 8][n % 8 * 2 + 1], c, -top));
          sum += w0 + w1;
          p[n / 4][n % 4] = pack_bf16(w0, w1);
        }
        if (t >= whole) {
          add_by_row<D, kPromptKeys>(o, p, smem + (2 + (t & 1)) * S::kTileBytes, 0, last_key - first_key(t), lane);
        } else {
          const uint32_t v_lane = column_address<D>(lds + (uint32_t)((2 + (t & 1)) * S::kTileBytes), lane);
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < kParts; ++i) o[i] = mfma32(read_columns<D>(v_lane, j, i), __builtin_bit_cast(bf16x8, p[j]), o[i]);
        }
      }
    }
  }

  sum = across_halves(sum, [](float x, float y) { return x + y; });
  const bool real = row < q.length;
  if (a.splits > 1) {
    if (!real) return;
    const int64_t at = ((int64_t)split * a.total_q + q.first + row) * a.q_heads + head;
    if (h == 0) *reinterpret_cast<float2*>(a.part_stats + 2 * at) = float2{top, sum};
    if (tiles == 0) return;
#pragma unroll
    for (int i = 0; i < kParts; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += 4) *reinterpret_cast<f32x4*>(a.part_sums + at * D + 32 * i + 2 * r + 4 * h) = f32x4{o[i][r], o[i][r + 1], o[i][r + 2], o[i][r + 3]};
    return;
  }
  store_columns<D>(o, sum == 0.f ? 0.f : 1.f / sum, a.out.at(q.first + min(row, q.length - 1), head), real, lane);
  if (real && h == 0) a.lse[(int64_t)head * a.total_q + q.first + row] = sum == 0.f ? -INFINITY : __builtin_fmaf(top, kLn2, __logf(sum));
}

// What the splits of a row (at most 64) have, joined: a wave for each row of a head, D / 64 dimensions a lane.
constexpr int kJoinRows = 4;
template <int D>
__global__ void __launch_bounds__(64 * kJoinRows) attention_join_kernel(PromptArgs a) {
  constexpr int kPer = D / 64;
  typedef __attribute__((ext_vector_type(kPer))) float vec;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const PromptPiece piece = prompt_piece((int)blockIdx.x, a.slots, a.q_heads, 1, a.num_xcd, a.sets);
  if (piece.turn < 0) return;
  const int head = piece.k_head;
  const TurnPlace place = find_turn(a.cu_q, a.total_q, a.cu_k, a.total_k, a.sequences, kJoinRows, piece.turn);
  const int row = place.tile * kJoinRows + wave;
  if (place.tile < 0 || row >= place.mine.length) return;
  const int64_t token = place.mine.first + row, step = (int64_t)a.total_q * a.q_heads, at = token * a.q_heads + head;
  float my_top = -FLT_MAX, my_sum = 0.f;                    // of split `lane`
  if (lane < a.splits) {
    const float2 x = *reinterpret_cast<const float2*>(a.part_stats + 2 * (at + lane * step));
    my_top = x.x;
    my_sum = x.y;
  }
  const float top = over_wave(my_top, [](float x, float y) { return fmaxf(x, y); });
  // a split without keys has a sum of 0 and has written nothing else
  const float weight = __builtin_amdgcn_exp2f(my_top - top), sum = over_wave(my_sum * weight, [](float x, float y) { return x + y; });
  vec o = 0.f;
  for (int s = 0; s < a.splits; ++s) {
    const float w = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(weight), s));
    if (__uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(my_sum), s)) != 0.f)
      o += *reinterpret_cast<const vec*>(a.part_sums + (at + s * step) * D + lane * kPer) * w;
  }
  const float f = sum == 0.f ? 0.f : 1.f / sum;
  uint16_t* to = a.out.at(token, head) + lane * kPer;
#pragma unroll
  for (int i = 0; i < kPer; ++i) to[i] = __builtin_bit_cast(uint16_t, (__bf16)(o[i] * f));
  if (lane == 0) a.lse[(int64_t)head * a.total_q + token] = sum == 0.f ? -INFINITY : __builtin_fmaf(top, kLn2, __logf(sum));
}

}  // namespace swz
