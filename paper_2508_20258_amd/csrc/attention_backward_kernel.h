// Attention over packed prompts, backward.
//
// With P = exp(scale q k^T - lse), dP = dout v^T and delta = sum over the dimensions of dout * out: dS = P (dP - delta), dq = scale dS k, dk = scale dS^T q, dv = P^T dout.
// Two kernels, one for dq with a row's keys in turn, one for dk and dv with a key's queries in turn: scores and dP are worked out in both (9 products with the forward pass, where 7
// would do), so that every sum has one owner and an order of its own, without atomics and without the scores in memory.
// P and dS are rounded to bfloat16 for the products that sum over them, as the instruction takes nothing else: dq and dk have 0.0025 relative error, where rounding the result
// alone has 0.0017; a second product with what the rounding leaves over would take a quarter more time.  delta comes from the rounded out: 0.0001 of that, 0.0002 with a few keys.
// With heads of 128 bound by power (1.57 and 1.67 GHz).  8227 tokens in six sequences, 32 heads of 128 sharing 8, causal: dq 275 us, 1090 TFLOP/s, dk and dv 431 us, 930; matrix units busy
// for 64 and 54 % of it, LDS for 32 and 41 %.  4 x 2048 tokens, 16 heads of 64: 70 and 85 us; matrix units 47 and 45 %, LDS 24 and 47 %, vector unit 60 and 50 %: none of them alone.
#pragma once

#include "attention_kernel.h"

namespace swz {

struct PromptBackArgs {
  PromptArgs f;                    // slots: of this launch
  Heads dout, dq, dk, dv;
  float *log_sums, *deltas;        // q_heads x total_q each: -lse / scale, and -(sum over the dimensions of dout * out)
};

// dq, and delta for the other kernel.  As the forward kernel, with a third product, dq^T += k^T dS^T, and without its maximum: lse is known.
template <int D, int NW, int HW, bool CAUSAL>
__global__ void __launch_bounds__(NW * 64, D == 64 ? 3 : 2) attention_dq_kernel(PromptBackArgs args) {
  const PromptArgs& a = args.f;
  using S = PromptShape<D, NW, HW>;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S::kLdsBytes];
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;

  const int group = a.q_heads / a.k_heads;
  const PromptPiece piece = prompt_piece((int)blockIdx.x, a.slots, a.k_heads, group / HW, a.num_xcd, a.sets);
  if (piece.turn < 0) return;
  const int k_head = piece.k_head, head = k_head * group + piece.member * HW + wave % HW;
  const TurnPlace place = find_turn(a.cu_q, a.total_q, a.cu_k, a.total_k, a.sequences, S::kRows, piece.turn);
  const Span q = place.mine, k = place.other;
  const int first = ((q.length + S::kRows - 1) / S::kRows - 1 - place.tile) * S::kRows;
  if (place.tile < 0 || first < 0) return;

  const int row0 = first + wave / HW * 32, row = row0 + (lane & 31);
  const bool real = row < q.length;
  const int ahead = k.length - q.length;
  auto keys_of = [&](int last_row) { return CAUSAL ? clamp_to(last_row + ahead + 1, 0, k.length) : k.length; };
  const int keys = keys_of(min(first + S::kRows, q.length) - 1);
  const int wave_keys = row0 < q.length ? keys_of(min(row0 + 32, q.length) - 1) : 0, all_keys = keys_of(row0);
  const int last_key = keys_of(row) - 1;
  const int tiles = (keys + kPromptKeys - 1) / kPromptKeys;

  const RowLoader<D, kPromptKeys, NW> load_k(a.k.at(k.first, k_head), a.k.token, k.length, wave, lane), load_v(a.v.at(k.first, k_head), a.v.token, k.length, wave, lane);
  auto fetch = [&](int t) {
    const uint32_t at = lds + (uint32_t)((t & 1) * S::kTileBytes);
    load_k(t * kPromptKeys, at);
    load_v(t * kPromptKeys, at + 2 * S::kTileBytes);
  };
  if (tiles > 0) fetch(0);

  const int64_t token = q.first + min(row, q.length - 1);
  bf16x8 qf[D / 16], gf[D / 16];
  load_fragments<D>(gf, args.dout.at(token, head), lane);
  load_fragments<D>(qf, a.out.at(token, head), lane);
  float delta = 0.f;
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) delta = __builtin_fmaf((float)gf[i][e], (float)qf[i][e], delta);
  delta = across_halves(delta, [](float x, float y) { return x + y; });
  const int64_t stat = (int64_t)head * a.total_q + token;
  float lse = a.lse[stat] * kLog2E;
  if (real && h == 0) {
    args.log_sums[stat] = lse == -INFINITY ? -INFINITY : -lse / (a.scale * kLog2E);
    args.deltas[stat] = -delta;
  }
  lse = lse == -INFINITY ? 0.f : lse;                       // a row that looks at nothing: its scores are -inf, and so its weights 0
  load_fragments<D>(qf, a.q.at(token, head), lane);
  f32x16 acc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) acc[i] = f32x16{};
  const float c = a.scale * kLog2E;

  auto mask = [&](f32x16& s, int first_key) __attribute__((always_inline)) {
    const int last = last_key - first_key - 4 * h;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 8 * (r / 4) + r % 4 <= last ? s[r] : -INFINITY;
  };
  constexpr int kSteps = D / 16, kParts = D / 32, kSlots = 4 * kSteps + 4 * kParts;
  uint32_t k_at[kSteps], t_at[kParts][2];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) keep(k_at[i] = row_address<D>(lds, lane) ^ (uint32_t)(i << 5));
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    keep(t_at[i][0] = column_address<D>(lds, lane) ^ (uint32_t)(i << 6));
    keep(t_at[i][1] = (column_address<D>(lds, lane) ^ (uint32_t)(i << 6) ^ 32u) + 16u * D);
  }
  // One tile in slots of one product each, with their share of the vector unit's work, blocks 0 and 1 of 32 keys: S0; dP0 and the weights of 0; S1 and the
  // gradients of the scores of 0; dP1 and the weights of 1; dq from 0 and the gradients of 1; dq from 1.
  auto tile_pass = [&](int t, auto parity, auto with_mask) __attribute__((always_inline)) {
    constexpr uint32_t kAt = (uint32_t)(decltype(parity)::value * S::kTileBytes);
    auto read = [&](auto slot) __attribute__((always_inline)) {
      constexpr int i = decltype(slot)::value, j = i - 4 * kSteps;
      if constexpr (j < 0) return read_rows_at<D>(k_at[i % kSteps], kAt + (uint32_t)((i / kSteps % 2 ? 2 * S::kTileBytes : 0) + i / (2 * kSteps) * 64 * D));
      else return read_columns_at<D>(t_at[j % kParts][0], t_at[j % kParts][1], kAt + (uint32_t)(j / kParts * 32 * D));
    };
    constexpr int kAhead = 2, kRing = kAhead + 1;
    bf16x8 f[kRing];
    for_each_index([&](auto slot) __attribute__((always_inline)) { f[decltype(slot)::value] = read(slot); }, std::make_integer_sequence<int, kAhead>{});
    f32x16 s[2], dp[2];
    u32x4 ds[4];
    __builtin_amdgcn_sched_barrier(0);
    for_each_index([&](auto slot) __attribute__((always_inline)) {
      constexpr int i = decltype(slot)::value, j = i - 4 * kSteps, b = i / (2 * kSteps);
      if constexpr (i + kAhead < kSlots) f[(i + kAhead) % kRing] = read(std::integral_constant<int, i + kAhead>{});
      if constexpr (j < 0 && i / kSteps % 2 == 0) s[b] = mfma32(f[i % kRing], qf[i % kSteps], i % kSteps ? s[b] : f32x16{});
      if constexpr (j < 0 && i / kSteps % 2 == 1) dp[b] = mfma32(f[i % kRing], gf[i % kSteps], i % kSteps ? dp[b] : f32x16{});
      if constexpr (j >= 0) acc[j % kParts] = mfma32(f[i % kRing], __builtin_bit_cast(bf16x8, ds[j / kParts]), acc[j % kParts]);
      if constexpr (decltype(with_mask)::value && j < 0 && i % (2 * kSteps) == kSteps - 1) mask(s[b], t * kPromptKeys + 32 * b);
      // pairs taken before a slot: weights of block 0 from slot kSteps on, ..
      constexpr auto pairs = [](int n, int slots) constexpr { return n <= 0 ? 0 : n >= slots ? 8 : (n * 8 + slots - 1) / slots; };
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int n = pairs(i - (1 + 2 * w) * kSteps, kSteps); n < pairs(i + 1 - (1 + 2 * w) * kSteps, kSteps); ++n)
#pragma unroll
          for (int e = 2 * n; e < 2 * n + 2; ++e) s[w][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[w][e], c, -lse));
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int n = pairs(i - (2 + 2 * w) * kSteps, w ? 2 * kParts : kSteps); n < pairs(i + 1 - (2 + 2 * w) * kSteps, w ? 2 * kParts : kSteps); ++n)
          ds[2 * w + n / 4][n % 4] = pack_bf16(s[w][2 * n] * (dp[w][2 * n] - delta), s[w][2 * n + 1] * (dp[w][2 * n + 1] - delta));
      __builtin_amdgcn_sched_barrier(0);
    }, std::make_integer_sequence<int, kSlots>{});
  };
  constexpr std::integral_constant<int, 0> kEven{};
  constexpr std::integral_constant<int, 1> kOdd{};
  auto turn = [&](int t) __attribute__((always_inline)) {
    publish();
    if (t + 1 < tiles) fetch(t + 1);
  };
  const int wave_tiles = (wave_keys + kPromptKeys - 1) / kPromptKeys, whole = min(all_keys / kPromptKeys, wave_tiles);       // tiles that this wave has, and without a mask
  int t = 0;
  for (; t + 1 < whole; t += 2) {
    turn(t);
    tile_pass(t, kEven, std::false_type{});
    turn(t + 1);
    tile_pass(t + 1, kOdd, std::false_type{});
  }
  for (; t < tiles; ++t) {
    turn(t);
    if (t >= wave_tiles) continue;
    if (t & 1) tile_pass(t, kOdd, std::true_type{});
    else tile_pass(t, kEven, std::true_type{});
  }
  if constexpr (CAUSAL) {            // a key that is no finite number and only some rows of a tile look at: as in the forward kernel
    const bool mine = __any(odd_sums(acc) != 0.f);
    if (__builtin_expect(any_wave<NW>(mine, smem, wave, lane), 0)) {
      if (tiles > 0) fetch(0);
      if (mine) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) acc[i] = f32x16{};
      }
      for (t = 0; t < tiles; ++t) {
        turn(t);
        if (!mine || t >= wave_tiles) continue;
        const uint32_t at = lds + (uint32_t)((t & 1) * S::kTileBytes);
        uint32_t l = (uint32_t)lane;
        keep(l);                     // or these addresses have registers all along
        const uint32_t k_lane = row_address<D>(at, (int)l), t_lane = column_address<D>(at, (int)l);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          f32x16 s = f32x16{}, dp = f32x16{};
#pragma unroll
          for (int i = 0; i < kSteps; ++i) {
            s = mfma32(read_rows<D>(k_lane, b, i), qf[i], s);
            dp = mfma32(read_rows<D>(k_lane + 2 * S::kTileBytes, b, i), gf[i], dp);
            __builtin_amdgcn_sched_barrier(0);              // one read at a time: few registers
          }
          mask(s, t * kPromptKeys + 32 * b);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -lse)) * (dp[r] - delta);
          const u32x4 ds[2] = {as_words(s, 0), as_words(s, 1)};
          if (t >= whole) {
            add_by_row<D, 32>(acc, ds, smem + (t & 1) * S::kTileBytes + b * 64 * D, 0, last_key - t * kPromptKeys - 32 * b, lane);
            continue;
          }
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < kParts; ++i) {
              acc[i] = mfma32(read_columns<D>(t_lane, 2 * b + j, i), __builtin_bit_cast(bf16x8, ds[j]), acc[i]);
              __builtin_amdgcn_sched_barrier(0);
            }
        }
      }
    }
  }
  store_columns<D>(acc, a.scale, args.dq.at(token, head), real, lane);
}

// dk and dv of 32 KW keys of a key head, summed over the queries of all its query heads.  A wave has 32 keys, as columns: with them as B, S = q k^T and dP = dout v^T have
// queries as rows, so that P and dS are B of dv^T += dout^T P and dk^T += q^T dS.  QP groups of KW waves take tiles of 32 queries in turn and add up what they have
// at the end: more waves for a key tile than one group of them would give, so that a tile that many queries look at is done sooner, and no atomics.
// The products start from the rows' -lse / scale and -delta, so that P = exp2(c S) and dS = P dP as they come.
constexpr int kBackRows = 32;      // queries of a tile
__device__ const float kMinusInfinity = -INFINITY;

template <int D, int KW, int QP>
struct BackShape {
  static constexpr int kKeys = 32 * KW, kThreads = 64 * KW * QP;
  static constexpr int kTileBytes = kBackRows * 2 * D;       // of q, or of dout
  static constexpr int kGroupBytes = 4 * kTileBytes;         // q and dout of one tile, then of the next
  static constexpr int kKeyBytes = kKeys * 2 * D, kKeysAt = QP * kGroupBytes, kStatsAt = kKeysAt + 2 * kKeyBytes;      // keys, values, statistics
  static constexpr int kLdsBytes = kStatsAt + QP * 2 * 2 * kBackRows * 4;
  static constexpr int kAccBytes = (D / 32) * 4096;     // of a wave: dk or dv
  static_assert(kLdsBytes <= 160 * 1024 && QP / 2 * KW * kAccBytes <= kLdsBytes, "LDS");
};

template <int D, int KW, int QP, bool CAUSAL>
__global__ void __launch_bounds__(64 * KW * QP, D == 64 ? 3 : 2) attention_dkv_kernel(PromptBackArgs args) {
  const PromptArgs& a = args.f;
  using S = BackShape<D, KW, QP>;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S::kLdsBytes];
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const int lane = threadIdx.x & 63, h = lane >> 5, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wave = w % KW, part = w / KW;

  const int group = a.q_heads / a.k_heads;
  const PromptPiece piece = prompt_piece((int)blockIdx.x, a.slots * a.splits, a.k_heads, 1, a.num_xcd, a.sets);
  if (piece.turn < 0) return;
  const int k_head = piece.k_head, split = a.splits == 1 ? 0 : piece.turn % a.splits;
  const TurnPlace place = find_turn(a.cu_k, a.total_k, a.cu_q, a.total_q, a.sequences, S::kKeys, a.splits == 1 ? piece.turn : piece.turn / a.splits);
  const Span q = place.other, k = place.mine;
  const int first = place.tile * S::kKeys;
  if (place.tile < 0 || first >= k.length) return;

  const int key0 = first + wave * 32, key = key0 + (lane & 31);
  const int ahead = k.length - q.length;
  const int from = CAUSAL ? clamp_to(first - ahead, 0, q.length) / kBackRows : 0;      // the first tile of queries that looks at a key of the workgroup
  const int tiles = (q.length + kBackRows - 1) / kBackRows - from, steps = tiles > 0 ? tiles * group : 0;
  const int stride = QP * a.splits, rounds = max(0, (steps - QP * split + stride - 1) / stride);        // of this split's groups

  const RowLoader<D, S::kKeys, KW * QP> load_k(a.k.at(k.first, k_head), a.k.token, k.length, w, lane), load_v(a.v.at(k.first, k_head), a.v.token, k.length, w, lane);
  if (rounds > 0) load_k(first, lds + S::kKeysAt), load_v(first, lds + S::kKeysAt + S::kKeyBytes);

  // this group's steps: query head k_head * group + member, tile `tile` of it, `stride` further each round
  RowLoader<D, kBackRows, KW> load_q(a.q.data, a.q.token, q.length, wave, lane), load_g(args.dout.data, args.dout.token, q.length, wave, lane);
  const uint32_t tile_lds = lds + (uint32_t)(part * S::kGroupBytes), stats_lds = lds + (uint32_t)(S::kStatsAt + part * 4 * kBackRows * 4);
  int member, tile;
  auto begin = [&]() {
    member = tiles > 0 ? (QP * split + part) / tiles : 0;
    tile = QP * split + part - member * tiles;
  };
  begin();
  auto advance = [&]() {
    tile += stride;
    while (tile >= tiles) tile -= tiles, ++member;
  };
  auto fetch = [&](int round) __attribute__((always_inline)) {         // of (member, tile), the round's
    if (member >= group) return;
    const int head = k_head * group + member, r0 = (from + tile) * kBackRows;
    const uint32_t at = tile_lds + (uint32_t)((round & 1) * 2 * S::kTileBytes);
    load_q.head = a.q.at(q.first, head);
    load_g.head = args.dout.at(q.first, head);
    load_q(r0, at);
    load_g(r0, at + S::kTileBytes);
    if (wave == 0) {
      const int r = r0 + (lane & 31);
      const float* stat = (lane < 32 ? args.log_sums : args.deltas) + (int64_t)head * a.total_q + q.first + r;
      load_word_to_lds(r < q.length ? stat : lane < 32 ? &kMinusInfinity : reinterpret_cast<const float*>(&kZeroChunk), stats_lds + (uint32_t)((round & 1) * 2 * kBackRows * 4));
    }
  };
  if (rounds > 0) fetch(0);

  constexpr int kSteps = D / 16, kParts = D / 32;
  f32x16 dk[kParts], dv[kParts];
#pragma unroll
  for (int i = 0; i < kParts; ++i) dk[i] = dv[i] = f32x16{};
  const float c = a.scale * kLog2E;
  uint32_t q_at = row_address<D>(tile_lds, lane), g_at = q_at + S::kTileBytes, column_at[kParts][2];
  keep(g_at);                        // or the compiler shares their steps' addresses, and has no registers for them
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    keep(column_at[i][0] = column_address<D>(tile_lds, lane) ^ (uint32_t)(i << 6));
    keep(column_at[i][1] = (column_address<D>(tile_lds, lane) ^ (uint32_t)(i << 6) ^ 32u) + 16u * D);
  }
  const uint32_t key_at = row_address<D>(lds + (uint32_t)(S::kKeysAt + wave * 64 * D), lane);
  uint32_t value_at = key_at + S::kKeyBytes;
  keep(value_at);
  typedef __attribute__((address_space(3))) const f32x4* stat_ptr;
  uint32_t stat_at = stats_lds + (uint32_t)(16 * h);

  auto start = [&](f32x16& x, uint32_t at) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 y = *(stat_ptr)(uintptr_t)(at + (uint32_t)(32 * i));
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * i + e] = y[e];
    }
  };
  constexpr bool kHold = D == 128;   // the wave's keys stay in registers (1% less time than reading them from LDS for every tile); with heads of 64 that would cost a wave of three
  bf16x8 held[kHold ? kSteps : 1];
  if constexpr (kHold) {
    publish();
    for_each_index([&](auto i) __attribute__((always_inline)) { held[decltype(i)::value] = read_rows<D>(key_at, 0, decltype(i)::value); }, std::make_integer_sequence<int, kSteps>{});
  }
  auto looks = [&](int r0) { return member < group && !(CAUSAL && r0 + kBackRows - 1 + ahead < key0); };      // some of these rows do, at a key of this wave
  auto masked = [&](int r0) { return (CAUSAL && r0 + ahead < key0 + 31) || key0 + 32 > k.length; };
  auto first_row = [&](int r0) { return key < k.length ? (CAUSAL ? key - ahead - r0 : 0) : kBackRows; };     // of those that look at the lane's key
  auto mask = [&](f32x16& s, int r0) __attribute__((always_inline)) {
    const int from_row = first_row(r0) - 4 * h;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 8 * (r / 4) + r % 4 >= from_row ? s[r] : -INFINITY;
  };
  for (int round = 0; round < rounds; ++round) {
    publish();
    const int r0 = (from + tile) * kBackRows;
    const bool mine = looks(r0);
    advance();
    if (round + 1 < rounds) fetch(round + 1);
    if (mine) {
      f32x16 s, dp;
      start(s, stat_at);
      // Slots of one product each: S, dP, dv, dk.
      constexpr int kAhead = 2, kRing = kAhead + 1;
      bf16x8 f[kRing], kf[kRing];
      auto read_a = [&](auto slot) __attribute__((always_inline)) {
        constexpr int i = decltype(slot)::value, j = i - 2 * kSteps;
        if constexpr (i < 2 * kSteps) return read_rows<D>(i < kSteps ? q_at : g_at, 0, i % kSteps);
        else return read_columns_at<D>(column_at[j % kParts][0], column_at[j % kParts][1], (uint32_t)((j < 2 * kParts ? S::kTileBytes : 0) + j / kParts % 2 * 32 * D));
      };
      auto read_k = [&](auto slot) __attribute__((always_inline)) {
        constexpr int i = decltype(slot)::value;
        if constexpr (!kHold || i >= kSteps) kf[i % kRing] = read_rows<D>(i < kSteps ? key_at : value_at, 0, i % kSteps);
      };
      constexpr int kSlots = 2 * kSteps + 4 * kParts, kPairs = 8;       // pairs of weights
      for_each_index([&](auto slot) __attribute__((always_inline)) {
        f[decltype(slot)::value] = read_a(slot);
        read_k(slot);
      }, std::make_integer_sequence<int, kAhead>{});
      __builtin_amdgcn_sched_barrier(0);
      for_each_index([&](auto slot) __attribute__((always_inline)) {
        constexpr int i = decltype(slot)::value;
        f[(i + kAhead) % kRing] = read_a(std::integral_constant<int, i + kAhead>{});
        read_k(std::integral_constant<int, i + kAhead>{});
        s = mfma32(f[i % kRing], kHold ? held[kHold ? i : 0] : kf[i % kRing], s);
        if constexpr (i == kSteps - 2) start(dp, stat_at + kBackRows * 4);
        __builtin_amdgcn_sched_barrier(0);
      }, std::make_integer_sequence<int, kSteps>{});
      if (masked(r0)) mask(s, r0);
      u32x4 p[2], ds[2];
      for_each_index([&](auto slot) __attribute__((always_inline)) {
        constexpr int u = decltype(slot)::value, i = kSteps + u, j = i - 2 * kSteps;
        if constexpr (i + kAhead < kSlots) f[(i + kAhead) % kRing] = read_a(std::integral_constant<int, i + kAhead>{});
        if constexpr (i + kAhead < 2 * kSteps) read_k(std::integral_constant<int, i + kAhead>{});
        if constexpr (i < 2 * kSteps) dp = mfma32(f[i % kRing], kf[i % kRing], dp);
        else if constexpr (j < 2 * kParts) dv[j % kParts] = mfma32(f[i % kRing], __builtin_bit_cast(bf16x8, p[j / kParts]), dv[j % kParts]);
        else dk[j % kParts] = mfma32(f[i % kRing], __builtin_bit_cast(bf16x8, ds[j / kParts - 2]), dk[j % kParts]);
        // weights while dP and the first half of dv are multiplied (half of them before any of dv, all before its second half), then the gradients of
        // the scores, half of them before any of dk
        constexpr int kW = kSteps + kParts, kD = 3 * kParts;
        constexpr auto weights_before = [](int n) constexpr { return n >= kW ? kPairs : n <= 0 ? 0 : (n * kPairs + kW - 1) / kW; };
        constexpr auto slopes_before = [](int n) constexpr { return n >= kD ? kPairs : n <= 0 ? 0 : (n * kPairs + kD - 1) / kD; };
#pragma unroll
        for (int n = weights_before(u); n < weights_before(u + 1); ++n) {
          const int e = 2 * n;
          s[e] = __builtin_amdgcn_exp2f(s[e] * c);
          s[e + 1] = __builtin_amdgcn_exp2f(s[e + 1] * c);
          p[e / 8][e % 8 / 2] = pack_bf16(s[e], s[e + 1]);
        }
#pragma unroll
        for (int n = slopes_before(j); n < slopes_before(j + 1); ++n) {
          const int e = 2 * n;
          ds[e / 8][e % 8 / 2] = pack_bf16(s[e] * dp[e], s[e + 1] * dp[e + 1]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }, std::make_integer_sequence<int, kSlots - kSteps>{});
    }
    // to the other tile
    q_at ^= 2 * S::kTileBytes;
    g_at ^= 2 * S::kTileBytes;
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      column_at[i][0] ^= 2 * S::kTileBytes;
      column_at[i][1] ^= 2 * S::kTileBytes;
    }
    stat_at ^= 2 * kBackRows * 4;
  }

  if constexpr (CAUSAL) {            // queries and gradients that are no finite numbers and look at some keys of a tile only: as in the forward kernel
    const bool odd = __any(odd_sums(dv, odd_sums(dk)) != 0.f);
    if (__builtin_expect(any_wave<KW * QP>(odd, smem, w, lane), 0)) {
      begin();
      if (rounds > 0) fetch(0);
      if (odd) {
#pragma unroll
        for (int i = 0; i < kParts; ++i) dk[i] = dv[i] = f32x16{};
      }
      for (int round = 0; round < rounds; ++round) {
        publish();
        const int r0 = (from + tile) * kBackRows;
        const bool mine = odd && looks(r0);
        advance();
        if (round + 1 < rounds) fetch(round + 1);
        if (!mine) continue;
        const int tiles_at = part * S::kGroupBytes + (round & 1) * 2 * S::kTileBytes;
        uint32_t l = (uint32_t)lane;
        keep(l);                     // or these addresses have registers all along
        const uint32_t q_lane = row_address<D>(lds + (uint32_t)tiles_at, (int)l), q_column = column_address<D>(lds + (uint32_t)tiles_at, (int)l);
        stat_at = stats_lds + (uint32_t)(16 * h + (round & 1) * 2 * kBackRows * 4);
        f32x16 s, dp;
        start(s, stat_at);
        start(dp, stat_at + kBackRows * 4);
        // (one read at a time: few registers)
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          s = mfma32(read_rows<D>(q_lane, 0, i), read_rows<D>(key_at, 0, i), s);
          __builtin_amdgcn_sched_barrier(0);
          dp = mfma32(read_rows<D>(q_lane + S::kTileBytes, 0, i), read_rows<D>(value_at, 0, i), dp);
          __builtin_amdgcn_sched_barrier(0);
        }
        mask(s, r0);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(s[r] * c);
        const u32x4 weights[2] = {as_words(s, 0), as_words(s, 1)};
        s *= dp;
        const u32x4 ds[2] = {as_words(s, 0), as_words(s, 1)};
        auto add = [&](f32x16 (&sum)[kParts], const u32x4 (&words)[2], int at) __attribute__((always_inline)) {
          if (masked(r0)) {
            add_by_row<D, kBackRows>(sum, words, smem + tiles_at + at, first_row(r0), kBackRows, lane);
            return;
          }
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < kParts; ++i) {
              sum[i] = mfma32(read_columns<D>(q_column + (uint32_t)at, j, i), __builtin_bit_cast(bf16x8, words[j]), sum[i]);
              __builtin_amdgcn_sched_barrier(0);
            }
        };
        add(dv, weights, S::kTileBytes);
        add(dk, ds, 0);
      }
    }
  }

  // the groups in halves, first dk, then dv: the upper one's sums go to the lower one
  auto join = [&](f32x16 (&x)[kParts]) __attribute__((always_inline)) {
#pragma unroll
    for (int half = QP / 2; half > 0; half /= 2) {
      publish();
      f32x4* held = reinterpret_cast<f32x4*>(smem) + lane;
      auto at = [&](int p, int i, int r) { return (((p * KW + wave) * kParts + i) * 4 + r) * 64; };
      if (part >= half && part < 2 * half) {
#pragma unroll
        for (int i = 0; i < kParts; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) held[at(part - half, i, r)] = f32x4{x[i][4 * r], x[i][4 * r + 1], x[i][4 * r + 2], x[i][4 * r + 3]};
      }
      publish();
      if (part < half) {
#pragma unroll
        for (int i = 0; i < kParts; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const f32x4 y = held[at(part, i, r)];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i][4 * r + e] += y[e];
          }
      }
    }
  };
  join(dk);
  join(dv);
  if (part > 0) return;
  const bool real = key < k.length;
  if (a.splits > 1) {                // splits x total_k x k_heads x (dk, dv) x D
    if (!real) return;
    float* to = a.part_sums + (((int64_t)split * a.total_k + k.first + key) * a.k_heads + k_head) * 2 * D + 4 * h;
#pragma unroll
    for (int i = 0; i < kParts; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        *reinterpret_cast<f32x4*>(to + 32 * i + 2 * r) = f32x4{dk[i][r], dk[i][r + 1], dk[i][r + 2], dk[i][r + 3]};
        *reinterpret_cast<f32x4*>(to + D + 32 * i + 2 * r) = f32x4{dv[i][r], dv[i][r + 1], dv[i][r + 2], dv[i][r + 3]};
      }
    return;
  }
  const int64_t token = k.first + min(key, k.length - 1);
  store_columns<D>(dk, a.scale, args.dk.at(token, k_head), real, lane);
  store_columns<D>(dv, 1.f, args.dv.at(token, k_head), real, lane);
}

// The splits' sums of a key, dk and dv, added up in their order: D / 4 lanes for a key, four dimensions of both a lane.
constexpr int kSumThreads = 256;
template <int D>
struct SumShape {
  static constexpr int kLanes = D / 4, kKeys = kSumThreads / kLanes;
};
template <int D>
__global__ void __launch_bounds__(kSumThreads) attention_dkv_sum_kernel(PromptBackArgs args) {
  const PromptArgs& a = args.f;
  using S = SumShape<D>;
  const PromptPiece piece = prompt_piece((int)blockIdx.x, a.slots, a.k_heads, 1, a.num_xcd, a.sets);
  if (piece.turn < 0) return;
  const TurnPlace place = find_turn(a.cu_k, a.total_k, a.cu_q, a.total_q, a.sequences, S::kKeys, piece.turn);
  const int key = place.tile * S::kKeys + (int)threadIdx.x / S::kLanes, d = (int)threadIdx.x % S::kLanes * 4;
  if (place.tile < 0 || key >= place.mine.length) return;
  const int64_t token = place.mine.first + key, step = (int64_t)a.total_k * a.k_heads * 2 * D;
  const float* from = a.part_sums + (token * a.k_heads + piece.k_head) * 2 * D + d;
  f32x4 dk = f32x4{}, dv = f32x4{};
#pragma unroll 4
  for (int s = 0; s < a.splits; ++s) {
    dk += *reinterpret_cast<const f32x4*>(from + s * step);
    dv += *reinterpret_cast<const f32x4*>(from + s * step + D);
  }
  dk *= a.scale;
  *reinterpret_cast<u32x2*>(args.dk.at(token, piece.k_head) + d) = u32x2{pack_bf16(dk[0], dk[1]), pack_bf16(dk[2], dk[3])};
  *reinterpret_cast<u32x2*>(args.dv.at(token, piece.k_head) + d) = u32x2{pack_bf16(dv[0], dv[1]), pack_bf16(dv[2], dv[3])};
}

}  // namespace swz
