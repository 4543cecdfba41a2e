// Attention over packed prompts, backward.
#pragma once

#include "attention_kernel.h"

namespace swz {

struct PromptBackArgs {
  PromptArgs f;                    // slots: of this launch
  Heads dout, dq, dk, dv;
  float* delta;                    // q_heads x total_q: sum over the dimensions of dout * out
};

// dq, and delta for the other kernel.  As the forward kernel, with a third product: dq^T += k^T dS^T.
template <int D, int NW, bool CAUSAL>
__global__ void __launch_bounds__(NW * 64, 2) attention_dq_kernel(PromptBackArgs args) {
  const PromptArgs& a = args.f;
  using S = PromptShape<D, NW>;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S::kLdsBytes];
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;

  const int group = a.q_heads / a.k_heads;
  const PromptPiece piece = prompt_piece((int)blockIdx.x, a.slots, a.k_heads, group, a.num_xcd, a.sets);
  if (piece.turn < 0) return;
  const int k_head = piece.k_head, head = k_head * group + piece.member;
  const TurnPlace place = find_turn(a.cu_q, a.total_q, a.cu_k, a.total_k, a.sequences, S::kRows, piece.turn);
  const Span q = place.mine, k = place.other;
  const int first = ((q.length + S::kRows - 1) / S::kRows - 1 - place.tile) * S::kRows;
  if (place.tile < 0 || first < 0) return;

  const int row0 = first + wave * 32, row = row0 + (lane & 31);
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
  if (real && h == 0) args.delta[stat] = delta;
  const float lse = a.lse[stat] * kLog2E;                   // -inf where a row looks at nothing: all of it is masked below
  load_fragments<D>(qf, a.q.at(token, head), lane);
  f32x16 acc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) acc[i] = f32x16{};
  const float c = a.scale * kLog2E;

  for (int t = 0; t < tiles; ++t) {
    publish();
    if (t + 1 < tiles) fetch(t + 1);
    const int k0 = t * kPromptKeys;
    if (k0 >= wave_keys) continue;
    const uint32_t at = lds + (uint32_t)((t & 1) * S::kTileBytes);
    const uint32_t k_lane = row_address<D>(at, lane), v_lane = row_address<D>(at + 2 * S::kTileBytes, lane), kt_lane = column_address<D>(at, lane);
    const bool masked = k0 + kPromptKeys > all_keys;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      f32x16 s = f32x16{}, dp = f32x16{};
#pragma unroll
      for (int i = 0; i < D / 16; ++i) s = mfma32(read_rows<D>(k_lane, b, i), qf[i], s);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) dp = mfma32(read_rows<D>(v_lane, b, i), gf[i], dp);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -lse)) * (dp[r] - delta);
      if (masked) {
        const int last = last_key - k0 - 32 * b - 4 * h;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 8 * (r / 4) + r % 4 <= last ? s[r] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const bf16x8 ds = as_operand(s, j);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) acc[i] = mfma32(read_columns<D>(kt_lane, 2 * b + j, i), ds, acc[i]);
      }
    }
  }
  store_columns<D>(acc, a.scale, args.dq.at(token, head), real, lane);
}

// dk and dv of 32 NW keys of a key head, summed over the queries of all its query heads.  A wave has 32 keys, as columns: their rows of k
// and v are B of S = q k^T and dP = dout v^T, whose rows are queries, so that P and dS are B of dv^T += dout^T P and dk^T += q^T dS.
constexpr int kBackRows = 32;      // queries of a tile

template <int D, int NW, bool CAUSAL>
__global__ void __launch_bounds__(NW * 64, 2) attention_dkv_kernel(PromptBackArgs args) {
  const PromptArgs& a = args.f;
  constexpr int kKeys = 32 * NW, kTileBytes = kBackRows * 2 * D;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * kTileBytes];
  __shared__ __attribute__((aligned(16))) float stats[2][2][kBackRows];
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;

  const int group = a.q_heads / a.k_heads;
  const PromptPiece piece = prompt_piece((int)blockIdx.x, a.slots, a.k_heads, 1, a.num_xcd, a.sets);
  if (piece.turn < 0) return;
  const int k_head = piece.k_head;
  const TurnPlace place = find_turn(a.cu_k, a.total_k, a.cu_q, a.total_q, a.sequences, kKeys, piece.turn);
  const Span q = place.other, k = place.mine;
  const int first = place.tile * kKeys;
  if (place.tile < 0 || first >= k.length) return;

  const int key0 = first + wave * 32, key = key0 + (lane & 31);
  const int ahead = k.length - q.length;
  const int from = CAUSAL ? clamp_to(first - ahead, 0, q.length) / kBackRows : 0;      // the first tile of queries that looks at a key of the workgroup
  const int tiles = (q.length + kBackRows - 1) / kBackRows - from, steps = tiles > 0 ? tiles * group : 0;

  const int64_t token = k.first + min(key, k.length - 1);
  bf16x8 kf[D / 16], vf[D / 16];
  load_fragments<D>(kf, a.k.at(token, k_head), lane);
  load_fragments<D>(vf, a.v.at(token, k_head), lane);
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) dk[i] = dv[i] = f32x16{};
  const float c = a.scale * kLog2E;

  RowLoader<D, kBackRows, NW> load_q(a.q.data, a.q.token, q.length, wave, lane), load_g(args.dout.data, args.dout.token, q.length, wave, lane);
  float stat = 0.f;                                         // thread i < 32: lse of row i, in units of log2; i < 64: delta of row i - 32
  auto fetch = [&](int n) {
    const int m = n / tiles, r0 = (from + n - m * tiles) * kBackRows, head = k_head * group + m;
    const uint32_t at = lds + (uint32_t)((n & 1) * kTileBytes);
    load_q.head = a.q.at(q.first, head);
    load_g.head = args.dout.at(q.first, head);
    load_q(r0, at);
    load_g(r0, at + 2 * kTileBytes);
    if (threadIdx.x < 64) {
      const int r = r0 + (lane & 31);
      const float* from_stat = lane < 32 ? a.lse : args.delta;
      stat = r < q.length ? from_stat[(int64_t)head * a.total_q + q.first + r] : 0.f;
      // rows past the end, and rows that look at nothing, get weights of 0
      if (lane < 32) stat = r < q.length && stat != -INFINITY ? stat * kLog2E : INFINITY;
    }
  };
  if (steps > 0) fetch(0);
  for (int n = 0; n < steps; ++n) {
    if (threadIdx.x < 64) stats[n & 1][lane >> 5][lane & 31] = stat;
    publish();
    if (n + 1 < steps) fetch(n + 1);
    const int m = n / tiles, r0 = (from + n - m * tiles) * kBackRows;
    if (CAUSAL && r0 + kBackRows - 1 + ahead < key0) continue;               // none of these rows looks at a key of this wave
    const uint32_t at = lds + (uint32_t)((n & 1) * kTileBytes);
    const uint32_t q_lane = row_address<D>(at, lane), g_lane = row_address<D>(at + 2 * kTileBytes, lane);
    f32x16 s = f32x16{}, dp = f32x16{};
#pragma unroll
    for (int i = 0; i < D / 16; ++i) s = mfma32(read_rows<D>(q_lane, 0, i), kf[i], s);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) dp = mfma32(read_rows<D>(g_lane, 0, i), vf[i], dp);
    const bool masked = (CAUSAL && r0 + ahead < key0 + 31) || key0 + 32 > k.length;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 lse = *reinterpret_cast<const f32x4*>(&stats[n & 1][0][8 * i + 4 * h]);
      const f32x4 delta = *reinterpret_cast<const f32x4*>(&stats[n & 1][1][8 * i + 4 * h]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 4 * i + e;
        s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -lse[e]));
        dp[r] = s[r] * (dp[r] - delta[e]);
      }
    }
    if (masked) {
      const int first_row = CAUSAL ? key - ahead - r0 - 4 * h : -1;          // of this key
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const bool looked_at = 8 * (r / 4) + r % 4 >= first_row && key < k.length;
        s[r] = looked_at ? s[r] : 0.f;
        dp[r] = looked_at ? dp[r] : 0.f;
      }
    }
    const uint32_t qt_lane = column_address<D>(at, lane), gt_lane = column_address<D>(at + 2 * kTileBytes, lane);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const bf16x8 p = as_operand(s, j), ds = as_operand(dp, j);
#pragma unroll
      for (int i = 0; i < D / 32; ++i) dv[i] = mfma32(read_columns<D>(gt_lane, j, i), p, dv[i]);
#pragma unroll
      for (int i = 0; i < D / 32; ++i) dk[i] = mfma32(read_columns<D>(qt_lane, j, i), ds, dk[i]);
    }
  }
  const bool real = key < k.length;
  store_columns<D>(dk, a.scale, args.dk.at(token, k_head), real, lane);
  store_columns<D>(dv, 1.f, args.dv.at(token, k_head), real, lane);
}

}  // namespace swz
