// Attention over packed prompts, forward.
#pragma once

#include "attention_tiles.h"

namespace swz {

constexpr int kPromptKeys = 64;        // keys of a tile
constexpr float kLazyRise = 8.f;       // a maximum that rises by less than 2^8 does not rescale what has been summed

template <int D, int NW>
struct PromptShape {
  static constexpr int kRows = 32 * NW;
  static constexpr int kTileBytes = kPromptKeys * 2 * D;
  static constexpr int kLdsBytes = 4 * kTileBytes;
};

// o += p v for the 32 keys from `first` on of a tile that the lane's row looks at (up to `last` of the tile), one at a time; p as the score product leaves it.
template <int D>
__device__ __forceinline__ void add_by_key(f32x16 (&o)[D / 32], const f32x16& p, const uint16_t* v_tile, int first, int last, int lane) {
  const int h = lane >> 5;
#pragma unroll 1
  for (int key = 0; key < 32; ++key) {
    float mine = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) mine = key == 8 * (r / 4) + 4 * h + r % 4 ? p[r] : mine;
    const float w = (float)(__bf16)across_halves(mine, [](float x, float y) { return x + y; });
    const int row = first + key;
    const bool seen = row <= last;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int part = 0; part < 4; ++part) {
        typedef __attribute__((ext_vector_type(4))) uint16_t u16x4;
        const int d = 32 * i + 8 * part + 4 * h;
        const u16x4 v = *reinterpret_cast<const u16x4*>(v_tile + row * D + (((d >> 3) ^ tile_key<D>(row)) << 3) + (d & 7));
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][4 * part + e] += seen ? w * __uint_as_float((uint32_t)v[e] << 16) : 0.f;
        __builtin_amdgcn_sched_barrier(0);                  // few registers at a time: this path is rare, and they are the kernel's
      }
  }
}

template <int D, int NW, bool CAUSAL>
__global__ void __launch_bounds__(NW * 64, D == 64 ? 4 : 2) attention_kernel(PromptArgs a) {
  using S = PromptShape<D, NW>;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S::kLdsBytes];
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;

  const int group = a.q_heads / a.k_heads;
  const int l = swz_xcd_renumber((int)blockIdx.x, (int)gridDim.x, a.num_xcd);
  const int k_head = l / (a.slots * group), rest = l - k_head * (a.slots * group), turn = rest / group;
  const int head = k_head * group + (rest - turn * group);
  const SlotPlace place = find_slot(a.cu_q, a.sequences, a.total_q, S::kRows, a.slots - 1 - turn);
  const Span q = sequence_span(a.cu_q, place.sequence, a.total_q), k = sequence_span(a.cu_k, place.sequence, a.total_k);
  const int first = place.tile * S::kRows;
  if (place.tile < 0 || first >= q.length) return;

  const int row0 = first + wave * 32, row = row0 + (lane & 31);
  const int ahead = k.length - q.length;                    // causal: query i looks at keys 0 .. i + ahead
  auto keys_of = [&](int last_row) { return CAUSAL ? clamp_to(last_row + ahead + 1, 0, k.length) : k.length; };
  const int keys = keys_of(min(first + S::kRows, q.length) - 1);              // of any row of the workgroup,
  const int wave_keys = row0 < q.length ? keys_of(min(row0 + 32, q.length) - 1) : 0, all_keys = keys_of(row0);   // any and every row of the wave
  const int last_key = keys_of(row) - 1;
  const int tiles = (keys + kPromptKeys - 1) / kPromptKeys;

  const uint16_t *k_rows = a.k.at(k.first, k_head), *v_rows = a.v.at(k.first, k_head);
  auto fetch = [&](int t) {
    const uint32_t at = lds + (uint32_t)((t & 1) * S::kTileBytes);
    load_rows<D, kPromptKeys, NW>(k_rows, a.k.token, t * kPromptKeys, k.length, at, wave, lane);
    load_rows<D, kPromptKeys, NW>(v_rows, a.v.token, t * kPromptKeys, k.length, at + 2 * S::kTileBytes, wave, lane);
  };
  bf16x8 qf[D / 16];
  load_fragments<D>(qf, a.q.at(q.first + min(row, q.length - 1), head), lane);
  f32x16 o[D / 32];
  const float c = a.scale * kLog2E;
  float top, sum;                                           // of scores times c; this lane's half of the sum

  // A weight of 0 times an infinity or NaN is NaN: where a value that only some rows of a tile look at is no finite number, the products carry it into the others.
  // The result shows it, and the tiles are then taken a second time, the masked ones key by key.
  auto all_tiles = [&](auto careful) __attribute__((always_inline)) {
    if (tiles > 0) fetch(0);
    top = -FLT_MAX;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = f32x16{};
    for (int t = 0; t < tiles; ++t) {
      publish();
      if (t + 1 < tiles) fetch(t + 1);
      const int k0 = t * kPromptKeys;
      if (k0 >= wave_keys) continue;
      const uint32_t at = lds + (uint32_t)((t & 1) * S::kTileBytes);
      const uint32_t k_lane = row_address<D>(at, lane), v_lane = column_address<D>(at + 2 * S::kTileBytes, lane);
      f32x16 s[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        s[b] = f32x16{};
#pragma unroll
        for (int i = 0; i < D / 16; ++i) s[b] = mfma32(read_rows<D>(k_lane, b, i), qf[i], s[b]);
      }
      const bool masked = k0 + kPromptKeys > all_keys;
      if (masked) {
        const int last = last_key - k0 - 4 * h;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[b][r] = 32 * b + 8 * (r / 4) + r % 4 <= last ? s[b][r] : -INFINITY;
      }
      float high = s[0][0];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) high = fmaxf(high, s[b][r]);
      high = across_halves(high, [](float x, float y) { return fmaxf(x, y); }) * c;
      if (__any(high > top + kLazyRise)) {
        const float now = fmaxf(top, high), less = __builtin_amdgcn_exp2f(top - now);
        sum *= less;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) o[i] *= less;
        top = now;
      }
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], c, -top));
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += s[b][r];
      }
      if (decltype(careful)::value && masked) {
        const uint16_t* v_tile = reinterpret_cast<const uint16_t*>(smem + (t & 1) * S::kTileBytes + 2 * S::kTileBytes);
        add_by_key<D>(o, s[0], v_tile, 0, last_key - k0, lane);
        add_by_key<D>(o, s[1], v_tile, 32, last_key - k0, lane);
        continue;
      }
      bf16x8 p[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) p[j] = as_operand(s[j / 2], j % 2);
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[i] = mfma32(read_columns<D>(v_lane, j, i), p[j], o[i]);
    }
  };
  all_tiles(std::false_type{});
  if constexpr (CAUSAL) {
    float odd = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) odd = __builtin_fmaf(o[i][r], 0.f, odd);
    if (__builtin_expect(__syncthreads_or(odd != 0.f), 0)) all_tiles(std::true_type{});
  }

  sum = across_halves(sum, [](float x, float y) { return x + y; });
  const bool real = row < q.length;
  store_columns<D>(o, sum == 0.f ? 0.f : 1.f / sum, a.out.at(q.first + min(row, q.length - 1), head), real, lane);
  if (real && h == 0) a.lse[(int64_t)head * a.total_q + q.first + row] = sum == 0.f ? -INFINITY : __builtin_fmaf(top, kLn2, __logf(sum));
}

}  // namespace swz
