// Norm and rotation of queries and keys, and their gradient.
#pragma once

#include "attention_tiles.h"

namespace swz {

struct NormArgs {
  Heads x[2], z[2], dx[2];           // queries, keys: input, output (or its gradient), gradient of the input
  const uint16_t* weight[2];
  const float *cos, *sin;
  const int32_t* positions;
  float* partial;                    // gradient of the weights: workgroups x 2 x D
  int rows[2], heads[2];             // rows: tokens * heads
  int blocks_q;                      // forward: workgroups that take queries
  int rotary, table_rows;
  float eps;
};

constexpr int kNormThreads = 256;
constexpr int kNormUnroll = 4;       // rows whose loads are on their way together

// Sum over the 8 or 16 neighbouring lanes that hold a row.
template <int LANES>
__device__ __forceinline__ float row_sum(float x) {
  auto dpp = [](float v, auto ctrl) __attribute__((always_inline)) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false));
  };
  x += dpp(x, std::integral_constant<int, 0xB1>{});        // quad_perm [1,0,3,2]
  x += dpp(x, std::integral_constant<int, 0x4E>{});        // quad_perm [2,3,0,1]
  x += dpp(x, std::integral_constant<int, 0x141>{});       // row_half_mirror
  if constexpr (LANES == 16) x += dpp(x, std::integral_constant<int, 0x140>{});   // row_mirror
  return x;
}

__device__ __forceinline__ void unpack8(const u32x4& v, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(v[e] << 16);
    x[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
  u32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
  return v;
}

// Which token and head the rows of a workgroup are: one division for its first row, the others are near it.
struct RowPlace {
  int token, head;
};
__device__ __forceinline__ RowPlace row_place(int first_token, int first_head, int step, int heads, float per_head) {
  const int x = first_head + step, t = (int)(((float)x + 0.5f) * per_head);       // x < 2^16 + heads: exact
  return {first_token + t, x - t * heads};
}

// The lane's 8 dimensions of a row and what turns them.
template <int D, bool INTERLEAVED>
struct Turn {
  int at, partner;                   // first of the lane's angles, -1 where its dimensions are not turned; the lane that has the other halves of its pairs
  float sign;                        // of the other half's part: -1 for the first half of a pair
  __device__ __forceinline__ Turn(int rotary, int lane) {
    const int d = (lane % (D / 8)) * 8, half = rotary / 2;
    at = d >= rotary ? -1 : INTERLEAVED ? d / 2 : d % half;
    partner = INTERLEAVED || d >= rotary ? lane : d < half ? lane + half / 8 : lane - half / 8;
    sign = d < half ? -1.f : 1.f;
  }
};

struct Angles {
  float c[8], s[8];
};
template <int D, bool INTERLEAVED>
__device__ __forceinline__ void load_angles(Angles& a, const NormArgs& n, const Turn<D, INTERLEAVED>& turn, int position) {
  constexpr int kAngles = INTERLEAVED ? 4 : 8;
  if ((unsigned)position >= (unsigned)n.table_rows) {
#pragma unroll
    for (int e = 0; e < kAngles; ++e) a.c[e] = a.s[e] = __builtin_nanf("");
  } else if (turn.at < 0) {
#pragma unroll
    for (int e = 0; e < kAngles; ++e) a.c[e] = 1.f, a.s[e] = 0.f;
  } else {
    const int64_t first = (int64_t)position * (n.rotary / 2) + turn.at;
#pragma unroll
    for (int e = 0; e < kAngles; e += 4) {
      const f32x4 c = *reinterpret_cast<const f32x4*>(n.cos + first + e), s = *reinterpret_cast<const f32x4*>(n.sin + first + e);
#pragma unroll
      for (int i = 0; i < 4; ++i) a.c[e + i] = c[i], a.s[e + i] = s[i];
    }
  }
}

// z = own * c -/+ other * s.  `back` turns the other way.
template <int D, bool INTERLEAVED>
__device__ __forceinline__ void turn_by(float (&x)[8], const float (&other)[8], const Angles& a, const Turn<D, INTERLEAVED>& turn, bool back) {
  if constexpr (INTERLEAVED) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float lo = x[2 * e], hi = x[2 * e + 1], s = back ? -a.s[e] : a.s[e];
      x[2 * e] = lo * a.c[e] - hi * s;
      x[2 * e + 1] = hi * a.c[e] + lo * s;
    }
  } else {
    const float sign = back ? -turn.sign : turn.sign;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = x[e] * a.c[e] + other[e] * (a.s[e] * sign);
  }
}

template <bool INTERLEAVED>
__device__ __forceinline__ u32x4 from_lane(const u32x4& v, int lane) {
  if constexpr (INTERLEAVED) return v;
  u32x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = (uint32_t)__builtin_amdgcn_ds_bpermute(lane * 4, (int)v[e]);
  return w;
}

template <int D, bool INTERLEAVED>
__global__ void __launch_bounds__(kNormThreads) qk_norm_kernel(NormArgs n) {
  constexpr int kLanes = D / 8, kRows = kNormThreads / kLanes;
  const int which = (int)blockIdx.x < n.blocks_q ? 0 : 1, block = (int)blockIdx.x - (which ? n.blocks_q : 0);
  const int rows = n.rows[which], heads = n.heads[which], lane = threadIdx.x & 63, d = ((int)threadIdx.x % kLanes) * 8;
  const Heads &in = n.x[which], &out = n.z[which];
  const int first = block * (kRows * kNormUnroll), token0 = first / heads, head0 = first - token0 * heads;
  const float per_head = 1.f / (float)heads;
  const Turn<D, INTERLEAVED> turn(n.rotary, lane);

  u32x4 x[kNormUnroll];
  RowPlace p[kNormUnroll];
  int position[kNormUnroll];
#pragma unroll
  for (int i = 0; i < kNormUnroll; ++i) {
    const int step = i * kRows + (int)threadIdx.x / kLanes;
    p[i] = row_place(token0, head0, min(step, rows - 1 - first), heads, per_head);      // past the end: the last row once more
    x[i] = *reinterpret_cast<const u32x4*>(in.at(p[i].token, p[i].head) + d);
    position[i] = n.positions[p[i].token];
  }
  float w[8], w_other[8];
  const u32x4 weight = *reinterpret_cast<const u32x4*>(n.weight[which] + d);
  unpack8(weight, w);
  unpack8(from_lane<INTERLEAVED>(weight, turn.partner), w_other);
#pragma unroll
  for (int i = 0; i < kNormUnroll; ++i) {
    Angles a;
    load_angles(a, n, turn, position[i]);
    float v[8], other[8];
    unpack8(x[i], v);
    unpack8(from_lane<INTERLEAVED>(x[i], turn.partner), other);
    float squares = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) squares = __builtin_fmaf(v[e], v[e], squares);
    const float r = __builtin_amdgcn_rsqf(row_sum<kLanes>(squares) * (1.f / D) + n.eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] *= r * w[e];
      other[e] *= r * w_other[e];
    }
    turn_by(v, other, a, turn, false);
    const int step = i * kRows + (int)threadIdx.x / kLanes;
    if (first + step < rows) *reinterpret_cast<u32x4*>(out.at(p[i].token, p[i].head) + d) = pack8(v);
  }
}

// With u = x r, y = u w: dy is dz turned back, dw = sum dy u, du = dy w, dx = r (du - u mean(du u)).  A workgroup goes over rows of queries, then of keys, in steps of the whole
// grid, each lane summing the weights' gradient of its dimensions; its sums go to `partial`, which norm_weights_kernel adds up.
template <int D, bool INTERLEAVED>
__global__ void __launch_bounds__(kNormThreads) qk_norm_backward_kernel(NormArgs n) {
  constexpr int kLanes = D / 8, kRows = kNormThreads / kLanes, kUnroll = 2;
  __shared__ float sums[kRows][D];
  const int lane = threadIdx.x & 63, d = ((int)threadIdx.x % kLanes) * 8, mine = (int)threadIdx.x / kLanes;
  const Turn<D, INTERLEAVED> turn(n.rotary, lane);
  for (int which = 0; which < 2; ++which) {
    const int rows = n.rows[which], heads = n.heads[which];
    const Heads &in = n.x[which], &grad = n.z[which], &out = n.dx[which];
    const float per_head = 1.f / (float)heads;
    float w[8], dw[8];
    unpack8(*reinterpret_cast<const u32x4*>(n.weight[which] + d), w);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[e] = 0.f;
    for (int64_t first64 = (int64_t)blockIdx.x * (kRows * kUnroll); first64 < rows; first64 += (int64_t)gridDim.x * (kRows * kUnroll)) {
      const int first = (int)first64, token0 = first / heads, head0 = first - token0 * heads;
      u32x4 x[kUnroll], g[kUnroll];
      RowPlace p[kUnroll];
      int position[kUnroll];
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) {
        p[i] = row_place(token0, head0, min(i * kRows + mine, rows - 1 - first), heads, per_head);
        x[i] = *reinterpret_cast<const u32x4*>(in.at(p[i].token, p[i].head) + d);
        g[i] = *reinterpret_cast<const u32x4*>(grad.at(p[i].token, p[i].head) + d);
        position[i] = n.positions[p[i].token];
      }
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) {
        const bool real = first + i * kRows + mine < rows;
        Angles a;
        load_angles(a, n, turn, position[i]);
        float u[8], dy[8], other[8];
        unpack8(x[i], u);
        unpack8(g[i], dy);
        unpack8(from_lane<INTERLEAVED>(g[i], turn.partner), other);
        turn_by(dy, other, a, turn, true);
        float squares = 0.f, along = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) squares = __builtin_fmaf(u[e], u[e], squares);
        const float r = __builtin_amdgcn_rsqf(row_sum<kLanes>(squares) * (1.f / D) + n.eps);
        float du[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[e] *= r;
          dw[e] += real ? dy[e] * u[e] : 0.f;
          du[e] = dy[e] * w[e];
          along = __builtin_fmaf(du[e], u[e], along);
        }
        along = row_sum<kLanes>(along) * (1.f / D);
#pragma unroll
        for (int e = 0; e < 8; ++e) du[e] = r * (du[e] - u[e] * along);
        if (real) *reinterpret_cast<u32x4*>(out.at(p[i].token, p[i].head) + d) = pack8(du);
      }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[mine][d + e] = dw[e];
    __syncthreads();
    if ((int)threadIdx.x < D) {
      float total = 0.f;
#pragma unroll
      for (int i = 0; i < kRows; ++i) total += sums[i][threadIdx.x];
      n.partial[((int64_t)blockIdx.x * 2 + which) * D + threadIdx.x] = total;
    }
  }
}

// Sums of `parts` rows of 2 D, 16 columns a workgroup: out[0][d], out[1][d].
__global__ void __launch_bounds__(256) norm_weights_kernel(const float* partial, int parts, int dims, float* q_weight, float* k_weight) {
  __shared__ float sums[16][17];
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4, column = (int)blockIdx.x * 16 + c;
  float total = 0.f;
  for (int i = r; i < parts; i += 16) total += partial[(int64_t)i * (2 * dims) + column];
  sums[r][c] = total;
  __syncthreads();
  if (r == 0) {
    total = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) total += sums[i][c];
    if (column < dims) q_weight[column] = total;
    else k_weight[column - dims] = total;
  }
}

}  // namespace swz
