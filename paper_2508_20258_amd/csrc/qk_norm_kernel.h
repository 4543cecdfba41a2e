// Norm and rotation of queries and keys, and their gradient.
//
// With r = 1 / sqrt(mean(x^2) + eps) and R the rotation of a token's position: z = R (x r w).  Backward: dy = R^T dz, u = x r, dw = sum over tokens and heads of dy u, and
// dx = r (dy w - u mean(dy w u)); r is worked out again from x, which is read anyway.  All of it in 32 bits, rounded once.
// HBM is the bound: every element is read once and written once.  32768 tokens of 32 + 8 heads of 128: 127 us, 5.4 TB/s of 6.0 that a copy reaches.  Backward, 12345 tokens: 75 us, 5.1 TB/s, and 5 us for the
// weights' sums; 4096 tokens of 16 + 16 heads of 64: 12.6 and 3.5.
#pragma once

#include "attention_tiles.h"
#include "norm_place.h"

namespace swz {

// Of queries or keys: input, output (or its gradient), gradient of the input.
struct NormSide {
  Heads x, z, dx;
  const uint16_t* weight;
  int heads, blocks, items;          // blocks of kNormHeads heads of a token; of all tokens
};
struct NormArgs {
  NormSide q, k;
  const float *cos, *sin;
  const int32_t* positions;
  float* partial;                    // gradient of the weights: workgroups x 2 x D
  int workgroups_q;                  // forward: those that take queries
  int rotary, table_rows;
  float eps;
};

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

// Which lane has the other halves of a lane's pairs, and whether the lane's dimensions have any.
struct Partner {
  int lane;
  uint32_t bits;                     // all where the lane's dimensions are turned, else none
};
template <int D, bool INTERLEAVED>
__device__ __forceinline__ Partner partner_of(int rotary, int lane) {
  const int d = (lane % (D / 8)) * 8, half = rotary / 2;
  return {INTERLEAVED || d >= rotary ? lane : d < half ? lane + half / 8 : lane - half / 8, d < rotary ? ~0u : 0u};
}
// The halves: of other lanes, or (interleaved) the neighbours.  0 for dimensions that are not turned: a sine of 0 would not keep an infinity or NaN out.
template <bool INTERLEAVED>
__device__ __forceinline__ void others(const u32x4& v, Partner partner, float (&other)[8]) {
  u32x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = (INTERLEAVED ? v[e] << 16 | v[e] >> 16 : (uint32_t)__builtin_amdgcn_ds_bpermute(partner.lane * 4, (int)v[e])) & partner.bits;
  unpack8(w, other);
}

// z[e] = x[e] c[e] + other[e] s[e] turns the lane's dimensions by the token's angles (back: the other way).  NaN for a position outside the tables.
struct Angles {
  float c[8], s[8];
};
template <int D, bool INTERLEAVED>
__device__ __forceinline__ void load_angles(Angles& a, const NormArgs& n, int position, int lane, bool back) {
  constexpr int kAngles = INTERLEAVED ? 4 : 8;
  const int d = (lane % (D / 8)) * 8, half = n.rotary / 2;
  const bool known = (unsigned)position < (unsigned)n.table_rows;
  f32x4 c[kAngles / 4], s[kAngles / 4];
#pragma unroll
  for (int i = 0; i < kAngles / 4; ++i) c[i] = 1.f, s[i] = 0.f;
  if (known && d < n.rotary) {
    const int64_t first = (int64_t)position * half + (INTERLEAVED ? d / 2 : d < half ? d : d - half);
#pragma unroll
    for (int i = 0; i < kAngles / 4; ++i) {
      c[i] = *reinterpret_cast<const f32x4*>(n.cos + first + 4 * i);
      s[i] = *reinterpret_cast<const f32x4*>(n.sin + first + 4 * i);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int i = INTERLEAVED ? e / 2 : e;
    const bool minus = (INTERLEAVED ? e % 2 == 0 : d < half) != back;             // the first of a pair loses what the second turns into it
    a.c[e] = known ? c[i / 4][i % 4] : __builtin_nanf("");
    a.s[e] = minus ? -s[i / 4][i % 4] : s[i / 4][i % 4];
  }
}

template <int D, bool INTERLEAVED>
__global__ void __launch_bounds__(kNormThreads) qk_norm_kernel(NormArgs n) {
  constexpr int kLanes = D / 8, kItems = kNormThreads / kLanes;
  const bool keys = (int)blockIdx.x >= n.workgroups_q;
  const NormSide side = keys ? n.k : n.q;
  const int lane = threadIdx.x & 63, d = ((int)threadIdx.x % kLanes) * 8;
  const NormPlace p = norm_place((int64_t)((int)blockIdx.x - (keys ? n.workgroups_q : 0)) * kItems + (int)threadIdx.x / kLanes, side.items, side.blocks);
  const int position = n.positions[p.token];
  u32x4 x[kNormHeads];
#pragma unroll
  for (int i = 0; i < kNormHeads; ++i) x[i] = *reinterpret_cast<const u32x4*>(side.x.at(p.token, min(p.head0 + i, side.heads - 1)) + d);
  const u32x4 weight = *reinterpret_cast<const u32x4*>(side.weight + d);
  const Partner partner = partner_of<D, INTERLEAVED>(n.rotary, lane);
  Angles a;
  load_angles<D, INTERLEAVED>(a, n, position, lane, false);
  float w[8], w_other[8];
  unpack8(weight, w);
  others<INTERLEAVED>(weight, partner, w_other);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    a.c[e] *= w[e];
    a.s[e] *= w_other[e];
  }
#pragma unroll
  for (int i = 0; i < kNormHeads; ++i) {
    float v[8], other[8], squares = 0.f;
    unpack8(x[i], v);
    others<INTERLEAVED>(x[i], partner, other);
#pragma unroll
    for (int e = 0; e < 8; ++e) squares = __builtin_fmaf(v[e], v[e], squares);
    const float r = __builtin_amdgcn_rsqf(row_sum<kLanes>(squares) * (1.f / D) + n.eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(v[e], a.c[e], other[e] * a.s[e]) * r;
    if (norm_stores(p, i, side.heads)) *reinterpret_cast<u32x4*>(side.z.at(p.token, p.head0 + i) + d) = pack8(v);
  }
}

// With u = x r, y = u w: dy is dz turned back, dw = sum dy u, du = dy w, dx = r (du - u mean(du u)).  A workgroup goes over blocks of heads of queries, then of keys, in steps of the
// whole grid, each lane summing the weights' gradient of its dimensions; its sums go to `partial`, which norm_weights_kernel adds up.
template <int D, bool INTERLEAVED>
__global__ void __launch_bounds__(kNormThreads, 4) qk_norm_backward_kernel(NormArgs n) {
  constexpr int kLanes = D / 8, kItems = kNormThreads / kLanes;
  __shared__ float sums[kItems][D];
  const int lane = threadIdx.x & 63, d = ((int)threadIdx.x % kLanes) * 8, mine = (int)threadIdx.x / kLanes;
  const Partner partner = partner_of<D, INTERLEAVED>(n.rotary, lane);
  for (int keys = 0; keys < 2; ++keys) {
    const NormSide side = keys ? n.k : n.q;
    float w[8], dw[8];
    unpack8(*reinterpret_cast<const u32x4*>(side.weight + d), w);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[e] = 0.f;
    // the last turn of a wave may be partly past the end: those lanes keep nothing
    for (int64_t first = (int64_t)blockIdx.x * kItems; first < side.items; first += (int64_t)gridDim.x * kItems) {
      const NormPlace p = norm_place(first + mine, side.items, side.blocks);
      const int position = n.positions[p.token];
      u32x4 x[kNormHeads], g[kNormHeads];
#pragma unroll
      for (int i = 0; i < kNormHeads; ++i) {
        const int head = min(p.head0 + i, side.heads - 1);
        x[i] = *reinterpret_cast<const u32x4*>(side.x.at(p.token, head) + d);
        g[i] = *reinterpret_cast<const u32x4*>(side.z.at(p.token, head) + d);
      }
      Angles a;
      load_angles<D, INTERLEAVED>(a, n, position, lane, true);
#pragma unroll
      for (int i = 0; i < kNormHeads; ++i) {
        const bool real = norm_stores(p, i, side.heads);
        float u[8], dy[8], other[8], squares = 0.f, along = 0.f;
        unpack8(x[i], u);
        unpack8(g[i], dy);
        others<INTERLEAVED>(g[i], partner, other);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          dy[e] = __builtin_fmaf(dy[e], a.c[e], other[e] * a.s[e]);
          squares = __builtin_fmaf(u[e], u[e], squares);
        }
        const float r = __builtin_amdgcn_rsqf(row_sum<kLanes>(squares) * (1.f / D) + n.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[e] *= r;
          dw[e] = real ? __builtin_fmaf(dy[e], u[e], dw[e]) : dw[e];
          dy[e] *= w[e];
          along = __builtin_fmaf(dy[e], u[e], along);
        }
        along = row_sum<kLanes>(along) * (1.f / D);
#pragma unroll
        for (int e = 0; e < 8; ++e) dy[e] = r * __builtin_fmaf(-u[e], along, dy[e]);
        if (real) *reinterpret_cast<u32x4*>(side.dx.at(p.token, p.head0 + i) + d) = pack8(dy);
      }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[mine][d + e] = dw[e];
    __syncthreads();
    if ((int)threadIdx.x < D) {
      float total = 0.f;
#pragma unroll
      for (int i = 0; i < kItems; ++i) total += sums[i][threadIdx.x];
      n.partial[((int64_t)blockIdx.x * 2 + keys) * D + threadIdx.x] = total;
    }
  }
}

// Sums of `parts` rows of 2 D, 4 columns a workgroup of 256 threads, a row each: out[0][d], out[1][d].
__global__ void __launch_bounds__(256) norm_weights_kernel(const float* partial, int parts, int dims, float* q_weight, float* k_weight) {
  __shared__ f32x4 sums[4];
  const int column = (int)blockIdx.x * 4, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  f32x4 total = f32x4{};
#pragma unroll 8
  for (int i = threadIdx.x; i < parts; i += 256) total += *reinterpret_cast<const f32x4*>(partial + (int64_t)i * (2 * dims) + column);
#pragma unroll
  for (int e = 0; e < 4; ++e) total[e] = over_wave(total[e], [](float x, float y) { return x + y; });
  if (lane == 0) sums[wave] = total;
  __syncthreads();
  if (threadIdx.x == 0) {
    total = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    *reinterpret_cast<f32x4*>(column < dims ? q_weight + column : k_weight + column - dims) = total;
  }
}

}  // namespace swz
