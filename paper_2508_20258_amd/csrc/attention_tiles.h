// What the kernels of attention over packed prompts share: which rows a workgroup has, tiles of heads in LDS, and their fragments
// for v_mfma_f32_32x32x16_bf16.
//
// The instruction multiplies A (32 x 16) by B (16 x 32).  Lane l = 32 h + i holds A[i][8 h .. + 7], B[8 h .. + 7][i], and of the product column i, rows
// 8 (r / 4) + 4 h + r % 4 in its registers r = 0..15.  Two products in a row need no exchange between lanes: where the first one's rows
// are what the second one sums over, registers 8 j .. 8 j + 7, rounded, are the second one's B for rows 16 j .. + 15, if its A is given in the same
// order: element e of lane half h is row 16 j + 8 (e / 4) + 4 h + e % 4.  The transposing reads below take four rows each, so they give that order.
//
// LDS: a row of a tile is a token's head, 2 D bytes, in 16-byte chunks; chunk c of row r is in slot c ^ tile_key(r).  Both reads are free of
// conflicts: one chunk of 16 consecutive rows is in 16 different 16-byte groups of the 256 bytes that the banks span, and the 4 rows that a half of
// a wave takes in a transposing read, 64 bytes of each, are in four different quarters of them.
#pragma once

#include <float.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gemm_kernel.h"

namespace swz {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

constexpr float kLog2E = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Heads of a tensor: pointer and distances in elements.
struct Heads {
  uint16_t* data;
  int64_t token, head;
  __device__ __forceinline__ uint16_t* at(int64_t t, int h) const { return data + t * token + (int64_t)h * head; }
};

struct PromptArgs {
  Heads q, k, v, out;
  float* lse;
  const int32_t *cu_q, *cu_k;
  int total_q, total_k, sequences, slots, q_heads, k_heads, num_xcd;
  float scale;
};

__device__ __forceinline__ int clamp_to(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// Tiles of `rows` rows of all sequences are numbered by slots: those of sequence b start at cu[b] / rows + PER * b.  With PER = 1 that leaves each sequence the
// ceil(length / rows) it needs, without a sum over the sequences before it; with PER = 2 one more, for tiles that do not start with the sequence.  There are
// total / rows + PER * sequences slots.  Which sequence a slot belongs to is a search over cu, 64 places at a time.
struct SlotPlace {
  int sequence, tile;
};
template <int PER = 1>
__device__ __forceinline__ SlotPlace find_slot(const int32_t* cu, int sequences, int total, int rows, int slot) {
  const int lane = threadIdx.x & 63;
  int lo = 0, span = sequences;
  while (span > 1) {
    const int stride = (span + 63) / 64, at = lo + lane * stride;
    const bool before = lane * stride < span && clamp_to(cu[at], 0, total) / rows + PER * at <= slot;
    int n = __popcll(__ballot(before));
    n = n > 1 ? n - 1 : 0;
    lo += n * stride;
    span = min(stride, span - n * stride);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  return {lo, slot - (clamp_to(__builtin_amdgcn_readfirstlane(cu[lo]), 0, total) / rows + PER * lo)};
}

// First token and length of a sequence, inside the tensor whatever cu holds.
struct Span {
  int first, length;
};
__device__ __forceinline__ Span sequence_span(const int32_t* cu, int sequence, int total) {
  const int a = clamp_to(__builtin_amdgcn_readfirstlane(cu[sequence]), 0, total);
  const int b = clamp_to(__builtin_amdgcn_readfirstlane(cu[sequence + 1]), a, total);
  return {a, b - a};
}

template <int D>
__device__ __forceinline__ int tile_key(int row) {
  if constexpr (D == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
  else return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}

// ROWS rows of a head, from `first` on, into LDS by all NW waves: 1024 bytes an instruction.  Rows at or past `length` come as zeros.
template <int D, int ROWS, int NW>
__device__ __forceinline__ void load_rows(const uint16_t* head, int64_t token, int first, int length, uint32_t lds, int wave, int lane) {
  constexpr int kChunks = D / 8, kRows = 64 / kChunks, kLoads = ROWS / kRows / NW;
  static_assert(kLoads * kRows * NW == ROWS, "whole instructions for every wave");
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int row = (wave * kLoads + i) * kRows + lane / kChunks, chunk = (lane % kChunks) ^ tile_key<D>(row), r = first + row;
    const void* from = r < length ? static_cast<const void*>(head + (int64_t)r * token + chunk * 8) : static_cast<const void*>(&kZeroChunk);
    load_to_lds(from, lds + (uint32_t)((wave * kLoads + i) * 1024));
  }
}

// This wave's loads have landed and its reads are done; then so are all waves'.
__device__ __forceinline__ void publish() {
  __builtin_amdgcn_sched_barrier(0);
  wait_vmcnt_lgkmcnt<0, 0>();
  __builtin_amdgcn_sched_barrier(0);
  block_barrier();
  __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// Rows 32 block .. + 31 of a tile as A, dimensions 16 step .. + 15.  `lane_row` is row_address(): the lane's row and the key's part of the chunk.
template <int D>
__device__ __forceinline__ uint32_t row_address(uint32_t lds, int lane) {
  return lds + (uint32_t)((lane & 31) * (2 * D) + (((lane >> 5) ^ tile_key<D>(lane & 31)) << 4));
}
template <int D>
__device__ __forceinline__ bf16x8 read_rows(uint32_t lane_row, int block, int step) {
  typedef __attribute__((address_space(3))) const bf16x8* ptr;
  return *(ptr)(uintptr_t)((lane_row ^ (uint32_t)(step << 5)) + (uint32_t)(block * 64 * D));
}

// Dimensions 32 part .. + 31 of rows 16 j .. + 15 as A, transposed: rows in the order above.
template <int D>
__device__ __forceinline__ uint32_t column_address(uint32_t lds, int lane) {
  const int s = lane & 15, h = lane >> 5, row = 4 * h + (s >> 2), chunk = 2 * ((lane >> 4) & 1) + ((s & 3) >> 1);
  return lds + (uint32_t)(row * (2 * D) + ((chunk ^ tile_key<D>(row)) << 4) + (s & 1) * 8);
}
template <int D>
__device__ __forceinline__ bf16x8 read_columns(uint32_t lane_column, int j, int part) {
  typedef __attribute__((address_space(3))) s16x4* ptr;
  const uint32_t at = lane_column ^ (uint32_t)(part << 6);               // chunk 4 part + ..
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(uintptr_t)(at + (uint32_t)(j * 32 * D)));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(uintptr_t)((at ^ 32u) + (uint32_t)(j * 32 * D + 16 * D)));   // rows + 8: key ^ 2
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// A head's row as B (columns are rows of the tensor), dimensions 16 step + 8 h .. + 7 for all steps.
template <int D>
__device__ __forceinline__ void load_fragments(bf16x8 (&f)[D / 16], const uint16_t* row, int lane) {
#pragma unroll
  for (int s = 0; s < D / 16; ++s) f[s] = *reinterpret_cast<const bf16x8*>(row + 16 * s + 8 * (lane >> 5));
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  bf16x2 p;
  p[0] = (__bf16)a;
  p[1] = (__bf16)b;
  return __builtin_bit_cast(uint32_t, p);
}

// Registers 8 j .. 8 j + 7 of a product, rounded, as B of the next one.
__device__ __forceinline__ bf16x8 as_operand(const f32x16& x, int j) {
  u32x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = pack_bf16(x[8 * j + 2 * e], x[8 * j + 2 * e + 1]);
  return __builtin_bit_cast(bf16x8, w);
}

// x of both halves of the wave: op over lanes l and l + 32.
template <class Op>
__device__ __forceinline__ float across_halves(float x, Op op) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return op(__uint_as_float(s[0]), __uint_as_float(s[1]));
}

// Column i of D / 32 products (dimensions 32 part + row) times `factor`, rounded and stored as a head's row: the halves trade registers so that each lane has 16 bytes.
template <int D>
__device__ __forceinline__ void store_columns(const f32x16 (&acc)[D / 32], float factor, uint16_t* row, bool real, int lane) {
#pragma unroll
  for (int part = 0; part < D / 32; ++part)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const auto s = __builtin_amdgcn_permlane32_swap(pack_bf16(acc[part][8 * i + 2 * e] * factor, acc[part][8 * i + 2 * e + 1] * factor),
                                                        pack_bf16(acc[part][8 * i + 4 + 2 * e] * factor, acc[part][8 * i + 5 + 2 * e] * factor), false, false);
        w[e] = s[0];
        w[2 + e] = s[1];
      }
      if (real) *reinterpret_cast<u32x4*>(row + 32 * part + 16 * i + 8 * (lane >> 5)) = w;
    }
}

}  // namespace swz
