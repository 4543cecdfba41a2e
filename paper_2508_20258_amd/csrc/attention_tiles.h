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
#include "prompt_order.h"

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
  int total_q, total_k, sequences, slots, q_heads, k_heads, num_xcd, sets;
  float scale;
  int splits;                        // of a row's keys, forward, or of a tile's queries, backward: each writes what it has to the parts
  float *part_sums, *part_stats;
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
__device__ __forceinline__ Span span_of(int from, int to, int total) {
  const int a = clamp_to(from, 0, total);
  return {a, clamp_to(to, a, total) - a};
}
__device__ __forceinline__ Span sequence_span(const int32_t* cu, int sequence, int total) {
  return span_of(__builtin_amdgcn_readfirstlane(cu[sequence]), __builtin_amdgcn_readfirstlane(cu[sequence + 1]), total);
}

// Sum of x over this lane and those before it.
__device__ __forceinline__ int sum_before(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);       // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);       // row_bcast:15, to rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);       // row_bcast:31, to rows 2 and 3
  return x;
}

// The turn-th tile of `rows` tokens of all sequences: which of its sequence's (-1: there is none), and the sequence's tokens on this side and the other.  Up to 64 sequences have a
// lane each.  Up to 16 take turns by the length of the other side, the longest first, which costs a few hundred clocks a workgroup; more of them even out as they come, and comparing 50
// of them costs more than it gives.  In that order and as they come: five prompts of 200 to 10000 keys 178 us and 198; a step of 16 sequences of up to 2048 tokens 245 and 259, of up to
// 300 57.0 and 55.5.
struct TurnPlace {
  Span mine, other;
  int tile;
};
__device__ __forceinline__ TurnPlace find_turn(const int32_t* cu, int total, const int32_t* other, int other_total, int sequences, int rows, int turn) {
  const int lane = threadIdx.x & 63;
  if (sequences > 64) {
    const SlotPlace p = find_slot(cu, sequences, total, rows, turn);
    return {sequence_span(cu, p.sequence, total), sequence_span(other, p.sequence, other_total), p.tile};
  }
  const int at = min(lane, sequences - 1);
  const Span a = span_of(cu[at], cu[at + 1], total), b = span_of(other[at], other[at + 1], other_total);
  const int tiles = lane < sequences ? (a.length + rows - 1) / rows : 0;
  int start = 0;
  if (sequences <= 16) {
    // all lengths of a row of lanes go by each: the longer ones, and of equal ones those before
    const int key = min(b.length, (1 << 27) - 1) << 4 | (15 - (lane & 15));
    for_each_index([&](auto i) __attribute__((always_inline)) {
      constexpr int kCtrl = 0x121 + decltype(i)::value;                  // row_ror:1 .. 15
      const int its_key = __builtin_amdgcn_mov_dpp(key, kCtrl, 0xf, 0xf, false), its_tiles = __builtin_amdgcn_mov_dpp(tiles, kCtrl, 0xf, 0xf, false);
      start += its_key > key ? its_tiles : 0;
    }, std::make_integer_sequence<int, 15>{});
  } else {
    start = sum_before(tiles) - tiles;
  }
  const uint64_t found = __ballot(turn >= start && turn < start + tiles);
  if (found == 0) return {{0, 0}, {0, 0}, -1};
  const int s = __ffsll((unsigned long long)found) - 1;
  return {{__builtin_amdgcn_readlane(a.first, s), __builtin_amdgcn_readlane(a.length, s)}, {__builtin_amdgcn_readlane(b.first, s), __builtin_amdgcn_readlane(b.length, s)},
          turn - __builtin_amdgcn_readlane(start, s)};
}

// Keeps the compiler from working a value out again where it is used.
__device__ __forceinline__ void keep(uint32_t& x) { asm volatile("" : "+v"(x)); }

template <int D>
__device__ __forceinline__ int tile_key(int row) {
  if constexpr (D == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
  else return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}

// ROWS rows of a head into LDS by NW waves, 1024 bytes an instruction.  Rows past the end are zeros: they are masked where it matters, but a weight of 0 times an infinity is
// NaN, so that copies of a real row would not do.  In whole tiles an instruction's rows
// are named by a wave-uniform base and 32-bit offsets, so the distance between tokens is less than 2^28 elements (7 rows of it fit 2^32 bytes).
template <int D, int ROWS, int NW>
struct RowLoader {
  static constexpr int kChunks = D / 8, kRows = 64 / kChunks, kLoads = ROWS / kRows / NW;
  static_assert(kLoads * kRows * NW == ROWS, "whole instructions for every wave");
  const uint16_t* head;
  int64_t token;
  int length, wave, lane;
  uint32_t row_part, chunk;          // bytes of the lane's row of an instruction; its chunk where the instruction starts at a row whose key is 0

  __device__ __forceinline__ RowLoader(const uint16_t* head_, int64_t token_, int length_, int wave_, int lane_) : head(head_), token(token_), length(length_), wave(wave_), lane(lane_) {
    const int r = lane / kChunks;
    row_part = (uint32_t)r * (uint32_t)(token * 2);
    chunk = (uint32_t)((lane % kChunks) ^ tile_key<D>(r)) << 4;
  }
  // first: of the tile, less than length
  __device__ __forceinline__ void operator()(int first, uint32_t lds) const {
    const uint32_t to = lds + (uint32_t)(wave * kLoads * 1024);
    if (first + ROWS <= length) {
      const uint16_t* base = head + (int64_t)(first + wave * kLoads * kRows) * token;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) load(base + i * kRows * token, row_part, i, to);
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        uint32_t l = (uint32_t)lane;
        keep(l);                     // or what this needs, once for a sequence, has registers all along
        const int from = first + (wave * kLoads + i) * kRows;
        const unsigned char* at = reinterpret_cast<const unsigned char*>(head + from * token) + (l / kChunks * (uint32_t)(token * 2) + (chunk ^ key_of(i)));
        load_to_lds(from + (int)(l / kChunks) < length ? at : reinterpret_cast<const unsigned char*>(&kZeroChunk), to + (uint32_t)(i * 1024));
      }
    }
  }
  __device__ __forceinline__ uint32_t key_of(int i) const { return (uint32_t)(tile_key<D>((wave * kLoads + i) * kRows) << 4); }
  __device__ __forceinline__ void load(const uint16_t* row, uint32_t rows, int i, uint32_t to) const {
    const uint64_t at = reinterpret_cast<uint64_t>(row);
    const uint64_t base = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
    load_to_lds_base_off(reinterpret_cast<const void*>(base), rows + (chunk ^ key_of(i)), to + (uint32_t)(i * 1024));
  }
};

// 4 bytes a lane, global -> LDS at lds + lane * 4 (load_to_lds has 16).
__device__ __forceinline__ void load_word_to_lds(const void* gptr, uint32_t lds_base) {
  const uint32_t lds_addr = __builtin_amdgcn_readfirstlane(lds_base);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds_addr), "v"(gptr) : "memory", "m0");
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

// The same with the lane's part of the address, a register, apart from the offset that is an instruction's constant.
template <int D>
__device__ __forceinline__ bf16x8 read_rows_at(uint32_t lane_step, uint32_t offset) {
  typedef __attribute__((address_space(3))) const bf16x8* ptr;
  return *(ptr)(uintptr_t)(lane_step + offset);
}
template <int D>
__device__ __forceinline__ bf16x8 read_columns_at(uint32_t lane_part, uint32_t lane_part_8, uint32_t offset) {
  typedef __attribute__((address_space(3))) s16x4* ptr;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(uintptr_t)(lane_part + offset));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(uintptr_t)(lane_part_8 + offset));
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
__device__ __forceinline__ u32x4 as_words(const f32x16& x, int j) {
  u32x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = pack_bf16(x[8 * j + 2 * e], x[8 * j + 2 * e + 1]);
  return w;
}

// x of both halves of the wave: op over lanes l and l + 32.
template <class Op>
__device__ __forceinline__ float across_halves(float x, Op op) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return op(__uint_as_float(s[0]), __uint_as_float(s[1]));
}

// x of all lanes.
template <class Op>
__device__ __forceinline__ float over_wave(float x, Op op) {
  auto dpp = [](float v, auto ctrl) __attribute__((always_inline)) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false));
  };
  x = op(x, dpp(x, std::integral_constant<int, 0xB1>{}));        // quad_perm [1,0,3,2]
  x = op(x, dpp(x, std::integral_constant<int, 0x4E>{}));        // quad_perm [2,3,0,1]
  x = op(x, dpp(x, std::integral_constant<int, 0x141>{}));       // row_half_mirror
  x = op(x, dpp(x, std::integral_constant<int, 0x140>{}));       // row_mirror
  const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return across_halves(op(__uint_as_float(s[0]), __uint_as_float(s[1])), op);
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
