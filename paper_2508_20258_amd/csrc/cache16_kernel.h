// A cache of keys and values in bfloat16: appending to it with the rotation on the way, and keeping an accepted path.
#pragma once

#include "attention_tiles.h"
#include "paged.h"

namespace swz {

// Which sequence owns a token: the last one that starts at it or before, if it has not ended.  Wave-uniform; sequence -1: none.
struct TokenPlace {
  int sequence, place, before;       // place in the sequence's block; what `before` holds for the sequence
};
__device__ __forceinline__ TokenPlace find_token(const int32_t* cu, const int32_t* before, int sequences, int total, int token) {
  if (sequences <= 64) {             // one round of loads
    const int at = min((int)(threadIdx.x & 63), sequences - 1);
    const int from = clamp_to(cu[at], 0, total), to = clamp_to(cu[at + 1], 0, total), mine = before[at];
    const uint64_t found = __ballot((int)(threadIdx.x & 63) < sequences && from <= token && token < to);
    if (found == 0) return {-1, 0, 0};
    const int s = 63 - __clzll((unsigned long long)found);
    return {s, token - __builtin_amdgcn_readlane(from, s), __builtin_amdgcn_readlane(mine, s)};
  }
  const SlotPlace p = find_slot<0>(cu, sequences, total, 1, token);
  const Span t = sequence_span(cu, p.sequence, total);
  if (token < t.first || token >= t.first + t.length) return {-1, 0, 0};
  return {p.sequence, token - t.first, __builtin_amdgcn_readfirstlane(before[p.sequence])};
}

struct Append16Args {
  PageTable c;
  uint16_t *k_pages, *v_pages;
  Heads q, k, v, q_out;
  const float *cos, *sin;
  const int32_t *positions, *cu, *before;
  int64_t table_rows;
  int total, sequences, q_heads, rotary, splits;   // rotary 0: nothing is turned
};

constexpr int kAppendThreads = 256, kAppendAhead = 3;

// HBM is the bound where tokens are many: 32768 of 32 + 8 + 8 heads of 128 in 139 us, 5.9 TB/s, in streaming loads and stores (159 without them), which are slower where all fits the memory-side cache (8192 tokens
// of 8 + 8 heads, 67 MB: 17.8 us, and 12.8 with regular ones).  A step's few tokens take 3.6 us, three loads one after another.
//
// A wave for each token, or for each of `splits` parts of its heads (queries, then keys, then values): 64 / kLanes heads at a time, 16 dimensions a lane.  The lane's two chunks of 8 hold both halves of its pairs: c and
// c + rotary / 16 of those that are turned, neighbours of the others.
template <int D, bool INTERLEAVED, bool STREAM>
__global__ void __launch_bounds__(kAppendThreads) cache16_append_kernel(Append16Args a) {
  constexpr int kLanes = D / 16, kHeads = 64 / kLanes;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int64_t id = (int64_t)blockIdx.x * (kAppendThreads / 64) + wave;
  const int token = (int)(id / a.splits), split = (int)(id - (int64_t)token * a.splits);
  if (token >= a.total) return;
  const int l = lane % kLanes, mine = lane / kLanes, heads = a.q_heads + 2 * a.c.k_heads;
  const bool turned = l < a.rotary / 16;
  const int d0 = 8 * (turned ? l : 2 * l), d1 = turned ? d0 + a.rotary / 2 : d0 + 8;

  const TokenPlace place = find_token(a.cu, a.before, a.sequences, a.total, token);
  if (place.sequence < 0) return;
  const int64_t position = (int64_t)place.before + place.place;
  const bool cached = place.before >= 0 && position < ((int64_t)a.c.table_width << a.c.page_shift);
  const int page = cached ? a.c.page_of(place.sequence, (int)position) : -1;

  f32x4 c[2] = {1.f, 1.f}, s[2] = {0.f, 0.f};
  if (turned) {
    const int64_t row = a.positions != nullptr ? (int64_t)a.positions[token] : position;
    c[0] = c[1] = __builtin_nanf("");
    if (row >= 0 && row < a.table_rows) {
      const float *cos = a.cos + row * (a.rotary / 2), *sin = a.sin + row * (a.rotary / 2);
      const int first = INTERLEAVED ? d0 / 2 : d0, second = INTERLEAVED ? d1 / 2 : d0 + 4;
      c[0] = *reinterpret_cast<const f32x4*>(cos + first), c[1] = *reinterpret_cast<const f32x4*>(cos + second);
      s[0] = *reinterpret_cast<const f32x4*>(sin + first), s[1] = *reinterpret_cast<const f32x4*>(sin + second);
    }
  }
  // kAppendAhead turns' loads are on their way together
  for (int first = split * kHeads + mine; first < heads; first += kAppendAhead * a.splits * kHeads) {
    u32x4 x[kAppendAhead], y[kAppendAhead];
#pragma unroll
    for (int i = 0; i < kAppendAhead; ++i) {
      const int head = min(first + i * a.splits * kHeads, heads - 1), k_head = head - a.q_heads, v_head = k_head - a.c.k_heads;
      const uint16_t* from = k_head < 0 ? a.q.at(token, head) : v_head < 0 ? a.k.at(token, k_head) : a.v.at(token, v_head);
      auto load = [](const uint16_t* p) { return STREAM ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)) : *reinterpret_cast<const u32x4*>(p); };
      x[i] = load(from + d0);
      y[i] = load(from + d1);
    }
#pragma unroll
    for (int i = 0; i < kAppendAhead; ++i) {
      const int head = first + i * a.splits * kHeads, k_head = head - a.q_heads, v_head = k_head - a.c.k_heads;
      if (head >= heads) break;
      if (turned && v_head < 0) {
        float p[8], q[8];
        unpack8(x[i], p);
        unpack8(y[i], q);
        if constexpr (INTERLEAVED) {
          auto turn = [&](float (&z)[8], const f32x4& c, const f32x4& s) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float u = z[2 * e], w = z[2 * e + 1];
              z[2 * e] = u * c[e] - w * s[e];
              z[2 * e + 1] = w * c[e] + u * s[e];
            }
          };
          turn(p, c[0], s[0]);
          turn(q, c[1], s[1]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float u = p[e], w = q[e], cosine = c[e / 4][e % 4], sine = s[e / 4][e % 4];
            p[e] = u * cosine - w * sine;
            q[e] = w * cosine + u * sine;
          }
        }
        x[i] = pack8(p);
        y[i] = pack8(q);
      }
      uint16_t* to = nullptr;
      if (k_head < 0) to = a.q_out.at(token, head);
      else if (page >= 0) to = v_head < 0 ? a.k_pages + a.c.token_at(page, k_head, (int)position) * D : a.v_pages + a.c.token_at(page, v_head, (int)position) * D;
      if (to != nullptr) {
        if constexpr (STREAM) {
          __builtin_nontemporal_store(x[i], reinterpret_cast<u32x4*>(to + d0));
          __builtin_nontemporal_store(y[i], reinterpret_cast<u32x4*>(to + d1));
        } else {
          *reinterpret_cast<u32x4*>(to + d0) = x[i];
          *reinterpret_cast<u32x4*>(to + d1) = y[i];
        }
      }
    }
  }
}

struct Keep16Args {
  PageTable c;
  uint16_t *k_pages, *v_pages;
  const int32_t *cu, *before, *path, *accepted;
  int total, sequences, blocks;      // workgroups of a sequence
};

constexpr int kKeepThreads = 256, kKeepAhead = 8;

// A thread for 8 dimensions of a key head's keys or values, which it moves in the path's order, kKeepAhead tokens at a time: a path rises, so a token that is written (to place i) is not the
// source of a later one (path[j] >= j > i).
// The waits bound it: a table of sources and targets for 64 tokens (three loads one after another), then the move.  16 blocks of 16 tokens 3.1 us, 128 of 64 with 8 heads of 128 3.7.
template <int D>
__global__ void __launch_bounds__(kKeepThreads) cache16_keep_kernel(Keep16Args a) {
  __shared__ int64_t from[64], to[64];                       // tokens of the cache before them, for head 0; -1: not moved
  const int sequence = (int)blockIdx.x / a.blocks, lane = threadIdx.x & 63;
  const Span t = sequence_span(a.cu, sequence, a.total);
  const int count = min(__builtin_amdgcn_readfirstlane(a.accepted[sequence]), t.length - 1), before = __builtin_amdgcn_readfirstlane(a.before[sequence]);
  if (before < 0) return;
  const int64_t last = (int64_t)a.c.table_width << a.c.page_shift;
  const int item = ((int)blockIdx.x - sequence * a.blocks) * kKeepThreads + (int)threadIdx.x, head = item / (2 * (D / 8)), chunk = item % (2 * (D / 8));
  uint16_t* pages = (chunk < D / 8 ? a.k_pages : a.v_pages) + ((int64_t)min(head, a.c.k_heads - 1) << a.c.page_shift) * D + chunk % (D / 8) * 8;
  for (int first = 1; first <= count; first += 64) {
    __syncthreads();
    if (threadIdx.x < 64) {
      const int i = first + lane;
      int64_t source = -1, target = -1;
      if (i <= count) {
        const int node = a.path[t.first + i];
        const int64_t at = (int64_t)before + node, there = (int64_t)before + i;
        if (node != i && node >= 0 && node < t.length && at < last && there < last) {
          const int p = a.c.page_of(sequence, (int)at), q = a.c.page_of(sequence, (int)there);
          if (p >= 0 && q >= 0) source = a.c.token_at(p, 0, (int)at), target = a.c.token_at(q, 0, (int)there);
        }
      }
      from[lane] = source;
      to[lane] = target;
    }
    __syncthreads();
    if (head >= a.c.k_heads) continue;
    for (int i = 0; i < min(64, count - first + 1); i += kKeepAhead) {
      u32x4 x[kKeepAhead];
#pragma unroll
      for (int e = 0; e < kKeepAhead; ++e)
        if (from[i + e] >= 0) x[e] = *reinterpret_cast<const u32x4*>(pages + from[i + e] * D);
#pragma unroll
      for (int e = 0; e < kKeepAhead; ++e)
        if (from[i + e] >= 0) *reinterpret_cast<u32x4*>(pages + to[i + e] * D) = x[e];
    }
  }
}

}  // namespace swz
