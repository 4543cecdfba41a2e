// Verification of drafted tokens: which of a tree's drafts stand, and the token after them, from given random numbers (the rule: include/swz_drafts.h).
//
// The tests need single probabilities, a lane for each node of the tree; only the row that the new token is drawn from is read whole.  It is cut into pieces of kPieceValues values, a workgroup each,
// which all make the tests for themselves and leave the sum of what is left of the target's probabilities in their piece; then a workgroup for each sequence finds the piece in which the sums exceed the
// random number's share, and in it the token.  Where children were drawn from a draft's probabilities and one fails that has siblings, what is left has to be summed before the next test: for trees of drawn
// children a launch before these makes the tests, a workgroup for each sequence.  Sums are 64-bit, in an order that depends on the sizes alone.
//
// What bounds it: the waits, and with many sequences the rows' bytes behind them.  Places, nodes, their probabilities and the row are loaded one after another: 16 sequences of 32000 values in bfloat16, next to no bytes,
// 4.7 us.  64 of 128000 floats, of both kinds, are 10.3 us at a copy's rate, and the sums take 15.0: every workgroup waits as long before its row's loads (pieces of 4096 values are 4 loads of 16 bytes a thread and row, all on their
// way), and all of them at the same time, while the vector unit issues for 44 % of the cycles.  The token's launch waits alike (4.9 us: sums, place in them, a piece of the row).
// Trees of drawn children: 8 sequences of 50257 floats 26 us for the tests, residuals of a row summed one after the other by a workgroup alone, whose compute unit's vector unit issues for 65 % of the cycles (512
// threads, or a division for each value: slower).  Each sum starts from the rows again and takes off all the failed children before it, so that the time goes with the square of their number: 8 trees whose root has 1, 2, 4, 8, 16, 32
// and 62 children that fail, and one more that passes, take 20, 33, 73, 202, 666, 2410 and 8650 us in all.  (The sums of a node follow from its two rows alone, whatever is drawn; they could be made for all nodes at once.)
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attention_tiles.h"

namespace swz {

constexpr int kVerifyThreads = 256, kPieceValues = 4096, kWalkThreads = 1024, kMostNodes = 64;

// What the tests of a sequence come to: the node whose row the new token is drawn from, how many drafts stand, how many (and which) of the node's children failed.
struct Walked {
  int node, accepted, failed;
  uint64_t failed_nodes;
};
struct LeftSum {
  double sum, inverse;
};
struct VerifyState {
  Walked walked;
  LeftSum sums[kMostNodes];            // drawn children: of what each failed one left
};

struct VerifyArgs {
  const void *target, *draft;
  int64_t target_pitch, draft_pitch;
  const int32_t *tokens, *parents, *cu;
  const float* uniforms;
  int32_t *accepted, *path, *token;
  int total, sequences, vocab, pieces;
  VerifyState* states;
  double* sums;                      // sequences x pieces x 2: of what is left after the last failed child, and before it
};

template <class T>
__device__ __forceinline__ double probability(const void* p, int64_t at) {
  if constexpr (sizeof(T) == 4) {
    const float x = static_cast<const float*>(p)[at];
    return x < 0.f ? 0. : (double)x;
  } else {
    const float x = __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[at] << 16);
    return x < 0.f ? 0. : (double)x;
  }
}

// 16 bytes of a row from value i on, those from `end` on 0; rows start anywhere.
template <class T>
__device__ __forceinline__ void load_values(const void* p, int64_t row, int i, int end, float (&x)[16 / sizeof(T)]) {
  constexpr int N = 16 / sizeof(T);
  const T* from = static_cast<const T*>(p) + row + i;
  T v[N];
  if (i + N <= end) {
    __builtin_memcpy(v, from, 16);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = i + e < end ? from[e] : T{};
  }
#pragma unroll
  for (int e = 0; e < N; ++e) {
    float f;
    if constexpr (sizeof(T) == 4) f = v[e];
    else f = __uint_as_float((uint32_t)v[e] << 16);
    x[e] = f < 0.f ? 0.f : f;
  }
}

// What a failed child leaves of p, but for the division by its sum.
__device__ __forceinline__ double take(double p, double q) {
  const double d = p - q;
  return d < 0. ? 0. : d;            // (NaN stays)
}
// d / sum: with the rounded reciprocal of the sum a quotient that its remainder corrects is the rounded one (Markstein), at three instructions instead of the division's dozen.
__device__ __forceinline__ LeftSum left_sum(double sum) { return {sum, 1. / sum}; }
// What is left of values p after `failed` children failed.
template <int N>
__device__ __forceinline__ void leave(double (&p)[N], const double (&q)[N], int failed, const LeftSum* sums) {
#pragma unroll 1
  for (int i = 0; i < failed; ++i) {
    const LeftSum s = sums[i];
    if (!(s.sum > 0.)) continue;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const double d = take(p[e], q[e]), quotient = d * s.inverse;
      p[e] = __builtin_fma(__builtin_fma(-quotient, s.sum, d), s.inverse, quotient);
    }
  }
}
__device__ __forceinline__ double left_of(double p, double q, int failed, const LeftSum* sums) {
  double x[1] = {p};
  const double y[1] = {q};
  leave<1>(x, y, failed, sums);
  return x[0];
}

__device__ __forceinline__ double lane_value(double x, int lane) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(b >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)b, lane));
}
// x of another lane of the wave, 0 where there is none.
template <int CTRL, int ROWS>
__device__ __forceinline__ double from_lane(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t low = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, CTRL, ROWS, 0xf, false), high = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}
// Sum of x over this lane and those before it.
__device__ __forceinline__ double sum_with(double x) {
  x += from_lane<0x111, 0xf>(x);     // row_shr:1, 2, 4, 8
  x += from_lane<0x112, 0xf>(x);
  x += from_lane<0x114, 0xf>(x);
  x += from_lane<0x118, 0xf>(x);
  x += from_lane<0x142, 0xa>(x);     // row_bcast:15, to rows 1 and 3
  x += from_lane<0x143, 0xc>(x);     // row_bcast:31, to rows 2 and 3
  return x;
}
__device__ __forceinline__ double add_over_wave(double x) { return lane_value(sum_with(x), 63); }

// A sequence's tests, all lanes alike; a lane has a node.
struct Nodes {
  int first, count;                  // tokens of the call; of the block, at most kMostNodes
  int token, parent;
  double uniform, p, q;              // of the token under the parent
  bool real;
};
template <class T, bool DRAWN>
__device__ __forceinline__ Nodes load_nodes(const VerifyArgs& a, int sequence) {
  const int lane = threadIdx.x & 63;
  const Span t = sequence_span(a.cu, sequence, a.total);
  Nodes n{};
  n.first = t.first;
  n.count = min(t.length, kMostNodes);
  n.token = n.parent = -1;
  if (lane > 0 && lane < n.count) {
    n.token = a.tokens[t.first + lane];
    n.parent = a.parents == nullptr ? lane - 1 : a.parents[t.first + lane];
    n.uniform = (double)a.uniforms[t.first + lane];
    n.real = n.token >= 0 && n.token < a.vocab && n.parent >= 0 && n.parent < lane;
  }
  if (n.real) {
    n.p = probability<T>(a.target, (t.first + n.parent) * a.target_pitch + n.token);
    if constexpr (DRAWN) n.q = probability<T>(a.draft, (t.first + n.parent) * a.draft_pitch + n.token);
  }
  return n;
}
// sum_left(node, failed): the sum of what is left of the node's row after that many failed children (drawn ones only), needed where another one is tested.
// The lane's entry of the path is returned in *path.
// SIBLINGS: a node may have more than one child.
template <bool DRAWN, bool SIBLINGS, class F>
__device__ __forceinline__ Walked walk(const Nodes& n, LeftSum* sums, int* path, F&& sum_left) {
  const int lane = threadIdx.x & 63;
  Walked s{};
  *path = lane == 0 ? 0 : -1;
  double mass = 1.;
  int at = 0;                        // the last node that was tested
  while (true) {
    const uint64_t children = __ballot(n.real && n.parent == s.node && lane > at);
    if (children == 0) break;
    at = __ffsll((unsigned long long)children) - 1;
    const double u = lane_value(n.uniform, at), p = lane_value(n.p, at);
    bool good;
    if constexpr (DRAWN) {
      const double q = lane_value(n.q, at);
      if constexpr (SIBLINGS) {
        if (s.failed > 0) sums[s.failed - 1] = left_sum(sum_left(s.node, s.failed));
        good = u * q < left_of(p, q, s.failed, sums);
      } else {
        good = u * q < p;
      }
    } else {
      const int token = __builtin_amdgcn_readlane(n.token, at);
      const double mine = __ballot(n.token == token && (s.failed_nodes >> lane & 1)) != 0 ? 0. : p, least = u * mass;
      good = mine > 0. && mine > least;                      // (a NaN on either side: no)
      if (!good) mass -= mine;
    }
    if (good) {
      s.node = at;
      ++s.accepted;
      s.failed = 0;
      s.failed_nodes = 0;
      mass = 1.;
      if (lane == s.accepted) *path = at;
    } else {
      ++s.failed;
      s.failed_nodes |= 1ull << at;
      if constexpr (!SIBLINGS) break;
    }
  }
  return s;
}

// The results but for the new token.
__device__ __forceinline__ void store_walk(const VerifyArgs& a, int sequence, const Nodes& n, const Walked& s, int path) {
  const int lane = threadIdx.x & 63;
  const Span t = sequence_span(a.cu, sequence, a.total);
  if (lane == 0) a.accepted[sequence] = s.accepted;
  for (int i = lane; i < t.length; i += 64) a.path[t.first + i] = i < 64 ? path : -1;
}

// Trees of drawn children: a workgroup makes the tests of a sequence.
template <class T>
__global__ void __launch_bounds__(kWalkThreads) verify_walk_kernel(VerifyArgs a) {
  constexpr int N = 16 / sizeof(T), kWaves = kWalkThreads / 64;
  __shared__ LeftSum sums[kMostNodes];
  __shared__ double parts[kWaves];
  const int sequence = (int)blockIdx.x, lane = threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  const Nodes n = load_nodes<T, true>(a, sequence);
  int path;
  const Walked s = walk<true, true>(n, sums, &path, [&](int node, int failed) {
    const int64_t p_row = (int64_t)(n.first + node) * a.target_pitch, q_row = (int64_t)(n.first + node) * a.draft_pitch;
    constexpr int kRounds = 8 / N, kStride = kRounds * kWalkThreads * N;     // the next rounds' loads are on their way while these are added up
    float p[2][kRounds][N], q[2][kRounds][N];
    auto load = [&](int to, int i) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < kRounds; ++j) {
        load_values<T>(a.target, p_row, i + j * kWalkThreads * N, a.vocab, p[to][j]);
        load_values<T>(a.draft, q_row, i + j * kWalkThreads * N, a.vocab, q[to][j]);
      }
    };
    double more[2] = {0., 0.};
    auto add = [&](int from) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < kRounds; ++j) {
        double x[N], y[N];
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = (double)p[from][j][e], y[e] = (double)q[from][j][e];
        leave<N>(x, y, failed - 1, sums);
#pragma unroll
        for (int e = 0; e < N; ++e) more[e % 2] += take(x[e], y[e]);
      }
    };
    const int first = (int)threadIdx.x * N;
    load(0, first);
#pragma unroll 1
    for (int64_t i = 0; i < a.vocab; i += 2 * kStride) {
      load(1, (int)min(i + kStride + first, (int64_t)a.vocab));
      add(0);
      load(0, (int)min(i + 2 * kStride + first, (int64_t)a.vocab));
      add(1);
    }
    double sum = more[0] + more[1];
    sum = add_over_wave(sum);
    __syncthreads();                                         // what was there has been read
    if (lane == 0) parts[wave] = sum;
    __syncthreads();
    sum = 0.;
    for (int w = 0; w < kWaves; ++w) sum += parts[w];
    return sum;
  });
  __syncthreads();
  VerifyState* to = a.states + sequence;
  if (threadIdx.x < kMostNodes) to->sums[threadIdx.x] = (int)threadIdx.x < s.failed - 1 ? sums[threadIdx.x] : LeftSum{0., 0.};
  if (wave == 0) {
    if (lane == 0) to->walked = s;
    store_walk(a, sequence, n, s, path);
  }
}

// Values of the row that the new token is drawn from: what is left after the last failed child, and before it.
template <bool DRAWN, int N>
__device__ __forceinline__ void left_at(const float (&p)[N], const float (&q)[N], const Walked& s, const LeftSum* sums, double (&now)[N], double (&before)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) now[e] = before[e] = (double)p[e];
  if constexpr (DRAWN) {
    if (s.failed == 0) return;
    double y[N];
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = (double)q[e];
    leave<N>(before, y, s.failed - 1, sums);
#pragma unroll
    for (int e = 0; e < N; ++e) now[e] = take(before[e], y[e]);
  }
}
// Whether token x is that of a failed child (points).
template <int N>
__device__ __forceinline__ void drop_failed(const VerifyArgs& a, int first, uint64_t failed, int i, float (&p)[N]) {
  while (failed != 0) {
    const int at = a.tokens[first + __ffsll((unsigned long long)failed) - 1] - i;
    failed &= failed - 1;
#pragma unroll
    for (int e = 0; e < N; ++e) p[e] = at == e ? 0.f : p[e];
  }
}

// WALKED: the tests have been made.
template <class T, bool DRAWN, bool WALKED>
__global__ void __launch_bounds__(kVerifyThreads) verify_sums_kernel(VerifyArgs a) {
  constexpr int N = 16 / sizeof(T), kTurns = kPieceValues / (kVerifyThreads * N);
  __shared__ double parts[kVerifyThreads / 64][2];
  const int sequence = (int)blockIdx.x / a.pieces, piece = (int)blockIdx.x - sequence * a.pieces, lane = threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  const Span t = sequence_span(a.cu, sequence, a.total);
  VerifyState* state = a.states + sequence;
  Walked s;
  if constexpr (WALKED) {
    s = state->walked;
  } else {
    const Nodes n = load_nodes<T, DRAWN>(a, sequence);
    int path;
    s = walk<DRAWN, !DRAWN>(n, nullptr, &path, [](int, int) { return 0.; });         // drawn children: of a chain
    if (piece == 0 && wave == 0) {
      if (lane == 0) state->walked = s;
      store_walk(a, sequence, n, s, path);
    }
  }
  if (t.length == 0) return;
  const int64_t p_row = (int64_t)(t.first + s.node) * a.target_pitch, q_row = (int64_t)(t.first + s.node) * a.draft_pitch;
  float p[kTurns][N], q[kTurns][N];
  const int first = piece * kPieceValues + (int)threadIdx.x * N;
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    load_values<T>(a.target, p_row, first + i * kVerifyThreads * N, a.vocab, p[i]);
    if (DRAWN && s.failed > 0) load_values<T>(a.draft, q_row, first + i * kVerifyThreads * N, a.vocab, q[i]);
  }
  double now = 0., before = 0.;
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    if constexpr (!DRAWN) drop_failed<N>(a, t.first, s.failed_nodes, first + i * kVerifyThreads * N, p[i]);
    double x[N], y[N];
    left_at<DRAWN, N>(p[i], q[i], s, state->sums, x, y);
#pragma unroll
    for (int e = 0; e < N; ++e) now += x[e], before += y[e];
  }
  now = add_over_wave(now);
  before = add_over_wave(before);
  if (lane == 0) parts[wave][0] = now, parts[wave][1] = before;
  __syncthreads();
  if (threadIdx.x < 2) {
    double sum = 0.;
#pragma unroll
    for (int w = 0; w < kVerifyThreads / 64; ++w) sum += parts[w][threadIdx.x];
    a.sums[((int64_t)sequence * a.pieces + piece) * 2 + threadIdx.x] = sum;
  }
}

// Numbers that are not negative, `mine` for each thread of a workgroup: the sum of those of the threads before it, and of all.
struct Before {
  double before, all;
};
__device__ __forceinline__ Before sum_before_threads(double mine, double (&waves)[kVerifyThreads / 64]) {
  const int lane = threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  const double with = sum_with(mine), before = from_lane<0x138, 0xf>(with);      // wave_shr:1
  if (lane == 63) waves[wave] = with;
  __syncthreads();
  double first = 0., all = 0.;
#pragma unroll
  for (int w = 0; w < kVerifyThreads / 64; ++w) {
    first = w < wave ? first + waves[w] : first;
    all += waves[w];
  }
  return {first + before, all};
}

// The first of a workgroup's numbers (N for each thread, from `first` on) with which their sum exceeds r, and the sum before it; where there is none (rounding may leave none at the very end of a piece) the last one above 0,
// and infinity.
struct Share {
  int at;
  double before;
};
struct WaveShare {
  int found, last;
  double before;
};
template <int N>
__device__ __forceinline__ Share find_share(const double (&x)[N], double before, int first, double r, WaveShare (&waves)[kVerifyThreads / 64]) {
  const int lane = threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  int at = -1, above = -1;
  double sum = before, at_before = 0.;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (x[i] > 0.) above = first + i;
    if (at < 0 && x[i] > 0. && sum + x[i] > r) at = first + i, at_before = sum;
    sum += x[i];
  }
  // a wave's first is its first lane's that has one
  const uint64_t found = __ballot(at >= 0), some = __ballot(above >= 0);
  const int its = found != 0 ? __ffsll((unsigned long long)found) - 1 : 0, last = some != 0 ? 63 - __clzll((unsigned long long)some) : 0;
  if (lane == its) waves[wave].found = at, waves[wave].before = at_before;
  if (lane == last) waves[wave].last = above;
  __syncthreads();
  Share s = {-1, INFINITY};
#pragma unroll
  for (int w = kVerifyThreads / 64 - 1; w >= 0; --w)
    if (waves[w].found >= 0) s = {waves[w].found, waves[w].before};
  if (s.at < 0)
#pragma unroll
    for (int w = 0; w < kVerifyThreads / 64; ++w) s.at = waves[w].last >= 0 ? waves[w].last : s.at;
  return s;
}

// COUNT consecutive values of a row (a multiple of 16 bytes of them) as numbers, those from `end` on 0.
template <class T, int COUNT>
__device__ __forceinline__ void load_run(const void* p, int64_t row, int i, int end, float (&x)[COUNT]) {
  constexpr int N = 16 / sizeof(T);
#pragma unroll
  for (int j = 0; j < COUNT; j += N) {
    float v[N];
    load_values<T>(p, row, i + j, end, v);
#pragma unroll
    for (int e = 0; e < N; ++e) x[j + e] = v[e];
  }
}

template <class T, bool DRAWN>
__global__ void __launch_bounds__(kVerifyThreads) verify_token_kernel(VerifyArgs a) {
  constexpr int kPer = kPieceValues / kVerifyThreads;
  __shared__ double waves[3][kVerifyThreads / 64];
  __shared__ WaveShare shares[2][kVerifyThreads / 64];
  const int sequence = (int)blockIdx.x;
  const Span t = sequence_span(a.cu, sequence, a.total);
  if (t.length == 0) {
    if (threadIdx.x == 0) a.token[sequence] = -1;
    return;
  }
  const VerifyState* state = a.states + sequence;
  const double* sums = a.sums + (int64_t)sequence * a.pieces * 2;
  // a thread's pieces: one, where there are no more pieces than threads
  const int per = (a.pieces + kVerifyThreads - 1) / kVerifyThreads, first_piece = (int)threadIdx.x * per, end_piece = min(first_piece + per, a.pieces);
  double now = 0., was = 0.;
  for (int i = first_piece; i < end_piece; ++i) now += sums[2 * i], was += sums[2 * i + 1];
  const Walked s = state->walked;
  const double u = (double)a.uniforms[t.first];
  Before b = sum_before_threads(now, waves[0]);
  const bool before = DRAWN && s.failed > 0 && !(b.all > 0.); // the last failed child left nothing: what there was before it
  if (before) {
    b = sum_before_threads(was, waves[1]);
    now = was;
  }
  if (!(b.all > 0.) || !(b.all < INFINITY)) {
    if (threadIdx.x == 0) a.token[sequence] = -1;
    return;
  }
  double r = u * b.all;
  const double mine[1] = {now};
  const Share found = find_share<1>(mine, b.before, (int)threadIdx.x, r, shares[0]);
  const int thread = found.at;
  r = found.before < INFINITY ? r - found.before : INFINITY;
  int piece = thread * per;
  if (per > 1) {                     // of the thread's pieces
    int last = piece;
    for (const int end = min(piece + per, a.pieces); piece < end; ++piece) {
      const double x = sums[2 * piece + (before ? 1 : 0)];
      if (x > r) break;
      last = x > 0. ? piece : last;
      r -= x;
      if (piece + 1 == end) {
        piece = last;
        r = INFINITY;
        break;
      }
    }
  }
  const int64_t p_row = (int64_t)(t.first + s.node) * a.target_pitch, q_row = (int64_t)(t.first + s.node) * a.draft_pitch;
  const int first = piece * kPieceValues + (int)threadIdx.x * kPer;
  float p[kPer], q[kPer];
  load_run<T, kPer>(a.target, p_row, first, a.vocab, p);
  if (DRAWN && s.failed > 0) load_run<T, kPer>(a.draft, q_row, first, a.vocab, q);
  if constexpr (!DRAWN) drop_failed<kPer>(a, t.first, s.failed_nodes, first, p);
  double x[kPer], y[kPer], sum = 0.;
  left_at<DRAWN, kPer>(p, q, s, state->sums, x, y);
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    x[e] = before ? y[e] : x[e];
    sum += x[e];
  }
  const Before c = sum_before_threads(sum, waves[2]);
  const Share token = find_share<kPer>(x, c.before, first, r, shares[1]);
  if (threadIdx.x == 0) a.token[sequence] = token.at;
}

}  // namespace swz
