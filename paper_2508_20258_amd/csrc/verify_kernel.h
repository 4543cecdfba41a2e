// Verification of drafted tokens: which of a tree's drafts stand, and the token after them, from given random numbers (the rule: include/swz_drafts.h).
//
// The tests need single probabilities, a lane for each node of the tree; only the row that the new token is drawn from is read whole.  It is cut into pieces of kPieceValues values, a workgroup each,
// which all make the tests for themselves and leave the sum of what is left of the target's probabilities in their piece; then a workgroup for each sequence finds the piece in which the sums exceed the
// random number's share, and in it the token.  Where children were drawn from a draft's probabilities and one fails that has siblings, what is left has to be summed before the next test: for trees of drawn
// children a launch before these makes the tests, a workgroup for each sequence.  Sums are 64-bit, in an order that depends on the sizes alone.
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
struct VerifyState {
  Walked walked;
  double sums[kMostNodes];           // drawn children: of what each failed one left
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

// What is left of p after `failed` children failed, but for the last division.
__device__ __forceinline__ double take(double p, double q) {
  const double d = p - q;
  return d < 0. ? 0. : d;            // (NaN stays)
}
__device__ __forceinline__ double left_of(double p, double q, int failed, const double* sums) {
  for (int i = 0; i < failed; ++i) {
    const double d = take(p, q);
    p = sums[i] > 0. ? d / sums[i] : p;
  }
  return p;
}

__device__ __forceinline__ double add_over_wave(double x) {
#pragma unroll
  for (int by = 1; by < 64; by *= 2) x += __shfl_xor(x, by);
  return x;
}

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
__device__ __forceinline__ double lane_value(double x, int lane) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(b >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)b, lane));
}

// sum_left(node, failed): the sum of what is left of the node's row after that many failed children (drawn ones only), needed where another one is tested.
// The lane's entry of the path is returned in *path.
template <bool DRAWN, class F>
__device__ __forceinline__ Walked walk(const Nodes& n, double* sums, int* path, F&& sum_left) {
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
      if (s.failed > 0) sums[s.failed - 1] = sum_left(s.node, s.failed);
      const double q = lane_value(n.q, at);
      good = u * q < left_of(p, q, s.failed, sums);
    } else {
      const int token = __builtin_amdgcn_readlane(n.token, at);
      const double mine = __ballot(n.token == token && (s.failed_nodes >> lane & 1)) != 0 ? 0. : p, least = u * mass;
      good = mine > (least > 0. ? least : 0.);
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
  __shared__ double sums[kMostNodes], parts[kWaves];
  const int sequence = (int)blockIdx.x, lane = threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  const Nodes n = load_nodes<T, true>(a, sequence);
  int path;
  const Walked s = walk<true>(n, sums, &path, [&](int node, int failed) {
    const int64_t p_row = (int64_t)(n.first + node) * a.target_pitch, q_row = (int64_t)(n.first + node) * a.draft_pitch;
    double sum = 0.;
#pragma unroll 2
    for (int i = (int)threadIdx.x * N; i < a.vocab; i += kWalkThreads * N) {
      float p[N], q[N];
      load_values<T>(a.target, p_row, i, a.vocab, p);
      load_values<T>(a.draft, q_row, i, a.vocab, q);
#pragma unroll
      for (int e = 0; e < N; ++e) sum += take(left_of((double)p[e], (double)q[e], failed - 1, sums), (double)q[e]);
    }
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
  if (threadIdx.x < kMostNodes) to->sums[threadIdx.x] = (int)threadIdx.x < s.failed - 1 ? sums[threadIdx.x] : 0.;
  if (wave == 0) {
    if (lane == 0) to->walked = s;
    store_walk(a, sequence, n, s, path);
  }
}

// Value i of the row that the new token is drawn from: what is left after the last failed child, and before it.
struct Left {
  double now, before;
};
template <bool DRAWN>
__device__ __forceinline__ Left left_at(double p, double q, const Walked& s, const double* sums) {
  if constexpr (DRAWN) {
    if (s.failed == 0) return {p, p};
    const double before = left_of(p, q, s.failed - 1, sums);
    return {take(before, q), before};
  }
  return {p, p};
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
    double none[1] = {0.};                                   // a chain: no node has a second child
    s = walk<DRAWN>(n, none, &path, [](int, int) { return 0.; });
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
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const Left x = left_at<DRAWN>((double)p[i][e], (double)q[i][e], s, state->sums);
      now += x.now;
      before += x.before;
    }
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

// The first of `count` numbers (value(i), not negative) with which their sum exceeds r, and the sum before it; -1: none.  The last one above 0 goes to *last.  A thread has `per` neighbours of
// kVerifyThreads * per >= count; all threads return the same.
struct Found {
  int at;
  double before;
};
template <class F>
__device__ __forceinline__ Found find_share(int count, int per, double r, int* last, double* total, F&& value) {
  __shared__ double waves[kVerifyThreads / 64], found_before;
  __shared__ int found_at, last_at;
  const int lane = threadIdx.x & 63, wave = (int)threadIdx.x >> 6, first = (int)threadIdx.x * per, end = min(first + per, count);
  double mine = 0.;
  int above = -1;
  for (int i = first; i < end; ++i) {
    const double x = value(i);
    mine += x;
    above = x > 0. ? i : above;
  }
  double with = mine;                // of this thread and those of its wave before it
#pragma unroll
  for (int by = 1; by < 64; by *= 2) {
    const double other = __shfl_up(with, by);
    if (lane >= by) with += other;
  }
  double without = __shfl_up(with, 1);
  without = lane > 0 ? without : 0.;
  __syncthreads();
  if (lane == 63) waves[wave] = with;
  if (threadIdx.x == 0) found_at = 0x7fffffff, last_at = -1;
  __syncthreads();
  double before = 0., all = 0.;
#pragma unroll
  for (int w = 0; w < kVerifyThreads / 64; ++w) {
    before = w < wave ? before + waves[w] : before;
    all += waves[w];
  }
  before += without;
  *total = all;
  if (above >= 0) atomicMax(&last_at, above);
  // rounding may leave sums that do not rise from thread to thread, by parts in 10^16: the first that exceeds counts
  double sum = before;
  int at = 0x7fffffff;
  double at_before = 0.;
  for (int i = first; i < end; ++i) {
    const double x = value(i);
    if (at == 0x7fffffff && sum + x > r && x > 0.) at = i, at_before = sum;
    sum += x;
  }
  if (at != 0x7fffffff) atomicMin(&found_at, at);
  __syncthreads();
  if (at != 0x7fffffff && at == found_at) found_before = at_before;
  __syncthreads();
  *last = last_at;
  const Found f = {found_at == 0x7fffffff ? -1 : found_at, found_before};
  return f;
}

template <class T, bool DRAWN>
__global__ void __launch_bounds__(kVerifyThreads) verify_token_kernel(VerifyArgs a) {
  constexpr int kPer = kPieceValues / kVerifyThreads;
  const int sequence = (int)blockIdx.x;
  const Span t = sequence_span(a.cu, sequence, a.total);
  if (t.length == 0) {
    if (threadIdx.x == 0) a.token[sequence] = -1;
    return;
  }
  const VerifyState* state = a.states + sequence;
  const Walked s = state->walked;
  const double* sums = a.sums + (int64_t)sequence * a.pieces * 2;
  const double u = (double)a.uniforms[t.first];
  int last;
  double total;
  const int per = (a.pieces + kVerifyThreads - 1) / kVerifyThreads;
  bool before = false;               // the last failed child left nothing: what there was before it
  find_share(a.pieces, per, 0., &last, &total, [&](int i) { return sums[2 * i]; });
  if (DRAWN && s.failed > 0 && !(total > 0.) && total == total) {
    before = true;
    find_share(a.pieces, per, 0., &last, &total, [&](int i) { return sums[2 * i + 1]; });
  }
  if (!(total > 0.) || !(total < INFINITY)) {
    if (threadIdx.x == 0) a.token[sequence] = -1;
    return;
  }
  double r = u * total;
  Found f = find_share(a.pieces, per, r, &last, &total, [&](int i) { return sums[2 * i + (before ? 1 : 0)]; });
  const int piece = f.at < 0 ? last : f.at;
  r = f.at < 0 ? INFINITY : r - f.before;
  const int64_t p_row = (int64_t)(t.first + s.node) * a.target_pitch, q_row = (int64_t)(t.first + s.node) * a.draft_pitch;
  const int start = piece * kPieceValues, count = min(kPieceValues, a.vocab - start);
  f = find_share(count, kPer, r, &last, &total, [&](int i) {
    float p[1] = {(float)probability<T>(a.target, p_row + start + i)};
    double q = 0.;
    if constexpr (DRAWN) q = s.failed > 0 ? probability<T>(a.draft, q_row + start + i) : 0.;
    else drop_failed<1>(a, t.first, s.failed_nodes, start + i, p);
    const Left x = left_at<DRAWN>((double)p[0], q, s, state->sums);
    return before ? x.before : x.now;
  });
  if (threadIdx.x == 0) a.token[sequence] = start + (f.at < 0 ? last : f.at);
}

}  // namespace swz
