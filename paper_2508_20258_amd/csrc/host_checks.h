// What the entry points of attention layers check and choose alike.  Host code only.
#pragma once

#include <stdint.h>

#include <type_traits>

#include "../../include/swz_attention.h"
#include "attention_tiles.h"
#include "launch.h"

namespace swz::host {

constexpr int64_t kTokens = (int64_t)1 << 31;      // fewer than these
constexpr int64_t kMostKeys = kTokens - 4096;      // of what is looked at (and looks): tiles and steps past the last one are 32-bit numbers too, and so is the sum of the steps of 64 sequences
constexpr int kMostHeads = 65536;

inline Heads device_heads(const swz_heads& h) { return {static_cast<uint16_t*>(h.data), h.token, h.head}; }

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Heads that a call reads or writes: there, aligned, and distances that keep 16-byte pieces aligned.
inline int check_heads(const swz_heads& h) {
  if (h.data == nullptr || h.token < 0 || h.head < 0) return SWZ_ERR_INVALID_ARG;
  return aligned(h.data, 16) && h.token % 8 == 0 && h.head % 8 == 0 ? SWZ_OK : SWZ_ERR_UNSUPPORTED;
}
template <class... H>
int check_heads(const swz_heads& h, const H&... more) {
  const int st = check_heads(h);
  return st != SWZ_OK ? st : check_heads(more...);
}

inline bool head_dim_ok(int d) { return d == 64 || d == 128; }

// f(integral_constant<int, D>) for the two sizes of a head.
template <class F>
auto for_head_dim(int d, F&& f) {
  return d == 128 ? f(std::integral_constant<int, 128>{}) : f(std::integral_constant<int, 64>{});
}
template <class F>
int for_flag(bool flag, F&& f) {
  return flag ? f(std::true_type{}) : f(std::false_type{});
}

inline int compute_units() {
  DeviceFacts f;
  return query_device(&f) == SWZ_OK && f.cus > 0 ? f.cus : kWholeCus;
}

}  // namespace swz::host
