// Where the positions of a sequence are in a cache of pages.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace swz {

struct PageTable {
  const int32_t* table;
  int64_t pages;
  int page_shift, k_heads, table_width;
  // The page of a position (not negative), or -1.
  __device__ __forceinline__ int page_of(int sequence, int position) const {
    const int j = position >> page_shift;
    if (j >= table_width) return -1;
    const int page = table[(int64_t)sequence * table_width + j];
    return page >= 0 && page < pages ? page : -1;
  }
  // Tokens of a head before this one in the cache.
  __device__ __forceinline__ int64_t token_at(int page, int head, int position) const {
    return (((int64_t)page * k_heads + head) << page_shift) + (position & ((1 << page_shift) - 1));
  }
};

}  // namespace swz
