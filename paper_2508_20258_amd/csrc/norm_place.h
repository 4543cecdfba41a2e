// Which heads a group of lanes has in the norm's kernels, and which of them it stores.  Host and device code.
#pragma once

#include "pid_decode.h"

namespace swz {

// D / 8 lanes take kNormHeads heads of a token (an item), 8 dimensions each: the token's angles are loaded once for them, and their product with the weight is
// taken once.  What turns is exchanged among lanes as it was loaded.
constexpr int kNormThreads = 256;
constexpr int kNormHeads = 4;

SWZ_HD int norm_blocks(int heads) { return (heads + kNormHeads - 1) / kNormHeads; }
// Workgroups that have an item for each of their D / 8 lanes.
SWZ_HD int norm_workgroups(int items, int head_dim) {
  const int per = kNormThreads / (head_dim / 8);
  return items / per + (items % per != 0);
}

struct NormPlace {
  int token, head0;
  bool there;
};
// Of `item` of `items`, `blocks` of a token.  Lanes past the end have the last item too, for the exchanges among lanes, but it is not theirs.
SWZ_HD NormPlace norm_place(int64_t item, int items, int blocks) {
  const bool there = item < items;
  const int i = there ? (int)item : items - 1, token = i / blocks;
  return {token, (i - token * blocks) * kNormHeads, there};
}
// Whether head `i` of the place is stored.  Each head by one group of lanes alone: where it is stored over what was loaded (the outputs may be the inputs), a second one could
// load what the first has stored.
SWZ_HD bool norm_stores(const NormPlace& p, int i, int heads) { return p.there && p.head0 + i < heads; }

}  // namespace swz
