// Which piece of an attention launch a workgroup computes.  Host and device code; pid_decode.h has the dispatch model.
//
// Tiles of tokens (turns) are computed for every query head (or key head, where a workgroup goes over the query heads that share it).  The query heads
// of a key head read the same keys and values, so they belong on one XCD, next to each other in time; and the turns of a head differ in length by up to the length of
// a sequence, so every XCD needs turns of all lengths, the longest first.  With X XCDs and H key heads: sets = gcd(H, X) of H / sets key heads, each served by X / sets
// XCDs, which are dealt (turn, key head) in that order, all `group` query heads of a pair at a time.  32768 tokens, 16 heads of 128 sharing 4, causal, with one run of
// (key head, turn) for each XCD instead, half of which then have the long turns: 1.4 times the time.
#pragma once

#include "pid_decode.h"

namespace swz {

struct PromptPiece {
  int turn, k_head, member;          // turn < 0: nothing to compute
};

SWZ_HD int prompt_sets(int k_heads, int num_xcd) {
  int a = k_heads, b = num_xcd;
  while (b != 0) {
    const int r = a % b;
    a = b;
    b = r;
  }
  return a;
}

// Workgroups of a launch: the same number for every XCD.
SWZ_HD int64_t prompt_workgroups(int64_t turns, int k_heads, int group, int num_xcd) {
  const int sets = prompt_sets(k_heads, num_xcd), share = num_xcd / sets;
  return (turns * (k_heads / sets) + share - 1) / share * group * num_xcd;
}

SWZ_HD PromptPiece prompt_piece(int w, int turns, int k_heads, int group, int num_xcd, int sets) {
  const int share = num_xcd / sets, heads = k_heads / sets;
  const int i = w / num_xcd, x = w - i * num_xcd, set = x / share;
  const int pair_of_xcd = i / group, pair = pair_of_xcd * share + (x - set * share), turn = pair / heads;
  return {turn < turns ? turn : -1, set * heads + (pair - turn * heads), i - pair_of_xcd * group};
}

}  // namespace swz
