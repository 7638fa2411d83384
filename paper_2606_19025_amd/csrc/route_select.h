// Selection of the largest logits and the local ids of the resident experts, shared by the
// router (route.hip) and the few-token layer (few.hip).
#pragma once
#include "common.h"

namespace moe {

// Local id (rank among resident experts, -1 for ghosts) of every expert, via
// ballots over chunks of 64 experts.  Executed by wave 0.
DEVI void build_local_map(const uint8_t* resident, int E, int* lmap) {
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int e0 = 0; e0 < E; e0 += 64) {
    const int e = e0 + lane;
    const bool r = (e < E) && resident[e] != 0;
    const uint64_t m = __ballot(r);
    const int below = __popcll(m & ((1ull << lane) - 1ull));
    if (e < E) lmap[e] = r ? base + below : -1;
    base += __popcll(m);
  }
}

// Logit as read for selection: NaN ranks as -inf (some expert is always
// picked) and -0 as +0 (they tie, as equal values do).
DEVI float sel_value(float v) { return (v != v) ? -INFINITY : v + 0.0f; }

// Order-preserving map of a float to uint32 (larger float -> larger key);
// every float maps above 0, the key of an empty slot.
DEVI uint32_t sel_key(float v) {
  const uint32_t u = __float_as_uint(v);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

constexpr int RT_KSEL = 8;

// Lane permutations within a row of 16 lanes (DPP), applied to a 64-bit value
// (its two halves moved alike): xor 1 and xor 2 inside each quad, then lane
// i <- 7 - i inside each half-row and lane i <- 15 - i inside the row.  After
// taking the maximum with each in turn, every lane of the row holds the row's
// maximum.
template <int CTRL>
DEVI uint64_t row_perm64(uint64_t v) {
  const int lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, 0xF, 0xF, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, 0xF, 0xF, false);
  return ((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo;
}
DEVI uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }
DEVI uint64_t row16_max64(uint64_t m) {
  m = max64(m, row_perm64<0xB1>(m));   // quad_perm [1, 0, 3, 2]
  m = max64(m, row_perm64<0x4E>(m));   // quad_perm [2, 3, 0, 1]
  m = max64(m, row_perm64<0x141>(m));  // row_half_mirror
  m = max64(m, row_perm64<0x140>(m));  // row_mirror
  return m;
}

}  // namespace moe
