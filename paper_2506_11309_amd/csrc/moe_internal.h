// Launches of the routers of a mixture of experts.
#pragma once
#include "ss_internal.h"

namespace ss {

// Tokens of a unit: as many as its waves take at one time, so that a prompt fills
// the chip, but at most 256 units (each grouping workgroup reads all their
// counts) as long as a unit's counts fit 16 bits.
constexpr int kLeast = 64;
inline int unit_tokens(int T, int k) {
  const int most = 65535 / k, need = (T + 255) / 256;
  return need < kLeast ? kLeast : need > most ? most : need;
}

// what the grouping knows of the tokens
struct GroupArgs {
  int T, E, k, tokens;  // tokens of a unit
  int32_t* experts;
  float* weights;
  int32_t *offsets, *rows, *pos;
  uint16_t* hist;  // [units][E rounded up to 4]
};

// The places of the pairs of `units` units of tokens whose counts are in hist.
void launch_group_units(const GroupArgs& a, int units, hipStream_t st);

struct RouteLaunch {
  const uint16_t* logits;  // null: the experts are given
  int ldl, T, E, k, renormalize;
  int32_t* experts;
  float* weights;
  int32_t *offsets, *rows, *pos;
  uint16_t* hist;  // route_hist_bytes
};
size_t route_hist_bytes(int T, int E, int k);  // T k < 2^28
void launch_moe_route(const RouteLaunch& L, hipStream_t st);


struct ScoredLaunch {
  GroupArgs group;  // all but tokens
  const void* logits;
  int ldl;
  bool wide, sigmoid, renormalize;  // wide: float scores, otherwise fp16
  const float* bias;
  int groups, top_groups, best;
  float scale;
};
void launch_moe_route_scored(const ScoredLaunch& L, hipStream_t st);

}  // namespace ss
