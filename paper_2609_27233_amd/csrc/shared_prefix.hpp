// The part of a shared decode call that its two sources have in common (gfx950).
#pragma once

#include "common.hpp"
#include "shared_plan.hpp"

namespace sm {

// A chunk's share of the attention over a prefix, for each vector (request i,
// query head h): the unnormalised output, its reference and its sum.
struct PrefixParts {
  float *o;       // [n][num_q_heads][chunks][head_dim]
  float *ml;      // [n][num_q_heads][chunks][2]; a sum of 0: no entries, below 0: unusable
  int32_t *flag;  // 1: the groups are no list of the requests
  int chunks;
};

struct PrefixArgs {
  const int32_t *prefix_ids, *group_offsets;
  int n, groups, max_prefix;
  SharedPlan plan;
  PrefixParts parts;
};

}  // namespace sm
