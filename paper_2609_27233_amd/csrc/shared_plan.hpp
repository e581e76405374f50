// How a batch's shared prefixes are cut: a rule on sizes (host code that needs
// no HIP, so that a test can compile it by itself).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace sm {

constexpr int kSharedVec = 128;        // query vectors of a workgroup
constexpr int kSharedStep = 128;       // entries that a chunk is a multiple of
constexpr int kSharedMostChunk = 8192;
constexpr int kSharedWgs = 256;        // workgroups that the cut aims at: one for each compute unit
constexpr int64_t kSharedVectors = (int64_t)kSharedWgs * kSharedVec;  // vectors x chunks, at most

struct SharedPlan {
  int chunk;   // entries of a chunk, a multiple of kSharedStep
  int chunks;  // chunks of the longest prefix
};

// Chunks that the workspace has room for: any plan stays within it.
inline int64_t shared_most_chunks(int64_t vectors, int max_prefix) {
  const int64_t all = ((int64_t)max_prefix + kSharedStep - 1) / kSharedStep;
  const int64_t most = kSharedVectors / vectors > 1 ? kSharedVectors / vectors : 1;
  const int64_t least = ((int64_t)max_prefix + kSharedMostChunk - 1) / kSharedMostChunk;
  const int64_t got = all < most ? all : most > least ? most : least;
  return got > 1 ? got : 1;
}

// n requests of G query heads on each of H kv heads, in `groups` groups.
inline SharedPlan plan_shared(int n, int H, int G, int groups, int max_prefix) {
  if (max_prefix <= 0) return SharedPlan{kSharedStep, 0};
  const int64_t per = ((int64_t)n + groups - 1) / groups * G;  // vectors of a group and kv head
  const int64_t most = shared_most_chunks((int64_t)n * G * H, max_prefix);
  const int64_t blocks = (per + kSharedVec - 1) / kSharedVec * groups * H;
  int64_t chunks = kSharedWgs / blocks;
  if (chunks > most) chunks = most;
  if (chunks < 1) chunks = 1;
  int64_t chunk = ((int64_t)max_prefix + chunks - 1) / chunks;
  chunk = (chunk + kSharedStep - 1) / kSharedStep * kSharedStep;
  if (chunk > kSharedMostChunk) chunk = kSharedMostChunk;
  return SharedPlan{(int)chunk, (int)(((int64_t)max_prefix + chunk - 1) / chunk)};
}

}  // namespace sm
