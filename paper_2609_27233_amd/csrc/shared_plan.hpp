// How a batch's shared prefixes are cut: a rule on sizes (host code that needs
// no HIP, so that a test can compile it by itself).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace sm {

// Query vectors of a workgroup: 32 for each of its four waves, which share the
// tiles of its keys.  (Waves over different keys, merged through LDS, and e4m3
// fragments straight from the pages, as for few prefill rows, measured slower:
// 128 requests behind 16,000 e4m3 entries 99 us for 87.)
constexpr int kSharedVec = 128;
constexpr int kSharedStep = 128;       // entries that a chunk is a multiple of
constexpr int kSharedMostChunk = 8192;
// Workgroups that the cut aims at: one for each compute unit, or two where that
// leaves their chunks long.  A second one hides the first's waits and its
// softmax; a chunk more costs the join a read of every row.  Us at 128, 256 and
// 512, 32/8 heads, D = 128, bf16 and e4m3 pages (chunk in entries at 256):
//   128 requests behind 4096 (512)    -, 47, 57 and -, 42, 49
//   behind 8192 (1024)                -, 57, 66 and -, 56, 59
//   behind 12,000 (1536)              -, 69, 73 and -, 72, 65
//   behind 16,000 (2048)              105, 82, 81 and 118, 86, 73
//   behind 32,000 (4096)              -, 143, 115 and -, 153, 108
//   64 behind 32,000 (2048)           -, 81, 73 and -, 87, 69
//   128 behind four of 6000 to 8192, 28/4 heads (1024)  74, 66, 78 and 74, 56, 63
//   8 behind each of 16 of 2000, 16/4 heads, D = 64 (512)  29, 22, 23 and 29, 21, 19
// Many requests' own chunks are the second workgroup anyway: 500 behind 4096
// (2048) -, 124, 140 and -, 103, 111.
constexpr int kSharedWgs = 256, kSharedLongChunk = 896, kSharedFewPairs = 2048;
constexpr int64_t kSharedVectors = 2 * (int64_t)kSharedWgs * kSharedVec;  // vectors x chunks, at most

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

// Where the prefixes' parts lie in the workspace, in bytes from the end of the
// requests' own: the flag in a line of its own, then each vector's and chunk's
// unnormalised output, read and written 16 bytes at a time (the statistics
// behind it: their 8 bytes come in any number).
constexpr int64_t kSharedLine = 256;
struct SharedParts {
  int64_t flag, o, ml, end;
};
inline SharedParts shared_parts(int64_t vectors, int64_t chunks, int head_dim) {
  const int64_t o = kSharedLine, ml = o + vectors * chunks * head_dim * 4;
  return SharedParts{0, o, ml, ml + vectors * chunks * 8};
}

// n requests of G query heads on each of H kv heads, in `groups` groups.
inline SharedPlan plan_shared(int n, int H, int G, int groups, int max_prefix) {
  if (max_prefix <= 0) return SharedPlan{kSharedStep, 0};
  const int64_t per = ((int64_t)n + groups - 1) / groups * G;  // vectors of a group and kv head
  const int64_t most = shared_most_chunks((int64_t)n * G * H, max_prefix);
  const int64_t blocks = (per + kSharedVec - 1) / kSharedVec * groups * H;
  int64_t chunks = 2 * kSharedWgs / blocks;
  if (chunks * kSharedLongChunk > max_prefix || (int64_t)n * H > kSharedFewPairs) chunks = kSharedWgs / blocks;
  if (chunks > most) chunks = most;
  if (chunks < 1) chunks = 1;
  int64_t chunk = ((int64_t)max_prefix + chunks - 1) / chunks;
  chunk = (chunk + kSharedStep - 1) / kSharedStep * kSharedStep;
  if (chunk > kSharedMostChunk) chunk = kSharedMostChunk;
  return SharedPlan{(int)chunk, (int)(((int64_t)max_prefix + chunk - 1) / chunk)};
}

}  // namespace sm
