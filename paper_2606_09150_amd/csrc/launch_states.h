// Launch interface of the state operators (internal to libuf.so).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "ufs.h"

namespace uf {
namespace lin {

constexpr int kD = 128;
constexpr int kState = kD * kD;              // floats of a state
constexpr int kChunk = 32;                   // tokens of a chunk

// Threads of a workgroup: of the walks and the parts' sums, and of all other kernels.  A launch has 2^32 - 1 threads at most.
constexpr int kWalkThreads = 512, kOtherThreads = 256;
constexpr int64_t most_groups(int threads) { return ((int64_t(1) << 32) - 1) / threads; }

// The cache's device table, the step: kHeader words (sequences, tokens, parts, chunks of a part), then kEntry words for
// each sequence: its number, its first token of the step, its new tokens, the tokens it held before, its first part.
constexpr int kHeader = 4;
constexpr int kEntry = 5;

// Sequences in a launch.  Workgroup or part k * kv_heads + h is part k of the launch and key head h: of plain tensors part
// k % parts of sequence k / parts, of a step the entry's whose first part is the last at or before k.
struct Geo {
  const float* decay;         // [kv_heads]
  const int32_t* lengths;     // plain tensors: [n] or null
  const int32_t* step;        // a step's table, or null
  int32_t n, tokens;          // sequences; tokens of each, or of the step
  int32_t kv_heads, group;
  int32_t parts, chunks;      // plain: parts of a sequence, a step: of all; chunks of a part (plain)
  int32_t max_seqs;           // a step: states of the pool
  int32_t scanned;            // the parts' own M were carried on by a launch of their own
  float scale;
};

struct Src {
  const uint16_t* p;
  int64_t batch, token, head;                // elements
};

// out_t = row weight x_t . M + sum of weights (x_t . y_j) z_j, M = sum of key weights y_j z_j^T: forwards over j <= t (o
// from q, k, v; dq from do, v, k), or backwards over j >= t (dk from v, do, q; dv from k, q, do).  dq and dk: first and starts
// hold M transposed.
struct Walk {
  Src x, y, z;
  uint16_t* out;
  const float* first;         // M where the walk begins, or null
  float* last;                // M where it ends, or null
  const float* starts;        // M where each part begins (scanned), or the parts' own; null: the only part begins with `first`
};
constexpr int kWalks = 3;
struct WalkArgs {
  Geo geo;
  Walk walk[kWalks];
  int32_t n;
};
// Parts' own M without the parts before (after) them, in their places of `starts`; forwards, where they are not carried on, `first` in
// the last part's, which no part comes after.
struct PartArgs {
  Geo geo;
  struct {
    Src y, z;
    const float* first;
    float* starts;
    int32_t back;
  } sum[2];
  int32_t n;
};

constexpr int kScanSlices = 16;              // of a state, workgroups of the scan
// Whether forward walks (o, dq) take two query heads an item, which share M's parts, y, z and the barriers.  One / two (us): 1 x 16,384
// tokens, 8 key heads of 4, forward 143 / 128, backward 325 / 317; 2 x 4,000, 16 of 2, 83 / 73, 184 / 182; 2 x 6,000, 8 of 8, 164 / 148,
// 447 / 423.  Odd groups take one head twice: 1 x 16,000, 6 of 3, 94 / 97, 190 / 197; 4 of 5, 85 / 81, 184 / 187; 4 of 7, 109 / 103,
// 247 / 246; 2 x 6,000, 8 of 5, 114 / 109, 287 / 285; 8 of 7, 139 / 133, 377 / 369; 4 x 2,000, 8 of 7, 100 / 95, 261 / 257.
inline bool two_heads(int group) { return group % 2 == 0 || group > 3; }
// exact: states are results in fp32, or bear on one
hipError_t launch_linear_parts(const PartArgs& a, int32_t groups, bool exact, hipStream_t stream);
hipError_t launch_linear_scan(const PartArgs& a, hipStream_t stream);
hipError_t launch_linear_fwd(const WalkArgs& a, int32_t groups, hipStream_t stream);
hipError_t launch_linear_bwd(const WalkArgs& a, int32_t groups, bool exact, hipStream_t stream);

// Few tokens a sequence: token by token.  So / in chunks (us): 1 sequence of 8 key heads, 4 tokens 5.0 / 7.1, 8 6.8 / 7.1; 24 of 8 heads of 2,
// 4 9.7 / 10.6, 5 10.8 / 10.5, 7 13.1 / 10.1; 64 of 8, 4 14.3 / 15.1, 6 17.4 / 15.4; 64 of 32, 4 46.6 / 52.5, 6 51.6 / 53.2, 8 58.6 /
// 52.7; 64 of 32 heads of 4, 4 60.2 / 63.8; 16 of 32 heads of 8, 2 18.9 / 26.1, 3 23.9 / 25.2, 4 30.0 / 26.5.  The rule goes by tokens, while a
// wave's way is tokens times query heads: large groups lose at 3 and 4 tokens, and gain below.  16 of 32 heads of 16, 2 27.1 / 37.0, 3 36.3 /
// 37.1, 4 45.8 / 37.5; 4 of 4 heads of 32, 2 19.1 / 36.8, 3 46.3 / 37.3, 4 60.9 / 37.4; 8 of one head of 64, 2 59.3 / 67.7, 4 115.8 / 68.2.
constexpr int kFewTokens = 4;
struct StepArgs {
  Geo geo;                    // of a step
  Src q, k, v;
  uint16_t* o;
  float* states;              // of the layer
  int32_t longest;
};
hipError_t launch_linear_step(const StepArgs& a, hipStream_t stream);

// (source, target) sequences in the launch's words
constexpr int kPairs = 400;
struct ForkArgs {
  float* pool;
  int64_t layer, seq;         // floats of a layer and of a sequence's states in it
  int32_t layers, n;
  int32_t words[2 * kPairs];
};
hipError_t launch_state_fork(const ForkArgs& a, hipStream_t stream);

constexpr int kMaxBeams = 64;
struct ReorderArgs {
  float* pool;
  int64_t layer, seq;
  const int32_t* parents;     // of the launch's groups
  int32_t layers, groups, beams;
  int32_t seqs[2 * kPairs];
};
hipError_t launch_state_reorder(const ReorderArgs& a, hipStream_t stream);

// Selection: slices of rows of logits, then what they hold per request.
constexpr int kMaxSelect = 64;
struct SelectArgs {
  const void* logits;
  int64_t group_stride, beam_stride;         // elements
  const float* scores;
  const uint8_t* done;
  float* best;
  int32_t* parents;
  int32_t* tokens;
  uint8_t* work;
  int32_t groups, beams, vocab, k, type, end;
  int32_t splits, slice;                     // slices of a row, vectors of 16 bytes of each
};
void plan_select(SelectArgs* a);
size_t select_work_bytes(const SelectArgs& a);
hipError_t launch_select(const SelectArgs& a, hipStream_t stream);

}  // namespace lin
}  // namespace uf
