// A workgroup's place in a launch of the linear attention kernels (device code).
#pragma once

#include "../launch_states.h"
#include "attn_common.h"

namespace uf {
namespace lin {

struct Place {
  int seq;              // plain tensors: of the batch; a step: of the pool; -1: none
  int h, part, parts;   // key head; part of the sequence
  int64_t row;          // first token: plain, of the sequence's tensors; a step, of the step's
  int tokens;           // of the sequence
  int chunk0, chunks;   // of the part
  int cut;              // chunks of the parts before the last one
  int rows;             // rows of the sequence in the outputs (with padding)
  bool held;            // the state before the walk counts
};

// Whole parts cover the same number of chunks; the last one has the rest.
__device__ inline void cut_into(Place& p, int chunks) {
  const int all = (p.tokens + kChunk - 1) / kChunk;
  p.cut = chunks;
  p.parts = (all + chunks - 1) / chunks;
  p.chunk0 = p.part * chunks;
  p.chunks = min(chunks, max(0, all - p.chunk0));
}

// Entry e of a step, as far as the launch reaches.
__device__ inline void entry_of(const Geo& g, int e, Place& p) {
  typedef const attn::const_i32* words;
  const words w = (words)(g.step + kHeader + kEntry * e);
  p.seq = w[0];
  p.row = w[1];
  p.tokens = max(0, min(w[2], g.tokens - w[1]));
  p.held = w[3] > 0;
  p.rows = p.tokens;
  if (uint32_t(p.seq) >= uint32_t(g.max_seqs)) p.seq = -1;
}

__device__ inline Place place(const Geo& g, int idx) {
  typedef const attn::const_i32* words;
  Place p;
  p.h = idx % g.kv_heads;
  const int k = idx / g.kv_heads;
  if (g.step == nullptr) {
    p.seq = k / g.parts;
    p.part = k - p.seq * g.parts;
    p.row = 0;
    p.tokens = g.lengths != nullptr ? min(max(((words)g.lengths)[p.seq], 0), g.tokens) : g.tokens;
    p.rows = g.tokens;
    p.held = true;
    cut_into(p, g.chunks);
    return p;
  }
  const words head = (words)g.step;
  const int n = min(g.n, head[0]), chunks = max(1, head[3]);
  int lo = 0, hi = n - 1;
  while (lo < hi) {                                      // the last entry whose first part is at or before k
    const int mid = (lo + hi + 1) >> 1;
    if (head[kHeader + kEntry * mid + 4] <= k) lo = mid;
    else hi = mid - 1;
  }
  p.seq = -1;
  if (n < 1 || k >= head[2]) return p;
  entry_of(g, lo, p);
  const int first = head[kHeader + kEntry * lo + 4];
  p.part = k - first;
  cut_into(p, chunks);
  // (a captured launch after a step that is cut otherwise: parts' states behind its own are not in its scratch)
  if (p.part >= p.parts || first + p.parts > g.parts) p.seq = -1;
  return p;
}

}  // namespace lin
}  // namespace uf
