// Launch interface of the token operators (internal to libuf.so).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "uft.h"

namespace uf {
namespace tok {

constexpr int kD = 128;
constexpr int kMaxTree = 64;      // nodes of a tree: bits of a node's word
constexpr int kInPlace = 16;      // rows that uft_keep moves in place

// Words of host metadata that ride in a launch's arguments: kWords at most, and where
// kFew do, a launch with arguments of that size (a host copy of 3.5 KB less).
constexpr int kWords = 880, kFew = 64;

// The device tables: the step (kHeader words, of which the first is its number of
// sequences, then kEntry words for each: sequence, first token of the step, tokens,
// length with them), then the page of each page_tokens tokens, [max_seqs][row].
constexpr int kHeader = 4;
constexpr int kEntry = 4;

struct Pool {
  uint8_t* base;            // of the layer, or of layer 0
  size_t layer_bytes;
  int32_t layers, n_pages, kv_heads, page_tokens;
};

// words[0 .. dense) go to table[dense_at ..]; then n_runs runs from words[runs] on:
// (at, count, value), of ascending values from `value` on.
struct PokeHead {
  int32_t* table;
  int32_t dense_at, dense, runs, n_runs;
};
// table rows: (source offset, target offset, count) triples
struct RowsHead {
  int32_t* table;
  int32_t n;
};
// (source page, target page, rows) triples, every layer; with them, from words[3 n] on,
// the words of a PokeHead (table null: none).
struct CopyHead {
  Pool pool;
  int32_t n;
  PokeHead poke;
};
// uft_keep.  In place: kKeepWords words a sequence: table offset, length, start, count,
// first index.  Into fresh pages: the same for a run of pages that follow one another,
// then the sequence's page that the run begins with, how many of the launch's pages
// came before, and the run's first page.
constexpr int kKeepWords = 8;
struct KeepHead {
  Pool pool;
  const int32_t* table;     // page table of all sequences
  const int32_t* index;
  int32_t n, n_pages;
};
template <class Head, int N>
struct Worded : Head {
  int32_t words[N];
};
using PokeArgs = Worded<PokeHead, kWords>;
using RowsArgs = Worded<RowsHead, kWords>;
using CopyArgs = Worded<CopyHead, kWords>;
using KeepArgs = Worded<KeepHead, kWords>;
// `used`: words of a that hold something
hipError_t launch_poke(const PokeArgs& a, int used, hipStream_t stream);
hipError_t launch_rows(const RowsArgs& a, hipStream_t stream);
hipError_t launch_copy_pages(const CopyArgs& a, int used, hipStream_t stream);
hipError_t launch_keep_in_place(const KeepArgs& a, hipStream_t stream);
hipError_t launch_keep_fresh(const KeepArgs& a, hipStream_t stream);

struct WriteArgs {
  const uint16_t* k;
  const uint16_t* v;
  int64_t k_token, k_head, v_token, v_head;   // elements
  Pool pool;                                  // base: the layer's
  const int32_t* step;
  const int32_t* table;
  int32_t n, longest, total, row;             // row: pages of a table row
  int32_t packed;                             // pages of all sequences, where workgroups are dealt to those; or 0
};
// Pages that so many new tokens of a sequence touch at most.
__host__ __device__ inline int write_spans(int count, int page_tokens) {
  return count > 0 ? (count - 1 + page_tokens - 1) / page_tokens + 1 : 0;
}
hipError_t launch_write(const WriteArgs& a, hipStream_t stream);

// Attention forward, from the cache or from plain tensors.
struct AttnArgs {
  const uint16_t* q;
  int64_t q_batch, q_token, q_head;           // elements
  uint16_t* o;
  float* lse;
  const int64_t* tree;
  // from the cache
  Pool pool;                                  // base: the layer's
  const int32_t* step;
  const int32_t* table;
  int32_t row;
  // from plain tensors
  const uint16_t* k;
  const uint16_t* v;
  int64_t k_batch, k_token, k_head, v_batch, v_token, v_head;
  const int32_t* lengths;
  int32_t tokens;
  int32_t n, total;                           // sequences; tokens of the step
  int32_t q_heads, kv_heads, group, window, sinks;
  float scale_log2;
  int32_t tiles;                              // row tiles of the longest sequence
  int32_t packed;                             // row tiles of all sequences, where workgroups are dealt to those; 0: `tiles` each
  int32_t least_rows, most_rows;              // sequences with other numbers of rows are not this launch's
  int32_t longest_rows;                       // the most rows of one of its sequences
  int32_t slice;                              // units of keys of a slice at least
  int32_t n_split;                            // slices at most
  float* work;                                // partials: O [tile][kv head][slice][row][D], then (offset, sum) of the same
};
constexpr int kRowTile = 128, kKeyUnit = 64;          // prompts: rows and keys of a tile
constexpr int kFewRows = 32, kFewUnit = 32;           // few rows: rows of a workgroup, keys of a unit
hipError_t launch_attn_rows(const AttnArgs& a, bool paged, hipStream_t stream);
hipError_t launch_attn_few(const AttnArgs& a, hipStream_t stream);

// The range of keys of a tile of queries at positions first .. last, in units of
// `unit` keys: units 0 .. sink-1 hold sinks that lie before the window's first unit
// `from`, then come units from .. to.  Unit u of the range is
// u < sink ? u : u - sink + from.
struct Range {
  int32_t sink, from, count, low;             // low: first key of the window of `first`
};
__host__ __device__ inline Range key_range(int first, int last, int window, int sinks, int unit) {
  Range r;
  r.low = (window > 0 && first - window + 1 > 0) ? first - window + 1 : 0;
  r.from = r.low / unit;
  const int s = (sinks + unit - 1) / unit;    // sinks <= 2^30
  r.sink = s < r.from ? s : r.from;
  r.count = r.sink + last / unit - r.from + 1;
  return r;
}
// Units of a slice of a range: `slice`, unless the range has more than n_split of them.
__host__ __device__ inline int slice_units(int count, int slice, int n_split) {
  const int least = (count + n_split - 1) / n_split;
  return slice > least ? slice : least;
}

// Backward.
struct BwdArgs {
  const uint16_t *q, *k, *v, *o, *dout;
  const float* lse;
  const int32_t* lengths;
  int64_t q_batch, q_token, q_head, k_batch, k_token, k_head, v_batch, v_token, v_head;
  uint16_t *dq, *dk, *dv;
  uint8_t* work;
  int32_t batch, tokens, q_heads, kv_heads, group, window, sinks;
  int32_t tiles;                              // row tiles of a sequence
  uint64_t group_div;                         // (2^64 - 1) / group: j / group == ((j + 1) * group_div) >> 64 for 0 <= j < 2^31
  float scale, scale_log2;
};
size_t bwd_work_bytes(const BwdArgs& a);
hipError_t launch_window_bwd(const BwdArgs& a, hipStream_t stream);

}  // namespace tok
}  // namespace uf
