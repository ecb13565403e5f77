// Device helpers shared by the token attention kernels (gfx950).
#pragma once

#include "attn_common.h"
#include "token_step.h"

namespace uf {
namespace tok {

using attn::bf16x2;
using attn::bf16x8;
using attn::f32x16;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;

__device__ inline bf16x8 lds_row(uint32_t at) {            // 16 bytes of a row
  return __builtin_bit_cast(bf16x8, *(const lds_u32x4*)(uintptr_t)at);
}
__device__ inline v4i16 lds_tr(uint32_t at) {              // transposing read
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(uintptr_t)at);
}
__device__ inline bf16x8 lds_tr2(uint32_t lo, uint32_t hi) {
  const v4i16 v[2] = {lds_tr(lo), lds_tr(hi)};
  return __builtin_bit_cast(bf16x8, v);
}

// Rows of 64 dimensions in LDS: 128 bytes, 16-byte chunk c of row r at c ^ swz_k(r % 16).
// Row reads (sixteen consecutive rows, one chunk) and transposing reads (four
// consecutive rows, 64 bytes of each) touch every bank once.
__device__ inline int swz_k(int r) { return ((r & 2) << 1) | (((r >> 1) ^ (r << 1)) & 2) | ((r >> 3) & 1); }

// Bits of the 64 keys from `key0` on that a query at position `pos` sees.
__device__ inline uint64_t bits_upto(int n) {              // bits 0 .. n-1
  return n >= 64 ? ~uint64_t(0) : (n <= 0 ? 0 : (uint64_t(1) << n) - 1);
}
__device__ inline uint64_t seen_bits(int pos, int key0, int window, int sinks) {
  uint64_t see = bits_upto(pos - key0 + 1);
  if (window > 0) see &= ~bits_upto(pos - window + 1 - key0) | bits_upto(sinks - key0);
  return see;
}
// The same for a node of a tree over `held` tokens.
__device__ inline uint64_t seen_bits_tree(int pos, int key0, int window, int sinks, int held, uint64_t node) {
  uint64_t see = window > 0 ? ~bits_upto(pos - window + 1 - key0) | bits_upto(sinks - key0) : ~uint64_t(0);
  const int d = held - key0;                               // the first node's bit
  see &= bits_upto(d);
  if (d >= 0) return see | (d < 64 ? node << d : 0);
  return see | (d > -64 ? node >> -d : 0);
}

// Rows one by one, where the tiles' products cannot be used.  dot_row: of 128 dimensions, 16 ks + 8 hl .. in registers, the
// other half in lane l ^ 32, with a row in memory.  add_row: dims d0 + 8 i .. + 3 (i < N) of w times such a row to out.
__device__ inline float dot_row(const bf16x8 (&q)[8], const uint8_t* row, int hl) {
  float s = 0.f;
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) {
    const bf16x8 x = attn::as_bf16x8(*reinterpret_cast<const uint4*>(row + (16 * ks + 8 * hl) * 2));
    bf16x8 y = q[ks];
    asm volatile("" : "+v"(y));   // (its fp32 form is made here, not held in 64 registers across the kernel)
#pragma unroll
    for (int e = 0; e < 8; ++e) s += float(y[e]) * float(x[e]);
  }
  return attn::pair_sum(s);
}
template <int N>
__device__ inline void add_row(float w, const uint8_t* row, bool on, int d0, float* out) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint2 x = *reinterpret_cast<const uint2*>(row + (d0 + 8 * i) * 2);
    const float y[4] = {__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16),
                        __uint_as_float(x.y & 0xffff0000u)};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (on) out[4 * i + e] += w * y[e];
  }
}
// One key's term of a lane's row of O.
template <int N>
__device__ inline void add_key(const bf16x8 (&q)[8], const uint8_t* k, const uint8_t* v, int hl, bool on, float c2, float m,
                               int d0, float* out) {
  add_row<N>(__builtin_amdgcn_exp2f(__builtin_fmaf(dot_row(q, k, hl), c2, -m)), v, on, d0, out);
}
__device__ inline bool not_finite(float x) { return !(fabsf(x) < INFINITY); }

// A sequence's part in a launch over the cache's step.
struct Part {
  int seq, at, count, held;    // new tokens `count` from token `at` of the step on, over `held` earlier ones
};
__device__ inline Part step_part(const AttnArgs& a, int e) {
  typedef const attn::const_i32* words;
  const words w = (words)(a.step + kHeader + kEntry * e);
  Part p;
  p.seq = w[0];
  p.at = w[1];
  p.count = min(w[2], a.total - w[1]);
  p.held = w[3] - w[2];
  return p;
}
// The sequence and tile of a launch's tile k, where it deals workgroups to the tiles there are.
__device__ inline Place tile_place(const AttnArgs& a, int k, int tile_rows) {
  Place w = place_of(a.step, a.n, k, [&](const int32_t* entry) {
    const int rows = min(entry[2], a.total - entry[1]) * a.group;
    return rows < a.least_rows || rows > a.most_rows ? 0 : min((rows + tile_rows - 1) / tile_rows, a.tiles);
  });
  if (uint32_t(w.tile) >= uint32_t(a.tiles)) w.entry = -1;
  return w;
}
// Where a launch's partial results of a (tile, key head, slice) start, in rows, and their number.
__device__ inline size_t work_at(const AttnArgs& a, int tile, int h, int slice, int tile_rows) {
  return ((size_t(tile) * a.kv_heads + h) * a.n_split + slice) * tile_rows;
}
__device__ inline size_t work_rows(const AttnArgs& a, int tile_rows) {
  return work_at(a, a.packed > 0 ? a.packed : a.n * a.tiles, 0, 0, tile_rows);
}

}  // namespace tok
}  // namespace uf
