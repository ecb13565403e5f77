// Linear attention with a decay for each head: whole sequences, prompts, pieces of
// prompts, and the gradients.
//
// All four results are one walk over a sequence in chunks of 32 tokens, with a matrix M
// [128 y-dims, 128 z-dims] that stands for what lies behind:
//     out_t = r_t M^T x_t + scale sum_j L^|t-j| (x_t.y_j) z_j     over the chunk's j <= t (>= t)
//     M     = L^32 M + sum_j c_j y_j z_j^T.
// o is the walk of (q, k, v), dq that of (do, v, k) with M transposed, and backwards dk that of (v,
// do, q) and dv that of (k, q, do), which add over the query heads of a key head.  Where
// sequences are few they are cut into parts: one launch forms the parts' own M, one
// carries them on from part to part, and the walks begin from those.
//
// Work split: a workgroup per (sequence, part, key head), four waves, each with 32
// z-dims of M and of the result; P^T = Y X^T is formed by each of them for itself (8 of
// 52 products a chunk), so that no wave waits for another but for the copies.  All products are
// v_mfma_f32_32x32x16_bf16: O^T = M^T X^T + Z^T P^T and M += Y^T (c Z), X and Y rows and
// transposed reads of Y and Z from LDS.  M stays in accumulators: its y-dims lie there as the
// k-slots of the next product want them (Y^T's operand is read with bits 2 and 3 of its
// dimensions swapped, which the accumulators swap back), so it is multiplied without leaving
// registers.
//
// Rounding: M and P enter their products as two bf16 parts each (one alone would add as much
// error as the result's own rounding), c Z in three, since M is a result in fp32 and carries
// each error on (two where it is none).  L^32 in fp32 would be off by the same 2^-25 in each of
// thousands of chunks: the part of it that fp32 drops is carried on and added to the next factor.
//
// Memory: three tiles of 8 KB an item (a chunk and query head), in two blocks of 64 dimensions in 128-byte
// rows (swz_k), copied by global_load_lds two items ahead into three buffers; one barrier
// an item.  Rows past the sequence's end take its last row, and weigh nothing.
#include "linear_place.h"
#include "token_common.h"

namespace uf {
namespace lin {
namespace {

using namespace attn;
using tok::bits_upto;
using tok::lds_row;
using tok::lds_tr2;
using tok::swz_k;

constexpr uint32_t kTile = 8192, kHalf = 4096, kStage = 3 * kTile;
constexpr int kStages = 3;
// LDS behind the stages, in floats: L^e for e = 0 .. 32, and the key weights of a whole chunk and of the last one.
constexpr int kPowers = 36;
constexpr uint32_t kShared = kStages * kStage + 4 * (kPowers + 2 * kChunk);

// x as parts of 8 bits each, the first ones cut off and the last one rounded.
__device__ inline bf16x8 top_part(float (&x)[8], bool rest) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = __builtin_amdgcn_perm(__float_as_uint(x[2 * i + 1]), __float_as_uint(x[2 * i]), 0x07060302u);
  if (rest)
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] -= __uint_as_float(__float_as_uint(x[i]) & 0xffff0000u);
  return as_bf16x8(make_uint4(w[0], w[1], w[2], w[3]));
}
__device__ inline bf16x8 last_part(const float (&x)[8]) {
  return as_bf16x8(make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])));
}
// Sign bits of the halves that are not finite (junk in the others).
__device__ inline uint32_t odd_halves(uint32_t u) { return (u & 0x7f807f80u) + 0x00800080u; }

__device__ inline double power(double g, int e) { return e == 0 ? 1.0 : exp(g * double(e)); }

// OUT: results are wanted, not M alone.  begin: M where the walk begins, or null; last: where to put it at the end, or null.
template <bool BACK, bool OUT, int PARTS>
__device__ __forceinline__ void walk(const Geo& geo, const Place& p, const Src& xs, const Src& ys, const Src& zs, uint16_t* out,
                                     const float* begin, bool trans, float* last, uint8_t* smem) {
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, hl = lane >> 5, ln = lane & 31, rp = lane & 15, gr = (lane >> 4) & 1;
  const int h = p.h, G = geo.group;
  const int rest = min(kChunk, p.tokens - (p.chunk0 + p.chunks - 1) * kChunk);   // tokens of the part's last chunk (by time)
  const uint32_t lds0 = lds_addr(smem);

  // copies: rows 8 wave + lane / 8 of each tile
  const int crow = 8 * wave + (lane >> 3);
  const uint32_t cchunk = uint32_t(16 * ((lane & 7) ^ swz_k(crow & 15)));
  const int n_items = p.chunks * G;
  int next_c = 0, next_g = 0;                          // the next item to copy
  auto issue = [&](uint32_t stage) {
    const int c = BACK ? p.chunk0 + p.chunks - 1 - next_c : p.chunk0 + next_c;
    const int t0 = c * kChunk, row = min(crow, p.tokens - 1 - t0);
    const uint32_t dst = __builtin_amdgcn_readfirstlane(lds0 + stage * kStage + uint32_t(wave) * 1024u);
    auto copy = [&](const Src& s, int head, uint32_t at) {
      const uint8_t* base = uniform_ptr(reinterpret_cast<const uint8_t*>(
          s.p + (geo.step == nullptr ? int64_t(p.seq) * s.batch : 0) + (p.row + t0) * s.token + int64_t(head) * s.head));
      const uint32_t off = uint32_t(row) * uint32_t(s.token * 2) + cchunk;
      dma16(base, off, dst + at);
      dma16(base + 128, off, dst + at + kHalf);
    };
    const int hg = h * G + next_g;
    if (OUT) copy(xs, BACK ? h : hg, 0);
    copy(ys, BACK ? hg : h, kTile);
    copy(zs, BACK ? hg : h, 2 * kTile);
    // past the end the last item is copied again, and not read
    if (next_g + 1 < G) ++next_g;
    else if (next_c + 1 < p.chunks) ++next_c, next_g = 0;
  };
  if (n_items > 0) {
    issue(0);
    issue(1);
  }

  // weights
  float* const tab = reinterpret_cast<float*>(smem + kStages * kStage);
  const double gd = double(geo.decay[h]);
  const float scale = geo.scale;
  if (tid < 33) tab[tid] = float(power(gd, tid));
  if (tid >= 64 && tid < 128) {
    const int j = tid & 31, n = tid < 96 ? kChunk : rest;
    tab[kPowers + tid - 64] = j >= n ? 0.f : BACK ? scale * float(power(gd, j + 1)) : float(power(gd, n - 1 - j));
  }
  const double dw = power(gd, kChunk);
  const float whole_hi = float(dw), whole_lo = float(dw - double(whole_hi)), rest_dec = float(power(gd, max(rest, 0)));
  __syncthreads();
  float pw[16];                                        // of (x_t.y_j), j = 8 (r / 4) + 4 hl + r % 4 of the chunk
  uint32_t see = 0;
  if (OUT) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int j = 8 * (r >> 2) + 4 * hl + (r & 3), age = BACK ? j - ln : ln - j;
      pw[r] = scale * tab[max(age, 0)];
      see |= uint32_t(age >= 0) << r;
    }
  }
  const float row_whole = BACK ? tab[31 - ln] : scale * tab[ln + 1];
  const float row_rest = BACK ? tab[max(rest - 1 - ln, 0)] : row_whole;

  // operand addresses within a stage
  uint32_t kr[4], yt[2][2], zt[2];
#pragma unroll
  for (int k = 0; k < 4; ++k) kr[k] = lds0 + uint32_t(ln * 128 + 16 * ((2 * k + hl) ^ swz_k(ln & 15)));
#pragma unroll
  for (int hh = 0; hh < 2; ++hh) {
    const int r = 8 * hh + 4 * hl + (rp >> 2);
#pragma unroll
    for (int m = 0; m < 2; ++m)                        // (units of four dimensions with bits 2 and 3 swapped)
      yt[hh][m] = lds0 + kTile + uint32_t(r * 128 + 16 * ((4 * m + 2 * gr + (rp & 1)) ^ swz_k(r)) + 8 * ((rp >> 1) & 1));
    zt[hh] = lds0 + 2 * kTile + uint32_t(wave >> 1) * kHalf +
             uint32_t(r * 128 + 16 * ((4 * (wave & 1) + 2 * gr + ((rp >> 1) & 1)) ^ swz_k(r)) + 8 * (rp & 1));
  }
  const uint32_t kwt = lds0 + kStages * kStage + 4 * (kPowers + 4 * hl);

  // M: y-dim 32 mt + 16 (r / 8) + 8 hl + r % 8, z-dim 32 wave + ln
  f32x16 S[4];
  const int zd = 32 * wave + ln;
#pragma unroll
  for (int mt = 0; mt < 4; ++mt) S[mt] = f32x16{};
  if (begin != nullptr) {
#pragma unroll
    for (int mt = 0; mt < 4; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int yd = 32 * mt + 16 * (r >> 3) + 8 * hl + (r & 7);
        S[mt][r] = trans ? begin[zd * kD + yd] : begin[yd * kD + zd];
      }
  }

  f32x16 o = f32x16{};
  uint2 pend[4];                                       // a result that waits to be stored
  uint16_t* pend_at = nullptr;
  auto flush = [&] {
    if (pend_at != nullptr)
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<uint2*>(pend_at + 8 * i) = pend[i];
  };
  const int out_heads = geo.kv_heads * (BACK ? 1 : G);
  uint16_t* const out_row = out + (p.row + (geo.step == nullptr ? int64_t(p.seq) * p.rows : 0)) * out_heads * kD + 32 * wave + 4 * hl;
  float err = 0.f;                                     // of the factors so far, relative
  int c = 0, g = 0;
  uint32_t stage = 0;
  for (int i = 0; i < n_items; ++i) {
    meet<OUT ? 6 : 4>();                               // this item has landed, and the last one's buffer is free
    if (OUT) flush();
    issue(stage == 0 ? 2 : stage - 1);
    const int chunk = BACK ? p.chunk0 + p.chunks - 1 - c : p.chunk0 + c;
    const int n = min(kChunk, p.tokens - chunk * kChunk);
    const bool full = n == kChunk;
    const uint32_t at = stage * kStage;

    // Z^T: z-dim zd, tokens 16 kk + 4 hl .. + 3 and 8 more
    bf16x8 z[2], zf[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) z[kk] = lds_tr2(zt[0] + at + kk * 2048, zt[1] + at + kk * 2048);
    if (!full) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (16 * kk + 8 * (e >> 2) + 4 * hl + (e & 3) >= n) z[kk][e] = (__bf16)0.f;
    }
    zf[0] = z[0];
    zf[1] = z[1];
    int odd = BACK ? -1 : kChunk;                      // the first (last) token whose value zd is not finite
    bool any_odd = false;
    if (OUT) {
      uint32_t bits = 0;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        const uint4 u = __builtin_bit_cast(uint4, z[kk]);
        bits |= odd_halves(u.x) | odd_halves(u.y) | odd_halves(u.z) | odd_halves(u.w);
      }
      any_odd = __ballot((bits & 0x80008000u) != 0) != 0;
      if (any_odd) {                                   // weights of zero would carry it to tokens that do not see it
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (tok::not_finite(float(z[kk][e]))) {
              const int j = 16 * kk + 8 * (e >> 2) + 4 * hl + (e & 3);
              odd = BACK ? max(odd, j) : min(odd, j);
              zf[kk][e] = (__bf16)0.f;
            }
        const int other = __shfl_xor(odd, 32);
        odd = BACK ? max(odd, other) : min(odd, other);
      }
    }

    if (OUT) {
      bf16x8 x[8];
      f32x16 s = f32x16{};
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        x[ks] = lds_row(kr[ks & 3] + at + (ks >> 2) * kHalf);
        const bf16x8 y = lds_row(kr[ks & 3] + at + kTile + (ks >> 2) * kHalf);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y, x[ks], s, 0, 0, 0);
      }
      if (!BACK || g == 0) {                           // (backwards the sum over the query heads begins)
        o = f32x16{};
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
          float m[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) m[e] = S[ks >> 1][8 * (ks & 1) + e];
          const bf16x8 hi = top_part(m, true), lo = last_part(m);
          o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(hi, x[ks], o, 0, 0, 0);
          o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lo, x[ks], o, 0, 0, 0);
        }
        o *= full ? row_whole : row_rest;
      }
      uint32_t mask = see;
      if (BACK && !full) {
        mask = 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int j = 8 * (r >> 2) + 4 * hl + (r & 3);
          mask |= uint32_t(j >= ln && j < n) << r;
        }
      }
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = (mask >> (8 * kk + e)) & 1u ? s[8 * kk + e] * pw[8 * kk + e] : 0.f;
        const bf16x8 hi = top_part(w, true), lo = last_part(w);
        o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(zf[kk], hi, o, 0, 0, 0);
        o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(zf[kk], lo, o, 0, 0, 0);
      }
      if (any_odd) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int of = __shfl(odd, 8 * (r >> 2) + 4 * hl + (r & 3));
          if (BACK ? ln <= of : ln >= of) o[r] = __builtin_nanf("");
        }
      }
      if (!BACK || g == G - 1) {
#pragma unroll
        for (int k = 0; k < 4; ++k) pend[k] = make_uint2(pack_bf16x2(o[4 * k], o[4 * k + 1]), pack_bf16x2(o[4 * k + 2], o[4 * k + 3]));
        pend_at = ln < n ? out_row + (int64_t(chunk * kChunk + ln) * out_heads + (BACK ? h : h * G + g)) * kD : nullptr;
      } else {
        pend_at = nullptr;
      }
    }

    // M past the chunk: forwards behind the last query head, backwards each one's own part
    if (BACK ? g == 0 : g == G - 1) {
      const float want = whole_lo + err;
      const float dec = full ? whole_hi + want : rest_dec;
      if (full) err = want - (dec - whole_hi);
#pragma unroll
      for (int mt = 0; mt < 4; ++mt) S[mt] *= dec;
    }
    if (BACK || g == G - 1) {
      const uint32_t kw = kwt + (full ? 0u : 4u * kChunk);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        float w[8];
        {
          const float4 a = __builtin_bit_cast(float4, *(const tok::lds_u32x4*)(uintptr_t)(kw + 64 * kk));
          const float4 b = __builtin_bit_cast(float4, *(const tok::lds_u32x4*)(uintptr_t)(kw + 64 * kk + 32));
          const float c8[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = float(z[kk][e]) * c8[e];
        }
        bf16x8 part[PARTS];
#pragma unroll
        for (int k = 0; k < PARTS; ++k) part[k] = k == PARTS - 1 ? last_part(w) : top_part(w, true);
#pragma unroll
        for (int mt = 0; mt < 4; ++mt) {
          const uint32_t ya = at + (mt >> 1) * kHalf + kk * 2048;
          const bf16x8 y = lds_tr2(yt[0][mt & 1] + ya, yt[1][mt & 1] + ya);
#pragma unroll
          for (int k = PARTS - 1; k >= 0; --k) S[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y, part[k], S[mt], 0, 0, 0);
        }
      }
    }
    stage = stage == 2 ? 0 : stage + 1;
    if (g + 1 < G) ++g;
    else g = 0, ++c;
  }
  meet<0>();                                           // no copy outlives the walk
  if (OUT) flush();
  if (last != nullptr) {
#pragma unroll
    for (int mt = 0; mt < 4; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) last[(32 * mt + 16 * (r >> 3) + 8 * hl + (r & 7)) * kD + zd] = S[mt][r];
  }
  if (OUT && geo.step == nullptr) {                    // padding
    const int from = max(p.tokens, p.part * geo.chunks * kChunk);
    const int to = p.part == geo.parts - 1 ? p.rows : min(p.rows, (p.part + 1) * geo.chunks * kChunk);
    const int heads = BACK ? 1 : G;
    uint16_t* const row0 = out + int64_t(p.seq) * p.rows * out_heads * kD + int64_t(h) * heads * kD;
    for (int64_t k = tid; k < int64_t(max(to - from, 0)) * heads * 16; k += 256) {
      const int64_t t = k / (heads * 16), w = k % (heads * 16);
      *reinterpret_cast<uint4*>(row0 + (from + t) * out_heads * kD + w * 8) = make_uint4(0, 0, 0, 0);
    }
  }
}

template <bool BACK, int PARTS>
__device__ __forceinline__ void run_walk(const Geo& geo, const Walk& w, int idx, uint8_t* smem) {
  const Place p = place(geo, idx);
  if (p.seq < 0) return;
  const size_t at = (size_t(p.seq) * geo.kv_heads + p.h) * kState;
  const bool ends = p.part == (BACK ? 0 : max(p.parts - 1, 0));
  const float* begin = nullptr;
  if (p.chunks > 0 && w.starts != nullptr) begin = w.starts + size_t(idx) * kState;
  else if (p.held && w.first != nullptr) begin = w.first + at;
  walk<BACK, true, PARTS>(geo, p, w.x, w.y, w.z, w.out, begin, w.trans != 0, ends && w.last != nullptr ? w.last + at : nullptr, smem);
}

__global__ __launch_bounds__(256, 2) void linear_fwd_kernel(WalkArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kShared];
  run_walk<false, 3>(a.geo, a.walk[0], blockIdx.x, smem);
}

// dk, dv and dq of eight workgroups' places one after the other: a place's three lie on one XCD, and share their reads there.
template <int PARTS>
__global__ __launch_bounds__(256, 2) void linear_bwd_kernel(WalkArgs a, int groups) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kShared];
  const int b = blockIdx.x / 24, r = blockIdx.x % 24, idx = 8 * b + r % 8;
  if (idx >= groups) return;
  if (r < 16) run_walk<true, PARTS>(a.geo, a.walk[r / 8], idx, smem);
  else run_walk<false, 2>(a.geo, a.walk[2], idx, smem);
}

template <int PARTS>
__global__ __launch_bounds__(256, 2) void linear_parts_kernel(PartArgs a, int groups) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kShared];
  const int idx = blockIdx.x % groups;
  const auto& s = a.sum[blockIdx.x / groups];
  const Place p = place(a.geo, idx);
  if (p.seq < 0 || p.chunks == 0) return;
  float* const to = s.starts + size_t(idx) * kState;
  if (s.back) {
    if (p.part > 0) walk<true, false, PARTS>(a.geo, p, s.y, s.y, s.z, nullptr, nullptr, false, to, smem);
  } else if (p.part < p.parts - 1) {
    walk<false, false, PARTS>(a.geo, p, s.y, s.y, s.z, nullptr, nullptr, false, to, smem);
  }
}

// Parts' beginnings from their own M, part by part.  A workgroup per (sequence, key head, eighth of M).
constexpr int kEighth = kState / 8;
__global__ __launch_bounds__(256) void linear_scan_kernel(PartArgs a) {
  const Geo& geo = a.geo;
  int k = blockIdx.x;
  const int eighth = k % 8;
  k /= 8;
  const int h = k % geo.kv_heads;
  k /= geo.kv_heads;
  const int e = k % geo.n;
  const auto& s = a.sum[k / geo.n];
  Place p;
  p.part = 0;
  int first;                                           // the sequence's first part in the launch
  if (geo.step == nullptr) {
    p = place(geo, e * geo.parts * geo.kv_heads);
    first = e * geo.parts;
  } else {
    typedef const const_i32* words;
    const words head = (words)geo.step;
    if (e >= head[0]) return;
    entry_of(geo, e, p);
    if (p.seq < 0) return;
    cut(p, max(1, head[3]));
    first = head[kHeader + kEntry * e + 4];
    if (first < 0 || first + p.parts > geo.parts) return;
  }
  const int chunks = geo.step == nullptr ? geo.chunks : max(1, ((const const_i32*)geo.step)[3]);
  const double gd = double(geo.decay[h]);
  const int at = eighth * kEighth + threadIdx.x * 4;
  constexpr int kV = kEighth / 1024;                   // float4 of a thread
  float4 m[kV];
#pragma unroll
  for (int v = 0; v < kV; ++v) m[v] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (s.first != nullptr && p.held) {
    const float* from = s.first + (size_t(p.seq) * geo.kv_heads + h) * kState + at;
#pragma unroll
    for (int v = 0; v < kV; ++v) m[v] = *reinterpret_cast<const float4*>(from + 1024 * v);
  }
  const int tail = p.tokens - (p.parts - 1) * chunks * kChunk;
  const double whole = power(gd, chunks * kChunk), part = power(gd, max(tail, 0));
  for (int i = 0; i < p.parts; ++i) {
    const int q = s.back ? p.parts - 1 - i : i;
    float* const slot = s.starts + (size_t(first + q) * geo.kv_heads + h) * kState + at;
    const double d = q == p.parts - 1 ? part : whole;
    const float hi = float(d), lo = float(d - double(hi));
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      float4* const to = reinterpret_cast<float4*>(slot + 1024 * v);
      const float4 own = i + 1 < p.parts ? *to : make_float4(0.f, 0.f, 0.f, 0.f);
      *to = m[v];
      m[v].x = __builtin_fmaf(m[v].x, hi, __builtin_fmaf(m[v].x, lo, own.x));
      m[v].y = __builtin_fmaf(m[v].y, hi, __builtin_fmaf(m[v].y, lo, own.y));
      m[v].z = __builtin_fmaf(m[v].z, hi, __builtin_fmaf(m[v].z, lo, own.z));
      m[v].w = __builtin_fmaf(m[v].w, hi, __builtin_fmaf(m[v].w, lo, own.w));
    }
  }
}

}  // namespace

hipError_t launch_linear_parts(const PartArgs& a, int32_t groups, bool exact, hipStream_t stream) {
  if (exact) linear_parts_kernel<3><<<dim3(unsigned(groups) * a.n), 256, 0, stream>>>(a, groups);
  else linear_parts_kernel<2><<<dim3(unsigned(groups) * a.n), 256, 0, stream>>>(a, groups);
  return hipGetLastError();
}

hipError_t launch_linear_scan(const PartArgs& a, hipStream_t stream) {
  linear_scan_kernel<<<dim3(unsigned(8 * a.geo.kv_heads) * a.geo.n * a.n), 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_linear_fwd(const WalkArgs& a, int32_t groups, hipStream_t stream) {
  linear_fwd_kernel<<<dim3(unsigned(groups)), 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_linear_bwd(const WalkArgs& a, int32_t groups, bool exact, hipStream_t stream) {
  const unsigned grid = (unsigned(groups) + 7) / 8 * 24;
  if (exact) linear_bwd_kernel<3><<<dim3(grid), 256, 0, stream>>>(a, groups);
  else linear_bwd_kernel<2><<<dim3(grid), 256, 0, stream>>>(a, groups);
  return hipGetLastError();
}

}  // namespace lin
}  // namespace uf
