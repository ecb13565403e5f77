// Gradients of the attention of whole sequences under a sliding window with sinks.
//
// With p = exp(scale q.k - lse) over the keys that a query sees, delta = <dO, O> and
// dS = p (dO.v - delta):
//   dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K,
// where the sums of dK and dV run over the queries of every head of the group.  Rows
// are (token, head of the group) pairs, row = token * G + head, so that a key sees the
// rows from key * G to (key + window) * G as one range and the heads add up by
// themselves.
//
// Kernels, all with 32x32x16 bf16 MFMA and fp32 accumulation:
//  * dq: one workgroup of four waves per 128 rows, two per CU: delta from the rows' dO and
//    O, then per 32 keys S^T = K Q^T, dP^T = V dO^T, dS^T and dQ^T += K^T dS^T (dS in two
//    parts).  It leaves -LSE/scale (-inf where there is no row, so that its weights vanish)
//    and -delta, corrected (see there), in the workspace, the seeds of dkdv's S and dP
//    accumulators;
//  * dkdv: one workgroup of eight waves per 128 keys of a head.  Waves w and w + 4
//    share 32 keys: wave w computes S = Q K^T and P, hands P to wave w + 4 through LDS
//    and accumulates dV^T += dO^T P, while wave w + 4 computes dP = dO V^T and, one unit
//    of 64 rows later, dS = P dP and dK^T += Q^T dS;
//  * sum: where a key tile's rows were cut into parts (the sinks', which every later row
//    sees), the parts' dK and dV in fp32, added in order.
// (A pass that copied Q and dO into records of 128 rows and formed delta took 123 us of
// 2,660 at 16,384 tokens, 32 heads, window 2,048, and 66 KB of workspace a record.)
// Rounding: scores, P, dP, dS and all sums are fp32.  What a product takes is bf16, the
// matrix cores' type for its other operand: P for dV, dS for dK, once each; dS for dQ in two
// parts.  Each such rounding is about as large as the result's own (1.7e-3 of its norm), so
// that dV and dK are 2.2e-3 to 2.5e-3 off and dQ 1.6e-3 to 2.2e-3.  A second part for dV or
// dK would be a quarter more products in a kernel that they bound.
// The transposed operands come from row-major LDS tiles through transposing reads.
// Every output row is owned by one workgroup and sums have one order: no atomics.
#include <type_traits>
#include <utility>

#include "token_common.h"

namespace uf {
namespace tok {
namespace {

using namespace attn;

constexpr int kT = 128;                        // rows of a dq tile, keys of a dkdv tile
constexpr size_t kSeeds = 1024;                // of 128 rows: -LSE/scale, then -delta, fp32
constexpr size_t kPartial = size_t(2) * kT * kD * 4;   // dV, dK of a part, fp32

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) f32x4 lds_f32x4;

// f(from), .., f(to - 1), each index a constant.
template <int FROM, class F, int... I>
__device__ __forceinline__ void each_of(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, FROM + I>{}), ...);
}
template <int FROM, int TO, class F>
__device__ __forceinline__ void each(F f) {
  each_of<FROM>(f, std::make_integer_sequence<int, TO - FROM>{});
}

__device__ inline float bf16f(uint32_t x) { return __uint_as_float(x << 16); }

__device__ inline int length_of(const BwdArgs& a, int b) {
  return a.lengths != nullptr ? min(max(((const const_i32*)a.lengths)[b], 0), a.tokens) : a.tokens;
}

// ---------------------------------------------------------------- dkdv ----

// LDS layout of rows of 128 dimensions: 16-byte chunk c of row r sits at position
// perm(c) ^ f(r) of the row, perm swapping bits 1 and 3 of c and f(r) =
// (r3, r1, r0, r2 ^ r3): row reads and transposing reads are free of bank conflicts.
__device__ inline int swz_perm(int c) { return (c & ~10) | ((c & 2) << 2) | ((c & 8) >> 2); }
__device__ inline int swz_f(int r) { return (r & 8) | ((r & 3) << 1) | (((r >> 2) ^ (r >> 3)) & 1); }
__device__ inline uint32_t swz_elem(int r, int c) {
  return uint32_t(r * 256 + ((swz_perm(c >> 3) ^ swz_f(r & 15)) << 4) + (c & 7) * 2);
}

// dma16 of the lanes in `mask` only (the whole wave is active around it).
__device__ inline void dma16_low(const void* base, uint32_t off, uint32_t lds, uint64_t mask) {
  asm volatile("s_mov_b32 m0, %2\n\ts_mov_b64 exec, %3\n\tglobal_load_lds_dwordx4 %0, %1\n\ts_mov_b64 exec, -1"
               : : "v"(off), "s"(base), "s"(lds), "s"(mask) : "memory");
}

// The key tiles' part of the launch: tiles 0 .. split-1 are cut into up to `parts` parts
// of `part_units` units, the others are whole.
struct Cut {
  int32_t tiles, split, parts, part_units;
  int32_t turn;                                // units of a tile of the window, 0 without a window
};
// Units (64 rows) of a sequence of `len` tokens that see keys of [k0, k0 + 128): first, end.
__host__ __device__ inline void unit_range(int len, int G, int k0, int window, int sinks, int* first, int* end) {
  const int64_t keys_end = k0 + kT < len ? k0 + kT : len;
  int64_t last = int64_t(len);                 // tokens k0 .. last-1
  if (window > 0 && k0 >= sinks && keys_end - 1 + window < last) last = keys_end - 1 + window;
  *first = int(int64_t(k0) * G / 64);
  *end = k0 < len ? int((last * G + 63) / 64) : *first;
}

// What bounds it: four products per pair on the matrix cores, busy 52 % of the cycles
// at 1.95 GHz: 930 to 980 TFLOP/s at 16,384 tokens, 32 heads over 8, window 2,048
// (1,050 to 1,110 us).  Phase s is unit s for
// group 0 and for group 1's dP, unit s-1 for group 1's dS and dK, one workgroup barrier
// after it.  Q rows live in a ring of four units, dO rows in a ring of three, so that a
// unit is requested two phases before it is used.
constexpr int kQRing = 4, kORing = 3, kLRing = 4;
constexpr int kAhead = 4;                      // operands in flight ahead of their product
constexpr int kKW = 4, W = 8, UQ = 64, NB = 2; // key blocks; waves; rows and 32-row blocks of a unit
constexpr uint32_t UB = UQ * 256;              // bytes of a unit's Q (or dO) rows
constexpr int kCopies = UB / 1024 / W;         // copies of a wave per unit and operand

__global__ __launch_bounds__(512, 2) void dkdv_kernel(BwdArgs a, Cut cut, float* partials) {
  __shared__ uint4 sQ[kQRing][UQ * 16];
  __shared__ uint4 sO[kORing][UQ * 16];
  __shared__ uint4 sP[2][kKW][NB * 2][64];     // P operands of a unit: [parity][wave pair][block, kk][lane]
  __shared__ float sLD[kLRing][2 * kT];        // the seeds of the unit's 128 rows, per unit

  const int H = a.kv_heads, G = a.group, BH = a.batch * H;
  const int bh = blockIdx.x % BH;
  const int item = blockIdx.x / BH;            // the parts of tile 0, of tile 1, ..., then whole tiles
  const bool splits = item < cut.split * cut.parts;
  const int t = splits ? item / cut.parts : item - cut.split * (cut.parts - 1);
  const int part = splits ? item % cut.parts : 0;
  const int h = bh % H, b = bh / H;
  const int len = length_of(a, b);
  int first, end;
  unit_range(len, G, t * kT, a.window, a.sinks, &first, &end);
  bool whole = true;
  if (splits && end - first > cut.part_units) {
    whole = false;
    first += part * cut.part_units;
    end = min(end, first + cut.part_units);
    if (first >= end) return;
  } else if (part > 0) {
    return;
  }
  const int U = end - first;
  // The order of the units.  Tiles side by side see rows that lie 128 tokens apart, so that in ascending order each
  // would read a unit when the other has long left it (32 tiles an XCD, 8 MB of Q and dO between the first and the last
  // of them: all of it past the L2, 4.0 GB at 16,384 tokens, 32 heads, window 2,048).  So they begin at the same unit, a
  // multiple of a tile's number of units, and take those before it at the end; without a window they begin at the
  // last unit.
  const int ahead = cut.turn > 0 && whole ? (first + cut.turn - 1) / cut.turn * cut.turn - first : 0;
  const int start = ahead < U ? ahead : 0;
  auto unit_at = [&](int s) {
    if (cut.turn == 0) return end - 1 - s;
    const int u = start + s;
    return first + (u < U ? u : u - U);
  };

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = wave / kKW, kw = wave % kKW;
  const int lane = tid & 63, hl = lane >> 5, ln = lane & 31, rp = lane & 15, gg = (lane >> 4) & 1;
  const int key = t * kT + kw * 32 + ln;       // this lane's key (result column)
  const bool key_ok = key < len;
  const uint8_t* seeds = a.work + size_t(bh) * a.tiles * kSeeds;

  bf16x8 bop[8];                               // B operands of the wave's keys: K (group 0) or V rows
  {
    const uint16_t* p = grp == 0 ? a.k + int64_t(b) * a.k_batch + int64_t(h) * a.k_head + int64_t(key_ok ? key : 0) * a.k_token
                                 : a.v + int64_t(b) * a.v_batch + int64_t(h) * a.v_head + int64_t(key_ok ? key : 0) * a.v_token;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      uint4 u = make_uint4(0, 0, 0, 0);
      if (key_ok) u = *reinterpret_cast<const uint4*>(p + 16 * ks + 8 * hl);
      bop[ks] = as_bf16x8(u);
    }
  }
  // rows that see the lane's key: [row_lo, row_hi); of the wave's keys, rows that see them all
  const int row_lo = int(min(int64_t(key) * G, int64_t(INT32_MAX)));
  const bool forever = a.window == 0 || key < a.sinks;
  const int row_hi = forever ? INT32_MAX : int(min((int64_t(key) + a.window) * G, int64_t(INT32_MAX)));
  const int k_first = t * kT + kw * 32;
  const int64_t all_lo = int64_t(k_first + 31) * G;
  const int64_t all_hi = a.window == 0 || k_first + 31 < a.sinks ? INT64_MAX : (int64_t(k_first) + a.window) * G;

  // Copies of a unit: Q and dO rows, and the seeds.  Copy i of wave w fills LDS chunks
  // [64*(8 i + w), +64), rows 32 i + 4 w + lane/16, whose low four bits do not depend
  // on i.  A row is found from the unit's first token and that token's rows before the
  // unit; rows past the last give way to it.
  const int lr = 4 * wave + (lane >> 4);
  const uint32_t chunk = uint32_t(swz_perm((lane & 15) ^ swz_f(lr & 15)) * 16);
  const uint32_t lq0 = lds_addr(&sQ[0][0]), lo0 = lds_addr(&sO[0][0]), ll0 = lds_addr(&sLD[0][0]);
  const uint8_t* const qb = reinterpret_cast<const uint8_t*>(a.q + int64_t(b) * a.q_batch + int64_t(h) * G * a.q_head);
  const uint8_t* const ob = reinterpret_cast<const uint8_t*>(a.dout + (size_t(b) * a.tokens * a.q_heads + size_t(h) * G) * kD);
  const float per_g = 1.f / float(G);
  const uint32_t qt2 = uint32_t(a.q_token) * 2, qh2 = uint32_t(a.q_head) * 2, ot2 = uint32_t(a.q_heads) * (kD * 2);
  struct Source {
    const uint8_t *q, *o, *seeds;
    uint32_t qslot, oslot;
  };
  uint32_t qoff[kCopies], ooff[kCopies];       // the lane's rows, from the unit's first token on
  bool placed = false;                         // for every whole unit
  // Unit s; past the end the last one is copied again, into a slot that nothing reads any more.
  auto source = [&](int s, uint32_t qslot, uint32_t oslot) {
    const int u = unit_at(min(s, U - 1));
    const int nt = div_nt(uint32_t(u) * UQ, a.group_div), nr = u * UQ - nt * G;
    const int top = len * G - 1 - nt * G;
    const bool same = UQ % G == 0 && top >= UQ - 1;    // the heads of a group divide a unit, and it is whole
    if (!placed || !same) {
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        const int rel = min(nr + 32 * i + lr, top);    // below 64 + G <= 2^17: the quotient is exact in fp32
        const uint32_t tok = uint32_t((float(rel) + 0.5f) * per_g), g = uint32_t(rel) - tok * uint32_t(G);
        qoff[i] = tok * qt2 + g * qh2 + chunk;
        ooff[i] = tok * ot2 + g * (kD * 2) + chunk;
      }
      placed = same;
    }
    return Source{qb + int64_t(nt) * a.q_token * 2, ob + int64_t(nt) * ot2, seeds + size_t(u >> 1) * kSeeds, qslot, oslot};
  };
  constexpr int kIssue = 2 * kCopies + 1;      // copies of a wave per unit
  auto issue = [&](const Source& c, int k) {
    if (k == 2 * kCopies) {
      constexpr uint32_t share = 2 * kT * 4 / W;
      dma16_low(c.seeds + uint32_t(wave) * share, uint32_t(lane) * 16u,
                ll0 + c.qslot * uint32_t(sizeof(sLD[0])) + uint32_t(wave) * share, (uint64_t(1) << (share / 16)) - 1);
      return;
    }
    const uint32_t at = uint32_t(wave) * 1024u + uint32_t(k >> 1) * W * 1024u;
    if (k & 1)
      dma16(c.o, ooff[k >> 1], lo0 + c.oslot * UB + at);
    else
      dma16(c.q, qoff[k >> 1], lq0 + c.qslot * UB + at);
  };
  auto issue_all = [&](const Source& c) {
#pragma unroll
    for (int k = 0; k < kIssue; ++k) issue(c, k);
  };

  f32x16 acc[4];                               // dV^T (group 0) or dK^T (group 1): [dim block][32 dims x 32 keys]
#pragma unroll
  for (int mb = 0; mb < 4; ++mb) acc[mb] = f32x16{};
  const float c2 = a.scale_log2;
  const float pad = key_ok ? 0.f : -INFINITY;  // keys that are none weigh nothing
  // P (at most 1) is handed over in fp16, 2^15 times as large: off by 2^-11 of itself, below weights of 2^-29 by 2^-40 at
  // most, where bf16's 2^-8 put 20 % on dK's error
  constexpr float kHandUp = 0x1p15f, kHandDown = 0x1p-15f;
  uint4* const pslot = &sP[0][kw][0][lane];
  constexpr uint32_t kPStep = sizeof(sP[0]) / 16;
  // Operand addresses within the current ring slots, advanced once per phase: tr,
  // transposing reads (k-slot kappa = row 16 kk + swap23(kappa)) of dO (group 0) or Q
  // (group 1); rt, row reads of Q (group 0) or dO (group 1).
  uint32_t tr[2][4], rt[8];
  {
    const uint32_t bt = grp == 0 ? lo0 : lq0, br = grp == 0 ? lq0 : lo0;
#pragma unroll
    for (int hh = 0; hh < 2; ++hh)
#pragma unroll
      for (int cb = 0; cb < 4; ++cb)
        tr[hh][cb] = bt + swz_elem(8 * hh + 4 * hl + (rp >> 2), 32 * cb + 16 * gg + 4 * (rp & 3));
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) rt[ks] = br + swz_elem(ln, 16 * ks + 8 * hl);
  }
  const uint32_t ld0 = ll0 + uint32_t(16 * hl + (grp == 0 ? 0 : 4 * kT));

  // A unit's products of one wave: 16 row products (X K^T or X V^T), then 16 transposed
  // ones (acc^T += X^T op).  Product i and its operand, read kAhead products earlier.
  constexpr int kRows = 8 * NB, kAll = 16 * NB;
  auto load = [&](int i) -> bf16x8 {
    if (i < kRows) return lds_row(rt[i & 7] + uint32_t((i >> 3) * 32 * 256));
    const int k = i - kRows;
    const uint32_t at = uint32_t(16 * (k >> 2) * 256);
    return lds_tr2(tr[0][k & 3] + at, tr[1][k & 3] + at);
  };
  auto row_product = [&](int i, const bf16x8& x, f32x16 (&v)[NB]) {
    v[i >> 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, bop[i & 7], v[i >> 3], 0, 0, 0);
  };
  auto tr_product = [&](int i, const bf16x8& x, const bf16x8 (&op)[NB][2]) {
    const int k = i - kRows, mb = k & 3;
    acc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, op[k >> 3][(k >> 2) & 1], acc[mb], 0, 0, 0);
  };
  auto seed = [&](uint32_t ld, f32x16 (&v)[NB]) {
#pragma unroll
    for (int qb = 0; qb < NB; ++qb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 c4 = *(const lds_f32x4*)(uintptr_t)(ld + uint32_t(4 * (qb * 32 + 8 * g)));
        v[qb][4 * g] = c4.x;
        v[qb][4 * g + 1] = c4.y;
        v[qb][4 * g + 2] = c4.z;
        v[qb][4 * g + 3] = c4.w;
      }
  };
  auto put = [&](bf16x8 (&op)[2], int e, float x0, float x1) {
    op[e >> 2][2 * (e & 3)] = (__bf16)x0;
    op[e >> 2][2 * (e & 3) + 1] = (__bf16)x1;
  };
  auto advance = [&](bool wrap, int ring) {
    const uint32_t d = wrap ? uint32_t(-(ring - 1) * int(UB)) : UB;
#pragma unroll
    for (int k = 0; k < 8; ++k) rt[k] += d;
  };
  auto advance_tr = [&](bool wrap, int ring) {
    const uint32_t d = wrap ? uint32_t(-(ring - 1) * int(UB)) : UB;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int cb = 0; cb < 4; ++cb) tr[k][cb] += d;
  };
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
  constexpr int kGap = kAll / kIssue;          // products between two of the next unit's copies
  // Group 0, unit at row `row`: S, P, the P slot, dV.
  auto unit0 = [&](int row, uint32_t ld, uint32_t par, const Source& next) {
    f32x16 sv[NB];
    bf16x8 op[NB][2], x[kAll];
    seed(ld, sv);
    const bool full = row >= all_lo && row + UQ <= all_hi;
    uint64_t see = 0;
    if (!full) see = (bits_upto(row_hi - row) & ~bits_upto(row_lo - row)) >> (4 * hl);
    auto mask = [&](int qb) {
      if (full) return;
      const uint32_t w = uint32_t(see >> (32 * qb));
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!((w >> (8 * (r >> 2) + (r & 3))) & 1u)) sv[qb][r] = -INFINITY;
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) x[i] = load(i);
    f16x8 hand;
    auto weights = [&](int qb, int e) {
      const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[qb][2 * e], c2, pad));
      const float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[qb][2 * e + 1], c2, pad));
      put(op[qb], e, w0, w1);
      hand[2 * (e & 3)] = (_Float16)__builtin_fmaf(w0, kHandUp, 0.f);        // (one mixed-type instruction each)
      hand[2 * (e & 3) + 1] = (_Float16)__builtin_fmaf(w1, kHandUp, 0.f);
      if ((e & 3) == 3) pslot[par * kPStep + (qb * 2 + (e >> 2)) * 64] = __builtin_bit_cast(uint4, hand);
    };
    fence();
    each<0, kAll>([&](auto ic) __attribute__((always_inline)) {
      constexpr int i = decltype(ic)::value;
      if constexpr (i == 8) mask(0);
      if constexpr (i == 16) mask(1);
      if constexpr (i < kRows) row_product(i, x[i], sv);
      else tr_product(i, x[i], op);
      if constexpr (i + kAhead < kAll) x[i + kAhead] = load(i + kAhead);
      if constexpr (i >= 8 && i < kAll - 8) weights((i - 8) >> 3, i & 7);
      if constexpr (i % kGap == kGap - 1 && i / kGap < kIssue) issue(next, i / kGap);
      fence();
    });
  };
  // Group 1: dP - delta of a unit (kDp) into nv, and dS (from the P slot and the dP of
  // the unit before, ov) and dK of that unit (kDk).
  auto unit1 = [&](auto dp, auto dk, uint32_t ld, uint32_t par, const f32x16 (&ov)[NB], f32x16 (&nv)[NB],
                   const Source& next) {
    constexpr bool kDp = decltype(dp)::value, kDk = decltype(dk)::value;
    constexpr int i0 = kDp ? 0 : kRows, i1 = kDk ? kAll : kRows;
    f16x8 pk[NB][2];
    bf16x8 op[NB][2], x[kAll];
    if (kDk) {
#pragma unroll
      for (int qb = 0; qb < NB; ++qb)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
          pk[qb][kk] = __builtin_bit_cast(f16x8, pslot[par * kPStep + (qb * 2 + kk) * 64]);
    }
    if (kDp) seed(ld, nv);
#pragma unroll
    for (int i = i0; i < i0 + kAhead; ++i) x[i] = load(i);
    auto ds = [&](int qb, int e) {
      put(op[qb], e, __builtin_fmaf(float(pk[qb][e >> 2][2 * (e & 3)]), kHandDown, 0.f) * ov[qb][2 * e],
          __builtin_fmaf(float(pk[qb][e >> 2][2 * (e & 3) + 1]), kHandDown, 0.f) * ov[qb][2 * e + 1]);
    };
    fence();
    if (kDk && !kDp) {
#pragma unroll
      for (int k = 0; k < kRows; ++k) ds(k >> 3, k & 7);
    }
    each<i0, i1>([&](auto ic) __attribute__((always_inline)) {
      constexpr int i = decltype(ic)::value;
      if constexpr (i < kRows) row_product(i, x[i], nv);
      else tr_product(i, x[i], op);
      if constexpr (i + kAhead < i1) x[i + kAhead] = load(i + kAhead);
      if constexpr (kDk && i < kRows) ds(i >> 3, i & 7);
      if constexpr (kDp && kDk && i % kGap == kGap - 1 && i / kGap < kIssue) issue(next, i / kGap);
      fence();
    });
  };
  auto run = [&](auto group) {
    constexpr int G0 = decltype(group)::value;
    f32x16 dpv[NB];
    uint32_t om = 0;                           // s % 3
    auto phase = [&](int s, auto start) {
      constexpr bool kFirst = decltype(start)::value;
      // unit s has landed; the slots of unit s+2 are free
      const Source next = source(s + 2, uint32_t(s + 2) & 3u, om == 0 ? 2u : om - 1u);
      const int u = unit_at(s);
      const uint32_t ld = ld0 + (uint32_t(s) & 3u) * uint32_t(sizeof(sLD[0])) + uint32_t(u & 1) * uint32_t(4 * UQ);
      if constexpr (G0 == 0) {
        unit0(u * UQ, ld, uint32_t(s) & 1u, next);
        advance((s & 3) == 3, kQRing);
        advance_tr(om == 2, kORing);
      } else {
        f32x16 nv[NB];
        if constexpr (kFirst) issue_all(next);
        unit1(std::true_type{}, std::bool_constant<!kFirst>{}, ld, uint32_t(s - 1) & 1u, dpv, nv, next);
#pragma unroll
        for (int qb = 0; qb < NB; ++qb) dpv[qb] = nv[qb];
        if constexpr (!kFirst) advance_tr((s & 3) == 0, kQRing);
        advance(om == 2, kORing);
      }
      om = om == 2 ? 0 : om + 1;
      meet<kIssue>();                          // unit s+1 has landed; unit s+2 may be in flight
    };
    meet<kIssue>();                            // unit 0 has landed, unit 1 may be in flight
    phase(0, std::true_type{});
    for (int s = 1; s < U; ++s) phase(s, std::false_type{});
    if constexpr (G0 == 1) {
      f32x16 nv[NB];
      unit1(std::false_type{}, std::true_type{}, 0, uint32_t(U - 1) & 1u, dpv, nv, Source{});
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0)); // no copy outlives the workgroup
  };
  if (U > 0) {
    issue_all(source(0, 0, 0));
    issue_all(source(1, 1, 1));
    if (grp == 0) run(std::integral_constant<int, 0>{});
    else run(std::integral_constant<int, 1>{});
    // A row that does not see a key has a weight of zero there, and zero times what is not finite in the row is not zero:
    // where any of the wave's results is not finite they are formed again row by row, each from the rows that see its key
    // (4 us a row; a few are enough to make the launch 20 times as long).
    float probe = 0.f;
#pragma unroll
    for (int mb = 0; mb < 4; ++mb)
#pragma unroll
      for (int r = 0; r < 16; ++r) probe += acc[mb][r];
    if (__ballot(not_finite(probe)) != 0) {
      bf16x8 kf[8], vf[8];
      const int64_t at = key_ok ? key : 0;
      const uint16_t* kp = a.k + int64_t(b) * a.k_batch + int64_t(h) * a.k_head + at * a.k_token + 8 * hl;
      const uint16_t* vp = a.v + int64_t(b) * a.v_batch + int64_t(h) * a.v_head + at * a.v_token + 8 * hl;
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        kf[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(kp + 16 * ks));
        vf[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(vp + 16 * ks));
      }
      float out[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) out[i] = 0.f;
      const int rows_end = min(end * UQ, len * G);
      for (int row = first * UQ; row < rows_end; ++row) {
        const bool on = key_ok && row >= row_lo && row < row_hi;
        if (__ballot(on) == 0) continue;
        const int tok = div_nt(uint32_t(row), a.group_div), g = row - tok * G;
        const uint8_t* qr = qb + int64_t(tok) * a.q_token * 2 + size_t(g) * qh2;
        const uint8_t* orow = ob + int64_t(tok) * ot2 + size_t(g) * (kD * 2);
        const float* seed = reinterpret_cast<const float*>(seeds + size_t(row / kT) * kSeeds) + row % kT;
        const float w = __builtin_amdgcn_exp2f((dot_row(kf, qr, hl) + seed[0]) * c2);
        if (grp == 0) add_row<16>(w, orow, on, 4 * hl, out);
        else add_row<16>(w * (dot_row(vf, orow, hl) + seed[kT]), qr, on, 4 * hl, out);
      }
#pragma unroll
      for (int mb = 0; mb < 4; ++mb)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[mb][r] = out[16 * mb + r];
    }
  }

  // lane holds key `key`, dims mb*32 + 8*(r/4) + 4*hl + r%4
  if (!whole) {
    float* dst = partials + (((size_t(bh) * cut.split + t) * cut.parts + part) * 2 + grp) * (kT * kD) + (kw * 32 + ln) * kD;
#pragma unroll
    for (int mb = 0; mb < 4; ++mb)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4*>(dst + mb * 32 + 8 * g + 4 * hl) =
            make_float4(acc[mb][4 * g], acc[mb][4 * g + 1], acc[mb][4 * g + 2], acc[mb][4 * g + 3]);
    return;
  }
  if (key < a.tokens) {
    uint16_t* dst = (grp ? a.dk : a.dv) + ((size_t(b) * a.tokens + key) * H + h) * kD + 4 * hl;
    const float f = grp ? a.scale : 1.f;
#pragma unroll
    for (int mb = 0; mb < 4; ++mb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        uint2 u = make_uint2(0, 0);
        if (key_ok) {
          u.x = pack_bf16x2(acc[mb][4 * g] * f, acc[mb][4 * g + 1] * f);
          u.y = pack_bf16x2(acc[mb][4 * g + 2] * f, acc[mb][4 * g + 3] * f);
        }
        *reinterpret_cast<uint2*>(dst + mb * 32 + 8 * g) = u;
      }
  }
}

// The parts of a cut tile: a thread adds four dims of one key of dK or dV, part by part.
__global__ __launch_bounds__(256) void sum_kernel(BwdArgs a, Cut cut, const float* partials) {
  const int H = a.kv_heads;
  const int rows = blockIdx.x * 8;                     // rows (bh, tile, kind, key), eight a workgroup
  const int r = rows + (threadIdx.x >> 5), c = (threadIdx.x & 31) * 4;
  const int k = r % kT, grp = (r / kT) & 1, bt = r / (2 * kT);
  const int t = bt % cut.split, bh = bt / cut.split, h = bh % H, b = bh / H;
  const int len = length_of(a, b), key = t * kT + k;
  int first, end;
  unit_range(len, a.group, t * kT, a.window, a.sinks, &first, &end);
  if (end - first <= cut.part_units || key >= a.tokens) return;
  const int n = (end - first + cut.part_units - 1) / cut.part_units;
  const float* src = partials + ((size_t(bt) * cut.parts) * 2 + grp) * (kT * kD) + k * kD + c;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p0 = 0; p0 < n; p0 += 4) {
    float4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const float4*>(src + size_t(min(p0 + i, n - 1)) * 2 * (kT * kD));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float on = p0 + i < n ? 1.f : 0.f;
      s.x = __builtin_fmaf(v[i].x, on, s.x);
      s.y = __builtin_fmaf(v[i].y, on, s.y);
      s.z = __builtin_fmaf(v[i].z, on, s.z);
      s.w = __builtin_fmaf(v[i].w, on, s.w);
    }
  }
  const float f = key < len ? (grp ? a.scale : 1.f) : 0.f;
  uint2 u;
  u.x = pack_bf16x2(s.x * f, s.y * f);
  u.y = pack_bf16x2(s.z * f, s.w * f);
  *reinterpret_cast<uint2*>((grp ? a.dk : a.dv) + ((size_t(b) * a.tokens + key) * H + h) * kD + c) = u;
}

// ------------------------------------------------------------------ dq ----
//
// The walk, the unit's layout and its copies are the forward's (token_attn.hip).  What
// bounds it: four products per pair on the matrix cores, busy 63 % of the cycles at 1.8
// GHz: 1,115 TFLOP/s at 16,384 tokens, 32 heads over 8, window 2,048 (924 us).  Two
// operands are read ahead: three to six, which the registers hold too, changed nothing.
// dS goes to its product in two bf16 parts, its rounding and the remainder: rounded once it
// puts 1.6e-3 on dQ.  The remainder's product costs 200 us of a backward of 1,950 at that
// size, in whichever order the two are issued.
//
// delta from the rounded O is off by 2e-3 of |dO| |O|, which is large where a row sees few
// keys (3.1e-3 of dQ and dK at a window of 6, 2.6e-3 at 16).  But P sums to 1, so that the sum
// of a row's dS, which the walk forms beside dS (up to 2 % of the backward), is what delta
// was off by: dkdv gets delta with that.  dQ has been formed with the other by then, and
// what it is off by is small where rows see many keys; tiles that see kFewKeys at most, whose walks
// are short, walk again with the corrected delta.  (dQ at 95 to 160 tokens 2.4e-3 without and
// 1.7e-3 with; 2 x 1,531 tokens, 6 heads, window 200: 44.1 and 44.8 us, 16,384 tokens 1,974 and
// 1,965.)
constexpr uint32_t kUnitBytes = 32768;
constexpr int kFewKeys = 128;

__global__ __launch_bounds__(256, 2) void dq_kernel(BwdArgs a) {
  __shared__ uint4 sbuf[2][kUnitBytes / 16];

  const int H = a.kv_heads, G = a.group, BH = a.batch * H;
  const int bh = blockIdx.x % BH;
  const int tile = a.tiles - 1 - blockIdx.x / BH;      // long ranges first
  const int h = bh % H, b = bh / H;
  const int len = length_of(a, b), rows = len * G, row0 = tile * kT;
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, hl = lane >> 5, ln = lane & 31, rp = lane & 15, g = (lane >> 4) & 1;
  const int q = wave * 32 + ln, row = row0 + q;
  auto target = [&](int r) {                           // of row r's gradient
    const int t = int(uint32_t(r) / uint32_t(G));
    return a.dq + ((size_t(b) * a.tokens + t) * a.q_heads + h * G + r - t * G) * kD + 4 * hl;
  };
  if (row0 >= rows) {                                  // padding
    if (row < a.tokens * G) {
      uint16_t* const dst = target(row);
#pragma unroll
      for (int i = 0; i < 16; ++i) *reinterpret_cast<uint2*>(dst + 8 * i) = make_uint2(0, 0);
    }
    return;
  }
  const int first = row0 / G, last = (min(row0 + kT, rows) - 1) / G;
  const Range range = key_range(first, last, a.window, a.sinks, kKeyUnit);
  const int w0 = row0 + wave * 32;
  const int pmin = w0 / G, pmax = (min(w0 + 32, rows) - 1) / G;
  const int pos = min(int(uint32_t(row) / uint32_t(G)), pmax);

  // Q^T and dO^T: lane holds row ln, dims 16 ks + 8 hl ..; delta from the chunks of dO and O
  bf16x8 qf[8], of[8];
  float nl = -INFINITY, nd = 0.f;
  {
    const int t = min(int(uint32_t(row) / uint32_t(G)), len - 1), head = h * G + (row < rows ? row - t * G : 0);
    const uint16_t* qp = a.q + int64_t(b) * a.q_batch + int64_t(t) * a.q_token + int64_t(head) * a.q_head + 8 * hl;
    const size_t off = ((size_t(b) * a.tokens + t) * a.q_heads + head) * kD + 8 * hl;
    uint4 vo[8];
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      qf[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(qp + 16 * ks));
      of[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(a.dout + off + 16 * ks));
      vo[ks] = *reinterpret_cast<const uint4*>(a.o + off + 16 * ks);
    }
    if (row < rows) nl = -a.lse[(size_t(b) * a.q_heads + head) * a.tokens + t] / a.scale;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      const uint32_t o[4] = {vo[ks].x, vo[ks].y, vo[ks].z, vo[ks].w};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        nd -= bf16f(o[e] & 0xffffu) * float(of[ks][2 * e]) + bf16f(o[e] >> 16) * float(of[ks][2 * e + 1]);
    }
    nd = pair_sum(nd);
    if (hl == 0) reinterpret_cast<float*>(a.work + (size_t(bh) * a.tiles + tile) * kSeeds)[q] = nl;
  }
  const float nd0 = nd;                                // from O as it was rounded
  const float c2 = a.scale_log2;
  nl *= c2;

  const uint32_t lds0 = lds_addr(&sbuf[0][0]);
  uint32_t kr[4], kt[2][2];                            // K rows (V rows 16 KB behind); K transposed
#pragma unroll
  for (int k = 0; k < 4; ++k) kr[k] = lds0 + uint32_t(ln * 128 + 16 * ((2 * k + hl) ^ swz_k(ln & 15)));
#pragma unroll
  for (int hh = 0; hh < 2; ++hh)
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int r = 8 * hh + 4 * hl + (rp >> 2);
      kt[hh][m] = lds0 + uint32_t(r * 128 + 16 * ((4 * m + 2 * g + ((rp >> 1) & 1)) ^ swz_k(r)) + 8 * (rp & 1));
    }
  struct Unit {
    const uint8_t *k, *v;
    int key0;
  };
  const uint32_t kstep = uint32_t(a.k_token) * 2, vstep = uint32_t(a.v_token) * 2;
  auto unit_of = [&](int u) {
    Unit x;
    x.key0 = (u < range.sink ? u : u - range.sink + range.from) * kKeyUnit;
    x.k = reinterpret_cast<const uint8_t*>(a.k + int64_t(b) * a.k_batch + int64_t(x.key0) * a.k_token + int64_t(h) * a.k_head);
    x.v = reinterpret_cast<const uint8_t*>(a.v + int64_t(b) * a.v_batch + int64_t(x.key0) * a.v_token + int64_t(h) * a.v_head);
    return x;
  };
  const uint32_t chunk = uint32_t(16 * ((lane & 7) ^ swz_k(8 * (wave & 1) + (lane >> 3))));
  struct Offsets {
    uint32_t k[2], v[2];
  };
  auto offsets = [&](const Unit& u) {
    Offsets o;
    const bool sink = u.key0 < range.from * kKeyUnit;
    const int top = sink ? min(63, a.sinks - 1 - u.key0) : min(63, last - u.key0);
    const int low = sink ? 0 : range.low - u.key0, srel = a.sinks - u.key0;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      int r = 8 * (wave + 4 * t) + (lane >> 3);
      r = min(r < srel ? r : max(r, low), top);
      o.k[t] = uint32_t(r) * kstep + chunk;
      o.v[t] = uint32_t(r) * vstep + chunk;
    }
    return o;
  };
  auto issue = [&](const Unit& u, const Offsets& o, uint32_t buf, int k) {
    const int t = k & 3;
    const uint32_t to = lds0 + buf * kUnitBytes + uint32_t(wave) * 1024u + uint32_t(t) * 4096u;
    if (k < 4)
      dma16(u.k + (t >> 1) * 128, o.k[t & 1], to);
    else
      dma16(u.v + (t >> 1) * 128, o.v[t & 1], to + 16384u);
  };
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };

  f32x16 dqt[4];                                       // [4 dim blocks][32 dims x 32 rows]
  float eps = 0.f;                                     // the row's sum of dS

  // Products of a unit: S0, dP0, S1, dP1, dQ0, dQ1 (eight each, per 32-key block).
  constexpr int kSP = 32, kReads = 2;
  auto load = [&](int k) -> bf16x8 {
    if (k < kSP) {
      const int n = k >> 4, ks = k & 7;
      return lds_row(kr[ks & 3] + uint32_t(n * 4096 + (ks >> 2) * 8192 + ((k & 8) ? 16384 : 0)));
    }
    const int m = k - kSP, n = m >> 3, kk = (m >> 2) & 1, mb = m & 3;
    const uint32_t at = uint32_t(n * 4096 + kk * 2048 + (mb >> 1) * 8192);
    return lds_tr2(kt[0][mb & 1] + at, kt[1][mb & 1] + at);
  };
  auto body = [&](const Unit& cur, const Unit& next, uint32_t nbuf) {
    f32x16 sv[2], dp[2];
    bf16x8 op[2][2], rest[2][2], x[48];   // dS and what its rounding leaves
    const Offsets no = offsets(next);
    const bool full = cur.key0 + 63 <= pmin &&
                      (a.window == 0 || cur.key0 >= pmax - a.window + 1 || cur.key0 + 63 < a.sinks);
    uint64_t see = 0;
    if (!full) see = seen_bits(pos, cur.key0, a.window, a.sinks) >> (4 * hl);
    auto mask = [&](int n) {
      if (full) return;
      const uint32_t w = uint32_t(see >> (32 * n));
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!((w >> (8 * (r >> 2) + (r & 3))) & 1u)) sv[n][r] = -INFINITY;
    };
    auto weight = [&](int n, int r) { sv[n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[n][r], c2, nl)); };
    auto ds = [&](int n, int e) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int at = 2 * (e & 3) + i;
        const float d = sv[n][2 * e + i] * (dp[n][2 * e + i] + nd);
        eps += d;
        op[n][e >> 2][at] = (__bf16)d;
        rest[n][e >> 2][at] = (__bf16)(d - float(op[n][e >> 2][at]));
      }
    };
#pragma unroll
    for (int k = 0; k < kReads; ++k) x[k] = load(k);
    fence();
    auto eight = [&](auto from) {                      // products from .. from + 7
      constexpr int k0 = decltype(from)::value;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int k = k0 + j;
        if constexpr (k0 < kSP) {
          const int n = k0 >> 4;
          if constexpr ((k0 & 8) == 0)
            sv[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[k], qf[j], j ? sv[n] : f32x16{}, 0, 0, 0);
          else
            dp[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[k], of[j], j ? dp[n] : f32x16{}, 0, 0, 0);
        } else {
          dqt[j & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[k], op[(k0 - kSP) >> 3][j >> 2], dqt[j & 3], 0, 0, 0);
          dqt[j & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[k], rest[(k0 - kSP) >> 3][j >> 2], dqt[j & 3], 0, 0, 0);
        }
        if (k + kReads < 48) x[k + kReads] = load(k + kReads);
        if constexpr (k0 < kSP && (k0 & 8) != 0) {     // beside dP of a block: its weights
          weight(k0 >> 4, 2 * j);
          weight(k0 >> 4, 2 * j + 1);
        }
        if constexpr (k0 == 16) ds(0, j);              // beside S of block 1
        if constexpr (k0 == 32) ds(1, j);              // beside dQ of block 0
        if (k % 2 == 1 && k < 16) issue(next, no, nbuf, k >> 1);
        fence();
      }
      if constexpr (k0 < kSP && (k0 & 8) != 0) asm volatile("" : "+v"(sv[k0 >> 4]));
      if constexpr (k0 == 16) asm volatile("" : "+v"(op[0][0]), "+v"(op[0][1]), "+v"(rest[0][0]), "+v"(rest[0][1]));
    };
    eight(std::integral_constant<int, 0>{});
    mask(0);
    eight(std::integral_constant<int, 8>{});
    eight(std::integral_constant<int, 16>{});
    mask(1);
    eight(std::integral_constant<int, 24>{});
    eight(std::integral_constant<int, 32>{});
    eight(std::integral_constant<int, 40>{});
  };
  const int U = range.count;
  const bool twice = min(int64_t(last) + 1, a.window > 0 ? int64_t(a.window) + a.sinks : INT64_MAX) <= kFewKeys;
  for (int pass = twice ? 0 : 1;; ++pass) {
#pragma unroll
    for (int mb = 0; mb < 4; ++mb) dqt[mb] = f32x16{};
    Unit cur = unit_of(0), next = unit_of(min(1, U - 1));
    {
      const Offsets co = offsets(cur);
#pragma unroll
      for (int k = 0; k < 8; ++k) issue(cur, co, 0, k);
    }
    int u = 0;
    do {
      meet<0>();                                       // unit u has landed; the other buffer is free
      const uint32_t nbuf = uint32_t(u + 1) & 1u;
      body(cur, next, nbuf);                           // past the end the last unit is copied again, and not read
      const uint32_t d = (u & 1) ? uint32_t(-int(kUnitBytes)) : kUnitBytes;
#pragma unroll
      for (int k = 0; k < 4; ++k) kr[k] += d;
#pragma unroll
      for (int k = 0; k < 4; ++k) kt[k >> 1][k & 1] += d;
      cur = next;
      next = unit_of(min(u + 2, U - 1));
    } while (++u < U);
    if (pass == 1) break;
    if (U & 1) {                                       // the units start in buffer 0 again
#pragma unroll
      for (int k = 0; k < 4; ++k) kr[k] -= kUnitBytes;
#pragma unroll
      for (int k = 0; k < 4; ++k) kt[k >> 1][k & 1] -= kUnitBytes;
    }
    nd -= pair_sum(eps);
    eps = 0.f;
    meet<0>();                                         // both buffers are free
  }
  __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));           // no copy outlives the workgroup
  eps = pair_sum(eps);
  // What is not finite in a key that a row does not see: as in the forward and in dkdv, key by key.
  float probe = 0.f;
#pragma unroll
  for (int mb = 0; mb < 4; ++mb)
#pragma unroll
    for (int r = 0; r < 16; ++r) probe += dqt[mb][r];
  if (__ballot(not_finite(probe)) != 0) {
    float out[64];
    nd = nd0;
    for (int pass = twice ? 0 : 1;; ++pass) {
      eps = 0.f;
#pragma unroll
      for (int i = 0; i < 64; ++i) out[i] = 0.f;
      for (int i = 0; i < U; ++i) {
        const Unit c = unit_of(i);
        const uint64_t see = seen_bits(pos, c.key0, a.window, a.sinks);
        for (int k = 0; k < kKeyUnit; ++k) {
          const bool on = row < rows && ((see >> k) & 1u);
          if (__ballot(on) == 0) continue;
          const uint8_t* kr1 = c.k + uint32_t(k) * kstep;
          const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(dot_row(qf, kr1, hl), c2, nl));
          const float d = w * (dot_row(of, c.v + uint32_t(k) * vstep, hl) + nd);
          if (on) eps += d;
          add_row<16>(d, kr1, on, 4 * hl, out);
        }
      }
      if (pass == 1) break;
      nd -= eps;
    }
#pragma unroll
    for (int mb = 0; mb < 4; ++mb)
#pragma unroll
      for (int r = 0; r < 16; ++r) dqt[mb][r] = out[16 * mb + r];
  }
  if (hl == 0) reinterpret_cast<float*>(a.work + (size_t(bh) * a.tiles + tile) * kSeeds)[kT + q] = nd - eps;
  int r_out = row;                                     // (its address is formed here, not held across the walk)
  asm volatile("" : "+v"(r_out));
  if (r_out >= a.tokens * G) return;
  uint16_t* const dst = target(r_out);
  const bool on = r_out < rows;                        // padding gets zeros
#pragma unroll
  for (int mb = 0; mb < 4; ++mb)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint2 u;
      u.x = on ? pack_bf16x2(dqt[mb][4 * k] * a.scale, dqt[mb][4 * k + 1] * a.scale) : 0;
      u.y = on ? pack_bf16x2(dqt[mb][4 * k + 2] * a.scale, dqt[mb][4 * k + 3] * a.scale) : 0;
      *reinterpret_cast<uint2*>(dst + mb * 32 + 8 * k) = u;
    }
}

// The sinks' key tiles are cut into parts of about a window tile's units, so that none
// outlasts the launch: a tile of the window is seen by (window + 127) G / 64 units, the
// sinks' by every unit behind them.  No more parts than give the sinks' tiles 1,024
// workgroups: many such tiles fill the GPU as they are, and a part's results are 128 KB.
constexpr int kMostParts = 1024;
Cut cut_of(const BwdArgs& a) {
  Cut c{};
  c.tiles = (a.tokens + kT - 1) / kT;
  c.parts = 1;
  if (a.window == 0) return c;
  const int64_t turn = ((int64_t(a.window < a.tokens ? a.window : a.tokens) + kT - 1) * a.group + 63) / 64;
  c.turn = int(turn);
  if (a.sinks == 0) return c;
  const int sinks = (a.sinks + kT - 1) / kT < c.tiles ? (a.sinks + kT - 1) / kT : c.tiles;
  int first, end;
  unit_range(a.tokens, a.group, 0, a.window, a.sinks, &first, &end);
  const int64_t near = (int64_t(a.window) + kT) * a.group / 64 + 1, all = end - first;
  const int64_t room = kMostParts / (int64_t(a.batch) * a.kv_heads * sinks);
  const int64_t parts = all / near < room ? all / near : room;
  if (parts < 2) return c;
  c.split = sinks;
  c.part_units = int((all + parts - 1) / parts);
  c.parts = int((all + c.part_units - 1) / c.part_units);
  return c;
}
size_t seed_bytes(const BwdArgs& a) { return size_t(a.batch) * a.kv_heads * a.tiles * kSeeds; }

}  // namespace

size_t bwd_work_bytes(const BwdArgs& a) {
  const Cut c = cut_of(a);
  return seed_bytes(a) + size_t(a.batch) * a.kv_heads * c.split * c.parts * kPartial;
}

hipError_t launch_window_bwd(const BwdArgs& a, hipStream_t stream) {
  const Cut c = cut_of(a);
  const unsigned BH = unsigned(a.batch) * unsigned(a.kv_heads);
  float* partials = reinterpret_cast<float*>(a.work + seed_bytes(a));
  dq_kernel<<<BH * unsigned(a.tiles), 256, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  dkdv_kernel<<<BH * unsigned(c.split * c.parts + c.tiles - c.split), 512, 0, stream>>>(a, c, partials);
  e = hipGetLastError();
  if (e != hipSuccess || c.split == 0) return e;
  sum_kernel<<<BH * unsigned(c.split) * 32u, 256, 0, stream>>>(a, c, partials);
  return hipGetLastError();
}

}  // namespace tok
}  // namespace uf
