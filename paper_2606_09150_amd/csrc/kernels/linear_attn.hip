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
// carries them on from part to part (or, of few parts, each walk sums those before it), and
// the walks begin from those.
//
// Work split: a workgroup per (sequence, part, key head), eight waves, each with 16
// z-dims of M and of the result; P^T = Y X^T is formed once, a quarter by each of four waves, and
// shared through LDS.  All products are v_mfma_f32_16x16x32_bf16: O^T = M^T X^T + Z^T P^T and
// M += Y^T (c Z), X and Y rows and transposed reads of Y and Z from LDS.  M stays in
// accumulators: its y-dims lie there as the k-slots of the next product want them (Y^T's rows
// are read in that order), so it is multiplied without leaving registers.  (Four waves of 32
// z-dims, by 32x32x16: two waves a SIMD hide less; one sequence of 32,768 tokens, 16 heads, in 8 parts 397 us
// for 336, in 32 216 for 207; the backward pass of 2 x 8,192 tokens, 32 heads, the same 465.  All of Y
// is read by twice the waves, and half of these reads' cycles are bank conflicts, for a wave's rows have
// one 8-byte half of each 16; rows of 16 dimensions side by side, with X read by 8 bytes, have none, a third
// less of LDS cycles, and the same times.)
//
// What bounds it is the issue of instructions.  A matrix instruction of 16x16x32 takes 16 cycles, and keeps 11 of
// them from vector instructions of every wave of its SIMD (32x32x16: 15 of 32; measured by loops of both).  A chunk
// has 46 of a wave, and 261 vector ones of 4 cycles, of which M's parts are 96: 3,100 cycles for a SIMD's two
// waves of a workgroup, where 4,200 pass (1 x 32,768 tokens, 16 heads, 159 us); each chunk has two barriers.
//
// Rounding: M and P enter their products as two bf16 parts each (one alone would add as much
// error as the result's own rounding), c Z in three, since M is a result in fp32 and carries
// each error on (two backwards, where it is none, as dq's never is).  L^32 in fp32 would be off by the same 2^-25 in each
// of thousands of chunks: the part of it that fp32 drops is carried on and added to the next factor.
//
// Memory: three tiles of 8 KB an item (a chunk and query head), in two blocks of 64 dimensions in 128-byte
// rows (swz_k), copied by global_load_lds two items ahead into three buffers.  Forward walks of several
// query heads take two an item, which share y, z, M's parts and the barriers: four tiles, an item ahead
// into two buffers.  Rows past the sequence's end take its last row, and weigh nothing.
#include "linear_place.h"
#include "token_common.h"

#include <algorithm>
#include <type_traits>

namespace uf {
namespace lin {
namespace {

using namespace attn;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) u32x2 lds_u32x2;

using tok::lds_row;
using tok::lds_tr2;
using tok::swz_k;

constexpr int kThreads = kWalkThreads;
constexpr uint32_t kTile = 8192, kHalf = 4096;
// LDS behind the stages: P, a row of 32 values in two parts (and 16 bytes, so that rows begin in banks of their own) for each
// token; then, in floats, L^e for e = 0 .. 32 and M's factors, the key weights of a period's chunks and of the last one, and what M is read with.
constexpr uint32_t kRow = 144;
constexpr int kPowers = 36;
constexpr int kPeriod = 4, kWeights = (kPeriod + 1) * kChunk;
// HEADS: query heads of an item.  One: tiles of x, y and z in three stages; two, whose x share y, z and M's parts: four tiles in two.
template <int HEADS>
struct Lds {
  static constexpr int kStages = HEADS == 1 ? 3 : 2;
  static constexpr uint32_t kY = HEADS * kTile, kZ = kY + kTile, kStage = kZ + kTile, kP = kStages * kStage, kTable = kP + HEADS * kChunk * kRow;
  static constexpr uint32_t kShared = kTable + 4 * (kPowers + kWeights + kPeriod);
  static_assert(2 * kShared <= 163840, "two workgroups a CU");
};
constexpr uint32_t kShared = Lds<1>::kShared;
static_assert(Lds<2>::kShared <= kShared);

// x as parts of 8 bits each, the first ones cut off and the last one rounded.  (Three operations a value and part; by dot products with
// (-1, 0), which leave out the masking, the copies and waits that those need cost as much.)
__device__ inline bf16x8 top_part(float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = __builtin_amdgcn_perm(__float_as_uint(x[2 * i + 1]), __float_as_uint(x[2 * i]), 0x07060302u);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] -= __uint_as_float(__float_as_uint(x[i]) & 0xffff0000u);
  return as_bf16x8(make_uint4(w[0], w[1], w[2], w[3]));
}
__device__ inline bf16x8 last_part(const float (&x)[8]) {
  return as_bf16x8(make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])));
}
// The workgroup's barrier behind its LDS accesses alone.
constexpr int waitcnt_lds() { return 15 | (7 << 4) | (0 << 8) | (3 << 14); }   // vmcnt 63: none, lgkmcnt 0
__device__ __forceinline__ void meet_lds() {
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __builtin_amdgcn_s_waitcnt(waitcnt_lds());
  __builtin_amdgcn_s_barrier();
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
}
// A branch that is hardly ever taken: nothing of it is done ahead of it.
__device__ inline bool seldom(bool x) {
  const bool y = __builtin_expect(x, 0);
  return y;
}
__device__ inline void stay() { asm volatile("" ::: "memory"); }
// Sign bits of the halves that are not finite (junk in the others).
__device__ inline uint32_t odd_halves(uint32_t u) { return (u & 0x7f807f80u) + 0x00800080u; }

__device__ inline double power_of(float g, int e) { return e == 0 ? 1.0 : exp(double(g) * double(e)); }
// The first powers of L: squares of exp(g), and the product of those that an exponent is made of (an exp costs as much as six of them).
struct Powers {
  static constexpr int BITS = 6;
  double square[BITS];
  __device__ explicit Powers(double g) {
    square[0] = exp(g);
#pragma unroll
    for (int i = 1; i < BITS; ++i) square[i] = square[i - 1] * square[i - 1];
  }
  __device__ double operator()(int e) const {
    double x = 1.0;
#pragma unroll
    for (int i = 0; i < BITS; ++i)
      if ((e >> i) & 1) x *= square[i];
    return x;
  }
};

// OUT: results are wanted, not M alone: a part's own M is summed against the walk, so that what is read last is what the
// walk reads first, with a factor for each chunk in the place of M's.  begin: M where the walk begins, or null; last: where
// to put it at the end, or null.
template <bool BACK, bool OUT, int PARTS, int HEADS>
__device__ __forceinline__ void walk(const Geo& geo, const Place& p, const Src& xs, const Src& ys, const Src& zs, uint16_t* out,
                                     const float* begin, const float* sums, bool trans, float* last, uint8_t* smem) {
  static_assert(HEADS == 1 || (OUT && !BACK));
  constexpr uint32_t kStage = Lds<HEADS>::kStage, kY = Lds<HEADS>::kY, kZ = Lds<HEADS>::kZ, kP = Lds<HEADS>::kP, kTable = Lds<HEADS>::kTable;
  constexpr int kStages = Lds<HEADS>::kStages;
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, q = lane >> 4, rp = lane & 15;
  const int h = p.h, G = geo.group;
  const int rest = min(kChunk, p.tokens - (p.chunk0 + p.chunks - 1) * kChunk);   // tokens of the part's last chunk (by time)
  const uint32_t lds0 = lds_addr(smem);

  // copies: rows 8 (wave % 4) + lane / 8 of a half of each tile
  const int crow = 8 * (wave & 3) + (lane >> 3), half = wave >> 2;
  const uint32_t cchunk = uint32_t(16 * ((lane & 7) ^ swz_k(crow & 15)));
  const int heads = OUT || BACK ? G : 1;               // items of a chunk
  constexpr bool kDown = OUT == BACK;                  // from the last chunk to the first
  // (the copies' sources move on by steps of a chunk, or of a query head)
  struct Tile {
    const uint8_t* at;
    int64_t head;
    int32_t token;
  };
  auto tile = [&](const Src& src, bool grouped) {
    Tile t;
    const int first = kDown ? p.chunk0 + p.chunks - 1 : p.chunk0;
    t.at = uniform_ptr(reinterpret_cast<const uint8_t*>(src.p + (geo.step == nullptr ? int64_t(p.seq) * src.batch : 0) +
                                                        (p.row + first * kChunk) * src.token + int64_t(grouped ? h * G : h) * src.head + 64 * half));
    t.head = grouped ? 2 * src.head : 0;
    t.token = int32_t(2 * src.token);                  // (at most 2^25)
    return t;
  };
  Tile tx = OUT ? tile(xs, !BACK) : Tile{}, ty = tile(ys, BACK), tz = tile(zs, BACK);
  int next_t = (kDown ? p.chunk0 + p.chunks - 1 : p.chunk0) * kChunk, next_c = 0, next_g = 0;   // the next item to copy
  const uint32_t mine = uint32_t(half) * kHalf + uint32_t(wave & 3) * 1024u;   // of a tile
  auto issue = [&](uint32_t stage) {
    const int row = min(crow, p.tokens - 1 - next_t);
    const uint32_t dst = __builtin_amdgcn_readfirstlane(lds0 + stage * kStage + mine);
    auto copy = [&](const uint8_t* from, const Tile& t, uint32_t at) { dma16(from, uint32_t(row) * uint32_t(t.token) + cchunk, dst + at); };
    if (OUT) copy(tx.at, tx, 0);
    if (HEADS == 2) copy(next_g + 1 < heads ? tx.at + tx.head : tx.at, tx, kTile);   // (or the last one once more)
    copy(ty.at, ty, kY);
    copy(tz.at, tz, kZ);
    // past the end the last item is copied again, and not read
    if (next_g + HEADS < heads) {
      next_g += HEADS;
      tx.at += HEADS * tx.head, ty.at += ty.head, tz.at += tz.head;
    } else if (next_c + 1 < p.chunks) {
      auto on = [&](Tile& t) { t.at += int64_t(kDown ? -kChunk : kChunk) * t.token - next_g * t.head; };
      on(tx), on(ty), on(tz);
      ++next_c, next_g = 0;
      next_t += kDown ? -kChunk : kChunk;
    }
  };
  if (p.chunks > 0) {
    issue(0);
    if (HEADS == 1) issue(1);
  }

  // M: y-dim 32 (b / 2) + 8 q + 4 (b % 2) + r, z-dim 16 wave + rp
  f32x4 S[8];
  const int zd = 16 * wave + rp;
  auto get_rows = [&](auto turned, f32x4& to, const float* from, int b) {
    const int y = 32 * (b >> 1) + 8 * q + 4 * (b & 1);
    if (decltype(turned)::value) to = *reinterpret_cast<const f32x4*>(from + zd * kD + y);
    else
#pragma unroll
      for (int r = 0; r < 4; ++r) to[r] = from[(y + r) * kD + zd];
  };
#pragma unroll
  for (int b = 0; b < 8; ++b) S[b] = f32x4{};
  // and the parts that were walked before: each row's place is loaded anew as soon as it is used
  auto get_state = [&](auto turned) {
    if (begin != nullptr)
#pragma unroll
      for (int b = 0; b < 8; ++b) get_rows(turned, S[b], begin, b);
    const int before_me = OUT && sums != nullptr ? (BACK ? p.parts - 1 - p.part : p.part) : 0;
    if (before_me > 0) {
      const int64_t stride = int64_t(BACK ? -geo.kv_heads : geo.kv_heads) * kState;
      const float* at = sums - before_me * stride;
      const double whole = power_of(geo.decay[h], p.cut * kChunk);
      double d = BACK ? power_of(geo.decay[h], p.tokens - (p.parts - 1) * p.cut * kChunk) : whole;
      f32x4 T[8];
#pragma unroll
      for (int b = 0; b < 8; ++b) get_rows(turned, T[b], at, b);
      auto add = [&](bool more) {
        const float hi = float(d), lo = float(d - double(hi));
        d = whole;
        at += stride;
#pragma unroll
        for (int b = 0; b < 8; ++b) {
#pragma unroll
          for (int r = 0; r < 4; ++r) S[b][r] = __builtin_fmaf(S[b][r], hi, __builtin_fmaf(S[b][r], lo, T[b][r]));
          if (more) get_rows(turned, T[b], at, b);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
#pragma unroll 1
      for (int i = 1; i < before_me; ++i) add(true);
      add(false);
    }
  };
  // (either way as a whole: branches between the loads would wait for them one by one)
  if (trans) get_state(std::true_type{});
  else get_state(std::false_type{});

  // weights
  float* const tab = reinterpret_cast<float*>(smem + kTable);
  const Powers power(double(geo.decay[h]));
  const float scale = geo.scale;
  // M is multiplied by L^32 not chunk by chunk, but for a period of four at once at its beginning; meanwhile it stands for the
  // period's end: parts join it with their weights there, and it is read with L^-32 for each chunk that is to come (1e10 at
  // most, so that what small gradients leave there stays in fp32's range: heads that forget faster have periods of one chunk).
  const double dw = power.square[5], dw4 = (dw * dw) * (dw * dw);
  const int period = __builtin_amdgcn_readfirstlane(OUT && dw4 > 1e-13 ? kPeriod : 1);
  if (tid < 33) tab[tid] = float(power(tid));
  if (tid < kWeights) {
    const int k = tid / kChunk, j = tid % kChunk, n = k < kPeriod ? kChunk : rest;
    double w = j >= n ? 0.0 : BACK ? double(scale) * power(j + 1) : power(n - 1 - j);
    if (k < kPeriod)
      for (int i = k + 1; i < period; ++i) w *= dw;
    tab[kPowers + tid] = float(w);
  }
  if (tid >= 192 && tid < 192 + kPeriod) {
    double f = 1.0;
    if (tid > 192)
      for (int i = tid - 192; i < period; ++i) f *= dw;
    tab[kPowers + kWeights + tid - 192] = float(1.0 / f);
  }
  const double dp = period == kPeriod ? dw4 : dw;
  // (M's factors, in two floats, and the last chunk's: in LDS, for a spilled register's load waits for the copies on their way)
  if (tid == 256) {
    tab[33] = float(dp);
    tab[34] = float(dp - double(float(dp)));
    tab[35] = float(power(max(rest, 0)));
  }
  meet_lds();                                          // (M and the first copies are on their way)
  // P: a quarter for each of the first four waves (of the second head for the others), x_t.y_j for j = pj .. pj + 3 and t = pt
  const bool scores = OUT && (HEADS == 2 || wave < 4);
  const int pj = 16 * ((wave >> 1) & (HEADS == 2 ? 1 : 3)) + 4 * q, pt = 16 * (wave & 1) + rp;
  float pw[4];
  bool seen[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int age = BACK ? pj + r - pt : pt - pj - r;
    pw[r] = scale * tab[min(max(age, 0), 32)];
    seen[r] = age >= 0;
  }
  float row_whole[2];                                  // of tokens rp and 16 + rp
#pragma unroll
  for (int tb = 0; tb < 2; ++tb) row_whole[tb] = BACK ? tab[31 - 16 * tb - rp] : scale * tab[16 * tb + rp + 1];

  // operand addresses within a stage (16 rows further: 2,048 bytes)
  uint32_t px[2], yt[2], zt, put;                      // (of the present stage)
  const int r0 = 4 * q + (rp >> 2);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    px[k] = lds0 + uint32_t(rp * 128 + 16 * ((4 * k + q) ^ swz_k(rp)));
    yt[k] = lds0 + kY + uint32_t(r0 * 128 + 16 * ((4 * k + (rp & 3)) ^ swz_k(r0)));
  }
  zt = lds0 + kZ + uint32_t(half) * kHalf + uint32_t(r0 * 128 + 16 * ((2 * (wave & 3) + ((rp >> 1) & 1)) ^ swz_k(r0)) + 8 * (rp & 1));
  const uint32_t py_at = kY + 2048 * uint32_t((wave >> 1) & 1), px_at = 2048 * uint32_t(wave & 1) + (HEADS == 2 ? kTile * uint32_t(half) : 0);
  // P's place of j: 8 (j % 16 / 4) + 4 (j / 16) + j % 4, as the k-slots of Z^T
  const uint32_t pput = lds0 + kP + (HEADS == 2 ? uint32_t(half) * kChunk * kRow : 0) + uint32_t(pt) * kRow + 2 * (8 * q + 4 * ((wave >> 1) & 1));
  const uint32_t pget = lds0 + kP + uint32_t(rp) * kRow + 16 * q;
  const uint32_t kwt = lds0 + kTable + 4 * (kPowers + 4 * q);

  f32x4 os[HEADS][2];                                  // O^T of tokens rp and 16 + rp
  const int out_heads = geo.kv_heads * (BACK ? 1 : G);
  // a result on its way: through the place of x in LDS, from where whole rows are stored, by the wave that then copies the next
  // item's rows there
  put = lds0 + uint32_t(half) * kHalf + uint32_t(rp * 128 + 16 * ((2 * (wave & 3) + (q >> 1)) ^ swz_k(rp)) + 8 * (q & 1));
  const uint32_t get = lds0 + mine + 16 * lane;
  uint16_t* const out_row = OUT ? out + (p.row + (geo.step == nullptr ? int64_t(p.seq) * p.rows : 0)) * out_heads * kD + 64 * half +
                                      int64_t(crow) * out_heads * kD + cchunk / 2 : nullptr;
  int held_n = 0, held_heads = 0;                      // its rows, or none
  int64_t held_at = 0;
  bf16x8 going[HEADS];
  auto fetch = [&](uint32_t stage) {
#pragma unroll
    for (int i = 0; i < HEADS; ++i) going[i] = lds_row(get + stage * kStage + i * kTile);
  };
  auto store = [&] {                                   // (waits for what was read: before the copies to its place)
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_waitcnt(waitcnt_lds());
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
#pragma unroll
    for (int i = 0; i < HEADS; ++i)
      if (crow < held_n && (i == 0 || held_heads > 1)) *reinterpret_cast<bf16x8*>(out_row + held_at + i * kD) = going[i];
    held_n = 0;
  };
  float err = 0.f;                                     // of the factors so far, relative
  double far = 1.0;                                    // without results: the chunk's factor
  uint32_t stage = 0;
  int chunk = 0, n = 0, phase = 0;                     // the chunk, its tokens, and its place in the period
  bool full = true;
  bf16x8 z;                                            // Z^T: z-dim zd, tokens 4 q .. + 3 and 16 more
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
  auto before = [&] { return stage == 0 ? kStages - 1 : stage - 1; };

  // An item's way to its result; FIRST: the first query head of the chunk.  Products and vector work are dealt out so that each
  // has the other to run beside.
  auto result = [&](auto first, int g) {
    constexpr bool kOfM = decltype(first)::value || !BACK;   // (backwards the sum over the query heads begins)
    // (its parts are formed anew for each item: held, they would take 32 registers that are not there)
    if (kOfM) asm volatile("" : "+v"(S[0]), "+v"(S[1]), "+v"(S[2]), "+v"(S[3]), "+v"(S[4]), "+v"(S[5]), "+v"(S[6]), "+v"(S[7]));
    // this wave's quarter of P^T = Y X^T
    f32x4 s = f32x4{};
    if (scores) {
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        const uint32_t c = px[ks & 1] + (ks >> 1) * kHalf;
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lds_row(c + py_at), lds_row(c + px_at), s, 0, 0, 0);
      }
    }
    // X of step u / HEADS, query head u % HEADS
    auto row = [&](int u, int tb) { return lds_row(px[(u / HEADS) & 1] + (u / HEADS >> 1) * kHalf + (u % HEADS) * kTile + 2048 * tb); };
    bf16x8 x[2][2];
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) x[0][tb] = row(0, tb);
    fence();
    store();
    issue(before());
    if (scores) {
      float w[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        w[r] = seen[r] ? s[r] * pw[r] : 0.f;
        if (BACK && pj + r >= n) w[r] = 0.f;
      }
      uint32_t top[2], low[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        top[i] = __builtin_amdgcn_perm(__float_as_uint(w[2 * i + 1]), __float_as_uint(w[2 * i]), 0x07060302u);
        low[i] = pack_bf16x2(w[2 * i] - __uint_as_float(__float_as_uint(w[2 * i]) & 0xffff0000u),
                             w[2 * i + 1] - __uint_as_float(__float_as_uint(w[2 * i + 1]) & 0xffff0000u));
      }
      *(lds_u32x2*)(uintptr_t)(pput) = u32x2{top[0], top[1]};
      *(lds_u32x2*)(uintptr_t)(pput + 64) = u32x2{low[0], low[1]};
    }
    if (kOfM) {
#pragma unroll
      for (int i = 0; i < 2 * HEADS; ++i) os[i >> 1][i & 1] = f32x4{};
      bf16x8 hi, lo;
#pragma unroll
      for (int u = 0; u < 4 * HEADS; ++u) {
        const int ks = u / HEADS, i = u % HEADS;
        fence();
        if (u + 1 < 4 * HEADS)
#pragma unroll
          for (int tb = 0; tb < 2; ++tb) x[(u + 1) & 1][tb] = row(u + 1, tb);
        if (i == 0) {
          float m[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) m[e] = S[2 * ks + (e >> 2)][e & 3];
          hi = top_part(m), lo = last_part(m);
        }
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) os[i][tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, x[u & 1][tb], os[i][tb], 0, 0, 0);
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) os[i][tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, x[u & 1][tb], os[i][tb], 0, 0, 0);
      }
    }
    fence();
    if (kOfM)
#pragma unroll
      for (int tb = 0; tb < 2; ++tb) {
        const float weight = (BACK && !full ? tab[max(rest - 1 - 16 * tb - rp, 0)] : row_whole[tb]) * tab[kPowers + kWeights + phase];
#pragma unroll
        for (int i = 0; i < HEADS; ++i) os[i][tb] *= weight;
      }
    bf16x8 zf = z;
    const uint4 u = __builtin_bit_cast(uint4, z);
    const uint32_t bits = odd_halves(u.x) | odd_halves(u.y) | odd_halves(u.z) | odd_halves(u.w);
    const bool any_odd = __ballot((bits & 0x80008000u) != 0) != 0;
    int odd = BACK ? -1 : kChunk;                      // the first (last) token whose value zd is not finite
    if (seldom(any_odd)) {                             // weights of zero would carry it to tokens that do not see it
      stay();
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (tok::not_finite(float(z[e]))) {
          const int j = 16 * (e >> 2) + 4 * q + (e & 3);
          odd = BACK ? max(odd, j) : min(odd, j);
          zf[e] = (__bf16)0.f;
        }
#pragma unroll
      for (int d = 16; d < 64; d <<= 1) {
        const int other = __shfl_xor(odd, d);
        odd = BACK ? max(odd, other) : min(odd, other);
      }
    }
    meet_lds();                                        // P is there, and nobody needs x any more
#pragma unroll
    for (int i = 0; i < HEADS; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
          os[i][tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(zf, lds_row(pget + 64 * k + 16 * kRow * tb + i * kChunk * kRow), os[i][tb], 0, 0, 0);
    if (seldom(any_odd)) {
      stay();
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int of = __shfl(odd, 4 * q + r);
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
          if (BACK ? 16 * tb + rp <= of : 16 * tb + rp >= of)
#pragma unroll
            for (int i = 0; i < HEADS; ++i) os[i][tb][r] = __builtin_nanf("");
      }
    }
  };
  auto keep = [&](int g) {                             // the result, to be stored behind the next barrier
#pragma unroll
    for (int i = 0; i < HEADS; ++i)
#pragma unroll
      for (int tb = 0; tb < 2; ++tb)
        *(lds_u32x2*)(uintptr_t)(put + 2048 * tb + i * kTile) =
            u32x2{pack_bf16x2(os[i][tb][0], os[i][tb][1]), pack_bf16x2(os[i][tb][2], os[i][tb][3])};
    held_n = n;
    held_heads = G - g;
    held_at = (int64_t(chunk) * kChunk * out_heads + (BACK ? h : h * G + g)) * kD;
  };
  // M past the chunk (of its first query head, backwards), and the present item's part.
  auto advance = [&](auto first, auto&& between) {
    // (a partial chunk: M as it is, and no period)
    const bool forget = OUT && decltype(first)::value && (phase == 0 || !full);
    float dec = 1.f;
    if (forget) {
      const float whole = tab[33], want = tab[34] + err;
      dec = full ? whole + want : tab[35] * tab[kPowers + kWeights + phase];
      if (full) err = want - (dec - whole);
    }
    const uint32_t kw = kwt + 4u * kChunk * uint32_t(full ? phase : kPeriod);
    if (forget) {
      stay();
#pragma unroll
      for (int b = 0; b < 8; ++b) S[b] *= dec;
    }
    auto operand = [&](int b) {                        // of the chunk's tokens, y-dims of S[b]
      const uint32_t a = yt[(b >> 1) & 1] + (b >> 2) * kHalf + 8 * (b & 1);
      return lds_tr2(a, a + 2048);
    };
    bf16x8 part[PARTS], y[3];
    y[0] = operand(0);
    y[1] = operand(1);
    {
      const float4 a = __builtin_bit_cast(float4, *(const tok::lds_u32x4*)(uintptr_t)(kw));
      const float4 b = __builtin_bit_cast(float4, *(const tok::lds_u32x4*)(uintptr_t)(kw + 64));
      const float c8[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = float(z[e]) * (OUT ? c8[e] : c8[e] * float(far));
#pragma unroll
      for (int k = 0; k < PARTS; ++k) part[k] = k == PARTS - 1 ? last_part(w) : top_part(w);
    }
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      fence();
      if (b + 2 < 8) y[(b + 2) % 3] = operand(b + 2);
#pragma unroll
      for (int k = PARTS - 1; k >= 0; --k) S[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y[b % 3], part[k], S[b], 0, 0, 0);
      if (b == 3) between();
    }
    fence();
  };
  auto begin_item = [&] {
    meet<HEADS == 2 ? 0 : OUT ? 3 : 2>();              // this item has landed, and the last one's buffer is free
    if (OUT) fetch(before());
    else issue(before());
    z = lds_tr2(zt, zt + 2048);
    if (seldom(!full)) {
      stay();
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (16 * (e >> 2) + 4 * q + (e & 3) >= n) z[e] = (__bf16)0.f;
    }
  };
  auto end_item = [&] {
    const uint32_t d = stage == kStages - 1 ? uint32_t(1 - kStages) * kStage : kStage;
    stage = stage == kStages - 1 ? 0 : stage + 1;
#pragma unroll
    for (int k = 0; k < 2; ++k) px[k] += d, yt[k] += d;
    zt += d, put += d;
  };
  const std::true_type yes;
  const std::false_type no;

  for (int c = 0; c < p.chunks; ++c) {
    chunk = kDown ? p.chunk0 + p.chunks - 1 - c : p.chunk0 + c;
    n = min(kChunk, p.tokens - chunk * kChunk);
    full = n == kChunk;
    begin_item();
    if (BACK) {
      if (OUT) result(yes, 0);
      advance(yes, [&] { if (OUT && G == 1) keep(0); });
      end_item();
      for (int g = 1; g < G; ++g) {
        begin_item();
        if (OUT) result(no, g);
        advance(no, [&] { if (OUT && g == G - 1) keep(0); });
        end_item();
      }
    } else {
      int g = 0;
      for (; g + HEADS < heads; g += HEADS) {          // (without results there is one item a chunk)
        result(yes, g);
        keep(g);
        end_item();
        begin_item();
      }
      if (OUT) result(yes, g);
      advance(yes, [&] { if (OUT) keep(g); });
      end_item();
    }
    if (!OUT) far *= full ? dw : double(tab[35]);
    phase = full && phase + 1 < period ? phase + 1 : 0;
  }
  meet<0>();                                           // no copy outlives the walk
  if (OUT) {
    fetch(before());
    store();
  }
  if (last != nullptr) {
    if (phase > 0)
#pragma unroll
      for (int b = 0; b < 8; ++b) S[b] *= tab[kPowers + kWeights + phase];
#pragma unroll
    for (int b = 0; b < 8; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) last[(32 * (b >> 1) + 8 * q + 4 * (b & 1) + r) * kD + zd] = S[b][r];
  }
  if (OUT && geo.step == nullptr) {                    // padding
    const int from = max(p.tokens, p.part * geo.chunks * kChunk);
    const int to = p.part == geo.parts - 1 ? p.rows : min(p.rows, (p.part + 1) * geo.chunks * kChunk);
    const int own = BACK ? 1 : G;
    uint16_t* const row0 = out + int64_t(p.seq) * p.rows * out_heads * kD + int64_t(h) * own * kD;
    for (int64_t k = tid; k < int64_t(max(to - from, 0)) * own * 16; k += kThreads) {
      const int64_t t = k / (own * 16), w = k % (own * 16);
      *reinterpret_cast<uint4*>(row0 + (from + t) * out_heads * kD + w * 8) = make_uint4(0, 0, 0, 0);
    }
  }
}

template <bool BACK, int PARTS, int HEADS>
__device__ __forceinline__ void run_walk(const Geo& geo, const Walk& w, bool trans, int idx, uint8_t* smem) {
  const Place p = place(geo, idx);
  if (p.seq < 0) return;
  const size_t at = (size_t(p.seq) * geo.kv_heads + p.h) * kState;
  const bool ends = p.part == (BACK ? 0 : max(p.parts - 1, 0));
  const float *begin = nullptr, *sums = nullptr;
  const float* const start = p.chunks > 0 && w.starts != nullptr ? w.starts + size_t(idx) * kState : nullptr;
  if (start != nullptr && geo.scanned) begin = start;
  else if (p.held && w.first != nullptr) {
    // (forwards the last part's place has a copy: that part may end, and put its M over the first one, before others begin)
    if (start != nullptr && !BACK) begin = start + int64_t(p.parts - 1 - p.part) * geo.kv_heads * kState;
    else begin = w.first + at;
  }
  if (!geo.scanned) sums = start;
  walk<BACK, true, PARTS, HEADS>(geo, p, w.x, w.y, w.z, w.out, begin, sums, trans, ends && w.last != nullptr ? w.last + at : nullptr, smem);
}

template <int HEADS>
__global__ __launch_bounds__(kThreads, 4) void linear_fwd_kernel(WalkArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kShared];
  run_walk<false, 3, HEADS>(a.geo, a.walk[0], false, blockIdx.x, smem);
}

// dk, dv and dq (dk's and dq's M are what is given transposed) of eight workgroups' places one after the other: a place's three lie on one XCD, and share their reads there.
// Places first .. groups - 1, as far as the launch reaches.
template <int PARTS, int HEADS>
__global__ __launch_bounds__(kThreads, 4) void linear_bwd_kernel(WalkArgs a, int first, int groups) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kShared];
  const int b = blockIdx.x / 24, r = blockIdx.x % 24, idx = first + 8 * b + r % 8;
  if (idx >= groups) return;
  if (r < 16) run_walk<true, PARTS, 1>(a.geo, a.walk[r / 8], r < 8, idx, smem);
  else run_walk<false, 2, HEADS>(a.geo, a.walk[2], true, idx, smem);
}

template <int PARTS>
__global__ __launch_bounds__(kThreads, 4) void linear_parts_kernel(PartArgs a, int groups) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kShared];
  const int idx = blockIdx.x % groups;
  const auto& s = a.sum[blockIdx.x / groups];
  const Place p = place(a.geo, idx);
  if (p.seq < 0 || p.chunks == 0) return;
  float* const to = s.starts + size_t(idx) * kState;
  if (s.back) {
    if (p.part > 0) walk<true, false, PARTS, 1>(a.geo, p, s.y, s.y, s.z, nullptr, nullptr, nullptr, false, to, smem);
  } else if (p.part == p.parts - 1) {
    if (a.geo.scanned || s.first == nullptr || !p.held) return;
    const float* const from = s.first + (size_t(p.seq) * a.geo.kv_heads + p.h) * kState;
    for (int i = 4 * threadIdx.x; i < kState; i += 4 * kThreads) *reinterpret_cast<f32x4*>(to + i) = *reinterpret_cast<const f32x4*>(from + i);
  } else {
    walk<false, false, PARTS, 1>(a.geo, p, s.y, s.y, s.z, nullptr, nullptr, nullptr, false, to, smem);
  }
}

// Parts' beginnings from their own M, part by part, kAhead of them read at once.  A workgroup per (sequence, key head,
// sixteenth of M).
constexpr int kAhead = 16;
static_assert(kScanSlices * 4 * kOtherThreads == kState);
__global__ __launch_bounds__(kOtherThreads) void linear_scan_kernel(PartArgs a) {
  const Geo& geo = a.geo;
  int k = blockIdx.x;
  const int slice = k % kScanSlices;
  k /= kScanSlices;
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
    cut_into(p, max(1, head[3]));
    first = head[kHeader + kEntry * e + 4];
    if (first < 0 || first + p.parts > geo.parts) return;
  }
  const int at = slice * 1024 + threadIdx.x * 4;
  float4 m = make_float4(0.f, 0.f, 0.f, 0.f);
  if (s.first != nullptr && p.held)
    m = *reinterpret_cast<const float4*>(s.first + (size_t(p.seq) * geo.kv_heads + h) * kState + at);
  const int tail = p.tokens - (p.parts - 1) * p.cut * kChunk;
  const double whole = power_of(geo.decay[h], p.cut * kChunk), part = power_of(geo.decay[h], max(tail, 0));
  auto slot = [&](int i) {
    const int q = s.back ? p.parts - 1 - i : i;
    return reinterpret_cast<float4*>(s.starts + (size_t(first + q) * geo.kv_heads + h) * kState + at);
  };
  for (int i0 = 0; i0 < p.parts; i0 += kAhead) {
    float4 own[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      own[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i0 + i + 1 < p.parts) own[i] = *slot(i0 + i);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (i0 + i >= p.parts) break;
      *slot(i0 + i) = m;
      const double d = (s.back ? i0 + i == 0 : i0 + i == p.parts - 1) ? part : whole;
      const float hi = float(d), lo = float(d - double(hi));
      m.x = __builtin_fmaf(m.x, hi, __builtin_fmaf(m.x, lo, own[i].x));
      m.y = __builtin_fmaf(m.y, hi, __builtin_fmaf(m.y, lo, own[i].y));
      m.z = __builtin_fmaf(m.z, hi, __builtin_fmaf(m.z, lo, own[i].z));
      m.w = __builtin_fmaf(m.w, hi, __builtin_fmaf(m.w, lo, own[i].w));
    }
  }
}

}  // namespace

hipError_t launch_linear_parts(const PartArgs& a, int32_t groups, bool exact, hipStream_t stream) {
  if (exact) linear_parts_kernel<3><<<dim3(unsigned(groups) * a.n), kThreads, 0, stream>>>(a, groups);
  else linear_parts_kernel<2><<<dim3(unsigned(groups) * a.n), kThreads, 0, stream>>>(a, groups);
  return hipGetLastError();
}

hipError_t launch_linear_scan(const PartArgs& a, hipStream_t stream) {
  linear_scan_kernel<<<dim3(unsigned(kScanSlices * a.geo.kv_heads) * a.geo.n * a.n), kOtherThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_linear_fwd(const WalkArgs& a, int32_t groups, hipStream_t stream) {
  if (!two_heads(a.geo.group)) linear_fwd_kernel<1><<<dim3(unsigned(groups)), kThreads, 0, stream>>>(a);
  else linear_fwd_kernel<2><<<dim3(unsigned(groups)), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_linear_bwd(const WalkArgs& a, int32_t groups, bool exact, hipStream_t stream) {
  // three walks a place: as many launches as their threads need (no walk waits for another)
  constexpr int32_t kMost = int32_t(most_groups(kThreads) / 24 * 8);
  for (int32_t first = 0; first < groups; first += std::min(kMost, groups - first)) {
    const unsigned grid = unsigned((std::min(kMost, groups - first) + 7) / 8 * 24);
    auto run = [&](auto kernel) { kernel<<<dim3(grid), kThreads, 0, stream>>>(a, first, groups); };
    if (!two_heads(a.geo.group)) exact ? run(linear_bwd_kernel<3, 1>) : run(linear_bwd_kernel<2, 1>);
    else exact ? run(linear_bwd_kernel<3, 2>) : run(linear_bwd_kernel<2, 2>);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

}  // namespace lin
}  // namespace uf
