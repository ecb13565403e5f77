// Attention of tokens under a sliding window with sinks, from the paged cache or from
// plain tensors: prompts, pieces of prompts, trees of drafted tokens, training.
//
// A workgroup takes 128 rows of one sequence and key head, a row being a (token, query
// head of the group) pair, so that heads that share keys share their copies and a tile
// spans few positions.  It walks the 64-key units that some row sees (the sinks' units,
// then the window's, key_range) with an online softmax.
//
// Work split: four waves of 32 rows, two workgroups per CU.  S^T = K Q^T and
// O^T += V^T P^T on v_mfma_f32_32x32x16_bf16, K and V from LDS as the A operand (V by
// transposing reads, since it lies row by row), Q^T and P^T in registers as the B
// operand: a lane owns one row's column, the weights rounded to bf16 in place are the
// PV operand, whose k-slots hold the keys of each group of 16 with bits 2 and 3 swapped.
//
// Memory: a unit is 32 KB, K and V as two blocks of 64 dimensions in 128-byte rows
// (swz_k), copied by global_load_lds one unit ahead into the other of two buffers; one
// barrier per unit.  Rows that no query of the tile sees are not copied: their places
// take a row that is seen, and weigh nothing.
//
// Softmax in base 2 with a lazy offset: weights exp2(c2 s - m), c2 = scale*log2(e).  The
// offset is raised, and O and l rescaled, on the first two units, on a lane's first
// seen key, and when a lane's 16 weights sum to more than kSumBound.  l adds the fp32
// weights; P is rounded to bf16 for the products (the matrix cores' type: half of O's
// error, the other half is its own rounding), O once at the end.
//
// What bounds it: the matrix cores under the power limit where the launch is large, 1,005
// to 1,040 TFLOP/s of seen pairs at 16,384 tokens, 32 heads over 8, window 4,096 (925 to
// 958 us by the card; a library product of 8,192 cubed reaches 1,082 to 1,125; matrix cores
// busy 55 % of the cycles at 1.85 GHz); where a CU has one workgroup, a unit takes 2,800 to
// 3,700 cycles for 1,024 of products: of a wave's cycles 46 % issue, 33 % are at wait counts
// and barriers and 21 % ready but not issued (360 tiles, window 1,024), or 35, 51 and 14 %
// (64 slices of two units).  (Eight waves a tile, each
// with one of a unit's key blocks, and four units in LDS took 17.9 us for 16.7 on tiles
// of 6 units and 87 for 89 on tiles of 65; reading three, five or six operands ahead
// changed nothing.)
#include "token_common.h"

#include <algorithm>

namespace uf {
namespace tok {
namespace {

using namespace attn;

constexpr uint32_t kUnitBytes = 32768;
constexpr float kSumBound = 4096.0f;
constexpr int kList = 1024;            // units taken into LDS at a time
constexpr int kReads = 4;              // operands in flight ahead of their product
constexpr int kExact = 2;              // units whose maxima always raise the offset

template <bool PAGED>
__global__ __launch_bounds__(256, 2) void attn_rows_kernel(AttnArgs a) {
  __shared__ uint4 sbuf[2][kUnitBytes / 16];
  __shared__ int32_t sunit[PAGED ? kList : 1], spage[PAGED ? kList + 1 : 1];   // the count last

  const int H = a.kv_heads, G = a.group;
  int idx = blockIdx.x;
  const int h = idx % H;
  idx /= H;
  int e, tile, slice, at_tile;                         // at_tile: of the launch
  if (PAGED && a.packed > 0) {
    slice = idx / a.packed;
    at_tile = a.packed - 1 - idx % a.packed;
    const Place w = tile_place(a, at_tile, kRowTile);
    if (w.entry < 0) return;
    e = w.entry;
    tile = w.tile;
  } else {
    e = idx % a.n;
    idx /= a.n;
    tile = a.tiles - 1 - idx % a.tiles;                // long ranges first
    slice = idx / a.tiles;
    at_tile = e * a.tiles + tile;
  }

  Part p;
  int rows_all;                                        // rows with an output
  if (PAGED) {
    if (e >= ((const const_i32*)a.step)[0]) return;
    p = step_part(a, e);
    rows_all = p.count * G;
    if (rows_all < a.least_rows || rows_all > a.most_rows) return;
  } else {
    p.seq = e;
    p.at = 0;
    p.count = a.lengths != nullptr ? min(max(((const const_i32*)a.lengths)[e], 0), a.tokens) : a.tokens;
    p.held = 0;
    rows_all = a.tokens * G;
  }
  const int row0 = tile * kRowTile;
  if (row0 >= rows_all) return;

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, hl = lane >> 5, ln = lane & 31, rp = lane & 15, g = (lane >> 4) & 1;
  const int row = row0 + wave * 32 + ln;
  const int token = int(uint32_t(row) / uint32_t(G));
  const int head = h * G + row - token * G;
  const bool stored = row < rows_all, live = stored && token < p.count;
  uint16_t* const op = a.o + (PAGED ? size_t(p.at) + token : size_t(e) * a.tokens + token) * a.q_heads * kD +
                       size_t(head) * kD + 4 * hl;
  float* const lp = a.lse == nullptr ? nullptr
                    : PAGED ? a.lse + (size_t(p.at) + token) * a.q_heads + head
                            : a.lse + (size_t(e) * a.q_heads + head) * a.tokens + token;
  const int tok0 = row0 / G, tok1 = min(min(row0 + kRowTile, rows_all) - 1, p.count * G - 1) / G;
  auto store_zero = [&] {
#pragma unroll
    for (int i = 0; i < 16; ++i) *reinterpret_cast<uint2*>(op + 8 * i) = make_uint2(0, 0);
    if (lp != nullptr && hl == 0) *lp = -INFINITY;
  };
  if (!PAGED && tok0 >= p.count) {                     // padding
    if (stored) store_zero();
    return;
  }
  const bool tree = PAGED && a.tree != nullptr;
  const int first = tree ? p.held : p.held + tok0, last = tree ? p.held + p.count - 1 : p.held + tok1;
  const Range range = key_range(first, last, a.window, a.sinks, kKeyUnit);
  const int units = slice_units(range.count, a.slice, a.n_split);
  const bool whole = units >= range.count;
  if (slice > 0 && (whole || slice * units >= range.count)) return;
  const int u0 = whole ? 0 : slice * units, n_units = whole ? range.count : min(units, range.count - u0);

  // this wave's positions, and the lane's
  const int w0 = row0 + wave * 32;
  const int pmin = tree ? p.held - 1 : p.held + w0 / G;
  const int pmax = tree ? last : p.held + min(min(w0 + 31, rows_all - 1) / G, p.count - 1);
  uint64_t node = 0;
  int pos = min(p.held + token, pmax);
  if (tree && live) {
    node = uint64_t(a.tree[p.at + token]) & bits_upto(p.count);
    pos = p.held + max(int(__popcll(node)) - 1, 0);
  }

  bf16x8 qf[8];                                        // Q^T: lane holds row ln, dims 16 ks + 8 hl ..
  {
    const uint16_t* qp = a.q + (PAGED ? 0 : int64_t(e) * a.q_batch) + int64_t(p.at + (live ? token : 0)) * a.q_token +
                         int64_t(live ? head : 0) * a.q_head + 8 * hl;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      uint4 u = make_uint4(0, 0, 0, 0);
      if (live) u = *reinterpret_cast<const uint4*>(qp + 16 * ks);
      qf[ks] = as_bf16x8(u);
    }
  }

  // operand addresses in the current buffer: K rows 32 kb + ln, V rows (keys) 16 kk ..
  const uint32_t lds0 = lds_addr(&sbuf[0][0]);
  uint32_t kr[4], vt[2][2];
#pragma unroll
  for (int k = 0; k < 4; ++k) kr[k] = lds0 + uint32_t(ln * 128 + 16 * ((2 * k + hl) ^ swz_k(ln & 15)));
#pragma unroll
  for (int hh = 0; hh < 2; ++hh)
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int r = 8 * hh + 4 * hl + (rp >> 2);
      vt[hh][m] = lds0 + 16384u + uint32_t(r * 128 + 16 * ((4 * m + 2 * g + ((rp >> 1) & 1)) ^ swz_k(r)) + 8 * (rp & 1));
    }

  struct Unit {
    const uint8_t *k, *v;
    int key0;
  };
  const uint32_t kstep = PAGED ? kD * 2 : uint32_t(a.k_token) * 2, vstep = PAGED ? kD * 2 : uint32_t(a.v_token) * 2;
  const int T = PAGED ? a.pool.page_tokens : 0;
  const size_t vbase = PAGED ? size_t(H) * T * kD * 2 : 0;
  auto tile_of = [&](int u) { return u < range.sink ? u : u - range.sink + range.from; };
  auto unit_of = [&](int t, int page) {                // t: 64-key tile of the sequence
    Unit u;
    u.key0 = t * kKeyUnit;
    if (PAGED) {
      u.k = a.pool.base + (size_t(page) * 2 * H + h) * size_t(T) * (kD * 2) + size_t(u.key0 & (T - 1)) * (kD * 2);
      u.v = u.k + vbase;
    } else {
      u.k = reinterpret_cast<const uint8_t*>(a.k + int64_t(e) * a.k_batch + int64_t(u.key0) * a.k_token + int64_t(h) * a.k_head);
      u.v = reinterpret_cast<const uint8_t*>(a.v + int64_t(e) * a.v_batch + int64_t(u.key0) * a.v_token + int64_t(h) * a.v_head);
    }
    return u;
  };
  // Copies: copy t of a wave fills block t/2, rows 8 (wave + 4 (t%2)) + lane/8.
  const uint32_t chunk = uint32_t(16 * ((lane & 7) ^ swz_k(8 * (wave & 1) + (lane >> 3))));
  struct Offsets {
    uint32_t k[2], v[2];
  };
  auto offsets = [&](const Unit& u) {
    Offsets o;
    const int top = u.key0 < range.from * kKeyUnit ? min(63, a.sinks - 1 - u.key0) : min(63, last - u.key0);
    const int low = u.key0 < range.from * kKeyUnit ? 0 : range.low - u.key0, srel = a.sinks - u.key0;
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
    const uint32_t dst = lds0 + buf * kUnitBytes + uint32_t(wave) * 1024u + uint32_t(t) * 4096u;
    if (k < 4)
      dma16(u.k + (t >> 1) * 128, o.k[t & 1], dst);
    else
      dma16(u.v + (t >> 1) * 128, o.v[t & 1], dst + 16384u);
  };
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };

  const float c2 = a.scale_log2;
  f32x16 o[4];                                         // O^T [4 x 32 dims][32 rows]
#pragma unroll
  for (int mb = 0; mb < 4; ++mb) o[mb] = f32x16{};
  float m = -INFINITY, moff = 0.f, l = 0.f, bound = -1.f;

  auto load = [&](int i) -> bf16x8 {
    if (i < 16) return lds_row(kr[i & 3] + uint32_t((i >> 3) * 4096 + ((i >> 2) & 1) * 8192));
    const int k = i - 16, kb = k >> 3, kk = (k >> 2) & 1, mb = k & 3;
    const uint32_t at = uint32_t(kb * 4096 + kk * 2048 + (mb >> 1) * 8192);
    return lds_tr2(vt[0][mb & 1] + at, vt[1][mb & 1] + at);
  };
  auto body = [&](const Unit& cur, const Unit& next, uint32_t nbuf) {
    bf16x8 x[32], pw[2][2];
    f32x16 s[2];
    float rs = 0.f;
    const Offsets no = offsets(next);
    const bool full = cur.key0 + 63 <= pmin &&
                      (a.window == 0 || cur.key0 >= pmax - a.window + 1 || cur.key0 + 63 < a.sinks);
    uint64_t see = 0;
    if (!full)
      see = tree ? seen_bits_tree(pos, cur.key0, a.window, a.sinks, p.held, node)
                 : seen_bits(pos, cur.key0, a.window, a.sinks);
    auto mask = [&](int kb) {
      if (full) return;
      const uint32_t w = uint32_t(see >> (32 * kb)) >> (4 * hl);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!((w >> (8 * (r >> 2) + (r & 3))) & 1u)) s[kb][r] = -INFINITY;
    };
    auto weight = [&](int kb, int r) {                 // elements r, r + 1
      const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][r], c2, -moff));
      const float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][r + 1], c2, -moff));
      pw[kb][r >> 3][r & 7] = (__bf16)w0;
      pw[kb][r >> 3][(r & 7) + 1] = (__bf16)w1;
      rs += w0 + w1;
    };
    auto check = [&](int kb) {
      asm volatile("" : "+v"(pw[kb][0]), "+v"(pw[kb][1]), "+v"(rs));
      if (__ballot(!(m > -INFINITY) || rs > bound) != 0) {
        float mx = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
        mx = pair_max(mx * c2);                        // c2 > 0
        const bool had = m > -INFINITY;
        const float sh = had ? fmaxf(mx - m, 0.f) : 0.f;
        const float alpha = __builtin_amdgcn_exp2f(-sh);
        m = had ? m + sh : mx;
        l *= alpha;
#pragma unroll
        for (int mb = 0; mb < 4; ++mb) o[mb] *= alpha;
        moff = (m > -INFINITY) ? m : 0.f;
        rs = 0.f;
#pragma unroll
        for (int r = 0; r < 16; r += 2) weight(kb, r);
      }
      l += rs;
      rs = 0.f;
    };
#pragma unroll
    for (int i = 0; i < kReads; ++i) x[i] = load(i);
    fence();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i], qf[i], i ? s[0] : f32x16{}, 0, 0, 0);
      x[i + kReads] = load(i + kReads);
      issue(next, no, nbuf, i);
      fence();
    }
    mask(0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[8 + i], qf[i], i ? s[1] : f32x16{}, 0, 0, 0);
      x[8 + i + kReads] = load(8 + i + kReads);
      weight(0, 2 * i);
      fence();
    }
    check(0);
    mask(1);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[16 + i], pw[0][i >> 2], o[i & 3], 0, 0, 0);
      x[16 + i + kReads] = load(16 + i + kReads);
      weight(1, 2 * i);
      fence();
    }
    check(1);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[24 + i], pw[1][i >> 2], o[i & 3], 0, 0, 0);
      if (i + kReads < 8) x[24 + i + kReads] = load(24 + i + kReads);
      fence();
    }
  };
  // A wave without a row only copies: in a loop of its own, since a branch around the body would have the compiler
  // keep two sets of accumulators and move one into the other (64 registers a unit: 2 % of a long prompt).
  const bool idle = row0 + wave * 32 >= min(rows_all, p.count * G);
  auto walk_idle = [&](int U, auto&& entry) {
    Unit cur = entry(0);
    for (int u = 0; u <= U; ++u) {
      const Offsets co = offsets(cur);
      if (u > 0) meet<0>();
#pragma unroll
      for (int k = 0; k < 8; ++k) issue(cur, co, uint32_t(u) & 1u, k);
      cur = entry(min(u + 1, U - 1));
    }
    meet<0>();
  };
  auto walk = [&](int U, auto&& entry) {
    if (idle) return walk_idle(U, entry);
    Unit cur = entry(0), next = entry(U > 1 ? 1 : 0);
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
      if (u == kExact - 1) bound = kSumBound;
      const uint32_t d = (u & 1) ? uint32_t(-int(kUnitBytes)) : kUnitBytes;
#pragma unroll
      for (int k = 0; k < 4; ++k) kr[k] += d;
#pragma unroll
      for (int k = 0; k < 4; ++k) vt[k >> 1][k & 1] += d;
      cur = next;
      next = entry(min(u + 2, U - 1));
    } while (++u < U);
    if (U & 1) {                                       // the next units start in buffer 0 again
#pragma unroll
      for (int k = 0; k < 4; ++k) kr[k] -= kUnitBytes;
#pragma unroll
      for (int k = 0; k < 4; ++k) vt[k >> 1][k & 1] -= kUnitBytes;
    }
    meet<0>();                                         // no copy outlives the walk
  };

  if constexpr (PAGED) {
    const int32_t* pages = a.table + size_t(p.seq) * a.row;
    for (int base = 0; base < n_units; base += kList) {
      // the units whose pages are there
      if (wave == 0) {
        int cnt = 0;
        const int end = min(n_units, base + kList);
        for (int b = base; b < end; b += 64) {
          const int u = b + lane;
          int page = -1;
          const int t = tile_of(u0 + min(u, n_units - 1));
          if (u < end) page = pages[uint32_t(t * kKeyUnit) / uint32_t(T)];
          const bool on = uint32_t(page) < uint32_t(a.pool.n_pages);
          const uint64_t bal = __ballot(on);
          const int at = cnt + __popcll(bal & ((uint64_t(1) << lane) - 1));
          if (on) {
            sunit[at] = t;
            spage[at] = page;
          }
          cnt += __popcll(bal);
        }
        if (lane == 0) spage[kList] = cnt;
      }
      meet<0>();
      const int U = __builtin_amdgcn_readfirstlane(spage[kList]);
      if (U > 0)
        walk(U, [&](int u) {
          return unit_of(__builtin_amdgcn_readfirstlane(sunit[u]), __builtin_amdgcn_readfirstlane(spage[u]));
        });
      else
        meet<0>();                                     // the table has been read
    }
  } else {
    walk(n_units, [&](int u) { return unit_of(tile_of(u), 0); });
  }

  // A weight of zero times a value that is not finite: a row that does not see the value has it all the same.  Where any
  // of the wave's results is not finite its rows are formed again key by key, each from the keys it sees.
  float probe = 0.f;
#pragma unroll
  for (int mb = 0; mb < 4; ++mb)
#pragma unroll
    for (int r = 0; r < 16; ++r) probe += o[mb][r];
  if (__ballot(not_finite(probe)) != 0) {
    float out[64];
#pragma unroll
    for (int i = 0; i < 64; ++i) out[i] = 0.f;
    for (int u = 0; u < n_units; ++u) {
      const int t = tile_of(u0 + u);
      int page = 0;
      if (PAGED) {
        page = __builtin_amdgcn_readfirstlane(a.table[size_t(p.seq) * a.row + uint32_t(t * kKeyUnit) / uint32_t(T)]);
        if (uint32_t(page) >= uint32_t(a.pool.n_pages)) continue;
      }
      const Unit c = unit_of(t, page);
      const uint64_t see = tree ? seen_bits_tree(pos, c.key0, a.window, a.sinks, p.held, node)
                                : seen_bits(pos, c.key0, a.window, a.sinks);
      for (int k = 0; k < kKeyUnit; ++k) {
        const bool on = live && ((see >> k) & 1u);
        if (__ballot(on) != 0)
          add_key<16>(qf, c.k + uint32_t(k) * kstep, c.v + uint32_t(k) * vstep, hl, on, c2, moff, 4 * hl, out);
      }
    }
#pragma unroll
    for (int mb = 0; mb < 4; ++mb)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[mb][r] = out[16 * mb + r];
  }
  l = pair_sum(l);
  if (!whole) {                                        // a slice: O relative to the offset, the offset and the sum
    if (live) {
      const size_t rows = work_rows(a, kRowTile);
      const size_t at = work_at(a, at_tile, h, slice, kRowTile) + (row - row0);
      float* wp = a.work + at * kD + 4 * hl;
#pragma unroll
      for (int mb = 0; mb < 4; ++mb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<float4*>(wp + mb * 32 + 8 * i) =
              make_float4(o[mb][4 * i], o[mb][4 * i + 1], o[mb][4 * i + 2], o[mb][4 * i + 3]);
      if (hl == 0) reinterpret_cast<float2*>(a.work + rows * kD)[at] = make_float2(m, l);
    }
    return;
  }
  if (live) {
    const float inv = l == 0.f ? 0.f : 1.f / l;       // (a sum that is no number stays one)
#pragma unroll
    for (int mb = 0; mb < 4; ++mb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint2 u;
        u.x = pack_bf16x2(o[mb][4 * i] * inv, o[mb][4 * i + 1] * inv);
        u.y = pack_bf16x2(o[mb][4 * i + 2] * inv, o[mb][4 * i + 3] * inv);
        *reinterpret_cast<uint2*>(op + mb * 32 + 8 * i) = u;
      }
    if (lp != nullptr && hl == 0) *lp = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
  } else if (stored) {
    store_zero();
  }
}

// ---------------------------------------------------------------- few rows ----
//
// At most 32 rows of a sequence and key head: a decoding step, or a small tree.  Nothing
// is multiplied often enough to fill the matrix cores, so HBM bounds it, and the latency of what
// stands before and after: 48 sequences x 8 heads x 4,100 keys in 148 us (5.4 TB/s), one
// of 131,072 keys in 93 (5.8), one of 200 keys and 4 heads in 8.  A workgroup takes a slice of the keys; each of its four
// waves walks every fourth 32-key unit by itself, its K and V copied into two stages
// of its own, so that no barrier stands in the loop, and the waves' states are
// merged through LDS at the end.
constexpr uint32_t kStage = 16384;     // K and V of a unit

__global__ __launch_bounds__(256, 1) void attn_few_kernel(AttnArgs a) {
  __shared__ uint4 sbuf[4][2][kStage / 16];
  __shared__ float sml[2][4][32];

  const int H = a.kv_heads, G = a.group;
  int idx = blockIdx.x;
  const int h = idx % H;
  idx /= H;
  const int sequences = a.packed > 0 ? a.packed : a.n;
  const int at_tile = idx % sequences, slice = idx / sequences;
  int e = at_tile;
  if (a.packed > 0) {
    e = tile_place(a, at_tile, kFewRows).entry;
    if (e < 0) return;
  }
  if (e >= ((const const_i32*)a.step)[0]) return;
  const Part p = step_part(a, e);
  const int rows = p.count * G;
  if (rows < a.least_rows || rows > a.most_rows) return;
  const bool tree = a.tree != nullptr;
  const int last = p.held + p.count - 1;
  const Range range = key_range(p.held, last, a.window, a.sinks, kFewUnit);
  const int units = slice_units(range.count, a.slice, a.n_split);
  const bool whole = units >= range.count;
  if (slice > 0 && (whole || slice * units >= range.count)) return;
  const int u0 = whole ? 0 : slice * units, n_units = whole ? range.count : min(units, range.count - u0);

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, hl = lane >> 5, ln = lane & 31, rp = lane & 15, g = (lane >> 4) & 1;
  const bool live = ln < rows;
  const int token = live ? int(uint32_t(ln) / uint32_t(G)) : p.count - 1;
  const int head = h * G + (live ? ln - token * G : 0);

  // units wave, wave + 4, ... of the slice; lane i keeps the page of the i-th of the next 64
  const int mine = (n_units - wave + 3) >> 2;
  const int32_t* pages = a.table + size_t(p.seq) * a.row;
  const int T = a.pool.page_tokens;
  auto key_of = [&](int i) {
    const int u = u0 + wave + 4 * i;
    return (u < range.sink ? u : u - range.sink + range.from) * kFewUnit;
  };
  int held_pages = -1;
  auto take_pages = [&](int i) {
    held_pages = i + lane < mine ? pages[uint32_t(key_of(i + lane)) / uint32_t(T)] : -1;
  };
  take_pages(0);

  uint64_t node = 0;
  int pos = p.held + token;
  if (tree) {
    node = uint64_t(a.tree[p.at + token]) & bits_upto(p.count);
    pos = p.held + max(int(__popcll(node)) - 1, 0);
  }
  const int pmin = tree ? p.held - 1 : p.held, pmax = last;
  bf16x8 qf[8];
  {
    const uint16_t* qp = a.q + int64_t(p.at + token) * a.q_token + int64_t(head) * a.q_head + 8 * hl;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      uint4 u = make_uint4(0, 0, 0, 0);
      if (live) u = *reinterpret_cast<const uint4*>(qp + 16 * ks);
      qf[ks] = as_bf16x8(u);
    }
  }

  const uint32_t lds0 = lds_addr(&sbuf[0][0][0]) + uint32_t(wave) * 2u * kStage;
  uint32_t kr[4], vt[2][2];                            // K [2 blocks][32 rows], V the same 8 KB behind
#pragma unroll
  for (int k = 0; k < 4; ++k) kr[k] = lds0 + uint32_t(ln * 128 + 16 * ((2 * k + hl) ^ swz_k(ln & 15)));
#pragma unroll
  for (int hh = 0; hh < 2; ++hh)
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int r = 8 * hh + 4 * hl + (rp >> 2);
      vt[hh][m] = lds0 + 8192u + uint32_t(r * 128 + 16 * ((4 * m + 2 * g + ((rp >> 1) & 1)) ^ swz_k(r)) + 8 * (rp & 1));
    }
  struct Unit {
    const uint8_t* k;
    int key0;
  };
  const size_t vbase = size_t(H) * T * (kD * 2);
  int taken = 0;                                       // units looked at
  auto fetch = [&](Unit& u) {
    while (taken < mine) {
      if (taken > 0 && (taken & 63) == 0) take_pages(taken);
      const int page = __builtin_amdgcn_readlane(held_pages, taken & 63);
      u.key0 = key_of(taken);
      ++taken;
      if (uint32_t(page) < uint32_t(a.pool.n_pages)) {
        u.k = a.pool.base + (size_t(page) * 2 * H + h) * size_t(T) * (kD * 2) + size_t(u.key0 & (T - 1)) * (kD * 2);
        return true;
      }
    }
    return false;
  };
  // Copy t fills rows 8 (t%4) + lane/8 of block t/4; rows that no query sees give way to one that is seen.
  auto issue = [&](const Unit& u, uint32_t stage) {
    const bool sink = u.key0 < range.from * kFewUnit;
    const int top = sink ? min(31, a.sinks - 1 - u.key0) : min(31, last - u.key0);
    const int low = sink ? 0 : range.low - u.key0, srel = a.sinks - u.key0;
    uint32_t off[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int at = 8 * t + (lane >> 3);
      const int r = min(at < srel ? at : max(at, low), top);
      off[t] = uint32_t(r) * (kD * 2) + uint32_t(16 * ((lane & 7) ^ swz_k(at & 15)));
    }
    const uint32_t dst = lds0 + stage * kStage;
#pragma unroll
    for (int t = 0; t < 8; ++t) dma16(u.k + (t >> 2) * 128, off[t & 3], dst + uint32_t(t) * 1024u);
#pragma unroll
    for (int t = 0; t < 8; ++t) dma16(u.k + vbase + (t >> 2) * 128, off[t & 3], dst + 8192u + uint32_t(t) * 1024u);
  };

  const float c2 = a.scale_log2;
  f32x16 o[4];
#pragma unroll
  for (int mb = 0; mb < 4; ++mb) o[mb] = f32x16{};
  float m = -INFINITY, moff = 0.f, l = 0.f, bound = -1.f;

  auto compute = [&](const Unit& cur, uint32_t stage) {
    const uint32_t st = stage * kStage;
    f32x16 s = f32x16{};
#pragma unroll
    for (int ks = 0; ks < 8; ++ks)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_row(kr[ks & 3] + st + uint32_t((ks >> 2) * 4096)), qf[ks], s, 0, 0, 0);
    bf16x8 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t at = st + uint32_t((i >> 2) * 2048 + ((i >> 1) & 1) * 4096);
      v[i] = lds_tr2(vt[0][i & 1] + at, vt[1][i & 1] + at);
    }
    const bool full = cur.key0 + 31 <= pmin &&
                      (a.window == 0 || cur.key0 >= pmax - a.window + 1 || cur.key0 + 31 < a.sinks);
    if (!full) {
      const uint64_t see = tree ? seen_bits_tree(pos, cur.key0, a.window, a.sinks, p.held, node)
                                : seen_bits(pos, cur.key0, a.window, a.sinks);
      const uint32_t w = uint32_t(see) >> (4 * hl);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!((w >> (8 * (r >> 2) + (r & 3))) & 1u)) s[r] = -INFINITY;
    }
    bf16x8 pw[2];
    auto weights = [&] {
      float rs = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c2, -moff));
        pw[r >> 3][r & 7] = (__bf16)w;
        rs += w;
      }
      return rs;
    };
    float rs = weights();
    if (__ballot(!(m > -INFINITY) || rs > bound) != 0) {
      float mx = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
      mx = pair_max(mx * c2);
      const bool had = m > -INFINITY;
      const float sh = had ? fmaxf(mx - m, 0.f) : 0.f;
      const float alpha = __builtin_amdgcn_exp2f(-sh);
      m = had ? m + sh : mx;
      l *= alpha;
#pragma unroll
      for (int mb = 0; mb < 4; ++mb) o[mb] *= alpha;
      moff = (m > -INFINITY) ? m : 0.f;
      rs = weights();
    }
    l += rs;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[i], pw[i >> 2], o[i & 3], 0, 0, 0);
  };

  Unit cur, next;
  bool has = fetch(cur);
  if (has) issue(cur, 0);
  uint32_t stage = 0;
  int done = 0;
  while (has) {
    const bool more = fetch(next);
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    if (more) {
      issue(next, stage ^ 1u);
      __builtin_amdgcn_s_waitcnt(waitcnt_vm(16));      // cur has landed, next may be in flight
    } else {
      __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    }
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    compute(cur, stage);
    if (++done == kExact) bound = kSumBound;
    // every operand has been read before the stage is copied into again
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_waitcnt((63 & 15) | (7 << 4) | (0 << 8) | ((63 >> 4) << 14));
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    cur = next;
    has = more;
    stage ^= 1u;
  }

  // ---- merge the waves: wave w takes dims 32 w .. ----
  l = pair_sum(l);
  float* xo = reinterpret_cast<float*>(&sbuf[0][0][0]);    // [4 waves][8: 4 blocks][16][64 lanes]: a wave's own stages
#pragma unroll
  for (int mb = 0; mb < 4; ++mb)
#pragma unroll
    for (int r = 0; r < 16; ++r) xo[((wave * 8 + mb) * 16 + r) * 64 + lane] = o[mb][r];
  if (hl == 0) {
    sml[0][wave][ln] = m;
    sml[1][wave][ln] = l;
  }
  __syncthreads();
  if (!live) return;
  float f[4], mm = -INFINITY, lt = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) mm = fmaxf(mm, sml[0][w][ln]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float mw = sml[0][w][ln];
    f[w] = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - mm);
    lt += sml[1][w][ln] * f[w];
  }
  float out[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    out[r] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) out[r] += xo[((w * 8 + wave) * 16 + r) * 64 + lane] * f[w];
  }
  const int d0 = wave * 32 + 4 * hl;
  float probe = 0.f;                                   // as above: a value that a row does not see
#pragma unroll
  for (int r = 0; r < 16; ++r) probe += out[r];
  if (__ballot(not_finite(probe)) != 0) {
#pragma unroll
    for (int r = 0; r < 16; ++r) out[r] = 0.f;
    for (int u = u0; u < u0 + n_units; ++u) {
      const int key0 = (u < range.sink ? u : u - range.sink + range.from) * kFewUnit;
      const int page = __builtin_amdgcn_readfirstlane(pages[uint32_t(key0) / uint32_t(T)]);
      if (uint32_t(page) >= uint32_t(a.pool.n_pages)) continue;
      const uint8_t* kp = a.pool.base + (size_t(page) * 2 * H + h) * size_t(T) * (kD * 2) + size_t(key0 & (T - 1)) * (kD * 2);
      const uint64_t see = tree ? seen_bits_tree(pos, key0, a.window, a.sinks, p.held, node)
                                : seen_bits(pos, key0, a.window, a.sinks);
      for (int k = 0; k < kFewUnit; ++k) {
        const bool on = (see >> k) & 1u;
        if (__ballot(on) != 0)
          add_key<4>(qf, kp + k * (kD * 2), kp + vbase + k * (kD * 2), hl, on, c2, mm == -INFINITY ? 0.f : mm, d0, out);
      }
    }
  }
  if (!whole) {
    const size_t all = work_rows(a, kFewRows);
    const size_t at = work_at(a, at_tile, h, slice, kFewRows) + ln;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<float4*>(a.work + at * kD + d0 + 8 * i) =
          make_float4(out[4 * i], out[4 * i + 1], out[4 * i + 2], out[4 * i + 3]);
    if (wave == 0 && hl == 0) reinterpret_cast<float2*>(a.work + all * kD)[at] = make_float2(mm, lt);
    return;
  }
  const float inv = lt == 0.f ? 0.f : 1.f / lt;
  uint16_t* op = a.o + (size_t(p.at) + token) * a.q_heads * kD + size_t(head) * kD + d0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint2 u;
    u.x = pack_bf16x2(out[4 * i] * inv, out[4 * i + 1] * inv);
    u.y = pack_bf16x2(out[4 * i + 2] * inv, out[4 * i + 3] * inv);
    *reinterpret_cast<uint2*>(op + 8 * i) = u;
  }
  if (a.lse != nullptr && wave == 0 && hl == 0)
    a.lse[(size_t(p.at) + token) * a.q_heads + head] = lt == 0.f ? -INFINITY : (mm + log2f(lt)) * 0.69314718055994531f;
}

// ---------------------------------------------------------------- join slices ----
//
// Sixteen lanes hold a row's dims, eight each, and LANES / 16 such groups share its
// slices: their offsets and sums first, then their O.  Latency bounds it (entry, range,
// slices, store): 16 lanes a row where slices are few, so that a wave holds four rows (a
// wave a row took 20 us for 32,768 rows of two slices, this 9), 64 where they are many
// (32 rows of 32 slices: 8.5 us with 16).
template <int TILE, int UNIT, int LANES>
__global__ __launch_bounds__(256) void join_kernel(AttnArgs a) {
  constexpr int kGroups = LANES / 16, kRows = 256 / LANES, kOwn = 64 / LANES;   // slices of a lane
  const int H = a.kv_heads, G = a.group;
  const int lane = threadIdx.x & (LANES - 1), c = lane & 15, grp = lane >> 4;
  const uint32_t blocks = uint32_t((a.packed > 0 ? min(a.longest_rows, TILE) : a.longest_rows) + kRows - 1) / kRows;
  const int eh = int(blockIdx.x / blocks);
  int row = int(blockIdx.x % blocks) * kRows + threadIdx.x / LANES;
  const int h = eh % H;
  int e = eh / H, at_tile;                             // of the launch
  if (a.packed > 0) {
    at_tile = e;
    const Place w = tile_place(a, at_tile, TILE);
    if (w.entry < 0) return;
    e = w.entry;
    row += w.tile * TILE;
  } else {
    at_tile = e * a.tiles + row / TILE;
  }
  if (e >= ((const const_i32*)a.step)[0]) return;
  const Part p = step_part(a, e);
  const int rows = p.count * G;
  if (rows < a.least_rows || rows > a.most_rows || row >= rows) return;
  const bool tree = a.tree != nullptr;
  const int row0 = row / TILE * TILE;
  const int first = tree ? p.held : p.held + row0 / G;
  const int last = tree ? p.held + p.count - 1 : p.held + (min(row0 + TILE, rows) - 1) / G;
  const Range range = key_range(first, last, a.window, a.sinks, UNIT);
  const int units = slice_units(range.count, a.slice, a.n_split);
  if (units >= range.count) return;                    // whole: written already
  const int n = (range.count + units - 1) / units;     // at most n_split <= 64
  const size_t all = work_rows(a, TILE), at = work_at(a, at_tile, h, 0, TILE) + (row - row0);
  const float2* mlp = reinterpret_cast<const float2*>(a.work + all * kD) + at;
  float f[kOwn], l[kOwn], mm = -INFINITY, lt = 0.f;
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane + LANES * i < n) ml = mlp[(lane + LANES * i) * TILE];
    f[i] = ml.x;
    l[i] = ml.y;
    mm = fmaxf(mm, ml.x);
  }
#pragma unroll
  for (int s = 1; s < LANES; s <<= 1) mm = fmaxf(mm, __shfl_xor(mm, s, LANES));
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    f[i] = f[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(f[i] - mm);
    lt += l[i] * f[i];
  }
#pragma unroll
  for (int s = 1; s < LANES; s <<= 1) lt += __shfl_xor(lt, s, LANES);
  float x[8] = {};
  const float4* op = reinterpret_cast<const float4*>(a.work + at * kD) + 2 * c;
#pragma unroll
  for (int i = 0; i < kOwn; ++i)
    for (int s0 = LANES * i; s0 < min(n, LANES * (i + 1)); s0 += 4 * kGroups) {
      float4 v[4][2];
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const float4* vp = op + min(s0 + s * kGroups + grp, n - 1) * TILE * (kD / 4);
        v[s][0] = vp[0];
        v[s][1] = vp[1];
      }
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        // 0 past the end, and where a slice's weight underflows: what is not finite there stays so (a row's O is finite
        // in slices that it does not see)
        const float w = __shfl(f[i], (s0 + s * kGroups + grp) & (LANES - 1), LANES);
        x[0] += v[s][0].x * w, x[1] += v[s][0].y * w, x[2] += v[s][0].z * w, x[3] += v[s][0].w * w;
        x[4] += v[s][1].x * w, x[5] += v[s][1].y * w, x[6] += v[s][1].z * w, x[7] += v[s][1].w * w;
      }
    }
#pragma unroll
  for (int s = 16; s < LANES; s <<= 1)
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] += __shfl_xor(x[i], s, LANES);
  if (grp != 0) return;
  const float inv = lt == 0.f ? 0.f : 1.f / lt;
  const int token = row / G, head = h * G + row - token * G;
  const size_t out = (size_t(p.at) + token) * a.q_heads + head;
  reinterpret_cast<uint4*>(a.o)[out * (kD / 8) + c] =
      make_uint4(pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv),
                 pack_bf16x2(x[4] * inv, x[5] * inv), pack_bf16x2(x[6] * inv, x[7] * inv));
  if (a.lse != nullptr && c == 0) a.lse[out] = lt == 0.f ? -INFINITY : (mm + log2f(lt)) * 0.69314718055994531f;
}

template <int TILE, int UNIT>
hipError_t launch_join(const AttnArgs& a, hipStream_t stream) {
  const unsigned pairs = unsigned(a.packed > 0 ? a.packed : a.n) * unsigned(a.kv_heads);
  const int rows = a.packed > 0 ? std::min(a.longest_rows, TILE) : a.longest_rows;
  if (a.n_split <= 4)
    join_kernel<TILE, UNIT, 16><<<unsigned(rows + 15) / 16 * pairs, 256, 0, stream>>>(a);
  else
    join_kernel<TILE, UNIT, 64><<<unsigned(rows + 3) / 4 * pairs, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_rows(const AttnArgs& a, bool paged, hipStream_t stream) {
  const unsigned tiles = a.packed > 0 ? unsigned(a.packed) : unsigned(a.n) * unsigned(a.tiles);
  const unsigned blocks = unsigned(a.kv_heads) * tiles * unsigned(a.n_split);
  if (paged)
    attn_rows_kernel<true><<<blocks, 256, 0, stream>>>(a);
  else
    attn_rows_kernel<false><<<blocks, 256, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_split == 1) return e;
  return launch_join<kRowTile, kKeyUnit>(a, stream);
}

hipError_t launch_attn_few(const AttnArgs& a, hipStream_t stream) {
  const unsigned blocks = unsigned(a.kv_heads) * unsigned(a.packed > 0 ? a.packed : a.n) * unsigned(a.n_split);
  attn_few_kernel<<<blocks, 256, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_split == 1) return e;
  return launch_join<kFewRows, kFewUnit>(a, stream);
}

}  // namespace tok
}  // namespace uf
