// The selection of a beam search: the k best continuations of each request's
// hypotheses, by score_w + (logit_wt - lse_w), equal ones by the lowest (w, t).
//
// What bounds it is one read of the logits.  One launch takes slices of rows: maximum and
// sum of exponentials online, and the slice's k + 1 largest logits; a second joins a request's
// slices, forms the scores, and selects among them.  Scores are rounded, so that different logits
// can give equal ones, and a slice's list, which goes by logits, may have left out an equal
// score of a lower token: where the last of a list has the score of the last selected, and the next smaller or larger logit
// has it too, that score is looked for in the slice again.
//
// A list holds 64-bit keys, the value in an order of integers, then the place, lowest
// first: all different, so that what is selected does not depend on the order in
// which it was found.  In a slice each wave keeps a list of its own in LDS, without a
// barrier: values above a bar join it, and the bar is the n-th largest, at first of the first
// block's maxima (two of each lane), later of the list's values (n values are at or above it, and
// what comes later has a higher place).  A list that might not hold the next block is cut down to its n largest.
//
// 32 requests of 8 beams over 131,072 tokens, bf16, k 16: 26 us of slices (67 MB at 2.6 TB/s) and 9 of joining.  A workgroup's
// eight blocks take 1.2 each, at which rate the slices would be read in 10; before them lie 3 until its first one is there, behind
// them and between, 5 of raising bars, summing and joining lists, at the same time in all workgroups.  One request of 32 beams
// over 200,000, k 64: 40 us (190 with the lists' entries all read by the join).
#include <algorithm>
#include <type_traits>

#include "../launch_states.h"

#include <hip/hip_fp16.h>

namespace uf {
namespace lin {
namespace {

constexpr int kThreads = kOtherThreads, kWaves = 4;
constexpr int kEach = 16;                              // values of a lane and block
constexpr int kBlock = 64 * kEach;                     // of a wave and block
constexpr int kRoom = kBlock + 128, kMine = kRoom / 64;   // keys of a wave's list; of a lane
constexpr int kSplits = 32;                            // slices of a row at most
constexpr int kFew = 128;                              // keys of a list that are put in order by counting
constexpr float kLog2e = 1.44269504f;
constexpr uint32_t kNone = 0x007fffffu;                // -inf in the order of integers: nothing at or below it is taken

// float32 in the order of unsigned integers, -0 as 0.
__device__ inline uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u ^ (uint32_t(int32_t(u) >> 31) | 0x80000000u);
}
__device__ inline float value_of(uint32_t o) { return __uint_as_float(o ^ (uint32_t(~int32_t(o) >> 31) | 0x80000000u)); }
__device__ inline int below_me(uint64_t mask) {        // lanes of the mask before this one
  return __builtin_amdgcn_mbcnt_hi(uint32_t(mask >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(mask), 0));
}
// The largest of the lanes' values.
__device__ inline uint32_t wave_max(uint32_t x) {
  auto step = [&](auto control) {
    x = max(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), decltype(control)::value, 0xf, 0xf, false)));
  };
  step(std::integral_constant<int, 0x111>{});       // from 1, 2, 4 and 8 lanes below in a row of 16
  step(std::integral_constant<int, 0x112>{});
  step(std::integral_constant<int, 0x114>{});
  step(std::integral_constant<int, 0x118>{});
  const uint32_t a = __builtin_amdgcn_readlane(x, 15), b = __builtin_amdgcn_readlane(x, 31), c = __builtin_amdgcn_readlane(x, 47),
                 d = __builtin_amdgcn_readlane(x, 63);
  return max(max(a, b), max(c, d));
}
// A t that n values are at or above, the largest whose last `rest` bits are 0, bit by bit from the first in which `low` and `high` differ: the
// n-th largest lies between them, or there are fewer than n above `low`, and t is at most `low`.  `above` counts over the wave.
// (Loops over bits stay loops here: a workgroup goes through this code once, and waits for every line of it to be fetched.)
template <class Above>
__device__ inline uint32_t nth(int n, uint32_t low, uint32_t high, int rest, Above above) {
  const int first = low == high ? -1 : 31 - __clz(low ^ high);
  uint32_t t = first < 0 ? low : first == 31 ? 0 : low >> (first + 1) << (first + 1);
#pragma unroll 1
  for (int bit = first; bit >= rest; --bit) {
    const uint32_t c = t | (1u << bit);
    if (above(c) >= n) t = c;
  }
  return t;
}

// A wave's list: the n largest keys of what it is shown, among others.  All calls by whole waves.
struct List {
  uint64_t* keys;
  int n;
  bool ascending;                                      // blocks come in the order of their places
  int rest;                                            // last bits that bars do not go by
  int count = 0, seen = 0;                             // keys; of them when the bar was last raised
  uint32_t bar = kNone;                                // values above it pass

  __device__ List(uint64_t* keys_, int n_, bool ascending_, int rest_) : keys(keys_), n(n_), ascending(ascending_), rest(rest_) {}
  // A bar that at least n of the values in a and b, one a lane each, are above.
  __device__ void begin(uint32_t a, uint32_t b) {
    const uint32_t low = ~wave_max(~min(a, b)), high = wave_max(max(a, b));
    bar = max(nth(n, low, high, rest, [&](uint32_t c) { return int(__popcll(__ballot(a >= c))) + int(__popcll(__ballot(b >= c))); }), kNone + 1) - 1;
  }
  // Places for `mine` keys of this lane, 31 at most: the first one.
  __device__ int claim(int mine) {
    int at = count;
#pragma unroll
    for (int b = 0; b < 5; ++b) {
      const uint64_t mask = __ballot((mine >> b) & 1);
      at += below_me(mask) << b;
      count += __popcll(mask) << b;
    }
    return at;
  }
  // Whether any of them passed.
  __device__ bool push(uint32_t order, uint32_t place) {
    const bool in = order > bar;
    const uint64_t mask = __ballot(in);
    if (mask == 0) return false;
    if (in) keys[count + below_me(mask)] = (uint64_t(order) << 32) | uint32_t(~place);
    count += __popcll(mask);
    return true;
  }
  // The bar up to the n-th largest of the list's values, but for its last bits, and what is below it out of the list.
  __device__ void raise() {
    const int lane = threadIdx.x & 63, m = (count + 63) / 64;
    uint32_t mine[kMine];
    uint32_t high = bar;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      mine[i] = 0;
      if (i >= m) break;
      if (lane + 64 * i < count) mine[i] = uint32_t(keys[lane + 64 * i] >> 32);
      high = max(high, mine[i]);
    }
    const uint32_t t = nth(n, bar, wave_max(high), rest, [&](uint32_t c) {
      int found = 0;
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        if (i >= m) break;
        found += __popcll(__ballot(mine[i] >= c));
      }
      return found;
    });
    if (t > kNone) bar = max(bar, ascending ? t : t - 1);
    keep(uint64_t(t) << 32);
  }
  // (in place: what is kept moves down)
  __device__ void keep(uint64_t low) {
    const int lane = threadIdx.x & 63;
    int left = 0;
#pragma unroll 1
    for (int i0 = 0; i0 < count; i0 += 64) {
      const uint64_t key = i0 + lane < count ? keys[i0 + lane] : 0;
      const bool in = i0 + lane < count && key >= low;
      const uint64_t mask = __ballot(in);
      if (in) keys[left + below_me(mask)] = key;
      left += __popcll(mask);
    }
    count = seen = left;
  }
  // Room for the next block, which may all pass; `now`: the bar in any case.
  __device__ void room(int most, bool now) {
    if (!now && count <= seen + 2 * n + 32 && count + most <= kRoom) return;
    raise();
    if (count + most > kRoom) cut();
  }
  // Down to the n largest, where many are equal.
  __device__ void cut() {
    if (count <= n) return;
    const int lane = threadIdx.x & 63;
    uint64_t t = 0;                                    // the n-th largest key, bit by bit
#pragma unroll 1
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t c = t | (uint64_t(1) << bit);
      int found = 0;
#pragma unroll 1
      for (int i0 = 0; i0 < count; i0 += 64) found += __popcll(__ballot(i0 + lane < count && keys[i0 + lane] >= c));
      if (found >= n) t = c;
    }
    keep(t);
    bar = max(bar, uint32_t(t >> 32) - (ascending ? 0u : 1u));
  }
};

// The lists of a workgroup's waves as one: s.out[0 .. n), in order, 0 behind the last.  By all threads; ends with a barrier.
struct Shared {
  uint64_t keys[kWaves][kRoom];
  uint64_t out[kMaxSelect];
  uint32_t low[kWaves];
  int count[2][kWaves], all;                           // (as they come, and cut down)
};
__device__ inline void join(Shared& s, List& list) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (lane == 0) s.low[wave] = list.bar, s.count[0][wave] = list.count;
  for (int i = threadIdx.x; i < list.n; i += kThreads) s.out[i] = 0;
  __syncthreads();
  // what is below any wave's n-th largest is left out (a list's own n-th may equal its bar)
  const uint32_t low = max(max(s.low[0], s.low[1]), max(s.low[2], s.low[3]));
  const bool many = max(max(s.count[0][0], s.count[0][1]), max(s.count[0][2], s.count[0][3])) > kFew;   // (the same for all waves)
  if (many) {
    list.keep(uint64_t(low) << 32);
    if (list.count > kFew) list.cut();
    if (lane == 0) s.count[1][wave] = list.count;
    __syncthreads();
  }
  if (wave == 0) {                                     // the others' into the first list
    list.keep(uint64_t(low) << 32);
    list.bar = low - 1;
#pragma unroll 1
    for (int w = 1; w < kWaves; ++w) {
      const int c = s.count[many][w];
#pragma unroll 1
      for (int i = lane; i - lane < c; i += 64) {
        const uint64_t key = i < c ? s.keys[w][i] : 0;
        list.push(uint32_t(key >> 32), ~uint32_t(key));
      }
    }
    if (list.count > kFew) list.raise();
    if (list.count > kFew) list.cut();
    if (lane == 0) s.all = list.count;
  }
  __syncthreads();
  const int all = s.all;                               // (at most kFew)
  if (int(threadIdx.x) < all) {
    const uint64_t mine = s.keys[0][threadIdx.x];
    int rank = 0;
#pragma unroll 8
    for (int k = 0; k < all; ++k) rank += s.keys[0][k] > mine;
    if (rank < list.n) s.out[rank] = mine;
  }
  __syncthreads();
}

// A row's logits in vectors of 16 bytes, counted from its first element wherever that lies: rows that are alike are
// taken apart alike, and their sums are the same bits.
template <int TYPE>
struct Logits {
  static constexpr int kSize = TYPE == UFS_FP32 ? 4 : 2, kE = 16 / kSize;
  static constexpr int kRest = TYPE == UFS_BF16 ? 16 : TYPE == UFS_FP16 ? 13 : 10;   // last bits: none of the type, or 2^-13
  const uint8_t* row;
  int vocab;
  __device__ Logits(const SelectArgs& a, int w, int g) {
    row = static_cast<const uint8_t*>(a.logits) + (g * a.group_stride + w * a.beam_stride) * kSize;
    vocab = a.vocab;
  }
  __device__ static float value(uint32_t bits) {
    if (TYPE == UFS_BF16) return __uint_as_float(bits << 16);
    if (TYPE == UFS_FP16) return __half2float(__ushort_as_half(uint16_t(bits)));
    return __uint_as_float(bits);
  }
  // The value next to a finite one, in the logits' own type.
  __device__ static float next(float x, bool up) {
    auto step = [&](uint32_t u, uint32_t sign) { return (u & ~sign) == 0 ? (up ? 1u : sign | 1u) : ((u & sign) != 0) == up ? u - 1 : u + 1; };
    if (TYPE == UFS_BF16) return value(step(__float_as_uint(x) >> 16, 0x8000u));
    if (TYPE == UFS_FP16) return value(step(__half_as_ushort(__float2half(x)), 0x8000u));
    return value(step(__float_as_uint(x), 0x80000000u));
  }
  // A vector's bits; elements that the row does not have are -inf.
  __device__ uint4 bits(int vector) const {
    const int t = vector * kE;
    if (t + kE <= vocab) {
      uint4 u;
      __builtin_memcpy(&u, row + int64_t(t) * kSize, 16);   // (one load: any alignment will do)
      return u;
    }
    uint32_t b[kE], w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < kE; ++e) {                     // (all of them in flight, the row's last one in the place of those it lacks)
      const int at = min(t + e, vocab - 1);
      b[e] = kSize == 2 ? uint32_t(reinterpret_cast<const uint16_t*>(row)[at]) : reinterpret_cast<const uint32_t*>(row)[at];
    }
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      if (t + e >= vocab) b[e] = TYPE == UFS_BF16 ? 0xff80u : TYPE == UFS_FP16 ? 0xfc00u : 0xff800000u;
      if (kSize == 2) w[e / 2] |= b[e] << (16 * (e & 1));
      else w[e] = b[e];
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ static void unpack(const uint4& u, float* x) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < kE; ++e) x[e] = kSize == 2 ? value((w[e / 2] >> (16 * (e & 1))) & 0xffffu) : value(w[e]);
  }
};

// A slice's results: its maximum, rounded up, and sum of exponentials by it, then its list of k + 1 (lanes bound a list to 64).
__device__ __host__ inline int listed_of(int k) { return k + 1 < 64 ? k + 1 : 64; }
__device__ __host__ inline size_t slice_bytes(int k) { return 16 + size_t(listed_of(k)) * 8; }

template <int TYPE>
__global__ __launch_bounds__(kThreads) void select_slices_kernel(SelectArgs a) {
  using L = Logits<TYPE>;
  constexpr int kE = L::kE;
  constexpr int kVectors = kEach / kE;                 // of a lane and block
  __shared__ Shared s;
  __shared__ float stop[kWaves];
  __shared__ double ssum[kWaves];
  const int row = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
  const float score = a.scores[row];                   // (both loads before either is looked at)
  const int ended = a.done != nullptr ? a.done[row] : 0;
  if (!(score > -INFINITY) || ended != 0) return;
  const L x(a, row % a.beams, row / a.beams);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // the waves take the slice's blocks in turn
  const int v1 = min((split + 1) * a.slice, (a.vocab + kE - 1) / kE), step = kWaves * 64 * kVectors;
  const int v0 = split * a.slice + wave * 64 * kVectors;

  List list(s.keys[wave], listed_of(a.k), true, L::kRest);
  // Exponentials go by the maximum so far rounded up to an integer, so that a sum is weighed anew only where it falls to 1 / e or
  // less; a block's sixteen are added in fp32, blocks in 64 bits (1,024 blocks of equal terms in fp32 had lse off by 1.5e-5).
  float top = -INFINITY;
  double sum = 0.0;
  uint4 next[2][kVectors];                             // two blocks ahead
  auto fetch = [&](uint4 (&to)[kVectors], int v) {
#pragma unroll
    for (int u = 0; u < kVectors; ++u) to[u] = x.bits(v + 64 * u + lane < v1 ? v + 64 * u + lane : (1 << 27));
  };
  auto block = [&](const uint4 (&bits)[kVectors], int v) {
    float y[kVectors][kE];
#pragma unroll
    for (int u = 0; u < kVectors; ++u) L::unpack(bits[u], y[u]);
    float half[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int u = 0; u < kVectors; ++u)
#pragma unroll
      for (int e = 0; e < kE; ++e) half[2 * u / kVectors] = fmaxf(half[2 * u / kVectors], y[u][e]);
    const float most = fmaxf(half[0], half[1]);
    if (most > top) {
      const float up = ceilf(most);
      sum *= double(__builtin_amdgcn_exp2f((top - up) * kLog2e));
      top = up;
    }
    const float off = top > -INFINITY ? top : 0.f;
    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < kVectors; ++u)
#pragma unroll
      for (int e = 0; e < kE; ++e) part[e & 3] += __builtin_amdgcn_exp2f((y[u][e] - off) * kLog2e);
    sum += double((part[0] + part[1]) + (part[2] + part[3]));
    if (v == v0) list.begin(ordered(half[0]), ordered(half[1]));
    // the bar as a value: -inf where all pass; the place between 0 and the largest value below it is no other value's
    const float bar = value_of(list.bar == 0x7fffffffu ? 0x7ffffffeu : list.bar);
    if (__ballot(most > bar) != 0) {
      int passed = 0;
#pragma unroll
      for (int u = 0; u < kVectors; ++u)
#pragma unroll
        for (int e = 0; e < kE; ++e) passed += y[u][e] > bar;
      uint64_t* to = list.keys + list.claim(passed);
#pragma unroll
      for (int u = 0; u < kVectors; ++u)
#pragma unroll
        for (int e = 0; e < kE; ++e)
          if (y[u][e] > bar) *to++ = (uint64_t(ordered(y[u][e])) << 32) | uint32_t(~uint32_t((v + 64 * u + lane) * kE + e));
    }
    list.room(kBlock, v + step >= v1 && list.count > max(2 * list.n, 24));
  };
  fetch(next[0], v0);
  fetch(next[1], v0 + step);
#pragma unroll 1
  for (int v = v0; v < v1; v += step) {
    uint4 now[kVectors];
#pragma unroll
    for (int u = 0; u < kVectors; ++u) now[u] = next[0][u], next[0][u] = next[1][u];
    if (v + 2 * step < v1) fetch(next[1], v + 2 * step);
    block(now, v);
  }
  // the slice's maximum and sum
  float all = top;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) all = fmaxf(all, __shfl_xor(all, d));
  if (lane == 0) stop[wave] = all;
  __syncthreads();
  all = fmaxf(fmaxf(stop[0], stop[1]), fmaxf(stop[2], stop[3]));
  double part = sum != 0.0 ? sum * double(__builtin_amdgcn_exp2f((top - all) * kLog2e)) : 0.0;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) part += __shfl_xor(part, d);
  if (lane == 0) ssum[wave] = part;
  join(s, list);
  uint8_t* const to = a.work + size_t(blockIdx.x) * slice_bytes(a.k);
  if (tid == 0) *reinterpret_cast<float2*>(to) = make_float2(all, float((ssum[0] + ssum[1]) + (ssum[2] + ssum[3])));
  if (tid < list.n) reinterpret_cast<uint64_t*>(to + 16)[tid] = s.out[tid];
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void select_join_kernel(SelectArgs a) {
  using L = Logits<TYPE>;
  constexpr int kE = L::kE;
  __shared__ Shared s;
  __shared__ float slse[kMaxBeams], sscore[kMaxBeams];
  __shared__ uint8_t skind[kMaxBeams];                 // 0: not in use, 1: goes on, 2: finished
  const int g = blockIdx.x, W = a.beams, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint8_t* const work = a.work + size_t(g) * W * a.splits * slice_bytes(a.k);
  auto slice_at = [&](int i) { return work + size_t(i) * slice_bytes(a.k); };
  const int n = listed_of(a.k), slices = W * a.splits, listed = slices * n;

  // A wave takes a quarter of the slices, their first entries before their second ones and so on: none of a slice's passes once one
  // has not, so that it is through when none of as many as it has slices did.  The first of them come while the sums are joined.
  constexpr int kHeld = 4;
  const int own = (slices + kWaves - 1) / kWaves;
  uint64_t held[kHeld];
  int from[kHeld];
  auto fetch = [&](uint64_t (&held)[kHeld], int (&from)[kHeld], int i0) {
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
      const int i = i0 + lane + 64 * u, level = i / own;
      from[u] = (i - level * own) * kWaves + wave;
      held[u] = level < n && from[u] < slices ? reinterpret_cast<const uint64_t*>(slice_at(from[u]) + 16)[level] : 0;
    }
  };
  fetch(held, from, 0);
  auto last_of = [&](int i) { return reinterpret_cast<const uint64_t*>(slice_at(i) + 16)[n - 1]; };
  const uint64_t last_held = tid < slices ? last_of(tid) : 0;
  // eight lanes a row
  for (int w0 = 0; w0 < W; w0 += kThreads / 8) {
    const int w = w0 + tid / 8, part = tid % 8;
    const float score = w < W ? a.scores[g * W + w] : -INFINITY;
    int kind = score > -INFINITY ? 1 : 0;
    if (w < W && a.done != nullptr && a.done[g * W + w] != 0) kind *= 2;
    float2 t[kSplits / 8];
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kSplits / 8; ++i) {
      t[i] = make_float2(-INFINITY, 0.f);              // (anything where the row is not read)
      if (w < W && part + 8 * i < a.splits) t[i] = *reinterpret_cast<const float2*>(slice_at(w * a.splits + part + 8 * i));
    }
#pragma unroll
    for (int i = 0; i < kSplits / 8; ++i) top = fmaxf(top, t[i].x);
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kSplits / 8; ++i) sum += t[i].y != 0.f ? double(t[i].y * __builtin_amdgcn_exp2f((t[i].x - top) * kLog2e)) : 0.0;
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) sum += __shfl_xor(sum, d);
    if (part == 0 && w < W) {
      slse[w] = kind == 1 ? float(double(top) + log(sum)) : 0.f;
      sscore[w] = score;
      skind[w] = uint8_t(kind);
    }
  }
  __syncthreads();
  auto score_of = [&](int w, float logit) { return sscore[w] + (logit - slse[w]); };   // (float32 each)
  auto order_of = [&](float score) { return score > -INFINITY ? ordered(score) : 0u; };   // NaN is no candidate
  // Whether a slice may have left out one that is selected, where `limit` is the lowest score selected: an equal one of a lower place than a
  // listed one, which has a larger logit then: the last one's next smaller logit has the limit's score too, or the last one's next larger.
  auto again = [&](int i, uint32_t limit) {
    const int w = i / a.splits;
    if (skind[w] != 1) return false;
    const uint64_t last = i == tid ? last_held : last_of(i);
    if (uint32_t(last >> 32) <= kNone) return false;   // (it has fewer: none was left out)
    const float x = value_of(uint32_t(last >> 32)), score = score_of(w, x);
    return order_of(score) > kNone && order_of(score) >= limit && (score_of(w, L::next(x, false)) == score || score_of(w, L::next(x, true)) == score);
  };
  // An entry of a slice as a candidate: its score, and its place.
  auto candidate = [&](int slice, uint64_t key, uint32_t* place) {
    const int w = min(slice / a.splits, W - 1);
    if (uint32_t(key >> 32) <= kNone || skind[w] != 1) return 0u;
    *place = uint32_t(w) * uint32_t(a.vocab) + uint32_t(~uint32_t(key));
    return order_of(score_of(w, value_of(uint32_t(key >> 32))));
  };
  auto finished = [&](List& list) {
    if (wave == 0) {
      list.room(64, false);
      const bool ends = lane < W && skind[lane] == 2;
      list.push(ends ? order_of(sscore[lane]) : 0u, uint32_t(lane) * uint32_t(a.vocab) + uint32_t(a.end));
    }
  };

  {
    List list(s.keys[wave], a.k, false, 10);
    uint32_t order[kHeld], places[kHeld];
    int last = 0;                                      // behind the last that passed
    for (int i0 = 0; i0 < n * own && i0 - last < own; i0 += 64 * kHeld) {
      uint64_t next[kHeld];
      int next_from[kHeld];
      fetch(next, next_from, i0 + 64 * kHeld);
      uint32_t top[2] = {0, 0};
#pragma unroll
      for (int u = 0; u < kHeld; ++u) {
        order[u] = candidate(from[u], held[u], &places[u]);
        top[2 * u / kHeld] = max(top[2 * u / kHeld], order[u]);
      }
      if (i0 == 0) list.begin(top[0], top[1]);
      list.room(64 * kHeld, false);
#pragma unroll
      for (int u = 0; u < kHeld; ++u)
        if (list.push(order[u], places[u])) last = i0 + 64 * (u + 1);
#pragma unroll
      for (int u = 0; u < kHeld; ++u) held[u] = next[u], from[u] = next_from[u];
    }
    finished(list);
    if (list.count > max(2 * list.n, 24)) list.raise();   // (few: the lists' join takes them as they are)
    join(s, list);
  }
  const uint32_t limit = uint32_t(s.out[a.k - 1] >> 32);
  int reads = 0;
  for (int i = tid; i < slices; i += kThreads) reads |= again(i, limit);
  if (__syncthreads_or(reads)) {
    // All scores above the limit are listed (a slice that left one out would list k of them).  Equal ones of those slices are looked for in the
    // order of their places, until there are k: rows of equal logits have them at once (one request, 131,072 of them: 176 us, of which
    // cutting the lists down to k takes most; 4,210 where slices were read to their ends, and each block's entries put in order).
    List list(s.keys[wave], a.k, false, 10);
    list.bar = limit - 1;
    for (int i0 = 0; i0 < listed; i0 += kThreads) {
      const int i = i0 + tid;
      uint32_t place = 0, o = 0;
      if (i < listed) o = candidate(i / n, reinterpret_cast<const uint64_t*>(slice_at(i / n) + 16)[i % n], &place);
      if (o == limit && again(i / n, limit)) o = 0;
      list.room(64, false);
      list.push(o, place);
    }
    finished(list);
    int found = 0;                                     // in the slices so far
    for (int i = 0; i < slices && found < a.k; ++i) {
      if (__ballot(again(i, limit)) == 0) continue;    // (the same for all threads)
      const int w = i / a.splits;
      const L x(a, w, g);
      const int v1 = min((i % a.splits + 1) * a.slice, (a.vocab + kE - 1) / kE);
      int own = 0;                                     // this wave's: k of them have lower places than what it has not read
      for (int v = (i % a.splits) * a.slice + wave * 64; v < v1 && own < a.k; v += kThreads) {
        float y[kE];
        L::unpack(x.bits(v + lane < v1 ? v + lane : (1 << 27)), y);
        list.room(64 * kE, false);
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          const bool equal = order_of(score_of(w, y[e])) == limit;
          list.push(equal ? limit : 0u, uint32_t(w) * uint32_t(a.vocab) + uint32_t((v + lane) * kE + e));
          own += __popcll(__ballot(equal));
        }
      }
      if (lane == 0) s.count[0][wave] = own;
      __syncthreads();
      found += (s.count[0][0] + s.count[0][1]) + (s.count[0][2] + s.count[0][3]);
      __syncthreads();
    }
    list.raise();
    __syncthreads();
    join(s, list);
  }
  if (tid < a.k) {
    const uint64_t key = s.out[tid];
    const bool there = uint32_t(key >> 32) > kNone;
    const uint32_t place = ~uint32_t(key);
    const int at = g * a.k + tid;
    a.best[at] = there ? value_of(uint32_t(key >> 32)) : -INFINITY;
    a.parents[at] = there ? int32_t(place / uint32_t(a.vocab)) : -1;
    a.tokens[at] = there ? int32_t(place % uint32_t(a.vocab)) : -1;
  }
}

template <int TYPE>
hipError_t run(const SelectArgs& a, hipStream_t stream) {
  select_slices_kernel<TYPE><<<dim3(unsigned(a.groups) * a.beams * a.splits), kThreads, 0, stream>>>(a);
  if (hipError_t e = hipGetLastError()) return e;
  select_join_kernel<TYPE><<<dim3(unsigned(a.groups)), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

// Rows are cut into slices for 1,024 workgroups (four a CU) in all, 32 slices at most.  256 / 512 / 1,024 / 2,048 / 4,096 workgroups, bf16
// (us): 32 x 8 rows of 131,072 tokens 45.0 / 35.6 / 33.7 / 38.3 / 47.2; 64 x 1 20.9 / 18.1 / 17.5 / 22.0 / 21.8; 8 x 8 of 200,000 28.8 / 24.9
// / 24.1 / 28.3 / 28.2; 64 x 4 of 32,000 21.9 / 19.1 / 18.8 / 22.6 / 22.8; but 1 x 32 of 200,000, one join for all, 29.5 / 30.8 / 35.4 / 35.5 /
// 35.3.  16 / 32 / 64 slices: 1 row of 2,000,000 43.2 / 30.6 / 24.0; 1 x 32 of 200,000 30.8 / 35.4 / 35.5; the others the same.
void plan_select(SelectArgs* a) {
  const int e = a->type == UFS_FP32 ? 4 : 8, block = kWaves * kBlock / e;
  const int64_t vectors = (int64_t(a->vocab) + e - 1) / e, rows = int64_t(a->groups) * a->beams;
  const int64_t blocks = (vectors + block - 1) / block;
  const int64_t splits = std::max<int64_t>(1, std::min<int64_t>({blocks, kSplits, (1024 + rows - 1) / rows}));
  a->slice = int32_t((blocks + splits - 1) / splits * block);
  a->splits = int32_t((vectors + a->slice - 1) / a->slice);
}

size_t select_work_bytes(const SelectArgs& a) { return size_t(a.groups) * a.beams * a.splits * slice_bytes(a.k); }

hipError_t launch_select(const SelectArgs& a, hipStream_t stream) {
  if (a.type == UFS_BF16) return run<UFS_BF16>(a, stream);
  if (a.type == UFS_FP16) return run<UFS_FP16>(a, stream);
  return run<UFS_FP32>(a, stream);
}

}  // namespace lin
}  // namespace uf
