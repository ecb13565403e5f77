// The selection of a beam search: the k best continuations of each request's
// hypotheses, by score_w + (logit_wt - lse_w), equal ones by the lowest (w, t).
//
// What bounds it is one read of the logits.  One launch takes slices of rows: maximum and
// sum of exponentials online, and the slice's k + 1 largest logits; a second joins a request's
// slices, forms the scores, and selects among them.  Scores are rounded, so that different logits
// can give equal ones, and a slice's list, which goes by logits, may have left out an equal
// score of a lower token: where the last of a list has the score of the last selected, and a smaller logit could have
// it too, that slice is read again by scores.
//
// A list holds 64-bit keys, the value in an order of integers, then the place, lowest
// first: all different, so that what is selected does not depend on the order in
// which threads add to it.  The first block's threshold comes from the lanes' maxima: each of
// four waves has ceil(n / 4) lanes at or above its own such maximum, so that n
// values are at or above the least of the four.  Later values pass only above it; what
// passes lies in LDS, and is cut down to the n largest where the next block might not fit.
#include <algorithm>

#include "../launch_states.h"

#include <hip/hip_fp16.h>

namespace uf {
namespace lin {
namespace {

constexpr int kThreads = 256, kVectors = 2;            // 16-byte vectors of a thread and block
constexpr int kBlock = kThreads * kVectors * 8;        // values of a block at most
constexpr int kRoom = kBlock + kThreads;               // keys in LDS
constexpr int kMine = kRoom / kThreads;                // of a thread
constexpr uint32_t kNone = 0x007fffffu;                // -inf in the order of integers: nothing at or below it is taken

// float32 in the order of unsigned integers, -0 as 0.
__device__ inline uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u ^ (uint32_t(int32_t(u) >> 31) | 0x80000000u);
}
__device__ inline float value_of(uint32_t o) { return __uint_as_float(o ^ (uint32_t(~int32_t(o) >> 31) | 0x80000000u)); }

struct Shared {
  uint64_t keys[kRoom];
  uint64_t out[kMaxSelect + 1];
  uint32_t count, sum[2];
  uint32_t low[4];
};

// The n largest keys of what a workgroup is shown.
struct Best {
  Shared& s;
  int n;
  bool ascending;                                      // blocks come in the order of their places
  uint32_t bar = kNone;                                // values above it pass

  __device__ Best(Shared& s_, int n_, bool ascending_) : s(s_), n(n_), ascending(ascending_) {
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
  }
  // A bar from the threads' largest values so far (`top`), of which at least n have to stay above it.
  __device__ void set_bar(uint32_t top) {
    const int want = (n + 3) / 4;
    uint32_t t = 0;
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t c = t | (1u << bit);
      if (__popcll(__ballot(top >= c)) >= want) t = c;
    }
    if ((threadIdx.x & 63) == 0) s.low[threadIdx.x >> 6] = t;
    __syncthreads();
    const uint32_t low = min(min(s.low[0], s.low[1]), min(s.low[2], s.low[3]));
    bar = max(low, kNone + 1) - 1;
    __syncthreads();
  }
  __device__ void push(uint32_t order, uint32_t place) {
    if (order > bar) s.keys[atomicAdd(&s.count, 1u)] = (uint64_t(order) << 32) | uint32_t(~place);
  }
  // Before a block of `most` values: room for them.  (Ends with a barrier.)
  __device__ void room(int most) {
    __syncthreads();
    const int c = int(s.count);
    __syncthreads();                                   // (nobody adds before all have read it)
    if (c + most > kRoom) shrink();
  }
  __device__ void shrink() {                           // by all threads
    uint64_t mine[kMine];
    const int c = int(s.count);
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int at = int(threadIdx.x) + i * kThreads;
      mine[i] = at < c ? s.keys[at] : 0;
    }
    if (c <= n) return;
    if (threadIdx.x < 2) s.sum[threadIdx.x] = 0;
    __syncthreads();
    uint64_t t = 0;                                    // the n-th largest, bit by bit
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t cand = t | (uint64_t(1) << bit);
      uint32_t found = 0;
#pragma unroll
      for (int i = 0; i < kMine; ++i) found += __popcll(__ballot(mine[i] >= cand));
      if ((threadIdx.x & 63) == 0) atomicAdd(&s.sum[bit & 1], found);
      __syncthreads();
      if (int(s.sum[bit & 1]) >= n) t = cand;
      if (threadIdx.x == 0) s.sum[(bit & 1) ^ 1] = 0;
      __syncthreads();
    }
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMine; ++i)
      if (mine[i] >= t) s.keys[atomicAdd(&s.count, 1u)] = mine[i];
    // what equals the last one has a higher place if it comes later, or may have a lower one
    bar = max(bar, uint32_t(t >> 32) - (ascending ? 0u : 1u));
    __syncthreads();
  }
  // s.out[0 .. n): the largest, in order, 0 behind the last.  (Ends with a barrier.)
  __device__ void finish() {
    __syncthreads();
    if (s.count > 2 * kThreads) shrink();
    const int c = int(s.count);
    for (int i = threadIdx.x; i < n; i += kThreads)
      if (i >= c) s.out[i] = 0;
    for (int i = threadIdx.x; i < c; i += kThreads) {
      const uint64_t mine = s.keys[i];
      int rank = 0;
      for (int k = 0; k < c; ++k) rank += s.keys[k] > mine;
      if (rank < n) s.out[rank] = mine;
    }
    __syncthreads();
  }
};

// A row's logits in vectors of 16 bytes, counted from its first element wherever that lies: rows that are alike are
// taken apart alike, and their sums are the same bits.
template <int TYPE>
struct Logits {
  static constexpr int kSize = TYPE == UFS_FP32 ? 4 : 2, kE = 16 / kSize;
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
  // The largest value below a finite one, in the logits' own type.
  __device__ static float below(float x) {
    auto down = [](uint32_t u, uint32_t sign) { return (u & ~sign) == 0 ? (sign | 1u) : (u & sign) ? u + 1 : u - 1; };
    if (TYPE == UFS_BF16) return value(down(__float_as_uint(x) >> 16, 0x8000u));
    if (TYPE == UFS_FP16) return value(down(__half_as_ushort(__float2half(x)), 0x8000u));
    return value(down(__float_as_uint(x), 0x80000000u));
  }
  // A vector's bits; elements that the row does not have are -inf.
  __device__ uint4 bits(int vector) const {
    const int t = vector * kE;
    if (t + kE <= vocab) {
      uint4 u;
      __builtin_memcpy(&u, row + int64_t(t) * kSize, 16);   // (one load: any alignment will do)
      return u;
    }
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      uint32_t b = TYPE == UFS_BF16 ? 0xff80u : TYPE == UFS_FP16 ? 0xfc00u : 0xff800000u;
      if (t + e < vocab)
        b = kSize == 2 ? uint32_t(reinterpret_cast<const uint16_t*>(row)[t + e]) : reinterpret_cast<const uint32_t*>(row)[t + e];
      if (kSize == 2) w[e / 2] |= b << (16 * (e & 1));
      else w[e] = b;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ static void unpack(const uint4& u, float* x) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < kE; ++e) x[e] = kSize == 2 ? value((w[e / 2] >> (16 * (e & 1))) & 0xffffu) : value(w[e]);
  }
};

// A slice's results: its maximum and sum of exponentials, then its list.
__device__ __host__ inline size_t slice_bytes(int k) { return 16 + size_t(k + 1) * 8; }
struct Slice {
  float top, sum;
  uint64_t unused;
};

__device__ inline bool in_use(const SelectArgs& a, int row) { return a.scores[row] > -INFINITY; }

template <int TYPE>
__global__ __launch_bounds__(kThreads) void select_slices_kernel(SelectArgs a) {
  using L = Logits<TYPE>;
  constexpr int kE = L::kE;
  __shared__ Shared s;
  __shared__ float stop[4];
  __shared__ double ssum[4];
  const int row = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
  if (!in_use(a, row) || (a.done != nullptr && a.done[row] != 0)) return;
  const L x(a, row % a.beams, row / a.beams);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int v0 = split * a.slice, v1 = min(v0 + a.slice, (a.vocab + kE - 1) / kE);

  Best best(s, a.k + 1, true);
  float top = -INFINITY, sum = 0.f;
  uint4 next[kVectors];
  auto fetch = [&](int v) {
#pragma unroll
    for (int u = 0; u < kVectors; ++u) next[u] = x.bits(v + u * kThreads + tid < v1 ? v + u * kThreads + tid : (1 << 27));
  };
  fetch(v0);
  for (int v = v0; v < v1; v += kThreads * kVectors) {
    float y[kVectors][kE];
#pragma unroll
    for (int u = 0; u < kVectors; ++u) L::unpack(next[u], y[u]);
    if (v + kThreads * kVectors < v1) fetch(v + kThreads * kVectors);
    float most = -INFINITY;
#pragma unroll
    for (int u = 0; u < kVectors; ++u)
#pragma unroll
      for (int e = 0; e < kE; ++e) most = fmaxf(most, y[u][e]);
    if (most > top) {
      sum *= __builtin_amdgcn_exp2f((top - most) * 1.44269504f);
      top = most;
    }
    const float off = top > -INFINITY ? top : 0.f;
#pragma unroll
    for (int u = 0; u < kVectors; ++u)
#pragma unroll
      for (int e = 0; e < kE; ++e) sum += __builtin_amdgcn_exp2f((y[u][e] - off) * 1.44269504f);
    const uint32_t order = ordered(most);
    if (v == v0) best.set_bar(order);
    else best.room(kThreads * kVectors * kE);
    if (order > best.bar) {
#pragma unroll
      for (int u = 0; u < kVectors; ++u)
#pragma unroll
        for (int e = 0; e < kE; ++e) best.push(ordered(y[u][e]), uint32_t((v + u * kThreads + tid) * kE + e));
    }
  }
  // the slice's maximum and sum
  float all = top;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) all = fmaxf(all, __shfl_xor(all, d));
  if (lane == 0) stop[wave] = all;
  __syncthreads();
  all = fmaxf(fmaxf(stop[0], stop[1]), fmaxf(stop[2], stop[3]));
  double part = sum != 0.f ? double(sum) * exp(double(top) - double(all)) : 0.0;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) part += __shfl_xor(part, d);
  if (lane == 0) ssum[wave] = part;
  best.finish();
  uint8_t* const to = a.work + size_t(blockIdx.x) * slice_bytes(a.k);
  if (tid == 0) {
    reinterpret_cast<float*>(to)[0] = all;
    reinterpret_cast<float*>(to)[1] = float(ssum[0] + ssum[1] + (ssum[2] + ssum[3]));
  }
  if (tid <= a.k) reinterpret_cast<uint64_t*>(to + 16)[tid] = s.out[tid];
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void select_join_kernel(SelectArgs a) {
  using L = Logits<TYPE>;
  constexpr int kE = L::kE;
  __shared__ Shared s;
  __shared__ float slse[kMaxBeams], sscore[kMaxBeams];
  __shared__ uint8_t skind[kMaxBeams];                 // 0: not in use, 1: goes on, 2: finished
  __shared__ int sagain;
  const int g = blockIdx.x, W = a.beams, tid = threadIdx.x;
  const uint8_t* const work = a.work + size_t(g) * W * a.splits * slice_bytes(a.k);
  auto slice_at = [&](int i) { return work + size_t(i) * slice_bytes(a.k); };
  for (int w = tid; w < W; w += kThreads) {
    const float score = a.scores[g * W + w];
    int kind = score > -INFINITY ? 1 : 0;
    if (a.done != nullptr && a.done[g * W + w] != 0) kind *= 2;
    float lse = 0.f;
    if (kind == 1) {
      float top = -INFINITY;
      for (int i = 0; i < a.splits; ++i) top = fmaxf(top, *reinterpret_cast<const float*>(slice_at(w * a.splits + i)));
      double sum = 0.0;
      for (int i = 0; i < a.splits; ++i) {
        const float2 t = *reinterpret_cast<const float2*>(slice_at(w * a.splits + i));
        sum += t.y != 0.f ? double(t.y) * exp(double(t.x) - double(top)) : 0.0;
      }
      lse = float(double(top) + log(sum));
    }
    slse[w] = lse;
    sscore[w] = score;
    skind[w] = uint8_t(kind);
  }
  __syncthreads();
  auto score_of = [&](int w, float logit) { return sscore[w] + (logit - slse[w]); };   // (float32 each)
  // NaN is no candidate
  auto order_of = [&](float score) { return score > -INFINITY ? ordered(score) : 0u; };

  // first by the slices' lists; then, where some have to be read again, by those slices' scores and the others' lists
  const int listed = W * a.splits * (a.k + 1);
  for (int pass = 0; pass < 2; ++pass) {
    Best best(s, a.k, false);
    const uint32_t limit = pass == 0 ? 0u : uint32_t(s.out[a.k - 1] >> 32);   // the score that decides
    auto again = [&](int i) {                          // whether slice i has to be read again
      const int w = i / a.splits;
      if (skind[w] != 1) return false;
      const uint64_t last = reinterpret_cast<const uint64_t*>(slice_at(i) + 16)[a.k];
      if (uint32_t(last >> 32) <= kNone) return false;   // (it has fewer: none was left out)
      const float x = value_of(uint32_t(last >> 32)), score = score_of(w, x);
      return order_of(score) > kNone && order_of(score) >= limit && score_of(w, L::below(x)) == score;
    };
    if (pass == 1) {
      if (tid == 0) sagain = 0;
      __syncthreads();
      for (int i = tid; i < W * a.splits; i += kThreads)
        if (again(i)) sagain = 1;
      __syncthreads();
      if (sagain == 0) break;
    }
    auto candidate = [&](int i, uint32_t* place) {      // entry i of the lists
      const int slice = i / (a.k + 1), w = slice / a.splits;
      if (i >= listed || skind[w] != 1) return 0u;
      const uint64_t key = reinterpret_cast<const uint64_t*>(slice_at(slice) + 16)[i - slice * (a.k + 1)];
      if (uint32_t(key >> 32) <= kNone || (pass == 1 && again(slice))) return 0u;
      *place = uint32_t(w) * uint32_t(a.vocab) + uint32_t(~uint32_t(key));
      return order_of(score_of(w, value_of(uint32_t(key >> 32))));
    };
    uint32_t top = 0, place = 0;
    for (int i = tid; i < listed; i += kThreads) top = max(top, candidate(i, &place));
    best.set_bar(top);
    for (int i0 = 0; i0 < listed; i0 += kThreads) {
      const uint32_t order = candidate(i0 + tid, &place);
      best.room(kThreads);
      best.push(order, place);
    }
    best.room(kThreads);
    if (tid < W && skind[tid] == 2) best.push(order_of(sscore[tid]), uint32_t(tid) * uint32_t(a.vocab) + uint32_t(a.end));
    if (pass == 1)
      for (int i = 0; i < W * a.splits; ++i) {
        if (!again(i)) continue;
        const int w = i / a.splits;
        const L x(a, w, g);
        const int v0 = (i % a.splits) * a.slice, v1 = min(v0 + a.slice, (a.vocab + kE - 1) / kE);
        for (int v = v0; v < v1; v += kThreads) {
          float y[kE];
          L::unpack(x.bits(v + tid < v1 ? v + tid : (1 << 27)), y);
          best.room(kThreads * kE);
#pragma unroll
          for (int e = 0; e < kE; ++e)
            best.push(order_of(score_of(w, y[e])), uint32_t(w) * uint32_t(a.vocab) + uint32_t((v + tid) * kE + e));
        }
      }
    best.finish();
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

void plan_select(SelectArgs* a) {
  const int e = a->type == UFS_FP32 ? 4 : 8, block = kThreads * kVectors;
  const int64_t vectors = (int64_t(a->vocab) + e - 1) / e, rows = int64_t(a->groups) * a->beams;
  const int64_t blocks = (vectors + block - 1) / block;
  const int64_t splits = std::max<int64_t>(1, std::min<int64_t>({blocks, 32, (1024 + rows - 1) / rows}));
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
