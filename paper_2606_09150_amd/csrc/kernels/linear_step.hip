// The recurrent form of linear attention (a few new tokens a sequence), and the states
// that move between sequences.
//
// What bounds all three is HBM: a state of 64 KB is read and written for 256 bytes of k and
// v, and products and sums are done in fp32 on the vector ALUs beside it.
//
// A step's wave holds 32 columns (of v: whole cache lines) of a state in registers, a lane four columns of 16
// rows, loads in flight all at once.  It takes its sequence's tokens one by one, S = L S + k v^T and
// o = scale S^T q, rows summed over lanes; no wave waits for another.  64 sequences of 32 key heads, one token: 41 us, 272 MB
// at 6.6 TB/s.  (Fewer columns a wave have XCDs read each other's lines: 192 states, 1 token, 6.9 us of 32 columns, 13 of
// 16, 19.6 of 8.)
//
// Where states are few a wave has 32 of their rows, all tokens' k, v and queries come through LDS at once,
// and the waves' sums meet there behind the last token: a wave's way through a token is as long as its part of a state.
// Rows split / whole (us): 192 states of 2 query heads, 4 tokens 9.6 / 10.9; 512 states, 2 tokens 14.9 / 11.8.
//
// L goes as two floats: one would be off by the same 2^-25 in each of thousands of steps.
#include <algorithm>

#include "linear_place.h"

namespace uf {
namespace lin {
namespace {

using namespace attn;

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = kOtherThreads;

// Sums over the lanes of the same columns (lane % 8), in all of them.
__device__ inline float column_sum(float x) {
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), 0x128, 0xf, 0xf, false));   // lane ^ 8
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}
template <int N>
struct Dims {                                          // N dimensions of a row, bf16
  typedef uint32_t words __attribute__((ext_vector_type(N / 2)));
  words w;
  __device__ static Dims of(const uint16_t* p) { return Dims{*reinterpret_cast<const words*>(p)}; }
  __device__ void unpack(float (&x)[N]) const {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};

constexpr int kCols = 32, kSums = 64;                  // columns of a wave; (token, query head) pairs whose sums LDS holds
// SPLIT: the waves of a workgroup have the rows of the same columns, or the columns of the same state.
template <bool SPLIT>
__global__ __launch_bounds__(kThreads) void linear_step_kernel(StepArgs a) {
  constexpr int kRows = SPLIT ? 4 : 16;                // of a lane
  __shared__ float sums[SPLIT ? kSums : 1][4][kCols];
  __shared__ __attribute__((aligned(16))) uint16_t sk[SPLIT ? kFewTokens : 1][kD], sv[SPLIT ? kFewTokens : 1][kCols], sq[SPLIT ? kSums : 1][kD];
  const Geo& geo = a.geo;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int slice = SPLIT ? blockIdx.x % 4 : wave, idx = SPLIT ? blockIdx.x / 4 : blockIdx.x;
  const int h = idx % geo.kv_heads, e = idx / geo.kv_heads;
  if (e >= min(geo.n, ((const const_i32*)geo.step)[0])) return;
  Place p;
  entry_of(geo, e, p);
  if (p.seq < 0 || p.tokens == 0) return;

  const int col = slice * kCols + 4 * (lane & 7), row0 = (SPLIT ? wave * 32 : 0) + kRows * (lane >> 3);
  float* const state = a.states + (size_t(p.seq) * geo.kv_heads + h) * kState + row0 * kD + col;
  f32x4 S[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    S[i] = f32x4{};
    if (p.held) S[i] = *reinterpret_cast<const f32x4*>(state + i * kD);
  }
  const int G = geo.group, tokens = min(p.tokens, a.longest);
  const uint16_t* const kp = a.k.p + p.row * a.k.token + int64_t(h) * a.k.head;
  const uint16_t* const vp = a.v.p + p.row * a.v.token + int64_t(h) * a.v.head + slice * kCols;
  const uint16_t* const qp = a.q.p + p.row * a.q.token + int64_t(h) * G * a.q.head;
  if (SPLIT) {                                         // chunks of 16 bytes: of q, of k, of v
    const int nq = tokens * G * 16, nk = nq + tokens * 16, all = nk + tokens * 4;
    for (int i = threadIdx.x; i < all; i += kThreads) {
      if (i < nq) {
        const int r = i / 16, t = r / G;
        *reinterpret_cast<uint4*>(&sq[r][8 * (i % 16)]) = *reinterpret_cast<const uint4*>(qp + t * a.q.token + (r - t * G) * a.q.head + 8 * (i % 16));
      } else if (i < nk) {
        const int t = (i - nq) / 16;
        *reinterpret_cast<uint4*>(&sk[t][8 * (i % 16)]) = *reinterpret_cast<const uint4*>(kp + t * a.k.token + 8 * (i % 16));
      } else {
        const int t = (i - nk) / 4;
        *reinterpret_cast<uint4*>(&sv[t][8 * (i % 4)]) = *reinterpret_cast<const uint4*>(vp + t * a.v.token + 8 * (i % 4));
      }
    }
    __syncthreads();
  }
  const double dd = exp(double(geo.decay[h]));
  const float hi = float(dd), lo = float(dd - double(hi));
  uint16_t* const op = a.o + (p.row * geo.kv_heads * G + h * G) * kD + col;
  auto keys = [&](int t) { return Dims<kRows>::of(SPLIT ? &sk[t][row0] : kp + t * a.k.token + row0); };
  auto values = [&](int t) { return *reinterpret_cast<const uint2*>(SPLIT ? &sv[t][4 * (lane & 7)] : vp + t * a.v.token + 4 * (lane & 7)); };
  auto queries = [&](int t, int g) { return Dims<kRows>::of(SPLIT ? &sq[t * G + g][row0] : qp + t * a.q.token + g * a.q.head + row0); };

  Dims<kRows> q = queries(0, 0);
#pragma unroll 1
  for (int t = 0; t < tokens; ++t) {
    {
      float x[kRows];
      keys(t).unpack(x);
      const uint2 w = values(t);
      const float y[4] = {__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                          __uint_as_float(w.y & 0xffff0000u)};
#pragma unroll
      for (int i = 0; i < kRows; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) S[i][c] = __builtin_fmaf(S[i][c], hi, __builtin_fmaf(S[i][c], lo, x[i] * y[c]));
    }
#pragma unroll 1
    for (int g = 0; g < G; ++g) {
      float x[kRows], o[4] = {0.f, 0.f, 0.f, 0.f};
      q.unpack(x);
      if (g + 1 < G || t + 1 < tokens) q = g + 1 < G ? queries(t, g + 1) : queries(t + 1, 0);   // the next ones
#pragma unroll
      for (int i = 0; i < kRows; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] = __builtin_fmaf(x[i], S[i][c], o[c]);
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] = column_sum(o[c]);
      if (SPLIT) {
        if (lane < 8) *reinterpret_cast<f32x4*>(&sums[t * G + g][wave][4 * lane]) = f32x4{o[0], o[1], o[2], o[3]};
      } else if (lane < 8) {
        *reinterpret_cast<uint2*>(op + (int64_t(t) * geo.kv_heads * G + g) * kD) =
            make_uint2(pack_bf16x2(geo.scale * o[0], geo.scale * o[1]), pack_bf16x2(geo.scale * o[2], geo.scale * o[3]));
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) *reinterpret_cast<f32x4*>(state + i * kD) = S[i];
  if (SPLIT) {
    __syncthreads();
    for (int k = threadIdx.x; k < tokens * G * (kCols / 2); k += kThreads) {
      const int i = k / (kCols / 2), c = 2 * (k % (kCols / 2)), t = i / G, g = i - t * G;
      const float2 s0 = *reinterpret_cast<const float2*>(&sums[i][0][c]), s1 = *reinterpret_cast<const float2*>(&sums[i][1][c]),
                   s2 = *reinterpret_cast<const float2*>(&sums[i][2][c]), s3 = *reinterpret_cast<const float2*>(&sums[i][3][c]);
      *reinterpret_cast<uint32_t*>(a.o + ((p.row + t) * geo.kv_heads * G + h * G + g) * kD + slice * kCols + c) =
          pack_bf16x2(geo.scale * ((s0.x + s1.x) + (s2.x + s3.x)), geo.scale * ((s0.y + s1.y) + (s2.y + s3.y)));
    }
  }
}

// States of a sequence in a layer, copied: a workgroup per (pair, layer, 16 KB).  A source is read for each of its copies: 8 sequences
// to 56, 32 layers of 8 heads, 316 us, 1.88 GB at 5.9 TB/s; 16 to 48, 4 layers, 25 us, 201 MB at 8.0 TB/s, for the sources of 34 MB
// stay in caches.
constexpr int kCopy = 4;                               // float4 of a thread
__global__ __launch_bounds__(kThreads) void state_fork_kernel(ForkArgs a) {
  const int64_t at = (int64_t(blockIdx.x) * kThreads * kCopy + threadIdx.x) * 4;
  float* const base = a.pool + int64_t(blockIdx.y) * a.layer + at;
  const float* const from = base + a.words[2 * blockIdx.z] * a.seq;
  float* const to = base + a.words[2 * blockIdx.z + 1] * a.seq;
  f32x4 x[kCopy];
#pragma unroll
  for (int i = 0; i < kCopy; ++i) x[i] = *reinterpret_cast<const f32x4*>(from + 4 * kThreads * i);
#pragma unroll
  for (int i = 0; i < kCopy; ++i) *reinterpret_cast<f32x4*>(to + 4 * kThreads * i) = x[i];
}

// A group's states, in place: a workgroup takes the same elements of all its beams, each thread
// holds its own in LDS before it stores any.  A parent is read once, whoever has it; who stays is
// neither read for itself nor written.  Elements of 16 bytes while 64 KB hold a workgroup's (two to a CU); 16 groups of 5
// beams, 4 layers of 8 key heads: 39 us, 230 MB at 5.9 TB/s.
template <class V, int BEAMS>
__global__ __launch_bounds__(kThreads) void state_reorder_kernel(ReorderArgs a) {
  __shared__ V held[BEAMS][kThreads];
  constexpr int kPer = sizeof(V) / 4;
  const int tid = threadIdx.x;
  const int32_t* const seqs = a.seqs + blockIdx.z * a.beams;
  const int32_t* const parents = a.parents + int64_t(blockIdx.z) * a.beams;
  const int mine = (tid & 63) < a.beams ? parents[tid & 63] : -1;    // the same in every wave
  const bool moves = uint32_t(mine) < uint32_t(a.beams) && mine != (tid & 63);
  const uint64_t moved = __ballot(moves);
  if (moved == 0) return;
  uint64_t wanted = 0;
  for (int i = 0; i < a.beams; ++i)
    if ((moved >> i) & 1) wanted |= uint64_t(1) << __builtin_amdgcn_readlane(mine, i);
  float* const base = a.pool + int64_t(blockIdx.y) * a.layer + (int64_t(blockIdx.x) * kThreads + tid) * kPer;
#pragma unroll 8
  for (int i = 0; i < BEAMS; ++i)
    if ((wanted >> i) & 1) held[i][tid] = *reinterpret_cast<const V*>(base + seqs[i] * a.seq);
#pragma unroll 8
  for (int i = 0; i < BEAMS; ++i)
    if ((moved >> i) & 1) *reinterpret_cast<V*>(base + seqs[i] * a.seq) = held[__builtin_amdgcn_readlane(mine, i)][tid];
}

}  // namespace

hipError_t launch_linear_step(const StepArgs& a, hipStream_t stream) {
  const int64_t units = int64_t(a.geo.n) * a.geo.kv_heads;
  // (256 states whole have a workgroup for each CU)
  if (units < 256 && int64_t(a.longest) * a.geo.group <= kSums)
    linear_step_kernel<true><<<dim3(unsigned(units * 4)), kThreads, 0, stream>>>(a);
  else
    linear_step_kernel<false><<<dim3(unsigned(units)), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_state_fork(const ForkArgs& a, hipStream_t stream) {
  state_fork_kernel<<<dim3(unsigned(a.seq / (4 * kThreads * kCopy)), unsigned(a.layers), unsigned(a.n)), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_state_reorder(const ReorderArgs& a, hipStream_t stream) {
  auto run = [&](auto v, auto kernel) {
    kernel<<<dim3(unsigned(a.seq * 4 / (kThreads * sizeof(v))), unsigned(a.layers), unsigned(a.groups)), kThreads, 0, stream>>>(a);
  };
  if (a.beams <= 8) run(float4{}, state_reorder_kernel<float4, 8>);
  else if (a.beams <= 16) run(float4{}, state_reorder_kernel<float4, 16>);
  else if (a.beams <= 32) run(float2{}, state_reorder_kernel<float2, 32>);
  else run(float{}, state_reorder_kernel<float, kMaxBeams>);
  return hipGetLastError();
}

}  // namespace lin
}  // namespace uf
