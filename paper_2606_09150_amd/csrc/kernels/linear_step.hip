// The recurrent form of linear attention (a few new tokens a sequence), and the states
// that move between sequences.
//
// What bounds all three is HBM: a state of 64 KB is read and written for 256 bytes of k and
// v, and products and sums are done in fp32 on the vector ALUs beside it.
//
// A step's workgroup holds COLS columns (of v) of a state in registers, 16 bytes a thread and row,
// loads in flight all at once, and takes its sequence's tokens one by one:
// S = L S + k v^T, o = scale S^T q, rows summed over lanes and then over waves through LDS.
// L goes as two floats: one would be off by the same 2^-25 in each of thousands of steps.
#include <algorithm>

#include "linear_place.h"

namespace uf {
namespace lin {
namespace {

using namespace attn;

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kHeads = 8;                              // query heads taken at a time

template <int COLS>
__global__ __launch_bounds__(kThreads) void linear_step_kernel(StepArgs a) {
  constexpr int kC4 = COLS / 4;                        // threads along a row
  constexpr int kGroups = kThreads / kC4;              // rows side by side
  constexpr int kRows = kD / kGroups;                  // rows of a thread: group + kGroups i
  constexpr int kLane = 64 / kC4;                      // groups of a wave
  constexpr int kSlices = kD / COLS;
  __shared__ float sk[kD], sv[COLS], sq[kHeads][kD];
  __shared__ float so[kHeads][4][COLS];

  const Geo& geo = a.geo;
  int idx = blockIdx.x;
  const int slice = idx % kSlices;
  idx /= kSlices;
  const int h = idx % geo.kv_heads, e = idx / geo.kv_heads;
  if (e >= ((const const_i32*)geo.step)[0]) return;
  Place p;
  entry_of(geo, e, p);
  if (p.seq < 0 || p.tokens == 0) return;

  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int c4 = tid % kC4, group = tid / kC4;
  float* const state = a.states + (size_t(p.seq) * geo.kv_heads + h) * kState + slice * COLS + 4 * c4;
  float4 S[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    S[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (p.held) S[i] = *reinterpret_cast<const float4*>(state + (group + kGroups * i) * kD);
  }
  const double gd = double(geo.decay[h]), dd = exp(gd);
  const float hi = float(dd), lo = float(dd - double(hi));
  const int G = geo.group;
  const int tokens = min(p.tokens, a.longest);

  // what a token and block of query heads bring: k, v and the queries, a pair of dimensions a thread
  constexpr int kPairs2 = (kD + COLS + kHeads * kD) / 2, kLoads = (kPairs2 + kThreads - 1) / kThreads;
  uint32_t next[kLoads];
  auto fetch = [&](int t, int g0) {
    const int64_t row = p.row + t;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      int k = 2 * (tid + kThreads * i);
      const uint16_t* from = nullptr;
      if (k < kD) {
        if (g0 == 0) from = a.k.p + row * a.k.token + int64_t(h) * a.k.head + k;
      } else if (k < kD + COLS) {
        if (g0 == 0) from = a.v.p + row * a.v.token + int64_t(h) * a.v.head + slice * COLS + (k - kD);
      } else {
        k -= kD + COLS;
        const int g = g0 + k / kD;
        if (k < kHeads * kD && g < G) from = a.q.p + row * a.q.token + int64_t(h * G + g) * a.q.head + k % kD;
      }
      next[i] = from != nullptr ? *reinterpret_cast<const uint32_t*>(from) : 0u;
    }
  };
  auto place_in_lds = [&](int g0) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      int k = 2 * (tid + kThreads * i);
      const float2 x = make_float2(__uint_as_float(next[i] << 16), __uint_as_float(next[i] & 0xffff0000u));
      if (k < kD) {
        if (g0 == 0) *reinterpret_cast<float2*>(&sk[k]) = x;
      } else if (k < kD + COLS) {
        if (g0 == 0) *reinterpret_cast<float2*>(&sv[k - kD]) = x;
      } else {
        k -= kD + COLS;
        if (k < kHeads * kD) *reinterpret_cast<float2*>(&sq[k / kD][k % kD]) = x;
      }
    }
  };
  fetch(0, 0);
  for (int t = 0; t < tokens; ++t) {
    for (int g0 = 0; g0 < G; g0 += kHeads) {
      const int heads = min(kHeads, G - g0);
      place_in_lds(g0);
      __syncthreads();
      {
        const bool more = g0 + kHeads < G;             // the next block, or the next token's first
        if (more || t + 1 < tokens) fetch(more ? t : t + 1, more ? g0 + kHeads : 0);
      }
      if (g0 == 0) {
        const float4 v = *reinterpret_cast<const float4*>(&sv[4 * c4]);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          const float k = sk[group + kGroups * i];
          S[i].x = __builtin_fmaf(S[i].x, hi, __builtin_fmaf(S[i].x, lo, k * v.x));
          S[i].y = __builtin_fmaf(S[i].y, hi, __builtin_fmaf(S[i].y, lo, k * v.y));
          S[i].z = __builtin_fmaf(S[i].z, hi, __builtin_fmaf(S[i].z, lo, k * v.z));
          S[i].w = __builtin_fmaf(S[i].w, hi, __builtin_fmaf(S[i].w, lo, k * v.w));
        }
      }
      for (int g = 0; g < heads; ++g) {
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          const float q = sq[g][group + kGroups * i];
          o.x = __builtin_fmaf(q, S[i].x, o.x);
          o.y = __builtin_fmaf(q, S[i].y, o.y);
          o.z = __builtin_fmaf(q, S[i].z, o.z);
          o.w = __builtin_fmaf(q, S[i].w, o.w);
        }
#pragma unroll
        for (int d = kC4; d < 64; d <<= 1) {           // the wave's groups
          o.x += __shfl_xor(o.x, d);
          o.y += __shfl_xor(o.y, d);
          o.z += __shfl_xor(o.z, d);
          o.w += __shfl_xor(o.w, d);
        }
        if (lane < kC4) *reinterpret_cast<float4*>(&so[g][wave][4 * lane]) = o;
      }
      __syncthreads();
      for (int k = 2 * tid; k < heads * COLS; k += 2 * kThreads) {
        const int g = k / COLS, c = k % COLS;
        float2 s = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          s.x += so[g][w][c];
          s.y += so[g][w][c + 1];
        }
        *reinterpret_cast<uint32_t*>(a.o + ((p.row + t) * geo.kv_heads * G + h * G + g0 + g) * kD + slice * COLS + c) =
            pack_bf16x2(geo.scale * s.x, geo.scale * s.y);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) *reinterpret_cast<float4*>(state + (group + kGroups * i) * kD) = S[i];
  static_assert(kLane * kC4 == 64, "whole groups in a wave");
}

// States of a sequence in a layer, copied: a workgroup per (pair, layer, 16 KB).
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
// neither read for itself nor written.
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
  if (units < 256)
    linear_step_kernel<32><<<dim3(unsigned(units * 4)), kThreads, 0, stream>>>(a);
  else
    linear_step_kernel<128><<<dim3(unsigned(units)), kThreads, 0, stream>>>(a);
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
