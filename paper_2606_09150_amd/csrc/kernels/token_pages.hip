// Pages of the token cache: table updates, new tokens' rows, copies of pages, and
// the moves of tokens that stay when others leave.
//
// All of it moves rows of 256 bytes (one head of one token) between places that the
// page tables name; nothing is computed.  What bounds the larger calls is HBM, the
// smaller ones launch latency.  Page numbers and positions come from device memory
// and are checked before they are used: what lies outside is skipped, or read as zeros.
#include "../launch_tokens.h"

namespace uf {
namespace tok {
namespace {

constexpr int kThreads = 256;
constexpr int kRowChunks = kD / 8;           // 16-byte chunks of a row

// First byte of head h's rows of a page: K (kv = 0) or V (kv = 1).
__device__ inline size_t page_rows(const Pool& p, int page, int kv, int h) {
  return ((size_t(page) * 2 + kv) * p.kv_heads + h) * size_t(p.page_tokens) * (kD * 2);
}

__global__ __launch_bounds__(1024) void poke_kernel(PokeArgs a) {
  for (int i = threadIdx.x; i < a.dense; i += 1024) a.table[a.dense_at + i] = a.words[i];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int r = wave; r < a.n_runs; r += 16) {
    const int at = a.words[a.runs + 3 * r], n = a.words[a.runs + 3 * r + 1], from = a.words[a.runs + 3 * r + 2];
    for (int i = lane; i < n; i += 64) a.table[at + i] = a.words[from + i];
  }
}

__global__ __launch_bounds__(kThreads) void rows_kernel(RowsArgs a) {
  const int b = blockIdx.x;
  const int from = a.words[3 * b], to = a.words[3 * b + 1], n = a.words[3 * b + 2];
  for (int i = threadIdx.x; i < n; i += kThreads) a.table[to + i] = a.table[from + i];
}

// One workgroup per (page, K or V, head; layer).  Loads before stores: the stores
// could alias them as far as the compiler knows.
__global__ __launch_bounds__(kThreads) void copy_pages_kernel(CopyArgs a) {
  const int heads = 2 * a.pool.kv_heads;
  const int i = blockIdx.x / heads, kvh = blockIdx.x % heads;
  const int rows = a.words[3 * i + 2];
  uint8_t* base = a.pool.base + size_t(blockIdx.y) * a.pool.layer_bytes;
  const uint4* src = reinterpret_cast<const uint4*>(base + page_rows(a.pool, a.words[3 * i], 0, kvh));
  uint4* dst = reinterpret_cast<uint4*>(base + page_rows(a.pool, a.words[3 * i + 1], 0, kvh));
  const int n = rows * kRowChunks;
  uint4 x[8];                                // 128 rows at most
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (threadIdx.x + k * kThreads < n) x[k] = src[threadIdx.x + k * kThreads];
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (threadIdx.x + k * kThreads < n) dst[threadIdx.x + k * kThreads] = x[k];
}

// Row at position `pos` of the sequence whose pages start at table[seq_row]: null
// where there is none.
__device__ inline const uint4* row_at(const KeepArgs& a, const uint8_t* base, int seq_row, int length, int pos, int kvh) {
  if (pos < 0 || pos >= length) return nullptr;
  const int page = a.table[size_t(seq_row) + pos / a.pool.page_tokens];
  if (uint32_t(page) >= uint32_t(a.pool.n_pages)) return nullptr;
  return reinterpret_cast<const uint4*>(base + page_rows(a.pool, page, 0, kvh)) + (pos % a.pool.page_tokens) * kRowChunks;
}

// Up to kInPlace rows of a sequence: one workgroup per (sequence, K or V, head; layer)
// holds them all before it stores any.
__global__ __launch_bounds__(kThreads) void keep_in_place_kernel(KeepArgs a) {
  static_assert(kInPlace * kRowChunks == kThreads, "a chunk each");
  const int heads = 2 * a.pool.kv_heads;
  const int32_t* w = a.words + kKeepWords * (blockIdx.x / heads);
  const int kvh = blockIdx.x % heads;
  uint8_t* base = a.pool.base + size_t(blockIdx.y) * a.pool.layer_bytes;
  const int r = threadIdx.x / kRowChunks, c = threadIdx.x % kRowChunks;
  uint4 x = make_uint4(0, 0, 0, 0);
  uint4* dst = nullptr;
  if (r < w[3]) {
    const uint4* src = row_at(a, base, w[0], w[1], a.index[w[4] + r], kvh);
    if (src != nullptr) x = src[c];
    dst = const_cast<uint4*>(row_at(a, base, w[0], w[1], w[2] + r, kvh));
  }
  __syncthreads();                           // every row has been read
  if (dst != nullptr) dst[c] = x;
}

// Rows into fresh pages: one workgroup per (page, K or V, head; layer).
template <int T>
__global__ __launch_bounds__(kThreads) void keep_fresh_kernel(KeepArgs a) {
  const int heads = 2 * a.pool.kv_heads;
  const int i = blockIdx.x / heads, kvh = blockIdx.x % heads;
  int lo = 0, hi = a.n - 1;                  // the last sequence whose pages start at or before page i
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.words[kKeepWords * mid + 6] <= i) lo = mid;
    else hi = mid - 1;
  }
  const int32_t* w = a.words + kKeepWords * lo;
  const int page = w[5] + i - w[6];          // of the sequence
  uint8_t* base = a.pool.base + size_t(blockIdx.y) * a.pool.layer_bytes;
  uint4* dst = reinterpret_cast<uint4*>(base + page_rows(a.pool, a.words[a.pages + i], 0, kvh));
  const int start = w[2], end = start + w[3];
  const int c = threadIdx.x % kRowChunks, r0 = threadIdx.x / kRowChunks;
  constexpr int kPer = T * kRowChunks / kThreads;
  int pos[kPer];
  uint4 x[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int to = page * T + r0 + k * (kThreads / kRowChunks);
    pos[k] = to < start ? to : (to < end ? a.index[w[4] + to - start] : -1);
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const uint4* src = row_at(a, base, w[0], w[1], pos[k], kvh);
    x[k] = make_uint4(0, 0, 0, 0);
    if (src != nullptr) x[k] = src[c];
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int r = r0 + k * (kThreads / kRowChunks);
    if (page * T + r < end) dst[r * kRowChunks + c] = x[k];
  }
}

// New tokens: a workgroup takes 2,048 chunks at a time (8 tokens of 8 heads) of one
// sequence.
__global__ __launch_bounds__(kThreads) void write_kernel(WriteArgs a) {
  const int e = blockIdx.y;
  if (e >= a.step[0]) return;
  const int32_t* entry = a.step + kHeader + kEntry * e;
  const int seq = entry[0], at = entry[1], count = min(entry[2], a.total - entry[1]), first = entry[3] - entry[2];
  const int H = a.pool.kv_heads, per = 2 * H * kRowChunks;   // chunks of a token
  const int64_t n = int64_t(count) * per;
  constexpr int kPer = 8;
  for (int64_t i0 = int64_t(blockIdx.x) * kPer * kThreads; i0 < n; i0 += int64_t(gridDim.x) * kPer * kThreads) {
    uint4 x[kPer];
    uint4* dst[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int64_t i = i0 + k * kThreads + threadIdx.x;
      dst[k] = nullptr;
      if (i < n) {
        const int t = int(i / per), r = int(i % per);
        const int kvh = r / kRowChunks, c = r % kRowChunks;
        const bool isv = kvh >= H;
        const int h = isv ? kvh - H : kvh;
        const int64_t off = isv ? int64_t(at + t) * a.v_token + int64_t(h) * a.v_head
                                : int64_t(at + t) * a.k_token + int64_t(h) * a.k_head;
        x[k] = *reinterpret_cast<const uint4*>((isv ? a.v : a.k) + off + 8 * c);
        const int pos = first + t;
        const int page = a.table[size_t(seq) * a.row + pos / a.pool.page_tokens];
        if (uint32_t(page) < uint32_t(a.pool.n_pages))
          dst[k] = reinterpret_cast<uint4*>(a.pool.base + page_rows(a.pool, page, 0, kvh)) +
                   (pos % a.pool.page_tokens) * kRowChunks + c;
      }
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (dst[k] != nullptr) *dst[k] = x[k];
  }
}

}  // namespace

hipError_t launch_poke(const PokeArgs& a, hipStream_t stream) {
  poke_kernel<<<1, 1024, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_rows(const RowsArgs& a, hipStream_t stream) {
  rows_kernel<<<unsigned(a.n), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_copy_pages(const CopyArgs& a, hipStream_t stream) {
  copy_pages_kernel<<<dim3(unsigned(a.n) * 2 * unsigned(a.pool.kv_heads), unsigned(a.pool.layers)), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_keep_in_place(const KeepArgs& a, hipStream_t stream) {
  keep_in_place_kernel<<<dim3(unsigned(a.n) * 2 * unsigned(a.pool.kv_heads), unsigned(a.pool.layers)), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_keep_fresh(const KeepArgs& a, hipStream_t stream) {
  const dim3 grid(unsigned(a.n_pages) * 2 * unsigned(a.pool.kv_heads), unsigned(a.pool.layers));
  if (a.pool.page_tokens == 128)
    keep_fresh_kernel<128><<<grid, kThreads, 0, stream>>>(a);
  else
    keep_fresh_kernel<64><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_write(const WriteArgs& a, hipStream_t stream) {
  const int64_t chunks = int64_t(a.longest) * 2 * a.pool.kv_heads * kRowChunks;
  const unsigned blocks = unsigned((chunks + 8 * kThreads - 1) / (8 * kThreads) < 65536 ? (chunks + 8 * kThreads - 1) / (8 * kThreads) : 65536);
  write_kernel<<<dim3(blocks, unsigned(a.n)), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace tok
}  // namespace uf
