// Pages of the token cache: table updates, new tokens' rows, copies of pages, and
// the moves of tokens that stay when others leave.
//
// All of it moves rows of 256 bytes (one head of one token) between places that the
// page tables name; nothing is computed.  What bounds the larger calls is HBM (a large
// copy: 4.9 TB/s), the smaller ones launch latency.  Page numbers and positions come from device memory
// and are checked before they are used: what lies outside is skipped, or read as zeros.
#include <cstring>

#include "token_step.h"

namespace uf {
namespace tok {
namespace {

constexpr int kThreads = 256;
constexpr int kRowChunks = kD / 8;           // 16-byte chunks of a row

// First byte of head h's rows of a page: K (kv = 0) or V (kv = 1).
__device__ inline size_t page_rows(const Pool& p, int page, int kv, int h) {
  return ((size_t(page) * 2 + kv) * p.kv_heads + h) * size_t(p.page_tokens) * (kD * 2);
}

// By a workgroup of THREADS.
template <int THREADS>
__device__ inline void poke(const PokeHead& a, const int32_t* words) {
  for (int i = threadIdx.x; i < a.dense; i += THREADS) a.table[a.dense_at + i] = words[i];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int r = wave; r < a.n_runs; r += THREADS / 64) {
    const int at = words[a.runs + 3 * r], n = words[a.runs + 3 * r + 1], value = words[a.runs + 3 * r + 2];
    for (int i = lane; i < n; i += 64) a.table[at + i] = value < 0 ? value : value + i;
  }
}
template <int N>
__global__ __launch_bounds__(1024) void poke_kernel(Worded<PokeHead, N> a) {
  poke<1024>(a, a.words);
}

template <int N>
__global__ __launch_bounds__(kThreads) void rows_kernel(Worded<RowsHead, N> a) {
  const int b = blockIdx.x;
  const int from = a.words[3 * b], to = a.words[3 * b + 1], n = a.words[3 * b + 2];
  for (int i = threadIdx.x; i < n; i += kThreads) a.table[to + i] = a.table[from + i];
}

// One workgroup per (page, K or V, head; layer), and one for the tables.  Loads before
// stores: the stores could alias them as far as the compiler knows.
template <int T, int N>
__global__ __launch_bounds__(kThreads) void copy_pages_kernel(Worded<CopyHead, N> a) {
  const int heads = 2 * a.pool.kv_heads;
  const int i = blockIdx.x / heads, kvh = blockIdx.x % heads;
  if (i == a.n) {
    if (blockIdx.y == 0) poke<kThreads>(a.poke, a.words + 3 * a.n);
    return;
  }
  const int rows = a.words[3 * i + 2];
  uint8_t* base = a.pool.base + size_t(blockIdx.y) * a.pool.layer_bytes;
  const uint4* src = reinterpret_cast<const uint4*>(base + page_rows(a.pool, a.words[3 * i], 0, kvh));
  uint4* dst = reinterpret_cast<uint4*>(base + page_rows(a.pool, a.words[3 * i + 1], 0, kvh));
  const int n = rows * kRowChunks;
  constexpr int kPer = T * kRowChunks / kThreads;
  uint4 x[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = threadIdx.x + k * kThreads;
    x[k] = make_uint4(0, 0, 0, 0);
    if (i < n) x[k] = src[i];
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = threadIdx.x + k * kThreads;
    if (i < n) dst[i] = x[k];
  }
}

// Row at position `pos` of the sequence whose pages start at table[seq_row]: null
// where there is none.
__device__ inline const uint4* row_at(const KeepHead& a, const uint8_t* base, int seq_row, int length, int pos, int kvh) {
  if (pos < 0 || pos >= length) return nullptr;
  const int page = a.table[size_t(seq_row) + pos / a.pool.page_tokens];
  if (uint32_t(page) >= uint32_t(a.pool.n_pages)) return nullptr;
  return reinterpret_cast<const uint4*>(base + page_rows(a.pool, page, 0, kvh)) + (pos % a.pool.page_tokens) * kRowChunks;
}

// Up to kInPlace rows of a sequence: one workgroup per (sequence, K or V, head; layer)
// holds them all before it stores any.
template <int N>
__global__ __launch_bounds__(kThreads) void keep_in_place_kernel(Worded<KeepHead, N> a) {
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

// Rows into fresh pages: one workgroup per (page, K or V, head; layer).  Every second of
// 4 x 30,000 tokens of 8 heads: 100 us, 4.9 TB/s.
template <int T, int N>
__global__ __launch_bounds__(kThreads) void keep_fresh_kernel(Worded<KeepHead, N> a) {
  const int heads = 2 * a.pool.kv_heads;
  const int i = blockIdx.x / heads, kvh = blockIdx.x % heads;
  int lo = 0, hi = a.n - 1;                  // the last run whose pages start at or before page i
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.words[kKeepWords * mid + 6] <= i) lo = mid;
    else hi = mid - 1;
  }
  const int32_t* w = a.words + kKeepWords * lo;
  const int page = w[5] + i - w[6];          // of the sequence
  uint8_t* base = a.pool.base + size_t(blockIdx.y) * a.pool.layer_bytes;
  uint4* dst = reinterpret_cast<uint4*>(base + page_rows(a.pool, w[7] + i - w[6], 0, kvh));
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

// New tokens of many: one workgroup per (page's worth of them, K or V, head; sequence),
// whose rows lie side by side in the page.  16,384 tokens of 8 heads: 25 us, 5.4 TB/s;
// 2,048 chunks of consecutive tokens a workgroup, all heads of one after the other: 51 us,
// and 14 for 5 at 16 x 48 tokens.  At fewer than 16 tokens a sequence most of a page's
// workgroups would find nothing: write_kernel.
template <int T>
__global__ __launch_bounds__(kThreads) void write_pages_kernel(WriteArgs a, int spans) {
  const int H = a.pool.kv_heads;
  int e = blockIdx.y, kvh = blockIdx.x / spans, s = blockIdx.x % spans;
  if (a.packed > 0) {                        // spans: of all sequences
    const Place w = place_of(a.step, a.n, s, [&](const int32_t* entry) {
      return write_spans(min(entry[2], a.total - entry[1]), T);
    });
    if (w.entry < 0) return;
    e = w.entry;
    s = w.tile;
  }
  typedef __attribute__((address_space(4))) int32_t uniform_i32;
  const uniform_i32* step = (const uniform_i32*)a.step;
  const uniform_i32* entry = step + kHeader + kEntry * e;
  if (e >= step[0]) return;
  const int seq = entry[0], at = entry[1], count = min(entry[2], a.total - at), first = entry[3] - entry[2];
  const uniform_i32* pages = (const uniform_i32*)(a.table + size_t(seq) * a.row);
  constexpr int kPer = T * kRowChunks / kThreads, kSlots = kThreads / kRowChunks;
  const int c = threadIdx.x % kRowChunks, slot = threadIdx.x / kRowChunks;
  const bool isv = kvh >= H;
  const int64_t ts = isv ? a.v_token : a.k_token;
  const uint16_t* src = isv ? a.v + int64_t(kvh - H) * a.v_head : a.k + int64_t(kvh) * a.k_head;
  for (; ; s += spans) {
    const int64_t p0 = (int64_t(first) / T + s) * T;     // first position of the page
    if (p0 >= int64_t(first) + count) return;
    const int page = pages[p0 / T];
    if (uint32_t(page) >= uint32_t(a.pool.n_pages)) continue;
    uint4* dst = reinterpret_cast<uint4*>(a.pool.base + page_rows(a.pool, page, 0, kvh)) + c;
    uint4 x[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int64_t t = p0 + slot + k * kSlots - first;
      x[k] = make_uint4(0, 0, 0, 0);
      if (t >= 0 && t < count) x[k] = *reinterpret_cast<const uint4*>(src + (at + t) * ts + 8 * c);
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int64_t t = p0 + slot + k * kSlots - first;
      if (t >= 0 && t < count) dst[(slot + k * kSlots) * kRowChunks] = x[k];
    }
  }
}

// New tokens of few: a workgroup takes `per` tokens of one sequence at a time, a row (token,
// K or V, head) in 16 lanes, eight rows a thread before the first is stored.
__global__ __launch_bounds__(kThreads) void write_kernel(WriteArgs a, int per) {
  const int e = blockIdx.y;
  typedef __attribute__((address_space(4))) int32_t uniform_i32;
  const uniform_i32* step = (const uniform_i32*)a.step;
  const uniform_i32* entry = step + kHeader + kEntry * e;
  if (e >= step[0]) return;
  const int seq = entry[0], at = entry[1], count = min(entry[2], a.total - at), first = entry[3] - entry[2];
  const int H = a.pool.kv_heads, T = a.pool.page_tokens;
  const int c = threadIdx.x % kRowChunks, slot = threadIdx.x / kRowChunks;
  const int32_t* pages = a.table + size_t(seq) * a.row;
  constexpr int kPer = 8, kSlots = kThreads / kRowChunks;
  for (int64_t t0 = int64_t(blockIdx.x) * per; t0 < count; t0 += int64_t(gridDim.x) * per) {
    const int rows = min(per, count - int(t0)) * 2 * H;
    for (int r0 = 0; r0 < rows; r0 += kPer * kSlots) {
      uint4 x[kPer];
      uint4* dst[kPer];
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const int r = r0 + k * kSlots + slot;
        dst[k] = nullptr;
        if (r < rows) {
          const int t = int(uint32_t(r) / uint32_t(2 * H)), kvh = r - t * 2 * H;
          const bool isv = kvh >= H;
          const int64_t token = at + t0 + t;
          const int64_t off = isv ? token * a.v_token + int64_t(kvh - H) * a.v_head : token * a.k_token + int64_t(kvh) * a.k_head;
          x[k] = *reinterpret_cast<const uint4*>((isv ? a.v : a.k) + off + 8 * c);
          const int pos = first + int(t0) + t;
          const int page = pages[uint32_t(pos) / uint32_t(T)];
          if (uint32_t(page) < uint32_t(a.pool.n_pages))
            dst[k] = reinterpret_cast<uint4*>(a.pool.base + page_rows(a.pool, page, 0, kvh)) + (pos & (T - 1)) * kRowChunks + c;
        }
      }
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if (dst[k] != nullptr) *dst[k] = x[k];
    }
  }
}

}  // namespace

namespace {

template <class Head>
Worded<Head, kFew> few(const Worded<Head, kWords>& a) {
  Worded<Head, kFew> f;
  static_cast<Head&>(f) = a;
  std::memcpy(f.words, a.words, sizeof(f.words));
  return f;
}

}  // namespace

hipError_t launch_poke(const PokeArgs& a, int used, hipStream_t stream) {
  if (used <= kFew)
    poke_kernel<kFew><<<1, 1024, 0, stream>>>(few(a));
  else
    poke_kernel<kWords><<<1, 1024, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_rows(const RowsArgs& a, hipStream_t stream) {
  if (3 * a.n <= kFew)
    rows_kernel<kFew><<<unsigned(a.n), kThreads, 0, stream>>>(few(a));
  else
    rows_kernel<kWords><<<unsigned(a.n), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_copy_pages(const CopyArgs& a, int used, hipStream_t stream) {
  const dim3 grid(unsigned(a.n) * 2 * unsigned(a.pool.kv_heads) + (a.poke.table != nullptr ? 1 : 0), unsigned(a.pool.layers));
  const bool wide = a.pool.page_tokens == 128;
  if (used <= kFew) {
    if (wide) copy_pages_kernel<128, kFew><<<grid, kThreads, 0, stream>>>(few(a));
    else copy_pages_kernel<64, kFew><<<grid, kThreads, 0, stream>>>(few(a));
  } else {
    if (wide) copy_pages_kernel<128, kWords><<<grid, kThreads, 0, stream>>>(a);
    else copy_pages_kernel<64, kWords><<<grid, kThreads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_keep_in_place(const KeepArgs& a, hipStream_t stream) {
  const dim3 grid(unsigned(a.n) * 2 * unsigned(a.pool.kv_heads), unsigned(a.pool.layers));
  if (kKeepWords * a.n <= kFew)
    keep_in_place_kernel<kFew><<<grid, kThreads, 0, stream>>>(few(a));
  else
    keep_in_place_kernel<kWords><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_keep_fresh(const KeepArgs& a, hipStream_t stream) {
  const dim3 grid(unsigned(a.n_pages) * 2 * unsigned(a.pool.kv_heads), unsigned(a.pool.layers));
  const bool wide = a.pool.page_tokens == 128;
  if (kKeepWords * a.n <= kFew) {
    if (wide) keep_fresh_kernel<128, kFew><<<grid, kThreads, 0, stream>>>(few(a));
    else keep_fresh_kernel<64, kFew><<<grid, kThreads, 0, stream>>>(few(a));
  } else {
    if (wide) keep_fresh_kernel<128, kWords><<<grid, kThreads, 0, stream>>>(a);
    else keep_fresh_kernel<64, kWords><<<grid, kThreads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_write(const WriteArgs& a, hipStream_t stream) {
  if (a.longest >= 16) {
    const int T = a.pool.page_tokens;
    const int spans = a.packed > 0 ? a.packed : write_spans(a.longest, T);
    const dim3 grid(unsigned(spans) * 2 * unsigned(a.pool.kv_heads), a.packed > 0 ? 1 : unsigned(a.n));
    if (T == 128)
      write_pages_kernel<128><<<grid, kThreads, 0, stream>>>(a, spans);
    else
      write_pages_kernel<64><<<grid, kThreads, 0, stream>>>(a, spans);
    return hipGetLastError();
  }
  const int per = a.pool.kv_heads < 64 ? 64 / a.pool.kv_heads : 1;     // 128 rows
  const int64_t blocks = (int64_t(a.longest) + per - 1) / per;
  write_kernel<<<dim3(unsigned(blocks), unsigned(a.n)), kThreads, 0, stream>>>(a, per);
  return hipGetLastError();
}

}  // namespace tok
}  // namespace uf
