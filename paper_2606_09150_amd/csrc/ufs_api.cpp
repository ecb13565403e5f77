// C ABI of the state operators: argument validation, what the sequences of a state
// cache hold, and kernel launches.  See include/ufs.h for the contract of every entry
// point.
//
// The host holds how many tokens each sequence has taken; kernels read a step's
// sequences from a table in device memory, whose words ride in launch arguments.  A call
// first checks, then launches, then commits: a failed call leaves the handle as it was, but
// for a step whose table or states some of its launches have changed, which is over.
#include <algorithm>
#include <climits>
#include <cmath>
#include <new>
#include <vector>

#include "launch_states.h"
#include "launch_tokens.h"
#include "status.h"

namespace {

using uf::fail;
using uf::ok;
namespace lin = uf::lin;
namespace tok = uf::tok;

constexpr size_t kStateBytes = size_t(lin::kState) * 4;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Every entry point: no exception leaves the library.
template <class F>
int guarded(F f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return fail(UF_ERR_ARG, "out of host memory");
  } catch (...) {
    return fail(UF_ERR_ARG, "unexpected failure");
  }
}

int check_hip(hipError_t e, const char* what) {
  if (e == hipSuccess) return UF_OK;
  return fail(UF_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
}

int check_stride(const uft_stride& s, const char* name) {
  if (s.token < 0 || s.head < 0 || s.batch < 0) return fail(UF_ERR_ARG, "%s must not be negative", name);
  if (s.token % 8 || s.head % 8 || s.batch % 8) return fail(UF_ERR_ARG, "%s must be multiples of 8", name);
  // a chunk's offsets are 32-bit: 32 tokens' strides in bytes
  if (s.token > (int64_t(1) << 24)) return fail(UF_ERR_ARG, "%s.token must be at most 2^24", name);
  if (s.head > (int64_t(1) << 30)) return fail(UF_ERR_ARG, "%s.head must be at most 2^30", name);
  return UF_OK;
}

int check_work(const void* work, size_t bytes, size_t need) {
  if (need == 0) return UF_OK;
  if (work == nullptr || !aligned(work, 16)) return fail(UF_ERR_ARG, "work must be 16-byte aligned and not null");
  if (bytes < need) return fail(UF_ERR_ARG, "work has %zu bytes, the call needs %zu", bytes, need);
  return UF_OK;
}

// Whether a launch of its own carries the states on from part to part, or each walk sums those of the parts before it.  `groups`:
// parts of all sequences' key heads.  Carried on / summed (us; one sequence, parts of 4 chunks): 2 / 4 / 8 parts of 4 heads
// 23.6 / 24.1 / 25.4, 22.0 / 24.6 / 30.3; of 64 heads 32.0 / 33.2 / 50.9, 22.3 / 28.8 / 44.0, and 16 parts 96 and 99.  Backward 3
// / 4 / 6 parts of 4 heads 24.9 / 25.5 / 26.8, 24.2 / 26.3 / 30.5; 4 / 8 of 64 heads 58.6 / 102, 58.4 / 116.
bool scanned(int64_t parts, double groups, int walks) { return parts > 4 && (walks > 1 || parts > 8 || groups < 256.0); }

// Chunks of a part: of n sequences with `all` chunks, the longest with `longest`, of `heads` key heads with `group` query heads
// each; `walks` 1, or the backward's 3 beside two sums.  Parts are walked side by side, and pay with a sum of each, a launch or two
// and their states' way through memory.  The time of either is estimated from what these launches took (us; c chunks a part, P
// parts of a sequence, W workgroups).  Walks: 1.8 c where a workgroup has a CU of its own (2.15 c where W = 256), 3.1 c where the first two
// share one, 3.8 c at W = 512, and rounds of these; the backward's 1.9 c, 2.1 c at 192, 3.75 c at 512, and less for what is left in a
// second round.  Sums 0.8 c, 1.9 c at 512; the states carried on 0.12 P, or 13 us for 512 of them, or summed 1.3 P (backward 1.5 P)
// with a launch less.  Measured (W: us): 1 x 32,768 tokens, 16 heads, 128: 336, 256: 221, 320: 254, 384: 234, 512: 211, 640: 238, 1,024: 238;
// 4 x 2,048 tokens, 8 heads, 128: 53, 256: 39, 320: 53, 512: 51; 1 x 16,384, 8 heads of 4, 192: 162, 256: 138, 512: 138, 592: 161.
// Backward (W: of walks, us) 2 x 8,192, 32 heads, 192 (whole): 547, 384: 502, 576: 521, 768: 509, 960: 489, 1,536: 502; 4 x 2,048, 8
// heads, 192: 95, 384: 77, 576: 87, 768: 83.
int32_t part_chunks(int64_t all, int64_t longest, int64_t n, int64_t heads, int walks, int group) {
  const int sums = walks > 1 ? 2 : 1;
  const double item = 0.35 + (walks == 1 && lin::two_heads(group) ? 0.58 : 0.65) * group, sum = walks > 1 ? 0.5 + 0.5 * group : 1.0;   // of a group's heads, for one's
  auto time = [&](int64_t c) {
    const double parts = double((longest + c - 1) / c);
    const double groups = double(heads) * (all == n * longest ? double(n) * parts
                                           : c < longest      ? std::ceil(double(all) / double(c)) + 0.5 * double(n - 1)
                                                              : double(n));
    // rounds of two workgroups a CU, and what is left
    const double all_walks = walks * groups, whole = std::floor(all_walks / 512.0), rest = all_walks - 512.0 * whole;
    double left = 0.0;
    if (walks > 1 && whole == 0.0) left = 1.9 + std::max(0.0, rest - 160.0) / 190.0;
    else if (walks > 1 && rest > 0.0) left = rest <= 256.0 ? 0.5 + rest / 183.0 : 1.9 + (rest - 256.0) / 160.0;
    else if (rest > 0.0) left = rest <= 256.0 ? std::max(1.8, 1.25 + rest / 285.0) : 3.1 + (rest - 256.0) / 365.0;
    const double walk = item * double(c) * (whole * (walks > 1 ? 3.75 : 3.8) + left);
    if (c >= longest) return 4.0 + walk;
    const double carry = scanned(int64_t(parts), groups, walks) ? std::max(0.12 * parts, 0.026 * sums * groups)
                                                                : (walks > 1 ? 1.5 * parts - 5.2 : 1.3 * parts - 4.5);
    return (walks > 1 ? 18.0 : 13.0) + walk + sum * double(c) * std::max(0.8, sums * groups / (walks > 1 ? 300.0 : 265.0)) + carry;
  };
  int64_t best = std::max<int64_t>(longest, 1);
  for (int64_t c = 1; c < longest; c += std::max<int64_t>(1, c / 32))
    if (time(c) < time(best)) best = c;
  return int32_t(best);
}

lin::Src src(const void* p, const uft_stride& s) { return lin::Src{static_cast<const uint16_t*>(p), s.batch, s.token, s.head}; }

}  // namespace

// ---- whole sequences ------------------------------------------------------------

namespace {

int check_linear(const ufs_linear_desc* d, int walks, lin::Geo* g) {
  if (d == nullptr) return fail(UF_ERR_ARG, "desc is null");
  if (d->batch < 1 || d->tokens < 1 || d->q_heads < 1 || d->kv_heads < 1)
    return fail(UF_ERR_ARG, "batch, tokens and heads must be >= 1");
  if (d->head_dim != lin::kD) return fail(UF_ERR_UNSUPPORTED, "head_dim %d: only 128 is built", d->head_dim);
  if (d->q_heads % d->kv_heads != 0)
    return fail(UF_ERR_ARG, "q_heads %d must be a multiple of kv_heads %d", d->q_heads, d->kv_heads);
  if (d->q_heads > 65536) return fail(UF_ERR_ARG, "q_heads must be at most 65536");
  if (d->tokens > (1 << 30)) return fail(UF_ERR_ARG, "tokens must be at most 2^30");
  if (!std::isfinite(d->scale)) return fail(UF_ERR_ARG, "scale must be finite");
  if (int s = check_stride(d->q, "q stride")) return s;
  if (int s = check_stride(d->k, "k stride")) return s;
  if (int s = check_stride(d->v, "v stride")) return s;
  *g = lin::Geo{};
  g->n = d->batch;
  g->tokens = d->tokens;
  g->kv_heads = d->kv_heads;
  g->group = d->q_heads / d->kv_heads;
  g->scale = d->scale;
  const int64_t chunks = (int64_t(d->tokens) + lin::kChunk - 1) / lin::kChunk;
  const double units = double(d->batch) * d->kv_heads;
  g->chunks = part_chunks(chunks * d->batch, chunks, d->batch, d->kv_heads, walks, g->group);
  g->parts = int32_t((chunks + g->chunks - 1) / g->chunks);
  g->scanned = scanned(g->parts, units * g->parts, walks);
  // (the backward's walks take as many launches as they need)
  const double sums = walks > 1 ? 2.0 : 1.0;
  if (units * g->parts > double(lin::most_groups(lin::kWalkThreads)) ||
      (g->parts > 1 && (units * g->parts * sums > double(lin::most_groups(lin::kWalkThreads)) ||
                        units * lin::kScanSlices * sums > double(lin::most_groups(lin::kOtherThreads)))) ||
      double(chunks) * g->group > 2.0e9)
    return fail(UF_ERR_ARG, "shape too large: batch * q_heads * tokens");
  return UF_OK;
}

// Bytes of one set of states at the parts' beginnings.
size_t starts_bytes(const lin::Geo& g) {
  return g.parts > 1 ? size_t(g.n) * g.kv_heads * size_t(g.parts) * kStateBytes : 0;
}

}  // namespace

extern "C" {

int ufs_linear_work_bytes(const ufs_linear_desc* d, size_t* bytes) {
  return guarded([&]() -> int {
    lin::Geo g;
    if (int s = check_linear(d, 1, &g)) return s;
    if (bytes == nullptr) return fail(UF_ERR_ARG, "bytes is null");
    *bytes = starts_bytes(g);
    return ok();
  });
}

int ufs_linear_bwd_work_bytes(const ufs_linear_desc* d, size_t* bytes) {
  return guarded([&]() -> int {
    lin::Geo g;
    if (int s = check_linear(d, 3, &g)) return s;
    if (bytes == nullptr) return fail(UF_ERR_ARG, "bytes is null");
    *bytes = 2 * starts_bytes(g);
    return ok();
  });
}

int ufs_linear_fwd(const ufs_linear_desc* d, const void* d_q, const void* d_k, const void* d_v, const float* d_decay,
                   const int32_t* d_lengths, const float* d_state, void* d_o, float* d_final, void* d_work,
                   size_t work_bytes, void* stream) {
  return guarded([&]() -> int {
    lin::WalkArgs a{};
    if (int s = check_linear(d, 1, &a.geo)) return s;
    for (const void* p : {d_q, d_k, d_v, static_cast<const void*>(d_o)}) {
      if (p == nullptr) return fail(UF_ERR_ARG, "q, k, v or o is null");
      if (!aligned(p, 16)) return fail(UF_ERR_ARG, "q, k, v and o must be 16-byte aligned");
    }
    if (d_decay == nullptr) return fail(UF_ERR_ARG, "decay is null");
    if (!aligned(d_decay, 4) || !aligned(d_lengths, 4)) return fail(UF_ERR_ARG, "decay and lengths must be 4-byte aligned");
    if (!aligned(d_state, 16) || !aligned(d_final, 16)) return fail(UF_ERR_ARG, "states must be 16-byte aligned");
    if (int s = check_work(d_work, work_bytes, starts_bytes(a.geo))) return s;
    hipStream_t st = static_cast<hipStream_t>(stream);
    a.geo.decay = d_decay;
    a.geo.lengths = d_lengths;
    const int32_t groups = a.geo.n * a.geo.parts * a.geo.kv_heads;
    float* starts = nullptr;
    if (a.geo.parts > 1) {
      starts = static_cast<float*>(d_work);
      lin::PartArgs p{};
      p.geo = a.geo;
      p.n = 1;
      p.sum[0] = {src(d_k, d->k), src(d_v, d->v), d_state, starts, 0};
      if (int s = check_hip(lin::launch_linear_parts(p, groups, true, st), "linear attention")) return s;
      if (a.geo.scanned)
        if (int s = check_hip(lin::launch_linear_scan(p, st), "linear attention")) return s;
    }
    a.n = 1;
    a.walk[0] = lin::Walk{src(d_q, d->q), src(d_k, d->k), src(d_v, d->v), static_cast<uint16_t*>(d_o), d_state, d_final, starts};
    if (int s = check_hip(lin::launch_linear_fwd(a, groups, st), "linear attention")) return s;
    return ok();
  });
}

int ufs_linear_bwd(const ufs_linear_desc* d, const void* d_q, const void* d_k, const void* d_v, const void* d_do,
                   const float* d_decay, const int32_t* d_lengths, const float* d_state, const float* d_dfinal,
                   void* d_dq, void* d_dk, void* d_dv, float* d_dstate, void* d_work, size_t work_bytes, void* stream) {
  return guarded([&]() -> int {
    lin::WalkArgs a{};
    if (int s = check_linear(d, 3, &a.geo)) return s;
    for (const void* p : {d_q, d_k, d_v, d_do, static_cast<const void*>(d_dq), static_cast<const void*>(d_dk),
                          static_cast<const void*>(d_dv)}) {
      if (p == nullptr) return fail(UF_ERR_ARG, "a tensor is null");
      if (!aligned(p, 16)) return fail(UF_ERR_ARG, "tensors must be 16-byte aligned");
    }
    if (d_decay == nullptr) return fail(UF_ERR_ARG, "decay is null");
    if (!aligned(d_decay, 4) || !aligned(d_lengths, 4)) return fail(UF_ERR_ARG, "decay and lengths must be 4-byte aligned");
    if (!aligned(d_state, 16) || !aligned(d_dfinal, 16) || !aligned(d_dstate, 16))
      return fail(UF_ERR_ARG, "states must be 16-byte aligned");
    if (int s = check_work(d_work, work_bytes, 2 * starts_bytes(a.geo))) return s;
    hipStream_t st = static_cast<hipStream_t>(stream);
    a.geo.decay = d_decay;
    a.geo.lengths = d_lengths;
    const int32_t groups = a.geo.n * a.geo.parts * a.geo.kv_heads;
    const bool exact = d_dstate != nullptr;             // (a result in fp32)
    // dO lies as O does
    const int64_t token = int64_t(d->q_heads) * lin::kD;
    const lin::Src q = src(d_q, d->q), k = src(d_k, d->k), v = src(d_v, d->v);
    const lin::Src g{static_cast<const uint16_t*>(d_do), token * d->tokens, token, lin::kD};
    float *forth = nullptr, *back = nullptr;
    if (a.geo.parts > 1) {
      forth = static_cast<float*>(d_work);
      back = forth + starts_bytes(a.geo) / 4;
      lin::PartArgs p{};
      p.geo = a.geo;
      p.n = 2;
      p.sum[0] = {k, v, d_state, forth, 0};
      p.sum[1] = {q, g, d_dfinal, back, 1};
      if (int s = check_hip(lin::launch_linear_parts(p, groups, exact, st), "linear attention backward")) return s;
      if (a.geo.scanned)
        if (int s = check_hip(lin::launch_linear_scan(p, st), "linear attention backward")) return s;
    }
    a.n = 3;
    a.walk[0] = lin::Walk{v, g, q, static_cast<uint16_t*>(d_dk), d_dfinal, nullptr, back};
    a.walk[1] = lin::Walk{k, q, g, static_cast<uint16_t*>(d_dv), d_dfinal, d_dstate, back};
    a.walk[2] = lin::Walk{g, v, k, static_cast<uint16_t*>(d_dq), d_state, nullptr, forth};
    if (int s = check_hip(lin::launch_linear_bwd(a, groups, exact, st), "linear attention backward")) return s;
    return ok();
  });
}

}  // extern "C"

// ---- states that a cache holds ------------------------------------------------------

namespace {

struct Entry {                  // a sequence of the step
  int32_t seq, at, count, held, part;
};

}  // namespace

struct ufs_cache {
  ufs_desc d;
  float* pool;
  int32_t* table;
  std::vector<int32_t> tokens;  // of each sequence
  std::vector<Entry> step;
  int32_t step_tokens = 0, step_longest = 0, step_parts = 0, step_most = 0;   // (parts: of all, and of a sequence at most)
  std::vector<uint8_t> seen;    // scratch of the checks, all 0 between calls

  bool dry() const { return (d.flags & UF_F_DRYRUN) != 0; }
  int64_t seq_floats() const { return int64_t(d.kv_heads) * lin::kState; }
  int64_t layer_floats() const { return seq_floats() * d.max_seqs; }
};

namespace {

int check_desc(const ufs_desc* d) {
  if (d == nullptr) return fail(UF_ERR_ARG, "desc is null");
  if (d->layers < 1 || d->layers > 65535) return fail(UF_ERR_ARG, "layers must be in [1, 65535] (got %d)", d->layers);
  if (d->kv_heads < 1 || d->kv_heads > 4096) return fail(UF_ERR_ARG, "kv_heads must be in [1, 4096] (got %d)", d->kv_heads);
  if (d->max_seqs < 1 || d->max_seqs > 65535)
    return fail(UF_ERR_ARG, "max_seqs must be in [1, 65535] (got %d)", d->max_seqs);
  if (d->flags & ~UF_F_DRYRUN) return fail(UF_ERR_ARG, "unknown flag bits 0x%x", d->flags);
  if (d->head_dim < 1) return fail(UF_ERR_ARG, "head_dim must be >= 1");
  if (d->head_dim != lin::kD) return fail(UF_ERR_UNSUPPORTED, "head_dim %d: only 128 is built", d->head_dim);
  if (double(d->layers) * d->kv_heads * d->max_seqs * double(kStateBytes) > 4.0e15)
    return fail(UF_ERR_ARG, "pool too large");
  return UF_OK;
}

// n sequence numbers, each once.
int check_seqs(ufs_cache* c, int64_t n, const int32_t* seqs, const char* name) {
  if (n < 1) return fail(UF_ERR_ARG, "n must be >= 1 (got %lld)", (long long)n);
  if (seqs == nullptr) return fail(UF_ERR_ARG, "%s is null", name);
  int s = UF_OK;
  int64_t i = 0;
  for (; i < n; ++i) {
    if (seqs[i] < 0 || seqs[i] >= c->d.max_seqs) {
      s = fail(UF_ERR_ARG, "%s[%lld] = %d is no sequence (0 .. %d)", name, (long long)i, seqs[i], c->d.max_seqs - 1);
      break;
    }
    if (c->seen[size_t(seqs[i])]) {
      s = fail(UF_ERR_ARG, "%s names sequence %d twice", name, seqs[i]);
      break;
    }
    c->seen[size_t(seqs[i])] = 1;
  }
  for (int64_t k = 0; k < i; ++k) c->seen[size_t(seqs[k])] = 0;
  return s;
}

void end_step(ufs_cache* c) {
  c->step.clear();
  c->step_tokens = c->step_longest = c->step_parts = c->step_most = 0;
}

// A step with one of these sequences is over.
void leave_step(ufs_cache* c, int64_t n, const int32_t* seqs) {
  for (int64_t i = 0; i < n; ++i) c->seen[size_t(seqs[i])] = 1;
  bool found = false;
  for (const Entry& e : c->step) found = found || c->seen[size_t(e.seq)];
  for (int64_t i = 0; i < n; ++i) c->seen[size_t(seqs[i])] = 0;
  if (found) end_step(c);
}

bool few(const ufs_cache* c) { return c->step_longest <= lin::kFewTokens; }
size_t step_bytes(const ufs_cache* c) {
  return !few(c) && c->step_most > 1 ? size_t(c->step_parts) * c->d.kv_heads * kStateBytes : 0;
}

}  // namespace

extern "C" {

int ufs_pool_bytes(const ufs_desc* desc, size_t* bytes) {
  if (int s = check_desc(desc)) return s;
  if (bytes == nullptr) return fail(UF_ERR_ARG, "bytes is null");
  *bytes = size_t(desc->layers) * desc->max_seqs * desc->kv_heads * kStateBytes;
  return ok();
}

int ufs_table_bytes(const ufs_desc* desc, size_t* bytes) {
  if (int s = check_desc(desc)) return s;
  if (bytes == nullptr) return fail(UF_ERR_ARG, "bytes is null");
  *bytes = 4 * (size_t(lin::kHeader) + size_t(desc->max_seqs) * lin::kEntry);
  return ok();
}

int ufs_create(const ufs_desc* desc, void* d_pool, size_t pool_bytes, void* d_table, size_t table_bytes, ufs_cache** out) {
  return guarded([&]() -> int {
    if (out == nullptr) return fail(UF_ERR_ARG, "out is null");
    size_t pool = 0, table = 0;
    if (int s = ufs_pool_bytes(desc, &pool)) return s;
    if (int s = ufs_table_bytes(desc, &table)) return s;
    const bool dry = (desc->flags & UF_F_DRYRUN) != 0;
    if (!dry && (d_pool == nullptr || d_table == nullptr)) return fail(UF_ERR_ARG, "pool or table is null");
    if (!aligned(d_pool, 256) || !aligned(d_table, 256)) return fail(UF_ERR_ARG, "pool and table must be 256-byte aligned");
    if (!dry && pool_bytes < pool) return fail(UF_ERR_CAPACITY, "pool has %zu bytes, the cache needs %zu", pool_bytes, pool);
    if (!dry && table_bytes < table)
      return fail(UF_ERR_CAPACITY, "table has %zu bytes, the cache needs %zu", table_bytes, table);
    ufs_cache* c = new ufs_cache();
    try {
      c->d = *desc;
      c->pool = static_cast<float*>(d_pool);
      c->table = static_cast<int32_t*>(d_table);
      c->tokens.assign(size_t(desc->max_seqs), 0);
      c->seen.assign(size_t(desc->max_seqs), 0);
    } catch (...) {
      delete c;
      throw;
    }
    *out = c;
    return ok();
  });
}

int ufs_destroy(ufs_cache* cache) {
  delete cache;
  return UF_OK;   // (the last error's text stays, as in uf_kv_destroy)
}

int ufs_extend(ufs_cache* c, int32_t n, const int32_t* seqs, const int32_t* counts, void* stream) {
  return guarded([&]() -> int {
    if (c == nullptr) return fail(UF_ERR_ARG, "handle is null");
    if (int s = check_seqs(c, n, seqs, "seqs")) return s;
    if (counts == nullptr) return fail(UF_ERR_ARG, "counts is null");
    int64_t total = 0, chunks = 0;
    int32_t longest = 0;
    for (int32_t i = 0; i < n; ++i) {
      if (counts[i] < 0) return fail(UF_ERR_ARG, "counts[%d] must be >= 0 (got %d)", i, counts[i]);
      if (int64_t(c->tokens[size_t(seqs[i])]) + counts[i] > INT32_MAX)
        return fail(UF_ERR_ARG, "sequence %d: more than 2^31 - 1 tokens", seqs[i]);
      total += counts[i];
      chunks += (int64_t(counts[i]) + lin::kChunk - 1) / lin::kChunk;
      longest = std::max(longest, counts[i]);
    }
    if (total > (1 << 30)) return fail(UF_ERR_ARG, "more than 2^30 new tokens");
    const int32_t part = part_chunks(chunks, (int64_t(longest) + lin::kChunk - 1) / lin::kChunk, n, c->d.kv_heads, 1, 1);
    std::vector<Entry> step;
    std::vector<int32_t> words = {n, int32_t(total), 0, part};
    step.reserve(size_t(n));
    words.reserve(size_t(lin::kHeader) + size_t(n) * lin::kEntry);
    int32_t at = 0, parts = 0, most = 0;
    for (int32_t i = 0; i < n; ++i) {
      const int32_t held = c->tokens[size_t(seqs[i])];
      step.push_back(Entry{seqs[i], at, counts[i], held, parts});
      words.insert(words.end(), {seqs[i], at, counts[i], held, parts});
      at += counts[i];
      const int32_t own = (counts[i] + lin::kChunk - 1) / lin::kChunk;   // (counts <= 2^30)
      parts += (own + part - 1) / part;
      most = std::max(most, (own + part - 1) / part);
    }
    words[2] = parts;
    // token by token, or walks, sums and what carries them on
    const double heads = c->d.kv_heads, other = double(lin::most_groups(lin::kOtherThreads));
    if (longest <= lin::kFewTokens ? n * heads > other
                                   : parts * heads > double(lin::most_groups(lin::kWalkThreads)) || (most > 1 && lin::kScanSlices * n * heads > other))
      return fail(UF_ERR_ARG, "step too large for one launch");
    if (!c->dry())
      for (size_t k = 0; k < words.size();) {
        tok::PokeArgs a;
        a.table = c->table;
        a.dense_at = int32_t(k);
        a.dense = a.runs = int32_t(std::min(words.size() - k, size_t(tok::kWords)));
        a.n_runs = 0;
        std::copy_n(words.begin() + k, a.dense, a.words);
        if (int s = check_hip(tok::launch_poke(a, a.dense, static_cast<hipStream_t>(stream)), "table")) {
          if (k > 0) end_step(c);                        // (the table is no step's any more)
          return s;
        }
        k += size_t(a.dense);
      }
    for (int32_t i = 0; i < n; ++i) c->tokens[size_t(seqs[i])] += counts[i];
    c->step.swap(step);
    c->step_tokens = int32_t(total);
    c->step_longest = longest;
    c->step_parts = parts;
    c->step_most = most;
    return ok();
  });
}

int ufs_attn_work_bytes(const ufs_cache* c, size_t* bytes) {
  return guarded([&]() -> int {
    if (c == nullptr) return fail(UF_ERR_ARG, "handle is null");
    if (bytes == nullptr) return fail(UF_ERR_ARG, "bytes is null");
    if (c->step.empty()) return fail(UF_ERR_EMPTY, "no step: ufs_extend first");
    *bytes = step_bytes(c);
    return ok();
  });
}

int ufs_attn(const ufs_cache* c, int32_t layer, const ufs_attn_desc* d, const void* d_q, const void* d_k, const void* d_v,
             const float* d_decay, void* d_o, void* d_work, size_t work_bytes, void* stream) {
  return guarded([&]() -> int {
    if (c == nullptr) return fail(UF_ERR_ARG, "handle is null");
    if (d == nullptr) return fail(UF_ERR_ARG, "desc is null");
    if (layer < 0 || layer >= c->d.layers) return fail(UF_ERR_ARG, "layer %d of %d", layer, c->d.layers);
    if (d->q_heads < 1 || d->q_heads % c->d.kv_heads != 0)
      return fail(UF_ERR_ARG, "q_heads %d must be a multiple of kv_heads %d", d->q_heads, c->d.kv_heads);
    if (d->q_heads > 65536) return fail(UF_ERR_ARG, "q_heads must be at most 65536");
    if (!std::isfinite(d->scale)) return fail(UF_ERR_ARG, "scale must be finite");
    if (int s = check_stride(d->q, "q stride")) return s;
    if (int s = check_stride(d->k, "k stride")) return s;
    if (int s = check_stride(d->v, "v stride")) return s;
    if (c->step.empty()) return fail(UF_ERR_EMPTY, "no step: ufs_extend first");
    const int32_t group = d->q_heads / c->d.kv_heads;
    if (double(c->step_longest) / lin::kChunk * group > 2.0e9) return fail(UF_ERR_ARG, "step too large: tokens * q_heads");
    if (c->dry() || c->step_tokens == 0) return ok();
    for (const void* p : {d_q, d_k, d_v, static_cast<const void*>(d_o)}) {
      if (p == nullptr) return fail(UF_ERR_ARG, "q, k, v or o is null");
      if (!aligned(p, 16)) return fail(UF_ERR_ARG, "q, k, v and o must be 16-byte aligned");
    }
    if (d_decay == nullptr || !aligned(d_decay, 4)) return fail(UF_ERR_ARG, "decay must be 4-byte aligned and not null");
    const size_t need = step_bytes(c);
    if (int s = check_work(d_work, work_bytes, need)) return s;
    hipStream_t st = static_cast<hipStream_t>(stream);
    float* const states = c->pool + layer * c->layer_floats();
    lin::Geo g{};
    g.decay = d_decay;
    g.step = c->table;
    g.n = int32_t(c->step.size());
    g.tokens = c->step_tokens;
    g.kv_heads = c->d.kv_heads;
    g.group = group;
    g.parts = c->step_parts;
    g.scanned = scanned(c->step_most, double(c->step_parts) * g.kv_heads, 1);
    g.max_seqs = c->d.max_seqs;
    g.scale = d->scale;
    if (few(c)) {
      lin::StepArgs a{};
      a.geo = g;
      a.q = src(d_q, d->q), a.k = src(d_k, d->k), a.v = src(d_v, d->v);
      a.o = static_cast<uint16_t*>(d_o);
      a.states = states;
      a.longest = c->step_longest;
      if (int s = check_hip(lin::launch_linear_step(a, st), "linear attention")) return s;
      return ok();
    }
    const int32_t groups = g.parts * g.kv_heads;
    float* starts = nullptr;
    if (need > 0) {
      starts = static_cast<float*>(d_work);
      lin::PartArgs p{};
      p.geo = g;
      p.n = 1;
      p.sum[0] = {src(d_k, d->k), src(d_v, d->v), states, starts, 0};
      if (int s = check_hip(lin::launch_linear_parts(p, groups, true, st), "linear attention")) return s;
      if (g.scanned)
        if (int s = check_hip(lin::launch_linear_scan(p, st), "linear attention")) return s;
    }
    lin::WalkArgs a{};
    a.geo = g;
    a.n = 1;
    a.walk[0] = lin::Walk{src(d_q, d->q), src(d_k, d->k), src(d_v, d->v), static_cast<uint16_t*>(d_o), states, states, starts};
    if (int s = check_hip(lin::launch_linear_fwd(a, groups, st), "linear attention")) return s;
    return ok();
  });
}

int ufs_fork(ufs_cache* c, int32_t n, const int32_t* src, const int32_t* dst, void* stream) {
  return guarded([&]() -> int {
    if (c == nullptr) return fail(UF_ERR_ARG, "handle is null");
    if (int s = check_seqs(c, n, dst, "dst")) return s;
    if (src == nullptr) return fail(UF_ERR_ARG, "src is null");
    for (int32_t i = 0; i < n; ++i) {
      if (src[i] < 0 || src[i] >= c->d.max_seqs)
        return fail(UF_ERR_ARG, "src[%d] = %d is no sequence (0 .. %d)", i, src[i], c->d.max_seqs - 1);
      if (c->tokens[size_t(dst[i])] != 0) return fail(UF_ERR_ARG, "sequence %d (dst) is not empty", dst[i]);
    }
    for (int32_t i = 0; i < n; ++i)
      if (c->tokens[size_t(src[i])] == 0) return fail(UF_ERR_EMPTY, "sequence %d (src) is empty", src[i]);
    if (!c->dry())
      for (int32_t i = 0; i < n;) {
        lin::ForkArgs a;
        a.pool = c->pool;
        a.layer = c->layer_floats();
        a.seq = c->seq_floats();
        a.layers = c->d.layers;
        for (a.n = 0; i < n && a.n < lin::kPairs; ++i, ++a.n) {
          a.words[2 * a.n] = src[i];
          a.words[2 * a.n + 1] = dst[i];
        }
        if (int s = check_hip(lin::launch_state_fork(a, static_cast<hipStream_t>(stream)), "fork")) return s;
      }
    for (int32_t i = 0; i < n; ++i) c->tokens[size_t(dst[i])] = c->tokens[size_t(src[i])];
    leave_step(c, n, dst);   // (one that the step names without a token)
    return ok();
  });
}

int ufs_reorder(ufs_cache* c, int32_t groups, int32_t beams, const int32_t* seqs, const int32_t* d_parents, void* stream) {
  return guarded([&]() -> int {
    if (c == nullptr) return fail(UF_ERR_ARG, "handle is null");
    if (groups < 1) return fail(UF_ERR_ARG, "groups must be >= 1 (got %d)", groups);
    if (beams < 1 || beams > lin::kMaxBeams) return fail(UF_ERR_ARG, "beams must be in [1, %d] (got %d)", lin::kMaxBeams, beams);
    const int64_t n = int64_t(groups) * beams;
    if (int s = check_seqs(c, n, seqs, "seqs")) return s;
    for (int64_t i = 0; i < n; ++i) {
      const int32_t held = c->tokens[size_t(seqs[i])], first = c->tokens[size_t(seqs[i / beams * beams])];
      if (held == 0) return fail(UF_ERR_EMPTY, "sequence %d is empty", seqs[i]);
      if (held != first)
        return fail(UF_ERR_ARG, "sequences of a group hold the same number of tokens (%d: %d, %d: %d)", seqs[i / beams * beams],
                    first, seqs[i], held);
    }
    if (!c->dry()) {
      if (d_parents == nullptr || !aligned(d_parents, 4)) return fail(UF_ERR_ARG, "parents must be 4-byte aligned and not null");
      const int32_t most = 2 * lin::kPairs / beams;
      for (int32_t g = 0; g < groups; g += most) {
        lin::ReorderArgs a;
        a.pool = c->pool;
        a.layer = c->layer_floats();
        a.seq = c->seq_floats();
        a.parents = d_parents + int64_t(g) * beams;
        a.layers = c->d.layers;
        a.groups = std::min(most, groups - g);
        a.beams = beams;
        std::copy_n(seqs + int64_t(g) * beams, a.groups * beams, a.seqs);
        if (int s = check_hip(lin::launch_state_reorder(a, static_cast<hipStream_t>(stream)), "reorder")) {
          if (g > 0) leave_step(c, int64_t(g) * beams, seqs);   // (those groups' states have moved)
          return s;
        }
      }
    }
    leave_step(c, n, seqs);
    return ok();
  });
}

int ufs_free(ufs_cache* c, int32_t n, const int32_t* seqs) {
  return guarded([&]() -> int {
    if (c == nullptr) return fail(UF_ERR_ARG, "handle is null");
    if (int s = check_seqs(c, n, seqs, "seqs")) return s;
    leave_step(c, n, seqs);
    for (int32_t i = 0; i < n; ++i) c->tokens[size_t(seqs[i])] = 0;
    return ok();
  });
}

int ufs_get_info(const ufs_cache* c, ufs_info* info) {
  if (c == nullptr || info == nullptr) return fail(UF_ERR_ARG, "null argument");
  info->step_seqs = int32_t(c->step.size());
  info->step_tokens = c->step_tokens;
  info->step_longest = c->step_longest;
  return ok();
}

int ufs_seq_tokens(const ufs_cache* c, int32_t seq, int32_t* tokens) {
  if (c == nullptr || tokens == nullptr) return fail(UF_ERR_ARG, "null argument");
  if (seq < 0 || seq >= c->d.max_seqs) return fail(UF_ERR_ARG, "%d is no sequence (0 .. %d)", seq, c->d.max_seqs - 1);
  *tokens = c->tokens[size_t(seq)];
  return ok();
}

}  // extern "C"

// ---- selection ------------------------------------------------------------------------

namespace {

int check_select(const ufs_select_desc* d, lin::SelectArgs* a) {
  if (d == nullptr) return fail(UF_ERR_ARG, "desc is null");
  if (d->groups < 1 || d->beams < 1 || int64_t(d->groups) * d->beams > (1 << 20) || d->beams > lin::kMaxBeams)
    return fail(UF_ERR_ARG, "groups and beams must be >= 1, beams at most %d, groups * beams at most 2^20", lin::kMaxBeams);
  if (d->vocab < 1 || d->vocab > (1 << 24)) return fail(UF_ERR_ARG, "vocab must be in [1, 2^24] (got %d)", d->vocab);
  if (d->k < 1 || d->k > lin::kMaxSelect) return fail(UF_ERR_ARG, "k must be in [1, %d] (got %d)", lin::kMaxSelect, d->k);
  if (d->type < UFS_BF16 || d->type > UFS_FP32) return fail(UF_ERR_UNSUPPORTED, "logits of type %d", d->type);
  const int64_t most = int64_t(1) << 40;
  if (d->group_stride < 0 || d->beam_stride < 0 || d->group_stride > most || d->beam_stride > most)
    return fail(UF_ERR_ARG, "strides must be in [0, 2^40]");
  *a = lin::SelectArgs{};
  a->groups = d->groups;
  a->beams = d->beams;
  a->vocab = d->vocab;
  a->k = d->k;
  a->type = d->type;
  a->end = d->end;
  a->group_stride = d->group_stride;
  a->beam_stride = d->beam_stride;
  lin::plan_select(a);
  return UF_OK;
}

}  // namespace

extern "C" {

int ufs_select_work_bytes(const ufs_select_desc* d, size_t* bytes) {
  return guarded([&]() -> int {
    lin::SelectArgs a;
    if (int s = check_select(d, &a)) return s;
    if (bytes == nullptr) return fail(UF_ERR_ARG, "bytes is null");
    *bytes = lin::select_work_bytes(a);
    return ok();
  });
}

int ufs_select(const ufs_select_desc* d, const void* d_logits, const float* d_scores, const uint8_t* d_done, float* d_best,
               int32_t* d_parents, int32_t* d_tokens, void* d_work, size_t work_bytes, void* stream) {
  return guarded([&]() -> int {
    lin::SelectArgs a;
    if (int s = check_select(d, &a)) return s;
    if (d_done != nullptr && (d->end < 0 || d->end >= d->vocab))
      return fail(UF_ERR_ARG, "end must be in [0, %d] (got %d)", d->vocab - 1, d->end);
    if (d_logits == nullptr || d_scores == nullptr || d_best == nullptr || d_parents == nullptr || d_tokens == nullptr)
      return fail(UF_ERR_ARG, "a tensor is null");
    if (!aligned(d_logits, d->type == UFS_FP32 ? 4 : 2)) return fail(UF_ERR_ARG, "logits must be aligned to their type");
    if (!aligned(d_scores, 4) || !aligned(d_best, 4) || !aligned(d_parents, 4) || !aligned(d_tokens, 4))
      return fail(UF_ERR_ARG, "scores, best, parents and tokens must be 4-byte aligned");
    if (int s = check_work(d_work, work_bytes, lin::select_work_bytes(a))) return s;
    a.logits = d_logits;
    a.scores = d_scores;
    a.done = d_done;
    a.best = d_best;
    a.parents = d_parents;
    a.tokens = d_tokens;
    a.work = static_cast<uint8_t*>(d_work);
    if (int s = check_hip(lin::launch_select(a, static_cast<hipStream_t>(stream)), "selection")) return s;
    return ok();
  });
}

}  // extern "C"
