// C ABI of the token operators: argument validation, the page tables of the token
// cache, and kernel launches.  See include/uft.h for the contract of every entry point.
//
// The host holds the truth about pages: the pages of every sequence, how many
// sequences use each page, and which are free.  Kernels read a copy of the tables in
// device memory, which every call that changes them brings up to date on its
// stream: the words ride in launch arguments, so that nothing is copied from host
// memory.  A call first plans, then launches, then commits: a failed call leaves the
// handle as it was.
#include <algorithm>
#include <climits>
#include <cmath>
#include <functional>
#include <new>
#include <queue>
#include <vector>

#include "launch_tokens.h"
#include "status.h"

namespace {

using uf::fail;
using uf::ok;
namespace tok = uf::tok;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

struct Seq {
  int32_t tokens = 0;
  std::vector<int32_t> pages;   // -1: trimmed
};

struct Entry {                  // a sequence of the step
  int32_t seq, at, count, tokens;
};

}  // namespace

struct uft_cache {
  uft_desc d;
  uint8_t* pool;
  int32_t* table;               // header, step, then page rows
  int32_t row;                  // pages of a sequence at most
  std::vector<Seq> seqs;
  std::vector<int32_t> uses;    // per page
  std::priority_queue<int32_t, std::vector<int32_t>, std::greater<int32_t>> free;
  std::vector<Entry> step;
  int32_t step_tokens = 0, step_longest = 0;
  std::vector<uint8_t> seen;    // scratch of the checks, all 0 between calls

  bool dry() const { return (d.flags & UF_F_DRYRUN) != 0; }
  int32_t rows_at() const { return tok::kHeader + tok::kEntry * d.max_seqs; }
  int32_t row_at(int32_t seq) const { return rows_at() + seq * row; }
  size_t layer_bytes() const { return size_t(d.n_pages) * d.kv_heads * d.page_tokens * 4 * tok::kD; }
  tok::Pool pool_of(int32_t layer) const {
    return tok::Pool{pool + size_t(layer) * layer_bytes(), layer_bytes(), d.layers, d.n_pages, d.kv_heads, d.page_tokens};
  }
  void release(int32_t page) {
    if (page >= 0 && --uses[size_t(page)] == 0) free.push(page);
  }
};

namespace {

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

int check_desc(const uft_desc* d) {
  if (d == nullptr) return fail(UF_ERR_ARG, "desc is null");
  if (d->layers < 1 || d->layers > 65535) return fail(UF_ERR_ARG, "layers must be in [1, 65535] (got %d)", d->layers);
  if (d->kv_heads < 1 || d->kv_heads > 4096) return fail(UF_ERR_ARG, "kv_heads must be in [1, 4096] (got %d)", d->kv_heads);
  if (d->n_pages < 1) return fail(UF_ERR_ARG, "n_pages must be >= 1 (got %d)", d->n_pages);
  if (d->max_seqs < 1 || d->max_seqs > 65535)
    return fail(UF_ERR_ARG, "max_seqs must be in [1, 65535] (got %d)", d->max_seqs);
  if (d->max_tokens < 1 || d->max_tokens > (1 << 30))
    return fail(UF_ERR_ARG, "max_tokens must be in [1, 2^30] (got %d)", d->max_tokens);
  if (d->flags & ~UF_F_DRYRUN) return fail(UF_ERR_ARG, "unknown flag bits 0x%x", d->flags);
  if (d->page_tokens < 1 || d->head_dim < 1) return fail(UF_ERR_ARG, "page_tokens and head_dim must be >= 1");
  if (d->head_dim != tok::kD) return fail(UF_ERR_UNSUPPORTED, "head_dim %d: only 128 is built", d->head_dim);
  if (d->page_tokens != 64 && d->page_tokens != 128)
    return fail(UF_ERR_UNSUPPORTED, "page_tokens %d: only 64 and 128 are built", d->page_tokens);
  const int64_t row = (int64_t(d->max_tokens) + d->page_tokens - 1) / d->page_tokens;
  if (tok::kHeader + int64_t(d->max_seqs) * (tok::kEntry + row) > INT32_MAX)
    return fail(UF_ERR_ARG, "tables too large: max_seqs * pages of max_tokens must fit in int32");
  // (exact in double up to 2^53; the largest pools are far below)
  if (double(d->layers) * d->n_pages * d->kv_heads * d->page_tokens * 4.0 * tok::kD > 4.0e15)
    return fail(UF_ERR_ARG, "pool too large");
  return UF_OK;
}

int check_hip(hipError_t e, const char* what) {
  if (e == hipSuccess) return UF_OK;
  return fail(UF_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
}

// n sequence numbers, each once.
int check_seqs(uft_cache* c, int32_t n, const int32_t* seqs, const char* name) {
  if (n < 1) return fail(UF_ERR_ARG, "n must be >= 1 (got %d)", n);
  if (seqs == nullptr) return fail(UF_ERR_ARG, "%s is null", name);
  int s = UF_OK;
  int32_t i = 0;
  for (; i < n; ++i) {
    if (seqs[i] < 0 || seqs[i] >= c->d.max_seqs) {
      s = fail(UF_ERR_ARG, "%s[%d] = %d is no sequence (0 .. %d)", name, i, seqs[i], c->d.max_seqs - 1);
      break;
    }
    if (c->seen[size_t(seqs[i])]) {
      s = fail(UF_ERR_ARG, "%s names sequence %d twice", name, seqs[i]);
      break;
    }
    c->seen[size_t(seqs[i])] = 1;
  }
  for (int32_t k = 0; k < i; ++k) c->seen[size_t(seqs[k])] = 0;
  return s;
}

// Pages taken for a call, lowest first; handed back if it fails.
class Taken {
 public:
  explicit Taken(uft_cache* c) : c_(c) {}
  ~Taken() {
    if (!kept_)
      for (int32_t p : pages_) {
        c_->uses[size_t(p)] = 0;
        c_->free.push(p);
      }
  }
  int32_t take() {
    const int32_t p = c_->free.top();
    pages_.push_back(p);   // (room was made by reserve: nothing throws after the pop)
    c_->free.pop();
    c_->uses[size_t(p)] = 1;
    return p;
  }
  int reserve(int64_t n) {
    if (n > int64_t(c_->free.size()))
      return fail(UF_ERR_CAPACITY, "%lld pages needed, %zu free", (long long)n, c_->free.size());
    pages_.reserve(size_t(n));
    return UF_OK;
  }
  void keep() { kept_ = true; }

 private:
  uft_cache* c_;
  std::vector<int32_t> pages_;
  bool kept_ = false;
};

// Changes of the device tables, sent in as many launches as their words need.
class Poke {
 public:
  explicit Poke(const uft_cache* c) : c_(c) {}
  std::vector<int32_t> dense;   // from word 0 of the table on
  // values for table words at ..: runs of ascending pages, or of -1
  void run(int32_t at, const int32_t* values, int32_t n) {
    for (int32_t i = 0; i < n;) {
      int32_t e = i + 1;
      while (e < n && values[e] == (values[i] < 0 ? values[i] : values[i] + e - i)) ++e;
      runs_.insert(runs_.end(), {at + i, e - i, values[i]});
      i = e;
    }
  }
  // All of it beside `used` words of another launch: its head, the words behind them.  False where it does not fit.
  bool join(tok::PokeHead* head, int32_t* words, int used) {
    if (size_t(used) + dense.size() + runs_.size() > size_t(tok::kWords)) return false;
    *head = tok::PokeHead{c_->table, 0, int32_t(dense.size()), int32_t(dense.size()), int32_t(runs_.size() / 3)};
    std::copy(dense.begin(), dense.end(), words + used);
    std::copy(runs_.begin(), runs_.end(), words + used + dense.size());
    return true;
  }
  int words() const { return int(dense.size() + runs_.size()); }
  int send(hipStream_t stream) {
    if (c_->dry()) return UF_OK;
    for (size_t di = 0, ri = 0; di < dense.size() || ri < runs_.size();) {
      tok::PokeArgs a;
      a.table = c_->table;
      a.dense_at = int32_t(di);
      a.dense = a.runs = int32_t(std::min(dense.size() - di, size_t(tok::kWords)));
      std::copy_n(dense.begin() + di, a.dense, a.words);
      di += size_t(a.dense);
      a.n_runs = int32_t(std::min((runs_.size() - ri) / 3, size_t(tok::kWords - a.dense) / 3));
      std::copy_n(runs_.begin() + ri, 3 * a.n_runs, a.words + a.runs);
      ri += size_t(3 * a.n_runs);
      if (int s = check_hip(tok::launch_poke(a, a.dense + 3 * a.n_runs, stream), "table")) return s;
    }
    return UF_OK;
  }

 private:
  const uft_cache* c_;
  std::vector<int32_t> runs_;   // (at, count, first value)
};

// Pages to copy and table changes: in one launch where their words fit.
int copy_and_poke(const uft_cache* c, const std::vector<int32_t>& triples, Poke& poke, hipStream_t stream) {
  if (c->dry()) return UF_OK;
  for (size_t i = 0; i < triples.size();) {
    tok::CopyArgs a;
    a.pool = c->pool_of(0);
    a.poke = tok::PokeHead{};
    const size_t n = std::min(triples.size() - i, size_t(tok::kWords / 3 * 3));
    std::copy_n(triples.begin() + i, n, a.words);
    a.n = int32_t(n / 3);
    i += n;
    const bool joined = i == triples.size() && poke.join(&a.poke, a.words, int(n));
    if (int s = check_hip(tok::launch_copy_pages(a, int(n) + (joined ? poke.words() : 0), stream), "page copy")) return s;
    if (joined) return UF_OK;
  }
  return poke.send(stream);
}

bool in_step(uft_cache* c, int32_t n, const int32_t* seqs) {
  for (int32_t i = 0; i < n; ++i) c->seen[size_t(seqs[i])] = 1;
  bool found = false;
  for (const Entry& e : c->step) found = found || c->seen[size_t(e.seq)];
  for (int32_t i = 0; i < n; ++i) c->seen[size_t(seqs[i])] = 0;
  return found;
}
void end_step(uft_cache* c) {
  c->step.clear();
  c->step_tokens = c->step_longest = 0;
}

int check_stride(const uft_stride* s, const char* name) {
  if (s == nullptr) return fail(UF_ERR_ARG, "%s is null", name);
  if (s->token < 0 || s->head < 0 || s->batch < 0) return fail(UF_ERR_ARG, "%s must not be negative", name);
  if (s->token % 8 || s->head % 8 || s->batch % 8) return fail(UF_ERR_ARG, "%s must be multiples of 8", name);
  // a tile's offsets are 32-bit: 64 tokens' strides in bytes
  if (s->token > (int64_t(1) << 24)) return fail(UF_ERR_ARG, "%s.token must be at most 2^24", name);
  if (s->head > (int64_t(1) << 30)) return fail(UF_ERR_ARG, "%s.head must be at most 2^30", name);
  return UF_OK;
}

int check_scale(float scale, float* log2) {
  *log2 = scale * 1.4426950408889634f;
  if (!(scale > 0.f) || !std::isfinite(scale) || !std::isnormal(*log2))
    return fail(UF_ERR_ARG, "scale must be positive, finite and normal");
  return UF_OK;
}

// Workgroups go to the tiles that sequences have (`tiles`; their waves look up whose theirs is), not to as many for each
// sequence as the longest has (`each`), where most of those would find nothing; 0: for each.  Measured (us, for each / to
// what there is): 255 single tokens and a piece of 512 over 1,000 earlier ones, 8 key heads, attention 408 / 237, write 32 /
// 11, and 4,160 / 16 MiB of scratch; 7 x 64 and 512 tokens 58 / 36.5; near to even, 3 x 256 and 512 tokens, 45.6 / 44.4; 1,023
// of 1,024 sequences with few rows 304 / 420 (looking up costs a round of 64 sequences after the other): the rule takes the
// first in those last two.
int32_t deal_packed(int64_t each, int64_t tiles) { return each > 2 * tiles && tiles <= INT32_MAX ? int32_t(tiles) : 0; }

int check_fork(uft_cache* c, int32_t n, const int32_t* src, const int32_t* dst) {
  if (int s = check_seqs(c, n, dst, "dst")) return s;
  if (src == nullptr) return fail(UF_ERR_ARG, "src is null");
  for (int32_t i = 0; i < n; ++i) {
    if (src[i] < 0 || src[i] >= c->d.max_seqs)
      return fail(UF_ERR_ARG, "src[%d] = %d is no sequence (0 .. %d)", i, src[i], c->d.max_seqs - 1);
    if (!c->seqs[size_t(dst[i])].pages.empty()) return fail(UF_ERR_ARG, "sequence %d (dst) is not empty", dst[i]);
  }
  for (int32_t i = 0; i < n; ++i)
    if (c->seqs[size_t(src[i])].pages.empty()) return fail(UF_ERR_EMPTY, "sequence %d (src) is empty", src[i]);
  return UF_OK;
}

}  // namespace

extern "C" {

int uft_pool_bytes(const uft_desc* desc, size_t* bytes) {
  if (int s = check_desc(desc)) return s;
  if (bytes == nullptr) return fail(UF_ERR_ARG, "bytes is null");
  *bytes = size_t(desc->layers) * desc->n_pages * desc->kv_heads * desc->page_tokens * 4 * tok::kD;
  return ok();
}

int uft_table_bytes(const uft_desc* desc, size_t* bytes) {
  if (int s = check_desc(desc)) return s;
  if (bytes == nullptr) return fail(UF_ERR_ARG, "bytes is null");
  const size_t row = (size_t(desc->max_tokens) + desc->page_tokens - 1) / desc->page_tokens;
  *bytes = 4 * (size_t(tok::kHeader) + size_t(desc->max_seqs) * (tok::kEntry + row));
  return ok();
}

int uft_create(const uft_desc* desc, void* d_pool, size_t pool_bytes, void* d_table, size_t table_bytes,
               uft_cache** out) {
  return guarded([&]() -> int {
    if (out == nullptr) return fail(UF_ERR_ARG, "out is null");
    size_t pool = 0, table = 0;
    if (int s = uft_pool_bytes(desc, &pool)) return s;
    if (int s = uft_table_bytes(desc, &table)) return s;
    const bool dry = (desc->flags & UF_F_DRYRUN) != 0;
    if (!dry && (d_pool == nullptr || d_table == nullptr)) return fail(UF_ERR_ARG, "pool or table is null");
    if (!aligned(d_pool, 256) || !aligned(d_table, 256)) return fail(UF_ERR_ARG, "pool and table must be 256-byte aligned");
    if (!dry && pool_bytes < pool) return fail(UF_ERR_CAPACITY, "pool has %zu bytes, the cache needs %zu", pool_bytes, pool);
    if (!dry && table_bytes < table)
      return fail(UF_ERR_CAPACITY, "table has %zu bytes, the cache needs %zu", table_bytes, table);
    uft_cache* c = new uft_cache();
    try {
      c->d = *desc;
      c->pool = static_cast<uint8_t*>(d_pool);
      c->table = static_cast<int32_t*>(d_table);
      c->row = (desc->max_tokens + desc->page_tokens - 1) / desc->page_tokens;
      c->seqs.resize(size_t(desc->max_seqs));
      c->seen.assign(size_t(desc->max_seqs), 0);
      c->uses.assign(size_t(desc->n_pages), 0);
      for (int32_t p = 0; p < desc->n_pages; ++p) c->free.push(p);   // (the heap never holds more)
    } catch (...) {
      delete c;
      throw;
    }
    *out = c;
    return ok();
  });
}

int uft_destroy(uft_cache* cache) {
  delete cache;
  return UF_OK;   // (the last error's text stays, as in uf_kv_destroy)
}

int uft_extend(uft_cache* c, int32_t n, const int32_t* seqs, const int32_t* counts, void* stream) {
  return guarded([&]() -> int {
    if (c == nullptr) return fail(UF_ERR_ARG, "handle is null");
    if (int s = check_seqs(c, n, seqs, "seqs")) return s;
    if (counts == nullptr) return fail(UF_ERR_ARG, "counts is null");
    const int32_t T = c->d.page_tokens;
    int64_t need = 0, total = 0;
    int32_t longest = 0;
    // pages whose sharers all grow: the last of them keeps the page, as its use count says then
    std::vector<int32_t> shared;
    for (int32_t i = 0; i < n; ++i) {
      const Seq& q = c->seqs[size_t(seqs[i])];
      if (counts[i] < 0) return fail(UF_ERR_ARG, "counts[%d] must be >= 0 (got %d)", i, counts[i]);
      if (int64_t(q.tokens) + counts[i] > c->d.max_tokens)
        return fail(UF_ERR_CAPACITY, "sequence %d: %d + %d tokens, at most %d", seqs[i], q.tokens, counts[i], c->d.max_tokens);
      need += (int64_t(q.tokens) + counts[i] + T - 1) / T - int64_t(q.pages.size());
      if (counts[i] > 0 && q.tokens % T != 0 && c->uses[size_t(q.pages.back())] > 1) shared.push_back(q.pages.back());
      total += counts[i];
      longest = std::max(longest, counts[i]);
    }
    if (total > INT32_MAX) return fail(UF_ERR_ARG, "more than 2^31 - 1 new tokens");
    std::sort(shared.begin(), shared.end());
    for (size_t i = 0; i < shared.size();) {
      size_t e = i;
      while (e < shared.size() && shared[e] == shared[i]) ++e;
      need += std::min(int64_t(e - i), int64_t(c->uses[size_t(shared[i])]) - 1);
      i = e;
    }
    Taken taken(c);
    if (int s = taken.reserve(need)) return s;

    struct Grown {
      int32_t own = -1, old = -1;      // copy on write
      std::vector<int32_t> fresh;
    };
    std::vector<Grown> grown(static_cast<size_t>(n));
    std::vector<int32_t> copies;
    std::vector<Entry> step;
    Poke poke(c);
    step.reserve(size_t(n));
    copies.reserve(3 * shared.size());
    poke.dense = {n, int32_t(total), 0, 0};
    std::vector<int32_t> gone(shared.size(), 0);   // uses given up so far, at a page's first place in `shared`
    int32_t at = 0;
    for (int32_t i = 0; i < n; ++i) {
      const Seq& q = c->seqs[size_t(seqs[i])];
      Grown& g = grown[size_t(i)];
      if (counts[i] > 0 && q.tokens % T != 0) {
        const int32_t last = q.pages.back();
        const size_t at = size_t(std::lower_bound(shared.begin(), shared.end(), last) - shared.begin());
        if (c->uses[size_t(last)] > 1 && c->uses[size_t(last)] - gone[at] > 1) {
          g.old = last;
          g.own = taken.take();
          ++gone[at];
          copies.insert(copies.end(), {last, g.own, q.tokens % T});
          poke.run(c->row_at(seqs[i]) + int32_t(q.pages.size()) - 1, &g.own, 1);
        }
      }
      const int32_t pages = int32_t((int64_t(q.tokens) + counts[i] + T - 1) / T);
      for (int32_t p = int32_t(q.pages.size()); p < pages; ++p) g.fresh.push_back(taken.take());
      if (!g.fresh.empty())
        poke.run(c->row_at(seqs[i]) + int32_t(q.pages.size()), g.fresh.data(), int32_t(g.fresh.size()));
      step.push_back(Entry{seqs[i], at, counts[i], q.tokens + counts[i]});
      poke.dense.insert(poke.dense.end(), {seqs[i], at, counts[i], q.tokens + counts[i]});
      at += counts[i];
    }
    for (int32_t i = 0; i < n; ++i)
      c->seqs[size_t(seqs[i])].pages.reserve(c->seqs[size_t(seqs[i])].pages.size() + grown[size_t(i)].fresh.size());
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (int s = copy_and_poke(c, copies, poke, st)) return s;
    taken.keep();
    for (int32_t i = 0; i < n; ++i) {
      Seq& q = c->seqs[size_t(seqs[i])];
      Grown& g = grown[size_t(i)];
      if (g.own >= 0) {
        c->release(g.old);
        q.pages.back() = g.own;
      }
      q.pages.insert(q.pages.end(), g.fresh.begin(), g.fresh.end());
      q.tokens += counts[i];
    }
    c->step.swap(step);
    c->step_tokens = int32_t(total);
    c->step_longest = longest;
    return ok();
  });
}

int uft_write(const uft_cache* c, int32_t layer, const void* d_k, const uft_stride* k_stride, const void* d_v,
              const uft_stride* v_stride, void* stream) {
  return guarded([&]() -> int {
    if (c == nullptr) return fail(UF_ERR_ARG, "handle is null");
    if (layer < 0 || layer >= c->d.layers) return fail(UF_ERR_ARG, "layer %d of %d", layer, c->d.layers);
    if (int s = check_stride(k_stride, "k_stride")) return s;
    if (int s = check_stride(v_stride, "v_stride")) return s;
    if (c->step.empty()) return fail(UF_ERR_EMPTY, "no step: uft_extend first");
    if (c->dry() || c->step_tokens == 0) return ok();
    if (d_k == nullptr || d_v == nullptr) return fail(UF_ERR_ARG, "k or v is null");
    if (!aligned(d_k, 16) || !aligned(d_v, 16)) return fail(UF_ERR_ARG, "k and v must be 16-byte aligned");
    tok::WriteArgs a{};
    a.k = static_cast<const uint16_t*>(d_k);
    a.v = static_cast<const uint16_t*>(d_v);
    a.k_token = k_stride->token;
    a.k_head = k_stride->head;
    a.v_token = v_stride->token;
    a.v_head = v_stride->head;
    a.pool = c->pool_of(layer);
    a.step = c->table;
    a.table = c->table + c->rows_at();
    a.n = int32_t(c->step.size());
    a.longest = c->step_longest;
    a.total = c->step_tokens;
    a.row = c->row;
    int64_t spans = 0;
    for (const Entry& e : c->step) spans += tok::write_spans(e.count, c->d.page_tokens);
    a.packed = deal_packed(int64_t(a.n) * tok::write_spans(a.longest, c->d.page_tokens), spans);
    if (int s = check_hip(tok::launch_write(a, static_cast<hipStream_t>(stream)), "token write")) return s;
    return ok();
  });
}

int uft_fork(uft_cache* c, int32_t n, const int32_t* src, const int32_t* dst, void* stream) {
  return guarded([&]() -> int {
    if (c == nullptr) return fail(UF_ERR_ARG, "handle is null");
    if (int s = check_fork(c, n, src, dst)) return s;
    for (int32_t i = 0; i < n; ++i) c->seqs[size_t(dst[i])].pages.reserve(c->seqs[size_t(src[i])].pages.size());
    if (!c->dry())
      for (int32_t i = 0; i < n;) {
        tok::RowsArgs a;
        a.table = c->table;
        a.n = 0;
        for (; i < n && a.n < tok::kWords / 3; ++i, ++a.n) {
          a.words[3 * a.n] = c->row_at(src[i]);
          a.words[3 * a.n + 1] = c->row_at(dst[i]);
          a.words[3 * a.n + 2] = int32_t(c->seqs[size_t(src[i])].pages.size());
        }
        if (int s = check_hip(tok::launch_rows(a, static_cast<hipStream_t>(stream)), "fork")) return s;
      }
    for (int32_t i = 0; i < n; ++i) {
      const Seq& from = c->seqs[size_t(src[i])];
      Seq& to = c->seqs[size_t(dst[i])];
      to.pages.assign(from.pages.begin(), from.pages.end());
      to.tokens = from.tokens;
      for (int32_t p : to.pages)
        if (p >= 0) ++c->uses[size_t(p)];
    }
    return ok();
  });
}

int uft_copy(uft_cache* c, int32_t n, const int32_t* src, const int32_t* dst, void* stream) {
  return guarded([&]() -> int {
    if (c == nullptr) return fail(UF_ERR_ARG, "handle is null");
    if (int s = check_fork(c, n, src, dst)) return s;
    const int32_t T = c->d.page_tokens;
    int64_t need = 0;
    for (int32_t i = 0; i < n; ++i)
      for (int32_t p : c->seqs[size_t(src[i])].pages) need += p >= 0;
    Taken taken(c);
    if (int s = taken.reserve(need)) return s;
    std::vector<std::vector<int32_t>> pages(static_cast<size_t>(n));
    std::vector<int32_t> copies;
    copies.reserve(size_t(3 * need));
    Poke poke(c);
    for (int32_t i = 0; i < n; ++i) {
      const Seq& from = c->seqs[size_t(src[i])];
      std::vector<int32_t>& to = pages[size_t(i)];
      for (size_t k = 0; k < from.pages.size(); ++k) {
        to.push_back(from.pages[k] < 0 ? -1 : taken.take());
        if (from.pages[k] >= 0)
          copies.insert(copies.end(), {from.pages[k], to.back(), std::min(T, from.tokens - int32_t(k) * T)});
      }
      poke.run(c->row_at(dst[i]), to.data(), int32_t(to.size()));
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (int s = copy_and_poke(c, copies, poke, st)) return s;
    taken.keep();
    for (int32_t i = 0; i < n; ++i) {
      c->seqs[size_t(dst[i])].pages.swap(pages[size_t(i)]);
      c->seqs[size_t(dst[i])].tokens = c->seqs[size_t(src[i])].tokens;
    }
    return ok();
  });
}

int uft_keep(uft_cache* c, int32_t n, const int32_t* seqs, const int32_t* starts, const int32_t* counts,
             const int32_t* d_index, void* stream) {
  return guarded([&]() -> int {
    if (c == nullptr) return fail(UF_ERR_ARG, "handle is null");
    if (int s = check_seqs(c, n, seqs, "seqs")) return s;
    if (starts == nullptr || counts == nullptr) return fail(UF_ERR_ARG, "starts or counts is null");
    const int32_t T = c->d.page_tokens;
    struct Move {
      int32_t first, end, index;   // pages written, first entry of the index
      bool fresh;
      std::vector<int32_t> pages;
    };
    std::vector<Move> moves(static_cast<size_t>(n));
    int64_t need = 0, index = 0;
    bool any = false;
    for (int32_t i = 0; i < n; ++i) {
      const Seq& q = c->seqs[size_t(seqs[i])];
      if (starts[i] < 0 || counts[i] < 0 || int64_t(starts[i]) + counts[i] > q.tokens)
        return fail(UF_ERR_ARG, "sequence %d: keep %d + %d of %d tokens", seqs[i], starts[i], counts[i], q.tokens);
      Move& m = moves[size_t(i)];
      m.first = starts[i] / T;
      m.end = (starts[i] + counts[i] + T - 1) / T;
      m.index = int32_t(index);
      m.fresh = counts[i] > tok::kInPlace;
      for (size_t p = size_t(m.first); p < q.pages.size(); ++p)
        if (q.pages[p] < 0)
          return fail(UF_ERR_ARG, "sequence %d: pages from token %d on were trimmed", seqs[i], starts[i]);
      if (counts[i] > 0) {
        any = true;
        for (int32_t p = m.first; p < m.end; ++p) m.fresh = m.fresh || c->uses[size_t(q.pages[size_t(p)])] > 1;
      }
      if (m.fresh) need += m.end - m.first;
      index += counts[i];
    }
    if (index > INT32_MAX) return fail(UF_ERR_ARG, "more than 2^31 - 1 tokens kept");
    if (any && !c->dry() && d_index == nullptr) return fail(UF_ERR_ARG, "index is null");
    if (any && !aligned(d_index, 4)) return fail(UF_ERR_ARG, "index must be 4-byte aligned");
    Taken taken(c);
    if (int s = taken.reserve(need)) return s;
    Poke poke(c);
    for (int32_t i = 0; i < n; ++i) {
      Move& m = moves[size_t(i)];
      if (!m.fresh) continue;
      for (int32_t p = m.first; p < m.end; ++p) m.pages.push_back(taken.take());
      poke.run(c->row_at(seqs[i]) + m.first, m.pages.data(), m.end - m.first);
    }
    if (!c->dry() && any) {
      hipStream_t st = static_cast<hipStream_t>(stream);
      tok::KeepArgs a;
      a.pool = c->pool_of(0);
      a.table = c->table + c->rows_at();
      a.index = d_index;
      auto words = [&](int32_t i) {
        const Move& m = moves[size_t(i)];
        int32_t* w = a.words + tok::kKeepWords * a.n++;
        w[0] = seqs[i] * c->row;
        w[1] = c->seqs[size_t(seqs[i])].tokens;
        w[2] = starts[i];
        w[3] = counts[i];
        w[4] = m.index;
        return w;
      };
      for (int32_t i = 0; i < n;) {
        a.n = 0;
        for (; i < n && a.n < tok::kWords / tok::kKeepWords; ++i)
          if (counts[i] > 0 && !moves[size_t(i)].fresh) words(i);
        if (a.n > 0)
          if (int s = check_hip(tok::launch_keep_in_place(a, st), "keep")) return s;
      }
      // fresh pages, run by run
      a.n = a.n_pages = 0;
      for (int32_t i = 0; i < n; ++i) {
        const Move& m = moves[size_t(i)];
        for (size_t k = 0; k < m.pages.size();) {
          size_t e = k + 1;
          while (e < m.pages.size() && m.pages[e] == m.pages[k] + int32_t(e - k)) ++e;
          int32_t* w = words(i);
          w[5] = m.first + int32_t(k);
          w[6] = a.n_pages;
          w[7] = m.pages[k];
          a.n_pages += int32_t(e - k);
          k = e;
          if (a.n == tok::kWords / tok::kKeepWords) {
            if (int s = check_hip(tok::launch_keep_fresh(a, st), "keep")) return s;
            a.n = a.n_pages = 0;
          }
        }
      }
      if (a.n > 0)
        if (int s = check_hip(tok::launch_keep_fresh(a, st), "keep")) return s;
      if (int s = poke.send(st)) return s;
    }
    if (in_step(c, n, seqs)) end_step(c);
    taken.keep();
    for (int32_t i = 0; i < n; ++i) {
      Seq& q = c->seqs[size_t(seqs[i])];
      const Move& m = moves[size_t(i)];
      if (m.fresh) {
        for (int32_t p = m.first; p < m.end; ++p) {
          c->release(q.pages[size_t(p)]);
          q.pages[size_t(p)] = m.pages[size_t(p - m.first)];
        }
      }
      for (size_t p = size_t(m.end); p < q.pages.size(); ++p) c->release(q.pages[p]);
      q.pages.resize(size_t(m.end));
      q.tokens = starts[i] + counts[i];
    }
    return ok();
  });
}

int uft_trim(uft_cache* c, int32_t n, const int32_t* seqs, int32_t window, int32_t sinks, void* stream) {
  return guarded([&]() -> int {
    if (c == nullptr) return fail(UF_ERR_ARG, "handle is null");
    if (int s = check_seqs(c, n, seqs, "seqs")) return s;
    if (window < 1) return fail(UF_ERR_ARG, "window must be >= 1 (got %d)", window);
    if (sinks < 0) return fail(UF_ERR_ARG, "sinks must be >= 0 (got %d)", sinks);
    const int64_t T = c->d.page_tokens;
    Poke poke(c);
    struct Hole { int32_t seq, from, to; };
    std::vector<Hole> holes;
    std::vector<int32_t> none(static_cast<size_t>(c->row), -1);
    for (int32_t i = 0; i < n; ++i) {
      const Seq& q = c->seqs[size_t(seqs[i])];
      const int64_t from = (int64_t(sinks) + T - 1) / T, to = (int64_t(q.tokens) - window + 1) / T;
      if (q.tokens + int64_t(1) < window || from >= to) continue;
      holes.push_back(Hole{seqs[i], int32_t(from), int32_t(to)});
      poke.run(c->row_at(seqs[i]) + int32_t(from), none.data(), int32_t(to - from));
    }
    // a step some of whose own tokens lose their place is over
    bool ends = false;
    if (!holes.empty()) {
      std::vector<int64_t> gone(size_t(c->d.max_seqs), 0);   // tokens before the hole's end
      for (const Hole& h : holes) gone[size_t(h.seq)] = h.to * T;
      for (const Entry& e : c->step) ends = ends || (e.count > 0 && gone[size_t(e.seq)] > e.tokens - e.count);
    }
    if (int s = poke.send(static_cast<hipStream_t>(stream))) return s;
    if (ends) end_step(c);
    for (const Hole& h : holes) {
      Seq& q = c->seqs[size_t(h.seq)];
      for (int32_t p = h.from; p < h.to; ++p) {
        c->release(q.pages[size_t(p)]);
        q.pages[size_t(p)] = -1;
      }
    }
    return ok();
  });
}

int uft_free(uft_cache* c, int32_t n, const int32_t* seqs) {
  return guarded([&]() -> int {
    if (c == nullptr) return fail(UF_ERR_ARG, "handle is null");
    if (int s = check_seqs(c, n, seqs, "seqs")) return s;
    if (in_step(c, n, seqs)) end_step(c);
    for (int32_t i = 0; i < n; ++i) {
      Seq& q = c->seqs[size_t(seqs[i])];
      for (int32_t p : q.pages) c->release(p);
      q.pages.clear();
      q.tokens = 0;
    }
    return ok();
  });
}

int uft_pack(uft_cache* c, int32_t* used_pages, void* stream) {
  return guarded([&]() -> int {
    if (c == nullptr) return fail(UF_ERR_ARG, "handle is null");
    const int32_t T = c->d.page_tokens, used = c->d.n_pages - int32_t(c->free.size());
    std::vector<int32_t> to(size_t(c->d.n_pages), -1), rows(size_t(c->d.n_pages), 0), copies;
    int32_t hole = 0;
    for (int32_t p = used; p < c->d.n_pages; ++p)
      if (c->uses[size_t(p)] > 0) {
        while (c->uses[size_t(hole)] > 0) ++hole;
        to[size_t(p)] = hole++;
      }
    for (const Seq& q : c->seqs)
      for (size_t k = 0; k < q.pages.size(); ++k)
        if (q.pages[k] >= 0)
          rows[size_t(q.pages[k])] = std::max(rows[size_t(q.pages[k])], std::min(T, q.tokens - int32_t(k) * T));
    for (int32_t p = used; p < c->d.n_pages; ++p)
      if (to[size_t(p)] >= 0) copies.insert(copies.end(), {p, to[size_t(p)], rows[size_t(p)]});
    Poke poke(c);
    for (int32_t s = 0; s < c->d.max_seqs; ++s) {
      const std::vector<int32_t>& pages = c->seqs[size_t(s)].pages;
      for (size_t k = 0; k < pages.size(); ++k)
        if (pages[k] >= 0 && to[size_t(pages[k])] >= 0) poke.run(c->row_at(s) + int32_t(k), &to[size_t(pages[k])], 1);
    }
    std::vector<int32_t> uses(size_t(c->d.n_pages), 0), left;
    left.reserve(size_t(c->d.n_pages));
    for (int32_t p = c->d.n_pages - 1; p >= used; --p) left.push_back(p);
    decltype(c->free) free(std::greater<int32_t>(), std::move(left));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (int s = copy_and_poke(c, copies, poke, st)) return s;
    for (Seq& q : c->seqs)
      for (int32_t& p : q.pages)
        if (p >= 0) {
          if (to[size_t(p)] >= 0) p = to[size_t(p)];
          ++uses[size_t(p)];
        }
    c->uses.swap(uses);
    c->free.swap(free);
    if (used_pages != nullptr) *used_pages = used;
    return ok();
  });
}

int uft_get_info(const uft_cache* c, uft_info* info) {
  if (c == nullptr || info == nullptr) return fail(UF_ERR_ARG, "null argument");
  info->free_pages = int32_t(c->free.size());
  info->step_seqs = int32_t(c->step.size());
  info->step_tokens = c->step_tokens;
  info->step_longest = c->step_longest;
  return ok();
}

int uft_seq_tokens(const uft_cache* c, int32_t seq, int32_t* tokens) {
  if (c == nullptr || tokens == nullptr) return fail(UF_ERR_ARG, "null argument");
  if (seq < 0 || seq >= c->d.max_seqs) return fail(UF_ERR_ARG, "%d is no sequence (0 .. %d)", seq, c->d.max_seqs - 1);
  *tokens = c->seqs[size_t(seq)].tokens;
  return ok();
}

int uft_seq_pages(const uft_cache* c, int32_t seq, int32_t* pages, int32_t cap, int32_t* n) {
  if (c == nullptr || n == nullptr || cap < 0 || (cap > 0 && pages == nullptr)) return fail(UF_ERR_ARG, "null argument");
  if (seq < 0 || seq >= c->d.max_seqs) return fail(UF_ERR_ARG, "%d is no sequence (0 .. %d)", seq, c->d.max_seqs - 1);
  const std::vector<int32_t>& p = c->seqs[size_t(seq)].pages;
  *n = int32_t(p.size());
  std::copy_n(p.begin(), std::min(p.size(), size_t(cap)), pages);
  return ok();
}

}  // extern "C"

namespace {

constexpr double kMostGroups = 16777215.0;   // workgroups of a launch: 2^32 - 1 threads

// One launch over the sequences of a step whose rows number least .. most.
struct Launch {
  bool run = false;
  int32_t least = 0, most = 0, longest = 0, tiles = 0, packed = 0, slice = 0, n_split = 1;
  size_t work_rows = 0;
};

// How a launch's time goes with its workgroups, in units of keys.  Measured (us, attention
// alone): 16 sequences x 8 heads x 2 tiles of 65 units, whole 95, in two slices 89, in three
// 103; 4 heads x 1 tile of 33 units, whole 44, slices of 5 units 15.7, of 2 14.6; few rows: one
// sequence of 4,096 units and 8 heads, in 4 slices 410, 8 217, 16 120, 32 100, 48 115, 64 104;
// 384 of 129 units, whole 154, in two slices 150, in four 159.
struct Cost {
  int64_t slots;      // workgroups that run side by side
  int32_t least;      // units of a slice at least
  double alone;       // time of a unit where a compute unit has one workgroup, of its time where it has all it holds
  double fixed;       // a workgroup's loads of queries, tables and its stores
  double join;        // the joining launch
  double partial;     // a slice's partial results, written and read, per slice
};

// Slices: the launch takes rounds of `slots` workgroups, each as long as a slice and
// its fixed cost; split launches add the joining launch and their partial results.
void choose_slices(const std::vector<int32_t>& counts, int32_t heads, int64_t n_cu, const Cost& cost, Launch* l) {
  int32_t most = 1;
  for (int32_t u : counts) most = std::max(most, u);
  l->slice = most;
  l->n_split = 1;
  if (n_cu <= 0 || int64_t(counts.size()) * heads >= 8 * cost.slots) return;
  static const int32_t kTry[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64};
  double best = 1e300;
  for (int32_t m : kTry) {
    const int32_t slice = (most + m - 1) / m;
    if (m > 1 && slice < cost.least) break;
    int64_t groups = 0;
    for (int32_t u : counts) groups += (u + slice - 1) / slice;
    groups *= heads;
    const double rounds = groups <= n_cu ? cost.alone : double((groups + cost.slots - 1) / cost.slots);
    const double time = rounds * (slice + cost.fixed) + (m > 1 ? cost.join + cost.partial * double(groups) : 0.0);
    if (time < best) {
      best = time;
      l->slice = slice;
      l->n_split = (most + slice - 1) / slice;
    }
  }
}

struct Plan {
  Launch few, rows;
  size_t bytes = 0;
};

int plan_attn(const uft_cache* c, const uft_attn_desc* d, Plan* p) {
  if (c == nullptr) return fail(UF_ERR_ARG, "handle is null");
  if (d == nullptr) return fail(UF_ERR_ARG, "desc is null");
  if (d->q_heads < 1 || d->q_heads % c->d.kv_heads != 0)
    return fail(UF_ERR_ARG, "q_heads %d must be a multiple of kv_heads %d", d->q_heads, c->d.kv_heads);
  if (d->q_heads > 65536) return fail(UF_ERR_ARG, "q_heads must be at most 65536");
  if (d->window < 0 || d->sinks < 0) return fail(UF_ERR_ARG, "window and sinks must be >= 0");
  if (d->n_cu < 0 || d->n_cu > 65536) return fail(UF_ERR_ARG, "n_cu must be in [0, 65536]");
  if (c->step.empty()) return fail(UF_ERR_EMPTY, "no step: uft_extend first");
  const int32_t H = c->d.kv_heads, G = d->q_heads / H, n = int32_t(c->step.size());
  const int32_t sinks = std::min(d->sinks, c->d.max_tokens);
  std::vector<int32_t> few, rows;
  int64_t tiles = 0, all_tiles = 0;
  int64_t few_rows = 0, many_rows = 0;
  for (const Entry& e : c->step) {
    const int64_t r = int64_t(e.count) * G;
    if (r == 0) continue;
    const int32_t first = e.tokens - e.count;
    (r <= tok::kFewRows ? few_rows : many_rows) = std::max(r <= tok::kFewRows ? few_rows : many_rows, r);
    if (r <= tok::kFewRows) {
      few.push_back(tok::key_range(first, e.tokens - 1, d->window, sinks, tok::kFewUnit).count);
      continue;
    }
    const int64_t t = (r + tok::kRowTile - 1) / tok::kRowTile;
    tiles = std::max(tiles, t);
    all_tiles += t;
    for (int64_t k = 0; k < t && rows.size() < size_t(8) * 65536; ++k) {
      const int32_t a = int32_t(k * tok::kRowTile / G);
      const int32_t b = int32_t(std::min(r, (k + 1) * tok::kRowTile) - 1) / G;
      rows.push_back(tok::key_range(first + a, first + b, d->window, sinks, tok::kKeyUnit).count);
      if (int64_t(rows.size()) * H >= int64_t(16) * d->n_cu) {   // enough without slices: see choose_slices
        rows.resize(size_t(16) * d->n_cu + 1, rows.back());
        break;
      }
    }
  }
  if (!few.empty()) {
    p->few.run = true;
    p->few.least = 1;
    p->few.most = tok::kFewRows;
    p->few.longest = int32_t(few_rows);
    p->few.tiles = 1;
    choose_slices(few, H, d->n_cu, Cost{d->n_cu, 4, 1.0, 6.0, 8.0, 0.004}, &p->few);
    p->few.packed = deal_packed(n, int64_t(few.size()));
  }
  if (!rows.empty()) {
    p->rows.run = true;
    p->rows.least = tok::kFewRows + 1;
    p->rows.most = INT32_MAX;
    p->rows.longest = int32_t(many_rows);
    p->rows.tiles = int32_t(tiles);
    choose_slices(rows, H, d->n_cu, Cost{int64_t(2) * d->n_cu, 2, 0.72, 4.0, 2.0, 0.014}, &p->rows);
    p->rows.packed = deal_packed(n * tiles, all_tiles);
  }
  for (Launch* l : {&p->few, &p->rows}) {
    const int32_t rows = l == &p->few ? tok::kFewRows : tok::kRowTile;
    const double groups = (l->packed > 0 ? double(l->packed) : double(n) * l->tiles) * H * l->n_split;
    // (a join takes a workgroup per four rows at least)
    if (groups > kMostGroups || (l->n_split > 1 && groups / l->n_split * (rows / 4) > kMostGroups) || double(many_rows) > 2.0e9)
      return fail(UF_ERR_ARG, "step too large for one launch");
    if (l->n_split > 1) l->work_rows = size_t(groups) * size_t(rows);
  }
  p->bytes = (p->few.work_rows + p->rows.work_rows) * (tok::kD + 2) * 4;
  return UF_OK;
}

}  // namespace

extern "C" {

int uft_attn_work_bytes(const uft_cache* c, const uft_attn_desc* desc, size_t* bytes) {
  return guarded([&]() -> int {
    if (bytes == nullptr) return fail(UF_ERR_ARG, "bytes is null");
    Plan p;
    if (int s = plan_attn(c, desc, &p)) return s;
    *bytes = p.bytes;
    return ok();
  });
}

int uft_attn(const uft_cache* c, int32_t layer, const uft_attn_desc* d, const void* d_q, const int64_t* d_tree, void* d_o,
             float* d_lse, void* d_work, size_t work_bytes, void* stream) {
  return guarded([&]() -> int {
    Plan p;
    if (int s = plan_attn(c, d, &p)) return s;
    if (layer < 0 || layer >= c->d.layers) return fail(UF_ERR_ARG, "layer %d of %d", layer, c->d.layers);
    if (int s = check_stride(&d->q, "q stride")) return s;
    tok::AttnArgs a{};
    if (int s = check_scale(d->scale, &a.scale_log2)) return s;
    if (d_tree != nullptr) {
      if (c->step_longest > tok::kMaxTree)
        return fail(UF_ERR_UNSUPPORTED, "a tree of %d nodes, at most %d", c->step_longest, tok::kMaxTree);
      if (d->window > 0 && d->window < c->step_longest)
        return fail(UF_ERR_ARG, "window %d is smaller than a tree of %d nodes", d->window, c->step_longest);
      if (!aligned(d_tree, 8)) return fail(UF_ERR_ARG, "tree must be 8-byte aligned");
    }
    if (c->dry() || c->step_tokens == 0) return ok();
    if (d_q == nullptr || d_o == nullptr) return fail(UF_ERR_ARG, "q or o is null");
    if (!aligned(d_q, 16) || !aligned(d_o, 16)) return fail(UF_ERR_ARG, "q and o must be 16-byte aligned");
    if (!aligned(d_lse, 4)) return fail(UF_ERR_ARG, "lse must be 4-byte aligned");
    if (p.bytes > 0) {
      if (d_work == nullptr || !aligned(d_work, 16)) return fail(UF_ERR_ARG, "work must be 16-byte aligned and not null");
      if (work_bytes < p.bytes) return fail(UF_ERR_ARG, "work has %zu bytes, the call needs %zu", work_bytes, p.bytes);
    }
    a.q = static_cast<const uint16_t*>(d_q);
    a.q_token = d->q.token;
    a.q_head = d->q.head;
    a.o = static_cast<uint16_t*>(d_o);
    a.lse = d_lse;
    a.tree = d_tree;
    a.pool = c->pool_of(layer);
    a.step = c->table;
    a.table = c->table + c->rows_at();
    a.row = c->row;
    a.n = int32_t(c->step.size());
    a.total = c->step_tokens;
    a.q_heads = d->q_heads;
    a.kv_heads = c->d.kv_heads;
    a.group = d->q_heads / c->d.kv_heads;
    a.window = d->window;
    a.sinks = std::min(d->sinks, c->d.max_tokens);
    a.work = static_cast<float*>(d_work);
    hipStream_t st = static_cast<hipStream_t>(stream);
    for (const Launch* l : {&p.few, &p.rows}) {
      if (!l->run) continue;
      a.least_rows = l->least;
      a.most_rows = l->most;
      a.longest_rows = l->longest;
      a.tiles = l->tiles;
      a.packed = l->packed;
      a.slice = l->slice;
      a.n_split = l->n_split;
      const hipError_t e = l == &p.few ? tok::launch_attn_few(a, st) : tok::launch_attn_rows(a, true, st);
      if (int s = check_hip(e, "attention")) return s;
      if (a.work != nullptr) a.work += l->work_rows * (tok::kD + 2);
    }
    return ok();
  });
}

}  // extern "C"

namespace {

int check_window(const uft_window_desc* d, float* log2) {
  if (d == nullptr) return fail(UF_ERR_ARG, "desc is null");
  if (d->batch < 1 || d->tokens < 1 || d->q_heads < 1 || d->kv_heads < 1)
    return fail(UF_ERR_ARG, "batch, tokens and heads must be >= 1");
  if (d->head_dim != tok::kD) return fail(UF_ERR_UNSUPPORTED, "head_dim %d: only 128 is built", d->head_dim);
  if (d->q_heads % d->kv_heads != 0)
    return fail(UF_ERR_ARG, "q_heads %d must be a multiple of kv_heads %d", d->q_heads, d->kv_heads);
  if (d->q_heads > 65536) return fail(UF_ERR_ARG, "q_heads must be at most 65536");
  if (d->tokens > (1 << 30)) return fail(UF_ERR_ARG, "tokens must be at most 2^30");
  if (d->window < 0 || d->sinks < 0) return fail(UF_ERR_ARG, "window and sinks must be >= 0");
  const double group = d->q_heads / d->kv_heads;
  if (double(d->batch) * d->kv_heads * (std::ceil(d->tokens * group / 128.0) + 2.0) > kMostGroups ||
      d->tokens * group > 2.0e9)
    return fail(UF_ERR_ARG, "shape too large: batch * q_heads * tokens");
  if (int s = check_stride(&d->q, "q stride")) return s;
  if (int s = check_stride(&d->k, "k stride")) return s;
  if (int s = check_stride(&d->v, "v stride")) return s;
  // the backward's offsets of a group's heads are 32-bit
  if (d->q.head * (d->q_heads / d->kv_heads) > (int64_t(1) << 30))
    return fail(UF_ERR_ARG, "the q stride's head times the query heads of a key head must be at most 2^30");
  if (int s = check_scale(d->scale, log2)) return s;
  // the backward seeds its products with LSE / scale
  if (d->scale < 0x1p-100f) return fail(UF_ERR_ARG, "scale must be at least 2^-100");
  return UF_OK;
}

tok::BwdArgs bwd_args(const uft_window_desc* d, float log2) {
  tok::BwdArgs a{};
  a.q_batch = d->q.batch, a.q_token = d->q.token, a.q_head = d->q.head;
  a.k_batch = d->k.batch, a.k_token = d->k.token, a.k_head = d->k.head;
  a.v_batch = d->v.batch, a.v_token = d->v.token, a.v_head = d->v.head;
  a.batch = d->batch;
  a.tokens = d->tokens;
  a.q_heads = d->q_heads;
  a.kv_heads = d->kv_heads;
  a.group = d->q_heads / d->kv_heads;
  a.group_div = ~uint64_t(0) / uint64_t(a.group);
  a.window = d->window;
  a.sinks = std::min(d->sinks, d->tokens);
  a.tiles = int32_t((int64_t(d->tokens) * a.group + 127) / 128);
  a.scale = d->scale;
  a.scale_log2 = log2;
  return a;
}

}  // namespace

extern "C" {

int uft_window_fwd(const uft_window_desc* d, const void* d_q, const void* d_k, const void* d_v, const int32_t* d_lengths,
                   void* d_o, float* d_lse, void* stream) {
  return guarded([&]() -> int {
    tok::AttnArgs a{};
    if (int s = check_window(d, &a.scale_log2)) return s;
    if (d_q == nullptr || d_k == nullptr || d_v == nullptr || d_o == nullptr) return fail(UF_ERR_ARG, "q, k, v or o is null");
    if (!aligned(d_q, 16) || !aligned(d_k, 16) || !aligned(d_v, 16) || !aligned(d_o, 16))
      return fail(UF_ERR_ARG, "q, k, v and o must be 16-byte aligned");
    if (!aligned(d_lse, 4) || !aligned(d_lengths, 4)) return fail(UF_ERR_ARG, "lse and lengths must be 4-byte aligned");
    a.q = static_cast<const uint16_t*>(d_q);
    a.k = static_cast<const uint16_t*>(d_k);
    a.v = static_cast<const uint16_t*>(d_v);
    a.o = static_cast<uint16_t*>(d_o);
    a.lse = d_lse;
    a.lengths = d_lengths;
    a.q_batch = d->q.batch, a.q_token = d->q.token, a.q_head = d->q.head;
    a.k_batch = d->k.batch, a.k_token = d->k.token, a.k_head = d->k.head;
    a.v_batch = d->v.batch, a.v_token = d->v.token, a.v_head = d->v.head;
    a.tokens = d->tokens;
    a.n = d->batch;
    a.q_heads = d->q_heads;
    a.kv_heads = d->kv_heads;
    a.group = d->q_heads / d->kv_heads;
    a.window = d->window;
    a.sinks = std::min(d->sinks, d->tokens);
    a.tiles = int32_t((int64_t(d->tokens) * a.group + tok::kRowTile - 1) / tok::kRowTile);
    a.least_rows = 0;
    a.most_rows = INT_MAX;
    a.n_split = 1;
    a.slice = INT_MAX;
    if (int s = check_hip(tok::launch_attn_rows(a, false, static_cast<hipStream_t>(stream)), "attention")) return s;
    return ok();
  });
}

int uft_window_bwd_work_bytes(const uft_window_desc* d, size_t* bytes) {
  return guarded([&]() -> int {
    float log2 = 0.f;
    if (int s = check_window(d, &log2)) return s;
    if (bytes == nullptr) return fail(UF_ERR_ARG, "bytes is null");
    *bytes = tok::bwd_work_bytes(bwd_args(d, log2));
    return ok();
  });
}

int uft_window_bwd(const uft_window_desc* d, const void* d_q, const void* d_k, const void* d_v, const void* d_o,
                   const float* d_lse, const void* d_do, const int32_t* d_lengths, void* d_dq, void* d_dk, void* d_dv,
                   void* d_work, size_t work_bytes, void* stream) {
  return guarded([&]() -> int {
    float log2 = 0.f;
    if (int s = check_window(d, &log2)) return s;
    for (const void* p : {d_q, d_k, d_v, d_o, d_do, static_cast<const void*>(d_dq), static_cast<const void*>(d_dk),
                          static_cast<const void*>(d_dv), static_cast<const void*>(d_work)}) {
      if (p == nullptr) return fail(UF_ERR_ARG, "a tensor or the workspace is null");
      if (!aligned(p, 16)) return fail(UF_ERR_ARG, "tensors and the workspace must be 16-byte aligned");
    }
    if (d_lse == nullptr) return fail(UF_ERR_ARG, "lse is null");
    if (!aligned(d_lse, 4) || !aligned(d_lengths, 4)) return fail(UF_ERR_ARG, "lse and lengths must be 4-byte aligned");
    tok::BwdArgs a = bwd_args(d, log2);
    const size_t need = tok::bwd_work_bytes(a);
    if (work_bytes < need) return fail(UF_ERR_ARG, "work has %zu bytes, the call needs %zu", work_bytes, need);
    a.q = static_cast<const uint16_t*>(d_q);
    a.k = static_cast<const uint16_t*>(d_k);
    a.v = static_cast<const uint16_t*>(d_v);
    a.o = static_cast<const uint16_t*>(d_o);
    a.dout = static_cast<const uint16_t*>(d_do);
    a.lse = d_lse;
    a.lengths = d_lengths;
    a.dq = static_cast<uint16_t*>(d_dq);
    a.dk = static_cast<uint16_t*>(d_dk);
    a.dv = static_cast<uint16_t*>(d_dv);
    a.work = static_cast<uint8_t*>(d_work);
    if (int s = check_hip(tok::launch_window_bwd(a, static_cast<hipStream_t>(stream)), "attention backward")) return s;
    return ok();
  });
}

}  // extern "C"
