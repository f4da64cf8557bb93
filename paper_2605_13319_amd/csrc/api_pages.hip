// Host side of the paged cache of operators: the handle, its bookkeeping, the passes.
#include <algorithm>
#include <new>
#include <vector>

#include "pages.h"
#include "rows.h"
#include "status.h"

using namespace pipesd;

namespace {
struct PagesSeq {
  int32_t len = 0;
  std::vector<int32_t> blocks;  // in token order
  std::vector<int32_t> sent;    // what the device has in the client's block table; -1: not known (all of them, where a launch failed)
  bool in_pass = false;         // of the pass that append and attend work on
};
template <class F>
int guarded(F f) {  // nothing throws over the boundary
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return PIPESD_ENOMEM;
  } catch (...) {
    return PIPESD_EINVAL;
  }
}
}  // namespace

struct pipesd_pages {
  pipesd_config cfg{};
  int32_t max_seqs = 0, n_blocks = 0;
  void* pool = nullptr;
  std::vector<int32_t> free_list;
  std::vector<int32_t> users;  // of a block: clients that hold it
  std::vector<PagesSeq> seqs;
  int n_cu = 256;
  // device memory of the library
  int32_t* table = nullptr;  // [max_seqs][n_blocks]
  float* part = nullptr;
  size_t part_cap = 0;  // floats
  unsigned* counters = nullptr;
  size_t counters_cap = 0;
  uint32_t* masks = nullptr;
  size_t masks_cap = 0;  // words
  std::vector<void*> old;  // buffers that have grown since
  // the pass
  std::vector<PagesClient> pass, next_pass;  // (next_..: where the next pass is made)
  std::vector<PagesLaunch> launches, next_launches;
  std::vector<int32_t> had, own, from, to;   // (a call's own)
  bool pass_open = false, attends = false, trees = false;
  bool rows_shared = false;  // a client outside the pass has become a copy, in the same blocks, of some of the pass's rows

  int32_t table_off(int32_t seq) const { return seq * n_blocks; }
  KvView view() const {
    KvView v;
    v.pool = pool;
    v.table = table;
    v.block_elems = cfg.n_kv_heads * kBlockTokens * cfg.head_dim;
    v.v_offset = (int64_t)n_blocks * v.block_elems;
    v.layer_stride = 2 * v.v_offset;
    v.n_kv_heads = cfg.n_kv_heads;
    v.head_dim = cfg.head_dim;
    return v;
  }
  int32_t take() {  // (the caller knows that there is one)
    const int32_t b = free_list.back();
    free_list.pop_back();
    users[b] = 1;
    return b;
  }
  void drop(int32_t b) {
    if (--users[b] == 0) free_list.push_back(b);  // (has room for every block)
  }
};

static int32_t pages_blocks(int32_t tokens) { return tokens / kBlockTokens + (tokens % kBlockTokens != 0); }
static bool pages_seq_ok(const pipesd_pages* pg, int32_t seq) { return pg && seq >= 0 && seq < pg->max_seqs; }
// every id in range, none twice
static bool pages_seqs_ok(const pipesd_pages* pg, int32_t n, const int32_t* ids) {
  bool rising = true;  // (as ids mostly are)
  for (int32_t i = 0; i < n; ++i) {
    if (!pages_seq_ok(pg, ids[i])) return false;
    rising = rising && (i == 0 || ids[i] > ids[i - 1]);
  }
  if (rising) return true;
  std::vector<char> seen(pg->max_seqs, 0);
  for (int32_t i = 0; i < n; ++i)
    if (seen[ids[i]]++) return false;
  return true;
}
static void pages_release(pipesd_pages* pg, PagesSeq& s, int32_t tokens) {
  const int32_t keep = pages_blocks(tokens);
  while ((int32_t)s.blocks.size() > keep) {
    pg->drop(s.blocks.back());
    s.blocks.pop_back();
  }
  s.len = tokens;
}
static void pages_close_pass(pipesd_pages* pg) {
  for (PagesSeq& s : pg->seqs) s.in_pass = false;
  pg->pass_open = false;
}

static bool pages_config_ok(const pipesd_config* c) {
  return c->n_layers >= 1 && c->n_kv_heads >= 1 && c->n_q_heads >= 1 && c->n_q_heads % c->n_kv_heads == 0 &&
         (c->head_dim == 64 || c->head_dim == 128) && (c->dtype == PIPESD_F32 || c->dtype == PIPESD_BF16) && c->n_kv_heads <= 65535 &&
         c->n_layers <= 65535 && c->n_q_heads / c->n_kv_heads <= 256;
}

extern "C" size_t pipesd_pages_block_bytes(const pipesd_config* cfg, int32_t block_tokens) {
  if (!cfg || block_tokens != kBlockTokens || !pages_config_ok(cfg)) return 0;
  return (size_t)cfg->n_layers * 2 * cfg->n_kv_heads * cfg->head_dim * kBlockTokens * (cfg->dtype == PIPESD_F32 ? 4 : 2);
}

// Grows a buffer of the pass.  The old one stays until the handle ends: the device may still be using it, and recorded calls hold its
// address (half as much again each time: all old ones together are less than twice the last).
template <class T>
static int pages_grow(pipesd_pages* pg, T** p, size_t* cap, size_t want, bool zero, size_t spare) {
  if (want <= *cap) return PIPESD_OK;
  want += spare;
  pg->old.reserve(pg->old.size() + 1);
  T* fresh = nullptr;
  if (hipMalloc((void**)&fresh, want * sizeof(T)) != hipSuccess) {
    (void)hipGetLastError();
    return PIPESD_ENOMEM;
  }
  hipError_t e = zero ? hipMemset(fresh, 0, want * sizeof(T)) : hipSuccess;
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    (void)hipFree(fresh);
    return hip_fail(e, "growing a buffer of the paged cache");
  }
  if (*p) pg->old.push_back(*p);
  *p = fresh;
  *cap = want;
  return PIPESD_OK;
}

extern "C" int pipesd_pages_destroy(pipesd_pages* pg) {
  if (!pg) return PIPESD_EINVAL;
  if (pg->pool) {
    (void)hipDeviceSynchronize();
    for (void* p : {(void*)pg->table, (void*)pg->part, (void*)pg->counters, (void*)pg->masks})
      if (p) (void)hipFree(p);
    for (void* p : pg->old) (void)hipFree(p);
  }
  delete pg;
  return PIPESD_OK;
}

extern "C" int pipesd_pages_create(const pipesd_config* cfg, int32_t max_seqs, int32_t block_tokens, void* pool, size_t pool_bytes,
                                   pipesd_pages** out) {
  if (!cfg || !out || max_seqs < 1 || !pages_config_ok(cfg)) return PIPESD_EINVAL;
  const size_t bb = pipesd_pages_block_bytes(cfg, block_tokens);
  if (bb == 0) return PIPESD_EINVAL;
  const size_t n = pool_bytes / bb;
  // tokens, slots of the block tables, elements of a block: 32-bit numbers
  if (n < 1 || n > (size_t)INT32_MAX / kBlockTokens || (uint64_t)max_seqs * n > (uint64_t)INT32_MAX) return PIPESD_EINVAL;
  if ((int64_t)cfg->n_kv_heads * kBlockTokens * cfg->head_dim > INT32_MAX) return PIPESD_EINVAL;
  if (pool && ((uintptr_t)pool & 255)) return PIPESD_EINVAL;
  pipesd_pages* pg = new (std::nothrow) pipesd_pages();
  if (!pg) return PIPESD_ENOMEM;
  int rc = guarded([&]() -> int {
    pg->cfg = *cfg;
    pg->max_seqs = max_seqs;
    pg->n_blocks = (int32_t)n;
    pg->seqs.resize(max_seqs);
    pg->users.assign(n, 0);
    pg->free_list.reserve(n);
    for (int32_t b = pg->n_blocks - 1; b >= 0; --b) pg->free_list.push_back(b);  // block 0 is handed out first
    if (!pool) return PIPESD_OK;
    pg->pool = pool;
    pg->n_cu = device_cu_count();
    if (pg->n_cu <= 0) return PIPESD_EHIP;
    const size_t entries = (size_t)max_seqs * n;
    if (hipMalloc((void**)&pg->table, entries * 4) != hipSuccess) {
      (void)hipGetLastError();
      return PIPESD_ENOMEM;
    }
    HIP_TRY(hipMemset(pg->table, 0, entries * 4));
    const int32_t clients = std::min(max_seqs, 16);
    const PagesNeeds most = pages_plan_most(clients, kPagesUsualRows, (int64_t)pg->n_blocks * kBlockTokens, cfg->dtype, cfg->head_dim, cfg->n_q_heads,
                                            cfg->n_kv_heads, pg->n_cu);
    int e;
    if ((e = pages_grow(pg, &pg->part, &pg->part_cap, most.part_tiles * 16 * (cfg->head_dim + kPagesPartPad), false, 0))) return e;
    if ((e = pages_grow(pg, &pg->counters, &pg->counters_cap, most.counters, true, 0))) return e;
    return pages_grow(pg, &pg->masks, &pg->masks_cap, (size_t)clients * kPagesUsualRows * kPagesMaskWords, false, 0);
  });
  if (rc) {
    pipesd_pages_destroy(pg);
    return rc;
  }
  *out = pg;
  return PIPESD_OK;
}

extern "C" int pipesd_pages_len(const pipesd_pages* pg, int32_t seq, int32_t* len) {
  if (!pages_seq_ok(pg, seq) || !len) return PIPESD_EINVAL;
  *len = pg->seqs[seq].len;
  return PIPESD_OK;
}
extern "C" int pipesd_pages_free_blocks(const pipesd_pages* pg, int32_t* n_free) {
  if (!pg || !n_free) return PIPESD_EINVAL;
  *n_free = (int32_t)pg->free_list.size();
  return PIPESD_OK;
}
extern "C" int pipesd_pages_seq_blocks(const pipesd_pages* pg, int32_t seq, int32_t* n_blocks) {
  if (!pages_seq_ok(pg, seq) || !n_blocks) return PIPESD_EINVAL;
  *n_blocks = (int32_t)pg->seqs[seq].blocks.size();
  return PIPESD_OK;
}

extern "C" int pipesd_pages_truncate(pipesd_pages* pg, int32_t n_seqs, const int32_t* seq_ids, const int32_t* new_len) {
  if (!pg || n_seqs < 1 || !seq_ids || !new_len) return PIPESD_EINVAL;
  return guarded([&]() -> int {
    if (!pages_seqs_ok(pg, n_seqs, seq_ids)) return PIPESD_EINVAL;
    for (int32_t i = 0; i < n_seqs; ++i)
      if (new_len[i] < 0 || new_len[i] > pg->seqs[seq_ids[i]].len) return PIPESD_ESTATE;
    bool touched = false;
    for (int32_t i = n_seqs - 1; i >= 0; --i) {  // (backwards: who asks for as much again, in the same order, gets the same blocks)
      PagesSeq& s = pg->seqs[seq_ids[i]];
      touched |= s.in_pass && new_len[i] < s.len;
      pages_release(pg, s, new_len[i]);
    }
    if (touched) pages_close_pass(pg);
    return PIPESD_OK;
  });
}

// What writes block tables, trees or tokens that the host says where they are is not recorded: a replay would do it again, when the
// blocks may be another client's, and until the first replay the device has not what the host takes it to have.
static int pages_not_recorded(hipStream_t st) {
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  HIP_TRY(hipStreamIsCapturing(st, &status));
  return status == hipStreamCaptureStatusNone ? PIPESD_OK : PIPESD_ESTATE;
}

// whether the device lacks entries of a client's block table, from one on
static bool pages_unsent(const PagesSeq& s, int32_t from) {
  if (s.sent.size() < s.blocks.size()) return true;
  if (!s.blocks.empty() && s.sent[0] < 0) return true;
  return !std::equal(s.blocks.begin() + from, s.blocks.end(), s.sent.begin() + from);
}

// Sends what is new of the block tables, the blocks to copy (pg->from, pg->to) and the trees of a pass (parents of all rows, or nullptr),
// some per launch.  (A block that a client gave back and got again is there already.)
static int pages_send(pipesd_pages* pg, int32_t n, const int32_t* seq_ids, const int32_t* from, bool own, const std::vector<PagesClient>& trees,
                      const int32_t* parents, hipStream_t st) {
  PagesBegin b;
  b.n = b.trees = b.own = 0;
  int32_t rows = 0;
  auto flush = [&]() -> int {
    if (b.n == 0 && b.trees == 0 && b.own == 0) return PIPESD_OK;
    HIP_TRY(launch_pages_begin(pg->cfg.dtype, pg->view(), pg->cfg.n_layers, b, pg->table, pg->masks, st));
    b.n = b.trees = b.own = rows = 0;
    return PIPESD_OK;
  };
  auto all = [&]() -> int {
    for (size_t i = 0; own && i < pg->from.size(); ++i) {
      if (b.own == kPagesOwnPerLaunch)
        if (int rc = flush()) return rc;
      b.own_from[b.own] = pg->from[i];
      b.own_to[b.own++] = pg->to[i];
    }
    for (int32_t k = 0; k < n; ++k) {
      PagesSeq& s = pg->seqs[seq_ids[k]];
      const int32_t off = pg->table_off(seq_ids[k]), nb = (int32_t)s.blocks.size();
      if ((int32_t)s.sent.size() < nb) s.sent.resize(nb, -1);
      for (int32_t i = from && nb > 0 && s.sent[0] >= 0 ? from[k] : 0; i < nb; ++i) {
        if (s.sent[i] == s.blocks[i]) continue;
        if (b.n == kPagesEntriesPerLaunch)
          if (int rc = flush()) return rc;
        b.at[b.n] = off + i;
        b.v[b.n++] = s.sent[i] = s.blocks[i];
      }
    }
    for (size_t i = 0; parents && i < trees.size(); ++i) {
      const PagesClient& c = trees[i];
      if (b.trees == kPagesPerLaunch || rows + c.n_rows > kPagesParentsPerLaunch)
        if (int rc = flush()) return rc;
      b.row_off[b.trees] = c.row_off;
      b.n_rows[b.trees] = c.n_rows;
      b.before[b.trees++] = c.len - c.n_rows;
      for (int32_t r = 0; r < c.n_rows; ++r) b.parent[rows++] = (int16_t)parents[c.row_off + r];
    }
    return flush();
  };
  const int rc = all();
  for (int32_t k = 0; rc && k < n; ++k) std::fill(pg->seqs[seq_ids[k]].sent.begin(), pg->seqs[seq_ids[k]].sent.end(), -1);
  return rc;
}

// What is left of a call whose launches failed, or were said to have (an error from before is the next launch's): clients whose bookkeeping
// is as it was get their block tables as they were, and a pass whose trees the device may have lost is over.
static void pages_take_back(pipesd_pages* pg, int32_t n, const int32_t* seq_ids, hipStream_t st) {
  pages_close_pass(pg);
  (void)pages_send(pg, n, seq_ids, nullptr, false, {}, nullptr, st);
}

// tokens (block * 16 + place) or blocks from pg->from to pg->to, some per launch
static int pages_moves(pipesd_pages* pg, bool blocks, hipStream_t st) {
  PagesMoves m;
  for (size_t i0 = 0; i0 < pg->from.size(); i0 += kPagesMovesPerLaunch) {
    m.n = (int32_t)std::min<size_t>(pg->from.size() - i0, kPagesMovesPerLaunch);
    std::copy_n(pg->from.begin() + i0, m.n, m.from);
    std::copy_n(pg->to.begin() + i0, m.n, m.to);
    HIP_TRY(blocks ? launch_pages_copy(pg->cfg.dtype, pg->view(), pg->cfg.n_layers, m, st) : launch_pages_move(pg->cfg.dtype, pg->view(), pg->cfg.n_layers, m, st));
  }
  return PIPESD_OK;
}

extern "C" int pipesd_pages_extend(pipesd_pages* pg, int32_t n_seqs, const int32_t* seq_ids, const int32_t* n_new, const int32_t* parents,
                                   void* stream) {
  if (!pg || n_seqs < 1 || n_seqs > PIPESD_PAGES_MAX_PASS_SEQS || !seq_ids || !n_new) return PIPESD_EINVAL;
  return guarded([&]() -> int {
    hipStream_t st = (hipStream_t)stream;
    if (!pages_seqs_ok(pg, n_seqs, seq_ids)) return PIPESD_EINVAL;
    const pipesd_config& cfg = pg->cfg;
    int64_t total = 0, blocks = 0;
    bool attends = true, chain = true;
    for (int32_t i = 0; i < n_seqs; ++i) {
      const PagesSeq& s = pg->seqs[seq_ids[i]];
      const int32_t n = n_new[i];
      if (n < 0 || n > (int32_t)(INT32_MAX / 2) - s.len || (parents && n > kPagesTreeRows) || total + n > INT32_MAX) return PIPESD_EINVAL;
      for (int32_t r = 0; parents && r < n; ++r) {
        const int32_t p = parents[total + r];
        if (p < -1 || p >= r) return PIPESD_EINVAL;
        chain = chain && p == r - 1;
      }
      total += n;
      blocks += pages_blocks(s.len + n) - (int32_t)s.blocks.size();
      attends = attends && n <= kPagesMaxRows;
    }
    if (total < 1) return PIPESD_EINVAL;
    const bool trees = parents && !chain;
    // A client whose last block has other users gets one of its own, unless all the others do: who comes last keeps it.
    std::vector<int32_t>&had = pg->had, &own = pg->own;
    had.resize(n_seqs);
    own.assign(n_seqs, -1);  // the block that is shared
    bool any_own = false;
    for (int32_t i = 0; i < n_seqs; ++i) {
      const PagesSeq& s = pg->seqs[seq_ids[i]];
      had[i] = (int32_t)s.blocks.size();
      if (n_new[i] == 0 || s.len % kBlockTokens == 0 || pg->users[s.blocks.back()] == 1) continue;
      own[i] = s.blocks.back();
      --pg->users[own[i]];
      any_own = true;
      ++blocks;
    }
    auto undo_own = [&] {
      for (int32_t i = 0; i < n_seqs; ++i)
        if (own[i] >= 0) ++pg->users[own[i]];
    };
    if (blocks > (int64_t)pg->free_list.size()) {
      undo_own();
      return PIPESD_ENOMEM;
    }

    std::vector<PagesClient>& plan = pg->next_pass;
    std::vector<PagesLaunch>& launches = pg->next_launches;
    auto prepare = [&]() -> int {
      plan.clear();
      launches.clear();
      plan.reserve(n_seqs);
      pg->from.clear();
      pg->to.clear();
      pg->from.reserve(n_seqs);
      pg->to.reserve(n_seqs);
      int32_t row = 0;
      for (int32_t i = 0; i < n_seqs; ++i) {
        PagesSeq& s = pg->seqs[seq_ids[i]];
        if (n_new[i]) plan.push_back(PagesClient{seq_ids[i], n_new[i], row, s.len + n_new[i], pg->table_off(seq_ids[i])});
        row += n_new[i];
        s.blocks.reserve(pages_blocks(s.len + n_new[i]));
        s.sent.reserve(pages_blocks(s.len + n_new[i]));
      }
      if (!pg->pool) return PIPESD_OK;
      PagesNeeds need{0, 0};
      if (attends) need = pages_plan(plan.data(), (int)plan.size(), cfg.dtype, cfg.head_dim, cfg.n_q_heads, cfg.n_kv_heads, pg->n_cu, launches);
      if (need.part_tiles > (size_t)INT32_MAX || need.counters > (size_t)INT32_MAX) return PIPESD_ENOMEM;
      const size_t parts = need.part_tiles * 16 * (cfg.head_dim + kPagesPartPad), words = trees ? (size_t)total * kPagesMaskWords : 0;
      int e;
      if (any_own || trees || parts > pg->part_cap || need.counters > pg->counters_cap)
        if ((e = pages_not_recorded(st))) return e;
      if ((e = pages_grow(pg, &pg->part, &pg->part_cap, parts, false, parts / 2))) return e;
      if ((e = pages_grow(pg, &pg->counters, &pg->counters_cap, need.counters, true, need.counters / 2))) return e;
      return pages_grow(pg, &pg->masks, &pg->masks_cap, words, false, words / 2);
    };
    int rc = PIPESD_ENOMEM;
    try {
      rc = prepare();
    } catch (const std::bad_alloc&) {
    }
    if (rc) {
      undo_own();
      return rc;
    }

    // from here on only the launches can fail: what they have not done is taken back
    for (int32_t i = 0; i < n_seqs; ++i) {
      PagesSeq& s = pg->seqs[seq_ids[i]];
      if (own[i] >= 0) {
        s.blocks.back() = pg->take();
        pg->from.push_back(own[i]);
        pg->to.push_back(s.blocks.back());
        --had[i];  // (blocks that stay as they were)
      }
      s.len += n_new[i];
      while ((int32_t)s.blocks.size() < pages_blocks(s.len)) s.blocks.push_back(pg->take());
    }
    auto launch = [&]() -> int {
      bool unsent = false;
      for (int32_t i = 0; i < n_seqs; ++i) unsent = unsent || pages_unsent(pg->seqs[seq_ids[i]], had[i]);
      if (unsent)
        if (int e = pages_not_recorded(st)) return e;
      return pages_send(pg, n_seqs, seq_ids, had.data(), true, plan, trees ? parents : nullptr, st);
    };
    if (pg->pool && (rc = launch())) {
      for (int32_t i = n_seqs - 1; i >= 0; --i) {  // (backwards: the free blocks' order too is as it was)
        PagesSeq& s = pg->seqs[seq_ids[i]];
        pages_release(pg, s, s.len - n_new[i]);
        if (own[i] >= 0) {
          pg->drop(s.blocks.back());
          s.blocks.back() = own[i];
        }
      }
      undo_own();
      if (rc == PIPESD_EHIP) pages_take_back(pg, n_seqs, seq_ids, st);
      return rc;
    }
    pages_close_pass(pg);
    for (int32_t i = 0; i < n_seqs; ++i) pg->seqs[seq_ids[i]].in_pass = true;
    pg->pass.swap(plan);
    pg->launches.swap(launches);
    pg->attends = attends;
    pg->trees = trees;
    pg->rows_shared = false;
    pg->pass_open = true;
    return PIPESD_OK;
  });
}

static bool pages_rows_ok(const pipesd_config& c, const void* p, int64_t stride, int heads) {
  const size_t e = c.dtype == PIPESD_F32 ? 4 : 2;
  return p && ((uintptr_t)p & 15) == 0 && stride >= (int64_t)heads * c.head_dim && (stride * e) % 16 == 0;
}

static void pages_add_range(PagesRanges& r, int32_t table_off, int32_t first, int32_t count, int32_t row_off) {
  r.table_off[r.n] = table_off;
  r.first[r.n] = first;
  r.count[r.n] = count;
  r.row_off[r.n++] = row_off;
  r.most = std::max(r.most, (first + count - 1) / kBlockTokens - first / kBlockTokens + 1);
}

extern "C" int pipesd_pages_append(pipesd_pages* pg, int32_t layer, const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* stream) {
  if (!pg || layer < 0 || layer >= pg->cfg.n_layers) return PIPESD_EINVAL;
  if (!pages_rows_ok(pg->cfg, k, k_stride, pg->cfg.n_kv_heads) || !pages_rows_ok(pg->cfg, v, v_stride, pg->cfg.n_kv_heads)) return PIPESD_EINVAL;
  if (!pg->pool || !pg->pass_open || pg->rows_shared) return PIPESD_ESTATE;
  PagesRanges r;
  r.n = r.most = 0;
  for (size_t i = 0; i < pg->pass.size(); ++i) {
    const PagesClient& c = pg->pass[i];
    pages_add_range(r, c.table_off, c.len - c.n_rows, c.n_rows, c.row_off);
    if (r.n == kPagesPerLaunch || i + 1 == pg->pass.size()) {
      HIP_TRY(launch_pages_store(pg->cfg.dtype, pg->view(), layer, r, k, v, k_stride, v_stride, (hipStream_t)stream));
      r.n = r.most = 0;
    }
  }
  return PIPESD_OK;
}

extern "C" int pipesd_pages_attend(pipesd_pages* pg, int32_t layer, const void* q, int64_t q_stride, void* out, int64_t out_stride, void* stream) {
  if (!pg || layer < 0 || layer >= pg->cfg.n_layers) return PIPESD_EINVAL;
  if (!pages_rows_ok(pg->cfg, q, q_stride, pg->cfg.n_q_heads) || !pages_rows_ok(pg->cfg, out, out_stride, pg->cfg.n_q_heads)) return PIPESD_EINVAL;
  // (results where the queries are: every workgroup reads its rows' queries before it, or who joins its splits, writes these rows)
  if (pg->pass_open && (q != out || q_stride != out_stride)) {
    const int64_t e = pg->cfg.dtype == PIPESD_F32 ? 4 : 2, rows = pg->pass.back().row_off + pg->pass.back().n_rows;
    if (rows_overlap(q, q_stride * e, out, out_stride * e, rows, (int64_t)pg->cfg.n_q_heads * pg->cfg.head_dim * e)) return PIPESD_EINVAL;
  }
  if (!pg->pool || !pg->pass_open || !pg->attends) return PIPESD_ESTATE;
  PagesAttend a{};
  a.view = pg->view();
  a.dtype = pg->cfg.dtype;
  a.n_q_heads = pg->cfg.n_q_heads;
  a.group = pg->cfg.n_q_heads / pg->cfg.n_kv_heads;
  a.layer = layer;
  a.q = q;
  a.out = out;
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.masks = pg->trees ? pg->masks : nullptr;
  a.part = pg->part;
  a.counters = pg->counters;
  for (const PagesLaunch& l : pg->launches) HIP_TRY(launch_pages_attend(a, l, (hipStream_t)stream));
  return PIPESD_OK;
}

extern "C" int pipesd_pages_read(const pipesd_pages* pg, int32_t n_seqs, const int32_t* seq_ids, const int32_t* first, const int32_t* count,
                                 int32_t layer0, int32_t n_layers, void* k_out, void* v_out, void* stream) {
  if (!pg || n_seqs < 1 || !seq_ids || !first || !count) return PIPESD_EINVAL;
  const pipesd_config& c = pg->cfg;
  if (layer0 < 0 || n_layers < 1 || n_layers > c.n_layers - layer0) return PIPESD_EINVAL;
  if (!k_out || !v_out || ((uintptr_t)k_out & 15) || ((uintptr_t)v_out & 15)) return PIPESD_EINVAL;
  int64_t total = 0;
  for (int32_t i = 0; i < n_seqs; ++i) {
    if (!pages_seq_ok(pg, seq_ids[i]) || first[i] < 0 || count[i] < 0) return PIPESD_EINVAL;
    if (count[i] > pg->seqs[seq_ids[i]].len - first[i]) return PIPESD_ESTATE;
    total += count[i];
  }
  if (total > INT32_MAX) return PIPESD_EINVAL;
  if (!pg->pool) return PIPESD_ESTATE;
  PagesRanges r;
  r.n = r.most = 0;
  int32_t row = 0;
  for (int32_t i = 0; i < n_seqs; ++i) {
    if (count[i] > 0) {
      pages_add_range(r, pg->table_off(seq_ids[i]), first[i], count[i], row);
      row += count[i];
    }
    if (r.n == kPagesPerLaunch || (i + 1 == n_seqs && r.n > 0)) {
      HIP_TRY(launch_pages_read(c.dtype, pg->view(), layer0, n_layers, r, total, k_out, v_out, (hipStream_t)stream));
      r.n = r.most = 0;
    }
  }
  return PIPESD_OK;
}

// what fork and copy check of their clients: sources (one may be several times there), targets that are none of them, lengths
static int pages_check_targets(const pipesd_pages* pg, int32_t n, const int32_t* seq_ids, const int32_t* into, const int32_t* len) {
  if (!pages_seqs_ok(pg, n, into)) return PIPESD_EINVAL;
  std::vector<char> target(pg->max_seqs, 0);
  for (int32_t i = 0; i < n; ++i) target[into[i]] = 1;
  for (int32_t i = 0; i < n; ++i)
    if (!pages_seq_ok(pg, seq_ids[i]) || target[seq_ids[i]]) return PIPESD_EINVAL;
  for (int32_t i = 0; i < n; ++i)
    if (len && (len[i] < 0 || len[i] > pg->seqs[seq_ids[i]].len)) return PIPESD_ESTATE;
  return PIPESD_OK;
}
static void pages_clear_targets(pipesd_pages* pg, int32_t n, const int32_t* into) {
  bool touched = false;
  for (int32_t i = n - 1; i >= 0; --i) {
    PagesSeq& t = pg->seqs[into[i]];
    touched |= t.in_pass;
    pages_release(pg, t, 0);
  }
  if (touched) pages_close_pass(pg);
}

extern "C" int pipesd_pages_fork(pipesd_pages* pg, int32_t n_seqs, const int32_t* seq_ids, const int32_t* into, const int32_t* len, void* stream) {
  if (!pg || n_seqs < 1 || !seq_ids || !into) return PIPESD_EINVAL;
  return guarded([&]() -> int {
    hipStream_t st = (hipStream_t)stream;
    if (int rc = pages_check_targets(pg, n_seqs, seq_ids, into, len)) return rc;
    if (pg->pool)
      if (int rc = pages_not_recorded(st)) return rc;
    for (int32_t i = 0; i < n_seqs; ++i) {
      const size_t nb = pages_blocks(len ? len[i] : pg->seqs[seq_ids[i]].len);
      pg->seqs[into[i]].blocks.reserve(nb);
      pg->seqs[into[i]].sent.reserve(nb);
    }
    pages_clear_targets(pg, n_seqs, into);  // (they are empty if a launch fails)
    PagesForks f;
    f.n = f.most = 0;
    int rc = PIPESD_OK;
    for (int32_t i = 0; i < n_seqs; ++i) {
      const PagesSeq& s = pg->seqs[seq_ids[i]];
      PagesSeq& t = pg->seqs[into[i]];
      t.len = len ? len[i] : s.len;
      t.blocks.assign(s.blocks.begin(), s.blocks.begin() + pages_blocks(t.len));
      for (int32_t b : t.blocks) ++pg->users[b];
      if (pg->pool && pages_unsent(s, 0) && !rc) rc = pages_send(pg, 1, &seq_ids[i], nullptr, false, {}, nullptr, st);
      if (pg->pool && pages_unsent(t, 0)) {
        f.from[f.n] = pg->table_off(seq_ids[i]);
        f.to[f.n] = pg->table_off(into[i]);
        f.blocks[f.n++] = (int32_t)t.blocks.size();
        f.most = std::max(f.most, (int32_t)t.blocks.size());
        if (t.sent.size() < t.blocks.size()) t.sent.resize(t.blocks.size());
        std::copy(t.blocks.begin(), t.blocks.end(), t.sent.begin());
      }
      if (f.n == kPagesPerLaunch || (i + 1 == n_seqs && f.n > 0)) {
        const hipError_t e = launch_pages_fork(f, pg->table, st);
        if (e != hipSuccess && !rc) rc = hip_fail(e, "forking clients of a paged cache");
        f.n = f.most = 0;
      }
    }
    for (int32_t i = 0; !rc && i < n_seqs; ++i) {
      if (!pg->seqs[seq_ids[i]].in_pass) continue;
      for (const PagesClient& c : pg->pass) pg->rows_shared = pg->rows_shared || (c.seq == seq_ids[i] && pg->seqs[into[i]].len > c.len - c.n_rows);
    }
    if (rc) {
      pages_clear_targets(pg, n_seqs, into);
      for (int32_t i = 0; i < n_seqs; ++i) std::fill(pg->seqs[into[i]].sent.begin(), pg->seqs[into[i]].sent.end(), -1);
    }
    return rc;
  });
}

extern "C" int pipesd_pages_copy(pipesd_pages* pg, int32_t n_seqs, const int32_t* seq_ids, const int32_t* into, const int32_t* len, void* stream) {
  if (!pg || n_seqs < 1 || !seq_ids || !into) return PIPESD_EINVAL;
  return guarded([&]() -> int {
    hipStream_t st = (hipStream_t)stream;
    if (int rc = pages_check_targets(pg, n_seqs, seq_ids, into, len)) return rc;
    if (pg->pool)
      if (int rc = pages_not_recorded(st)) return rc;
    int64_t need = 0, have = (int64_t)pg->free_list.size();
    for (int32_t i = 0; i < n_seqs; ++i) need += pages_blocks(len ? len[i] : pg->seqs[seq_ids[i]].len);
    for (int32_t i = 0; i < n_seqs; ++i)  // what the targets hold alone is given up first
      for (int32_t b : pg->seqs[into[i]].blocks) have += --pg->users[b] == 0;
    for (int32_t i = 0; i < n_seqs; ++i)
      for (int32_t b : pg->seqs[into[i]].blocks) ++pg->users[b];
    if (need > have) return PIPESD_ENOMEM;
    pg->from.clear();
    pg->to.clear();
    pg->from.reserve(need);
    pg->to.reserve(need);
    for (int32_t i = 0; i < n_seqs; ++i) {
      const size_t nb = pages_blocks(len ? len[i] : pg->seqs[seq_ids[i]].len);
      pg->seqs[into[i]].blocks.reserve(nb);
      pg->seqs[into[i]].sent.reserve(nb);
    }
    pages_clear_targets(pg, n_seqs, into);  // (they are empty if a launch fails)
    for (int32_t i = 0; i < n_seqs; ++i) {
      const PagesSeq& s = pg->seqs[seq_ids[i]];
      PagesSeq& t = pg->seqs[into[i]];
      t.len = len ? len[i] : s.len;
      for (int32_t b = 0; b < pages_blocks(t.len); ++b) {
        t.blocks.push_back(pg->take());
        pg->from.push_back(s.blocks[b]);
        pg->to.push_back(t.blocks[b]);
      }
    }
    if (!pg->pool) return PIPESD_OK;
    const bool few = pg->from.size() <= (size_t)kPagesOwnPerLaunch;  // (go with the tables' entries: a launch less)
    int rc = few ? PIPESD_OK : pages_moves(pg, true, st);
    if (!rc) rc = pages_send(pg, n_seqs, into, nullptr, few, {}, nullptr, st);
    if (rc) pages_clear_targets(pg, n_seqs, into);
    return rc;
  });
}

extern "C" int pipesd_pages_compact(pipesd_pages* pg, int32_t n_seqs, const int32_t* seq_ids, const int32_t* first, const int32_t* n_kept,
                                    const int32_t* kept, void* stream) {
  if (!pg || n_seqs < 1 || !seq_ids || !first || !n_kept) return PIPESD_EINVAL;
  return guarded([&]() -> int {
    hipStream_t st = (hipStream_t)stream;
    if (!pages_seqs_ok(pg, n_seqs, seq_ids)) return PIPESD_EINVAL;
    int64_t total = 0;
    for (int32_t i = 0; i < n_seqs; ++i) {
      if (first[i] < 0 || n_kept[i] < 0) return PIPESD_EINVAL;
      if (first[i] > pg->seqs[seq_ids[i]].len) return PIPESD_ESTATE;
      const int32_t rows = pg->seqs[seq_ids[i]].len - first[i];
      if (n_kept[i] > 0 && !kept) return PIPESD_EINVAL;
      for (int32_t j = 0; j < n_kept[i]; ++j) {
        const int32_t at = kept[total + j];
        if (at < 0 || (j > 0 && at <= kept[total + j - 1])) return PIPESD_EINVAL;
        if (at >= rows) return PIPESD_ESTATE;
      }
      total += n_kept[i];
    }
    // Where tokens go to, a block with other users is replaced.  Clients one after the other: if several share one, who comes last keeps
    // it, and writes it when the others' tokens have been read.
    pg->from.clear();
    pg->to.clear();
    pg->from.reserve(total + (size_t)n_seqs * kBlockTokens);
    pg->to.reserve(total + (size_t)n_seqs * kBlockTokens);
    std::vector<int32_t>&moved = pg->had, &own = pg->own;  // how many tokens of each stay where they are; blocks that are replaced
    moved.resize(n_seqs);
    own.clear();
    struct Range {
      int32_t b0, b1;
    };
    auto range = [&](int32_t i) {
      if (moved[i] == n_kept[i]) return Range{0, 0};
      return Range{(first[i] + moved[i]) / kBlockTokens, pages_blocks(first[i] + n_kept[i])};
    };
    size_t most = 0;
    int64_t k0 = 0;
    for (int32_t i = 0; i < n_seqs; ++i) {
      moved[i] = 0;
      while (moved[i] < n_kept[i] && kept[k0 + moved[i]] == moved[i]) ++moved[i];
      k0 += n_kept[i];
      const Range r = range(i);
      most += r.b1 - r.b0;
    }
    own.reserve(most);
    for (int32_t i = 0; i < n_seqs; ++i) {
      const Range r = range(i);
      for (int32_t b = r.b0; b < r.b1; ++b) {
        const int32_t blk = pg->seqs[seq_ids[i]].blocks[b];
        if (pg->users[blk] > 1) own.push_back(blk), --pg->users[blk];
      }
    }
    for (int32_t blk : own) ++pg->users[blk];
    if (own.size() > pg->free_list.size()) return PIPESD_ENOMEM;
    const bool work = most > 0;
    if (pg->pool && work)
      if (int rc = pages_not_recorded(st)) return rc;
    struct Replaced {
      int32_t seq, at, blk;
    };
    std::vector<Replaced> replaced;
    replaced.reserve(own.size());
    k0 = 0;
    for (int32_t i = 0; i < n_seqs; ++i) {
      PagesSeq& s = pg->seqs[seq_ids[i]];
      const Range r = range(i);
      auto place = [&](int32_t pos) { return s.blocks[pos / kBlockTokens] * kBlockTokens + pos % kBlockTokens; };
      const bool whole = r.b0 < r.b1 && pg->users[s.blocks[r.b0]] > 1;  // (then what stays in the first block comes along)
      const int32_t lead = whole ? (first[i] + moved[i]) % kBlockTokens : 0;
      for (int32_t j = moved[i] - lead; j < moved[i]; ++j) pg->from.push_back(place(first[i] + j));
      for (int32_t j = moved[i]; j < n_kept[i]; ++j) pg->from.push_back(place(first[i] + kept[k0 + j]));
      for (int32_t b = r.b0; b < r.b1; ++b)
        if (pg->users[s.blocks[b]] > 1) {
          replaced.push_back(Replaced{seq_ids[i], b, s.blocks[b]});
          --pg->users[s.blocks[b]];
          s.blocks[b] = pg->take();
        }
      for (int32_t j = moved[i] - lead; pg->to.size() < pg->from.size(); ++j) pg->to.push_back(place(first[i] + j));
      k0 += n_kept[i];
    }
    if (pg->pool && work) {
      auto launch = [&]() -> int {
        std::vector<int32_t> from(n_seqs);
        for (int32_t i = 0; i < n_seqs; ++i) from[i] = range(i).b0;
        if (int e = pages_moves(pg, false, st)) return e;
        return replaced.empty() ? PIPESD_OK : pages_send(pg, n_seqs, seq_ids, from.data(), false, {}, nullptr, st);
      };
      if (int rc = launch()) {  // (tokens behind `first` may have been moved, as by a call that has run)
        for (size_t j = replaced.size(); j-- > 0;) {
          PagesSeq& s = pg->seqs[replaced[j].seq];
          pg->drop(s.blocks[replaced[j].at]);
          s.blocks[replaced[j].at] = replaced[j].blk;
          ++pg->users[replaced[j].blk];
        }
        if (rc == PIPESD_EHIP) pages_take_back(pg, n_seqs, seq_ids, st);
        return rc;
      }
    }
    bool touched = false;
    for (int32_t i = n_seqs - 1; i >= 0; --i) {
      PagesSeq& s = pg->seqs[seq_ids[i]];
      touched |= s.in_pass && first[i] + n_kept[i] < s.len;
      pages_release(pg, s, first[i] + n_kept[i]);
    }
    if (touched) pages_close_pass(pg);
    return PIPESD_OK;
  });
}
