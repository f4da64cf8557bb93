// Host side of the 4-bit cache: the handle, its bookkeeping, the passes.
#include <algorithm>
#include <new>
#include <vector>

#include "kv4.h"
#include "status.h"

using namespace pipesd;

namespace {
struct Kv4Seq {
  int32_t len = 0;
  std::vector<int32_t> blocks;  // in token order
  int32_t which = 0;            // of the client's two block tables
  std::vector<int32_t> sent[2]; // what the device has in them
  bool in_pass = false;         // of the pass that store and attend work on
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

struct pipesd_kv4 {
  pipesd_config cfg{};
  int32_t max_seqs = 0, n_blocks = 0;
  uint8_t* pool = nullptr;
  std::vector<int32_t> free_list;
  std::vector<Kv4Seq> seqs;
  int n_cu = 256;
  // device memory of the library
  int32_t* table = nullptr;  // [2 max_seqs][n_blocks]
  float* part = nullptr;
  size_t part_cap = 0;  // floats
  unsigned* counters = nullptr;
  size_t counters_cap = 0;
  float* lse = nullptr;
  size_t lse_cap = 0;
  std::vector<void*> old;  // buffers that have grown since
  // the pass
  std::vector<Kv4Client> pass, next_pass;  // (next_..: where the next pass is made)
  std::vector<Kv4Launch> launches, next_launches;
  std::vector<int32_t> idle, next_idle;    // its clients without new rows
  std::vector<int32_t> had;
  bool pass_open = false, attends = false;

  int32_t table_off(int32_t seq) const { return (2 * seq + seqs[seq].which) * n_blocks; }
  Kv4View view() const { return Kv4View{pool, table, n_blocks, cfg.n_layers, cfg.n_kv_heads}; }
};

static int32_t kv4_blocks(int32_t tokens) { return tokens / kBlockTokens + (tokens % kBlockTokens != 0); }
static bool kv4_seq_ok(const pipesd_kv4* kv, int32_t seq) { return kv && seq >= 0 && seq < kv->max_seqs; }
// every id in range, none twice
static bool kv4_seqs_ok(const pipesd_kv4* kv, int32_t n, const int32_t* ids) {
  for (int32_t i = 0; i < n; ++i)
    if (!kv4_seq_ok(kv, ids[i])) return false;
  bool rising = true;  // (as ids mostly are)
  for (int32_t i = 1; i < n; ++i) rising = rising && ids[i] > ids[i - 1];
  if (rising) return true;
  std::vector<char> seen(kv->max_seqs, 0);
  for (int32_t i = 0; i < n; ++i)
    if (seen[ids[i]]++) return false;
  return true;
}
static void kv4_release(pipesd_kv4* kv, Kv4Seq& s, int32_t tokens) {
  const int32_t keep = kv4_blocks(tokens);
  while ((int32_t)s.blocks.size() > keep) {
    kv->free_list.push_back(s.blocks.back());  // (has room for every block)
    s.blocks.pop_back();
  }
  s.len = tokens;
}
static void kv4_close_pass(pipesd_kv4* kv) {
  for (Kv4Seq& s : kv->seqs) s.in_pass = false;
  kv->pass_open = false;
}

static bool kv4_config_ok(const pipesd_config* c) {
  return c->n_layers >= 1 && c->n_kv_heads >= 1 && c->n_q_heads >= 1 && c->n_q_heads % c->n_kv_heads == 0 &&
         (c->head_dim == 64 || c->head_dim == 128) && (c->dtype == PIPESD_F32 || c->dtype == PIPESD_BF16) && c->n_kv_heads <= 65535 &&
         c->n_layers <= 65535 && (int64_t)c->n_layers * c->n_kv_heads <= INT32_MAX && c->n_q_heads / c->n_kv_heads <= 256;
}

extern "C" size_t pipesd_kv4_block_bytes(const pipesd_config* cfg, int32_t block_tokens) {
  if (!cfg || block_tokens != kBlockTokens || !kv4_config_ok(cfg)) return 0;
  return (size_t)cfg->n_layers * cfg->n_kv_heads * kv4_record_bytes(cfg->head_dim);
}

// Grows a buffer of the pass.  The old one stays until the handle ends: the device may still be using it, and recorded calls hold its
// address (half as much again each time: all old ones together are less than twice the last).
template <class T>
static int kv4_grow(pipesd_kv4* kv, T** p, size_t* cap, size_t want, bool zero, size_t spare) {
  if (want <= *cap) return PIPESD_OK;
  want += spare;
  kv->old.reserve(kv->old.size() + 1);
  T* fresh = nullptr;
  if (hipMalloc((void**)&fresh, want * sizeof(T)) != hipSuccess) {
    (void)hipGetLastError();
    return PIPESD_ENOMEM;
  }
  hipError_t e = zero ? hipMemset(fresh, 0, want * sizeof(T)) : hipSuccess;
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    (void)hipFree(fresh);
    return hip_fail(e, "growing a buffer of the 4-bit cache");
  }
  if (*p) kv->old.push_back(*p);
  *p = fresh;
  *cap = want;
  return PIPESD_OK;
}

extern "C" int pipesd_kv4_destroy(pipesd_kv4* kv) {
  if (!kv) return PIPESD_EINVAL;
  if (kv->pool) {
    (void)hipDeviceSynchronize();
    for (void* p : {(void*)kv->table, (void*)kv->part, (void*)kv->counters, (void*)kv->lse})
      if (p) (void)hipFree(p);
    for (void* p : kv->old) (void)hipFree(p);
  }
  delete kv;
  return PIPESD_OK;
}

extern "C" int pipesd_kv4_create(const pipesd_config* cfg, int32_t max_seqs, int32_t block_tokens, void* pool, size_t pool_bytes,
                                 pipesd_kv4** out) {
  if (!cfg || !out || max_seqs < 1 || !kv4_config_ok(cfg)) return PIPESD_EINVAL;
  const size_t bb = pipesd_kv4_block_bytes(cfg, block_tokens);
  if (bb == 0) return PIPESD_EINVAL;
  const size_t n = pool_bytes / bb;
  // tokens, slots of both block tables: 32-bit numbers
  if (n < 1 || n > (size_t)INT32_MAX / kBlockTokens || 2 * (uint64_t)max_seqs * n > (uint64_t)INT32_MAX) return PIPESD_EINVAL;
  if (pool && ((uintptr_t)pool & 255)) return PIPESD_EINVAL;
  pipesd_kv4* kv = new (std::nothrow) pipesd_kv4();
  if (!kv) return PIPESD_ENOMEM;
  int rc = guarded([&]() -> int {
    kv->cfg = *cfg;
    kv->max_seqs = max_seqs;
    kv->n_blocks = (int32_t)n;
    kv->seqs.resize(max_seqs);
    kv->pass.reserve(max_seqs);
    kv->free_list.reserve(n);
    for (int32_t b = kv->n_blocks - 1; b >= 0; --b) kv->free_list.push_back(b);  // block 0 is handed out first
    if (!pool) return PIPESD_OK;
    kv->pool = (uint8_t*)pool;
    kv->n_cu = device_cu_count();
    if (kv->n_cu <= 0) return PIPESD_EHIP;
    const size_t entries = 2 * (size_t)max_seqs * n;
    if (hipMalloc((void**)&kv->table, entries * 4) != hipSuccess) {
      (void)hipGetLastError();
      return PIPESD_ENOMEM;
    }
    HIP_TRY(hipMemset(kv->table, 0, entries * 4));
    const int32_t clients = std::min(max_seqs, 16);
    const Kv4PlanNeeds most = kv4_plan_most(clients, kMaxRows, (int64_t)kv->n_blocks * kBlockTokens, cfg->dtype, cfg->head_dim, cfg->n_q_heads,
                                            cfg->n_kv_heads, kv->n_cu);
    int e;
    if ((e = kv4_grow(kv, &kv->part, &kv->part_cap, most.part_tiles * 16 * (cfg->head_dim + kKv4PartPad), false, 0))) return e;
    if ((e = kv4_grow(kv, &kv->counters, &kv->counters_cap, most.counters, true, 0))) return e;
    return kv4_grow(kv, &kv->lse, &kv->lse_cap, (size_t)clients * kMaxRows * cfg->n_q_heads, false, 0);
  });
  if (rc) {
    pipesd_kv4_destroy(kv);
    return rc;
  }
  *out = kv;
  return PIPESD_OK;
}

extern "C" int pipesd_kv4_len(const pipesd_kv4* kv, int32_t seq, int32_t* len) {
  if (!kv4_seq_ok(kv, seq) || !len) return PIPESD_EINVAL;
  *len = kv->seqs[seq].len;
  return PIPESD_OK;
}
extern "C" int pipesd_kv4_free_blocks(const pipesd_kv4* kv, int32_t* n_free) {
  if (!kv || !n_free) return PIPESD_EINVAL;
  *n_free = (int32_t)kv->free_list.size();
  return PIPESD_OK;
}
extern "C" int pipesd_kv4_seq_blocks(const pipesd_kv4* kv, int32_t seq, int32_t* n_blocks) {
  if (!kv4_seq_ok(kv, seq) || !n_blocks) return PIPESD_EINVAL;
  *n_blocks = (int32_t)kv->seqs[seq].blocks.size();
  return PIPESD_OK;
}

extern "C" int pipesd_kv4_truncate(pipesd_kv4* kv, int32_t n_seqs, const int32_t* seq_ids, const int32_t* new_len) {
  if (!kv || n_seqs < 1 || !seq_ids || !new_len) return PIPESD_EINVAL;
  return guarded([&]() -> int {
    if (!kv4_seqs_ok(kv, n_seqs, seq_ids)) return PIPESD_EINVAL;
    for (int32_t i = 0; i < n_seqs; ++i)
      if (new_len[i] < 0 || new_len[i] > kv->seqs[seq_ids[i]].len) return PIPESD_ESTATE;
    bool touched = false;
    for (int32_t i = n_seqs - 1; i >= 0; --i) {  // (backwards: who asks for as much again, in the same order, gets the same blocks)
      Kv4Seq& s = kv->seqs[seq_ids[i]];
      touched |= s.in_pass && new_len[i] < s.len;
      kv4_release(kv, s, new_len[i]);
    }
    if (touched) kv4_close_pass(kv);
    return PIPESD_OK;
  });
}

// What writes block tables is not recorded: a replay would write them again, when the blocks may be another client's, and until the
// first replay the device has not what the host takes it to have.
static int kv4_not_recorded(hipStream_t st) {
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  HIP_TRY(hipStreamIsCapturing(st, &status));
  return status == hipStreamCaptureStatusNone ? PIPESD_OK : PIPESD_ESTATE;
}

// sends what is new of the block tables, some per launch.  (A block that a client gave back and got again is there already.)
static int kv4_send(pipesd_kv4* kv, int32_t n, const int32_t* seq_ids, const int32_t* from, hipStream_t st) {
  Kv4TableUpdate u;
  u.n = 0;
  auto flush = [&]() -> int {
    if (u.n == 0) return PIPESD_OK;
    if (int rc = kv4_not_recorded(st)) return rc;
    HIP_TRY(launch_kv4_table(u, kv->table, st));
    u.n = 0;
    return PIPESD_OK;
  };
  for (int32_t k = 0; k < n; ++k) {
    Kv4Seq& s = kv->seqs[seq_ids[k]];
    const int32_t off = kv->table_off(seq_ids[k]);
    std::vector<int32_t>& sent = s.sent[s.which];
    const int32_t nb = (int32_t)s.blocks.size();
    if ((int32_t)sent.size() < nb) sent.resize(nb, -1);
    for (int32_t i = from ? from[k] : 0; i < nb; ++i) {
      if (sent[i] == s.blocks[i]) continue;
      if (u.n == kKv4EntriesPerLaunch)
        if (int rc = flush()) return rc;
      u.at[u.n] = off + i;
      u.v[u.n++] = sent[i] = s.blocks[i];
    }
  }
  return flush();
}

extern "C" int pipesd_kv4_extend(pipesd_kv4* kv, int32_t n_seqs, const int32_t* seq_ids, const int32_t* n_new, void* stream) {
  if (!kv || n_seqs < 1 || n_seqs > PIPESD_KV4_MAX_PASS_SEQS || !seq_ids || !n_new) return PIPESD_EINVAL;
  return guarded([&]() -> int {
    hipStream_t st = (hipStream_t)stream;
    if (!kv4_seqs_ok(kv, n_seqs, seq_ids)) return PIPESD_EINVAL;
    const pipesd_config& cfg = kv->cfg;
    int64_t total = 0, blocks = 0;
    bool attends = true;
    for (int32_t i = 0; i < n_seqs; ++i) {
      const Kv4Seq& s = kv->seqs[seq_ids[i]];
      if (n_new[i] < 0 || n_new[i] > (int32_t)(INT32_MAX / 2) - s.len) return PIPESD_EINVAL;
      total += n_new[i];
      blocks += kv4_blocks(s.len + n_new[i]) - (int32_t)s.blocks.size();
      attends = attends && n_new[i] <= kKv4MaxRows;
    }
    if (total < 1 || total > INT32_MAX) return PIPESD_EINVAL;
    if (blocks > (int64_t)kv->free_list.size()) return PIPESD_ENOMEM;

    std::vector<Kv4Client>& plan = kv->next_pass;
    std::vector<Kv4Launch>& launches = kv->next_launches;
    std::vector<int32_t>& had = kv->had;
    plan.clear();
    launches.clear();
    std::vector<int32_t>& idle = kv->next_idle;
    had.resize(n_seqs);
    plan.reserve(n_seqs);
    idle.clear();
    int32_t row = 0;
    for (int32_t i = 0; i < n_seqs; ++i) {
      had[i] = (int32_t)kv->seqs[seq_ids[i]].blocks.size();
      if (n_new[i]) plan.push_back(Kv4Client{seq_ids[i], n_new[i], row, kv->seqs[seq_ids[i]].len + n_new[i]});
      else idle.push_back(seq_ids[i]);
      row += n_new[i];
    }
    if (kv->pool && attends) {
      const Kv4PlanNeeds need = kv4_plan(plan.data(), (int)plan.size(), cfg.dtype, cfg.head_dim, cfg.n_q_heads, cfg.n_kv_heads, kv->n_cu, launches);
      if (need.part_tiles > (size_t)INT32_MAX || need.counters > (size_t)INT32_MAX) return PIPESD_ENOMEM;
      for (Kv4Launch& l : launches)
        for (int32_t j = 0; j < l.c.n; ++j) l.c.table_off[j] = kv->table_off(l.c.seq[j]);
      const size_t parts = need.part_tiles * 16 * (cfg.head_dim + kKv4PartPad), sums = (size_t)total * cfg.n_q_heads;
      int e;
      if (parts > kv->part_cap || need.counters > kv->counters_cap || sums > kv->lse_cap)
        if ((e = kv4_not_recorded(st))) return e;
      if ((e = kv4_grow(kv, &kv->part, &kv->part_cap, parts, false, parts / 2))) return e;
      if ((e = kv4_grow(kv, &kv->counters, &kv->counters_cap, need.counters, true, need.counters / 2))) return e;
      if ((e = kv4_grow(kv, &kv->lse, &kv->lse_cap, sums, false, sums / 2))) return e;
    }
    for (int32_t i = 0; i < n_seqs; ++i) {
      Kv4Seq& s = kv->seqs[seq_ids[i]];
      s.blocks.reserve(kv4_blocks(s.len + n_new[i]));
      s.sent[s.which].reserve(kv4_blocks(s.len + n_new[i]));
    }

    // from here on only the launches can fail: what they have not done is taken back
    for (int32_t i = 0; i < n_seqs; ++i) {
      Kv4Seq& s = kv->seqs[seq_ids[i]];
      s.len += n_new[i];
      while ((int32_t)s.blocks.size() < kv4_blocks(s.len)) {
        s.blocks.push_back(kv->free_list.back());
        kv->free_list.pop_back();
      }
    }
    if (kv->pool) {
      if (int rc = kv4_send(kv, n_seqs, seq_ids, had.data(), st)) {
        for (int32_t i = n_seqs - 1; i >= 0; --i) {  // (backwards: the free blocks' order too is as it was)
          Kv4Seq& s = kv->seqs[seq_ids[i]];
          std::fill(s.sent[s.which].begin() + had[i], s.sent[s.which].end(), -1);
          kv4_release(kv, s, s.len - n_new[i]);
        }
        return rc;
      }
    }
    kv4_close_pass(kv);
    for (int32_t i = 0; i < n_seqs; ++i) kv->seqs[seq_ids[i]].in_pass = true;
    kv->pass.swap(plan);
    kv->launches.swap(launches);
    kv->idle.swap(idle);
    kv->attends = attends;
    kv->pass_open = true;
    return PIPESD_OK;
  });
}

static bool kv4_rows_ok(const pipesd_config& c, const void* p, int64_t stride, int heads) {
  const size_t e = c.dtype == PIPESD_F32 ? 4 : 2;
  return p && ((uintptr_t)p & 15) == 0 && stride >= (int64_t)heads * c.head_dim && (stride * e) % 16 == 0;
}

// Whether a row of a and a row of b share bytes: `rows` of `width` bytes each, strides of at least that.
static bool kv4_rows_overlap(const void* a, int64_t a_stride, const void* b, int64_t b_stride, int64_t rows, int64_t width) {
  if ((uintptr_t)a > (uintptr_t)b) std::swap(a, b), std::swap(a_stride, b_stride);
  int64_t at = (int64_t)((uintptr_t)b - (uintptr_t)a);  // of b's first row, from a's
  if (at >= (rows - 1) * a_stride + width) return false;
  if (a_stride == b_stride) {  // (columns of one matrix) b's rows lie between the same two rows of a each, or behind the last
    const int64_t before = at / a_stride;
    return at % a_stride < width || (before + 1 < rows && a_stride - at % a_stride < width);
  }
  for (int64_t i = 0, j = 0; i < rows && j < rows;) {
    if (at >= width) ++i, at -= a_stride;
    else if (at <= -width) ++j, at += b_stride;
    else return true;
  }
  return false;
}

static void kv4_add_range(Kv4Ranges& r, int32_t table_off, int32_t first, int32_t count, int32_t row_off) {
  r.table_off[r.n] = table_off;
  r.first[r.n] = first;
  r.count[r.n] = count;
  r.row_off[r.n++] = row_off;
  r.most = std::max(r.most, count);
}

extern "C" int pipesd_kv4_append(pipesd_kv4* kv, int32_t layer, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                 void* stream) {
  if (!kv || layer < 0 || layer >= kv->cfg.n_layers) return PIPESD_EINVAL;
  if (!kv4_rows_ok(kv->cfg, k, k_stride, kv->cfg.n_kv_heads) || !kv4_rows_ok(kv->cfg, v, v_stride, kv->cfg.n_kv_heads)) return PIPESD_EINVAL;
  if (!kv->pool || !kv->pass_open) return PIPESD_ESTATE;
  Kv4Ranges r;
  r.n = r.most = 0;
  for (size_t i = 0; i < kv->pass.size(); ++i) {
    const Kv4Client& c = kv->pass[i];
    kv4_add_range(r, kv->table_off(c.seq), c.len - c.n_rows, c.n_rows, c.row_off);
    if (r.n == kKv4ClientsPerLaunch || i + 1 == kv->pass.size()) {
      HIP_TRY(launch_kv4_store(kv->cfg.dtype, kv->cfg.head_dim, kv->view(), layer, r, k, v, k_stride, v_stride, (hipStream_t)stream));
      r.n = r.most = 0;
    }
  }
  return PIPESD_OK;
}

extern "C" int pipesd_kv4_attend(pipesd_kv4* kv, int32_t layer, const void* q, int64_t q_stride, const int32_t* limits, void* out,
                                 int64_t out_stride, float* mass, int64_t mass_stride, float decay, void* stream) {
  if (!kv || layer < 0 || layer >= kv->cfg.n_layers) return PIPESD_EINVAL;
  if (!kv4_rows_ok(kv->cfg, q, q_stride, kv->cfg.n_q_heads) || !kv4_rows_ok(kv->cfg, out, out_stride, kv->cfg.n_q_heads)) return PIPESD_EINVAL;
  if (((uintptr_t)limits & 3) || ((uintptr_t)mass & 3)) return PIPESD_EINVAL;
  // Results where the queries are: every workgroup reads its rows' queries before it, or who joins its splits, writes these rows.
  // The weights are formed from the queries again, when all results have been written.
  if (kv->pass_open && (mass || q != out || q_stride != out_stride)) {
    const int64_t e = kv->cfg.dtype == PIPESD_F32 ? 4 : 2, rows = kv->pass.back().row_off + kv->pass.back().n_rows;
    if (kv4_rows_overlap(q, q_stride * e, out, out_stride * e, rows, (int64_t)kv->cfg.n_q_heads * kv->cfg.head_dim * e)) return PIPESD_EINVAL;
  }
  if (!kv->pool || !kv->pass_open || !kv->attends) return PIPESD_ESTATE;
  if (mass) {
    if (!(decay >= 0.f) || !(decay <= 1.f)) return PIPESD_EINVAL;
    for (const Kv4Client& c : kv->pass)
      if (c.len > mass_stride) return PIPESD_EINVAL;
    for (int32_t seq : kv->idle)
      if (kv->seqs[seq].len > mass_stride) return PIPESD_EINVAL;
  }
  hipStream_t st = (hipStream_t)stream;
  Kv4AttendCall a{};
  a.view = kv->view();
  a.dtype = kv->cfg.dtype;
  a.head_dim = kv->cfg.head_dim;
  a.n_q_heads = kv->cfg.n_q_heads;
  a.group = kv->cfg.n_q_heads / kv->cfg.n_kv_heads;
  a.layer = layer;
  a.q = q;
  a.out = out;
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.limits = limits;
  a.part = kv->part;
  a.counters = kv->counters;
  a.lse = mass ? kv->lse : nullptr;
  a.mass = mass;
  a.mass_stride = mass_stride;
  a.decay = decay;
  for (const Kv4Launch& l : kv->launches) {
    HIP_TRY(launch_kv4_attend(a, l, st));
    if (mass) HIP_TRY(launch_kv4_mass(a, l.c, st));
  }
  if (mass && decay != 1.f) {
    Kv4Idle idle;
    idle.n = idle.most = 0;
    for (size_t i = 0; i < kv->idle.size(); ++i) {
      idle.seq[idle.n] = kv->idle[i];
      idle.len[idle.n] = kv->seqs[kv->idle[i]].len;
      idle.most = std::max(idle.most, idle.len[idle.n++]);
      if (idle.n == kKv4ClientsPerLaunch || i + 1 == kv->idle.size()) {
        HIP_TRY(launch_kv4_decay(a, idle, st));
        idle.n = idle.most = 0;
      }
    }
  }
  return PIPESD_OK;
}

extern "C" int pipesd_kv4_read(const pipesd_kv4* kv, int32_t n_seqs, const int32_t* seq_ids, const int32_t* first, const int32_t* count,
                               int32_t layer0, int32_t n_layers, void* k_out, void* v_out, void* stream) {
  if (!kv || n_seqs < 1 || !seq_ids || !first || !count) return PIPESD_EINVAL;
  const pipesd_config& c = kv->cfg;
  if (layer0 < 0 || n_layers < 1 || n_layers > c.n_layers - layer0) return PIPESD_EINVAL;
  if (!k_out || !v_out || ((uintptr_t)k_out & 15) || ((uintptr_t)v_out & 15)) return PIPESD_EINVAL;
  int64_t total = 0;
  for (int32_t i = 0; i < n_seqs; ++i) {
    if (!kv4_seq_ok(kv, seq_ids[i]) || first[i] < 0 || count[i] < 0) return PIPESD_EINVAL;
    if (count[i] > kv->seqs[seq_ids[i]].len - first[i]) return PIPESD_ESTATE;
    total += count[i];
  }
  if (total > INT32_MAX) return PIPESD_EINVAL;
  if (!kv->pool) return PIPESD_ESTATE;
  Kv4Ranges r;
  r.n = r.most = 0;
  int32_t row = 0;
  for (int32_t i = 0; i < n_seqs; ++i) {
    if (count[i] > 0) {
      kv4_add_range(r, kv->table_off(seq_ids[i]), first[i], count[i], row);
      row += count[i];
    }
    if (r.n == kKv4ClientsPerLaunch || (i + 1 == n_seqs && r.n > 0)) {
      HIP_TRY(launch_kv4_read(c.dtype, c.head_dim, kv->view(), layer0, n_layers, r, total, k_out, v_out, (hipStream_t)stream));
      r.n = r.most = 0;
    }
  }
  return PIPESD_OK;
}

extern "C" int pipesd_kv4_evict(pipesd_kv4* kv, int32_t n_seqs, const int32_t* seq_ids, const int32_t* into, int32_t keep, int32_t recent,
                                float* mass, int64_t mass_stride, int32_t* kept, void* stream) {
  if (!kv || n_seqs < 1 || !seq_ids || !into || keep < 1 || recent < 0 || recent > keep) return PIPESD_EINVAL;
  if (!mass || ((uintptr_t)mass & 3) || !kept || ((uintptr_t)kept & 3)) return PIPESD_EINVAL;
  return guarded([&]() -> int {
    hipStream_t st = (hipStream_t)stream;
    if (!kv4_seqs_ok(kv, n_seqs, seq_ids) || !kv4_seqs_ok(kv, n_seqs, into)) return PIPESD_EINVAL;
    // a client is cut in place or into one that is not itself being cut
    std::vector<char> cut(kv->max_seqs, 0);
    for (int32_t i = 0; i < n_seqs; ++i) cut[seq_ids[i]] = 1;
    for (int32_t i = 0; i < n_seqs; ++i)
      if (into[i] != seq_ids[i] && cut[into[i]]) return PIPESD_EINVAL;
    int64_t have = (int64_t)kv->free_list.size();
    for (int32_t i = 0; i < n_seqs; ++i) {
      const int32_t len = kv->seqs[seq_ids[i]].len;
      if (len < keep) return PIPESD_ESTATE;
      if (len > mass_stride) return PIPESD_EINVAL;
      if (into[i] != seq_ids[i]) have += (int64_t)kv->seqs[into[i]].blocks.size();  // what the target holds is given up first
    }
    if (!kv->pool) return PIPESD_ESTATE;
    if (int rc = kv4_not_recorded(st)) return rc;
    const int32_t nb = kv4_blocks(keep);
    if ((int64_t)nb * n_seqs > have) return PIPESD_ENOMEM;

    std::vector<std::vector<int32_t>> fresh(n_seqs);
    for (auto& f : fresh) f.reserve(nb);
    for (int32_t i = 0; i < n_seqs; ++i)
      for (auto& sent : kv->seqs[into[i]].sent) sent.reserve(nb);
    for (int32_t i = 0; i < n_seqs; ++i)
      if (into[i] != seq_ids[i]) kv->seqs[into[i]].blocks.reserve(nb);
    std::vector<int32_t> from_off(n_seqs), len(n_seqs);
    for (int32_t i = 0; i < n_seqs; ++i) {
      from_off[i] = kv->table_off(seq_ids[i]);
      len[i] = kv->seqs[seq_ids[i]].len;
    }
    // what was in the targets is gone from here on, also if a launch fails: then they are empty, and clients cut in place whole
    bool touched = false;
    for (int32_t i = 0; i < n_seqs; ++i) touched |= kv->seqs[into[i]].in_pass;  // (a client copied into another stays as it is)
    if (touched) kv4_close_pass(kv);
    for (int32_t i = 0; i < n_seqs; ++i)
      if (into[i] != seq_ids[i]) kv4_release(kv, kv->seqs[into[i]], 0);
    std::vector<std::vector<int32_t>> old(n_seqs);
    for (int32_t i = 0; i < n_seqs; ++i) {
      Kv4Seq& t = kv->seqs[into[i]];
      for (int32_t b = 0; b < nb; ++b) {
        fresh[i].push_back(kv->free_list.back());
        kv->free_list.pop_back();
      }
      old[i].swap(t.blocks);
      t.blocks.swap(fresh[i]);
      t.which ^= 1;
      std::fill(t.sent[t.which].begin(), t.sent[t.which].end(), -1);
    }
    auto launch = [&]() -> int {
      if (int rc = kv4_send(kv, n_seqs, into, nullptr, st)) return rc;
      Kv4Cuts cuts;
      cuts.keep = keep;
      cuts.recent = recent;
      const int64_t per = (int64_t)kv->cfg.n_layers * kv->cfg.n_kv_heads * keep;
      for (int32_t i0 = 0; i0 < n_seqs; i0 += kKv4ClientsPerLaunch) {
        cuts.n = std::min(n_seqs - i0, kKv4ClientsPerLaunch);
        for (int32_t i = 0; i < cuts.n; ++i) {
          cuts.seq[i] = seq_ids[i0 + i];
          cuts.into[i] = into[i0 + i];
          cuts.len[i] = len[i0 + i];
          cuts.from_off[i] = from_off[i0 + i];
          cuts.to_off[i] = kv->table_off(into[i0 + i]);
        }
        HIP_TRY(launch_kv4_select(kv->view(), cuts, mass, mass_stride, kept + i0 * per, st));
        HIP_TRY(launch_kv4_move(kv->cfg.head_dim, kv->view(), cuts, kept + i0 * per, st));
      }
      return PIPESD_OK;
    };
    const int rc = launch();
    for (int32_t i = 0; i < n_seqs; ++i) {
      Kv4Seq& t = kv->seqs[into[i]];
      if (rc) {  // back to the blocks before
        t.blocks.swap(old[i]);
        t.which ^= 1;
      } else {
        t.len = keep;
      }
      for (int32_t b : old[i]) kv->free_list.push_back(b);
    }
    return rc;
  });
}
