// The paged cache of operators in the model's own type: its layout, the plan of a pass, and the launchers.
//
// A block holds 16 tokens, as the model's own cache does (KvView): per layer all key blocks [kv_head][token][head_dim], then all
// value blocks [kv_head][head_dim][token].  Blocks may belong to several clients: what writes gets its own first.
#pragma once

#include <math.h>
#include "common.h"

namespace pipesd {

constexpr int kPagesMaxRows = kMaxPromptRows;  // query rows of one client in a pass that attends
constexpr int kPagesTreeRows = 256;            // and of a tree
constexpr int kPagesUsualRows = 64;            // what creation provides for, of 16 clients
// What a row of a tree sees of its pass: a bit a token, 32 neighbours (as the walk over the cache takes them) a word, from the 32 on
// that the pass begins in; tokens before the pass have theirs set.
constexpr int kPagesMaskWords = (31 + kPagesTreeRows + 31) / 32;

// ---- the plan of a pass ------------------------------------------------------------------------
// A client's query rows are taken with the heads that share a head of the cache: row rr of a cache head is pass row rr /
// group, head rr % group of the group; 16 of them make a tile.  A workgroup has `tiles` of them, of one client and cache head, and a
// span of the context.
constexpr int kPagesFewWaves = 8;  // of a workgroup of one or two tiles
constexpr int kPagesWaves = 4;     // of one of more
constexpr int kPagesStep = 128;    // spans are a multiple of so many tokens
constexpr int kPagesMaxSplits = 64;
// a client's last split takes up to so many tokens more than the others
constexpr int kPagesSplitSlack = 64;
inline int pages_splits(int64_t len, int64_t span) { return (int)std::max<int64_t>(1, (len - kPagesSplitSlack + span - 1) / span); }
constexpr int kPagesCutRounds = 4;  // workgroups whose rows are to be joined, in rounds that fill the device: bounds the partial rows

constexpr int kPagesPartPad = 4;  // a partial row is [head_dim values, max, sum, 2 unused]
constexpr int kPagesPerLaunch = 32;     // clients of a launch, by value
constexpr int kPagesMaxItems = 65535;   // workgroups of a grid in y
struct PagesClients {
  int32_t n, items, span;               // span: tokens of a split
  int32_t apart;                        // splits are joined by a kernel of their own, not by their last workgroup
  int32_t first[kPagesPerLaunch];       // item (beyond the last client: the number of items)
  int32_t table_off[kPagesPerLaunch], len[kPagesPerLaunch];  // len: with the pass's own rows
  int32_t n_rows[kPagesPerLaunch], row_off[kPagesPerLaunch];
  int32_t groups[kPagesPerLaunch], nsplit[kPagesPerLaunch];
  int32_t part_off[kPagesPerLaunch];    // tiles; the client's partials are [cache head][group][split][tiles of a workgroup]
  int32_t count_off[kPagesPerLaunch];   // arrival counters [cache head][group]
};
struct PagesClient {
  int32_t seq, n_rows, row_off, len, table_off;
};
struct PagesLaunch {
  int32_t tiles;
  PagesClients c;
};
struct PagesNeeds {
  size_t part_tiles, counters;
};

// What workgroups of one, two, four and eight tiles take: tokens of a step, its time in us on a compute unit by itself and with as many
// workgroups as one holds, and what a workgroup's beginning and end add.  One or two tiles ask for as much as a compute unit gets (58 GB/s).
// Fitted to 8 heads of 128: 4096 tokens more of one client 36, 38, 78 and 107 us with 8 workgroups; 64 rows behind 32768 75 us with
// 512 of four tiles, 70 with 512 of eight, 78 with 256 of them.  Heads of 64: 9 rows behind 65536, 43.5 us where two groups of two tiles
// walk them, 39 with one of four.
struct PagesCost {
  int tokens, resident;
  double alone, full, begin;
};
constexpr int kPagesTiles[4] = {1, 2, 4, 8};
constexpr PagesCost pages_cost(int tiles, int dtype, int head_dim) {
  const double part = head_dim == 128 ? 1 : tiles <= 2 ? 0.5 : 0.75;  // (the weights' instructions do not get fewer)
  if (dtype == PIPESD_F32) return tiles == 1 ? PagesCost{128, 1, 2.9 * part, 2.9 * part, 3.5} : tiles == 2 ? PagesCost{128, 1, 4.5 * part, 4.5 * part, 5.5} : PagesCost{32, 1, 1e30, 1e30, 5};
  if (tiles == 1) return PagesCost{256, 1, 2.25 * part, 2.25 * part, 3.5};
  if (tiles == 2) return PagesCost{256, 1, 2.35 * part, 2.35 * part, 5.5};
  if (tiles == 4) return PagesCost{64, 2, 1.3 * part, 1.7 * part, 5};
  return PagesCost{32, 2, 0.92 * part, 1.6 * part, 5};
}
constexpr double kPagesLaunchUs = 2, kPagesJoinUs = 3, kPagesApartUs = 4;  // a launch; what joins splits, in the last workgroup and apart
constexpr double kPagesMemory = 5.8e6, kPagesCaches = 12e6, kPagesParts = 3.5e6;  // bytes a us: of the cache once, again, of partial rows (there and back)

// Whether splits of `rows` query rows of a cache head are joined by a kernel of their own: always those of more than two tiles, others
// where the last workgroup would go to memory 4 times and more.
inline bool pages_apart(int tiles, int64_t rows, int nsplit, int head_dim) {
  if (nsplit == 1 || tiles > 2) return nsplit > 1;
  const int threads = kPagesFewWaves * 64, tasks = (int)std::min<int64_t>(rows, tiles * 16) * (head_dim / 4);
  int shares = 1;
  while (2 * shares * tasks <= threads) shares *= 2;
  return (tasks + threads - 1) / threads * ((nsplit + 8 * shares - 1) / (8 * shares)) > 3;
}

// What joins splits apart: workgroups per cache head, for the groups that have splits (kPagesCutRounds bounds them, however many others
// there are), and threads that share the splits of 4 channels: more while one would go to memory again, up to 8, or 1024 workgroups.
struct PagesJoin {
  int32_t log_shares;
  int32_t first[kPagesPerLaunch];  // workgroup of a client (of one without splits: the next one's)
};
inline int pages_join_plan(const PagesClients& c, int rows, int head_dim, PagesJoin* join) {
  int groups = 0, most = 1;
  for (int i = 0; i < c.n; ++i)
    if (c.nsplit[i] > 1) groups += c.groups[i], most = std::max(most, c.nsplit[i]);
  int per_group = rows / (1024 / head_dim), log = 0, wgs = 0;
  while (log < 3 && most > 8 << log && 2 * groups * per_group <= 1024) per_group *= 2, ++log;
  join->log_shares = log;
  for (int i = 0; i < kPagesPerLaunch; ++i) {
    join->first[i] = wgs;
    if (i < c.n && c.nsplit[i] > 1) wgs += c.groups[i] * per_group;
  }
  return wgs;
}

// The launches of a pass, at most kPagesPerLaunch clients in one.  All splits are as long, some part of the longest context: as short
// as pays for what begins and joins them, in rounds of workgroups that fill the device.  So what a row's sums are cut into depends on
// the pass, not on timing.
template <class Out>  // std::vector<PagesLaunch>
inline PagesNeeds pages_plan(const PagesClient* cl, int n, int dtype, int head_dim, int n_q_heads, int n_kv_heads, int n_cu, Out& out) {
  out.clear();
  const int group = n_q_heads / n_kv_heads;
  PagesNeeds need{0, 0};
  auto sets = [&](const PagesClient& c, int tiles) { return ((int64_t)group * c.n_rows + 16 * tiles - 1) / (16 * tiles); };
  int longest = 0;
  double once = 0;  // tokens of all clients and heads
  for (int i = 0; i < n; ++i)
    if (cl[i].n_rows > 0) longest = std::max(longest, (int)cl[i].len), once += (double)n_kv_heads * cl[i].len;
  if (longest == 0) return need;
  const double token_bytes = 2. * head_dim * (dtype == PIPESD_F32 ? 4 : 2), row_bytes = 4. * (head_dim + kPagesPartPad);
  auto best = [&](int tiles, int64_t* span) {
    PagesCost cost = pages_cost(tiles, dtype, head_dim);
    const int64_t room = (int64_t)cost.resident * n_cu, cut = std::max<int64_t>(1, longest - kPagesSplitSlack);
    double walked = 0, worked = 0, time = 1e300;  // tokens: walked by all workgroups, and by waves that have rows
    for (int i = 0; i < n; ++i) {
      const double tokens = (double)n_kv_heads * cl[i].len;
      walked += tokens * sets(cl[i], tiles);
      worked += tokens * (((int64_t)group * cl[i].n_rows + 31) / 32 * 2) / tiles;
    }
    // (waves of eight tiles that have no rows leave the compute unit to others: 16 clients of up to 33 rows behind up to 4096 49 us, 52 with
    // four tiles)
    if (tiles == 8) cost.full = cost.alone + (cost.full - cost.alone) * worked / walked;
    // (workgroups that walk the same tokens do it side by side: what the second one asks for is often not in the caches yet)
    const double memory = std::max(once / kPagesMemory + std::min(once, walked - once) / kPagesCaches, walked / kPagesCaches) * token_bytes;
    int64_t last = 0;
    for (int halves = 2; halves <= 2 * kPagesMaxSplits; halves += halves < 16 ? 1 : 2) {  // half parts of the longest context
      const int64_t s = ((2 * cut + halves - 1) / halves + kPagesStep - 1) / kPagesStep * kPagesStep;
      if (s == last) continue;
      last = s;
      int64_t groups = 0, cut_groups = 0;
      double cut_rows = 0;
      bool apart = false;
      for (int i = 0; i < n; ++i) {
        if (cl[i].n_rows == 0) continue;
        const int nsplit = pages_splits(cl[i].len, s);
        const int64_t g = (int64_t)n_kv_heads * sets(cl[i], tiles) * nsplit;
        groups += g;
        if (nsplit > 1) cut_groups += g, cut_rows += (double)n_q_heads * cl[i].n_rows * nsplit;
        apart = apart || pages_apart(tiles, (int64_t)group * cl[i].n_rows, nsplit, head_dim);
      }
      if (cut_groups > kPagesCutRounds * room) break;  // (more still with shorter ones)
      const double walk = std::max(1., (double)std::min<int64_t>(s + kPagesSplitSlack, longest) / cost.tokens);
      // rounds of workgroups that all walk as far as the longest does, or all walks shared evenly and then one of the longest
      const int64_t rounds = groups / room, left = groups % room;
      const double by_rounds = rounds * (walk * cost.full + cost.begin) + (left ? walk * (left <= n_cu ? cost.alone : cost.full) + cost.begin : 0);
      const double by_tokens = walked / cost.tokens * cost.full / room + walk * cost.alone + (1 + (double)groups / room) * cost.begin;
      const double walks = n > 1 ? std::min(by_rounds, by_tokens) : by_rounds;
      // (work and memory that take as long do not quite run side by side)
      const double t = kPagesLaunchUs + sqrt(sqrt(walks * walks * walks * walks + memory * memory * memory * memory)) +
                       (s >= cut ? 0 : !apart ? kPagesJoinUs : kPagesApartUs + cut_rows * row_bytes / kPagesParts);
      if (t < time) time = t, *span = s;
    }
    return time;
  };
  int tiles = 1;
  int64_t span = 0;
  double time = 1e300;
  for (int k : kPagesTiles) {
    int64_t its = 0;
    const double t = best(k, &its);
    if (t < time) time = t, tiles = k, span = its;
  }
  PagesLaunch l{};
  auto flush = [&] {
    if (l.c.n == 0) return;
    for (int i = l.c.n; i < kPagesPerLaunch; ++i) l.c.first[i] = l.c.items;
    for (int i = 0; i < l.c.n; ++i)
      if (pages_apart(tiles, (int64_t)group * l.c.n_rows[i], l.c.nsplit[i], head_dim)) l.c.apart = 1;
    out.push_back(l);
    l = PagesLaunch{};
  };
  for (int i = 0; i < n; ++i) {
    if (cl[i].n_rows == 0) continue;
    const int groups = (int)sets(cl[i], tiles), nsplit = pages_splits(cl[i].len, span);
    if (l.c.n == kPagesPerLaunch || (int64_t)l.c.items + (int64_t)groups * nsplit > kPagesMaxItems) flush();
    const int j = l.c.n++;
    l.tiles = tiles;
    l.c.span = (int)span;
    l.c.first[j] = l.c.items;
    l.c.table_off[j] = cl[i].table_off;
    l.c.len[j] = cl[i].len;
    l.c.n_rows[j] = cl[i].n_rows;
    l.c.row_off[j] = cl[i].row_off;
    l.c.groups[j] = groups;
    l.c.nsplit[j] = nsplit;
    l.c.items += groups * nsplit;
    l.c.part_off[j] = (int)need.part_tiles;
    l.c.count_off[j] = (int)need.counters;
    need.counters += (size_t)n_kv_heads * groups;
    if (nsplit > 1) need.part_tiles += (size_t)n_kv_heads * groups * nsplit * tiles;
  }
  flush();
  return need;
}

// At least what pages_plan needs for any pass of up to `clients` clients of up to `rows` rows and `len` tokens each.
inline PagesNeeds pages_plan_most(int clients, int rows, int64_t len, int dtype, int head_dim, int n_q_heads, int n_kv_heads, int n_cu) {
  const int64_t all = ((int64_t)(n_q_heads / n_kv_heads) * rows + 15) / 16;
  const int64_t splits = std::min<int64_t>(kPagesMaxSplits, pages_splits(len, kPagesStep));
  size_t most = 0;
  for (int tiles : kPagesTiles) {
    const int64_t cut = std::min<int64_t>((int64_t)clients * n_kv_heads * ((all + tiles - 1) / tiles) * splits,
                                          (int64_t)kPagesCutRounds * pages_cost(tiles, dtype, head_dim).resident * n_cu);
    if (splits > 1) most = std::max(most, (size_t)(cut * tiles));
  }
  return PagesNeeds{most, (size_t)clients * n_kv_heads * all};
}

// ---- bookkeeping on the device -----------------------------------------------------------------
// Entries of the block tables that changed, blocks that are copied and the trees of a pass, by value: no copy that the host would have
// to keep.
constexpr int kPagesEntriesPerLaunch = 128;
constexpr int kPagesParentsPerLaunch = 1024;
constexpr int kPagesOwnPerLaunch = 32;
struct PagesBegin {
  int32_t own;                                                      // blocks that clients get for one that others hold as well
  int32_t own_from[kPagesOwnPerLaunch], own_to[kPagesOwnPerLaunch];
  int32_t n;                                                        // entries
  int32_t at[kPagesEntriesPerLaunch], v[kPagesEntriesPerLaunch];    // table[at[i]] = v[i]
  int32_t trees;
  int32_t row_off[kPagesPerLaunch], n_rows[kPagesPerLaunch], before[kPagesPerLaunch];  // before: tokens in front of the pass
  int16_t parent[kPagesParentsPerLaunch];                           // the trees' rows one after the other: within the tree, -1 for none
};
hipError_t launch_pages_begin(int dtype, const KvView& v, int n_layers, const PagesBegin& b, int32_t* table, uint32_t* masks, hipStream_t st);
// rows of block tables copied on the device
struct PagesForks {
  int32_t n, most;
  int32_t from[kPagesPerLaunch], to[kPagesPerLaunch], blocks[kPagesPerLaunch];
};
hipError_t launch_pages_fork(const PagesForks& f, int32_t* table, hipStream_t st);

// ---- the operators -----------------------------------------------------------------------------
struct PagesRanges {  // tokens of clients, and the rows that stand for them
  int32_t n, most;    // most: blocks that the longest touches
  int32_t table_off[kPagesPerLaunch], first[kPagesPerLaunch], count[kPagesPerLaunch], row_off[kPagesPerLaunch];
};
hipError_t launch_pages_store(int dtype, const KvView& v, int layer, const PagesRanges& r, const void* k, const void* val, int64_t k_stride,
                              int64_t v_stride, hipStream_t st);
// out [n_layers][total_rows][n_kv_heads][head_dim]
hipError_t launch_pages_read(int dtype, const KvView& v, int layer0, int n_layers, const PagesRanges& r, int64_t total_rows, void* k, void* val,
                             hipStream_t st);
// Tokens from place to place (block * 16 + token) in all layers; all of a launch are read before any is written by the same workgroup,
// which has them all for its channels.
constexpr int kPagesMovesPerLaunch = 448;
struct PagesMoves {
  int32_t n;
  int32_t from[kPagesMovesPerLaunch], to[kPagesMovesPerLaunch];
};
hipError_t launch_pages_move(int dtype, const KvView& v, int n_layers, const PagesMoves& m, hipStream_t st);
// whole blocks in all layers (from, to: blocks)
hipError_t launch_pages_copy(int dtype, const KvView& v, int n_layers, const PagesMoves& m, hipStream_t st);

struct PagesAttend {
  KvView view;
  int dtype, n_q_heads, group, layer;  // group: query heads of a cache head
  const void* q;
  void* out;
  int64_t q_stride, out_stride;        // elements between rows
  const uint32_t* masks;               // [rows][kPagesMaskWords], or nullptr: a row sees all up to its own
  float* part;
  unsigned* counters;
};
hipError_t launch_pages_attend(const PagesAttend& a, const PagesLaunch& l, hipStream_t st);

}  // namespace pipesd
