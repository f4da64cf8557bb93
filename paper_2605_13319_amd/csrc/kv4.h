// The 4-bit cache: its layout, the plan of a pass, and the launchers.
//
// A value is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 or their negatives (e2m1: the magnitudes are the codes 0..7, 8 is the
// sign) times a power of two that 32 neighbouring channels of a token and head share; a power is a byte e + 127.  All values are
// finite, and exact as bf16 numbers.
//
// Per (layer, block of 16 tokens, head of the cache) the pool holds one record: the codes of the keys, of the values, the
// powers of the keys, of the values.
//   keys          [token][head_dim / 2 bytes], the even channel in the low half: a wave reads a block with one load, lane (token,
//                 quarter) its quarter of the channels, which at head_dim 128 share one power
//   values        [token / 4][unit 0..15][token % 4][head_dim / 32 bytes]; unit r holds channels r * head_dim / 16 and on.  Lane (r,
//                 quarter g) reads its unit of the tokens 4g .. 4g + 3, side by side: what pairs of tokens are made of
//   key powers    [token][head_dim / 32]
//   value powers  [token / 4][head_dim / 32][token % 4]: those of a lane's four tokens are one word
#pragma once

#include "common.h"

namespace pipesd {

constexpr int kKv4MaxRows = kMaxPromptRows;  // query rows of one client in a pass that attends

template <int HD>
struct Kv4Record {
  static constexpr int kUnit = HD / 32;  // bytes of a unit, and powers of a token
  static constexpr int kKeys = 0, kValues = kBlockTokens * HD / 2, kKeyPow = 2 * kValues, kValPow = kKeyPow + kBlockTokens * kUnit,
                       kBytes = kValPow + kBlockTokens * kUnit;
};
inline int kv4_record_bytes(int head_dim) { return head_dim == 128 ? Kv4Record<128>::kBytes : Kv4Record<64>::kBytes; }

struct Kv4View {
  uint8_t* pool;
  const int32_t* table;  // all clients' block tables [2 max_seqs][n_blocks]: one in use, one to build the next in
  int32_t n_blocks, n_layers, n_kv_heads;
};
template <int HD>
__device__ __forceinline__ int64_t kv4_record(const Kv4View& v, int layer, int blk, int kvh) {
  return (((int64_t)layer * v.n_blocks + blk) * v.n_kv_heads + kvh) * Kv4Record<HD>::kBytes;
}

// ---- the plan of a pass ------------------------------------------------------------------------
// A client's query rows are taken with the heads that share a head of the cache: row rr of a cache head is pass row rr /
// group, head rr % group of the group; 16 of them make a tile.
//   few tiles    the waves of a workgroup take every WAVES-th 32 tokens of a span for the same one or two tiles, and
//                join their sums
//   many tiles   each of four waves takes two tiles of its own, over tokens that they convert together
constexpr int kKv4WideWaves = 4;
constexpr int kKv4WideTiles = 2 * kKv4WideWaves;  // of a workgroup
constexpr int kKv4MaxSplits = 64;
// A client's last split takes up to so many tokens more than the others: a context of some power of two and a few new rows is not cut
// once more for the rows.
constexpr int kKv4SplitSlack = 64;
inline int kv4_splits(int64_t len, int64_t span) { return (int)std::max<int64_t>(1, (len - kKv4SplitSlack + span - 1) / span); }
constexpr int kv4_few_waves(int tiles) { return tiles == 1 ? 8 : 4; }

// Clients of a launch, by value.  Workgroups: (cache head, item); a client's items are its splits, the groups of tiles of a
// split side by side, for they read the same tokens.
constexpr int kKv4ClientsPerLaunch = 32;
constexpr int kKv4MaxItems = 65535;  // workgroups of a grid in y
struct Kv4Clients {
  int32_t n, items, span;  // span: tokens of a split
  int32_t apart;           // splits are joined by a kernel of their own, not by their last workgroup
  int32_t first[kKv4ClientsPerLaunch];  // item (beyond the last client: the number of items)
  int32_t seq[kKv4ClientsPerLaunch], table_off[kKv4ClientsPerLaunch], len[kKv4ClientsPerLaunch];  // len: with the pass's own rows
  int32_t n_rows[kKv4ClientsPerLaunch], row_off[kKv4ClientsPerLaunch];
  int32_t groups[kKv4ClientsPerLaunch], nsplit[kKv4ClientsPerLaunch];
  int32_t part_off[kKv4ClientsPerLaunch];   // tiles; the client's partials are [cache head][group][split][tiles of a workgroup]
  int32_t count_off[kKv4ClientsPerLaunch];  // arrival counters [cache head][group]
};
struct Kv4Client {
  int32_t seq, n_rows, row_off, len;
};
struct Kv4Launch {
  int32_t wide, tiles;  // tiles: of a workgroup
  Kv4Clients c;
};
struct Kv4PlanNeeds {
  size_t part_tiles, counters;
};

// What a launch takes on a device of 256 compute units, in us: `start`, and `step` for each 32 tokens of a workgroup's tiles and
// compute unit.  Two tiles in a workgroup share the conversion of keys and values, but leave registers for half the waves; eight share it
// through LDS, four times as many rows to join.  Measured, query heads 4 to a cache head: 4 clients of 8 rows behind 2048 tokens 13.5 us
// with one tile, 18.2 with two; 32 clients behind 4096 46.6 and 45.0; 32 rows behind 65536 tokens 67 with two, 71 with eight; 2048 rows behind 6144
// of head dim 64 225 with two, 186 with eight, of head dim 128 349 and 265.  Two in fp32 were never faster: 4 clients of 9 rows behind 4096 tokens 32.9 us, 21.9 with one.
struct Kv4Cost {
  double start, step;
};
constexpr Kv4Cost kv4_cost(int tiles, int dtype, int head_dim) {
  if (dtype == PIPESD_F32) {
    if (tiles == 2) return Kv4Cost{1e30, 1e30};
    if (tiles == 1) return head_dim == 128 ? Kv4Cost{12, 0.15} : Kv4Cost{10, 0.105};
    return head_dim == 128 ? Kv4Cost{25, 1.1} : Kv4Cost{18, 0.7};
  }
  if (tiles == 1) return head_dim == 128 ? Kv4Cost{8, 0.14} : Kv4Cost{8, 0.086};
  if (tiles == 2) return head_dim == 128 ? Kv4Cost{14, 0.185} : Kv4Cost{13, 0.12};
  return head_dim == 128 ? Kv4Cost{24, 0.6} : Kv4Cost{18, 0.39};
}

// The launches of a pass: clients of few and of many tiles apart, at most kKv4ClientsPerLaunch in one.  All splits of a kind
// are as long: as short as leaves the workgroups of the pass one round on the device, and no shorter than a step of the
// workgroup.  So what a row's sums are cut into depends on the pass, not on timing.
template <class Out>  // std::vector<Kv4Launch>
inline Kv4PlanNeeds kv4_plan(const Kv4Client* cl, int n, int dtype, int head_dim, int n_q_heads, int n_kv_heads, int n_cu, Out& out) {
  out.clear();
  const int group = n_q_heads / n_kv_heads;
  Kv4PlanNeeds need{0, 0};
  const Kv4Cost one = kv4_cost(1, dtype, head_dim), two = kv4_cost(2, dtype, head_dim), eight = kv4_cost(kKv4WideTiles, dtype, head_dim);
  auto tiles_of = [&](const Kv4Client& c) { return attn_query_tiles(group, c.n_rows); };
  auto sets = [&](const Kv4Client& c, int tiles) { return (tiles_of(c) + tiles - 1) / tiles; };
  // Many tiles: clients whose steps are cheaper so, if together they save what the other launch costs.
  auto gain = [&](const Kv4Client& c) { return std::min(one.step * sets(c, 1), two.step * sets(c, 2)) - eight.step * sets(c, kKv4WideTiles); };
  double saved = 0;
  bool few = false;
  for (int i = 0; i < n; ++i) {
    if (cl[i].n_rows > 0 && gain(cl[i]) > 0) saved += gain(cl[i]) * n_kv_heads * cl[i].len / 32 / n_cu;
    else few |= cl[i].n_rows > 0;
  }
  const bool any_wide = saved > eight.start - (few ? 0 : one.start);
  for (int wide = 0; wide < 2; ++wide) {
    auto mine = [&](const Kv4Client& c) { return c.n_rows > 0 && (any_wide && gain(c) > 0) == (wide != 0); };
    int longest = 0;
    double work1 = 0, work2 = 0;  // steps of 32 tokens of all workgroups, of one tile and of two
    for (int i = 0; i < n; ++i) {
      if (!mine(cl[i])) continue;
      longest = std::max(longest, (int)cl[i].len);
      work1 += (double)n_kv_heads * sets(cl[i], 1) * cl[i].len / 32;
      work2 += (double)n_kv_heads * sets(cl[i], 2) * cl[i].len / 32;
    }
    if (longest == 0) continue;
    int wg_tiles = kKv4WideTiles, step = 256, resident = 2;  // resident: workgroups that a compute unit holds at once
    if (wide) {
      if (head_dim == 128 && dtype == PIPESD_F32) resident = 1;
    } else {
      wg_tiles = one.start + one.step * work1 / n_cu <= two.start + two.step * work2 / n_cu ? 1 : 2;
      step = kv4_few_waves(wg_tiles) * 32;
    }
    auto workgroups = [&](int64_t span) {
      int64_t w = 0;
      for (int i = 0; i < n; ++i)
        if (mine(cl[i])) w += (int64_t)n_kv_heads * sets(cl[i], wg_tiles) * kv4_splits(cl[i].len, span);
      return w;
    };
    // (a split costs what joins it, about the time of three steps: none below 768 tokens)
    const int64_t room = (int64_t)resident * n_cu;
    int64_t span = std::max<int64_t>(step, longest <= 768 ? longest : 0);
    span = std::max<int64_t>(span, std::min<int64_t>(workgroups(1) / room, longest));  // (no shorter one would do)
    span = (span + step - 1) / step * step;
    while (workgroups(span) > room && span < longest) span += span < 16 * step ? step : span / 16 / step * step;
    span = std::max<int64_t>(span, ((longest + kKv4MaxSplits - 1) / kKv4MaxSplits + step - 1) / step * step);
    Kv4Launch l{};
    auto flush = [&] {
      if (l.c.n == 0) return;
      for (int i = l.c.n; i < kKv4ClientsPerLaunch; ++i) l.c.first[i] = l.c.items;
      for (int i = 0; i < l.c.n; ++i) {  // (few tiles: where the last workgroup would go to memory 4 times and more.  4 rows
        // behind 20000 tokens: 15.3 us apart, 17.2 not; 4 such clients, 2 times: 26.3 and 24.9)
        const int threads = kv4_few_waves(wg_tiles) * 64, tasks = std::min(group * l.c.n_rows[i], wg_tiles * 16) * (head_dim / 4);
        int shares = 1;
        while (2 * shares * tasks <= threads) shares *= 2;
        const int turns = (tasks + threads - 1) / threads * ((l.c.nsplit[i] + 8 * shares - 1) / (8 * shares));
        if (l.c.nsplit[i] > 1 && (wide || turns > 3)) l.c.apart = 1;
      }
      out.push_back(l);
      l = Kv4Launch{};
    };
    for (int i = 0; i < n; ++i) {
      if (!mine(cl[i])) continue;
      const int groups = sets(cl[i], wg_tiles), nsplit = kv4_splits(cl[i].len, span);
      if (l.c.n == kKv4ClientsPerLaunch || l.c.items + groups * nsplit > kKv4MaxItems) flush();
      const int j = l.c.n++;
      l.wide = wide;
      l.tiles = wg_tiles;
      l.c.span = (int)span;
      l.c.first[j] = l.c.items;
      l.c.seq[j] = cl[i].seq;
      l.c.len[j] = cl[i].len;
      l.c.n_rows[j] = cl[i].n_rows;
      l.c.row_off[j] = cl[i].row_off;
      l.c.groups[j] = groups;
      l.c.nsplit[j] = nsplit;
      l.c.items += l.c.groups[j] * l.c.nsplit[j];
      l.c.part_off[j] = (int)need.part_tiles;
      l.c.count_off[j] = (int)need.counters;
      need.counters += (size_t)n_kv_heads * l.c.groups[j];
      if (l.c.nsplit[j] > 1) need.part_tiles += (size_t)n_kv_heads * l.c.groups[j] * l.c.nsplit[j] * wg_tiles;
    }
    flush();
  }
  return need;
}

// block-table entries that changed, by value: no copy that the host would have to keep
constexpr int kKv4EntriesPerLaunch = 256;
struct Kv4TableUpdate {
  int32_t n;
  int32_t at[kKv4EntriesPerLaunch], v[kKv4EntriesPerLaunch];  // table[at[i]] = v[i]
};
hipError_t launch_kv4_table(const Kv4TableUpdate& u, int32_t* table, hipStream_t st);

// ---- the operators -----------------------------------------------------------------------------
struct Kv4Ranges {  // tokens of clients, and the rows that stand for them
  int32_t n, most;  // most: largest count
  int32_t table_off[kKv4ClientsPerLaunch], first[kKv4ClientsPerLaunch], count[kKv4ClientsPerLaunch], row_off[kKv4ClientsPerLaunch];
};
hipError_t launch_kv4_store(int dtype, int head_dim, const Kv4View& v, int layer, const Kv4Ranges& r, const void* k, const void* val,
                            int64_t k_stride, int64_t v_stride, hipStream_t st);
// out [n_layers][total_rows][n_kv_heads][head_dim]
hipError_t launch_kv4_read(int dtype, int head_dim, const Kv4View& v, int layer0, int n_layers, const Kv4Ranges& r, int64_t total_rows,
                           void* k, void* val, hipStream_t st);

struct Kv4AttendCall {
  Kv4View view;
  int dtype, head_dim, n_q_heads, group, layer;  // group: query heads of a cache head
  const void* q;
  void* out;
  int64_t q_stride, out_stride;  // elements between rows
  const int32_t* limits;         // tokens that each row sees, or nullptr: all up to its own
  float* part;
  unsigned* counters;
  float* lse;                    // [rows][n_q_heads], or nullptr: base-2 logarithm of each row's sum of weights
  // weights given to the cached tokens (launch_kv4_mass)
  float* mass;                   // [max_seqs][n_layers][n_kv_heads][mass_stride]
  int64_t mass_stride;
  float decay;
};
constexpr int kKv4PartPad = 4;  // a partial row is [head_dim values, max, sum, 2 unused]
hipError_t launch_kv4_attend(const Kv4AttendCall& c, const Kv4Launch& l, hipStream_t st);
hipError_t launch_kv4_mass(const Kv4AttendCall& c, const Kv4Clients& clients, hipStream_t st);

struct Kv4Cuts {
  int32_t n, keep, recent;
  int32_t seq[kKv4ClientsPerLaunch], into[kKv4ClientsPerLaunch], len[kKv4ClientsPerLaunch];
  int32_t from_off[kKv4ClientsPerLaunch], to_off[kKv4ClientsPerLaunch];  // entries to the tables of the old and of the new blocks
};
// kept [n][n_layers][n_kv_heads][keep]
hipError_t launch_kv4_select(const Kv4View& v, const Kv4Cuts& c, float* mass, int64_t mass_stride, int32_t* kept, hipStream_t st);
hipError_t launch_kv4_move(int head_dim, const Kv4View& v, const Kv4Cuts& c, const int32_t* kept, hipStream_t st);

}  // namespace pipesd
