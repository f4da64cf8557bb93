// The 4-bit cache: its layout, the plan of a pass, and the launchers.
//
// A value is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 or their negatives (e2m1: the magnitudes are the codes 0..7, 8 is the
// sign) times a power of two that 32 neighbouring channels of a token and head share; a power is a byte e + 127.  That is
// what the matrix cores multiply as it is.  All values are finite.
//
// Per (layer, block of 16 tokens, head of the cache) the pool holds one record: the codes of the keys, of the values, the
// powers of the keys, of the values.
//   keys          [token][head_dim / 2 bytes], the even channel in the low half.  Operand A of S^T = K Q^T (16 tokens x 128
//                 channels): lane (token, quarter) holds 32 channels, which share one power.
//   values        [token / 4][unit 0..15][token % 4][head_dim / 32 bytes]; unit r holds channels r * head_dim / 16 and on.
//                 Operand A of O^T = V^T P^T: lane (r, quarter g) holds its unit of the tokens 4g .. 4g + 3, side by side.
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
//   many tiles   each of four waves takes tiles of its own
constexpr int kKv4ManyTiles = 16;  // (from here on)
constexpr int kKv4WideWaves = 4;
constexpr int kv4_wide_tiles(int dtype, int head_dim) { return dtype == PIPESD_BF16 && head_dim == 64 ? 4 : 2; }  // of a wave
constexpr int kKv4MaxSplits = 64;
constexpr int kv4_few_waves(int tiles) { return tiles == 1 ? 8 : 4; }

// Clients of a launch, by value.  Workgroups: (cache head, item); a client's items are its splits, the groups of tiles of a
// split side by side, for they read the same tokens.
constexpr int kKv4ClientsPerLaunch = 32;
struct Kv4Clients {
  int32_t n, items, span;  // span: tokens of a split
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
  int32_t wide, tiles;  // tiles: of a workgroup (few), of a wave (many)
  Kv4Clients c;
};
struct Kv4PlanNeeds {
  size_t part_tiles, counters;
};

// One tile a workgroup or two.  Two share the conversion of keys and values (a step of 32 tokens takes 1.5 times as long, not
// twice), but leave registers for half the waves and twice the rows to join: measured on a device of 256 compute units, a
// launch takes 8 us + 0.14 us per step and compute unit of one tile, 14 us + 0.215 us of two (head dim 64: 0.086 and 0.10).
// Two in fp32 were never faster: 4 clients of 9 rows behind 4096 tokens 32.9 us, 21.9 with one.
inline int kv4_few_tiles(int dtype, int head_dim, double work1, double work2, int n_cu) {
  if (dtype == PIPESD_F32) return 1;
  const double one = head_dim == 128 ? 0.14 : 0.086, two = head_dim == 128 ? 0.215 : 0.10;
  return 8 + one * work1 / n_cu <= 14 + two * work2 / n_cu ? 1 : 2;
}

// The launches of a pass: clients of few and of many tiles apart, at most kKv4ClientsPerLaunch in one.  All splits of a kind
// are as long: as short as leaves the workgroups of the pass one round on the device, and no shorter than a step of the
// workgroup.  So what a row's sums are cut into depends on the pass, not on timing.
template <class Out>  // std::vector<Kv4Launch>
inline Kv4PlanNeeds kv4_plan(const Kv4Client* cl, int n, int dtype, int head_dim, int n_q_heads, int n_kv_heads, int n_cu, Out& out) {
  out.clear();
  const int group = n_q_heads / n_kv_heads;
  Kv4PlanNeeds need{0, 0};
  for (int wide = 0; wide < 2; ++wide) {
    auto tiles_of = [&](const Kv4Client& c) { return attn_query_tiles(group, c.n_rows); };
    auto mine = [&](const Kv4Client& c) { return c.n_rows > 0 && (tiles_of(c) >= kKv4ManyTiles) == (wide != 0); };
    int longest = 0;
    double work[3] = {0, 0, 0};  // [tiles]: steps of 32 tokens of all workgroups' sets of tiles
    for (int i = 0; i < n; ++i) {
      if (!mine(cl[i])) continue;
      longest = std::max(longest, (int)cl[i].len);
      for (int tiles = 1; tiles <= 2; ++tiles) work[tiles] += (double)n_kv_heads * ((tiles_of(cl[i]) + tiles - 1) / tiles) * cl[i].len / 32;
    }
    if (longest == 0) continue;
    int tiles, wg_tiles, step, resident = 2;  // resident: workgroups that a compute unit holds at once
    if (wide) {
      tiles = kv4_wide_tiles(dtype, head_dim);
      wg_tiles = kKv4WideWaves * tiles;
      step = 512;
      if (head_dim == 128 && dtype == PIPESD_F32) resident = 1;
    } else {
      tiles = kv4_few_tiles(dtype, head_dim, work[1], work[2], n_cu);
      wg_tiles = tiles;
      step = kv4_few_waves(tiles) * 32;
    }
    auto workgroups = [&](int64_t span) {
      int64_t w = 0;
      for (int i = 0; i < n; ++i)
        if (mine(cl[i])) w += (int64_t)n_kv_heads * ((tiles_of(cl[i]) + wg_tiles - 1) / wg_tiles) * ((cl[i].len + span - 1) / span);
      return w;
    };
    // (a split costs what joins it, about the time of three steps: none below 768 tokens)
    const int64_t room = (int64_t)resident * n_cu;
    int64_t span = std::max<int64_t>(step, longest <= 768 ? longest : 0);
    span = std::max<int64_t>(span, (int64_t)(workgroups(1) / room));  // (no shorter one would do)
    span = (span + step - 1) / step * step;
    while (workgroups(span) > room && span < longest) span += span < 16 * step ? step : span / 16 / step * step;
    span = std::max<int64_t>(span, ((longest + kKv4MaxSplits - 1) / kKv4MaxSplits + step - 1) / step * step);
    Kv4Launch l{};
    auto flush = [&] {
      if (l.c.n == 0) return;
      for (int i = l.c.n; i < kKv4ClientsPerLaunch; ++i) l.c.first[i] = l.c.items;
      out.push_back(l);
      l = Kv4Launch{};
    };
    for (int i = 0; i < n; ++i) {
      if (!mine(cl[i])) continue;
      if (l.c.n == kKv4ClientsPerLaunch) flush();
      const int j = l.c.n++;
      l.wide = wide;
      l.tiles = tiles;
      l.c.span = (int)span;
      l.c.first[j] = l.c.items;
      l.c.seq[j] = cl[i].seq;
      l.c.len[j] = cl[i].len;
      l.c.n_rows[j] = cl[i].n_rows;
      l.c.row_off[j] = cl[i].row_off;
      l.c.groups[j] = (tiles_of(cl[i]) + wg_tiles - 1) / wg_tiles;
      l.c.nsplit[j] = (int)((cl[i].len + span - 1) / span);
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
