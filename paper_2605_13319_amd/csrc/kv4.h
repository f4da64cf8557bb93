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
//   few tiles    the eight waves of a workgroup take every eighth 32 tokens of a span for the same one or two tiles, and
//                join their sums
//   many tiles   each of four waves takes two tiles of its own, over tokens that they convert together
constexpr int kKv4WideWaves = 4;
constexpr int kKv4WideTiles = 2 * kKv4WideWaves;  // of a workgroup
constexpr int kKv4MaxSplits = 64;
// A client's last split takes up to so many tokens more than the others: a context of some power of two and a few new rows is not cut
// once more for the rows.
constexpr int kKv4SplitSlack = 64;
inline int kv4_splits(int64_t len, int64_t span) { return (int)std::max<int64_t>(1, (len - kKv4SplitSlack + span - 1) / span); }
constexpr int kKv4FewWaves = 8;
// Workgroups of a kind whose rows are to be joined, in rounds that fill the device: no pass has more, which bounds the partial rows.
// (By the cost below none of 60000 ragged passes would take more; with four, 193 of them would be cut less, and take up to 11 %
// longer.)
constexpr int kKv4CutRounds = 6;

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

// What workgroups of one, two or eight tiles take, in us: a launch (with what joins eight tiles' splits), a workgroup to begin and end, 32 tokens
// of it by compute unit with all `resident` workgroups that a compute unit holds, how much longer one takes alone, and a join.  Two
// tiles share the conversion of keys and values, but leave registers for half the workgroups; eight share it through LDS, four times as
// many rows to join.  Measured on the same inputs again and again, 4 query heads on each of 8 cache heads of 128: 32 clients of 8 rows
// behind 4096 tokens 37.7 us with one tile, 33.5 with two; 4 of 4 rows behind 20000 24.1 and 27.6; 32 rows behind 65536 65 with two, 67
// to 69 with eight; 64 rows 113 and 105; 2048 rows behind 6144 382 and 301 to 307, of head dim 64 276 and 197.  In fp32 2048 rows behind
// 2048 291 with one, 262 to 272 with eight; two were never faster, 4 clients of 9 rows behind 4096 tokens 32.9 and 21.9 with one (weights of
// 16 bits then; 22.1 now).  (40 cache heads, 4 clients of 17 rows behind 8192, inputs changing: 57.8; two tiles in four waves, two such
// workgroups to a compute unit, 52.9, but 10 to 15 % longer wherever the rounds fit.)
struct Kv4Cost {
  double start, begin, step, alone, join;
  int resident;
};
constexpr Kv4Cost kv4_cost(int tiles, int dtype, int head_dim) {
  const bool f32 = dtype == PIPESD_F32, wide = head_dim == 128;
  if (tiles == 1) return Kv4Cost{2, 2.5, f32 ? (wide ? 0.157 : 0.109) : (wide ? 0.14 : 0.08), 1.15, 3, 2};
  if (tiles == 2) return Kv4Cost{1, 7, f32 ? 1e30 : (wide ? 0.195 : 0.125), 1, 4, 1};
  return Kv4Cost{10, 5, f32 ? (wide ? 1.22 : 0.73) : (wide ? 0.6 : 0.39), f32 && wide ? 1. : 1.8, 5, f32 && wide ? 1 : 2};
}

// The launches of a pass: clients of few and of many tiles apart, at most kKv4ClientsPerLaunch in one.  All splits of a kind are as
// long, some part of the longest context: as short as pays for what begins and joins them, in rounds of workgroups that fill the
// device.  So what a row's sums are cut into depends on the pass, not on timing.
template <class Out>  // std::vector<Kv4Launch>
inline Kv4PlanNeeds kv4_plan(const Kv4Client* cl, int n, int dtype, int head_dim, int n_q_heads, int n_kv_heads, int n_cu, Out& out) {
  out.clear();
  const int group = n_q_heads / n_kv_heads;
  Kv4PlanNeeds need{0, 0};
  const Kv4Cost one = kv4_cost(1, dtype, head_dim), two = kv4_cost(2, dtype, head_dim), eight = kv4_cost(kKv4WideTiles, dtype, head_dim);
  auto tiles_of = [&](const Kv4Client& c) { return attn_query_tiles(group, c.n_rows); };
  auto sets = [&](const Kv4Client& c, int tiles) { return (tiles_of(c) + tiles - 1) / tiles; };
  // The best span for workgroups of `tiles`, and the time that it takes, of the clients that `mine` picks: by rounds of workgroups that
  // all walk as far as the longest does.  Among many short contexts a long one is then not worth a cut, though the pass waits for
  // it.  So there is a second measure, all walks divided among the compute units and then one of the longest, and a span that takes
  // less than two thirds by it is taken instead.  (One context of 131072 tokens among 51 of 300, 40 heads of 128: 165 us, 754 uncut;
  // among 255, 8 heads: 77 and 616.)
  auto best = [&](int tiles, const Kv4Cost& cost, auto mine, int64_t* span) {
    const int64_t step = 32 * kKv4FewWaves, room = (int64_t)cost.resident * n_cu;
    int longest = 0;
    double tokens = 0;  // that all workgroups walk
    for (int i = 0; i < n; ++i)
      if (mine(cl[i])) {
        longest = std::max(longest, (int)cl[i].len);
        tokens += (double)n_kv_heads * sets(cl[i], tiles) * cl[i].len;
      }
    double time = 1e300;
    int64_t last = 0;
    const int64_t cut = std::max<int64_t>(1, longest - kKv4SplitSlack);
    int64_t even_span = 0;
    double even = 1e300, even_least = 1e300;  // the second measure, of *span and of even_span
    bool rounds_end = false;                  // rounds of shorter spans are not tried
    // half parts of the longest context
    for (int halves = 2; halves <= 2 * kKv4MaxSplits; halves += rounds_end ? halves : halves < 16 ? 1 : 2) {
      const int64_t s = ((2 * cut + halves - 1) / halves + step - 1) / step * step;
      if (s == last) continue;
      last = s;
      int64_t groups = 0, cut_groups = 0;
      for (int i = 0; i < n; ++i)
        if (mine(cl[i])) {
          const int nsplit = kv4_splits(cl[i].len, s);
          const int64_t g = (int64_t)n_kv_heads * sets(cl[i], tiles) * nsplit;
          groups += g;
          if (nsplit > 1) cut_groups += g;
        }
      if (cut_groups > kKv4CutRounds * room) break;  // (more still with shorter ones)
      const double walk = std::min<double>(s, longest) / 32 * cost.step;
      const int64_t rounds = groups / room, left = groups % room;  // whole rounds, and what the last has
      const double t = cost.start + rounds * (walk * cost.resident + cost.begin) +
                       (left ? walk * (left <= n_cu ? cost.alone : cost.resident) + cost.begin : 0) + (s < cut ? cost.join : 0);
      const double t_even = n == 1 ? t : cost.start + tokens / 32 * cost.step / n_cu + walk * cost.alone + (1 + (double)groups / room) * cost.begin + (s < cut ? cost.join : 0);
      if (!rounds_end && t < time) time = t, *span = s, even = t_even;
      if (t_even < even_least) even_least = t_even, even_span = s;
      if (rounds > 3) {
        if (n == 1) break;
        rounds_end = true;
      }
    }
    if (even_least < 2. / 3 * std::min(even, time)) *span = even_span;
    return time;
  };
  // Many tiles: clients whose steps are cheaper so, if that pays for the other launch.
  auto all = [&](const Kv4Client& c) { return c.n_rows > 0; };
  auto many = [&](const Kv4Client& c) { return c.n_rows > 0 && eight.step * sets(c, kKv4WideTiles) < std::min(one.step * sets(c, 1), two.step * sets(c, 2)); };
  auto others = [&](const Kv4Client& c) { return c.n_rows > 0 && !many(c); };
  bool any = false, any_many = false, any_others = false;
  for (int i = 0; i < n; ++i) any |= all(cl[i]), any_many |= many(cl[i]), any_others |= others(cl[i]);
  if (!any) return need;
  int64_t span1 = 0, span2 = 0, span8 = 0;
  double time1 = best(1, one, all, &span1), time2 = best(2, two, all, &span2);
  bool any_wide = false;
  if (any_many) {
    int64_t s1 = 0, s2 = 0;
    const double t1 = any_others ? best(1, one, others, &s1) : 0, t2 = any_others ? best(2, two, others, &s2) : 0;
    any_wide = std::min(t1, t2) + best(kKv4WideTiles, eight, many, &span8) < std::min(time1, time2);
    if (any_wide) time1 = t1, time2 = t2, span1 = s1, span2 = s2;
  }
  for (int wide = 0; wide < 2; ++wide) {
    if (wide ? !any_wide : any_wide && !any_others) continue;
    auto mine = [&](const Kv4Client& c) { return c.n_rows > 0 && (any_wide && many(c)) == (wide != 0); };
    const int wg_tiles = wide ? kKv4WideTiles : time1 <= time2 ? 1 : 2;
    const int64_t span = wide ? span8 : wg_tiles == 1 ? span1 : span2;
    Kv4Launch l{};
    auto flush = [&] {
      if (l.c.n == 0) return;
      for (int i = l.c.n; i < kKv4ClientsPerLaunch; ++i) l.c.first[i] = l.c.items;
      for (int i = 0; i < l.c.n; ++i) {  // (few tiles: where the last workgroup would go to memory 4 times and more.  4 rows
        // behind 20000 tokens: 15.3 us apart, 17.2 not; 4 such clients, 2 times: 26.3 and 24.9)
        const int threads = kKv4FewWaves * 64, tasks = std::min(group * l.c.n_rows[i], wg_tiles * 16) * (head_dim / 4);
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

// At least what kv4_plan needs for any pass of up to `clients` clients of up to `rows` rows and `len` tokens each.
inline Kv4PlanNeeds kv4_plan_most(int clients, int rows, int64_t len, int dtype, int head_dim, int n_q_heads, int n_kv_heads, int n_cu) {
  const int all = attn_query_tiles(n_q_heads / n_kv_heads, rows);
  const int64_t splits = std::min<int64_t>(kKv4MaxSplits, kv4_splits(len, 32 * kKv4FewWaves));
  auto tiles = [&](int wg_tiles) {
    const int64_t sets = (all + wg_tiles - 1) / wg_tiles;
    const int64_t cut = std::min<int64_t>((int64_t)clients * n_kv_heads * sets * splits, (int64_t)kKv4CutRounds * kv4_cost(wg_tiles, dtype, head_dim).resident * n_cu);
    return splits > 1 ? (size_t)(cut * wg_tiles) : 0;
  };
  const double one = kv4_cost(1, dtype, head_dim).step, two = kv4_cost(2, dtype, head_dim).step, eight = kv4_cost(kKv4WideTiles, dtype, head_dim).step;
  const bool wide = eight < std::min(one * all, two * ((all + 1) / 2));  // (some client may have many tiles)
  return Kv4PlanNeeds{std::max(tiles(1), tiles(2)) + (wide ? tiles(kKv4WideTiles) : 0), (size_t)clients * n_kv_heads * all};
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
struct Kv4Idle {  // clients of a pass without rows: their weights are decayed, no more
  int32_t n, most;  // most: largest length
  int32_t seq[kKv4ClientsPerLaunch], len[kKv4ClientsPerLaunch];
};
hipError_t launch_kv4_decay(const Kv4AttendCall& c, const Kv4Idle& clients, hipStream_t st);

struct Kv4Cuts {
  int32_t n, keep, recent;
  int32_t seq[kKv4ClientsPerLaunch], into[kKv4ClientsPerLaunch], len[kKv4ClientsPerLaunch];
  int32_t from_off[kKv4ClientsPerLaunch], to_off[kKv4ClientsPerLaunch];  // entries to the tables of the old and of the new blocks
};
// kept [n][n_layers][n_kv_heads][keep]
hipError_t launch_kv4_select(const Kv4View& v, const Kv4Cuts& c, float* mass, int64_t mass_stride, int32_t* kept, hipStream_t st);
hipError_t launch_kv4_move(int head_dim, const Kv4View& v, const Kv4Cuts& c, const int32_t* kept, hipStream_t st);

}  // namespace pipesd
