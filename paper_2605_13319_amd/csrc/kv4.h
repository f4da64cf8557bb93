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
// group, head rr % group of the group; 16 of them make a tile.  Few tiles: the four waves of a workgroup take every fourth
// 32 tokens of a span for the same T tiles and join their sums.  Many tiles: each wave takes T tiles of its own.
constexpr int kKv4Waves = 4;
constexpr int kKv4TilesBf16 = 4, kKv4TilesF32 = 2;  // tiles of a wave at most
constexpr int kKv4ManyTiles = 16;  // from here on they do
constexpr int kKv4MaxSplits = 64;

struct Kv4Client {
  int32_t seq, n_rows, row_off, len;  // len: cached tokens, the pass's own rows included
  int32_t table_off;                  // entries to the client's block table
  int32_t wide, tiles, groups;        // tiles of a workgroup; workgroups for all tiles of a cache head
  int32_t span, nsplit;               // tokens of a split
  int32_t item_off, count_off;        // first item, first arrival counter
  int32_t part_off;                   // partial sums, in tiles of 16 rows
};
struct Kv4Item {  // one workgroup per cache head
  int32_t row_off, n_rows, len, table_off;
  int32_t group, groups, span, split;
  int32_t nsplit, part_off, count_off, seq;  // the client's: partials [cache head][group][split][tile], counters [cache head][group]
};

// The split of one client; its results do not depend on who shares the pass.
inline void kv4_plan_client(Kv4Client& c, int dtype, int n_q_heads, int n_kv_heads, int n_cu) {
  const int most = dtype == PIPESD_F32 ? kKv4TilesF32 : kKv4TilesBf16;
  const int nqt = std::max(1, attn_query_tiles(n_q_heads / n_kv_heads, c.n_rows));
  c.wide = nqt >= kKv4ManyTiles;
  c.tiles = c.wide ? kKv4Waves * most : std::min(nqt, most);
  c.groups = (nqt + c.tiles - 1) / c.tiles;
  const int step = c.wide ? 32 : kKv4Waves * 32;
  const int least = c.wide ? 512 : 128 * c.tiles;
  const long want = std::min<long>(kKv4MaxSplits, std::max<long>(1, 4L * n_cu / ((long)n_kv_heads * c.groups)));
  const long span = std::max<long>(least, (c.len + want - 1) / want);
  c.span = (int)((span + step - 1) / step * step);
  c.nsplit = std::max(1, (c.len + c.span - 1) / c.span);
}

// What begins a pass: block-table entries that changed and the clients, some per launch (by value: no copy that the host
// would have to keep).
constexpr int kKv4ClientsPerLaunch = 32, kKv4EntriesPerLaunch = 256;
struct Kv4PassUpdate {
  int32_t n_clients, n_entries;
  Kv4Client client[kKv4ClientsPerLaunch];
  int32_t at[kKv4EntriesPerLaunch], v[kKv4EntriesPerLaunch];  // table[at[i]] = v[i]
};
// where a new row goes, and whose it is
struct Kv4Row {
  int32_t table_off, pos;
};
hipError_t launch_kv4_begin(const Kv4PassUpdate& u, int32_t* table, Kv4Row* rows, Kv4Item* items, hipStream_t st);

// ---- the operators -----------------------------------------------------------------------------
hipError_t launch_kv4_store(int dtype, int head_dim, const Kv4View& v, int layer, int n_rows, const Kv4Row* rows, const void* k,
                            const void* val, int64_t k_stride, int64_t v_stride, hipStream_t st);

constexpr int kKv4SeqsPerLaunch = 64;
struct Kv4Ranges {
  int32_t n;
  int32_t table_off[kKv4SeqsPerLaunch], first[kKv4SeqsPerLaunch], count[kKv4SeqsPerLaunch], row_off[kKv4SeqsPerLaunch];
  int32_t most;  // largest count
};
// out [n_layers][total_rows][n_kv_heads][head_dim]
hipError_t launch_kv4_read(int dtype, int head_dim, const Kv4View& v, int layer0, int n_layers, const Kv4Ranges& r, int64_t total_rows,
                           void* k, void* val, hipStream_t st);

struct Kv4AttendCall {
  Kv4View view;
  int dtype, head_dim, n_q_heads, layer;
  const void* q;
  void* out;
  int64_t q_stride, out_stride;  // elements between rows
  const int32_t* limits;         // tokens that each row sees, or nullptr: all up to its own
  const Kv4Item* items;
  int32_t item0, n_items;        // this launch's
  int32_t wide, tiles;
  float* part;
  unsigned* counters;
  float* lse;                    // [rows][n_q_heads], or nullptr: base-2 logarithm of each row's sum of weights
  // weights given to the cached tokens (launch_kv4_mass; clients one after the other)
  float* mass;                   // [max_seqs][n_layers][n_kv_heads][mass_stride]
  int64_t mass_stride;
  float decay;
};
constexpr int kKv4PartPad = 4;  // a partial row is [head_dim values, max, sum, 2 unused]
hipError_t launch_kv4_attend(const Kv4AttendCall& c, hipStream_t st);

struct Kv4MassClients {
  int32_t n, most;  // most: the largest len
  int32_t seq[kKv4SeqsPerLaunch], table_off[kKv4SeqsPerLaunch], n_rows[kKv4SeqsPerLaunch], row_off[kKv4SeqsPerLaunch], len[kKv4SeqsPerLaunch];
};
hipError_t launch_kv4_mass(const Kv4AttendCall& c, const Kv4MassClients& clients, hipStream_t st);

struct Kv4Cuts {
  int32_t n, keep, recent;
  int32_t seq[kKv4SeqsPerLaunch], into[kKv4SeqsPerLaunch], len[kKv4SeqsPerLaunch];
  int32_t from_off[kKv4SeqsPerLaunch], to_off[kKv4SeqsPerLaunch];  // entries to the tables of the old and of the new blocks
};
// kept [n][n_layers][n_kv_heads][keep]
hipError_t launch_kv4_select(const Kv4View& v, const Kv4Cuts& c, float* mass, int64_t mass_stride, int32_t* kept, hipStream_t st);
hipError_t launch_kv4_move(int head_dim, const Kv4View& v, const Kv4Cuts& c, const int32_t* kept, hipStream_t st);

}  // namespace pipesd
