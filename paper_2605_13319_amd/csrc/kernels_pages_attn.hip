// Attention of the rows of a pass over the paged cache of operators, chains and trees.
//
//   o_r = sum_t p_rt v_t,   p_rt = exp(s_rt) / sum_t' exp(s_rt'),   s_rt = q_r . k_t / sqrt(head_dim),
// over the tokens before the pass, the row's ancestors in it and the row itself.
//
// bf16: keys, values and queries are operands as they are; weights are cut into two bf16 numbers, 16 bits where results have 8, as in
// the other attentions of the library.  fp32: products of fp32 numbers on the matrix cores.  Maxima and sums are fp32.
//
// One pass over the cache with a running maximum and sum.  Few rows are bound by what a compute unit can ask for: keys and values go
// from memory into the registers that the products take them from, each wave has tokens of its own, and the waves' states are joined
// through LDS at the end.  Many rows are bound by products and exponentials: waves have rows of their own over tokens in LDS.  A context
// that is cut into splits is joined by the last workgroup that arrives, or by a kernel of its own.
#include "device_attend.h"
#include "device_dma.h"
#include "lds_limit.h"
#include "pages.h"

namespace pipesd {

struct PagesItem {
  int ci, group, split;
};
__device__ __forceinline__ PagesItem find_item(const PagesClients& cl, int item, int lane) {
  int ci = 0;
  if (cl.n > 1) ci = __popcll(__ballot(lane < kPagesPerLaunch && item >= cl.first[lane & (kPagesPerLaunch - 1)] && lane < cl.n)) - 1;
  ci = __builtin_amdgcn_readfirstlane(ci);
  const int i = item - cl.first[ci], groups = cl.groups[ci], split = div_by(i, __builtin_amdgcn_rcpf((float)groups));
  return PagesItem{ci, groups - 1 - (i - split * groups), split};  // (the last rows see most: first)
}

// What a workgroup knows of its client, and how rows leave it.
template <int HD, typename T>
struct PagesWork {
  const PagesAttend& a;
  int kvh, len, n_rows, row_off, nsplit, group_rows, first_row;  // group_rows: query rows of the cache head; first_row: the group's first
  float group_rinv;
  const int32_t* table;
  float* all;  // partial rows of the group's splits: [split][tiles of a workgroup][16][ROW]
  unsigned* counter;
  static constexpr int ROW = HD + kPagesPartPad;

  __device__ __forceinline__ PagesWork(const PagesAttend& call, const PagesClients& c, const PagesItem& it, int kvh_, int tiles)
      : a(call), kvh(kvh_), len(c.len[it.ci]), n_rows(c.n_rows[it.ci]), row_off(c.row_off[it.ci]), nsplit(c.nsplit[it.ci]) {
    group_rows = n_rows * a.group;
    first_row = it.group * tiles * 16;
    group_rinv = __builtin_amdgcn_rcpf((float)a.group);
    table = a.view.table + c.table_off[it.ci];
    all = a.part + ((size_t)c.part_off[it.ci] + ((size_t)kvh * c.groups[it.ci] + it.group) * nsplit * tiles) * (16 * ROW);
    counter = a.counters + c.count_off[it.ci] + kvh * c.groups[it.ci] + it.group;
  }
  __device__ __forceinline__ TileRow row(int rr) const { return tile_row(rr, a.group, group_rinv, n_rows, row_off, kvh); }

  static __device__ __forceinline__ float inverse(float l) {  // (a row sees itself: l is 0 only where all its scores are -inf, and then there is no number)
    const float inv = __builtin_amdgcn_rcpf(l);
    return inv * (2.f - l * inv);
  }
  static __device__ __forceinline__ void store(T* out, const f32x4& y) {
    if constexpr (sizeof(T) == 4) *(f32x4*)out = y;
    else *(uint2*)out = make_uint2(pack2_bf16(y[0], y[1]), pack2_bf16(y[2], y[3]));
  }
  __device__ __forceinline__ void finish(int rr, int e0, const f32x4& o, float l) const {  // 4 channels of a row: o / l
    const TileRow tr = row(rr);
    if (tr.live) store((T*)a.out + tr.row * a.out_stride + tr.head * HD + e0, o * inverse(l));
  }

  // The partial rows have been written through; whoever of the splits arrives last joins them.  All threads of the workgroup.
  __device__ __forceinline__ bool arrives_last(int* word) const {
    Xwg<true>::drain();
    __syncthreads();
    if (threadIdx.x == 0) {
      const unsigned prev = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      const int last = prev == (unsigned)nsplit - 1u;
      if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // ready for the next launch
      *word = last;
    }
    __syncthreads();
    return *word != 0;
  }
};

// The splits of a workgroup's rows joined.  Their maxima and sums come to LDS at once; each thread then has a task (a row, 4 channels),
// or several one after the other, and takes its splits 8 at a time.  Threads that the tasks leave over share the splits of a task:
// thread (share, task) takes splits share, share + shares, .., and the shares are joined through LDS in order.
template <int ROWS, int NT>
constexpr int join_floats() { return 2 * kPagesMaxSplits * ROWS + NT * 5; }
template <int HD, typename T, int ROWS, int NT>
__device__ __forceinline__ void join_splits(const PagesWork<HD, T>& wk, float* lds, int tid) {
  constexpr int BATCH = 8, TPR = HD / 4, ROW = HD + kPagesPartPad;
  const int rows_here = min(ROWS, wk.group_rows - wk.first_row), tasks = rows_here * TPR;
  f32x2* stats = (f32x2*)lds;                       // [split][row]
  float* joined = lds + 2 * kPagesMaxSplits * ROWS;  // [share][task] 4 sums, the sum of weights
  for (int i = tid; i < wk.nsplit * ROWS; i += NT)
    if (i % ROWS < rows_here) stats[i] = *(const f32x2*)(wk.all + (size_t)i * ROW + HD);
  int log_tasks = 31 - __builtin_clz(TPR);  // (their number made a power of two)
  while ((1 << log_tasks) < tasks) ++log_tasks;
  const int shares = max(1, NT >> log_tasks);
  __syncthreads();
#pragma unroll 1
  for (int k0 = 0; k0 < tasks; k0 += NT) {
    const int task = k0 + (tid & ((1 << log_tasks) - 1)), share = tid >> log_tasks;
    const int mr = min(task / TPR, rows_here - 1), e0 = (task % TPR) * 4;
    const float* p0 = wk.all + (size_t)mr * ROW + e0;
    float m = -INFINITY, l = 0.f;
#pragma unroll 4
    for (int sp = 0; sp < wk.nsplit; ++sp) m = fmaxf(m, stats[sp * ROWS + mr].x);
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int s0 = share; s0 < wk.nsplit; s0 += BATCH * shares) {
      f32x4 ob[BATCH];
#pragma unroll
      for (int j = 0; j < BATCH; ++j) ob[j] = *(const f32x4*)(p0 + (size_t)min(s0 + j * shares, wk.nsplit - 1) * (ROWS * ROW));
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        const int sp = s0 + j * shares;
        const f32x2 ml = stats[min(sp, wk.nsplit - 1) * ROWS + mr];
        if (sp < wk.nsplit && ml.x != -INFINITY) {
          const float sw = __builtin_amdgcn_exp2f(ml.x - m);
          l += ml.y * sw;
          o += ob[j] * sw;
        }
      }
    }
    if (shares > 1) {
      float* x = joined + (size_t)tid * 5;
      x[0] = o[0], x[1] = o[1], x[2] = o[2], x[3] = o[3], x[4] = l;
      __syncthreads();
      if (share == 0)
        for (int sh = 1; sh < shares; ++sh) {
          const float* y = joined + (size_t)((sh << log_tasks) + tid) * 5;
          o += f32x4{y[0], y[1], y[2], y[3]};
          l += y[4];
        }
    }
    if (share == 0 && task < tasks) wk.finish(wk.first_row + mr, e0, o, l);
  }
}

// States of waves that shared rows, [wave][row] in LDS, joined: rows of the result, or a split's partial rows (written
// through, unless a kernel of its own reads them).
template <int HD, typename T, int ROWS, int SHARES, int NT>
__device__ __forceinline__ void join_waves(const PagesWork<HD, T>& wk, int split, bool apart, const float* lds, int tid) {
  constexpr int TPR = HD / 4, ROW = HD + kPagesPartPad;
  const float(*states)[ROWS][ROW] = (const float(*)[ROWS][ROW])lds;
  const int tasks = min(ROWS, wk.group_rows - wk.first_row) * TPR;  // a task: (row, 4 channels)
#pragma unroll 1
  for (int task = tid; task < tasks; task += NT) {
    const int mr = task / TPR, e0 = (task % TPR) * 4;
    f32x2 ml[SHARES];
    float m = -INFINITY;
#pragma unroll
    for (int ww = 0; ww < SHARES; ++ww) {
      ml[ww] = *(const f32x2*)&states[ww][mr][HD];
      m = fmaxf(m, ml[ww].x);
    }
    const float m_ref = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ww = 0; ww < SHARES; ++ww) {
      const float sw = __builtin_amdgcn_exp2f(ml[ww].x - m_ref);
      l += ml[ww].y * sw;
      o += *(const f32x4*)&states[ww][mr][e0] * sw;
    }
    if (wk.nsplit == 1) {
      wk.finish(wk.first_row + mr, e0, o, l);
    } else {
      float* dst = wk.all + ((size_t)split * ROWS + mr) * ROW;
      const f32x4 stats = f32x4{partial_maximum(m, l), l, 0.f, 0.f};
      if (apart) {
        *(f32x4*)(dst + e0) = o;
        if (e0 == 0) *(f32x4*)(dst + HD) = stats;
      } else {
        Xwg<true>::st4f(dst + e0, o);
        if (e0 == 0) Xwg<true>::st4f(dst + HD, stats);
      }
    }
  }
}

typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
template <typename T>
__device__ __forceinline__ bool not_finite(T x) {
  if constexpr (sizeof(T) == 4) return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u;
  else return (x & 0x7f80u) == 0x7f80u;
}

// In a step that all rows see, an infinity is multiplied with both pieces of a bf16 model's weights, which is no number where the lower one
// is zero or of the other sign.  A wave whose sums are none comes by here with its states: such a sum holds a value that is not finite, so
// it is what all of those give, weighted once more.  (Lane (c, g): row c, channels 16 j + 4 g + ...  What it needs it finds again: registers
// that the walk kept for it would spill in the walk.)  8 heads of 128, 9 rows behind 2048 tokens: 11.3 us, 13.2 with an infinity, 22.5 with
// one in every 64th token, 106 where all values are NaN.  The test for it costs calls without any 0.1 to 0.3 us.
template <int HD, int TILES>
__device__ __forceinline__ void weigh_infinities(const PagesAttend& a, const PagesClients& clients, float* state, int first, int step, int end) {
  constexpr int HT = HD / 16, ROW = HD + kPagesPartPad;
  int lane = threadIdx.x & 63, item = blockIdx.y, kvh = blockIdx.x;
  asm volatile("" : "+v"(lane), "+s"(item), "+s"(kvh));  // (found again, not kept)
  const PagesWork<HD, uint16_t> wk(a, clients, find_item(clients, item, lane), kvh, TILES);
  const int c = lane & 15, g = lane >> 4, before = wk.len - wk.n_rows;
  const KvView& view = wk.a.view;
  const uint16_t* keys = (const uint16_t*)view.pool + (int64_t)wk.a.layer * view.layer_stride + (int64_t)wk.kvh * kBlockTokens * HD;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
  for (int t = 0; t < TILES; ++t) {
    const TileRow tr = wk.row(wk.first_row + t * 16 + c);
    const uint16_t* q = (const uint16_t*)wk.a.q + tr.row * wk.a.q_stride + tr.head * HD;
    float* mine = state + (t * 16 + c) * ROW;
    const float m = mine[HD];
    f32x4 o[HT];
#pragma unroll
    for (int j = 0; j < HT; ++j) {
      o[j] = *(f32x4*)(mine + j * 16 + 4 * g);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[j][e] = o[j][e] != o[j][e] ? 0.f : o[j][e];
    }
#pragma unroll 1
    for (int tok0 = first; tok0 < end; tok0 += step) {
      // bit x: a channel of token tok0 + x (lane: channels 16 j + c, tokens 8 g .. + 7)
      uint32_t odd = 0;
      const int piece = tok0 + 8 * g;
      const uint16_t* v = keys + view.v_offset + (int64_t)wk.table[piece < wk.len ? piece / kBlockTokens : 0] * view.block_elems + c * kBlockTokens + piece % kBlockTokens;
#pragma unroll 1
      for (int j = 0; j < HT; ++j) {
        const uint4 x = *(const uint4*)(v + j * 16 * kBlockTokens);
        const uint16_t* xs = (const uint16_t*)&x;
#pragma unroll
        for (int i = 0; i < 8; ++i) odd |= not_finite(xs[i]) && piece + i < wk.len ? 1u << (8 * g + i) : 0u;
      }
      uint32_t sees = ~0u;
      if (wk.a.masks == nullptr) {
        const int n = before + 1 + tr.row - wk.row_off - tok0;
        sees = n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
      } else if (tok0 >= (before & ~31)) {
        sees = wk.a.masks[(size_t)tr.row * kPagesMaskWords + min((tok0 - (before & ~31)) >> 5, kPagesMaskWords - 1)];
      }
#pragma unroll 1
      for (int tok = 0; tok < 32; ++tok) {
        if (__ballot((odd >> tok) & 1) == 0) continue;
        const uint16_t* key = keys + (int64_t)wk.table[(tok0 + tok) / kBlockTokens] * view.block_elems;
        const uint16_t* val = key + view.v_offset + (tok0 + tok) % kBlockTokens;
        key += (tok0 + tok) % kBlockTokens * HD;
        float score = 0.f;
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) {
          const k4u32x4 x = *(const k4u32x4*)(q + g * (HD / 4) + i * 8), y = *(const k4u32x4*)(key + g * (HD / 4) + i * 8);
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            score = fmaf(__uint_as_float(x[d] << 16), __uint_as_float(y[d] << 16), score);
            score = fmaf(__uint_as_float(x[d] & 0xffff0000u), __uint_as_float(y[d] & 0xffff0000u), score);
          }
        }
        const float p = __builtin_amdgcn_exp2f(fmaf(fold_groups(score, LaneAdd{}), attend_scale<HD>(), -m));
#pragma unroll
        for (int j = 0; j < HT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint16_t x = val[(j * 16 + 4 * g + e) * kBlockTokens];
            if (not_finite(x) && ((sees >> tok) & 1)) o[j][e] += p * bf16_bits_to_f32(x);
          }
      }
    }
#pragma unroll
    for (int j = 0; j < HT; ++j) *(f32x4*)(mine + j * 16 + 4 * g) = o[j];
  }
}

// ---- few rows: waves share one or two tiles of 16 ----
// Eight waves take every eighth step of the span, 32 tokens of bf16 numbers or 16 of fp32 ones.  Of a step a lane (c, g) has the scores of
// query row c with 8 or 4 tokens:
//   bf16  tokens 8 g .. + 7: what a product over 32 tokens takes of their weights, and of a channel's values with one load.  The
//         first four are row 4 g + .. of the first 16 x 16 product of keys, the others of the second: row r of product tt is token
//         8 (r / 4) + 4 tt + r % 4.
//   fp32  tokens 4 g .. + 3; a load of 4 channels of a key, or 4 tokens of a value, serves 4 products (k = 4).
// What bounds it: a compute unit gets 58 GB/s, with 4 waves asking as with 8: 256 tokens of 128 bf16 channels take 2.25 us for one tile
// and 2.35 for two, so two are taken where there are the rows.  fp32 products take as long as their operands' way: 128 tokens of 128
// channels 2.9 us for one tile, 4.5 for two, 3.4 of them products.  fp32 numbers cut into three bf16 pieces, for six bf16 products
// instead of one, took 4.2 in registers and 5.7 through LDS.
// 8 heads of 128, bf16: behind 2048 tokens 1 row 9.3 us, 9 rows 10.9, 64 rows 16.5 (launch, table, keys, 3 us to join: trips to memory
// one after the other); fp32: 1 row behind 2048 12.8, behind 131071 183 (5.9 TB/s).
// LDS: states [wave][row], later what joins the splits; then the queries that registers do not hold; a word
template <int HD, int TILES>
constexpr size_t state_floats() { return (size_t)TILES * kPagesFewWaves * 16 * (HD + kPagesPartPad); }
template <int HD, typename T, int TILES>
constexpr bool queries_in_lds() { return TILES * HD * (int)sizeof(T) > 512; }  // (more than 32 registers)
template <int HD, typename T, int TILES>
constexpr size_t attend_lds_bytes() {
  return state_floats<HD, TILES>() * sizeof(float) + (queries_in_lds<HD, T, TILES>() ? (size_t)TILES * HD * sizeof(T) * 16 : 0) + 16;
}
// sets of keys and values that a wave has on their way
template <int HD, typename T, int TILES>
constexpr int few_sets() { return sizeof(T) == 2 && TILES * HD > 128 ? 1 : 2; }

template <int HD, typename T, int TILES>
__global__ __launch_bounds__(kPagesFewWaves * 64, 2) void pages_attend_kernel(PagesAttend a, PagesClients clients) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int HT = HD / 16, ROW = HD + kPagesPartPad, WAVES = kPagesFewWaves, NT = WAVES * 64, SETS = few_sets<HD, T, TILES>();
  constexpr int NB = F32 ? 1 : 2, TOKENS = NB * kBlockTokens, STEP = WAVES * TOKENS;  // blocks and tokens of a wave's step; of the workgroup's
  constexpr int NX = 4 * NB;                   // scores of a lane
  constexpr int NK = F32 ? HD / 16 : HD / 32;  // 16-byte pieces of a key that a lane has
  constexpr int NV = HT;                       // and of values
  constexpr bool Q_LDS = queries_in_lds<HD, T, TILES>();
  extern __shared__ float lds[];
  int* word = (int*)((char*)lds + attend_lds_bytes<HD, T, TILES>() - 16);

  const int kvh = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, g = lane >> 4;
  const PagesItem it = find_item(clients, blockIdx.y, lane);
  const PagesWork<HD, T> wk(a, clients, it, kvh, TILES);
  const int len = wk.len, before = len - wk.n_rows, span0 = it.split * clients.span, first = span0 + w * TOKENS;

  // 64 steps' blocks sit in the lanes: lane L has those of step L
  int step_blk[NB];
  auto load_blocks = [&](int it0) {
#pragma unroll
    for (int tt = 0; tt < NB; ++tt) {
      const int64_t tok = (int64_t)first + (int64_t)(it0 + lane) * STEP + tt * 16;
      step_blk[tt] = wk.table[tok < len ? (int)(tok / kBlockTokens) : 0];
    }
  };
  load_blocks(0);

  // ---- queries, and how far the rows see ----
  // [piece]: the lane's part of the row, as its keys lie
  k4u32x4 q[Q_LDS ? 1 : TILES][NK];
  k4u32x4* q_lds = (k4u32x4*)(lds + state_floats<HD, TILES>()) + lane;
  int row_of[TILES];  // lane's column: row of the pass
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const TileRow tr = wk.row(wk.first_row + t * 16 + c);
    row_of[t] = tr.row;
    const char* part = (const char*)((const T*)a.q + tr.row * a.q_stride + tr.head * HD) + g * 16;
#pragma unroll
    for (int s = 0; s < NK; ++s) q[Q_LDS ? 0 : t][s] = *(const k4u32x4*)(part + s * 64);
    if constexpr (Q_LDS) {  // (the waves write the same)
#pragma unroll
      for (int s = 0; s < NK; ++s) q_lds[(t * NK + s) * 64] = q[0][s];
    }
  }
  auto query = [&](int t, int s) {
    if constexpr (Q_LDS) return q_lds[(t * NK + s) * 64];
    else return q[t][s];
  };
  // All rows see the first `lo` tokens, none sees any from `hi` on.
  int lo = before, hi = len;
  if (a.masks == nullptr) {
    lo = before + 1 + div_by(wk.first_row, wk.group_rinv);
    hi = before + 1 + div_by(min(wk.first_row + TILES * 16, wk.group_rows) - 1, wk.group_rinv);
  }
  const int end = min(it.split + 1 < wk.nsplit ? span0 + clients.span : len, hi);
  const int nsteps = end > first ? (end - first + STEP - 1) / STEP : 0;
  // which of a step's tokens a row sees
  auto seen = [&](int t, int tok0) -> uint32_t {
    if (a.masks != nullptr) {
      const int at = tok0 - (before & ~31);
      return a.masks[(size_t)row_of[t] * kPagesMaskWords + min(at >> 5, kPagesMaskWords - 1)] >> (at & 31);
    }
    const int n = before + 1 + row_of[t] - wk.row_off - tok0;
    return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
  };
  // (the first that are asked for travel with the keys)
  const int first_masked = first > lo - TOKENS ? 0 : (lo - TOKENS - first) / STEP + 1;
  uint32_t next_seen[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) next_seen[t] = first_masked < nsteps ? seen(t, first + first_masked * STEP) : 0u;

  Running<HT> run[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) run[t].clear();
  const float c1 = attend_scale<HD>();

  // Keys and values of a step travel from where those of the step before (or of the one before that, with registers for two) have been
  // used until they are.
  k4u32x4 k[SETS][NB][NK], v[SETS][NV];
  const char* head_base = (const char*)((const T*)a.view.pool + (int64_t)a.layer * a.view.layer_stride + (int64_t)kvh * kBlockTokens * HD);
  auto at_block = [&](int blk) { return head_base + (int64_t)blk * a.view.block_elems * (int)sizeof(T); };
  auto block_base = [&](int i, int tt) { return at_block(__builtin_amdgcn_readlane(step_blk[tt], i & 63)); };
  auto request_keys = [&](int i, int set) {
    if (i >= nsteps) return;
    if (i > 0 && (i & 63) == 0) load_blocks(i);
    if constexpr (F32) {
      const char* p = block_base(i, 0) + c * HD * 4 + g * 16;
#pragma unroll
      for (int s = 0; s < NK; ++s) k[set][0][s] = *(const k4u32x4*)(p + s * 64);
    } else {
      const char *b0 = block_base(i, 0), *b1 = block_base(i, 1);
#pragma unroll
      for (int tt = 0; tt < NB; ++tt) {
        const char* p = (c >> 3 ? b1 : b0) + (8 * ((c >> 2) & 1) + 4 * tt + (c & 3)) * HD * 2 + g * 16;
#pragma unroll
        for (int s = 0; s < NK; ++s) k[set][tt][s] = *(const k4u32x4*)(p + s * 64);
      }
    }
  };
  auto request_values = [&](int i, int set) {
    if (i >= nsteps) return;
    const int64_t off = a.view.v_offset * (int)sizeof(T);
    if constexpr (F32) {
      const char* p = block_base(i, 0) + off + c * 64 + g * 16;
#pragma unroll
      for (int j = 0; j < NV; ++j) v[set][j] = *(const k4u32x4*)(p + j * 1024);
    } else {
      const char *b0 = block_base(i, 0) + off, *b1 = block_base(i, 1) + off;
      const char* p = (g >> 1 ? b1 : b0) + c * 32 + (g & 1) * 16;
#pragma unroll
      for (int j = 0; j < NV; ++j) v[set][j] = *(const k4u32x4*)(p + j * 512);
    }
  };
  auto token_of = [&](int x) { return NX * g + x; };  // the lane's token of score x, of the step's

  // Values of tokens that not every row sees.  Behind the client's last token there may be anything: 0 instead.  A value that is not
  // finite must reach the rows that see its token and no other, but a product would take it times 0 to all: it becomes 0 here, too, and
  // `apart_of` has a bit for its token.
  auto drop_values = [&](k4u32x4 (&v)[NV], int tok0, uint32_t& apart_of) {
    uint32_t odd = 0;  // bit x: of the lane's token x
    if constexpr (F32) {
      uint32_t largest = 0;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (tok0 + token_of(i) >= len) v[j][i] = 0u;
          largest = max(largest, v[j][i] & 0x7fffffffu);
        }
      if (__ballot(largest >= 0x7f800000u) != 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if ((v[j][i] & 0x7f800000u) == 0x7f800000u) odd |= 1u << i, v[j][i] = 0u;
      }
    } else {
      if (tok0 + TOKENS > len) {
        const int n = min(8, max(0, len - tok0 - 8 * g));
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int j = 0; j < NV; ++j) v[j][d] &= n >= 2 * d + 2 ? ~0u : n == 2 * d + 1 ? 0xffffu : 0u;
      }
      u16x2 largest = u16x2{0, 0};
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int d = 0; d < 4; ++d) largest = __builtin_elementwise_max(largest, __builtin_bit_cast(u16x2, v[j][d] & 0x7fff7fffu));
      if (__ballot(max(largest.x, largest.y) >= 0x7f80) != 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const uint32_t bad = ((v[j][d] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;  // (an exponent of ones carries)
            if (bad & 0x8000u) odd |= 1u << (2 * d), v[j][d] &= 0xffff0000u;
            if (bad & 0x80000000u) odd |= 2u << (2 * d), v[j][d] &= 0xffffu;
          }
      }
    }
    apart_of = 0;
    if (__ballot(odd != 0) == 0) return;
#pragma unroll
    for (int x = 0; x < NX; ++x) {
      const unsigned long long who = __ballot((odd >> x) & 1);
#pragma unroll
      for (int gg = 0; gg < 4; ++gg)
        if ((who >> (16 * gg)) & 0xffff) apart_of |= 1u << (NX * gg + x);
    }
  };
  // those values, for the rows that see them (LDS: the wave's own states, which nobody reads before its walk has ended; the block is asked
  // for: the lanes may have the next 64 steps' already)
  float* scratch = lds + (size_t)w * TILES * 16 * ROW;
  auto add_apart = [&](Running<HT>& r, const float (&p)[NX], uint32_t sees, uint32_t apart_of, int tok0) {
#pragma unroll
    for (int x = 0; x < NX; ++x) scratch[c * 33 + token_of(x)] = p[x];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
    for (uint32_t left = apart_of; left != 0; left &= left - 1) {
      const int tok = __builtin_ctz(left);
      const T* from = (const T*)(at_block(wk.table[(unsigned)(tok0 + tok) / kBlockTokens]) + a.view.v_offset * (int)sizeof(T)) + tok % kBlockTokens;
      const float pt = scratch[c * 33 + tok];
#pragma unroll
      for (int j = 0; j < HT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const T x = from[(j * 16 + 4 * g + e) * kBlockTokens];
          if (not_finite(x) && ((sees >> tok) & 1)) r.acc[j][e] += pt * (F32 ? (float)x : bf16_bits_to_f32((uint16_t)x));
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };

#pragma unroll
  for (int set = 0; set < SETS; ++set) request_keys(set, set), request_values(set, set);
  auto step = [&](int i, auto which) {
    constexpr int SET = decltype(which)::value;
    const int tok0 = first + i * STEP;
    const bool masked = tok0 + TOKENS > lo;  // (of the wave) some row does not see all tokens
    f32x4 score[TILES][NB];
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int tt = 0; tt < NB; ++tt) score[t][tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < NK; ++s)
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const k4u32x4 qs = query(t, s);
        if constexpr (F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            score[t][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[SET][0][s][e]), __uint_as_float(qs[e]), score[t][0], 0, 0, 0);
        } else {
#pragma unroll
          for (int tt = 0; tt < NB; ++tt)
            score[t][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[SET][tt][s]), __builtin_bit_cast(bf16x8, qs), score[t][tt], 0, 0, 0);
        }
      }
    request_keys(i + SETS, SET);
    settle(score);
    float p[TILES][NX];
    uint32_t sees[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
#pragma unroll
      for (int x = 0; x < NX; ++x) p[t][x] = score[t][x >> 2][x & 3];
      if (masked) {
        sees[t] = next_seen[t];
        if (i + 1 < nsteps) next_seen[t] = seen(t, tok0 + STEP);
#pragma unroll
        for (int x = 0; x < NX; ++x)
          if (!((sees[t] >> token_of(x)) & 1)) p[t][x] = -INFINITY;
      }
      float top = max3(p[t][0], p[t][1], p[t][2]);
      if constexpr (NX == 8) top = max3(max3(top, p[t][3], p[t][4]), max3(p[t][5], p[t][6], p[t][7]), p[t][7]);
      else top = max3(top, p[t][3], p[t][3]);
      if (__ballot(top > run[t].moves) != 0) run[t].move_to(top, c1);
#pragma unroll
      for (int x = 0; x < NX; ++x) p[t][x] = __builtin_amdgcn_exp2f(fmaf(p[t][x], c1, run[t].neg_m));
#pragma unroll
      for (int x = 0; x < NX; x += 4) run[t].l += (p[t][x] + p[t][x + 1]) + (p[t][x + 2] + p[t][x + 3]);
    }
    uint32_t apart_of = 0;
    if (masked) drop_values(v[SET], tok0, apart_of);
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      if constexpr (F32) {
#pragma unroll
        for (int x = 0; x < NX; ++x)
#pragma unroll
          for (int j = 0; j < HT; ++j)
            run[t].acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[SET][j][x]), p[t][x], run[t].acc[j], 0, 0, 0);
      } else {
        unsigned pw[4][2];
#pragma unroll
        for (int d = 0; d < 4; ++d) split_weights(p[t][2 * d], p[t][2 * d + 1], pw[d]);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int j = 0; j < HT; ++j)
            run[t].acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v[SET][j]), __builtin_bit_cast(bf16x8, k4u32x4{pw[0][m], pw[1][m], pw[2][m], pw[3][m]}),
                                                                    run[t].acc[j], 0, 0, 0);
      }
    }
    settle(run);
    if (apart_of != 0) {
#pragma unroll
      for (int t = 0; t < TILES; ++t) add_apart(run[t], p[t], sees[t], apart_of, tok0);
    }
    request_values(i + SETS, SET);
  };
#pragma unroll 1
  for (int i = 0; i < nsteps; i += SETS) {
    step(i, std::integral_constant<int, 0>{});
    if constexpr (SETS == 2)
      if (i + 1 < nsteps) step(i + 1, std::integral_constant<int, 1>{});
  }
  bool none = false;  // (fp32 weights are one piece)
#pragma unroll
  for (int t = 0; !F32 && t < TILES; ++t) none |= run[t].no_number();
  float(*states)[TILES * 16][ROW] = (float(*)[TILES * 16][ROW])lds;  // [wave][row] its channels, its maximum and sum
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
#pragma unroll
    for (int j = 0; j < HT; ++j) *(f32x4*)&states[w][t * 16 + c][j * 16 + 4 * g] = run[t].acc[j];
    const float l = fold_groups(run[t].l, LaneAdd{});
    if (g == 0) *(f32x2*)&states[w][t * 16 + c][HD] = f32x2{partial_maximum(run[t].maximum(), l), l};
  }
  if constexpr (!F32) {
    if (__builtin_expect(lo > first && __ballot(none) != 0, 0)) weigh_infinities<HD, TILES>(a, clients, &states[w][0][0], first, STEP, end);
  }
  __syncthreads();
  join_waves<HD, T, TILES * 16, WAVES, NT>(wk, it.split, clients.apart, lds, tid);
  if (wk.nsplit == 1 || clients.apart || !wk.arrives_last(word)) return;
  static_assert(join_floats<TILES * 16, NT>() <= (int)state_floats<HD, TILES>(), "what joins fits the states' LDS");
  join_splits<HD, T, TILES * 16, NT>(wk, lds, tid);
}

// ---- many rows: waves have 32 rows each, over tokens that all of them read from LDS ----
// bf16, products of 32 x 32 x 16.  WR waves have different rows, the others the same rows over other tokens: a workgroup has WR * 32
// rows and takes 128 / WR tokens at a time (a stage).  Stages are copied from memory straight into a ring of LDS, one or two ahead: a wave
// copies the keys or the values of a block.
//
// Layout of a product: operand lane (r, h) holds row (column) r, k = 8 h .. + 7; the result's register 4 u + i holds row 8 u + 4 h + i
// of column r.  Row 8 a + 4 h + i of a block's keys is its token 8 h + 4 a + i: then a lane has the scores of 8 neighbouring tokens
// of each block, which is what a product takes of their weights, and of a channel's values with one read.
// What bounds it: a wave's chain of products, maximum, exponentials, products, 0.92 us for a stage of 32 tokens of 128 channels with one
// workgroup on a compute unit, 1.6 with two, where products alone take 0.32 each; scores of the next stage multiplied under this one's
// weights took 1.16.  Where 64 rows are enough, two waves over 32 other tokens take 1.3 and 1.7 us for 64 tokens.  8 heads of 128:
// 2048 rows behind 6144 347 us, 0.69 PFLOP/s, 1.04 with the weights' second product (a large bf16 product reaches 1.21); 9 rows
// behind 131071 102 us, 5.3 TB/s with the join.
// LDS of 32 tokens: [block][keys, values], as the pool has them but for the order of 16-byte pieces, in which lanes that read together
// find theirs in different banks: a key's piece c at c ^ (token), a channel's half u of its tokens at u ^ (channel / 4 % 2).
template <int HD, int WR>
struct Wide {
  static constexpr int kShares = kPagesWaves / WR, kRows = WR * 32, kTokens = kShares * 32;  // of a workgroup; of a stage
  static constexpr int kPart = kBlockTokens * HD * 2, kStage = kShares * 4 * kPart;          // bytes of a block's keys; of a stage
  static constexpr int kRing = WR == 4 ? 3 : 2;
  static constexpr size_t kStates = kShares > 1 ? (size_t)kShares * kRows * (HD + kPagesPartPad) * sizeof(float) : 0;
  static constexpr size_t kLds = kRing * kStage > (int)kStates ? kRing * kStage : kStates;
};

template <int HD, int WR>
__global__ __launch_bounds__(kPagesWaves * 64, 2) void pages_attend_wide_kernel(PagesAttend a, PagesClients clients) {
  typedef Wide<HD, WR> W;
  constexpr int KS = HD / 16, HT = HD / 32, ROW = HD + kPagesPartPad, SHARES = W::kShares, ROWS = W::kRows, STAGE = W::kTokens, RING = W::kRing;
  constexpr int COPIES = HD / 32;  // instructions, of 1 KB, for a block's keys
  extern __shared__ float lds[];

  const int kvh = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 31, h = lane >> 5, wr = w % WR, share = w / WR;
  const PagesItem it = find_item(clients, blockIdx.y, lane);
  const PagesWork<HD, uint16_t> wk(a, clients, it, kvh, ROWS / 16);
  const int len = wk.len, before = len - wk.n_rows, span0 = it.split * clients.span;

  // All rows of the workgroup see the first `lo` tokens, none sees any from `hi` on.
  int lo = before, hi = len;
  if (a.masks == nullptr) {
    lo = before + 1 + div_by(wk.first_row, wk.group_rinv);
    hi = before + 1 + div_by(min(wk.first_row + ROWS, wk.group_rows) - 1, wk.group_rinv);
  }
  const int end = min(it.split + 1 < wk.nsplit ? span0 + clients.span : len, hi);
  const int nstages = end > span0 ? (end - span0 + STAGE - 1) / STAGE : 0;

  // Copies: wave w has part w % 2 of block w / 2 of each 32 tokens.  64 stages' blocks sit in the lanes.
  const bool values = w & 1;
  int stage_blk[SHARES];
  auto load_blocks = [&](int it0) {
#pragma unroll
    for (int sh = 0; sh < SHARES; ++sh) {
      const int64_t tok = (int64_t)span0 + (int64_t)(it0 + lane) * STAGE + sh * 32 + (w >> 1) * 16;
      stage_blk[sh] = wk.table[tok < len ? (int)(tok / kBlockTokens) : 0];
    }
  };
  load_blocks(0);
  unsigned from[COPIES];  // lane's bytes in the part
#pragma unroll
  for (int i = 0; i < COPIES; ++i) {
    const int x = i * 64 + lane;  // where the piece lies in LDS
    constexpr int PPT = HD / 8;   // pieces of a token
    from[i] = values ? (x >> 1) * 32 + (((x & 1) ^ ((x >> 3) & 1)) << 4) : (x / PPT) * (HD * 2) + (((x % PPT) ^ (x / PPT % PPT)) << 4);
  }
  const char* part_base = (const char*)((const uint16_t*)a.view.pool + (int64_t)a.layer * a.view.layer_stride + (values ? a.view.v_offset : 0) +
                                        (int64_t)kvh * kBlockTokens * HD);
  const unsigned lds0 = (unsigned)(unsigned long long)(__attribute__((address_space(3))) char*)lds;
  auto copy = [&](int i) {
    if ((i & 63) == 0 && i > 0 && i < nstages) load_blocks(i);
    const unsigned to = lds0 + (i % RING) * W::kStage + w * W::kPart;
#pragma unroll
    for (int sh = 0; sh < SHARES; ++sh) {
      const char* p = part_base + (int64_t)__builtin_amdgcn_readlane(stage_blk[sh], i & 63) * a.view.block_elems * 2;
#pragma unroll
      for (int n = 0; n < COPIES; ++n) lds_dma16(p, from[n], to + sh * 4 * W::kPart + n * 1024);
    }
  };

  // queries as operand B
  const TileRow tr = wk.row(wk.first_row + wr * 32 + r);
  const bool idle = wk.first_row + wr * 32 >= wk.group_rows;  // (of the wave) there are no such rows
  k4u32x4 q[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) q[s] = *(const k4u32x4*)((const uint16_t*)a.q + tr.row * a.q_stride + tr.head * HD + s * 16 + h * 8);
  // Which of the 32 tokens from tok0 on the row sees.  The words of a tree of up to 97 rows come with the queries: a load in the walk
  // would wait for all copies.
  constexpr int AHEAD = 4;
  const uint32_t* words = a.masks + (size_t)tr.row * kPagesMaskWords;
  uint32_t early[AHEAD] = {0, 0, 0, 0};
  if (a.masks != nullptr) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) early[i] = words[i];
  }
  auto seen = [&](int tok0) -> uint32_t {
    if (a.masks == nullptr) {
      const int n = before + 1 + tr.row - wk.row_off - tok0;
      return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
    }
    const int at = (tok0 - (before & ~31)) >> 5;
    if (at < 0) return ~0u;
    if (at >= AHEAD) return words[min(at, kPagesMaskWords - 1)];
    uint32_t word = early[0];
#pragma unroll
    for (int i = 1; i < AHEAD; ++i) {
      word = at == i ? early[i] : word;
      asm("" : "+v"(word));  // (or the compiler makes a table of them in memory)
    }
    return word;
  };

  f32x16 acc[1][HT];
  float neg_m, moves, l;  // as of a Running
  auto maximum = [&] { return moves == -INFINITY ? -INFINITY : -neg_m; };
  const float c1 = attend_scale<HD>();

  // where the lane finds a key and a channel in a part
  const int kt = 8 * ((r >> 2) & 1) + 4 * ((r >> 3) & 1) + (r & 3);
  const unsigned key_at = (unsigned)((r >> 4) * 2 * W::kPart + kt * (HD * 2) + ((h ^ (kt % (HD / 8))) << 4));
  const unsigned value_at = (unsigned)(W::kPart + r * 32 + ((h ^ ((r >> 2) & 1)) << 4));

  auto step = [&](const char* at, int tok0) {
    const bool masked = tok0 + 32 > lo;  // (of the workgroup) some row does not see all 32 tokens
    f32x16 score[1][1];
#pragma unroll
    for (int x = 0; x < 16; ++x) score[0][0][x] = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const k4u32x4 key = *(const k4u32x4*)(at + (key_at ^ (32u * s)));
      score[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, key), __builtin_bit_cast(bf16x8, q[s]), score[0][0], 0, 0, 0);
    }
    k4u32x4 v[2][HT];  // [block]: tokens 8 h .. + 7 of a channel
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int j = 0; j < HT; ++j) v[s][j] = *(const k4u32x4*)(at + s * 2 * W::kPart + value_at + j * 1024);
    settle(score);
    float p[16];
#pragma unroll
    for (int x = 0; x < 16; ++x) p[x] = score[0][0][x];
    uint32_t sees = ~0u, odd = 0;  // odd: (see the kernel of few rows) bits 8 s + x: token 16 s + 8 h + x
    if (masked) {
      sees = seen(tok0);
#pragma unroll
      for (int x = 0; x < 16; ++x)
        if (!((sees >> (16 * (x >> 3) + 8 * h + (x & 7))) & 1)) p[x] = -INFINITY;
      if (tok0 + 32 > len) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int n = min(8, max(0, len - tok0 - 16 * s - 8 * h));
#pragma unroll
          for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int j = 0; j < HT; ++j) v[s][j][d] &= n >= 2 * d + 2 ? ~0u : n == 2 * d + 1 ? 0xffffu : 0u;
        }
      }
      u16x2 largest = u16x2{0, 0};
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int j = 0; j < HT; ++j)
#pragma unroll
          for (int d = 0; d < 4; ++d) largest = __builtin_elementwise_max(largest, __builtin_bit_cast(u16x2, v[s][j][d] & 0x7fff7fffu));
      if (__ballot(max(largest.x, largest.y) >= 0x7f80) != 0) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int j = 0; j < HT; ++j)
#pragma unroll
            for (int d = 0; d < 4; ++d) {
              const uint32_t bad = ((v[s][j][d] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;  // (an exponent of ones carries)
              odd |= (bad & 0x8000u ? 1u << (8 * s + 2 * d) : 0u) | (bad & 0x80000000u ? 2u << (8 * s + 2 * d) : 0u);
              v[s][j][d] &= (bad & 0x8000u ? 0u : 0xffffu) | (bad & 0x80000000u ? 0u : 0xffff0000u);
            }
      }
    }
    float top = max3(p[0], p[1], p[2]);
#pragma unroll
    for (int x = 3; x < 15; x += 2) top = max3(top, p[x], p[x + 1]);
    top = max3(top, p[15], p[15]);
    if (__ballot(top > moves) != 0) {  // (the maximum moves only when a score passes it by 2^8)
      const float m_old = maximum(), m_new = fmaxf(m_old, fold32(top, LaneMax{}) * c1);
      const float alpha = m_new == m_old ? 1.f : __builtin_amdgcn_exp2f(m_old - m_new);
      if (m_new != -INFINITY) {
        neg_m = -m_new;
        moves = (m_new + 8.f) * (1.f / c1);
      }
      l *= alpha;
#pragma unroll
      for (int j = 0; j < HT; ++j)
#pragma unroll
        for (int x = 0; x < 16; ++x) acc[0][j][x] *= alpha;
    }
    unsigned pw[8][2];
#pragma unroll
    for (int x = 0; x < 16; ++x) p[x] = __builtin_amdgcn_exp2f(fmaf(p[x], c1, neg_m));
#pragma unroll
    for (int x = 0; x < 16; x += 4) l += (p[x] + p[x + 1]) + (p[x + 2] + p[x + 3]);
#pragma unroll
    for (int d = 0; d < 8; ++d) split_weights(p[2 * d], p[2 * d + 1], pw[d]);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int j = 0; j < HT; ++j)
          acc[0][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[s][j]), __builtin_bit_cast(bf16x8, k4u32x4{pw[4 * s][m], pw[4 * s + 1][m], pw[4 * s + 2][m], pw[4 * s + 3][m]}),
                                                              acc[0][j], 0, 0, 0);
    settle(acc);
    if (__ballot(odd != 0) != 0) {  // values that are no numbers, for the rows that see them
      uint32_t apart_of = 0;
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const unsigned long long who = __ballot((odd >> x) & 1);
        apart_of |= ((uint32_t)who ? 1u << (16 * (x >> 3) + (x & 7)) : 0u) | ((who >> 32) ? 1u << (16 * (x >> 3) + 8 + (x & 7)) : 0u);
      }
#pragma unroll 1
      for (; apart_of != 0; apart_of &= apart_of - 1) {
        const int tok = __builtin_ctz(apart_of), x = 8 * (tok >> 4) + (tok & 7);
        float pt = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) pt = x == i ? p[i] : pt;
        pt = __shfl(pt, r + 32 * ((tok >> 3) & 1), 64);
#pragma unroll
        for (int j = 0; j < HT; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int ch = j * 32 + 8 * (e >> 2) + 4 * h + (e & 3);
            const uint16_t y = *(const uint16_t*)(at + (tok >> 4) * 2 * W::kPart + W::kPart + ch * 32 + ((((tok >> 3) & 1) ^ ((ch >> 2) & 1)) << 4) + (tok & 7) * 2);
            if (not_finite(y) && ((sees >> tok) & 1)) acc[0][j][e] += pt * bf16_bits_to_f32(y);
          }
      }
    }
  };

  constexpr int PER = SHARES * COPIES;  // copies of a stage that a wave has on their way
  // Once, and again where sums are no numbers behind steps that all rows see (see weigh_infinities): then such values are apart in all.  9 rows
  // behind 131071 tokens 103 us, 159 with an infinity, 322 with one in every 64th token.
#pragma unroll 1
  for (;;) {
#pragma unroll
    for (int j = 0; j < HT; ++j)
#pragma unroll
      for (int x = 0; x < 16; ++x) acc[0][j][x] = 0.f;
    neg_m = l = 0.f;
    moves = -INFINITY;
#pragma unroll
    for (int i = 0; i < RING - 1; ++i)
      if (i < nstages) copy(i);
#pragma unroll
    for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(q[s]));  // (here: a wait in the walk would be one for copies, which the compiler does not count)
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) asm volatile("" : "+v"(early[i]));
#pragma unroll 1
    for (int i = 0; i < nstages; ++i) {
      if (RING == 3 && i + 1 < nstages) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(PER) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();  // the stage has landed, and what the next copies go over has been read
      if (i + RING - 1 < nstages) copy(i + RING - 1);
      const int tok0 = span0 + i * STAGE + share * 32;
      if (!idle && tok0 < end) {
        const char* at = (const char*)lds + (i % RING) * W::kStage + share * 4 * W::kPart;
        step(at, tok0);
      }
    }
    if (lo <= span0) break;
    bool none = false;
#pragma unroll
    for (int j = 0; j < HT; ++j)
#pragma unroll
      for (int x = 0; x < 16; ++x) none |= acc[0][j][x] != acc[0][j][x];
    if (!__syncthreads_or(none)) break;
    lo = 0;
    load_blocks(0);
  }
  if constexpr (SHARES == 1) {  // the rows are the wave's own
    l = fold32(l, LaneAdd{});
    if (!tr.live) return;
    const float inv = wk.inverse(l);
    uint16_t* out = (uint16_t*)a.out + tr.row * a.out_stride + tr.head * HD;
    float* dst = wk.all + ((size_t)it.split * ROWS + wr * 32 + r) * ROW;
#pragma unroll
    for (int j = 0; j < HT; ++j)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const f32x4 o = f32x4{acc[0][j][4 * u], acc[0][j][4 * u + 1], acc[0][j][4 * u + 2], acc[0][j][4 * u + 3]};
        const int e0 = j * 32 + 8 * u + 4 * h;
        if (wk.nsplit == 1) wk.store(out + e0, o * inv);
        else *(f32x4*)(dst + e0) = o;
      }
    if (wk.nsplit > 1 && h == 0) *(f32x2*)(dst + HD) = f32x2{partial_maximum(maximum(), l), l};
  } else {
    __syncthreads();
    float(*states)[ROWS][ROW] = (float(*)[ROWS][ROW])lds;
#pragma unroll
    for (int j = 0; j < HT; ++j)
#pragma unroll
      for (int u = 0; u < 4; ++u)
        *(f32x4*)&states[share][wr * 32 + r][j * 32 + 8 * u + 4 * h] = f32x4{acc[0][j][4 * u], acc[0][j][4 * u + 1], acc[0][j][4 * u + 2], acc[0][j][4 * u + 3]};
    l = fold32(l, LaneAdd{});
    if (h == 0) *(f32x2*)&states[share][wr * 32 + r][HD] = f32x2{partial_maximum(maximum(), l), l};
    __syncthreads();
    join_waves<HD, uint16_t, ROWS, SHARES, kPagesWaves * 64>(wk, it.split, true, lds, tid);
  }
}

// The splits of a workgroup's rows joined apart: workgroup (cache head, some rows of a client's group), a thread 4 channels of a row and of
// every `shares`-th split, 8 at a time.  The shares of a task are joined through LDS in order.  Bound by trips to memory, 1.7 us for 8 splits:
// 64 splits of 36 rows (8 heads of 128) 6.9 us with eight threads a task, 13 to 15 with one; 2 to 4 splits 6.3.
template <int HD, typename T, int ROWS>
__global__ __launch_bounds__(256) void pages_join_kernel(PagesAttend a, PagesClients clients, PagesJoin join) {
  constexpr int TPR = HD / 4, ROW = HD + kPagesPartPad, PER = 256 / TPR, BATCH = 8;
  __shared__ float joined[256][6];
  const int tid = threadIdx.x, lane = tid & 63, shares = 1 << join.log_shares, per = PER >> join.log_shares, wgs = ROWS / per;
  const int ci = __builtin_amdgcn_readfirstlane(__popcll(__ballot(lane < clients.n && (int)blockIdx.y >= join.first[lane & (kPagesPerLaunch - 1)])) - 1);
  const int at = blockIdx.y - join.first[ci];
  const PagesWork<HD, T> wk(a, clients, PagesItem{ci, at / wgs, 0}, blockIdx.x, ROWS / 16);
  const int row0 = at % wgs * per, share = tid / (per * TPR), mr = row0 + tid / TPR % per, e0 = tid % TPR * 4;
  if (wk.first_row + row0 >= wk.group_rows) return;  // (whole workgroup)
  const float* from = wk.all + (size_t)min(mr, wk.group_rows - wk.first_row - 1) * ROW;
  float m = -INFINITY, l = 0.f;
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int s0 = share; s0 < wk.nsplit; s0 += BATCH * shares) {
    f32x4 ob[BATCH];
    f32x2 ml[BATCH];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const int sp = s0 + j * shares;
      const float* p = from + (size_t)min(sp, wk.nsplit - 1) * (ROWS * ROW);
      ob[j] = *(const f32x4*)(p + e0);
      ml[j] = *(const f32x2*)(p + HD);
      if (sp >= wk.nsplit) ml[j].x = -INFINITY;
    }
    float top = m;
#pragma unroll
    for (int j = 0; j < BATCH; ++j) top = fmaxf(top, ml[j].x);
    const float back = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
    l *= back;
    o *= back;
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      if (ml[j].x == -INFINITY) continue;
      const float sw = __builtin_amdgcn_exp2f(ml[j].x - top);
      l += ml[j].y * sw;
      o += ob[j] * sw;
    }
    m = top;
  }
  if (shares > 1) {
    float* x = joined[tid];
    x[0] = o[0], x[1] = o[1], x[2] = o[2], x[3] = o[3], x[4] = l, x[5] = m;
    __syncthreads();
    if (share > 0) return;
    float top = m;
    for (int sh = 1; sh < shares; ++sh) top = fmaxf(top, joined[sh * per * TPR + tid][5]);
    const float own = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
    l *= own;
    o *= own;
    for (int sh = 1; sh < shares; ++sh) {
      const float* y = joined[sh * per * TPR + tid];
      if (y[5] == -INFINITY) continue;
      const float sw = __builtin_amdgcn_exp2f(y[5] - top);
      l += y[4] * sw;
      o += f32x4{y[0], y[1], y[2], y[3]} * sw;
    }
  }
  wk.finish(wk.first_row + mr, e0, o, l);
}

template <class Kernel, class Join>
static hipError_t launch(Kernel kernel, Join join, std::atomic<uint64_t>& allowed, size_t bytes, int waves, int rows, const PagesAttend& a,
                         const PagesClients& c, hipStream_t st) {
  if (bytes > 65536) {
    const hipError_t e = allow_lds(allowed, (const void*)kernel, bytes);
    if (e != hipSuccess) return e;
  }
  kernel<<<dim3(a.view.n_kv_heads, c.items), waves * 64, bytes, st>>>(a, c);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !c.apart) return e;
  PagesJoin how;
  const int wgs = pages_join_plan(c, rows, a.view.head_dim, &how);
  join<<<dim3(a.view.n_kv_heads, wgs), 256, 0, st>>>(a, c, how);
  return hipGetLastError();
}
template <int HD, typename T, int TILES>
static hipError_t launch_few(const PagesAttend& a, const PagesClients& c, hipStream_t st) {
  static std::atomic<uint64_t> allowed;
  return launch(pages_attend_kernel<HD, T, TILES>, pages_join_kernel<HD, T, TILES * 16>, allowed, attend_lds_bytes<HD, T, TILES>(), kPagesFewWaves, TILES * 16, a, c, st);
}
template <int HD, int WR>
static hipError_t launch_wide(const PagesAttend& a, const PagesClients& c, hipStream_t st) {
  static std::atomic<uint64_t> allowed;
  return launch(pages_attend_wide_kernel<HD, WR>, pages_join_kernel<HD, uint16_t, WR * 32>, allowed, Wide<HD, WR>::kLds, kPagesWaves, WR * 32, a, c, st);
}

hipError_t launch_pages_attend(const PagesAttend& a, const PagesLaunch& l, hipStream_t st) {
  auto go = [&](auto hd) {
    constexpr int HD = decltype(hd)::value;
    if (a.dtype == PIPESD_F32) {
      if (l.tiles == 1) return launch_few<HD, float, 1>(a, l.c, st);
      return l.tiles == 2 ? launch_few<HD, float, 2>(a, l.c, st) : hipErrorInvalidValue;
    }
    if (l.tiles == 1) return launch_few<HD, uint16_t, 1>(a, l.c, st);
    if (l.tiles == 2) return launch_few<HD, uint16_t, 2>(a, l.c, st);
    if (l.tiles == 4) return launch_wide<HD, 2>(a, l.c, st);
    return l.tiles == 8 ? launch_wide<HD, 4>(a, l.c, st) : hipErrorInvalidValue;
  };
  return a.view.head_dim == 128 ? go(std::integral_constant<int, 128>{}) : go(std::integral_constant<int, 64>{});
}

}  // namespace pipesd
