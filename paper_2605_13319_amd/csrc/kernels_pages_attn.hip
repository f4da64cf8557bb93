// Attention of the rows of a pass over the paged cache of operators, chains and trees.
//
//   o_r = sum_t p_rt v_t,   p_rt = exp(s_rt) / sum_t' exp(s_rt'),   s_rt = q_r . k_t / sqrt(head_dim),
// over the tokens before the pass, the row's ancestors in it and the row itself.
//
// bf16: keys, values and queries are operands as they are; weights are cut into two bf16 numbers, 16 bits where results have 8, as in
// the other attentions of the library.  fp32: products of fp32 numbers on the matrix cores.  Maxima and sums are fp32.
//
// One pass over the cache: keys and values go from memory into the registers that the products take them from and are not kept.  The
// waves of a workgroup share its tiles of query rows, take every fourth 32 tokens of the span and join their states through LDS at the
// end; a context that is cut into splits is joined by the last workgroup that arrives, or by a kernel of its own.
#include "device_attend.h"
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

  __device__ __forceinline__ void finish(int rr, int e0, const f32x4& o, float l) const {  // 4 channels of a row: o / l
    const TileRow tr = row(rr);
    if (!tr.live) return;
    float inv = __builtin_amdgcn_rcpf(l);  // (a row sees itself: l is 0 only where all its scores are -inf, and then there is no number)
    inv = inv * (2.f - l * inv);
    const f32x4 y = o * inv;
    T* out = (T*)a.out + tr.row * a.out_stride + tr.head * HD + e0;
    if constexpr (sizeof(T) == 4) *(f32x4*)out = y;
    else *(uint2*)out = make_uint2(pack2_bf16(y[0], y[1]), pack2_bf16(y[2], y[3]));
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

template <typename T>
__device__ __forceinline__ bool not_finite(T x) {
  if constexpr (sizeof(T) == 4) return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u;
  else return (x & 0x7f80u) == 0x7f80u;
}

// LDS: states [tile][wave][row], later what joins the splits; then the queries that registers do not hold; a word
template <int HD, int TILES>
constexpr size_t state_floats() { return (size_t)TILES * kPagesWaves * 16 * (HD + kPagesPartPad); }
template <int HD, typename T, int TILES>
constexpr bool queries_in_lds() { return TILES * HD * (int)sizeof(T) > 512; }  // (more than 32 registers)
template <int HD, typename T, int TILES>
constexpr size_t attend_lds_bytes() {
  return state_floats<HD, TILES>() * sizeof(float) + (queries_in_lds<HD, T, TILES>() ? (size_t)TILES * HD * sizeof(T) * 16 : 0) + 16;
}

// A wave walks tokens 32 at a time (a step): scores, weights, products with the values.  Of a step a lane (c, g) has the scores of
// query row c with 8 tokens:
//   bf16  tokens 8 g .. + 7: what a product over 32 tokens takes of their weights, and of a channel's values with one load.  The
//         first four are row 4 g + .. of the first 16 x 16 product of keys, the others of the second: row r of product tt is token
//         8 (r / 4) + 4 tt + r % 4.
//   fp32  tokens 4 g .. + 3 of both blocks; a load of 4 channels of a key, or 4 tokens of a value, serves 4 products (k = 4).
template <int HD, typename T, int TILES>
__global__ __launch_bounds__(kPagesWaves * 64, 2) void pages_attend_kernel(PagesAttend a, PagesClients clients) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int HT = HD / 16, ROW = HD + kPagesPartPad, WAVES = kPagesWaves, STEP = kPagesStep, NT = WAVES * 64;
  constexpr int NK = F32 ? HD / 16 : HD / 32;  // 16-byte pieces of a key that a lane has
  constexpr int NV = F32 ? 2 * HT : HT;        // and of values
  constexpr bool Q_LDS = queries_in_lds<HD, T, TILES>();
  extern __shared__ float lds[];
  int* word = (int*)((char*)lds + attend_lds_bytes<HD, T, TILES>() - 16);

  const int kvh = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, g = lane >> 4;
  const PagesItem it = find_item(clients, blockIdx.y, lane);
  const PagesWork<HD, T> wk(a, clients, it, kvh, TILES);
  const int len = wk.len, before = len - wk.n_rows, span0 = it.split * clients.span, first = span0 + w * 32;

  // 64 steps' blocks sit in the lanes: lane L has the two of step L
  int step_blk[2];
  auto load_blocks = [&](int it0) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
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
  // which of the 32 tokens from tok0 on a row sees
  auto seen = [&](int t, int tok0) -> uint32_t {
    if (a.masks != nullptr) return a.masks[(size_t)row_of[t] * kPagesMaskWords + min((tok0 - (before & ~31)) >> 5, kPagesMaskWords - 1)];
    const int n = before + 1 + row_of[t] - wk.row_off - tok0;
    return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
  };
  // (the first that are asked for travel with the keys)
  const int first_masked = first > lo - 32 ? 0 : (lo - 32 - first) / STEP + 1;
  uint32_t next_seen[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) next_seen[t] = first_masked < nsteps ? seen(t, first + first_masked * STEP) : 0u;

  Running<HT> run[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) run[t].clear();
  const float c1 = attend_scale<HD>();

  // Keys and values of a step travel from where those of the step before have been used until they are.
  k4u32x4 k[2][NK], v[NV];
  const char* head_base = (const char*)((const T*)a.view.pool + (int64_t)a.layer * a.view.layer_stride + (int64_t)kvh * kBlockTokens * HD);
  auto block_base = [&](int i, int tt) {
    return head_base + (int64_t)__builtin_amdgcn_readlane(step_blk[tt], i & 63) * a.view.block_elems * (int)sizeof(T);
  };
  auto request_keys = [&](int i) {
    if (i >= nsteps) return;
    if (i > 0 && (i & 63) == 0) load_blocks(i);
    const char *b0 = block_base(i, 0), *b1 = block_base(i, 1);
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const char* p;
      if constexpr (F32) p = (tt ? b1 : b0) + c * HD * 4 + g * 16;
      else p = (c >> 3 ? b1 : b0) + (8 * ((c >> 2) & 1) + 4 * tt + (c & 3)) * HD * 2 + g * 16;
#pragma unroll
      for (int s = 0; s < NK; ++s) k[tt][s] = *(const k4u32x4*)(p + s * 64);
    }
  };
  auto request_values = [&](int i) {
    if (i >= nsteps) return;
    const char *b0 = block_base(i, 0) + a.view.v_offset * (int)sizeof(T), *b1 = block_base(i, 1) + a.view.v_offset * (int)sizeof(T);
    if constexpr (F32) {
#pragma unroll
      for (int j = 0; j < NV; ++j) v[j] = *(const k4u32x4*)((j / HT ? b1 : b0) + ((j % HT) * 16 + c) * 64 + g * 16);
    } else {
      const char* p = (g >> 1 ? b1 : b0) + c * 32 + (g & 1) * 16;
#pragma unroll
      for (int j = 0; j < NV; ++j) v[j] = *(const k4u32x4*)(p + j * 512);
    }
  };
  // the lane's token of score x, of the step's 32
  auto token_of = [&](int x) { return F32 ? 16 * (x >> 2) + 4 * g + (x & 3) : 8 * g + x; };

  // Values of tokens that not every row sees.  Behind the client's last token there may be anything: 0 instead.  A value that is not
  // finite must reach the rows that see its token and no other, but a product would take it times 0 to all: it becomes 0 here, too, and
  // `apart_of` has a bit for its token.
  auto drop_values = [&](int tok0, uint32_t& apart_of) {
    uint32_t odd = 0;  // bit x: of the lane's token x
    if constexpr (F32) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int x = (j / HT) * 4 + i;
          const bool there = tok0 + token_of(x) < len, bad = (v[j][i] & 0x7f800000u) == 0x7f800000u;
          if (there && bad) odd |= 1u << x;
          if (!there || bad) v[j][i] = 0u;
        }
    } else {
      const int n = min(8, max(0, len - tok0 - 8 * g));
      uint32_t any = 0;  // (an exponent of ones carries into the sign)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const uint32_t keep = n >= 2 * d + 2 ? ~0u : n == 2 * d + 1 ? 0xffffu : 0u;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          v[j][d] &= keep;
          any |= (v[j][d] & 0x7f807f80u) + 0x00800080u;
        }
      }
      if (__ballot((any & 0x80008000u) != 0) != 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const uint32_t bad = ((v[j][d] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
            if (bad & 0x8000u) odd |= 1u << (2 * d), v[j][d] &= 0xffff0000u;
            if (bad & 0x80000000u) odd |= 2u << (2 * d), v[j][d] &= 0xffffu;
          }
      }
    }
    apart_of = 0;
    if (__ballot(odd != 0) == 0) return;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const unsigned long long who = __ballot((odd >> x) & 1);
#pragma unroll
      for (int gg = 0; gg < 4; ++gg)
        if ((who >> (16 * gg)) & 0xffff) apart_of |= 1u << (F32 ? 16 * (x >> 2) + 4 * gg + (x & 3) : 8 * gg + x);
    }
  };
  // those values, for the rows that see them (LDS: the wave's own states, which nobody reads before its walk has ended)
  float* scratch = lds + (size_t)w * 16 * ROW;
  auto add_apart = [&](Running<HT>& r, const float (&p)[8], uint32_t sees, uint32_t apart_of, int i, int tok0) {
#pragma unroll
    for (int x = 0; x < 8; ++x) scratch[c * 33 + token_of(x)] = p[x];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
    for (uint32_t left = apart_of; left != 0; left &= left - 1) {
      const int tok = __builtin_ctz(left);
      const T* from = (const T*)(block_base(i, tok >> 4) + a.view.v_offset * (int)sizeof(T)) + (tok & 15);
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

  request_keys(0);
  request_values(0);
#pragma unroll 1
  for (int i = 0; i < nsteps; ++i) {
    const int tok0 = first + i * STEP;
    const bool masked = tok0 + 32 > lo;  // (of the wave) some row does not see all 32 tokens
    f32x4 score[TILES][2];
#pragma unroll
    for (int t = 0; t < TILES; ++t) score[t][0] = score[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < NK; ++s)
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const k4u32x4 qs = query(t, s);
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
          if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              score[t][tt] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[tt][s][e]), __uint_as_float(qs[e]), score[t][tt], 0, 0, 0);
          } else {
            score[t][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[tt][s]), __builtin_bit_cast(bf16x8, qs), score[t][tt], 0, 0, 0);
          }
        }
      }
    request_keys(i + 1);
    settle(score);
    float p[TILES][8];
    uint32_t sees[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      float sc[8] = {score[t][0][0], score[t][0][1], score[t][0][2], score[t][0][3], score[t][1][0], score[t][1][1], score[t][1][2], score[t][1][3]};
      if (masked) {
        sees[t] = next_seen[t];
        if (i + 1 < nsteps) next_seen[t] = seen(t, tok0 + STEP);
#pragma unroll
        for (int x = 0; x < 8; ++x)
          if (!((sees[t] >> token_of(x)) & 1)) sc[x] = -INFINITY;
      }
      const float top = top_of(sc);
      if (__ballot(top > run[t].moves) != 0) run[t].move_to(top, c1);
#pragma unroll
      for (int x = 0; x < 8; ++x) p[t][x] = __builtin_amdgcn_exp2f(fmaf(sc[x], c1, run[t].neg_m));
      run[t].l += ((p[t][0] + p[t][1]) + (p[t][2] + p[t][3])) + ((p[t][4] + p[t][5]) + (p[t][6] + p[t][7]));
    }
    uint32_t apart_of = 0;
    if (masked) drop_values(tok0, apart_of);
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      if constexpr (F32) {
#pragma unroll
        for (int x = 0; x < 8; ++x)
#pragma unroll
          for (int j = 0; j < HT; ++j)
            run[t].acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[(x >> 2) * HT + j][x & 3]), p[t][x], run[t].acc[j], 0, 0, 0);
      } else {
        unsigned pw[4][2];
#pragma unroll
        for (int d = 0; d < 4; ++d) split_weights(p[t][2 * d], p[t][2 * d + 1], pw[d]);
#pragma unroll
        for (int j = 0; j < HT; ++j)
#pragma unroll
          for (int m = 0; m < 2; ++m)
            run[t].acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v[j]), __builtin_bit_cast(bf16x8, k4u32x4{pw[0][m], pw[1][m], pw[2][m], pw[3][m]}),
                                                                    run[t].acc[j], 0, 0, 0);
      }
    }
    settle(run);
    if (apart_of != 0) {
#pragma unroll
      for (int t = 0; t < TILES; ++t) add_apart(run[t], p[t], sees[t], apart_of, i, tok0);
    }
    request_values(i + 1);
  }

  // ---- the waves' states joined: rows, or a split's partial rows (written through) ----
  constexpr int ROWS = TILES * 16, TPR = HD / 4;
  const int rows_here = min(ROWS, wk.group_rows - wk.first_row), tasks = rows_here * TPR;  // a task: (row, 4 channels)
  float(*states)[WAVES][16][ROW] = (float(*)[WAVES][16][ROW])lds;  // a row: its channels, its maximum and sum
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
#pragma unroll
    for (int j = 0; j < HT; ++j) *(f32x4*)&states[t][w][c][j * 16 + 4 * g] = run[t].acc[j];
    const float l = fold_groups(run[t].l, LaneAdd{});
    if (g == 0) *(f32x2*)&states[t][w][c][HD] = f32x2{partial_maximum(run[t].maximum(), l), l};
  }
  __syncthreads();
#pragma unroll 1
  for (int task = tid; task < tasks; task += NT) {
    const int mr = task / TPR, e0 = (task % TPR) * 4;
    const float(*rows)[16][ROW] = states[mr / 16];
    f32x2 ml[WAVES];
    float m = -INFINITY;
#pragma unroll
    for (int ww = 0; ww < WAVES; ++ww) {
      ml[ww] = *(const f32x2*)&rows[ww][mr % 16][HD];
      m = fmaxf(m, ml[ww].x);
    }
    const float m_ref = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ww = 0; ww < WAVES; ++ww) {
      const float sw = __builtin_amdgcn_exp2f(ml[ww].x - m_ref);
      l += ml[ww].y * sw;
      o += *(const f32x4*)&rows[ww][mr % 16][e0] * sw;
    }
    if (wk.nsplit == 1) {
      wk.finish(wk.first_row + mr, e0, o, l);
    } else {
      float* dst = wk.all + ((size_t)it.split * ROWS + mr) * ROW;
      Xwg<true>::st4f(dst + e0, o);
      if (e0 == 0) Xwg<true>::st4f(dst + HD, f32x4{partial_maximum(m, l), l, 0.f, 0.f});
    }
  }
  if (wk.nsplit == 1 || clients.apart || !wk.arrives_last(word)) return;
  static_assert(join_floats<ROWS, NT>() <= (int)state_floats<HD, TILES>(), "what joins fits the states' LDS");
  join_splits<HD, T, ROWS, NT>(wk, lds, tid);
}

// The splits of clients that their last workgroup would take long to join: workgroup (cache head, client's group of tiles).
template <int HD, typename T, int TILES>
__global__ __launch_bounds__(kPagesWaves * 64) void pages_join_kernel(PagesAttend a, PagesClients clients) {
  __shared__ float lds[join_floats<TILES * 16, kPagesWaves * 64>()];
  int group = blockIdx.y, ci = 0;
  while (group >= clients.groups[ci]) group -= clients.groups[ci++];
  if (clients.nsplit[ci] == 1) return;  // (whole workgroup)
  const PagesWork<HD, T> wk(a, clients, PagesItem{ci, group, 0}, blockIdx.x, TILES);
  join_splits<HD, T, TILES * 16, kPagesWaves * 64>(wk, lds, threadIdx.x);
}

template <int HD, typename T, int TILES>
static hipError_t launch(const PagesAttend& a, const PagesClients& c, hipStream_t st) {
  static std::atomic<uint64_t> allowed;
  constexpr size_t bytes = attend_lds_bytes<HD, T, TILES>();
  if (bytes > 65536) {
    const hipError_t e = allow_lds(allowed, (const void*)pages_attend_kernel<HD, T, TILES>, bytes);
    if (e != hipSuccess) return e;
  }
  pages_attend_kernel<HD, T, TILES><<<dim3(a.view.n_kv_heads, c.items), kPagesWaves * 64, bytes, st>>>(a, c);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !c.apart) return e;
  int groups = 0;
  for (int i = 0; i < c.n; ++i) groups += c.groups[i];
  pages_join_kernel<HD, T, TILES><<<dim3(a.view.n_kv_heads, groups), kPagesWaves * 64, 0, st>>>(a, c);
  return hipGetLastError();
}

hipError_t launch_pages_attend(const PagesAttend& a, const PagesLaunch& l, hipStream_t st) {
  auto tiles = [&](auto hd, auto t) {
    typedef decltype(t) T;
    constexpr int HD = decltype(hd)::value;
    return l.tiles == 1 ? launch<HD, T, 1>(a, l.c, st) : launch<HD, T, 2>(a, l.c, st);
  };
  typedef std::integral_constant<int, 64> H64;
  typedef std::integral_constant<int, 128> H128;
  if (a.view.head_dim == 128) return a.dtype == PIPESD_F32 ? tiles(H128{}, float{}) : tiles(H128{}, uint16_t{});
  return a.dtype == PIPESD_F32 ? tiles(H64{}, float{}) : tiles(H64{}, uint16_t{});
}

}  // namespace pipesd
