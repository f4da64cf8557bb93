// Attention over the 4-bit cache, and the weights it gave to the cached tokens.
//
//   o_r = sum_t p_rt v_t,   p_rt = exp(s_rt) / sum_t' exp(s_rt'),   s_rt = q_r . k_t / sqrt(head_dim),
// over the first lim_r tokens; a row with none has no weights, and o_r = 0.  mass_t = sum over rows and heads of p_rt.
//
// Keys and values become bf16 on their way to the matrix cores, exactly (two bits and a power of two).  The queries of a bf16
// model are operands as they are, those of an fp32 model are cut into three bf16 numbers (24 bits, so exactly): scores are as
// good as fp32 ones.  So are an fp32 model's weights, cut into three bf16 numbers too.  Those of a bf16 model are cut into two, 16
// bits where its results have 8, as in the attention over its bf16 cache: only the cache itself is coarse.  Maxima and sums are fp32.
//
// (The products that take 4-bit codes with their powers as operands need no conversion of the keys, but cut the addends of a
// sum about 2^15 below the largest: with the queries in two e4m3 pieces scores were off by 2^-20 to 2^-16 of sum |q k|, where
// bf16 products are off by 2^-27 to 2^-24.)
#include "device_gemm.h"
#include "kv4.h"
#include "lds_limit.h"

namespace pipesd {

typedef __attribute__((ext_vector_type(4))) unsigned k4u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned k4u32x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

template <int HD>
__device__ __forceinline__ float kv4_scale() { return (HD == 128 ? 0.08838834764831845f : 0.125f) * 1.44269504088896341f; }  // log2(e) / sqrt(HD)

// Queries as operand B.  A lane holds 8 channels of its row in each step of a product; in step s these are 8 s .. + 7 of the
// lane's own part of the row, so that what it needs of a key in all steps is one load.  (Columns beyond the last row have the last
// row's once more: nothing reads theirs.)
template <int NP, int NS, typename T>
__device__ __forceinline__ void load_queries(const T* part, k4u32x4 (&out)[NP][NS]) {
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const T* p = part + s * 8;
    if constexpr (sizeof(T) == 2) {
      out[0][s] = *(const k4u32x4*)p;
    } else {
      const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
      float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
#pragma unroll
      for (int m = 0; m < NP; ++m) {  // the upper half of each float is a bf16 number; what it leaves goes on
        unsigned w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const unsigned lo = __float_as_uint(x[2 * i]), hi = __float_as_uint(x[2 * i + 1]);
          w[i] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
          x[2 * i] -= __uint_as_float(lo & 0xffff0000u);
          x[2 * i + 1] -= __uint_as_float(hi & 0xffff0000u);
        }
        out[m][s] = k4u32x4{w[0], w[1], w[2], w[3]};
      }
    }
  }
}

// step s of a lane's keys as operand A: 8 channels of one word of codes
__device__ __forceinline__ bf16x8 key_operand(unsigned codes, float power) {
  auto two = [&](auto byte) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, decltype(byte)::value));
  };
  return __builtin_bit_cast(bf16x8, k4u32x4{two(std::integral_constant<int, 0>{}), two(std::integral_constant<int, 1>{}),
                                            two(std::integral_constant<int, 2>{}), two(std::integral_constant<int, 3>{})});
}

// The values of a lane's unit for its four tokens of a block, channels 2 b and 2 b + 1 of the unit, as half of an operand each:
// bf16 pairs (channel, next channel) of every token, regrouped to pairs of tokens.
template <int HD, class Codes>
__device__ __forceinline__ void value_operands(const Codes& v, unsigned powers, int b, k4u32x2& even, k4u32x2& odd) {
  const float p0 = __uint_as_float(powers << 23), p1 = __uint_as_float(powers << 15), p2 = __uint_as_float(powers << 7),
              p3 = __uint_as_float(powers >> 1);  // (only the exponent's bits count)
  unsigned x[4];
  auto cvt = [&](unsigned w, float pw, auto byte) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, pw, decltype(byte)::value));
  };
  auto at_byte = [&](auto byte) {
    if constexpr (HD == 128) {
      x[0] = cvt(v.x, p0, byte);
      x[1] = cvt(v.y, p1, byte);
      x[2] = cvt(v.z, p2, byte);
      x[3] = cvt(v.w, p3, byte);
    } else {
      typedef std::integral_constant<int, decltype(byte)::value + 2> upper;
      x[0] = cvt(v.x, p0, byte);
      x[1] = cvt(v.x, p1, upper{});
      x[2] = cvt(v.y, p2, byte);
      x[3] = cvt(v.y, p3, upper{});
    }
  };
  if (b == 0) at_byte(std::integral_constant<int, 0>{});
  if (b == 1) at_byte(std::integral_constant<int, 1>{});
  if constexpr (HD == 128) {
    if (b == 2) at_byte(std::integral_constant<int, 2>{});
    if (b == 3) at_byte(std::integral_constant<int, 3>{});
  }
  even = k4u32x2{__builtin_amdgcn_perm(x[1], x[0], 0x05040100u), __builtin_amdgcn_perm(x[3], x[2], 0x05040100u)};
  odd = k4u32x2{__builtin_amdgcn_perm(x[1], x[0], 0x07060302u), __builtin_amdgcn_perm(x[3], x[2], 0x07060302u)};
}
__device__ __forceinline__ bf16x8 both_blocks(const k4u32x2 (&x)[2]) {
  return __builtin_bit_cast(bf16x8, k4u32x4{x[0].x, x[0].y, x[1].x, x[1].y});
}
// What lies behind a client's last token may be anything.  Its weights are 0; its values must be numbers: of a lane's four
// tokens the first `left` stay.
template <int HD, class Codes>
__device__ __forceinline__ void drop_values(Codes& v, unsigned& powers, int left) {
  const int n = min(4, max(0, left));
  if constexpr (HD == 128) {
    v.x = n > 0 ? v.x : 0u;
    v.y = n > 1 ? v.y : 0u;
    v.z = n > 2 ? v.z : 0u;
    v.w = n > 3 ? v.w : 0u;
  } else {
    const unsigned long long keep = n >= 4 ? ~0ull : (1ull << (16 * n)) - 1ull;
    v.x &= (unsigned)keep;
    v.y &= (unsigned)(keep >> 32);
  }
  const unsigned km = n >= 4 ? ~0u : (1u << (8 * n)) - 1u;
  powers = (powers & km) | (0x7f7f7f7fu & ~km);
}

// Wait states behind the last products of sums, tied to all of them: whoever reads them next may be in another basic block,
// where the compiler pads too few.
template <bool ACC = false, int N, int M, class V>  // ACC: the sums are held in accumulation registers
__device__ __forceinline__ void settle(V (&x)[N][M]) {
#if defined(__HIP_DEVICE_COMPILE__)
  auto tie = [](V& v) {
    if constexpr (ACC) asm volatile("" : "+a"(v));
    else asm volatile("" : "+v"(v));
  };
#pragma unroll
  for (int i = 1; i < N * M; ++i) tie(x[i / M][i % M]);
  if constexpr (ACC) asm volatile("s_nop 15\n\ts_nop 1" : "+a"(x[0][0]));  // (in order: the products of all others come before)
  else asm volatile("s_nop 15\n\ts_nop 1" : "+v"(x[0][0]));
#pragma unroll
  for (int i = 1; i < N * M; ++i) tie(x[i / M][i % M]);
#endif
}

__device__ __forceinline__ float plain(float x) {  // in an ordinary register
  asm("" : "+v"(x));
  return x;
}

// where lane (c, g) finds its part of a record
template <int HD>
struct LaneOffsets {
  int k, v, kp, vp;
  __device__ __forceinline__ LaneOffsets(int c, int g) {
    typedef Kv4Record<HD> R;
    k = R::kKeys + c * (HD / 2) + g * (HD / 8);
    v = R::kValues + (g * 16 + c) * 4 * R::kUnit;
    kp = R::kKeyPow + c * R::kUnit + g * R::kUnit / 4;
    vp = R::kValPow + (g * R::kUnit + c / (512 / HD)) * 4;
  }
};

// n / m for 0 <= n < 2^20, 1 <= m, rinv = 1 / m to within an ulp: (n + 0.5) / m is at least 0.5 / m from an integer, more than
// the roundings' 2^-22 (n + 0.5) / m.  (An integer division is 30 instructions, and code is what a short call waits for.)
__device__ __forceinline__ int div_by(int n, float rinv) { return (int)(((float)n + 0.5f) * rinv); }

// the rows of a tile: lane's column
struct TileRow {
  int row, head;  // of the pass; of the model
  bool live;
};
__device__ __forceinline__ TileRow tile_row(int rr, int group, float group_rinv, int n_rows, int row_off, int kvh) {
  const int r = div_by(rr, group_rinv);
  return TileRow{row_off + min(r, n_rows - 1), kvh * group + rr - r * group, r < n_rows};
}
__device__ __forceinline__ int row_limit(const int32_t* limits, int row, int row_off, int n_rows, int len) {
  return limits ? min(max(limits[row], 0), len) : len - n_rows + (row - row_off) + 1;
}

// ------------------------------------------------------------------------------------------------
// attention
// ------------------------------------------------------------------------------------------------
__device__ __forceinline__ float max3(float a, float b, float c) {  // (through fmaxf the compiler quiets every operand first)
  float d;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}
// Two weights as NW pairs of bf16 numbers, each what the ones before leave (exactly).  (Dot products with (-1, 0) and (0, -1) give what is
// left in half the instructions, but wait for the matrix cores: two beside a 32 x 32 x 16 product take 53 cycles, where four of any others
// hide in its 32.)
template <int NW>
__device__ __forceinline__ void split_weights(float p0, float p1, unsigned (&out)[NW]) {
#pragma unroll
  for (int m = 0; m < NW; ++m) {
    out[m] = pack2_bf16(p0, p1);
    p0 -= __uint_as_float(out[m] << 16);
    p1 -= __uint_as_float(out[m] & 0xffff0000u);
  }
}

// which client and split a workgroup is for
struct Kv4Item {
  int ci, group, split;
};
__device__ __forceinline__ Kv4Item find_item(const Kv4Clients& cl, int item, int lane) {
  int ci = 0;
  if (cl.n > 1) ci = __popcll(__ballot(lane < kKv4ClientsPerLaunch && item >= cl.first[lane & (kKv4ClientsPerLaunch - 1)] && lane < cl.n)) - 1;
  ci = __builtin_amdgcn_readfirstlane(ci);
  const int i = item - cl.first[ci], groups = cl.groups[ci], split = div_by(i, __builtin_amdgcn_rcpf((float)groups));
  return Kv4Item{ci, groups - 1 - (i - split * groups), split};  // (the last rows see most: first)
}

// A wave walks tokens 32 at a time (a step): scores of the step, weights, products with the values.
template <typename T>
constexpr int pieces() { return sizeof(T) == 4 ? 3 : 1; }  // of a query
template <typename T>
constexpr int weight_pieces() { return sizeof(T) == 4 ? 3 : 2; }

// What a workgroup knows of its client, and how rows leave it.
template <int HD, typename T>
struct Work {
  const Kv4AttendCall& a;
  int kvh, len, n_rows, row_off, groups, nsplit, group_rows, first_row;  // group_rows: query rows of the cache head; first_row: the group's first
  float group_rinv;
  const int32_t* table;
  float* all;   // partial rows of the group's splits: [split][tiles of a workgroup][16][ROW]
  unsigned* counter;
  static constexpr int ROW = HD + kKv4PartPad;

  __device__ __forceinline__ Work(const Kv4AttendCall& call, const Kv4Clients& c, const Kv4Item& it, int kvh_, int wg_tiles)
      : a(call), kvh(kvh_), len(c.len[it.ci]), n_rows(c.n_rows[it.ci]), row_off(c.row_off[it.ci]), groups(c.groups[it.ci]),
        nsplit(c.nsplit[it.ci]) {
    group_rows = n_rows * a.group;
    first_row = it.group * wg_tiles * 16;
    group_rinv = __builtin_amdgcn_rcpf((float)a.group);
    table = a.view.table + c.table_off[it.ci];
    all = a.part + ((size_t)c.part_off[it.ci] + ((size_t)kvh * groups + it.group) * nsplit * wg_tiles) * (16 * ROW);
    counter = a.counters + c.count_off[it.ci] + kvh * groups + it.group;
  }
  __device__ __forceinline__ TileRow row(int rr) const { return tile_row(rr, a.group, group_rinv, n_rows, row_off, kvh); }
  __device__ __forceinline__ int limit(const TileRow& tr) const { return row_limit(a.limits, tr.row, row_off, n_rows, len); }

  // 4 channels of a row: o / l, and once a row what launch_kv4_mass needs
  __device__ __forceinline__ void finish(int rr, int e0, const f32x4& o, float m, float l) const {
    const TileRow tr = row(rr);
    if (!tr.live) return;
    float inv = __builtin_amdgcn_rcpf(l);
    inv = l == 0.f ? 0.f : inv * (2.f - l * inv);
    const f32x4 y = o * inv;
    T* out = (T*)a.out + tr.row * a.out_stride + tr.head * HD + e0;
    if constexpr (sizeof(T) == 4) *(f32x4*)out = y;
    else *(uint2*)out = make_uint2(pack2_bf16(y[0], y[1]), pack2_bf16(y[2], y[3]));
    if (a.lse && e0 == 0) a.lse[(size_t)tr.row * a.n_q_heads + tr.head] = l == 0.f ? INFINITY : m + __builtin_amdgcn_logf(l);
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

// The running softmax of a tile of 16 query rows: its state, per row (lane's column), and a step's weights.
template <int HT>
struct Running {
  f32x4 acc[HT];  // O^T
  // -(running maximum) (0 while nothing has been seen), the score that moves it, the lane's own sum of weights
  float neg_m, moves, l;

  __device__ __forceinline__ void clear() {
    neg_m = 0.f;
    moves = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int j = 0; j < HT; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ float maximum() const { return moves == -INFINITY ? -INFINITY : -neg_m; }
  // The maximum moves only when a score passes it by 2^8 (any scale will do for fp32 sums: most steps then need no exchange
  // between lanes and no rescaling).
  __device__ __forceinline__ void move_to(float top, float c1) {  // all lanes
    const float m_old = maximum(), m_new = fmaxf(m_old, fold_groups(top, LaneMax{}) * c1);
    const float alpha = m_new == m_old ? 1.f : __builtin_amdgcn_exp2f(m_old - m_new);
    if (m_new != -INFINITY) {
      neg_m = -m_new;
      moves = (m_new + 8.f) * (1.f / c1);
    }
    l *= alpha;
#pragma unroll
    for (int j = 0; j < HT; ++j) acc[j] *= alpha;
  }
  template <int NW>
  __device__ __forceinline__ void weights(const float (&sc)[8], float c1, bf16x8 (&out)[NW]) {
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], c1, neg_m));
    l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    unsigned w[4][NW];
#pragma unroll
    for (int i = 0; i < 4; ++i) split_weights(p[2 * i], p[2 * i + 1], w[i]);
#pragma unroll
    for (int m = 0; m < NW; ++m) out[m] = __builtin_bit_cast(bf16x8, k4u32x4{w[0][m], w[1][m], w[2][m], w[3][m]});
  }
};
__device__ __forceinline__ float top_of(const float (&sc)[8]) {
  return max3(max3(sc[0], sc[1], sc[2]), max3(sc[3], sc[4], sc[5]), max3(sc[6], sc[7], sc[7]));
}
__device__ __forceinline__ void hide(float (&sc)[8], int tok, int lim) {  // tok: the lane's first token of the first block
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (tok + (i >> 2) * 16 + (i & 3) >= lim) sc[i] = -INFINITY;
}
// What a split leaves as its row's maximum.  None means that it saw nothing and is passed over; a row of NaN, whose maximum never
// moves, must not be.
__device__ __forceinline__ float partial_maximum(float m, float l) { return l != l ? INFINITY : m; }

template <int N, int HT>
__device__ __forceinline__ void settle(Running<HT> (&x)[N]) {
  f32x4 acc[N][HT];
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int j = 0; j < HT; ++j) acc[t][j] = x[t].acc[j];
  settle(acc);
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int j = 0; j < HT; ++j) x[t].acc[j] = acc[t][j];
}

// ---- few tiles: the waves share them, take every WAVES-th 32 tokens of the span and join their states through LDS at the end ----
// One pass over the cache: keys and values go from memory into registers, become operands there and are not kept.  Eight waves with
// one tile have 128 registers each and are four to a SIMD, which hides the way to memory; with two tiles they convert once for
// both and are two to a SIMD.  Bound by memory for a row or a few over a long context (1 row behind 131071 tokens, 32 query heads on 8 of 128: 34 us, 4.2 TB/s; 32
// clients of 4 rows behind 8192: 57 us, 5.0 TB/s), by the conversion and the products for more rows (0.14 us for each 32 tokens of a
// tile and compute unit), and by latency where there is little (9 rows behind 2048 tokens 8.9 us: 1.2 until the first keys are
// asked for, 1.5 for them and their products, 1.2 for the waves' states, 3.5 to join the splits).
// LDS: states [tile][wave][row], later what joins the splits; then the queries that registers do not hold; words
template <int HD, int TILES, int WAVES>
constexpr size_t state_floats() { return (size_t)TILES * WAVES * 16 * (HD + kKv4PartPad); }
template <int HD, typename T, int TILES>
constexpr bool queries_in_lds() { return TILES * pieces<T>() * (HD / 8) > 32; }
template <int HD, typename T, int TILES, int WAVES>
constexpr size_t few_lds_bytes() {
  return state_floats<HD, TILES, WAVES>() * sizeof(float) + (queries_in_lds<HD, T, TILES>() ? (size_t)TILES * pieces<T>() * (HD / 32) * 1024 : 0) + 16;
}

template <int HD, typename T, int TILES, int WAVES>
__global__ __launch_bounds__(WAVES * 64, TILES == 1 ? 4 : 2) void kv4_attend_kernel(Kv4AttendCall a, Kv4Clients clients) {
  constexpr int NP = pieces<T>(), NS = HD / 32, HT = HD / 16, ROW = HD + kKv4PartPad, STEP = WAVES * 32;
  constexpr int NW = weight_pieces<T>(), SETS = sizeof(T) == 2 && HD == 64 ? 2 : 1;
  constexpr bool Q_LDS = queries_in_lds<HD, T, TILES>();
  typedef typename std::conditional<HD == 128, k4u32x4, k4u32x2>::type Codes;
  extern __shared__ float lds[];
  int* word = (int*)((char*)lds + few_lds_bytes<HD, T, TILES, WAVES>() - 16);

  const int kvh = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, g = lane >> 4;
  const Kv4Item it = find_item(clients, blockIdx.y, lane);
  const Work<HD, T> wk(a, clients, it, kvh, TILES);
  const int len = wk.len, span0 = it.split * clients.span, first = span0 + w * 32;

  // 64 steps' blocks sit in the lanes: lane L has the two of step L
  int step_blk[2];
  const int64_t block_bytes = (int64_t)a.view.n_kv_heads * Kv4Record<HD>::kBytes;
  const uint8_t* head_base = a.view.pool + (int64_t)a.layer * a.view.n_blocks * block_bytes + kvh * Kv4Record<HD>::kBytes;
  auto load_blocks = [&](int it0) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const int64_t tok = (int64_t)first + (int64_t)(it0 + lane) * STEP + tt * 16;
      step_blk[tt] = wk.table[tok < len ? (int)(tok / kBlockTokens) : 0];
    }
  };
  load_blocks(0);

  // ---- queries, and how far each row sees ----
  // (in registers, or where the sums leave no room for them in LDS: [tile][piece][step][lane])
  k4u32x4 q[Q_LDS ? 1 : TILES][NP][NS];
  k4u32x4* q_lds = (k4u32x4*)(lds + state_floats<HD, TILES, WAVES>()) + lane;
  int lim[TILES];
  int lo = len, hi = 0;
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const TileRow tr = wk.row(wk.first_row + t * 16 + c);
    load_queries<NP, NS>((const T*)a.q + tr.row * a.q_stride + tr.head * HD + g * (HD / 4), q[Q_LDS ? 0 : t]);
    if constexpr (Q_LDS) {  // (the waves write the same)
#pragma unroll
      for (int i = 0; i < NP * NS; ++i) q_lds[(t * NP * NS + i) * 64] = q[0][i / NS][i % NS];
    }
    lim[t] = wk.limit(tr);
    if (tr.live) lo = min(lo, lim[t]), hi = max(hi, lim[t]);
  }
  auto fold = [&](auto n) {
    constexpr int N = decltype(n)::value;
    lo = min(lo, (int)lanes_ror<N>((unsigned)lo));
    hi = max(hi, (int)lanes_ror<N>((unsigned)hi));
  };
  fold(std::integral_constant<int, 8>{});
  fold(std::integral_constant<int, 4>{});
  fold(std::integral_constant<int, 2>{});
  fold(std::integral_constant<int, 1>{});
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  const int end = min(it.split + 1 < wk.nsplit ? span0 + clients.span : len, hi);
  const int nsteps = end > first ? (end - first + STEP - 1) / STEP : 0;
  auto query = [&](int t, int piece, int st) {
    if constexpr (Q_LDS) return __builtin_bit_cast(bf16x8, q_lds[((t * NP + piece) * NS + st) * 64]);
    else return __builtin_bit_cast(bf16x8, q[t][piece][st]);
  };

  Running<HT> run[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) run[t].clear();
  const LaneOffsets<HD> at(c, g);
  const float c1 = kv4_scale<HD>();

  // (Keys and values of a step travel from where those of the step before have been used until they are, or with registers for two
  // sets from a step earlier: 32 clients of 4 rows behind 8192 tokens of head dim 64 38.7 us, 40.6 with one.)
  Codes k[SETS][2], v[SETS][2];
  unsigned kp[SETS][2], vp[SETS][2];
  auto record = [&](int i, int tt) {
    return head_base + (int64_t)__builtin_amdgcn_readlane(step_blk[tt], i & 63) * block_bytes;
  };
  auto request_keys = [&](int i, int set) {
    if (i >= nsteps) return;
    if (i > 0 && (i & 63) == 0) load_blocks(i);
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const uint8_t* rec = record(i, tt);
      k[set][tt] = *(const Codes*)(rec + at.k);
      kp[set][tt] = rec[at.kp];
    }
  };
  auto request_values = [&](int i, int set) {
    if (i >= nsteps) return;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const uint8_t* rec = record(i, tt);
      v[set][tt] = *(const Codes*)(rec + at.v);
      vp[set][tt] = *(const unsigned*)(rec + at.vp);
    }
  };
#pragma unroll
  for (int set = 0; set < SETS; ++set) request_keys(set, set), request_values(set, set);
  auto step = [&](int i, auto which) {
    constexpr int SET = decltype(which)::value;
    const int tok0 = first + i * STEP;
    const bool masked = tok0 + 32 > lo;  // (of the wave) some row does not see all 32 tokens
    f32x4 score[TILES][2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const float power = __uint_as_float(kp[SET][tt] << 23);
#pragma unroll
      for (int t = 0; t < TILES; ++t) score[t][tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        const bf16x8 key = key_operand(k[SET][tt][st], power);
#pragma unroll
        for (int m = NP - 1; m >= 0; --m)
#pragma unroll
          for (int t = 0; t < TILES; ++t) score[t][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, query(t, m, st), score[t][tt], 0, 0, 0);
      }
    }
    request_keys(i + SETS, SET);
    settle(score);
    bf16x8 p[TILES][NW];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      const f32x4 s0 = score[t][0], s1 = score[t][1];
      float sc[8] = {s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]};
      if (masked) hide(sc, tok0 + g * 4, lim[t]);
      const float top = top_of(sc);
      if (__ballot(top > run[t].moves) != 0) run[t].move_to(top, c1);
      run[t].weights(sc, c1, p[t]);
    }
    if (masked) {
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) drop_values<HD>(v[SET][tt], vp[SET][tt], len - (tok0 + tt * 16 + g * 4));
    }
#pragma unroll
    for (int b = 0; b < HT / 2; ++b) {
      k4u32x2 even2[2], odd2[2];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) value_operands<HD>(v[SET][tt], vp[SET][tt], b, even2[tt], odd2[tt]);
      const bf16x8 even = both_blocks(even2), odd = both_blocks(odd2);
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        f32x4& x = run[t].acc[2 * b];
        f32x4& y = run[t].acc[2 * b + 1];
#pragma unroll
        for (int m = 0; m < NW; ++m) {
          x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, p[t][m], x, 0, 0, 0);
          y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, p[t][m], y, 0, 0, 0);
        }
      }
    }
    request_values(i + SETS, SET);
    settle(run);
  };
#pragma unroll 1
  for (int i = 0; i < nsteps; i += SETS) {
    step(i, std::integral_constant<int, 0>{});
    if constexpr (SETS == 2)
      if (i + 1 < nsteps) step(i + 1, std::integral_constant<int, 1>{});
  }

  // ---- the waves' states joined: rows, or a split's partial rows (written through) ----
  constexpr int ROWS = TILES * 16, TPR = HD / 4, NT = WAVES * 64;
  const int rows_here = min(ROWS, wk.group_rows - wk.first_row), tasks = rows_here * TPR;  // a task: (row, 4 channels)
  float(*states)[WAVES][16][ROW] = (float(*)[WAVES][16][ROW])lds;  // a row: its channels, its maximum and sum
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < HT; j += 4)
        *(f32x4*)&states[t][w][c][(4 * g + i) * HT + j] = f32x4{run[t].acc[j][i], run[t].acc[j + 1][i], run[t].acc[j + 2][i], run[t].acc[j + 3][i]};
    const float l = fold_groups(run[t].l, LaneAdd{});
    if (g == 0) *(f32x2*)&states[t][w][c][HD] = f32x2{run[t].maximum(), l};
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
      wk.finish(wk.first_row + mr, e0, o, m, l);
    } else {
      float* dst = wk.all + ((size_t)it.split * ROWS + mr) * ROW;
      Xwg<true>::st4f(dst + e0, o);
      if (e0 == 0) Xwg<true>::st4f(dst + HD, f32x4{partial_maximum(m, l), l, 0.f, 0.f});
    }
  }
  if (wk.nsplit == 1 || clients.apart || !wk.arrives_last(word)) return;

  // ---- the splits joined ----
  // Their maxima and sums come to LDS at once; each thread then has a task, or several one after the other, and takes its
  // splits 8 at a time.  Threads that the tasks leave over share the splits of a task: thread (share, task) takes splits
  // share, share + shares, .., and the shares are joined through LDS in order.
  constexpr int BATCH = 8;
  static_assert(2 * kKv4MaxSplits * ROWS + NT * 5 <= (int)state_floats<HD, TILES, WAVES>(), "maxima, sums and shares fit the states' LDS");
  f32x2* stats = (f32x2*)lds;                      // [split][row]
  float* joined = lds + 2 * kKv4MaxSplits * ROWS;  // [share][task] 4 sums, the sum of weights
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
        const float sw = sp < wk.nsplit && ml.x != -INFINITY ? __builtin_amdgcn_exp2f(ml.x - m) : 0.f;
        l += ml.y * sw;
        o += ob[j] * sw;
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
    if (share == 0 && task < tasks) wk.finish(wk.first_row + mr, e0, o, m, l);
  }
}

// ---- many tiles: each of four waves has two of its own, 32 rows ----
// Keys and values are converted once, a block by each wave, into operands in LDS that all read; a barrier for every 64 tokens.
// Products of 32 x 32 x 16: 8 for a step's scores, 16 for its values (24 and 24 of an fp32 model), multiplied a step later: those, which depend
// on nothing of the step, travel with the weights' instructions, the score products with half of the next round's conversion.  (The
// matrix cores leave a wave 28 of a product's 32 cycles for other instructions, and one after another, products and instructions
// would take both times.)  Chunks that the compiler keeps in order do it: left to itself it puts the products side by side.
// Bound by the matrix cores' power: 2048 rows behind 6144 tokens, 32 query heads on 8 of 128, 300 to 320 us, 750 to 800
// TFLOP/s and, with two weights for each, 1.13 to 1.19 PFLOP/s of products, where a large matrix product of random numbers reaches
// 1.24; on zeros, which draw less, 250 us.  With two tiles more a wave and its SIMD's registers to itself, half the LDS reads:
// 337 us where this took 326, and the longest rows end alone.
//
// Layout of a product: operand lane (r, h) holds row (column) r, k = 8 h .. + 7; the result's register 4 u + i holds row 8 u + 4 h + i
// of column r.  Scores: k is channel h * HD / 2 + 8 s .. of step s.  Values: row r of product j is channel
// r % 16 * HD / 16 + r / 16 * HD / 32 + j, so that what 32 lanes store lies side by side, and k the tokens 4 h .. + 3 and 8 + 4 h .. + 3
// of a block, which is how the weights lie.
// LDS: keys [2 times 64 tokens][2 steps][HD / 16][lane], values [2 times 64 tokens][2 steps][HD / 32][block][lane] (before the walk: a
// few words)
template <int HD>
constexpr size_t many_lds_bytes() { return (size_t)8 * (HD / 16) * 64 * 16; }
typedef __attribute__((ext_vector_type(16))) float f32x16;

// whether a wave takes a SIMD's registers alone, half of them accumulation registers: then O^T is there
template <int HD, typename T>
constexpr bool alone() { return HD * pieces<T>() > 192; }

template <int HD, typename T>
__global__ __launch_bounds__(kKv4WideWaves * 64, (alone<HD, T>() ? 1 : 2)) void kv4_attend_many_kernel(Kv4AttendCall a, Kv4Clients clients) {
  constexpr int NP = pieces<T>(), NW = weight_pieces<T>(), KS = HD / 16, HT = HD / 32, ROW = HD + kKv4PartPad;
  constexpr int WAVES = kKv4WideWaves, WG_ROWS = WAVES * 32;
  constexpr bool ALONE = alone<HD, T>();
  typedef typename std::conditional<HD == 128, k4u32x4, k4u32x2>::type Codes;
  extern __shared__ float lds[];
  k4u32x4* key_lds = (k4u32x4*)lds;
  k4u32x4* value_lds = key_lds + 4 * KS * 64;
  int* word = (int*)lds;

  const int kvh = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, g = lane >> 4, gv = (g & 1) * 2 + (g >> 1), col = lane & 31, half = lane >> 5;
  const Kv4Item it = find_item(clients, blockIdx.y, lane);
  const Work<HD, T> wk(a, clients, it, kvh, WG_ROWS / 16);
  const int len = wk.len, span0 = it.split * clients.span;

  // the wave converts every fourth block: its next 64 sit in the lanes
  int my_blk;
  const int64_t block_bytes = (int64_t)a.view.n_kv_heads * Kv4Record<HD>::kBytes;
  const uint8_t* head_base = a.view.pool + (int64_t)a.layer * a.view.n_blocks * block_bytes + kvh * Kv4Record<HD>::kBytes;
  auto load_blocks = [&](int it0) {
    const int64_t tok = (int64_t)span0 + (int64_t)(it0 + lane) * 64 + w * 16;
    my_blk = wk.table[tok < len ? (int)(tok / kBlockTokens) : 0];
  };
  load_blocks(0);

  // ---- queries, and how far each row sees ----
  const int row0 = wk.first_row + w * 32;
  const bool idle = row0 >= wk.group_rows;  // (the wave has no row, and only converts)
  k4u32x4 q[NP][KS];
  const TileRow tr = wk.row(row0 + col);
  load_queries<NP, KS>((const T*)a.q + tr.row * a.q_stride + tr.head * HD + half * (HD / 2), q);
  const int lim = wk.limit(tr);
  int lo = tr.live ? lim : len, hi = tr.live ? lim : 0;
#pragma unroll
  for (int m = 1; m < 32; m *= 2) lo = min(lo, __shfl_xor(lo, m)), hi = max(hi, __shfl_xor(hi, m));
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  if (lane == 0) word[w] = hi;  // all waves walk as far as one of them has to
  __syncthreads();
#pragma unroll
  for (int ww = 0; ww < WAVES; ++ww) hi = max(hi, word[ww]);
  const int end = min(it.split + 1 < wk.nsplit ? span0 + clients.span : len, __builtin_amdgcn_readfirstlane(hi));
  const int rounds = end > span0 ? (end - span0 + 63) / 64 : 0;
  __syncthreads();

  // O^T; the row's -(running maximum) (infinity while nothing has been seen), the lane's own sum of weights
  f32x16 acc[1][HT];
  float neg_m = INFINITY, sum = 0.f;
#pragma unroll
  for (int j = 0; j < HT; ++j) acc[0][j] = f32x16{};
  const LaneOffsets<HD> at(c, g), at_v(c, gv);
  const float c1 = kv4_scale<HD>();

  // ---- this wave's block of a round: requested two rounds before it is converted ----
  Codes k_raw[2], v_raw[2];  // of even rounds, of odd ones
  unsigned k_pow[2], v_pow[2];
  auto record = [&](int i) { return head_base + (int64_t)__builtin_amdgcn_readlane(my_blk, i & 63) * block_bytes; };
  auto request_keys = [&](int i, int set) {
    if (i >= rounds) return;
    if (i > 0 && (i & 63) == 0) load_blocks(i);
    const uint8_t* rec = record(i);
    k_raw[set] = *(const Codes*)(rec + at.k);
    k_pow[set] = rec[at.kp];
  };
  auto request_values = [&](int i, int set) {  // (after the keys')
    if (i >= rounds) return;
    const uint8_t* rec = record(i);
    v_raw[set] = *(const Codes*)(rec + at_v.v);
    v_pow[set] = *(const unsigned*)(rec + at_v.vp);
  };
  // In pieces, so that little of each goes between two products.  (An LDS store of 16 bytes a lane takes 13 cycles of the compute unit,
  // a load 4: a round's stores are spread over its two steps.)
  k4u32x4* key_to;
  k4u32x2* value_to;
  auto open_keys = [&](int i) { key_to = key_lds + (((i & 1) * 2 + (w >> 1)) * KS + (g & 1) * (KS / 2)) * 64 + (g >> 1) * 32 + (w & 1) * 16 + c; };
  auto convert_keys = [&](int piece, int set) {  // lane (token c, quarter g): channels g * HD / 4 + 8 piece .. + 7
    key_to[piece * 64] = __builtin_bit_cast(k4u32x4, key_operand(k_raw[set][piece], __uint_as_float(k_pow[set] << 23)));
  };
  auto open_values = [&](int i, int set) {
    value_to = (k4u32x2*)(value_lds + (((i & 1) * 2 + (w >> 1)) * HT * 2 + (w & 1)) * 64 + (gv & 1) * 32 + c) + (gv >> 1);
    const int left = len - (span0 + i * 64 + w * 16);
    if (left < 16) drop_values<HD>(v_raw[set], v_pow[set], left - gv * 4);
  };
  auto convert_values = [&](int piece, int set) {  // lane (unit c, quarter gv): two channels of the unit, of tokens 4 gv .. + 3
    const int ch = 2 * piece;
    k4u32x2 even, odd;
    value_operands<HD>(v_raw[set], v_pow[set], piece, even, odd);
    value_to[(ch % HT * 2 * 64 + ch / HT * 16) * 2] = even;
    value_to[((ch + 1) % HT * 2 * 64 + (ch + 1) / HT * 16) * 2] = odd;
  };

  // A step's weights as NW operands a block.  Two sets: the step's, and those of the step before, whose products are still to come.
  unsigned weight[2][8][NW];
#pragma unroll
  for (int x = 0; x < 8; ++x)
#pragma unroll
    for (int m = 0; m < NW; ++m) weight[1][x][m] = 0u;
  auto operand = [](const unsigned (&x)[8][NW], int block, int m) {
    return __builtin_bit_cast(bf16x8, k4u32x4{x[4 * block][m], x[4 * block + 1][m], x[4 * block + 2][m], x[4 * block + 3][m]});
  };

  k4u32x4 key[KS];
  auto step = [&](int n, auto second, auto odd) {
    constexpr int NOW = decltype(second)::value, BEFORE = 1 - NOW, NEXT = 1 - decltype(odd)::value;  // of a round's two steps; the next round's set
    if constexpr (NOW == 0) open_keys(n / 2 + 1);
    else open_values(n / 2 + 1, NEXT);
    // Half of the next round's operands (behind the last round: nobody's).
    auto convert = [&](int piece) {
      if constexpr (NOW == 0) convert_keys(piece, NEXT);
      else convert_values(piece, NEXT);
    };
    auto request = [&] {
      if constexpr (NOW == 0) request_keys(n / 2 + 3, NEXT);
      else request_values(n / 2 + 3, NEXT);
    };
    if (idle) {
#pragma unroll
      for (int piece = 0; piece < KS / 2; ++piece) convert(piece);
      request();
      return;
    }
    const int tok0 = span0 + n * 32;
    const bool masked = tok0 + 32 > lo;  // (of the wave) some row does not see all 32 tokens
    const k4u32x4* from = value_lds + ((n == 0 ? 0 : n - 1) & 3) * HT * 2 * 64 + lane;  // (for the first step's weights of 0: its own)
    k4u32x4 value[2][HT];
    f32x16 score[1][1];
    score[0][0] = f32x16{};
#pragma unroll
    for (int st = 0; st < KS; ++st) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = NP - 1; m >= 0; --m)
        score[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, key[st]), __builtin_bit_cast(bf16x8, q[m][st]), score[0][0], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (st % 2 == 0) convert(st / 2);
      if (st == KS - 2) request();
      if (st >= KS - HT) value[0][st - (KS - HT)] = from[(st - (KS - HT)) * 2 * 64];
    }
    __builtin_amdgcn_sched_barrier(0);
    settle<ALONE>(score);
    float sc[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) sc[j] = plain(score[0][0][j]);
    if (masked) {
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (tok0 + (j >> 2) * 8 + half * 4 + (j & 3) >= lim) sc[j] = -INFINITY;
    }
    // The step before's products, and between them two weights of this step at a time; a step's last keys are read for the next.
    constexpr int PRODUCTS = 2 * NW * HT;  // an eighth of them for each pair of weights
    float total = 0.f, p[2];
    auto weigh = [&](int x, float neg) {
      p[0] = __builtin_amdgcn_exp2f(fmaf(sc[2 * x], c1, neg));
      p[1] = __builtin_amdgcn_exp2f(fmaf(sc[2 * x + 1], c1, neg));
    };
    auto keep = [&](int x) {
      split_weights(p[0], p[1], weight[NOW][x]);
      total += p[0] + p[1];
    };
    const k4u32x4* keys = key_lds + ((n + 1) & 3) * KS * 64 + lane;
    unsigned long long move = 0;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const int first = x * PRODUCTS / 8, behind = (x + 1) * PRODUCTS / 8;
#pragma unroll
      for (int y = first; y < behind; ++y) {
        const int block = y / (NW * HT), m = y / HT % NW, j = y % HT;
        __builtin_amdgcn_sched_barrier(0);
        acc[0][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, value[block][j]), operand(weight[BEFORE], block, m), acc[0][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if (y == first) {
          if (x == 0) weigh(0, neg_m);
          keep(x);
          asm volatile("" ::"v"(weight[NOW][x][NW - 1]));  // (here, not behind the branch below)
          if (x < HT) value[1][x] = from[(x * 2 + 1) * 64];
          if (x >= 8 - KS) key[x - (8 - KS)] = keys[(x - (8 - KS)) * 64];
          if (x == 7) move = __ballot(!(total <= 4096.f));  // (before the last product: the branch need not wait for it)
        }
        if (y == behind - 1 && x < 7) weigh(x + 1, neg_m);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    // A maximum moves only when the weights it leaves have grown to 2^12 (any scale will do for fp32 sums), or when a row sees
    // something for the first time: an infinite total, or none.
    if (move != 0) {
      settle<ALONE>(acc);
      float top = max3(max3(sc[0], sc[1], sc[2]), max3(sc[3], sc[4], sc[5]), max3(sc[6], sc[7], sc[8]));
      top = max3(top, max3(sc[9], sc[10], sc[11]), max3(sc[12], sc[13], max3(sc[14], sc[15], top)));
      const float m_old = -neg_m, m_new = fmaxf(m_old, fold32(top, LaneMax{}) * c1);
      const float alpha = m_new == m_old ? 1.f : __builtin_amdgcn_exp2f(m_old - m_new);
      neg_m = -m_new;
      sum *= alpha;
#pragma unroll
      for (int j = 0; j < HT; ++j) acc[0][j] *= alpha;
      total = 0.f;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        weigh(x, m_new == -INFINITY ? 0.f : -m_new);
        keep(x);
      }
    }
    sum += total;
  };

  if (rounds > 0) {
    request_keys(0, 0);
    request_values(0, 0);
    request_keys(1, 1);
    request_values(1, 1);
    open_keys(0);
    open_values(0, 0);
#pragma unroll
    for (int piece = 0; piece < KS / 2; ++piece) convert_keys(piece, 0), convert_values(piece, 0);
    request_keys(2, 0);
    request_values(2, 0);
    __syncthreads();
#pragma unroll
    for (int st = 0; st < KS; ++st) key[st] = key_lds[st * 64 + lane];
    // Between two barriers, the second step of round i - 1 and the first of round i: they read keys of round i, as operands of the
    // steps to come, and values of round i - 1, and write values of round i and keys of round i + 1.
    typedef std::integral_constant<int, 0> Zero;
    typedef std::integral_constant<int, 1> One;
#pragma unroll 1
    for (int i = 0; i < rounds; i += 2) {
      step(2 * i, Zero{}, Zero{});
      __syncthreads();
      step(2 * i + 1, One{}, Zero{});
      if (i + 1 == rounds) break;
      step(2 * i + 2, Zero{}, One{});
      __syncthreads();
      step(2 * i + 3, One{}, One{});
    }
    const k4u32x4* from = value_lds + ((2 * rounds - 1) & 3) * HT * 2 * 64 + lane;
#pragma unroll
    for (int block = 0; block < 2; ++block)
#pragma unroll
      for (int j = 0; j < HT; ++j) {
        const bf16x8 value = __builtin_bit_cast(bf16x8, from[(j * 2 + block) * 64]);
#pragma unroll
        for (int m = 0; m < NW; ++m) acc[0][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value, operand(weight[1], block, m), acc[0][j], 0, 0, 0);
      }
    settle<ALONE>(acc);
  }
  if (idle) return;

  // ---- rows, or a split's partial rows ----
  const float m = -neg_m, l = fold32(sum, LaneAdd{});
  float* dst = wk.all + ((size_t)it.split * WG_ROWS + w * 32 + col) * ROW;
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < HD / 16; e += 4) {  // of unit 8 u + 4 half + i
        const int ch = (8 * u + 4 * half + i) * (HD / 16) + e;
        f32x4 o;
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = acc[0][(e + k) % HT][4 * (u + (e + k) / HT * 2) + i];
        if (wk.nsplit == 1) wk.finish(row0 + col, ch, o, m, l);
        else if (rounds > 0 && tr.live) *(f32x4*)(dst + ch) = o;  // (nothing seen: nothing to read)
      }
  if (wk.nsplit > 1 && half == 0 && tr.live) *(f32x2*)(dst + HD) = f32x2{partial_maximum(m, l), l};
}

// ---- the splits of a group of tiles joined by a kernel of its own: a group's splits have a workgroup each, as in the walk, for its share
// of the rows.  What a join takes is the way to memory, 1.7 us for a thread's next 8 splits of its next 4 channels: by the walk's last
// workgroup alone (which starts 2 us sooner) 16 splits of 32 rows took 13 us, 8 of 128 rows 40. ----
// Partial sums of splits s0, s0 + step, .. added to a row's.
template <int N>
__device__ __forceinline__ void add_splits(const f32x4 (&ob)[N], const f32x2 (&ml)[N], int s0, int step, int nsplit, float& m, float& l, f32x4& o) {
  float m_new = m;
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (s0 + j * step < nsplit) m_new = fmaxf(m_new, ml[j].x);
  if (m_new == -INFINITY) return;
  const float alpha = m_new == m ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
  l *= alpha;
  o *= alpha;
  m = m_new;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (s0 + j * step >= nsplit || ml[j].x == -INFINITY) continue;  // (a split that saw nothing may have written no values)
    const float sw = __builtin_amdgcn_exp2f(ml[j].x - m);
    l += ml[j].y * sw;
    o += ob[j] * sw;
  }
}
// A thread has 4 channels of a row (a task); threads that the tasks leave over share a task's splits: thread (share, task) takes splits
// share, share + shares, .., 8 at a time, and the shares are joined through LDS in order.
template <int HD, typename T, int WG_ROWS>
__global__ __launch_bounds__(256) void kv4_join_kernel(Kv4AttendCall a, Kv4Clients clients) {
  constexpr int ROW = HD + kKv4PartPad, TPR = HD / 4, NT = 256, BATCH = 8;
  __shared__ float joined[NT * 6];
  const int tid = threadIdx.x;
  const Kv4Item it = find_item(clients, blockIdx.y, tid & 63);
  const Work<HD, T> wk(a, clients, it, blockIdx.x, WG_ROWS / 16);
  if (wk.nsplit == 1) return;
  const int per = (WG_ROWS + wk.nsplit - 1) / wk.nsplit, from = it.split * per;
  const int tasks = min(per, min(WG_ROWS, wk.group_rows - wk.first_row) - from) * TPR;
  if (tasks <= 0) return;
  int log_tasks = 31 - __builtin_clz(TPR);  // (their number made a power of two)
  while ((1 << log_tasks) < tasks) ++log_tasks;
  const int shares = max(1, NT >> log_tasks), share = shares > 1 ? tid >> log_tasks : 0;
#pragma unroll 1
  for (int k0 = 0; k0 < tasks; k0 += NT) {
    const int task = k0 + (tid & ((1 << log_tasks) - 1)), mr = from + min(task, tasks - 1) / TPR, e0 = (task % TPR) * 4;
    const float* p0 = wk.all + (size_t)mr * ROW;
    float m = -INFINITY, l = 0.f;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s0 = share; s0 < wk.nsplit; s0 += BATCH * shares) {
      f32x4 ob[BATCH];
      f32x2 ml[BATCH];
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        const float* ps = p0 + (size_t)min(s0 + j * shares, wk.nsplit - 1) * (WG_ROWS * ROW);
        ml[j] = *(const f32x2*)(ps + HD);
        ob[j] = *(const f32x4*)(ps + e0);
      }
      add_splits(ob, ml, s0, shares, wk.nsplit, m, l, o);
    }
    if (shares > 1) {  // (then this is the only turn)
      float* x = joined + tid * 6;
      x[0] = o[0], x[1] = o[1], x[2] = o[2], x[3] = o[3], x[4] = l, x[5] = m;
      __syncthreads();
      for (int sh = 1; share == 0 && sh < shares; ++sh) {
        const float* y = joined + ((sh << log_tasks) + tid) * 6;
        const f32x4 one_o[1] = {f32x4{y[0], y[1], y[2], y[3]}};
        const f32x2 one_ml[1] = {f32x2{y[5], y[4]}};
        add_splits(one_o, one_ml, 0, 1, 1, m, l, o);
      }
    }
    if (share == 0 && task < tasks) wk.finish(wk.first_row + mr, e0, o, m, l);
  }
}

template <class K>
static hipError_t allow_and_launch(K kernel, std::atomic<uint64_t>& allowed, size_t lds, int threads, const Kv4AttendCall& c, const Kv4Clients& cl,
                                   hipStream_t st) {
  if (lds > 64 * 1024) {
    const hipError_t e = allow_lds(allowed, (const void*)kernel, lds);
    if (e != hipSuccess) return e;
  }
  if (cl.items > kKv4MaxItems) return hipErrorInvalidValue;  // (the plan's launches have no more)
  kernel<<<dim3(c.view.n_kv_heads, cl.items), threads, lds, st>>>(c, cl);
  return hipGetLastError();
}
template <int HD, typename T, int WG_ROWS>
static hipError_t join(hipError_t e, const Kv4AttendCall& c, const Kv4Clients& cl, hipStream_t st) {
  if (e != hipSuccess || !cl.apart) return e;
  kv4_join_kernel<HD, T, WG_ROWS><<<dim3(c.view.n_kv_heads, cl.items), 256, 0, st>>>(c, cl);
  return hipGetLastError();
}
template <int HD, typename T, int TILES>
static hipError_t attend_few(const Kv4AttendCall& c, const Kv4Clients& cl, hipStream_t st) {
  static std::atomic<uint64_t> allowed{0};
  constexpr int WAVES = kKv4FewWaves;
  return join<HD, T, TILES * 16>(
      allow_and_launch(kv4_attend_kernel<HD, T, TILES, WAVES>, allowed, few_lds_bytes<HD, T, TILES, WAVES>(), WAVES * 64, c, cl, st), c, cl, st);
}
template <int HD, typename T>
static hipError_t attend_of(const Kv4AttendCall& c, const Kv4Launch& l, hipStream_t st) {
  static std::atomic<uint64_t> allowed{0};
  if (l.wide)
    return join<HD, T, kKv4WideTiles * 16>(
        allow_and_launch(kv4_attend_many_kernel<HD, T>, allowed, many_lds_bytes<HD>(), kKv4WideWaves * 64, c, l.c, st), c, l.c, st);
  if (l.tiles == 1) return attend_few<HD, T, 1>(c, l.c, st);
  if constexpr (sizeof(T) == 2)
    if (l.tiles == 2) return attend_few<HD, T, 2>(c, l.c, st);
  return hipErrorInvalidValue;
}
hipError_t launch_kv4_attend(const Kv4AttendCall& c, const Kv4Launch& l, hipStream_t st) {
  if (c.head_dim == 128) return c.dtype == PIPESD_F32 ? attend_of<128, float>(c, l, st) : attend_of<128, uint16_t>(c, l, st);
  return c.dtype == PIPESD_F32 ? attend_of<64, float>(c, l, st) : attend_of<64, uint16_t>(c, l, st);
}

// ------------------------------------------------------------------------------------------------
// weights given to the cached tokens, once the rows' sums are known
// ------------------------------------------------------------------------------------------------
// Workgroup (cache head, tokens, client): each wave has TT * 16 tokens' keys in registers and meets all query rows, whose
// tiles the four waves bring through LDS four at a time.  One writer per token, sums in a fixed order.  The scores are formed again: kept,
// they would be 30 times the keys' bytes at 32 rows of 4 heads.  Bound by the way from block table to keys to products that each
// short workgroup goes: 32 rows behind 12001 tokens of 8 heads of 64 8.0 us, 38 behind 65536 of 128 (64 tokens a wave in place of
// 32: 10.9 and 39.9).  For many rows by what stands behind every tile's products, their wait and the exponentials: 2048 rows behind 6144
// tokens, 32 query heads on 8 of 128, 289 us beside the attention's 307, where the products alone are 96; in fp32 527 and 589.
template <int HD, typename T>
__global__ __launch_bounds__(256) void kv4_mass_kernel(Kv4AttendCall a, Kv4Clients cl, int first_piece) {
  constexpr int NP = pieces<T>(), NS = HD / 32, TT = 2;
  typedef typename std::conditional<HD == 128, k4u32x4, k4u32x2>::type Codes;
  __shared__ k4u32x4 q_lds[4][NP * NS][64];
  __shared__ float lse_lds[4][16];
  __shared__ int lim_lds[4][16];
  const int kvh = blockIdx.x, ci = blockIdx.z, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int c = lane & 15, g = lane >> 4;
  const int len = cl.len[ci], n_rows = cl.n_rows[ci], row_off = cl.row_off[ci];
  const int piece = first_piece + (int)blockIdx.y, tok0 = (piece * 4 + w) * TT * 16;
  if (piece * 4 * TT * 16 >= len) return;  // (whole workgroup)
  const int group = a.group;
  const float group_rinv = __builtin_amdgcn_rcpf((float)group);
  const int nqt = (n_rows * group + 15) / 16;
  const int32_t* table = a.view.table + cl.table_off[ci];
  const LaneOffsets<HD> at(c, g);
  const float c1 = kv4_scale<HD>();
  bf16x8 k[TT][NS];
  float sum[TT][4];
#pragma unroll
  for (int tt = 0; tt < TT; ++tt) {
    const int t = tok0 + tt * 16;
    const uint8_t* rec = a.view.pool + kv4_record<HD>(a.view, a.layer, table[t < len ? t / kBlockTokens : 0], kvh);
    const Codes codes = *(const Codes*)(rec + at.k);
    const float power = __uint_as_float((unsigned)rec[at.kp] << 23);
#pragma unroll
    for (int st = 0; st < NS; ++st) k[tt][st] = key_operand(codes[st], power);
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[tt][i] = 0.f;
  }
  for (int q0 = 0; q0 < nqt; q0 += 4) {
    if (q0 > 0) __syncthreads();  // the tiles before have been read
    {
      const TileRow tr = tile_row((q0 + w) * 16 + c, group, group_rinv, n_rows, row_off, kvh);
      k4u32x4 q[NP][NS];
      load_queries<NP, NS>((const T*)a.q + tr.row * a.q_stride + tr.head * HD + g * (HD / 4), q);
#pragma unroll
      for (int i = 0; i < NP * NS; ++i) q_lds[w][i][lane] = q[i / NS][i % NS];
      if (g == 0) {
        lse_lds[w][c] = tr.live ? a.lse[(size_t)tr.row * a.n_q_heads + tr.head] : INFINITY;
        lim_lds[w][c] = tr.live ? row_limit(a.limits, tr.row, row_off, n_rows, len) : 0;
      }
    }
    __syncthreads();
#pragma unroll 1
    for (int t = 0; t < min(4, nqt - q0); ++t) {
      const float lse = lse_lds[t][c];
      const int lim = lim_lds[t][c];
      if (__ballot(lim > tok0) == 0) continue;
      f32x4 score[1][TT];
#pragma unroll
      for (int tt = 0; tt < TT; ++tt) score[0][tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = NP * NS - 1; i >= 0; --i) {
        const bf16x8 q = __builtin_bit_cast(bf16x8, q_lds[t][i][lane]);
#pragma unroll
        for (int tt = 0; tt < TT; ++tt) score[0][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[tt][i % NS], q, score[0][tt], 0, 0, 0);
      }
      settle(score);
      float p[2][4];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[tt][i] = __builtin_amdgcn_exp2f(fmaf(score[0][tt][i], c1, -lse));
      if (__ballot(lim < tok0 + 32) != 0) {  // some row does not see all of the wave's tokens
        asm volatile("");                    // (a branch: eight selections for every tile would be a third of its time)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int i = 0; i < 4; ++i) p[tt][i] = tok0 + tt * 16 + g * 4 + i < lim ? p[tt][i] : 0.f;
      }
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[tt][i] += p[tt][i];
    }
  }
  float* out = a.mass + (((int64_t)cl.seq[ci] * a.view.n_layers + a.layer) * a.view.n_kv_heads + kvh) * a.mass_stride;
#pragma unroll
  for (int tt = 0; tt < TT; ++tt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x = sum[tt][i];
      x += __uint_as_float(lanes_ror<8>(__float_as_uint(x)));
      x += __uint_as_float(lanes_ror<4>(__float_as_uint(x)));
      x += __uint_as_float(lanes_ror<2>(__float_as_uint(x)));
      x += __uint_as_float(lanes_ror<1>(__float_as_uint(x)));
      const int t = tok0 + tt * 16 + g * 4 + i;
      if (c == 0 && t < len) out[t] = (a.decay != 0.f && t < len - n_rows ? a.decay * out[t] : 0.f) + x;
    }
}

template <int HD, typename T>
static hipError_t mass_of(const Kv4AttendCall& a, const Kv4Clients& cl, hipStream_t st) {
  int most = 0;
  for (int i = 0; i < cl.n; ++i) most = std::max(most, (int)cl.len[i]);
  const int pieces = most / 128 + (most % 128 != 0);
  for (int first = 0; first < pieces; first += kKv4MaxItems)
    kv4_mass_kernel<HD, T><<<dim3(a.view.n_kv_heads, std::min(pieces - first, kKv4MaxItems), cl.n), 256, 0, st>>>(a, cl, first);
  return hipGetLastError();
}
hipError_t launch_kv4_mass(const Kv4AttendCall& c, const Kv4Clients& cl, hipStream_t st) {
  if (c.head_dim == 128) return c.dtype == PIPESD_F32 ? mass_of<128, float>(c, cl, st) : mass_of<128, uint16_t>(c, cl, st);
  return c.dtype == PIPESD_F32 ? mass_of<64, float>(c, cl, st) : mass_of<64, uint16_t>(c, cl, st);
}

// Of a client without rows nothing is added.  Workgroup (cache head, 1024 tokens, client); what it reads and writes bounds it.
constexpr int kDecayPer = 4;
__global__ __launch_bounds__(256) void kv4_decay_kernel(Kv4AttendCall a, Kv4Idle cl, int first_piece) {
  const int ci = blockIdx.z, len = cl.len[ci];
  float* out = a.mass + (((int64_t)cl.seq[ci] * a.view.n_layers + a.layer) * a.view.n_kv_heads + blockIdx.x) * a.mass_stride;
  const int t0 = (first_piece + (int)blockIdx.y) * (256 * kDecayPer) + (int)threadIdx.x;
#pragma unroll
  for (int i = 0; i < kDecayPer; ++i) {
    const int t = t0 + i * 256;
    if (t < len) out[t] = a.decay != 0.f ? a.decay * out[t] : 0.f;  // (0: whatever was there)
  }
}
hipError_t launch_kv4_decay(const Kv4AttendCall& c, const Kv4Idle& cl, hipStream_t st) {
  constexpr int kPiece = 256 * kDecayPer;
  const int pieces = cl.most / kPiece + (cl.most % kPiece != 0);
  for (int first = 0; first < pieces; first += kKv4MaxItems)
    kv4_decay_kernel<<<dim3(c.view.n_kv_heads, std::min(pieces - first, kKv4MaxItems), cl.n), 256, 0, st>>>(c, cl, first);
  return hipGetLastError();
}

}  // namespace pipesd
