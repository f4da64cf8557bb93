// Attention over the 4-bit cache, and the weights it gave to the cached tokens.
//
//   o_r = sum_t p_rt v_t,   p_rt = exp(s_rt) / sum_t' exp(s_rt'),   s_rt = q_r . k_t / sqrt(head_dim),
// over the first lim_r tokens; a row with none has no weights, and o_r = 0.  mass_t = sum over rows and heads of p_rt.
//
// Keys and values become bf16 on their way to the matrix cores, exactly (two bits and a power of two).  The queries of a bf16
// model are operands as they are, those of an fp32 model are cut into three bf16 numbers (24 bits, so exactly): scores are as
// good as fp32 ones.  Weights are cut into two bf16 numbers (16 bits), as everywhere in this library: only the cache itself
// is coarse.  Maxima and sums are fp32.
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

template <int HD, int NP>
struct Queries {  // one tile of 16 rows as operand B: piece p, step s
  k4u32x4 q[NP][HD / 32];
};

template <int HD>
__device__ __forceinline__ float kv4_scale() { return (HD == 128 ? 0.08838834764831845f : 0.125f) * 1.44269504088896341f; }  // log2(e) / sqrt(HD)

// Lane (c, g) of a product's operands holds 8 channels of row c; in step s these are g * HD / 4 + 8 s .. + 7, so that what a lane
// needs of a key in all steps is one load, and of one power.
template <int HD, int NP, typename T>
__device__ __forceinline__ void load_queries(const T* row, bool live, int g, Queries<HD, NP>& out) {
#pragma unroll
  for (int s = 0; s < HD / 32; ++s) {
    const T* p = row + g * (HD / 4) + s * 8;
    if constexpr (sizeof(T) == 2) {
      const k4u32x4 x = *(const k4u32x4*)p;
      out.q[0][s] = live ? x : k4u32x4{0u, 0u, 0u, 0u};
    } else {
      const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
      float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = live ? x[i] : 0.f;
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
        out.q[m][s] = k4u32x4{w[0], w[1], w[2], w[3]};
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
template <int TILES, int HT>
__device__ __forceinline__ void settle(f32x4 (&acc)[TILES][HT]) {
#pragma unroll
  for (int t = TILES - 1; t >= 0; --t) {
    auto& x = acc[t];
    if (t == 0) {
      if constexpr (HT == 8)
        asm volatile("s_nop 15\n\ts_nop 1" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]), "+v"(x[6]), "+v"(x[7]));
      else if constexpr (HT == 2)
        asm volatile("s_nop 15\n\ts_nop 1" : "+v"(x[0]), "+v"(x[1]));
      else
        asm volatile("s_nop 15\n\ts_nop 1" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]));
    } else {
      if constexpr (HT == 2)
        asm volatile("" : "+v"(x[0]), "+v"(x[1]));
      else if constexpr (HT == 8)
        asm volatile("" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]), "+v"(x[6]), "+v"(x[7]));
      else
        asm volatile("" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]));
    }
  }
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
// p = hi + lo, each four pairs of bf16 numbers.  lo rounds p - hi, which is exact: a product with (-1, 0) or (0, -1) and a sum.
// (Through the builtin the product accumulates in place, a copy each, and a factor that is a constant of the instruction sits
// in the other half than the compiler takes it to.  Three wait states before anything reads such a product's result.)
__device__ __forceinline__ void split_weights(const float (&p)[8], unsigned (&hi)[4], unsigned (&lo)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) hi[i] = pack2_bf16(p[2 * i], p[2 * i + 1]);
#if defined(__HIP_DEVICE_COMPILE__)
  float r[8];
  asm("s_nop 0\n\t"
      "v_dot2_f32_bf16 %0, %8, %20, %12\n\t"
      "v_dot2_f32_bf16 %1, %8, %21, %13\n\t"
      "v_dot2_f32_bf16 %2, %9, %20, %14\n\t"
      "v_dot2_f32_bf16 %3, %9, %21, %15\n\t"
      "v_dot2_f32_bf16 %4, %10, %20, %16\n\t"
      "v_dot2_f32_bf16 %5, %10, %21, %17\n\t"
      "v_dot2_f32_bf16 %6, %11, %20, %18\n\t"
      "v_dot2_f32_bf16 %7, %11, %21, %19\n\t"
      "s_nop 3"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
      : "v"(hi[0]), "v"(hi[1]), "v"(hi[2]), "v"(hi[3]), "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "v"(p[4]), "v"(p[5]), "v"(p[6]),
        "v"(p[7]), "s"(0x0000bf80u), "s"(0xbf800000u));
#pragma unroll
  for (int i = 0; i < 4; ++i) lo[i] = pack2_bf16(r[2 * i], r[2 * i + 1]);
#endif
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

// A wave walks tokens 32 at a time.  Per tile of 16 query rows it keeps a running maximum, sum and O^T in registers; the maximum moves
// only when a score passes it by 2^8 (any scale will do for fp32 sums: most steps then need no exchange between lanes and
// no rescaling).
// FEW tiles: the waves share them and join their states through LDS at the end.  MANY: each wave has its own; keys and values
// are converted once, by the four waves in turn (one a block's keys, one its values), into operands in LDS that all read:
// two steps by turns, one barrier a step.
// LDS: states [tile][wave][row], later what joins the splits, or operands [2 steps]([2 blocks][steps of a product][lane] keys,
// [tile of channels][lane] values); then the queries that registers do not hold; words
template <int HD, int TILES, int WAVES, bool WIDE>
constexpr size_t state_floats() {
  return WIDE ? 2 * (2 * (HD / 32) + HD / 16) * 64 * 4 : (size_t)TILES * WAVES * 16 * (HD + kKv4PartPad);
}
template <typename T>
constexpr int pieces() { return sizeof(T) == 4 ? 3 : 1; }
template <int HD, typename T, int TILES, bool WIDE>
constexpr bool queries_in_lds() { return !WIDE && TILES * pieces<T>() * (HD / 8) > 32; }
template <int HD, typename T, int TILES, int WAVES, bool WIDE>
constexpr size_t attend_lds_bytes() {
  return state_floats<HD, TILES, WAVES, WIDE>() * sizeof(float) + (queries_in_lds<HD, T, TILES, WIDE>() ? (size_t)TILES * sizeof(Queries<HD, pieces<T>()>) * 64 : 0) + 32;
}
template <int HD, typename T, int TILES, bool WIDE>
constexpr int attend_waves_per_simd() { return WIDE ? (sizeof(T) == 4 ? 2 : 3) : TILES == 1 ? 4 : 2; }

template <int HD, typename T, int TILES, int WAVES, bool WIDE>
__global__ __launch_bounds__(WAVES * 64, (attend_waves_per_simd<HD, T, TILES, WIDE>())) void kv4_attend_kernel(Kv4AttendCall a, Kv4Clients clients) {
  constexpr int NP = pieces<T>(), NS = HD / 32, HT = HD / 16, ROW = HD + kKv4PartPad;
  constexpr bool Q_LDS = queries_in_lds<HD, T, TILES, WIDE>();
  constexpr int WG_TILES = WIDE ? WAVES * TILES : TILES;
  constexpr int STEP = WIDE ? 32 : WAVES * 32;
  typedef typename std::conditional<HD == 128, k4u32x4, k4u32x2>::type Codes;
  extern __shared__ float lds[];
  int* last_lds = (int*)((char*)lds + attend_lds_bytes<HD, T, TILES, WAVES, WIDE>() - 32);

  const int kvh = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, g = lane >> 4;
  const Kv4Item it = find_item(clients, blockIdx.y, lane);
  const int len = clients.len[it.ci], n_rows = clients.n_rows[it.ci], row_off = clients.row_off[it.ci];
  const int groups = clients.groups[it.ci], nsplit = clients.nsplit[it.ci];
  const int group = a.group;
  const float group_rinv = __builtin_amdgcn_rcpf((float)group);
  const int R = n_rows * group;
  const int tile0 = it.group * WG_TILES + (WIDE ? w * TILES : 0);
  const int span0 = it.split * clients.span;
  const int32_t* table = a.view.table + clients.table_off[it.ci];

  const int first = span0 + (WIDE ? 0 : w * 32);
  // the records of 64 steps' blocks sit in the lanes: lane L has where the two of step L begin
  int64_t step_rec[2];
  const int64_t block_bytes = (int64_t)a.view.n_kv_heads * Kv4Record<HD>::kBytes;
  const uint8_t* head_base = a.view.pool + (int64_t)a.layer * a.view.n_blocks * block_bytes + kvh * Kv4Record<HD>::kBytes;
  auto load_blocks = [&](int it0) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const int64_t tok = (int64_t)first + (int64_t)(it0 + lane) * STEP + tt * 16;
      step_rec[tt] = table[tok < len ? (int)(tok / kBlockTokens) : 0] * block_bytes;
    }
  };
  load_blocks(0);

  // ---- queries, and how far each row sees ----
  // (in registers, or where the sums leave no room for them in LDS: [tile][piece][step][lane])
  Queries<HD, NP> q[Q_LDS ? 1 : TILES];
  k4u32x4* q_lds = (k4u32x4*)(lds + state_floats<HD, TILES, WAVES, WIDE>()) + lane;
  int lim[TILES];
  int lo = len, hi = 0;
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const TileRow tr = tile_row((tile0 + t) * 16 + c, group, group_rinv, n_rows, row_off, kvh);
    load_queries<HD, NP>((const T*)a.q + tr.row * a.q_stride + tr.head * HD, tr.live, g, q[Q_LDS ? 0 : t]);
    if constexpr (Q_LDS) {  // (the waves of one set of tiles write the same)
#pragma unroll
      for (int i = 0; i < NP * NS; ++i) q_lds[(t * NP * NS + i) * 64] = q[0].q[i / NS][i % NS];
    }
    lim[t] = row_limit(a.limits, tr.row, row_off, n_rows, len);
    if (tr.live) lo = min(lo, lim[t]), hi = max(hi, lim[t]);
  }
#pragma unroll
  for (int m = 1; m < 16; m *= 2) lo = min(lo, __shfl_xor(lo, m)), hi = max(hi, __shfl_xor(hi, m));
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  const int wave_hi = hi;
  if constexpr (WIDE) {  // all waves walk as far as one of them has to
    if (lane == 0) last_lds[w] = hi;
    __syncthreads();
#pragma unroll
    for (int ww = 0; ww < WAVES; ++ww) hi = max(hi, last_lds[ww]);
    hi = __builtin_amdgcn_readfirstlane(hi);
  }
  const int end = min(min(span0 + clients.span, len), hi);
  const int nsteps = end > first ? (end - first + STEP - 1) / STEP : 0;

  f32x4 acc[TILES][HT];
  // per row: -(running maximum) (0 while nothing has been seen), the score that moves it, the sum of weights
  float neg_m[TILES], moves[TILES], l_run[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    neg_m[t] = 0.f;
    moves[t] = -INFINITY;
    l_run[t] = 0.f;
#pragma unroll
    for (int j = 0; j < HT; ++j) acc[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  auto query = [&](int t, int piece, int st) {
    if constexpr (Q_LDS) return __builtin_bit_cast(bf16x8, q_lds[((t * NP + piece) * NS + st) * 64]);
    else return __builtin_bit_cast(bf16x8, q[t].q[piece][st]);
  };
  const LaneOffsets<HD> at(c, g);
  const float c1 = kv4_scale<HD>();

  struct Raw {
    Codes k[2], v[2];
    unsigned kp[2], vp[2];
  };
  // (Keys and values of a step travel from where those of the step before have been used until they are.)
  constexpr int DEPTH = 1;
  Raw raw[DEPTH];
  Raw& r = raw[0];  // (MANY)
  auto record = [&](int i, int tt) {
    const unsigned lo = __builtin_amdgcn_readlane((unsigned)step_rec[tt], i & 63), hi = __builtin_amdgcn_readlane((unsigned)(step_rec[tt] >> 32), i & 63);
    return head_base + (int64_t)(((uint64_t)hi << 32) | lo);
  };
  auto request_keys = [&](Raw& r, int i) {
    if (i >= nsteps) return;
    if (i > 0 && (i & 63) == 0) load_blocks(i);
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const uint8_t* rec = record(i, tt);
      r.k[tt] = *(const Codes*)(rec + at.k);
      r.kp[tt] = rec[at.kp];
    }
  };
  auto request_values = [&](Raw& r, int i) {
    if (i >= nsteps) return;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const uint8_t* rec = record(i, tt);
      r.v[tt] = *(const Codes*)(rec + at.v);
      r.vp[tt] = *(const unsigned*)(rec + at.vp);
    }
  };
  // MANY: this wave's part of a step is one block's keys (tt), or its values
  k4u32x4* ops = (k4u32x4*)lds;
  constexpr int OPS = (2 * NS + HT) * 64;  // of a step
  auto part_of_step = [&](int i) { return (w + 2 * (i & 1)) & 3; };
  auto request_part = [&](int i) {
    if (i >= nsteps) return;
    if (i > 0 && (i & 63) == 0) load_blocks(i);
    const int part = part_of_step(i);
    const uint8_t* rec = record(i, part & 1);
    if (part < 2) {
      r.k[0] = *(const Codes*)(rec + at.k);
      r.kp[0] = rec[at.kp];
    } else {
      r.k[0] = *(const Codes*)(rec + at.v);
      r.kp[0] = *(const unsigned*)(rec + at.vp);
    }
  };
  auto convert_part = [&](int i) {
    if (i >= nsteps) return;
    const int part = part_of_step(i), tt = part & 1;
    k4u32x4* to = ops + (i & 1) * OPS + lane;
    if (part < 2) {
      const float power = __uint_as_float(r.kp[0] << 23);
#pragma unroll
      for (int st = 0; st < NS; ++st) to[(tt * NS + st) * 64] = __builtin_bit_cast(k4u32x4, key_operand(r.k[0][st], power));
    } else {
      const int left = len - (first + i * STEP + tt * 16);
      if (left < 16) drop_values<HD>(r.k[0], r.kp[0], left - g * 4);
#pragma unroll
      for (int b = 0; b < HT / 2; ++b) {
        k4u32x2 even, odd;
        value_operands<HD>(r.k[0], r.kp[0], b, even, odd);
        ((k4u32x2*)(to + (2 * NS + 2 * b) * 64))[tt] = even;
        ((k4u32x2*)(to + (2 * NS + 2 * b + 1) * 64))[tt] = odd;
      }
    }
  };
  if constexpr (WIDE) {
    request_part(0);
    convert_part(0);
    request_part(1);
  } else {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      request_keys(raw[d], d);
      request_values(raw[d], d);
    }
  }
  auto step = [&](Raw& r, int i) {
    const int tok0 = first + i * STEP;
    const k4u32x4* op = ops + (i & 1) * OPS + lane;
    if constexpr (WIDE) {
      __syncthreads();  // step i's operands are there, and those of step i - 1 have been read
      convert_part(i + 1);
      request_part(i + 2);
      if (tok0 >= wave_hi) return;
    }
    const bool masked = tok0 + 32 > lo;  // (of the wave) some row does not see all 32 tokens
    bf16x8 ph[TILES], pl[TILES];
    f32x4 score[TILES][2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const float power = WIDE ? 0.f : __uint_as_float(r.kp[tt] << 23);
#pragma unroll
      for (int t = 0; t < TILES; ++t) score[t][tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        bf16x8 k;
        if constexpr (WIDE) k = __builtin_bit_cast(bf16x8, op[(tt * NS + st) * 64]);
        else k = key_operand(r.k[tt][st], power);
#pragma unroll
        for (int m = NP - 1; m >= 0; --m)
#pragma unroll
          for (int t = 0; t < TILES; ++t) score[t][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, query(t, m, st), score[t][tt], 0, 0, 0);
      }
    }
    settle(score);
    if constexpr (!WIDE) request_keys(r, i + DEPTH);
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      const f32x4 s0 = score[t][0], s1 = score[t][1];
      float sc[8] = {s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]};
      if (masked) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (tok0 + (i >> 2) * 16 + g * 4 + (i & 3) >= lim[t]) sc[i] = -INFINITY;
      }
      float top = max3(max3(sc[0], sc[1], sc[2]), max3(sc[3], sc[4], sc[5]), max3(sc[6], sc[7], sc[7]));
      if (__ballot(top > moves[t]) != 0) {
        const float m_old = moves[t] == -INFINITY ? -INFINITY : -neg_m[t];
        const float m_new = fmaxf(m_old, fold_groups(top, LaneMax{}) * c1);
        const float alpha = m_new == m_old ? 1.f : __builtin_amdgcn_exp2f(m_old - m_new);
        if (m_new != -INFINITY) {
          neg_m[t] = -m_new;
          moves[t] = (m_new + 8.f) * (1.f / c1);
        }
        l_run[t] *= alpha;
#pragma unroll
        for (int j = 0; j < HT; ++j) acc[t][j] *= alpha;
      }
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], c1, neg_m[t]));
      l_run[t] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      unsigned h[4], l[4];
      split_weights(p, h, l);
      ph[t] = __builtin_bit_cast(bf16x8, k4u32x4{h[0], h[1], h[2], h[3]});
      pl[t] = __builtin_bit_cast(bf16x8, k4u32x4{l[0], l[1], l[2], l[3]});
    }
    if (!WIDE && masked) {
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) drop_values<HD>(r.v[tt], r.vp[tt], len - (tok0 + tt * 16 + g * 4));
    }
#pragma unroll
    for (int b = 0; b < HT / 2; ++b) {
      bf16x8 even, odd;
      if constexpr (WIDE) {
        even = __builtin_bit_cast(bf16x8, op[(2 * NS + 2 * b) * 64]);
        odd = __builtin_bit_cast(bf16x8, op[(2 * NS + 2 * b + 1) * 64]);
      } else {
        k4u32x2 even2[2], odd2[2];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) value_operands<HD>(r.v[tt], r.vp[tt], b, even2[tt], odd2[tt]);
        even = both_blocks(even2);
        odd = both_blocks(odd2);
      }
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        acc[t][2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, ph[t], acc[t][2 * b], 0, 0, 0);
        acc[t][2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, ph[t], acc[t][2 * b + 1], 0, 0, 0);
        acc[t][2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, pl[t], acc[t][2 * b], 0, 0, 0);
        acc[t][2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, pl[t], acc[t][2 * b + 1], 0, 0, 0);
      }
    }
    settle(acc);
    if constexpr (!WIDE) request_values(r, i + DEPTH);
  };
  for (int i = 0; i < nsteps; i += DEPTH)
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
      if (i + d < nsteps) step(raw[d], i + d);
#pragma unroll
  for (int t = 0; t < TILES; ++t) l_run[t] = fold_groups(l_run[t], LaneAdd{});
  auto maximum = [&](int t) { return moves[t] == -INFINITY ? -INFINITY : -neg_m[t]; };

  // ---- what leaves the workgroup: rows, or a split's partial rows (written through) ----
  float* all = a.part + ((size_t)clients.part_off[it.ci] + ((size_t)kvh * groups + it.group) * nsplit * WG_TILES) * (16 * ROW);
  float* part = all + (size_t)it.split * WG_TILES * 16 * ROW;
  auto finish = [&](int rr, int e0, const f32x4& o, float m, float l) {  // 4 channels of a row
    const TileRow tr = tile_row(rr, group, group_rinv, n_rows, row_off, kvh);
    if (!tr.live) return;
    float inv = __builtin_amdgcn_rcpf(l);
    inv = l == 0.f ? 0.f : inv * (2.f - l * inv);
    const f32x4 y = o * inv;
    T* out = (T*)a.out + tr.row * a.out_stride + tr.head * HD + e0;
    if constexpr (sizeof(T) == 4) *(f32x4*)out = y;
    else *(uint2*)out = make_uint2(pack2_bf16(y[0], y[1]), pack2_bf16(y[2], y[3]));
    if (a.lse && e0 == 0) a.lse[(size_t)tr.row * a.n_q_heads + tr.head] = l == 0.f ? INFINITY : m + __builtin_amdgcn_logf(l);
  };
  if constexpr (WIDE) {
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      if ((tile0 + t) * 16 >= R) break;
      const float m = maximum(t);
      float* dst = part + ((size_t)(w * TILES + t) * 16 + c) * ROW;
      // lane (c, g): channels (4 g + i) * HT + j of row c
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < HT; j += 4) {
          const int ch = (4 * g + i) * HT + j;
          const f32x4 o = f32x4{acc[t][j][i], acc[t][j + 1][i], acc[t][j + 2][i], acc[t][j + 3][i]};
          if (nsplit == 1) finish((tile0 + t) * 16 + c, ch, o, m, l_run[t]);
          else if (wave_hi > first) Xwg<true>::st4f(dst + ch, o);  // (nothing seen: nothing to read)
        }
      if (nsplit > 1 && g == 0) Xwg<true>::st4f(dst + HD, f32x4{m, l_run[t], 0.f, 0.f});
    }
  } else {
    float(*states)[WAVES][16][ROW] = (float(*)[WAVES][16][ROW])lds;  // a row: its channels, its maximum and sum
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < HT; j += 4)
          *(f32x4*)&states[t][w][c][(4 * g + i) * HT + j] = f32x4{acc[t][j][i], acc[t][j + 1][i], acc[t][j + 2][i], acc[t][j + 3][i]};
      if (g == 0) *(f32x2*)&states[t][w][c][HD] = f32x2{maximum(t), l_run[t]};
    }
    __syncthreads();
    const int live = min(WG_TILES * 16, R - tile0 * 16) * (HD / 4);
#pragma unroll 1
    for (int k = tid; k < live; k += WAVES * 64) {  // (row, 4 channels)
      const int mr = k / (HD / 4), e0 = (k % (HD / 4)) * 4;
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
      if (nsplit == 1) {
        finish(tile0 * 16 + mr, e0, o, m, l);
      } else {
        float* dst = part + (size_t)mr * ROW;
        Xwg<true>::st4f(dst + e0, o);
        if (e0 == 0) Xwg<true>::st4f(dst + HD, f32x4{m, l, 0.f, 0.f});
      }
    }
  }
  if (nsplit == 1) return;

  // ---- count in; the last of the splits to arrive joins them ----
  Xwg<true>::drain();
  __syncthreads();
  if (tid == 0) {
    unsigned* counter = a.counters + clients.count_off[it.ci] + kvh * groups + it.group;
    const unsigned prev = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const int last = prev == (unsigned)nsplit - 1u;
    if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // ready for the next launch
    *last_lds = last;
  }
  __syncthreads();
  if (*last_lds == 0) return;
  const size_t split_stride = (size_t)WG_TILES * 16 * ROW;
  constexpr int TPR = HD / 4, NT = WAVES * 64;
  const int rows_here = min(WG_TILES * 16, R - it.group * WG_TILES * 16), tasks = rows_here * TPR;
  if constexpr (!WIDE) {
    // The maxima and sums of all (split, row) come to LDS at once; each thread then has 4 channels of a row, or of several
    // one after the other, and takes its splits 8 at a time.  Threads that the rows leave over share the splits of a row:
    // thread (share, row, 4 channels) takes splits share, share + shares, .., and the shares are joined through LDS in order.
    constexpr int BATCH = 8, ROWS = WG_TILES * 16;
    static_assert(2 * kKv4MaxSplits * ROWS + NT * 5 <= (int)state_floats<HD, TILES, WAVES, WIDE>(), "maxima, sums and shares fit the states' LDS");
    f32x2* stats = (f32x2*)lds;                           // [split][row]
    float* joined = lds + 2 * kKv4MaxSplits * ROWS;       // [share][row, 4 channels] 4 sums, the sum of weights
    for (int i = tid; i < nsplit * ROWS; i += NT)
      if (i % ROWS < rows_here) stats[i] = *(const f32x2*)(all + (size_t)i * ROW + HD);
    int log_tasks = 31 - __builtin_clz(TPR);  // (rows made a power of two)
    while ((1 << log_tasks) < tasks) ++log_tasks;
    const int shares = max(1, NT >> log_tasks);
    __syncthreads();
#pragma unroll 1
    for (int k0 = 0; k0 < tasks; k0 += NT) {
      const int k = k0 + (tid & ((1 << log_tasks) - 1)), share = tid >> log_tasks;
      const int mr = min(k / TPR, rows_here - 1), e0 = (k % TPR) * 4;
      const float* p0 = all + (size_t)mr * ROW + e0;
      float m = -INFINITY, l = 0.f;
#pragma unroll 4
      for (int sp = 0; sp < nsplit; ++sp) m = fmaxf(m, stats[sp * ROWS + mr].x);
      f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
      for (int s0 = share; s0 < nsplit; s0 += BATCH * shares) {
        f32x4 ob[BATCH];
#pragma unroll
        for (int j = 0; j < BATCH; ++j) ob[j] = *(const f32x4*)(p0 + min(s0 + j * shares, nsplit - 1) * split_stride);
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
          const int sp = s0 + j * shares;
          const f32x2 ml = stats[min(sp, nsplit - 1) * ROWS + mr];
          const float sw = sp < nsplit && ml.x != -INFINITY ? __builtin_amdgcn_exp2f(ml.x - m) : 0.f;
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
      if (share == 0 && k < tasks) finish(it.group * WG_TILES * 16 + mr, e0, o, m, l);
    }
  } else {
    constexpr int BATCH = 8;
    for (int k = tid; k < tasks; k += NT) {
      const int mr = k / TPR, e0 = (k % TPR) * 4;
      const float* p0 = all + (size_t)mr * ROW;
      float m = -INFINITY, l = 0.f;
      f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int s0 = 0; s0 < nsplit; s0 += BATCH) {
        f32x4 ob[BATCH];
        f32x2 ml[BATCH];
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
          const float* ps = p0 + min(s0 + j, nsplit - 1) * split_stride;
          ml[j] = *(const f32x2*)(ps + HD);
          ob[j] = *(const f32x4*)(ps + e0);
        }
        float m_new = m;
#pragma unroll
        for (int j = 0; j < BATCH; ++j)
          if (s0 + j < nsplit) m_new = fmaxf(m_new, ml[j].x);
        if (m_new == -INFINITY) continue;
        const float alpha = __builtin_amdgcn_exp2f(m - m_new);
        l *= alpha;
        o *= alpha;
        m = m_new;
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
          if (s0 + j >= nsplit || ml[j].x == -INFINITY) continue;  // (a split that saw nothing wrote no values)
          const float sw = __builtin_amdgcn_exp2f(ml[j].x - m);
          l += ml[j].y * sw;
          o += ob[j] * sw;
        }
      }
      finish(it.group * WG_TILES * 16 + mr, e0, o, m, l);
    }
  }
}

template <int HD, typename T, int TILES, int WAVES, bool WIDE>
static hipError_t attend_kernel(const Kv4AttendCall& c, const Kv4Clients& cl, hipStream_t st) {
  constexpr size_t lds = attend_lds_bytes<HD, T, TILES, WAVES, WIDE>();
  if constexpr (lds > 64 * 1024) {
    static std::atomic<uint64_t> allowed{0};
    const hipError_t e = allow_lds(allowed, (const void*)kv4_attend_kernel<HD, T, TILES, WAVES, WIDE>, lds);
    if (e != hipSuccess) return e;
  }
  if (cl.items > 65535) return hipErrorInvalidValue;  // (a client has at most 2048 * group / 16 * 64 of them, and 32 share a launch)
  kv4_attend_kernel<HD, T, TILES, WAVES, WIDE><<<dim3(c.view.n_kv_heads, cl.items), WAVES * 64, lds, st>>>(c, cl);
  return hipGetLastError();
}
template <int HD, typename T>
static hipError_t attend_of(const Kv4AttendCall& c, const Kv4Launch& l, hipStream_t st) {
  if (l.wide) return attend_kernel<HD, T, kv4_wide_tiles(sizeof(T) == 4 ? PIPESD_F32 : PIPESD_BF16, HD), kKv4WideWaves, true>(c, l.c, st);
  if (l.tiles == 1) return attend_kernel<HD, T, 1, kv4_few_waves(1), false>(c, l.c, st);
  if constexpr (sizeof(T) == 2)
    if (l.tiles == 2) return attend_kernel<HD, T, 2, kv4_few_waves(2), false>(c, l.c, st);
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
// tiles the four waves bring through LDS four at a time.  One writer per token, sums in a fixed order.
template <int HD, typename T, int TT>
__global__ __launch_bounds__(256) void kv4_mass_kernel(Kv4AttendCall a, Kv4Clients cl) {
  constexpr int NP = pieces<T>(), NS = HD / 32;
  typedef typename std::conditional<HD == 128, k4u32x4, k4u32x2>::type Codes;
  __shared__ k4u32x4 q_lds[4][NP * NS][64];
  __shared__ float lse_lds[4][16];
  __shared__ int lim_lds[4][16];
  const int kvh = blockIdx.x, ci = blockIdx.z, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int c = lane & 15, g = lane >> 4;
  const int len = cl.len[ci], n_rows = cl.n_rows[ci], row_off = cl.row_off[ci];
  const int tok0 = ((int)blockIdx.y * 4 + w) * TT * 16;
  if ((int)blockIdx.y * 4 * TT * 16 >= len) return;  // (whole workgroup)
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
      Queries<HD, NP> q;
      load_queries<HD, NP>((const T*)a.q + tr.row * a.q_stride + tr.head * HD, tr.live, g, q);
#pragma unroll
      for (int i = 0; i < NP * NS; ++i) q_lds[w][i][lane] = q.q[i / NS][i % NS];
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
#pragma unroll
      for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = __builtin_amdgcn_exp2f(fmaf(score[0][tt][i], c1, -lse));
          sum[tt][i] += tok0 + tt * 16 + g * 4 + i < lim ? p : 0.f;
        }
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
  auto go = [&](auto tt) {
    constexpr int TT = decltype(tt)::value;
    const dim3 grid(a.view.n_kv_heads, (most + 64 * TT - 1) / (64 * TT), cl.n);
    kv4_mass_kernel<HD, T, TT><<<grid, 256, 0, st>>>(a, cl);
  };
  if (most <= 32768) go(std::integral_constant<int, 2>{});
  else go(std::integral_constant<int, 4>{});
  return hipGetLastError();
}
hipError_t launch_kv4_mass(const Kv4AttendCall& c, const Kv4Clients& cl, hipStream_t st) {
  if (c.head_dim == 128) return c.dtype == PIPESD_F32 ? mass_of<128, float>(c, cl, st) : mass_of<128, uint16_t>(c, cl, st);
  return c.dtype == PIPESD_F32 ? mass_of<64, float>(c, cl, st) : mass_of<64, uint16_t>(c, cl, st);
}

}  // namespace pipesd
