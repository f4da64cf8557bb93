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

// the rows of a tile: lane's column
struct TileRow {
  int row, head;  // of the pass; of the model
  bool live;
};
__device__ __forceinline__ TileRow tile_row(int rr, int group, int n_rows, int row_off, int kvh) {
  const int r = rr / group;
  return TileRow{row_off + min(r, n_rows - 1), kvh * group + rr % group, r < n_rows};
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
// (a, b) = hi + lo, each a pair of bf16 numbers
__device__ __forceinline__ void split_weights(float a, float b, unsigned& hi, unsigned& lo) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  hi = pack2_bf16(a, b);
  const bf16x2 h = __builtin_bit_cast(bf16x2, hi);
  // a - the lower half, b - the upper half: exact.  (The factors -1 come in registers: as a constant of the instruction the
  // number sits in the other half than the compiler takes it to.)
  unsigned low = 0x0000bf80u, high = 0xbf800000u;
  asm("" : "+s"(low), "+s"(high));
  lo = pack2_bf16(__builtin_amdgcn_fdot2_f32_bf16(h, __builtin_bit_cast(bf16x2, low), a, false),
                  __builtin_amdgcn_fdot2_f32_bf16(h, __builtin_bit_cast(bf16x2, high), b, false));
}

// which client and split a workgroup is for
struct Kv4Item {
  int ci, group, split;
};
__device__ __forceinline__ Kv4Item find_item(const Kv4Clients& cl, int item, int lane) {
  int ci = 0;
  if (cl.n > 1) ci = __popcll(__ballot(lane < kKv4ClientsPerLaunch && item >= cl.first[lane & (kKv4ClientsPerLaunch - 1)] && lane < cl.n)) - 1;
  ci = __builtin_amdgcn_readfirstlane(ci);
  const int i = item - cl.first[ci], groups = cl.groups[ci];
  return Kv4Item{ci, i % groups, i / groups};
}

// A wave walks tokens 32 at a time.  Per tile of 16 query rows it keeps a running maximum, sum and O^T in registers; the maximum moves
// only when a score passes it by 2^8 (any scale will do for fp32 sums: most steps then need no exchange between lanes and
// no rescaling).
// LDS: where the waves share tiles their states to be joined; then the queries that registers do not hold; a word
template <int HD, int WAVES, bool WIDE>
constexpr size_t state_floats() { return WIDE ? 0 : (size_t)WAVES * 16 * (HD + kKv4PartPad) + 2 * WAVES * 16; }
template <typename T>
constexpr int pieces() { return sizeof(T) == 4 ? 3 : 1; }
template <int HD, typename T, int TILES>
constexpr bool queries_in_lds() { return TILES * pieces<T>() * (HD / 8) > 32; }
template <int HD, typename T, int TILES, int WAVES, bool WIDE>
constexpr size_t attend_lds_bytes() {
  return state_floats<HD, WAVES, WIDE>() * sizeof(float) +
         (queries_in_lds<HD, T, TILES>() ? (size_t)(WIDE ? WAVES : 1) * TILES * sizeof(Queries<HD, pieces<T>()>) * 64 : 0) + 16;
}

template <int HD, typename T, int TILES, int WAVES, bool WIDE>
__global__ __launch_bounds__(WAVES * 64, TILES == 1 ? 4 : 2) void kv4_attend_kernel(Kv4AttendCall a, Kv4Clients clients) {
  constexpr int NP = pieces<T>(), NS = HD / 32, HT = HD / 16, ROW = HD + kKv4PartPad;
  constexpr bool Q_LDS = queries_in_lds<HD, T, TILES>();
  constexpr int WG_TILES = WIDE ? WAVES * TILES : TILES;
  constexpr int STEP = WIDE ? 32 : WAVES * 32;
  typedef typename std::conditional<HD == 128, k4u32x4, k4u32x2>::type Codes;
  extern __shared__ float lds[];
  float(*o_lds)[16][ROW] = (float(*)[16][ROW])lds;
  float(*m_lds)[16] = (float(*)[16])(lds + (size_t)WAVES * 16 * ROW);
  float(*l_lds)[16] = m_lds + WAVES;
  int* last_lds = (int*)((char*)lds + attend_lds_bytes<HD, T, TILES, WAVES, WIDE>() - 16);

  const int kvh = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, g = lane >> 4;
  const Kv4Item it = find_item(clients, blockIdx.y, lane);
  const int len = clients.len[it.ci], n_rows = clients.n_rows[it.ci], row_off = clients.row_off[it.ci];
  const int groups = clients.groups[it.ci], nsplit = clients.nsplit[it.ci];
  const int group = a.n_q_heads / a.view.n_kv_heads;
  const int R = n_rows * group;
  const int tile0 = it.group * WG_TILES + (WIDE ? w * TILES : 0);
  const int span0 = it.split * clients.span;
  const int32_t* table = a.view.table + clients.table_off[it.ci];

  const int first = span0 + (WIDE ? 0 : w * 32);
  // the blocks of 64 steps sit in the lanes: lane L has the two of step L
  int step_blk[2];
  auto load_blocks = [&](int it0) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const int64_t tok = (int64_t)first + (int64_t)(it0 + lane) * STEP + tt * 16;
      step_blk[tt] = table[tok < len ? (int)(tok / kBlockTokens) : 0];
    }
  };
  load_blocks(0);

  // ---- queries, and how far each row sees ----
  // (in registers, or where the sums leave no room for them in LDS: [tile][piece][step][lane])
  Queries<HD, NP> q[Q_LDS ? 1 : TILES];
  k4u32x4* q_lds = (k4u32x4*)(lds + state_floats<HD, WAVES, WIDE>()) + (WIDE ? w * TILES * NP * NS * 64 : 0) + lane;
  int lim[TILES];
  int lo = len, hi = 0;
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const TileRow tr = tile_row((tile0 + t) * 16 + c, group, n_rows, row_off, kvh);
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
  Raw r;
  // (step i's: keys and values travel from where those of the step before have been used until they are)
  auto record = [&](int i, int tt) {
    return a.view.pool + kv4_record<HD>(a.view, a.layer, __builtin_amdgcn_readlane(step_blk[tt], i & 63), kvh);
  };
  auto request_keys = [&](int i) {
    if (i >= nsteps) return;
    if (i > 0 && (i & 63) == 0) load_blocks(i);
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const uint8_t* rec = record(i, tt);
      r.k[tt] = *(const Codes*)(rec + at.k);
      r.kp[tt] = rec[at.kp];
    }
  };
  auto request_values = [&](int i) {
    if (i >= nsteps) return;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const uint8_t* rec = record(i, tt);
      r.v[tt] = *(const Codes*)(rec + at.v);
      r.vp[tt] = *(const unsigned*)(rec + at.vp);
    }
  };
  request_keys(0);
  request_values(0);
  for (int i = 0; i < nsteps; ++i) {
    const int tok0 = first + i * STEP;
    const bool masked = tok0 + 32 > lo;  // (of the wave) some row does not see all 32 tokens
    bf16x8 ph[TILES], pl[TILES];
    f32x4 score[TILES][2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const float power = __uint_as_float(r.kp[tt] << 23);
#pragma unroll
      for (int t = 0; t < TILES; ++t) score[t][tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        const bf16x8 k = key_operand(r.k[tt][st], power);
#pragma unroll
        for (int m = NP - 1; m >= 0; --m)
#pragma unroll
          for (int t = 0; t < TILES; ++t) score[t][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, query(t, m, st), score[t][tt], 0, 0, 0);
      }
    }
    settle(score);
    request_keys(i + 1);
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
#pragma unroll
      for (int i = 0; i < 4; ++i) split_weights(p[2 * i], p[2 * i + 1], h[i], l[i]);
      ph[t] = __builtin_bit_cast(bf16x8, k4u32x4{h[0], h[1], h[2], h[3]});
      pl[t] = __builtin_bit_cast(bf16x8, k4u32x4{l[0], l[1], l[2], l[3]});
    }
    if (masked) {  // what lies behind the last token may be anything: its weights are 0, its values must be numbers
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const int n = min(4, max(0, len - (tok0 + tt * 16 + g * 4)));  // of this lane's four tokens
        const unsigned long long keep = n >= 4 ? ~0ull : (1ull << (16 * n)) - 1ull;
        if constexpr (HD == 128) {
          r.v[tt].x = n > 0 ? r.v[tt].x : 0u;
          r.v[tt].y = n > 1 ? r.v[tt].y : 0u;
          r.v[tt].z = n > 2 ? r.v[tt].z : 0u;
          r.v[tt].w = n > 3 ? r.v[tt].w : 0u;
        } else {
          r.v[tt].x &= (unsigned)keep;
          r.v[tt].y &= (unsigned)(keep >> 32);
        }
        const unsigned km = n >= 4 ? ~0u : (1u << (8 * n)) - 1u;
        r.vp[tt] = (r.vp[tt] & km) | (0x7f7f7f7fu & ~km);
      }
    }
    // two neighbouring channels at a time: bf16 pairs (channel, channel + 1) of each token, regrouped to pairs of tokens
#pragma unroll
    for (int b = 0; b < HT / 2; ++b) {
      unsigned x[2][4];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const float p0 = __uint_as_float(r.vp[tt] << 23), p1 = __uint_as_float(r.vp[tt] << 15),
                    p2 = __uint_as_float(r.vp[tt] << 7), p3 = __uint_as_float(r.vp[tt] >> 1);  // (only the exponent's bits count)
        auto cvt = [&](unsigned w, float pw, auto byte) {
          return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, pw, decltype(byte)::value));
        };
        auto at_byte = [&](auto byte) {
          if constexpr (HD == 128) {
            x[tt][0] = cvt(r.v[tt].x, p0, byte);
            x[tt][1] = cvt(r.v[tt].y, p1, byte);
            x[tt][2] = cvt(r.v[tt].z, p2, byte);
            x[tt][3] = cvt(r.v[tt].w, p3, byte);
          } else {
            typedef std::integral_constant<int, decltype(byte)::value + 2> upper;
            x[tt][0] = cvt(r.v[tt].x, p0, byte);
            x[tt][1] = cvt(r.v[tt].x, p1, upper{});
            x[tt][2] = cvt(r.v[tt].y, p2, byte);
            x[tt][3] = cvt(r.v[tt].y, p3, upper{});
          }
        };
        if (b == 0) at_byte(std::integral_constant<int, 0>{});
        if (b == 1) at_byte(std::integral_constant<int, 1>{});
        if constexpr (HD == 128) {
          if (b == 2) at_byte(std::integral_constant<int, 2>{});
          if (b == 3) at_byte(std::integral_constant<int, 3>{});
        }
      }
      auto tokens = [&](unsigned halves) {
        return __builtin_bit_cast(bf16x8, k4u32x4{__builtin_amdgcn_perm(x[0][1], x[0][0], halves), __builtin_amdgcn_perm(x[0][3], x[0][2], halves),
                                                  __builtin_amdgcn_perm(x[1][1], x[1][0], halves), __builtin_amdgcn_perm(x[1][3], x[1][2], halves)});
      };
      const bf16x8 even = tokens(0x05040100u), odd = tokens(0x07060302u);
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        acc[t][2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, ph[t], acc[t][2 * b], 0, 0, 0);
        acc[t][2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, ph[t], acc[t][2 * b + 1], 0, 0, 0);
        acc[t][2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, pl[t], acc[t][2 * b], 0, 0, 0);
        acc[t][2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, pl[t], acc[t][2 * b + 1], 0, 0, 0);
      }
    }
    settle(acc);
    request_values(i + 1);
  }
#pragma unroll
  for (int t = 0; t < TILES; ++t) l_run[t] = fold_groups(l_run[t], LaneAdd{});
  auto maximum = [&](int t) { return moves[t] == -INFINITY ? -INFINITY : -neg_m[t]; };

  // ---- what leaves the workgroup: rows, or a split's partial rows (written through) ----
  float* all = a.part + ((size_t)clients.part_off[it.ci] + ((size_t)kvh * groups + it.group) * nsplit * WG_TILES) * (16 * ROW);
  float* part = all + (size_t)it.split * WG_TILES * 16 * ROW;
  auto finish = [&](int rr, int e0, const f32x4& o, float m, float l) {  // 4 channels of a row
    const TileRow tr = tile_row(rr, group, n_rows, row_off, kvh);
    if (!tr.live) return;
    const f32x4 y = l == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o / l;
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
          else if (nsteps > 0) Xwg<true>::st4f(dst + ch, o);
        }
      if (nsplit > 1 && g == 0) Xwg<true>::st4f(dst + HD, f32x4{m, l_run[t], 0.f, 0.f});
    }
  } else {
    // thread -> (row, 4 channels); a workgroup of more than 16 * HD / 4 threads leaves some idle, one of fewer goes round
    constexpr int TPR = HD / 4, TASKS = 16 * TPR;
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      if ((tile0 + t) * 16 >= R) break;
      if (t > 0) __syncthreads();  // the tile before has been read
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < HT; j += 4)
          *(f32x4*)&o_lds[w][c][(4 * g + i) * HT + j] = f32x4{acc[t][j][i], acc[t][j + 1][i], acc[t][j + 2][i], acc[t][j + 3][i]};
      if (g == 0) {
        m_lds[w][c] = maximum(t);
        l_lds[w][c] = l_run[t];
      }
      __syncthreads();
      const int live = min(16, R - (tile0 + t) * 16) * TPR;
#pragma unroll
      for (int k0 = 0; k0 < TASKS; k0 += WAVES * 64) {
        const int k = k0 + tid, mr = k / TPR, e0 = (k % TPR) * 4;
        if (k >= live) continue;
        float m = m_lds[0][mr];
#pragma unroll
        for (int ww = 1; ww < WAVES; ++ww) m = fmaxf(m, m_lds[ww][mr]);
        const float m_ref = m == -INFINITY ? 0.f : m;
        float l = 0.f;
        f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ww = 0; ww < WAVES; ++ww) {
          const float sw = __builtin_amdgcn_exp2f(m_lds[ww][mr] - m_ref);
          l += l_lds[ww][mr] * sw;
          o += *(const f32x4*)&o_lds[ww][mr][e0] * sw;
        }
        if (nsplit == 1) {
          finish((tile0 + t) * 16 + mr, e0, o, m, l);
        } else {
          float* dst = part + ((size_t)t * 16 + mr) * ROW;
          Xwg<true>::st4f(dst + e0, o);
          if (e0 == 0) Xwg<true>::st4f(dst + HD, f32x4{m, l, 0.f, 0.f});
        }
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
  // Threads that the rows leave over divide the splits among them: thread (share, row, 4 channels) takes splits share,
  // share + shares, ..; the shares of a row and channels are joined through LDS in order.
  constexpr int TPR = HD / 4, NT = WAVES * 64, BATCH = 8;
  static_assert(WIDE || NT * 6 * sizeof(float) <= state_floats<HD, WAVES, WIDE>() * sizeof(float), "the shares fit the states' LDS");
  const size_t split_stride = (size_t)WG_TILES * 16 * ROW;
  const int rows_here = min(WG_TILES * 16, R - it.group * WG_TILES * 16), tasks = rows_here * TPR;
  const int shares = WIDE || tasks >= NT ? 1 : min(NT / tasks, nsplit);
  for (int k0 = 0; k0 < tasks; k0 += NT) {
    const int k = shares > 1 ? tid % tasks : k0 + tid, share = shares > 1 ? tid / tasks : 0;
    const int mr = k / TPR, e0 = (k % TPR) * 4;
    const bool on = k < tasks && share < shares;
    const float* p0 = all + (size_t)(on ? mr : 0) * ROW;
    float m = -INFINITY, l = 0.f;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s0 = share; on && s0 < nsplit; s0 += BATCH * shares) {
      f32x4 ob[BATCH];
      f32x2 ml[BATCH];
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        const float* ps = p0 + min(s0 + j * shares, nsplit - 1) * split_stride;
        ml[j] = *(const f32x2*)(ps + HD);
        ob[j] = *(const f32x4*)(ps + e0);
      }
      float m_new = m;
#pragma unroll
      for (int j = 0; j < BATCH; ++j)
        if (s0 + j * shares < nsplit) m_new = fmaxf(m_new, ml[j].x);
      if (m_new == -INFINITY) continue;
      const float alpha = __builtin_amdgcn_exp2f(m - m_new);
      l *= alpha;
      o *= alpha;
      m = m_new;
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        if (s0 + j * shares >= nsplit || ml[j].x == -INFINITY) continue;  // (a split that saw nothing wrote no values)
        const float sw = __builtin_amdgcn_exp2f(ml[j].x - m);
        l += ml[j].y * sw;
        o += ob[j] * sw;
      }
    }
    if (shares > 1) {
      float* x = lds + (size_t)tid * 6;
      x[0] = o[0], x[1] = o[1], x[2] = o[2], x[3] = o[3], x[4] = m, x[5] = l;
      __syncthreads();
      if (share == 0) {
        for (int sh = 1; sh < shares; ++sh) {
          const float* y = lds + (size_t)(sh * tasks + k) * 6;
          const float m_new = fmaxf(m, y[4]);
          if (m_new == -INFINITY) continue;
          const float sa = __builtin_amdgcn_exp2f(m - m_new), sb = y[4] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(y[4] - m_new);
          l = l * sa + y[5] * sb;
          o = o * sa + f32x4{y[0], y[1], y[2], y[3]} * sb;
          m = m_new;
        }
        finish(it.group * WG_TILES * 16 + mr, e0, o, m, l);
      }
    } else if (on) {
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
  if (l.wide) return attend_kernel<HD, T, sizeof(T) == 4 ? kKv4WideTilesF32 : kKv4WideTilesBf16, kKv4WideWaves, true>(c, l.c, st);
  if (l.tiles == 1) return attend_kernel<HD, T, 1, 8, false>(c, l.c, st);
  return attend_kernel<HD, T, 2, 4, false>(c, l.c, st);
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
  const int group = a.n_q_heads / a.view.n_kv_heads;
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
      const TileRow tr = tile_row((q0 + w) * 16 + c, group, n_rows, row_off, kvh);
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
