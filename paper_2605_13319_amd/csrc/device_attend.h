// What the attention kernels over caches of operators share: the running softmax of a tile of query rows, its weights as operands,
// the wait states of sums.
#pragma once

#include "device_gemm.h"

namespace pipesd {

typedef __attribute__((ext_vector_type(4))) unsigned k4u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned k4u32x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(16))) float f32x16;

template <int HD>
__device__ __forceinline__ float attend_scale() { return (HD == 128 ? 0.08838834764831845f : 0.125f) * 1.44269504088896341f; }  // log2(e) / sqrt(HD)

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

// n / m for 0 <= n < 2^20, 1 <= m, rinv = 1 / m to within an ulp: (n + 0.5) / m is at least 0.5 / m from an integer, more than
// the roundings' 2^-22 (n + 0.5) / m.  (An integer division is 30 instructions, and code is what a short call waits for.)
__host__ __device__ __forceinline__ int div_by(int n, float rinv) { return (int)(((float)n + 0.5f) * rinv); }

// The rows of a tile: lane's column.  Columns behind the last row are that row once more: the workgroup's own, where the last heads of a row may
// be another's, which may have written its results over the queries.
struct TileRow {
  int row, head;  // of the pass; of the model
  bool live;
};
__host__ __device__ __forceinline__ TileRow tile_row(int rr, int group, float group_rinv, int n_rows, int row_off, int kvh) {
  const int last = n_rows * group - 1, at = rr < last ? rr : last, r = div_by(at, group_rinv);
  return TileRow{row_off + r, kvh * group + at - r * group, rr <= last};
}
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
  __device__ __forceinline__ bool no_number() const {
    bool none = false;
#pragma unroll
    for (int j = 0; j < HT; ++j)
#pragma unroll
      for (int e = 0; e < 4; e += 2) none |= __builtin_isunordered(acc[j][e], acc[j][e + 1]);
    return none;
  }
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

}  // namespace pipesd
