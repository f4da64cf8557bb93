// The 4-bit cache: block tables, rounding rows into it, reading them back, and cutting a client to a budget.
#include "kv4.h"

namespace pipesd {

__global__ __launch_bounds__(256) void kv4_table_kernel(Kv4TableUpdate u, int32_t* table) {
  if ((int)threadIdx.x < u.n) table[u.at[threadIdx.x]] = u.v[threadIdx.x];
}
static_assert(kKv4EntriesPerLaunch <= 256, "a thread an entry");
hipError_t launch_kv4_table(const Kv4TableUpdate& u, int32_t* table, hipStream_t st) {
  kv4_table_kernel<<<1, 256, 0, st>>>(u, table);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------
// numbers to codes and back
// ------------------------------------------------------------------------------------------------
// 16 lanes share a (token, head): lane r has its unit of HD / 16 neighbouring channels, 512 / HD lanes a power.
template <int HD, typename T>
__device__ __forceinline__ void load_unit(const T* p, float (&x)[HD / 16]) {
  constexpr int N = HD / 16;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 v = *(const float4*)(p + i);
      x[i] = v.x, x[i + 1] = v.y, x[i + 2] = v.z, x[i + 3] = v.w;
    }
  } else {
    uint32_t w[N / 2];
    if constexpr (N == 8) {
      const uint4 v = *(const uint4*)p;
      w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else {
      const uint2 v = *(const uint2*)p;
      w[0] = v.x, w[1] = v.y;
    }
#pragma unroll
    for (int i = 0; i < N / 2; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// The unit's codes, and its power's byte.  The power is the smallest 2^e with max|x| <= 7 * 2^e, e in [-125, 125]: of the
// 32 values only those above 6 * 2^e are cut, by at most a seventh.  That has the least error on normal numbers (rms
// 0.1119 of theirs; 0.1155 where nothing may be cut, 0.1149 where up to 8 * 2^e is).  The format holds finite values only:
// infinities are taken as the largest float, NaN as 0.
template <int HD>
__device__ __forceinline__ uint32_t encode_unit(float (&x)[HD / 16], uint32_t& power) {
  constexpr int N = HD / 16;
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float lim = fminf(fmaxf(x[i], -3.4028234663852886e38f), 3.4028234663852886e38f);
    x[i] = x[i] != x[i] ? 0.f : lim;
    top = fmaxf(top, fabsf(x[i]));
  }
#pragma unroll
  for (int m = 1; m < 512 / HD; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
  // top = 1.f * 2^E: 7 * 2^e = 1.75 * 2^(e + 2) holds it for e = E - 2 up to f = .75, for E - 1 beyond
  const uint32_t bits = __float_as_uint(top);
  const int e = (int)(bits >> 23) - 129 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  power = (uint32_t)(min(max(e, -125), 125) + 127);
  const float scale = __uint_as_float(power << 23);
  uint32_t codes = 0;  // (the conversion: to nearest, ties to the even code, cut at 6)
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], scale, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], scale, 1);
  if constexpr (N == 8) {
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], scale, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], scale, 3);
  }
  return codes;
}

template <int HD>
__device__ __forceinline__ void decode_unit(uint32_t codes, uint32_t power, uint32_t (&w)[HD / 32]) {  // bf16 pairs: exact
  const float scale = __uint_as_float(power << 23);
  w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  if constexpr (HD == 128) {
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  }
}

// where unit r of a token (its place in the block) is, keys and values, and its power
template <int HD>
__device__ __forceinline__ int key_unit(int tok, int r) { return Kv4Record<HD>::kKeys + (tok * 16 + r) * Kv4Record<HD>::kUnit; }
template <int HD>
__device__ __forceinline__ int value_unit(int tok, int r) {
  return Kv4Record<HD>::kValues + (((tok >> 2) * 16 + r) * 4 + (tok & 3)) * Kv4Record<HD>::kUnit;
}
template <int HD>
__device__ __forceinline__ int key_power(int tok, int b) { return Kv4Record<HD>::kKeyPow + tok * Kv4Record<HD>::kUnit + b; }
template <int HD>
__device__ __forceinline__ int value_power(int tok, int b) {
  return Kv4Record<HD>::kValPow + ((tok >> 2) * Kv4Record<HD>::kUnit + b) * 4 + (tok & 3);
}
template <int HD>
using unit_t = typename std::conditional<HD == 128, uint32_t, uint16_t>::type;

// ------------------------------------------------------------------------------------------------
// store: a wave takes 4 neighbouring rows of a head, 16 lanes each, which find a power with two exchanges between lanes and write a
// unit of codes.  Bound by memory where rows are many (2048 rows of 40 heads of 128: 14.5 us, 3.7 TB/s read and written; of 8
// heads 5.4 us), by the launch where they are few (16 clients' new rows 3.3 us).
// ------------------------------------------------------------------------------------------------
template <int HD, typename T>
__global__ __launch_bounds__(256) void kv4_store_kernel(Kv4View v, int layer, Kv4Ranges rg, const T* k, const T* val, int64_t k_stride,
                                                        int64_t v_stride) {
  constexpr int N = HD / 16;
  const int lane = threadIdx.x & 63, r = lane & 15;
  const int kvh = blockIdx.x, c = blockIdx.z, i = (blockIdx.y * 4 + (threadIdx.x >> 6)) * 4 + (lane >> 4);
  if (i >= rg.count[c]) return;  // (whole groups of 16 lanes)
  const int64_t row = rg.row_off[c] + i;
  const int pos = rg.first[c] + i, tok = pos % kBlockTokens;
  float x[N], y[N];
  load_unit<HD>(k + row * k_stride + kvh * HD + r * N, x);
  load_unit<HD>(val + row * v_stride + kvh * HD + r * N, y);
  const int blk = v.table[rg.table_off[c] + pos / kBlockTokens];
  uint8_t* rec = v.pool + kv4_record<HD>(v, layer, blk, kvh);
  uint32_t kp, vp;
  const uint32_t kc = encode_unit<HD>(x, kp), vc = encode_unit<HD>(y, vp);
  *(unit_t<HD>*)(rec + key_unit<HD>(tok, r)) = (unit_t<HD>)kc;
  *(unit_t<HD>*)(rec + value_unit<HD>(tok, r)) = (unit_t<HD>)vc;
  if (r % (512 / HD) == 0) {
    rec[key_power<HD>(tok, r / (512 / HD))] = (uint8_t)kp;
    rec[value_power<HD>(tok, r / (512 / HD))] = (uint8_t)vp;
  }
}

template <class F>
static void by_type(int dtype, int head_dim, F go) {
  typedef std::integral_constant<int, 64> H64;
  typedef std::integral_constant<int, 128> H128;
  if (head_dim == 128) {
    if (dtype == PIPESD_F32) go(H128{}, float{}); else go(H128{}, uint16_t{});
  } else {
    if (dtype == PIPESD_F32) go(H64{}, float{}); else go(H64{}, uint16_t{});
  }
}

// (a grid has at most 65535 workgroups in y: rows by the piece)
static Kv4Ranges part_of(const Kv4Ranges& r, int i0, int n) {
  Kv4Ranges p = r;
  p.most = std::min(r.most - i0, n);
  for (int c = 0; c < r.n; ++c) {
    p.first[c] += i0;
    p.row_off[c] += i0;
    p.count[c] = std::max(0, std::min(r.count[c] - i0, n));
  }
  return p;
}

hipError_t launch_kv4_store(int dtype, int head_dim, const Kv4View& v, int layer, const Kv4Ranges& r, const void* k, const void* val,
                            int64_t k_stride, int64_t v_stride, hipStream_t st) {
  constexpr int kMost = 65535 * 16;
  for (int i0 = 0; i0 < r.most; i0 += kMost) {
    const Kv4Ranges p = part_of(r, i0, kMost);
    by_type(dtype, head_dim, [&](auto hd, auto t) {
      typedef decltype(t) T;
      kv4_store_kernel<decltype(hd)::value, T><<<dim3(v.n_kv_heads, (p.most + 15) / 16, p.n), 256, 0, st>>>(v, layer, p, (const T*)k, (const T*)val,
                                                                                                       k_stride, v_stride);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ------------------------------------------------------------------------------------------------
// read: the same division of the lanes.  Bound by what it writes: 2048 tokens of 8 heads of 128 in 32 layers 61 us, 5.6 TB/s.
// ------------------------------------------------------------------------------------------------
template <int HD, typename T>
__device__ __forceinline__ void store_unit(T* p, const uint32_t (&w)[HD / 32]) {
  if constexpr (sizeof(T) == 2) {
    if constexpr (HD == 128) *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
    else *(uint2*)p = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int i = 0; i < HD / 32; i += 2)
      *(float4*)(p + 2 * i) = make_float4(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u),
                                          __uint_as_float(w[i + 1] << 16), __uint_as_float(w[i + 1] & 0xffff0000u));
  }
}

template <int HD, typename T>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4View v, int layer0, Kv4Ranges rg, int64_t total_rows, T* k,
                                                       T* val) {
  constexpr int N = HD / 16;
  const int lane = threadIdx.x & 63, r = lane & 15, wave = threadIdx.x >> 6;
  const int c = blockIdx.z, layer = blockIdx.y / v.n_kv_heads, kvh = blockIdx.y % v.n_kv_heads;
  const int i = (blockIdx.x * 4 + wave) * 4 + (lane >> 4);
  if (i >= rg.count[c]) return;
  const int pos = rg.first[c] + i, tok = pos % kBlockTokens;
  const int blk = v.table[rg.table_off[c] + pos / kBlockTokens];
  const uint8_t* rec = v.pool + kv4_record<HD>(v, layer0 + layer, blk, kvh);
  const uint32_t kc = *(const unit_t<HD>*)(rec + key_unit<HD>(tok, r)), vc = *(const unit_t<HD>*)(rec + value_unit<HD>(tok, r));
  const uint32_t kp = rec[key_power<HD>(tok, r / (512 / HD))], vp = rec[value_power<HD>(tok, r / (512 / HD))];
  uint32_t w[HD / 32], x[HD / 32];
  decode_unit<HD>(kc, kp, w);
  decode_unit<HD>(vc, vp, x);
  const int64_t at = (((int64_t)layer * total_rows + rg.row_off[c] + i) * v.n_kv_heads + kvh) * HD + r * N;
  store_unit<HD>(k + at, w);
  store_unit<HD>(val + at, x);
}

hipError_t launch_kv4_read(int dtype, int head_dim, const Kv4View& v, int layer0, int n_layers, const Kv4Ranges& r, int64_t total_rows,
                           void* k, void* val, hipStream_t st) {
  // (a grid has at most 65535 workgroups in y: layers by the piece)
  const int per = std::max(1, 65535 / v.n_kv_heads);
  for (int l0 = 0; l0 < n_layers; l0 += per) {
    const int nl = std::min(per, n_layers - l0);
    const dim3 grid((r.most + 15) / 16, nl * v.n_kv_heads, r.n);
    by_type(dtype, head_dim, [&](auto hd, auto t) {
      typedef decltype(t) T;
      const int64_t off = (int64_t)l0 * total_rows * v.n_kv_heads * head_dim;
      kv4_read_kernel<decltype(hd)::value, T><<<grid, 256, 0, st>>>(v, layer0 + l0, r, total_rows, (T*)k + off, (T*)val + off);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ------------------------------------------------------------------------------------------------
// evict: which tokens stay
// ------------------------------------------------------------------------------------------------
// Workgroup (cache head, layer, client).  Of the tokens before the newest `recent` the keep - recent heaviest stay, the
// lower index first among equals: the weights as integers in their order, the (keep - recent)-th largest found 8 bits at
// a time from the counts of each value of the 8 bits, then one walk in order that numbers the tokens that stay.  Bound by the
// turns: four of counting and one for each 4096 tokens of the walk.  8192 tokens of 256 (layer, head) pairs 14 us; 18 with the
// weights read again for each digit.
constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64, kSelPer = 4, kSelHold = 8;

// order of floats as an order of integers; NaN counts as 0, as does -0
__device__ __forceinline__ uint32_t weight_key(float x) {
  x = x != x ? 0.f : x + 0.f;
  const uint32_t b = __float_as_uint(x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__global__ __launch_bounds__(kSelThreads) void kv4_select_kernel(Kv4Cuts c, int n_layers, int n_kv_heads, float* mass,
                                                                 int64_t mass_stride, int32_t* kept) {
  __shared__ uint32_t count[256];
  __shared__ uint32_t found[2];  // the digit; how many of the larger ones it left to take
  __shared__ uint32_t wave_eq[kSelWaves], wave_keep[kSelWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int kvh = blockIdx.x, layer = blockIdx.y, ci = blockIdx.z;
  const int64_t row = ((int64_t)layer * n_kv_heads + kvh) * mass_stride;
  const int64_t per_seq = (int64_t)n_layers * n_kv_heads * mass_stride;
  const float* src = mass + c.seq[ci] * per_seq + row;
  float* dst = mass + c.into[ci] * per_seq + row;
  int32_t* out = kept + (((int64_t)ci * n_layers + layer) * n_kv_heads + kvh) * c.keep;
  const int len = c.len[ci], old = len - c.recent, want = c.keep - c.recent;

  // threshold: keys above it stay, and the first `ties` of those equal to it
  uint32_t prefix = 0, mask = 0, left = (uint32_t)want;
  if (want > 0 && want < old) {
    // (the first kSelHold a thread stay in registers; what is behind comes again for every digit, as many requested at once)
    float held[kSelHold];
    auto load = [&](int t0, float (&x)[kSelHold]) {
#pragma unroll
      for (int i = 0; i < kSelHold; ++i) {
        const int t = t0 + i * kSelThreads + tid;
        x[i] = src[min(t, old - 1)];
      }
    };
    auto add = [&](int t0, const float (&x)[kSelHold], int shift) {
#pragma unroll
      for (int i = 0; i < kSelHold; ++i) {
        if (t0 + i * kSelThreads >= old) break;
        const uint32_t key = weight_key(x[i]);
        if (t0 + i * kSelThreads + tid < old && (key & mask) == prefix) atomicAdd(&count[(key >> shift) & 255u], 1u);
      }
    };
    load(0, held);
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) count[tid] = 0;
      __syncthreads();
      add(0, held, shift);
      for (int t0 = kSelHold * kSelThreads; t0 < old; t0 += kSelHold * kSelThreads) {
        float x[kSelHold];
        load(t0, x);
        add(t0, x, shift);
      }
      __syncthreads();
      if (tid < 64) {  // lane l: digits 255 - 4 l down to 252 - 4 l
        uint32_t n[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += n[i] = count[255 - 4 * lane - i];
        uint32_t before = (uint32_t)scan_wave(sum) - sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (before < left && left <= before + n[i]) {
            found[0] = (uint32_t)(255 - 4 * lane - i);
            found[1] = left - before;
          }
          before += n[i];
        }
      }
      __syncthreads();
      prefix |= found[0] << shift;
      mask |= 255u << shift;
      left = found[1];
    }
  }
  const bool all = want >= old, none = want <= 0;

  // in order; a thread has kSelPer neighbours
  uint32_t base_keep = 0, base_eq = 0;
  for (int t0 = 0; t0 < len; t0 += kSelThreads * kSelPer) {
    float x[kSelPer];
    uint32_t eq = 0, gt = 0;  // bit i: token i is equal to the threshold / stays anyway
#pragma unroll
    for (int i = 0; i < kSelPer; ++i) {
      const int t = t0 + tid * kSelPer + i;
      x[i] = t < len ? src[t] : 0.f;
      const uint32_t key = weight_key(x[i]);
      if (t < len && (t >= old || all || (!none && key > prefix))) gt |= 1u << i;
      else if (t < old && !none && key == prefix) eq |= 1u << i;
    }
    // equal ones before this thread
    const uint32_t n_eq = __popc(eq);
    const uint32_t in_eq = (uint32_t)scan_wave(n_eq);
    if (lane == 63) wave_eq[wave] = in_eq;
    __syncthreads();  // (also: all of this chunk has been read)
    uint32_t eq_before = base_eq + in_eq - n_eq, eq_all = base_eq;
    for (int w = 0; w < kSelWaves; ++w) {
      if (w < wave) eq_before += wave_eq[w];
      eq_all += wave_eq[w];
    }
    uint32_t stay = gt;
#pragma unroll
    for (int i = 0; i < kSelPer; ++i)
      if (eq >> i & 1u) {
        if (eq_before < left) stay |= 1u << i;
        ++eq_before;
      }
    const uint32_t n_stay = __popc(stay);
    const uint32_t in_stay = (uint32_t)scan_wave(n_stay);
    if (lane == 63) wave_keep[wave] = in_stay;
    __syncthreads();
    uint32_t at = base_keep + in_stay - n_stay, keep_all = base_keep;
    for (int w = 0; w < kSelWaves; ++w) {
      if (w < wave) at += wave_keep[w];
      keep_all += wave_keep[w];
    }
#pragma unroll
    for (int i = 0; i < kSelPer; ++i)
      if (stay >> i & 1u) {  // (into the client's own weights: at or before the place it was read from)
        out[at] = t0 + tid * kSelPer + i;
        dst[at] = x[i];
        ++at;
      }
    base_eq = eq_all;
    base_keep = keep_all;
  }
}

hipError_t launch_kv4_select(const Kv4View& v, const Kv4Cuts& c, float* mass, int64_t mass_stride, int32_t* kept, hipStream_t st) {
  kv4_select_kernel<<<dim3(v.n_kv_heads, v.n_layers, c.n), kSelThreads, 0, st>>>(c, v.n_layers, v.n_kv_heads, mass, mass_stride, kept);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------
// evict: their bytes to the new blocks.  A wave fills one record.  Bound by what it reads beside the kept tokens: values of four
// neighbouring tokens share their lines.  2048 of 8192 tokens of 8 heads of 128 in 32 layers: 68 us for 71 MB kept, about 170 MB
// read and 71 written.
// ------------------------------------------------------------------------------------------------
template <int HD>
__global__ __launch_bounds__(256) void kv4_move_kernel(Kv4View v, Kv4Cuts c, const int32_t* kept, int first) {
  constexpr int U = Kv4Record<HD>::kUnit;
  const int lane = threadIdx.x & 63;
  const int kvh = blockIdx.x % v.n_kv_heads, layer = blockIdx.x / v.n_kv_heads, ci = blockIdx.z;
  const int b = (first + (int)blockIdx.y) * 4 + (int)(threadIdx.x >> 6);
  if (b * kBlockTokens >= c.keep) return;
  const int32_t* idx = kept + (((int64_t)ci * v.n_layers + layer) * v.n_kv_heads + kvh) * c.keep + b * kBlockTokens;
  const int n = min(kBlockTokens, c.keep - b * kBlockTokens);
  // lane t of each 16: the token that comes to place t (beyond the last: the last once more, unwritten)
  const int from = idx[min(lane & 15, n - 1)];
  const int64_t rec = kv4_record<HD>(v, layer, v.table[c.from_off[ci] + from / kBlockTokens], kvh);
  const int tok = from % kBlockTokens;
  uint8_t* to = v.pool + kv4_record<HD>(v, layer, v.table[c.to_off[ci] + b], kvh);
  auto of = [&](int place, int& place_tok) {  // record and place of the token that comes to `place`
    place_tok = __shfl(tok, place);
    const unsigned lo = __shfl((unsigned)rec, place), hi = __shfl((unsigned)(rec >> 32), place);
    return v.pool + (int64_t)(((uint64_t)hi << 32) | lo);
  };
  int st;
  // keys: four lanes a token
  const uint8_t* src = of(lane >> 2, st);
  uint4 k16;
  uint2 k8;
  if constexpr (HD == 128) k16 = *(const uint4*)(src + key_unit<HD>(st, (lane & 3) * 4));
  else k8 = *(const uint2*)(src + key_unit<HD>(st, (lane & 3) * 4));
  // values: lane = (unit, token % 4), four tokens at a time
  unit_t<HD> val[4];
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const uint8_t* s = of(4 * g + (lane & 3), st);
    val[g] = *(const unit_t<HD>*)(s + value_unit<HD>(st, lane >> 2));
  }
  // powers: a byte each
  const uint8_t* kps = of((lane / U) & 15, st);
  const uint8_t kp = kps[key_power<HD>(st, lane % U)];
  const int vt = (lane / (4 * U)) * 4 + (lane & 3);
  const uint8_t* vps = of(vt & 15, st);
  const uint8_t vp = vps[value_power<HD>(st, (lane >> 2) % U)];
  if ((lane >> 2) < n) {
    if constexpr (HD == 128) *(uint4*)(to + key_unit<HD>(lane >> 2, (lane & 3) * 4)) = k16;
    else *(uint2*)(to + key_unit<HD>(lane >> 2, (lane & 3) * 4)) = k8;
  }
#pragma unroll
  for (int g = 0; g < 4; ++g)
    if (4 * g + (lane & 3) < n) *(unit_t<HD>*)(to + value_unit<HD>(4 * g + (lane & 3), lane >> 2)) = val[g];
  if (lane < kBlockTokens * U && lane / U < n) to[key_power<HD>(lane / U, lane % U)] = kp;
  if (lane < kBlockTokens * U && vt < n) to[value_power<HD>(vt, (lane >> 2) % U)] = vp;
}

hipError_t launch_kv4_move(int head_dim, const Kv4View& v, const Kv4Cuts& c, const int32_t* kept, hipStream_t st) {
  const int n = c.keep / (4 * kBlockTokens) + 1;
  for (int first = 0; first < n; first += kKv4MaxItems) {
    const dim3 grid(v.n_kv_heads * v.n_layers, std::min(n - first, kKv4MaxItems), c.n);
    if (head_dim == 128) kv4_move_kernel<128><<<grid, 256, 0, st>>>(v, c, kept, first);
    else kv4_move_kernel<64><<<grid, 256, 0, st>>>(v, c, kept, first);
  }
  return hipGetLastError();
}

}  // namespace pipesd
