// The decision on a tree of drafts (Sec. 2.2 with several continuations a round): which drafts stand, and the token behind them.
//
// A row's children x_1, x_2, .. were drawn from q one after the other (distinct: without putting back), and are tried in order
// against what the target still wants: r_0 = p; draft i is taken with probability min(1, r(x_i) / s(x_i)), s = q without the drafts that
// were refused, over its sum S; if it is not, r becomes max(0, r - s) over its sum.  That keeps the target's distribution whatever the
// tree.  With r = max(0, p - a q) / T,
//   r - s = (p - (a + T / S) q) / T   wherever q is still there, and a refused draft has r < s, so nothing left,
// so all that a refusal changes is a += T / S: one number a row, and T = sum over the vocabulary of max(0, p - a q).
//
// T and the draw are sums of whole numbers floor(2^40 w): they have no order, and the decision is the same whoever sums.
//
// Rows whose children are tried need their sums one after the other, but rows do not need each other's: a launch forms the sums of all
// rows for their second children, the next for the third ones, and rows that the walk cannot come by are left out.  Bound by latency: a launch
// goes to memory for the trees, the drafts' p and q, the sums, and what all workgroups found; 64 rows of up to four children over
// 128256 tokens take three such launches of 2.8 us and the draw's 10.4, 16 clients over 32000 two of 5.8 and 10.6.
#include "tree.h"

namespace pipesd {

constexpr int kTThreads = 256;
constexpr int kTHold = 8;  // values of p and of q that a thread asks for at once
constexpr int kNone = 0x7fffffff;
static_assert(kTreeRows <= kTThreads, "a thread a row");

__device__ __forceinline__ float left_of(float p, float q, float a) { return fmaxf(0.f, fmaf(-a, q, p)); }  // p - a q rounded once
// floor(2^40 w) in two parts, high * 2^24 + low, of w < 256: both steps are exact, and cost a quarter of a conversion to 64 bits.
struct Fixed {
  unsigned high, low;
};
__device__ __forceinline__ Fixed fixed(float w) {
  const float x = w * 65536.f;
  const unsigned high = (unsigned)x;
  return Fixed{high, (unsigned)((x - (float)high) * 16777216.f)};
}
constexpr float kFixedBelow = 256.f;
__device__ __forceinline__ unsigned long long fixed_wide(float w) { return (unsigned long long)((double)w * 1099511627776.0); }
__device__ __forceinline__ unsigned long long lane_u64(unsigned long long v, int src) {
  return ((unsigned long long)__shfl((unsigned)(v >> 32), src, 64) << 32) | __shfl((unsigned)v, src, 64);
}

// A client's tree.  Thread r has row r; what others have to know of it is in LDS.
struct TreeShared {
  int parent[kTreeRows], children[kTreeRows];
  int taken[kTreeRows];      // the child that was taken, kTreeRows: none
  float a[kTreeRows];        // behind the last child that was tested
  float refused[kTreeRows];  // q of that child's token
  unsigned char alive[kTreeRows];
  int list[kTreeRows], count;
  int path[kTreeRows], length, at;  // the walk
  float u0;
};
struct TreeMine {
  int up, nth;
  float p, q, u;  // of the row's token where its parent drew it
  float2 ab;      // what an earlier launch left for its test
  bool child;
};
__device__ __forceinline__ TreeMine tree_rows(const TreeCall& t, int ci, TreeShared& s) {  // all threads
  const int r = threadIdx.x, n = t.rows[ci], row0 = t.row_off[ci];
  TreeMine m{0, 0, 0.f, 0.f, 0.f, make_float2(0.f, 1.f), false};
  const TreeRow first = t.row[min(r, kTreeRows - 1)];  // (of the launch's first client: asked for before it is known which client this is)
  if (r < n) {
    const TreeRow row = row0 == 0 ? first : t.row[row0 + r];
    m.ab = t.ws.ab[row0 + r];
    m.child = r > 0;
    m.up = max(0, (int)row.parent);
    m.nth = row.nth;
    m.u = row.u;
    if (m.child && t.q != nullptr) {
      m.p = t.p[(int64_t)(row0 + m.up) * t.p_stride + row.token];
      m.q = t.q[(int64_t)(row0 + m.up) * t.q_stride + row.token];
    }
    // (a child before this one was taken, or the row cannot be come by, and there is nothing: then it is not asked for, either)
    if (m.nth == 0) m.ab = make_float2(0.f, 1.f);
    s.parent[r] = m.up;
    s.children[r] = row.children;
    if (r == 0) s.u0 = row.u;
  }
  return m;
}

// What is known when the children up to the stage-th of every row have been tested; (a, b): what this row is tested with.
__device__ __forceinline__ void tree_tests(TreeShared& s, const TreeMine& m, int n, int stage, float a, float b) {
  const int r = threadIdx.x;
  const bool tested = m.child && m.nth < stage;
  if (r < n) {
    s.taken[r] = kTreeRows;
    s.a[r] = 0.f;
  }
  __syncthreads();
  const float ratio = left_of(m.p, m.q, a) / (b * m.q);
  if (tested && (ratio >= 1.f || m.u < ratio)) atomicMin(&s.taken[m.up], r);  // (u < 1; 0 / 0 is neither)
  if (tested && m.nth == min(stage, s.children[m.up]) - 1) {
    s.a[m.up] = a + b;
    s.refused[m.up] = m.q;
  }
  __syncthreads();
  if (r < n) s.alive[r] = r == 0 || (tested ? s.taken[m.up] == r : s.taken[m.up] == kTreeRows);
  if (r == 0) s.count = 0;
  __syncthreads();
}
// The rows that the walk may come by, whose children before the stage-th were all refused and that have another.  (In any order: what
// belongs to a row has its place by the row.)
__device__ __forceinline__ int tree_needs(TreeShared& s, int n, int stage) {
  const int r = threadIdx.x;
  bool need = r < n && s.children[r] > stage && s.taken[r] == kTreeRows;
  for (int j = r; need && j > 0; j = s.parent[j]) need = s.alive[j];
  if (need) s.list[atomicAdd(&s.count, 1)] = r;
  __syncthreads();
  return s.count;
}
__device__ __forceinline__ void tree_walk(TreeShared& s) {
  if (threadIdx.x == 0) {
    int at = 0, length = 0;
    while (s.taken[at] < kTreeRows) s.path[length++] = at = s.taken[at];
    s.at = at;
    s.length = length;
  }
  __syncthreads();
}
template <int NT>
__device__ __forceinline__ void tree_report(const TreeCall& t, int ci, const TreeShared& s, int token) {  // all threads
  int32_t* out = t.result + ci * t.result_stride;
  for (int64_t i = threadIdx.x; i < t.result_stride; i += NT)
    out[i] = i == 0 ? s.length : i == 1 ? token : i - 2 < s.length ? s.path[i - 2] : -1;
}

// what is left of a row: max(0, p - a q), and floor(2^40 ..) of it
struct TreeLeft {
  const float *p, *q;
  float a;
  int V;
  bool residual;
  __device__ __forceinline__ TreeLeft(const TreeCall& t, int row, float a_, bool residual_) : a(a_), V(t.V), residual(residual_) {
    p = t.p + (int64_t)row * t.p_stride;
    q = t.q + (int64_t)row * t.q_stride;
  }
  // of the tokens i0, i0 + step, .. (kTHold of them; nothing from `end` on)
  __device__ __forceinline__ void rest(int i0, int step, int end, float (&w)[kTHold]) const {
    float pv[kTHold], qv[kTHold];
#pragma unroll
    for (int j = 0; j < kTHold; ++j) {
      const int i = min(i0 + j * step, V - 1);
      pv[j] = p[i];
      qv[j] = residual ? q[i] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < kTHold; ++j) w[j] = i0 + j * step < end ? left_of(pv[j], qv[j], a) : 0.f;
  }
  static __device__ __forceinline__ bool large(const float (&w)[kTHold]) {  // masses that no distribution has
    float top = w[0];
#pragma unroll
    for (int j = 1; j < kTHold; ++j) top = fmaxf(top, w[j]);
    return __ballot(!(top < kFixedBelow)) != 0;
  }
  // sum over [lo, hi), to all threads
  template <int NT>
  __device__ __forceinline__ unsigned long long sum(int lo, int hi, unsigned long long* red) const {
    unsigned long long x = 0;
    for (int base = lo; base < hi; base += NT * kTHold) {
      float w[kTHold];
      rest(base + threadIdx.x, NT, hi, w);
      if (large(w)) {
#pragma unroll
        for (int j = 0; j < kTHold; ++j) x += fixed_wide(w[j]);
      } else {
        unsigned high = 0, low = 0;
#pragma unroll
        for (int j = 0; j < kTHold; ++j) {
          const Fixed f = fixed(w[j]);
          high += f.high;
          low += f.low;
        }
        x += ((unsigned long long)high << 24) + low;
      }
    }
    x = sum_wave(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) x += red[i];
    return x;
  }
  // the first token of [lo, hi) whose running sum, `run` before the first, exceeds `bound`; hi - 1 if none does
  template <int NT>
  __device__ __forceinline__ int find(int lo, int hi, unsigned long long run, unsigned long long bound, unsigned long long* red, int* next) const {
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    if (tid == 0) *next = kNone;
    for (int base = lo; base < hi; base += NT * kTHold) {  // thread t has the kTHold tokens behind base + t * kTHold
      const int i0 = base + tid * kTHold;
      float rest_w[kTHold];
      unsigned long long wt[kTHold], own = 0;
      rest(i0, 1, hi, rest_w);
      const bool wide = large(rest_w);
#pragma unroll
      for (int j = 0; j < kTHold; ++j) {
        const Fixed f = fixed(rest_w[j]);
        wt[j] = wide ? fixed_wide(rest_w[j]) : ((unsigned long long)f.high << 24) + f.low;
        own += wt[j];
      }
      const unsigned long long inc = scan_wave(own);
      __syncthreads();
      if (lane == 63) red[w] = inc;
      __syncthreads();
      unsigned long long at = run + inc - own;
#pragma unroll
      for (int ww = 0; ww < NT / 64; ++ww) {
        if (ww < w) at += red[ww];
        run += red[ww];
      }
      int found = kNone;
#pragma unroll
      for (int j = 0; j < kTHold; ++j) {
        at += wt[j];
        if (at > bound) found = min(found, i0 + j);
      }
      if (found != kNone) atomicMin(next, found);
      __syncthreads();
      if (*next != kNone) break;
    }
    __syncthreads();
    return min(*next, hi - 1);
  }
  // the lowest index of the largest p (where nothing is left)
  template <int NT>
  __device__ __forceinline__ int best(unsigned long long* red) const {
    float x = -INFINITY;
    int xi = kNone;
    auto take = [&](float o, int oi) {
      if (o > x || (o == x && oi < xi)) x = o, xi = oi;
    };
    for (int i = threadIdx.x; i < V; i += NT) take(p[i], i);
    for (int o = 32; o > 0; o >>= 1) take(__shfl_xor(x, o, 64), __shfl_xor(xi, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = ((unsigned long long)__float_as_uint(x) << 32) | (unsigned)xi;
    __syncthreads();
    for (int i = 0; i < NT / 64; ++i) take(__uint_as_float((unsigned)(red[i] >> 32)), (int)(unsigned)red[i]);
    return min(xi, V - 1);
  }
};
__device__ __forceinline__ unsigned long long draw_bound(unsigned long long W, float u) {  // floor(2^24 u) W / 2^24
  const unsigned long long ui = (unsigned long long)(u * 16777216.0f);
  return (__umul64hi(W, ui) << 40) | ((W * ui) >> 24);
}

// Large vocabularies: a launch for the second children's sums, one for the third ones', .., and one for the walk and the draw.
// Workgroup (chunk of the vocabulary, client); the last one of a client that arrives goes on with what all have found.
__device__ __forceinline__ bool tree_arrives_last(const TreeCall& t, int ci, int* last) {  // thread 0 has written through
  if (threadIdx.x == 0) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    *last = atomicInc(&t.ws.counters[ci * 4], (unsigned)t.chunks - 1u) == (unsigned)t.chunks - 1u;  // (zero again behind the last)
  }
  __syncthreads();
  return *last;
}

__global__ __launch_bounds__(kTThreads) void tree_stage_kernel(TreeCall t, int stage) {
  __shared__ TreeShared s;
  __shared__ int last;
  __shared__ unsigned long long red[kTThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, ci = blockIdx.y, n = t.rows[ci], row0 = t.row_off[ci];
  const TreeMine m = tree_rows(t, ci, s);
  __syncthreads();
  tree_tests(s, m, n, stage, m.ab.x, m.ab.y);
  const int many = tree_needs(s, n, stage);
  if (many == 0) return;
  const int per = (t.V + t.chunks - 1) / t.chunks, lo = blockIdx.x * per, hi = min(t.V, lo + per);
#pragma unroll 1
  for (int i = 0; i < many; ++i) {
    const int r = s.list[i];
    const unsigned long long sum = TreeLeft(t, row0 + r, s.a[r], true).sum<kTThreads>(lo, hi, red);
    if (tid == 0) __hip_atomic_store(&t.ws.partial[(size_t)(row0 + r) * kTreeChunks + blockIdx.x], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  if (!tree_arrives_last(t, ci, &last)) return;
  for (int i = tid >> 6; i < many; i += kTThreads / 64) {
    const int r = s.list[i];
    const unsigned long long whole = sum_wave(
        lane < t.chunks ? __hip_atomic_load(&t.ws.partial[(size_t)(row0 + r) * kTreeChunks + lane], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0ull);
    double mass = 1.0;
    if (t.distinct) {
      mass = fmax((stage == 1 ? 1.0 : t.ws.mass[row0 + r]) - (double)s.refused[r], 1.0 / 16777216.0);
      if (lane == 0) t.ws.mass[row0 + r] = mass;
    }
    const float b = (float)((double)whole * (1.0 / 1099511627776.0) / mass);
    for (int c = lane; c < n; c += 64)
      if (c > 0 && s.parent[c] == r && t.row[row0 + c].nth == stage) t.ws.ab[row0 + c] = make_float2(s.a[r], b);
  }
}

__global__ __launch_bounds__(kTThreads) void tree_draw_kernel(TreeCall t) {
  __shared__ TreeShared s;
  __shared__ int last, next;
  __shared__ unsigned long long red[kTThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, ci = blockIdx.y, n = t.rows[ci], row0 = t.row_off[ci];
  const TreeMine m = tree_rows(t, ci, s);
  __syncthreads();
  tree_tests(s, m, n, t.stages, m.ab.x, m.ab.y);
  tree_walk(s);
  const TreeLeft left(t, row0 + s.at, s.a[s.at], s.children[s.at] > 0);
  const int per = (t.V + t.chunks - 1) / t.chunks, lo = blockIdx.x * per, hi = min(t.V, lo + per);
  const unsigned long long sum = left.sum<kTThreads>(lo, hi, red);
  unsigned long long* partial = t.ws.partial + (size_t)row0 * kTreeChunks;
  if (tid == 0) __hip_atomic_store(&partial[blockIdx.x], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (!tree_arrives_last(t, ci, &last)) return;
  const unsigned long long mine = lane < t.chunks ? __hip_atomic_load(&partial[lane], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0ull;
  const unsigned long long upto = scan_wave(mine), W = lane_u64(upto, 63);
  if (W == 0) {
    tree_report<kTThreads>(t, ci, s, left.best<kTThreads>(red));
    return;
  }
  const unsigned long long bound = draw_bound(W, s.u0);
  const int above = __ffsll((long long)__ballot(upto > bound)), b = above > 0 ? above - 1 : t.chunks - 1;  // the chunk that passes it
  const int clo = b * per, chi = min(t.V, clo + per);
  tree_report<kTThreads>(t, ci, s, left.find<kTThreads>(clo, chi, lane_u64(upto, b) - lane_u64(mine, b), bound, red, &next));
}

// Small vocabularies: one workgroup goes through all of it, 8.7 us for 6 rows over 4096 tokens (a call 10 to 12; 14 in launches that
// hand on).
constexpr int kTSmallThreads = 512;
__global__ __launch_bounds__(kTSmallThreads) void tree_small_kernel(TreeCall t) {
  __shared__ TreeShared s;
  __shared__ float2 s_ab[kTreeRows];
  __shared__ double s_mass[kTreeRows];
  __shared__ int next;
  __shared__ unsigned long long red[kTSmallThreads / 64];
  const int tid = threadIdx.x, ci = blockIdx.x, n = t.rows[ci], row0 = t.row_off[ci];
  const TreeMine m = tree_rows(t, ci, s);
  if (tid < n) s_mass[tid] = 1.0, s_ab[tid] = make_float2(0.f, 1.f);
  __syncthreads();
#pragma unroll 1
  for (int stage = 1; stage < t.stages; ++stage) {
    const float2 ab = s_ab[min(tid, n - 1)];
    tree_tests(s, m, n, stage, ab.x, ab.y);
    const int many = tree_needs(s, n, stage);
    if (many == 0) continue;  // (a later stage's rows are some of this one's, too)
#pragma unroll 1
    for (int i = 0; i < many; ++i) {
      const int r = s.list[i];
      const unsigned long long whole = TreeLeft(t, row0 + r, s.a[r], true).sum<kTSmallThreads>(0, t.V, red);
      if (m.child && m.up == r && m.nth == stage) {
        double mass = 1.0;
        if (t.distinct) s_mass[r] = mass = fmax(s_mass[r] - (double)s.refused[r], 1.0 / 16777216.0);
        s_ab[tid] = make_float2(s.a[r], (float)((double)whole * (1.0 / 1099511627776.0) / mass));
      }
    }
    __syncthreads();
  }
  const float2 ab = s_ab[min(tid, n - 1)];
  tree_tests(s, m, n, t.stages, ab.x, ab.y);
  tree_walk(s);
  const TreeLeft left(t, row0 + s.at, s.a[s.at], s.children[s.at] > 0);
  const unsigned long long W = left.sum<kTSmallThreads>(0, t.V, red);
  tree_report<kTSmallThreads>(t, ci, s,
                              W == 0 ? left.best<kTSmallThreads>(red) : left.find<kTSmallThreads>(0, t.V, 0ull, draw_bound(W, s.u0), red, &next));
}

// ------------------------------------------------------------------------------------------------
// token matching: the largest probability of every row in chunks, then the walk
// ------------------------------------------------------------------------------------------------
__device__ __forceinline__ void take_best(float& x, int& xi, float o, int oi) {
  if (o > x || (o == x && oi < xi)) x = o, xi = oi;
}
__global__ __launch_bounds__(kTThreads) void tree_best_kernel(TreeCall t) {
  __shared__ float rb[kTThreads / 64];
  __shared__ int ri[kTThreads / 64];
  const int tid = threadIdx.x, row = blockIdx.y;
  const float* p = t.p + (int64_t)row * t.p_stride;
  const int per = (t.V + t.chunks - 1) / t.chunks, lo = blockIdx.x * per, hi = min(t.V, lo + per);
  float best = -INFINITY;
  int bi = kNone;
  for (int base = lo; base < hi; base += kTThreads * kTHold) {
    float pv[kTHold];
#pragma unroll
    for (int j = 0; j < kTHold; ++j) pv[j] = p[min(base + tid + j * kTThreads, t.V - 1)];
#pragma unroll
    for (int j = 0; j < kTHold; ++j) {
      const int i = base + tid + j * kTThreads;
      if (i < hi && pv[j] > best) best = pv[j], bi = i;
    }
  }
  for (int o = 32; o > 0; o >>= 1) take_best(best, bi, __shfl_xor(best, o, 64), __shfl_xor(bi, o, 64));
  if ((tid & 63) == 0) rb[tid >> 6] = best, ri[tid >> 6] = bi;
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < kTThreads / 64; ++i) take_best(best, bi, rb[i], ri[i]);
    t.ws.partial[(size_t)row * kTreeChunks + blockIdx.x] = ((unsigned long long)__float_as_uint(best) << 32) | (unsigned)bi;
  }
}
__global__ __launch_bounds__(kTThreads) void tree_match_kernel(TreeCall t) {
  __shared__ TreeShared s;
  __shared__ int best_of[kTreeRows];
  const int tid = threadIdx.x, lane = tid & 63, ci = blockIdx.x, n = t.rows[ci], row0 = t.row_off[ci];
  const TreeMine m = tree_rows(t, ci, s);
  for (int r = tid >> 6; r < n; r += kTThreads / 64) {
    float best = -INFINITY;
    int bi = kNone;
    if (lane < t.chunks) {
      const unsigned long long x = t.ws.partial[(size_t)(row0 + r) * kTreeChunks + lane];
      best = __uint_as_float((unsigned)(x >> 32));
      bi = (int)(unsigned)x;
    }
    for (int o = 32; o > 0; o >>= 1) take_best(best, bi, __shfl_xor(best, o, 64), __shfl_xor(bi, o, 64));
    if (lane == 0) best_of[r] = min(bi, t.V - 1);
  }
  if (tid < n) s.taken[tid] = kTreeRows;
  __syncthreads();
  if (m.child && t.row[row0 + tid].token == best_of[m.up]) atomicMin(&s.taken[m.up], tid);
  __syncthreads();
  tree_walk(s);
  tree_report<kTThreads>(t, ci, s, best_of[s.at]);
}

hipError_t launch_tree_accept(const TreeCall& c, hipStream_t st) {
  if (c.q == nullptr) {
    const int rows = c.row_off[c.n - 1] + c.rows[c.n - 1];
    tree_best_kernel<<<dim3(c.chunks, rows), kTThreads, 0, st>>>(c);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    tree_match_kernel<<<c.n, kTThreads, 0, st>>>(c);
    return hipGetLastError();
  }
  if (c.V <= kTreeSmall) {
    tree_small_kernel<<<c.n, kTSmallThreads, 0, st>>>(c);
    return hipGetLastError();
  }
  for (int stage = 1; stage < c.stages; ++stage) {
    tree_stage_kernel<<<dim3(c.chunks, c.n), kTThreads, 0, st>>>(c, stage);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  tree_draw_kernel<<<dim3(c.chunks, c.n), kTThreads, 0, st>>>(c);
  return hipGetLastError();
}

}  // namespace pipesd
