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
#include "tree.h"

namespace pipesd {

constexpr int kTThreads = 256;
constexpr int kTHold = 8;  // values of p and of q that a thread asks for at once
static_assert(kTreeRows <= kTThreads, "a thread a row");

__device__ __forceinline__ float left_of(float p, float q, float a) {  // max(0, p - a q) rounded once: the product is exact in 64 bits
  return fmaxf(0.f, (float)((double)p - (double)a * (double)q));
}
__device__ __forceinline__ unsigned long long fixed(float w) { return (unsigned long long)((double)w * 1099511627776.0); }

// What is known of a client's tree when the children up to the stage-th of every row have been tested.  All threads of the workgroup.
struct TreeState {
  int parent[kTreeRows];
  int taken[kTreeRows];   // the child that was taken, kTreeRows: none
  float a[kTreeRows];     // behind the last child that was tested
  float refused[kTreeRows];  // q of that child's token
  unsigned char alive[kTreeRows];
};
__device__ __forceinline__ void tree_state(const TreeCall& t, int ci, int stage, TreeState& s) {
  const int r = threadIdx.x, n = t.rows[ci], row0 = t.row_off[ci], at = row0 + min(r, n - 1);
  const int up = max(0, (int)t.parent[at]), nth = t.nth[at];
  const bool child = r > 0 && r < n, tested = child && nth < stage;
  float p = 0.f, q = 0.f, a = 0.f, b = 1.f;
  if (tested) {
    const int x = t.token[at];
    p = t.p[(int64_t)(row0 + up) * t.p_stride + x];
    q = t.q[(int64_t)(row0 + up) * t.q_stride + x];
    if (nth > 0) {  // (left by an earlier launch, unless a child before this one was taken or the row cannot be come by)
      const float2 ab = t.ws.ab[at];
      a = ab.x;
      b = ab.y;
    }
  }
  if (r < n) {
    s.parent[r] = up;
    s.taken[r] = kTreeRows;
    s.a[r] = 0.f;
  }
  __syncthreads();
  const float ratio = left_of(p, q, a) / (b * q);
  const bool good = tested && (ratio >= 1.f || t.u[at] < ratio);  // (u < 1; 0 / 0 is neither)
  if (good) atomicMin(&s.taken[up], r);
  if (tested && nth == min(stage, (int)t.children[row0 + up]) - 1) {
    s.a[up] = a + b;
    s.refused[up] = q;
  }
  __syncthreads();
  if (r < n) s.alive[r] = r == 0 || (tested ? s.taken[up] == r : s.taken[up] == kTreeRows);
  __syncthreads();
}

// Sums T of rows that the walk may come by and whose children before the stage-th were refused.  Workgroup (chunk of the vocabulary, client);
// the last one of a client joins the sums and leaves what the rows' next children are tested with.
__global__ __launch_bounds__(kTThreads) void tree_stage_kernel(TreeCall t, int stage) {
  __shared__ TreeState s;
  __shared__ int list[kTreeRows];
  __shared__ int count, last;
  __shared__ unsigned long long red[kTThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, ci = blockIdx.y, n = t.rows[ci], row0 = t.row_off[ci];
  if (tid == 0) count = 0;
  tree_state(t, ci, stage, s);
  bool need = tid < n && t.children[row0 + min(tid, n - 1)] > stage && s.taken[min(tid, n - 1)] == kTreeRows;
  for (int j = tid; need && j > 0; j = s.parent[j]) need = s.alive[j];
  if (need) list[atomicAdd(&count, 1)] = tid;  // (in any order: every workgroup has its own places, by row)
  __syncthreads();
  const int many = count;
  if (many == 0) return;
  const int per = (t.V + kTreeChunks - 1) / kTreeChunks, lo = blockIdx.x * per, hi = min(t.V, lo + per);
#pragma unroll 1
  for (int i = 0; i < many; ++i) {
    const int r = list[i];
    const float* p = t.p + (int64_t)(row0 + r) * t.p_stride;
    const float* q = t.q + (int64_t)(row0 + r) * t.q_stride;
    const float a = s.a[r];
    unsigned long long sum = 0;
    for (int base = lo; base < hi; base += kTThreads * kTHold) {
      float pv[kTHold], qv[kTHold];
#pragma unroll
      for (int j = 0; j < kTHold; ++j) {
        const int x = min(base + tid + j * kTThreads, t.V - 1);
        pv[j] = p[x];
        qv[j] = q[x];
      }
#pragma unroll
      for (int j = 0; j < kTHold; ++j) sum += base + tid + j * kTThreads < hi ? fixed(left_of(pv[j], qv[j], a)) : 0ull;
    }
    sum = sum_wave(sum);
    __syncthreads();
    if (lane == 0) red[w] = sum;
    __syncthreads();
    if (tid == 0)
      __hip_atomic_store(&t.ws.partial[(size_t)(row0 + r) * kTreeChunks + blockIdx.x], red[0] + red[1] + red[2] + red[3], __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
  }
  if (tid == 0) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    last = atomicInc(&t.ws.counters[ci * 4], (unsigned)kTreeChunks - 1u) == (unsigned)kTreeChunks - 1u;  // (zero again behind the last)
  }
  __syncthreads();
  if (!last) return;
  for (int i = w; i < many; i += kTThreads / 64) {
    const int r = list[i];
    const unsigned long long whole =
        sum_wave(__hip_atomic_load(&t.ws.partial[(size_t)(row0 + r) * kTreeChunks + lane], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    double mass = 1.0;
    if (t.distinct) {
      mass = fmax((stage == 1 ? 1.0 : t.ws.mass[row0 + r]) - (double)s.refused[r], 1.0 / 16777216.0);
      if (lane == 0) t.ws.mass[row0 + r] = mass;
    }
    const float b = (float)((double)whole * (1.0 / 1099511627776.0) / mass);
    for (int c = lane; c < n; c += 64)
      if (c > 0 && t.parent[row0 + c] == r && t.nth[row0 + c] == stage) t.ws.ab[row0 + c] = make_float2(s.a[r], b);
  }
}

__device__ __forceinline__ unsigned long long lane_u64(unsigned long long v, int src) {
  return ((unsigned long long)__shfl((unsigned)(v >> 32), src, 64) << 32) | __shfl((unsigned)v, src, 64);
}

// the walk as it came out: the accepted rows and the row that it ends at
__device__ __forceinline__ int tree_walk(const int* taken, int* path, int& at) {
  int length = 0;
  at = 0;
  while (taken[at] < kTreeRows) path[length++] = at = taken[at];
  return length;
}
__device__ __forceinline__ void tree_report(const TreeCall& t, int ci, int length, const int* path, int token) {  // all threads
  int32_t* out = t.result + ci * t.result_stride;
  for (int64_t i = threadIdx.x; i < t.result_stride; i += kTThreads)
    out[i] = i == 0 ? length : i == 1 ? token : i - 2 < length ? path[i - 2] : -1;
}

// The walk, and the draw from what is left where it ends: the integer inverse CDF of the chain's decision.  Workgroup (chunk, client).
__global__ __launch_bounds__(kTThreads) void tree_draw_kernel(TreeCall t) {
  constexpr int kWaves = kTThreads / 64, kNone = 0x7fffffff;
  __shared__ TreeState s;
  __shared__ int path[kTreeRows], s_at, s_length, s_last, s_next;
  __shared__ unsigned long long red[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, ci = blockIdx.y, row0 = t.row_off[ci];
  tree_state(t, ci, t.stages, s);
  if (tid == 0) {
    int at;
    s_length = tree_walk(s.taken, path, at);
    s_at = at;
    s_next = kNone;
  }
  __syncthreads();
  const int at = s_at, length = s_length;
  const bool residual = t.children[row0 + at] > 0;
  const float a = s.a[at];
  const float* p = t.p + (int64_t)(row0 + at) * t.p_stride;
  const float* q = t.q + (int64_t)(row0 + at) * t.q_stride;
  auto weights = [&](int i0, int step, int end, unsigned long long (&out)[kTHold]) {
    float pv[kTHold], qv[kTHold];
#pragma unroll
    for (int j = 0; j < kTHold; ++j) {
      const int i = min(i0 + j * step, t.V - 1);
      pv[j] = p[i];
      qv[j] = residual ? q[i] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < kTHold; ++j) out[j] = i0 + j * step < end ? fixed(left_of(pv[j], qv[j], a)) : 0ull;
  };
  const int per = (t.V + kTreeChunks - 1) / kTreeChunks, lo = blockIdx.x * per, hi = min(t.V, lo + per);
  unsigned long long sum = 0, wt[kTHold];
  for (int base = lo; base < hi; base += kTThreads * kTHold) {
    weights(base + tid, kTThreads, hi, wt);
#pragma unroll
    for (int j = 0; j < kTHold; ++j) sum += wt[j];
  }
  sum = sum_wave(sum);
  if (lane == 0) red[w] = sum;
  __syncthreads();
  unsigned long long* partial = t.ws.partial + (size_t)row0 * kTreeChunks;
  if (tid == 0) {
    __hip_atomic_store(&partial[blockIdx.x], red[0] + red[1] + red[2] + red[3], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    s_last = atomicInc(&t.ws.counters[ci * 4], (unsigned)kTreeChunks - 1u) == (unsigned)kTreeChunks - 1u;
  }
  __syncthreads();
  if (!s_last) return;

  const unsigned long long mine = __hip_atomic_load(&partial[lane], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const unsigned long long upto = scan_wave(mine), W = lane_u64(upto, 63);
  if (W == 0) {  // lowest-index maximum of the target row
    float best = -INFINITY;
    int bi = kNone;
    for (int i = tid; i < t.V; i += kTThreads)
      if (p[i] > best) best = p[i], bi = i;
    for (int o = 32; o > 0; o >>= 1) {
      const float ob = __shfl_xor(best, o, 64);
      const int oi = __shfl_xor(bi, o, 64);
      if (ob > best || (ob == best && oi < bi)) best = ob, bi = oi;
    }
    __syncthreads();
    if (lane == 0) red[w] = ((unsigned long long)__float_as_uint(best) << 32) | (unsigned)bi;
    __syncthreads();
    best = __uint_as_float((unsigned)(red[0] >> 32));
    bi = (int)(unsigned)red[0];
    for (int i = 1; i < kWaves; ++i) {
      const float ob = __uint_as_float((unsigned)(red[i] >> 32));
      const int oi = (int)(unsigned)red[i];
      if (ob > best || (ob == best && oi < bi)) best = ob, bi = oi;
    }
    tree_report(t, ci, length, path, min(bi, t.V - 1));
    return;
  }
  const unsigned long long ui = (unsigned long long)(t.u[row0] * 16777216.0f);  // floor(u * 2^24)
  const unsigned long long bound = (__umul64hi(W, ui) << 40) | ((W * ui) >> 24);
  const int above = __ffsll((long long)__ballot(upto > bound)), b = above > 0 ? above - 1 : kTreeChunks - 1;
  unsigned long long run = lane_u64(upto, b) - lane_u64(mine, b);
  const int clo = b * per, chi = min(t.V, clo + per);
  for (int base = clo; base < chi; base += kTThreads * kTHold) {  // thread t has the kTHold tokens behind base + t * kTHold
    const int i0 = base + tid * kTHold;
    weights(i0, 1, chi, wt);
    unsigned long long own = 0;
#pragma unroll
    for (int j = 0; j < kTHold; ++j) own += wt[j];
    const unsigned long long inc = scan_wave(own);
    if (lane == 63) red[w] = inc;
    __syncthreads();
    unsigned long long sum_at = run + inc - own;
#pragma unroll
    for (int ww = 0; ww < kWaves; ++ww) {
      if (ww < w) sum_at += red[ww];
      run += red[ww];
    }
    int found = kNone;
#pragma unroll
    for (int j = 0; j < kTHold; ++j) {
      sum_at += wt[j];
      if (sum_at > bound) found = min(found, i0 + j);
    }
    if (found != kNone) atomicMin(&s_next, found);
    __syncthreads();
    if (s_next != kNone) break;
  }
  __syncthreads();
  tree_report(t, ci, length, path, min(s_next, chi - 1));
}

// ------------------------------------------------------------------------------------------------
// token matching: the largest probability of every row in chunks, then the walk
// ------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(kTThreads) void tree_best_kernel(TreeCall t) {
  __shared__ float rb[kTThreads / 64];
  __shared__ int ri[kTThreads / 64];
  const int tid = threadIdx.x, row = blockIdx.y;
  const float* p = t.p + (int64_t)row * t.p_stride;
  const int per = (t.V + kTreeChunks - 1) / kTreeChunks, lo = blockIdx.x * per, hi = min(t.V, lo + per);
  float best = -INFINITY;
  int bi = 0x7fffffff;
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
  for (int o = 32; o > 0; o >>= 1) {
    const float ob = __shfl_xor(best, o, 64);
    const int oi = __shfl_xor(bi, o, 64);
    if (ob > best || (ob == best && oi < bi)) best = ob, bi = oi;
  }
  if ((tid & 63) == 0) rb[tid >> 6] = best, ri[tid >> 6] = bi;
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < kTThreads / 64; ++i)
      if (rb[i] > best || (rb[i] == best && ri[i] < bi)) best = rb[i], bi = ri[i];
    t.ws.partial[(size_t)row * kTreeChunks + blockIdx.x] = ((unsigned long long)__float_as_uint(best) << 32) | (unsigned)bi;
  }
}
__global__ __launch_bounds__(kTThreads) void tree_match_kernel(TreeCall t) {
  __shared__ int best_of[kTreeRows], taken[kTreeRows], path[kTreeRows], s_at, s_length;
  const int tid = threadIdx.x, lane = tid & 63, ci = blockIdx.x, n = t.rows[ci], row0 = t.row_off[ci];
  for (int r = tid >> 6; r < n; r += kTThreads / 64) {
    const unsigned long long x = t.ws.partial[(size_t)(row0 + r) * kTreeChunks + lane];
    float best = __uint_as_float((unsigned)(x >> 32));
    int bi = (int)(unsigned)x;
    for (int o = 32; o > 0; o >>= 1) {
      const float ob = __shfl_xor(best, o, 64);
      const int oi = __shfl_xor(bi, o, 64);
      if (ob > best || (ob == best && oi < bi)) best = ob, bi = oi;
    }
    if (lane == 0) best_of[r] = min(bi, t.V - 1);
  }
  if (tid < n) taken[tid] = kTreeRows;
  __syncthreads();
  if (tid > 0 && tid < n) {
    const int up = t.parent[row0 + tid];
    if (t.token[row0 + tid] == best_of[up]) atomicMin(&taken[up], tid);
  }
  __syncthreads();
  if (tid == 0) {
    int at;
    s_length = tree_walk(taken, path, at);
    s_at = at;
  }
  __syncthreads();
  tree_report(t, ci, s_length, path, best_of[s_at]);
}

hipError_t launch_tree_accept(const TreeCall& c, hipStream_t st) {
  if (c.q == nullptr) {
    const int rows = c.row_off[c.n - 1] + c.rows[c.n - 1];
    tree_best_kernel<<<dim3(kTreeChunks, rows), kTThreads, 0, st>>>(c);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    tree_match_kernel<<<c.n, kTThreads, 0, st>>>(c);
    return hipGetLastError();
  }
  for (int stage = 1; stage < c.stages; ++stage) {
    tree_stage_kernel<<<dim3(kTreeChunks, c.n), kTThreads, 0, st>>>(c, stage);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  tree_draw_kernel<<<dim3(kTreeChunks, c.n), kTThreads, 0, st>>>(c);
  return hipGetLastError();
}

}  // namespace pipesd
