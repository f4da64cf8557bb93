// The paged cache of operators: block tables and the masks of trees, rows in and out, tokens and blocks moved.
#include "pages.h"

namespace pipesd {

// 16 bytes
typedef __attribute__((ext_vector_type(4))) unsigned piece_t;
struct BlockPieces {  // blocks in pieces
  piece_t* pool;
  int64_t layer, v;  // between layers; from keys to values
  int block;
  BlockPieces(int dtype, const KvView& view) {
    const int elems = dtype == PIPESD_F32 ? 4 : 8;  // (a block of a head is a multiple)
    pool = (piece_t*)view.pool;
    layer = view.layer_stride / elems;
    v = view.v_offset / elems;
    block = view.block_elems / elems;
  }
  // part: 2 * layer, and 1 for values
  __device__ __forceinline__ void copy(int part, int from_block, int to_block) const {
    piece_t* base = pool + (part >> 1) * layer + (part & 1 ? v : 0);
    const piece_t* from = base + (int64_t)from_block * block;
    piece_t* to = base + (int64_t)to_block * block;
    constexpr int N = 4;
    int i = threadIdx.x;
    for (; i + (N - 1) * 256 < block; i += N * 256) {
      piece_t x[N];
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = from[i + j * 256];
#pragma unroll
      for (int j = 0; j < N; ++j) to[i + j * 256] = x[j];
    }
    for (; i < block; i += 256) to[i] = from[i];
  }
};

// ------------------------------------------------------------------------------------------------
// what a pass begins with: new entries of the block tables, what every row of its trees sees, and blocks copied for clients that write
// into one that others hold as well
// ------------------------------------------------------------------------------------------------
// The first workgroups have a tree each, a thread a row, which walks up to the root (the very first also writes the entries); the others the
// keys or values of a block and layer.  One launch, because it is nothing but latency: 1.3 us for entries and trees, 3.5 with 15 blocks of
// two layers copied beside them.
__global__ __launch_bounds__(kPagesTreeRows) void pages_begin_kernel(BlockPieces pool, PagesBegin b, int32_t* table, uint32_t* masks) {
  __shared__ int parent[kPagesTreeRows];
  __shared__ uint32_t bits[kPagesTreeRows][kPagesMaskWords];
  const int tid = threadIdx.x, tree = blockIdx.x;
  if (tree == 0 && tid < b.n) table[b.at[tid]] = b.v[tid];
  if (tree >= b.trees) {  // (whole workgroup)
    const int i = tree - b.trees;
    if (b.own) pool.copy(i / b.own, b.own_from[i % b.own], b.own_to[i % b.own]);
    return;
  }
  int first = 0;  // of the tree's rows among the launch's
  for (int i = 0; i < tree; ++i) first += b.n_rows[i];
  const int n = b.n_rows[tree], lead = b.before[tree] & 31;
  if (tid < n) parent[tid] = b.parent[first + tid];
  __syncthreads();
  if (tid < n) {
#pragma unroll
    for (int w = 0; w < kPagesMaskWords; ++w) bits[tid][w] = w == 0 ? (1u << lead) - 1u : 0u;
    for (int j = tid; j >= 0; j = parent[j]) bits[tid][(lead + j) >> 5] |= 1u << ((lead + j) & 31);
  }
  __syncthreads();
  uint32_t* out = masks + (size_t)b.row_off[tree] * kPagesMaskWords;
  const uint32_t* from = &bits[0][0];
  for (int i = tid; i < n * kPagesMaskWords; i += kPagesTreeRows) out[i] = from[i];
}
static_assert(kPagesEntriesPerLaunch <= kPagesTreeRows && kPagesTreeRows == 256, "a thread an entry; threads that copy");
hipError_t launch_pages_begin(int dtype, const KvView& v, int n_layers, const PagesBegin& b, int32_t* table, uint32_t* masks, hipStream_t st) {
  pages_begin_kernel<<<std::max(1, b.trees + b.own * 2 * n_layers), kPagesTreeRows, 0, st>>>(BlockPieces(dtype, v), b, table, masks);
  return hipGetLastError();
}

__global__ __launch_bounds__(256) void pages_fork_kernel(PagesForks f, int32_t* table) {
  const int c = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
  if (i < f.blocks[c]) table[f.to[c] + i] = table[f.from[c] + i];
}
hipError_t launch_pages_fork(const PagesForks& f, int32_t* table, hipStream_t st) {
  pages_fork_kernel<<<dim3((f.most + 255) / 256, f.n), 256, 0, st>>>(f, table);
  return hipGetLastError();
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

// ------------------------------------------------------------------------------------------------
// store and read: a workgroup has a block of a head.  Keys lie as the rows do; values go through LDS to lie token beside token, which is
// how the attention's products take them: turned once here and not in every pass.  Stores of some rows are latency (the table, then the
// rows with what the block holds): 3.7 to 4.1 us.  Long ones are bound by memory: 131071 rows of 8 heads of 128 stored 193 us, 5.6 TB/s both
// ways; 6200 tokens of four layers read 30.8 us, 6.5 TB/s.
// ------------------------------------------------------------------------------------------------
template <typename T, int HD>
struct Piece {  // 16 bytes
  static constexpr int kElems = 16 / sizeof(T), kOfRow = HD / kElems, kOfTokens = kBlockTokens / kElems;  // of a token's row; of a channel's tokens
};
template <typename T, int HD>
struct Tile {  // a block's values, and room between channels that keeps a wave's stores in different banks
  T v[HD][kBlockTokens + 2];
};

template <int HD, typename T>
__global__ __launch_bounds__(256) void pages_store_kernel(KvView v, int layer, PagesRanges rg, const T* k, const T* val, int64_t k_stride,
                                                          int64_t v_stride) {
  typedef Piece<T, HD> P;
  __shared__ Tile<T, HD> tile;
  const int tid = threadIdx.x, kvh = blockIdx.y, c = blockIdx.z;
  const int first = rg.first[c], end = first + rg.count[c];
  const int b = first / kBlockTokens + blockIdx.x, t0 = b * kBlockTokens;
  if (t0 >= end) return;  // (whole workgroup)
  const int lo = max(first, t0) - t0, hi = min(end, t0 + kBlockTokens) - t0;  // of the block's tokens
  const int64_t base = (int64_t)layer * v.layer_stride + (int64_t)v.table[rg.table_off[c] + b] * v.block_elems + (int64_t)kvh * kBlockTokens * HD;
  T* kb = (T*)v.pool + base;
  T* vb = (T*)v.pool + base + v.v_offset;
  const int64_t row0 = rg.row_off[c] + (t0 - first);  // (of the block's first token; before the rows where the pass begins in it)
  // What other tokens of a block have is written again: the workgroup is the only one that writes there.  (It is asked for with the rows.)
  constexpr int PIECES = HD * P::kOfTokens, PER = (PIECES + 255) / 256;
  const bool whole = lo == 0 && hi == kBlockTokens;
  uint4 there[PER];
#pragma unroll
  for (int n = 0; n < PER; ++n) there[n] = make_uint4(0, 0, 0, 0);
  if (!whole) {
#pragma unroll
    for (int n = 0; n < PER; ++n)
      if (tid + n * 256 < PIECES) there[n] = ((const uint4*)vb)[tid + n * 256];
  }
  for (int i = tid; i < kBlockTokens * P::kOfRow; i += 256) {
    const int t = i / P::kOfRow, e = i % P::kOfRow * P::kElems;
    if (t < lo || t >= hi) continue;
    *(uint4*)(kb + t * HD + e) = *(const uint4*)(k + (row0 + t) * k_stride + kvh * HD + e);
    const uint4 x = *(const uint4*)(val + (row0 + t) * v_stride + kvh * HD + e);
    const T* xs = (const T*)&x;
#pragma unroll
    for (int j = 0; j < P::kElems; ++j) tile.v[e + j][t] = xs[j];
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < PER; ++n) {
    const int i = tid + n * 256, e = i / P::kOfTokens, t = i % P::kOfTokens * P::kElems;
    if (i >= PIECES) break;
    T* xs = (T*)&there[n];
    bool any = false;
#pragma unroll
    for (int j = 0; j < P::kElems; ++j)
      if (t + j >= lo && t + j < hi) xs[j] = tile.v[e][t + j], any = true;
    if (any) ((uint4*)vb)[i] = there[n];
  }
}

hipError_t launch_pages_store(int dtype, const KvView& v, int layer, const PagesRanges& r, const void* k, const void* val, int64_t k_stride,
                              int64_t v_stride, hipStream_t st) {
  by_type(dtype, v.head_dim, [&](auto hd, auto t) {
    typedef decltype(t) T;
    pages_store_kernel<decltype(hd)::value, T><<<dim3(r.most, v.n_kv_heads, r.n), 256, 0, st>>>(v, layer, r, (const T*)k, (const T*)val, k_stride,
                                                                                               v_stride);
  });
  return hipGetLastError();
}

template <int HD, typename T>
__global__ __launch_bounds__(256) void pages_read_kernel(KvView v, int layer0, PagesRanges rg, int64_t total_rows, T* k, T* val) {
  typedef Piece<T, HD> P;
  __shared__ Tile<T, HD> tile;
  const int tid = threadIdx.x, c = blockIdx.z, layer = blockIdx.y / v.n_kv_heads, kvh = blockIdx.y % v.n_kv_heads;
  const int first = rg.first[c], end = first + rg.count[c];
  const int b = first / kBlockTokens + blockIdx.x, t0 = b * kBlockTokens;
  if (t0 >= end) return;
  const int lo = max(first, t0) - t0, hi = min(end, t0 + kBlockTokens) - t0;
  const int64_t base = (int64_t)(layer0 + layer) * v.layer_stride + (int64_t)v.table[rg.table_off[c] + b] * v.block_elems + (int64_t)kvh * kBlockTokens * HD;
  const T* kb = (const T*)v.pool + base;
  const T* vb = (const T*)v.pool + base + v.v_offset;
  for (int i = tid; i < HD * P::kOfTokens; i += 256) {
    const int e = i / P::kOfTokens, t = i % P::kOfTokens * P::kElems;
    const uint4 x = *(const uint4*)(vb + e * kBlockTokens + t);
    const T* xs = (const T*)&x;
#pragma unroll
    for (int j = 0; j < P::kElems; ++j) tile.v[e][t + j] = xs[j];
  }
  __syncthreads();
  const int64_t row0 = (int64_t)layer * total_rows + rg.row_off[c] + (t0 - first);
  for (int i = tid; i < kBlockTokens * P::kOfRow; i += 256) {
    const int t = i / P::kOfRow, e = i % P::kOfRow * P::kElems;
    if (t < lo || t >= hi) continue;
    const int64_t at = ((row0 + t) * v.n_kv_heads + kvh) * HD + e;
    *(uint4*)(k + at) = *(const uint4*)(kb + t * HD + e);
    uint4 x;
    T* xs = (T*)&x;
#pragma unroll
    for (int j = 0; j < P::kElems; ++j) xs[j] = tile.v[e + j][t];
    *(uint4*)(val + at) = x;
  }
}

hipError_t launch_pages_read(int dtype, const KvView& v, int layer0, int n_layers, const PagesRanges& r, int64_t total_rows, void* k, void* val,
                             hipStream_t st) {
  const int per = std::max(1, 65535 / v.n_kv_heads);  // (a grid has at most 65535 workgroups in y: layers by the piece)
  for (int l0 = 0; l0 < n_layers; l0 += per) {
    const int nl = std::min(per, n_layers - l0);
    by_type(dtype, v.head_dim, [&](auto hd, auto t) {
      typedef decltype(t) T;
      const int64_t off = (int64_t)l0 * total_rows * v.n_kv_heads * v.head_dim;
      pages_read_kernel<decltype(hd)::value, T><<<dim3(r.most, nl * v.n_kv_heads, r.n), 256, 0, st>>>(v, layer0 + l0, r, total_rows, (T*)k + off,
                                                                                                     (T*)val + off);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ------------------------------------------------------------------------------------------------
// move: workgroup (a cache line of a token's key, or some channels of its value; layer and head), for keys eight threads a token, for
// values one.  What the tokens of a launch are moved over may be other tokens of it: all are read first, by the workgroup that writes
// them, and no wait between workgroups is needed.  Made for the rows of trees: some tens of tokens of four layers 4 us (latency), 448
// tokens of four layers and 8 heads of 64 6.0 us, 1.2 TB/s; with 16 bytes of a key to a workgroup, which eight chiplets' caches then fetch
// and write apart, 15 to 20.
// ------------------------------------------------------------------------------------------------
template <int HD, typename T>
__global__ __launch_bounds__(kPagesMovesPerLaunch) void pages_move_kernel(KvView v, int layer0, PagesMoves m) {
  typedef Piece<T, HD> P;
  constexpr int SLICE = 8, SLICES = P::kOfRow / SLICE;  // pieces of a key that a workgroup has: a cache line
  const int tid = threadIdx.x, layer = layer0 + blockIdx.y / v.n_kv_heads, kvh = blockIdx.y % v.n_kv_heads;
  T* keys = (T*)v.pool + (int64_t)layer * v.layer_stride + (int64_t)kvh * kBlockTokens * HD;
  if (blockIdx.x < SLICES) {
    const int e = (blockIdx.x * SLICE + tid % SLICE) * P::kElems, per = blockDim.x / SLICE;
    auto at = [&](int place) { return (piece_t*)(keys + (int64_t)(place / kBlockTokens) * v.block_elems + place % kBlockTokens * HD + e); };
    piece_t x[SLICE];
#pragma unroll
    for (int j = 0; j < SLICE; ++j) x[j] = *at(m.from[min(j * per + tid / SLICE, m.n - 1)]);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int j = 0; j < SLICE; ++j)
      if (j * per + tid / SLICE < m.n) *at(m.to[j * per + tid / SLICE]) = x[j];
    return;
  }
  const int e = (blockIdx.x - SLICES) * P::kElems;
  auto at = [&](int place) { return keys + v.v_offset + (int64_t)(place / kBlockTokens) * v.block_elems + e * kBlockTokens + place % kBlockTokens; };
  T xs[P::kElems];
  const T* from = at(m.from[min(tid, m.n - 1)]);
#pragma unroll
  for (int j = 0; j < P::kElems; ++j) xs[j] = from[j * kBlockTokens];
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid < m.n) {
    T* to = at(m.to[tid]);
#pragma unroll
    for (int j = 0; j < P::kElems; ++j) to[j * kBlockTokens] = xs[j];
  }
}

hipError_t launch_pages_move(int dtype, const KvView& v, int n_layers, const PagesMoves& m, hipStream_t st) {
  const int per = std::max(1, 65535 / v.n_kv_heads);
  for (int l0 = 0; l0 < n_layers; l0 += per) {
    const int nl = std::min(per, n_layers - l0);
    by_type(dtype, v.head_dim, [&](auto hd, auto t) {
      typedef decltype(t) T;
      constexpr int HD = decltype(hd)::value;
      pages_move_kernel<HD, T><<<dim3(Piece<T, HD>::kOfRow / 8 + Piece<T, HD>::kOfRow, nl * v.n_kv_heads), (m.n + 63) / 64 * 64, 0, st>>>(v, l0, m);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ------------------------------------------------------------------------------------------------
// copy: workgroup (block, its keys or values of a layer), four pieces of 16 bytes a thread at a time.  65536 tokens of four layers (8 heads
// of 128, 2.1 GB both ways) 400 us, 5.4 TB/s: a large copy.
// ------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void pages_copy_kernel(BlockPieces pool, int part0, PagesMoves m) {
  pool.copy(part0 + blockIdx.y, m.from[blockIdx.x], m.to[blockIdx.x]);
}
hipError_t launch_pages_copy(int dtype, const KvView& v, int n_layers, const PagesMoves& m, hipStream_t st) {
  for (int p0 = 0; p0 < 2 * n_layers; p0 += 65534) {
    pages_copy_kernel<<<dim3(m.n, std::min(65534, 2 * n_layers - p0)), 256, 0, st>>>(BlockPieces(dtype, v), p0, m);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace pipesd
