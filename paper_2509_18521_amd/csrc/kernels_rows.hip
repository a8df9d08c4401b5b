// Rows chosen by an index, and their gradients: the embedding's rows of tokens, tokens' rows in their experts' batches.  gfx950.
//
// All sums of rows are in fp32, in an order that the indexes alone decide (a stable sort, then ascending rows): no atomics on values.
#include <algorithm>

#include "train.h"

namespace april {
namespace {

// ---------------------------------------------------------------------------
// Stable sort of n small keys: passes over digits of 9 bits, in tiles of 4096 keys.  A wavefront ranks 64 keys at a time: the lanes
// with an equal digit by nine ballots, those of earlier steps by its own counters in LDS.
// ---------------------------------------------------------------------------
constexpr int BITS = 9, BINS = 1 << BITS;
constexpr int SORT_THREADS = 1024, SORT_WAVES = 16, SORT_STEPS = 4, SORT_TILE = SORT_THREADS * SORT_STEPS;

struct SortIn {
  const void* ids;         // the caller's, where keys is null; one outside 0 .. limit - 1 counts as limit
  bool i64;
  int limit, n;
  const int *keys, *rows;  // an earlier pass's result
  __device__ int key(int i) const {
    if (keys != nullptr) return keys[i];
    const long long v = index_at(ids, i64, i);
    return v >= 0 && v < limit ? (int)v : limit;
  }
  __device__ int row(int i) const { return rows != nullptr ? rows[i] : i; }
};

__global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(SortIn in, int shift, int* hist) {
  __shared__ int bins[BINS];
  const int tid = threadIdx.x;
  if (tid < BINS) bins[tid] = 0;
  __syncthreads();
#pragma unroll
  for (int s = 0; s < SORT_STEPS; ++s) {
    const long long i = (long long)blockIdx.x * SORT_TILE + s * SORT_THREADS + tid;
    if (i < in.n) atomicAdd(&bins[(in.key((int)i) >> shift) & (BINS - 1)], 1);
  }
  __syncthreads();
  if (tid < BINS) hist[(size_t)blockIdx.x * BINS + tid] = bins[tid];
}

// hist[tile][bin] -> where the tile's first key of that bin goes.  One workgroup.  starts (experts): bins are experts, each begins at
// a multiple of `align`; entry n_bins is the end of the last one.
__global__ __launch_bounds__(BINS) void sort_offsets_kernel(int* hist, int n_tiles, int n_bins, int align, int* starts) {
  __shared__ int wave_sum[BINS / 64];
  const int b = threadIdx.x, lane = b & 63;
  int total = 0;
  for (int t = 0; t < n_tiles; ++t) total += hist[(size_t)t * BINS + b];
  const int room = b < n_bins ? (total + align - 1) / align * align : 0;
  int incl = room;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int o = __shfl_up(incl, off, 64);
    if (lane >= off) incl += o;
  }
  if (lane == 63) wave_sum[b >> 6] = incl;
  __syncthreads();
  for (int w = 0; w < b >> 6; ++w) incl += wave_sum[w];
  int at = incl - room;
  if (starts != nullptr && b <= n_bins) starts[b] = at;
  for (int t = 0; t < n_tiles; ++t) {
    const int c = hist[(size_t)t * BINS + b];
    hist[(size_t)t * BINS + b] = at;
    at += c;
  }
}

// Where each of the tile's keys goes: at(i, key, destination) for every one of them.
template <class F>
__device__ inline void sort_tile(const SortIn& in, int shift, const int* offsets, F at) {
  __shared__ int count[SORT_WAVES][BINS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < SORT_WAVES * BINS; i += SORT_THREADS) count[0][i] = 0;
  __syncthreads();
  volatile int* mine = count[wave];
  int key[SORT_STEPS], rank[SORT_STEPS];
  const long long first = (long long)blockIdx.x * SORT_TILE + wave * (64 * SORT_STEPS) + lane;
#pragma unroll
  for (int s = 0; s < SORT_STEPS; ++s) key[s] = first + 64 * s < in.n ? in.key((int)(first + 64 * s)) : -1;
#pragma unroll
  for (int s = 0; s < SORT_STEPS; ++s) {
    const int d = (key[s] >> shift) & (BINS - 1);
    unsigned long long same = __ballot(key[s] >= 0);
#pragma unroll
    for (int b = 0; b < BITS; ++b) {
      const unsigned long long has = __ballot((d >> b) & 1);
      same &= (d >> b) & 1 ? has : ~has;
    }
    const int before = mine[d];
    __builtin_amdgcn_wave_barrier();
    const int below = __popcll(same & ((1ull << lane) - 1));
    rank[s] = before + below;
    if (key[s] >= 0 && below == 0) mine[d] = before + __popcll(same);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  if (tid < BINS) {
    int sum = offsets[(size_t)blockIdx.x * BINS + tid];
#pragma unroll
    for (int w = 0; w < SORT_WAVES; ++w) {
      const int c = count[w][tid];
      count[w][tid] = sum;
      sum += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int s = 0; s < SORT_STEPS; ++s)
    if (key[s] >= 0) at((int)(first + 64 * s), key[s], count[wave][(key[s] >> shift) & (BINS - 1)] + rank[s]);
}

__global__ __launch_bounds__(SORT_THREADS) void sort_move_kernel(SortIn in, int shift, const int* offsets, int* keys, int* rows) {
  sort_tile(in, shift, offsets, [&](int i, int key, int to) { keys[to] = key; rows[to] = in.row(i); });
}

__global__ __launch_bounds__(SORT_THREADS) void expert_place_kernel(SortIn in, const int* offsets, int* source, int* position) {
  sort_tile(in, 0, offsets, [&](int i, int key, int to) {
    position[i] = key < in.limit ? to : -1;
    if (key < in.limit) source[to] = i;
  });
}

__global__ __launch_bounds__(256) void fill_i32_kernel(int* p, int v, int n) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = v;
}

int blocks_of(long long n, int per) { return (int)((n + per - 1) / per); }

// ---------------------------------------------------------------------------
// Rows as vectors of V elements: loads and stores of 16 bytes of the wider type where every row allows them, else single elements.
// ---------------------------------------------------------------------------
template <typename T, int V>
struct Pack {
  typedef T type __attribute__((ext_vector_type(V)));
};
template <typename T>
struct Pack<T, 1> {
  typedef T type;
};
template <typename T, int V>
__device__ inline void load(float (&x)[V], const T* p) {
  if constexpr (V * sizeof(T) > 16) {
    float a[V / 2], b[V / 2];
    load<T, V / 2>(a, p);
    load<T, V / 2>(b, p + V / 2);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) { x[i] = a[i]; x[V / 2 + i] = b[i]; }
  } else if constexpr (V == 1) {
    x[0] = (float)*p;
  } else {
    const auto v = *reinterpret_cast<const typename Pack<T, V>::type*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = (float)v[i];
  }
}
template <typename T, int V>
__device__ inline void store(T* p, const float (&x)[V]) {
  if constexpr (V == 1) {
    *p = (T)x[0];
  } else {
    typename Pack<T, V>::type v;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (T)x[i];
    *reinterpret_cast<typename Pack<T, V>::type*>(p) = v;
  }
}
template <int V>
__device__ inline void zero(float (&x)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = 0.f;
}

template <typename T> constexpr int wide() { return 16 / (int)sizeof(T); }
template <typename A, typename B> constexpr int wide() { return 16 / (int)std::max(sizeof(A), sizeof(B)); }

bool rows_aligned(const void* p, long long row, size_t element, int v) {
  return reinterpret_cast<uintptr_t>(p) % (v * element) == 0 && row % v == 0;
}

// A workgroup of 256 threads takes 256 vectors at a time of the `per_row` x rows ones.
constexpr int ROWS_THREADS = 256;
struct At {
  long long row;
  int col;                 // in vectors
};
__device__ inline At vector_at(long long first, int tid, int per_row) {
  const long long r = first / per_row;
  const unsigned off = (unsigned)(first - r * per_row) + tid, q = off / (unsigned)per_row;
  return At{r + q, (int)(off - q * per_row)};
}
dim3 vector_grid(long long rows, int per_row) {
  const long long n = (rows * per_row + ROWS_THREADS - 1) / ROWS_THREADS;
  return dim3((unsigned)std::max<long long>(1, std::min<long long>(n, 1 << 22)));
}
#define FOR_VECTORS(rows, per_row)                                                                                       \
  for (long long first_ = (long long)blockIdx.x * ROWS_THREADS; first_ < (long long)(rows) * (per_row); first_ += (long long)gridDim.x * ROWS_THREADS) \
    if (const At at = vector_at(first_, threadIdx.x, per_row); at.row < (rows))

// ---------------------------------------------------------------------------
// Embedding: rows of the table, scaled.
// ---------------------------------------------------------------------------
template <typename TT, typename TO, int V>
__global__ __launch_bounds__(ROWS_THREADS) void embed_kernel(Embed a, int per_row) {
  FOR_VECTORS(a.n_rows, per_row) {
    const long long tok = index_at(a.tokens, a.i64, at.row);
    float x[V];
    zero(x);
    if (tok >= 0 && tok < a.vocab) load<TT, V>(x, static_cast<const TT*>(a.table) + tok * a.table_row + (long long)at.col * V);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = tok < a.vocab ? x[i] * a.scale : NAN;
    if (tok < 0) zero(x);
    store<TO, V>(static_cast<TO*>(a.out) + at.row * a.out_row + (long long)at.col * V, x);
  }
}

template <typename TT, typename TO>
hipError_t embed(hipStream_t st, const Embed& a) {
  constexpr int V = wide<TT, TO>();
  const bool vec = a.d % V == 0 && rows_aligned(a.table, a.table_row, sizeof(TT), V) && rows_aligned(a.out, a.out_row, sizeof(TO), V);
  const int per_row = vec ? a.d / V : a.d;
  const dim3 grid = vector_grid(a.n_rows, per_row), block(ROWS_THREADS);
  return vec ? enqueue(embed_kernel<TT, TO, V>, grid, block, st, a, per_row) : enqueue(embed_kernel<TT, TO, 1>, grid, block, st, a, per_row);
}

// ---------------------------------------------------------------------------
// The embedding's gradient.  Rows sorted by token; a token's rows are added in ascending order.  A run of more than PIECE rows is
// added up in pieces of the sorted order's blocks of PIECE (each block holds the end of one such run at most and the beginning of
// another: two partial sums), and the pieces are added in order.
// ---------------------------------------------------------------------------
constexpr int PIECE = 128;

struct Sorted {
  const int *keys, *rows, *starts;     // starts[t]: first row of token t; starts[vocab]: rows that have a token
  float* partial;                      // [blocks][2][d]
};

// A thread for each token: the first of the sorted keys that is no less.
__global__ __launch_bounds__(256) void run_starts_kernel(const int* keys, int n, int vocab, int* starts) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t > vocab) return;
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    if (keys[mid] < t) lo = mid + 1;
    else hi = mid;
  }
  starts[t] = lo;
}

template <typename TO, int V>
__device__ inline void add_rows(float (&sum)[V], const EmbedGrad& a, const int* rows, int n, int col) {
  const TO* g = static_cast<const TO*>(a.grad_out) + (long long)col * V;
  for (int i = 0; i < n; ++i) {
    float x[V];
    load<TO, V>(x, g + (long long)rows[i] * a.out_row);
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] += x[j];
  }
}
template <typename TT, int V>
__device__ inline void put_sum(const EmbedGrad& a, long long token, int col, float (&sum)[V]) {
  TT* to = static_cast<TT*>(a.grad_table) + token * a.table_row + (long long)col * V;
  float x[V];
  zero(x);
  if (a.accumulate) load<TT, V>(x, to);
#pragma unroll
  for (int j = 0; j < V; ++j) x[j] += a.scale * sum[j];
  store<TT, V>(to, x);
}

template <typename TO, typename TT, int V>
__global__ __launch_bounds__(ROWS_THREADS) void embed_grad_kernel(EmbedGrad a, Sorted s, int per_row) {
  FOR_VECTORS(a.vocab, per_row) {
    const int first = s.starts[at.row], n = s.starts[at.row + 1] - first;
    if (n > PIECE || (n == 0 && a.accumulate)) continue;
    float sum[V];
    zero(sum);
    add_rows<TO, V>(sum, a, s.rows + first, n, at.col);
    put_sum<TT, V>(a, at.row, at.col, sum);
  }
}
template <typename TO, int V>
__global__ __launch_bounds__(ROWS_THREADS) void embed_pieces_kernel(EmbedGrad a, Sorted s, int per_row) {
  const int n = s.starts[a.vocab], p0 = blockIdx.x * PIECE, p1 = min(p0 + PIECE, n);
  if (p0 >= n) return;
  const int t[2] = {s.keys[p0], s.keys[p1 - 1]};
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const int first = s.starts[t[w]], end = s.starts[t[w] + 1];
    if (end - first <= PIECE || (w == 0) != (first < p0)) continue;
    const int from = max(first, p0), to = min(end, p1);
    for (int col = threadIdx.x; col < per_row; col += ROWS_THREADS) {
      float sum[V];
      zero(sum);
      add_rows<TO, V>(sum, a, s.rows + from, to - from, col);
      store<float, V>(s.partial + ((size_t)blockIdx.x * 2 + w) * a.d + (size_t)col * V, sum);
    }
  }
}
template <typename TT, int V>
__global__ __launch_bounds__(ROWS_THREADS) void embed_join_kernel(EmbedGrad a, Sorted s, int per_row) {
  const int n = s.starts[a.vocab], p0 = blockIdx.x * PIECE, p1 = min(p0 + PIECE, n);
  if (p0 >= n) return;
  const int t = s.keys[p1 - 1], first = s.starts[t], end = s.starts[t + 1];
  if (end - first <= PIECE || first < p0) return;
  for (int col = threadIdx.x; col < per_row; col += ROWS_THREADS) {
    float sum[V];
    load<float, V>(sum, s.partial + ((size_t)blockIdx.x * 2 + 1) * a.d + (size_t)col * V);
    for (int b = blockIdx.x + 1; (long long)b * PIECE < end; ++b) {
      float x[V];
      load<float, V>(x, s.partial + (size_t)b * 2 * a.d + (size_t)col * V);
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] += x[j];
    }
    put_sum<TT, V>(a, t, col, sum);
  }
}

// The workspace: hist, two sets of keys and rows, starts, partial sums, each 16-byte aligned.
struct GradSpace {
  int *hist, *keys[2], *rows[2], *starts;
  float* partial;
  size_t bytes;
  explicit GradSpace(const EmbedGrad& a) {
    char* p = static_cast<char*>(a.ws);
    size_t at = 0;
    auto take = [&](size_t n) { char* q = p + at; at += (n + 15) / 16 * 16; return q; };
    const size_t n = a.n_rows;
    hist = (int*)take((size_t)blocks_of(n, SORT_TILE) * BINS * 4);
    for (int i = 0; i < 2; ++i) { keys[i] = (int*)take(n * 4); rows[i] = (int*)take(n * 4); }
    starts = (int*)take(((size_t)a.vocab + 1) * 4);
    partial = (float*)take((size_t)blocks_of(n, PIECE) * 2 * a.d * 4);
    bytes = at;
  }
};

template <typename TO, typename TT>
hipError_t embed_grad(hipStream_t st, const EmbedGrad& a) {
  const GradSpace w(a);
  const dim3 block(ROWS_THREADS);
  const int tiles = blocks_of(a.n_rows, SORT_TILE), blocks = blocks_of(a.n_rows, PIECE);
  SortIn in{a.tokens, a.i64, a.vocab, a.n_rows, nullptr, nullptr};
  hipError_t e = hipSuccess;
  int set = 0;
  for (int shift = 0; a.n_rows > 0 && (shift == 0 || a.vocab >> shift > 0); shift += BITS, set ^= 1) {
    if (e == hipSuccess) e = enqueue(sort_count_kernel, dim3(tiles), dim3(SORT_THREADS), st, in, shift, w.hist);
    if (e == hipSuccess) e = enqueue(sort_offsets_kernel, dim3(1), dim3(BINS), st, w.hist, tiles, BINS, 1, (int*)nullptr);
    if (e == hipSuccess) e = enqueue(sort_move_kernel, dim3(tiles), dim3(SORT_THREADS), st, in, shift, (const int*)w.hist, w.keys[set], w.rows[set]);
    in.keys = w.keys[set];
    in.rows = w.rows[set];
  }
  const Sorted s{in.keys, in.rows, w.starts, w.partial};
  if (e == hipSuccess) e = enqueue(run_starts_kernel, dim3(blocks_of((long long)a.vocab + 1, 256)), dim3(256), st, s.keys, a.n_rows, a.vocab, w.starts);
  constexpr int V = wide<TO, TT>();
  const bool vec = a.d % V == 0 && rows_aligned(a.grad_out, a.out_row, sizeof(TO), V) && rows_aligned(a.grad_table, a.table_row, sizeof(TT), V);
  const int per_row = vec ? a.d / V : a.d;
  const dim3 grid = vector_grid(a.vocab, per_row);
  if (e == hipSuccess) e = vec ? enqueue(embed_grad_kernel<TO, TT, V>, grid, block, st, a, s, per_row) : enqueue(embed_grad_kernel<TO, TT, 1>, grid, block, st, a, s, per_row);
  if (a.n_rows <= PIECE) return e;
  if (e == hipSuccess) e = vec ? enqueue(embed_pieces_kernel<TO, V>, dim3(blocks), block, st, a, s, per_row) : enqueue(embed_pieces_kernel<TO, 1>, dim3(blocks), block, st, a, s, per_row);
  if (e == hipSuccess) e = vec ? enqueue(embed_join_kernel<TT, V>, dim3(blocks), block, st, a, s, per_row) : enqueue(embed_join_kernel<TT, 1>, dim3(blocks), block, st, a, s, per_row);
  return e;
}

// ---------------------------------------------------------------------------
// Tokens' rows in their experts' batches.
// ---------------------------------------------------------------------------
// Rows of no assignment are zeros.
template <typename T, int V>
__global__ __launch_bounds__(ROWS_THREADS) void expert_gather_kernel(ExpertRows a, int per_row) {
  const long long n = (long long)a.n_rows * a.k;
  FOR_VECTORS(a.n_packed, per_row) {
    const int from = a.source[at.row];
    float x[V];
    zero(x);
    if (from >= 0 && from < n) load<T, V>(x, static_cast<const T*>(a.rows) + (long long)(from / a.k) * a.row + (long long)at.col * V);
    store<T, V>(static_cast<T*>(a.out) + at.row * a.packed_row + (long long)at.col * V, x);
  }
}

template <typename T, int V>
__global__ __launch_bounds__(ROWS_THREADS) void expert_combine_kernel(ExpertRows a, int per_row) {
  FOR_VECTORS(a.n_rows, per_row) {
    float sum[V];
    zero(sum);
    for (int j = 0; j < a.k; ++j) {
      const int from = a.position[at.row * a.k + j];
      if (from < 0 || from >= a.n_packed) continue;
      const float w = a.weights ? a.weights[at.row * a.k + j] : 1.f;
      float x[V];
      load<T, V>(x, static_cast<const T*>(a.packed) + (long long)from * a.packed_row + (long long)at.col * V);
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] += w * x[i];
    }
    store<T, V>(static_cast<T*>(a.out) + at.row * a.row + (long long)at.col * V, sum);
  }
}

// One wavefront a packed row: its gradient, and its weight's.
template <typename T, int V>
__global__ __launch_bounds__(ROWS_THREADS) void expert_combine_grad_kernel(ExpertRows a, int per_row) {
  const int lane = threadIdx.x & 63;
  const long long n = (long long)a.n_rows * a.k;
  for (long long p = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); p < a.n_packed; p += (long long)gridDim.x * 4) {
    const int from = a.source[p];
    const bool there = from >= 0 && from < n;
    const float w = there && a.weights ? a.weights[from] : 1.f;
    float dot = 0.f;
    for (int col = lane; col < per_row; col += 64) {
      float g[V], y[V];
      zero(g);
      if (there) {
        load<T, V>(g, static_cast<const T*>(a.rows) + (long long)(from / a.k) * a.row + (long long)col * V);
        if (a.grad_weights) {
          load<T, V>(y, static_cast<const T*>(a.packed) + p * a.packed_row + (long long)col * V);
#pragma unroll
          for (int i = 0; i < V; ++i) dot += g[i] * y[i];
        }
      }
#pragma unroll
      for (int i = 0; i < V; ++i) g[i] *= w;
      if (a.grad_packed) store<T, V>(static_cast<T*>(a.grad_packed) + p * a.grad_row + (long long)col * V, g);
    }
    dot = wave_sum_f32(dot);
    if (there && a.grad_weights && lane == 0) a.grad_weights[from] = dot;
  }
}
// Weights of assignments that are nowhere.
__global__ __launch_bounds__(256) void expert_lost_kernel(ExpertRows a) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i < (long long)a.n_rows * a.k && (a.position[i] < 0 || a.position[i] >= a.n_packed)) a.grad_weights[i] = 0.f;
}

bool vectors(const ExpertRows& a, int v) {
  const size_t e = a.f32 ? 4 : 2;
  auto fine = [&](const void* p, long long row) { return p == nullptr || rows_aligned(p, row, e, v); };
  return a.d % v == 0 && fine(a.rows, a.row) && fine(a.packed, a.packed_row) && fine(a.grad_packed, a.grad_row);
}

}  // namespace

hipError_t launch_embed(hipStream_t st, const Embed& a) {
  if (a.table_f32) return a.out_f32 ? embed<float, float>(st, a) : embed<float, bf16_t>(st, a);
  return a.out_f32 ? embed<bf16_t, float>(st, a) : embed<bf16_t, bf16_t>(st, a);
}

size_t embed_grad_workspace(const EmbedGrad& a) { return GradSpace(a).bytes; }

hipError_t launch_embed_grad(hipStream_t st, const EmbedGrad& a) {
  if (a.out_f32) return a.table_f32 ? embed_grad<float, float>(st, a) : embed_grad<float, bf16_t>(st, a);
  return a.table_f32 ? embed_grad<bf16_t, float>(st, a) : embed_grad<bf16_t, bf16_t>(st, a);
}

size_t expert_sort_workspace(const ExpertSort& a) { return (size_t)blocks_of(a.n, SORT_TILE) * BINS * 4; }

hipError_t launch_expert_sort(hipStream_t st, const ExpertSort& a) {
  const int tiles = blocks_of(a.n, SORT_TILE);
  const SortIn in{a.ids, a.i64, a.n_experts, a.n, nullptr, nullptr};
  int* hist = static_cast<int*>(a.ws);
  hipError_t e = hipSuccess;
  if (a.n_packed > 0) e = enqueue(fill_i32_kernel, dim3(blocks_of(a.n_packed, 256)), dim3(256), st, a.source, -1, a.n_packed);
  if (e == hipSuccess && tiles > 0) e = enqueue(sort_count_kernel, dim3(tiles), dim3(SORT_THREADS), st, in, 0, hist);
  if (e == hipSuccess) e = enqueue(sort_offsets_kernel, dim3(1), dim3(BINS), st, hist, tiles, a.n_experts, a.align, a.starts);
  if (e == hipSuccess && tiles > 0) e = enqueue(expert_place_kernel, dim3(tiles), dim3(SORT_THREADS), st, in, (const int*)hist, a.source, a.position);
  return e;
}

hipError_t launch_expert_gather(hipStream_t st, const ExpertRows& a) {
  constexpr int F = wide<float>(), B = wide<bf16_t>();
  ExpertRows c = a;
  c.packed = a.out;                                     // (for the alignment's test)
  const bool vec = vectors(c, a.f32 ? F : B);
  const int per_row = vec ? a.d / (a.f32 ? F : B) : a.d;
  const dim3 grid = vector_grid(a.n_packed, per_row), block(ROWS_THREADS);
  if (a.f32) return vec ? enqueue(expert_gather_kernel<float, F>, grid, block, st, a, per_row) : enqueue(expert_gather_kernel<float, 1>, grid, block, st, a, per_row);
  return vec ? enqueue(expert_gather_kernel<bf16_t, B>, grid, block, st, a, per_row) : enqueue(expert_gather_kernel<bf16_t, 1>, grid, block, st, a, per_row);
}

hipError_t launch_expert_combine(hipStream_t st, const ExpertRows& a) {
  constexpr int F = wide<float>(), B = wide<bf16_t>();
  ExpertRows c = a;
  c.rows = a.out;
  const bool vec = vectors(c, a.f32 ? F : B);
  const int per_row = vec ? a.d / (a.f32 ? F : B) : a.d;
  const dim3 grid = vector_grid(a.n_rows, per_row), block(ROWS_THREADS);
  if (a.f32) return vec ? enqueue(expert_combine_kernel<float, F>, grid, block, st, a, per_row) : enqueue(expert_combine_kernel<float, 1>, grid, block, st, a, per_row);
  return vec ? enqueue(expert_combine_kernel<bf16_t, B>, grid, block, st, a, per_row) : enqueue(expert_combine_kernel<bf16_t, 1>, grid, block, st, a, per_row);
}

hipError_t launch_expert_combine_grad(hipStream_t st, const ExpertRows& a) {
  constexpr int F = wide<float>(), B = wide<bf16_t>();
  const bool vec = vectors(a, a.f32 ? F : B);
  const int per_row = vec ? a.d / (a.f32 ? F : B) : a.d;
  const dim3 grid(std::max(1, std::min(blocks_of(a.n_packed, 4), 1 << 22))), block(ROWS_THREADS);
  hipError_t e;
  if (a.f32) e = vec ? enqueue(expert_combine_grad_kernel<float, F>, grid, block, st, a, per_row) : enqueue(expert_combine_grad_kernel<float, 1>, grid, block, st, a, per_row);
  else e = vec ? enqueue(expert_combine_grad_kernel<bf16_t, B>, grid, block, st, a, per_row) : enqueue(expert_combine_grad_kernel<bf16_t, 1>, grid, block, st, a, per_row);
  if (e == hipSuccess && a.grad_weights && a.n_rows > 0) e = enqueue(expert_lost_kernel, dim3(blocks_of((long long)a.n_rows * a.k, 256)), dim3(256), st, a);
  return e;
}

}  // namespace april
