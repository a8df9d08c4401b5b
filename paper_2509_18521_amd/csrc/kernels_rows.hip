// Rows chosen by an index, and their gradients: the embedding's rows of tokens, tokens' rows in their experts' batches.  gfx950.
//
// All sums of rows are in fp32, in an order that the indexes alone decide (a stable sort, then ascending rows): no atomics on values.
#include <algorithm>

#include "train.h"

namespace april {
namespace {

// ---------------------------------------------------------------------------
// Stable sort of n small keys: passes over digits of 9 bits, in tiles of 4096 keys.  A wavefront ranks 64 keys at a time: the lanes
// with an equal digit by nine ballots, those of earlier steps by its own counters in LDS.  A pass is two launches, digits counted for each tile, then moved: a
// tile's workgroup adds up the other tiles' counts itself (up to 256 tiles; beyond, a launch between does).  One tile is sorted in one launch.
// Bound by latency: 32768 tokens 15 us a pass, 111 k experts' ids 14, one tile of them 9.
// ---------------------------------------------------------------------------
constexpr int BITS = 9, BINS = 1 << BITS;
constexpr int SORT_THREADS = 1024, SORT_WAVES = 16, SORT_STEPS = 4, SORT_TILE = SORT_THREADS * SORT_STEPS;
constexpr int ADD_TILES = 256;
// Passes over keys up to `limit` (four from 2^27 on; a shift by 36 is none).
__host__ __device__ inline int sort_passes(int limit) { return limit >> BITS == 0 ? 1 : limit >> 2 * BITS == 0 ? 2 : limit >> 3 * BITS == 0 ? 3 : 4; }

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

// Zeros that a launch of the sort's writes beside its own work, on the workgroups behind the tiles': units `first` .. `end` - 1, each a row, or of
// adjacent rows 64 KB.
struct Zeros {
  char* p;
  bool streaming;
  long long unit, stride, total, first, end;      // bytes of a unit, from one to the next, of all (-1: every unit is whole); units
};
__device__ inline void write_zeros(const Zeros& z, int group, int groups) {
  const int tid = threadIdx.x, nt = blockDim.x;
  for (long long u = z.first + group; u < z.end; u += groups) {
    char* p = z.p + u * z.stride;
    const long long n = z.total < 0 ? z.unit : min(z.unit, z.total - u * z.stride);          // (a multiple of 2)
    const int head = (int)min(n, (long long)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15));
    const long long body = (n - head) / 16 * 16;
    for (int i = 2 * tid; i < head; i += 2 * nt) *reinterpret_cast<short*>(p + i) = 0;
    typedef int vec __attribute__((ext_vector_type(4)));
    vec* at = reinterpret_cast<vec*>(p + head);
    if (z.streaming)
      for (long long i = tid; i < body / 16; i += nt) __builtin_nontemporal_store(vec{0, 0, 0, 0}, at + i);
    else
      for (long long i = tid; i < body / 16; i += nt) at[i] = vec{0, 0, 0, 0};
    for (long long i = head + body + 2 * tid; i < n; i += 2 * nt) *reinterpret_cast<short*>(p + i) = 0;
  }
}

__global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(SortIn in, int shift, int tiles, int* hist, Zeros z) {
  if ((int)blockIdx.x >= tiles) return write_zeros(z, blockIdx.x - tiles, gridDim.x - tiles);
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

// Sum over the bins before the thread's (thread b < 512: bin b's value; all threads call).
__device__ inline int sum_before(int v) {
  __shared__ int wave_sum[BINS / 64];
  const int tid = threadIdx.x, lane = tid & 63;
  int incl = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int o = __shfl_up(incl, off, 64);
    if (lane >= off) incl += o;
  }
  __syncthreads();
  if (lane == 63 && tid < BINS) wave_sum[tid >> 6] = incl;
  __syncthreads();
  for (int w = 0; w < BINS / 64; ++w) incl += w < tid >> 6 ? wave_sum[w] : 0;
  return incl - v;
}

// hist[tile][bin]: counts -> the tiles' sums before it; row `tiles`: the whole.  A thread a bin.
__global__ __launch_bounds__(64) void sort_add_kernel(int* hist, int tiles) {
  const int b = blockIdx.x * 64 + threadIdx.x;
  int sum = 0;
  for (int t = 0; t < tiles; t += 8) {
    int c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = t + i < tiles ? hist[(size_t)(t + i) * BINS + b] : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (t + i < tiles) hist[(size_t)(t + i) * BINS + b] = sum;
      sum += c[i];
    }
  }
  hist[(size_t)tiles * BINS + b] = sum;
}

struct SortShared {
  int count[SORT_WAVES][BINS];
};
struct TileKeys {
  int key[SORT_STEPS], rank[SORT_STEPS];       // -1: none
  __device__ static long long place(int s) { return (threadIdx.x >> 6) * (64 * SORT_STEPS) + 64 * s + (threadIdx.x & 63); }      // in the tile
  __device__ void load(const SortIn& in, int tile) {
#pragma unroll
    for (int s = 0; s < SORT_STEPS; ++s) {
      const long long i = (long long)tile * SORT_TILE + place(s);
      key[s] = i < in.n ? in.key((int)i) : -1;
    }
  }
  // Ranks within the wavefront's keys of the same digit; its counts are left in sh.count.
  __device__ void count(SortShared& sh, int shift) {
    const int tid = threadIdx.x, lane = tid & 63;
    for (int i = tid; i < SORT_WAVES * BINS; i += SORT_THREADS) sh.count[0][i] = 0;
    __syncthreads();
    volatile int* mine = sh.count[tid >> 6];
#pragma unroll
    for (int s = 0; s < SORT_STEPS; ++s) {
      const int d = (key[s] >> shift) & (BINS - 1);
      unsigned long long same = __ballot(key[s] >= 0);
#pragma unroll
      for (int b = 0; b < BITS; ++b) {
        const unsigned long long has = __ballot((d >> b) & 1);
        same &= (d >> b) & 1 ? has : ~has;
      }
      const int before = mine[d], below = __popcll(same & ((1ull << lane) - 1));
      __builtin_amdgcn_wave_barrier();
      rank[s] = before + below;
      if (key[s] >= 0 && below == 0) mine[d] = before + __popcll(same);
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
  }
  // The tile's keys of the thread's bin.
  __device__ static int total(const SortShared& sh) {
    int sum = 0;
#pragma unroll
    for (int w = 0; w < SORT_WAVES; ++w) sum += sh.count[w][threadIdx.x];
    return sum;
  }
  // first: where the tile's first key of the thread's bin goes (threads below 512) -> ranks become places
  __device__ void place_from(SortShared& sh, int shift, int first) {
    if (threadIdx.x < BINS) {
#pragma unroll
      for (int w = 0; w < SORT_WAVES; ++w) {
        const int c = sh.count[w][threadIdx.x];
        sh.count[w][threadIdx.x] = first;
        first += c;
      }
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < SORT_STEPS; ++s)
      if (key[s] >= 0) rank[s] += sh.count[threadIdx.x >> 6][(key[s] >> shift) & (BINS - 1)];
  }
};
// Of the thread's bin: all keys, and those of the tiles before.
__device__ inline void tiles_sums(const int* hist, int tile, int tiles, int& all, int& before) {
  const int b = threadIdx.x;
  all = before = 0;
  if (b >= BINS) return;
  if (tiles > ADD_TILES) {
    before = hist[(size_t)tile * BINS + b];
    all = hist[(size_t)tiles * BINS + b];
    return;
  }
  for (int t = 0; t < tiles; t += 8) {
    int c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = t + i < tiles ? hist[(size_t)(t + i) * BINS + b] : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      all += c[i];
      before += t + i < tile ? c[i] : 0;
    }
  }
}

__global__ __launch_bounds__(SORT_THREADS) void sort_move_kernel(SortIn in, int shift, int tiles, const int* hist, int* keys, int* rows, Zeros z) {
  if ((int)blockIdx.x >= tiles) return write_zeros(z, blockIdx.x - tiles, gridDim.x - tiles);
  __shared__ SortShared sh;
  const int tile = blockIdx.x;
  TileKeys t;
  t.load(in, tile);
  int all, before;
  tiles_sums(hist, tile, tiles, all, before);
  t.count(sh, shift);
  t.place_from(sh, shift, sum_before(all) + before);
#pragma unroll
  for (int s = 0; s < SORT_STEPS; ++s)
    if (t.key[s] >= 0) {
      keys[t.rank[s]] = t.key[s];
      rows[t.rank[s]] = in.row((int)((long long)tile * SORT_TILE + t.place(s)));
    }
}

// Up to one tile, all passes.
__global__ __launch_bounds__(SORT_THREADS) void sort_tile_kernel(SortIn in, int* keys, int* rows, Zeros z) {
  if (blockIdx.x > 0) return write_zeros(z, blockIdx.x - 1, gridDim.x - 1);
  __shared__ SortShared sh;
  __shared__ int key_of[SORT_TILE], row_of[SORT_TILE];
  TileKeys t;
  t.load(in, 0);
  int row[SORT_STEPS];
#pragma unroll
  for (int s = 0; s < SORT_STEPS; ++s) row[s] = (int)t.place(s);
  for (int shift = 0, end = sort_passes(in.limit) * BITS; shift < end; shift += BITS) {
    t.count(sh, shift);
    const int tid = threadIdx.x;
    t.place_from(sh, shift, sum_before(tid < BINS ? t.total(sh) : 0));
#pragma unroll
    for (int s = 0; s < SORT_STEPS; ++s)
      if (t.key[s] >= 0) { key_of[t.rank[s]] = t.key[s]; row_of[t.rank[s]] = row[s]; }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < SORT_STEPS; ++s)
      if (t.place(s) < in.n) { t.key[s] = key_of[t.place(s)]; row[s] = row_of[t.place(s)]; }
    __syncthreads();
  }
#pragma unroll
  for (int s = 0; s < SORT_STEPS; ++s)
    if (t.place(s) < in.n) { keys[t.place(s)] = t.key[s]; rows[t.place(s)] = row[s]; }
}

// Experts: one pass places them.  Expert e's rows begin at a multiple of `align`; what lies behind its last one and behind the last expert's is no row.
__global__ __launch_bounds__(SORT_THREADS) void expert_place_kernel(SortIn in, int tiles, const int* hist, ExpertSort a) {
  __shared__ SortShared sh;
  __shared__ int end_of[BINS + 1], first_of[BINS + 1];
  const int tid = threadIdx.x, tile = blockIdx.x, n_experts = in.limit;
  TileKeys t;
  t.load(in, tile);
  int all, before;
  if (hist != nullptr) tiles_sums(hist, tile, tiles, all, before);
  t.count(sh, 0);
  if (hist == nullptr) {
    all = tid < BINS ? t.total(sh) : 0;
    before = 0;
  }
  const int room = tid < n_experts ? (all + a.align - 1) / a.align * a.align : 0, first = sum_before(room);
  if (tid < BINS) {
    first_of[tid] = first;
    end_of[tid] = first + (tid < n_experts ? all : 0);
    if (tile == 0) {
      if (tid <= n_experts) a.starts[tid] = first;
      if (a.counts != nullptr && tid < n_experts) a.counts[tid] = all;
    }
  }
  t.place_from(sh, 0, first + before);
#pragma unroll
  for (int s = 0; s < SORT_STEPS; ++s)
    if (t.key[s] >= 0) {
      const int i = (int)((long long)tile * SORT_TILE + t.place(s));
      const bool there = t.key[s] < n_experts;
      a.position[i] = there ? t.rank[s] : -1;
      if (there) a.source[t.rank[s]] = a.per_row == 1 ? i : i / a.per_row;
    }
  // (n_experts is at most 511: entry n_experts begins where the last one's room ends)
  // a wavefront fills the room behind an expert's last row, all threads what lies behind the last expert's
  const int lane = tid & 63;
  for (int e = tile * SORT_WAVES + (tid >> 6); e < n_experts; e += gridDim.x * SORT_WAVES)
    for (long long p = end_of[e] + lane; p < first_of[e + 1]; p += 64) a.source[p] = -1;      // (the last rows may end within 64 of 2^31)
  for (long long p = end_of[n_experts] + (long long)tile * SORT_THREADS + tid; p < a.n_packed; p += (long long)gridDim.x * SORT_THREADS) a.source[p] = -1;
  for (int g = tile * SORT_THREADS + tid; g < a.n_groups; g += gridDim.x * SORT_THREADS) {
    int lo = 0, hi = n_experts;                              // the last expert that begins at the group's first row or before
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (first_of[mid] <= g * a.align) lo = mid;
      else hi = mid - 1;
    }
    a.groups[g] = lo < n_experts ? lo : -1;
  }
}

int blocks_of(long long n, int per) { return (int)((n + per - 1) / per); }

// ---------------------------------------------------------------------------
// Rows as vectors of V elements, 16 bytes of the wider type, at any address of an element (the hardware takes 16-byte accesses there; rows of single elements took
// 2 to 4 times as long); a row's last vector may have fewer, n (TAIL: rows where it has).
// ---------------------------------------------------------------------------
template <typename T, int V>
struct Raw {
  static constexpr int PARTS = V * sizeof(T) > 16 ? 2 : 1, N = V / PARTS;
  typedef T vec __attribute__((ext_vector_type(N)));
  typedef vec at_element __attribute__((aligned(sizeof(T))));
  vec v[PARTS];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < PARTS; ++i) v[i] = vec{};
  }
  template <bool STREAM = false>
  __device__ __forceinline__ void load(const T* p, int n = V) {
    if (n == V) {
#pragma unroll
      for (int i = 0; i < PARTS; ++i) {
        const at_element* q = reinterpret_cast<const at_element*>(p + i * N);
        v[i] = STREAM ? __builtin_nontemporal_load(q) : *q;
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i / N][i % N] = i < n ? p[i] : (T)0.f;
    }
  }
  template <bool STREAM = false>
  __device__ __forceinline__ void store(T* p, int n = V) const {
    if (n == V) {
#pragma unroll
      for (int i = 0; i < PARTS; ++i) {
        if (STREAM) __builtin_nontemporal_store(v[i], reinterpret_cast<at_element*>(p + i * N));
        else *reinterpret_cast<at_element*>(p + i * N) = v[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i < n) p[i] = v[i / N][i % N];
    }
  }
  __device__ __forceinline__ float operator[](int i) const { return (float)v[i / N][i % N]; }
};
template <typename T, int V, bool STREAM = false>
__device__ inline void load(float (&x)[V], const T* p, int n) {
  Raw<T, V> r;
  r.template load<STREAM>(p, n);
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = r[i];
}
template <typename T, int V, bool STREAM = false>
__device__ inline void store(T* p, const float (&x)[V], int n) {
  Raw<T, V> r;
#pragma unroll
  for (int i = 0; i < V; ++i) r.v[i / r.N][i % r.N] = (T)x[i];
  r.template store<STREAM>(p, n);
}
template <int V>
__device__ inline void zero(float (&x)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = 0.f;
}
// Elements of vector `col` of a row of d.
template <int V, bool TAIL>
__device__ inline int elements(int d, int col) { return TAIL ? min(V, d - col * V) : V; }

template <typename T> constexpr int wide() { return 16 / (int)sizeof(T); }
template <typename A, typename B> constexpr int wide() { return 16 / (int)std::max(sizeof(A), sizeof(B)); }

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
template <typename TT, typename TO, int V, bool TAIL, bool STREAM>
__global__ __launch_bounds__(ROWS_THREADS) void embed_kernel(Embed a, int per_row) {
  FOR_VECTORS(a.n_rows, per_row) {
    const long long tok = index_at(a.tokens, a.i64, at.row);
    const int n = elements<V, TAIL>(a.d, at.col);
    float x[V];
    zero(x);
    if (tok >= 0 && tok < a.vocab) load<TT, V>(x, static_cast<const TT*>(a.table) + tok * a.table_row + (long long)at.col * V, n);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = tok < a.vocab ? x[i] * a.scale : NAN;
    if (tok < 0) zero(x);
    store<TO, V, STREAM>(static_cast<TO*>(a.out) + at.row * a.out_row + (long long)at.col * V, x, n);
  }
}

template <typename TT, typename TO>
hipError_t embed(hipStream_t st, const Embed& a) {
  constexpr int V = wide<TT, TO>();
  const int per_row = blocks_of(a.d, V);
  // (streaming stores here and of the gradient's zeros: 32768 rows of 2560 and a table of 151936, lookup and gradient 277 -> 264 us; either alone nothing; in the sums too 257)
  const bool stream = streams((long long)a.n_rows * a.d * (long long)sizeof(TO)), whole = a.d % V == 0;
  const auto kernel = stream ? (whole ? embed_kernel<TT, TO, V, false, true> : embed_kernel<TT, TO, V, true, true>) : (whole ? embed_kernel<TT, TO, V, false, false> : embed_kernel<TT, TO, V, true, false>);
  return enqueue(kernel, vector_grid(a.n_rows, per_row), dim3(ROWS_THREADS), st, a, per_row);
}

// ---------------------------------------------------------------------------
// The embedding's gradient.  Rows sorted by token; the sorted order in blocks of 32 rows, a wavefront to a block and 64 vectors of the row: it adds a token's rows in order, writes
// the sums of tokens that lie in the block, and leaves those of the first and the last token, where they go on outside, as partial sums.  A second launch adds the partial
// sums of a token in order.  So the work is even whatever the tokens' shares are (a thread for each vector of the table was 326 us for 32768 rows of 2560,
// frequent tokens its tail; this 54 into a table that is there, 5.3 TB/s), and the table's zeros are written while the tokens are sorted.
// ---------------------------------------------------------------------------
constexpr int PIECE = 32;

struct Sorted {
  const int *keys, *rows;
  float* partial;                      // [blocks][2][d]: of the token that goes on from the block before; of the one that begins and goes on behind
};

template <typename TT, int V, bool STREAM = false>
__device__ inline void put_sum(const EmbedGrad& a, int token, int col, const float (&sum)[V], int n) {
  TT* to = static_cast<TT*>(a.grad_table) + (long long)token * a.table_row + (long long)col * V;
  float x[V];
  zero(x);
  if (a.accumulate) load<TT, V>(x, to, n);
#pragma unroll
  for (int j = 0; j < V; ++j) x[j] += a.scale * sum[j];
  store<TT, V, STREAM>(to, x, n);
}

template <typename TO, typename TT, int V, bool TAIL, bool STREAM>
__global__ __launch_bounds__(256) void embed_sums_kernel(EmbedGrad a, Sorted s, int per_row, int chunks) {
  const int lane = threadIdx.x & 63;
  for (long long id = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);; id += (long long)gridDim.x * 4) {
    const int block = (int)(id / chunks), col = (int)(id - (long long)block * chunks) * 64 + lane;
    const long long p0 = (long long)block * PIECE;
    if (p0 >= a.n_rows) return;
    // lanes 0..31: the block's tokens and rows; 32: the token behind it; 33: the one before
    const long long at = lane <= PIECE ? p0 + lane : p0 - 1;
    const int key = lane <= PIECE + 1 && at >= 0 && at < a.n_rows ? s.keys[at] : -1, row = lane < PIECE && at < a.n_rows ? s.rows[at] : 0;
    const int n = __popcll(__ballot(lane < PIECE && key >= 0 && key < a.vocab));
    const TO* g = static_cast<const TO*>(a.grad_out) + (long long)col * V;
    const bool mine = col < per_row;
    const int here = elements<V, TAIL>(a.d, col);
    float sum[V];
    zero(sum);
    int last = __builtin_amdgcn_readlane(key, PIECE + 1);      // the token of the row before
    bool inside = false;                                       // the sum's token begins in the block
    constexpr int U = 8;
    for (int i0 = 0; i0 < n; i0 += U) {
      Raw<TO, V> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        x[u].clear();
        if (i0 + u < n && mine) x[u].template load<STREAM>(g + (long long)__builtin_amdgcn_readlane(row, i0 + u) * a.out_row, here);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u;
        if (i >= n) continue;
        const int token = __builtin_amdgcn_readlane(key, i);
        if (token != last) {
          inside = true;
          zero(sum);
          last = token;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += x[u][j];
        if (token == __builtin_amdgcn_readlane(key, i + 1)) {  // it goes on, in the block or behind it
          if (i == PIECE - 1 && mine) store<float, V>(s.partial + ((size_t)block * 2 + (inside ? 1 : 0)) * a.d + (size_t)col * V, sum, here);
        } else if (mine) {
          if (inside) put_sum<TT, V, STREAM>(a, token, col, sum, here);
          else store<float, V>(s.partial + (size_t)block * 2 * a.d + (size_t)col * V, sum, here);
        }
      }
    }
  }
}

// A token that begins in the block and goes on behind it: four wavefronts a quarter of its partial sums each, then theirs in order.
template <typename TT, int V, bool TAIL>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedGrad a, Sorted s, int per_row, int chunks) {
  __shared__ float part[4][64 * V];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (long long id = blockIdx.x;; id += gridDim.x) {
    const int block = (int)(id / chunks), col = (int)(id - (long long)block * chunks) * 64 + lane;
    const long long p0 = (long long)block * PIECE;
    if (p0 + PIECE >= a.n_rows) return;
    const int token = s.keys[p0 + PIECE - 1];
    if (token >= a.vocab || s.keys[p0 + PIECE] != token) continue;
    if (s.keys[p0] == token && p0 > 0 && s.keys[p0 - 1] == token) continue;
    int n = 1;                                                 // blocks that hold rows of it: 64 of the following ones' first tokens at a time
    for (unsigned long long more = ~0ull; more == ~0ull; n += __popcll(more)) {
      const long long at = (block + (long long)n + lane) * PIECE;
      more = __ballot(at < a.n_rows && s.keys[at] == token);
    }
    const int from = (int)((long long)n * wave / 4), to = (int)((long long)n * (wave + 1) / 4);
    const bool mine = col < per_row;
    const int here = elements<V, TAIL>(a.d, col);
    float sum[V];
    zero(sum);
    constexpr int U = 8;
    for (int i0 = from; i0 < to; i0 += U) {
      float x[U][V];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        zero(x[u]);
        if (i0 + u < to && mine) load<float, V>(x[u], s.partial + (((size_t)block + i0 + u) * 2 + (i0 + u == 0 ? 1 : 0)) * a.d + (size_t)col * V, here);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += x[u][j];
    }
    __syncthreads();                                           // (the last round's are read)
#pragma unroll
    for (int j = 0; j < V; ++j) part[wave][j * 64 + lane] = sum[j];
    __syncthreads();
    if (wave > 0 || !mine) continue;
#pragma unroll
    for (int w = 1; w < 4; ++w)
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] += part[w][j * 64 + lane];
    put_sum<TT, V>(a, token, col, sum, here);
  }
}

// The workspace: counts, two sets of keys and rows, partial sums, each 16-byte aligned.
struct GradSpace {
  int *hist, *keys[2], *rows[2];
  float* partial;
  size_t bytes;
  explicit GradSpace(const EmbedGrad& a) {
    char* p = static_cast<char*>(a.ws);
    size_t at = 0;
    auto take = [&](size_t n) { char* q = p + at; at += (n + 15) / 16 * 16; return q; };
    const size_t n = a.n_rows;
    hist = (int*)take(n > 0 ? ((size_t)blocks_of(n, SORT_TILE) + 1) * BINS * 4 : 0);
    for (int i = 0; i < 2; ++i) { keys[i] = (int*)take(n * 4); rows[i] = (int*)take(n * 4); }
    partial = (float*)take((size_t)blocks_of(n, PIECE) * 2 * a.d * 4);
    bytes = at;
  }
};

template <typename TO, typename TT>
hipError_t embed_grad(hipStream_t st, const EmbedGrad& a) {
  const GradSpace w(a);
  const int tiles = blocks_of(a.n_rows, SORT_TILE), passes = sort_passes(a.vocab);
  const int launches = tiles > 1 ? 2 * passes : 1;
  // the table's zeros, in as many shares as there are launches
  const long long row = (long long)a.d * sizeof(TT), stride = a.table_row * (long long)sizeof(TT);
  Zeros z{static_cast<char*>(a.grad_table), streams(row * a.vocab), row, stride, -1, 0, 0};
  long long units = a.vocab;
  if (a.table_row == a.d || a.vocab == 1) {
    z.unit = z.stride = 64 << 10;
    z.total = row * a.vocab;
    units = (z.total + z.unit - 1) / z.unit;
  }
  if (a.accumulate) units = 0;
  int share = 0;
  auto grid = [&](int groups) {
    z.first = units * share / launches;
    z.end = units * ++share / launches;
    return dim3((unsigned)(groups + std::min<long long>(z.end - z.first, 2048)));
  };
  SortIn in{a.tokens, a.i64, a.vocab, a.n_rows, nullptr, nullptr};
  hipError_t e = hipSuccess;
  auto run = [&](auto... args) { if (e == hipSuccess) e = enqueue(args...); };
  if (tiles <= 1) {
    run(sort_tile_kernel, grid(1), dim3(SORT_THREADS), st, in, w.keys[0], w.rows[0], z);
    in.keys = w.keys[0];
    in.rows = w.rows[0];
  }
  for (int pass = 0; tiles > 1 && pass < passes; ++pass) {
    run(sort_count_kernel, grid(tiles), dim3(SORT_THREADS), st, in, pass * BITS, tiles, w.hist, z);
    if (tiles > ADD_TILES) run(sort_add_kernel, dim3(BINS / 64), dim3(64), st, w.hist, tiles);
    run(sort_move_kernel, grid(tiles), dim3(SORT_THREADS), st, in, pass * BITS, tiles, (const int*)w.hist, w.keys[pass & 1], w.rows[pass & 1], z);
    in.keys = w.keys[pass & 1];
    in.rows = w.rows[pass & 1];
  }
  if (a.n_rows == 0) return e;
  const Sorted s{in.keys, in.rows, w.partial};
  constexpr int V = wide<TO, TT>();
  const bool whole = a.d % V == 0;
  const int per_row = blocks_of(a.d, V), chunks = blocks_of(per_row, 64), blocks = blocks_of(a.n_rows, PIECE);
  const long long groups = (long long)blocks * chunks;
  auto most = [](long long n) { return dim3((unsigned)std::min<long long>(n, 1 << 22)); };
  const auto sums = streams((long long)a.n_rows * a.d * (long long)sizeof(TO)) ? (whole ? embed_sums_kernel<TO, TT, V, false, true> : embed_sums_kernel<TO, TT, V, true, true>)
                                                                              : (whole ? embed_sums_kernel<TO, TT, V, false, false> : embed_sums_kernel<TO, TT, V, true, false>);
  run(sums, most((groups + 3) / 4), dim3(256), st, a, s, per_row, chunks);
  if (a.n_rows > PIECE) run(whole ? embed_join_kernel<TT, V, false> : embed_join_kernel<TT, V, true>, most(groups), dim3(256), st, a, s, per_row, chunks);
  return e;
}

// ---------------------------------------------------------------------------
// Tokens' rows in their experts' batches.
// ---------------------------------------------------------------------------
// Zeros in the packed rows of no assignment, a wavefront 16 of them, on the workgroups behind the tokens'.
template <typename T, int V, bool TAIL, bool STREAM>
__device__ inline void write_zero_rows(const ExpertRows& a, T* out, long long row, int per_row, int row_groups) {
  const long long n = (long long)a.n_rows * a.k;
  const int lane = threadIdx.x & 63;
  for (long long p0 = ((long long)(blockIdx.x - row_groups) * 4 + (threadIdx.x >> 6)) * 16; p0 < a.n_packed; p0 += (long long)(gridDim.x - row_groups) * 64) {
    const int from = lane < 16 && p0 + lane < a.n_packed ? a.source[p0 + lane] : 0;
    float x[V];
    zero(x);
    for (unsigned long long none = __ballot(lane < 16 && p0 + lane < a.n_packed && (from < 0 || from >= n)); none != 0; none &= none - 1)
      for (int col = lane; col < per_row; col += 64) store<T, V, STREAM>(out + (p0 + __ffsll((long long)none) - 1) * row + (long long)col * V, x, elements<V, TAIL>(a.d, col));
  }
}

// The tokens' rows, each read once and stored at its k places.
template <typename T, int V, bool TAIL, bool STREAM>
__global__ __launch_bounds__(ROWS_THREADS) void expert_gather_kernel(ExpertRows a, int per_row, int row_groups) {
  T* out = static_cast<T*>(a.out);
  if ((int)blockIdx.x >= row_groups) return write_zero_rows<T, V, TAIL, STREAM>(a, out, a.packed_row, per_row, row_groups);
  for (long long first = (long long)blockIdx.x * ROWS_THREADS; first < (long long)a.n_rows * per_row; first += (long long)row_groups * ROWS_THREADS) {
    const At at = vector_at(first, threadIdx.x, per_row);
    if (at.row >= a.n_rows) continue;
    const int n = elements<V, TAIL>(a.d, at.col);
    Raw<T, V> x;
    x.load(static_cast<const T*>(a.rows) + at.row * a.row + (long long)at.col * V, n);
    const int* position = a.position + at.row * a.k;
    for (int j0 = 0; j0 < a.k; j0 += 8) {
      int to[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) to[j] = j0 + j < a.k ? position[j0 + j] : -1;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (to[j] >= 0 && to[j] < a.n_packed) x.template store<STREAM>(out + (long long)to[j] * a.packed_row + (long long)at.col * V, n);
    }
  }
}

// Eight of a token's packed rows in flight, added in order.
template <typename T, int V, bool TAIL, bool STREAM>
__global__ __launch_bounds__(ROWS_THREADS) void expert_combine_kernel(ExpertRows a, int per_row) {
  FOR_VECTORS(a.n_rows, per_row) {
    const int n = elements<V, TAIL>(a.d, at.col);
    float sum[V];
    zero(sum);
    const int* position = a.position + at.row * a.k;
    const float* weights = a.weights + at.row * a.k;
    const T* packed = static_cast<const T*>(a.packed) + (long long)at.col * V;
    for (int j0 = 0; j0 < a.k; j0 += 8) {
      Raw<T, V> x[8];
      float w[8];
      int from[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        from[j] = j0 + j < a.k ? position[j0 + j] : -1;
        w[j] = a.weights != nullptr && j0 + j < a.k ? weights[j0 + j] : 1.f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (from[j] >= 0 && from[j] < a.n_packed) x[j].template load<STREAM>(packed + (long long)from[j] * a.packed_row, n);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (from[j] >= 0 && from[j] < a.n_packed) {
#pragma unroll
          for (int i = 0; i < V; ++i) sum[i] = fmaf(w[j], x[j][i], sum[i]);
        }
    }
    store<T, V, STREAM>(static_cast<T*>(a.out) + at.row * a.row + (long long)at.col * V, sum, n);
  }
}

// A token's rows again: its gradient is read once and stored at its k places, eight packed rows in flight for the weights' gradients.  WAVES wavefronts a token.  Bound by HBM:
// 16384 tokens of 2048 in bf16 with 8 experts each 185 us (5.8 TB/s); by packed rows, which read a token's gradient k times, 208.
template <typename T, int V, bool TAIL, bool STREAM, int WAVES>
__global__ __launch_bounds__(ROWS_THREADS) void expert_combine_grad_kernel(ExpertRows a, int per_row, int row_groups) {
  T* out = static_cast<T*>(a.grad_packed);
  if ((int)blockIdx.x >= row_groups) return write_zero_rows<T, V, TAIL, STREAM>(a, out, a.grad_row, per_row, row_groups);
  constexpr int ROWS = ROWS_THREADS / 64 / WAVES;            // of a workgroup at a time
  __shared__ float part[4][8];
  const int tid = threadIdx.x & (64 * WAVES - 1), wave = threadIdx.x >> 6;
  for (long long r0 = (long long)blockIdx.x * ROWS; r0 < a.n_rows; r0 += (long long)row_groups * ROWS) {
    const long long r = r0 + wave / WAVES;
    const bool row = r < a.n_rows;
    for (int j0 = 0; j0 < a.k; j0 += 8) {
      int at[8];
      float w[8], dot[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        at[j] = row && j0 + j < a.k ? a.position[r * a.k + j0 + j] : -1;
        if (at[j] >= a.n_packed) at[j] = -1;
        w[j] = a.weights != nullptr && at[j] >= 0 ? a.weights[r * a.k + j0 + j] : 1.f;
        dot[j] = 0.f;
      }
      for (int col = tid; row && col < per_row; col += 64 * WAVES) {
        const int n = elements<V, TAIL>(a.d, col);
        float g[V];
        load<T, V>(g, static_cast<const T*>(a.rows) + r * a.row + (long long)col * V, n);
        if (a.grad_weights) {
          Raw<T, V> y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (at[j] >= 0) y[j].template load<STREAM>(static_cast<const T*>(a.packed) + at[j] * a.packed_row + (long long)col * V, n);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (at[j] >= 0) {
#pragma unroll
              for (int i = 0; i < V; ++i) dot[j] = fmaf(g[i], y[j][i], dot[j]);
            }
        }
        if (out != nullptr) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (at[j] >= 0) {
              float x[V];
#pragma unroll
              for (int i = 0; i < V; ++i) x[i] = w[j] * g[i];
              store<T, V, STREAM>(out + at[j] * a.grad_row + (long long)col * V, x, n);
            }
        }
      }
      if (!a.grad_weights) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) dot[j] = wave_sum_f32(dot[j]);
      if (WAVES > 1) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
          for (int j = 0; j < 8; ++j) part[wave][j] = dot[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) dot[j] = (part[0][j] + part[1][j]) + (part[2][j] + part[3][j]);
      }
      if (row && tid == 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j0 + j < a.k) a.grad_weights[r * a.k + j0 + j] = at[j] >= 0 ? dot[j] : 0.f;
      }
    }
  }
}

// The packed rows are streamed, read or written, where they are many (13900 tokens of 2048 in bf16 with 8 experts each, gathered and summed, 249 -> 204 us, 16384 with all gradients
// 583 -> 525; only the gradients' 562, only the stores 548).
template <typename T>
bool streamed(const ExpertRows& a) { return streams((long long)a.n_packed * a.d * (long long)sizeof(T)); }
#define EXPERT_KERNEL(name, T, V) \
  (streamed<T>(a) ? (a.d % V == 0 ? name<T, V, false, true> : name<T, V, true, true>) : (a.d % V == 0 ? name<T, V, false, false> : name<T, V, true, false>))

template <typename T>
hipError_t expert_gather(hipStream_t st, const ExpertRows& a) {
  constexpr int V = wide<T>();
  const int per_row = blocks_of(a.d, V), row_groups = a.n_rows > 0 ? (int)vector_grid(a.n_rows, per_row).x : 0;
  const dim3 grid(row_groups + std::min(blocks_of(a.n_packed, 64), 1 << 20));
  return enqueue(EXPERT_KERNEL(expert_gather_kernel, T, V), grid, dim3(ROWS_THREADS), st, a, per_row, row_groups);
}
template <typename T>
hipError_t expert_combine(hipStream_t st, const ExpertRows& a) {
  constexpr int V = wide<T>();
  const int per_row = blocks_of(a.d, V);
  return enqueue(EXPERT_KERNEL(expert_combine_kernel, T, V), vector_grid(a.n_rows, per_row), dim3(ROWS_THREADS), st, a, per_row);
}
template <typename T>
hipError_t expert_combine_grad(hipStream_t st, const ExpertRows& a) {
  constexpr int V = wide<T>();
  const int per_row = blocks_of(a.d, V), waves = per_row > 64 ? 4 : 1;
  const int row_groups = std::min(blocks_of(a.n_rows, 4 / waves), 1 << 22), zeros = a.grad_packed ? std::min(blocks_of(a.n_packed, 64), 1 << 20) : 0;
  auto run = [&](auto whole, auto tail, auto whole_streamed, auto tail_streamed) {
    return enqueue(streamed<T>(a) ? (a.d % V == 0 ? whole_streamed : tail_streamed) : (a.d % V == 0 ? whole : tail), dim3(row_groups + zeros), dim3(ROWS_THREADS), st, a, per_row, row_groups);
  };
#define KERNEL(TAIL, STREAM) expert_combine_grad_kernel<T, V, TAIL, STREAM, W>
  if (waves == 4) {
    constexpr int W = 4;
    return run(KERNEL(false, false), KERNEL(true, false), KERNEL(false, true), KERNEL(true, true));
  }
  constexpr int W = 1;
  return run(KERNEL(false, false), KERNEL(true, false), KERNEL(false, true), KERNEL(true, true));
#undef KERNEL
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

// (one tile needs no counts of the others)
size_t expert_sort_workspace(const ExpertSort& a) { return a.n > SORT_TILE ? ((size_t)blocks_of(a.n, SORT_TILE) + 1) * BINS * 4 : 0; }

hipError_t launch_expert_sort(hipStream_t st, const ExpertSort& a) {
  const int tiles = std::max(1, blocks_of(a.n, SORT_TILE));
  const SortIn in{a.ids, a.i64, a.n_experts, a.n, nullptr, nullptr};
  int* hist = tiles > 1 ? static_cast<int*>(a.ws) : nullptr;
  hipError_t e = hipSuccess;
  if (tiles > 1) e = enqueue(sort_count_kernel, dim3(tiles), dim3(SORT_THREADS), st, in, 0, tiles, hist, Zeros{});
  if (tiles > ADD_TILES && e == hipSuccess) e = enqueue(sort_add_kernel, dim3(BINS / 64), dim3(64), st, hist, tiles);
  return e == hipSuccess ? enqueue(expert_place_kernel, dim3(tiles), dim3(SORT_THREADS), st, in, tiles, (const int*)hist, a) : e;
}

hipError_t launch_expert_gather(hipStream_t st, const ExpertRows& a) { return a.f32 ? expert_gather<float>(st, a) : expert_gather<bf16_t>(st, a); }
hipError_t launch_expert_combine(hipStream_t st, const ExpertRows& a) { return a.f32 ? expert_combine<float>(st, a) : expert_combine<bf16_t>(st, a); }
hipError_t launch_expert_combine_grad(hipStream_t st, const ExpertRows& a) { return a.f32 ? expert_combine_grad<float>(st, a) : expert_combine_grad<bf16_t>(st, a); }

}  // namespace april
