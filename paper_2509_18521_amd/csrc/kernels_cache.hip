// Kernels of the 4-bit KV cache (gfx950): tables from request lengths, the store, the attention that reads it.
#include <algorithm>
#include <cmath>
#include <tuple>

#include "cache.h"
#include <float.h>

namespace april {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <typename... P, typename... A>
hipError_t launch(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t st, A... args) {
  std::tuple<P...> held{static_cast<P>(args)...};
  void* ptrs[sizeof...(P)];
  std::apply([&](auto&... x) { int i = 0; ((ptrs[i++] = (void*)&x), ...); }, held);
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, ptrs, 0, st);
}

// ---------------------------------------------------------------------------
// Tables.  One workgroup: lengths -> exclusive sums over the sequences of pages given back, pages lacked and rows gained;
// then the status (nothing has been written yet), then the items of each kind, dealt to the threads flat: an item finds its sequence
// by a binary search in the sums.  Latency is all there is; but the many rows of prompts, and the pages that they open, are left to a second
// launch over the whole chip (the pages from the one workgroup: 19.5 and not 11.5 us for 384 prompts of up to 1999 tokens).
// ---------------------------------------------------------------------------
constexpr int EXT_THREADS = 1024;

// Exclusive sums of three values over the workgroup, and their totals; the three go through the same two barriers.
template <typename I>
__device__ void block_scan(I (&v)[3], I (*s_wave)[EXT_THREADS / 64], I (&total)[3]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  I x[3] = {v[0], v[1], v[2]};
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    I y[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) y[k] = __shfl_up(x[k], d, 64);
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (lane >= d) x[k] += y[k];
  }
  __syncthreads();                                   // (the last call's sums have been read)
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (lane == 63) s_wave[k][wave] = x[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    I base = 0;
    total[k] = 0;
#pragma unroll
    for (int w = 0; w < EXT_THREADS / 64; ++w) {
      const I s = s_wave[k][w];
      if (w < wave) base += s;
      total[k] += s;
    }
    v[k] = base + x[k] - v[k];
  }
}

// largest i in 0..n-1 with s[i] <= k (s: exclusive sums, s[0] <= k)
template <typename P, typename K>
__device__ int find_in(P s, int n, K k) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s[mid] <= k) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ inline void put_row(const CacheExtend& a, int r, int page, int pos) {
  a.slot_map[r] = page < 0 ? -1 : (long long)page * CACHE_PAGE + (pos & (CACHE_PAGE - 1));
  a.positions[r] = page < 0 ? -1 : pos;
}

enum { EXT_PAGES, EXT_ROWS, EXT_SUMS };              // the pages that are taken; the rows' slots too; neither (cache_rows_kernel does both)
// I: int where no sum can pass 31 bits, else long long.
template <typename I>
__global__ __launch_bounds__(EXT_THREADS) void cache_extend_kernel(CacheExtend a, int what) {
  const bool rows = what == EXT_ROWS;
  enum { REL, LACK, ROW };                           // pages given back, pages lacked, rows gained
  __shared__ I s_wave[3][EXT_THREADS / 64], s_sum[3][EXT_THREADS];
  __shared__ int s_len[EXT_THREADS], s_flags;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n_chunks = (a.n_seqs + EXT_THREADS - 1) / EXT_THREADS;
  const int top = *a.free_top;
  const long long cap = min((long long)a.max_pages * CACHE_PAGE, (1ll << 31) - CACHE_PAGE);       // (rounded up to pages, still 31 bits)
  I sum[3], total[3];                                // this thread's sequence: sums before it in its chunk; the chunk's totals
  int len, add;
  bool bad = false;
  if (tid == 0) s_flags = 0;
  auto table_row = [&](int b) { return a.block_table + (size_t)(a.row_of != nullptr ? a.row_of[b] : b) * a.table_stride; };
  int last_page = 0;                                 // of this thread's sequence, where it is not full
  auto scan = [&](int chunk) {
    const int b = chunk * EXT_THREADS + tid;
    len = b < a.n_seqs && a.lens != nullptr ? a.lens[b] : 0;
    add = b < a.n_seqs ? a.new_lens[b] : 0;
    const bool off = len < 0 || len > cap || (add > 0 && (long long)len + add > cap);
    bad |= off;
    if (rows && !off && add > 0 && (len & (CACHE_PAGE - 1))) last_page = table_row(b)[len / CACHE_PAGE];
    const int held = off ? 0 : (len + CACHE_PAGE - 1) / CACHE_PAGE;
    const int want = off || add < 0 ? 0 : (int)(((long long)len + add + CACHE_PAGE - 1) / CACHE_PAGE);
    sum[REL] = !off && add < 0 ? held : 0;
    sum[LACK] = want > held ? want - held : 0;
    sum[ROW] = off || add < 0 ? 0 : add;
    block_scan<I>(sum, s_wave, total);
#pragma unroll
    for (int k = 0; k < 3; ++k) s_sum[k][tid] = sum[k];
    s_len[tid] = len;
    __syncthreads();
  };
  I all[3] = {0, 0, 0};
  for (int c = 0; c < n_chunks; ++c) {
    scan(c);
#pragma unroll
    for (int k = 0; k < 3; ++k) all[k] += total[k];
  }
  // Decode iterations: a thread sees to its sequence's few rows itself, without searches (192 sequences 6.1 and not 7.2 us).
  constexpr int FEW = 4;
  if (bad) atomicOr(&s_flags, 1);
  if (n_chunks > 1 || add > FEW) atomicOr(&s_flags, 2);
  __syncthreads();
  const long long have = (long long)top + all[REL];
  int status = 0;
  if ((s_flags & 1) || (a.row_of == nullptr && all[ROW] > a.n_rows) || top < 0 || have > a.n_pages) status = 2;
  else if (all[LACK] > have) status = 1;
  if (tid == 0) {
    *a.status = status;
    *a.free_top_out = status ? top : (int)(have - all[LACK]);
    if (a.q_start != nullptr) a.q_start[0] = 0;
  }
  I base = 0;
  if (status == 0 && all[REL] > 0) {                 // pages given back
    for (int c = 0; c < n_chunks; ++c) {
      if (n_chunks > 1) scan(c);
      const int n = min(EXT_THREADS, a.n_seqs - c * EXT_THREADS);
      for (I k = tid; k < total[REL]; k += EXT_THREADS) {
        const int s = find_in(s_sum[REL], n, k);
        a.free_pages[top + base + k] = table_row(c * EXT_THREADS + s)[k - s_sum[REL][s]];
      }
      base += total[REL];
      if (n_chunks > 1) __syncthreads();             // the sums are used up
    }
    __syncthreads();
  }
  base = 0;
  I row_base = 0;
  for (int c = 0; c < n_chunks; ++c) {               // lengths, first rows, pages taken, slots
    if (n_chunks > 1) scan(c);
    const int b = c * EXT_THREADS + tid, n = min(EXT_THREADS, a.n_seqs - c * EXT_THREADS);
    if (b < a.n_seqs) {
      const int now = status ? len : (add < 0 ? 0 : len + add);
      if (a.lens_out != nullptr) a.lens_out[b] = now;
      if (a.q_start != nullptr) a.q_start[b + 1] = status ? 0 : (int)(row_base + sum[ROW] + (add < 0 ? 0 : add));
      if (a.held_of != nullptr && status == 0) a.held_of[a.row_of[b]] = (now + CACHE_PAGE - 1) / CACHE_PAGE;
    }
    if (status == 0 && what != EXT_SUMS) {
      const int* taken = a.free_pages + (have - 1 - base);       // page k of the chunk: taken[-k]
      if (rows && !(s_flags & 2)) {
        if (add > 0) {
          const int held = (len + CACHE_PAGE - 1) / CACHE_PAGE;
          int page = 0;
          if (len + add > held * CACHE_PAGE) {
            page = taken[-(long long)sum[LACK]];
            table_row(b)[held] = page;
          }
#pragma unroll
          for (int i = 0; i < FEW; ++i)
            if (i < add) put_row(a, (int)sum[ROW] + i, (len + i) / CACHE_PAGE < held ? last_page : page, len + i);
        }
        break;                                       // (one chunk)
      }
      if (total[LACK] <= EXT_THREADS) {
        if (tid < total[LACK]) {
          const int s = find_in(s_sum[LACK], n, (I)tid);
          table_row(c * EXT_THREADS + s)[(s_len[s] + CACHE_PAGE - 1) / CACHE_PAGE + (int)(tid - s_sum[LACK][s])] = taken[-tid];
        }
      } else {                                       // prompts: a wavefront per sequence, no searches
        for (int s = wave; s < n; s += EXT_THREADS / 64) {
          const I first = s_sum[LACK][s], count = (s + 1 < n ? s_sum[LACK][s + 1] : total[LACK]) - first;
          if (count == 0) continue;
          int* to = table_row(c * EXT_THREADS + s) + (s_len[s] + CACHE_PAGE - 1) / CACHE_PAGE;
          for (I k = lane; k < count; k += 64) to[k] = taken[-(long long)(first + k)];
        }
      }
      if (rows)
        for (I k = tid; k < total[ROW]; k += EXT_THREADS) {
          // (a page taken just now comes from the stack: the table's entry is another thread's)
          const int s = find_in(s_sum[ROW], n, k), pos = s_len[s] + (int)(k - s_sum[ROW][s]), i = pos / CACHE_PAGE - (s_len[s] + CACHE_PAGE - 1) / CACHE_PAGE;
          put_row(a, (int)(row_base + k), i < 0 ? table_row(c * EXT_THREADS + s)[pos / CACHE_PAGE] : taken[-(long long)(s_sum[LACK][s] + i)], pos);
        }
    }
    base += total[LACK];
    row_base += total[ROW];
    if (n_chunks > 1) __syncthreads();
  }
  if (rows)
    for (int r = (status ? 0 : (int)all[ROW]) + tid; r < a.n_rows; r += EXT_THREADS) put_row(a, r, -1, 0);
}

// Many rows and the pages that they open, a thread each, from what the kernel above has left.  Rows that begin a page take the pages
// in their order: the k-th of them the k-th from the top.  k is counted within the workgroup by ballots, before it from the lengths.
__global__ __launch_bounds__(256) void cache_rows_kernel(CacheExtend a) {
  __shared__ int s_begin, s_sum[2][4], s_starts[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = blockIdx.x * 256 + tid, total = a.q_start[a.n_seqs];
  if ((int)blockIdx.x * 256 >= total) {
    if (r < a.n_rows) put_row(a, r, -1, 0);
    return;
  }
  auto pages = [](int tokens) { return (tokens + CACHE_PAGE - 1) / CACHE_PAGE; };
  const bool valid = r < total;
  const int b = find_in(a.q_start, a.n_seqs, valid ? r : total - 1), rows_end = a.q_start[b + 1], now = a.lens_out[b];
  const int pos = now - (rows_end - r), held = pages(now - (rows_end - a.q_start[b]));
  if (tid == 0) s_begin = b;
  __syncthreads();
  int sum[2] = {0, 0};                               // pages taken by the sequences before the first row's; by all
#pragma unroll 4
  for (int s = tid; s < a.n_seqs; s += 256) {
    const int n = a.lens_out[s], lack = pages(n) - pages(n - (a.q_start[s + 1] - a.q_start[s]));
    sum[0] += s < s_begin ? lack : 0;
    sum[1] += lack;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) { sum[0] += __shfl_xor(sum[0], d, 64); sum[1] += __shfl_xor(sum[1], d, 64); }
  const bool starts = valid && (pos & (CACHE_PAGE - 1)) == 0;
  const unsigned long long here = __ballot(starts);
  if (tid == 0) sum[0] += pages(pos) - held;         // (and by the first row's own, before it)
  if (lane == 0) { s_sum[0][wave] = sum[0]; s_sum[1][wave] = sum[1]; s_starts[wave] = __popcll(here); }
  __syncthreads();
  if (!valid) {
    if (r < a.n_rows) put_row(a, r, -1, 0);
    return;
  }
  int k = s_sum[0][0] + s_sum[0][1] + s_sum[0][2] + s_sum[0][3] + __popcll(here & (~0ull >> (63 - lane))) - 1;
  for (int w = 0; w < wave; ++w) k += s_starts[w];
  int* entry = a.block_table + (size_t)b * a.table_stride + pos / CACHE_PAGE;
  const int page = pos / CACHE_PAGE < held ? *entry : a.free_pages[*a.free_top_out + s_sum[1][0] + s_sum[1][1] + s_sum[1][2] + s_sum[1][3] - 1 - k];
  if (starts) *entry = page;
  put_row(a, r, page, pos);
}

}  // namespace

hipError_t launch_cache_extend(hipStream_t st, const CacheExtend& a) {
  // one launch up to 4 rows a thread: 1 sequence of 4000 new tokens 6.7 us, with the second launch 7.9; 200 of 1-35 10.1 and 10.4
  const bool rows = a.n_rows > 0 && a.n_rows <= 4 * EXT_THREADS;
  const bool small = (long long)a.n_seqs * a.max_pages * CACHE_PAGE < (1ll << 30);
  const int what = rows ? EXT_ROWS : a.n_rows > 0 ? EXT_SUMS : EXT_PAGES;
  hipError_t e = small ? launch(cache_extend_kernel<int>, dim3(1), dim3(EXT_THREADS), st, a, what)
                       : launch(cache_extend_kernel<long long>, dim3(1), dim3(EXT_THREADS), st, a, what);
  if (e == hipSuccess && what == EXT_SUMS) e = launch(cache_rows_kernel, dim3(((unsigned)a.n_rows + 255) / 256), dim3(256), st, a);
  return e;
}

// ---------------------------------------------------------------------------
// Store.  A wavefront takes 16 rows of one (head, block of 32): 4 lanes to a row, 8 dimensions each, keys then values.
// Bound by HBM where a page's rows come together, as a prompt's do: 32768 rows of 8 heads of 128 with the values 125 us in fp32 (4.6 TB/s), 63 in
// bf16 (4.8); rows whose slots are a random permutation write lone pieces of 16 bytes, 160 and 97 us (3.6 and 3.1 TB/s).
// ---------------------------------------------------------------------------
namespace {

// maximum over the 4 lanes of a quad
__device__ inline unsigned quad_max(unsigned v) {
  v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false));    // quad_perm 1 0 3 2
  return max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, false)); // quad_perm 2 3 0 1
}

// 8 values of a block of 32 that a quad shares -> their codes; e: the block's biased exponent
__device__ inline unsigned cache_codes(const float (&x)[8], unsigned& e) {
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = quad_max(top);
  const bool bad = top >= 0x7f800000u;
  // 2^21 = a quarter of the fraction's range: from 1.75 on the next power, so that the largest code, 6, is the nearest
  const unsigned p = (top + 0x200000u) >> 23;
  e = bad ? 255u : min(max(p, 4u) - 2u, 252u);      // (every value then is a normal number)
  const float inv = __uint_as_float((254u - (bad ? 127u : e)) << 23);
  unsigned c = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float y0 = bad ? 0.f : x[2 * i] * inv, y1 = bad ? 0.f : x[2 * i + 1] * inv;
    if (i == 0) c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y0, y1, 1.0f, 0);
    if (i == 1) c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y0, y1, 1.0f, 1);
    if (i == 2) c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y0, y1, 1.0f, 2);
    if (i == 3) c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y0, y1, 1.0f, 3);
  }
  return c;
}

// 8 codes times their power, in bf16 (exact); a power of 255 makes them NaN
__device__ inline bf16x8 cache_open(unsigned c, unsigned e) {
  const float s = __uint_as_float(e << 23);
  union { bf16x2 h[4]; bf16x8 v; } o;
  o.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0);
  o.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1);
  o.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2);
  o.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3);
  return o.v;
}

// A lane's 8 of a block's 32 dimensions: what lets the quad's accesses of 16 bytes lie together.  bf16: 8 part .. + 7; fp32: 4 part .. + 3 and
// 16 + 4 part .. + 3.
template <typename T> constexpr int SECOND = sizeof(T) == 2 ? 4 : 16;        // first of its second four, from its first
template <typename T> __device__ inline int first_dim(int part) { return part * (sizeof(T) == 2 ? 8 : 4); }

template <typename T, bool VEC>
__device__ inline void load8(const T* p, float (&x)[8]) {
  if constexpr (!VEC) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)p[i < 4 ? i : SECOND<T> + i - 4];
  } else if constexpr (sizeof(T) == 2) {
    const bf16x8 v = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
  } else {
    const f32x4 u = *reinterpret_cast<const f32x4*>(p), v = *reinterpret_cast<const f32x4*>(p + SECOND<T>);
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = u[i]; x[4 + i] = v[i]; }
  }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheAppend a) {
  const int nb = a.dh / 32;
  const int unit = blockIdx.y * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (unit >= a.Hkv * nb) return;
  const int row = blockIdx.x * 16 + (lane >> 2), r = min(row, a.n_rows - 1), part = lane & 3, head = unit / nb, blk = unit % nb;
  // (the rows' values are requested with their slots, not behind them)
  const long long slot = a.slot_map[r];
  float x[2][8];
  load8<T, VEC>(reinterpret_cast<const T*>(a.k) + r * a.k_row + head * a.k_head + blk * 32 + first_dim<T>(part), x[0]);
  load8<T, VEC>(reinterpret_cast<const T*>(a.v) + r * a.v_row + head * a.v_head + blk * 32 + first_dim<T>(part), x[1]);
  __builtin_amdgcn_sched_barrier(0);
  if (row >= a.n_rows || slot < 0 || slot >= (long long)a.n_pages * CACHE_PAGE) return;
  const int tok = (int)(slot % CACHE_PAGE);
  unsigned char* page = a.pool + ((size_t)(slot / CACHE_PAGE) * a.Hkv + head) * cache_block_bytes(a.dh);
  unsigned e[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const unsigned c = cache_codes(x[q], e[q]);
    unsigned w = c;                                  // the codes of 8 adjacent dimensions
    int at = part * 4;
    if constexpr (sizeof(T) == 4) {                  // pairs of lanes trade: the first halves to the even one, the second halves to the odd one
      const unsigned other = (unsigned)__builtin_amdgcn_update_dpp(0, (int)c, 0xB1, 0xf, 0xf, false);
      w = part & 1 ? (other >> 16) | (c & 0xffff0000u) : (c & 0xffffu) | (other << 16);
      at = (part & 1) * 8 + (part >> 1) * 4;
    }
    *reinterpret_cast<unsigned*>(page + cache_code_off(a.dh, q, blk, tok) + at) = w;
    void* values = q ? a.v_values : a.k_values;
    if (values == nullptr) continue;
    const bf16x8 v = cache_open(c, e[q]);
    T* dst = reinterpret_cast<T*>(values) + ((size_t)r * a.Hkv + head) * a.dh + blk * 32 + first_dim<T>(part);
    if constexpr (sizeof(T) == 2) *reinterpret_cast<bf16x8*>(dst) = v;
    else {
#pragma unroll
      for (int i = 0; i < 8; i += 4) *reinterpret_cast<f32x4*>(dst + (i ? SECOND<T> : 0)) = f32x4{(float)v[i], (float)v[i + 1], (float)v[i + 2], (float)v[i + 3]};
    }
  }
  if (part == 0) *reinterpret_cast<unsigned short*>(page + cache_scale_off(a.dh, 0, blk, tok)) = (unsigned short)(e[0] | e[1] << 8);
}

}  // namespace

hipError_t launch_cache_append(hipStream_t st, const CacheAppend& a, bool f32) {
  const dim3 grid((a.n_rows + 15) / 16, (a.Hkv * (a.dh / 32) + 3) / 4);
  auto at16 = [&](const void* p, long long row, long long head) {
    const int e = f32 ? 4 : 8;
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && row % e == 0 && head % e == 0;
  };
  const bool vec = at16(a.k, a.k_row, a.k_head) && at16(a.v, a.v_row, a.v_head);
  if (f32) return vec ? launch(cache_append_kernel<float, true>, grid, dim3(256), st, a) : launch(cache_append_kernel<float, false>, grid, dim3(256), st, a);
  return vec ? launch(cache_append_kernel<bf16_t, true>, grid, dim3(256), st, a) : launch(cache_append_kernel<bf16_t, false>, grid, dim3(256), st, a);
}

// ---------------------------------------------------------------------------
// Attention of few rows: one workgroup (W wavefronts) per (sequence, KV head, split of the context), up to 16 CT columns, CT 1, 2 or 4
// (row of the sequence, query head of the KV head).  The wavefronts take the split's tiles of 32 tokens in turn, each with an online
// softmax in registers; they meet in LDS, the splits of a context in a second small kernel, both in a fixed order.
//
// Products on v_mfma_f32_16x16x32_bf16, transposed, so that the scores' accumulators are the probabilities' operand:
//   S^T[token, column] = K . Q^T,  O^T[dim, column] = V^T . P^T.
// K: the order of a contraction is free, so lane (token t, g) takes the dimensions g dh / 4 .. of its token, which lie together
// with one scale (dh 128: exactly a block of 32), and Q is loaded in the same order; codes become bf16 in
// registers, exactly.  (A scaled product straight from the codes, v_mfma_scale_f32_16x16x128_f8f6f4 with Q split into two e4m3
// terms, was tried: its sums keep about 17 bits, 4.5e-6 of a score against 8e-9 here, and a short row's lse showed it.)
// V: a fragment wants 8 tokens of one dimension, the store 32 dimensions of one token (so that a token is appended without
// touching its neighbours): lanes open the blocks that they loaded into a tile of LDS, [token][dim], and
// read it back transposed (ds_read_b64_tr_b16).  Rows of dh + 16 elements put the rows of a read on different banks.
// ---------------------------------------------------------------------------
namespace {

constexpr int CA_MOST = 4096;                    // tokens of a split, at most: a lane holds 4 page ids

typedef short s16x4 __attribute__((ext_vector_type(4)));
// Four rows (tokens) of 16 bf16 columns each; lane i of 16 points at row i / 4, columns 4 (i % 4).. and gets column i, rows 0..3.
__device__ inline bf16x4 read_transposed(const bf16_t* p) {
  union { s16x4 s; bf16x4 b; } u;
#if defined(__HIP_DEVICE_COMPILE__)
  u.s = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p));
#else
  u.b = *reinterpret_cast<const bf16x4*>(p);
#endif
  return u.b;
}

struct Split { int chunk, n, waves; };           // tokens of a split, splits of the longest context, wavefronts of a workgroup (few rows)

// Where a row's head's dimension goes: rows with strides, or (engine) the fragment-tiled layout of the products behind it.
template <int DH, bool ENGINE> __device__ inline bf16_t* out_at(const CacheAttn& a, int r, int h, int d) {
  return ENGINE ? a.out + act_index<true>(r, h * DH + d, a.Hq * DH) : a.out + r * a.out_row + h * a.out_head + d;
}

template <int DH> struct KRaw;
template <> struct KRaw<32> { typedef unsigned type; };
template <> struct KRaw<64> { typedef uint2 type; };
template <> struct KRaw<128> { typedef uint4 type; };
template <int DH> __device__ inline unsigned k_word(const typename KRaw<DH>::type& r, int c) {
  if constexpr (DH == 32) return r;
  else if constexpr (DH == 64) return c ? r.y : r.x;
  else return c == 0 ? r.x : c == 1 ? r.y : c == 2 ? r.z : r.w;
}

// Blocks of NaN among the values that a column with `vis` visible tokens sees on the page whose first token is t0 (a bit each; every
// lane of the wavefront calls, each with its own column).
template <int DH> __device__ inline unsigned nan_blocks(const CacheAttn& a, int page, int kvh, int t0, int len, int vis) {
  const int lane = threadIdx.x & 63, blk = lane >> 4, tok = lane & 15;
  bool nan = false;
  if ((unsigned)page < (unsigned)a.n_pages && blk < DH / 32 && t0 + tok < len)
    nan = a.pool[((size_t)page * a.Hkv + kvh) * cache_block_bytes(DH) + cache_scale_off(DH, 1, blk, tok)] == 255;
  const unsigned long long m = __ballot(nan);
  const unsigned seen = vis > t0 ? 0xffffu >> (16 - min(16, vis - t0)) : 0u;
  unsigned bits = 0;
#pragma unroll
  for (int q = 0; q < DH / 32; ++q) bits |= ((unsigned)(m >> (16 * q)) & seen) ? 1u << q : 0u;
  return bits;
}

// Partial results of a split: per (row, head) maximum and sum, then the unnormalised output.  Rows are counted by sequence where that makes
// fewer than n_rows (a padded batch).
__device__ inline int part_row(const CacheAttn& a, int r, int b, int i) { return a.ws_rows < a.n_rows ? b * a.max_q + i : r; }
__device__ inline float* part_ml(const CacheAttn& a, int split, int pr, int h) { return a.ws + (((size_t)split * a.ws_rows + pr) * a.Hq + h) * 2; }
template <int DH> __device__ inline float* part_o(const CacheAttn& a, int n_splits, int split, int pr, int h) {
  return a.ws + (size_t)n_splits * a.ws_rows * a.Hq * 2 + (((size_t)split * a.ws_rows + pr) * a.Hq + h) * DH;
}

// Whose rows: a caller's (the operator), or the engine's decode iteration, with the queries given or (fused) with the projection's partials.
enum { CA_ROWS, CA_ENGINE, CA_FUSED };
// ENGINE: the work list of a decode iteration, entry 0 = {number}, entry 1 + i = {row, split, slot, position} (see launch_sched).
template <int DH, int CT, int W, int MODE>
__global__ __launch_bounds__(64 * W, CT == 1 ? 4 : CT == 2 ? 2 : 1) void cache_attn_kernel(CacheAttn a, Split sp, CacheRows er, CacheRope f) {
  constexpr bool ENGINE = MODE != CA_ROWS, FUSED = MODE == CA_FUSED;
  constexpr int KC = DH / 32, DT = DH / 16, NV = DH == 128 ? 2 : 1;
  constexpr int VS = DH + 16, OS = DH + 4;            // row strides in LDS: opened values, merged outputs
  constexpr int REC = CT * 16 * (2 + OS);             // floats of a wavefront's result
  constexpr int REGION = REC * 4 > 32 * VS * 2 ? REC * 4 : 32 * VS * 2;
  typedef typename KRaw<DH>::type kraw_t;
  __shared__ __align__(16) unsigned char lds[W][REGION];
  __shared__ __align__(16) uint4 s_new[FUSED ? 2 * (DH / 32) : 1];       // the new token's codes, key and value, and their scales
  __shared__ unsigned s_new_scale[FUSED ? 2 * (DH / 32) : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hh = lane & 15, g = lane >> 4;
  const int G = a.Hq / a.Hkv;
  // KV heads go round first: the heads of one sequence on different XCDs; splits last: only long contexts have the later ones
  const int kvh = (int)(blockIdx.x % a.Hkv), rest = (int)(blockIdx.x / a.Hkv);
  int b, split, first, count = 1, len_raw;
  if (ENGINE) {
    const int4 head = er.items[0], it = er.items[1 + rest];
    if (er.ctl->y || rest >= head.x) return;
    first = it.x; split = it.y; b = it.z; len_raw = it.w + 1;
  } else {
    b = rest % a.n_seqs;
    split = rest / a.n_seqs;
    first = a.q_start != nullptr ? a.q_start[b] : b;
    if (a.q_start != nullptr) count = a.q_start[b + 1] - first;
    len_raw = a.lens[b];
  }
  if (first < 0 || count <= 0 || first >= a.n_rows) return;
  const int nq = min(min(count, a.max_q), a.n_rows - first);
  bool bad = len_raw < 0 || len_raw > a.max_len;
  const int len = bad ? 0 : len_raw;
  const int t_begin = split * sp.chunk;
  if (split > 0 && t_begin >= len) return;
  const int t_end = min(len, t_begin + sp.chunk), n_tiles = (t_end - t_begin + 31) >> 5, n_pages = (t_end - t_begin + 15) >> 4;

  // page ids of the split, one per lane and register (loading them as the tiles come to them, in a branch, had every wait in the loop be
  // for all loads: 245 against 238 us); ids outside the pool are noticed and not followed
  const int* bt = a.block_table + (size_t)b * a.table_stride + (t_begin >> 4);
  int my_page[CA_MOST / 1024];
#pragma unroll
  for (int q = 0; q < CA_MOST / 1024; ++q) {
    const int i = q * 64 + lane;
    my_page[q] = n_pages > q * 64 ? bt[i < n_pages ? i : n_pages - 1] : 0;
    const bool out = (unsigned)my_page[q] >= (unsigned)a.n_pages;
    bad |= __any(out);
    if (out) my_page[q] = 0;
  }

  // what this lane takes of a page's block: keys, their scale; values, theirs
  const int kblk = g * DH / 128, kbyte = (g * (DH / 4) % 32) / 2;
  const int off_k = cache_code_off(DH, 0, kblk, hh) + kbyte, off_ks = cache_scale_off(DH, 0, kblk, hh);
  const int vblk = DH == 128 ? g : DH == 64 ? g & 1 : 0;
  const int vpage = DH == 128 ? 0 : DH == 64 ? g >> 1 : g & 1;            // (dh 128: both pages, one after the other)
  const int off_v = cache_code_off(DH, 1, vblk, hh), off_vs = cache_scale_off(DH, 1, vblk, hh);
  constexpr int R = 2;                                // tiles in flight
  kraw_t kr[R][2];
  uint4 vr[R][NV];
  unsigned ks[R][2], vs[R][NV];
  auto request = [&](int u, int i) {
    const int tile = min(wave + i * W, n_tiles - 1);
    const unsigned char* base[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int pl = __builtin_amdgcn_readfirstlane(min(2 * tile + p, n_pages - 1));
      int page = __builtin_amdgcn_readlane(my_page[0], pl & 63);
#pragma unroll
      for (int q = 1; q < CA_MOST / 1024; ++q)
        if ((pl >> 6) == q) page = __builtin_amdgcn_readlane(my_page[q], pl & 63);
      base[p] = a.pool + ((size_t)page * a.Hkv + kvh) * cache_block_bytes(DH);
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      kr[u][p] = *reinterpret_cast<const kraw_t*>(base[p] + off_k);
      if constexpr (DH == 128) {
        vr[u][p] = *reinterpret_cast<const uint4*>(base[p] + off_v);
        ks[u][p] = *reinterpret_cast<const unsigned short*>(base[p] + off_ks);       // key's and value's scale
      } else {
        ks[u][p] = base[p][off_ks];
      }
    }
    if constexpr (DH != 128) {
      const unsigned char* vb = vpage ? base[1] : base[0];
      vr[u][0] = *reinterpret_cast<const uint4*>(vb + off_v);
      vs[u][0] = vb[off_vs];
    }
  };
  const int cnt = n_tiles > wave ? (n_tiles - wave + W - 1) / W : 0;
  auto first_tiles = [&]() {
#pragma unroll
    for (int u = 0; u < R; ++u)
      if (u < cnt) request(u, u);
  };
  const bool has_new = FUSED && len > 0 && t_end == len;          // the split of the token that this iteration adds
  bf16_t* s_q = reinterpret_cast<bf16_t*>(lds);        // [head][DH + 8] until the queries are in registers
  if (FUSED) {
    // The workgroup sums the projection's partials of its query heads and rotates them, a pair (i, i + DH / 2) per thread, and in the
    // last split the new token's key (rotated) and value, "heads" G and G + 1; those are rounded by 4 lanes a block, stored in the page
    // and kept for the tile that holds them.  The partials are requested before the first tiles, so the sums run while those arrive.
    // (A kernel of its own for this costs a launch a layer: 96 sequences of 1000 tokens, 8 layers: 0.410 against 0.362 ms an iteration.
    // Four partials of two pairs at a time: 8 have head dim 128 spill and gain nothing.)
    constexpr int HALF = DH / 2, U = 2, QB = 4, QS = DH + 8;
    float* s_kv = reinterpret_cast<float*>(s_q + 16 * QS);               // [key | value][DH]
    const int n_pairs = (has_new ? G + 2 : G) * HALF, np = f.n_partials, pos = max(len - 1, 0);
    const float* src = f.q_src + (size_t)first * f.q_ld;
    const float* cs = f.rope_cos + (size_t)pos * HALF;
    const float* sn = f.rope_sin + (size_t)pos * HALF;
    auto trip = [&](int p0, auto requests) {
      const float* col[U];
      float cv[U], sv[U], x[U], y[U], vx[U][QB], vy[U][QB];
      int hd[U], ii[U];
      auto load = [&](int q0) {
#pragma unroll
        for (int q = 0; q < QB; ++q)
          if (q0 + q < np) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
              const float* c = col[u] + (size_t)(q0 + q) * f.partial_stride;
              vx[u][q] = c[0]; vy[u][q] = c[HALF];
            }
          }
      };
      auto add = [&](int q0) {                         // in the order p = 0, 1, ...
#pragma unroll
        for (int q = 0; q < QB; ++q)
          if (q0 + q < np) {
#pragma unroll
            for (int u = 0; u < U; ++u) { x[u] = q0 + q ? x[u] + vx[u][q] : vx[u][q]; y[u] = q0 + q ? y[u] + vy[u][q] : vy[u][q]; }
          }
      };
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int e = min(p0 + u * 64 * W + (int)threadIdx.x, n_pairs - 1);
        hd[u] = e / HALF; ii[u] = e % HALF;
        col[u] = src + (size_t)(hd[u] < G ? kvh * G + hd[u] : a.Hq + (hd[u] - G) * a.Hkv + kvh) * DH + ii[u];
        cv[u] = cs[ii[u]]; sv[u] = sn[ii[u]];
        x[u] = y[u] = 0.f;
      }
      load(0);
      __builtin_amdgcn_sched_barrier(0);
      if (requests) first_tiles();
      __builtin_amdgcn_sched_barrier(0);
      add(0);
      for (int q0 = QB; q0 < np; q0 += QB) { load(q0); add(q0); }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (p0 + u * 64 * W + (int)threadIdx.x >= n_pairs) continue;
        const int i = ii[u];
        const float ra = rope_first(x[u], y[u], cv[u], sv[u]), rb = rope_second(x[u], y[u], cv[u], sv[u]);
        if (hd[u] < G) {
          s_q[hd[u] * QS + i] = (bf16_t)ra;
          s_q[hd[u] * QS + i + HALF] = (bf16_t)rb;
        } else {
          const bool key = hd[u] == G;
          float* to = s_kv + (key ? 0 : DH) + i;
          to[0] = key ? ra : x[u];
          to[HALF] = key ? rb : y[u];
        }
      }
    };
    trip(0, std::true_type{});
    for (int p0 = U * 64 * W; p0 < n_pairs; p0 += U * 64 * W) trip(p0, std::false_type{});
    __syncthreads();
    if (has_new && (int)threadIdx.x < 2 * DH / 8) {
      const int val = threadIdx.x / (DH / 8), blk = threadIdx.x % (DH / 8) / 4, part = threadIdx.x % 4, tok = pos % CACHE_PAGE, new_page = bt[(pos - t_begin) / CACHE_PAGE];
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = s_kv[val * DH + blk * 32 + part * 8 + i];
      unsigned e;
      const unsigned c = cache_codes(x, e);
      reinterpret_cast<unsigned*>(s_new)[(val * (DH / 32) + blk) * 4 + part] = c;
      unsigned char* to = f.pool + ((size_t)new_page * a.Hkv + kvh) * cache_block_bytes(DH);
      const bool in_pool = (unsigned)new_page < (unsigned)a.n_pages;
      if (in_pool) *reinterpret_cast<unsigned*>(to + cache_code_off(DH, val, blk, tok) + part * 4) = c;
      if (part == 0) {
        s_new_scale[val * (DH / 32) + blk] = e;
        if (in_pool) to[cache_scale_off(DH, val, blk, tok)] = (unsigned char)e;
      }
    }
  } else {
    first_tiles();
  }

  // queries, and the tokens that each column sees
  bf16x8 qf[CT][KC];
  int vis[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int col = ct * 16 + hh, i = col / G, h = col - i * G;
    const bool used = i < nq;
    vis[ct] = used ? len - count + i + 1 : 0;
    const bf16_t* q = a.q + (first + (used ? i : 0)) * a.q_row + (kvh * G + h) * a.q_head + g * (DH / 4);
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const bf16x8 v = *reinterpret_cast<const bf16x8*>(FUSED ? s_q + (used ? h : 0) * (DH + 8) + g * (DH / 4) + 8 * c : q + 8 * c);
      qf[ct][c] = used ? v : bf16x8{};
    }
  }
  if (FUSED) __syncthreads();                          // (the tiles' memory held the queries)
  const int vis_min = len - count + 1;                // what the sequence's first row sees
  float m_run[CT], l_run[CT];
  unsigned poison[CT];                                // bit: this column sees a NaN among the values of that block
  f32x4 oacc[CT][DT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    m_run[ct] = -INFINITY; l_run[ct] = 0.f; poison[ct] = bad ? 15u : 0u;
#pragma unroll
    for (int d = 0; d < DT; ++d) oacc[ct][d] = f32x4{};
  }
  bf16_t* vl = reinterpret_cast<bf16_t*>(lds[wave]);
  bool nan_seen = false;

  auto compute = [&](int u, int i) {
    const int t0 = t_begin + (wave + i * W) * 32;
    if (FUSED && has_new && t0 + 32 >= len) {          // the new token, wherever its page's copy may be
      const int pp = (len - 1 - t0) >> 4, tin = (len - 1) & 15;
      if (hh == tin) {
#pragma unroll
        for (int p = 0; p < 2; ++p)
          if (p == pp) {
            kr[u][p] = *reinterpret_cast<const kraw_t*>(reinterpret_cast<const unsigned char*>(s_new) + kblk * 16 + kbyte);
            ks[u][p] = s_new_scale[kblk];
            if (DH == 128) { vr[u][p % NV] = s_new[DH / 32 + vblk]; ks[u][p] |= s_new_scale[DH / 32 + vblk] << 8; }
          }
        if (DH != 128 && vpage == pp) { vr[u][0] = s_new[DH / 32 + vblk]; vs[u][0] = s_new_scale[DH / 32 + vblk]; }
      }
    }
    // values into LDS: zeros behind the context's end (what lies there is anything) and for blocks of NaN, which would reach
    // columns that do not see them; the columns that do are marked behind the loop
#pragma unroll
    for (int p = 0; p < NV; ++p) {
      __builtin_amdgcn_sched_barrier(0);
      const int row = (DH == 128 ? p : vpage) * 16 + hh;
      uint4 c = vr[u][p];
      unsigned e = DH == 128 ? ks[u][p] >> 8 : vs[u][p];
      if (t0 + 32 > len && t0 + row >= len) { c = uint4{0, 0, 0, 0}; e = 127; }
      if (__any(e == 255)) {
        nan_seen = true;
        if (e == 255) { c = uint4{0, 0, 0, 0}; e = 127; }
      }
      if (DH > 32 || g < 2) {
        bf16x8* to = reinterpret_cast<bf16x8*>(vl + row * VS + vblk * 32);
        to[0] = cache_open(c.x, e);
        to[1] = cache_open(c.y, e);
        to[2] = cache_open(c.z, e);
        to[3] = cache_open(c.w, e);
      }
    }
    f32x4 sacc[CT][2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      __builtin_amdgcn_sched_barrier(0);               // (one page's opened fragments at a time: registers)
      const unsigned e = DH == 128 ? ks[u][p] & 255 : ks[u][p];
      bf16x8 kf[KC];
#pragma unroll
      for (int c = 0; c < KC; ++c) kf[c] = cache_open(k_word<DH>(kr[u][p], c), e);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        sacc[ct][p] = f32x4{};
#pragma unroll
        for (int c = 0; c < KC; ++c) sacc[ct][p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[c], qf[ct][c], sacc[ct][p], 0, 0, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    // Softmax in base 2; the running maximum may lag by 2^8 (probabilities then reach 256, which costs no precision), so that a
    // tile seldom needs a shuffle.  It is a score, subtracted before the scale: of scores beyond 2^30 a rounded multiple of it would leave
    // exponents of hundreds.  Probabilities are rounded to bf16 for the second product, their sum is not: an output is off by at most
    // 2^-8 of the mean |v| under its weights (relative 2-norm 0.0023, of which the rounded output alone is 0.0017).  A second bf16 term of
    // each would take that away and double the second product, the opened values' reads with it.
    bf16x8 pf[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      float s[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = sacc[ct][e >> 2][e & 3];
      if (t0 + 32 > vis_min) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (t0 + (e >> 2) * 16 + 4 * g + (e & 3) >= vis[ct]) s[e] = -INFINITY;
      }
      float mx = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
      if (__any(mx > m_run[ct] + a.lag)) {
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const bool grow = mx > m_run[ct] + a.lag;
        const float corr = grow ? __builtin_amdgcn_exp2f((m_run[ct] - mx) * a.c2) : 1.0f;
        m_run[ct] = grow ? mx : m_run[ct];
        l_run[ct] *= corr;
#pragma unroll
        for (int d = 0; d < DT; ++d) oacc[ct][d] *= corr;
      }
      const float m = m_run[ct] == -INFINITY ? 0.f : m_run[ct];          // nothing seen yet: exponentials of -inf
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float pe = __builtin_amdgcn_exp2f((s[e] - m) * a.c2);
        sum[e & 1] += pe;
        pf[ct][e] = (bf16_t)pe;
      }
      l_run[ct] += sum[0] + sum[1];
    }
    asm volatile("" ::: "memory");                     // (LDS serves a wavefront's accesses in their order)
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      if (d % 4 == 0) __builtin_amdgcn_sched_barrier(0);
      const bf16_t* at = vl + (4 * g + (hh >> 2)) * VS + d * 16 + 4 * (hh & 3);
      union { bf16x4 h[2]; bf16x8 v; } vf;
      vf.h[0] = read_transposed(at);
      vf.h[1] = read_transposed(at + 16 * VS);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) oacc[ct][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf.v, pf[ct], oacc[ct][d], 0, 0, 0);
    }
    asm volatile("" ::: "memory");
  };
  // A slot is requested again as soon as its tile is done; behind the last tile that is the last tile once more, so that no load is in a
  // branch (a wait behind one would be for all loads).  Two copies of the loop's body: every compute unit has to fetch the code of a
  // launch (with steady state and tail apart, five copies, 61 sequences of 100-2003 tokens took 20.7 us and not 17.4; the loop has 124 registers then, not 168: 192 of
  // 576-4608 tokens, 32 + 8 heads of 128, 131 and 121; with all that came later 15.2 and 116).
  for (int i = 0; i < cnt; i += R) {
#pragma unroll
    for (int u = 0; u < R; ++u) {
      if (u == 0 || i + u < cnt) compute(u, i + u);
      __builtin_amdgcn_sched_barrier(0);
      request(u, i + u + R);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  if (nan_seen)                                      // some block of this wavefront's values is NaN: mark the columns that see it
#pragma clang loop unroll(disable)
    for (int i = 0; i < 2 * cnt; ++i) {
      const int pg = 2 * (wave + (i >> 1) * W) + (i & 1);
      if (pg >= n_pages) continue;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) poison[ct] |= nan_blocks<DH>(a, bt[pg], kvh, t_begin + pg * CACHE_PAGE, len, vis[ct]);
    }

  // the wavefronts meet: each publishes (m, l, O), then merges its share of the columns' outputs
  float* mine = reinterpret_cast<float*>(lds[wave]);
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    unsigned p = poison[ct];
    p |= __shfl_xor((int)p, 16, 64);
    p |= __shfl_xor((int)p, 32, 64);
    float l = l_run[ct];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (bad) l = NAN;
    if (g == 0) { mine[ct * 16 + hh] = m_run[ct]; mine[CT * 16 + ct * 16 + hh] = l; }
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      f32x4 o = oacc[ct][d];
      if (p >> (d / 2) & 1) o = f32x4{NAN, NAN, NAN, NAN};
      *reinterpret_cast<f32x4*>(mine + CT * 32 + (ct * 16 + hh) * OS + d * 16 + 4 * g) = o;
    }
  }
  __syncthreads();
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int col = ct * 16 + hh, qi = col / G, h = kvh * G + col - qi * G, r = first + qi;
    float M = -INFINITY, wgt[W], lsum = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) M = fmaxf(M, reinterpret_cast<const float*>(lds[w])[col]);
    const float Mu = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float* p = reinterpret_cast<const float*>(lds[w]);
      wgt[w] = __builtin_amdgcn_exp2f((p[col] - Mu) * a.c2);
      lsum += wgt[w] * p[CT * 16 + col];
    }
    const float inv = lsum == 0.f ? 0.f : 1.0f / lsum;
    if (qi >= nq || (split > 0 && vis[ct] <= t_begin)) continue;
    const bool whole = vis[ct] <= sp.chunk;            // the row's tokens are all in the first split
    const int pr = part_row(a, r, b, qi);
    for (int d = wave; d < DT; d += W) {
      f32x4 o = f32x4{};
#pragma unroll
      for (int w = 0; w < W; ++w) o += *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(lds[w]) + CT * 32 + col * OS + d * 16 + 4 * g) * wgt[w];
      if (whole) {
        bf16x4 ob;
#pragma unroll
        for (int e = 0; e < 4; ++e) ob[e] = (bf16_t)(o[e] * inv);
        *reinterpret_cast<bf16x4*>(out_at<DH, ENGINE>(a, r, h, d * 16 + 4 * g)) = ob;
      } else {
        *reinterpret_cast<f32x4*>(part_o<DH>(a, sp.n, split, pr, h) + d * 16 + 4 * g) = o;
      }
    }
    if (wave == 0 && g == 0) {
      if (!whole) *reinterpret_cast<float2*>(part_ml(a, split, pr, h)) = float2{M, lsum};
      else if (a.lse != nullptr) a.lse[(size_t)r * a.Hq + h] = lsum == 0.f ? -INFINITY : (M * a.c2 + log2f(lsum)) * 0.6931471805599453f;
    }
  }
}

// Joins the splits of the rows that see tokens of several, in their order: 4 dimensions of a head per thread, 1024 elements of a row per
// workgroup.  The loads of 4 splits go out together.  (A workgroup per row, a split at a time: 34 us of the 71 of 7 rows of 32 heads over
// up to 19 splits.)
template <int DH, bool ENGINE>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheAttn a, Split sp, CacheRows er) {
  const int b = ENGINE ? (int)blockIdx.x : (int)blockIdx.x / a.max_q, i = ENGINE ? 0 : (int)blockIdx.x % a.max_q;
  if (ENGINE && (er.ctl->y || b >= er.ctl->x)) return;
  const int first = !ENGINE && a.q_start != nullptr ? a.q_start[b] : b, count = !ENGINE && a.q_start != nullptr ? a.q_start[b + 1] - first : 1, r = first + i;
  const int len = ENGINE ? er.row_pos[b] + 1 : a.lens[b];
  if (first < 0 || i >= count || r >= a.n_rows || len < 0 || len > a.max_len || len - count + i + 1 <= sp.chunk) return;
  const int n_splits = (len - count + i + sp.chunk) / sp.chunk;
  const int e = blockIdx.y * 256 + threadIdx.x, h = e / (DH / 4), d = 4 * (e % (DH / 4));
  if (h >= a.Hq) return;
  const int pr = part_row(a, r, b, i);
  const float* ml = part_ml(a, 0, pr, h);
  const float* po = part_o<DH>(a, sp.n, 0, pr, h) + d;
  const size_t ml_step = (size_t)a.ws_rows * a.Hq * 2, o_step = (size_t)a.ws_rows * a.Hq * DH;
  constexpr int U = 4;
  float M = -INFINITY;
  for (int s = 0; s < n_splits; s += 2 * U) {
    float v[2 * U];
#pragma unroll
    for (int u = 0; u < 2 * U; ++u) v[u] = ml[min(s + u, n_splits - 1) * ml_step];
#pragma unroll
    for (int u = 0; u < 2 * U; ++u) M = fmaxf(M, v[u]);
  }
  const float Mu = M == -INFINITY ? 0.f : M;
  float lsum = 0.f;
  f32x4 o = f32x4{};
  for (int s = 0; s < n_splits; s += U) {
    float2 v[U];
    f32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = min(s + u, n_splits - 1);
      v[u] = *reinterpret_cast<const float2*>(ml + at * ml_step);
      x[u] = *reinterpret_cast<const f32x4*>(po + at * o_step);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s + u < n_splits) {
        const float w = __builtin_amdgcn_exp2f((v[u].x - Mu) * a.c2);
        lsum += w * v[u].y;
        o += x[u] * w;
      }
  }
  const float inv = lsum == 0.f ? 0.f : 1.0f / lsum;
  bf16x4 ob;
#pragma unroll
  for (int q = 0; q < 4; ++q) ob[q] = (bf16_t)(o[q] * inv);
  *reinterpret_cast<bf16x4*>(out_at<DH, ENGINE>(a, r, h, d)) = ob;
  if (!ENGINE && d == 0 && a.lse != nullptr) a.lse[(size_t)r * a.Hq + h] = lsum == 0.f ? -INFINITY : (M * a.c2 + log2f(lsum)) * 0.6931471805599453f;
}
template <int DH> dim3 join_grid(const CacheAttn& a, int rows) { return dim3(rows, (a.Hq * (DH / 4) + 255) / 256); }

// ---------------------------------------------------------------------------
// Attention of many rows: a workgroup (4 wavefronts) owns 256 columns (row, query head) of one (sequence, KV head) and walks over
// the tokens that they see in stages of 64: each block of 32 codes is opened to bf16 once per workgroup, into LDS, and serves all
// of its columns.  A wavefront takes 64 columns, two tiles of v_mfma_f32_32x32x16_bf16, transposed products as above:
//   S^T[token, column] = K . Q^T,  O^T[dim, column] = V^T . P^T;
// the accumulators of the first, rounded to bf16 in place, are the operand of the second, whose V fragment is read transposed.
// Two stage buffers: while one is worked on, the codes of the next are opened into the other and those of the one behind it
// requested.  Rows of LDS are 8 (keys) and 16 (values) elements apart beyond their length, which puts the rows of a read on different
// banks.
// At head dim 128 accumulators and queries take 192 of the 256 registers that two wavefronts a SIMD leave; one register too many
// has the loop wait for its reload and with it for the codes on their way.  So the codes go past the registers (copied into LDS), and what follows
// from a lane's number is computed where it is used.  A fragment's read from LDS takes as long as four products, so two are in flight
// (left to itself the compiler reads into the registers just used, and waits), and the exponentials of a half's second 16
// tokens run beside the products of its first.  Probabilities are rounded to bf16 for the second product, as above.
// 21 prompts of 1-1999 tokens, 32 + 8 heads, us in short runs: 358; without
// spills 325, fragments ahead 317, queries and outputs as whole rows 304, exponentials beside products 288, scores less
// their maximum before the scale 300 (without it scores beyond 2^30 overflow).  Such a run is too short for the clock: of 300 calls in a row the
// first 20 take 339 under the profiler, from the 150th on 269 to 278 (827 TFLOP/s and more).  What is left, in those runs:
// queries, outputs and the first stage alone take 110 us (2 x 172 MB), opening and barriers 46; priorities for either kind of phase,
// three fragments in flight and the codes requested later changed nothing.
constexpr int RA_STAGE = 64, RA_COLS = 256;
typedef unsigned u32x4_8 __attribute__((ext_vector_type(4), aligned(8)));      // outputs are 8-byte aligned

__device__ inline void copy_to_lds(const void* src_lane, uint4* lds_base) {      // 64 lanes x 16 bytes, past the registers
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds(src_lane, lds_base, 16, 0, 0);
#else
  (void)src_lane; (void)lds_base;
#endif
}
__device__ inline void loads_done() {                // vmcnt(0)
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_s_waitcnt(0x0f70);
#endif
  asm volatile("" ::: "memory");
}

__device__ inline int again(int x) {                 // what is derived from it is computed where it is used, not kept in registers
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(x));
#endif
  return x;
}

__device__ inline float max_of_halves(float x) {      // of lanes l and l ^ 32
#if defined(__HIP_DEVICE_COMPILE__)
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const unsigned lower = r[0], upper = r[1];
  return fmaxf(__uint_as_float(lower), __uint_as_float(upper));
#else
  return x;
#endif
}

// ENGINE: items {slot, first row of the sequence, its tokens, first position of the tile} of er.q_tile positions (see launch_attn_prefill).
template <int DH, bool ENGINE>
__global__ __launch_bounds__(256, 2) void cache_attn_rows_kernel(CacheAttn a, Split sp, int n_qt, CacheRows er) {
  constexpr int KC = DH / 16, DT = DH / 32, CT = 2, NV = DH == 128 ? 2 : 1;
  constexpr int KS = DH + 8, VS = DH + 16;                   // row strides in LDS
  __shared__ __align__(16) bf16_t s_kv[2 * RA_STAGE * (KS + VS)];
  bf16_t (*s_k)[RA_STAGE * KS] = reinterpret_cast<bf16_t (*)[RA_STAGE * KS]>(s_kv);                            // [buffer][token][dim]
  bf16_t (*s_v)[RA_STAGE * VS] = reinterpret_cast<bf16_t (*)[RA_STAGE * VS]>(s_kv + 2 * RA_STAGE * KS);
  __shared__ __align__(16) uint4 s_raw[4][NV][64];           // the next stage's codes, each wavefront's own
  __shared__ int s_nan;                                      // some block of the values is NaN
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), cl = lane & 31, hf = lane >> 5;
  const int G = a.Hq / a.Hkv;
  // KV heads first (different XCDs), the tiles with the most tokens before the others, splits last
  const int kvh = (int)(blockIdx.x % a.Hkv);
  int rest = (int)(blockIdx.x / a.Hkv);
  int b, split = 0, first, count = 1, len_raw, n_cols, col0;
  if (ENGINE) {
    const int4 it = er.items[rest];
    b = it.x; first = it.y; count = len_raw = it.z;
    col0 = it.w * G;
    n_cols = min(count, it.w + er.q_tile) * G;
  } else {
    b = rest % a.n_seqs;
    rest /= a.n_seqs;
    split = rest / n_qt;
    first = a.q_start != nullptr ? a.q_start[b] : b;
    if (a.q_start != nullptr) count = a.q_start[b + 1] - first;
    len_raw = a.lens[b];
    if (first < 0 || count <= 0 || first >= a.n_rows) return;
    col0 = (n_qt - 1 - rest % n_qt) * RA_COLS;
    n_cols = min(min(count, a.max_q), a.n_rows - first) * G;
  }
  if (col0 >= n_cols) return;
  bool bad = len_raw < 0 || len_raw > a.max_len;
  const int len = bad ? 0 : len_raw;
  const int t_begin = split * sp.chunk;
  const int seen = max(0, len - count + min(n_cols - 1, col0 + RA_COLS - 1) / G + 1);       // by the workgroup's last column
  if (split > 0 && t_begin >= seen) return;
  const int t_end = min(seen, t_begin + sp.chunk), n_stages = max(0, t_end - t_begin + RA_STAGE - 1) / RA_STAGE;
  const int last_page = max(0, t_end - 1) / CACHE_PAGE - t_begin / CACHE_PAGE;
  const int* bt = a.block_table + (size_t)b * a.table_stride + t_begin / CACHE_PAGE;

  // what this thread opens of a stage
  const bool opens = DH > 32 || wave < 2;
  int my_page = 0;                                   // page ids of 16 stages, one per lane
  unsigned scale = 127;                              // (dh 128: of the key and, above it, of the value)
  auto request = [&](int st) {
    const int lane = again(threadIdx.x) & 63, hh = lane & 15, g = lane >> 4;
    const int my_pg = DH == 128 ? wave : DH == 64 ? 2 * (wave & 1) + (g >> 1) : g, my_blk = DH == 128 ? g : DH == 64 ? g & 1 : 0;
    if ((st & 15) == 0) {
      const int i = st * 4 + lane;
      my_page = bt[i < last_page ? i : last_page];
      const bool out = (unsigned)my_page >= (unsigned)a.n_pages;
      bad |= __any(out);
      if (out) my_page = 0;
    }
    const int i = st * 4 + my_pg;
    const int page = __shfl(my_page, (i < last_page ? i : last_page) & 63, 64);
    if (!opens) return;
    const unsigned char* blk = a.pool + ((size_t)page * a.Hkv + kvh) * cache_block_bytes(DH);
    if constexpr (DH == 128) {
#pragma unroll
      for (int p = 0; p < NV; ++p) copy_to_lds(blk + cache_code_off(DH, p, my_blk, hh), s_raw[wave][p]);
      scale = *reinterpret_cast<const unsigned short*>(blk + cache_scale_off(DH, 0, my_blk, hh));
    } else {
      const int value = DH == 64 ? wave >> 1 : wave;
      copy_to_lds(blk + cache_code_off(DH, value, my_blk, hh), s_raw[wave][0]);
      scale = blk[cache_scale_off(DH, value, my_blk, hh)];
    }
  };
  auto open = [&](int st) {
    const int lane = again(threadIdx.x) & 63, hh = lane & 15, g = lane >> 4;
    const int my_pg = DH == 128 ? wave : DH == 64 ? 2 * (wave & 1) + (g >> 1) : g, my_blk = DH == 128 ? g : DH == 64 ? g & 1 : 0;
    const int my_row = my_pg * CACHE_PAGE + hh;
    const int buf = st & 1;
    loads_done();
#pragma unroll
    for (int p = 0; p < NV; ++p) {
      const int value = DH == 128 ? p : DH == 64 ? wave >> 1 : wave;
      uint4 c = s_raw[wave][p][lane];
      unsigned e = DH == 128 ? (p ? scale >> 8 : scale & 255) : scale;
      if (value == 1) {
        // zeros behind the context's end, where anything may lie, and for blocks of NaN: the columns that see them are marked
        if (t_begin + st * RA_STAGE + my_row >= len) { c = uint4{0, 0, 0, 0}; e = 127; }
        if (e == 255) { c = uint4{0, 0, 0, 0}; e = 127; if (opens) s_nan = 1; }
      }
      if (!opens) continue;
      bf16x8* to = reinterpret_cast<bf16x8*>(value ? &s_v[buf][my_row * VS + my_blk * 32] : &s_k[buf][my_row * KS + my_blk * 32]);
      to[0] = cache_open(c.x, e);
      to[1] = cache_open(c.y, e);
      to[2] = cache_open(c.z, e);
      to[3] = cache_open(c.w, e);
    }
  };
  if (threadIdx.x == 0) s_nan = 0;
  if (n_stages > 0) request(0);

  // Queries: whole rows into LDS, 16 bytes a lane (a row's pieces exchanged by its number: rows apart by a multiple of 256 bytes are then
  // read from different banks), from there column cl of tile ct; lane half hf holds dims 16 c + 8 hf .. + 7.  Outputs go the same way back.
  constexpr int P = DH / 8, RPI = 64 / P;                    // pieces of a row, rows of an access
  bf16_t* s_mine = s_kv + wave * 64 * DH;
  const int c_first = col0 + wave * 64, i_first = c_first / G, c_rem = c_first - i_first * G;
  const unsigned inv_g = ((1u << 20) + G - 1) / G;           // (c * inv_g) >> 20 == c / G for c < 64 + G
  auto head_row = [&](int row, int& i, int& h) {             // of row `row` of the wavefront's 64
    const int c = c_rem + row, di = (int)((unsigned)c * inv_g >> 20);
    i = i_first + di; h = kvh * G + c - di * G;
  };
  auto swap_piece = [](int row, int piece) { return piece ^ ((row * P / 16) & (P - 1)); };
  if (c_first < n_cols) {
#pragma unroll
    for (int n = 0; n < 64 / RPI; ++n) {
      const int row = n * RPI + lane / P, piece = swap_piece(row, lane % P);
      int i, h;
      head_row(min(row, n_cols - 1 - c_first), i, h);
      copy_to_lds(a.q + (first + i) * a.q_row + h * a.q_head + 8 * piece, reinterpret_cast<uint4*>(s_mine + n * RPI * DH));
    }
  }
  loads_done();
  bf16x8 qf[CT][KC];
  int vis[CT], vis_first[CT];
  int wave_seen = 0;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int c0 = c_first + ct * 32, row = ct * 32 + cl;
    int i, h;
    head_row(row, i, h);
    const bool used = c_first + row < n_cols;
    vis[ct] = used ? len - count + i + 1 : 0;
    vis_first[ct] = len - count + c0 / G + 1;
    if (c0 < n_cols) wave_seen = max(wave_seen, len - count + min(n_cols - 1, c0 + 31) / G + 1);
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const bf16x8 v = *reinterpret_cast<const bf16x8*>(s_mine + row * DH + 8 * swap_piece(row, 2 * c + hf));
      qf[ct][c] = used ? v : bf16x8{};
    }
  }
  float m_run[CT], l_run[CT];
  unsigned poison[CT];
  f32x16 oacc[CT][DT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    m_run[ct] = -FLT_MAX; l_run[ct] = 0.f; poison[ct] = 0;
#pragma unroll
    for (int d = 0; d < DT; ++d) oacc[ct][d] = f32x16{};
  }
  __syncthreads();                                   // (the flag is clear)
  if (n_stages > 0) open(0);
  if (n_stages > 1) request(1);
  __syncthreads();

  for (int st = 0; st < n_stages; ++st) {
    if (st + 1 < n_stages) open(st + 1);
    if (st + 2 < n_stages) request(st + 2);
    const int buf = st & 1, ts = t_begin + st * RA_STAGE;
#pragma unroll
    for (int half = 0; half < RA_STAGE / 32; ++half) {
      const int t0 = ts + half * 32;
      if (t0 >= wave_seen) continue;
      f32x16 sacc[CT];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) sacc[ct] = f32x16{};
      const int ln = again(threadIdx.x) & 63;
      const bf16_t* kl = &s_k[buf][(half * 32 + (ln & 31)) * KS + 8 * (ln >> 5)];
      {
        constexpr int AHEAD = KC < 2 ? KC : 2;
        bf16x8 kf[KC];
#pragma unroll
        for (int c = 0; c < KC; ++c) kf[c] = *reinterpret_cast<const bf16x8*>(kl + 16 * c);
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) sacc[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[c], qf[ct][c], sacc[ct], 0, 0, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          __builtin_amdgcn_sched_group_barrier(0x8, CT, 0);
          if (c + AHEAD < KC) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
      }
      float mx[CT];
      bool grow[CT];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        if (t0 + 32 > vis_first[ct]) {               // some column of the tile does not see all 32 tokens
          const int lim = vis[ct] - t0 - 4 * ((again(threadIdx.x) >> 5) & 1);
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (8 * (i >> 2) + (i & 3) >= lim) sacc[ct][i] = -INFINITY;
        }
      }
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        mx[ct] = sacc[ct][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx[ct] = fmaxf(mx[ct], sacc[ct][i]);
        mx[ct] = max_of_halves(mx[ct]);
        grow[ct] = mx[ct] > m_run[ct] + a.lag;
      }
      if (__any(grow[0] || grow[1])) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          const float corr = grow[ct] ? __builtin_amdgcn_exp2f((m_run[ct] - mx[ct]) * a.c2) : 1.0f;
          m_run[ct] = grow[ct] ? mx[ct] : m_run[ct];
          l_run[ct] *= corr;
#pragma unroll
          for (int d = 0; d < DT; ++d) oacc[ct][d] *= corr;
        }
      }
      bf16x8 pf[CT][2];
      const int lv = again(threadIdx.x) & 63;
      const bf16_t* vl = &s_v[buf][(half * 32 + 4 * (lv >> 5) + ((lv & 15) >> 2)) * VS + 16 * (lv >> 4 & 1) + 4 * (lv & 3)];
      float sum[CT][2] = {};
      __builtin_amdgcn_sched_barrier(0);
      {
        constexpr int VA = 2;
        union vfrag { bf16x4 h[2]; bf16x8 v; } vf[2 * DT];
#pragma unroll
        for (int n = 0; n < 2 * DT; ++n)
#pragma unroll
          for (int j = 0; j < 2; ++j) vf[n].h[j] = read_transposed(vl + (n / DT * 16 + j * 8) * VS + n % DT * 32);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int i = 8 * k; i < 8 * k + 8; ++i) {
              const float pe = __builtin_amdgcn_exp2f((sacc[ct][i] - m_run[ct]) * a.c2);
              sum[ct][i & 1] += pe;
              pf[ct][k][i & 7] = (bf16_t)pe;
            }
#pragma unroll
          for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) oacc[ct][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[k * DT + d].v, pf[ct][k], oacc[ct][d], 0, 0, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * VA, 0);
        __builtin_amdgcn_sched_group_barrier(0x2, 56, 0);
#pragma unroll
        for (int n = 0; n < 2 * DT; ++n) {
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            if (n < DT) __builtin_amdgcn_sched_group_barrier(0x2, 7, 0);
          }
          if (n + VA < 2 * DT) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) l_run[ct] += sum[ct][0] + sum[ct][1];
    }
    __syncthreads();
  }
  if (s_nan)                                         // (rare: which columns see it)
#pragma clang loop unroll(disable)
    for (int pg = 0; pg * CACHE_PAGE < t_end - t_begin; ++pg)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) poison[ct] |= nan_blocks<DH>(a, bt[pg], kvh, t_begin + pg * CACHE_PAGE, len, vis[ct]);

  const int n_mine = min(64, n_cols - c_first), lane_o = again(threadIdx.x) & 63, cl_o = lane_o & 31, hf_o = lane_o >> 5;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    unsigned p = poison[ct];
    float l = l_run[ct] + __shfl_xor(l_run[ct], 32, 64);
    if (bad) { l = NAN; p = 15; }
    const int row = ct * 32 + cl_o;
    int i, h;
    head_row(row, i, h);
    const bool whole = vis[ct] <= sp.chunk;
    const int r = first + i, pr = part_row(a, r, b, i);
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    const bool mine = row < n_mine && !(split > 0 && vis[ct] <= t_begin);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int dim = d * 32 + 8 * q + 4 * hf_o;
        f32x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = p >> d & 1 ? NAN : oacc[ct][d][4 * q + e];
        if (mine && !whole) *reinterpret_cast<f32x4*>(part_o<DH>(a, sp.n, split, pr, h) + dim) = o;
        bf16x4 ob;
#pragma unroll
        for (int e = 0; e < 4; ++e) ob[e] = (bf16_t)(o[e] * inv);
        *reinterpret_cast<bf16x4*>(s_mine + row * DH + 8 * swap_piece(row, dim / 8) + 4 * hf_o) = ob;
      }
    if (hf_o == 0 && mine) {
      if (!whole) *reinterpret_cast<float2*>(part_ml(a, split, pr, h)) = float2{l == 0.f ? -INFINITY : m_run[ct], l};
      else if (a.lse != nullptr) a.lse[(size_t)r * a.Hq + h] = l == 0.f ? -INFINITY : (m_run[ct] * a.c2 + log2f(l)) * 0.6931471805599453f;
    }
  }
  asm volatile("" ::: "memory");                     // (LDS serves a wavefront's accesses in their order)
#pragma unroll
  for (int n = 0; n < 64 / RPI; ++n) {
    const int row = n * RPI + lane_o / P, piece = lane_o % P;
    int i, h;
    head_row(row, i, h);
    const int seen_here = len - count + i + 1;
    if (row >= n_mine || seen_here > sp.chunk || (split > 0 && seen_here <= t_begin)) continue;
    *reinterpret_cast<u32x4_8*>(out_at<DH, ENGINE>(a, first + i, h, 8 * piece)) = *reinterpret_cast<const u32x4_8*>(s_mine + row * DH + 8 * swap_piece(row, piece));
  }
}

// Up to 64 columns go to the kernel of few rows, whose wavefronts share out the tokens: with all four on the same 64 columns the other one
// would leave three idle.
int ws_rows(const CacheAttn& a) { return (int)std::min<long long>(a.n_rows, (long long)a.n_seqs * a.max_q); }
bool few_rows(const CacheAttn& a) { return (long long)a.max_q * (a.Hq / a.Hkv) <= 64; }
int row_tiles(const CacheAttn& a) { return (int)(((long long)a.max_q * (a.Hq / a.Hkv) + RA_COLS - 1) / RA_COLS); }

// Splits of the longest context, and the wavefronts that share a split's tiles.  Few rows: 8 wavefronts where the sequences and their KV heads
// leave compute units with one or two workgroups.  A split saves 0.6 to 0.75 us for each of its 128 tokens and 4 wavefronts and costs 0.1 us of
// the join, which takes 2.5 us besides: least in all for about 10 sqrt(length) tokens, until the workgroups fill the chip; from 128 sequences and heads on
// it does not pay below what a workgroup can hold; half of that, up to 1280 workgroups, where the longest context has to be split anyway: with 4096 | 2048 and
// 8 wavefronts 40 of 4000-9000 72 | 66, 30 of 8000-16000 89 | 86, 70 of 1000-9000 with 14 + 2 heads of 64 27 | 20 (but 20 of 1000-4000 23.4 | 24.9,
// 100 of 500-4000 with 14 + 2 heads of 64 17.5 | 18.7).
// us, one row of 32 + 8 heads of 128, 4 wavefronts in splits of 512 | 1024 | 2048 | 4096, 8 in the same (shorter contexts: whole), and by the rule:
//   1 sequence of 300 tokens 6.9, 6.1, 6.1; 1000 10.2 | 10.6, 9.5 | 8.9, 8.9; 2000 10.6 | 13.3 | 17.3, 9.8 | 11.6 | 13.2, 9.8
//     4000 11.3 | 13.7 | 20.1 | 30.3, 10.8 | 11.9 | 16.1 | 21.7, 11.0; 16000 19.0 | 17.8 | 22.4 | 34.8, 19.8 | 16.4 | 18.7 | 26.6, 17.3
//   8 of 1000 10.9, 10.5 | 9.4, 9.4; 4000 16.6 | 15.8 | 21.6 | 31.7, 17.2 | 15.0 | 18.5 | 23.5, 17.5
//   16 of 4000 22.3 | 19.9 | 22.2 | 31.8, 25.8 | 20.5 | 19.6 | 23.4, 23.7
//   20 of 1000 14.5 | 11.6, 15.2 | 10.5, 10.6; 4000 26.3 | 24.5 | 27.4 | 31.9, 30.4 | 25.9 | 26.9 | 24.0, 24.1
//   40 of 40 5.7, 5.9, 5.6; 1000 17.9 | 15.8, 19.7 | 15.5, 15.5; 4000 46.6 | 42.7 | 44.2 | 43.6, 56.8 | 44.7 | 42.8 | 46.1, 46.1
//   40 of 4000-9000 72 | 66 | 68 | 73, 93 | 72 | 66 | 72, 64; 30 of 8000-16000 98 | 88 | 88 | 92, 124 | 95 | 86 | 89, 86
//   192 of 576-4608 129 | 117 | 115 | 118, 173 | 134 | 116 | 111, 116
//   (16 wavefronts, before the last steps: 1 of 4000 11.9 | 12.8 | 20.0 in 512 | 1024 | 4096, 20 of 4000 46 | 37 | 23.5, 40 of 1000 28 | 21.6.)
// Where it is not best: 128 sequences and heads of up to 4096 tokens, whole (16 of 4000: 24 against 20; 40 of 4000: 46 against 43).
//
// Many rows: as many splits as fill the two workgroups that a compute unit holds, none shorter than 256 tokens; of whole prompts, whose
// workgroups see half of the tokens on average, half again as many.  us with 256 | 512 | 1024 | 2048 | 4096 | no splits (32 + 8 heads of 128): 3 sequences of
// 16384 tokens, 300 rows (120 workgroups) 709 | 498 | 383 | 350 | 327 | 858; one of 8000, 100 rows (16) 50 | 51 | 72 | 120 | 222 | 414; whole prompts:
// one of 1000 (128) 45 | 49 | 61, of 2000 (256) 114 | 96 | 95 | 114, 768: 85, four of 1000 (512) 123 | 93 | 74.
Split split_of(const CacheAttn& a) {
  const bool few = few_rows(a);
  const long long groups = std::max<long long>(1, (long long)a.n_seqs * a.Hkv * (few ? 1 : row_tiles(a)));
  const bool joined = groups >= 128 && a.max_len > CA_MOST;
  const int least = !few ? 256 : joined ? CA_MOST / 2 : groups >= 128 ? CA_MOST : a.max_len <= 1152 ? 1152 : ((int)(10 * std::sqrt((double)a.max_len)) + 127) / 128 * 128;
  const long long most = few ? ((joined ? 1280 : 640) + groups - 1) / groups : std::max<long long>(1, (2ll * a.max_q > a.max_len ? 768 : 512) / groups);
  long long n = std::max<long long>(1, std::min<long long>(most, few ? (a.max_len + least - 1) / least : a.max_len / least));
  if (few) n = std::max<long long>(n, (a.max_len + CA_MOST - 1) / CA_MOST);
  Split s;
  s.chunk = (int)std::max<long long>(128, ((a.max_len + n - 1) / n + 127) / 128 * 128);
  if (few) s.chunk = std::min(s.chunk, CA_MOST);
  s.n = std::max(1, (a.max_len + s.chunk - 1) / s.chunk);
  s.waves = groups <= 512 && a.max_len > 128 && (long long)a.max_q * (a.Hq / a.Hkv) <= 32 ? 8 : 4;
  return s;
}

long long attention_groups(const CacheAttn& a, const Split& sp) { return (long long)a.Hkv * a.n_seqs * sp.n * (few_rows(a) ? 1 : row_tiles(a)); }

template <int DH> hipError_t attention(hipStream_t st, CacheAttn a) {
  const Split sp = split_of(a);
  const int n_qt = row_tiles(a);
  const long long cols = (long long)a.max_q * (a.Hq / a.Hkv);
  a.ws_rows = ws_rows(a);
  const dim3 grid((unsigned)attention_groups(a, sp));
  hipError_t e = !few_rows(a) ? launch(cache_attn_rows_kernel<DH, false>, grid, dim3(256), st, a, sp, n_qt, CacheRows{})
                 : cols <= 16 ? (sp.waves == 8 ? launch(cache_attn_kernel<DH, 1, 8, CA_ROWS>, grid, dim3(512), st, a, sp, CacheRows{}, CacheRope{})
                                               : launch(cache_attn_kernel<DH, 1, 4, CA_ROWS>, grid, dim3(256), st, a, sp, CacheRows{}, CacheRope{}))
                 : cols <= 32 ? (sp.waves == 8 ? launch(cache_attn_kernel<DH, 2, 8, CA_ROWS>, grid, dim3(512), st, a, sp, CacheRows{}, CacheRope{})
                                               : launch(cache_attn_kernel<DH, 2, 4, CA_ROWS>, grid, dim3(256), st, a, sp, CacheRows{}, CacheRope{}))
                              : launch(cache_attn_kernel<DH, 4, 4, CA_ROWS>, grid, dim3(256), st, a, sp, CacheRows{}, CacheRope{});
  if (e == hipSuccess && sp.n > 1) e = launch(cache_join_kernel<DH, false>, join_grid<DH>(a, a.n_seqs * a.max_q), dim3(256), st, a, sp, CacheRows{});
  return e;
}

}  // namespace

// Whether the launches of a call are possible: a dimension of a grid has fewer than 2^32 threads, and columns are counted in 31 bits.
bool cache_attention_fits(const CacheAttn& a) {
  if ((long long)a.max_q * (a.Hq / a.Hkv) > (1ll << 31) - RA_COLS) return false;
  // (before splits, in floating point: nothing below this bound overflows)
  if ((double)a.n_seqs * a.Hkv * (few_rows(a) ? 1.0 : (double)row_tiles(a)) * 256 >= 4294967296.0) return false;
  const Split sp = split_of(a);
  return attention_groups(a, sp) * 64 * (few_rows(a) ? sp.waves : 4) < 1ll << 32 && (sp.n == 1 || (long long)a.n_seqs * a.max_q * 256 < 1ll << 32);
}

size_t cache_attention_workspace(const CacheAttn& a, int dh) {
  const Split sp = split_of(a);
  return sp.n > 1 ? (size_t)sp.n * ws_rows(a) * a.Hq * (dh + 2) * sizeof(float) : 0;
}

// The engine's passes: decode iterations over the scheduler's work list, prefill over its tiles of query positions.  Splits have the
// engine's length, whatever the batch, so that a rollout's sums depend on its own length alone.
void launch_cache_decode(hipStream_t st, const CacheAttn& a, int dh, const CacheRows& er, int rows, int chunk, int max_splits, int grid_splits, const CacheRope* f) {
  const Split sp{chunk, max_splits, 4};
  const dim3 grid((unsigned)rows * grid_splits * a.Hkv);
#define CACHE_DECODE(DH)                                                                        \
  if (f != nullptr) launch(cache_attn_kernel<DH, 1, 4, CA_FUSED>, grid, dim3(256), st, a, sp, er, *f);           \
  else launch(cache_attn_kernel<DH, 1, 4, CA_ENGINE>, grid, dim3(256), st, a, sp, er, CacheRope{});                \
  if (grid_splits > 1) launch(cache_join_kernel<DH, true>, join_grid<DH>(a, rows), dim3(256), st, a, sp, er)
  switch (dh) {
    case 32: CACHE_DECODE(32); break;
    case 64: CACHE_DECODE(64); break;
    default: CACHE_DECODE(128); break;
  }
#undef CACHE_DECODE
}
void launch_cache_prefill(hipStream_t st, const CacheAttn& a, int dh, const CacheRows& er, int n_items) {
  if (n_items <= 0) return;
  const Split sp{0x7fffff80, 1, 4};
  const dim3 grid((unsigned)n_items * a.Hkv);
  switch (dh) {
    case 32: launch(cache_attn_rows_kernel<32, true>, grid, dim3(256), st, a, sp, 1, er); break;
    case 64: launch(cache_attn_rows_kernel<64, true>, grid, dim3(256), st, a, sp, 1, er); break;
    default: launch(cache_attn_rows_kernel<128, true>, grid, dim3(256), st, a, sp, 1, er); break;
  }
}

// ---------------------------------------------------------------------------
// The engine's rotary embedding and store where the attention does not do them itself (prompts; APRIL_FUSE_ROPE=0): a workgroup per row.  Sums the projection's partials, rotates the queries (bf16 rows) and
// the key, and stores key and value in the row's page; they meet in LDS, where a block's 32 dimensions lie together.
// ---------------------------------------------------------------------------
namespace {

__global__ __launch_bounds__(256) void cache_rope_kernel(RowCtx rc, Slots s, CacheRope f, int dh, int Hkv) {
  extern __shared__ float s_kv[];                     // [key | value][Hkv * dh]
  const int r = blockIdx.x;
  ROW_GUARD(rc, r);
  const int slot = rc.row_slot[r], pos = rc.row_pos[r], half = dh >> 1, nkv = Hkv * dh;
  const float* cs = f.rope_cos + (size_t)pos * half;
  const float* sn = f.rope_sin + (size_t)pos * half;
  auto value = [&](const float* src, int col) {
    float x = src[col];
    for (int p = 1; p < f.n_partials; ++p) x += src[p * f.partial_stride + col];        // in the order p = 0, 1, ...
    return x;
  };
  const float* q = f.q_src + (size_t)r * f.q_ld;
  const float* kv = f.kv_src + (size_t)r * f.kv_ld;
  for (int e = threadIdx.x; e < (f.Hq + (f.store ? Hkv : 0)) * half; e += 256) {
    const int hd = e / half, i = e - hd * half;
    const float* src = hd < f.Hq ? q + hd * dh : kv + (hd - f.Hq) * dh;
    const float a = value(src, i), b = value(src, i + half), ra = rope_first(a, b, cs[i], sn[i]), rb = rope_second(a, b, cs[i], sn[i]);
    if (hd < f.Hq) {
      bf16_t* to = f.q + ((size_t)r * f.Hq + hd) * dh + i;
      to[0] = (bf16_t)ra;
      to[half] = (bf16_t)rb;
    } else {
      s_kv[(hd - f.Hq) * dh + i] = ra;
      s_kv[(hd - f.Hq) * dh + i + half] = rb;
    }
  }
  if (!f.store) return;
  for (int e = threadIdx.x; e < nkv; e += 256) s_kv[nkv + e] = value(kv, nkv + e);
  __syncthreads();
  const int page = s.block_table[(size_t)slot * s.max_blocks + pos / CACHE_PAGE], tok = pos % CACHE_PAGE;
  unsigned char* base = f.pool + (size_t)page * Hkv * cache_block_bytes(dh);
  // (2 nkv / 8 pieces, a multiple of 4: a block's four lanes take every trip together)
  for (int e = threadIdx.x; e < nkv / 4; e += 256) {
    const int at = e * 8, val = at >= nkv, d = at - val * nkv, head = d / dh, blk = d % dh / 32, part = d % 32 / 8;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = s_kv[at + i];
    unsigned ex;
    const unsigned c = cache_codes(x, ex);
    unsigned char* to = base + (size_t)head * cache_block_bytes(dh);
    *reinterpret_cast<unsigned*>(to + cache_code_off(dh, val, blk, tok) + part * 4) = c;
    if (part == 0) to[cache_scale_off(dh, val, blk, tok)] = (unsigned char)ex;
  }
}

}  // namespace

void launch_cache_rope(hipStream_t st, RowCtx rc, Slots s, const CacheRope& f, int dh, int Hkv) {
  hipLaunchKernelGGL(cache_rope_kernel, dim3(rc.max_rows), dim3(256), f.store ? 2 * Hkv * dh * sizeof(float) : 0, st, rc, s, f, dh, Hkv);
}

hipError_t launch_cache_attention(hipStream_t st, const CacheAttn& a, int dh) {
  return dh == 32 ? attention<32>(st, a) : dh == 64 ? attention<64>(st, a) : attention<128>(st, a);
}

}  // namespace april
