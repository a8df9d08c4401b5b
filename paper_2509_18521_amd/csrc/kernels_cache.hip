// Kernels of the 4-bit KV cache (gfx950): tables from request lengths, the store, the attention that reads it.
#include <tuple>

#include "cache.h"

namespace april {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <typename... P, typename... A>
hipError_t launch(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t st, A... args) {
  std::tuple<P...> held{static_cast<P>(args)...};
  void* ptrs[sizeof...(P)];
  std::apply([&](auto&... x) { int i = 0; ((ptrs[i++] = (void*)&x), ...); }, held);
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, ptrs, 0, st);
}

// ---------------------------------------------------------------------------
// Tables.  One workgroup: lengths -> exclusive sums over the sequences of pages given back, pages lacked and rows gained;
// then the verdict (nothing has been written yet), then the items of each kind, dealt to the threads flat: an item finds its sequence
// by a binary search in the sums.  Latency is all there is.
// ---------------------------------------------------------------------------
constexpr int EXT_THREADS = 1024;

// exclusive sum over the workgroup; total: of all of it
template <typename I>
__device__ I block_scan(I v, I* s_wave, I& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  I x = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const I y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  if (lane == 63) s_wave[wave] = x;
  __syncthreads();
  I base = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < EXT_THREADS / 64; ++w) {
    const I s = s_wave[w];
    if (w < wave) base += s;
    total += s;
  }
  __syncthreads();
  return base + x - v;
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

// I: int where no sum can pass 31 bits, else long long.  rows: the rows' slots too (else cache_rows_kernel).
template <typename I>
__global__ __launch_bounds__(EXT_THREADS) void cache_extend_kernel(CacheExtend a, int rows) {
  __shared__ I s_wave[EXT_THREADS / 64], s_rel[EXT_THREADS], s_lack[EXT_THREADS], s_row[EXT_THREADS];
  __shared__ int s_len[EXT_THREADS];
  const int tid = threadIdx.x, n_chunks = (a.n_seqs + EXT_THREADS - 1) / EXT_THREADS;
  const int top = *a.free_top;
  const long long cap = (long long)a.max_pages * CACHE_PAGE;
  I rel, lack, row, t_rel, t_lack, t_row;           // this thread's sequence: sums before it in its chunk; the chunk's totals
  int len, add;
  bool bad;
  auto scan = [&](int chunk) {
    const int b = chunk * EXT_THREADS + tid;
    len = b < a.n_seqs ? a.lens[b] : 0;
    add = b < a.n_seqs ? a.new_lens[b] : 0;
    bad = len < 0 || len > cap || (add > 0 && (long long)len + add > cap);
    const int held = bad ? 0 : (len + CACHE_PAGE - 1) / CACHE_PAGE;
    const int want = bad || add < 0 ? 0 : (int)(((long long)len + add + CACHE_PAGE - 1) / CACHE_PAGE);
    rel = block_scan<I>(!bad && add < 0 ? held : 0, s_wave, t_rel);
    lack = block_scan<I>(want > held ? want - held : 0, s_wave, t_lack);
    row = block_scan<I>(bad || add < 0 ? 0 : add, s_wave, t_row);
    s_rel[tid] = rel; s_lack[tid] = lack; s_row[tid] = row; s_len[tid] = len;
    __syncthreads();
  };
  I all_rel = 0, all_lack = 0, all_row = 0;
  int any_bad = 0;
  for (int c = 0; c < n_chunks; ++c) {
    scan(c);
    any_bad |= __syncthreads_or(bad);
    all_rel += t_rel; all_lack += t_lack; all_row += t_row;
  }
  const long long have = (long long)top + all_rel;
  int status = 0;
  if (any_bad || all_row > a.n_rows || top < 0 || have > a.n_pages) status = 2;
  else if (all_lack > have) status = 1;
  if (tid == 0) {
    *a.status = status;
    *a.free_top_out = status ? top : (int)(have - all_lack);
    a.q_start[0] = 0;
  }
  I base = 0;
  for (int c = 0; c < n_chunks; ++c) {              // lengths, first rows, pages given back
    if (n_chunks > 1) scan(c);
    const int b = c * EXT_THREADS + tid;
    if (status == 0) {
      const int n = min(EXT_THREADS, a.n_seqs - c * EXT_THREADS);
      for (I k = tid; k < t_rel; k += EXT_THREADS) {
        const int s = find_in(s_rel, n, k);
        a.free_pages[top + base + k] = a.block_table[(size_t)(c * EXT_THREADS + s) * a.table_stride + (size_t)(k - s_rel[s])];
      }
      base += t_rel;
    }
    if (n_chunks > 1) __syncthreads();               // the sums are used up
  }
  __syncthreads();
  base = 0;
  I row_base = 0;
  for (int c = 0; c < n_chunks; ++c) {              // pages taken
    if (n_chunks > 1) scan(c);
    const int b = c * EXT_THREADS + tid, n = min(EXT_THREADS, a.n_seqs - c * EXT_THREADS);
    if (b < a.n_seqs) {
      a.lens_out[b] = status ? len : (add < 0 ? 0 : len + add);
      a.q_start[b + 1] = status ? 0 : (int)(row_base + row + (add < 0 ? 0 : add));
    }
    if (status == 0) {
      for (I k = tid; k < t_lack; k += EXT_THREADS) {
        const int s = find_in(s_lack, n, k);
        a.block_table[(size_t)(c * EXT_THREADS + s) * a.table_stride + (s_len[s] + CACHE_PAGE - 1) / CACHE_PAGE + (size_t)(k - s_lack[s])] =
            a.free_pages[have - 1 - (base + k)];
      }
      if (rows) {
        __syncthreads();
        for (I k = tid; k < t_row; k += EXT_THREADS) {
          const int s = find_in(s_row, n, k), pos = s_len[s] + (int)(k - s_row[s]);
          put_row(a, (int)(row_base + k), a.block_table[(size_t)(c * EXT_THREADS + s) * a.table_stride + pos / CACHE_PAGE], pos);
        }
      }
      base += t_lack;
      row_base += t_row;
    }
    if (n_chunks > 1) __syncthreads();
  }
  if (rows)
    for (int r = (status ? 0 : (int)all_row) + tid; r < a.n_rows; r += EXT_THREADS) put_row(a, r, -1, 0);
}

// The slots of many rows, one thread each, from what the kernel above has left.
__global__ __launch_bounds__(256) void cache_rows_kernel(CacheExtend a) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r >= a.n_rows) return;
  if (r >= a.q_start[a.n_seqs]) { put_row(a, r, -1, 0); return; }
  const int b = find_in(a.q_start, a.n_seqs, r);
  const int pos = a.lens_out[b] - (a.q_start[b + 1] - r);
  put_row(a, r, a.block_table[(size_t)b * a.table_stride + pos / CACHE_PAGE], pos);
}

}  // namespace

hipError_t launch_cache_extend(hipStream_t st, const CacheExtend& a) {
  const bool rows = a.n_rows <= 4096;
  const bool small = (long long)a.n_seqs * a.max_pages * CACHE_PAGE < (1ll << 30);
  hipError_t e = small ? launch(cache_extend_kernel<int>, dim3(1), dim3(EXT_THREADS), st, a, rows ? 1 : 0)
                       : launch(cache_extend_kernel<long long>, dim3(1), dim3(EXT_THREADS), st, a, rows ? 1 : 0);
  if (e == hipSuccess && !rows) e = launch(cache_rows_kernel, dim3((a.n_rows + 255) / 256), dim3(256), st, a);
  return e;
}

// ---------------------------------------------------------------------------
// Store.  A wavefront takes 16 rows of one (head, block of 32): 4 lanes to a row, 8 dimensions each, keys then values.
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

template <typename T, bool VEC>
__device__ inline void load8(const T* p, float (&x)[8]) {
  if constexpr (!VEC) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)p[i];
  } else if constexpr (sizeof(T) == 2) {
    const bf16x8 v = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
  } else {
    const f32x4 u = *reinterpret_cast<const f32x4*>(p), v = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = u[i]; x[4 + i] = v[i]; }
  }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheAppend a) {
  const int nb = a.dh / 32;
  const int unit = blockIdx.y * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (unit >= a.Hkv * nb) return;
  const int r = blockIdx.x * 16 + (lane >> 2), part = lane & 3, head = unit / nb, blk = unit % nb;
  if (r >= a.n_rows) return;
  const long long slot = a.slot_map[r];
  if (slot < 0 || slot >= (long long)a.n_pages * CACHE_PAGE) return;
  const int tok = (int)(slot % CACHE_PAGE);
  unsigned char* page = a.pool + ((size_t)(slot / CACHE_PAGE) * a.Hkv + head) * cache_block_bytes(a.dh);
  float x[2][8];
  load8<T, VEC>(reinterpret_cast<const T*>(a.k) + r * a.k_row + head * a.k_head + blk * 32 + part * 8, x[0]);
  load8<T, VEC>(reinterpret_cast<const T*>(a.v) + r * a.v_row + head * a.v_head + blk * 32 + part * 8, x[1]);
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    unsigned e;
    const unsigned c = cache_codes(x[q], e);
    *reinterpret_cast<unsigned*>(page + cache_code_off(a.dh, q, blk, tok) + part * 4) = c;
    if (part == 0) page[cache_scale_off(a.dh, q, blk, tok)] = (unsigned char)e;
    void* values = q ? a.v_values : a.k_values;
    if (values == nullptr) continue;
    const bf16x8 v = cache_open(c, e);
    T* dst = reinterpret_cast<T*>(values) + ((size_t)r * a.Hkv + head) * a.dh + blk * 32 + part * 8;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<bf16x8*>(dst) = v;
    else {
#pragma unroll
      for (int i = 0; i < 8; i += 4) *reinterpret_cast<f32x4*>(dst + i) = f32x4{(float)v[i], (float)v[i + 1], (float)v[i + 2], (float)v[i + 3]};
    }
  }
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
// Attention, simple form: a wavefront per (row, query head), a token per trip, online softmax.
// ---------------------------------------------------------------------------
namespace {

__device__ inline float cache_value(const unsigned char* page, int dh, int value, int tok, int d) {
  const unsigned byte = page[cache_code_off(dh, value, d / 32, tok) + (d % 32) / 2];
  const unsigned e = page[cache_scale_off(dh, value, d / 32, tok)];
  const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(byte, __uint_as_float(e << 23), 0);
  return (float)p[d & 1];
}

__global__ __launch_bounds__(64) void cache_attn_simple_kernel(CacheAttn a, int dh) {
  const int b = blockIdx.x / a.max_q, i = blockIdx.x % a.max_q, h = blockIdx.y, lane = threadIdx.x;
  const int first = a.q_start != nullptr ? a.q_start[b] : b, c = a.q_start != nullptr ? a.q_start[b + 1] - first : 1, r = first + i;
  if (first < 0 || i >= c || r >= a.n_rows) return;
  const int len = a.lens[b];
  bool bad = len < 0 || len > a.max_len;
  const int seen = bad ? 0 : min(len, len - c + i + 1), kvh = h / (a.Hq / a.Hkv);
  const bf16_t* q = a.q + r * a.q_row + h * a.q_head;
  const bool has0 = lane < dh, has1 = lane + 64 < dh;
  const float q0 = has0 ? (float)q[lane] : 0.f, q1 = has1 ? (float)q[lane + 64] : 0.f;
  float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
  if (!bad)
    for (int p = 0; p * CACHE_PAGE < len; ++p) bad |= (unsigned)a.block_table[(size_t)b * a.table_stride + p] >= (unsigned)a.n_pages;
  if (!bad)
    for (int t = 0; t < seen; ++t) {
      const unsigned char* page = a.pool + ((size_t)a.block_table[(size_t)b * a.table_stride + t / CACHE_PAGE] * a.Hkv + kvh) * cache_block_bytes(dh);
      float part = 0.f;
      if (has0) part += q0 * cache_value(page, dh, 0, t % CACHE_PAGE, lane);
      if (has1) part += q1 * cache_value(page, dh, 0, t % CACHE_PAGE, lane + 64);
      for (int d = 32; d; d >>= 1) part += __shfl_xor(part, d, 64);
      const float s = part * a.c2, m_new = fmaxf(m, s);
      const float corr = m == -INFINITY ? 0.f : exp2f(m - m_new), w = exp2f(s - m_new);
      l = l * corr + w;
      o0 = o0 * corr + w * (has0 ? cache_value(page, dh, 1, t % CACHE_PAGE, lane) : 0.f);
      o1 = o1 * corr + w * (has1 ? cache_value(page, dh, 1, t % CACHE_PAGE, lane + 64) : 0.f);
      m = m_new;
    }
  const float inv = bad ? NAN : (l == 0.f ? 0.f : 1.0f / l);
  bf16_t* out = a.out + r * a.out_row + h * a.out_head;
  if (has0) out[lane] = (bf16_t)(o0 * inv);
  if (has1) out[lane + 64] = (bf16_t)(o1 * inv);
  if (a.lse != nullptr && lane == 0) a.lse[(size_t)r * a.Hq + h] = bad ? NAN : (l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f);
}

}  // namespace

size_t cache_attention_workspace(const CacheAttn&, int) { return 0; }

hipError_t launch_cache_attention(hipStream_t st, const CacheAttn& a, int dh) {
  return launch(cache_attn_simple_kernel, dim3(a.n_seqs * a.max_q, a.Hq), dim3(64), st, a, dh);
}

}  // namespace april
