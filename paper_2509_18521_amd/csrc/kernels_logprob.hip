// Log-probabilities of given tokens with the row's entropy and its most likely alternatives, and the gradient of the
// logits.  gfx950.
//
// x = logits / T.  With m the row's maximum, s = sum e^(x_j - m) and E = sum e^(x_j - m) (x_j - m):
//   logprob = x_t - m - log s,   entropy = -sum p log p = log s - E / s  (E <= 0: both terms positive, no cancellation),
//   d logits_j = (1/T) [ a (delta_jt - p_j) + z p_j - h p_j (log p_j + entropy) ]   for gradients a, h, z of logprob, entropy
//   and lse = m + log s.
// Kept in powers of two: c2 = log2(e) / T, exponentials are exp2((x - m) c2), E in units of c2.
#include <float.h>

#include <algorithm>

#include "train.h"

namespace april {
namespace {

constexpr float LN2 = 0.69314718055994530942f;

template <typename T> struct Vec;
template <> struct Vec<float> { static constexpr int N = 4; typedef f32x4 type; };
template <> struct Vec<bf16_t> { static constexpr int N = 8; typedef bf16x8 type; };

// A part of a row's softmax: m a reference no smaller than -FLT_MAX (so that m - x is no NaN for an x of -infinity), s and e
// relative to it.  A NaN or +infinity among the logits ends in an s of NaN.
struct Part {
  float m = -FLT_MAX, s = 0.f, e = 0.f;
};
// d = (old reference - new one) * c2, kept finite: 0 * infinity would be NaN
__device__ inline void rebase(Part& p, float m, float c2) {
  const float d = fmaxf((p.m - m) * c2, -1e30f), f = exp2f(d);
  p.e = f * (p.e + p.s * d);
  p.s *= f;
  p.m = m;
}
// (in natural units: a mask of the type's lowest value stays finite)
__device__ inline float log_p(float x, float m, float l2, float inv_t) { return (x - m) * inv_t - l2 * LN2; }

// A run of a row's elements as the threads of a workgroup see it: `head` single elements up to the first 16-byte border, vectors, and what is left behind
// them.  The singles are element e of thread e.
template <typename T>
struct Run {
  static constexpr int V = Vec<T>::N;
  const T* p;
  int n, head, nv, singles;
  __device__ Run(const T* p, int n) : p(p), n(n) {
    const int off = (int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
    head = off == 0 ? 0 : min(n, V - off);
    nv = (n - head) / V;
    singles = n - nv * V;
  }
  __device__ int single(int e) const { return e < head ? e : e + nv * V; }      // its place in the run
  __device__ const typename Vec<T>::type* at(int v) const { return reinterpret_cast<const typename Vec<T>::type*>(p + head + (size_t)v * V); }
  template <bool STREAM = false>
  __device__ typename Vec<T>::type vector(int v) const { return STREAM ? __builtin_nontemporal_load(at(v)) : *at(v); }
  __device__ int place(int v) const { return head + v * V; }                    // of a vector's first element
};

// ---------------------------------------------------------------------------
// The scan.  32 elements of a thread at a time (8 vectors of fp32: with 4 in flight 192 rows of 151936 took 29.7 us instead of 27.3; 8 of bf16 spill) share one test whether the running reference still serves: exponents may reach LAG.  (They are rounded
// relative to their size, so the few that make up the sum lose digits by it: with 30 a temperature of 0.6 left the entropy 4e-7 off, with 4 it is 6e-8; 4 costs up
// to 3 % in bf16.)  The largest element is kept apart, and all threads go over to the row's at the end.
// ---------------------------------------------------------------------------
constexpr float LAG = 4.f;

// A thread's vectors of a run in at most 8 sections of this many (a multiple of eight, or four of a short run).
constexpr int SECTIONS = 8;
template <int NT>
__device__ inline int section_vectors(int nv) {
  const int each = (nv + NT * SECTIONS - 1) / (NT * SECTIONS);
  return each <= 4 ? 4 : (each + 7) / 8 * 8;
}

template <typename T, bool ENT, int NT, bool STREAM>
struct Scan {
  static constexpr int V = Vec<T>::N, U = 32 / V;      // vectors of a thread in flight
  Part p;
  float top = -INFINITY;           // the thread's largest element
  float c2;

  __device__ __forceinline__ void add(float x) {
    const float d = (x - p.m) * c2, v = exp2_of(d);
    p.s += v;
    if (ENT) p.e = fmaf(v, fmaxf(d, -1e30f), p.e);
  }
  template <int K>
  __device__ __forceinline__ void feed(const typename Vec<T>::type (&x)[K]) {
    float m = top;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) m = fmaxf(m, (float)x[k][i]);
    top = m;
    if ((m - p.m) * c2 > LAG) rebase(p, m, c2);
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) add((float)x[k][i]);
  }
  // vectors v, v + NT, ... below `end`
  __device__ __forceinline__ void vectors(const Run<T>& r, int v, int end) {
    typedef typename Vec<T>::type vec;
    for (; v + (U - 1) * NT < end; v += U * NT) {
      vec x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = r.template vector<STREAM>(v + u * NT);
      feed(x);
    }
    for (; v < end; v += NT) {
      const vec x[1] = {r.template vector<STREAM>(v)};
      feed(x);
    }
  }
  __device__ __forceinline__ void single(const Run<T>& r, int tid) {
    if (tid >= r.singles) return;
    const float x = (float)r.p[r.single(tid)];
    top = fmaxf(top, x);
    if ((x - p.m) * c2 > LAG) rebase(p, x, c2);
    add(x);
  }
  __device__ __forceinline__ void run(const Run<T>& r, int tid) {
    vectors(r, tid, r.nv);
    single(r, tid);
  }
  // The same, with the largest element of each of the thread's sections left in tops[section][thread].
  template <class S>
  __device__ __forceinline__ void run(const Run<T>& r, int tid, S& sh) {
    const int each = section_vectors<NT>(r.nv) * NT;
    float all = -INFINITY;
    for (int i = 0; i * each < r.nv; ++i) {
      top = -INFINITY;
      vectors(r, i * each + tid, min((i + 1) * each, r.nv));
      sh.tops[i][tid] = top;
      all = fmaxf(all, top);
    }
    top = all;
    single(r, tid);
  }
  __device__ static __forceinline__ float exp2_of(float d) { return __builtin_amdgcn_exp2f(d); }
};

// ---------------------------------------------------------------------------
// The k largest of a run, by value and then by index.  256 groups of threads have a largest element each; where k of those reach a bound, so do k
// elements, and only sections of a thread whose own largest reaches it have candidates: their vectors are read again, one to a thread
// (4 to 40 of 16 bytes in lines of their own: whole threads' vectors instead of sections cost 4096 rows of 128256 in bf16 277 us where these took 226: now 210, and 174 without a search).  The
// bound is searched bit by bit in registers, by every wavefront for itself.  More candidates than the list holds: those above the exact k-th largest of the groups
// (no more than k - 1 groups have any), and then those equal to it in the run's order until there are k; where even the former are too
// many, k passes over the run.
// ---------------------------------------------------------------------------
template <int NT> constexpr int groups = NT < 256 ? NT : 256;
template <int NT> constexpr int max_cand = NT < 256 ? 512 : 2048;

template <int NT>
struct TopShared {
  alignas(16) unsigned group[groups<NT>];
  float tops[SECTIONS][NT];
  unsigned short hot[SECTIONS * NT];      // section * NT + thread
  alignas(16) unsigned long long cand[max_cand<NT> + 8];
  unsigned long long best[NT / 64];
  static_assert(NT == 64 || NT == 256 || NT == 512, "one or two threads a group");
  alignas(8) unsigned char bits[NT];
  int n_hot, n_cand;
};
__device__ inline unsigned long long pair_of(unsigned key, int place) { return ((unsigned long long)key << 32) | (unsigned)~place; }
__device__ inline float key_value(unsigned key) { return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key); }

// The largest bound that k of the wavefront's keys reach (four a lane, of 64 groups x alone; 0 where fewer are there); unless `exact`, one of 16 bits, or one that exactly k reach.
template <int NT>
__device__ inline unsigned bound_of(const uint4& g, int k, bool exact) {
  unsigned t = 0;
  for (unsigned bit = 0x80000000u; bit != (exact ? 0u : 0x8000u); bit >>= 1) {
    const unsigned u = t | bit;
    int n = __popcll(__ballot(g.x >= u));
    if (NT > 64) n += __popcll(__ballot(g.y >= u)) + __popcll(__ballot(g.z >= u)) + __popcll(__ballot(g.w >= u));
    if (n >= k) t = u;
    if (n == k && !exact) break;
  }
  return t;
}

// Candidates: elements whose key is `from` or more, of the sections in the list (all threads call).
template <typename T, int NT>
__device__ void collect(TopShared<NT>& sh, const Run<T>& r, unsigned from) {
  constexpr int V = Vec<T>::N;
  const int n_hot = sh.n_hot, each = section_vectors<NT>(r.nv);
  for (int i = threadIdx.x; i < n_hot * each; i += NT) {
    if (*static_cast<volatile int*>(&sh.n_cand) > max_cand<NT>) break;                 // (more than the list holds: the count does not matter)
    const int h = i / each, at = sh.hot[h], v = ((at / NT) * each + i - h * each) * NT + at % NT;
    if (v >= r.nv) continue;
    const auto x = r.vector(v);
    unsigned key[V], hits = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      key[j] = f2key((float)x[j]);
      hits |= (key[j] >= from ? 1u : 0u) << j;
    }
    if (hits == 0) continue;
    int to = atomicAdd(&sh.n_cand, __popc(hits));
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (hits >> j & 1) {
        if (to < max_cand<NT>) sh.cand[to] = pair_of(key[j], r.place(v) + j);
        ++to;
      }
  }
  if ((int)threadIdx.x < r.singles) {
    const int place = r.single(threadIdx.x);
    const unsigned key = f2key((float)r.p[place]);
    if (key >= from) {
      const int to = atomicAdd(&sh.n_cand, 1);
      if (to < max_cand<NT>) sh.cand[to] = pair_of(key, place);
    }
  }
  __syncthreads();
}

// The candidates equal to `least` in the run's order, `need` of them, behind those that are there (all threads call).
template <typename T, int NT>
__device__ void collect_equal(TopShared<NT>& sh, const Run<T>& r, unsigned least, int need) {
  constexpr int V = Vec<T>::N;
  const int tid = threadIdx.x, lane = tid & 63;
  auto single = [&](int e) {
    if (need <= 0 || f2key((float)r.p[r.single(e)]) != least) return;
    if (tid == 0) sh.cand[sh.n_cand++] = pair_of(least, r.single(e));
    --need;
  };
  for (int e = 0; e < r.head; ++e) single(e);
  for (int v0 = 0; v0 < r.nv && need > 0; v0 += NT) {
    unsigned bits = 0;
    if (v0 + tid < r.nv) {
      const auto x = r.vector(v0 + tid);
#pragma unroll
      for (int i = 0; i < V; ++i) bits |= (f2key((float)x[i]) == least ? 1u : 0u) << i;
    }
    sh.bits[tid] = (unsigned char)bits;
    __syncthreads();
    // every wavefront counts; the first one writes
    unsigned long long b = lane < NT / 8 ? reinterpret_cast<const unsigned long long*>(sh.bits)[lane] : 0ull;
    int before = __popcll(b);
    const int own = before;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int o = __shfl_up(before, off, 64);
      if (lane >= off) before += o;
    }
    const int all = __shfl(before, 63, 64);
    before -= own;
    if (tid < 64) {
      const int base = sh.n_cand;
      for (; b != 0 && before < need; ++before, b &= b - 1) {
        const int bit = __ffsll((long long)b) - 1;
        sh.cand[base + before] = pair_of(least, r.place(v0 + lane * 8 + bit / 8) + bit % 8);
      }
      if (lane == 0) sh.n_cand = base + min(all, need);
    }
    need -= min(all, need);
    __syncthreads();
  }
  for (int e = r.head; e < r.singles; ++e) single(e);
  __syncthreads();
}

// k passes, each for the next one below the last (all threads call).
template <typename T, int NT>
__device__ void collect_one_by_one(TopShared<NT>& sh, const Run<T>& r, int k) {
  const int tid = threadIdx.x;
  unsigned long long last = ~0ull;
  for (int j = 0; j < k; ++j) {
    unsigned long long best = 0;
    for (int i = tid; i < r.n; i += NT) {
      const unsigned long long key = pair_of(f2key((float)r.p[i]), i);
      if (key < last && key > best) best = key;
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
      const unsigned long long o = __shfl_xor(best, off, 64);
      best = o > best ? o : best;
    }
    if ((tid & 63) == 0) sh.best[tid >> 6] = best;
    __syncthreads();
    for (int w = 0; w < NT / 64; ++w) best = sh.best[w] > best ? sh.best[w] : best;
    last = best;
    if (tid == 0) { sh.cand[j] = best; sh.n_cand = j + 1; }
    __syncthreads();
  }
}

// All threads call; the candidates, k of them or more if the run has as many, are complete behind it.  top: the thread's largest element, if it has any.
template <typename T, int NT>
__device__ void find_top(TopShared<NT>& sh, const Run<T>& r, int k, float top, bool any) {
  const int tid = threadIdx.x, lane = tid & 63;
  const unsigned mine = any ? f2key(top) : 0u;
  if (NT <= 256) {
    sh.group[tid] = mine;
  } else {
    const unsigned pair = max(mine, (unsigned)__builtin_amdgcn_update_dpp(0, (int)mine, 0xB1, 0xf, 0xf, false));      // (its neighbour's)
    if ((tid & 1) == 0) sh.group[tid >> 1] = pair;
  }
  if (tid == 0) { sh.n_hot = 0; sh.n_cand = 0; }
  __syncthreads();
  const uint4 g = NT == 64 ? uint4{mine, 0u, 0u, 0u} : reinterpret_cast<const uint4*>(sh.group)[NT == 64 ? 0 : lane];
  unsigned least = bound_of<NT>(g, k, false);
  const int each = section_vectors<NT>(r.nv) * NT;
  for (int i = 0; i * each < r.nv; ++i) {
    const unsigned long long hot = __ballot(i * each + tid < r.nv && f2key(sh.tops[i][tid]) >= least);
    if (hot == 0) continue;
    int at = 0;
    if (lane == 0) at = atomicAdd(&sh.n_hot, __popcll(hot));
    at = __builtin_amdgcn_readfirstlane(at) + __popcll(hot & ((1ull << lane) - 1));
    if (hot >> lane & 1) sh.hot[at] = (unsigned short)(i * NT + tid);
  }
  __syncthreads();
  collect(sh, r, least);
  if (sh.n_cand <= max_cand<NT>) return;
  least = bound_of<NT>(g, k, true);
  __syncthreads();
  if (tid == 0) sh.n_cand = 0;
  __syncthreads();
  collect(sh, r, least + 1);
  const int above = sh.n_cand;
  __syncthreads();
  if (above <= max_cand<NT> - k) collect_equal(sh, r, least, k - above);
  else collect_one_by_one(sh, r, k);
}

// put(rank, candidate) for the k first of n candidates (no two are equal).
// All threads call; the list has room for 7 more.
template <int NT, class F>
__device__ inline void rank_candidates(unsigned long long* cand, int n, int k, F put) {
  const int end = (n + 7) / 8 * 8;
  if ((int)threadIdx.x < end - n) cand[n + threadIdx.x] = 0ull;
  __syncthreads();
  for (int c = threadIdx.x; c < n; c += NT) {
    const unsigned long long own = cand[c];
    int rank = 0;
    for (int j = 0; j < end; j += 8) {
      ulonglong2 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = reinterpret_cast<const ulonglong2*>(cand + j)[i];
#pragma unroll
      for (int i = 0; i < 4; ++i) rank += (x[i].x > own) + (x[i].y > own);
    }
    if (rank < k) put(rank, own);
  }
}

template <int NT>
struct RowShared {
  float m[NT / 64], s[NT / 64], e[NT / 64];
};
// Every thread's part -> the workgroup's, relative to its largest element (all threads call, and have it).
template <bool ENT, int NT>
__device__ inline Part join_threads(RowShared<NT>& sh, Part p, float top, float c2) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float m = wave_max_f32(fmaxf(top, -FLT_MAX));
  if (lane == 0) sh.m[wave] = m;
  __syncthreads();
  m = sh.m[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) m = fmaxf(m, sh.m[w]);
  rebase(p, m, c2);
  const float s = wave_sum_f32(p.s), e = ENT ? wave_sum_f32(p.e) : 0.f;
  if (lane == 0) { sh.s[wave] = s; sh.e[wave] = e; }
  __syncthreads();
  Part all{m, sh.s[0], sh.e[0]};
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) { all.s += sh.s[w]; all.e += sh.e[w]; }
  return all;
}

__device__ inline void padding_row(const Logprobs& a, int r, int tid, int nt) {
  if (tid == 0) {
    if (a.logprob) a.logprob[r] = 0.f;
    if (a.entropy) a.entropy[r] = 0.f;
    if (a.lse) a.lse[r] = 0.f;
    if (a.norm) reinterpret_cast<float2*>(a.norm)[r] = float2{0.f, 0.f};
  }
  for (int i = tid; i < a.n_top; i += nt) { a.top_logprobs[(size_t)r * a.n_top + i] = 0.f; a.top_ids[(size_t)r * a.n_top + i] = -1; }
}
// One thread: the row's numbers.
template <typename T>
__device__ inline void put_row(const Logprobs& a, int r, const T* row, long long tok, const Part& p, float l2) {
  if (a.logprob) a.logprob[r] = tok < a.vocab ? log_p((float)row[tok], p.m, l2, a.inv_t) : NAN;
  if (a.entropy) a.entropy[r] = (l2 - p.e / p.s) * LN2;
  if (a.lse) a.lse[r] = p.m * a.inv_t + l2 * LN2;
  if (a.norm) reinterpret_cast<float2*>(a.norm)[r] = float2{p.m, l2};
}
__device__ inline void put_top(const Logprobs& a, int r, int rank, unsigned long long cand, const Part& p, float l2) {
  a.top_ids[(size_t)r * a.n_top + rank] = (int)~(unsigned)cand;
  a.top_logprobs[(size_t)r * a.n_top + rank] = log_p(key_value((unsigned)(cand >> 32)), p.m, l2, a.inv_t);
}
// A row with a NaN, +infinity or nothing but -infinity has no alternatives.
__device__ inline bool no_top(const Logprobs& a, int r, const Part& p, int tid, int nt) {
  if (p.s > 0.f) return false;
  for (int i = tid; i < a.n_top; i += nt) { a.top_logprobs[(size_t)r * a.n_top + i] = NAN; a.top_ids[(size_t)r * a.n_top + i] = -1; }
  return true;
}

// One workgroup a row, one pass over it.  Bound by HBM: 12288 rows of 151936 in bf16 544 us (6.9 TB/s), 192 in fp32 27
// (4.3; 22 where they lie in the last cache).  Registers before wavefronts: with 8 a SIMD the scan of bf16 spills, and 8192 rows of 128256 take 389 us instead of 350 (before
// their loads were streamed).
template <typename T, bool ENT, bool TOP, int NT, bool STREAM>
__global__ __launch_bounds__(NT, 5) void logprobs_kernel(Logprobs a) {
  __shared__ RowShared<NT> sh;
  __shared__ std::conditional_t<TOP, TopShared<NT>, int> st;
  const int tid = threadIdx.x;
  for (long long at = blockIdx.x; at < a.n_rows; at += gridDim.x) {      // (a row past the last may have a number beyond 2^31)
    const int r = (int)at;
    const T* row = static_cast<const T*>(a.logits) + (long long)r * a.row;
    const long long tok = index_at(a.tokens, a.i64, r);
    if (tok < 0) {
      padding_row(a, r, tid, NT);
      continue;
    }
    const Run<T> run(row, a.vocab);
    Scan<T, ENT, NT, STREAM> scan;
    scan.c2 = a.c2;
    if constexpr (TOP) scan.run(run, tid, st);
    else scan.run(run, tid);
    const Part p = join_threads<ENT, NT>(sh, scan.p, scan.top, a.c2);
    const float l2 = log2f(p.s);
    if (tid == 0) put_row(a, r, row, tok, p, l2);
    if constexpr (TOP) {
      if (!no_top(a, r, p, tid, NT)) {
        find_top<T, NT>(st, run, a.n_top, scan.top, tid < run.nv || tid < run.singles);
        rank_candidates<NT>(st.cand, min(st.n_cand, max_cand<NT>), a.n_top, [&](int rank, unsigned long long c) { put_top(a, r, rank, c, p, l2); });
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Few rows: `parts` workgroups a row, each with a run of its vectors (the first with the singles before, the last with those behind), and a second
// launch that joins them.  Of the workspace a part has its m, s, e and then its candidates.
// ---------------------------------------------------------------------------
__host__ __device__ constexpr int part_words(int n_top) { return 4 + 2 * n_top; }      // (a multiple of 8 bytes)

template <typename T, bool ENT, bool TOP, int NT>
__global__ __launch_bounds__(NT, 8) void logprobs_part_kernel(Logprobs a, int parts) {
  __shared__ RowShared<NT> sh;
  __shared__ std::conditional_t<TOP, TopShared<NT>, int> st;
  const int tid = threadIdx.x, r = blockIdx.x / parts, part = blockIdx.x - r * parts;
  const T* row = static_cast<const T*>(a.logits) + (long long)r * a.row;
  if (index_at(a.tokens, a.i64, r) < 0) return;
  const Run<T> whole(row, a.vocab);
  const int v0 = (int)((long long)whole.nv * part / parts), v1 = (int)((long long)whole.nv * (part + 1) / parts);
  const int from = part == 0 ? 0 : whole.place(v0), to = part == parts - 1 ? a.vocab : whole.place(v1);
  const Run<T> run(row + from, to - from);
  Scan<T, ENT, NT, false> scan;
  scan.c2 = a.c2;
  if constexpr (TOP) scan.run(run, tid, st);
  else scan.run(run, tid);
  const Part p = join_threads<ENT, NT>(sh, scan.p, scan.top, a.c2);
  float* out = a.ws + (size_t)blockIdx.x * part_words(a.n_top);
  if (tid == 0) { out[0] = p.m; out[1] = p.s; out[2] = p.e; }
  if constexpr (TOP) {
    find_top<T, NT>(st, run, a.n_top, scan.top, tid < run.nv || tid < run.singles);
    const int n = min(st.n_cand, max_cand<NT>);
    unsigned long long* cand = reinterpret_cast<unsigned long long*>(out + 4);
    for (int i = n + tid; i < a.n_top; i += NT) cand[i] = 0ull;
    // (places count from the row's first element on; the order of equal values stays)
    rank_candidates<NT>(st.cand, n, a.n_top, [&](int rank, unsigned long long c) { cand[rank] = pair_of((unsigned)(c >> 32), (int)~(unsigned)c + from); });
  }
}

constexpr int JOIN_THREADS = 256, MAX_PARTS = 32, MAX_JOIN = 512;

// The parts' candidates are in descending order.  Each part has `depth` elements no smaller than its depth-th, so where parts x depth is n_top or
// more, nothing below the smallest of those is among the n_top largest.
template <typename T>
__global__ __launch_bounds__(JOIN_THREADS) void logprobs_join_kernel(Logprobs a, int parts) {
  __shared__ alignas(16) unsigned long long cand[MAX_JOIN + 8];
  __shared__ unsigned long long least;
  __shared__ int n_cand;
  const int tid = threadIdx.x, r = blockIdx.x;
  const T* row = static_cast<const T*>(a.logits) + (long long)r * a.row;
  const long long tok = index_at(a.tokens, a.i64, r);
  if (tok < 0) {
    padding_row(a, r, tid, JOIN_THREADS);
    return;
  }
  const int words = part_words(a.n_top), lane = tid & 63;
  const float* in = a.ws + (size_t)r * parts * words;
  auto entry = [&](int part, int i) { return reinterpret_cast<const unsigned long long*>(in + (size_t)part * words + 4)[i]; };
  Part p;
  if (lane < parts) p = Part{in[lane * words], in[lane * words + 1], in[lane * words + 2]};
  if (tid == 0) { n_cand = 0; least = ~0ull; }
  __syncthreads();
  if (a.n_top > 0 && tid < parts) atomicMin(&least, entry(tid, (a.n_top + parts - 1) / parts - 1));
  rebase(p, wave_max_f32(p.m), a.c2);
  p.s = wave_sum_f32(p.s);
  p.e = wave_sum_f32(p.e);
  const float l2 = log2f(p.s);
  if (tid == 0) put_row(a, r, row, tok, p, l2);
  if (no_top(a, r, p, tid, JOIN_THREADS)) return;
  __syncthreads();
  for (int i = tid; i < parts * a.n_top; i += JOIN_THREADS) {
    const unsigned long long c = entry(i / a.n_top, i % a.n_top);
    if (c != 0ull && c >= least) cand[atomicAdd(&n_cand, 1)] = c;
  }
  __syncthreads();
  rank_candidates<JOIN_THREADS>(cand, n_cand, a.n_top, [&](int rank, unsigned long long c) { put_top(a, r, rank, c, p, l2); });
}

// Workgroups a row is shared out between: about 256 for the call (one a compute unit), from 16 KB of a row on for each, and no more than 512 candidates a row
// in the second launch.  us unshared | so, without, with 5 and with 64 alternatives: 16 rows of 151936 in fp32 14.6 | 7.9, 17.8 | 12.4, 20.9 | 16.7; 48 rows 15.9 | 10.1, 19.1 | 17.0, 22.2 | 21.3; 64
// 18.4 | 12.1, 20.8 | 19.6, 24.0 | 22.9; 128 19.4 | 19.0, 21.6 | 22.1, 25.0 | 25.7; of 128256 in bf16 16 rows 12.2 | 6.6, 17.4 | 11.8, 19.7 | 15.3; 64 12.3 | 9.0, 17.5 | 13.4, 19.9 | 16.5; 128 14.5 | 13.0,
// 19.0 | 17.0, 21.6 | 20.3.  Three parts lose with alternatives in fp32: 96 rows of 151936 18.9 | 16.6, but 21.3 | 24.6 and 24.7 | 28.3 (in two parts 20.1 and 23.6; sections of four vectors, as three parts have them, are loaded
// one at a time).  192 rows in two parts without: 22.2 | 24.0; 16 rows with 64 alternatives in 8 parts 14.5, in 32 19.8.
int row_parts(const Logprobs& a) {
  if (a.n_rows > 128) return 1;
  const long long bytes = (long long)a.vocab * (a.f32 ? 4 : 2);
  long long parts = std::min<long long>((255 + a.n_rows) / a.n_rows, bytes >> 14);
  if (a.n_top > 0) parts = std::min<long long>(parts, MAX_JOIN / a.n_top);
  return (int)std::max<long long>(1, std::min<long long>(parts, MAX_PARTS));
}

template <typename T, bool ENT, bool TOP>
hipError_t logprobs(hipStream_t st, const Logprobs& a) {
  const int parts = row_parts(a);
  if (parts == 1) {
    const dim3 grid(std::min(a.n_rows, 1 << 20));
    // (streaming loads: 8192 rows of 128256 in bf16 348 -> 325 us; what the last cache holds may lie there already, and still when the gradient reads it again)
    const bool stream = streams((long long)a.n_rows * a.vocab * (long long)sizeof(T) / 2);
    auto rows = [&](auto kernel, auto streaming, int nt) { return enqueue(stream ? streaming : kernel, grid, dim3(nt), st, a); };
    // Short rows, a wavefront a row where there are many (us of workgroups of 64 | 256 threads: 16384 rows of 5000 in bf16 with 20 alternatives 51 | 118, of 512 in fp32 without 9.6 | 19,
    // 2048 of 16000 in bf16 with 32 alternatives 25.6 | 26.4; 1024 of them 21.5 | 14.7).  With more than 32 alternatives the largest elements of 64 lanes are no bound to speak of.
    const long long bytes = (long long)a.vocab * sizeof(T);
    if (a.n_rows >= 2048 && a.n_top <= 32 && bytes < (TOP ? 32 << 10 : 4 << 10)) return rows(logprobs_kernel<T, ENT, TOP, 64, false>, logprobs_kernel<T, ENT, TOP, 64, true>, 64);
    // (workgroups of 256 | 512 threads: 4096 rows of 5000 in bf16 11.2 | 15.5 us, of 32003 with 20 alternatives 73 | 100, of 128256 with 20 307 | 277, of 151936 in fp32 440 | 432)
    if (bytes < (128 << 10)) return rows(logprobs_kernel<T, ENT, TOP, 256, false>, logprobs_kernel<T, ENT, TOP, 256, true>, 256);
    return rows(logprobs_kernel<T, ENT, TOP, 512, false>, logprobs_kernel<T, ENT, TOP, 512, true>, 512);
  }
  const hipError_t e = enqueue(logprobs_part_kernel<T, ENT, TOP, 512>, dim3(a.n_rows * parts), dim3(512), st, a, parts);
  return e == hipSuccess ? enqueue(logprobs_join_kernel<T>, dim3(a.n_rows), dim3(JOIN_THREADS), st, a, parts) : e;
}

// ---------------------------------------------------------------------------
// Gradient: one pass, every element by itself.  A workgroup takes four vectors a thread of one row.  Bound by HBM: 16384 rows of 151936 in bf16, a quarter of
// them padding (not read), 1527 us (5.7 TB/s).
// ---------------------------------------------------------------------------
constexpr int GRAD_THREADS = 256, GRAD_VECS = 4;

template <typename T, bool ENT>
struct GradRow {
  float m, c2, l2, q, hl, add, inv_t, none;
  // d logits = (p * (q + hl * log2 p) + `add` at the token) / T.  The temperature comes last: gradients over a small one may be infinite, their difference and their product with a p of 0 are not.
  // Where p is 0, log2 p may be -infinity: `none`, which is 0 for finite gradients.  (A p above 0 keeps hl * log2 p finite for gradients of the entropy up to 3e36.)
  __device__ __forceinline__ float operator()(float x, float at_token = 0.f) const {
    const float lp = (x - m) * c2 - l2, p = __builtin_amdgcn_exp2f(lp);
    return ((p == 0.f ? none : ENT ? p * fmaf(hl, lp, q) : p * q) + at_token) * inv_t;
  }
};

template <typename T, bool ENT, bool STREAM>
__global__ __launch_bounds__(GRAD_THREADS) void logprobs_grad_kernel(LogprobsGrad a, int chunks) {
  typedef typename Vec<T>::type vec;
  typedef vec at_element __attribute__((aligned(sizeof(T))));     // (grad's rows may lie to a 16-byte border otherwise than the logits')
  constexpr int V = Vec<T>::N;
  const long long items = (long long)a.n_rows * chunks;
  for (long long item = blockIdx.x; item < items; item += gridDim.x) {
    const int r = (int)(item / chunks), chunk = (int)(item - (long long)r * chunks);
    const T* row = static_cast<const T*>(a.logits) + (long long)r * a.row;
    T* out = static_cast<T*>(a.grad) + (long long)r * a.grad_row;
    const long long tok = index_at(a.tokens, a.i64, r);
    const bool pad = tok < 0;
    const float2 norm = reinterpret_cast<const float2*>(a.norm)[r];
    const float g = tok < a.vocab ? (a.g_logprob ? a.g_logprob[r] : 0.f) : NAN, z = a.g_lse ? a.g_lse[r] : 0.f;
    const float h = ENT ? a.g_entropy[r] : 0.f, ent = ENT ? a.entropy[r] : 0.f;
    const GradRow<T, ENT> f{norm.x, a.c2, norm.y, z - g - h * ent, -h * LN2, g, a.inv_t, 0.f + (g * 0.f + (h * 0.f + z * 0.f))};
    auto single = [&](int i) {
      const float v = pad ? 0.f : f((float)row[i], i == tok ? f.add : 0.f);
      out[i] = (T)v;
    };
    const Run<T> run(row, a.vocab);
    T* to = out + run.head;
    const int v0 = chunk * (GRAD_THREADS * GRAD_VECS) + threadIdx.x;
    vec x[GRAD_VECS];
    if (!pad) {
#pragma unroll
      for (int u = 0; u < GRAD_VECS; ++u)
        if (v0 + u * GRAD_THREADS < run.nv) x[u] = run.template vector<STREAM>(v0 + u * GRAD_THREADS);
    }
#pragma unroll
    for (int u = 0; u < GRAD_VECS; ++u) {
      const int v = v0 + u * GRAD_THREADS;
      if (v >= run.nv) break;
      vec y{};
      if (!pad) {
        const long long at = tok - run.place(v);
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = (T)f((float)x[u][i]);
        if (at >= 0 && at < V) {
#pragma unroll
          for (int i = 0; i < V; ++i)
            if (i == at) y[i] = (T)f((float)x[u][i], f.add);
        }
      }
      at_element* place = reinterpret_cast<at_element*>(to + (size_t)v * V);
      if (STREAM) __builtin_nontemporal_store(y, place);
      else *place = y;
    }
    if (chunk == 0 && (int)threadIdx.x < run.singles) single(run.single(threadIdx.x));
  }
}

template <typename T, bool ENT>
hipError_t logprobs_grad(hipStream_t st, const LogprobsGrad& a) {
  const int per = GRAD_THREADS * GRAD_VECS * Vec<T>::N, chunks = std::max(1, (a.vocab - 1) / per + 1);
  const dim3 grid((unsigned)std::min<long long>((long long)a.n_rows * chunks, 1 << 22));
  // (streaming accesses: 16384 rows of 151936 in bf16, a quarter of them padding, 1570 -> 1520 us, and 740 -> 650 for the
  // forward pass behind it)
  const bool stream = streams((long long)a.n_rows * a.vocab * (long long)sizeof(T));
  return enqueue(stream ? logprobs_grad_kernel<T, ENT, true> : logprobs_grad_kernel<T, ENT, false>, grid, dim3(GRAD_THREADS), st, a, chunks);
}

}  // namespace

size_t logprobs_workspace(const Logprobs& a) {
  const int parts = a.n_rows > 0 ? row_parts(a) : 1;
  return parts > 1 ? (size_t)a.n_rows * parts * part_words(a.n_top) * 4 : 0;
}

hipError_t launch_logprobs(hipStream_t st, const Logprobs& a) {
  const bool ent = a.entropy != nullptr, top = a.n_top > 0;
  auto of = [&](auto t) {
    typedef decltype(t) T;
    if (top) return ent ? logprobs<T, true, true>(st, a) : logprobs<T, false, true>(st, a);
    return ent ? logprobs<T, true, false>(st, a) : logprobs<T, false, false>(st, a);
  };
  return a.f32 ? of(float{}) : of(bf16_t{});
}

hipError_t launch_logprobs_grad(hipStream_t st, const LogprobsGrad& a) {
  const bool ent = a.g_entropy != nullptr;
  if (a.f32) return ent ? logprobs_grad<float, true>(st, a) : logprobs_grad<float, false>(st, a);
  return ent ? logprobs_grad<bf16_t, true>(st, a) : logprobs_grad<bf16_t, false>(st, a);
}

}  // namespace april
