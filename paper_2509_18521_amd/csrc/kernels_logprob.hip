// Log-probabilities of given tokens with the row's entropy and its most likely alternatives, and the gradient of the
// logits.  gfx950.
//
// x = logits / T.  With m the row's maximum, s = sum e^(x_j - m) and E = sum e^(x_j - m) (x_j - m):
//   logprob = x_t - m - log s,   entropy = -sum p log p = log s - E / s  (E <= 0: both terms positive, no cancellation),
//   d logits_j = (1/T) [ a (delta_jt - p_j) + z p_j - h p_j (log p_j + entropy) ]   for gradients a, h, z of logprob, entropy
//   and lse = m + log s.
// Kept in powers of two: c2 = log2(e) / T, exponentials are exp2((x - m) c2), E in units of c2.
#include <float.h>

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
__device__ inline void feed(Part& p, float x, float c2) {
  if (x > p.m) rebase(p, x, c2);
  const float d = (x - p.m) * c2, v = exp2f(d);
  p.s += v;
  p.e += v * fmaxf(d, -1e30f);
}

// (in natural units: a mask of the type's lowest value stays finite)
__device__ inline float log_p(float x, float m, float l2, float inv_t) { return (x - m) * inv_t - l2 * LN2; }

constexpr int ROW_THREADS = 1024;
constexpr int ROW_WAVES = ROW_THREADS / 64;

// One workgroup a row.
template <typename T>
__global__ __launch_bounds__(ROW_THREADS) void logprobs_kernel(Logprobs a) {
  __shared__ float red_m[ROW_WAVES], red_s[ROW_WAVES], red_e[ROW_WAVES];
  __shared__ unsigned long long red_k[ROW_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
    const T* row = static_cast<const T*>(a.logits) + (long long)r * a.row;
    const long long tok = index_at(a.tokens, a.i64, r);
    if (tok < 0) {
      if (tid == 0) {
        if (a.logprob) a.logprob[r] = 0.f;
        if (a.entropy) a.entropy[r] = 0.f;
        if (a.lse) a.lse[r] = 0.f;
        if (a.norm) a.norm[2 * (size_t)r] = a.norm[2 * (size_t)r + 1] = 0.f;
      }
      for (int i = tid; i < a.n_top; i += ROW_THREADS) { a.top_logprobs[(size_t)r * a.n_top + i] = 0.f; a.top_ids[(size_t)r * a.n_top + i] = -1; }
      continue;
    }
    Part p;
    for (int i = tid; i < a.vocab; i += ROW_THREADS) feed(p, (float)row[i], a.c2);
    float m = wave_max_f32(p.m);
    if (lane == 0) red_m[wave] = m;
    __syncthreads();
    m = red_m[0];
    for (int w = 1; w < ROW_WAVES; ++w) m = fmaxf(m, red_m[w]);
    rebase(p, m, a.c2);
    const float ws = wave_sum_f32(p.s), we = wave_sum_f32(p.e);
    if (lane == 0) { red_s[wave] = ws; red_e[wave] = we; }
    __syncthreads();
    float s = red_s[0], e = red_e[0];
    for (int w = 1; w < ROW_WAVES; ++w) { s += red_s[w]; e += red_e[w]; }
    const float l2 = log2f(s);
    if (tid == 0) {
      if (a.logprob) a.logprob[r] = tok < a.vocab ? log_p((float)row[tok], m, l2, a.inv_t) : NAN;
      if (a.entropy) a.entropy[r] = (l2 - e / s) * LN2;
      if (a.lse) a.lse[r] = m * a.inv_t + l2 * LN2;
      if (a.norm) { a.norm[2 * (size_t)r] = m; a.norm[2 * (size_t)r + 1] = l2; }
    }
    unsigned long long last = ~0ull;
    for (int k = 0; k < a.n_top; ++k) {                    // the next one below the last, by value and then by index
      unsigned long long best = 0;
      for (int i = tid; i < a.vocab; i += ROW_THREADS) {
        const unsigned long long key = ((unsigned long long)f2key((float)row[i]) << 32) | (unsigned)~i;
        if (key < last && key > best) best = key;
      }
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) {
        const unsigned long long o = __shfl_xor(best, off, 64);
        best = o > best ? o : best;
      }
      __syncthreads();
      if (lane == 0) red_k[wave] = best;
      __syncthreads();
      for (int w = 0; w < ROW_WAVES; ++w) best = red_k[w] > best ? red_k[w] : best;
      last = best;
      if (tid == 0) {
        const int id = ~(int)(unsigned)best;
        const bool bad = !(s > 0.f);
        a.top_ids[(size_t)r * a.n_top + k] = bad ? -1 : id;
        a.top_logprobs[(size_t)r * a.n_top + k] = bad ? NAN : log_p((float)row[id], m, l2, a.inv_t);
      }
    }
    __syncthreads();
  }
}

constexpr int GRAD_THREADS = 256;

template <typename T>
__global__ __launch_bounds__(GRAD_THREADS) void logprobs_grad_kernel(LogprobsGrad a) {
  for (int r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
    const T* row = static_cast<const T*>(a.logits) + (long long)r * a.row;
    T* out = static_cast<T*>(a.grad) + (long long)r * a.grad_row;
    const long long tok = index_at(a.tokens, a.i64, r);
    const float m = a.norm[2 * (size_t)r], l2 = a.norm[2 * (size_t)r + 1];
    float g = a.g_logprob ? a.g_logprob[r] : 0.f;
    const float h = a.g_entropy ? a.g_entropy[r] : 0.f, z = a.g_lse ? a.g_lse[r] : 0.f, ent = a.g_entropy ? a.entropy[r] : 0.f;
    if (tok >= a.vocab) g = NAN;
    for (int i = threadIdx.x; i < a.vocab; i += GRAD_THREADS) {
      float v = 0.f;
      if (tok >= 0) {
        const float lp2 = ((float)row[i] - m) * a.c2 - l2, p = exp2f(lp2);
        v = p * (z - g - h * (fmaxf(lp2, -1e30f) * LN2 + ent));
        if (i == tok) v += g;
        v *= a.inv_t;
      }
      out[i] = (T)v;
    }
  }
}

}  // namespace

size_t logprobs_workspace(const Logprobs&) { return 0; }

hipError_t launch_logprobs(hipStream_t st, const Logprobs& a) {
  const dim3 grid(a.n_rows < (1 << 20) ? a.n_rows : 1 << 20), block(ROW_THREADS);
  return a.f32 ? enqueue(logprobs_kernel<float>, grid, block, st, a) : enqueue(logprobs_kernel<bf16_t>, grid, block, st, a);
}

hipError_t launch_logprobs_grad(hipStream_t st, const LogprobsGrad& a) {
  const dim3 grid(a.n_rows < (1 << 20) ? a.n_rows : 1 << 20), block(GRAD_THREADS);
  return a.f32 ? enqueue(logprobs_grad_kernel<float>, grid, block, st, a) : enqueue(logprobs_grad_kernel<bf16_t>, grid, block, st, a);
}

}  // namespace april
