// Operators that score rollouts and train on them, on the caller's tensors: arguments as their kernels take them (see april.h), and the launchers.
#pragma once
#include <type_traits>

#include "kernels.h"

namespace april {

// A launch whose own error comes back (the sticky one of an earlier call is left alone).
template <class... A>
hipError_t enqueue(void (*kernel)(A...), dim3 grid, dim3 block, hipStream_t st, std::common_type_t<A>... args) {
  void* ptrs[] = {&args...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, ptrs, 0, st);
}

__device__ inline long long index_at(const void* p, bool i64, size_t i) {
  return i64 ? static_cast<const long long*>(p)[i] : (long long)static_cast<const int*>(p)[i];
}

// Whether an array of so many bytes is read or written past the last cache (256 MB): whoever reads a result of more than half of it writes as much again and finds little there,
// and its lines are written back among the next kernels' reads.
inline bool streams(long long bytes) { return bytes > (128ll << 20); }

// Element types are template arguments of the kernels; `f32`, `i64` say which one an argument is.
struct Logprobs {
  int n_rows, vocab, n_top;
  bool f32, i64;
  float inv_t, c2;                 // 1 / temperature, log2(e) / temperature
  long long row;
  const void *logits, *tokens;
  float *logprob, *entropy, *lse, *norm, *top_logprobs;
  int* top_ids;
  float* ws;
};
size_t logprobs_workspace(const Logprobs& a);
hipError_t launch_logprobs(hipStream_t st, const Logprobs& a);

struct LogprobsGrad {
  int n_rows, vocab;
  bool f32, i64;
  float inv_t, c2;
  long long row, grad_row;
  const void *logits, *tokens;
  const float *norm, *entropy, *g_logprob, *g_entropy, *g_lse;
  void* grad;
};
hipError_t launch_logprobs_grad(hipStream_t st, const LogprobsGrad& a);

struct Embed {
  int n_rows, vocab, d;
  bool table_f32, out_f32, i64;
  float scale;
  long long table_row, out_row;
  const void *table, *tokens;
  void* out;
};
hipError_t launch_embed(hipStream_t st, const Embed& a);

struct EmbedGrad {
  int n_rows, vocab, d;
  bool out_f32, table_f32, i64, accumulate;
  float scale;
  long long out_row, table_row;
  const void *grad_out, *tokens;
  void *grad_table, *ws;
};
size_t embed_grad_workspace(const EmbedGrad& a);
hipError_t launch_embed_grad(hipStream_t st, const EmbedGrad& a);

struct ExpertSort {
  int n, n_experts, align, n_packed;        // n: rows x experts of a row
  bool i64;
  const void* ids;
  int *starts, *source, *position;
  void* ws;
  // the engine's dispatch: source[p] is the assignment divided by `per_row`, an expert's assignments are counted, and groups[g] is the expert that owns packed rows
  // [g * align, (g + 1) * align), -1 past the end
  int per_row = 1;
  int* counts = nullptr;
  int* groups = nullptr;
  int n_groups = 0;
};
size_t expert_sort_workspace(const ExpertSort& a);
hipError_t launch_expert_sort(hipStream_t st, const ExpertSort& a);

struct ExpertRows {
  int n_rows, k, d, n_packed;
  bool f32;
  long long row, packed_row, grad_row;      // strides of rows in the token's order, of packed rows, of the packed rows' gradient
  const void* rows;                         // x or the gradient of the sums
  const void* packed;                       // what the experts made
  const int *position, *source;
  const float* weights;                     // null: 1
  void *out, *grad_packed;
  float* grad_weights;
};
hipError_t launch_expert_gather(hipStream_t st, const ExpertRows& a);         // out: packed rows
hipError_t launch_expert_combine(hipStream_t st, const ExpertRows& a);        // out: rows in the token's order
hipError_t launch_expert_combine_grad(hipStream_t st, const ExpertRows& a);

}  // namespace april
