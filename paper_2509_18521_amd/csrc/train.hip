// C entry points of the operators that score rollouts and train on them: the arguments' checks, then the launch.  They need no context.
#include <cmath>
#include <limits>

#include "../../include/april.h"
#include "train.h"

using namespace april;

namespace {

#define REFUSE(...) return fail_no_ctx(APRIL_EINVAL, __VA_ARGS__)

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
bool dtype_ok(int t) { return t == APRIL_DTYPE_FP32 || t == APRIL_DTYPE_BF16; }
bool bits_ok(int b) { return b == 32 || b == 64; }
size_t element(int t) { return t == APRIL_DTYPE_FP32 ? 4 : 2; }
int launched(const char* name, hipError_t e) {
  return e == hipSuccess ? APRIL_OK : fail_no_ctx(APRIL_EDEVICE, "%s: launch failed: %s", name, hipGetErrorString(e));
}

// Rows of `len` elements of `size` bytes, `row` elements apart.
struct Rows {
  const void* p;
  int64_t n, row, len;
  size_t size;
  int64_t step() const { return n > 1 ? row : 0; }
};
bool rows_overlap(const Rows& a) { return a.n > 1 && a.row > -a.len && a.row < a.len; }
// Whether the two share a byte; where the strides differ, whether their ranges of addresses do.
bool meet(const Rows& a, const Rows& b) {
  if (a.n < 1 || b.n < 1 || a.len < 1 || b.len < 1) return false;
  typedef __int128 wide;
  auto ends = [](const Rows& r, wide& lo, wide& hi) {
    const wide at = (wide) reinterpret_cast<uintptr_t>(r.p), far = at + (wide)r.step() * (wide)(r.n - 1) * (wide)r.size;
    lo = at < far ? at : far;
    hi = (at < far ? far : at) + (wide)r.len * (wide)r.size;
  };
  wide al, ah, bl, bh;
  ends(a, al, ah);
  ends(b, bl, bh);
  if (ah <= bl || bh <= al) return false;
  const wide step = (wide)a.step() * (wide)a.size;
  if (a.n == 1 || b.n == 1 || step <= 0 || step != (wide)b.step() * (wide)b.size) return true;
  wide off = ((wide) reinterpret_cast<uintptr_t>(b.p) - (wide) reinterpret_cast<uintptr_t>(a.p)) % step;   // of b's rows from a's
  if (off < 0) off += step;
  return off < (wide)a.len * (wide)a.size || off + (wide)b.len * (wide)b.size > step;
}

bool temperature_ok(float t, float* inv_t, float* c2) {
  *inv_t = (float)(1.0 / (double)t);
  *c2 = (float)(1.4426950408889634074 / (double)t);
  // (a factor of a normal number: a distance of infinity times it stays infinite)
  return t > 0.f && *c2 < std::numeric_limits<float>::max() && *inv_t >= std::numeric_limits<float>::min();
}

int logprobs_sizes(const april_logprobs_args* a, Logprobs* o) {
  if (!a) REFUSE("april_logprobs: null argument");
  if (a->n_rows < 0 || a->vocab < 1 || a->vocab > (1 << 30)) REFUSE("april_logprobs: n_rows must not be negative, vocab in 1..2^30");
  if (!dtype_ok(a->dtype) || !bits_ok(a->index_bits)) REFUSE("april_logprobs: bad dtype or index_bits");
  if (a->n_top < 0 || a->n_top > 64 || a->n_top > a->vocab) REFUSE("april_logprobs: n_top must be in 0..64 and at most vocab");
  *o = Logprobs{};
  if (!temperature_ok(a->temperature, &o->inv_t, &o->c2)) REFUSE("april_logprobs: temperature must be positive and finite, as its inverse");
  o->n_rows = a->n_rows; o->vocab = a->vocab; o->n_top = a->n_top; o->f32 = a->dtype == APRIL_DTYPE_FP32; o->i64 = a->index_bits == 64;
  return APRIL_OK;
}

int embed_grad_sizes(const april_embed_grad_args* a, EmbedGrad* o) {
  if (!a) REFUSE("april_embed_grad: null argument");
  if (a->n_rows < 0 || a->n_rows > (1 << 30) || a->vocab < 1 || a->vocab > (1 << 30) || a->d < 1 || a->d > (1 << 24))
    REFUSE("april_embed_grad: n_rows must be in 0..2^30, vocab in 1..2^30, d in 1..2^24");
  if (!dtype_ok(a->out_dtype) || !dtype_ok(a->table_dtype) || !bits_ok(a->index_bits)) REFUSE("april_embed_grad: bad dtype or index_bits");
  *o = EmbedGrad{};
  o->n_rows = a->n_rows; o->vocab = a->vocab; o->d = a->d; o->out_f32 = a->out_dtype == APRIL_DTYPE_FP32;
  o->table_f32 = a->table_dtype == APRIL_DTYPE_FP32; o->i64 = a->index_bits == 64; o->accumulate = a->accumulate != 0; o->scale = a->scale;
  return APRIL_OK;
}

int expert_sizes(const char* name, int64_t n_rows, int64_t k, int64_t n_packed) {
  if (n_rows < 0 || k < 1 || k > 64 || n_rows * k > ((1ll << 31) - 1 - 4096) || n_packed < 0)
    REFUSE("%s: n_rows and n_packed must not be negative, k in 1..64, n_rows * k below 2^31 - 4096", name);
  return APRIL_OK;
}
int expert_sort_sizes(const april_expert_sort_args* a, ExpertSort* o) {
  if (!a) REFUSE("april_expert_sort: null argument");
  if (const int rc = expert_sizes("april_expert_sort", a->n_rows, a->k, a->n_packed); rc != APRIL_OK) return rc;
  if (a->n_experts < 1 || a->n_experts > 511 || a->align < 1 || a->align > 4096 || !bits_ok(a->index_bits))
    REFUSE("april_expert_sort: n_experts must be in 1..511, align in 1..4096, index_bits 32 or 64");
  const int64_t n = (int64_t)a->n_rows * a->k, most = n + (n < a->n_experts ? n : a->n_experts) * (a->align - 1);
  if (a->n_packed < most / a->align * a->align) REFUSE("april_expert_sort: n_packed must be at least %lld", (long long)(most / a->align * a->align));
  *o = ExpertSort{};
  o->n = (int)n; o->n_experts = a->n_experts; o->align = a->align; o->n_packed = a->n_packed; o->i64 = a->index_bits == 64;
  return APRIL_OK;
}
int expert_rows(const char* name, int32_t n_rows, int32_t k, int32_t d, int32_t n_packed, int32_t dtype, int32_t reserved, ExpertRows* o) {
  if (const int rc = expert_sizes(name, n_rows, k, n_packed); rc != APRIL_OK) return rc;
  if (d < 1 || d > (1 << 24)) REFUSE("%s: d must be in 1..2^24", name);
  if (!dtype_ok(dtype) || reserved) REFUSE("%s: bad dtype, or reserved is not 0", name);
  *o = ExpertRows{};
  o->n_rows = n_rows; o->k = k; o->d = d; o->n_packed = n_packed; o->f32 = dtype == APRIL_DTYPE_FP32;
  return APRIL_OK;
}

}  // namespace

extern "C" {

int64_t april_logprobs_workspace(const april_logprobs_args* a) {
  Logprobs k;
  if (const int rc = logprobs_sizes(a, &k); rc != APRIL_OK) return rc;
  return (int64_t)logprobs_workspace(k);
}

int april_logprobs(const april_logprobs_args* a) {
  Logprobs k;
  if (const int rc = logprobs_sizes(a, &k); rc != APRIL_OK) return rc;
  if (a->n_rows == 0) return APRIL_OK;
  if (!a->logits || !a->tokens || (a->n_top > 0 && (!a->top_logprobs || !a->top_ids))) REFUSE("april_logprobs: null array");
  if (!aligned(a->logits, element(a->dtype)) || !aligned(a->tokens, a->index_bits / 8)) REFUSE("april_logprobs: logits and tokens must be aligned to their elements");
  if (!aligned(a->logprob, 4) || !aligned(a->entropy, 4) || !aligned(a->lse, 4) || !aligned(a->top_logprobs, 4) || !aligned(a->top_ids, 4) || !aligned(a->norm, 8))
    REFUSE("april_logprobs: results must be aligned to their elements, norm to 8 bytes");
  const size_t need = logprobs_workspace(k);
  if (need > 0 && (!a->workspace || a->workspace_bytes < (int64_t)need || !aligned(a->workspace, 16)))
    REFUSE("april_logprobs: needs %zu bytes of 16-byte aligned workspace (april_logprobs_workspace)", need);
  k.row = a->n_rows > 1 ? a->logits_row : 0;
  k.logits = a->logits; k.tokens = a->tokens; k.logprob = a->logprob; k.entropy = a->entropy; k.lse = a->lse; k.norm = a->norm;
  k.top_logprobs = a->top_logprobs; k.top_ids = a->top_ids; k.ws = (float*)a->workspace;
  return launched("april_logprobs", launch_logprobs((hipStream_t)a->stream, k));
}

int april_logprobs_grad(const april_logprobs_grad_args* a) {
  if (!a) REFUSE("april_logprobs_grad: null argument");
  LogprobsGrad k{};
  if (a->n_rows < 0 || a->vocab < 1 || a->vocab > (1 << 30)) REFUSE("april_logprobs_grad: n_rows must not be negative, vocab in 1..2^30");
  if (!dtype_ok(a->dtype) || !bits_ok(a->index_bits) || a->reserved) REFUSE("april_logprobs_grad: bad dtype or index_bits, or reserved is not 0");
  if (!temperature_ok(a->temperature, &k.inv_t, &k.c2)) REFUSE("april_logprobs_grad: temperature must be positive and finite, as its inverse");
  if (a->n_rows == 0) return APRIL_OK;
  if (!a->logits || !a->tokens || !a->norm || !a->grad || (a->grad_entropy && !a->entropy)) REFUSE("april_logprobs_grad: null array");
  const size_t e = element(a->dtype);
  if (!aligned(a->logits, e) || !aligned(a->grad, e) || !aligned(a->tokens, a->index_bits / 8) || !aligned(a->norm, 8) || !aligned(a->entropy, 4) ||
      !aligned(a->grad_logprob, 4) || !aligned(a->grad_entropy, 4) || !aligned(a->grad_lse, 4))
    REFUSE("april_logprobs_grad: arrays must be aligned to their elements, norm to 8 bytes");
  const Rows in{a->logits, a->n_rows, a->logits_row, a->vocab, e}, out{a->grad, a->n_rows, a->grad_row, a->vocab, e};
  if (rows_overlap(out)) REFUSE("april_logprobs_grad: rows of grad overlap");
  if (!(in.p == out.p && in.step() == out.step()) && meet(in, out)) REFUSE("april_logprobs_grad: grad overlaps the logits and is not the same array");
  k.n_rows = a->n_rows; k.vocab = a->vocab; k.f32 = a->dtype == APRIL_DTYPE_FP32; k.i64 = a->index_bits == 64;
  k.row = in.step(); k.grad_row = out.step(); k.logits = a->logits; k.tokens = a->tokens; k.norm = a->norm; k.entropy = a->entropy;
  k.g_logprob = a->grad_logprob; k.g_entropy = a->grad_entropy; k.g_lse = a->grad_lse; k.grad = a->grad;
  return launched("april_logprobs_grad", launch_logprobs_grad((hipStream_t)a->stream, k));
}

int april_embed(const april_embed_args* a) {
  if (!a) REFUSE("april_embed: null argument");
  if (a->n_rows < 0 || a->vocab < 1 || a->vocab > (1 << 30) || a->d < 1 || a->d > (1 << 24)) REFUSE("april_embed: n_rows must not be negative, vocab in 1..2^30, d in 1..2^24");
  if (!dtype_ok(a->table_dtype) || !dtype_ok(a->out_dtype) || !bits_ok(a->index_bits) || a->reserved) REFUSE("april_embed: bad dtype or index_bits, or reserved is not 0");
  if (!std::isfinite(a->scale)) REFUSE("april_embed: scale must be finite");
  if (a->n_rows == 0) return APRIL_OK;
  if (!a->table || !a->tokens || !a->out) REFUSE("april_embed: null array");
  if (!aligned(a->table, element(a->table_dtype)) || !aligned(a->out, element(a->out_dtype)) || !aligned(a->tokens, a->index_bits / 8))
    REFUSE("april_embed: arrays must be aligned to their elements");
  const Rows out{a->out, a->n_rows, a->out_row, a->d, element(a->out_dtype)}, table{a->table, a->vocab, a->table_row, a->d, element(a->table_dtype)};
  if (rows_overlap(out)) REFUSE("april_embed: rows of out overlap");
  if (meet(out, table)) REFUSE("april_embed: out overlaps the table");
  const Embed k{a->n_rows, a->vocab, a->d, a->table_dtype == APRIL_DTYPE_FP32, a->out_dtype == APRIL_DTYPE_FP32, a->index_bits == 64, a->scale,
                table.step(), out.step(), a->table, a->tokens, a->out};
  return launched("april_embed", launch_embed((hipStream_t)a->stream, k));
}

int64_t april_embed_grad_workspace(const april_embed_grad_args* a) {
  EmbedGrad k;
  if (const int rc = embed_grad_sizes(a, &k); rc != APRIL_OK) return rc;
  return (int64_t)embed_grad_workspace(k);
}

int april_embed_grad(const april_embed_grad_args* a) {
  EmbedGrad k;
  if (const int rc = embed_grad_sizes(a, &k); rc != APRIL_OK) return rc;
  if (!std::isfinite(a->scale)) REFUSE("april_embed_grad: scale must be finite");
  if (a->accumulate != 0 && a->accumulate != 1) REFUSE("april_embed_grad: accumulate must be 0 or 1");
  if (!a->grad_table || (a->n_rows > 0 && (!a->grad_out || !a->tokens))) REFUSE("april_embed_grad: null array");
  if (!aligned(a->grad_out, element(a->out_dtype)) || !aligned(a->grad_table, element(a->table_dtype)) || !aligned(a->tokens, a->index_bits / 8))
    REFUSE("april_embed_grad: arrays must be aligned to their elements");
  const Rows out{a->grad_out, a->n_rows, a->out_row, a->d, element(a->out_dtype)}, table{a->grad_table, a->vocab, a->table_row, a->d, element(a->table_dtype)};
  if (rows_overlap(table)) REFUSE("april_embed_grad: rows of grad_table overlap");
  if (meet(out, table)) REFUSE("april_embed_grad: grad_table overlaps grad_out");
  const size_t need = embed_grad_workspace(k);
  if (need > 0 && (!a->workspace || a->workspace_bytes < (int64_t)need || !aligned(a->workspace, 16)))
    REFUSE("april_embed_grad: needs %zu bytes of 16-byte aligned workspace (april_embed_grad_workspace)", need);
  k.out_row = out.step(); k.table_row = table.step(); k.grad_out = a->grad_out; k.tokens = a->tokens; k.grad_table = a->grad_table; k.ws = a->workspace;
  if (k.n_rows == 0 && k.accumulate) return APRIL_OK;
  return launched("april_embed_grad", launch_embed_grad((hipStream_t)a->stream, k));
}

int64_t april_expert_sort_workspace(const april_expert_sort_args* a) {
  ExpertSort k;
  if (const int rc = expert_sort_sizes(a, &k); rc != APRIL_OK) return rc;
  return (int64_t)expert_sort_workspace(k);
}

int april_expert_sort(const april_expert_sort_args* a) {
  ExpertSort k;
  if (const int rc = expert_sort_sizes(a, &k); rc != APRIL_OK) return rc;
  if (!a->starts || (k.n > 0 && (!a->ids || !a->position)) || (k.n_packed > 0 && !a->source)) REFUSE("april_expert_sort: null array");
  if (!aligned(a->ids, a->index_bits / 8) || !aligned(a->starts, 4) || !aligned(a->source, 4) || !aligned(a->position, 4)) REFUSE("april_expert_sort: arrays must be aligned to their elements");
  const size_t need = expert_sort_workspace(k);
  if (need > 0 && (!a->workspace || a->workspace_bytes < (int64_t)need || !aligned(a->workspace, 16)))
    REFUSE("april_expert_sort: needs %zu bytes of 16-byte aligned workspace (april_expert_sort_workspace)", need);
  k.ids = a->ids; k.starts = a->starts; k.source = a->source; k.position = a->position; k.ws = a->workspace;
  return launched("april_expert_sort", launch_expert_sort((hipStream_t)a->stream, k));
}

int april_expert_gather(const april_expert_gather_args* a) {
  if (!a) REFUSE("april_expert_gather: null argument");
  ExpertRows k;
  if (const int rc = expert_rows("april_expert_gather", a->n_rows, a->k, a->d, a->n_packed, a->dtype, a->reserved, &k); rc != APRIL_OK) return rc;
  if (a->n_packed == 0) return APRIL_OK;
  if (!a->source || !a->packed || (a->n_rows > 0 && (!a->x || !a->position))) REFUSE("april_expert_gather: null array");
  const size_t e = element(a->dtype);
  if (!aligned(a->x, e) || !aligned(a->packed, e) || !aligned(a->source, 4) || !aligned(a->position, 4)) REFUSE("april_expert_gather: arrays must be aligned to their elements");
  const Rows x{a->x, a->n_rows, a->x_row, a->d, e}, out{a->packed, a->n_packed, a->packed_row, a->d, e};
  if (rows_overlap(out)) REFUSE("april_expert_gather: rows of packed overlap");
  if (meet(x, out)) REFUSE("april_expert_gather: packed overlaps x");
  k.row = x.step(); k.packed_row = out.step(); k.rows = a->x; k.position = a->position; k.source = a->source; k.out = a->packed;
  return launched("april_expert_gather", launch_expert_gather((hipStream_t)a->stream, k));
}

int april_expert_combine(const april_expert_combine_args* a) {
  if (!a) REFUSE("april_expert_combine: null argument");
  ExpertRows k;
  if (const int rc = expert_rows("april_expert_combine", a->n_rows, a->k, a->d, a->n_packed, a->dtype, a->reserved, &k); rc != APRIL_OK) return rc;
  if (a->n_rows == 0) return APRIL_OK;
  if (!a->position || !a->out || (a->n_packed > 0 && !a->packed)) REFUSE("april_expert_combine: null array");
  const size_t e = element(a->dtype);
  if (!aligned(a->packed, e) || !aligned(a->out, e) || !aligned(a->position, 4) || !aligned(a->weights, 4)) REFUSE("april_expert_combine: arrays must be aligned to their elements");
  const Rows y{a->packed, a->n_packed, a->packed_row, a->d, e}, out{a->out, a->n_rows, a->out_row, a->d, e};
  if (rows_overlap(out)) REFUSE("april_expert_combine: rows of out overlap");
  if (meet(y, out)) REFUSE("april_expert_combine: out overlaps packed");
  k.row = out.step(); k.packed_row = y.step(); k.packed = a->packed; k.position = a->position; k.weights = a->weights; k.out = a->out;
  return launched("april_expert_combine", launch_expert_combine((hipStream_t)a->stream, k));
}

int april_expert_combine_grad(const april_expert_combine_grad_args* a) {
  if (!a) REFUSE("april_expert_combine_grad: null argument");
  ExpertRows k;
  if (const int rc = expert_rows("april_expert_combine_grad", a->n_rows, a->k, a->d, a->n_packed, a->dtype, a->reserved, &k); rc != APRIL_OK) return rc;
  if ((a->n_packed == 0 || !a->grad_packed) && (a->n_rows == 0 || !a->grad_weights)) return APRIL_OK;
  if ((a->n_packed > 0 && (!a->source || (a->grad_weights && !a->packed))) || (a->n_rows > 0 && (!a->grad_out || !a->position))) REFUSE("april_expert_combine_grad: null array");
  const size_t e = element(a->dtype);
  if (!aligned(a->grad_out, e) || !aligned(a->packed, e) || !aligned(a->grad_packed, e) || !aligned(a->source, 4) || !aligned(a->position, 4) || !aligned(a->weights, 4) ||
      !aligned(a->grad_weights, 4))
    REFUSE("april_expert_combine_grad: arrays must be aligned to their elements");
  const Rows g{a->grad_out, a->n_rows, a->out_row, a->d, e}, y{a->packed, a->grad_weights ? a->n_packed : 0, a->packed_row, a->d, e},
      out{a->grad_packed, a->grad_packed ? a->n_packed : 0, a->grad_packed_row, a->d, e};
  if (rows_overlap(out)) REFUSE("april_expert_combine_grad: rows of grad_packed overlap");
  if (meet(g, out) || meet(y, out)) REFUSE("april_expert_combine_grad: grad_packed overlaps grad_out or packed");
  k.row = g.step(); k.packed_row = y.step(); k.grad_row = out.step(); k.rows = a->grad_out; k.packed = a->grad_weights ? a->packed : nullptr;
  k.position = a->position; k.source = a->source; k.weights = a->weights; k.grad_packed = a->grad_packed; k.grad_weights = a->grad_weights;
  return launched("april_expert_combine_grad", launch_expert_combine_grad((hipStream_t)a->stream, k));
}

}  // extern "C"
