// C entry points of the 4-bit KV cache's operators: the arguments' checks, then the launch.  They need no context.
#include <algorithm>
#include <cmath>
#include <utility>

#include "../../include/april.h"
#include "cache.h"

using namespace april;

namespace {

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
bool head_dim_ok(int dh) { return dh == 32 || dh == 64 || dh == 128; }
int launched(const char* name, hipError_t e) {
  return e == hipSuccess ? APRIL_OK : fail_no_ctx(APRIL_EDEVICE, "%s: launch failed: %s", name, hipGetErrorString(e));
}

// Whether some two of n x m runs of `len` elements, `row` and `head` elements apart, share one.
bool runs_overlap(int64_t n, int64_t row, int64_t m, int64_t head, int64_t len) {
  auto dist = [](int64_t x) { return x < 0 ? 0 - (uint64_t)x : (uint64_t)x; };      // (as is the order of rows and heads, a sign is nothing here)
  uint64_t s[2] = {dist(row), dist(head)}, c[2] = {(uint64_t)n, (uint64_t)m}, l = (uint64_t)len;
  if (c[0] <= 1 || (c[1] > 1 && s[1] < s[0])) { std::swap(s[0], s[1]); std::swap(c[0], c[1]); }
  if (c[0] <= 1) return false;
  if (s[0] < l) return true;
  if (c[1] <= 1) return false;
  const unsigned __int128 span = (unsigned __int128)s[0] * (c[0] - 1) + l;           // of the nearer ones
  if (s[1] >= span) return false;
  for (uint64_t j = 1; j < c[1]; ++j) {                                            // rare: the two interleave
    const unsigned __int128 at = (unsigned __int128)s[1] * j;
    if (at >= span) return false;
    const uint64_t rest = (uint64_t)(at % s[0]), below = (uint64_t)(at / s[0]);
    if ((rest < l && below < c[0]) || (s[0] - rest < l && below + 1 < c[0])) return true;
  }
  return false;
}

#define REFUSE(...) return fail_no_ctx(APRIL_EINVAL, __VA_ARGS__)

// What both the workspace query and the call check: the sizes.
int attention_sizes(const april_cache_attention_args* a, CacheAttn* o) {
  if (!a) REFUSE("april_cache_attention: null argument");
  if (!head_dim_ok(a->head_dim)) REFUSE("april_cache_attention: head_dim must be 32, 64 or 128");
  if (a->n_kv_heads < 1 || a->n_q_heads < 1 || a->n_q_heads % a->n_kv_heads || a->n_q_heads / a->n_kv_heads > 16 || a->n_q_heads > 65536)
    REFUSE("april_cache_attention: n_q_heads must be a multiple of n_kv_heads, at most 16 times it");
  if (a->n_pages < 1 || a->n_seqs < 0 || a->n_rows < 0 || a->max_pages < 1 || a->max_q < 1 || a->max_len < 0)
    REFUSE("april_cache_attention: bad n_pages, n_seqs, n_rows, max_pages, max_q or max_len");
  if (!(a->scale >= 0.f) || std::isinf(1.4426950408889634f * a->scale)) REFUSE("april_cache_attention: scale must be positive, or 0 for 1 / sqrt(head_dim)");
  *o = CacheAttn{};
  o->Hq = a->n_q_heads; o->Hkv = a->n_kv_heads; o->n_pages = a->n_pages; o->n_seqs = a->n_seqs; o->max_pages = a->max_pages;
  o->n_rows = a->n_rows;
  o->max_q = a->max_q < a->n_rows ? a->max_q : (a->n_rows > 0 ? a->n_rows : 1);
  // (the block table bounds a length too, and positions are counted in 30 bits)
  o->max_len = (int)std::min<long long>({a->max_len, (long long)a->max_pages * CACHE_PAGE, 1ll << 30});
  if (!cache_attention_fits(*o)) REFUSE("april_cache_attention: n_seqs, n_kv_heads, max_q and max_len bound more work than one call takes");
  o->set_scale(a->scale > 0.f ? a->scale : 1.0f / sqrtf((float)a->head_dim));
  return APRIL_OK;
}

}  // namespace

extern "C" {

int april_cache_block_bytes(int32_t head_dim) {
  if (!head_dim_ok(head_dim)) REFUSE("april_cache_block_bytes: head_dim must be 32, 64 or 128");
  return cache_block_bytes(head_dim);
}

int april_cache_extend(const april_cache_extend_args* a) {
  if (!a) REFUSE("april_cache_extend: null argument");
  if (a->n_seqs < 1 || a->n_seqs > 65536 || a->max_pages < 1 || a->n_pages < 1 || a->n_rows < 0)
    REFUSE("april_cache_extend: n_seqs must be in 1..65536, max_pages and n_pages positive, n_rows not negative");
  if (a->max_pages > (1 << 27)) REFUSE("april_cache_extend: max_pages beyond 2^27");
  if (a->table_stride < a->max_pages && a->n_seqs > 1) REFUSE("april_cache_extend: rows of the block table overlap");
  if (!a->lens || !a->new_lens || !a->free_top || !a->block_table || !a->free_pages || !a->lens_out || !a->free_top_out || !a->q_start ||
      !a->status || (a->n_rows > 0 && (!a->slot_map || !a->positions)))
    REFUSE("april_cache_extend: null array");
  if (!aligned(a->slot_map, 8)) REFUSE("april_cache_extend: slot_map must be 8-byte aligned");
  const CacheExtend k{a->n_seqs, a->max_pages, a->n_pages, a->n_rows, (size_t)a->table_stride, a->lens, a->new_lens, a->free_top, a->block_table,
                      a->free_pages, a->lens_out, a->free_top_out, a->q_start, reinterpret_cast<long long*>(a->slot_map), a->positions, a->status, nullptr, nullptr};
  return launched("april_cache_extend", launch_cache_extend((hipStream_t)a->stream, k));
}

int april_cache_append(const april_cache_append_args* a) {
  if (!a) REFUSE("april_cache_append: null argument");
  if (!head_dim_ok(a->head_dim)) REFUSE("april_cache_append: head_dim must be 32, 64 or 128");
  if (a->n_pages < 1 || a->n_kv_heads < 1 || a->n_kv_heads > 4096 || a->n_rows < 0)
    REFUSE("april_cache_append: n_pages must be positive, n_kv_heads in 1..4096, n_rows not negative");
  if (a->n_rows > 16 * ((1 << 24) - 1)) REFUSE("april_cache_append: n_rows beyond 2^28 - 16");      // (16 a workgroup; a launch has fewer than 2^32 threads)
  if (a->dtype != APRIL_DTYPE_FP32 && a->dtype != APRIL_DTYPE_BF16) REFUSE("april_cache_append: bad dtype");
  if (a->reserved) REFUSE("april_cache_append: reserved must be 0");
  if (a->n_rows == 0) return APRIL_OK;
  if (!a->k || !a->v || !a->slot_map || !a->pool) REFUSE("april_cache_append: null array");
  const size_t e = a->dtype == APRIL_DTYPE_FP32 ? 4 : 2;
  if (!aligned(a->pool, 16) || !aligned(a->slot_map, 8) || !aligned(a->k, e) || !aligned(a->v, e))
    REFUSE("april_cache_append: the pool must be 16-byte aligned, slot_map, k and v to their elements");
  if ((a->k_values && !aligned(a->k_values, 16)) || (a->v_values && !aligned(a->v_values, 16)))
    REFUSE("april_cache_append: k_values and v_values must be 16-byte aligned");
  const CacheAppend k{a->n_pages, a->n_kv_heads, a->head_dim, a->n_rows, a->k_row, a->k_head, a->v_row, a->v_head, a->k, a->v, a->k_values, a->v_values,
                      reinterpret_cast<const long long*>(a->slot_map), (unsigned char*)a->pool};
  return launched("april_cache_append", launch_cache_append((hipStream_t)a->stream, k, a->dtype == APRIL_DTYPE_FP32));
}

int64_t april_cache_attention_workspace(const april_cache_attention_args* a) {
  CacheAttn k;
  const int rc = attention_sizes(a, &k);
  if (rc != APRIL_OK) return rc;
  return (int64_t)cache_attention_workspace(k, a->head_dim);
}

int april_cache_attention(const april_cache_attention_args* a) {
  CacheAttn k;
  const int rc = attention_sizes(a, &k);
  if (rc != APRIL_OK) return rc;
  if (a->n_seqs == 0 || a->n_rows == 0) return APRIL_OK;
  if (!a->q || !a->pool || !a->block_table || !a->lens || !a->out) REFUSE("april_cache_attention: null array");
  if (!a->q_start && a->n_rows < a->n_seqs) REFUSE("april_cache_attention: fewer rows than sequences, and no q_start");
  // (a stride over a single row or head is not used)
  const int64_t q_row = a->n_rows > 1 ? a->q_row : 0, q_head = a->n_q_heads > 1 ? a->q_head : 0, out_row = a->n_rows > 1 ? a->out_row : 0,
                out_head = a->n_q_heads > 1 ? a->out_head : 0;
  if (!aligned(a->q, 16) || q_row % 8 || q_head % 8 || !aligned(a->pool, 16)) REFUSE("april_cache_attention: q's heads and the pool must be 16-byte aligned");
  if (!aligned(a->out, 8) || out_row % 4 || out_head % 4) REFUSE("april_cache_attention: out's heads must be 8-byte aligned");
  if (runs_overlap(a->n_rows, out_row, a->n_q_heads, out_head, a->head_dim)) REFUSE("april_cache_attention: heads of out overlap");
  if (a->table_stride < a->max_pages && a->n_seqs > 1) REFUSE("april_cache_attention: rows of the block table overlap");
  const size_t need = cache_attention_workspace(k, a->head_dim);
  if (need > 0 && (!a->workspace || a->workspace_bytes < (int64_t)need || !aligned(a->workspace, 16)))
    REFUSE("april_cache_attention: needs %zu bytes of 16-byte aligned workspace (april_cache_attention_workspace)", need);
  k.table_stride = a->table_stride; k.q_row = q_row; k.q_head = q_head; k.out_row = out_row; k.out_head = out_head;
  k.q = (const bf16_t*)a->q; k.pool = (const unsigned char*)a->pool; k.block_table = a->block_table; k.lens = a->lens; k.q_start = a->q_start;
  k.out = (bf16_t*)a->out; k.lse = a->lse; k.ws = (float*)a->workspace;
  return launched("april_cache_attention", launch_cache_attention((hipStream_t)a->stream, k, a->head_dim));
}

}  // extern "C"
