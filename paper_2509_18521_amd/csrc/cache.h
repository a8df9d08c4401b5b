// The 4-bit KV cache: its page layout, and the launchers of the kernels in kernels_cache.hip.
#pragma once
#include "kernels.h"

namespace april {

// A page's block of one KV head: codes of the keys, of the values, then the scales (see april.h).  A sixteenth of a
// kilobyte-sized run per piece: [block of 32 dims][token][16 bytes] puts the 16 tokens of a block next to each other, so
// that 64 lanes read 1 KiB of a page in one load and a prompt's tokens are stored in runs of 256 bytes.
constexpr int CACHE_PAGE = 16;
__host__ __device__ constexpr int cache_block_bytes(int dh) { return 17 * dh; }
__host__ __device__ constexpr int cache_code_off(int dh, int value, int blk, int tok) { return value * 8 * dh + (blk * 16 + tok) * 16; }
__host__ __device__ constexpr int cache_scale_off(int dh, int value, int blk, int tok) { return 16 * dh + (blk * 16 + tok) * 2 + value; }

struct CacheExtend {
  int n_seqs, max_pages, n_pages, n_rows;
  size_t table_stride;
  const int *lens, *new_lens, *free_top;
  int *block_table, *free_pages, *lens_out, *free_top_out, *q_start;
  long long* slot_map;
  int *positions, *status;
  // the engine's admission: sequence b is row row_of[b] of the table, holds nothing yet (lens null), and its pages are counted
  // in held_of[row]; no rows, lengths or first rows are wanted (null)
  const int* row_of;
  int* held_of;
};
hipError_t launch_cache_extend(hipStream_t st, const CacheExtend& a);

struct CacheAppend {
  int n_pages, Hkv, dh, n_rows;
  long long k_row, k_head, v_row, v_head;
  const void *k, *v;
  void *k_values, *v_values;
  const long long* slot_map;
  unsigned char* pool;
};
hipError_t launch_cache_append(hipStream_t st, const CacheAppend& a, bool f32);

struct CacheAttn {
  int Hq, Hkv, n_pages, n_seqs, max_pages, n_rows, max_q, max_len;
  float c2;                        // scale * log2(e)
  float lag;                       // by how much a score may pass the running maximum: its exponential then is 2^8
  void set_scale(float scale) {
    c2 = 1.4426950408889634f * scale;
    lag = 8.0f / c2 < 1e38f ? 8.0f / c2 : 1e38f;
  }
  long long table_stride, q_row, q_head, out_row, out_head;
  const bf16_t* q;
  const unsigned char* pool;
  const int *block_table, *lens, *q_start;
  bf16_t* out;
  float* lse;
  float* ws;
  int ws_rows;                     // rows that the workspace holds (at most n_rows)
};
// The engine's rows (decode: items = the scheduler's work list; prefill: tiles of q_tile positions).
struct CacheRows {
  const int4* items;
  const int2* ctl;
  const int* row_pos;
  int q_tile;
};
// Queries rotated to bf16 rows [row][Hq][dh] (Hq 0: none); keys and values (kv_src: a row's keys, then its values) into the rows' pages if `store`.
struct CacheRope {
  const float *q_src, *kv_src;     // partial p of row r: src + p * partial_stride + r * ld
  int q_ld, kv_ld, n_partials;
  size_t partial_stride;
  const float *rope_cos, *rope_sin;
  bf16_t* q;
  unsigned char* pool;             // the layer's pages
  int Hq, store;
};
void launch_cache_rope(hipStream_t st, RowCtx rc, Slots s, const CacheRope& f, int dh, int Hkv);
// f: the kernel does launch_cache_rope's work itself (a.q is not read); its rows' keys and values are then the tokens of this iteration.
void launch_cache_decode(hipStream_t st, const CacheAttn& a, int dh, const CacheRows& er, int rows, int chunk, int max_splits, int grid_splits, const CacheRope* f);
void launch_cache_prefill(hipStream_t st, const CacheAttn& a, int dh, const CacheRows& er, int n_items);
bool cache_attention_fits(const CacheAttn& a);       // of the sizes alone; workspace and launch only where it is true
size_t cache_attention_workspace(const CacheAttn& a, int dh);
hipError_t launch_cache_attention(hipStream_t st, const CacheAttn& a, int dh);

}  // namespace april
