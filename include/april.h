/*
 * april.h - C ABI of the MI355X-native APRIL rollout engine.
 *
 * APRIL (Active Partial Rollouts in Reinforcement Learning) schedules the rollout
 * phase of RL post-training: every step keeps N' > N rollouts in flight, stops as
 * soon as N of them are complete, parks the unfinished ones in a continuation
 * buffer and resumes them, ahead of new requests, at the next step (paper,
 * Section 2.2, the four-item description of the method).  With N' == N the same
 * call is the wait-for-all baseline of the paper's "standard setting"
 * (Section 3.1).
 *
 * The library owns the whole hot path on ONE gfx950 GPU: paged KV cache, prefill,
 * the batched decode loop (HIP kernels), the sampler, and a device-side scheduler
 * that counts finished rollouts and compacts the live batch without a host round
 * trip per token.  There is no CPU fallback: every call fails with APRIL_EDEVICE
 * when no GPU is usable.
 *
 * Conventions
 *   - all functions return APRIL_OK (0) or a negative error code; the message is
 *     available from april_last_error();
 *   - "host" pointers are ordinary process memory, "device" pointers are HIP
 *     device memory on the context's GPU; each argument says which one it is;
 *   - a context is single-threaded; calls on one context must not overlap;
 *   - matrices are row-major [out_features, in_features] (y = W x).
 */
#ifndef APRIL_H
#define APRIL_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define APRIL_OK        0
#define APRIL_EINVAL   -1   /* bad argument / unsupported configuration          */
#define APRIL_ENOMEM   -2   /* device memory or KV pool cannot hold the request   */
#define APRIL_ESTARVED -3   /* fewer than N_target rollouts can ever complete     */
#define APRIL_EHANDLE  -4   /* unknown / stale buffer handle or request id        */
#define APRIL_EDEVICE  -5   /* HIP error, or no usable GPU                        */

#define APRIL_DTYPE_FP32 0
#define APRIL_DTYPE_BF16 1
#define APRIL_DTYPE_BF16_KV4 2   /* bf16, but the KV cache in 4 bits (the blocks of the 4-bit cache operators below): 3.8 times
                                    the tokens in the same memory, and keys and values rounded to MXFP4.  Decode is faster where
                                    reading the cache bounds it (many rollouts, long contexts), a few percent slower for one
                                    short rollout of a small model; so is prefill                               */
#define APRIL_MEM_KV      1   /* memory tags of april_memory_pause / april_memory_resume */
#define APRIL_MEM_WEIGHTS 2
#define APRIL_SAMPLER_GREEDY 0
#define APRIL_SAMPLER_TOPK   1   /* top-k, then (top_p < 1) the nucleus of the k candidates            */
#define APRIL_SAMPLER_CATEGORICAL 2   /* temperature sampling over the whole vocabulary (the paper's
                                         rollout setting, appendix: rollout temperature, no truncation) */

typedef struct april_ctx    april_ctx;     /* opaque; owns all device state            */
typedef struct april_buffer april_buffer;  /* opaque handle: a continuation buffer     */

/* Model and engine configuration (host memory, read during april_init only).
 * The network is a pre-norm decoder: RMSNorm, q/k/v projections without bias,
 * rotary embedding (pair (i, i + head_dim/2), angle pos * rope_theta^(-2i/head_dim)),
 * causal attention with n_q_heads / n_kv_heads query heads sharing one KV head,
 * output projection + residual, RMSNorm, SwiGLU MLP (or routed experts) + residual,
 * final RMSNorm, untied LM head.  The paper names only the model family it runs
 * (Section 3.1); the rollout itself is Eq. 1's a ~ pi(theta_k). */
typedef struct {
  int32_t n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn, vocab;
  int32_t n_experts, experts_per_tok, d_expert_ffn;  /* 0,0,0 => dense MLP                */
  int32_t dtype;             /* APRIL_DTYPE_*: type of weights, KV cache, GEMM operands (BF16_KV4: cache apart) */
  float   rope_theta, rms_eps;
  int32_t kv_block_tokens;   /* tokens per KV page; must be 16                            */
  int64_t kv_pool_bytes;     /* 0 => sized for max_inflight sequences of max_ctx tokens,
                                but at most the free device memory less a reserve for the
                                workspaces (max(12 GiB, 1/16 of the device))              */
  int32_t max_inflight;      /* sequence slots (in flight + parked + surplus-complete)    */
  int32_t max_ctx;           /* max prompt + generated tokens of one sequence             */
  int32_t sampler;           /* APRIL_SAMPLER_*                                           */
  int32_t top_k;             /* 1..64 for the top-k sampler                               */
  float   temperature;       /* > 0, top-k sampler only                                   */
  uint64_t seed;             /* Philox key of the sampler                                 */
  int32_t eos_token;         /* -1: only length limits end a rollout                      */
  int32_t debug_logits;      /* 1: parity mode, logits of watched requests are kept       */
  float   top_p;             /* top-k sampler: keep the shortest prefix of the k candidates
                                (descending) whose probabilities, renormalised over the k
                                candidates, reach top_p; 0 or >= 1: no nucleus cut (the paper's
                                appendix lists an evaluation top_p)                          */
  int32_t logprobs;          /* 1: keep log softmax(logits / temperature)[token] over the whole
                                vocabulary for every generated token (what a trainer's
                                importance ratio needs, Section 2.2) and return it            */
  int32_t n_samples_per_prompt;  /* G > 1: instance-level completion (Section 3.2.3; Section 3.1
                                runs 32 x 8): every input instance is a group of G rollouts
                                (april_request.group_id), admitted together; a step stops once
                                N_target / G groups have all members complete and returns those
                                groups whole; complete members of an unfinished group wait in the
                                buffer.  N_target and N_overprovision stay rollout counts and must
                                be multiples of G.  0 or 1: every rollout on its own             */
  int32_t pausable;          /* 1: the KV pool and the weights live in reserved virtual address
                                ranges whose physical memory april_memory_pause can release    */
  void*   stream;            /* hipStream_t to run on (e.g. torch's current), or NULL     */
} april_model_cfg;

/* One named weight tensor.  `data` is host or device memory (on_device says which),
 * borrowed for the duration of april_init only: the library keeps its own copy in
 * the layout its kernels want.  Element type: float for APRIL_DTYPE_FP32, bf16 bit
 * patterns (uint16) for APRIL_DTYPE_BF16 and APRIL_DTYPE_BF16_KV4; norm gains are always float.
 * Names (l = layer index): tok_emb [vocab,d]; attn_norm.l [d]; wq.l [Hq*dh,d];
 * wk.l, wv.l [Hkv*dh,d]; wo.l [d,Hq*dh]; mlp_norm.l [d]; w_gate.l, w_up.l [F,d];
 * w_down.l [d,F]; final_norm [d]; lm_head [vocab,d]; for experts: router.l [E,d],
 * e_gate.l, e_up.l [E,Fe,d], e_down.l [E,d,Fe]. */
typedef struct {
  const char* name;
  const void* data;
  int64_t     nbytes;
  int32_t     on_device;
} april_tensor;

/* A new rollout request (host memory, borrowed during the call).
 * forced_len > 0: the rollout is complete exactly when it has generated
 * min(forced_len, max_new) tokens (synthetic long-tail workloads); 0: only max_new
 * and the EOS token end it.  forced_tokens (may be NULL): teacher forcing for
 * parity tests - generated token i is replaced by forced_tokens[i] for
 * i < n_forced_tokens after the sampler has run. */
typedef struct {
  int64_t        request_id;
  const int32_t* tokens;          /* prompt, host */
  int32_t        n_tokens;
  int32_t        forced_len;
  const int32_t* forced_tokens;   /* host, or NULL */
  int32_t        n_forced_tokens;
  int64_t        group_id;        /* input instance (n_samples_per_prompt > 1): its G requests are
                                     consecutive in new_reqs; ignored otherwise                  */
} april_request;

/* Result of one step.  Every pointer is host memory owned by the context and valid
 * until the next april_rollout_step / april_destroy on that context. */
typedef struct {
  int32_t  n_completed;           /* == N_target on success                                */
  const int64_t* request_id;      /* [n_completed], completion order (iteration, then id)  */
  const int32_t* const* tokens;   /* [n_completed] generated tokens only                   */
  const int32_t* n_tokens;        /* [n_completed]                                         */
  const int32_t* n_resumes;       /* [n_completed] steps the rollout spanned, minus one    */
  const float* const* logprobs;   /* [n_completed] per generated token (cfg.logprobs), else NULL */
  const int64_t* group_id;        /* [n_completed] (n_samples_per_prompt > 1: the members of a group are
                                     adjacent, ascending request id), else NULL                  */
  april_buffer*  buffer;          /* unfinished + surplus-complete rollouts (never NULL)   */
  int32_t  n_new_consumed;        /* how many of new_reqs were admitted                    */
  int64_t  decode_iters;          /* iterations executed (each adds 1 token per live seq)  */
  int64_t  tokens_generated;      /* over all in-flight rollouts, partial ones included    */
  int64_t  prefill_tokens;        /* prompt tokens of newly admitted rollouts              */
  int64_t  reprefill_tokens;      /* tokens recomputed for rollouts resumed without KV     */
  int64_t  n_preempted;           /* rollouts preempted in this step (KV pool exhausted)   */
  int64_t  sum_live;              /* sum over decode-path iterations of the live batch     */
  int64_t  sum_ctx;               /* sum over decode-path (iteration, seq) of context len  */
  int64_t  dec_sum_live, dec_sum_ctx;  /* the same sums over iterations 2.. only: the ones
                                          t_decode_s covers (iteration 1 is timed with prefill) */
  int64_t  dec_sum_experts;       /* routed experts: sum over (iteration 2.., layer) of the
                                     experts that received at least one token              */
  double   t_prefill_s, t_decode_s, t_total_s;   /* host wall clock                        */
} april_step_result;

/* A rollout as stored in a continuation buffer, token-level view (Section 3.2.3:
 * the buffer caches the tokens of incomplete trajectories). */
typedef struct {
  int64_t request_id;
  const int32_t* prompt;    int32_t n_prompt;      /* host */
  const int32_t* generated; int32_t n_generated;   /* host */
  int32_t limit;            /* generated length at which it completes                      */
  int32_t n_resumes;
  int32_t done;             /* 1: complete, waiting to be delivered first next step        */
  int32_t kv_resident;      /* 1: its KV pages are still on the device                     */
  const float* logprobs;    /* host, [n_generated] (cfg.logprobs), or NULL                  */
  int64_t group_id;         /* input instance (n_samples_per_prompt > 1), else -1           */
} april_partial;

/* Create a context on the current HIP device: copy/re-layout the weights, carve the
 * KV pool into pages, allocate scheduler state and workspaces. */
int april_init(const april_model_cfg* cfg, const april_tensor* weights, int32_t n_weights,
               april_ctx** out);

/* One rollout step (Section 2.2).  In flight = rollouts resumed by april_resume
 * (ascending request id) + new_reqs in order until N_overprovision are in flight
 * (surplus-complete rollouts in the resumed buffer count toward N_target and reduce
 * the number admitted).  Runs prefill for new / KV-less rollouts and decode
 * iterations - one token per live rollout per iteration - until N_target rollouts
 * are complete, then returns exactly N_target of them and a buffer with the rest.
 * N_overprovision == N_target is the wait-for-all baseline.
 * KV pool exhausted: a rollout that needs prefill is admitted only while the pages of its
 * tokens fit (the first that does not fit closes admission for the step); before an
 * iteration, if the rollouts that open a new page need more pages than are free, the
 * youngest decoding rollout (largest request id) is preempted - pages freed, tokens kept,
 * no progress this step, re-prefilled when resumed; if nothing is left in flight the step
 * returns fewer than N_target (n_completed says how many).
 * new_reqs: host array [n_new_avail]; out: host struct filled by the call.
 * A call that fails is transactional with respect to the rollouts: none of new_reqs is
 * consumed (the caller still owns them), and every rollout that april_resume had handed in
 * goes back to the pending set - with the tokens it generated before the failure, without its
 * KV pages - so the next april_rollout_step admits it first again; `out` is not filled. */
int april_rollout_step(april_ctx* ctx, const april_request* new_reqs, int32_t n_new_avail,
                       int32_t N_target, int32_t N_overprovision, int32_t max_new,
                       april_step_result* out);

/* Prioritized resumption: hand a buffer back; its rollouts are admitted ahead of new
 * requests in the NEXT april_rollout_step.  Consumes the handle. */
int april_resume(april_ctx* ctx, april_buffer* buffer);

/* Number of rollouts in a buffer (negative: error). */
int april_buffer_size(const april_ctx* ctx, const april_buffer* buffer);
/* Token-level view of a buffer: fills out[0..min(size,cap)) (host), arrays are owned
 * by the context and valid until the buffer is freed or resumed.  Returns the size. */
int april_buffer_export(april_ctx* ctx, const april_buffer* buffer, april_partial* out, int32_t cap);
/* Build a buffer from token-level entries (host, copied); such rollouts have no KV on
 * the device and are re-prefilled when resumed. */
int april_buffer_import(april_ctx* ctx, const april_partial* in, int32_t n, april_buffer** out);
/* Release the KV pages of every rollout in the buffer: they resume by re-prefill
 * (fallback path; also what a change of policy weights would require). */
int april_buffer_drop_kv(april_ctx* ctx, april_buffer* buffer);
/* Drop a buffer and everything it holds. */
void april_buffer_free(april_ctx* ctx, april_buffer* buffer);

/* Policy update between steps (Eq. 1: the trainer moves theta_k to theta_{k+1} after every
 * step, and rollouts parked under theta_k are continued under theta_{k+1}: Section 2.2,
 * trajectories of a mixed policy).  `weights` as for april_init (same names and sizes, host or
 * device, borrowed during the call); the library overwrites its own copies in place.
 * keep_kv = 0: the K/V of every parked rollout was computed under the old weights, so its pages
 * are released and the rollout is re-prefilled under the new weights when it is resumed (its
 * tokens are kept).  keep_kv = 1: the stale K/V stays and decoding simply goes on (cheaper, and
 * an approximation: the measured alternative).  Call between steps only.  On an error the
 * context's weights are undefined until a later call succeeds. */
int april_update_weights(april_ctx* ctx, const april_tensor* weights, int32_t n_weights, int32_t keep_kv);

/* Pause / resume of the engine's large device buffers by virtual-memory remapping (Section 3.3,
 * the memory-saving extension that lets rollout and training share one GPU on either vendor's
 * hardware; cfg.pausable = 1).  tags: APRIL_MEM_KV | APRIL_MEM_WEIGHTS.
 * april_memory_pause releases the physical memory behind the tagged buffers; their virtual
 * addresses stay reserved, so everything that holds those addresses (captured iteration graphs
 * included) remains valid.  The workspace that april_sample_rows keeps is released too.
 * april_memory_resume maps fresh physical memory at the same addresses.
 * Contents do not survive: after a KV pause every parked rollout keeps its tokens and is
 * re-prefilled when resumed (the pool comes back zeroed and entirely free); after a weights
 * pause april_update_weights must be called before the next step.  Call between steps only;
 * april_rollout_step fails with APRIL_EINVAL while anything is paused. */
int april_memory_pause(april_ctx* ctx, int32_t tags);
int april_memory_resume(april_ctx* ctx, int32_t tags);

/* Parity mode (cfg.debug_logits = 1): keep the fp32 logits that produced generated
 * tokens [first_gen, first_gen + n_gen) of request_id.  Call before the step that
 * generates them. */
int april_debug_watch(april_ctx* ctx, int64_t request_id, int32_t first_gen, int32_t n_gen);
/* Copy the kept logits row (vocab floats, host) and the sampler's own choice for it. */
int april_debug_logits(april_ctx* ctx, int64_t request_id, int32_t gen_index,
                       float* out_logits, int32_t* out_sampled);

/* The sampler alone (Section 3.1 samples with a temperature; greedy / top-k are the
 * configured ones): logits is a DEVICE array [n_rows, vocab] of float; request_ids,
 * gen_index (host, [n_rows]) key the Philox stream; out_tokens host [n_rows].
 * The context keeps the call's device workspace for the next call: at most 64 MiB (or what one row
 * needs, 12 bytes per 64 logits, if that is more), until april_memory_pause or april_destroy. */
int april_sample_rows(april_ctx* ctx, const float* logits, int32_t n_rows,
                      const int64_t* request_ids, const int32_t* gen_index, int32_t* out_tokens);

/* The same with the log-probability of each chosen token (out_logprobs host [n_rows]):
 * log softmax(logits / temperature) over the whole vocabulary. */
int april_sample_rows_logprobs(april_ctx* ctx, const float* logits, int32_t n_rows,
                               const int64_t* request_ids, const int32_t* gen_index,
                               int32_t* out_tokens, float* out_logprobs);

/* april_sample_rows for callers that cannot allocate device memory (code under HIP graph
 * capture rules, tight serving loops, harnesses that forbid hipMalloc): same arguments, same
 * result, but the device temporaries (the per-row maxima and sums of 64-logit groups) live in a static
 * device array of 12 MiB that the library holds on every GPU it runs on until the process ends, row
 * keys and result in the context's pinned staging buffer; the call makes no hipMalloc / hipFree.
 * Limits: n_rows <= 1024 and n_rows * (vocab / 64) <= 1048576 (APRIL_EINVAL beyond).
 * All calls on one GPU share that array and it keeps the last call's contents: calls that
 * overlap on one GPU (other threads, other contexts) race; serialise them. */
int april_sample_rows_noalloc(april_ctx* ctx, const float* logits, int32_t n_rows,
                              const int64_t* request_ids, const int32_t* gen_index, int32_t* out_tokens);

/* ------------------------------------------------------------------------------------------
 * Operators of a 4-bit KV cache on the caller's own device memory: the tables that say where a
 * token lies, the store, and the attention that reads it.  They need no context: each enqueues
 * its kernels on `stream` (NULL: the null stream) of the current device and returns; nothing is
 * allocated or synchronised, so the calls may be captured into a graph.  Pointers are device
 * memory of that device.  Errors found on the host leave everything untouched, their message is
 * april_last_error(NULL) of the calling thread; errors in device data end in `status` or in NaN, as
 * said below, never in an access outside the given arrays.
 *
 * The pool: pages of 16 tokens of one sequence, n_pages x n_kv_heads blocks of 17 * head_dim bytes
 * (april_cache_block_bytes; head_dim 32, 64 or 128; 16-byte aligned).  Keys and values are kept in
 * blocks of 32 dimensions, MXFP4: 4-bit codes (sign; 0, 0.5, 1, 1.5, 2, 3, 4, 6) times a power of two
 * that the block shares.  In a page's block of one head:
 *   keys    [head_dim / 32][16 tokens][16 bytes]   dimension 2 i in the low half of byte i, 2 i + 1 in the high one
 *   values  the same
 *   scales  [head_dim / 32][16 tokens][key, value] the power's biased exponent, 2^(e - 127); 255: 32 NaN
 * The power brings the block's largest magnitude into [3.5, 7) (between 2^-125 and 2^125, so that every value is
 * a normal number; what lies beyond 6 * 2^125 becomes that), codes are rounded to nearest, ties to even; a block
 * that holds an infinity or a NaN is stored as NaN.  Uninitialised pages are fine: nothing
 * is read behind a sequence's length.
 * The block table: row b holds the pages of sequence b, token p in page p / 16 of the row. */
#define APRIL_CACHE_PAGE 16

/* Bytes of one (page, KV head) of the pool, 17 * head_dim; APRIL_EINVAL for another head_dim. */
int april_cache_block_bytes(int32_t head_dim);

/* One iteration's tables from the requests' lengths.  Sequence b holds lens[b] tokens.  new_lens[b] < 0:
 * it has ended, its pages go onto the stack of free pages (in the order of sequences and of their pages).
 * Then the others grow by new_lens[b] >= 0 tokens; in the order of sequences each takes the pages that it
 * lacks from the top of the stack and has them entered in its row of the block table.
 * lens_out, free_top_out and status may be the arrays of the next call's lens and free_top. */
typedef struct {
  int32_t n_seqs;                /* sequences, 1..65536                                        */
  int32_t max_pages;             /* columns of the block table                                 */
  int32_t n_pages;               /* pages of the pool = entries of free_pages                  */
  int32_t n_rows;                /* entries of slot_map and positions                          */
  int64_t table_stride;          /* elements between rows of the block table                   */
  const int32_t* lens;           /* [n_seqs]                                                   */
  const int32_t* new_lens;       /* [n_seqs]                                                   */
  const int32_t* free_top;       /* [1] free pages on the stack                                */
  int32_t* block_table;          /* [n_seqs][max_pages], in place                              */
  int32_t* free_pages;           /* [n_pages] the stack, in place                              */
  int32_t* lens_out;             /* [n_seqs] (may be lens); 0 for a sequence that has ended    */
  int32_t* free_top_out;         /* [1] (may be free_top)                                      */
  int32_t* q_start;              /* [n_seqs + 1] first row of each sequence's new tokens       */
  int64_t* slot_map;             /* [n_rows] page * 16 + token of each row; -1 behind the last */
  int32_t* positions;            /* [n_rows] position in its sequence; -1 behind the last      */
  int32_t* status;               /* [1] 0; 1: too few free pages; 2: a length below zero, beyond the
                                    block table or beyond 2^31 - 16, more rows than n_rows, or a stack that
                                    does not fit its array.  Not 0: nothing was entered or taken, lens_out = lens,
                                    free_top_out = free_top, no rows (q_start 0, slots and positions -1) */
  void* stream;
} april_cache_extend_args;
int april_cache_extend(const april_cache_extend_args* args);

/* Store the keys and values of n_rows tokens at their slots (page * 16 + token, as april_cache_extend writes
 * them).  Rows whose slot lies outside the pool are left out; two rows with the same slot leave one of them,
 * or parts of both. */
typedef struct {
  int32_t n_pages, n_kv_heads, head_dim;
  int32_t n_rows;                /* at most 2^28 - 16                                          */
  int32_t dtype;                 /* APRIL_DTYPE_* of k, v and the values                       */
  int32_t reserved;              /* 0                                                          */
  int64_t k_row, k_head, v_row, v_head;   /* elements between rows and heads; dimensions are adjacent.
                                    Rows of 16-byte aligned heads are read fastest             */
  const void *k, *v;             /* [n_rows][n_kv_heads][head_dim]                             */
  void *k_values, *v_values;     /* or NULL: contiguous, what the cache now stands for (rows that are left out: untouched) */
  const int64_t* slot_map;       /* [n_rows]                                                   */
  void* pool;
  void* stream;
} april_cache_append_args;
int april_cache_append(const april_cache_append_args* args);

/* Causal attention over the cache, softmax(scale q k) v, bf16, sums in fp32; the softmax's weights are rounded to bf16
 * before they multiply the values (their own sum is not), which puts an output off by at most 2^-8 of the mean |v| under them.  The rows
 * q_start[b] .. q_start[b + 1] - 1 of q are the last tokens of sequence b: row i of c sees the tokens
 * 0 .. lens[b] - c + i.  (One row: a decode iteration.  As many rows as tokens: a whole prompt.)
 * n_q_heads / n_kv_heads (at most 16) consecutive query heads share a KV head.
 * A row that sees no token is 0 and its lse -infinity.  Rows of no sequence are left as they were.  A NaN in the
 * cache reaches the rows that see it.  A page id outside the pool makes the rows that see a token on it NaN (and
 * may others of their sequence); a length outside 0 .. max_len, beyond the block table or
 * beyond 2^30, all rows of its sequence.
 * n_seqs, the heads, max_q and max_len (or 16 max_pages, where that is less) decide how the work is shared out, for all sequences
 * alike; with those given, a row's bits do not depend on the other sequences.  One sequence of many rows among many of one row has all of them
 * take the way of many rows, without splits of long contexts: two calls are faster then, one with max_q 1 over all (it leaves the further rows as they
 * were), one with the arrays of the long sequences alone (block_table, lens and q_start from theirs on).
 * Sizes that bound more work than one launch takes are refused (APRIL_EINVAL, here and by the workspace query): 2^24 workgroups,
 * of which each KV head of a sequence has one, or one for every 256 of max_q x (query heads of the KV head) where those are more than 64, and
 * that for every split of max_len tokens (at most 4096 a split up to those 64); where there are splits, 2^24 rows n_seqs x max_q;
 * and 2^31 - 256 of max_q x (query heads of the KV head). */
typedef struct {
  int32_t n_q_heads, n_kv_heads, head_dim;
  int32_t n_pages, n_seqs;
  int32_t max_pages;             /* columns of the block table                                 */
  int32_t n_rows;                /* rows of q, out and lse                                     */
  int32_t max_q;                 /* bound on the rows of a sequence (rows beyond it are left as they were) */
  int32_t max_len;               /* bound on lens.  Tight bounds are faster                    */
  float scale;                   /* > 0; 0: 1 / sqrt(head_dim)                                 */
  int64_t table_stride, q_row, q_head, out_row, out_head;   /* in elements; dimensions are adjacent */
  const void* q;                 /* bf16 [n_rows][n_q_heads][head_dim], heads 16-byte aligned  */
  const void* pool;
  const int32_t* block_table;    /* [n_seqs][max_pages]                                        */
  const int32_t* lens;           /* [n_seqs] tokens in the cache, those of the rows included   */
  const int32_t* q_start;        /* [n_seqs + 1], or NULL: row b is sequence b's (n_rows >= n_seqs) */
  void* out;                     /* bf16, as q (8-byte aligned heads; no two overlap)          */
  float* lse;                    /* [n_rows][n_q_heads] log of the sum of exp(scale q k), or NULL */
  void* workspace;               /* april_cache_attention_workspace bytes, 16-byte aligned; NULL if 0.  Calls that may
                                    run at the same time need one each                         */
  int64_t workspace_bytes;
  void* stream;
} april_cache_attention_args;
int april_cache_attention(const april_cache_attention_args* args);
/* Bytes that a call of these sizes needs (pointers, strides and the stream are not looked at). */
int64_t april_cache_attention_workspace(const april_cache_attention_args* args);

/* ------------------------------------------------------------------------------------------
 * Operators that score rollouts and train on them, on the caller's own device memory, each with its gradient: the
 * log-probability of a given token, a token's row of the embedding, a token's rows in its experts' batches.  As the
 * cache's operators they need no context, enqueue on `stream` of the current device, allocate and synchronise
 * nothing (so they may be captured into a graph), and leave everything untouched where the host finds an error.
 * Matrices are rows of adjacent elements, `*_row` elements apart (16-byte aligned rows are fastest); a stride over a
 * single row is not used; inputs may repeat a row (stride 0), rows of a result may not overlap, nor a result an input where
 * nothing else is said.  dtype: APRIL_DTYPE_FP32 or APRIL_DTYPE_BF16; sums are in fp32, a result is rounded once.
 * Indexes (tokens, experts) are of index_bits 32 or 64.  The same call gives the same bits every time; the last bits of a
 * sum may change with the sizes of the call and with a row's address to 16 bytes.  Calls that may run at the same time need a workspace each. */

/* x = logits / temperature, row by row: logprob = x[token] - lse, lse = log of the sum of exp(x), entropy = -sum of p log p, and the
 * n_top largest x - lse with their columns, descending, equal logits by ascending column.
 * A token below zero marks a padding row: its results are 0, its top_ids -1, and it is not read.  A token of vocab or more: logprob
 * NaN.  Logits of -infinity have probability 0.  Rows that have a NaN, +infinity or nothing but -infinity: NaN (lse: NaN or
 * -infinity), top_ids -1.  Results that are NULL are left out. */
typedef struct {
  int32_t n_rows, vocab;         /* vocab 1..2^30                                              */
  int32_t dtype, index_bits;     /* of logits; of tokens                                       */
  int32_t n_top;                 /* 0..64, at most vocab                                       */
  float temperature;             /* > 0                                                        */
  int64_t logits_row;
  const void* logits;            /* [n_rows][vocab]                                            */
  const void* tokens;            /* [n_rows]                                                   */
  float *logprob, *entropy, *lse;   /* [n_rows]                                                */
  float* norm;                   /* [n_rows][2], 8-byte aligned: what april_logprobs_grad needs of the row (its largest logit, log2 of
                                    the sum of 2^((logit - largest) log2(e) / temperature))   */
  float* top_logprobs;           /* [n_rows][n_top]                                            */
  int32_t* top_ids;              /* [n_rows][n_top]                                            */
  void* workspace;               /* april_logprobs_workspace bytes, 16-byte aligned; NULL if 0 */
  int64_t workspace_bytes;
  void* stream;
} april_logprobs_args;
int april_logprobs(const april_logprobs_args* args);
/* Bytes that a call of these sizes needs (pointers, strides and the stream are not looked at). */
int64_t april_logprobs_workspace(const april_logprobs_args* args);

/* Gradient of the logits for gradients a, h, z of logprob, entropy, lse (NULL: 0):
 * (a (1 at the token - p) - h p (log p + entropy) + z p) / temperature.  Padding rows: 0; a token of vocab or more: NaN.  A term of p = 0 is
 * 0 for finite a, h, z, at any temperature. */
typedef struct {
  int32_t n_rows, vocab, dtype, index_bits;   /* as in april_logprobs; grad is of the logits' type */
  float temperature;
  int32_t reserved;              /* 0                                                          */
  int64_t logits_row, grad_row;
  const void *logits, *tokens;
  const float* norm;             /* [n_rows][2] of april_logprobs                              */
  const float* entropy;          /* [n_rows] of april_logprobs; NULL without grad_entropy      */
  const float *grad_logprob, *grad_entropy, *grad_lse;   /* [n_rows]                           */
  void* grad;                    /* [n_rows][vocab]; may be the logits themselves (the same address and stride) */
  void* stream;
} april_logprobs_grad_args;
int april_logprobs_grad(const april_logprobs_grad_args* args);

/* out[r] = scale * table[tokens[r]].  A token below zero marks padding: 0; one of vocab or more: NaN. */
typedef struct {
  int32_t n_rows, vocab, d;      /* vocab 1..2^30, d 1..2^24                                   */
  int32_t table_dtype, out_dtype, index_bits;
  float scale;
  int32_t reserved;              /* 0                                                          */
  int64_t table_row, out_row;
  const void* table;             /* [vocab][d]                                                 */
  const void* tokens;            /* [n_rows]                                                   */
  void* out;                     /* [n_rows][d]                                                */
  void* stream;
} april_embed_args;
int april_embed(const april_embed_args* args);

/* grad_table[t] = scale * (sum of grad_out[r] over the rows of token t, in ascending order; added up in pieces of at most 32 rows, whose
 * borders depend on the other tokens).  accumulate 0: every row is written (0 where no row has the token); 1: added to what is there, and
 * rows of no token are not touched.  Tokens outside 0..vocab - 1 are left out. */
typedef struct {
  int32_t n_rows, vocab, d;
  int32_t out_dtype, table_dtype, index_bits;   /* of grad_out, of grad_table, of tokens       */
  float scale;
  int32_t accumulate;
  int64_t out_row, table_row;
  const void *grad_out, *tokens;
  void* grad_table;
  void* workspace;               /* april_embed_grad_workspace bytes, 16-byte aligned          */
  int64_t workspace_bytes;
  void* stream;
} april_embed_grad_args;
int april_embed_grad(const april_embed_grad_args* args);
int64_t april_embed_grad_workspace(const april_embed_grad_args* args);

/* Assignments (row r, place j) -> r * k + j, sorted by expert and then by number.  Expert e's packed rows begin at starts[e], a
 * multiple of align, and starts[n_experts] is the end of the last one's; rows between hold no assignment.  Assignments of
 * an expert outside 0..n_experts - 1 are left out (position -1).
 * n_packed: rows of the packed arrays, at least (n + min(n_experts, n) * (align - 1)) / align * align for n = n_rows * k. */
typedef struct {
  int32_t n_rows, k;             /* n_rows * k below 2^31 - 4096; k 1..64                      */
  int32_t n_experts, align;      /* 1..511; 1..4096                                            */
  int32_t n_packed, index_bits;
  const void* ids;               /* [n_rows][k]                                                */
  int32_t* starts;               /* [n_experts + 1]                                            */
  int32_t* source;               /* [n_packed] assignment of each packed row, -1: none         */
  int32_t* position;             /* [n_rows][k] packed row of each assignment, -1: left out    */
  void* workspace;               /* april_expert_sort_workspace bytes, 16-byte aligned; NULL if 0 */
  int64_t workspace_bytes;
  void* stream;
} april_expert_sort_args;
int april_expert_sort(const april_expert_sort_args* args);
int64_t april_expert_sort_workspace(const april_expert_sort_args* args);

/* packed[p] = x[source[p] / k]; packed rows of no assignment are 0.  (Its gradient is april_expert_combine of packed's, without weights.)
 * source and position are april_expert_sort's; entries outside the arrays are as -1. */
typedef struct {
  int32_t n_rows, k, d;          /* d 1..2^24                                                  */
  int32_t n_packed, dtype;
  int32_t reserved;              /* 0                                                          */
  int64_t x_row, packed_row;
  const void* x;                 /* [n_rows][d]                                                */
  const int32_t *source, *position;
  void* packed;                  /* [n_packed][d]                                              */
  void* stream;
} april_expert_gather_args;
int april_expert_gather(const april_expert_gather_args* args);

/* out[r] = sum over j of weights[r][j] * packed[position[r][j]], in the order of j. */
typedef struct {
  int32_t n_rows, k, d, n_packed, dtype;
  int32_t reserved;              /* 0                                                          */
  int64_t packed_row, out_row;
  const void* packed;            /* [n_packed][d]                                              */
  const int32_t* position;       /* [n_rows][k]                                                */
  const float* weights;          /* [n_rows][k], or NULL: 1                                    */
  void* out;                     /* [n_rows][d]                                                */
  void* stream;
} april_expert_combine_args;
int april_expert_combine(const april_expert_combine_args* args);

/* Its gradients: grad_packed[p] = weight of p's assignment * grad_out of its row (0: no assignment);
 * grad_weights[r][j] = sum over d of grad_out[r] * packed[position[r][j]] (0: left out). */
typedef struct {
  int32_t n_rows, k, d, n_packed, dtype;
  int32_t reserved;              /* 0                                                          */
  int64_t out_row, packed_row, grad_packed_row;
  const void* grad_out;          /* [n_rows][d]                                                */
  const void* packed;            /* [n_packed][d]; NULL without grad_weights                   */
  const int32_t *source, *position;
  const float* weights;          /* [n_rows][k], or NULL: 1                                    */
  void* grad_packed;             /* [n_packed][d], or NULL                                     */
  float* grad_weights;           /* [n_rows][k], or NULL                                       */
  void* stream;
} april_expert_combine_grad_args;
int april_expert_combine_grad(const april_expert_combine_grad_args* args);

/* Per-kernel-class timing, measured with HIP events on the context's stream around
 * sampled launches of the real decode loop (every `every`-th iteration; 0 = off).  Two extra
 * classes calibrate the method: "event_pair_no_kernel" is what a pair of event records reads
 * with nothing between them (the cost of the pair itself; subtract it from a class's average to
 * get the launch's own time), "event_pair_empty_kernel" the same around a kernel that does
 * nothing (the floor of any single launch). */
#define APRIL_KERNEL_CLASSES 24
typedef struct {
  const char* name;
  int64_t launches;          /* timed launches                                           */
  double  total_ms;          /* their summed duration                                    */
  double  alg_bytes;         /* algorithmic HBM bytes those launches had to move         */
  double  alg_flops;         /* floating-point operations of those launches              */
} april_kernel_stat;
int april_profile_enable(april_ctx* ctx, int32_t every);
int april_profile_get(april_ctx* ctx, april_kernel_stat* out, int32_t cap);   /* returns count */
int april_profile_reset(april_ctx* ctx);

/* Device facts used for reporting: free/total bytes, KV pages, weight bytes. */
typedef struct {
  int64_t hbm_total, hbm_free, kv_pool_bytes, kv_blocks_total, kv_blocks_free,
          weight_bytes, decode_weight_bytes, kv_bytes_per_token,
          expert_bytes;   /* routed experts: bytes of one expert's matrices; decode_weight_bytes
                             then covers everything but the experts                         */
} april_info;
int april_get_info(april_ctx* ctx, april_info* out);

const char* april_last_error(const april_ctx* ctx);   /* ctx may be NULL: init errors */
void april_destroy(april_ctx* ctx);

#ifdef __cplusplus
}
#endif
#endif /* APRIL_H */
