/*
 * rgd.h - C ABI of the MI355X (gfx950) refusal-gated decoding library.
 *
 * Refusal-gated decoding (Section 3, Algorithm 1): a prompt's KV cache is
 * computed once and shared; a short greedy probe decodes against it and is
 * checked after every token for compatibility with a table of refusal
 * prefixes; a probe that stays compatible to a stop token or the length cap is
 * returned as the greedy response, otherwise the probe's own positions are
 * dropped and N high-temperature continuations are sampled from the prompt.
 *
 * Conventions (all entry points):
 *  - Every function returns an rgd_status (int32).  On failure the reason is
 *    available from rgd_last_error() (thread-local, valid until the next call
 *    on the same thread).  Arguments are validated before any HIP call; an
 *    invalid argument leaves all state untouched.
 *  - "dev" pointers are device memory (e.g. PyTorch tensors on the GPU) and
 *    "host" pointers ordinary host memory.  The caller owns every buffer it
 *    passes; the library never frees them.  The library owns its handles and
 *    the workspace it allocates in the *_create calls; no entry point on the
 *    decode path allocates device memory.
 *  - stream is a hipStream_t (NULL = the null stream).  Work is enqueued on it;
 *    calls documented as synchronous wait for that stream.
 *  - Layouts are row-major with the last index fastest.  bf16 values are IEEE
 *    bfloat16 bit patterns, fp32 values IEEE binary32.
 *  - Results are deterministic: reductions use a fixed order and no floating
 *    point atomics, so equal inputs and seeds give bit-identical outputs.
 *  - A model and its KV state hold the workspace, staging buffers and page
 *    pool every call on them uses: calls on one model (or its KV states) must
 *    not overlap, from several threads or on several streams.  Different
 *    models are independent.
 */
#ifndef RGD_H
#define RGD_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct rgd_model rgd_model;
typedef struct rgd_kv rgd_kv;
typedef struct rgd_table rgd_table;
typedef void* rgd_stream; /* hipStream_t */

enum rgd_status {
  RGD_OK = 0,
  RGD_E_INVALID_ARG = 1, /* null pointer, size out of range, bad enum */
  RGD_E_OOM = 2,         /* page pool or workspace exhausted */
  RGD_E_HIP = 3,         /* a HIP runtime call failed */
  RGD_E_UNSUPPORTED = 4, /* dtype or shape the library does not handle */
  RGD_E_NONFINITE = 5,   /* a logit row had a non-finite maximum */
  RGD_E_STATE = 6        /* entry points called out of order */
};

enum rgd_dtype { RGD_DTYPE_F32 = 0, RGD_DTYPE_BF16 = 1 };

/* Decisive probe events (Algorithm 1: incompatibility, stop, length cap). */
enum rgd_event { RGD_EVENT_INCOMPAT = 0, RGD_EVENT_STOP = 1, RGD_EVENT_MAXLEN = 2,
                 RGD_EVENT_SKIPPED = 3 /* pre-check score <= theta: sampled without a check */ };

/* Target model M: a pre-norm decoder (RMSNorm, grouped-query attention with
 * rotate-half RoPE, SwiGLU feed-forward, untied LM head).  The paper runs
 * pretrained models of this family (Section 4).  d_model = n_heads * head_dim
 * is not required; n_heads must be a multiple of n_kv_heads. */
typedef struct rgd_model_config {
  int32_t n_layers;
  int32_t d_model;
  int32_t n_heads;    /* query heads Hq */
  int32_t n_kv_heads; /* key/value heads Hkv */
  int32_t head_dim;   /* D */
  int32_t ffn_dim;
  int32_t vocab;
  int32_t dtype;      /* rgd_dtype of weights, KV cache and activations */
  float rms_eps;
  float rope_theta;
  int32_t max_pos;    /* largest position any call may use, exclusive */
} rgd_model_config;

/* Per-layer weights, device pointers in the model dtype, W[out][in] row-major
 * (y = W x).  wq [Hq*D][d_model], wk/wv [Hkv*D][d_model], wo [d_model][Hq*D],
 * w_gate/w_up [ffn][d_model], w_down [d_model][ffn].  Norm gains are fp32
 * [d_model]. */
typedef struct rgd_layer_weights {
  const void* attn_norm;
  const void* wq;
  const void* wk;
  const void* wv;
  const void* wo;
  const void* ffn_norm;
  const void* w_gate;
  const void* w_up;
  const void* w_down;
} rgd_layer_weights;

/* embed [vocab][d_model] and lm_head [vocab][d_model] in the model dtype,
 * final_norm fp32 [d_model]; layers is a host array of n_layers entries. */
typedef struct rgd_weights {
  const void* embed;
  const void* final_norm;
  const void* lm_head;
  const rgd_layer_weights* layers;
} rgd_weights;

/* Library version string (static storage). */
const char* rgd_version(void);

/* Message for the last failing call on this thread ("" if none). */
const char* rgd_last_error(void);

/* Creates a model.  bf16 weight matrices are repacked here, once, into
 * library-owned buffers in the layout the GEMM kernels stream (16-row panels
 * of 64-wide k blocks); the caller's matrices are not read afterwards.  The
 * embedding table, the norm gains and fp32 matrices are used in place and
 * must outlive the handle.  max_rows bounds the rows of any decode step
 * (probe prompts, or prompts x branches) and the tokens processed per prefill
 * chunk; the workspace for that many rows is allocated here.  bf16 models
 * require head_dim == 128 and d_model, Hq*D, ffn multiples of 128. */
int32_t rgd_model_create(const rgd_model_config* cfg, const rgd_weights* w, int32_t max_rows,
                         rgd_model** out);
void rgd_model_destroy(rgd_model* m);

/* KV state for up to max_prompts prompts of up to max_prefix positions each.
 * All caches are KV-head-major, so the positions of one head form contiguous
 * runs; values are stored transposed (head dim before position) in blocks of
 * 64 positions.  VP = max_prefix rounded up to a multiple of 64:
 *  prefix_k: dev [n_layers][max_prompts][Hkv][max_prefix][D]
 *  prefix_v: dev [n_layers][max_prompts][Hkv][VP/64][D][64]
 *    - the shared prompt KV (rotated keys), written only by rgd_prefill_kv
 *    or by the caller, read in place by every probe and branch, never copied.
 *  pool_k: dev [n_layers][n_pages][Hkv][page_size][D]
 *  pool_v: dev [n_layers][n_pages][Hkv][D][page_size]
 *    - pages of the per-row tails (probe positions, branch positions).
 * bf16 models need page_size % 16 == 0.  The handle keeps per-prompt prefix
 * lengths, page tables and the page free list.  All four buffers are caller
 * owned. */
int32_t rgd_kv_create(const rgd_model* m, int32_t max_prompts, int32_t max_prefix, int32_t n_pages,
                      int32_t page_size, void* prefix_k, void* prefix_v, void* pool_k, void* pool_v,
                      rgd_kv** out);
void rgd_kv_destroy(rgd_kv* kv);

/* Declares that positions [0, len) of prompt `prompt` hold valid KV written by
 * the caller (e.g. a synthetic prefix).  Host-side bookkeeping only. */
int32_t rgd_kv_set_prefix_len(rgd_kv* kv, int32_t prompt, int32_t len);

/* Refusal-prefix table P (Section 3; token-level matching with a minimum match
 * length, Appendix D), copied to the device.  CSR on the host: entry e is
 * tokens[offsets[e] .. offsets[e+1]).  owner (host [n_entries] or NULL):
 * owner[e] = -1 makes the entry apply to every prompt, p >= 0 to prompt p only.
 * Entries shorter than min_match tokens never match.  n_entries may be 0 (every
 * probe is then incompatible at its first token). */
int32_t rgd_table_create(const int32_t* offsets, const int32_t* tokens, int32_t n_entries,
                         const int32_t* owner, int32_t min_match, rgd_table** out);
void rgd_table_destroy(rgd_table* t);

/* Prefill (Algorithm 1, first line; the prompt KV reused by both stages):
 * tokens dev int32 [B][n] for prompts 0..B-1 at positions
 * [start_pos, start_pos + n); each prompt must already hold start_pos valid
 * positions.  Writes their K/V into the prefix, sets each prefix length to
 * start_pos + n and writes the logits of each prompt's last position to
 * last_logits dev fp32 [B][vocab].  Asynchronous. */
int32_t rgd_prefill_kv(rgd_model* m, rgd_kv* kv, const int32_t* tokens, int32_t B, int32_t n,
                       int32_t start_pos, float* last_logits, rgd_stream stream);

/* rgd_prefill_kv plus the residual-stream classifier pre-check (Appendix A):
 * for each prompt b, scores[b] = 1 / (1 + exp(-(cls_w . h_b + cls_b))) where
 * h_b is the fp32 residual stream of the prompt's last position after block
 * cls_layer (1..n_layers; 0 = the embedding).  cls_w dev fp32 [d_model]
 * (caller-owned), scores dev fp32 [B].  The logits and the KV written are those
 * of rgd_prefill_kv.  Asynchronous. */
int32_t rgd_prefill_kv_scored(rgd_model* m, rgd_kv* kv, const int32_t* tokens, int32_t B, int32_t n,
                              int32_t start_pos, float* last_logits, int32_t cls_layer, const float* cls_w,
                              float cls_b, float* scores, rgd_stream stream);

/* Greedy probe (Algorithm 1: the c-token gate G_M and the post-cap probe B_M)
 * for prompts 0..B-1.  Token 1 is the argmax of last_logits (dev fp32
 * [B][vocab]); each further token is the argmax after feeding the probe, whose
 * K/V goes to pages of the prompt's probe tail.  After every token the probe
 * is checked against tbl: incompatible -> INCOMPAT, token == eos_id (eos_id <
 * 0: none) -> STOP, k tokens -> MAXLEN.  The host polls the device state after
 * each of the first c tokens and then every c tokens, and stops launching
 * steps once no prompt is undecided (early exit); the decision does not depend
 * on c.  Outputs (dev): probe_tokens int32 [B][k], probe_len int32 [B],
 * event int32 [B] (rgd_event).  Synchronous.  tbl NULL: no refusal set, every
 * probe stays compatible, so the probe runs to k tokens (or eos): the
 * fixed-length probe of the paper's ablations.  On success the probe tails are
 * held until rgd_gate; a probe that fails after validation (a HIP error) waits
 * for its stream and releases them itself. */
int32_t rgd_probe(rgd_model* m, rgd_kv* kv, const float* last_logits, const rgd_table* tbl,
                  int32_t B, int32_t k, int32_t c, int32_t eos_id, int32_t* probe_tokens,
                  int32_t* probe_len, int32_t* event, rgd_stream stream);

/* Probe without the compatibility gate (Appendix B's fixed-probe ablation;
 * with k = L, the naive greedy-then-high-temperature approach of Section 3):
 * greedy decoding always runs to k tokens, or to eos_id when it is set, and
 * the refusal detector (the table's compatibility predicate, tbl NULL = no
 * refusal set, every probe passes) is applied to the finished probe: event
 * INCOMPAT when the probe is incompatible with every entry (a miss), else
 * STOP or MAXLEN (a hit).  By prefix closure the decision equals rgd_probe's;
 * only the decoded tokens differ (k instead of stopping at the first
 * incompatible one).  Arguments, outputs, page use and the c cadence (host
 * polls after tokens 1..c and every c tokens, which only ends prompts that
 * reached eos) as rgd_probe.  Synchronous. */
int32_t rgd_probe_fixed(rgd_model* m, rgd_kv* kv, const float* last_logits, const rgd_table* tbl,
                        int32_t B, int32_t k, int32_t c, int32_t eos_id, int32_t* probe_tokens,
                        int32_t* probe_len, int32_t* event, rgd_stream stream);

/* Probe with the soft compatibility gate (Appendix C, the soft-gate
 * algorithm); arguments and outputs as rgd_probe.  Tokens 1..c are soft steps:
 * when the greedy token would make the probe incompatible, the topk most
 * probable next tokens (softmax of the logits at temperature 1 over the whole
 * vocabulary; equal logits: lower id first) are examined, and if those that
 * keep the probe compatible carry a probability mass >= rho, the most probable
 * of them is appended instead and the probe goes on.  Otherwise the failing
 * greedy token is recorded with event INCOMPAT.  Tokens after c follow the
 * hard rule of rgd_probe (there c only sets the polling cadence; here it is
 * also the number of soft steps).  1 <= topk <= 32 and topk <= vocab; rho is
 * any non-NaN value (rho > 1 never accepts: the hard gate).  The probe tokens
 * then hold the substituted tokens, which is what a hit returns.
 * Synchronous. */
int32_t rgd_probe_soft(rgd_model* m, rgd_kv* kv, const float* last_logits, const rgd_table* tbl,
                       int32_t B, int32_t k, int32_t c, int32_t eos_id, int32_t topk, float rho,
                       int32_t* probe_tokens, int32_t* probe_len, int32_t* event, rgd_stream stream);

/* The adaptive gate (Appendix A): prompts whose pre-check score (scores dev
 * fp32 [B], from rgd_prefill_kv_scored) is <= theta skip the greedy check: they
 * get event RGD_EVENT_SKIPPED and probe_len 0 (a miss for rgd_gate, sampled
 * without any check token); the others are probed as by rgd_probe (topk 0) or
 * rgd_probe_soft (topk >= 1, with rho).  Synchronous. */
int32_t rgd_probe_adaptive(rgd_model* m, rgd_kv* kv, const float* last_logits, const rgd_table* tbl,
                           int32_t B, int32_t k, int32_t c, int32_t eos_id, int32_t topk, float rho,
                           const float* scores, float theta, int32_t* probe_tokens, int32_t* probe_len,
                           int32_t* event, rgd_stream stream);

/* Gate (Algorithm 1, the return branches): prompt b is a hit (return the
 * greedy probe) iff event[b] is STOP or MAXLEN, otherwise (INCOMPAT, SKIPPED)
 * a miss (sample from the prompt).  Releases every probe-tail page (the probe's K/V is dropped,
 * never copied; the shared prefix is untouched).  event dev int32 [B].
 * decision_host int32 [B] (1 = hit, 0 = miss), *n_miss_host, miss_idx_host
 * int32 [B] (first *n_miss_host entries: missed prompts in increasing order).
 * Synchronous. */
int32_t rgd_gate(rgd_kv* kv, const int32_t* event, int32_t B, int32_t* decision_host,
                 int32_t* n_miss_host, int32_t* miss_idx_host, rgd_stream stream);

/* S_{T,theta}(M, p) (Section 3) with temperature-scaled min-p truncation for
 * the n prompts listed in prompt_idx (host int32 [n]), N branches each, `steps`
 * tokens per branch.  Branch j of listed prompt i is row r = i*N + j; it uses
 * Philox key seeds[r] (dev uint64 [n*N]) and counter (s, 0) for token s.
 * Token 0 is drawn from last_logits (dev fp32 [B][vocab], row prompt_idx[i]);
 * token s >= 1 from the logits after feeding token s-1 at position
 * prefix_len + s - 1 (the branch restarts from the prompt; probe positions are
 * not visible).  T == 0 is greedy argmax.  A token i is kept iff
 * exp((z_i - max z)/T) >= min_p; the draw is the smallest kept id whose running
 * kept weight exceeds u * (total kept weight).
 *  forced (dev int32 [n*N][steps] or NULL): if given, token forced[r][s-1] is
 *    fed at step s instead of the drawn one (teacher forcing for tests).
 *  logits_tap (dev fp32 [steps][n*N][vocab] or NULL): receives every step's
 *    logits (tests).
 *  out: dev int32 [n][N][steps].
 * Asynchronous.  Requires every probe tail to have been released (rgd_gate). */
int32_t rgd_sample_continuations(rgd_model* m, rgd_kv* kv, const float* last_logits,
                                 const int32_t* prompt_idx, int32_t n, int32_t N, int32_t steps,
                                 float T, float min_p, const uint64_t* seeds, const int32_t* forced,
                                 float* logits_tap, int32_t* out, rgd_stream stream);

/* As rgd_sample_continuations, with p-less truncation in place of min-p (the
 * truncation Section 4 samples with; its rule, from the cited p-less paper:
 * with p = softmax(z/T), keep token i iff p_i >= sum_j p_j^2, which is
 * exp((z_i - max z)/T) >= S2/S1 for S1, S2 the sums of those weights and of
 * their squares).  No parameter besides T; T == 0 is greedy argmax.  The
 * vocabulary must be a multiple of 4 (RGD_E_UNSUPPORTED otherwise). */
int32_t rgd_sample_continuations_pless(rgd_model* m, rgd_kv* kv, const float* last_logits,
                                       const int32_t* prompt_idx, int32_t n, int32_t N, int32_t steps,
                                       float T, const uint64_t* seeds, const int32_t* forced,
                                       float* logits_tap, int32_t* out, rgd_stream stream);

/* Checks the device status flag raised by the sampler (non-finite row
 * maximum) and clears it.  Synchronous. */
int32_t rgd_check_status(rgd_model* m, rgd_stream stream);

/* ---- in-situ kernel timing (measurement hooks for the benchmark) ---- */

/* Timed units: the LM-head GEMM; the whole attention stage (shared-prefix
 * kernel, tail kernel and combine); the shared-prefix attention kernel alone;
 * the min-p sampler kernel of a decode step; one whole decode step (all layers,
 * LM head and token selection). */
enum rgd_timer {
  RGD_TIMER_LM_HEAD = 0,
  RGD_TIMER_ATTENTION = 1,
  RGD_TIMER_ATTN_PREFIX = 2,
  RGD_TIMER_SAMPLER = 3,
  RGD_TIMER_STEP = 4,
  RGD_TIMER_COUNT = 5
};

/* period >= 1: from now on the model records HIP events on the work stream
 * around timed units.  Inside rgd_sample_continuations, decode step s (s >= 1)
 * is timed when (s - 1) % period == 0, and only one unit is timed in such a
 * step: unit ((s - 1) / period) % RGD_TIMER_COUNT (LM head, attention stage,
 * shared-prefix attention kernel, sampler, whole step, in turn), so that no
 * unit's measurement holds another unit's event records; the draw from the
 * prompt's logits is never timed.  Elsewhere every launch of every unit is
 * timed (the prefix kernel's events then sit inside the attention stage's).
 * At most 8192 timed launches per unit between reads; later launches are not
 * timed.  Each event record leaves a small idle gap on the stream.  period == 0
 * stops recording; negative is RGD_E_INVALID_ARG.  Events are created on the
 * first enable, not on the decode path. */
int32_t rgd_timing_enable(rgd_model* m, int32_t period);

/* Waits for the recorded events and returns, per timed unit, the summed
 * duration in milliseconds (ms[RGD_TIMER_COUNT]) and the number of launches
 * (launches[RGD_TIMER_COUNT]); then clears the records.  Synchronous. */
int32_t rgd_timing_read(rgd_model* m, double* ms, int64_t* launches);

/* ---- kernel-level entry points (used by the tests and the benchmark) ---- */

/* Decode attention for R rows of one layer: q dev [R][Hq][D] (model dtype)
 * over prompt row_prompt[r]'s first plen[r] prefix positions followed by
 * tail_len positions of the row's own tail.  row_prompt and plen are HOST int32
 * [R]; rows of one prompt must be contiguous.  prefix_k, prefix_v, pool_k,
 * pool_v are one layer of the layouts of rgd_kv_create; pages dev int32
 * [R][max_pages] (may be NULL when tail_len == 0).  out dev
 * [R][Hq*D] (model dtype).  splits = 0 picks the prefix split count.
 * Asynchronous. */
int32_t rgd_kernel_attention(rgd_model* m, const void* q, int32_t R, const int32_t* row_prompt,
                             const int32_t* plen, const void* prefix_k, const void* prefix_v,
                             int32_t max_prompts, int32_t max_prefix, const void* pool_k,
                             const void* pool_v, int32_t page_size, const int32_t* pages,
                             int32_t max_pages, int32_t tail_len, int32_t splits, void* out,
                             rgd_stream stream);

/* LM head: logits dev fp32 [R][vocab] = h W_lm^T with h dev [R][d_model]
 * (model dtype, the already normalised final hidden state).  Asynchronous. */
int32_t rgd_kernel_lm_head(rgd_model* m, const void* h, int32_t R, float* logits, rgd_stream stream);

/* Bytes of caller-provided device workspace the sampler entry points below
 * need for R rows of V logits. */
uint64_t rgd_sampler_workspace_bytes(int32_t R, int32_t V);

/* Greedy token of each row of z dev fp32 [R][V] (first index of the maximum)
 * -> out dev int32 [R].  workspace: dev, rgd_sampler_workspace_bytes(R, V)
 * bytes, 256-byte aligned.  Asynchronous. */
int32_t rgd_kernel_argmax(const float* z, int32_t R, int32_t V, void* workspace, int32_t* out,
                          rgd_stream stream);

/* min-p draws on z dev fp32 [R][V] (V a multiple of 4, V <= 1048576, T > 0,
 * 0 <= min_p <= 1): draw d of row r uses Philox key seeds[r] (dev uint64 [R])
 * and counter (ctr, stream0 + d); out dev int32 [R][draws].  workspace as for
 * rgd_kernel_argmax.  Asynchronous. */
int32_t rgd_kernel_sample(const float* z, int32_t R, int32_t V, float T, float min_p,
                          const uint64_t* seeds, uint32_t ctr, uint32_t stream0, int32_t draws,
                          void* workspace, int32_t* out, rgd_stream stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the draws of
 * rgd_kernel_sample, same arguments without the workspace, which is taken from
 * a fixed array of RGD_NOALLOC_SCRATCH_BYTES the library holds on each device
 * it runs on until the process ends.  Allocates nothing.  Calls with
 * rgd_sampler_workspace_bytes(R, V) > RGD_NOALLOC_SCRATCH_BYTES are rejected
 * (RGD_E_INVALID_ARG) before any HIP call.  Every call on one device shares
 * that array: calls that overlap on one device (several streams or threads)
 * race and must be serialised by the caller.  The first call on a device
 * looks up the array's device address (hipGetSymbolAddress) with that device
 * current.  Asynchronous. */
#define RGD_NOALLOC_SCRATCH_BYTES 1048576
int32_t rgd_kernel_sample_noalloc(const float* z, int32_t R, int32_t V, float T, float min_p,
                                  const uint64_t* seeds, uint32_t ctr, uint32_t stream0, int32_t draws,
                                  int32_t* out, rgd_stream stream);

/* p-less draws on z dev fp32 [R][V] (keep p_i >= sum_j p_j^2 of softmax(z/T),
 * see rgd_sample_continuations_pless; V a multiple of 4, V <= 1048576,
 * T > 0); seeds, counters, workspace and out as for rgd_kernel_sample.
 * Asynchronous. */
int32_t rgd_kernel_sample_pless(const float* z, int32_t R, int32_t V, float T, const uint64_t* seeds,
                                uint32_t ctr, uint32_t stream0, int32_t draws, void* workspace,
                                int32_t* out, rgd_stream stream);

/* One probe step (Algorithm 1, or the soft gate of Appendix C when topk > 0)
 * for prompts 0..R-1 of the table, given their next-token logits dev fp32
 * [R][vocab of m] and their probe state probe_tokens dev int32 [R][k],
 * probe_len, event dev int32 [R] (updated in place; prompts whose event is
 * not -1 are left alone): appends one token and sets the event as rgd_probe
 * and rgd_probe_soft do for their step (c: soft steps when topk > 0; tbl NULL:
 * no table).  Uses m's workspace, so calls on one model must not overlap.
 * Asynchronous. */
int32_t rgd_kernel_probe_step(rgd_model* m, const float* logits, int32_t R, const rgd_table* tbl,
                              int32_t k, int32_t c, int32_t eos_id, int32_t topk, float rho,
                              int32_t* probe_tokens, int32_t* probe_len, int32_t* event,
                              rgd_stream stream);

/* ---- paged sequences: a cache whose sequences differ in length, share pages
 * and are forked, rolled back and compacted on the device ----
 *
 * A plain description of caller-owned device buffers (no handle; the fields are
 * read during the call).  Sequence s holds positions [0, lens[s]); position t
 * lies in slot t % page_size of page pages[s][t / page_size].  Several
 * sequences may hold the same page; refs[p] counts the table entries that hold
 * page p, 0 for a free one.  A cache starts with lens and refs 0.  The entry
 * points below keep these arrays in line, take them in stream order and leave
 * the host out of it, so a step of them can be captured into a graph.
 * Entries of a table behind a sequence's pages say nothing.  A length outside
 * [0, max_pages * page_size] counts as the nearest one inside; positions whose
 * table entry is outside [0, n_pages) are neither written nor attended to. */
typedef struct rgd_paged_cache {
  int32_t n_layers;   /* at most 65536 */
  int32_t n_pages;    /* at most 2^20 */
  int32_t n_kv_heads; /* Hkv, at most 1024 */
  int32_t page_size;  /* positions per page: a multiple of 16, at most 4096 */
  int32_t head_dim;   /* D: 32, 64 or 128 */
  int32_t dtype;      /* rgd_dtype of K and V */
  int32_t max_seqs;   /* S, at most 65536 */
  int32_t max_pages;  /* table entries per sequence, at most 2^30 positions */
  void* pool_k;       /* dev [n_layers][n_pages][Hkv][page_size][D], as in rgd_kv_create */
  void* pool_v;       /* dev [n_layers][n_pages][Hkv][D][page_size] */
  int32_t* pages;     /* dev [S][max_pages] */
  int32_t* lens;      /* dev [S] */
  int32_t* refs;      /* dev [n_pages] */
  int32_t* status;    /* dev [1]: set to 1 by an rgd_paged_reserve that found no room */
} rgd_paged_cache;

/* Bytes of caller-provided device workspace (256-byte aligned) that
 * rgd_paged_select, rgd_paged_reserve and rgd_paged_compact need; 0 for a
 * description they refuse.  Calls that share a workspace must not overlap; a
 * workspace and what a call writes are apart from its inputs and from the cache. */
uint64_t rgd_paged_workspace_bytes(const rgd_paged_cache* cache);

/* Forks, reorders, rolls back and frees, all sequences at once: sequence s
 * becomes the first min(keep[s], len) positions of what sequence parent[s] was
 * before the call.  No K or V is copied: the pages are shared.  parent dev
 * int32 [S] (NULL, or an entry outside [0, S): s itself), keep dev int32 [S]
 * (NULL or negative: every position; 0 frees the sequence).  refs follows;
 * table entries that a sequence no longer has become -1.  workspace may be
 * NULL when parent is.  Asynchronous. */
int32_t rgd_paged_select(const rgd_paged_cache* cache, const int32_t* parent, const int32_t* keep, void* workspace,
                         rgd_stream stream);

/* Makes room for grow[s] more positions (dev int32 [S]; negative counts as 0)
 * behind each sequence and adds them to lens.  New pages are the lowest free
 * ones, in the order of the sequences.  A sequence that grows and whose last
 * page is partly filled and held by another table entry too gets a copy of that
 * page (every layer) in its place, so the new positions are its own.  That goes by
 * refs before the call: where all N holders of a page grow, each gets a copy, which takes
 * N free pages, and the original is free afterwards.  If the
 * pool has too few free pages or a table too few entries, status[0] is set to 1
 * and nothing else is changed.  Asynchronous. */
int32_t rgd_paged_reserve(const rgd_paged_cache* cache, const int32_t* grow, void* workspace, rgd_stream stream);

/* As rgd_paged_reserve; granted (dev int32 [S]; grow itself, or apart from it) receives how many positions
 * each sequence got: max(grow[s], 0), or 0 for every sequence where there was no room.  What is queued
 * behind a reserve without the host's look at status takes its counts from here: an append and an
 * attention with n_new = granted, and a roll-back to lens - granted + kept, leave a cache that had no room
 * as it is, where grow would have them write over and drop older positions. */
int32_t rgd_paged_reserve_granted(const rgd_paged_cache* cache, const int32_t* grow, int32_t* granted,
                                  void* workspace, rgd_stream stream);

/* Moves pages so that the pages held by any sequence (refs > 0) are the pages
 * [0, n): those at or above n go, in order, to the free ones below it, in every
 * layer; tables and refs follow.  live dev int32 [1] receives n.  Asynchronous. */
int32_t rgd_paged_compact(const rgd_paged_cache* cache, int32_t* live, void* workspace, rgd_stream stream);

/* Writes the K and V of each sequence's last n_new[s] positions (dev int32 [S],
 * counts outside [0, n] as the nearest inside; NULL: n of each) of one layer:
 * token i of sequence s goes to position lens[s] - n_new[s] + i, whatever is there (a reserve
 * that had room has made it, so that no other sequence holds its page; behind one that may have had none,
 * n_new is what rgd_paged_reserve_granted granted; positions before 0 are left out).  k, v dev in the cache's type:
 * row s * n + i at k + (s * n + i) * ldk elements, [Hkv][D] each; keys already
 * rotated.  ldk, ldv >= Hkv * D; k, v and their row strides 16-byte aligned.
 * Asynchronous. */
int32_t rgd_paged_append(const rgd_paged_cache* cache, int32_t layer, const void* k, const void* v, int64_t ldk,
                         int64_t ldv, int32_t n, const int32_t* n_new, rgd_stream stream);

/* Bytes of device workspace (256-byte aligned) for rgd_paged_attention with up
 * to n new tokens per sequence and n_heads query heads; 0 for arguments it
 * refuses. */
uint64_t rgd_paged_attention_workspace_bytes(const rgd_paged_cache* cache, int32_t n, int32_t n_heads);

/* Causal attention of each sequence's last n_new[s] positions (as for
 * rgd_paged_append, whose K and V are in the cache) over the whole sequence, one
 * layer: token i sees positions [0, lens[s] - n_new[s] + i].  q dev in the
 * cache's type, row s * n + i at q + (s * n + i) * ldq elements, [n_heads][D]
 * (16-byte aligned rows); query head h reads KV head h / (n_heads / Hkv), scores
 * are scaled by 1/sqrt(D).  out dev [S * n][n_heads * D] in the cache's type
 * (16-byte aligned), lse dev fp32 [S * n][n_heads] or NULL:
 * the log of the sum of exponentiated scores, for joining with attention over
 * other positions.  out, lse and the workspace overlap neither each other, nor q, n_new or the cache.  A token that
 * sees nothing gets 0 and -inf; rows at or behind
 * n_new[s] are left as they were.  Slots behind a length and free pages may hold
 * anything.  A value of V that is not finite makes its dimension of the tokens
 * that see it inf or NaN and no other; sums are fp32, so a sequence's sum of |V|
 * in a dimension must stay below 2^128.  1 <= n <= 1024, S * n <= 2^24, n_heads <= 1024.  Meant for few tokens: every 64
 * query vectors (tokens x query heads per KV head; 32 in fp32 with D = 128) of a sequence read its K and
 * V once.  The same call gives the same bits; how a sequence's sums are associated also depends on the other
 * sequences' lengths and on max_pages, so its last bits may differ in another batch.  Asynchronous. */
int32_t rgd_paged_attention(const rgd_paged_cache* cache, int32_t layer, const void* q, int64_t ldq, int32_t n,
                            const int32_t* n_new, int32_t n_heads, void* workspace, void* out, float* lse,
                            rgd_stream stream);

/* ---- verification of drafted tokens ---- */

/* Bytes of device workspace (256-byte aligned) for rgd_verify_drafts; 0 for
 * sizes it refuses. */
uint64_t rgd_verify_workspace_bytes(int32_t S, int32_t K, int32_t V);

/* Checks up to K drafted tokens of each of S sequences against the target's
 * distribution, so that the tokens kept are distributed as if they had been
 * sampled from the target one by one.  target dev fp32 [S][K+1][V]: row i holds
 * the logits after the first i drafts.  draft dev fp32 [S][K][V]: the logits
 * draft_tokens (dev int32 [S][K]) were sampled from with the same T and min_p,
 * or NULL: the drafts carry no distribution (a greedy probe, a lookup), each
 * counts as certain.  n_draft dev int32 [S] or NULL (K of each; counts outside
 * [0, K] as the nearest inside).  u dev fp32 [S][K+1]: uniform in [0, 1).
 * With p_i the distribution of rgd_sample_continuations on target row i
 * (temperature T, then min-p; T == 0: the first maximum has everything) and q_i
 * that of draft row i (one-hot at the draft without draft logits or at T == 0):
 * draft x_i is accepted while u[i] q_i(x_i) < p_i(x_i).  At the first refusal the next
 * token is drawn from max(p_i - q_i, 0), after n_draft acceptances from p_i, by
 * u[K]: the smallest id whose running weight exceeds u[K] times the total.
 * Kept ids are those with z_i - max z >= T ln(min_p) in fp64; the sampler goes by the weight in fp32, so an id
 * whose weight is within 1e-5 of itself of min_p may be kept by one of the two only.
 * out dev int32 [S][K+1]: the accepted drafts, the drawn token, then -1;
 * n_accepted dev int32 [S]; these and the workspace overlap neither each other nor an input.  A draft
 * outside [0, V) is refused.  NaN logits
 * count as -inf.  A target row whose maximum is not finite has no distribution:
 * its draft is refused and -1 stands for the drawn token; such a draft row has
 * q = 0.  1 <= S <= 65536, 1 <= K <= 255, 2 <= V <= 1048576, S (2 K + 1)
 * ceil(V / 8192) <= 2^23, T >= 0, min_p in [0, 1].  Sums are taken in fp64, so
 * that the draw is the exact one unless u[K] meets the border of two tokens by
 * 1e-11 of p's sum (not of the rest's, which is small where q is near p).  Asynchronous. */
int32_t rgd_verify_drafts(const float* target, const float* draft, const int32_t* draft_tokens,
                          const int32_t* n_draft, int32_t S, int32_t K, int32_t V, float T, float min_p,
                          const float* u, void* workspace, int32_t* out, int32_t* n_accepted, rgd_stream stream);

/* ---- rotary positions and head norms of a paged cache's new tokens ---- */

/* How the frequencies theta^(-2j/dim) of a rotation are changed for contexts longer than the trained one
 * (`context` positions) by `factor`. */
enum rgd_rotary_kind {
  RGD_ROTARY_LINEAR = 1,       /* each over factor */
  RGD_ROTARY_BASE = 2,         /* theta times factor^(dim / (dim - 2)): the first kept, the last over factor */
  RGD_ROTARY_BY_ROTATIONS = 3, /* by the turns r a pair makes over context: over factor for r <= low, kept for
                                  r >= high, in between linear in r */
  RGD_ROTARY_BY_INDEX = 4      /* linear in the pair's index between the pair (rounded down) that makes `high` turns
                                  and the one (rounded up) that makes `low`; cosine and sine are scaled by
                                  1 + ln(factor) / 10 */
};

typedef struct rgd_rotary_scaling {
  int32_t kind;   /* rgd_rotary_kind */
  double factor;  /* >= 1 */
  double context; /* > 0 (the last two kinds) */
  double low;     /* 0 < low < high (the last two kinds) */
  double high;
} rgd_rotary_scaling;

/* The frequencies of a rotation of `dim` dimensions (even, 2 to 128): freq host fp64 [dim / 2] receives the radians per
 * position of each pair, scale host [1] the factor of cosine and sine.  scaling NULL: theta^(-2j/dim) and 1.
 * theta > 1; RGD_ROTARY_BASE needs dim > 2.  No HIP call. */
int32_t rgd_rotary_frequencies(int32_t dim, double theta, const rgd_rotary_scaling* scaling, double* freq,
                               float* scale);

/* A rotation of the first dim dimensions of a head: pair j, of dimensions (j, j + dim / 2) or, interleaved,
 * (2 j, 2 j + 1), turns by position * freq[j] radians: (a, b) -> scale (a cos - b sin, b cos + a sin).  Read during the
 * call. */
typedef struct rgd_rotary {
  int32_t dim;         /* even, 0 (no rotation) to head_dim */
  int32_t interleaved;
  float scale;
  const double* freq;  /* host [dim / 2], finite; of any source */
} rgd_rotary;

/* rgd_paged_append for rows as a fused projection leaves them, together with what attention needs of q: the heads of
 * q and k are normed, x / sqrt(mean(x^2) + eps) times a gain for each dimension (q_norm, k_norm dev fp32 [D]; NULL:
 * that one is left as it is), rotated by their token's position, and k and v are written to the pages of one layer as
 * rgd_paged_append does, q to q_out.  Token i of sequence s has the position lens[s] - n_new[s] + i, or
 * positions[s * n + i] (dev int32 [S * n], any value) where positions is given; the slot in the cache stays
 * the former.  q, k, v dev in the cache's type, row s * n + i at q + (s * n + i) * ldq elements [n_heads][D],
 * k and v [Hkv][D]; q_out alike, with ldo: q itself with its stride, or apart from every input.  Values are rounded
 * once, to the cache's type; norms, angles' remainders (taken in fp64) and rotations are fp32, so a head's sum of squares is to lie
 * within fp32's normal numbers, or below them with an eps that does not.  Rows at or behind n_new[s]
 * are left as they were; a token before position 0 or on a page outside the pool gets its q and no K and V.
 * rotary NULL: no rotation.  ld* at least a row's elements; rows 16-byte aligned; eps >= 0 and finite; 1 <= n,
 * S * n <= 2^24, n_heads a multiple of Hkv, at most 1024.  The inputs are apart from the cache.  Asynchronous. */
int32_t rgd_paged_append_rotated(const rgd_paged_cache* cache, int32_t layer, const void* q, const void* k,
                                 const void* v, int64_t ldq, int64_t ldk, int64_t ldv, int32_t n,
                                 const int32_t* n_new, int32_t n_heads, const int32_t* positions,
                                 const rgd_rotary* rotary, const float* q_norm, const float* k_norm, float eps,
                                 void* q_out, int64_t ldo, rgd_stream stream);

/* ---- attention of sequences that share leading pages ---- */

/* Bytes of the plan (256-byte aligned device memory) that rgd_paged_share writes for up to n new tokens per sequence
 * and n_heads query heads; 0 for arguments it refuses.  Besides rgd_paged_attention's limits, max_seqs * n * n_heads is at
 * most 2^22, max_seqs * n * (n_heads / Hkv)^2 below 2^31, and the tables hold at most 2^38 units of the work of all groups,
 * a unit a step of 32 or 64 positions of 16 to 128 query vectors of one KV head. */
uint64_t rgd_paged_share_bytes(const rgd_paged_cache* cache, int32_t n, int32_t n_heads);

/* Finds what the sequences of each group share, once for all layers of a turn: sequences with equal labels in
 * group (dev int32 [S]; one outside [0, S): a sequence by itself; NULL: all are one group) that have new tokens (n_new
 * dev int32 [S], counts outside [0, n] as the nearest inside; NULL: n of each) share the leading table entries that
 * are the same in all of them, as far as whole pages in front of each one's new tokens go.  Labels are hints: a group
 * that shares nothing costs nothing but the search, and one label for all finds what all share.  plan receives
 * this for rgd_paged_attention_shared; it holds for these lens, tables and counts.  shared (dev int32 [S], or NULL)
 * receives the positions that each sequence shares, 0 where it is its group's only one with new tokens.  Asynchronous. */
int32_t rgd_paged_share(const rgd_paged_cache* cache, int32_t n, const int32_t* n_new, int32_t n_heads,
                        const int32_t* group, void* plan, int32_t* shared, rgd_stream stream);

/* Bytes of device workspace (256-byte aligned) for rgd_paged_attention_shared with these n and n_heads; 0 for
 * arguments it refuses. */
uint64_t rgd_paged_attention_shared_workspace_bytes(const rgd_paged_cache* cache, int32_t n, int32_t n_heads);

/* rgd_paged_attention with the counts of a plan, whose shared positions are read once for all sequences of their group: the
 * same outputs but for the rounding of their sums, the same rows, limits and handling of bad pages and of values that
 * are not finite.  plan: written by rgd_paged_share for the same n, n_heads and sizes of the cache; where it was
 * not, every row of out and lse is left as it was.  Asynchronous. */
int32_t rgd_paged_attention_shared(const rgd_paged_cache* cache, int32_t layer, const void* q, int64_t ldq, int32_t n,
                                   int32_t n_heads, const void* plan, void* workspace, void* out, float* lse,
                                   rgd_stream stream);

/* ---- sampling with limits for each row ---- */

/* Bytes of device workspace (256-byte aligned) for rgd_sample_truncated; 0 for sizes it refuses. */
uint64_t rgd_sample_truncated_workspace_bytes(int32_t R, int32_t V);

/* Draws one id from each row of logits z (dev fp32, row r at z + r * ldz, V ids) under limits of its own.  The ids are
 * ordered by logit, equal ones lower id first, and weighted w = exp((z - max z) / T).  Kept are, in this order,
 *   the first top_k ids (dev int32 [R]; below 1, or NULL: no limit),
 *   of these, every id with less than top_p of their weight in front of it (dev fp32 [R]; 1 and above, NaN, or
 *   NULL: no limit; the first id is always kept),
 *   of these, every id with z - max z >= T ln(min_p) (dev fp32 [R]; 0 and below, NaN, or NULL: no limit; above 1 as 1).
 * The id drawn is the smallest one whose running kept weight, in the order of the ids, exceeds u (dev fp32 [R], uniform in
 * [0, 1); outside as the nearest inside, NaN as 0) times the kept weight.  T dev fp32 [R] (NULL: 1); where it is 0,
 * negative or NaN the first maximum is drawn.  out dev int32 [R]; logp dev fp32 [R] or NULL: the logarithm of the drawn
 * id's share of the kept weight.  NaN logits count as -inf, which is never kept; a row whose maximum is not finite gives
 * -1 and -inf.  Weights are taken in 64 bits, to 2^-46 of themselves and then to 2^-44 of the largest (less weighs nothing),
 * and sums are of whole multiples of 2^-43, so that they do not depend on their order: the draw is the exact one unless u or a
 * limit meets the border of two ids by 2^-43 of the largest weight for each id or less.  The same row gives the same id in any batch.  1 <= R <= 65536,
 * 1 <= V <= 2^20, ldz >= V.  out, logp and the workspace overlap neither each other nor an input.  Asynchronous. */
int32_t rgd_sample_truncated(const float* z, int64_t ldz, int32_t R, int32_t V, const float* T, const int32_t* top_k,
                             const float* top_p, const float* min_p, const float* u, void* workspace, int32_t* out,
                             float* logp, rgd_stream stream);

#ifdef __cplusplus
}
#endif

#endif /* RGD_H */
