/*
 * tasp.h - C ABI of the compiled structured-sparse decoder runtime for MI355X (gfx950).
 *
 * A structured mask removes, per decoder layer, whole GQA KV groups together with their query
 * heads, single query heads inside a kept group, and SwiGLU channels (gate row, up row and down
 * column together). The mask is closed under those dependencies (paper, Sec. "Dependency-Closed
 * Masks and Cache-Consistent Routing") and then compiled once into a plan: the retained rows and
 * columns of every projection are copied into dense INT8 panels (same section, and the appendix
 * paragraph "Backing-store semantics"), so that every later decode step and prefill launches only
 * the smaller contractions. One plan serves a whole request, its prefill and all of its decode
 * steps; a cache filled under one mask is refused by a plan of another mask (same section).
 *
 * Model: Llama-3 style decoder layer. Per layer and token, with residual r (float32):
 *   n = RMSNorm(r; gamma_attn); [q; k; v] = Wqkv n; RoPE(q, k) at the token position;
 *   append BF16 k, v to the cache; o = softmax(q K^T / sqrt(d_h)) V per retained head;
 *   r += Wo o; n2 = RMSNorm(r; gamma_ffn); h = silu(Wg n2) * (Wu n2); r += Wd h.
 * A stack applies L layers, then logits = W_lm RMSNorm(r; gamma_final) with a dense BF16 LM head.
 *
 * Conventions used by every entry point
 *   - Weights: INT8, row-major [out][in], one float32 scale per output row (W = q * s).
 *   - Query head h belongs to KV group h / (n_q_heads / n_kv_heads); heads are never regrouped.
 *   - RoPE: rotate-half pairs (i, i + d_h/2), angle = pos * theta^(-2i/d_h).
 *   - KV cache: BF16, K and V separate, [n_layers][batch][n_kv_heads][max_seq][head_dim]. Only
 *     retained groups' rows are read or written. Decode at `pos` writes row `pos` and attends
 *     over rows 0..pos inclusive, reading the stored BF16 values.
 *   - Activations x / out: float32; rows of `d_model` (decode: [batch][d_model]).
 *   - Pointers marked (device) are HIP device pointers; (host) are host pointers.
 *   - Streams are `hipStream_t` passed as void*; NULL is the default stream.
 *   - Every device buffer is owned by the caller. The library allocates no device memory and owns
 *     only a plan's host metadata until tasp_plan_destroy.
 *   - Errors: all arguments are validated on the host before any work is enqueued; on error
 *     nothing is enqueued and the status says why. tasp_last_error() gives thread-local detail.
 *     HIP failures map to TASP_ERR_HIP with the runtime's message. No C++ exception crosses the ABI.
 */
#ifndef TASP_H
#define TASP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t tasp_status;
enum {
  TASP_OK = 0,
  TASP_ERR_INVALID_ARG = -1,      /* null pointer, negative size, wrong enum value        */
  TASP_ERR_SHAPE = -2,            /* model or call shape not supported / inconsistent      */
  TASP_ERR_MASK = -3,             /* mask byte other than 0 or 1                           */
  TASP_ERR_WORKSPACE = -4,        /* workspace too small or misaligned                     */
  TASP_ERR_POS_RANGE = -5,        /* pos / pos0 + T outside the cache or the plan's limits */
  TASP_ERR_CACHE_PLAN_MISMATCH = -6, /* cache bound to a plan of another mask              */
  TASP_ERR_HIP = -7,              /* HIP runtime error                                     */
  TASP_ERR_UNSUPPORTED = -8,      /* valid request this build does not implement           */
  TASP_ERR_INTERNAL = -9          /* device result disagrees with the host's check         */
};

typedef struct tasp_plan_s* tasp_plan;   /* opaque; immutable after tasp_compile_plan */

/* Model geometry and the plan's capacity limits.
 *   n_layers >= 1; d_model % 16 == 0; head_dim in {64, 128}; n_q_heads % n_kv_heads == 0 with
 *   n_q_heads / n_kv_heads <= 8; d_ffn % 16 == 0; vocab = 0 for a bare layer stack (decode
 *   returns the residual) or > 0 for a stack ending in the BF16 LM head (decode returns logits).
 *   max_batch in 1..8 (decode batch), max_seq = cache rows per sequence, max_prefill = largest
 *   prefill chunk T (0: prefill unused, no prefill scratch is reserved). */
typedef struct {
  int32_t n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn, vocab;
  int32_t max_batch, max_seq, max_prefill;
  float rms_eps;
  float reserved0;
  double rope_theta;
} tasp_model_desc;

typedef struct {
  const int8_t* w;        /* (device) int8 [out][in], row-major, 16-byte aligned */
  const float* scale;     /* (device) float32 [out] */
} tasp_qmat;

/* One layer of the INT8 store: wq [Hq*dh][d], wk/wv [Hkv*dh][d], wo [d][Hq*dh],
 * wg/wu [d_ffn][d], wd [d][d_ffn]; attn_norm / ffn_norm are BF16 gains [d] (device). */
typedef struct {
  tasp_qmat wq, wk, wv, wo, wg, wu, wd;
  const uint16_t* attn_norm;
  const uint16_t* ffn_norm;
} tasp_layer;

/* The store: layers (host array of n_layers), and for vocab > 0 the final BF16 norm gain [d]
 * and the dense BF16 LM head [vocab][d] (device). The plan copies what it needs, so the store
 * may be freed once tasp_compile_plan's stream work has completed. */
typedef struct {
  const tasp_layer* layers;
  const uint16_t* final_norm;
  const uint16_t* lm_head;
} tasp_store;

/* Host bytes in {0, 1}: q_keep [n_layers][n_q_heads], kv_keep [n_layers][n_kv_heads] (NULL: all
 * kept), ffn_keep [n_layers][d_ffn]. A NULL tasp_mask* means the dense (all-kept) plan. A mask
 * that is not dependency-closed is closed, not rejected: a head in a dropped group is dropped,
 * and a group with no retained head is dropped. */
typedef struct {
  const uint8_t* q_keep;
  const uint8_t* kv_keep;
  const uint8_t* ffn_keep;
} tasp_mask;

/* A caller-owned KV cache (device BF16 arrays, layout above). plan_sig records the plan the
 * cache contents belong to; it is set by tasp_kv_bind and checked by decode and prefill. */
typedef struct {
  void* k;
  void* v;
  int32_t batch;          /* sequences in the cache, 1..max_batch */
  int32_t max_seq;        /* rows per sequence, <= the plan's max_seq */
  uint64_t plan_sig;
} tasp_kv_cache;

/* Index lists of tasp_plan_indices. */
enum { TASP_IDX_Q = 0, TASP_IDX_KV = 1, TASP_IDX_QKVSLOT = 2, TASP_IDX_FFN = 3 };
/* Panels of tasp_plan_panel. */
enum { TASP_PANEL_QKV = 0, TASP_PANEL_O = 1, TASP_PANEL_GATE = 2, TASP_PANEL_UP = 3,
       TASP_PANEL_DOWN = 4 };

/* Workspace bytes that tasp_compile_plan needs for this mask (paper, Sec. "Dependency-Closed
 * Masks and Cache-Consistent Routing": each mask's retained units are packed into contiguous
 * tensors; Eqs. flop-attn and flop-mlp give the retained panel shapes): panels, copies of the
 * gains and LM head, RoPE table, decode and prefill scratch. The mask is closed on the host to
 * size it. desc, mask: host; *bytes (host) receives the size. Errors: TASP_ERR_SHAPE for an
 * unsupported desc, TASP_ERR_MASK for a byte other than 0 / 1. */
tasp_status tasp_plan_workspace_bytes(const tasp_model_desc* desc, const tasp_mask* mask,
                                      size_t* bytes);

/* Compile a plan (paper, Sec. "Dependency-Closed Masks and Cache-Consistent Routing": one
 * compiled launch plan per mask over the INT8 store). Uploads the mask, runs the closure/index kernel (one workgroup per layer; integer-only), gathers
 * the retained rows / columns and their scales into the panels inside `workspace` (device, 256-byte
 * aligned, >= tasp_plan_workspace_bytes), and zeroes the decode scratch. Synchronises `stream`
 * once to read the index lists back; returns TASP_ERR_INTERNAL if they differ from the host's
 * closure. The workspace must outlive the plan and must not be shared between plans. */
tasp_status tasp_compile_plan(const tasp_model_desc* desc, const tasp_store* store,
                              const tasp_mask* mask, void* workspace, size_t workspace_bytes,
                              void* stream, tasp_plan* out);

/* ---- shared-store plans (paper, appendix "Backing-store semantics": every mask indexes one
 * immutable packed store and owns no weight bytes, so memory grows only by plan metadata; Table
 * "configuration": symmetric groupwise INT8, group size 128, BF16 scales).
 *
 * Groupwise matrix: w int8 [out][in] row-major (16-byte aligned), scale BF16 bits
 * [out][in / 128] (2-byte aligned); W[o][i] = w[o][i] * scale[o][i / 128]. */
typedef struct {
  const int8_t* w;
  const uint16_t* scale;
} tasp_gqmat;

/* One layer of the packed groupwise store: wqkv [(n_q_heads + 2 n_kv_heads) head_dim][d] holds
 * every query head's rows, then every K row, then every V row; wo [d][n_q_heads head_dim];
 * wg / wu [d_ffn][d]; wd [d][d_ffn]; gains BF16 [d] (device). */
typedef struct {
  tasp_gqmat wqkv, wo, wg, wu, wd;
  const uint16_t* attn_norm;
  const uint16_t* ffn_norm;
} tasp_glayer;

/* The packed store (host array of n_layers layers; final BF16 gain and dense BF16 LM head
 * [vocab][d] on the device for vocab > 0). Plans keep pointers into it: it must outlive them. */
typedef struct {
  const tasp_glayer* layers;
  const uint16_t* final_norm;
  const uint16_t* lm_head;
} tasp_gstore;

/* Bytes of a shared-store plan (paper, appendix "Backing-store semantics": a plan over the one
 * store is block-selection and launch metadata). *plan_bytes: masks, index lists, the maps into
 * the store and the RoPE table, the same for every mask. *scratch_bytes: the decode (max_batch
 * sequences) and prefill (max_prefill tokens) scratch, which any number of shared plans of equal
 * scratch size may share (see tasp_compile_shared_plan). d_model, n_q_heads * head_dim and d_ffn
 * must be divisible by 128. */
tasp_status tasp_shared_plan_workspace_bytes(const tasp_model_desc* desc, size_t* plan_bytes,
                                             size_t* scratch_bytes);

/* Compile a plan over the shared store: closes the mask (as tasp_compile_plan), builds on the
 * device the maps from plan rows / column pieces to store rows / columns (QKV rows of the
 * retained heads and groups, W_o columns of the retained heads, gate / up rows and W_down column
 * blocks of the retained channels) and checks them on the host; copies no weights. The retained
 * channels of every layer must come in aligned blocks of 16 (else TASP_ERR_UNSUPPORTED; the
 * paper's channel groups are 1,024 wide). Such a plan serves every call a per-row plan serves
 * (decode at batch 1..max_batch, prefill, tasp_generate, tasp_serve_turn, the profiling calls),
 * reading the store in place: batch 1 with per-lane group scales, batches and prefill on the
 * matrix cores, a group's sum times its scale (batches where 128 retained columns are not one group:
 * each weight times its scale, split exactly into BF16 hi and lo parts);
 * only tasp_plan_panel returns TASP_ERR_UNSUPPORTED (there are no panels). Its signature differs
 * from a per-row plan of the same mask, so caches are not shared between the two formats.
 * `workspace` (256-byte aligned, plan_bytes) holds the plan's metadata. `scratch` (256-byte
 * aligned, scratch_bytes) is its scratch arena and may be passed to several shared plans: their
 * calls, and this compile (it clears the arena's counters), must then be ordered one after
 * another (one stream, or synchronised streams); overlapping calls race. With scratch NULL the
 * arena is the workspace's tail (workspace_bytes >= plan_bytes + scratch_bytes). Both buffers stay
 * owned by the caller and must outlive the plan. Synchronises `stream`. */
tasp_status tasp_compile_shared_plan(const tasp_model_desc* desc, const tasp_gstore* store,
                                     const tasp_mask* mask, void* workspace,
                                     size_t workspace_bytes, void* scratch, size_t scratch_bytes,
                                     void* stream, tasp_plan* out);

/* Retained counts of one layer after closure (paper, Eqs. flop-attn and flop-mlp: m^q, m^kv and
 * c of that layer): query heads, KV groups, SwiGLU channels, written to host int32s.
 * TASP_ERR_INVALID_ARG for a NULL pointer or a layer outside 0..n_layers-1. */
tasp_status tasp_plan_counts(tasp_plan plan, int32_t layer, int32_t* m_q, int32_t* m_kv,
                             int32_t* n_ffn);

/* Copy one ascending index list of a layer as computed on the device by the closure (paper,
 * Sec. "Dependency-Closed Masks and Cache-Consistent Routing": a KV group stays active while any
 * of its query heads is retained, heads keep their group, and a SwiGLU channel is kept or removed
 * in gate, up and down together) into host dst of cap entries: TASP_IDX_Q retained query heads,
 * TASP_IDX_KV retained KV groups, TASP_IDX_QKVSLOT the rank of each retained head's group among
 * the retained groups, TASP_IDX_FFN retained channels. *n (if not NULL) receives the list length; dst NULL
 * only queries it. TASP_ERR_INVALID_ARG if the length exceeds cap, or for a bad layer / `which`. */
tasp_status tasp_plan_indices(tasp_plan plan, int32_t layer, int32_t which, int32_t* dst,
                              int32_t cap, int32_t* n);

/* Where a panel of a layer lives (paper, appendix "Backing-store semantics": the contiguous
 * retained tensors a plan launches on): device int8 rows [rows][ld] (columns >= cols are zero)
 * and its float32 scales [rows], both inside the plan's workspace (not owned by the caller's
 * pointers; valid until tasp_plan_destroy). QKV rows: retained q heads, then K, then V rows of
 * retained groups. TASP_ERR_UNSUPPORTED for a shared-store plan (it has no panels). */
tasp_status tasp_plan_panel(tasp_plan plan, int32_t layer, int32_t which, const int8_t** w,
                            const float** scale, int64_t* rows, int64_t* cols, int64_t* ld);

/* Analytical active-FLOP ratio of the decoder projections (paper, Eqs. flop-attn and flop-mlp;
 * LM head excluded), retained INT8 weight bytes, float32 scale bytes, and the plan signature
 * (a hash of the model shape and the closed mask; equal masks give equal signatures). */
tasp_status tasp_plan_ledger(tasp_plan plan, double* active_flop_ratio, uint64_t* weight_bytes,
                             uint64_t* scale_bytes, uint64_t* signature);

/* Release a plan's host metadata (paper, appendix "Backing-store semantics": a mask owns plan
 * metadata only). The workspace given to the compile call stays the caller's to free once the
 * plan's queued work has completed. NULL is accepted. */
tasp_status tasp_plan_destroy(tasp_plan plan);

/* Adopt a cache whose rows 0..pos-1 were filled outside the library (already rotated keys) for
 * this plan (paper, Sec. "Dependency-Closed Masks and Cache-Consistent Routing": cache contents
 * belong to one mask and are not carried to an incompatible one): checks its shape against the
 * plan (TASP_ERR_SHAPE: batch outside 1..max_batch, max_seq above the plan's) and sets
 * cache->plan_sig (host struct; the device arrays are not touched). */
tasp_status tasp_kv_bind(tasp_plan plan, tasp_kv_cache* cache);

/* One decode step (paper, Sec. "Dependency-Closed Masks and Cache-Consistent Routing": the
 * plan chosen for a turn runs every decode step; Table "systems": the timed decode latency) for
 * cache->batch sequences that share `pos` (prior positions, 0 <= pos < cache->max_seq, else
 * TASP_ERR_POS_RANGE; a cache bound to another plan gives TASP_ERR_CACHE_PLAN_MISMATCH). x (device) float32 [batch][d_model]; out (device) float32 [batch][d_model], or
 * logits [batch][vocab] when the plan has an LM head. x and out may not overlap. Stream-ordered
 * and asynchronous; launches only the plan's kernels and allocates nothing, so it may be captured
 * into a HIP graph. Calls on one plan must be ordered (they share the plan's scratch). */
tasp_status tasp_decode_step(tasp_plan plan, const float* x, tasp_kv_cache* cache, int32_t pos,
                             float* out, void* stream);

/* Prefill of T tokens of one sequence (cache->batch must be 1) at positions pos0..pos0+T-1
 * (paper, Sec. "Dependency-Closed Masks and Cache-Consistent Routing": the plan fixed at the start
 * of a turn serves the prompt and every later decode step; Table "configuration": the timed
 * request begins with a prefill). 1 <= T <= max_prefill (TASP_ERR_UNSUPPORTED for a plan compiled with
 * max_prefill 0), pos0 + T <= cache->max_seq (else TASP_ERR_POS_RANGE). x (device) float32
 * [T][d_model]; out (device, not overlapping x) float32 [T][d_model], or logits [T][vocab] with
 * an LM head. Token t attends causally over rows 0..pos0+t; rows pos0..pos0+T-1 of every
 * retained group receive the BF16 k and v of the tokens. pos0 == 0 binds the cache to the plan;
 * pos0 > 0 requires it bound (else TASP_ERR_CACHE_PLAN_MISMATCH). Projections run
 * on the INT8 matrix cores over 24-bit fixed-point activations (one scale per token), those of a token
 * with outliers, where such digits would hold less than a hi/lo BF16 pair, on the BF16 ones; attention
 * on the BF16 ones with q and P split into hi/lo pairs. Stream-ordered, capturable;
 * calls on one plan must be ordered (they share the plan's scratch). */
tasp_status tasp_prefill(tasp_plan plan, const float* x, int32_t T, tasp_kv_cache* cache,
                         int32_t pos0, float* out, void* stream);

/* The same prefill returning only the last token's logits (paper, Sec. "Dependency-Closed Masks
 * and Cache-Consistent Routing" and Table "configuration": greedy decoding continues from the
 * prompt's last position, so no other position's logits are needed). Arguments and errors as
 * tasp_prefill, with out (device, not overlapping x) float32 [vocab]: the final RMSNorm and LM
 * head of token T - 1 only, by the decode LM head kernel (TASP_ERR_UNSUPPORTED without an LM
 * head). The cache rows and every other effect are those of tasp_prefill. tasp_generate and
 * tasp_serve_turn prefill this way. */
tasp_status tasp_prefill_last(tasp_plan plan, const float* x, int32_t T, tasp_kv_cache* cache,
                              int32_t pos0, float* out, void* stream);

/* One request under the plan (paper, Sec. "Dependency-Closed Masks and Cache-Consistent Routing":
 * the plan stays fixed through prefill and every decode step; Table "configuration": the timed
 * request is a prefill followed by greedy decoding). The prompt's ids (device int32 [T]) are
 * embedded from the dense INT8 table (device int8 [vocab][d_model] with float32 row scales
 * [vocab]), prefilled at positions 0..T-1 (binding the cache), and the greedy id of the last
 * position goes to out_ids[0]; then n_new decode steps feed out_ids[i] at position T + i and
 * write the greedy id of its logits to out_ids[i + 1]. Greedy = highest logit, lowest id on ties;
 * ids stay on the device, so nothing waits for the host between tokens.
 *   Requires an LM head (else TASP_ERR_UNSUPPORTED), cache batch 1, 1 <= T <= max_prefill and
 *   T + n_new <= cache->max_seq (else TASP_ERR_POS_RANGE).
 *   out_ids: device int32 [n_new + 1]; x_scratch: device float32 [T][d_model]; logits: device
 *   float32 [T][vocab] (holds the last step's logits afterwards). Stream-ordered. */
tasp_status tasp_generate(tasp_plan plan, const int8_t* embed, const float* embed_scale,
                          const int32_t* prompt, int32_t T, int32_t n_new, tasp_kv_cache* cache,
                          int32_t* out_ids, float* x_scratch, float* logits, void* stream);

/* Profiling variant of tasp_prefill (per-kernel split of the prefill time of Table "systems"):
 * an event pair around every kernel; kinds as for tasp_decode_step_timed, plus 7 for the RoPE /
 * cache-append kernel. kernel_ms, kinds: host arrays of cap entries; *n the kernels launched.
 * Synchronises `stream`. */
tasp_status tasp_prefill_timed(tasp_plan plan, const float* x, int32_t T, tasp_kv_cache* cache,
                               int32_t pos0, float* out, void* stream, float* kernel_ms,
                               int32_t* kinds, int32_t cap, int32_t* n);

/* Profiling variant of tasp_decode_step (per-kernel split of the decode latency of Table
 * "systems"): records a HIP event pair around every kernel it launches,
 * synchronises `stream`, and writes each kernel's duration in milliseconds to kernel_ms[i] and a
 * kernel-kind code to kinds[i] (0 QKV, 1 attention, 2 O, 3 gate/up, 4 down, 5 LM head, 6 batched
 * operand preparation) for up to
 * cap kernels; *n receives the number launched. Not capturable (it synchronises). */
tasp_status tasp_decode_step_timed(tasp_plan plan, const float* x, tasp_kv_cache* cache,
                                   int32_t pos, float* out, void* stream, float* kernel_ms,
                                   int32_t* kinds, int32_t cap, int32_t* n);

/* Profiling (the timing protocol of Sec. "Experimental Design": back-to-back runs between
 * events, here for one stage): average duration of one stage of layer `layer`, measured as n_plans * reps
 * back-to-back launches between two HIP events on `stream` (layer -1: every layer that has the stage,
 * in order, so that each launch of a stack reads another layer's panel). Stage `kind`: 1 attention at `pos`
 * (split-KV partials, merged by the last split of each group slot; rewrites cache row pos with
 * the same values, or for layer -1 every layer's row pos with the last decoded layer's k, v), 3 the gate/up projection (RMSNorm + SwiGLU), 4 the down projection (writes the plan's
 * scratch, not a caller buffer). Launch i uses plans[i % n_plans] with caches[i % n_plans] (bound
 * to that plan; its batch selects the batch-1 or the batched kernels), so distinct plan copies
 * keep every launch streaming from HBM rather than from cache. Each plan must have run a
 * tasp_decode_step with that cache at `pos` (its scratch holds the stage's input). Synchronises
 * `stream`; writes the mean milliseconds per launch. Not capturable. */
tasp_status tasp_profile_stage(const tasp_plan* plans, const tasp_kv_cache* caches,
                               int32_t n_plans, int32_t layer, int32_t kind, int32_t pos,
                               int32_t reps, void* stream, float* ms_per_launch);

/* Greedy dependency-closed mask construction (paper, Sec. "Dependency-Closed Masks and
 * Cache-Consistent Routing"; costs from Eqs. flop-attn and flop-mlp). Candidates are every query
 * head and every SwiGLU group of `granule` consecutive channels (gate row, up row and down column
 * jointly). They are ranked by score / active FLOPs in float64 (a head: 4 d d_h plus 1/r of its
 * KV group's 4 d d_h; a channel group: 6 d granule), equal keys by ascending candidate index
 * (layer-major, a layer's heads before its channel groups), and accepted in that order when the
 * marginal cost (a head whose KV group is not open yet also pays the group) fits the budget
 * floor(target x full-width decoder FLOPs); a candidate that does not fit is skipped. Outputs are
 * dependency-closed by construction.
 *   head_scores (device) float32 [n_layers][n_q_heads]; chan_scores (device) float32
 *   [n_layers][d_ffn / granule]; all finite (else TASP_ERR_INVALID_ARG).
 *   q_keep [L][Hq], kv_keep [L][Hkv], ffn_keep [L][d_ffn] (device, caller-owned) receive 0/1.
 *   granule must divide d_ffn (else TASP_ERR_SHAPE); 0 <= target <= 1.
 *   workspace: device, 256-byte aligned, at least tasp_mask_workspace_bytes.
 * Synchronises `stream` (it reads back the status and the FLOPs spent, *flops_spent if given). */
tasp_status tasp_mask_workspace_bytes(const tasp_model_desc* desc, int32_t granule, size_t* bytes);
tasp_status tasp_build_mask(const tasp_model_desc* desc, const float* head_scores,
                            const float* chan_scores, int32_t granule, double target,
                            void* workspace, size_t workspace_bytes, uint8_t* q_keep,
                            uint8_t* kv_keep, uint8_t* ffn_keep, uint64_t* flops_spent,
                            void* stream);

/* ---- routing (paper, Sec. "Dependency-Closed Masks and Cache-Consistent Routing": a three-layer
 * MLP router picks one task plan per user turn, or the dense plan when its temperature-scaled
 * confidence is below tau; appendix "Router feature specification": the feature vector).
 *
 * Feature vector of a prompt (float32, proj_dim + 11 entries, in this order):
 *   [0, proj_dim)  proj x tf, tf[bin] = (number of the prompt's byte trigrams, ASCII letters
 *                  case-folded, whose 32-bit FNV-1a hash is bin modulo n_bins) / max(1, bytes - 2);
 *   then ln(1 + bytes), the proxy-LM mean token log-probability (an input), ln(1 + count) of
 *   digits, of operators (+ - * / = < > % ^), of code punctuation ({ } [ ] ( ) ; _ # ` \ | &) and
 *   of question marks, and five 0/1 descriptors: numbered list (a line opening with 1-3 digits,
 *   '.' or ')', a space), code fence (three backticks), translate cue ("translat", case-folded),
 *   multiple-choice pattern (lines opening with option labels A and B, as "X.", "X)" or "(X)"
 *   then a space), retrieval cue (case-folded who / when / where / which at a word start and
 *   not followed by a letter).
 * MLP: h1 = ReLU(w1 f + b1), h2 = ReLU(w2 h1 + b2), z = w3 h2 + b3; p = softmax(z / temperature);
 * choice = the lowest task index of max p, or -1 (dense plan) when max p < tau. float32
 * arithmetic; the text scan is integer. */
#define TASP_ROUTER_SCALARS 11
#define TASP_ROUTER_MAX_TASKS 16
#define TASP_ROUTER_MAX_BINS 16384

typedef struct {
  int32_t n_bins;       /* hashed trigram bins (paper: 2,048), 1..16384 */
  int32_t proj_dim;     /* width of the frozen random projection (paper: 256), >= 1 */
  int32_t hidden1;      /* MLP hidden widths (paper: 512 and 256), >= 1 */
  int32_t hidden2;
  int32_t n_tasks;      /* task plans (paper: 5), 1..16 */
  float temperature;    /* > 0; divides the logits */
  float tau;            /* confidence threshold of the dense fallback (paper: 0.85) */
  const float* proj;    /* device float32 [proj_dim][n_bins] */
  const float* w1;      /* device float32 [hidden1][proj_dim + 11] */
  const float* b1;      /* [hidden1] */
  const float* w2;      /* [hidden2][hidden1] */
  const float* b2;      /* [hidden2] */
  const float* w3;      /* [n_tasks][hidden2] */
  const float* b3;      /* [n_tasks] */
} tasp_router;

/* Device workspace bytes for routing n_prompts prompts (also covers tasp_serve_turn with
 * n_prompts = 1). */
tasp_status tasp_router_workspace_bytes(const tasp_router* router, int32_t n_prompts,
                                        size_t* bytes);

/* Route n_prompts prompts. text (device bytes, n_text of them) holds the prompts back to back;
 * offsets (device int32 [n_prompts + 1]) bounds prompt i as [offsets[i], offsets[i + 1]), each
 * bound clamped to [0, n_text] on the device (a decreasing pair is an empty prompt); offsets NULL
 * means one prompt, the whole text (n_prompts must be 1). proxy_logprob: device float32
 * [n_prompts]. Outputs (device): features float32 [n_prompts][proj_dim + 11] (may be NULL),
 * probs float32 [n_prompts][n_tasks], choice int32 [n_prompts]. workspace: device, 256-byte
 * aligned, at least tasp_router_workspace_bytes. Stream-ordered and asynchronous (five kernels,
 * no allocation), so it may be captured into a HIP graph. Errors: TASP_ERR_INVALID_ARG for NULL
 * pointers, sizes out of range (n_prompts 1..65535, n_text >= 0) or a temperature <= 0;
 * TASP_ERR_WORKSPACE for a short workspace. */
tasp_status tasp_route(const tasp_router* router, const uint8_t* text, int32_t n_text,
                       const int32_t* offsets, int32_t n_prompts, const float* proxy_logprob,
                       void* workspace, size_t workspace_bytes, float* features, float* probs,
                       int32_t* choice, void* stream);

/* Routing for callers that cannot allocate (code under HIP graph capture, serving loops and
 * harnesses that forbid allocation): tasp_route without a workspace argument. Its scratch is a
 * fixed TASP_ROUTE_NOALLOC_SCRATCH_BYTES array that the library holds in each GPU's memory
 * until the process ends; the call allocates nothing. A call whose scratch need
 * (tasp_router_workspace_bytes for the same router and n_prompts) exceeds that size returns
 * TASP_ERR_WORKSPACE and enqueues nothing (about 12 KB per prompt at the paper's router shape,
 * so ~340 prompts per call). Every call on one GPU uses that GPU's one array: calls that overlap
 * on one GPU (concurrent streams, or host threads without ordering) race and must be serialised
 * by the caller; calls on one stream are ordered. The array's contents are left over from the
 * last call and need no clearing (every byte a call reads, that call writes first). The first
 * call on a device looks up the array's device address (not enqueued). Arguments, outputs and
 * errors otherwise as tasp_route; the results equal tasp_route's bit for bit. */
#define TASP_ROUTE_NOALLOC_SCRATCH_BYTES ((size_t)4 << 20)
tasp_status tasp_route_noalloc(const tasp_router* router, const uint8_t* text, int32_t n_text,
                               const int32_t* offsets, int32_t n_prompts,
                               const float* proxy_logprob, float* features, float* probs,
                               int32_t* choice, void* stream);

/* One user turn with routing and dispatch (paper, Sec. "Dependency-Closed Masks and
 * Cache-Consistent Routing"): one routing decision per turn; the plan it picks runs all of that
 * turn's prefill and decode work; cache rows written under one closed mask are kept only when the
 * same plan serves the next turn, and are otherwise discarded and rebuilt.
 *   1. routes the turn's text (device bytes [n_text], one prompt) with proxy_logprob (device
 *      float32 [1]) and waits for the decision (this synchronises `stream`);
 *   2. takes task_plans[choice], or dense_plan for choice -1 (all n_tasks + 1 plans must share
 *      one model shape with an LM head);
 *   3. if 0 < n_cached < T and the cache is bound to the chosen plan, its rows 0..n_cached-1 (the
 *      conversation so far, written under that plan) are kept and prompt ids n_cached..T-1 are
 *      prefilled at those positions (*reused = 1); otherwise the cache is invalidated: all T ids
 *      are prefilled from position 0 and the cache is bound to the chosen plan (*reused = 0);
 *   4. decodes greedily as tasp_generate: out_ids[0] from the last prompt position, then n_new
 *      steps. After the turn the cache holds T + n_new valid rows (the last id is not fed).
 *   prompt: device int32 [T] (the whole conversation's ids); x_scratch: device float32
 *   [T][d_model]; logits: device float32 [T][vocab]; out_ids: device int32 [n_new + 1];
 *   workspace: tasp_router_workspace_bytes(router, 1). *chosen receives the choice (-1 dense).
 *   Errors as tasp_route and tasp_generate; T - prefilled start must fit the plan's max_prefill. */
tasp_status tasp_serve_turn(const tasp_router* router, const tasp_plan* task_plans,
                            tasp_plan dense_plan, const uint8_t* text, int32_t n_text,
                            const float* proxy_logprob, const int8_t* embed,
                            const float* embed_scale, const int32_t* prompt, int32_t T,
                            int32_t n_cached, int32_t n_new, tasp_kv_cache* cache,
                            int32_t* out_ids, float* x_scratch, float* logits, void* workspace,
                            size_t workspace_bytes, int32_t* chosen, int32_t* reused,
                            void* stream);

/* ---- sequences of their own lengths and trees of drafted tokens (paper, Sec. "Dependency-Closed
 * Masks and Cache-Consistent Routing": the plan fixed for a turn runs every decode step; here several
 * drafted tokens of a sequence, for instance from a sparser plan, are run and verified in one step).
 *
 * A typed cache holds, per layer, sequence and KV head, max_seq rows of head_dim values in BF16 or in 8
 * bits (INT8 or E4M3) with one float32 scale per row: value = code * scale. len (device) is the
 * number of rows each sequence holds: no call needs it on the host. Lengths outside 0..max_seq are not an
 * error that a call can report: such a sequence is passed over (nothing written, zeros returned).
 *
 * The T nodes of a tree: parent (device int32 [batch][T]) is -1 for a root, an earlier node, or anything else
 * for an absent node (shorter trees of a batch; nodes below an absent one, and nodes whose row would not fit
 * max_seq, are absent too). NULL: a chain, parent[t] = t - 1. Node t of a sequence has cache row len + t
 * and position len + its depth. T <= TASP_TREE_MAX with a tree. */
#define TASP_TREE_MAX 64
#define TASP_SEQ_MAX_BATCH 256
enum { TASP_BF16 = 0, TASP_F32 = 1, TASP_INT8 = 2, TASP_E4M3 = 3 };

typedef struct {
  void* k;                /* (device) [n_layers][batch][n_kv_heads][max_seq][head_dim], 16-byte aligned */
  void* v;
  float* k_scale;         /* (device) [n_layers][batch][n_kv_heads][max_seq]; NULL for TASP_BF16 */
  float* v_scale;
  int32_t* len;           /* (device) [batch] */
  int32_t type;           /* TASP_BF16, TASP_INT8 or TASP_E4M3 */
  int32_t n_layers, batch, n_kv_heads, max_seq, head_dim;   /* batch 1..TASP_SEQ_MAX_BATCH, heads 1..64,
                             head_dim 64 or 128, max_seq * head_dim < 2^30 */
  uint64_t plan_sig;      /* the plan the rows belong to (tasp_tree_step), 0: none */
} tasp_seq_cache;

/* Rows of head vectors (device): element strides from one sequence, token and head to the next; the
 * values of a head are contiguous. Address and strides keep every row 16-byte aligned. */
typedef struct {
  void* p;
  int64_t seq, token, head;
} tasp_rows;

/* Rotary positions. layout: pairs (i, i + rot_dim / 2) or (2 i, 2 i + 1) of a head's first rot_dim values (a
 * multiple of 16, up to head_dim; the others pass unchanged), turned by pos * f_i, f_i = theta^(-2 i / rot_dim) (theta above 1),
 * and multiplied by mscale. For contexts beyond orig_len positions the frequencies are scaled:
 *   LINEAR      f / factor
 *   WAVELENGTH  by the turns n = orig_len f / 2 pi: f for n >= high, f / factor for n <= low, between them
 *               f (g + (1 - g) / factor), g = (n - low) / (high - low)
 *   INDEX       by the pair's index: f ((1 - g) + g / factor), g = clamp((i - a) / (b - a)), a and b the indices
 *               (rounded down and up, cut to 0..rot_dim - 1; b - a at least 0.001) of the pairs that make high
 *               and low turns over orig_len */
enum { TASP_ROPE_HALF = 0, TASP_ROPE_INTERLEAVED = 1 };
enum { TASP_ROPE_NONE = 0, TASP_ROPE_LINEAR = 1, TASP_ROPE_WAVELENGTH = 2, TASP_ROPE_INDEX = 3 };
typedef struct {
  int32_t layout, rot_dim, scaling, orig_len;
  double theta, factor, low, high, mscale;
} tasp_rope;

/* Write T tokens' k and v behind every sequence of layer `layer` (rows len..len + T - 1; len itself
 * stays) and rotate q: q and k are turned by the nodes' positions (rope NULL: not at all), v is taken as it
 * is, and rows of an 8-bit cache are quantised as they are written (scale = the row's largest magnitude
 * / 127 or 448, codes rounded to nearest even; a row that holds an infinity or a NaN reads back as NaN). k, v: rows of
 * n_kv_heads heads; q, q_out: n_q_heads (0: no queries, both NULL), neither q_out overlapping q, k or
 * v; all of act_type TASP_BF16 or TASP_F32. Rows of absent nodes are not written, their q_out are zeros. Only
 * k and v of a packed BF16 cache may be given this way too (rope NULL), to convert it. Arithmetic in float32, angles in
 * float64. Stream-ordered, asynchronous, capturable, no workspace. Errors: TASP_ERR_INVALID_ARG (NULL, types,
 * misaligned rows), TASP_ERR_SHAPE (cache fields, layer, T, head counts, rot_dim). */
tasp_status tasp_seq_append(const tasp_seq_cache* cache, int32_t layer, const tasp_rope* rope,
                            const int32_t* parent, int32_t T, int32_t act_type, const tasp_rows* q,
                            const tasp_rows* k, const tasp_rows* v, int32_t n_q_heads,
                            const tasp_rows* q_out, void* stream);

/* Read rows first[b]..first[b] + n - 1 (device int32 [batch]; NULL: 0) of layer `layer` back as out_type
 * TASP_BF16 or TASP_F32 values (token stride: from row to row); rows outside 0..max_seq - 1 read as zeros. n is at least
 * 1 and n * head_dim at most 2^35 - 2^11.
 * Stream-ordered, capturable. Errors as tasp_seq_append. */
tasp_status tasp_seq_read(const tasp_seq_cache* cache, int32_t layer, const int32_t* first,
                          int32_t n, int32_t out_type, const tasp_rows* k_out,
                          const tasp_rows* v_out, void* stream);

/* Attention of T nodes (1..TASP_TREE_MAX; their rows already appended) of every sequence: node t sees rows
 * 0..len - 1, its ancestors' rows and its own, with scores scale * q . k. q, out: n_q_heads heads (a multiple
 * of n_kv_heads, at most 8 per KV head; query head h reads KV head h / (n_q_heads / n_kv_heads)) of act_type;
 * out must not overlap q or the cache. Outputs of absent nodes are zeros, and what absent or unseen
 * rows hold (NaN, infinities) reaches no output (in a row that is seen they leave nothing finite in their dimension: an
 * infinite v of a node's row comes out as it is, of a cached row perhaps as NaN). TASP_BF16: q and V exact, probabilities in 16 bits, sums in float32;
 * TASP_F32: everything to 24 bits. The ends of float32: rows seen times the largest |v| stay below 2^120 (sums are divided
 * at the end, a row's share in them is up to 2^8), and of a probability times a row's scale what lies below 2^-126
 * may be lost. max_len: the largest length expected (0..max_seq): it sizes launches and
 * workspace; longer sequences are served too. workspace: device, 256-byte aligned, at least
 * tasp_tree_attention_workspace_bytes for the same cache shape, n_q_heads, T and max_len; its contents need
 * no clearing; calls that overlap need one each. Stream-ordered, capturable (one or two kernels). Errors as
 * tasp_seq_append, TASP_ERR_WORKSPACE. */
tasp_status tasp_tree_attention_workspace_bytes(const tasp_seq_cache* cache, int32_t n_q_heads,
                                                int32_t T, int32_t max_len, size_t* bytes);
tasp_status tasp_tree_attention(const tasp_seq_cache* cache, int32_t layer, const int32_t* parent,
                                int32_t T, int32_t act_type, const tasp_rows* q, int32_t n_q_heads,
                                double scale, int32_t max_len, const tasp_rows* out,
                                void* workspace, size_t workspace_bytes, void* stream);

/* Verify the drafted tokens of `batch` trees against the target's distributions and take one more token from
 * given random numbers. logits (device float32 [batch][T][vocab]) are the target's behind each node, p_v =
 * softmax(logits[v] / temperature); tokens (device int32 [batch][T]): node 0 is the last token of the text (a
 * root), nodes t >= 1 are drafted; u (device float32 [batch][T], in [0, 1); NULL with temperature 0). From node
 * 0 on, the current node v's children are tried in node order:
 *   without draft_logits, child c is accepted when u[c] (1 - the share of the earlier children's distinct tokens
 *   in p_v) < p_v(tokens[c]), a token tried before having no share;
 *   with draft_logits (device float32 [batch][T - 1][vocab], behind nodes 0..T - 2; parent must be NULL) when
 *   u[c] q_v(tokens[c]) < p_v(tokens[c]), q_v = softmax(draft_logits[v] / temperature).
 * An accepted child becomes the current node. Where none is, the last token is the lowest one whose
 * cumulative weight exceeds u[0] times the total, the weights being p_v without the children's tokens, or
 * max(p_v - q_v, 0) at a refused child with draft_logits (p_v, should rounding leave no weight). Either way the emitted
 * tokens are distributed as the target's own samples. temperature 0: p_v is the lowest index of the
 * largest logit, draft_logits are not read. T = 1 samples one token from logits. NaN logits count as -inf;
 * a row without a finite or +inf logit yields token -1; drafted tokens outside the vocabulary are never accepted.
 * It knows no cache: nodes whose rows did not fit one have to be absent in `parent` (tasp_tree_step sees to that itself).
 *   n (device int32 [batch]): tokens emitted, the accepted ones and one more; ids (device int32 [batch][T]): those
 *   tokens, then -1; path (device int32 [batch][T]): the nodes 0, ... of the accepted path (n entries), then -1.
 * All sums in float64. workspace: device, 256-byte aligned, at least tasp_verify_workspace_bytes, needs no clearing;
 * calls that overlap need one each. Stream-ordered, capturable. Errors: TASP_ERR_INVALID_ARG (NULL, a temperature
 * neither 0 nor in 1e-30..1e30, draft_logits with a tree), TASP_ERR_SHAPE (batch, T, vocab), TASP_ERR_WORKSPACE. */
tasp_status tasp_verify_workspace_bytes(int32_t batch, int32_t T, int32_t vocab, size_t* bytes);
tasp_status tasp_verify(const float* logits, const int32_t* tokens, const float* u,
                        const int32_t* parent, const float* draft_logits, int32_t batch, int32_t T,
                        int32_t vocab, double temperature, int32_t* ids, int32_t* path, int32_t* n,
                        void* workspace, size_t workspace_bytes, void* stream);

/* Keep an accepted path: in every layer, sequence and KV head, row len + path[b][i] moves to row len + i for
 * i < n[b] (entries of path outside 0..T - 1 and rows past max_seq stay where they are), and len_out[b] = len[b] + n[b],
 * cut to max_seq (device int32 [batch]; it may lie over cache->len, n or path). path [batch][T] and n as tasp_verify
 * returns them, T <= TASP_TREE_MAX. Stream-ordered, capturable. Errors as tasp_seq_append. */
tasp_status tasp_seq_commit(const tasp_seq_cache* cache, const int32_t* path, const int32_t* n,
                            int32_t T, int32_t* len_out, void* stream);

/* Adopt a typed cache's rows for a plan (as tasp_kv_bind does for a tasp_kv_cache): checks that it has the plan's
 * layers, KV heads and head_dim (TASP_ERR_SHAPE) and sets cache->plan_sig. Rows may come from tasp_seq_append of
 * a prefilled tasp_kv_cache of the same plan (rope NULL: its keys are rotated already). */
tasp_status tasp_seq_bind(tasp_plan plan, tasp_seq_cache* cache);

/* Workspace bytes of a plan's step over trees of T nodes: tasp_tree_step's, enough for tasp_tree_forward. The step
 * runs in the plan's prefill scratch, so cache->batch * T <= max_prefill (TASP_ERR_SHAPE; TASP_ERR_UNSUPPORTED for
 * max_prefill 0). max_len as for tasp_tree_attention. */
tasp_status tasp_tree_step_workspace_bytes(tasp_plan plan, const tasp_seq_cache* cache, int32_t T,
                                           int32_t max_len, size_t* bytes);

/* The plan's layers over trees of T nodes of every sequence (any plan format; projections as tasp_prefill, attention
 * as tasp_tree_attention with TASP_F32 over the retained groups): x (device) float32 [batch][T][d_model], out (device, not overlapping
 * x; both 16-byte aligned) float32 [batch][T][vocab], or [batch][T][d_model] without an LM head. Appends the nodes' k and v to every
 * layer (positions len + depth, rotate-half RoPE with the plan's base; only retained groups' rows are written);
 * the lengths stay. Rows of out of absent nodes hold values of no meaning. The cache must be bound to the plan
 * (else TASP_ERR_CACHE_PLAN_MISMATCH). Stream-ordered, capturable; calls on one plan must be ordered. */
tasp_status tasp_tree_forward(tasp_plan plan, const float* x, const int32_t* parent, int32_t T,
                              const tasp_seq_cache* cache, int32_t max_len, float* out,
                              void* workspace, size_t workspace_bytes, void* stream);

/* One step of decoding with drafted tokens: embeds tokens (device int32 [batch][T]; node 0 the last token of the
 * text, whose row is not in the cache yet), runs tasp_tree_forward, verifies the drafts (tasp_verify; arguments as
 * there) and keeps the accepted path (tasp_seq_commit, cache->len grows by n). The next step's node 0 is
 * ids[b][n[b] - 1]. Nodes whose rows do not fit max_seq are absent for the verification too: they are never accepted, and a
 * sequence whose node 0 is absent (no row left, a length outside 0..max_seq, or parent[b][0] other than -1) emits nothing:
 * n[b] = 0, ids and path -1, its length and rows as they were. Nothing waits for the host: lengths, tokens and acceptance stay on the device, and a step can be
 * captured into a HIP graph and replayed with new tokens in the same arrays (max_len then is an upper bound for the
 * replays). embed, embed_scale as tasp_generate; x_scratch float32 [batch][T][d_model]; logits float32
 * [batch][T][vocab] receive the target's logits (both 16-byte aligned). A drafted token outside the vocabulary is not
 * accepted, and reaches its descendants alone. T = 1 decodes one token of every sequence by sampling or
 * greedily. Requires an LM head (else TASP_ERR_UNSUPPORTED). */
tasp_status tasp_tree_step(tasp_plan plan, const int8_t* embed, const float* embed_scale,
                           const int32_t* tokens, const int32_t* parent, const float* u,
                           const float* draft_logits, double temperature, int32_t T, int32_t max_len,
                           const tasp_seq_cache* cache, int32_t* ids, int32_t* path, int32_t* n,
                           float* x_scratch, float* logits, void* workspace, size_t workspace_bytes,
                           void* stream);

/* ---- caches in pages: many conversations of one pool (paper, Sec. "Dependency-Closed Masks and Cache-Consistent
 * Routing": a plan's prefill and decode over its own cache rows; here for any mixture of prompts, chunks of
 * prompts and single tokens of several sequences in one call).
 *
 * A pool holds, per layer, n_pages pages of page_rows rows of every KV head, in BF16 or in 8 bits (INT8 or E4M3: value =
 * code * scale, one float32 scale per page and head). Row r of sequence b lies in page table[b][r / page_rows] at r % page_rows.
 * A table entry outside 0..n_pages - 1 is no page: its rows are not written, not seen and read as zeros. len (device) is
 * the number of rows each sequence holds; as for a tasp_seq_cache no call needs it on the host, and a sequence with a length
 * outside 0..max_pages * page_rows is passed over. Sequences may share pages that are read (a common prefix); a page
 * that a call writes rows of must be one sequence's only, and in its table once (else its contents are undefined).
 *
 * Scales: a page and head's scale is the largest magnitude / 127 or 448 of what was written into it since its row 0 was
 * (rows given up by a smaller len still count). A call whose rows raise it rounds the page's older codes again, code' = round(code *
 * old / new); new rows are round(x / scale), ties to even. A page and head that was given an infinity or a NaN has
 * the scale NaN: all of it reads as NaN until its row 0 is written again.
 *
 * Packed tokens: a call's n_tokens new tokens (1..TASP_PAGE_MAX_TOKENS) lie one after the other, those of sequence b at
 * start[b]..start[b + 1] - 1 (device int32 [batch + 1]; a pair that falls or leaves 0..n_tokens: no tokens; ranges must not
 * overlap). start NULL: one token for every sequence (n_tokens = batch). The i-th token of a sequence is cache row and
 * position len + i; one beyond the table's pages is absent. Rows of tokens that are no sequence's (in front of start[0], behind
 * start[batch]) are not written, and what they hold reaches nothing. */
#define TASP_PAGE_MAX_TOKENS 262143
typedef struct {
  void* k;                /* (device) [n_layers][n_pages][n_kv_heads][page_rows][head_dim], 16-byte aligned */
  void* v;
  float* k_scale;         /* (device) [n_layers][n_pages][n_kv_heads]; NULL for TASP_BF16 */
  float* v_scale;
  const int32_t* table;   /* (device) [batch][max_pages] */
  int32_t* len;           /* (device) [batch] */
  int32_t type;           /* TASP_BF16, TASP_INT8 or TASP_E4M3 */
  int32_t n_layers, n_pages, n_kv_heads, page_rows, head_dim, batch, max_pages;   /* heads 1..64 of 64 or 128,
                             page_rows 16, 32, 64 or 128, batch 1..TASP_SEQ_MAX_BATCH, max_pages * page_rows at most 2^23 */
  uint64_t plan_sig;      /* the plan the rows belong to (tasp_page_forward), 0: none */
} tasp_page_cache;

/* Write the tokens' k and v into their sequences' pages of layer `layer` (len itself stays) and rotate q: q and k are
 * turned by the tokens' positions (rope NULL: not at all), v is taken as it is. k, v: rows of n_kv_heads heads; q, q_out:
 * n_q_heads (0: no queries, both NULL); all of act_type TASP_BF16 or TASP_F32 (seq strides are not used). Rows of q_out must not
 * overlap those of q, k or v. q_out of absent tokens are zeros. Arithmetic in float32, angles in float64.
 * Stream-ordered, asynchronous, capturable, no workspace. Errors: TASP_ERR_INVALID_ARG (NULL, types, misaligned rows),
 * TASP_ERR_SHAPE (cache fields, layer, n_tokens, head counts, rot_dim). */
tasp_status tasp_page_append(const tasp_page_cache* cache, int32_t layer, const tasp_rope* rope,
                             const int32_t* start, int32_t n_tokens, int32_t act_type, const tasp_rows* q,
                             const tasp_rows* k, const tasp_rows* v, int32_t n_q_heads,
                             const tasp_rows* q_out, void* stream);

/* Read rows first[b]..first[b] + n - 1 (device int32 [batch]; NULL: 0) of layer `layer` back as out_type
 * TASP_BF16 or TASP_F32 values, [batch][n_kv_heads][n] by the strides (token stride: from row to row); rows outside the table
 * read as zeros. n as for tasp_seq_read. Stream-ordered, capturable. Errors as tasp_page_append. */
tasp_status tasp_page_read(const tasp_page_cache* cache, int32_t layer, const int32_t* first,
                           int32_t n, int32_t out_type, const tasp_rows* k_out,
                           const tasp_rows* v_out, void* stream);

/* Causal attention of packed tokens (their rows already appended): token i of a sequence sees its rows 0..len + i that have
 * pages, with scores scale * q . k. q, out: rows of n_q_heads heads (a multiple of n_kv_heads, at most 8 per KV head; query head
 * h reads KV head h / (n_q_heads / n_kv_heads)) of act_type; out must not overlap q or the cache. Outputs of absent tokens and of
 * tokens that see no row are zeros, and what unseen rows hold (NaN, infinities, values of any size) reaches no output (a page's scale
 * belongs to all of its rows). TASP_BF16: q exact, sums in float32, probabilities in 16 bits, or, with more than 32 query rows of a
 * sequence and cache head (batch 1: of n_tokens tokens), in 11 to 16 bits, and lost per row up to 2^-34 of the largest |v|
 * seen (8-bit pages: 2^-30 of the row's own); TASP_F32: everything to 24 bits. The ends of float32 as for tasp_tree_attention.
 * max_len, max_new: the largest length and the largest number of new tokens of a sequence that are expected (max_len
 * 0..max_pages * page_rows, max_new at least 1): they size launches and workspace; more is served too.
 * workspace: device, 256-byte aligned, at least tasp_page_attention_workspace_bytes for the same cache shape, n_q_heads,
 * n_tokens, max_len and max_new; its contents need no clearing; calls that overlap need one each. Stream-ordered,
 * capturable. Errors as tasp_page_append, TASP_ERR_WORKSPACE. */
tasp_status tasp_page_attention_workspace_bytes(const tasp_page_cache* cache, int32_t n_q_heads,
                                                int32_t n_tokens, int32_t max_len, int32_t max_new,
                                                size_t* bytes);
tasp_status tasp_page_attention(const tasp_page_cache* cache, int32_t layer, const int32_t* start,
                                int32_t n_tokens, int32_t act_type, const tasp_rows* q,
                                int32_t n_q_heads, double scale, int32_t max_len, int32_t max_new,
                                const tasp_rows* out, void* workspace, size_t workspace_bytes,
                                void* stream);

/* Lengths grow by the call's tokens, cut to the table's pages: len[b] += start[b + 1] - start[b] (a sequence that is passed
 * over keeps its length). Behind the last layer of a step. Stream-ordered, capturable. Errors as tasp_page_append. */
tasp_status tasp_page_advance(const tasp_page_cache* cache, const int32_t* start, int32_t n_tokens, void* stream);

/* A plan over packed tokens of many sequences: prompts, chunks of prompts and single tokens in one call. tasp_page_bind
 * adopts a pool for a plan as tasp_seq_bind does. tasp_page_forward runs the plan's layers (any plan format; projections as
 * tasp_prefill, attention as tasp_page_attention with TASP_F32 over the retained groups): x (device) float32
 * [n_tokens][d_model], out (device, not overlapping x; both 16-byte aligned) float32 [n_tokens][vocab], or
 * [n_tokens][d_model] without an LM head. It appends the tokens' k and v to every layer (rotate-half RoPE with the plan's base; only
 * retained groups' rows are written); the lengths stay (tasp_page_advance). Rows of out of absent tokens and of tokens
 * that are no sequence's hold values of no meaning. n_tokens <= max_prefill (TASP_ERR_SHAPE; TASP_ERR_UNSUPPORTED for max_prefill 0):
 * the step runs in the plan's prefill scratch. The cache must be bound to the plan (else TASP_ERR_CACHE_PLAN_MISMATCH).
 * max_len, max_new, workspace: as for tasp_page_attention. Stream-ordered, capturable; calls on one plan must be ordered. */
tasp_status tasp_page_bind(tasp_plan plan, tasp_page_cache* cache);
tasp_status tasp_page_forward_workspace_bytes(tasp_plan plan, const tasp_page_cache* cache,
                                              int32_t n_tokens, int32_t max_len, int32_t max_new,
                                              size_t* bytes);
tasp_status tasp_page_forward(tasp_plan plan, const float* x, const int32_t* start, int32_t n_tokens,
                              const tasp_page_cache* cache, int32_t max_len, int32_t max_new,
                              float* out, void* workspace, size_t workspace_bytes, void* stream);

/* Scores of given tokens. logits (device): `rows` rows of vocab values, TASP_F32 or TASP_BF16, row_stride elements (vocab at
 * least) from one to the next; tokens (device int32 [rows]); p = softmax(row / temperature). Per row:
 *   logprob (float32 [rows])   log p(token); 0 for a token outside the vocabulary (padding)
 *   entropy (float32 [rows])   of p in nats; may be NULL
 *   rank (int32 [rows])        tokens before this one in the order of logits, equal ones by id (0: the most likely); -1 for
 *                              padding; may be NULL
 *   top_ids, top_logprobs      ([rows][n_top], n_top 0..TASP_TOP_MAX) the n_top first tokens in that order with their log
 *                              probabilities; -1 and -inf behind the last token above -inf
 * mean (float32 [n_seqs], with start device int32 [n_seqs + 1]; both may be NULL): the mean logprob of rows start[i]..start[i + 1] - 1
 * whose tokens lie in the vocabulary (0 where there are none; bounds are cut to 0..rows): what tasp_route takes as
 * proxy_logprob, over a prompt's rows of logits and next tokens.
 * NaN logits count as -inf, magnitudes of 2^126 / max(1, log2(e) / temperature) and more as infinite; infinite logits share the
 * whole probability evenly. A row without a logit above -inf has logprob -inf and entropy 0. Terms in float32, sums joined in
 * float64 behind every 512 terms of a thread.
 * workspace: device, 256-byte aligned, at least tasp_token_logprobs_workspace_bytes, needs no clearing; calls that overlap need
 * one each. Stream-ordered, capturable. Errors: TASP_ERR_INVALID_ARG (NULL, types, a temperature outside 1e-30..1e30),
 * TASP_ERR_SHAPE (rows, vocab 1..2^24, row_stride, n_top, n_seqs), TASP_ERR_WORKSPACE. */
#define TASP_TOP_MAX 32
tasp_status tasp_token_logprobs_workspace_bytes(int32_t rows, int32_t vocab, int32_t n_top, size_t* bytes);
tasp_status tasp_token_logprobs(const void* logits, int32_t logits_type, int64_t row_stride,
                                const int32_t* tokens, int32_t rows, int32_t vocab, double temperature,
                                int32_t n_top, float* logprob, float* entropy, int32_t* rank,
                                int32_t* top_ids, float* top_logprobs, const int32_t* start,
                                int32_t n_seqs, float* mean, void* workspace, size_t workspace_bytes,
                                void* stream);

/* Plain streaming copy of `bytes` (multiple of 16) from src to dst (device, not overlapping):
 * the reference kernel whose counter readings calibrate memory-traffic measurements (the byte
 * ledger of appendix "FLOP and storage validation" checked against hardware counters).
 * TASP_ERR_INVALID_ARG for NULL pointers or a size not a multiple of 16. */
tasp_status tasp_copy_probe(void* dst, const void* src, size_t bytes, void* stream);

/* Text of a status code, and the thread-local detail of the last failing call on this thread
 * (static / thread-owned strings; the caller does not free them). They report the host-side
 * validation that precedes every enqueue (all entry points above). */
const char* tasp_status_string(tasp_status s);
const char* tasp_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* TASP_H */
