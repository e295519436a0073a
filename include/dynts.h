/*
 * dynts.h -- C ABI of the MI355X (gfx950) DynTS decode hot path.
 *
 * DynTS (Dynamic Thinking-Token Selection) decodes over a budget-bounded KV cache: per
 * layer the cache of a sequence is the question window (M prompt slots, never evicted),
 * the selection window and the local window (Sec. 4.2).  Every decode step attends over
 * the retained slots (Eq. attn-score, Eq. attn-o), every cached thinking token carries an
 * importance score (Eq. importance-score, kept here in running form per layer and KV
 * head), and on a trigger the top-k thinking tokens of the selection window are kept and
 * the rest evicted.
 *
 * Conventions
 *  - All array arguments are DEVICE pointers unless a comment says "host".  The caller
 *    owns every buffer; the context owns host metadata only and never allocates device
 *    memory.  bf16 arrays are passed as uint16_t (raw bits).
 *  - Every call enqueues its kernels on the caller's stream (a hipStream_t passed as
 *    void*, NULL = the null stream) and returns without synchronising the host.  Calls on
 *    one context must be stream-ordered with respect to each other.
 *  - Return value: DYNTS_OK or a negative error.  Argument errors are found on the host
 *    before anything is launched.  Conditions only the device can see (a sequence that
 *    would overflow `capacity`) are latched into the bound `status` word: bit 0 = an
 *    append was dropped because the cache was full; bit 1 (value 2) = keep_idx too short for a sequence
 *    (dynts_select_evict left it alone); bit 2 (value 4) = the page pool of the paged layout ran dry; bit 3
 *    (value 8) = a chunk of question tokens behind thinking tokens (dynts_chunk_append); bit 4 (value 16) = a leaf that is
 *    none of its sequence's drafted tokens (dynts_tree_keep).
 *  - Layout (C order, L = n_layers, Nb = batch, Hkv = n_kv_heads, cap = capacity, d = head_dim):
 *      K, V      bf16  [L][Nb][Hkv][cap][d]   rows in position order
 *      S         fp32  [L][Nb][Hkv][cap]      importance score; +inf on question slots
 *      pos       int32 [L][Nb][Hkv][cap]      original token position of each slot
 *      seq_len   int32 [L][Nb]                slots in use (equal for all KV heads)
 *      next_pos  int32 [L][Nb]                position the next appended token receives
 *      n_prompt  int32 [Nb]                   M of each sequence
 *  - Query head hq reads KV head hq / G, G = n_q_heads / n_kv_heads (grouped-query
 *    attention, Sec. 2 "Attention Mechanism").  Supported: head_dim 64 or 128, G <= 16.
 *  - `active` (uint8 [Nb], may be NULL = all active) masks finished sequences of a ragged
 *    batch: nothing is appended, attended or written for them.
 */
#ifndef DYNTS_H
#define DYNTS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DYNTS_OK 0
#define DYNTS_EINVAL (-1)     /* a value outside its documented range */
#define DYNTS_ENULL (-2)      /* a required pointer is NULL */
#define DYNTS_ESHAPE (-3)     /* unsupported shape: head_dim, group size, divisibility */
#define DYNTS_ECAPACITY (-4)  /* capacity < budget + window + evict_every, or an index stride too small */
#define DYNTS_ENOTBOUND (-5)  /* dynts_bind has not been called */
#define DYNTS_EWORKSPACE (-6) /* workspace smaller than dynts_workspace_bytes, or misaligned */
#define DYNTS_EHIP (-7)       /* the HIP runtime refused a launch */
#define DYNTS_EPENDING (-8)   /* rows would move while a score update is still deferred */
#define DYNTS_ECODES (-9)     /* the context's cache holds codes (dynts_bind_codes), the call takes bf16 caches */

#define DYNTS_SCORE_ACCUMULATE 0 /* score = attention received so far (Eq. importance-score) */
#define DYNTS_SCORE_EXTERNAL 1   /* score supplied at append (the predictor's output, Sec. 4.1) */

typedef struct dynts_config {
  int32_t n_layers;
  int32_t batch;
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t capacity;     /* cap: slots per (sequence, KV head); >= prompt + budget + window + evict_every, <= 2^22 */
  int32_t budget;       /* selection-window slots kept by a trigger (the k of top-k, default k_keep) */
  int32_t window;       /* local-window slots, always kept */
  int32_t evict_every;  /* trigger period in steps = eviction volume K of Sec. 5 */
  float softmax_scale;  /* 0 => 1/sqrt(head_dim) (Eq. attn-score) */
  int32_t score_mode;   /* DYNTS_SCORE_* */
} dynts_config;

typedef struct dynts_ctx dynts_ctx;

/* Library version, major*10000 + minor*100 + patch. */
int dynts_version(void);
/* Static text for an error code. */
const char *dynts_strerror(int code);

/* Validate `cfg` and make a host-side context.  No device work, no HIP call. */
int dynts_create(const dynts_config *cfg, dynts_ctx **out);
int dynts_destroy(dynts_ctx *ctx);

/* Bytes of device scratch the kernels need for `cfg` (split partials, the saved query and softmax statistics of the
 * deferred score update, the kept logits of one layer).  0 if cfg is invalid. */
size_t dynts_workspace_bytes(const dynts_config *cfg);

/* Launch shape of the attention kernel, for tuning and for tests that must reach a particular shape at a
 * small size: the cache of a (sequence, KV head) is split over about target_workgroups / (batch * n_kv_heads)
 * workgroups (at least one; 0 = the default, one workgroup per compute unit) of waves_per_workgroup waves
 * (4 or 8; 0 = the default, 8).  Results do not depend on the shape beyond rounding order.  Changes the
 * workspace layout: call it before dynts_bind (it unbinds), and size the workspace with
 * dynts_ctx_workspace_bytes. */
int dynts_set_launch_shape(dynts_ctx *ctx, int32_t target_workgroups, int32_t waves_per_workgroup);
/* Bytes of workspace with which this context has all its forms: what it needs (dynts_workspace_bytes(cfg), another size if the launch
 * shape was changed) and behind it, on caches whose steps dynts_decode_loop can make in runs and that are split over several workgroups,
 * room for the partials of 16 to 64 steps, 4 * (head_dim + 2) bytes a step, workgroup and query head of its group, 64 MB at most.  A workspace
 * without that room is accepted: the loop then makes every step a launch of its own.  Paged contexts never use it. */
size_t dynts_ctx_workspace_bytes(const dynts_ctx *ctx);

/* Attach the caller's device buffers (layout above).  `workspace` must be 256-byte aligned
 * and zero-filled once by the caller before first use; `status` is one int32, zeroed by
 * the caller.  Binding resets the context's deferred-update bookkeeping. */
int dynts_bind(dynts_ctx *ctx, uint16_t *K, uint16_t *V, float *S, int32_t *pos,
               int32_t *seq_len, int32_t *next_pos, int32_t *n_prompt, void *workspace,
               size_t workspace_bytes, int32_t *status);

/* Paged (block-table) layout instead of one dense [cap][d] array per unit: K_pool, V_pool bf16
 * [n_pages][64][d] hold the rows of ALL layers, sequences and KV heads; slot j of a unit is row j % 64 of page
 * block_table[layer][b][h][j / 64] (int32 [L][Nb][Hkv][max_pages], max_pages * 64 >= capacity).  Pages are taken
 * from and returned to a device-side free stack: free_stack int32 [n_pages] lists page ids, *free_top (device
 * int32) is the number of free ones (entries [0, *free_top) are free).  The caller initialises the stack (all
 * pages free: free_stack[i] = i, *free_top = n_pages) and leaves the block table alone; appends and
 * dynts_prefill pop, dynts_compact gives the pages past the new length back, so evicted memory can be taken by
 * any other sequence.  dynts_prefill expects the layer's units to hold no pages.  When the stack runs dry the
 * row is dropped and bit 2 (value 4) of the status word is latched; results are undefined from then on.
 * The pools must hold finite values before first use (zero-filled, say): rows beyond a sequence's length may be
 * read, with zero weight.  S, pos and the per-sequence arrays keep the dense layout.  Everything else behaves as after dynts_bind.
 * The ORDER of the ids in the initial stack is the caller's choice and decides where a unit's pages lie.  With ids in
 * order, sequences that append in step get neighbouring pages round after round, so a unit's pages lie a fixed
 * power-of-two stride apart: good for caches streamed from HBM, but a cache small enough to stay in the 256 MB
 * memory-side cache then runs up to 25 % slower than with a shuffled stack (measured, 159 MB of K/V: 35 - 40 us per
 * attend launch in order, 31.5 us shuffled, 30 us dense); beyond that size a shuffled stack costs 3 - 5 %. */
int dynts_bind_paged(dynts_ctx *ctx, uint16_t *K_pool, uint16_t *V_pool, int32_t n_pages, int32_t *block_table,
                     int32_t max_pages, int32_t *free_stack, int32_t *free_top, float *S, int32_t *pos,
                     int32_t *seq_len, int32_t *next_pos, int32_t *n_prompt, void *workspace,
                     size_t workspace_bytes, int32_t *status);

/* Question window (Sec. 4.2, first paragraph): copy the prompt rows of one layer,
 * K0, V0 bf16 [Nb][Hkv][m_max][d], m int32 [Nb] with m[b] <= m_max, into slots [0, m[b]);
 * scores +inf, pos = slot, seq_len = next_pos = n_prompt = m. */
int dynts_prefill(dynts_ctx *ctx, int32_t layer, const uint16_t *K0, const uint16_t *V0,
                  int32_t m_max, const int32_t *m, void *stream);

/* Append the current token (Sec. 4.2, second paragraph): k_new, v_new bf16 [Nb][Hkv][d] go
 * to slot seq_len[b] of every KV head; score 0, or s_new fp32 [Nb][Hkv] when score_mode is
 * DYNTS_SCORE_EXTERNAL (then s_new is required); pos = next_pos++; seq_len++. */
int dynts_append(dynts_ctx *ctx, int32_t layer, const uint16_t *k_new, const uint16_t *v_new,
                 const float *s_new, const uint8_t *active, void *stream);

/* Decode attention (Eq. attn-score, Eq. attn-o): for each active sequence and query head,
 * out[b][hq][:] = sum_j softmax_j(q.k_j * scale) v_j over slots [0, seq_len[b]).
 * q bf16 [Nb][Hq][d]; out fp32 [Nb][Hq][d]; lse fp32 [Nb][Hq] (may be NULL) receives
 * log sum_j exp(logit_j).  Leaves what dynts_update_scores needs in the workspace.
 * Where the last two such calls of the layer were each followed by its dynts_update_scores, before another attention that
 * keeps its logits or a fused step of the layer (the first call of a context counts as such), and the group is small enough
 * for it to pay, the call also leaves its logits there, 4 bytes per slot and query head: it takes up to a fifth longer, and
 * the update adds them up instead of reading K again.  There is room for one layer's logits; under stream capture none are
 * left. */
int dynts_decode_attend(dynts_ctx *ctx, int32_t layer, const uint16_t *q, const uint8_t *active,
                        float *out, float *lse, void *stream);

/* Score accumulation (Eq. importance-score in running form; App. B.1 sums over heads):
 * S[b][h][j] += sum over the G heads of the group of alpha[g][j], for every thinking slot
 * j >= n_prompt[b] the last attend call of this layer saw.  A no-op when nothing is
 * outstanding or score_mode is external. */
int dynts_update_scores(dynts_ctx *ctx, int32_t layer, void *stream);

/* dynts_decode_attend with the score accumulation fused into the same pass over K: the
 * accumulation owed by the PREVIOUS attend call of this layer is applied while this call
 * streams the cache, and this call's own accumulation becomes the outstanding one.  S
 * therefore lags by one step until dynts_update_scores (or dynts_select_evict, which
 * applies it first) is called. */
int dynts_decode_attend_update(dynts_ctx *ctx, int32_t layer, const uint16_t *q,
                               const uint8_t *active, float *out, float *lse, void *stream);

/* One whole decode step of a layer in one pass: dynts_append + dynts_decode_attend_update.  A sequence whose
 * cache is already full is left alone in this step (nothing appended, attended or scored; status bit 0). */
int dynts_decode_step(dynts_ctx *ctx, int32_t layer, const uint16_t *q, const uint16_t *k_new,
                      const uint16_t *v_new, const float *s_new, const uint8_t *active,
                      float *out, float *lse, void *stream);

/* dynts_decode_step for callers that cannot allocate device memory and want to hand over as little as possible
 * (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): the same step, but
 * the launch's scratch -- the split partials and the ticket counters, i.e. everything in the workspace that
 * does not have to survive the call -- lives in an array that is part of the library's code object on each
 * GPU (DYNTS_STATIC_SCRATCH_BYTES = 8 MiB, held until the process ends) instead of the head of the
 * bound workspace.  The call allocates nothing and frees nothing, on the host side of HIP or the device side.
 * The state that carries over between steps (saved queries and softmax statistics of the deferred score
 * update) stays in the bound workspace, so this call and dynts_decode_step may be mixed freely on a context.
 *  - DYNTS_EWORKSPACE if the context's shape needs more scratch than the array holds: the partials take
 *    batch * n_kv_heads * chunks * group * (head_dim + 2) * 8 bytes of its upper 7 MiB (chunks being what
 *    dynts_set_launch_shape describes; with the default shape 2 MiB on the 32-sequence Qwen-shaped workload,
 *    nothing once there are as many (sequence, KV head) units as compute units), the counters 4 bytes per
 *    unit and per sequence of 512 KiB each.  Nothing is launched then.
 *  - All calls on one GPU share that GPU's array, from every context and stream: calls that may overlap in
 *    time on one GPU race with each other -- keep them on one stream or order them with events.  (Calls that
 *    are stream-ordered leave the array as the next one needs it, whatever its shape: counters live in a part
 *    of the array that holds nothing else and are back at zero when a launch ends, partials are tagged with
 *    a serial number that no other launch of the process uses.)
 *  - The first call on a GPU looks the array up and clears it with a small kernel on the caller's stream. */
#define DYNTS_STATIC_SCRATCH_BYTES (8u << 20)
int dynts_decode_step_static(dynts_ctx *ctx, int32_t layer, const uint16_t *q, const uint16_t *k_new,
                             const uint16_t *v_new, const float *s_new, const uint8_t *active,
                             float *out, float *lse, void *stream);

/* Optional announcement: the next fused step of this layer (dynts_decode_step, dynts_decode_step_static or
 * dynts_decode_attend_update) will be followed by a trigger (dynts_select_evict).  That step then keeps its
 * logits (4 bytes per slot and query head of the group, in the workspace), and the score accumulation it owes
 * is applied from them when dynts_select_evict / dynts_update_scores asks for it, instead of by a second pass
 * over K.  Results are the same up to fp32 rounding order; without the announcement everything works as before.
 * dynts_decode_loop makes it itself on the steps flagged in evict_steps.  No effect with external scores. */
int dynts_hint_trigger(dynts_ctx *ctx, int32_t layer);

/* KV-cache selection (Sec. 4.2, third paragraph): for every sequence with trigger[b] != 0
 * (uint8 [Nb], NULL = all) and every KV head keep all question slots, the last `window`
 * slots, and of the slots between them the k_keep with the highest score (ties: lower
 * position first -- decided by SLOT order: the kernel never reads `pos`, it relies on the
 * invariant that slots are in position order, which appends and the stable compaction keep).  keep_idx int32 [Nb][Hkv][keep_stride] receives the retained slots in
 * ascending order, new_len int32 [Nb] their count (seq_len[b] where not triggered or when
 * the selection window holds <= k_keep slots).  k_keep < 0 means cfg.budget.  Applies an
 * outstanding score accumulation first.  NaN scores give an unspecified (in-bounds) choice. */
int dynts_select_evict(dynts_ctx *ctx, int32_t layer, const uint8_t *trigger, int32_t k_keep,
                       int32_t *keep_idx, int32_t keep_stride, int32_t *new_len, void *stream);

/* Eviction (Sec. 4.2): stable in-place gather of the K, V, S and pos rows listed in
 * keep_idx to slots [0, new_len[b]) and seq_len[b] = new_len[b], for triggered sequences.
 * keep_idx rows must be strictly ascending and < seq_len[b] (indices are clamped into the
 * cache, never followed out of bounds).  DYNTS_EPENDING if a score accumulation is
 * outstanding for this layer. */
int dynts_compact(dynts_ctx *ctx, int32_t layer, const uint8_t *trigger, const int32_t *keep_idx,
                  int32_t keep_stride, const int32_t *new_len, void *stream);

/* Native decode loop: enqueue n_steps whole steps of every layer without returning to the
 * caller -- per step and layer dynts_decode_step, and on steps with evict_steps[i] != 0
 * (host uint8 [n_steps]) dynts_select_evict(k_keep = budget) + dynts_compact for the
 * sequences flagged in trigger (device uint8 [n_steps][Nb], NULL = all).
 *   q      bf16 [n_steps][L][Nb][Hq][d]      k_new, v_new bf16 [n_steps][L][Nb][Hkv][d]
 *   s_new  fp32 [n_steps][Nb][Hkv] (external mode, same score for every layer) or NULL
 *   active uint8 [n_steps][Nb] or NULL
 *   out    fp32 [L][Nb][Hq][d], overwritten every step (out_step_stride = 0) or one slab
 *          per step (out_step_stride = L*Nb*Hq*d elements)
 *   keep_idx int32 [Nb][Hkv][cap], new_len int32 [Nb]: scratch for the triggers.
 * On dense caches that the chip's registers hold, runs of three or more steps between two triggers are made a layer at a time, by one to three
 * launches, with the results of a launch per step, and the cache is read once a run.  That serves callers who have the inputs of several steps in
 * hand: replay of a known text, teacher forcing, scoring.  A model that forms step t + 1's query from step t's output calls with n_steps = 1, and
 * pays a launch a step.  Launches whose kernel events are asked for (below), recorded ones, and those on a workspace without the
 * room that dynts_ctx_workspace_bytes counts, stay one per step. */
int dynts_decode_loop(dynts_ctx *ctx, int32_t n_steps, const uint16_t *q, const uint16_t *k_new,
                      const uint16_t *v_new, const float *s_new, const uint8_t *active,
                      const uint8_t *evict_steps, const uint8_t *trigger, float *out,
                      size_t out_step_stride, int32_t *keep_idx, int32_t *new_len, void *stream);

/* Measurement hook: when both are non-NULL hipEvent_t handles (created by the caller with
 * timing enabled), every later attend launch of this context attaches them to the dispatch
 * of its streaming kernel (attention + deferred score update, the kernel that moves the K/V
 * bytes; behind an unfused attention also its score update, from K or from kept logits): `start` is
 * stamped when that kernel begins, `stop` when it ends, so hipEventElapsedTime(start, stop) is the kernel's own duration.  Pass NULLs to switch it off. */
int dynts_set_kernel_events(dynts_ctx *ctx, void *start, void *stop);

/* The same for a run of launches: `starts` and `stops` are host arrays of n hipEvent_t handles; the
 * next n attend launches of this context (in call order, e.g. inside dynts_decode_loop) take one pair
 * each, after which the hook is off again.  n = 0 clears the list. */
int dynts_set_kernel_event_list(dynts_ctx *ctx, void *const *starts, void *const *stops, int32_t n);

/* Importance score from a block of queries at once (Eq. importance-score with its sum over the K
 * answer tokens; App. B.1: the answer-by-thinking sub-matrix of the attention weights summed over
 * heads and over the answer dimension):
 *   dst[b][h][j] (+)= sum over the n_queries block queries i and the G heads g of the group of
 *                    alpha_{(i,g), j},   for the cached slots j < seq_len[b],
 * where query i's softmax (Eq. attn-score) runs over the cached slots and, when k_blk is given, over
 * block keys 0..i (causal, as in one forward pass over the block; block tokens receive no score).
 *   q_blk bf16 [Nb][n_queries][Hq][d]     k_blk bf16 [Nb][n_queries][Hkv][d] or NULL
 *   dst fp32 [Nb][Hkv][cap]: every slot j < seq_len[b] is written (question slots too).  dst = NULL
 *     means the layer's score array S; then slots below n_prompt[b] keep their +inf.
 *   accumulate != 0 adds to dst, 0 overwrites it.
 *   scratch: >= dynts_score_block_scratch_bytes(cfg, n_queries) bytes of device memory, 4-byte
 *     aligned, contents irrelevant before and after.  (The first pass may cut the keys into up to four ranges with
 *     denominators of their own; with less, down to the room of one range, there are fewer ranges.)
 * Independent of the deferred accumulation of the fused decode calls (sums commute).  The cache is
 * only read. */
size_t dynts_score_block_scratch_bytes(const dynts_config *cfg, int32_t n_queries);
int dynts_score_block(dynts_ctx *ctx, int32_t layer, const uint16_t *q_blk, const uint16_t *k_blk,
                      int32_t n_queries, const uint8_t *active, float *dst, int32_t accumulate,
                      void *scratch, size_t scratch_bytes, void *stream);

/* Importance Predictor (Sec. 4.1; App. A "Predictor Overhead", App. C for the sizes): the three-layer
 * MLP d -> m1 -> m2 -> 1 on the final hidden state of the current token,
 *   s[b] = w3 . act(W2 act(W1 h[b] + b1) + b2) + b3,
 * whose output is the score the paper's inference mode appends with the token (dynts_append / dynts_decode_step
 * with score_mode DYNTS_SCORE_EXTERNAL take it as s_new).  Weights are device pointers, bf16 row-major
 * [out][in]; biases fp32 or NULL.  The paper calls the MLP "linear" and names no activation: it is a
 * parameter.  Products are accumulated in fp32 and nothing is rounded to bf16 between the layers.
 *   h bf16 [batch][d], batch <= 128;  d and m1 multiples of 32, m2 a multiple of 16.
 *   s_out fp32 [batch][n_rep]: the score of sequence b written n_rep times (n_rep = n_kv_heads gives the
 *     [Nb][Hkv] layout of s_new: one score per token for every head, as in the paper).
 *   scratch: >= dynts_predict_scratch_bytes bytes, 256-byte aligned, contents irrelevant before and after (it may be shared by calls
 *     that are stream-ordered with respect to each other).  What serves a batch serves every smaller one.
 *   start/stop: optional hipEvent_t handles attached to the first and the last kernel of the call. */
#define DYNTS_ACT_NONE 0
#define DYNTS_ACT_RELU 1
#define DYNTS_ACT_SILU 2
typedef struct dynts_predictor {
  int32_t d, m1, m2;
  int32_t activation; /* DYNTS_ACT_* */
  int32_t packed;     /* 0: W1, W2 row-major [out][in]; 1: both in the tiled layout of dynts_predictor_pack */
  const uint16_t *W1; /* [m1][d] */
  const float *b1;    /* [m1] or NULL */
  const uint16_t *W2; /* [m2][m1] */
  const float *b2;    /* [m2] or NULL */
  const uint16_t *w3; /* [m2] */
  const float *b3;    /* [1] or NULL */
} dynts_predictor;
/* One-off repacking of a row-major bf16 weight matrix W [m][K] (m a multiple of 16, K of 32) into tiles of
 * 16 rows x 32 columns stored contiguously, W_packed [m/16][K/32][16][32] (same size, must not alias W).
 * With packed weights every load instruction of the GEMM reads one contiguous kilobyte instead of 16 pieces a
 * whole weight row apart, which is what lets the weight stream run at memory speed. */
int dynts_predictor_pack(const uint16_t *W, int32_t m, int32_t K, uint16_t *W_packed, void *stream);
size_t dynts_predict_scratch_bytes(const dynts_predictor *w, int32_t batch);
int dynts_predict_scores(const dynts_predictor *w, const uint16_t *h, int32_t batch, float *s_out,
                         int32_t n_rep, void *scratch, size_t scratch_bytes, void *start, void *stop,
                         void *stream);

/* ---- chunks of new tokens ----------------------------------------------------------------------------------------
 * Several new tokens of every sequence at once: a prompt, the next question, a tool's answer, drafted tokens to be
 * checked, a known answer that is scored.  A chunk of m tokens is what m single steps are (Eq. attn-score, Eq. attn-o,
 * Eq. importance-score), up to the roundings below: every token enters the cache, attends to what is there and to itself, and its
 * attention weights are added to the scores of the thinking slots; but K and V are read once a chunk.  Dense and paged layouts.
 *   n_tokens: tokens of the longest chunk, the row count of the arrays, 1 <= n_tokens <= 2^20.
 *   n_new int32 [Nb] or NULL (= n_tokens each): tokens of each sequence (clamped to [0, n_tokens]); the rows behind
 *     them are padding, not read as keys or written as outputs.  A sequence with none is left alone: no output of any of these
 *     calls is written for it, the dst of dynts_chunk_scores neither, whatever `accumulate` says.
 *   scratch: >= dynts_chunk_scratch_bytes(cfg, n_tokens) bytes of device memory, 256-byte aligned, contents irrelevant
 *     before and after (what serves a chunk serves every smaller one; it may be shared by calls that are
 *     stream-ordered with respect to each other).
 * Arrays that are written overlap no other argument.  Outputs are bf16, as what a projection reads next, and the weights are rounded to bf16 for their
 * product with V, half a step of 2^-8 each (a single step keeps 16 bits of a weight and returns fp32); sums, products, statistics and the weights that
 * slots receive are fp32.
 * A token's weights of rows that it does not see are 0, and 0 times a NaN or an infinity is NaN: rows of V that are hidden from a token, those of the chunk's
 * later tokens among them, have to be finite, or elements of its output are NaN where theirs are not.  (On codes one element of 2^126 and more makes 32 such.)
 * Rows of K need not: hidden logits are -inf whatever they were. */

/* What is done to the logits of a chunk, in this order (s the scaled product of a query at position p and a key at
 * position j; positions are those of the `pos` array, not slots: evictions leave gaps in them):
 *   softcap > 0      s = softcap * tanh(s / softcap), off by 6 * 2^-24 of softcap at most up to a softcap of 128, above by 24 * 2^-24 of s
 *                    (and slower on long chunks; a softcap so small that 3 * scale / softcap overflows is refused)
 *   slope            s = s - slope[hq] * |p - j|
 *   hidden keys      s = -inf unless max(first[b][i], p - window + 1) <= j <= last[b][i]
 * first, last: positions token i of the chunk sees from and up to (`last` may lie behind the token's own position: a
 * prefix whose tokens see each other; `first` at the start of a document keeps documents apart).  Positions are taken to
 * be 0 or more and below 2^31 - 1.  A token that sees nothing gets zeros and lse = -inf.
 * n_tokens = 1 is the form for single tokens, and the only one: dynts_decode_step, dynts_decode_loop and dynts_score_block know no shaping.  A model that
 * has one pays a score launch a token, and has no runs of steps and no logits kept for a trigger. */
typedef struct dynts_shaping {
  float softcap;        /* 0: none */
  int32_t window;       /* positions a token sees, its own the last of them; 0: all */
  const float *slope;   /* fp32 [Hq] or NULL */
  const int32_t *first; /* int32 [Nb][n_tokens] or NULL: 0 */
  const int32_t *last;  /* int32 [Nb][n_tokens] or NULL: the token's own position */
} dynts_shaping;

/* Bytes of scratch for chunks of up to n_tokens tokens; 0 if cfg or n_tokens is invalid. */
size_t dynts_chunk_scratch_bytes(const dynts_config *cfg, int32_t n_tokens);

/* dynts_append for a chunk: k_new, v_new bf16 [Nb][n_tokens][Hkv][d] go to slots seq_len[b] and on; score 0, or s_new fp32
 * [Nb][n_tokens][Hkv] when score_mode is DYNTS_SCORE_EXTERNAL (then required); pos = next_pos and on; both lengths advance.
 * question != 0: the tokens are question slots (score +inf, never evicted; s_new is not read) and n_prompt[b] becomes the new length,
 * so a sequence may get its question in several chunks, or another one before its first thinking token.
 * A chunk that does not fit leaves its whole sequence alone, and latches in the status word: bit 0 = more than `capacity` slots, bit 2
 * (value 4) = more pages than the pool has (the sequence keeps what it had, unlike after a dry dynts_append),
 * bit 3 (value 8) = a question behind thinking tokens (seq_len[b] > n_prompt[b]). */
int dynts_chunk_append(dynts_ctx *ctx, int32_t layer, const uint16_t *k_new, const uint16_t *v_new, const float *s_new,
                       int32_t n_tokens, const int32_t *n_new, int32_t question, void *scratch, size_t scratch_bytes,
                       void *stream);

/* Attention of the LAST n_new[b] tokens in the cache (at most seq_len[b]): token i of them sees the slots up to its own, or what
 * `shaping` (host struct of device pointers, or NULL) says.  q bf16 [Nb][n_tokens][Hq][d]; out bf16 [Nb][n_tokens][Hq][d];
 * lse fp32 [Nb][n_tokens][Hq] or NULL: log of the softmax denominators.  Reads the cache only; what dynts_update_scores owes is
 * not touched.  A NaN in a row of K makes out and lse of the tokens and heads that see the row NaN, and so what the slots that they see receive
 * (dynts_chunk_scores). */
int dynts_chunk_attend(dynts_ctx *ctx, int32_t layer, const uint16_t *q, int32_t n_tokens, const int32_t *n_new,
                       const dynts_shaping *shaping, uint16_t *out, float *lse, void *scratch, size_t scratch_bytes,
                       void *stream);

/* The attention weight that every cached slot receives from those tokens, summed over them and over the heads of its group:
 *   dst[b][h][j] (+)= sum over tokens i and heads g of exp(logit - lse[b][i][hq]),  j < seq_len[b],
 * with the lse of dynts_chunk_attend for the same arguments.  dst fp32 [Nb][Hkv][cap], or NULL: the layer's scores S, then slots
 * below n_prompt[b] keep their +inf.  accumulate != 0 adds to dst, 0 overwrites it.  Commutes with what
 * dynts_update_scores owes. */
int dynts_chunk_scores(dynts_ctx *ctx, int32_t layer, const uint16_t *q, int32_t n_tokens, const int32_t *n_new,
                       const dynts_shaping *shaping, const float *lse, float *dst, int32_t accumulate, void *stream);

/* A chunk's whole step: dynts_chunk_append, dynts_chunk_attend and, unless the tokens are question slots or scores come from outside,
 * dynts_chunk_scores into S.  A sequence whose chunk does not fit is left alone in all of them.
 * The weights of all its tokens are in S then, and stay there.  Drafted tokens that may be dropped again take the parts instead: dynts_chunk_append and
 * dynts_chunk_attend; then dynts_compact with the slots that stay (it gives a paged sequence's pages back, which a smaller seq_len alone would lose; a
 * score update owed by a single step has to be applied before), next_pos[b] reduced by the number dropped; then dynts_chunk_scores with the same q and
 * lse and n_new = the number that stays. */
int dynts_chunk_step(dynts_ctx *ctx, int32_t layer, const uint16_t *q, const uint16_t *k_new, const uint16_t *v_new,
                     const float *s_new, int32_t n_tokens, const int32_t *n_new, int32_t question,
                     const dynts_shaping *shaping, uint16_t *out, float *lse, void *scratch, size_t scratch_bytes,
                     void *stream);

/* ---- caches of 8-bit codes ----------------------------------------------------------------------------------------
 * Rows are quantised as they are written: a block of 32 neighbouring elements of a row shares a scale byte s, and
 *   value = code * 2^(s - 127),   s the least, 27 at least, with  max |x| <= top * 2^(s - 127)  over the block,
 * codes rounded to nearest, ties to even.  33 bytes in place of 64 a block; every value is exact in bf16.
 *   DYNTS_CODE_E4M3  a float of 4 bits of exponent, 3 of mantissa, top 448: off by 2^-4 of the value at most, or by 2^-10 of 2^(s - 127)
 *   DYNTS_CODE_INT8  a whole number, two's complement, top 127: off by half of 2^(s - 127) at most
 * A block with an infinity, a NaN or a magnitude of 2^126 and more has s = 255 and reads as NaN.
 *
 * dynts_bind_codes takes such a cache in place of dynts_bind's or (block_table not NULL) dynts_bind_paged's: K, V uint8 [L][Nb][Hkv][cap][d] with scales
 * [L][Nb][Hkv][cap][d / 32], or pools [n_pages][64][d] with scales [n_pages][64][d / 32]; everything else as there.
 * 16-byte aligned; pools zero-filled before first use.  Chunks (dynts_chunk_append, _attend, _scores, _step; n_tokens = 1 is the form for single tokens, question = 1 fills a prompt), drafts
 * (dynts_tree_*), dynts_read_rows, dynts_select_evict, dynts_compact and dynts_update_scores (which has nothing to do) serve it; the new tokens of a
 * chunk see each other's rows as the cache holds them.  Roundings are those of chunks, one token or many: outputs in bf16 and weights rounded to bf16, where
 * dynts_decode_step on a bf16 cache has fp32 and 16 bits.  The other calls on rows return DYNTS_ECODES: dynts_prefill, dynts_append, dynts_decode_attend,
 * dynts_decode_attend_update, dynts_decode_step, dynts_decode_step_static, dynts_hint_trigger, dynts_score_block, dynts_decode_loop. */
#define DYNTS_CODE_E4M3 1
#define DYNTS_CODE_INT8 2
typedef struct dynts_codes {
  int32_t code; /* DYNTS_CODE_* */
  uint8_t *K, *V;
  uint8_t *K_scale, *V_scale;
  /* pages, as in dynts_bind_paged; block_table NULL: the dense layout */
  int32_t n_pages, max_pages;
  int32_t *block_table, *free_stack, *free_top;
} dynts_codes;
int dynts_bind_codes(dynts_ctx *ctx, const dynts_codes *codes, float *S, int32_t *pos, int32_t *seq_len, int32_t *next_pos,
                     int32_t *n_prompt, void *workspace, size_t workspace_bytes, int32_t *status);

/* dynts_chunk_scratch_bytes for a cache of codes, and for drafts on one.  Where a chunk has many rows there is room in it for one layer's rows as bf16. */
size_t dynts_codes_scratch_bytes(const dynts_config *cfg, int32_t n_tokens);

/* Rows of a layer as bf16, of any cache: slot first[b] + i (first int32 [Nb], NULL: 0) of every KV head goes to row i of K_out, V_out bf16
 * [Nb][Hkv][n_rows][d], n_rows <= capacity.  Rows of slots that the sequence does not have are left as they were. */
int dynts_read_rows(dynts_ctx *ctx, int32_t layer, const int32_t *first, int32_t n_rows, uint16_t *K_out, uint16_t *V_out,
                    void *stream);

/* ---- drafts that branch -----------------------------------------------------------------------------------------------
 * Drafted tokens that form trees over the cache: a token sees the whole cache, its ancestors and itself.  A step of a model that drafts:
 *   dynts_tree_build once, then in every layer dynts_tree_step; when the model has chosen, in every layer dynts_tree_keep with the last token that is
 *   accepted, and dynts_chunk_scores with the q and lse that it has gathered.
 * Rotary positions are the caller's: a token of depth t lies t behind the first of the draft.  Dense and paged caches, bf16 or codes.
 *   n_tokens: tokens of the largest draft, 1 <= n_tokens <= 4096; n_new int32 [Nb] or NULL as for chunks, the rest of the arrays is padding.
 *   seen uint32 [Nb][n_tokens][ceil(n_tokens / 32)]: bit j % 32 of word j / 32 of token i says that it sees token j of the draft.  What
 *     dynts_tree_build writes, or any other pattern; bits of tokens behind the sequence's last count as 0.
 * Arrays that are written overlap no other argument.  Rows of V that a token of the draft does not see have to be finite, rows of K need not. */

/* seen, and depth int32 [Nb][n_tokens] (0 for a token whose parent is the cache; may be NULL), from parents int32 [Nb][n_tokens]: the draft's
 * token before it that a token follows, or -1, the cache (as does any number that is not of a token before it).  Padding gets zeros. */
int dynts_tree_build(const int32_t *parents, const int32_t *n_new, int32_t batch, int32_t n_tokens, uint32_t *seen,
                     int32_t *depth, void *stream);

/* dynts_chunk_attend for a draft: the LAST n_new[b] tokens in the cache see what lies before them, and of each other what `seen` says.  A token
 * that sees nothing gets zeros and lse = -inf.  scratch as dynts_chunk_scratch_bytes (or dynts_codes_scratch_bytes) says. */
int dynts_tree_attend(dynts_ctx *ctx, int32_t layer, const uint16_t *q, int32_t n_tokens, const int32_t *n_new,
                      const uint32_t *seen, uint16_t *out, float *lse, void *scratch, size_t scratch_bytes, void *stream);

/* dynts_chunk_append of the draft (as thinking tokens, in their order) and dynts_tree_attend.  n_taken int32 [Nb] receives the tokens of each sequence that
 * the cache took, n_new[b] or 0 (see dynts_chunk_append): dynts_tree_keep wants it. */
int dynts_tree_step(dynts_ctx *ctx, int32_t layer, const uint16_t *q, const uint16_t *k_new, const uint16_t *v_new,
                    const float *s_new, int32_t n_tokens, const int32_t *n_new, const uint32_t *seen, int32_t *n_taken,
                    uint16_t *out, float *lse, void *scratch, size_t scratch_bytes, void *stream);

/* Of the last n_taken[b] (NULL: n_tokens; no more than the sequence has) tokens in the cache those stay that token leaf[b] sees, in order, right
 * behind what lay before the draft; leaf[b] = -1: none.  Applies an outstanding score accumulation first.  Scores move with the rows, positions are those of a
 * chunk, both lengths and the pages follow; rows behind the new length keep what they held.  n_kept int32 [Nb] receives the number that stays.  q_kept and lse_kept (NULL, or of the shapes of q and
 * lse, those of dynts_tree_step) receive the rows of q and lse of the tokens that stay, one after the other; rows behind them are left
 * alone: dynts_chunk_scores takes them with n_new = n_kept.  A leaf that is not one of the n_taken[b] tokens keeps none and latches bit 4
 * (value 16) in the status word. */
int dynts_tree_keep(dynts_ctx *ctx, int32_t layer, int32_t n_tokens, const int32_t *n_taken, const uint32_t *seen,
                    const int32_t *leaf, const uint16_t *q, const float *lse, uint16_t *q_kept, float *lse_kept,
                    int32_t *n_kept, void *stream);

/* Rotary positions with several axes (time, height and width of an image's patches, say): pair p of every head, elements (a, b), is
 * turned by theta = positions[axis[p]][t] * freq[p],
 *   a' = a cos theta - b sin theta,  b' = b cos theta + a sin theta,
 * elements behind the pairs are copied.  inverse != 0 turns by -theta: the gradient with respect to the input.  Whole turns are
 * taken off in 64 bits, one rounding to bf16 at the end.
 *   q bf16 [n_tokens][q_heads][head_dim], k bf16 [n_tokens][k_heads][head_dim] or NULL; q_out, k_out of the same shapes, the same
 *   arrays or others (that do not overlap).  positions int32 [n_axes][n_tokens].
 * n_tokens below 2^24, head_dim a multiple of 8, n_pairs a multiple of 8, at most 128 and head_dim / 2.  An axis[p] past the last one counts as that one. */
#define DYNTS_PAIR_HALVES 0   /* pair p: elements p and n_pairs + p */
#define DYNTS_PAIR_ADJACENT 1 /* pair p: elements 2 p and 2 p + 1 */
typedef struct dynts_rotary {
  int32_t head_dim, n_pairs;
  int32_t pairing; /* DYNTS_PAIR_* */
  int32_t n_axes;
  const float *freq;   /* device fp32 [n_pairs], radians a position */
  const uint8_t *axis; /* device [n_pairs] or NULL: all of axis 0 */
} dynts_rotary;
int dynts_rotate(const dynts_rotary *r, const uint16_t *q, int32_t q_heads, const uint16_t *k, int32_t k_heads,
                 const int32_t *positions, int32_t n_tokens, int32_t inverse, uint16_t *q_out, uint16_t *k_out,
                 void *stream);

/* Measurement aid, not part of the method: one launch of a plain read stream over `bytes` (a multiple
 * of 16, buf 16-byte aligned) of device memory, 16 bytes per lane per load, n_workgroups x 256 lanes,
 * grid-stride.  Nothing is written unless the XOR of all words equals `magic` (then sink[0], one
 * device uint32, receives it).  start/stop: hipEvent_t handles attached to the dispatch as in
 * dynts_set_kernel_events, or both NULL.  Its rate on a buffer of the cache's size is the bandwidth
 * the simplest kernel reaches, to set beside the published peak. */
int dynts_probe_read_stream(const void *buf, size_t bytes, int32_t n_workgroups, uint32_t magic,
                            uint32_t *sink, void *start, void *stop, void *stream);

/* Measurement aid, not part of the method: one launch in which every lane of n_workgroups x 256 lanes performs
 * iters x 8 exponentials 2^x followed by a subtraction (the loop holds nothing else), 16 * iters instructions per
 * wave.  The exponentials delivered per second are the second roofline of dynts_score_block, which needs one
 * per (query row, slot) and pass (Eq. attn-score's softmax).  sink: one device float, written only on a value
 * that cannot occur.  start/stop: hipEvent_t handles attached to the dispatch, or both NULL. */
int dynts_probe_exp_rate(int32_t n_workgroups, int32_t iters, float *sink, void *start, void *stop, void *stream);

/* Measurement aid, not part of the method: the instruction mix of dynts_score_block's kernels (head_dim 128) with
 * no memory access.  Every wave of n_workgroups x 256 lanes runs iters rounds of what one chunk of 32 streamed
 * rows costs it there: what & 1: 16 bf16 MFMAs (32x32x16) on two independent accumulators; what & 2: 32 x
 * (multiply-add, 2^x, add) on independent registers; what = 3: both, interleaved by the compiler.  The time per
 * round and SIMD is the floor of a chunk (32 rows x 64 columns) that instruction issue and the two pipes set (Eq.
 * attn-score's softmax needs the three vector instructions per logit).  sink, start/stop as for
 * dynts_probe_exp_rate. */
int dynts_probe_issue_mix(int32_t n_workgroups, int32_t iters, int32_t what, float *sink, void *start, void *stop,
                          void *stream);

#ifdef __cplusplus
}
#endif
#endif /* DYNTS_H */
