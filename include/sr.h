/*
 * sr.h -- C boundary of the selective-rollout decode library for AMD MI355X (gfx950).
 *
 * The library runs the group-batched multi-turn rollout of one GRPO step and the
 * Selective-Rollout gate that retires converged groups mid-batch:
 *
 *   - G samples per prompt ("group") advance one environment step ("turn") at a time;
 *     each turn an observation chunk is appended to every live sequence and an action
 *     is decoded token by token (paper Section 2.2 and Appendix C.1/C.2: token layout
 *     [prompt, o_1, a_1, o_2, a_2, ...], one model call per step per trajectory);
 *   - after turn K the mean pairwise prefix edit distance d_K of each group's action
 *     sequences (Section 3.2) is compared with the threshold d_L and a group is cut iff
 *     d_K < d_L (Eq. 2); a cut group stops generating and leaves the batch (Section 3.2,
 *     paragraph "The gate"; Appendix C.1).
 *
 * Behind the rollout it has the losses over the kept trajectories' logits with their gradients, the
 * clipping of a list of gradients (sr_policy_loss, sr_preference_loss, sr_clip_grad_norm), and what surrounds
 * the matrix products of the decoder being trained: embedding, residual + norm and dropout with their gradients.
 *
 * Conventions
 *   - Every function returns SR_OK (0) or a negative sr_status; nothing throws or exits.
 *   - "device" pointers are HIP device memory of the current device; "host" pointers are
 *     ordinary host memory.  The caller owns every buffer it passes in.  The library owns
 *     its packed weight copy, the KV page pool, page tables, the action table and all
 *     scratch; they are released by sr_destroy.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  Calls are
 *     asynchronous on that stream unless stated otherwise.  One context must be driven
 *     from one stream at a time.  Page tables and row maps reach the device through pinned
 *     staging slots guarded by events, so sr_prefill_chunk, sr_decode_step, sr_gate and
 *     sr_finish_sequences do not wait for the stream; sr_retire_and_compact waits once, for
 *     the retire mask (the page allocator lives on the host).
 *   - Batch rows are ordered group-major: while no sequence has finished early, live row r
 *     belongs to live group r / G, member r % G.  Retirement removes whole groups,
 *     sr_finish_sequences single members; both keep the order of the survivors
 *     (sr_get_live_map names the original sequence of every row).
 *   - All live sequences have the same length at all times (lock-step turns).
 *   - bf16 tensors are raw 16-bit patterns; matrices are row-major [out_features][in_features].
 */
#ifndef SR_H
#define SR_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    SR_OK = 0,
    SR_E_ARG = -1,    /* null pointer, bad shape, turn out of range, chunk_len <= 0, G < 2, ... */
    SR_E_NOMEM = -2,  /* KV page pool exhausted (checked on the host before any launch) or allocation failed */
    SR_E_STATE = -3,  /* call out of order: decode before prefill, gate with too few recorded actions, ... */
    SR_E_HIP = -4,    /* a HIP runtime call failed; sr_strerror gives the text */
    SR_E_LIMIT = -5   /* a size beyond the fixed capacity of an entry point that allocates nothing */
} sr_status;

typedef struct sr_ctx sr_ctx;

/* Decoder shape: pre-norm blocks, RMSNorm, rotate-half RoPE, grouped-query attention,
 * SwiGLU FFN.  head_dim must be 64 or 128; n_q_heads % n_kv_heads == 0.  (The paper names the
 * model family only -- Section 3.1; these fields describe any decoder of that family.) */
typedef struct {
    int32_t n_layers, hidden, n_q_heads, n_kv_heads, head_dim, ffn, vocab;
    float rms_eps, rope_theta;
    int32_t qkv_bias;     /* 1: q/k/v projections add a bias vector */
    int32_t tied_lm_head; /* 1: the LM head is the embedding matrix (sr_weights.lm_head is ignored and may be
                             NULL); 0: a separate [vocab][hidden] matrix */
} sr_model_shape;

typedef struct {
    int32_t page_tokens;     /* tokens per KV page: 32, 64 or 128 */
    int32_t max_seq_len;     /* longest context any sequence will reach */
    int32_t max_turns;       /* width of the per-sequence action table */
    int32_t action_mod;      /* action id of a turn = (first decoded token of the turn) % action_mod;
                                0 = the host supplies action ids with sr_set_actions */
    int32_t max_prefill_rows;/* rows (sequences x chunk tokens) processed per prefill pass; 0 = default 8192 */
    uint64_t kv_pool_bytes;  /* size of the KV page pool (K and V, all layers) */
    float temperature;       /* 0 = greedy decoding; > 0 = sample from softmax(logits / temperature) (the paper's
                                rollouts use 0.7, Section 3.1) by the Gumbel-max rule:
                                token = argmax_v (logit_v / T - ln(-ln(u_v))), lowest index on ties, with
                                u_v = (top 23 bits of SplitMix64(key, counter v) + 0.5) / 2^23 and key derived from
                                (sample_seed, original sequence id, position of the token): reproducible, and
                                independent of where the sequence sits in the batch */
    uint64_t sample_seed;
    float tau_H;             /* 0 = the one-clause gate of Eq. 2; > 0 = sr_gate also retires a group when the
                                fraction of its members that have finished (sr_finish_sequences) is >= tau_H
                                (Appendix E, Eq. 3) */
    int32_t fp32_debug;      /* 1 = debugging build of the path: every activation, the stored keys and values
                                and the attention probabilities stay in single precision (weights are the same
                                bf16 values, widened exactly) and the contractions run as plain fp32
                                multiply-adds.  Paging, copy-on-write, the split of the context and of the
                                projections' inner dimension, the order in which partial results are added,
                                token selection, gate and compaction are the ones of the normal path, so a
                                difference from an exact evaluation beyond single-precision rounding (logits:
                                1e-4) points at indexing rather than at bf16 operands.  Slow; a KV page takes
                                twice the bytes, so kv_pool_bytes holds half as many pages. */
} sr_options;

/* bf16 device pointers; borrowed only for the duration of sr_load_weights. */
typedef struct {
    const void *wq, *wk, *wv;   /* [n_q*d][hidden], [n_kv*d][hidden], [n_kv*d][hidden] */
    const void *wo;             /* [hidden][n_q*d] */
    const void *wg, *wu;        /* [ffn][hidden] */
    const void *wd;             /* [hidden][ffn] */
    const void *bq, *bk, *bv;   /* [n_q*d], [n_kv*d], [n_kv*d]; ignored when qkv_bias == 0 */
    const void *norm1, *norm2;  /* [hidden] RMSNorm gains before attention / before the FFN */
} sr_layer_weights;

typedef struct {
    const void *embed;              /* [vocab][hidden] */
    const void *lm_head;            /* [vocab][hidden]; ignored when tied_lm_head == 1 */
    const void *final_norm;         /* [hidden] */
    const sr_layer_weights *layers; /* HOST array of n_layers entries (of device pointers) */
} sr_weights;

typedef struct {
    int64_t decoded_tokens;   /* tokens appended by sr_decode_step, summed over sequences */
    int64_t prefill_tokens;   /* tokens appended by sr_prefill_chunk (shared prompt counted once per group) */
    int32_t n_live_groups, n_live_seq, seq_len, turn;
    int32_t pages_total, pages_in_use;
    int32_t groups_retired;   /* total over all gates so far */
    int32_t pages_freed;      /* total over all gates so far */
    int32_t cow_page_copies;  /* pages duplicated because a member appended into a shared page */
    int32_t seqs_finished;    /* sequences taken out by sr_finish_sequences */
    int32_t groups_finished;  /* groups that left because their last member finished (not retired by the gate) */
} sr_stats_t;

/*
 * Create a context for n_groups groups of G sequences each and threshold d_L
 * (Eq. 2; resolved to the rational round(d_L*1e6)/1e6).  Allocates the KV pool and all
 * scratch on the current device.  *out is set on success.
 * SR_E_ARG: null pointers, G < 2, unsupported shape/options; SR_E_NOMEM / SR_E_HIP: allocation failed.
 */
int sr_init(sr_ctx **out, const sr_model_shape *shape, int n_groups, int G, double threshold,
            const sr_options *opt);

/* Release everything the context owns.  Synchronises the device.  NULL is allowed. */
void sr_destroy(sr_ctx *ctx);

/*
 * Copy the weights into the library's own packed layout (device -> device, on `stream`)
 * and wait for completion; the caller may free its tensors afterwards.
 */
int sr_load_weights(sr_ctx *ctx, const sr_weights *w, void *stream);

/*
 * Append chunk_len tokens to every live sequence and leave the logits that follow the
 * last of them (Section 2.2: the environment's observation is appended before each action;
 * Appendix C.2: observation tokens are injected, not generated).
 *   shared_per_group = 1: tokens is device int32 [n_live_groups][chunk_len]; the chunk is the
 *       prompt common to the G members of a group; its KV pages are computed once and
 *       shared by the members (copy-on-write).  Only legal while every sequence is empty.
 *   shared_per_group = 0: tokens is device int32 [n_live_seq][chunk_len], one chunk per
 *       sequence; starts a new turn (the next sr_decode_step records the turn's action).
 * SR_E_ARG: bad arguments or max_seq_len exceeded; SR_E_NOMEM: not enough free KV pages
 * (nothing is launched); SR_E_STATE: shared prefill on non-empty sequences, weights not loaded.
 * With no live group the call is a no-op returning SR_OK.
 */
int sr_prefill_chunk(sr_ctx *ctx, const int32_t *tokens, int chunk_len, int shared_per_group,
                     void *stream);

/*
 * One generation step of every live trajectory (Section 2.2: rollout is token-by-token sampling, one
 * model call per environment step and trajectory, and is what dominates the wall-clock; Appendix C.1:
 * the per-step loop over the group's trajectories that the gate interrupts).
 * Decode one token for every live sequence: pick token = forced[r] if forced != NULL, else
 * the library's own choice -- greedy (largest current logit, lowest index on ties) or, with
 * temperature > 0, the sampled token; append it and compute the logits that follow it.
 * out_tokens (device int32 [n_live_seq], may be NULL) always receives the library's own
 * choice, also under forcing.  On the first decode step after a
 * per-sequence prefill the turn's action id (token % action_mod, from the token actually
 * appended) is recorded in the action table.
 * SR_E_STATE before any prefill; SR_E_ARG when max_seq_len would be exceeded; SR_E_NOMEM
 * when a needed KV page cannot be allocated.
 */
int sr_decode_step(sr_ctx *ctx, const int32_t *forced, int32_t *out_tokens, void *stream);

/*
 * Evaluate the gate after turn K = `turn` (1-based count of recorded actions compared):
 * for each live group S_K = sum over the G(G-1)/2 member pairs of the Levenshtein distance
 * between their first K action ids (Section 3.2; all members hold K actions, so
 * d_K = S_K / (C(G,2)*K)), and retire = [d_K < d_L] (Eq. 2, strict) evaluated in integers as
 * S_K < ceil(round(d_L*1e6) * C(G,2) * K / 1e6).
 * out_sums (device int32 [n_live_groups]) and out_retire (device uint8 [n_live_groups]) may
 * be NULL; the mask is also kept inside the context for sr_retire_and_compact.
 * SR_E_ARG: turn < 1 or > max_turns; SR_E_STATE: fewer than `turn` actions recorded.
 */
int sr_gate(sr_ctx *ctx, int turn, int32_t *out_sums, uint8_t *out_retire, void *stream);

/*
 * The cut itself (Section 3.2, paragraph "The gate": when the gate fires, every trajectory of the group
 * that has not ended yet is stopped after step K and the remaining steps are never generated; Appendix
 * C.1: the cut group is skipped by the trainer).
 * Apply the mask of the preceding sr_gate: rows of retired groups are removed from every
 * per-sequence array (order of survivors kept), their KV pages are released (a shared
 * prompt page returns to the pool when its last holder leaves) and the batch shrinks.
 * This call waits for the mask on the host (the one synchronisation per gate turn) and
 * stores the number of surviving groups in *host_n_live_groups (may be NULL).
 * Retiring every group is legal; later prefill/decode calls are then no-ops.
 * SR_E_STATE: no gate since the last compaction.
 */
int sr_retire_and_compact(sr_ctx *ctx, int *host_n_live_groups, void *stream);

/*
 * Take single sequences out of the batch because their trajectory has ended (success or failure
 * reported by the environment) while other members of their group go on (Section 3.2, paragraph
 * "The gate", cuts only the trajectories that have not ended by step K, so some may have; Appendix B
 * defines the fraction that has, tau_K).  host_done: HOST uint8 [n_live_seq], non-zero = finished.  Call
 * between a turn's last sr_decode_step and the next sr_prefill_chunk: the sequence is recorded as
 * finished after `turn` environment steps.  Its private KV pages are freed and its references to
 * the shared prompt pages dropped; its action prefix is kept, because a later sr_gate still
 * compares it with the other members' (a pair is then divided by the longer of the two prefix
 * lengths, Section 3.2, and the member counts towards tau_K).  A group whose last member
 * finishes leaves the batch without being retired.  Rows keep their order; page table and row
 * maps are re-uploaded behind the work already queued.  *host_n_live_seq (may be NULL) receives
 * the number of sequences left.  SR_E_STATE: before the first turn, in the middle of one, or between
 * sr_gate and sr_retire_and_compact (the pending mask is indexed by the groups live at the gate).
 * After this call sr_gate writes to out_sums the plain sum of the pair distances.
 */
int sr_finish_sequences(sr_ctx *ctx, const uint8_t *host_done, int *host_n_live_seq, void *stream);

/*
 * Stand-alone gate over many groups and several prefix lengths (no context needed).
 * actions: device int32 [n_groups][G][stride]; prefix_lens: HOST int [n_lens], each in
 * [1, min(stride, 32)]; sums: device int32 [n_lens][n_groups]; retire: device uint8
 * [n_lens][n_groups] (either may be NULL).  2 <= G <= 16, n_lens <= 8.
 */
int sr_gate_batch(const int32_t *actions, int n_groups, int G, int stride, const int *prefix_lens,
                  int n_lens, double threshold, int32_t *sums, uint8_t *retire, void *stream);

/*
 * sr_gate_batch computed by the other work decomposition -- one workgroup per group, every pair's
 * Levenshtein table advanced one anti-diagonal at a time with the last three anti-diagonals in LDS --
 * for measuring the two side by side.  Same arguments, same results bit for bit (Section 3.2, Eq. 2).
 */
int sr_gate_batch_antidiag(const int32_t *actions, int n_groups, int G, int stride, const int *prefix_lens,
                           int n_lens, double threshold, int32_t *sums, uint8_t *retire, void *stream);

/*
 * Teacher-forced scoring (Appendix C.2).  Appends chunk_len given tokens to every live sequence
 * exactly like sr_prefill_chunk(..., shared_per_group = 0) -- their K/V are computed and the
 * logits at the chunk's last position are kept -- and adds, for every chunk position t whose
 * action_mask entry is non-zero, log softmax(logits at the position before t)[tokens[t]] to the
 * sequence's running log-likelihood  log p(tau) = sum over action-token positions.  A token is scored
 * by the distribution computed from everything before it, so the chunk's first token is scored by the
 * logits the previous prefill / scoring / decode call left and the context must not be empty
 * (SR_E_STATE).  Observation tokens are either passed with mask 0 or, cheaper, appended with
 * sr_prefill_chunk, which computes no LM head for them.
 *
 * tokens: device int32 [n_live_seq][chunk_len]; action_mask: device uint8, same shape, or NULL
 * (every token counts); out_token_logprob: device float [n_live_seq][chunk_len] receiving the
 * per-token values (0 where masked), or NULL.  Arithmetic: bf16 operands, fp32 accumulation and
 * fp32 log-sum-exp per row; the per-sequence sums are kept in double, added in token order.
 * The running sums follow their sequences through sr_retire_and_compact.
 */
int sr_score_chunk(sr_ctx *ctx, const int32_t *tokens, const uint8_t *action_mask, int chunk_len,
                   float *out_token_logprob, void *stream);

/* Copy the running log-likelihoods of the live sequences to dst: device double [n_live_seq]. */
int sr_get_logprob(sr_ctx *ctx, double *dst, void *stream);

/*
 * Policy-gradient loss of Section 2.1:  L = -(1/N) sum_i A_i log p(tau_i)  over the N = n_groups * G
 * trajectories, with the group-relative advantages of Eq. 1 (population standard deviation;
 * every advantage of a group whose rewards are all equal is exactly 0).  No context needed.
 * logprob: device double [n_groups][G]; rewards: device float [n_groups][G]; advantages: device
 * float [n_groups][G] or NULL; group_scratch: device double [n_groups], overwritten; loss: device
 * double [1].  Groups are added in index order, so the result is reproducible.
 */
int sr_grpo_loss(const double *logprob, const float *rewards, int n_groups, int G, double eps,
                 float *advantages, double *group_scratch, double *loss, void *stream);

/*
 * sr_grpo_loss for callers that cannot allocate device memory or bring a workspace: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments without group_scratch,
 * same kernel, same results bit for bit; the per-group shares go to a fixed device array inside the library
 * (SR_GRPO_STATIC_MAX_GROUPS doubles = 512 KiB, held by every GPU the library runs on until the process
 * ends).  The call allocates and frees nothing.  n_groups above the limit: SR_E_LIMIT, nothing is launched.
 * All calls on one GPU share that array: calls that may overlap on one GPU (different streams) race and
 * must be serialised by the caller; nothing of an earlier call's contents is read.
 */
#define SR_GRPO_STATIC_MAX_GROUPS 65536
int sr_grpo_loss_static(const double *logprob, const float *rewards, int n_groups, int G, double eps,
                        float *advantages, double *loss, void *stream);

/*
 * The update half of a GRPO step, from the logits that the policy being trained gives to the tokens of the kept
 * trajectories (Appendix C.2: one causal forward, log softmax at action-token positions; Section 2.1: the loss over them)
 * to gradients that an optimizer can take.  No context needed; the caller brings every buffer.
 *
 * Rows.  Row t of `logits` is the distribution of token targets[t].  The rows of a sequence lie together, the sequences
 * one behind another: sequence i owns rows [seq_start[i], seq_start[i + 1]), some possibly none.  A row counts unless its
 * mask entry is 0 or it lies outside [seq_start[0], seq_start[n_seq]) (padding).  Rows that do not count are not read; they
 * receive log-probability 0 and a gradient of exactly 0.  An entry of -infinity is a token that cannot occur; a row whose
 * entries are all -infinity, or that holds NaN or +infinity, has log-probability NaN, and so has a counting row whose target
 * lies outside the vocabulary.  seq_start must not decrease; other values give unspecified results, but no access outside
 * the buffers.  A token of probability 0 has log-probability -infinity and, with a reference that allows it, an infinite kl.
 *
 * Arithmetic: the logits are widened to single precision; maximum, sum of exponentials, loss and slopes are single
 * precision, sums over tokens double, added in a fixed order (the results are the same bit for bit from call to call); the
 * gradient is rounded once, to the type of the logits.
 *
 * Outputs overlap neither each other, nor the workspace, nor an input; the gradient alone may lie in the place of the logits.
 * That token_logprob shares nothing with old_logprob and ref_logprob is checked: different workgroups would read and write it.
 */
typedef enum {
    SR_F32 = 0, SR_BF16 = 1, SR_F16 = 2,
    SR_E4M3 = 3, SR_E5M2 = 4   /* 8 bits: outputs of sr_add_norm alone (largest finite values 448 and 57344) */
} sr_dtype;

typedef struct {
    const void *logits;        /* device [n_rows][ld_logits], of type dtype, any alignment that the type allows */
    void *grad;                /* device [n_rows][ld_grad], same type: d(loss * grad_scale) / d(logits); may be `logits` itself
                                  (with the same row stride), must not overlap it otherwise; NULL: the loss alone */
    int64_t ld_logits, ld_grad;/* elements from one row to the next, >= vocab */
    const int32_t *targets;    /* device [n_rows] */
    const uint8_t *mask;       /* device [n_rows], 0 = the row does not count; NULL: all count */
    const int32_t *seq_start;  /* device [n_seq + 1] */
    float *token_logprob;      /* device [n_rows], written; may be NULL; shares no element with old_logprob and ref_logprob */
    int32_t dtype;             /* sr_dtype of logits and grad */
    int32_t n_rows, vocab, n_seq;
    float grad_scale;          /* multiplies the gradient only (loss scaling for 16-bit gradients) */
    int32_t reserved;
} sr_token_rows;

/* Bytes of device memory, 16-byte aligned, that the two losses need as workspace.  Nothing in it outlives the call, and
 * calls that may overlap (different streams) need one each. */
#define SR_TOKEN_LOSS_WORKSPACE(n_rows, n_seq) (65536 + (size_t)64 * (size_t)(n_rows) + (size_t)32 * (size_t)(n_seq))

/*
 * Clipped policy loss with a KL term.  With l the log-probability of a counting row's token, A the advantage of its
 * sequence (Eq. 1; sr_grpo_loss writes them), r = exp(l - old_logprob) and, where ref_logprob is given, d = ref_logprob - l:
 *     surrogate = min(r A, clip(r, 1 - clip_low, 1 + clip_high) A)        kl = exp(d) - d - 1
 *     loss = mean(kl_coef * kl - surrogate)
 * (kl is the estimate, never negative, of KL(policy | reference) from the sampled token.)  The mean is one of
 *     SR_MEAN_TOKENS     over all counting rows
 *     SR_MEAN_SEQUENCES  over the rows of a sequence, then over the sequences that have any
 *     SR_MEAN_SUMS       of the sums over a sequence's rows, over the sequences that have any: with r = 1 and kl_coef = 0 the
 *                        gradient of the loss of Section 2.1
 * and 0 where nothing counts.  The gradient of a row is slope * (onehot(target) - softmax), slope = weight *
 * (kl_coef * (1 - exp(d)) - r A [r A <= clip(r) A]).
 * stats: device float [4]: loss, mean surrogate, mean kl (0 without ref_logprob), mean of [r A > clip(r) A] (the fraction of
 * tokens that the clip takes out of the gradient).
 * old_logprob, ref_logprob: device float [n_rows], as sr_score_chunk writes them; ref_logprob may be NULL if kl_coef == 0.
 * advantages: device float [n_seq].
 * SR_E_ARG: null pointers, a bad dtype, shape, stride or option, token_logprob overlapping old_logprob or ref_logprob, a workspace
 * that is too small or not 16-byte aligned;
 * SR_E_LIMIT: more than 2^26 - 4 rows or 2^23 sequences, or more threads than a launch may have (2^32 - 1; a row of more than
 * 8 KiB takes 256, and so does every 16 KiB of a preference loss's gradient).  n_rows may be 0.
 */
typedef enum { SR_MEAN_TOKENS = 0, SR_MEAN_SEQUENCES = 1, SR_MEAN_SUMS = 2 } sr_reduce;
typedef struct {
    float clip_low, clip_high; /* 0 <= clip_low <= 1, clip_high >= 0 */
    float kl_coef;
    int32_t reduce;            /* sr_reduce */
} sr_policy_options;
int sr_policy_loss(const sr_token_rows *rows, const float *old_logprob, const float *ref_logprob, const float *advantages,
                   const sr_policy_options *opt, float *stats, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Preference loss over pairs of sequences: sequence 2 i is the one preferred to sequence 2 i + 1 (two members of a group with
 * different rewards, for example).  With the log ratio L of a sequence = sum over its counting rows of (l - ref_logprob) and
 * the margin m_i = beta (L_{2i} - L_{2i+1}):
 *     loss = mean over pairs of  -(1 - label_smoothing) log sigmoid(m) - label_smoothing log sigmoid(-m)
 * A sequence without counting rows has L = 0.  The gradient of a row of sequence 2 i is s_i (onehot(target) - softmax), of
 * sequence 2 i + 1 the same with -s_i, s_i = beta / pairs * (label_smoothing sigmoid(m_i) - (1 - label_smoothing) sigmoid(-m_i)).
 * stats: device float [4]: loss, fraction of pairs with m > 0, mean of beta L over the preferred and over the other sequences.
 * log_ratio: device float [n_seq] receiving L, or NULL.  ref_logprob: device float [n_rows], or NULL (taken as 0).
 * SR_E_ARG as above, and n_seq odd, beta not finite, label_smoothing outside [0, 1].
 */
int sr_preference_loss(const sr_token_rows *rows, const float *ref_logprob, float beta, float label_smoothing, float *log_ratio,
                       float *stats, void *workspace, size_t workspace_bytes, void *stream);

/*
 * The global 2-norm of a list of gradient tensors, and the list scaled down to a largest norm.
 *     norm = |scale| * sqrt(sum over all tensors and elements of g^2)        c = max_norm / norm if norm > max_norm, else 1
 *     out = scale * c * g
 * norm: device float [1].  Squares are added in double, in a fixed order, so that neither 1e30 nor 1e-30 is lost and
 * the norm is the same bit for bit from call to call.  A norm that is infinite or NaN as it is written (a float: beyond FLT_MAX it is
 * infinite) leaves c = 1, out = scale * g: for the caller who looks at the norm.
 * host_tensors: HOST array, read during the call only; the data are device memory, contiguous, any alignment that the type
 * allows.  `out` may be `data` itself or NULL (in place; then nothing is written where scale * c is 1) and must not overlap any
 * tensor otherwise; its type is that of the data, or SR_F32.  sr_grad_norm reads `data` only.
 * workspace: SR_GRAD_NORM_WORKSPACE bytes of device memory, 16-byte aligned.  Nothing in it outlives the call, and calls that may
 * overlap (different streams) need one each; it, `norm` and the tensors share no memory.
 * SR_E_ARG: null pointers, n < 0 or > 2^36, a bad type, scale or max_norm not finite, max_norm < 0.  The list and its tensors may
 * be empty.
 */
typedef struct {
    void *data;
    void *out;
    int64_t n;                 /* elements */
    int32_t dtype, out_dtype;  /* sr_dtype; out_dtype is ignored where out is NULL */
} sr_tensor;
#define SR_GRAD_NORM_WORKSPACE 65536
int sr_grad_norm(const sr_tensor *host_tensors, int n_tensors, float scale, float *norm, void *workspace, size_t workspace_bytes,
                 void *stream);
int sr_clip_grad_norm(const sr_tensor *host_tensors, int n_tensors, float scale, float max_norm, float *norm, void *workspace,
                      size_t workspace_bytes, void *stream);

/*
 * The same for a list that stays: sr_plan_tensors copies it to `table` (device memory of the caller, 16-byte aligned,
 * SR_TENSOR_TABLE_BYTES(n_tensors) bytes, kept as long as the plan is used), waits for the stream, and fills *host_plan.  The planned
 * calls then take any number of tensors in one launch a pass, on any stream.  A plan names addresses: it has to be made again when
 * a tensor moves, and a list that moves at every step is cheaper in the arguments of the calls above.  Results are those of the calls
 * above but for the order in which the squares are added.
 * SR_E_ARG as above; SR_E_LIMIT: more than 2^31 pieces of 8192 elements; SR_E_NOMEM, SR_E_HIP.
 */
#define SR_TENSOR_TABLE_BYTES(n_tensors) ((size_t)64 + (size_t)24 * (size_t)(n_tensors))
typedef struct {
    const void *table;
    int64_t chunks, keep;      /* the library's */
    int32_t n_tensors, reserved;
} sr_tensor_plan;
int sr_plan_tensors(const sr_tensor *host_tensors, int n_tensors, void *table, size_t table_bytes, sr_tensor_plan *host_plan, void *stream);
int sr_planned_grad_norm(const sr_tensor_plan *host_plan, float scale, float *norm, void *workspace, size_t workspace_bytes, void *stream);
int sr_planned_clip_grad_norm(const sr_tensor_plan *host_plan, float scale, float max_norm, float *norm, void *workspace,
                              size_t workspace_bytes, void *stream);

/*
 * What surrounds the matrix products of the decoder being trained (sr_model_shape: an embedding, pre-norm blocks, RMSNorm), forward
 * and backward.  No context needed; the caller brings every buffer.  Rows of any width, at any address their type allows, with any
 * distance >= width between them; what lies between rows is neither read nor written.  Arithmetic, sums and statistics are in single
 * precision, every output is rounded once, and results are the same bit for bit from call to call.
 *
 * Types: a call has one type T of SR_F32, SR_BF16, SR_F16 and a second one for what is wider, T itself or SR_F32 (a residual in single
 * precision beside 16-bit branches).  Outputs overlap neither each other, nor an input, nor the workspace, except where a call says that
 * one may lie in the place of an input: then with the same address, type and row distance.
 */
typedef struct {
    void *data;                /* device [rows][ld]; NULL: not there */
    int64_t ld;                /* elements from one row to the next, >= width */
    int32_t dtype;             /* sr_dtype */
    int32_t reserved;
} sr_rows;

/*
 * Rows of a table for a list of tokens:  out[i] = scale * table[tokens[i]].  A token outside the vocabulary (padding) has a row of zeros.
 * table [vocab][width] of type T, out [n][width] of T or SR_F32; tokens: device int32 [n].
 * SR_E_ARG: null pointers, bad types, sizes or strides, a scale that is not finite; SR_E_LIMIT: width > 2^20, more than 2^31 - 1 threads.
 */
int sr_embed(const sr_rows *table, int vocab, int width, const int32_t *tokens, int n, float scale, const sr_rows *out, void *stream);

/*
 * Its gradient:  d_table[v] = scale * sum of d_out[i] over all i with tokens[i] = v, zeros for every other v; with accumulate != 0 this is
 * added to what d_table holds, and rows of tokens that do not occur are not touched.  Sums run over ascending i, in parts whose length
 * depends on sizes and types alone.  d_out [n][width] of type T, d_table [vocab][width] of T or SR_F32.
 * workspace: device memory, 16-byte aligned, SR_EMBED_GRAD_WORKSPACE(n, width) bytes; nothing in it outlives the call, and calls that
 * may overlap (different streams) need one each.
 * SR_E_ARG as above; SR_E_LIMIT: n > 2^20 (a larger batch goes in parts that accumulate), width > 2^20, too many rows for a launch.
 */
#define SR_EMBED_GRAD_SUMS(n, width) ((size_t)(n) / 8 * 4 * (size_t)(width))
#define SR_EMBED_GRAD_WORKSPACE(n, width) \
    (65536 + (size_t)32 * (size_t)(n) + (size_t)256 * (size_t)(width) + \
     (SR_EMBED_GRAD_SUMS(n, width) < (size_t)1 << 22 ? SR_EMBED_GRAD_SUMS(n, width) : (size_t)1 << 22))
int sr_embed_grad(const sr_rows *d_out, const int32_t *tokens, int n, float scale, const sr_rows *d_table, int vocab, int width,
                  int accumulate, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Dropout.  Its mask is a function of numbers and is never stored: element (row r, column c) of a batch of `width` columns is dropped iff
 *     (bits >> 16 (c % 4)) % 2^16 < D,   bits = word (first_row + r) * ceil(width / 4) + c / 4
 *     D = min(65535, round(65536 p))
 * of the SplitMix64 stream keyed (seed, mask + *step): the same mask forward and backward, whatever the types, strides and the operator,
 * and whatever part of the rows a call is given (first_row).  What is kept is multiplied by 65536 / (65536 - D), the reciprocal of the
 * share that these bits keep; what is dropped is 0, also where the input is not finite.  So p below 2^-17 drops nothing, and however near
 * p is to 1, one element in 65536 is kept.
 * `step` (device, may be NULL) is read when the kernel runs, so that a replayed graph draws another mask at every step.
 */
typedef struct {
    float p;                   /* 0 <= p < 1; D / 65536 of it counts */
    uint32_t reserved;
    uint64_t seed;
    uint64_t mask;             /* which mask of that seed: a layer's number, for example */
    uint64_t first_row;        /* number of the first row */
    const uint64_t *step;      /* device: added to `mask`; NULL: 0 */
} sr_mask;

/*
 * out = dropout(x), or residual + dropout(x).  The backward pass is the same call on the gradient, without the residual.
 * x [rows][width] of type T; residual (NULL, or data NULL: none) of T or SR_F32; out of the residual's type, or T.  out may lie in the
 * place of x or of the residual.
 * SR_E_ARG: null pointers, p outside [0, 1), bad types, sizes or strides; SR_E_LIMIT: width > 2^30, more than 2^31 - 1 threads.
 */
int sr_dropout(const sr_rows *x, const sr_rows *residual, const sr_rows *out, int rows, int width, const sr_mask *mask, void *stream);

/*
 * Residual + branch, and the root-mean-square norm of the sum:
 *     total = residual + dropout(x), rounded to the residual's type
 *     rstd = 1 / sqrt(mean over a row of total^2 + eps)          out = total * rstd * gain
 * The norm is that of the sum as it is stored.  x.data NULL: total = residual.  x.dtype is T in any case.
 * out of type T, or in 8 bits with scales: for each block of scale_block columns (32, 64 or 128; the last one of a row may be shorter), or
 * for each row (0), scale = max(largest |out| of the block / largest finite value of the type, 2^-126), and the stored code is out / scale,
 * rounded to nearest even.  NaN does not enter the scale; its code is NaN.
 * A row whose squares' sum is beyond single precision has rstd 0, one whose squares all vanish in it 1 / sqrt(eps): with eps 0 infinity,
 * and NaN where the row is 0.
 * SR_E_ARG: null pointers (rstd, total and dropout may be NULL), bad types, sizes, strides or options, eps < 0 or not finite;
 * SR_E_LIMIT: width > 16384, more than 2^32 - 1 threads.  rows may be 0.
 */
typedef struct {
    sr_rows x;                 /* branch [rows][width] of type T, or no data */
    sr_rows residual;          /* of type T or SR_F32 */
    sr_rows total;             /* of the residual's type; may lie in its place; no data: not stored */
    sr_rows out;               /* of type T (may lie in the place of x), SR_E4M3 or SR_E5M2 */
    const void *gain;          /* device [width], of type T or SR_F32 */
    float *rstd;               /* device [rows], or NULL */
    float *scales;             /* device [rows][ceil(width / scale_block)], or [rows] where scale_block is 0; 8-bit outputs only */
    const sr_mask *dropout;    /* HOST, NULL: none */
    int32_t gain_dtype, rows, width, scale_block;
    float eps;
    int32_t reserved;
} sr_norm_rows;
int sr_add_norm(const sr_norm_rows *rows, void *stream);

/*
 * Its gradients.  With n = total * rstd and g = d_out * gain:
 *     d_residual = rstd * (g - n * mean over the row of g n) + d_total       d_x = dropout(d_residual)       d_gain = sum over rows of d_out * n
 * d_total is the gradient that reaches the sum from behind it (no data: none); d_x is formed from d_residual before that is rounded.
 * d_gain is overwritten, or added to with accumulate != 0.  Any of the three outputs may be left out, not all.  With an 8-bit output d_out is the
 * gradient of what its codes and scales stand for.
 * workspace (only with d_gain): device memory, 16-byte aligned, SR_NORM_GRAD_WORKSPACE(rows, width) bytes; nothing in it outlives the
 * call, and calls that may overlap (different streams) need one each.
 * Errors as above.  rows may be 0: d_gain is then zeros, or stays.
 */
typedef struct {
    sr_rows d_out;             /* [rows][width] of type T */
    sr_rows total;             /* as sr_add_norm stored it (without a branch: the residual), of type T or SR_F32 */
    sr_rows d_total;           /* of total's type, or no data */
    sr_rows d_residual;        /* of total's type; may lie in the place of d_total; or no data */
    sr_rows d_x;               /* of type T; may lie in the place of d_out; or no data */
    const float *rstd;         /* device [rows] */
    const void *gain;          /* device [width], of type T or SR_F32 */
    void *d_gain;              /* device [width], of type T or SR_F32, or NULL */
    const sr_mask *dropout;    /* HOST, NULL: none */
    int32_t gain_dtype, d_gain_dtype, rows, width, accumulate, reserved;
} sr_norm_grad_rows;
#define SR_NORM_GRAD_MOST(width) \
    ((width) <= 1024 ? (size_t)8192 * (size_t)(width) : (width) <= 4096 ? (size_t)1 << 23 : (size_t)2048 * (size_t)(width))
#define SR_NORM_GRAD_WORKSPACE(rows, width) \
    (256 + ((size_t)4 * (size_t)(rows) * (size_t)(width) < SR_NORM_GRAD_MOST(width) ? (size_t)4 * (size_t)(rows) * (size_t)(width) \
                                                                                    : SR_NORM_GRAD_MOST(width)))
int sr_add_norm_grad(const sr_norm_grad_rows *rows, void *workspace, size_t workspace_bytes, void *stream);

/*
 * The in-group divergence signals of Appendix B at step K, and the gates of Eq. 2 and of
 * Appendix E (Eq. 3), for groups whose members may have finished early (no context needed).
 *
 * Member i of a group finished after end_step[i] environment steps (any value > stride while
 * it is still running; values below 0 count as 0), so at step K it contributes the prefix
 * a_i[0 : len_i], len_i = min(K, end_step[i]).
 *   d_K            mean over the C(G,2) pairs of the Levenshtein distance of the two prefixes
 *                  divided by the longer of their lengths (Section 3.2); a pair of empty
 *                  prefixes counts 0
 *   lev_scaled     the same sum before the division by C(G,2), exact, in units of
 *                  1 / lcm(1..32) = 1 / 144403552893600
 *   lev_sum        the plain sum over pairs of the Levenshtein distances (S_K when nobody has
 *                  finished early)
 *   bigram_jaccard mean over pairs of 1 - |A n B| / |A u B|, A and B the SETS of consecutive
 *                  action pairs of the two prefixes; two empty sets count as identical (0)
 *   unique_prefix  number of distinct prefixes among the G members (the ratio is this / G)
 *   n_at_step      members whose prefix reaches step K; the next three are taken over them
 *   unique_action  distinct step-K actions a_{i,K}; unique_obs: distinct step-K observation
 *                  ids o_{i,K} (0 if obs is NULL); action_entropy: Shannon entropy of the
 *                  step-K action, natural logarithm
 *   n_done         members that had finished by step K (end_step <= K); tau_K = n_done / G
 *   cut_d          d_K < d_L (Eq. 2, strict), decided in integers with d_L read as
 *                  round(d_L * 1e6) / 1e6;  cut_or: cut_d or tau_K >= tau_H (Eq. 3), tau_H
 *                  read the same way (a tau_H above 1 switches the second clause off)
 * Pair terms are added in the order (0,1), (0,2), ..., (G-2,G-1), so d_K and bigram_jaccard
 * are reproducible bit for bit.
 *
 * actions, obs: device int32 [n_groups][G][stride] (obs may be NULL); end_step: device int32
 * [n_groups][G] or NULL (nobody has finished); prefix_lens: HOST int [n_lens], each in
 * [1, min(stride, 32)]; out: device [n_lens][n_groups].  2 <= G <= 16, n_lens <= 8.
 * SR_E_ARG on anything else.  Asynchronous on `stream`; the caller owns every buffer.
 */
typedef struct {
    double d_K;
    int64_t lev_scaled;
    double bigram_jaccard;
    double action_entropy;
    int32_t unique_prefix, n_at_step, unique_action, unique_obs, n_done;
    int32_t lev_sum;
    uint8_t cut_d, cut_or;
    uint8_t reserved[6];
} sr_signals_t;
int sr_signals_batch(const int32_t *actions, const int32_t *obs, const int32_t *end_step, int n_groups, int G,
                     int stride, const int *prefix_lens, int n_lens, double d_L, double tau_H,
                     sr_signals_t *out, void *stream);

/* Overwrite the action ids of turn `turn` (1-based) for all live sequences:
 * ids is device int32 [n_live_seq].  For action_mod == 0, or for tests. */
int sr_set_actions(sr_ctx *ctx, int turn, const int32_t *ids, void *stream);

/* Copy the action table of the live sequences: dst is device int32 [n_live_seq][max_turns];
 * turns not yet recorded hold -1. */
int sr_get_actions(sr_ctx *ctx, int32_t *dst, void *stream);

/* Copy the current logits: dst is device float [n_live_seq][vocab]. */
int sr_get_logits(sr_ctx *ctx, float *dst, void *stream);

/* Original sequence index (group*G + member at sr_init time) of every live row:
 * host int32 [n_live_seq].  Host-side bookkeeping only; does not touch the stream. */
int sr_get_live_map(sr_ctx *ctx, int32_t *host_orig_seq_ids);

/* Counters (host struct). */
int sr_stats(sr_ctx *ctx, sr_stats_t *host_stats);

/*
 * Per-kernel timing for benchmarks.  While enabled, every kernel launch of sr_prefill_chunk /
 * sr_decode_step is bracketed by HIP events on the caller's stream (this perturbs the stream
 * slightly; enable it for sampled steps only).  sr_profile_read waits for the stream, adds the
 * elapsed times up per kernel class and clears the record.  Classes are numbered by
 * sr_kernel_class; `out` is a HOST array of SR_KC_COUNT entries.
 */
typedef enum {
    SR_KC_NORM = 0,        /* residual add + RMSNorm (+ embedding gather) */
    SR_KC_GEMM_QKV,
    SR_KC_QKV_POST,        /* split-K sum + bias + RoPE + KV page write */
    SR_KC_ATTN_DECODE,     /* decode attention: shared-prompt phase and private phase in one launch */
    SR_KC_ATTN_PREFILL,
    SR_KC_ATTN_MERGE,
    SR_KC_GEMM_O,
    SR_KC_GEMM_GATE_UP,    /* with the SwiGLU epilogue */
    SR_KC_GEMM_DOWN,
    SR_KC_GEMM_LM_HEAD,
    SR_KC_ARGMAX,
    SR_KC_COUNT
} sr_kernel_class;

typedef struct {
    int64_t launches;
    double total_ms;
} sr_kernel_time;

int sr_profile(sr_ctx *ctx, int enable);
int sr_profile_read(sr_ctx *ctx, sr_kernel_time *host_out /* [SR_KC_COUNT] */, void *stream);

/*
 * Measured ceilings of the chip, for the roofline report next to the published peaks (HBM 8 TB/s, dense
 * bf16 matrix cores 2.5 PFLOP/s).  Both calls launch probe kernels on `stream`, time `iters` launches with
 * HIP events, wait for them and write the rate to a HOST double.  They are not part of the method.
 *   sr_probe_hbm: src (device, `bytes` long; use well over 256 MiB so that no cache holds it) is streamed by
 *     4096 wavefronts with 16-byte loads -- mode 0 with the non-temporal hint of the weight-streaming kernels,
 *     mode 1 with default loads, mode 2 copied to dst (device, `bytes` long; read + written bytes are counted).
 *     For modes 0 and 1 dst must point at >= 16 device bytes (never written in practice).
 *   sr_probe_mfma_bf16: register-resident 32x32x16 bf16 matrix-core loop on 1024 workgroups; scratch is
 *     device memory of at least 1 MiB that receives one float per thread.
 */
int sr_probe_hbm(const void *src, void *dst, size_t bytes, int mode, int iters, void *stream, double *host_GBs);
int sr_probe_mfma_bf16(void *scratch, size_t scratch_bytes, int iters, void *stream, double *host_TFLOPs);

/*
 * The matrix-core loop with operand-sized loads beside it, for telling what the operand traffic of a tiled GEMM leaves
 * of the matrix pipe: 256 workgroups of eight wavefronts; every wavefront alternates sixteen register-resident
 * 32x32x16 bf16 MFMAs with loads_per_16 (2, 4 or 8; 0 with path 0) wavefront-wide loads of 16 bytes per lane from buf,
 * into registers (path 1) or straight into LDS (path 2); lds_reads != 0 adds twelve 16-byte LDS reads per sixteen MFMAs
 * (paths 0 and 2).  A 256 x 256 x 32 GEMM step on eight computing wavefronts corresponds to loads_per_16 = 4.
 * buf: device memory, buf_bytes a power of two >= 64 KiB (small = L2 resident; read only).  scratch: device memory of
 * at least 512 KiB that receives one float per thread.  Waits for the stream; writes the matrix rate and the rate of
 * the loads to HOST doubles (host_load_GBs may be null).  SR_E_ARG for any other combination.
 */
int sr_probe_mfma_under_loads(const void *buf, size_t buf_bytes, void *scratch, size_t scratch_bytes, int path,
                              int loads_per_16, int lds_reads, int iters, void *stream, double *host_TFLOPs,
                              double *host_load_GBs);

/*
 * One layer's decode attention launch at the 7B attention shape (28 query / 4 kv heads of 128, 64-token pages) on
 * synthetic pages, for studying its phases apart: phases = 1 the shared-prompt phase alone (one unit per group, the
 * members' query rows batched over each prompt block), 2 the private phase alone (one unit per sequence, priv_splits
 * splits of priv_tokens tokens), 3 both in one launch as sr_decode_step runs them; adding 4 puts the launch that merges
 * the partial results behind each attention launch (the duration is then that of the pair).  hot != 0: every page-table entry
 * names one of a few pages, so all K/V loads are cache hits.  Allocates and frees its own buffers, waits for the
 * stream, and writes the mean launch duration in microseconds and the K/V bytes one launch has to read to HOST doubles.
 */
int sr_probe_decode_attention(int n_groups, int G, int shared_tokens, int priv_tokens, int priv_splits, int phases,
                              int hot, int iters, void *stream, double *host_us, double *host_kv_bytes);

/* Text for a status code; for SR_E_HIP the text of the last HIP error seen by this thread. */
const char *sr_strerror(int status);

#ifdef __cplusplus
}
#endif
#endif /* SR_H */
