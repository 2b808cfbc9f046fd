/*
 * sapo.h — C ABI of the SAPO policy-scoring library for NVIDIA B200 (sm_100a).
 *
 * One SAPO node's policy update (paper Algorithm 1: the steps that put the training set
 * together and update the policy) scores a batch made of I locally generated and J swarm-sampled
 * rollouts per question.  This library runs the data-parallel part of that update:
 *
 *   sapo_pack_rollouts     training set T^n = {local picks} U {external picks}
 *                          (Section 3.2, training-set equation) as a varlen layout
 *   sapo_group_advantages  GRPO group-relative advantages (Section 4.2)
 *   sapo_policy_loss_fwd   LM-head log-probs of the chosen tokens (Section 3.2: rollouts
 *                          are re-encoded and their token-level values computed under the
 *                          node's own policy) + clipped-ratio surrogate, KL weight 0,
 *                          separate lower/upper clip thresholds (Section 4.2)
 *   sapo_policy_loss_bwd   gradient of that loss w.r.t. the final hidden states and the
 *                          LM-head weight (Algorithm 1, the policy-gradient step)
 *   sapo_policy_loss_fwd_bwd  the two above in one call that passes over the logits once
 *                          (bf16 operands; the fastest way through a training step)
 *
 * and, around them:
 *   sapo_select_external            filter and sample the shared pool (Section 3.2 / Section 5)
 *   sapo_policy_loss_bwd_active     backward over the tokens with a gradient only
 *   sapo_policy_loss_fwd_bwd_gather the single-pass call reading the hidden states in place from the
 *                                   rollout stores (the pack then copies none)
 *   sapo_lmhead_lse_partial, sapo_policy_loss_from_partials, sapo_policy_loss_bwd_shard
 *                                   the same loss with W_head sharded by vocabulary over ranks
 *   sapo_adam_step                  the optimiser step of Section 4.2 on the LM head
 *   sapo_preference_loss            a preference loss over the completions of a question (paired log
 *                                   ratios), from per-token log-probs to gscale
 *   sapo_preference_loss_fwd_bwd    the same through the LM head, with both gradients
 *   sapo_norm_fwd, sapo_norm_bwd    the norm in front of the LM head (layer norm, RMS norm)
 *   sapo_ckpt8_store, sapo_ckpt8_restore, sapo_norm_replay
 *                                   activations kept in 8 bits between forward and backward
 *   sapo_sample                     draws the next tokens from logits (the answers of a round)
 *   sapo_fp8_store, sapo_fp8_matmul matrices in 8-bit floating point and their product (the head that
 *                                   answers)
 *   sapo_adamw_step                 AdamW over many tensors, states in 32 or 8 bits
 *   sapo_policy_loss_fwd_static     the forward for callers that may not allocate device memory
 *   sapo_group_advantages_warp, sapo_workspace_bytes[_min], sapo_status_string, sapo_timing_*,
 *   sapo_launch_count, sapo_debug_wait_timeout, sapo_debug_bounds_violations
 *                                   sizes, texts, measurement and test hooks
 *
 * General rules
 *   - Every pointer is a DEVICE pointer unless its name starts with h_.  The caller owns
 *     all buffers; the library allocates and frees nothing and keeps no pointer after a
 *     call returns.  Scratch memory is passed in as `workspace`.
 *   - Calls enqueue work on `stream` (a cudaStream_t passed as void*) and return without
 *     synchronising.  Results are valid once the stream has drained.
 *   - Return value: SAPO_OK or a negative host-detected error.  Conditions only the device
 *     can see (capacity overflow, index out of range, a bounded wait that ran out) are
 *     OR-ed as SAPO_ST_* bits into *status (int32 in device memory, zeroed by the caller);
 *     the kernels never trap and never spin without a limit.
 *   - Matrices are row-major with the H (hidden) index contiguous.  Base pointers of
 *     hidden / W_head / dhidden / dW_head / workspace must be 16-byte aligned and the
 *     leading dimensions, in bytes, multiples of 16.
 *   - There is no CPU fallback: without a CUDA device every call returns SAPO_ERR_CUDA.
 *   - Threads.  The calls keep a few per-device values they look up on first use (the driver's
 *     tensor-map encoder, the SM count, the shared-memory opt-in and resident CTA pairs of each
 *     kernel, the address of the built-in scratch of sapo_policy_loss_fwd_static) without locks.
 *     Make the first call of each entry point on each device from one thread (a warm-up step does
 *     it); after that, calls from several threads are safe as long as each uses its own stream,
 *     workspace and outputs.  sapo_timing_* and sapo_launch_count are for one thread only.
 */
#ifndef SAPO_H_
#define SAPO_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* host-detected errors (return values) */
#define SAPO_OK                      0
#define SAPO_ERR_INVALID_ARG        -1
#define SAPO_ERR_UNSUPPORTED_SHAPE  -2
#define SAPO_ERR_WORKSPACE_TOO_SMALL -3
#define SAPO_ERR_CUDA               -4
#define SAPO_ERR_STATIC_SCRATCH_EXCEEDED -5  /* sizes beyond the built-in scratch of the _static call */

/* device-detected conditions (bits of *status) */
#define SAPO_ST_TOKEN_OVERFLOW   0x01  /* packed tokens exceed max_tokens; output truncated   */
#define SAPO_ST_SEQ_OVERFLOW     0x02  /* selected sequences exceed max_seqs; nothing packed  */
#define SAPO_ST_BAD_INDEX        0x04  /* a selection index is outside its rollout buffer     */
#define SAPO_ST_EMPTY_SEQUENCE   0x08  /* a selected rollout has no tokens                    */
#define SAPO_ST_BAD_TOKEN_ID     0x10  /* ids[t] outside [0, V): token scored as masked       */
#define SAPO_ST_WAIT_TIMEOUT     0x20  /* a bounded in-kernel wait ran out; results invalid   */
#define SAPO_ST_NONFINITE_REWARD 0x40  /* a reward is NaN or infinite                         */
#define SAPO_ST_EXP_RANGE        0x80  /* fused call: old_logp[t] is so far from the current
                                          log-prob that exp(z - c_t) left the safe range; the
                                          token is scored as masked: use the separate calls   */
#define SAPO_ST_NONFINITE_INPUT  0x100 /* old_logp[t] or the advantage of its sequence is NaN or
                                          infinite: the token is scored as masked               */

/* element types of hidden / W_head */
#define SAPO_DTYPE_BF16 0
#define SAPO_DTYPE_F32  1  /* converted on the device to split bf16; see sapo_policy_loss_fwd */

/* kinds of norm */
#define SAPO_NORM_LAYER 0
#define SAPO_NORM_RMS   1

/* kinds of preference loss, and which pairs of a question enter it */
#define SAPO_PREF_SIGMOID 0
#define SAPO_PREF_SQUARED 1
#define SAPO_PREF_HINGE   2
#define SAPO_PREF_ALL        0
#define SAPO_PREF_BEST_WORST 1

/* `which` of sapo_workspace_bytes */
#define SAPO_WS_FWD 0
#define SAPO_WS_BWD 1
#define SAPO_WS_BWD_ACTIVE 2
#define SAPO_WS_FUSED 3
#define SAPO_WS_PREFERENCE 4     /* sapo_preference_loss_fwd_bwd */
#define SAPO_WS_OUT_BF16 0x100   /* OR into `which`: the gradients will be asked for in bf16 */
#define SAPO_WS_GATHER   0x200   /* OR into `which`: for sapo_policy_loss_fwd_bwd_gather          */

/* A rollout store: n_rollouts completions laid end to end (Section 3.1: a node's answers
 * to its questions; Section 3.2: the tuples other nodes broadcast).
 *   hidden   [n_tokens, H]  final hidden state at the position that predicts ids[t]
 *   ids      [n_tokens]     chosen token
 *   old_logp [n_tokens]     log-prob of ids[t] under the pre-update policy
 *   offsets  [n_rollouts+1] token offset of each completion (offsets[0] = 0)
 *   rewards  [n_rollouts]   reward of each completion */
typedef struct sapo_rollout_buf {
  const void*    hidden;
  const int32_t* ids;
  const float*   old_logp;
  const int64_t* offsets;
  const float*   rewards;
  int32_t        n_rollouts;
} sapo_rollout_buf;

/* Which rollouts enter the training set: for question q the local picks are
 * local_idx[q_offsets_local[q] .. q_offsets_local[q+1]) and the external picks
 * ext_idx[q_offsets_ext[q] .. q_offsets_ext[q+1]).  Either side may be empty. */
typedef struct sapo_selection {
  const int32_t* q_offsets_local;  /* [Q+1] */
  const int32_t* local_idx;
  const int32_t* q_offsets_ext;    /* [Q+1] */
  const int32_t* ext_idx;
  int32_t        Q;
} sapo_selection;

/* Output of sapo_pack_rollouts.  Capacities max_tokens / max_seqs are set by the caller.
 *   hidden [max_tokens, H], ids, old_logp [max_tokens], rewards [max_seqs]
 *   cu_seqlens [max_seqs+1] exclusive prefix sum of sequence lengths
 *   seq_group [max_seqs] question of each sequence;  seq_is_ext [max_seqs] 0 local / 1 external
 *   seq_src [max_seqs] index of the rollout inside its buffer
 *   tok_seq [max_tokens] sequence of each token;  tok_mask [max_tokens] 1 for t < T else 0
 *   group_offsets [Q+1] first sequence of each question
 *   n_tokens, n_seqs: device scalars T and S
 *   tok_src [max_tokens] (optional, may be NULL): where each packed token's row lives in its source
 *     buffer: row index, plus 2^62 when it is the external buffer; -1 for unused slots.  With it the
 *     loss can read the hidden states in place (sapo_policy_loss_fwd_bwd_gather) and `hidden` may
 *     be NULL: the pack then copies no hidden rows at all. */
typedef struct sapo_packed {
  void*    hidden;
  int32_t* ids;
  float*   old_logp;
  float*   rewards;
  int32_t* cu_seqlens;
  int32_t* seq_group;
  uint8_t* seq_is_ext;
  int32_t* seq_src;
  int32_t* tok_seq;
  uint8_t* tok_mask;
  int32_t* group_offsets;
  int32_t* n_tokens;
  int32_t* n_seqs;
  int64_t  max_tokens;
  int32_t  max_seqs;
  int64_t* tok_src;
} sapo_packed;

/* Loss parameters.  The paper's run uses eps_low 0.2, eps_high 0.28 and no KL term
 * (Section 4.2).  grad_scale multiplies the per-token gradient factor (upstream dL).
 * loss_agg: 0 = mean over sequences of the token mean (the default reading), 1 = mean over all
 * tokens (the aggregation of DAPO, which Section 4.2 cites).  kl_beta: weight of a penalty
 * towards a reference policy, per token exp(d) - d - 1 with d = ref_logp[t] - logp[t], aggregated
 * like the surrogate; 0 (the paper's choice) leaves ref_logp unused.  ref_logp: device pointer,
 * [T], may be NULL when kl_beta is 0.  entropy: device pointer [T] or NULL; when given, the forward
 * also writes the entropy of the policy's next-token distribution at every scored position,
 * H_t = - sum_v p[t,v] log p[t,v] (nats), a by-product of the same pass over the logits that RL
 * runs log beside the reward; it does not enter the loss.  Tokens that belong to no sequence get 0. */
typedef struct sapo_loss_cfg {
  float eps_low;
  float eps_high;
  float grad_scale;
  int32_t loss_agg;
  float kl_beta;
  const float* ref_logp;
  float* entropy;
} sapo_loss_cfg;

/* Section 3.2, training-set equation / Algorithm 1, where the training set is put together.
 * Gathers the selected rollouts into one token-major batch.  Sequence order: questions in
 * order; inside a question its local picks in list order, then its external picks in list
 * order.  Copies are byte-exact.  H is the row width in elements, `dtype` a SAPO_DTYPE_*.
 * Slots [T, max_tokens) of hidden, ids and old_logp are zero-filled (tok_mask 0, tok_seq -1),
 * so a caller that must not read n_tokens back can score the whole capacity: the loss calls
 * treat tokens that belong to no sequence as masked.
 * Errors: a NULL struct, a NULL array that the sizes say will be touched (outputs when the
 * capacities are positive, the members of a rollout buffer that holds rollouts; the index lists
 * may be NULL when empty) or a negative size returns SAPO_ERR_INVALID_ARG before anything is
 * launched; a bad index, an empty rollout or a capacity overflow sets the matching status bit
 * (bad or empty picks are packed as length-0 sequences, tokens beyond max_tokens are dropped). */
int sapo_pack_rollouts(const sapo_rollout_buf* h_local, const sapo_rollout_buf* h_ext,
                       const sapo_selection* h_sel, int32_t H, int32_t dtype,
                       const sapo_packed* h_out, int32_t* status, void* stream);

/* Section 4.2 (GRPO): for each question g with members group_offsets[g]..group_offsets[g+1):
 *   mean_g = average reward, std_g = sqrt(sum (r-mean_g)^2 / (G - ddof)),
 *   adv[s] = (rewards[s] - mean_g) / (std_g + adv_eps).
 * The group covers all its completions, local and external alike.  fp32 in, fp32 out; the sums
 * carry their rounding errors along (compensated fp32), so an advantage is within 6 fp32 ulp of
 * the exactly computed value for groups of up to 16 rewards whatever their common offset, and an
 * all-equal group gives exactly 0.  mean / std may be NULL.  A non-finite reward sets
 * SAPO_ST_NONFINITE_REWARD.  Up to 4095 questions run on the warp-level kernel (two lanes per
 * question, a 16-byte vector of rewards each), more on a thread-per-question kernel; sapo_group_advantages_warp always takes the
 * warp-level one (same arguments and results; it exists so that kernel can be measured alone). */
int sapo_group_advantages(const float* rewards, const int32_t* group_offsets, int32_t Q,
                          float adv_eps, int32_t ddof, float* adv, float* mean, float* std,
                          int32_t* status, void* stream);
int sapo_group_advantages_warp(const float* rewards, const int32_t* group_offsets, int32_t Q,
                               float adv_eps, int32_t ddof, float* adv, float* mean, float* std,
                               int32_t* status, void* stream);

/* Section 3.2 (token-level values under the node's own policy) + Section 4.2 (clipped
 * surrogate, KL weight 0).  For T packed tokens in S sequences:
 *   z[t,v] = <hidden[t,:], W_head[v,:]>,  lse[t] = log sum_v exp z[t,v],
 *   logp[t] = z[t, ids[t]] - lse[t],      ratio[t] = exp(logp[t] - old_logp[t]),
 *   surr[t] = min(ratio*A, clip(ratio, 1-eps_low, 1+eps_high)*A),  A = adv[seq of t],
 *   loss    = -(1/S) sum_s (1/T_s) sum_{t in s} surr[t]   (variants: see sapo_loss_cfg),
 *   gscale[t] = dloss/dlogp[t] = -grad_scale * A * ratio / (S*T_s) where the unclipped term
 *               is the min (ties included), else 0.
 * The [T,V] logits are never written to memory: the projection runs on the tensor cores and
 * its epilogue keeps a running max / sum-exp / target logit per token.
 * hidden [T, ld_hidden], W_head [V, ld_W] of `dtype`; for SAPO_DTYPE_F32 the operands are
 * split on the device into bf16 high and low parts (3 products), which keeps log-probs at
 * fp32 accuracy.  adv [S], cu_seqlens [S+1].  Outputs logp, lse, ratio, surr, gscale [T]
 * and loss [1] (float32); seq_surr [S] (token-mean surrogate per sequence) may be NULL.
 * cu_seqlens must be non-decreasing with every entry in [0, T]; normally cu_seqlens[0] = 0 and
 * cu_seqlens[S] = T, but T may also be the capacity of the buffers (sapo_pack_rollouts leaves the
 * token count on the device): tokens of [0, T) before cu_seqlens[0] or from cu_seqlens[S] on
 * belong to no sequence and are scored as masked (all five per-token outputs 0, no gradient).
 * Their hidden rows are still read by the projection and must hold finite numbers
 * (sapo_pack_rollouts zero-fills them).  An entry of cu_seqlens outside [0, T] or below its
 * predecessor is clamped and sets SAPO_ST_BAD_INDEX.  A NaN or infinite old_logp[t] or adv[s]
 * sets SAPO_ST_NONFINITE_INPUT and masks the token(s) (ratio = surr = gscale = 0).
 * workspace: at least sapo_workspace_bytes(SAPO_WS_FWD, ...) bytes.
 * Errors: bad arguments / unaligned pointers -> SAPO_ERR_INVALID_ARG; H or V beyond the
 * supported range -> SAPO_ERR_UNSUPPORTED_SHAPE; small workspace ->
 * SAPO_ERR_WORKSPACE_TOO_SMALL; ids outside [0,V) -> SAPO_ST_BAD_TOKEN_ID and the token
 * gets logp = 0 contribution (surr = gscale = 0). */
int sapo_policy_loss_fwd(const void* hidden, const void* W_head, int32_t dtype,
                         int64_t T, int32_t H, int32_t V, int64_t ld_hidden, int64_t ld_W,
                         const int32_t* ids, const float* old_logp, const float* adv,
                         const int32_t* cu_seqlens, int32_t S, const sapo_loss_cfg* h_cfg,
                         float* logp, float* lse, float* ratio, float* surr, float* gscale,
                         float* seq_surr, float* loss,
                         void* workspace, size_t workspace_bytes,
                         int32_t* status, void* stream);

/* Algorithm 1 "Policy update" (gradient of the loss above through the LM head):
 *   dz[t,v]      = gscale[t] * ([v == ids[t]] - exp(z[t,v] - lse[t]))
 *   dhidden[t,:] = sum_v dz[t,v] W_head[v,:]        [T, H] of out_dtype
 *   dW_head[v,:] = sum_t dz[t,v] hidden[t,:]        [V, H] of out_dtype
 * Logit tiles are recomputed on the tensor cores; dz is rounded to bf16 and kept in a
 * bounded panel inside `workspace` (token chunks x vocab padded to 128, stored as 16 KB tiles
 * of 128 tokens x 64 vocab entries), from which two tensor-core contractions form dhidden and
 * dW_head.  accumulate_dW != 0 adds into dW_head instead of
 * overwriting it.  lse and gscale come from sapo_policy_loss_fwd.  For SAPO_DTYPE_F32 the
 * operands are rounded to bf16.
 * out_dtype: SAPO_DTYPE_F32, or SAPO_DTYPE_BF16 for gradients that feed a bf16 backward pass and
 * optimiser: contiguous [T, H] / [V, H] of that type, 16-byte aligned; sums are always formed in
 * fp32 and rounded once (when the panel holds fewer than T tokens, or accumulate_dW is set,
 * dW_head is summed in an fp32 copy inside `workspace` and rounded, or added to the caller's
 * values and rounded, at the end: ask sapo_workspace_bytes for SAPO_WS_BWD | SAPO_WS_OUT_BF16).
 * workspace: sapo_workspace_bytes(SAPO_WS_BWD, ...) is the preferred size; any size down to
 * the one for 128 tokens works (smaller panels mean more passes over dW_head). */
int sapo_policy_loss_bwd(const void* hidden, const void* W_head, int32_t dtype,
                         int64_t T, int32_t H, int32_t V, int64_t ld_hidden, int64_t ld_W,
                         const int32_t* ids, const float* lse, const float* gscale,
                         void* dhidden, void* dW_head, int32_t out_dtype, int32_t accumulate_dW,
                         void* workspace, size_t workspace_bytes,
                         int32_t* status, void* stream);

/* The loss over a vocabulary that is sharded across ranks (no counterpart in the paper, whose
 * nodes each hold a whole model; it lets one node's LM head span several GPUs).  Rank r holds
 * W_shard = rows [vocab_offset, vocab_offset + V_shard) of W_head and every token's hidden state.
 *   1. sapo_lmhead_lse_partial: the projection of the shard on the tensor cores, reduced per token
 *      to triple[0][t] = max_v z log2(e), triple[1][t] = sum_v 2^(z log2(e) - max), triple[2][t] =
 *      z[t, ids[t]] if the chosen token lies in the shard, else 0   (float32 [3][T]).
 *      workspace: sapo_workspace_bytes(SAPO_WS_FWD, T, H, V_shard, dtype).
 *   2. the caller gathers the triples of all ranks into local memory, [n_parts][3][T] (one
 *      all-gather of 12 T bytes per rank);
 *   3. sapo_policy_loss_from_partials: merges them (log-sum-exp over the parts) and evaluates the
 *      loss tail exactly as sapo_policy_loss_fwd does; every rank computes the same values.
 *      ids are the global token ids, V the whole vocabulary.  h_cfg->entropy must be NULL.
 *   4. sapo_policy_loss_bwd_shard: sapo_policy_loss_bwd on the shard with the global lse:
 *      dW_shard [V_shard, H] is this rank's rows of dW_head; dhidden is this shard's share of
 *      the sum over the vocabulary, to be added up over the ranks (one all-reduce of T H values).
 * The library itself moves nothing between GPUs; a kernel only ever reads local memory. */
int sapo_lmhead_lse_partial(const void* hidden, const void* W_shard, int32_t dtype,
                            int64_t T, int32_t H, int32_t V_shard, int64_t ld_hidden, int64_t ld_W,
                            const int32_t* ids, int32_t vocab_offset, float* triple,
                            void* workspace, size_t workspace_bytes, int32_t* status, void* stream);
int sapo_policy_loss_from_partials(const float* triples, int32_t n_parts, int64_t T, int32_t V,
                                   const int32_t* ids, const float* old_logp, const float* adv,
                                   const int32_t* cu_seqlens, int32_t S, const sapo_loss_cfg* h_cfg,
                                   float* logp, float* lse, float* ratio, float* surr, float* gscale,
                                   float* seq_surr, float* loss, int32_t* status, void* stream);
int sapo_policy_loss_bwd_shard(const void* hidden, const void* W_shard, int32_t dtype,
                               int64_t T, int32_t H, int32_t V_shard, int64_t ld_hidden, int64_t ld_W,
                               const int32_t* ids, int32_t vocab_offset, const float* lse,
                               const float* gscale, void* dhidden, void* dW_shard, int32_t out_dtype,
                               int32_t accumulate_dW, void* workspace, size_t workspace_bytes,
                               int32_t* status, void* stream);

/* The same gradient, computed over the active tokens only (gscale[t] != 0).  Sequences of a
 * zero-advantage group — which the paper's experiments drop from the shared pool as
 * uninformative (Section 5) — and tokens clipped on the binding side have gscale = 0 and add
 * nothing to either gradient; this call compacts them away first (order kept), gathers the
 * hidden rows of the rest, runs the three contractions on those rows and writes dhidden rows
 * back to their token positions (inactive rows are zero).  The active count is read on the
 * device by the kernels, so the call does not synchronise; if n_active_out (device int32) is not
 * NULL the count is also copied there.  Results equal sapo_policy_loss_bwd up to fp32 summation
 * order.  workspace: sapo_workspace_bytes(SAPO_WS_BWD_ACTIVE, ...) (the regular backward's plus
 * a compacted copy of hidden and four per-token vectors). */
int sapo_policy_loss_bwd_active(const void* hidden, const void* W_head, int32_t dtype,
                                int64_t T, int32_t H, int32_t V, int64_t ld_hidden, int64_t ld_W,
                                const int32_t* ids, const float* lse, const float* gscale,
                                void* dhidden, void* dW_head, int32_t out_dtype, int32_t accumulate_dW,
                                int32_t* n_active_out,
                                void* workspace, size_t workspace_bytes,
                                int32_t* status, void* stream);

/* Loss (Section 3.2 + Section 4.2) and both gradients (Algorithm 1 "Policy update") in ONE call
 * that passes over the logits once.  Same definitions and outputs as sapo_policy_loss_fwd followed
 * by sapo_policy_loss_bwd; what changes is how the softmax is carried from the forward to the
 * backward contraction.  With a per-token reference
 *   c_t = z[t, ids[t]] - old_logp[t]          (one dot product per token, computed first)
 * — equal to lse[t] if the policy has not moved since old_logp was taken, and off by
 * log ratio[t] otherwise — the forward epilogue forms e[t,v] = exp(z[t,v] - c_t), adds it up per
 * token in fp32 (lse[t] = c_t + log sum_v e[t,v]; no running maximum is needed) and keeps e,
 * rounded to bf16, in a panel inside `workspace` (token chunks x vocab padded to 128, 16 KB tiles
 * of 128 tokens x 64 vocab entries).  Then, with sum_t = sum_v e[t,v] and a_t = -gscale[t] / sum_t,
 *   dz[t,v] = gscale[t] ([v == ids[t]] - e[t,v] / sum_t) = a_t e'[t,v],  e' = e - [v == ids[t]] sum_t,
 * so after patching one panel entry per token
 *   dhidden[t,:] = a_t sum_v e'[t,v] W_head[v,:]     (row scale in the epilogue)
 *   dW_head[v,:] = sum_t e'[t,v] (a_t hidden[t,:])   (scaled bf16 copy of hidden as operand)
 * are two tensor-core contractions over the panel: 6 T V H flops instead of the 8 T V H of the
 * separate calls, which recompute the logits.  The price is the range of e: if old_logp[t] is so
 * stale that |log ratio| approaches 69 (the sum of e reaches 2^100 or drops below 2^-100), the token
 * is scored as masked (surr = gscale = 0) and SAPO_ST_EXP_RANGE is set; such batches need the
 * separate calls.  bf16 operands only (SAPO_DTYPE_F32 returns SAPO_ERR_UNSUPPORTED_SHAPE).
 * Arguments as in the two separate calls.  workspace: sapo_workspace_bytes(SAPO_WS_FUSED, ...)
 * is the preferred size (a panel of up to 32768 tokens); any size down to
 * sapo_workspace_bytes_min(SAPO_WS_FUSED, ...) works, the batch is then processed in token
 * chunks and dW_head accumulated over them.  seq_surr may be NULL (then S <= T is required). */
int sapo_policy_loss_fwd_bwd(const void* hidden, const void* W_head, int32_t dtype,
                             int64_t T, int32_t H, int32_t V, int64_t ld_hidden, int64_t ld_W,
                             const int32_t* ids, const float* old_logp, const float* adv,
                             const int32_t* cu_seqlens, int32_t S, const sapo_loss_cfg* h_cfg,
                             float* logp, float* lse, float* ratio, float* surr, float* gscale,
                             float* seq_surr, float* loss,
                             void* dhidden, void* dW_head, int32_t out_dtype, int32_t accumulate_dW,
                             void* workspace, size_t workspace_bytes,
                             int32_t* status, void* stream);

/* sapo_policy_loss_fwd_bwd with the hidden states read in place.  The training set is a union of
 * index picks (Section 3.2, training-set equation), so it need not be copied: every packed token
 * names its row in the local or the external rollout store (tok_src, written by
 * sapo_pack_rollouts, which then copies no hidden rows when its `hidden` output is NULL), the
 * projection's row loads follow the runs of consecutive rows that whole sequences form, and the
 * per-token kernels read their row through the same map.  local_hidden [n_local_tokens, ld_hidden],
 * ext_hidden [n_ext_tokens, ld_hidden] (bf16, the same row pitch, 16-byte aligned; fewer than 2^31
 * rows each); everything else, results included, as in sapo_policy_loss_fwd_bwd.  A packed slot
 * without a token (tok_src -1) is scored as masked; a tok_src that points outside its store sets
 * SAPO_ST_BAD_INDEX.  workspace: sapo_workspace_bytes(SAPO_WS_FUSED | SAPO_WS_GATHER, ...). */
int sapo_policy_loss_fwd_bwd_gather(const void* local_hidden, int64_t n_local_tokens,
                                    const void* ext_hidden, int64_t n_ext_tokens, const int64_t* tok_src,
                                    const void* W_head, int32_t dtype,
                                    int64_t T, int32_t H, int32_t V, int64_t ld_hidden, int64_t ld_W,
                                    const int32_t* ids, const float* old_logp, const float* adv,
                                    const int32_t* cu_seqlens, int32_t S, const sapo_loss_cfg* h_cfg,
                                    float* logp, float* lse, float* ratio, float* surr, float* gscale,
                                    float* seq_surr, float* loss,
                                    void* dhidden, void* dW_head, int32_t out_dtype, int32_t accumulate_dW,
                                    void* workspace, size_t workspace_bytes,
                                    int32_t* status, void* stream);

/* Section 3.2 (nodes filter and sample what the swarm shares) / Section 5 (the experiments'
 * policy: discard rollouts with zero advantage, then sample uniformly from the rest).
 * The pool holds n_entries rollouts; entry g is a question's group of completions with rewards
 * rewards[group_offsets[g] .. group_offsets[g+1]).  An entry whose rewards are all equal has zero
 * advantage throughout and is dropped; of the others, J are drawn uniformly without replacement
 * (all of them if there are fewer than J): entry g gets the key
 * (philox4x32-10(counter = (g,0,0,0), key = (seed low, seed high))[0] << 32) | g and the J
 * smallest keys win, so the draw depends only on the seed and the pool.  selected [J] receives
 * the chosen entries in pool order, *n_selected how many there are, *n_candidates how many passed
 * the filter (all device memory).  workspace: sapo_select_workspace_bytes(n_entries), 8-byte
 * aligned. */
int sapo_select_external(const float* rewards, const int32_t* group_offsets, int32_t n_entries,
                         int32_t J, uint64_t seed, int32_t* selected, int32_t* n_selected,
                         int32_t* n_candidates, void* workspace, size_t workspace_bytes, void* stream);
size_t sapo_select_workspace_bytes(int32_t n_entries);

/* Parameters of the preference loss.  beta > 0; label_smoothing in [0, 0.5), sigmoid kind only;
 * grad_scale multiplies the gradient (upstream dL); kind SAPO_PREF_SIGMOID / _SQUARED / _HINGE;
 * pairs SAPO_PREF_ALL / _BEST_WORST; length_norm 1: R_s is the mean over the tokens of s. */
typedef struct sapo_pref_cfg {
  float beta;
  float label_smoothing;
  float grad_scale;
  int32_t kind;
  int32_t pairs;
  int32_t length_norm;
} sapo_pref_cfg;

/* A preference loss over the completions of a question (no counterpart in the paper, whose update is
 * the clipped policy loss above): the rewards only order the completions of a question.
 *   R_s  = sum_{t in s} (logp[t] - ref_logp[t])       (length_norm: divided by T_s)
 *   h_ij = beta (R_i - R_j) for every pair of one question with rewards[i] > rewards[j]
 *          (SAPO_PREF_ALL), or for its best against its worst completion only, the first of each
 *          in packed order where rewards tie (SAPO_PREF_BEST_WORST)
 *   l    = (1-e) softplus(-h) + e softplus(h), e = label_smoothing     (SAPO_PREF_SIGMOID)
 *          (R_i - R_j - 1/(2 beta))^2                                  (SAPO_PREF_SQUARED)
 *          max(0, 1 - h)                                               (SAPO_PREF_HINGE)
 *   q_loss[q] = mean of l over the pairs of question q (0 if it has none), loss = (1/Q) sum_q q_loss[q]
 *   seq_grad[s] = grad_scale dloss/dR_s,  gscale[t] = grad_scale dloss/dlogp[t]
 *   q_margin[q] = mean of h over the pairs, q_pairs[q] their number (each may be NULL)
 * gscale is what sapo_policy_loss_bwd takes, so that call turns it into dhidden and dW_head.
 * cu_seqlens [S+1] and group_offsets [Q+1] (first sequence of each question) as sapo_pack_rollouts
 * writes them, rewards [S]; all sums in fp32 or wider and in a fixed order (the same inputs give the
 * same bits).  A completion without tokens or with a reward that is not finite
 * (SAPO_ST_NONFINITE_REWARD) joins no pair; a pair whose h left the fp32 range is left out.  A token whose logp or
 * ref_logp is not finite (SAPO_ST_NONFINITE_INPUT) is left out of its sum and gets gscale 0.  Tokens
 * and sequences that belong to no question get zeros.  Offsets outside their range or below their
 * predecessor are clamped (SAPO_ST_BAD_INDEX).  T may be 0; Q, S >= 1. */
int sapo_preference_loss(const float* logp, const float* ref_logp, int64_t T, const int32_t* cu_seqlens,
                         int32_t S, const float* rewards, const int32_t* group_offsets, int32_t Q,
                         const sapo_pref_cfg* h_cfg, float* gscale, float* seq_logratio, float* seq_grad,
                         float* q_loss, float* q_margin, int32_t* q_pairs, float* loss,
                         int32_t* status, void* stream);

/* The preference loss through the LM head: log-probs of the chosen tokens under (hidden, W_head) as
 * in sapo_policy_loss_fwd, the loss above on them, and its gradients dhidden and dW_head as in
 * sapo_policy_loss_bwd (arguments, alignment, out_dtype and accumulate_dW as there; bf16 operands only,
 * SAPO_ERR_UNSUPPORTED_SHAPE for fp32: those go through sapo_policy_loss_fwd, sapo_preference_loss and
 * sapo_policy_loss_bwd).
 * logp, lse, gscale [T]; a token with an id outside [0, V) gets logp 0 (SAPO_ST_BAD_TOKEN_ID), is left
 * out of its sequence's sum and gets no gradient.  The same holds for a token whose log ratio is beyond
 * +-69 (SAPO_ST_EXP_RANGE): its exponentials are taken relative to exp(ref_logp).
 * lse and logp are not sapo_policy_loss_fwd's to the bit: here a part of what the tensor cores truncate from a logit is put
 * back (they add in fp32 rounded towards zero; lse is short by about 1e-9 H E_p[z] without it, and a sequence sums that),
 * and a log ratio is formed without the rounding of its lse.
 * workspace: sapo_workspace_bytes(SAPO_WS_PREFERENCE, ...), at least sapo_workspace_bytes_min of it.  With a workspace
 * whose panel holds the whole batch (what the first returns up to 40960 tokens: 2 (V + H) bytes a token and a little,
 * 13.8 GB at 40960 tokens, V 151936, H 1536 with bf16 gradients) the call takes 6 T V H flops, with a smaller one
 * 8 T V H: a pair's factor is known only when both its sequences have been scored.
 * Precision of the gradients: the tensor cores take bf16 operands and add in fp32.  In one pass the exponentials and the
 * rows g_t hidden_t / sum_t are rounded to bf16, in two passes the entries of dz.  Error against 64 bits, of the norm
 * (T 2048, V 20000, H 896): fp32 gradients 4e-5 (dhidden) and 1.7e-3 (dW_head) in one pass, 1.2e-3 (both) in two; bf16
 * gradients 1.7e-3 and 2.3e-3 in one pass, 2.0e-3 in two, where the exact ones rounded to bf16 are off by 1.7e-3. */
int sapo_preference_loss_fwd_bwd(const void* hidden, const void* W_head, int32_t dtype,
                                 int64_t T, int32_t H, int32_t V, int64_t ld_hidden, int64_t ld_W,
                                 const int32_t* ids, const float* ref_logp, const int32_t* cu_seqlens, int32_t S,
                                 const float* rewards, const int32_t* group_offsets, int32_t Q,
                                 const sapo_pref_cfg* h_cfg, float* logp, float* lse, float* gscale,
                                 float* seq_logratio, float* seq_grad, float* q_loss, float* q_margin,
                                 int32_t* q_pairs, float* loss,
                                 void* dhidden, void* dW_head, int32_t out_dtype, int32_t accumulate_dW,
                                 void* workspace, size_t workspace_bytes, int32_t* status, void* stream);

/* An activation [T, H] kept in 8 bits: data [T, ld], and one fp32 scale per row and group of 128
 * columns, scale [T, ld_scale] with ld_scale >= ceil(H / 128).  Element (t, c) stands for
 * data[t, c] * scale[t, c / 128].  Storing takes a = max |x| of the group, scale = a (1/127) and
 * data = rint(x (127 (1/a))), each product and quotient rounded to fp32, so a value is off by at
 * most a / 254 and a little rounding; a group with a below 2^-119 is stored as zeros.  A group that holds a NaN or an infinity is stored
 * with scale NaN (SAPO_ST_NONFINITE_INPUT): all its values read back as NaN. */
typedef struct sapo_ckpt8 {
  int8_t* data;
  float*  scale;
  int64_t ld, ld_scale;
} sapo_ckpt8;

/* x [T, ld_x] to a checkpoint and back.  x_dtype: SAPO_DTYPE_BF16 or SAPO_DTYPE_F32.  For these
 * calls and the norms below H is in [1, 16384] (SAPO_ERR_UNSUPPORTED_SHAPE beyond) and T may be 0.  Any H and any leading
 * dimension from H up will do; rows that start on 16-byte boundaries (8 for the 8-bit data) are read
 * and written in vectors, others element by element. */
int sapo_ckpt8_store(const void* x, int32_t x_dtype, int64_t T, int32_t H, int64_t ld_x,
                     const sapo_ckpt8* h_out, int32_t* status, void* stream);
int sapo_ckpt8_restore(const sapo_ckpt8* h_in, int64_t T, int32_t H, void* x, int32_t x_dtype, int64_t ld_x,
                       void* stream);

/* kind SAPO_NORM_LAYER or SAPO_NORM_RMS; eps >= 0 is added to the variance (mean square); w_dtype:
 * element type of gamma and beta. */
typedef struct sapo_norm_cfg {
  int32_t kind;
  float   eps;
  int32_t w_dtype;
} sapo_norm_cfg;

/* The norm in front of the LM head (no counterpart in the paper; hidden of the loss calls is its
 * output), row by row over H columns:
 *   layer: mean = (1/H) sum x, rstd = ((1/H) sum (x - mean)^2 + eps)^-1/2;  rms: mean = 0
 *   xh = (x - mean) rstd,  y = xh gamma + beta          (gamma NULL: ones, beta NULL: zeros)
 * x [T, ld_x] and y [T, ld_y] of x_dtype / y_dtype (bf16 or fp32, any mix); statistics in fp32 from
 * one read of x.  mean (layer) and rstd [T] are what the backward wants; each may be NULL.  h_ckpt
 * (may be NULL; `status` is then not used): x is also stored as an 8-bit checkpoint, in the same pass.  y may be x. */
int sapo_norm_fwd(const void* x, int32_t x_dtype, int64_t T, int32_t H, int64_t ld_x,
                  const void* gamma, const void* beta, const sapo_norm_cfg* h_cfg,
                  void* y, int32_t y_dtype, int64_t ld_y, float* mean, float* rstd,
                  const sapo_ckpt8* h_ckpt, int32_t* status, void* stream);

/* y again, from the checkpoint and the statistics that the forward stored (cfg.eps is not used): for
 * a backward that wants hidden after its memory has been given up. */
int sapo_norm_replay(const sapo_ckpt8* h_x, int64_t T, int32_t H, const void* gamma, const void* beta,
                     const sapo_norm_cfg* h_cfg, const float* mean, const float* rstd,
                     void* y, int32_t y_dtype, int64_t ld_y, void* stream);

/* Gradient of sapo_norm_fwd: with g = dy gamma,
 *   dx = rstd (g - [layer] mean_c(g) - xh mean_c(g xh)),  dgamma = sum_t dy xh,  dbeta = sum_t dy.
 * Exactly one of x (the forward's input) and h_ckpt (its 8-bit checkpoint, read in place) is given; mean (layer) and rstd
 * come from the forward.  dy, x, dx each bf16 or fp32; dx may be dy.  dgamma and dbeta (fp32 [H],
 * either may be NULL) are overwritten, or added to with accumulate != 0; their sums over the rows are
 * formed in fp32 in a fixed order.  workspace: sapo_norm_workspace_bytes(T, H), not needed when both
 * are NULL. */
int sapo_norm_bwd(const void* dy, int32_t dy_dtype, int64_t ld_dy,
                  const void* x, int32_t x_dtype, int64_t ld_x, const sapo_ckpt8* h_ckpt,
                  int64_t T, int32_t H, const void* gamma, const sapo_norm_cfg* h_cfg,
                  const float* mean, const float* rstd, void* dx, int32_t dx_dtype, int64_t ld_dx,
                  float* dgamma, float* dbeta, int32_t accumulate,
                  void* workspace, size_t workspace_bytes, void* stream);
size_t sapo_norm_workspace_bytes(int64_t T, int32_t H);

/* Section 4.2: the policy is updated with Adam (default hyper-parameters, learning rate 0.001).
 * One Adam step (Kingma & Ba, Algorithm 1) on a [rows, cols] weight such as W_head, from the
 * fp32 gradient sapo_policy_loss_bwd wrote:
 *   m <- beta1 m + (1-beta1) g;  v <- beta2 v + (1-beta2) g^2;
 *   master <- master - lr * (m / (1-beta1^step)) / (sqrt(v / (1-beta2^step)) + eps).
 * master, m, v, grad: fp32 [rows, cols], contiguous, 16-byte aligned, updated in place (grad is
 * only read).  w_bf16 (may be NULL): bf16 [rows, ld_w] copy of the new master weight, rounded to
 * nearest even — the operand the next forward reads.  step counts from 1.  cols % 4 == 0. */
int sapo_adam_step(float* master, float* m, float* v, const float* grad, void* w_bf16,
                   int64_t rows, int32_t cols, int64_t ld_w, int32_t step,
                   float lr, float beta1, float beta2, float eps, void* stream);

/* AdamW over a list of tensors (Loshchilov & Hutter; no counterpart in the paper, whose run is plain
 * Adam: sapo_adam_step).  Per element, with g = grad (* *grad_scale), lr_i = lr lr_factor:
 *   m <- beta1 m + (1-beta1) g;  v <- beta2 v + (1-beta2) g g;
 *   master <- master (1 - lr_i weight_decay) - lr_i (m / (1-beta1^step)) / (sqrt(v / (1-beta2^step)) + eps)
 * and copy_bf16 (may be NULL) = master rounded to bf16.  An element whose g is not finite is left as it
 * was (SAPO_ST_NONFINITE_INPUT; 8-bit moments are rounded anew with their group); v stops at the largest fp32.
 * A tensor has n elements in one run of memory, of any n (0 too) and any alignment of its element type;
 * arrays on 16-byte boundaries are faster.  The _out arrays receive the new values: the same pointers as
 * the old ones for a step in place, or other arrays (the weights of the policy before the step stay).
 * state_bits 32: m, v are fp32.  state_bits 8: m and v are e4m3 codes [n] with an fp32 scale per 128
 * elements, [ceil(n / 128)]: m = code * m_scale, and the SECOND array holds the root: sqrt(v) = code *
 * v_scale.  The step itself uses the new m and v before they are rounded.  With a the largest magnitude of
 * a group, scale = a (1/448) (0, and codes 0, if a < 2^-119); m (448 (1/a)) is rounded to the nearest code.  For the
 * root, t = max(sqrt(v) (448 (1/a)), 2^-6) (0 if v is 0) is rounded up or down to a code so that it is right on average: of
 * the bits of t as fp32 those of weight below 2^20 are cut off after 16 r + 8 has been added, r being 16 random
 * bits; element i of tensor `number` in the list takes half i % 8 (low half of a word first) of
 * philox4x32-10(counter = (i / 8 low, i / 8 high, number, step), key = (seed low, seed high)).  Each product and sum of
 * the state is rounded to fp32 by itself, so that the state is defined to the bit (but for a last bit of about one root
 * in 10^5; the root of a v below the normal numbers is 0).  Zeroed codes and scales are a fresh state. */
typedef struct sapo_adamw_tensor {
  const float* master;
  float*       master_out;
  const void*  grad;          /* grad_dtype */
  const void*  m;
  const void*  v;
  void*        m_out;
  void*        v_out;
  const float* m_scale;       /* state_bits 8 only */
  const float* v_scale;
  float*       m_scale_out;
  float*       v_scale_out;
  void*        copy_bf16;
  int64_t      n;
  float        lr_factor;
  float        weight_decay;
  int32_t      grad_dtype;
  int32_t      state_bits;
} sapo_adamw_tensor;

/* step counts from 1.  lr_dev, step_dev (each may be NULL): device memory that is read instead of lr and
 * step, so that a captured call follows a schedule.  grad_scale (may be NULL): one float in device memory, e.g. the
 * factor of a clipped gradient norm. */
typedef struct sapo_adamw_cfg {
  double   lr, beta1, beta2, eps;
  uint64_t seed;
  int32_t  step;
  const int32_t* step_dev;
  const float*   lr_dev;
  const float*   grad_scale;
} sapo_adamw_cfg;

int sapo_adamw_step(const sapo_adamw_tensor* h_tensors, int32_t n_tensors, const sapo_adamw_cfg* h_cfg,
                    int32_t* status, void* stream);

/* A matrix [R, C] in 8-bit floating point: e4m3 codes data [R, ld], and one fp32 scale per row and 128
 * columns (blocks 0: scale [R, ld_scale]) or per block of 128 rows and 128 columns (blocks 1: scale
 * [ceil(R / 128), ld_scale]), ld_scale >= ceil(C / 128).  An element stands for code * scale. */
typedef struct sapo_fp8 {
  void*   data;
  float*  scale;
  int64_t ld, ld_scale;
  int32_t blocks;
} sapo_fp8;

/* x [R, ld_x] (bf16 or fp32) into 8 bits: a = the largest |x| of a group, scale = a (1/448), code = x (448 (1/a)) rounded
 * to the nearest, each product and quotient rounded to fp32 (a below 2^-119: scale and codes 0).  A group that holds a NaN or an infinity gets scale NaN and
 * codes 0 (SAPO_ST_NONFINITE_INPUT).  Any C and any leading dimension from C up; R may be 0. */
int sapo_fp8_store(const void* x, int32_t x_dtype, int64_t R, int32_t C, int64_t ld_x, const sapo_fp8* h_out,
                   int32_t* status, void* stream);

/* y [T, ld_y] (bf16 or fp32) = x W^T for x [T, K] with scales per row (blocks 0) and W [N, K] with scales
 * per block (blocks 1); products of one block of 128 along K are formed on the tensor cores, scaled and added up in
 * fp32, and rounded once.  data of both 16-byte aligned, ld a multiple of 16 where there is more than one row (codes
 * behind column K are not read).  Any N, K >= 1, T >= 0; y on 16-byte boundaries with ld_y in bytes a multiple of 16 is
 * written faster.  *status: SAPO_ST_WAIT_TIMEOUT. */
int sapo_fp8_matmul(const sapo_fp8* h_x, int64_t T, const sapo_fp8* h_w, int32_t N, int32_t K, void* y, int32_t y_dtype,
                    int64_t ld_y, int32_t* status, void* stream);

/* How a row is drawn: temperature >= 0 (0: the largest logit), top_k (<= 0: off), top_p (>= 1: off; <= 0: the
 * largest logit), min_p in [0, 1] (0: off).  The _rows pointers (device, [B], each may be NULL) give every row a value of its own
 * in place of the common one. */
typedef struct sapo_sample_cfg {
  float   temperature;
  int32_t top_k;
  float   top_p;
  float   min_p;
  const float*   temperature_rows;
  const int32_t* top_k_rows;
  const float*   top_p_rows;
  const float*   min_p_rows;
} sapo_sample_cfg;

/* Draws one token of every row of logits [B, ld] (V columns, bf16 or fp32): the answers of a round
 * (Section 3.1: a node's own completions), whose log-probs the training batch keeps as old_logp.
 * With w_i = exp((z_i - max z) / temperature), tokens stay in the draw that are
 *   among the top_k largest logits (equal logits: lower index first),
 *   in that order the first ones whose predecessors' weight is below top_p of the top_k tokens' weight,
 *   and have w_i >= min_p;
 * the largest always stays.  Of these, token i wins with probability w_i / sum w: ids[b] = the one with the smallest
 * e_i / w_i, e_i = -log(1 - (n_i + 1/2) 2^-32), where the 32 bits n_i come from the row's random number
 * seeds[b]: upper 16 bits half i % 8 (low half of a word first) of philox4x32-10(counter = (i / 8, 0, 0, 0), key = (seed low,
 * seed high)), lower 16 bits the same of counter (i / 8, 1, 0, 0).  The same number draws the same token.
 * logp[b] = log softmax(z)[ids[b]], at temperature 1 and over all tokens: old_logp of the loss calls.
 * Logits of -inf rule a token out.  A row of -inf only gets id -1 and logp 0; so does a row with a NaN, with
 * +inf, or with a temperature, top_p or min_p that is NaN or out of range (SAPO_ST_NONFINITE_INPUT).
 * V in [1, 524287], up to 1474048 bytes of logits a row (SAPO_ERR_UNSUPPORTED_SHAPE beyond); B may be 0.  Rows on 16-byte boundaries
 * are read faster; ld may be 0 (several draws from one row). */
int sapo_sample(const void* logits, int32_t dtype, int32_t B, int32_t V, int64_t ld, const int64_t* seeds,
                const sapo_sample_cfg* h_cfg, int32_t* ids, float* logp, int32_t* status, void* stream);

/* Bytes of scratch the forward (SAPO_WS_FWD), backward (SAPO_WS_BWD, SAPO_WS_BWD_ACTIVE),
 * fused (SAPO_WS_FUSED) or preference (SAPO_WS_PREFERENCE) call wants for these sizes; OR SAPO_WS_OUT_BF16 into `which` for a call
 * with bf16 gradient outputs.  Returns 0 for invalid arguments. */
size_t sapo_workspace_bytes(int32_t which, int64_t T, int32_t H, int32_t V, int32_t dtype);

/* Smallest backward or fused workspace that still works (one 128-token panel). */
size_t sapo_workspace_bytes_min(int32_t which, int64_t T, int32_t H, int32_t V, int32_t dtype);

/* Forward pass without caller-provided scratch (the paper has no counterpart; this exists for
 * hosts that are not allowed to allocate device memory: a component embedded in a process whose
 * memory pool is fixed once at start-up, or a loop that must never reach cudaMalloc because it
 * synchronises the whole device).  Same arguments and results as sapo_policy_loss_fwd, and the
 * same argument checks in the same order, except that `workspace` is gone: the scratch is an
 * array of SAPO_STATIC_SCRATCH_BYTES that is part of the library image, so every GPU that loads
 * the library carries it until the process ends.  The call itself allocates and frees nothing.
 * Limits, checked after the common argument checks: bf16 operands only
 * (SAPO_ERR_UNSUPPORTED_SHAPE otherwise), and
 *     24 * T bytes  (+ 4 * S, rounded up to 256, when seq_surr is NULL)  <=  SAPO_STATIC_SCRATCH_BYTES,
 * i.e. up to 174,762 tokens (32 * T and 131,072 tokens when h_cfg->entropy is given); beyond that
 * the call does nothing and returns SAPO_ERR_STATIC_SCRATCH_EXCEEDED.  The forward keeps 24 (32)
 * bytes per token and vocab split; this
 * entry takes as many of the splits the regular call would use as fit in the array.  When all of
 * them fit the results are bit-identical to sapo_policy_loss_fwd; with fewer splits they agree up
 * to the order in which a token's partial sums are added (and large batches of few tokens per SM
 * pair run somewhat slower).
 * The first call on each device looks up the array's device address (that device must be
 * current); make that first call outside any stream capture, and from one thread.  All calls on
 * a device share the one array and it keeps whatever the previous call left: nothing in it needs
 * clearing between calls, but two calls that may run on the GPU at the same time (different
 * streams, or different threads) race on it and must be ordered by the caller. */
#define SAPO_STATIC_SCRATCH_BYTES (4 * 1024 * 1024)
int sapo_policy_loss_fwd_static(const void* hidden, const void* W_head, int32_t dtype,
                                int64_t T, int32_t H, int32_t V, int64_t ld_hidden, int64_t ld_W,
                                const int32_t* ids, const float* old_logp, const float* adv,
                                const int32_t* cu_seqlens, int32_t S, const sapo_loss_cfg* h_cfg,
                                float* logp, float* lse, float* ratio, float* surr, float* gscale,
                                float* seq_surr, float* loss, int32_t* status, void* stream);

/* Optional per-kernel timing for benchmarks (no counterpart in the paper).  While enabled,
 * every kernel launch of the library is bracketed by two CUDA events recorded on the call's
 * stream.  sapo_timing_read waits for the recorded events, writes the summed milliseconds and
 * the number of launches per kernel id (arrays of SAPO_K_COUNT) and forgets them; at most 16384
 * launches are kept between reads.  The events are created on the first enable.  Not thread-safe.
 * sapo_launch_count returns how many kernels the library has launched in this process. */
#define SAPO_K_PACK_SCAN  0
#define SAPO_K_PACK_COPY  1
#define SAPO_K_GROUP_ADV  2
#define SAPO_K_SPLIT_BF16 3
#define SAPO_K_FWD_GEMM   4
#define SAPO_K_LOSS_TAIL  5
#define SAPO_K_LOSS_FINAL 6
#define SAPO_K_BWD_DZ     7
#define SAPO_K_BWD_DH     8
#define SAPO_K_BWD_DW     9
#define SAPO_K_STREAMK_FIXUP 10
#define SAPO_K_COMPACT   11
#define SAPO_K_SELECT    12
#define SAPO_K_ADAM      13
#define SAPO_K_TARGET_LOGIT 14
#define SAPO_K_FWD_EXP   15
#define SAPO_K_FUSED_TAIL 16
#define SAPO_K_NORM_FWD   17
#define SAPO_K_NORM_BWD   18
#define SAPO_K_NORM_REDUCE 19
#define SAPO_K_CKPT8      20
#define SAPO_K_PREFERENCE 21
#define SAPO_K_PREF_SCORE 22
#define SAPO_K_SAMPLE     23
#define SAPO_K_FP8_STORE  24
#define SAPO_K_FP8_MATMUL 25
#define SAPO_K_ADAMW      26
#define SAPO_K_COUNT      27
int sapo_timing_enable(int32_t on);
int sapo_timing_read(float* h_ms, int32_t* h_launches);
int64_t sapo_launch_count(void);

/* The library's in-kernel waits (on the barriers between the copy, tensor-core and epilogue
 * roles of the GEMM kernels) are bounded: a wait that runs out makes the kernel set
 * SAPO_ST_WAIT_TIMEOUT, let its copies in flight land, free its tensor memory and return, so the
 * context stays usable.  This call (no counterpart in the paper) exercises exactly that code on a
 * barrier nobody arrives at: one thread waits limit_clocks SM clocks (at most 10^8, about 50 ms),
 * then sets the bit in *status.  For tests of a caller's error handling. */
int sapo_debug_wait_timeout(int64_t limit_clocks, int32_t* status, void* stream);

/* Checked builds (the library compiled with -DSAPO_BOUNDS_CHECK, see build.py): the kernels compare
 * every index they compute before a global-memory access with the extent of its array, count a
 * violation and leave the access out.  Returns the number of violations counted so far in this
 * process, or -1 when the library is a regular build. */
int64_t sapo_debug_bounds_violations(void);

/* Text for a return code. */
const char* sapo_status_string(int32_t code);

#ifdef __cplusplus
}
#endif
#endif /* SAPO_H_ */
