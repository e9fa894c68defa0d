/*
 * rollout.h -- C ABI of the MI355X GRPO rollout library (librollout.so).
 *
 * The library runs the rollout phase of a GRPO training step (paper section 3,
 * "Background"): for each of B prompts it generates a group of G sampled
 * completions with a dense decoder-only transformer, and it computes each
 * completion's advantage relative to its own group.  Generation concurrency
 * (sequences in flight), group size, completion length, temperature and top-p
 * are per-call arguments, never cached at initialisation: they are the knobs a
 * power controller moves between calls (sections 4.1, 4.3 and 6.4, Table 4).
 *
 * Conventions for every entry point:
 *  - C linkage, no exceptions cross the boundary, plain pointers and sizes.
 *  - "d_" pointers are device (HBM) pointers owned by the caller; "h_"/plain
 *    struct pointers are host pointers owned by the caller.  The library never
 *    frees caller memory.  rollout_ctx is opaque host state owned by the
 *    library between rollout_init and rollout_destroy.
 *  - Device work is enqueued on the stream given to rollout_init (or passed
 *    directly) and the call returns; outputs are valid after that stream is
 *    synchronised or after rollout_sync.
 *  - Arguments are validated before anything is enqueued; on error nothing is
 *    enqueued and a message is available from rollout_last_error.
 *  - Sequence order is group-major: completion g of prompt p is sequence
 *    s = p * G + g, so every group is contiguous (section 4.3 keeps the
 *    generation batch a multiple of G).
 *  - Token ids are int32; logits, uniforms, rewards and advantages are fp32.
 */
#ifndef ROLLOUT_H
#define ROLLOUT_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t rollout_status;
#define ROLLOUT_OK 0
#define ROLLOUT_EINVAL (-1)      /* bad argument; nothing enqueued */
#define ROLLOUT_ENOMEM (-2)      /* arena or HBM budget too small for the request */
#define ROLLOUT_EDEVICE (-3)     /* HIP runtime error (message in rollout_last_error) */
#define ROLLOUT_ESTATE (-4)      /* call order violated (decode before prefill, context full) */
#define ROLLOUT_EUNSUPPORTED (-5) /* shape the kernels do not implement */

#define ROLLOUT_DTYPE_FP32 0     /* fp32 weights, cache and activations */
#define ROLLOUT_DTYPE_BF16 1     /* bf16 weights/cache/GEMM operands, fp32 residual and logits */
#define ROLLOUT_DTYPE_INT4 2     /* as BF16, but the layer projections (q, k, v, o, gate, up, down) are
                                    weight-only int4: groups of 128 inputs of one output row, each with an
                                    fp32 scale s = (hi - lo) / 15 and a zero point z = rint(-lo / s) in
                                    [0, 15], codes q = clamp(rint(w / s) + z, 0, 15) (the AWQ storage format
                                    of the 72B generation proxy, sections 5 and 6.6, which fix no format).
                                    The model multiplies with the group-quantised weight's plain value
                                    (q - z) * s, never rounded to bf16: each group's scale multiplies its
                                    integer dot product in fp32.  Embedding and LM head stay bf16.  Needs
                                    d_model, n_heads*head_dim and d_ff to be multiples of 128. */

#define ROLLOUT_DTYPE_E4M3 3     /* 8 bits: sign, 4 exponent bits (bias 7), 3 mantissa bits, largest value 448, no
                                    infinity.  Outputs and optimiser states of the update side, always with a power of
                                    two as fp32 scale: what is stored stands for code * scale.  No model's type. */

typedef struct rollout_ctx rollout_ctx;

/*
 * Model and capacity description; immutable after rollout_init.
 * The model is a dense decoder (section 5 runs the Qwen2.5 family): RMSNorm,
 * grouped-query attention with rotate-half RoPE, SwiGLU MLP, untied LM head,
 * no biases.  Weights are synthesised on the device from weight_seed with the
 * SplitMix64-based counter hash (Irwin-Hall(4) values of standard deviation
 * weight_std; norm gains 1).
 * Supported shapes: head_dim in {32, 64, 128}; n_heads a multiple of
 * n_kv_heads with n_heads / n_kv_heads <= 16; d_model, n_heads*head_dim and
 * d_ff multiples of 32; vocab a multiple of 16; kv_block_size in {8, 16, 32}.
 */
typedef struct {
  int32_t n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ff, vocab;
  float rms_eps, rope_theta;
  int32_t dtype;               /* ROLLOUT_DTYPE_* */
  uint64_t weight_seed;
  double weight_std;           /* standard deviation of the synthesised weights */
  int32_t kv_block_size;       /* tokens per paged-KV block */
  int32_t max_prompt_len;      /* longest prompt any call may pass */
  int32_t max_new_tokens;      /* longest completion any call may request */
  int32_t max_seqs_in_flight;  /* requested concurrency ceiling; the plan may lower it */
  uint64_t hbm_budget_bytes;   /* 0 = free device memory reported by the runtime */
} rollout_model_config;

/* Result of planning: how many sequences fit and how big the arena must be. */
typedef struct {
  int32_t seqs_in_flight_max;  /* multiple of group_size; 0 never returned with OK */
  int32_t kv_blocks;           /* paged-KV blocks in the pool */
  uint64_t arena_bytes;        /* device bytes the caller must provide to rollout_init */
  uint64_t weight_bytes;       /* of which model weights */
  uint64_t kv_block_bytes;     /* bytes of one block across all layers, K and V */
  uint64_t kv_bytes;           /* bytes of the whole pool */
  uint64_t work_bytes;         /* activations, logits and split-K workspace */
} rollout_plan_t;

/*
 * Size the arena (section 4.3: the generation batch must be a multiple of G).
 * Host-only unless cfg->hbm_budget_bytes == 0, in which case the free memory
 * of the current HIP device is queried.  seqs_in_flight_max is the largest
 * multiple of group_size, at most cfg->max_seqs_in_flight, whose weights,
 * KV blocks (prompt blocks shared inside a group), activations, logits and
 * workspace fit in the budget.
 * Errors: EINVAL (bad config or group_size < 1), EUNSUPPORTED (shape),
 * ENOMEM (not even one group fits), EDEVICE (memory query failed).
 */
rollout_status rollout_plan(const rollout_model_config* cfg, int32_t group_size, rollout_plan_t* out);

/*
 * Set up the rollout engine of section 3's rollout phase: the model of section 5 (a dense decoder of the
 * Qwen2.5 family, here with synthetic weights) resident in HBM, ready to generate groups of completions.
 * Bind a context to a caller-owned device arena of arena_bytes (>= the plan's
 * arena_bytes for group size 1 at cfg->max_seqs_in_flight, or the value
 * returned by rollout_plan for the group size that will be used), enqueue
 * weight synthesis on hip_stream (a hipStream_t; NULL = default stream) and
 * return the context in *out.  The arena must stay allocated until
 * rollout_destroy.  Errors: EINVAL, EUNSUPPORTED, ENOMEM (arena too small),
 * EDEVICE.
 */
rollout_status rollout_init(const rollout_model_config* cfg, void* d_arena, uint64_t arena_bytes,
                            void* hip_stream, rollout_ctx** out);

/*
 * Section 3's rollout phase, first forward: a batch of B prompts, each the prompt of a group of G
 * candidate completions.
 * Start a wave: n_prompts prompts of prompt_len tokens (d_prompts, int32,
 * row-major [n_prompts, prompt_len]), each expanded to group_size sequences.
 * Each prompt is run through the model once; its KV blocks are shared by the
 * group's sequences (a partially filled last block is copied per sequence).
 * Writes the last-position logits of every sequence, fp32 row-major
 * [n_prompts * group_size, vocab], to d_logits (rows of a group are equal).
 * Any previous wave is discarded.  Errors: EINVAL (sizes, prompt_len >
 * max_prompt_len), ENOMEM (more sequences than the plan admits), EDEVICE.
 * Token ids outside [0, vocab) set the device error flag (see rollout_sync).
 */
rollout_status rollout_prefill(rollout_ctx* ctx, const int32_t* d_prompts, int32_t n_prompts,
                               int32_t prompt_len, int32_t group_size, float* d_logits);

/*
 * One autoregressive step of section 3's rollout phase (every candidate of every group extends by one
 * token; completion length is the knob of Table 4's third row, section 6.4).
 * One decode step of the current wave: append token d_tokens[s] (int32
 * [n_seqs]) to every sequence s at its next position and write the logits of
 * that position, fp32 [n_seqs, vocab], to d_logits.  n_seqs is the wave's
 * sequence count.  Errors: ESTATE (no wave, or the context would exceed
 * max_prompt_len + max_new_tokens), EDEVICE.
 */
rollout_status rollout_decode_step(rollout_ctx* ctx, const int32_t* d_tokens, float* d_logits);

/*
 * The draw that makes a group's G candidates differ (section 3: G sampled answers to the same prompt).
 * The paper names no sampler settings; temperature and top-p are per-call knobs with the definition below.
 * Draw one token per row of d_logits (fp32 [n_seqs, vocab]) with one uniform
 * per row (d_uniforms, fp32 [n_seqs], values in [0, 1)) into d_tokens_out
 * (int32 [n_seqs]).  temperature 0 is greedy (lowest id among equal maxima).
 * Otherwise e_i = exp(z_i / T - max) in fp32; with top_p < 1 the kept set is
 * the shortest prefix, in (e descending, id ascending) order, whose mass
 * reaches top_p of the total; the token is the first kept id, in ascending
 * id order, whose running mass exceeds u times the kept mass.
 * Errors: EINVAL (n_seqs < 1, temperature < 0, top_p outside (0, 1]), EDEVICE.
 */
rollout_status rollout_sample(rollout_ctx* ctx, const float* d_logits, int32_t n_seqs, float temperature,
                              float top_p, const float* d_uniforms, int32_t* d_tokens_out);

/*
 * Group-relative advantages (section 3: each candidate's reward against its
 * own group; GRPO's normalisation by the group's standard deviation).
 * d_rewards fp32 [n_groups * group_size] in group-major order; d_adv receives
 * A = (r - mean) / (std + eps) with std using divisor group_size - std_ddof;
 * groups whose rewards are all equal (or group_size == 1) get A = 0 and are
 * counted into *d_zero_var_groups (int32, device; overwritten; may be NULL),
 * the zero-variance-group statistic of section 4.2.  Enqueued on hip_stream.
 * Errors: EINVAL (n_groups < 1, group_size < 1, std_ddof not 0 or 1, eps < 0,
 * NULL rewards or advantages), EDEVICE.
 */
rollout_status grpo_advantages(const float* d_rewards, int32_t n_groups, int32_t group_size, float eps,
                               int32_t std_ddof, float* d_adv, int32_t* d_zero_var_groups, void* hip_stream);

/*
 * The whole rollout for n_prompts prompts (d_prompts int32 [n_prompts,
 * prompt_len]): waves of whole groups, at most seqs_in_flight sequences each
 * (snapped down to a multiple of group_size, section 4.3), each wave prefilled
 * once then decoded max_new_tokens - 1 times, drawing token t of sequence s
 * with d_uniforms[s * max_new_tokens + t] (fp32 [n_prompts * group_size,
 * max_new_tokens]) into d_tokens_out[s * max_new_tokens + t] (int32, same
 * shape).  Exactly max_new_tokens tokens per completion (no end-of-sequence).
 * Errors: EINVAL, ENOMEM (one group does not fit), EDEVICE.
 */
rollout_status rollout_generate(rollout_ctx* ctx, const int32_t* d_prompts, int32_t n_prompts,
                                int32_t prompt_len, int32_t group_size, int32_t seqs_in_flight,
                                int32_t max_new_tokens, float temperature, float top_p,
                                const float* d_uniforms, int32_t* d_tokens_out);

/*
 * Completions that end at a stop token, served by continuous batching.  The
 * paper's controller counts T_k, the non-padding tokens a batch produced
 * (section 4.5, eq. 4), and its runs reward closeness to a length target
 * (section 5): both presuppose completions that end when the model draws a
 * stop token.
 *
 * Draws are those of rollout_generate (token t of completion s = p * G + g
 * with d_uniforms[s * max_new_tokens + t]); completion s ends after drawing a
 * token of the stop set (d_stop_ids, n_stop device int32 ids in [0, vocab);
 * n_stop = 0: no stop set) or after max_new_tokens tokens.  Outputs (device,
 * caller-owned): d_tokens_out int32 [n_prompts * G, max_new_tokens], -1 after
 * the end; d_lengths_out int32 [n_prompts * G], tokens including the stop
 * token; d_admit_step_out int32 [n_prompts * G] or NULL, the decode step at
 * which each completion was admitted; *h_decode_steps_out (host, or NULL) the
 * decode steps run.
 *
 * Scheduling: every refill_interval decode steps the host reads the slots'
 * ended flags and refills, in slot order, in completion order.
 *  - whole_groups = 1: min(seqs_in_flight snapped to whole groups (section
 *    4.3), n_prompts * G) slots in ranges of G; a range whose G completions
 *    have all ended takes the next prompt's group (prefilled there, token 0
 *    drawn from its logits).
 *  - whole_groups = 0: min(seqs_in_flight, context rows - 1, n_prompts * G)
 *    slots; a slot whose completion has ended takes the next completion.  A
 *    group's prompt is prefilled once, when its first completion is admitted,
 *    into a prompt record of KV blocks shared by its members (at most slots + 1
 *    records are alive); every member's token 0 is drawn then, so group_size
 *    must not exceed the context's sequence rows (else ENOMEM).  Needs
 *    (slots + 1) * ceil(prompt / block) + slots * (blocks from the last full
 *    prompt block to the end) KV blocks; fewer slots are used if the pool is
 *    smaller.
 * The call returns when every completion has been admitted and has ended.
 * Ended completions keep running in their slot until it is refilled (their
 * rows are the padding that T_k excludes).  Errors: EINVAL (bad argument, or
 * a stop id outside [0, vocab), reported by rollout_sync), ENOMEM, EDEVICE.
 */
rollout_status rollout_generate_eos(rollout_ctx* ctx, const int32_t* d_prompts, int32_t n_prompts,
                                    int32_t prompt_len, int32_t group_size, int32_t seqs_in_flight,
                                    int32_t max_new_tokens, float temperature, float top_p,
                                    const float* d_uniforms, const int32_t* d_stop_ids, int32_t n_stop,
                                    int32_t refill_interval, int32_t whole_groups, int32_t* d_tokens_out,
                                    int32_t* d_lengths_out, int32_t* d_admit_step_out,
                                    int32_t* h_decode_steps_out);

/*
 * Length-target reward of section 5 (its formula is not given; reading:
 * r = 1 - min(1, |L - target| / target), 1 at the target, 0 at distance
 * >= target) for n completion lengths d_lengths (device int32), into
 * d_rewards (device fp32 [n]); *d_total_tokens (device int64, or NULL)
 * receives the sum of the lengths, the batch's non-padding token count T_k
 * (section 4.5).  Enqueued on hip_stream.  Errors: EINVAL, EDEVICE.
 */
rollout_status rollout_length_rewards(const int32_t* d_lengths, int32_t n, int32_t target, float* d_rewards,
                                      int64_t* d_total_tokens, void* hip_stream);

/* Wait for the context's stream and report the device error flag (EINVAL if a
 * token id outside [0, vocab) was seen since the last call; the flag is then
 * cleared).  Errors: EINVAL, EDEVICE. */
rollout_status rollout_sync(rollout_ctx* ctx);

/* Release the context's host state (never the caller's arena). NULL is a no-op. */
void rollout_destroy(rollout_ctx* ctx);

/* Last error message of ctx, or of the calling thread's last context-free
 * call when ctx is NULL.  Never NULL; valid until the next call. */
const char* rollout_last_error(const rollout_ctx* ctx);

/* ------------------------------------------------------------------------ */
/* Allocation-free draw                                                      */
/* ------------------------------------------------------------------------ */

/*
 * For callers that cannot allocate device memory (code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc): the draw of
 * rollout_sample without a context.  Same definition and arguments as
 * rollout_sample, plus the row width vocab and hip_stream (a hipStream_t of
 * the current device; NULL = its default stream); enqueued on that stream.
 * Nothing is allocated: the sampler kernels' scratch is one fixed device array
 * of ROLLOUT_SAMPLE_NOALLOC_SCRATCH_BYTES, held on every GPU the call runs on
 * until the process ends, and rows are drawn in batches that fit it.  Every
 * call on a GPU shares that GPU's array, so calls that overlap on one GPU
 * (several streams or threads) race on it and must be serialised by the
 * caller.  Errors (message from rollout_last_error(NULL)): EINVAL (NULL
 * buffer, n_seqs < 1, vocab < 2, temperature < 0, top_p outside (0, 1], a
 * stream of another device), ENOMEM (one row needs more scratch than the
 * array holds: vocab above 16,724,608), EDEVICE.
 */
#define ROLLOUT_SAMPLE_NOALLOC_SCRATCH_BYTES (64ull << 20)
rollout_status rollout_sample_noalloc(const float* d_logits, int32_t n_seqs, int32_t vocab, float temperature,
                                      float top_p, const float* d_uniforms, int32_t* d_tokens_out,
                                      void* hip_stream);

/* ------------------------------------------------------------------------ */
/* The update side of a GRPO step                                            */
/* ------------------------------------------------------------------------ */
/*
 * After the rollout a step scores its tokens, forms the clipped loss over the
 * groups' advantages and carries its gradient back (section 3's update phase,
 * of which the paper gives no arithmetic: the definitions are below).  These
 * entry points need no context.  hip_stream is a hipStream_t of the current
 * device (NULL = its default stream; a stream of another device: EINVAL), and
 * every buffer is the caller's, on that device.  A workspace is device memory
 * aligned to 16 bytes, at least as large as the call's _workspace query says
 * for the same sizes (for larger ones it says no less, so the workspace of the
 * largest call serves them all); nothing is kept in it from one call to the
 * next, and calls that may run at the same time (two streams, two captured
 * graphs) need one each.  Buffers are aligned to their element's size, and no output and no
 * workspace shares a byte with another one or with an input, but for the one case named
 * below (EINVAL; the space between the rows of logits belongs to no one).  Nothing is
 * allocated or waited for, so every call can be captured into a HIP graph.  Messages:
 * rollout_last_error(NULL).
 *
 * dtype of a matrix: ROLLOUT_DTYPE_FP32 or ROLLOUT_DTYPE_BF16.  Arithmetic is
 * fp32 or wider, outputs are rounded once (to nearest, ties to even).  Results
 * do not depend on scheduling: no floating-point atomics.
 * A token id < 0 is padding (rollout_generate_eos fills with -1).
 */

/*
 * Log probabilities of given tokens under softmax(z / temperature), with the
 * rows' entropies and most likely alternatives.  d_logits: n_rows rows of vocab
 * values of dtype, row_stride elements apart (>= vocab; rows may start at any
 * element); d_tokens int32 [n_rows].  Outputs, each fp32 and NULL if not
 * wanted:
 *   d_logp [n_rows]      log p of the row's token;
 *   d_entropy [n_rows]   -sum p log p;
 *   d_stats [n_rows, 2]  max z, and log sum exp((z - max z) / temperature): what the
 *                        gradient needs.  (Their sum, the log-sum-exp of the row, would
 *                        lose the second where the logits stand far from zero.)
 *   d_top_ids int32, d_top_logp [n_rows, n_top]  the n_top ids with the largest
 *                        logits, equal ones by lowest id, and their log p; both needed
 *                        when n_top > 0 (at most 32 and vocab), unused when it is 0.
 * The distribution is the whole one: a draw's top-p does not enter.
 * Padding rows are not read and get zeros (top ids -1).  A token >= vocab gets
 * log p NaN.  Logits of -inf have probability 0; a row of nothing else has log p
 * -inf, entropy 0, statistics -inf and the lowest ids as alternatives.  A row
 * with NaN or +inf gets NaN everywhere and top ids -1.  d_tokens NULL: no row
 * is padding, and d_logp must be NULL.
 * Errors: EINVAL (sizes, types, alignment, NULL buffers, temperature not > 0, no
 * output), EUNSUPPORTED (n_rows or vocab above 2^30, vocab above 327,680 with n_top > 0), ENOMEM
 * (workspace too small), EDEVICE.
 */
rollout_status rollout_token_logprobs_workspace(int32_t n_rows, int32_t vocab, int32_t n_top, uint64_t* h_bytes);
rollout_status rollout_token_logprobs(const void* d_logits, int32_t dtype, int64_t row_stride, int32_t n_rows,
                                      int32_t vocab, float temperature, const int32_t* d_tokens, int32_t n_top,
                                      float* d_logp, float* d_entropy, float* d_stats, int32_t* d_top_ids,
                                      float* d_top_logp, void* d_workspace, uint64_t workspace_bytes,
                                      void* hip_stream);

/*
 * Gradient of the above with respect to the logits.  With p = softmax(z / T), H
 * its entropy, g = d_grad_logp and h = d_grad_entropy (fp32 [n_rows]; h NULL: 0):
 *   dz_i = (g (1[i = token] - p_i) - h p_i (log p_i + H)) / T
 * into d_grad_logits, n_rows rows of vocab values of dtype, grad_stride elements
 * apart; it may be d_logits itself at the same stride (any other overlap of the
 * two, from first to last row: EINVAL).  d_stats and d_entropy (needed only with h) are the forward call's.
 * What lies between the rows is left alone.  Rows that are padding, have g = h = 0
 * or hold nothing but -inf get zeros and are not read; a token >= vocab makes
 * its row NaN.  Errors: EINVAL, EUNSUPPORTED (n_rows or vocab above 2^30), EDEVICE.
 */
rollout_status rollout_token_logprobs_backward(const void* d_logits, int32_t dtype, int64_t row_stride, int32_t n_rows,
                                               int32_t vocab, float temperature, const int32_t* d_tokens,
                                               const float* d_stats, const float* d_entropy, const float* d_grad_logp,
                                               const float* d_grad_entropy, void* d_grad_logits, int64_t grad_stride,
                                               void* hip_stream);

/*
 * The clipped policy loss over groups of completions, and its gradient.  All matrices
 * are fp32 [n_seqs, max_len], sequence s being completion s of the rollout and
 * its tokens 0 .. len_s - 1 counted (d_lengths int32 [n_seqs] as rollout_generate_eos
 * leaves them, taken into [0, max_len]; NULL: max_len each); what lies
 * behind them is not used and gets gradient 0.  With lp = d_logp, A = d_adv[s]
 * (grpo_advantages), r = exp(lp - old), x = ref - lp:
 *   tok  = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl_coef (exp(x) - 1 - x) - entropy_coef H
 *   loss = sum_s w_s sum_t tok,  w_s by mean:
 *     ROLLOUT_MEAN_SEQUENCE  1 / (n_seqs len_s)      each completion weighs the same
 *     ROLLOUT_MEAN_TOKEN     1 / sum len             each token weighs the same
 *     ROLLOUT_MEAN_FIXED     1 / (n_seqs max_len)    lengths do not enter
 *   (a divisor of 0 counts as 1: nothing but empty sequences has loss 0)
 *   dlp  = w_s (-A r where the ratio is not clipped - kl_coef (exp(x) - 1)),  dH = -entropy_coef w_s
 * A token is clipped where A > 0 and r > 1 + clip_high, or A < 0 and r < 1 - clip_low;
 * with A = 0 the first term is 0 whatever the ratio.  d_old_logp NULL: the
 * log probabilities themselves, held constant (r = 1).  d_ref_logp NULL: no penalty
 * (kl_coef must be 0).  d_entropy NULL: no entropy term (entropy_coef must be 0).
 * A coefficient of 0 leaves its term out of loss and gradients (the statistics stay), so
 * that a term which overflows can still be watched.  Terms are fp32: an exponential of
 * more than 88.7 is infinite.  A log probability of -inf (a masked id) has ratio 0 and
 * exp(x) - 1 - x = inf; where lp and old (or lp and ref) are both infinite their
 * difference, and what follows from it, is NaN.
 * Outputs, each NULL if not wanted: d_loss fp32 [1]; d_stats fp32 [5], means over the counted
 * tokens of r, of exp(x) - 1 - x, of tokens clipped below, clipped above, of H; d_grad_logp,
 * d_grad_entropy fp32 [n_seqs, max_len].  Sums are fp64.
 * Errors: EINVAL (sizes, clip_low outside [0, 1], clip_high < 0, coefficients, mean,
 * NULL buffers, overlap, no output), EUNSUPPORTED (2^31 tokens or more), ENOMEM
 * (workspace too small), EDEVICE.
 */
#define ROLLOUT_MEAN_SEQUENCE 0
#define ROLLOUT_MEAN_TOKEN 1
#define ROLLOUT_MEAN_FIXED 2
rollout_status grpo_policy_loss_workspace(int32_t n_seqs, int32_t max_len, uint64_t* h_bytes);
rollout_status grpo_policy_loss(const float* d_logp, const float* d_old_logp, const float* d_ref_logp,
                                const float* d_entropy, const float* d_adv, const int32_t* d_lengths, int32_t n_seqs,
                                int32_t max_len, float clip_low, float clip_high, float kl_coef, float entropy_coef,
                                int32_t mean, float* d_loss, float* d_stats, float* d_grad_logp, float* d_grad_entropy,
                                void* d_workspace, uint64_t workspace_bytes, void* hip_stream);

/*
 * Embedding lookup: d_out [n_tokens, dim] of out_dtype, row n being scale times row
 * d_tokens[n] of d_table [vocab, dim] of table_dtype (tensor 0 of rollout_export_weight,
 * say).  Padding gives zeros, an id >= vocab NaN.  Both matrices are dense and do not
 * overlap.  Errors: EINVAL (sizes, types, alignment, NULL buffers, overlap, scale not finite),
 * EUNSUPPORTED (vocab or dim above 2^30, n_tokens above 2^28), EDEVICE.
 */
rollout_status rollout_embedding(const void* d_table, int32_t table_dtype, int32_t vocab, int32_t dim,
                                 const int32_t* d_tokens, int32_t n_tokens, float scale, void* d_out, int32_t out_dtype,
                                 void* hip_stream);

/*
 * Its gradient: row v of d_grad_table [vocab, dim] of table_dtype becomes scale times the
 * sum of the rows of d_grad [n_tokens, dim] of grad_dtype whose token is v.  With accumulate
 * 0 every row is written (rows without tokens with zeros); with 1 the sum is added
 * to what the row holds, rounded once, and rows without tokens are left alone.
 * Ids outside [0, vocab) contribute nothing.  Tokens are sorted by id and a row's are
 * added in fp32 in an order that the call's sizes and tokens fix: the same call gives the
 * same bits, but other ids in the batch may move a row's sum by roundings.  Errors as above, EUNSUPPORTED also where
 * n_tokens ceil(dim / 1024) is above 2^25, and ENOMEM (workspace too small).
 */
rollout_status rollout_embedding_backward_workspace(int32_t n_tokens, int32_t vocab, int32_t dim, uint64_t* h_bytes);
rollout_status rollout_embedding_backward(const void* d_grad, int32_t grad_dtype, const int32_t* d_tokens, int32_t n_tokens,
                                          int32_t vocab, int32_t dim, float scale, int32_t accumulate, void* d_grad_table,
                                          int32_t table_dtype, void* d_workspace, uint64_t workspace_bytes,
                                          void* hip_stream);

/*
 * The update through the layers: attention over packed sequences and its gradient, the norm of the
 * residual stream and its gradient, and the optimiser's step.  What else a layer has, matrix products, rotary embedding
 * and the gated activation, is the caller's, with its gradients.
 *
 * Attention.  Sequences lie one behind the other in matrices of tokens, d_q [n_q, n_heads * head_dim] and
 * d_k, d_v [n_k, n_kv_heads * head_dim], whose rows are a stride of elements apart (so that the three
 * may be columns of one projection's output; n_heads / n_kv_heads query heads share a key's).  Sequence
 * s has the rows from starts[s] on, lens[s] of them, at most up to starts[s + 1] (d_q_starts, d_k_starts
 * int32 [n_seqs + 1], ascending; d_q_lens, d_k_lens int32 [n_seqs], NULL: all of them.  Values are taken
 * into [0, rows]; with starts that descend it is not said which rows are written).  A padded batch has
 * starts s * max_len and its lengths.  d_k_starts NULL: keys lie where the queries do (n_k = n_q).
 *   s_ij = scale q_i k_j;  lse_i = log sum_j exp(s_ij);  out_i = sum_j exp(s_ij - lse_i) v_j
 * over all keys of the sequence or, causal, over keys j <= i + len_k - len_q (the queries are the last
 * of the keys' tokens).  A query without keys gets out 0 and lse -inf.  Rows of no sequence are neither
 * read nor written, in the outputs either.  What is not finite in a sequence may reach all of its rows,
 * and none of another one's.
 * d_out as d_q, d_lse fp32 [n_heads, n_q].
 * dtype FP32 (fp32 products) or BF16 (probabilities and their gradients enter products as bf16; sums
 * and statistics are fp32; in calls of at most 16,384 pairs, n_q n_heads n_k / n_seqs, what that rounding takes is multiplied
 * too).  A sequence's last bits depend on the shape that it is called with, not on the other sequences' values.
 * Matrices and strides are multiples of 16 bytes, rows at most 2^25 bytes apart.
 * The workspace is for 64 parts that a query's keys may be cut into, each n_q n_heads (head_dim + 4) fp32, and 256 MiB at most;
 * it goes by these alone, whether or not the call is cut, so that a larger call's serves smaller ones.
 * Errors: EINVAL (shape, NULL buffers, alignment, strides, overlap), EUNSUPPORTED (head_dim not 32, 64 or
 * 128, n_heads / n_kv_heads above 64, n_heads times tokens above 2^26, n_heads times sequences above 2^23, strides), ENOMEM
 * (workspace too small), EDEVICE.
 */
typedef struct {
  int32_t dtype;               /* ROLLOUT_DTYPE_FP32 or _BF16: of all matrices */
  int32_t n_heads, n_kv_heads, head_dim;
  int32_t n_seqs;
  int32_t n_q, n_k;            /* rows of the queries' and of the keys' matrices */
  int32_t causal;              /* 0 or 1 */
  float scale;                 /* of the products, in [2^-100, 2^100] */
} rollout_attention_shape;

rollout_status rollout_attention_workspace(const rollout_attention_shape* shape, uint64_t* h_bytes);
rollout_status rollout_attention(const rollout_attention_shape* shape, const void* d_q, int64_t q_stride, const void* d_k,
                                 int64_t k_stride, const void* d_v, int64_t v_stride, const int32_t* d_q_starts,
                                 const int32_t* d_q_lens, const int32_t* d_k_starts, const int32_t* d_k_lens, void* d_out,
                                 int64_t out_stride, float* d_lse, void* d_workspace, uint64_t workspace_bytes,
                                 void* hip_stream);

/*
 * Its gradient: with p_ij = exp(s_ij - lse_i) and D_i = sum grad_out_i out_i, out and lse being the forward call's,
 *   grad_v_j = sum_i p_ij grad_out_i;  ds_ij = p_ij (grad_out_i v_j - D_i)
 *   grad_k_j = scale sum_i ds_ij q_i;  grad_q_i = scale sum_j ds_ij k_j
 * each over the query heads that share the key's.  Every row of a sequence is written (keys that no query
 * attends, and queries without keys, get 0).  The gradients' rows may be columns of one matrix.  The workspace holds 8 bytes
 * for every query and head, and the parts' sums, 256 MiB of them at most.
 * Errors as above.
 */
rollout_status rollout_attention_backward_workspace(const rollout_attention_shape* shape, uint64_t* h_bytes);
rollout_status rollout_attention_backward(const rollout_attention_shape* shape, const void* d_q, int64_t q_stride,
                                          const void* d_k, int64_t k_stride, const void* d_v, int64_t v_stride,
                                          const int32_t* d_q_starts, const int32_t* d_q_lens, const int32_t* d_k_starts,
                                          const int32_t* d_k_lens, const void* d_out, int64_t out_stride, const float* d_lse,
                                          const void* d_grad_out, int64_t grad_out_stride, void* d_grad_q,
                                          int64_t grad_q_stride, void* d_grad_k, int64_t grad_k_stride, void* d_grad_v,
                                          int64_t grad_v_stride, void* d_workspace, uint64_t workspace_bytes,
                                          void* hip_stream);

/*
 * Root-mean-square norm of rows of dim values, behind the addition to the residual stream:
 *   h = x + delta (rounded to x_dtype);  rstd = 1 / sqrt(mean h^2 + eps);  y = h rstd gain
 * d_x [n_rows, dim] of x_dtype, d_delta of delta_dtype with d_h of x_dtype (which may be d_x), or both NULL (h = x);
 * d_gain fp32 [dim], NULL: 1; d_y of y_dtype; d_rstd fp32 [n_rows], NULL if not wanted (the gradient needs it).  Squares are
 * summed in fp32: a row whose sum of squares is above 3.4e38 gets rstd 0.
 * x and delta are FP32 or BF16.  y is FP32, BF16 or E4M3: then d_scales [n_rows] (otherwise NULL) receives
 * the smallest power of two, 2^-126 at least, for which no finite |y| of the row, over it, is above 448, and d_y the codes of
 * y over it, to nearest, ties to even (NaN where y is not finite).  Matrices are dense, and rows may start at any element.
 * Errors: EINVAL (sizes, types, alignment, NULL buffers, overlap), EUNSUPPORTED (dim above 32,768,
 * rows whose launch would have 2^32 threads: some 2^26 up to dim 1,024, 2^22 from 4,097 on), EDEVICE.
 */
rollout_status rollout_rms_norm(const void* d_x, int32_t x_dtype, const void* d_delta, int32_t delta_dtype,
                                const float* d_gain, int32_t n_rows, int32_t dim, float eps, void* d_h, void* d_y,
                                int32_t y_dtype, float* d_scales, float* d_rstd, void* hip_stream);

/*
 * Its gradient.  d_h are the normed rows (d_h of the forward call, or d_x without an addition), d_rstd its statistics,
 * d_grad_h of grad_x_dtype the gradient that reaches h by the residual stream (NULL: none; it may be d_grad_x):
 *   t = grad_y gain;  xhat = h rstd;  grad_x = grad_h + rstd (t - xhat mean(t xhat));  grad_gain = sum over rows of grad_y xhat
 * grad_x is the gradient of x and of delta alike.  d_grad_gain fp32 [dim], NULL: not wanted (and no workspace
 * needed); accumulate 1 adds to what it holds.  Errors as above, and ENOMEM (workspace too small).
 */
rollout_status rollout_rms_norm_backward_workspace(int32_t n_rows, int32_t dim, uint64_t* h_bytes);
rollout_status rollout_rms_norm_backward(const void* d_grad_y, int32_t grad_y_dtype, const void* d_h, int32_t h_dtype,
                                         const float* d_gain, const float* d_rstd, int32_t n_rows, int32_t dim,
                                         const void* d_grad_h, void* d_grad_x, int32_t grad_x_dtype, float* d_grad_gain,
                                         int32_t accumulate, void* d_workspace, uint64_t workspace_bytes,
                                         void* hip_stream);

/*
 * AdamW over many tensors in one launch.  A table names them: rollout_adamw_table writes it to host memory
 * (rollout_adamw_table_bytes of it), the caller copies it to the device once, and it serves every step as long as
 * the buffers stay where they are, the gradients' among them (a program that allocates these anew for every step makes the
 * table anew as well).  A tensor of n >= 0 elements:
 *   d_param of param_dtype (FP32 or BF16), d_grad of grad_dtype (FP32 or BF16);
 *   d_m, d_v: first and second moment, fp32 (state_dtype FP32), or E4M3 codes with d_m_scales, d_v_scales fp32
 *     [ceil(n / 128)], one scale for 128 elements: m = code scale, sqrt(v) = code scale.  Zeros are a fresh state;
 *   d_copy: bf16 copy of fp32 weights that the step writes (to nearest), or NULL.
 * Buffers are aligned to their elements; one that is written shares no byte with any other of the table.
 * The step, with g = grad_scale grad and t = step:
 *   m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2
 *   param = param (1 - lr weight_decay) - lr m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps)
 * in fp32, a moment's products, sum and root each rounded to nearest, with the new moments before they are rounded further
 * (one of less than 2^-126 may count as 0; eps is 0 or at least that).  BF16 weights and E4M3 states are rounded up or
 * down with the probability that keeps their expectation (to nearest they would not move by steps that are small beside
 * them), by 16 bits r of a counter hash of (seed, t, the tensor's place in the table, the element): bf16 drops 16 bits of
 * the fp32 value's magnitude after adding r, e4m3 drops 20 after adding 16 r + 8 (below 2^-6, where values are 2^-9 apart,
 * from the magnitude plus 2^-6).  A scale is the smallest power of two, 2^-126 at least, that leaves no finite magnitude of
 * its 128 above 448 (a moment that is not finite becomes NaN, and no other one of the 128 changes by it); a second moment
 * of 2^-126 or more keeps a code above 0.  Of h = f(i * 0x9E3779B1 + k) for element i, m takes the low 16 bits and v the high ones; a weight the low ones of f(h + (k >> 32)).  f is MurmurHash3's 32-bit
 * finaliser, k = F(F(seed + G t) + G (1 + tensor + 2^20 floor(i / 2^32))) with SplitMix64's finaliser F and constant G.
 * d_grad_scale fp32 [1] (a clipping factor, say; NULL: 1): where it is not finite nothing changes.  d_lr fp32 [1] and d_step
 * int64 [1] replace lr and step if not NULL (a captured call reads them at every replay; a step below 1 counts as 1).
 * n_chunks is what rollout_adamw_table said; d_table has to hold what it wrote.
 * Errors: EINVAL (types, alignment, NULL buffers, overlap, factors), EUNSUPPORTED (more than 2^20 tensors,
 * 2^36 elements or 2^24 - 8 chunks of them), ENOMEM (table too small), EDEVICE.
 */
typedef struct {
  void* d_param;
  const void* d_grad;
  void *d_m, *d_v;
  float *d_m_scales, *d_v_scales;   /* E4M3 states only */
  void* d_copy;
  int64_t n;
  int32_t param_dtype, grad_dtype, state_dtype;
  float weight_decay;
} rollout_adamw_tensor;

rollout_status rollout_adamw_table_bytes(int32_t n_tensors, uint64_t* h_bytes);
rollout_status rollout_adamw_table(const rollout_adamw_tensor* h_tensors, int32_t n_tensors, void* h_table,
                                   uint64_t table_bytes, int64_t* h_chunks);
rollout_status rollout_adamw(const void* d_table, int32_t n_tensors, int64_t n_chunks, double lr, double beta1, double beta2,
                             double eps, int64_t step, uint64_t seed, const float* d_grad_scale, const float* d_lr,
                             const int64_t* d_step, void* hip_stream);

/* ------------------------------------------------------------------------ */
/* Inspection and measurement                                                */
/* ------------------------------------------------------------------------ */

/* Weight tensor ids of the synthesis hash: embedding 0; layer l:
 * 1 + 9 l + {1 Wq, 2 Wk, 3 Wv, 4 Wo, 6 Wgate, 7 Wup, 8 Wdown}; LM head
 * 2 + 9 n_layers.  Copies the logical [out, in] matrix, as fp32 (bf16 values
 * widened exactly), into d_out (caller-owned, rows*cols floats), whatever the
 * physical layout the kernels keep it in.  Errors: EINVAL (not a matrix id). */
rollout_status rollout_export_weight(rollout_ctx* ctx, int32_t tensor_id, float* d_out);

/* Per-kernel-class timing of one instrumented decode step of the current
 * wave, with HIP events around every launch on the context's stream.  The
 * step is run for real (it appends d_tokens like rollout_decode_step).
 * Classes: 0 projection GEMMs (QKV, O, gate/up, down, LM head), 1 decode
 * attention (+ its combine), 2 everything else.  ms[c] = summed duration,
 * launches[c] = launch count, bytes[c] = algorithmic HBM bytes (weights read
 * once, cache read once per sequence, activations), flops[c] = useful flops. */
typedef struct {
  double ms[3];
  int32_t launches[3];
  double bytes[3];
  double flops[3];
} rollout_step_profile;
rollout_status rollout_profile_decode_step(rollout_ctx* ctx, const int32_t* d_tokens, float* d_logits,
                                           rollout_step_profile* out);

/* Average duration of the projection GEMMs of one decode step of the current
 * wave, in the launch mode the rollout uses: the step's projection launches
 * (per layer QKV, O, gate/up with SwiGLU, down; then the LM head, into
 * d_logits, fp32 [n_seqs, vocab]) are captured as one HIP graph and replayed
 * reps times between two HIP events on the context's stream.  (Where the
 * rollout's O and down add to the residual stream, above 64 rows, they write
 * to the workspace here.)  Only the
 * split-K workspace, the SwiGLU output and d_logits are written (the wave's
 * KV cache, residual stream and positions are untouched).  out: launches per
 * step, average microseconds per launch, algorithmic bytes (weights once,
 * activations and outputs once) and flops per launch on average.
 * Errors: EINVAL (reps < 1, NULL; int4 weights with more than 64 rows in the
 * wave, whose projections dequantise first), ESTATE (no wave), EDEVICE. */
typedef struct {
  int32_t launches;
  double avg_us;
  double bytes_per_launch;
  double flops_per_launch;
} rollout_projection_profile;
rollout_status rollout_profile_projections(rollout_ctx* ctx, int32_t reps, float* d_logits,
                                           rollout_projection_profile* out);

#ifdef __cplusplus
}
#endif
#endif /* ROLLOUT_H */
