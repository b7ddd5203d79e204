/*
 * vla.h -- C-ABI of the MI355X (gfx950) library for the batched VLA policy rollout step and
 * the PPO/GRPO log-probability recompute.
 *
 * The operations follow the paper's statement of the problem:
 *   - generation: at every simulator step the policy infers an action (chunk) from the current
 *     observation, a_t ~ pi_theta(. | o_t), for all parallel environments (sections III-A,
 *     III-C); an atomic action is M tokens, one per action dimension, a chunk is C atomic
 *     actions (section III-B);
 *   - token-level log-probabilities pi(d_{t,i,j} | o_t, d_{t,i,:j-1}) (section IV-C.1);
 *   - the recompute of log pi_theta on stored (o_t, a_t) that the importance ratio
 *     rho = pi_theta / pi_theta_old of the PPO and GRPO objectives needs (appendix I-B, I-C);
 *   - a lightweight value head attached to the language model (section IV-C.2).
 * The decoder itself is a Llama-style pre-norm transformer (RMSNorm, rotary with half-split
 * pairing, multi-head causal attention without biases, SwiGLU); action tokens are the last
 * n_bins = 256 vocabulary ids and every distribution is over those 256 bins only.
 *
 * Conventions for every function below
 *   - Pointers marked DEVICE are device memory owned by the caller; pointers marked HOST are
 *     host memory.  The three hot calls never allocate or free device memory.
 *   - All device work is enqueued on `stream` (a hipStream_t passed as void*; NULL is the
 *     default stream).  No call synchronises; outputs are valid once the caller has
 *     synchronised the stream.  Calls that share a KV buffer or workspace must be ordered by
 *     the caller (same stream, or events).
 *   - Return value: VLA_OK (0) or a negative error code.  On error nothing has been enqueued
 *     (except for VLA_EHIP, which reports a failed launch) and vla_last_error() returns a
 *     thread-local, NUL-terminated HOST string describing it.  No exception crosses the ABI.
 *   - "dtype" below means the storage type selected by vla_config.dtype: float (VLA_DTYPE_F32)
 *     or bfloat16 (VLA_DTYPE_BF16).  Weight matrices, patch embeddings, slot embeddings and the
 *     KV cache use it; norm gains, the value head, noise and every output are fp32.
 *     Accumulation, the residual stream, norms, softmax and the action-bin head are fp32.
 *   - Weight matrices are row-major [out, in].
 */
#ifndef VLA_H
#define VLA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define VLA_VERSION 1

#define VLA_OK          0
#define VLA_EINVAL     (-1)  /* null pointer, negative or zero size, bad enum              */
#define VLA_ESHAPE     (-2)  /* exceeds max_batch / max_seq, or unsupported dimensions      */
#define VLA_EWORKSPACE (-3)  /* workspace (or KV buffer) smaller than required              */
#define VLA_EDTYPE     (-4)  /* unknown dtype                                               */
#define VLA_EHIP       (-5)  /* a HIP call or kernel launch failed                          */

#define VLA_DTYPE_F32  0
#define VLA_DTYPE_BF16 1

#define VLA_MODE_AR             0  /* autoregressive: token j+1 conditioned on tokens 1..j   */
#define VLA_MODE_PARALLEL_CHUNK 1  /* all A slots in one forward, bidirectional among slots  */

#define VLA_ENTRY_PREFILL   0
#define VLA_ENTRY_DECODE    1
#define VLA_ENTRY_RECOMPUTE 2

#define VLA_N_BINS 256

typedef struct vla_config {
    int32_t n_layers, hidden, n_heads, ffn, vocab;
    int32_t n_bins;      /* must be 256; bin k is token id vocab - 256 + k                   */
    int32_t dtype;       /* VLA_DTYPE_*                                                      */
    float   rms_eps;     /* RMSNorm epsilon                                                  */
    float   rope_theta;  /* rotary base                                                      */
    int32_t max_batch;   /* capacity: sequences per call                                     */
    int32_t max_seq;     /* capacity: positions per sequence (prefix + action rows); also the
                            position stride of the KV buffer                                 */
    int32_t value_dim;   /* outputs of the value head: 1 = one scalar per observation (chunk-level
                            value), C = one value per atomic action of the chunk (action-level
                            value, section IV-C.2); 0 is read as 1                            */
} vla_config;

/* DEVICE pointers.  attn_norm, ffn_norm: fp32 [hidden].  wq, wk, wv, wo: dtype [hidden, hidden].
 * w_gate, w_up: dtype [ffn, hidden].  w_down: dtype [hidden, ffn]. */
typedef struct vla_layer_weights {
    const void *attn_norm, *wq, *wk, *wv, *wo, *ffn_norm, *w_gate, *w_up, *w_down;
} vla_layer_weights;

/* embed, lm_head: DEVICE dtype [vocab, hidden] (only the last 256 rows of lm_head are read).
 * final_norm: DEVICE fp32 [hidden].  value_w: DEVICE fp32 [value_dim, hidden] or NULL (no value head).
 * value_b: scalar bias added to every value output; value_bias: DEVICE fp32 [value_dim] added per
 * output, or NULL.  layers: HOST array of n_layers entries, copied by vla_create. */
typedef struct vla_weights {
    const void *embed, *lm_head, *final_norm, *value_w;
    float value_b;
    const vla_layer_weights *layers;
    const void *value_bias;
} vla_weights;

typedef struct vla_model vla_model;

int vla_version(void);

/* HOST string describing the calling thread's last error ("" if none). */
const char *vla_last_error(void);

/* Create a host-side model object.  It stores the configuration and the weight POINTERS only;
 * the weights stay owned by the caller and must outlive the model.  Checks the dimensions:
 * hidden = n_heads * head_dim with head_dim a multiple of 16 and at most 256; n_bins = 256
 * <= vocab; positive sizes.  Touches no device. */
int vla_create(const vla_config *cfg, const vla_weights *weights, vla_model **out);
int vla_destroy(vla_model *model);

/* Optional repacked copy of the decoder-layer projection weights for the multi-row (prefill, parallel chunk,
 * recompute) forwards of bf16 models.  The large GEMM loads its operands straight into LDS; with the weights
 * stored [K / 32][rows][32] instead of row-major [rows, K] every such load reads whole cache lines.
 * vla_prepack_bytes: size of the copy for this configuration, 0 if the configuration has no use for it
 *   (fp32 storage, head_dim other than 128, widths that are not tile aligned).
 * vla_prepack: enqueues the repack of all layers on `stream` into `buffer` (DEVICE, 256-byte aligned, at least
 *   vla_prepack_bytes bytes, caller owned) and makes the model use it from then on; the caller orders later
 *   calls after it (same stream, or events) and keeps the buffer alive and unchanged while the model uses it.
 *   buffer = NULL detaches.  Decode forwards stream the copy too where they can, the original weights stay in use
 *   elsewhere (tail rows, the backward).  Results with and without the copy are bit-identical. */
size_t vla_prepack_bytes(const vla_config *cfg);
int vla_prepack(vla_model *model, void *buffer, size_t bytes, void *stream);

/* Bytes of the caller-allocated KV buffer for B sequences of up to max_pos positions
 * (max_pos <= cfg->max_seq; the buffer is always laid out with cfg->max_seq positions per
 * sequence, so the same B must be used by every call sharing it).  Layout is opaque.
 * Returns 0 on invalid arguments (see vla_last_error). */
size_t vla_kv_bytes(const vla_config *cfg, int B, int max_pos);

/* Bytes of workspace the given entry point needs for B sequences, prefix length S and A action
 * tokens (for VLA_ENTRY_RECOMPUTE, B is the number of stored rollouts N; the call processes
 * them in micro-batches, so the size stops growing beyond an internal micro-batch).  The
 * workspace holds no state between calls.  Returns 0 on invalid arguments. */
size_t vla_workspace_bytes(const vla_config *cfg, int entry, int B, int S, int A);

/* Prefill (sections III-A, III-C: the observation o_t enters the policy).  For each of B
 * environments, the prefix rows x_p = patch[p] (p < P), x_{P+t} = embed[ids[t]] run through all
 * decoder layers with causal attention; K and V of every prefix row are written to `kv`.
 *   kv        DEVICE, >= vla_kv_bytes(cfg, B, P+T)        ws  DEVICE workspace, ws_bytes long
 *   patch     DEVICE dtype [B, P, hidden] (P may be 0)     ids DEVICE int32 [B, T] in [0, vocab)
 *   h_last    DEVICE fp32 [B, hidden] out: final-norm output of the last prefix row
 *   value     DEVICE fp32 [B, value_dim] out or NULL: value_w . h_last + bias (section IV-C.2)
 * Requires P + T >= 1, B <= max_batch, P + T <= max_seq, and B * (P + T) rows within what one
 * pass can hold: the residual stream [rows, hidden] fp32 and the widest activation
 * [rows + 256 + pad, max(hidden, ffn)] in the storage dtype each below 2 GiB (32-bit byte
 * offsets in the kernels; 97,254 rows at the 7B shape in bf16).  Beyond that VLA_ESHAPE: split
 * the batch over several calls (each with its own kv). */
int vla_prefill(vla_model *model, void *kv, void *ws, size_t ws_bytes,
                const void *patch, const int32_t *ids, int B, int P, int T,
                float *h_last, float *value, void *stream);

/* Decode A action tokens per environment after vla_prefill on the same kv with the same B
 * (section III-C generation; token factorisation of section IV-C.1).
 *   mode VLA_MODE_AR: token 1 is read from h_last; for j = 1..A-1 token id vocab-256+bin_j is
 *     embedded at position S+j-1 and run through the decoder against the cache (its K, V are
 *     appended); token j+1 is read from that row.  The sampled bin feeds the next forward on
 *     the device.  The last token is not fed back.
 *   mode VLA_MODE_PARALLEL_CHUNK: one forward over A slot rows with inputs slot_embed[s] at
 *     positions S+s; slot rows attend to all S prefix rows and all A slot rows; slot s is read
 *     from its own row.  h_last is ignored.
 *   For every token: y = z / temperature over the 256 bins, bin = argmax_k (y_k + gumbel_k)
 *   (lowest k wins ties; gumbel NULL = greedy), logp = y_bin - logsumexp(y),
 *   entropy = -sum_k p_k log p_k (nats).
 *   h_last     DEVICE fp32 [B, hidden] from vla_prefill    S   prefix length P+T of that prefill
 *   slot_embed DEVICE dtype [A, hidden] (mode 1) or NULL   temperature > 0
 *   gumbel     DEVICE fp32 [B, A, 256] or NULL
 *   bins       DEVICE int32 [B, A] out                     logp, entropy DEVICE fp32 [B, A] out
 *   logits     DEVICE fp32 [B, A, 256] out or NULL: untempered z, for parity checks
 * Requires A >= 1 and S + A - 1 <= max_seq (mode 0), S + A <= max_seq (mode 1); mode 1 also
 * B * A rows within one pass (see vla_prefill). */
int vla_decode_actions(vla_model *model, void *kv, void *ws, size_t ws_bytes,
                       const float *h_last, int B, int S, int A, int mode,
                       const void *slot_embed, float temperature, const float *gumbel,
                       int32_t *bins, float *logp, float *entropy, float *logits, void *stream);

/* Log-probability recompute for the policy update (appendix I-B: rho needs log pi_theta of
 * the stored actions under the current weights).  Teacher-forced forward over N stored
 * rollouts without a persistent KV cache.
 *   mode VLA_MODE_AR: rows = prefix, then the stored tokens 1..A-1 (S + A - 1 rows, causal);
 *     token j is read from row S + j - 2 (1-based j).
 *   mode VLA_MODE_PARALLEL_CHUNK: rows = prefix, then the A slot inputs; prefix rows causal,
 *     slot rows see all rows.
 *   bins   DEVICE int32 [N, A], each in [0, 256): the stored actions
 *   logp   DEVICE fp32 [N, A] out: log-prob of the stored bin at the given temperature
 *   entropy DEVICE fp32 [N, A] out      value DEVICE fp32 [N, value_dim] out or NULL (last prefix row)
 *   logits DEVICE fp32 [N, A, 256] out or NULL
 * N may exceed max_batch: rollouts are processed in internal micro-batches of max_batch rollouts
 * (fewer if that many rows do not fit one pass, see vla_prefill) and the result does not depend
 * on the split. */
int vla_logprob_recompute(vla_model *model, void *ws, size_t ws_bytes,
                          const void *patch, const int32_t *ids, const int32_t *bins,
                          int N, int P, int T, int A, int mode, const void *slot_embed,
                          float temperature, float *logp, float *entropy, float *value,
                          float *logits, void *stream);

/* ---- profiling (auxiliary; process-wide, not thread safe) --------------------------------------
 * While enabled, every kernel launch of the three hot calls is bracketed by a pair of HIP events
 * recorded on the launch stream, tagged with a label and with the launch's algorithmic work (flops
 * for contractions, bytes for streaming kernels).  Events add a few microseconds per launch, so
 * timed throughput runs keep profiling off.
 *   vla_profile_enable(on)   turn recording on (1) or off (0); turning it on clears old records.
 *   vla_profile_report(buf, n) synchronises the recorded events and writes, into the HOST buffer
 *     buf of n bytes, one line per label: "label count total_ms total_work" (NUL terminated,
 *     truncated to n).  Returns the number of labels, or a negative error code. */
int vla_profile_enable(int on);
int vla_profile_report(char *buf, size_t n);

/* Triage aid (process-wide, not thread safe): a bit mask of steps that take the shape-generic kernel even where a
 * gfx950 fast path applies -- 1 large GEMM, 2 decode GEMM, 4 multi-row attention, 8 decode attention, 16 rotary / KV
 * write / RMSNorm; in the gradient pass 1 also takes the LoRA products, 4 the attention, 16 the rotation and SwiGLU that
 * ride their projections; 0 (the default) selects every fast path.  Results stay within the parity tolerances either way;
 * the tests use it to run the generic kernels on shapes that would otherwise never reach them. */
int vla_debug_force_generic(int mask);

/* Calibration aid for hardware-counter runs: a plain copy kernel (`bytes` must be a multiple of 16;
 * dst, src DEVICE, 16-byte aligned) that reads and writes exactly `bytes` bytes, so that HBM
 * traffic counters collected around the hot kernels can be scaled by what they read for it. */
int vla_calibration_copy(void *dst, const void *src, size_t bytes, void *stream);

/* ---- consumers of the recomputed log-probabilities in the policy update ------------------------
 * All arrays DEVICE fp32 (flags and masks int32), row-major; launches on `stream`, no sync.  Sums are
 * taken in a fixed order (no atomics), so results are bit-reproducible.
 *
 * vla_gae -- generalized advantage estimation (appendix I-B):
 *   delta_t = r_t + gamma V(s_{t+1}) - V(s_t),  A_t = sum_k (gamma lambda)^k delta_{t+k}.
 *   rewards [n, T]; values [n, T+1] (column T bootstraps the last step); dones [n, T] or NULL: a
 *   non-zero done_t ends an episode at step t inside the row (partial reset), cutting both the
 *   bootstrap term and the sum.  Outputs adv [n, T] and returns = adv + V [n, T] (returns may be NULL).
 *
 * vla_grpo_advantage -- group-relative advantage (appendix I-C): for each group of G consecutive
 *   trajectories A_i = (R_i - mean) / std with the population standard deviation.  total_reward
 *   [n_groups * G]; adv out, same shape; keep [n_groups] out or NULL: 0 for groups whose returns are
 *   all equal (advantages 0; the success-rate filter of section IV-C.3 drops them), else 1.
 *
 * vla_policy_objective -- clipped surrogate of PPO / GRPO (appendix I-B, I-C, II-C.2):
 *   s = min(rho A, clip(rho, 1 - clip_low, 1 + clip_high) A), rho = exp(logp_new - logp_old).
 *   logp_new, logp_old [n_traj, T]; adv [n_traj, T] if adv_per_step else [n_traj]; mask [n_traj, T]
 *   (non-zero = valid step) or NULL.  per_trajectory = 0: objective = mean of s over all valid steps
 *   (PPO's E_t); 1: (1/n_traj) sum_i (1/T_i) sum_t s with T_i the valid steps of trajectory i (GRPO
 *   with the valid-action mask; a trajectory without valid steps contributes 0).
 *   ws: DEVICE scratch of vla_policy_objective_workspace_bytes(n_traj) bytes.
 *   Outputs: objective [1]; per_step [n_traj, T] or NULL (masked s); clip_frac [1] or NULL (share of
 *   valid steps where the clipped branch is the smaller one).
 *
 * vla_logp_aggregate -- log-probability granularity (section IV-C.1): out[i] = sum of the `inner`
 *   consecutive entries logp[i * inner ...], i < n_out: token -> action with inner = tokens per action,
 *   action -> chunk with inner = actions per chunk. */
int vla_gae(const float *rewards, const float *values, const int32_t *dones, int n, int T, float gamma,
            float lambda, float *adv, float *returns, void *stream);
int vla_grpo_advantage(const float *total_reward, int n_groups, int G, float *adv, int32_t *keep, void *stream);
size_t vla_policy_objective_workspace_bytes(int n_traj);
int vla_policy_objective(const float *logp_new, const float *logp_old, const float *adv, int adv_per_step,
                         const int32_t *mask, int n_traj, int T, float clip_low, float clip_high,
                         int per_trajectory, void *ws, size_t ws_bytes, float *objective, float *per_step,
                         float *clip_frac, void *stream);
int vla_logp_aggregate(const float *logp, size_t n_out, int inner, float *out, void *stream);

/* ---- backward pass of the log-probability recompute: LoRA gradients (section IV-B.2; appendix I-B, I-C) -------------
 * The policy update differentiates the clipped surrogate through rho = exp(logp_theta - logp_old) only, so what it
 * needs from the model is the gradient of  L = sum_{n,j} coef[n,j] * logp_theta[n,j]  with coef = dJ/dlogp (rho * A-hat
 * where the unclipped branch is active, 0 elsewhere; the per_step output of vla_policy_objective times the caller's
 * normalisation).  The trainable parameters are the LoRA factors of the seven projections of every decoder layer:
 * W_eff = W + scale * B A, A [rank, in], B [out, rank].  The model's weights are the EFFECTIVE ones (the caller keeps
 * them merged); with X a projection's input and dY the gradient at its output,
 *     dL/dB = scale * dY^T (X A^T)   [out, rank],      dL/dA = scale * (dY B)^T X   [rank, in].
 * Embeddings, norm gains, the action head and the value head are frozen.
 *
 * vla_lora_layer: DEVICE pointers, storage dtype, per projection a [rank, in] and b [out, rank]
 *   (in / out: hidden / hidden for q, k, v, o; hidden / ffn for gate, up; ffn / hidden for down).
 * vla_lora_layer_grads: DEVICE fp32 outputs of the same shapes, overwritten.
 * vla_logprob_backward: teacher-forced forward over the N stored rollouts exactly as vla_logprob_recompute (same
 *   arguments, same modes), then the backward.  lora, grads: HOST arrays of n_layers entries.  coef DEVICE fp32 [N, A].
 *   logp DEVICE fp32 [N, A] out or NULL: the forward's log-probabilities of the stored bins (equal to the output of
 *   vla_logprob_recompute up to the rounding differences of two evaluations).  Rollouts are processed in
 *   micro-batches of max_batch; gradients are summed over micro-batches in order, every sum in a fixed order, so the
 *   result is reproducible bit for bit.  Gradient operands of the GEMMs are rounded to the storage dtype.
 *   keep_activations = 0: the first pass runs the lower layers with the kernels of vla_logprob_recompute, keeping the
 *   residual stream at every layer input, and the top one or two (two where 4 A is at most the rows of a rollout and the
 *   workspace has room) with the unfused kernels, which leave what their backward reads; the lower ones are run a second
 *   time for theirs.  ws: DEVICE, at least vla_backward_workspace_bytes(cfg, N, P + T, A, rank) bytes (grows with
 *   max_batch; 11.7 GB at the 7B shape with max_batch 32).  keep_activations = 1: the first pass keeps what every layer's
 *   backward reads for one micro-batch and no layer is run twice; ws at least vla_backward_keep_workspace_bytes(...) bytes
 *   (78 GB there): for GPUs with memory to spare.  Same gradients up to rounding (all layers then use the unfused kernels). */
typedef struct { const void *a, *b; } vla_lora_factor;
typedef struct { vla_lora_factor q, k, v, o, gate, up, down; } vla_lora_layer;
typedef struct { float *da, *db; } vla_lora_grad;
typedef struct { vla_lora_grad q, k, v, o, gate, up, down; } vla_lora_layer_grads;
size_t vla_backward_workspace_bytes(const vla_config *cfg, int N, int S, int A, int rank);
size_t vla_backward_keep_workspace_bytes(const vla_config *cfg, int N, int S, int A, int rank);
int vla_logprob_backward(vla_model *model, void *ws, size_t ws_bytes, const void *patch, const int32_t *ids,
                         const int32_t *bins, const float *coef, int N, int P, int T, int A, int mode,
                         const void *slot_embed, float temperature, int rank, float scale, int keep_activations,
                         const vla_lora_layer *lora, const vla_lora_layer_grads *grads, float *logp, void *stream);

/* vla_policy_objective_noalloc -- vla_policy_objective for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): same arguments without the workspace,
 * same kernels, same results bit for bit.  The per-trajectory partial sums live in an array built into the library
 * (786,432 bytes of device memory per GPU, held until the process ends), so n_traj is limited to
 * vla_policy_objective_noalloc_max_traj() = 65,536; beyond that VLA_ESHAPE and nothing is enqueued.  The call
 * allocates and frees nothing, on the device or through any library; the first call on a GPU looks the array's
 * address up once (hipGetSymbolAddress).  Every call on one GPU shares that GPU's array: two calls that overlap in
 * time on the same GPU (different streams or threads) race and must be ordered by the caller.  Nothing of an
 * earlier call is read: every slot the second kernel reads is written by the first. */
int vla_policy_objective_noalloc_max_traj(void);
int vla_policy_objective_noalloc(const float *logp_new, const float *logp_old, const float *adv, int adv_per_step,
                                 const int32_t *mask, int n_traj, int T, float clip_low, float clip_high,
                                 int per_trajectory, float *objective, float *per_step, float *clip_frac,
                                 void *stream);

/* ---- paged KV cache: append, attention, sampling (generation, section III-C, over ragged batches) ----------------------
 * The rollout calls above serve batches of one prefix length on a cache of their own layout.  These serve sequences of any
 * lengths on pages that the caller hands out, and decoders with grouped heads, norms of q and k, capped scores, biases by
 * distance, prefix masks and windows.  Token ids and positions are whole numbers below 2^31; sizes below are per call.
 *
 * vla_paged_cache: one layer's cache.  k, v: DEVICE dtype [n_pages][n_kv_heads][page_size][head_dim], 16-byte aligned;
 *   page_size a power of two from 16 to 1024; head_dim a multiple of 16, at most 256.  Position p of a sequence lies in page
 *   page_table[sequence][p / page_size], row p % page_size.
 * vla_paged_batch: rows of n_seq sequences, one after the other: sequence s has rows row_start[s] .. row_start[s + 1] - 1
 *   (row_start ascending from 0), the newest of its kv_len[s] positions: row i of its n_s rows is at position
 *   kv_len[s] - n_s + i.  A sequence may have no rows.  Rows from row_start[n_seq] to n_rows - 1 are padding: whatever they
 *   hold changes nothing, and nothing is written for them.  max_rows, max_len (HOST): bounds of n_s and kv_len that the launches are sized by; work beyond them is left out, and so are
 *   pages whose id is not in [0, n_pages): the rows are not written, and read as zeros.  The arrays are read on the device, so a captured call follows them as they change.
 *   table_stride: entries per sequence in page_table, at least max_len / page_size rounded up; entries of pages that hold no
 *   visible position are never read.
 *   page_table must not give one page to two sequences that both write to it (sequences may read shared pages).
 *
 * vla_paged_append: the new rows' q, k and v (outputs of a projection, in_dtype, row strides in elements, heads packed within
 *   a row) -> K and V in their pages and q_out, in the cache's dtype.  Per head of q and of k: x / sqrt(mean(x^2) + eps) * gain
 *   where a gain is given, then the rotation of the first rot_dim dims by position * inv_freq[i]: of the pairs (i, i + rot_dim / 2),
 *   or (2 i, 2 i + 1) where interleaved; cos and sin times `scale`.  v is rounded alone.  fp32 arithmetic, angles in fp64,
 *   one rounding at the end.  q and q_out may both be NULL (k and v alone), and q_out may be q itself (same dtype and stride).
 *   Rows at negative positions (kv_len[s] < n_s) are left out.
 *   vla_rotary: inv_freq DEVICE fp64 [rot_dim / 2] (scaled as the model has it; NULL with rot_dim 0), rot_dim even, at most
 *   head_dim; q_gain, k_gain DEVICE fp32 [head_dim] or NULL.
 *
 * vla_paged_attention: rows q [n_rows, n_heads, head_dim] (the cache's dtype, row stride in elements; n_heads a multiple of
 *   n_kv_heads, heads of a group consecutive) against the pages, which already hold the new rows' K and V.  With p the row's
 *   position and j a key's:  s = scale q.k,  s = softcap tanh(s / softcap) (softcap > 0),  s -= slopes[head] |p - j| (slopes not
 *   NULL);  visible are j < kv_len with  (j <= p and (window == 0 or j > p - window))  or  j < prefix_len[sequence];
 *   out = sum softmax(s) v, fp32 sums; weights enter the products with v with 16 bits at least, but on a bf16 cache as bf16 where
 *   n_heads / n_kv_heads times max_rows is above 32 (prompts).  lse (fp32 [n_rows, n_heads] or NULL) = ln sum exp(s).  A row that sees no
 *   key gets zeros and -inf; a head of a row with a visible score that is NaN or +inf gets NaN in both, however the keys are split (so
 *   may one with an infinite k whose score is -inf).  K and V of visible positions are taken to be finite where any row of the call masks them.
 *   vla_paged_mask: scale > 0; softcap, window >= 0; slopes DEVICE fp32 [n_heads]; prefix_len DEVICE int32 [n_seq]; shared_len
 *   (HOST): a multiple of page_size; the first shared_len positions of all sequences lie in the same pages, which are read once
 *   for the whole batch, through sequence 0's table (sequence 0 and every sequence with rows hold shared_len positions
 *   or more); not together with a window.
 *   out does not overlap q.  ws: DEVICE, 16-byte aligned, of vla_paged_attention_workspace_bytes (from HOST numbers alone) bytes: partial sums of
 *   split key ranges; no state, but calls that overlap in time need one each.
 *   Sums are added in a fixed order: the same call gives the same bits; the split depends on the HOST numbers.
 *
 * vla_sample_logits: one token per row of logits (DEVICE dtype [n, vocab], row stride in elements), vocab at most 262,144.
 *   With T = temperature[i] and w_k = exp((z_k - max z) / T):  of the tokens the top_k[i] largest are kept (ties: lowest id first;
 *   <= 0: all), of these the shortest leading run, largest first, that holds top_p[i] of their mass (>= 1: all), of these those
 *   with w_k >= min_p[i] (above 1: 1).  token[i] = the lowest id at which the kept tokens' running mass, in id order, exceeds u[i] times its
 *   total; u in [0, 1).  T <= 0, or u NULL: the largest (lowest id).  The largest is always kept; NaN and -inf never are; where +inf occurs only
 *   those are, at equal weights.  A row without any gets token -1, n_kept 0 and log-probabilities -inf.
 *   temperature, top_p, min_p, u: DEVICE fp32 [n]; top_k DEVICE int32 [n]; each may be NULL (1, all, all, greedy, all).
 *   logp (or NULL): log-probability under softmax(z / T), as the recompute gives it; logp_kept (or NULL): among the kept tokens;
 *   n_kept (or NULL).  With T <= 0 or u NULL the cuts still apply to n_kept and logp_kept; T <= 0 counts as 1 in all of them.  Masses are summed as 64-bit fixed point numbers,
 *   in any order the same, so equal inputs give equal tokens.  ws: DEVICE, of vla_sample_logits_workspace_bytes bytes. */
/* vla_forward_paged: the decoder over a ragged batch's new rows: a prefill of prefixes of any lengths, a decode step, or both at once.
 *   Row r is the embedding of token ids[r], or, where ids[r] < 0, row -1 - ids[r] of patch (DEVICE dtype [n_patch, hidden]; ids and rows out of
 *   range are clamped).  Every layer appends its K and V to its cache, layer l at cache->k, v + l * layer_stride elements, and attends:
 *   causally, but for positions below prefix_len[sequence] (or NULL), which every row sees; shared_len as in vla_paged_mask.  The cache
 *   has the model's dtype, heads and head_dim; any max_len (the model's max_batch and max_seq do not bind it).
 *   h_last  DEVICE fp32 [n_seq, hidden] out: final-norm output of each sequence's last new row (zeros' where it has none)
 *   logits  DEVICE fp32 [n_seq, 256] out or NULL: the action bins' (token id vocab - 256 + bin), what vla_sample_logits takes
 *   value   DEVICE fp32 [n_seq, value_dim] out or NULL
 *   ws      DEVICE, of vla_forward_paged_workspace_bytes bytes.  n_rows within one pass (see vla_prefill). */
typedef struct vla_paged_cache {
    void *k, *v;
    int32_t dtype, n_pages, page_size, n_kv_heads, head_dim;
} vla_paged_cache;
typedef struct vla_paged_batch {
    int32_t n_seq, n_rows, max_rows, max_len, table_stride;
    const int32_t *row_start, *kv_len, *page_table;   /* DEVICE [n_seq + 1], [n_seq], [n_seq, table_stride] */
} vla_paged_batch;
typedef struct vla_rotary {
    const double *inv_freq;
    int32_t rot_dim, interleaved;
    float scale, eps;
    const float *q_gain, *k_gain;
} vla_rotary;
typedef struct vla_paged_mask {
    float scale, softcap;
    const float *slopes;
    const int32_t *prefix_len;
    int32_t window, shared_len;
} vla_paged_mask;
/* The largest tree of drafted rows of one sequence, and the most pages of a sequence that are chosen from. */
#define VLA_TREE_ROWS 1024
#define VLA_SELECT_PAGES 8192
int vla_paged_append(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_rotary *rotary, const void *q,
                     const void *k, const void *v, int in_dtype, int n_heads, int64_t q_stride, int64_t k_stride,
                     int64_t v_stride, void *q_out, int64_t q_out_stride, void *stream);
size_t vla_paged_attention_workspace_bytes(const vla_paged_cache *cache, const vla_paged_batch *batch,
                                           const vla_paged_mask *mask, int n_heads);
int vla_paged_attention(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask, const void *q,
                        int n_heads, int64_t q_stride, void *out, int64_t out_stride, float *lse, void *ws, size_t ws_bytes,
                        void *stream);
size_t vla_sample_logits_workspace_bytes(int n, int vocab);
size_t vla_forward_paged_workspace_bytes(const vla_config *cfg, const vla_paged_cache *cache, const vla_paged_batch *batch,
                                         int shared_len);
int vla_forward_paged(vla_model *model, const vla_paged_cache *cache, size_t layer_stride, const vla_paged_batch *batch,
                      const int32_t *ids, const void *patch, int n_patch, const int32_t *prefix_len, int shared_len, void *ws,
                      size_t ws_bytes, float *h_last, float *logits, float *value, void *stream);
int vla_sample_logits(const void *logits, int dtype, int64_t row_stride, int n, int vocab, const float *temperature,
                      const int32_t *top_k, const float *top_p, const float *min_p, const float *u, int32_t *token,
                      float *logp, float *logp_kept, int32_t *n_kept, void *ws, size_t ws_bytes, void *stream);

/* ---- reading less per token: drafted trees, sparse pages, eviction --------------------------------------------------------
 * A decode step on the paged cache reads all K and V of a sequence for one token.  These take several drafted tokens through one such
 * step, read only the pages that matter to a row, or cut the cache to the positions that mattered.  Cache, batch, mask, padding, page ids
 * out of range, streams and workspaces are as above.
 *
 * vla_paged_append_at: vla_paged_append with the rotation's position of every row in `position` (DEVICE int32 [n_rows], not negative)
 *   instead of its place in the cache: a drafted node's is its depth behind the cache, and behind a cache that was cut places have moved.
 *
 * Drafted trees.  The new rows of a sequence (n_s of them, at most VLA_TREE_ROWS) are the nodes of a tree: the first is the last committed
 * token, the others drafts, each behind its parent.  parent: DEVICE int32 [n_rows], the parent's number among the sequence's rows, smaller
 * than the node's own (of the first row, and wherever it is not in 0 .. i - 1: none, the node stands on the cache itself).
 * vla_paged_tree: seen [n_rows][words] out, DEVICE int32: bit j % 32 of word j / 32 says that the row sees its sequence's new row j: its
 *   ancestors and itself; position [n_rows] out or NULL: kv_len - n_s + depth.  words: at least max_rows / 32 rounded up, at most 32.
 * vla_paged_tree_attention: as vla_paged_attention, but a row sees the positions below kv_len - n_s and of the new rows those whose
 *   bits are set in its `seen` (any bits: not only a tree's; K and V of the new rows are finite).  mask: scale, softcap and shared_len (at most kv_len - n_s of every sequence with rows) alone;
 *   slopes and prefix_len NULL, window 0.  On a bf16 cache weights enter the products with v with 16 bits whatever the number of rows.
 *   ws: of vla_paged_attention_workspace_bytes bytes.
 * vla_paged_accept: the drafts that the model agrees with.  ids: DEVICE int32 [n_rows], the rows' tokens; chosen: DEVICE int32
 *   [n_rows], the model's own token behind each row (vla_sample_logits of its logits).  From the first row on, the path goes to the
 *   lowest row whose parent is the path's last and whose id is what that chose (a negative choice: none), until there is none.  path
 *   [n_seq, max_rows] out: the rows of the path, then -1; n_accepted [n_seq] out: how many; next [n_seq] out or NULL: what the last of
 *   them chose (-1 without rows); new_len [n_seq] out or NULL: kv_len - n_s + n_accepted.  In each of n_layers layers, layer l at
 *   cache->k, v + l * layer_stride elements, K and V of row path[i] move to position kv_len - n_s + i (n_layers may be 0: nothing moves).  The rows behind
 *   new_len keep what they hold.  No output overlaps parent, ids, chosen, kv_len or row_start.  The pages of the new rows belong to their sequence alone.  Rows at negative positions are nowhere, and new_len is not below 0.
 *   Page bounds that a caller keeps (below) are behind it those of rows that have left or moved: vla_paged_bounds, with n_accepted's running sums as row_start, new_len as
 *   kv_len and the other numbers of this batch, computes those from position kv_len - n_s on again.  Mass (below) of
 *   these positions is the caller's to set, for no weights of a tree's rows are summed.
 *
 * Sparse attention over pages.
 * vla_paged_bounds: bounds, DEVICE cache's dtype [n_pages][n_kv_heads][2][head_dim], 16-byte aligned: the least and the largest K of each dim over the
 *   positions below kv_len of a page, for every page that holds one of the batch's rows (positions kv_len - n_s on; a batch whose rows
 *   are all positions: every page).  K of these positions is finite; pages of other rows keep their bounds.
 * vla_paged_select: for each row and key head, the pages to read.  score(page) = sum over the heads h of the group and the dims of
 *   max(q_h lo, q_h hi), no less than the sum of the heads' q.k for any key of the page; fp64 (bounds are finite; q may not be).  Of the pages 0 .. p / page_size of a row at
 *   position p the first `first` and the last `recent` (at least 1) are taken, then those with the largest scores (ties: lowest page
 *   first; a score that is NaN comes last), until there are n_select (at least first + recent).  selected [n_rows][n_kv_heads][n_select]
 *   out, DEVICE int32: numbers of pages within the sequence, ascending, then -1.  Rows at negative positions get none.  max_len / page_size at most VLA_SELECT_PAGES.
 * vla_paged_sparse_attention: as vla_paged_attention, but a row's heads see the positions j <= p, j < kv_len of the pages in their `selected` alone
 *   (any ascending list; it ends at the first negative entry, and an entry not above the one before it is left out).  mask: scale and
 *   softcap alone.  Each row reads its own pages: for few rows per sequence.
 *
 * Eviction by accumulated weight.
 * vla_paged_weights: mass [n_seq][n_kv_heads][mass_stride], DEVICE fp32: to every position j < kv_len - n_s that a row sees is added, and every
 *   new position gets, the sum over the call's rows and the heads of the group of exp(s - lse), with s and the visibility of
 *   vla_paged_attention under the same mask (shared_len changes nothing) and lse its output [n_rows, n_heads].  A row whose lse is -inf adds nothing.
 *   mass_stride: at least max_len.  Sums in fp32 in a fixed order.
 * vla_paged_evict: each sequence and key head keeps `keep` positions: the first `first` and the last `recent`, then those of the largest
 *   mass (ties: lowest position first; NaN comes last); all where there are no more.  kept [n_seq][n_kv_heads][keep] out: positions,
 *   ascending, then -1.  K, V and mass of the i-th go to position i: K and V in page to_table[sequence][i / page_size] (to_stride entries per
 *   sequence, at least keep / page_size rounded up), mass to mass_out [n_seq][n_kv_heads][mass_out_stride] (mass itself with its stride, or apart
 *   from it; entries behind the last keep what they hold).  new_len [n_seq] out or NULL: min(kv_len, keep), apart from kv_len.  to_table's pages hold nothing that the call reads, but that a sequence
 *   with no more than `keep` may name its own pages again (nothing moves).  The bounds of to_table's pages are
 *   to be computed again (vla_paged_bounds of a batch whose rows are all positions).  One layer a call.  Of the batch it uses the sequences, not their rows. */
/* vla_forward_paged_rows: vla_forward_paged with these, and with the logits of every row (a tree's nodes are all read).
 *   position, seen (words to a row), prefix_len: as above, each or NULL; bounds: [n_layers] of vla_paged_bounds' arrays or NULL: kept up with the
 *   new rows (behind vla_paged_accept and vla_paged_evict: see there); n_select above 0 (bounds given): rows read the pages that vla_paged_select takes with first and recent; mass
 *   [n_layers][n_seq][n_kv_heads][mass_stride] or NULL: vla_paged_weights of every layer.  A tree, selected pages, and weights or a prefix mask exclude each other.
 *   logits  DEVICE fp32 [n_rows, 256] out (of padding rows: of no meaning).  ws: of vla_forward_paged_rows_workspace_bytes bytes. */
typedef struct vla_paged_rows {
    const int32_t *position, *seen, *prefix_len;
    void *bounds;
    float *mass;
    int64_t mass_stride;
    int32_t words, n_select, first, recent;
} vla_paged_rows;
size_t vla_forward_paged_rows_workspace_bytes(const vla_config *cfg, const vla_paged_cache *cache, const vla_paged_batch *batch,
                                              const vla_paged_rows *rows, int shared_len);
int vla_forward_paged_rows(vla_model *model, const vla_paged_cache *cache, size_t layer_stride, const vla_paged_batch *batch,
                           const vla_paged_rows *rows, const int32_t *ids, const void *patch, int n_patch, int shared_len, void *ws,
                           size_t ws_bytes, float *logits, void *stream);
int vla_paged_append_at(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_rotary *rotary, const int32_t *position,
                        const void *q, const void *k, const void *v, int in_dtype, int n_heads, int64_t q_stride, int64_t k_stride,
                        int64_t v_stride, void *q_out, int64_t q_out_stride, void *stream);
int vla_paged_tree(const vla_paged_cache *cache, const vla_paged_batch *batch, const int32_t *parent, int32_t *seen, int words, int32_t *position,
                   void *stream);
int vla_paged_tree_attention(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask, const int32_t *seen,
                             int words, const void *q, int n_heads, int64_t q_stride, void *out, int64_t out_stride, float *lse, void *ws,
                             size_t ws_bytes, void *stream);
int vla_paged_accept(const vla_paged_cache *cache, int n_layers, size_t layer_stride, const vla_paged_batch *batch, const int32_t *parent,
                     const int32_t *ids, const int32_t *chosen, int32_t *path, int32_t *n_accepted, int32_t *next, int32_t *new_len,
                     void *stream);
int vla_paged_bounds(const vla_paged_cache *cache, const vla_paged_batch *batch, void *bounds, void *stream);
size_t vla_paged_select_workspace_bytes(const vla_paged_cache *cache, const vla_paged_batch *batch);
int vla_paged_select(const vla_paged_cache *cache, const vla_paged_batch *batch, const void *bounds, const void *q, int n_heads,
                     int64_t q_stride, int n_select, int first, int recent, int32_t *selected, void *ws, size_t ws_bytes, void *stream);
size_t vla_paged_sparse_attention_workspace_bytes(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask,
                                                  int n_heads, int n_select);
int vla_paged_sparse_attention(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask,
                               const int32_t *selected, int n_select, const void *q, int n_heads, int64_t q_stride, void *out,
                               int64_t out_stride, float *lse, void *ws, size_t ws_bytes, void *stream);
size_t vla_paged_weights_workspace_bytes(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask, int n_heads);
int vla_paged_weights(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask, const void *q, int n_heads,
                      int64_t q_stride, const float *lse, float *mass, int64_t mass_stride, void *ws, size_t ws_bytes, void *stream);
int vla_paged_evict(const vla_paged_cache *cache, const vla_paged_batch *batch, const float *mass, int64_t mass_stride, int keep, int first,
                    int recent, const int32_t *to_table, int to_stride, int32_t *kept, float *mass_out, int64_t mass_out_stride,
                    int32_t *new_len, void *stream);

/* ---------------------------------------------------------------- GPU allocation modes (section IV-A)
 * Host-only arithmetic (no device work, all pointers HOST): the rollout-time model behind the
 * automatic placement.  One rollout epoch is m_chunks steps, each a Generation phase (t_gen for the
 * environments of one Generation GPU) followed by a Simulator phase (t_sim likewise).
 *
 * vla_pipeline_time -- k = 1, collocated mode: *out = m_chunks (t_gen + t_sim), the section's t_1.
 *   k = 2, hybrid mode with fine-grained pipelining: the environments are split in two sub-batches that
 *   take turns on the Generation and on the Simulator partition (times are then per sub-batch):
 *   *out = 2 m_chunks max(t_gen, t_sim) + min(t_gen, t_sim).  The section gives no formula for
 *   t_2, only that it is an estimate for pipelined execution; this is the makespan of the schedule it describes.  Other k: VLA_EINVAL.
 *
 * vla_profile_lookup -- profile[i] is a component's measured time at batch 2^i, i < n_prof (the
 *   section profiles batch sizes 2^0 ... n_S); other batches are interpolated linearly between the two
 *   neighbours.  batch < 1 or above 2^(n_prof-1): VLA_ESHAPE.
 *
 * vla_auto_placement -- min over k in {1, 2} and N_G + N_S = n_gpus of the rollout time.  k = 1 uses
 *   all n_gpus for both components with ceil(n_envs / n_gpus) environments each; k = 2 gives n_gen GPUs
 *   to Generation and n_sim = n_gpus - n_gen to the Simulator, each sub-batch holding
 *   ceil(n_envs / (2 n_gen)) resp. ceil(n_envs / (2 n_sim)) environments per GPU (splits that leave a
 *   GPU without an environment are skipped).  *best receives the fastest candidate (the first on ties,
 *   in the order k = 1, then n_gen = 1, 2, ...); if `all` is not NULL up to all_cap candidates are
 *   written in that order and *n_all (if not NULL) receives their total number. */
typedef struct {
    int32_t k;        /* pipeline stages: 1 collocated, 2 hybrid with pipelining */
    int32_t n_gen;    /* GPUs running Generation (all of them when k = 1)        */
    int32_t n_sim;    /* GPUs running the Simulator (all of them when k = 1)     */
    double time;      /* modelled time of one rollout epoch                       */
} vla_placement;
int vla_pipeline_time(double t_gen, double t_sim, int k, int m_chunks, double *out);
int vla_profile_lookup(const double *profile, int n_prof, double batch, double *out);
int vla_auto_placement(const double *t_gen, const double *t_sim, int n_prof, int n_envs, int n_gpus,
                       int m_chunks, vla_placement *best, vla_placement *all, int all_cap, int *n_all);

#ifdef __cplusplus
}
#endif
#endif /* VLA_H */
