/*
 * pda_ops.h -- the steps around attention in a rollout, log-prob and update
 * program, in the same library and with the conventions of pda.h (device
 * pointers owned by the caller, host checks before any HIP call, asynchronous on
 * `stream`, the stream's workspace, HIP graphs, pda_last_error(),
 * pda_read_device_status()).
 *
 *   before attention  norms of queries and keys per head and the position
 *                     rotation in one pass, into the paged cache (decode steps,
 *                     verification, chunked prefill, the log-prob forward) or
 *                     as a training forward, and its gradient
 *   after the model   log-probabilities and entropies of tokens from logits, and
 *                     the clipped policy loss with its gradient at the logits
 *
 * These are the attention inputs of the models of the paper's Sec. 6.1 and the
 * compute_log_prob and update_actor phases of its Table 2 (Sec. 6.3).
 */
#ifndef PDA_OPS_H
#define PDA_OPS_H

#include "pda.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Further bits of pda_read_device_status(): 32 = a position outside the table of
 * angles was clamped into it, 64 = a target at or past the vocabulary was
 * ignored. */

/* Sizes and types of the norm and rotation of queries and keys.
 *
 * For a head's row x [D] of a token at position p, with weights w:
 *     r = 1 / sqrt(mean x^2 + eps),  n = x r w       (n = x without weights)
 *     y_i = n_i cos - n_j sin,  y_j = n_j cos + n_i sin
 * over the pairs (i, j) of the head's first rotary_dim dims, i-th angle of row p
 * of the table: (i, i + rotary_dim / 2), or (2 i, 2 i + 1) if interleaved. Dims
 * past rotary_dim stay n. Arithmetic and sums are float32; results are rounded
 * once.
 *
 *   q            [T, Hq, D], k (and v) [T, Hkv, D] dtype: a token's heads are
 *                contiguous, tokens q_stride (k_stride, v_stride) elements apart,
 *                so that the parts of a packed projection need no copy
 *   q_weight, k_weight  [D] weight_dtype, both or neither (no norm)
 *   cos_sin      [max_positions, rotary_dim] f32: rotary_dim / 2 cosines, then as
 *                many sines
 *
 * Strides of 0 mean contiguous tokens. Pointers and strides must keep every row
 * 16-byte aligned. */
typedef struct pdaops_rope_problem {
  int32_t num_tokens;     /* T */
  int32_t num_q_heads;    /* Hq */
  int32_t num_kv_heads;   /* Hkv */
  int32_t head_dim;       /* D: 64 or 128 */
  int32_t rotary_dim;     /* a multiple of 16, at most D */
  int32_t max_positions;  /* rows of cos_sin */
  int32_t interleaved;    /* 0: pairs (i, i + rotary_dim / 2); 1: (2 i, 2 i + 1) */
  int32_t dtype;          /* q, k, v: PDA_DTYPE_F32 or PDA_DTYPE_BF16 */
  int32_t out_dtype;      /* rotated q and k: F32 or BF16 (the gradients have dtype) */
  int32_t weight_dtype;   /* F32 or BF16 */
  float eps;
  int64_t q_stride, k_stride, v_stride;
  int64_t q_out_stride, k_out_stride;    /* also of their gradients */
  int64_t grad_q_stride, grad_k_stride;  /* of the gradients of q and k */
} pdaops_rope_problem;

/* The paged cache that an append writes (layouts and limits of pda.h). */
typedef struct pdaops_cache {
  int32_t num_seqs;            /* B */
  int32_t block_size;          /* 16 */
  int32_t max_blocks_per_seq;  /* block_table row stride */
  int32_t max_seq_len;         /* host bound on seq_lens (0 = max_blocks_per_seq * 16) */
  int64_t num_blocks;
  int32_t kv_dtype;            /* PDA_DTYPE_F32, PDA_DTYPE_BF16 or PDA_DTYPE_FP8_E4M3 */
} pdaops_cache;

/*
 * The steps between the projections and attention, in one launch: norm and
 * rotation of the new tokens' queries and keys, keys and values written into the
 * paged cache.
 *
 *   q_offsets    [B + 1] int32, or NULL: T / B tokens of every sequence. Rows
 *                q_offsets[b] .. q_offsets[b+1]-1 are the last tokens of sequence
 *                b, as for pda_paged_prefill_attention
 *   seq_lens     [B] int32: lengths with the new tokens, as the attention call
 *                that follows takes them; token i of n_b sits at position
 *                seq_lens[b] - n_b + i and goes to that slot of the cache
 *   positions    [T] int32 rows of cos_sin, or NULL: the position in the sequence
 *   q_out        [T, Hq, D] out_dtype (may be q itself where types agree)
 *   k_cache, v_cache, kv_scales, block_table: as for pda_paged_kv_append (an fp8
 *                cache takes finite values)
 *
 * An fp8 cache keeps each (block, KV head) tile's scales by the rule of
 * pda_paged_kv_append, with the tile's new tokens taken together: where their
 * largest value exceeds 448 * scale, or the tile's slot 0 is among them, the scale
 * becomes that value / 448 (at least 2^-126) and the tile's earlier codes are
 * re-encoded. One token per sequence gives what that call gives. Sequences must
 * not append into the same block of an fp8 cache.
 *
 * Device-checked: lengths are clamped (status bit 1), tokens whose block-table
 * entry lies outside [0, num_blocks) are not written (bit 2), positions outside the
 * table are clamped into it (bit 32). Offsets that are not non-decreasing within
 * [0, T] set bit 8: a sequence whose own two are not in order is left out, and
 * tokens of the call's other sequences may be too (keys and values, q_out rows, or
 * both); what is written is right. Tokens before position 0 (n_b > seq_lens[b]) are
 * turned as at position 0 and not written; q_out rows of no sequence are not
 * written.
 *
 * Errors: PDA_EINVAL for bad sizes, types, strides, NULL or misaligned pointers
 * (16 bytes for all but the int32 arrays and kv_scales), T not a multiple of B
 * without offsets, or too much work for one call: T ((Hq + Hkv) / (512 / D) + 2) or
 * 2 Hkv times the bound on the call's cache tiles (T / 16 + 2 B with offsets, B ((T / B +
 * 14) / 16 + 1) without) past 2^25, quotients rounded down; PDA_EUNSUPPORTED for head_dim
 * not in {64, 128}, rotary_dim not a multiple of 16 or block_size != 16.
 */
int pdaops_paged_qk_norm_rope_append(const void* q,
                                     const void* k,
                                     const void* v,
                                     const void* q_weight,
                                     const void* k_weight,
                                     const float* cos_sin,
                                     const int32_t* positions,
                                     const int32_t* q_offsets,
                                     void* q_out,
                                     void* k_cache,
                                     void* v_cache,
                                     float* kv_scales,
                                     const int32_t* block_table,
                                     const int32_t* seq_lens,
                                     const pdaops_rope_problem* problem,
                                     const pdaops_cache* cache,
                                     hipStream_t stream);

/* The same norm and rotation without a cache: q_out [T, Hq, D] and k_out [T, Hkv,
 * D] (out_dtype; q and k themselves where types and strides agree), at positions
 * [T] int32. Errors and status bits as above; T ((Hq + Hkv) / (512 / D) + 2) may reach
 * 2^26, here and for the gradient. */
int pdaops_qk_norm_rope(const void* q,
                        const void* k,
                        const void* q_weight,
                        const void* k_weight,
                        const float* cos_sin,
                        const int32_t* positions,
                        void* q_out,
                        void* k_out,
                        const pdaops_rope_problem* problem,
                        hipStream_t stream);

/*
 * Gradient of pdaops_qk_norm_rope: from grad_q_out, grad_k_out (of q_out and
 * k_out; dtype), grad_q and grad_k (of q and k; dtype; grad_q_out and grad_k_out
 * themselves where strides agree), and with weights grad_q_weight, grad_k_weight
 * [D] f32, summed over all tokens and heads:
 *     g = grad turned back,  dw = sum g x r,  dx = r (g w - x r mean(g w x r)).
 * q and k are the forward's inputs (without weights they are not read and may be
 * NULL). The sums are in a fixed order: repeated calls give identical results.
 * Uses the stream's workspace (with weights 32,768 D bytes, whatever the call's size: room
 * for the parts of 4 workgroups on each of up to 1,024 compute units).
 */
int pdaops_qk_norm_rope_backward(const void* q,
                                 const void* k,
                                 const void* q_weight,
                                 const void* k_weight,
                                 const float* cos_sin,
                                 const int32_t* positions,
                                 const void* grad_q_out,
                                 const void* grad_k_out,
                                 void* grad_q,
                                 void* grad_k,
                                 float* grad_q_weight,
                                 float* grad_k_weight,
                                 const pdaops_rope_problem* problem,
                                 hipStream_t stream);

/* Logits and the tokens whose log-probabilities are wanted.
 *
 *   logits   [T, V] dtype, rows row_stride elements apart (0 = V)
 *   targets  [T] int64 or int32; a negative target marks a row that takes no part
 *            (log-probability, entropy and gradient 0; its logits are not read),
 *            one at or past V too, with status bit 64
 *
 * Logits need the alignment of their elements only. -inf marks a masked word; a
 * row of nothing else has log-probability -inf, entropy 0 and gradient 0. NaN or
 * +inf makes its own row's results NaN and no other's. */
typedef struct pdaops_logits_problem {
  int32_t num_tokens;     /* T */
  int32_t vocab;          /* V */
  int64_t row_stride;
  int32_t dtype;          /* PDA_DTYPE_F32 or PDA_DTYPE_BF16 */
  int32_t targets_int64;  /* 1: targets are int64, 0: int32 */
  float temperature;      /* > 0: the distribution is that of logits / temperature */
} pdaops_logits_problem;

/*
 * Log-probabilities of the target tokens (and entropies, unless NULL) [T] f32:
 *     z = logits / temperature,  logprob = z_y - log sum exp z,  entropy = -sum p log p
 * in float32, each row read once. Few rows are cut into parts that several
 * workgroups read, by a rule on T and V alone; the last of them, or a second
 * launch, joins them in a fixed order.
 *
 * Errors: PDA_EINVAL for bad sizes, types, strides, temperature, NULL or misaligned
 * pointers, or more than 2^22 rows (rows in parts are few: at most 1,023 of them). Uses
 * the stream's workspace (16 bytes per part).
 */
int pdaops_token_logprobs(const void* logits,
                          const void* targets,
                          float* logprobs,
                          float* entropy,
                          const pdaops_logits_problem* problem,
                          hipStream_t stream);

/* Coefficients of the policy loss. */
typedef struct pdaops_policy_options {
  float clip_low;        /* the ratio is clipped to [1 - clip_low, 1 + clip_high] */
  float clip_high;
  float dual_clip;       /* > 1: for a negative advantage A the term is at most -A dual_clip; 0: off */
  float kl_coef;         /* of the KL term (needs ref_logprobs unless 0) */
  float entropy_coef;
  float grad_scale;      /* factor of dlogits (the loss scale; 1 / accumulated steps) */
  int64_t dlogits_stride;  /* elements between dlogits' rows (0 = V) */
} pdaops_policy_options;

/*
 * The clipped policy loss of RLVR's update with its KL and entropy terms, and its
 * gradient at the logits, in one pass over them. Per row, with lp its target's
 * log-probability (pdaops_token_logprobs) and H its entropy:
 *     d = clamp(lp - old_logprobs, +-20),  ratio = e^d,  A = advantages
 *     policy = max(-A ratio, -A clip(ratio, 1 - clip_low, 1 + clip_high)),
 *              at most -A dual_clip where A < 0 and dual_clip is set
 *     u = clamp(ref_logprobs - lp, +-20),  kl = e^u - 1 - u   (0 without ref_logprobs)
 *     loss = sum over rows of weights (policy + kl_coef kl - entropy_coef H)
 * and dlogits [T, V] of the logits' type (may be the logits themselves; NULL: the
 * loss alone) = grad_scale * dloss / dlogits, 0 through a clamp or clip that
 * holds. `weights` carry the mask and the mean (1 / tokens, or 1 / (sequences *
 * tokens of the sequence)); a row of weight 0 has gradient 0 whatever its logits.
 *
 *   old_logprobs, advantages, weights [T] f32; ref_logprobs [T] f32 or NULL
 *   stats    [8] f32: sums over rows of weights times loss, policy, kl, entropy,
 *            clipped (1 where a clip holds), ratio, e^-d - 1 + d and 1. The seventh,
 *            a distance from the rollout's policy (0 where they agree, else positive),
 *            has the mean KL(policy || rollout) over tokens drawn from the policy;
 *            over the rollout's own tokens its mean is no KL but chi-square less KL,
 *            both of (rollout || policy)
 *   logprobs, entropy  [T] f32, or NULL
 *
 * Rows of up to 458,752 bytes stay in a workgroup's registers and LDS between the
 * sums and the gradient: the logits are read once. Longer rows, and few long ones
 * (which are cut into parts), are read twice. The sums are in a fixed order.
 *
 * Errors as for pdaops_token_logprobs, and PDA_EINVAL for coefficients that are
 * negative or not finite, or more than 2^20 rows. Uses the stream's workspace (32 bytes per row, 16 per part).
 */
int pdaops_policy_loss(const void* logits,
                       const void* targets,
                       const float* old_logprobs,
                       const float* ref_logprobs,
                       const float* advantages,
                       const float* weights,
                       float* stats,
                       void* dlogits,
                       float* logprobs,
                       float* entropy,
                       const pdaops_logits_problem* problem,
                       const pdaops_policy_options* options,
                       hipStream_t stream);

#ifdef __cplusplus
}  /* extern "C" */
#endif

#endif  /* PDA_OPS_H */
