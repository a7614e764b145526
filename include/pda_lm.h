/*
 * pda_lm.h -- a language model's steps between its blocks and behind its head, in
 * the same library and with the conventions of pda.h and pda_ops.h (device
 * pointers owned by the caller, host checks before any HIP call, asynchronous on
 * `stream`, the stream's workspace, HIP graphs, pda_last_error(),
 * pda_read_device_status()).
 *
 *   between the blocks  a block's output added to the residual stream, the
 *                       stream's root-mean-square norm, rounded to what the next
 *                       projection reads (fp8 with scales among it), and the
 *                       gradient
 *   behind the head     the most likely alternatives of every row of logits with
 *                       their log-probabilities: a server's answer, or what a
 *                       teacher hands to its student; and the loss by which a
 *                       student learns from such lists, with its gradient
 */
#ifndef PDA_LM_H
#define PDA_LM_H

#include "pda_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Further bit of pda_read_device_status(): 128 = a teacher's token that its list
 * holds twice was taken once. */

/* The most alternatives of a row, and entries of a teacher's list. */
#define PDALM_MAX_TOP 256

/* Sizes and types of the residual stream's norm.
 *
 * For a token's row x [H] with weights w:
 *     h = x + residual, rounded to dtype   (h = x without residual)
 *     r = 1 / sqrt(mean h^2 + eps),  y = h r w
 * The norm sees the stream as it is kept, so that a later call on h alone, and
 * the gradient, which reads h, see the same. Arithmetic and sums are float32;
 * results are rounded once.
 *
 * Strides are elements from one token's row to the next (0 = H). Pointers and
 * strides must keep every row 16-byte aligned (8-byte for an fp8 out). */
typedef struct pdalm_norm_problem {
  int32_t num_tokens;    /* T */
  int32_t width;         /* H: a multiple of 8, at most 32768 */
  int32_t dtype;         /* x, residual, stream, gradients: PDA_DTYPE_F32 or PDA_DTYPE_BF16 */
  int32_t out_dtype;     /* F32, BF16 or FP8_E4M3 */
  int32_t weight_dtype;  /* F32 or BF16 */
  int32_t scale_group;   /* fp8: neighbouring elements that share a scale: 0 (all of a row), 64 or 128 */
  float eps;
  int64_t x_stride;         /* x; the gradient's h */
  int64_t residual_stride;  /* residual; grad_residual */
  int64_t sum_stride;       /* residual_out; grad_h */
  int64_t out_stride;       /* out; grad_out */
} pdalm_norm_problem;

/*
 * out [T, H] out_dtype = y, and residual_out [T, H] = h (dtype; may be x or residual
 * itself, or NULL: not kept).
 *
 *   x         [T, H] dtype;  residual [T, H] dtype, or NULL
 *   weight    [H] weight_dtype
 *   out       may be x or residual where types and strides agree
 *   scales    [T, H / scale_group] f32 ([T] for scale_group 0) for an fp8 out, else
 *             NULL: scale = max(max |y| / 448, 2^-126) of a group, out = y / scale to
 *             nearest even, so that out * scale stands for y
 *
 * A row's results are the same in every call of its width, whatever the other rows.
 * A row whose stream holds NaN gives NaN in its whole out (in fp8 code 0x7f, and every
 * scale of the row 2^-126) and in no other row's; a weight's NaN stays in its column.
 * Squares are summed in float32, where their sum passes it those of the row times 2^-72:
 * a row gives 0 (NaN where it is infinite) where the mean square itself passes float32
 * (3.4e38). With eps 0 a row of zeros gives NaN, and values below 1e-19 lose digits.
 *
 * Errors: PDA_EINVAL for bad sizes, types, strides, NULL or misaligned pointers, more
 * than 2^22 rows, or as many of a width above 8192 (which the gradient takes);
 * PDA_EUNSUPPORTED for a width that is no multiple of 8 or above 32768, and a
 * scale_group other than 0, 64 and 128 or that does not divide the width.
 */
int pdalm_add_rms_norm(const void* x,
                       const void* residual,
                       const void* weight,
                       void* residual_out,
                       void* out,
                       float* scales,
                       const pdalm_norm_problem* problem,
                       hipStream_t stream);

/*
 * Gradient of the norm at h (the forward's residual_out, or its x without
 * residual), all of problem's dtype: from grad_out [T, H] (of out) and grad_residual
 * [T, H] (of residual_out, from the stream's further way; or NULL)
 *     grad_h = grad_residual + r (g w - y' mean(g w y')),  y' = h r,  g = grad_out
 * which is the gradient of x and of residual alike, and
 *     grad_weight [H] f32 = sum over tokens of g y'   (NULL: not wanted)
 * r is the forward's (0 for a row whose mean square passes float32).
 * grad_h may be grad_out or grad_residual where strides agree. The sums are in a
 * fixed order: repeated calls give identical results. out_dtype and scale_group
 * are not read. Uses the stream's workspace (with grad_weight: 4 bytes for each weight and each of 1,024
 * workgroups, 512 from a width of 1,025 and 256 from 8,193 on). Errors as above.
 */
int pdalm_add_rms_norm_backward(const void* h,
                                const void* weight,
                                const void* grad_out,
                                const void* grad_residual,
                                void* grad_h,
                                float* grad_weight,
                                const pdalm_norm_problem* problem,
                                hipStream_t stream);

/*
 * The num_top most likely words of every row of logits (pdaops_logits_problem), and
 * their log-probabilities at the problem's temperature, read once:
 *
 *   top_ids       [T, num_top] int32, the largest logit first; equal logits in the
 *                 order of their words
 *   top_logprobs  [T, num_top] f32
 *   targets       [T] int64 or int32, or NULL: no row has one
 *   logprobs      [T] f32 of the targets (NULL: not wanted; needs targets)
 *   entropy       [T] f32, or NULL
 *
 * num_top is 1 .. PDALM_MAX_TOP. Words of logit -inf are masked and never listed: places that no
 * word is left for hold id -1 and -inf, as does the whole list of a row whose target
 * is negative (or at or past V, status bit 64): such a row takes no part, its
 * logits are not read, its log-probability and entropy are 0. A row of -inf alone has
 * log-probability -inf and entropy 0. NaN or +inf makes its own row's log-probabilities and
 * entropy NaN; NaN is listed before +inf.
 *
 * Errors as for pdaops_token_logprobs, and PDA_EINVAL for num_top out of range. Uses the stream's workspace where
 * few rows are cut into parts (16 + 8 num_top bytes per part).
 */
int pdalm_top_logprobs(const void* logits,
                       const void* targets,
                       int32_t* top_ids,
                       float* top_logprobs,
                       float* logprobs,
                       float* entropy,
                       const pdaops_logits_problem* problem,
                       int32_t num_top,
                       hipStream_t stream);

/* Sizes and coefficients of the distillation loss. */
typedef struct pdalm_distill_options {
  int32_t num_listed;      /* K: places of a teacher's list, 1 .. PDALM_MAX_TOP */
  int32_t rest;            /* 1: the words outside of the list are one more outcome; 0: they are left out */
  float reverse;           /* b in [0, 1]: weight of the reverse divergence */
  float grad_scale;        /* factor of dlogits */
  int64_t dlogits_stride;  /* elements between dlogits' rows (0 = V) */
} pdalm_distill_options;

/*
 * Distillation from a teacher's lists of likely tokens, and its gradient at the
 * student's logits, which are read once (few long rows, and the end of very long ones, twice). A row's list gives words i_k and the
 * teacher's log-probabilities tau_k (as pdalm_top_logprobs writes them, at the same
 * temperature). With t = e^tau, log p the student's log-probabilities, a = log p - tau, sums over the
 * list, S = sum t, P = sum p:
 *     forward = -sum t a,  reverse = sum p a
 * and with rest, t_r = max(1 - S, 2^-24), p_r the student's probability of all words
 * that are not listed, a_r = log p_r - log t_r:
 *     forward = -sum t a - t_r a_r,  reverse = sum p a + p_r a_r
 * (the two divergences of the distributions over listed words and the rest; no rest
 * where no other word has a logit above -inf).
 *     loss = sum over rows of weights ((1 - b) forward + b reverse)
 * dlogits [T, V] of the logits' type (may be the logits themselves; NULL: the loss
 * alone) = grad_scale * dloss / dlogits.
 *
 *   teacher_ids       [T, K] int32, in any order; a place with a negative id or tau =
 *                     -inf is empty (lists may be of different lengths). Ids at or past V are
 *                     ignored (status bit 64). A word's second place in a list is ignored
 *                     (status bit 128).
 *   teacher_logprobs  [T, K] f32
 *   weights           [T] f32: mask and mean, as for pdaops_policy_loss; a row of weight 0 has
 *                     gradient 0 whatever its logits
 *   stats             [6] f32: sums over rows of weights times loss, forward, reverse, S, P, 1
 *   losses            [T] f32: the rows' (1 - b) forward + b reverse, or NULL
 *
 * A listed word whose student's logit is -inf makes forward +inf, and its gradient stays finite; a row of
 * -inf alone has reverse 0, P 0 and gradient 0. NaN or +inf makes its own row's results NaN (and
 * stats, if its weight is not 0).
 *
 * The sums are in a fixed order. Errors as for pdaops_policy_loss (targets_int64 is not used), and
 * PDA_EINVAL for options out of range. Uses the stream's workspace (32 bytes per row, and where
 * few or very long rows are cut into parts 16 per part and 8 K per row).
 */
int pdalm_distill_loss(const void* logits,
                       const int32_t* teacher_ids,
                       const float* teacher_logprobs,
                       const float* weights,
                       float* stats,
                       float* losses,
                       void* dlogits,
                       const pdaops_logits_problem* problem,
                       const pdalm_distill_options* options,
                       hipStream_t stream);

#ifdef __cplusplus
}  /* extern "C" */
#endif

#endif  /* PDA_LM_H */
