// Internal interface between the host code of the operators around attention
// (pda_ops_host.cpp) and their kernels (pda_rope.hip, pda_policy.hip).
#pragma once

#include "pda_internal.h"

#include <hip/hip_runtime.h>

namespace pda {

// Further device-side status bits (pda_internal.h has the first).
constexpr int kStatusBadPosition = 32;  // a rotation position outside the table was clamped
constexpr int kStatusBadTarget = 64;    // a target at or past the vocabulary was ignored

// Head norms and rotation (pda_rope.hip): the cache append, the training
// forward and its gradient. Strides are elements from one token's row to the next.
struct RopeArgs {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  const void *wq, *wk;       // [D] norm weights; null: no norm
  const float* table;        // [P, R]: R / 2 cosines, R / 2 sines of a position's angles
  const int32_t* positions;  // [T] rows of the table; null: the token's place in its sequence
  void *q_out, *k_out;
  int64_t qo_stride, ko_stride;
  int32_t T, Hq, Hkv, D, R, P;
  int32_t in_bf16, out_bf16, w_bf16, interleaved;
  float eps;
  int32_t* status;
  // append
  const int32_t* q_offsets;  // [B + 1], or null: n tokens of every sequence
  const int32_t* seq_lens;   // [B] lengths with the new tokens
  const int32_t* block_table;
  void *k_cache, *v_cache;
  float* kv_scales;
  int32_t B, n, max_blocks, len_cap;
  int64_t num_blocks;
  int32_t tiles;             // bound on the cache tiles of one KV head that the new tokens touch
  int32_t tiles_per_seq;     // with n: of each sequence
  // gradient: of the rotated queries and keys (in), of the inputs (out)
  const void *gq, *gk;
  int64_t gq_stride, gk_stride;
  void *dq, *dk;
  int64_t dq_stride, dk_stride;
  float *dwq, *dwk;          // [D]
  float* dw_part;            // [workgroups, 2, D]
  int32_t wgs;               // of the gradient's kernel
  uint64_t* counts;          // null: the weights' gradients are summed by a launch of their own
  uint32_t epoch;
  // the launcher's: chunks of `rows` rows that a token's heads are cut into, one wave each
  int32_t chunks, rows;
};

// Log-probabilities of tokens and the policy loss (pda_policy.hip).
constexpr int kMaxSplits = 64;  // parts that a row of logits is cut into, one lane each to merge them
constexpr int kTerms = 8;       // sums of the loss: loss, policy, kl, entropy, clipped, ratio, old_kl, weight

struct LogitsArgs {
  const void* logits;   // [T, V], rows `stride` elements apart
  int64_t stride;
  const void* targets;  // [T] int32 or int64
  int32_t targets64, T, V, bf16;
  float inv_temp;
  float* logp;          // [T]
  float* ent;           // [T] or null
  int32_t splits, chunk;  // parts of a row, 16-byte vectors of each
  float4* part;         // [T, splits] {max, sum, weighted sum, target's logit}
  int32_t* status;
  // policy loss
  const float *old_logp, *ref_logp, *adv, *weight;
  float* stats;         // [kTerms]
  void* dlogits;        // [T, V] of logits' type, rows d_stride elements apart; null: no gradient
  int64_t d_stride;
  float* terms;         // [T, kTerms]
  float clip_low, clip_high, dual, kl, ent_coef, grad_scale;
  // arrival counts (one, or one of each row); null: rows and sums are finished by launches of their own
  uint64_t* counts;
  uint32_t epoch;
};

// Calls outside of a capture whose workgroups count their arrivals, so that the
// last one finishes the work: up to this many rows (policy loss), workgroups
// (weights' gradients) or, with a word each, kShortUnits rows in parts
// (log-probabilities). us per call, with a further launch / counted: log-probabilities of
// 64 x 131,072 10.0 / 8.5, of 1 x 150,000 7.9 / 6.0; gradient of 1 token 8.0 / 6.7, of 50
// 8.2 / 7.9 (63 workgroups); policy loss of 20 x 4,046 8.0 / 6.7, of 32 x 8,000 8.2 / 7.3,
// of 64 x 8,000 8.3 / 8.1, of 512 x 2,000 8.7 / 16.8 (arrivals at one word take turns).
constexpr int kCountedRows = 32, kCountedWgs = 64;

// Vectors of a row that one workgroup's registers and LDS hold: 1,024 threads' 19 and 9.
constexpr int kRowVectors = 1024 * (19 + 9);

hipError_t launch_token_logprobs(const LogitsArgs& a, hipStream_t s);
hipError_t launch_policy_loss(const LogitsArgs& a, hipStream_t s);

hipError_t launch_rope_append(const RopeArgs& a, KvType kv, hipStream_t s);
hipError_t launch_rope(const RopeArgs& a, hipStream_t s);
hipError_t launch_rope_backward(const RopeArgs& a, hipStream_t s);

}  // namespace pda
