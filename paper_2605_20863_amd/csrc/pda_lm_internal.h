// Internal interface between the host code of include/pda_lm.h (pda_lm_host.cpp)
// and its kernels (pda_norm.hip, pda_top.hip, pda_distill.hip).
#pragma once

#include "pda_ops_internal.h"

namespace pda {

constexpr int kStatusTwice = 128;  // a teacher's token that its list holds twice was taken once

constexpr int kMaxTop = 256;       // alternatives of a row, entries of a list
constexpr int kMaxWidth = 32768;   // of the residual stream
constexpr int kLongWidth = 8192;   // above it the norm has 1,024 threads a row, however many rows there are

enum class OutType : int { F32 = 0, BF16 = 1, FP8 = 2 };

// The residual stream's norm (pda_norm.hip). Strides are elements from one
// token's row to the next.
struct NormArgs {
  const void *x, *res, *w;  // x: the gradient's h; res, or null: the gradient's grad_residual
  void *sum, *out;          // sum, or null; the gradient's grad_h, and its grad_out (which is only read)
  float* scales;
  int64_t x_stride, res_stride, sum_stride, out_stride;
  int32_t T, H, bf16, w_bf16, group;
  OutType type;
  float eps;
  float* dw;       // [H], or null
  float* dw_part;  // [wgs, H]
  int32_t wgs;
};

// The most likely words of rows of logits (pda_top.hip).
struct TopArgs {
  LogitsArgs z;     // targets and logp may be null
  int32_t K;
  int32_t* ids;     // [T, K]
  float* tops;      // [T, K]
  uint64_t* keys;   // [T, splits, K]
};

// Distillation from a teacher's lists (pda_distill.hip).
constexpr int kDistillStats = 6;
// Vectors of a row that one workgroup takes: 20 and 4 of 1,024 threads in registers and LDS, beside the words' bits, and 40 more
// that are read twice.
constexpr int kListedMore = 40, kListedVectors = 1024 * (20 + 4 + kListedMore);
struct DistillArgs {
  LogitsArgs z;     // no targets; weight, terms, stats, dlogits as for the policy loss
  const int32_t* ids;  // [T, K]
  const float* tau;    // [T, K]
  int32_t K, rest;
  float rev;
  float* losses;    // [T], or null
  float* listed;    // [T, K] of rows in parts: {a place's word's logit, 1, or 0 if the word has an earlier place}
};

hipError_t launch_norm(const NormArgs& a, hipStream_t s);
hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s);
hipError_t launch_top_logprobs(const TopArgs& a, hipStream_t s);
hipError_t launch_distill_loss(const DistillArgs& a, hipStream_t s);

}  // namespace pda
