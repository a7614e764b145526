// Host side of include/pda_lm.h: argument checks (host code only, before any HIP
// call), the split of the work, and the launches.

#include "pda_lm.h"

#include "pda_checks.h"
#include "pda_lm_internal.h"

namespace {

using namespace pda;

// *out: the stride in elements; rows of H elements must not overlap and stay aligned to `align` bytes.
int check_stride(const char* name, int64_t stride, const pdalm_norm_problem* pr, int size, int align, int64_t* out) {
  if (stride == 0) stride = pr->width;
  if (stride < pr->width) return host_fail(PDA_EINVAL, "%s = %lld is less than the width %d", name, (long long)stride, pr->width);
  if (stride > INT64_MAX / 8 / (pr->num_tokens + 1ll)) return host_fail(PDA_EINVAL, "%s = %lld is too large", name, (long long)stride);
  if (stride * size % align) return host_fail(PDA_EINVAL, "%s = %lld elements is not a multiple of %d bytes", name, (long long)stride, align);
  *out = stride;
  return PDA_OK;
}

int check_norm(const pdalm_norm_problem* pr, bool gradient, NormArgs* a) {
  if (!pr) return host_fail(PDA_EINVAL, "problem is NULL");
  if (pr->num_tokens < 0 || pr->num_tokens > kMaxWaves / 16)
    return host_fail(PDA_EINVAL, "num_tokens = %d (0 .. 2^22)", pr->num_tokens);
  if (pr->width < 1) return host_fail(PDA_EINVAL, "width = %d < 1", pr->width);
  if (pr->width % 8 || pr->width > kMaxWidth)
    return host_fail(PDA_EUNSUPPORTED, "width = %d (supported: multiples of 8 up to %d)", pr->width, kMaxWidth);
  // the norm's launch: 1,024 threads for each of the longest rows (the gradient's workgroups take rows in turn)
  if (!gradient && pr->width > kLongWidth && pr->num_tokens == kMaxWaves / 16)
    return host_fail(PDA_EINVAL, "num_tokens = %d (below 2^22 for widths above %d)", pr->num_tokens, kLongWidth);
  if (!float_type(pr->dtype)) return host_fail(PDA_EINVAL, "dtype = %d (supported: F32, BF16)", pr->dtype);
  if (!float_type(pr->weight_dtype)) return host_fail(PDA_EINVAL, "weight_dtype = %d (supported: F32, BF16)", pr->weight_dtype);
  if (!(pr->eps >= 0.f) || !std::isfinite(pr->eps)) return host_fail(PDA_EINVAL, "eps is negative or not finite");
  const int e = size_of(pr->dtype);
  const bool fp8 = !gradient && pr->out_dtype == PDA_DTYPE_FP8_E4M3;
  if (!gradient) {
    if (!fp8 && !float_type(pr->out_dtype)) return host_fail(PDA_EINVAL, "out_dtype = %d is not a pda_dtype", pr->out_dtype);
    if (fp8 && pr->scale_group != 0 && pr->scale_group != 64 && pr->scale_group != 128)
      return host_fail(PDA_EUNSUPPORTED, "scale_group = %d (supported: 0, 64, 128)", pr->scale_group);
    if (fp8 && pr->scale_group && pr->width % pr->scale_group)
      return host_fail(PDA_EUNSUPPORTED, "scale_group = %d does not divide the width %d", pr->scale_group, pr->width);
  }
  int rc;
  if ((rc = check_stride("x_stride", pr->x_stride, pr, e, 16, &a->x_stride)) != PDA_OK ||
      (rc = check_stride("residual_stride", pr->residual_stride, pr, e, 16, &a->res_stride)) != PDA_OK ||
      (rc = check_stride("sum_stride", pr->sum_stride, pr, e, 16, &a->sum_stride)) != PDA_OK ||
      (rc = check_stride("out_stride", pr->out_stride, pr, gradient ? e : fp8 ? 1 : size_of(pr->out_dtype), fp8 ? 8 : 16,
                         &a->out_stride)) != PDA_OK)
    return rc;
  a->T = pr->num_tokens;
  a->H = pr->width;
  a->bf16 = pr->dtype == PDA_DTYPE_BF16;
  a->w_bf16 = pr->weight_dtype == PDA_DTYPE_BF16;
  a->type = fp8 ? OutType::FP8 : pr->out_dtype == PDA_DTYPE_BF16 ? OutType::BF16 : OutType::F32;
  a->group = fp8 ? pr->scale_group : 0;
  a->eps = pr->eps;
  return PDA_OK;
}

int norm_run(const void* x, const void* residual, const void* weight, void* residual_out, void* out, float* scales,
             const pdalm_norm_problem* pr, hipStream_t stream) {
  host_clear_error();
  NormArgs a = {};
  int rc = check_norm(pr, false, &a);
  if (rc != PDA_OK) return rc;
  const bool fp8 = a.type == OutType::FP8;
  if (residual_out && !residual) return host_fail(PDA_EINVAL, "residual_out without residual: the stream is x");
  if (scales && !fp8) return host_fail(PDA_EINVAL, "scales for an out that is not fp8");
  if (a.T == 0) return PDA_OK;
  rc = check_pointers({{x, 16, "x", true}, {residual, 16, "residual", false}, {weight, 16, "weight", true},
                       {residual_out, 16, "residual_out", false}, {out, fp8 ? 8u : 16u, "out", true},
                       {scales, 4, "scales", fp8}});
  if (rc != PDA_OK) return rc;
  a.x = x;
  a.res = residual;
  a.w = weight;
  a.sum = residual_out;
  a.out = out;
  a.scales = scales;
  const hipError_t e = launch_norm(a, stream);
  return e == hipSuccess ? PDA_OK : host_fail_hip(e, "residual norm kernel launch");
}

int norm_backward_run(const void* h, const void* weight, const void* grad_out, const void* grad_residual, void* grad_h,
                      float* grad_weight, const pdalm_norm_problem* pr, hipStream_t stream) {
  host_clear_error();
  NormArgs a = {};
  int rc = check_norm(pr, true, &a);
  if (rc != PDA_OK) return rc;
  const bool any = a.T > 0;
  if (!any && !grad_weight) return PDA_OK;
  rc = check_pointers({{h, 16, "h", any}, {weight, 16, "weight", any}, {grad_out, 16, "grad_out", any},
                       {grad_residual, 16, "grad_residual", false}, {grad_h, 16, "grad_h", any},
                       {grad_weight, 4, "grad_weight", false}});
  if (rc != PDA_OK) return rc;
  // room for the parts of the weights' gradient; long rows have fewer (backward_for)
  constexpr int64_t kWgsPerCu = 4, kMostWgs = 1024;
  const int64_t room = a.H <= 1024 ? kMostWgs : a.H <= 8192 ? 512 : 256;
  HeldWorkspace ws;
  if ((rc = hold_workspace(stream, kHeader + (grad_weight ? room * a.H * 4 : 0), &ws)) != PDA_OK) return rc;
  a.x = h;
  a.res = grad_residual;
  a.w = weight;
  a.sum = grad_h;
  a.out = const_cast<void*>(grad_out);
  a.dw = grad_weight;
  a.dw_part = reinterpret_cast<float*>(ws.base + kHeader);
  a.wgs = (int32_t)(kWgsPerCu * ws.cus < room ? kWgsPerCu * ws.cus : room);
  const hipError_t e = launch_norm_backward(a, stream);
  return e == hipSuccess ? PDA_OK : host_fail_hip(e, "residual norm gradient kernel launch");
}

int top_run(const void* logits, const void* targets, int32_t* top_ids, float* top_logprobs, float* logprobs,
            float* entropy, const pdaops_logits_problem* pr, int32_t num_top, hipStream_t stream) {
  host_clear_error();
  TopArgs g = {};
  LogitsArgs& a = g.z;
  int rc = check_logits(pr, &a);
  if (rc != PDA_OK) return rc;
  if (num_top < 1 || num_top > kMaxTop) return host_fail(PDA_EINVAL, "num_top = %d (1 .. %d)", num_top, kMaxTop);
  if (logprobs && !targets) return host_fail(PDA_EINVAL, "logprobs without targets");
  if (a.T == 0) return PDA_OK;
  rc = check_pointers({{logits, a.bf16 ? 2u : 4u, "logits", true}, {targets, a.targets64 ? 8u : 4u, "targets", false},
                       {top_ids, 4, "top_ids", true}, {top_logprobs, 4, "top_logprobs", true}, {logprobs, 4, "logprobs", false},
                       {entropy, 4, "entropy", false}});
  if (rc != PDA_OK) return rc;
  // a part's own chain (a bar, K keys to hand on) is longer than a sum's: parts of at least 2,048 vectors (us per call of 512 /
  // 1,024 / 2,048 / 4,096; bf16: 64 x 131,072, 20 alternatives 17.1 / 17.1 / 14.9 / 16.6, 64: 17.4 / 17.5 / 16.4 / 19.7, 256: 40 / 41 / 31 /
  // 33; 1 x 131,072, 20: 12.5 / 11.9 / 12.5 / 14.2; f32: 2 x 150,001, 5: 16.0 / 13.4 / 12.8 / 16.5)
  split_rows(&a, 2048);
  if ((int64_t)a.T * a.splits > kMaxWaves / 16) return host_fail(PDA_EINVAL, "num_tokens = %d is too much for one call", a.T);
  const int64_t parts = a.splits > 1 ? (int64_t)a.T * a.splits : 0;
  HeldWorkspace ws;
  if ((rc = hold_workspace(stream, kHeader + parts * (16 + 8 * (int64_t)num_top), &ws)) != PDA_OK) return rc;
  a.logits = logits;
  a.targets = targets;
  a.logp = logprobs;
  a.ent = entropy;
  a.status = status_word(ws.base);
  a.part = reinterpret_cast<float4*>(ws.base + kHeader);
  g.keys = reinterpret_cast<uint64_t*>(ws.base + kHeader + parts * 16);
  if (a.splits > 1 && a.T <= kShortUnits && (rc = count(stream, ws, &a)) != PDA_OK) return rc;
  g.K = num_top;
  g.ids = top_ids;
  g.tops = top_logprobs;
  const hipError_t e = launch_top_logprobs(g, stream);
  return e == hipSuccess ? PDA_OK : host_fail_hip(e, "top log-probability kernel launch");
}

int distill_run(const void* logits, const int32_t* teacher_ids, const float* teacher_logprobs, const float* weights,
                float* stats, float* losses, void* dlogits, const pdaops_logits_problem* pr,
                const pdalm_distill_options* op, hipStream_t stream) {
  host_clear_error();
  DistillArgs g = {};
  LogitsArgs& a = g.z;
  int rc = check_logits(pr, &a);
  if (rc != PDA_OK) return rc;
  if (!op) return host_fail(PDA_EINVAL, "options is NULL");
  if (op->num_listed < 1 || op->num_listed > kMaxTop)
    return host_fail(PDA_EINVAL, "num_listed = %d (1 .. %d)", op->num_listed, kMaxTop);
  if (op->rest != 0 && op->rest != 1) return host_fail(PDA_EINVAL, "rest = %d (0 or 1)", op->rest);
  if (!(op->reverse >= 0.f && op->reverse <= 1.f)) return host_fail(PDA_EINVAL, "reverse must be in [0, 1]");
  if (!std::isfinite(op->grad_scale)) return host_fail(PDA_EINVAL, "grad_scale is not finite");
  a.d_stride = op->dlogits_stride ? op->dlogits_stride : a.V;
  if (a.d_stride < a.V || a.d_stride > INT64_MAX / 8 / (a.T + 1ll))
    return host_fail(PDA_EINVAL, "dlogits_stride = %lld", (long long)op->dlogits_stride);
  const bool any = a.T > 0;
  const uintptr_t e = a.bf16 ? 2 : 4;
  rc = check_pointers({{logits, e, "logits", any}, {teacher_ids, 4, "teacher_ids", any},
                       {teacher_logprobs, 4, "teacher_logprobs", any}, {weights, 4, "weights", any}, {stats, 4, "stats", true},
                       {losses, 4, "losses", false}, {dlogits, e, "dlogits", false}});
  if (rc != PDA_OK) return rc;
  if (a.T > kMaxWaves / 64) return host_fail(PDA_EINVAL, "num_tokens = %d is too much for one call", a.T);
  // A workgroup a row where it can take one and rows are short or as many as a 220th of their vectors; otherwise in parts, read twice
  // (us per call, rows / parts, 64 places; bf16: 16,000 words, 1 row 9.4 / 12.1, 200 12.2 / 16.7; 32,000, 1 11.8 / 12.5, 64 14.0 / 15.5;
  // 50,000, 8 14.5 / 13.4, 32 15.0 / 14.4, 64 15.2 / 17.2; 131,072, 1 22 / 12, 64 24.0 / 19.4, 96 24.5 / 24.5, 160 26 / 36; 200,000, 64 34 / 23,
  // 128 35 / 37; f32: 20,000, 1 10.6 / 12.0; 50,001, 32 16.5 / 15.0, 64 16.9 / 16.7, 128 18.4 / 21.7; 110,000, 64 27 / 22, 128 32 / 36).
  constexpr int kShortVectors = 4096, kShare = 220, kMany = 128;
  const int v = vectors_of(a);
  const bool rows = v <= kListedVectors && (v <= kShortVectors || a.T >= kMany || (int64_t)a.T * kShare >= v);
  if (any && !rows) split_rows(&a);
  const int64_t terms = ((int64_t)a.T * kTerms * 4 + 255) / 256 * 256, parts = (int64_t)a.T * a.splits * 16;
  HeldWorkspace ws;
  if ((rc = hold_workspace(stream, kHeader + terms + parts + (parts ? (int64_t)a.T * op->num_listed * 8 : 0), &ws)) != PDA_OK) return rc;
  a.logits = logits;
  a.weight = weights;
  a.stats = stats;
  a.dlogits = dlogits;
  a.grad_scale = op->grad_scale;
  a.terms = reinterpret_cast<float*>(ws.base + kHeader);
  a.status = status_word(ws.base);
  g.ids = teacher_ids;
  g.tau = teacher_logprobs;
  g.K = op->num_listed;
  g.rest = op->rest;
  g.rev = op->reverse;
  g.losses = losses;
  a.part = reinterpret_cast<float4*>(ws.base + kHeader + terms);
  g.listed = reinterpret_cast<float*>(ws.base + kHeader + terms + parts);
  if (any && a.T <= kCountedRows && (rc = count(stream, ws, &a)) != PDA_OK) return rc;
  const hipError_t h = launch_distill_loss(g, stream);
  return h == hipSuccess ? PDA_OK : host_fail_hip(h, "distillation kernel launch");
}

}  // namespace

extern "C" {

int pdalm_add_rms_norm(const void* x, const void* residual, const void* weight, void* residual_out, void* out, float* scales,
                       const pdalm_norm_problem* problem, hipStream_t stream) {
  return entry([&] { return norm_run(x, residual, weight, residual_out, out, scales, problem, stream); });
}

int pdalm_add_rms_norm_backward(const void* h, const void* weight, const void* grad_out, const void* grad_residual,
                                void* grad_h, float* grad_weight, const pdalm_norm_problem* problem, hipStream_t stream) {
  return entry([&] { return norm_backward_run(h, weight, grad_out, grad_residual, grad_h, grad_weight, problem, stream); });
}

int pdalm_top_logprobs(const void* logits, const void* targets, int32_t* top_ids, float* top_logprobs, float* logprobs,
                       float* entropy, const pdaops_logits_problem* problem, int32_t num_top, hipStream_t stream) {
  return entry([&] { return top_run(logits, targets, top_ids, top_logprobs, logprobs, entropy, problem, num_top, stream); });
}

int pdalm_distill_loss(const void* logits, const int32_t* teacher_ids, const float* teacher_logprobs, const float* weights,
                       float* stats, float* losses, void* dlogits, const pdaops_logits_problem* problem,
                       const pdalm_distill_options* options, hipStream_t stream) {
  return entry([&] {
    return distill_run(logits, teacher_ids, teacher_logprobs, weights, stats, losses, dlogits, problem, options, stream);
  });
}

}  // extern "C"
