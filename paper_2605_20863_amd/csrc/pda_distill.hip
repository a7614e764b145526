// HIP kernels for the distillation loss from a teacher's lists of likely tokens,
// with its gradient at the student's logits, on MI355X (gfx950).
//
// For a row of logits l [V], z = l / temperature, a list of words i_k with the
// teacher's log-probabilities tau_k, t = e^tau, S = sum t, the student's log p, p,
// P = sum p over the list, a = log p - tau; of the words outside of it p_r, t_r = max(1 - S, 2^-24),
// a_r = log p_r - log t_r (rest; t_r = p_r = 0 without):
//     F = -sum t a - t_r a_r,  R = sum p a + p_r a_r,  loss = (1 - b) F + b R
//     dF / dz_v = p_v (S + t_r) - t_v,  p_v (S + t_r - t_r / p_r) outside
//     dR / dz_v = p_v (a_v - R),        p_v (a_r - R) outside             (rest)
//               = p_v (a_v + 1 - R - P), -p_v (R + P) outside            (without)
//
// The words outside of the list are summed by themselves, against their own largest logit,
// so that a small p_r is as exact as a large one (1 - P would not be); the gradient outside is
// one factor a row times a word's share of the rest. With a bit in LDS for every listed word a vector of 16 bytes
// costs one LDS read to leave them out.
//
// With rest, sum p + p_r = 1 turns the divergences into sums of terms that are not
// negative, which keeps their digits where teacher and student are close:
//     F = sum t (e^a - 1 - a) + (S + t_r - 1),  R = sum p (e^-a - 1 + a) - (S + t_r - 1).

#include "pda_lm_internal.h"
#include "pda_rows.h"

namespace pda {
namespace {

constexpr int kWindow = 1 << 17;         // words whose bits LDS holds at a time
constexpr double kLeastRest = 0x1p-24;  // half a step of float32 below 1: what a sum of t can tell from it

// A row's list: places that hold a word, each word once.
struct List {
  int id[kMaxTop];  // -1: empty
  float tau[kMaxTop], l[kMaxTop];
  float d[kMaxTop];  // gradient by the word's logit / (w / temperature)
};

// e^x - 1 - x
__device__ __forceinline__ float phi(float x) {
  if (fabsf(x) > 0.25f) return expm1f(x) - x;
  // the series to x^8: what is left is below 2^-24 of it
  float y = 1.f / 40320.f;
  y = fmaf(y, x, 1.f / 5040.f);
  y = fmaf(y, x, 1.f / 720.f);
  y = fmaf(y, x, 1.f / 120.f);
  y = fmaf(y, x, 1.f / 24.f);
  y = fmaf(y, x, 1.f / 6.f);
  y = fmaf(y, x, 0.5f);
  return y * x * x;
}

// The sum over the workgroup, in every thread.
template <typename X>
__device__ __forceinline__ X group_total(X x) {
  __shared__ X parts[kPartThreads / 64];
#pragma unroll
  for (int o = 1; o < 64; o *= 2) x += __shfl_xor(x, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x / 64] = x;
  __syncthreads();
  x = parts[0];
#pragma unroll
  for (int w = 1; w < kPartThreads / 64; ++w) x += parts[w];
  return x;
}

// The list's places of row t, by thread k its k-th.
template <typename T>
__device__ __forceinline__ void load_list(const DistillArgs& g, int t, const T* row, List& s) {
  const int k = (int)threadIdx.x;
  int id = -1;
  float tau = 0.f;
  if (k < g.K) {
    id = g.ids[(int64_t)t * g.K + k];
    tau = g.tau[(int64_t)t * g.K + k];
    if (id >= g.z.V) {
      atomicOr(g.z.status, kStatusBadTarget);
      id = -1;
    }
    if (id < 0 || tau == -__builtin_huge_valf()) id = -1;
    s.id[k] = id;
  }
  __syncthreads();
  bool twice = false;
  for (int j = 0; j < min(k, g.K); ++j) twice |= id >= 0 && s.id[j] == id;
  __syncthreads();
  if (twice) {
    atomicOr(g.z.status, kStatusTwice);
    id = -1;
  }
  if (k < g.K) {
    s.id[k] = id;
    s.tau[k] = tau;
    s.l[k] = id >= 0 ? load1(row + id) : 0.f;
  }
  __syncthreads();
}

struct Row {
  float loss;
  float terms[kTerms];
  float m, log2_s, outside;  // gradient outside of the list: exp2((l - m) c - log2_s) outside
  bool zero;
};

// From the sums of the words outside of the list, and the list.
__device__ __forceinline__ Row finish_row(const DistillArgs& g, int t, const Soft& r, List& s, float c) {
  const LogitsArgs& a = g.z;
  const int k = (int)threadIdx.x;
  const bool in = k < g.K && s.id[k] >= 0;
  const float l = in ? s.l[k] : kLowest, tau = in ? s.tau[k] : 0.f;
  __syncthreads();  // the merge before this one has been read
  // the row's own largest logit and sum
  Soft x = none();
  if (in) add1(x, l, c);
  x = merge(group_merge<kPartThreads>(x, c), r, c);
  const bool some = x.s != 0.f;  // NaN too
  const float log_s = logf(x.s);
  const float lp = some ? (l - x.m) * a.inv_temp - log_s : -__builtin_huge_valf();
  const float p = in ? expf(lp) : 0.f;
  const double t64 = in ? exp((double)tau) : 0.;
  const float tk = (float)t64, ak = in ? lp - tau : 0.f;
  const double S64 = group_total(t64);
  const float S = (float)S64, P = group_total(p), b = g.rev;
  const float pa = p == 0.f ? 0.f : p * ak, ta = tk == 0.f ? 0.f : tk * ak;
  Row o;
  float F, R, total = S, d;
  float tr = 0.f, pr = 0.f, ar = 0.f;
  if (g.rest) {
    float over = (float)(S64 - 1.);
    if (r.s != 0.f) {
      const double t_rest = fmax(1. - S64, kLeastRest);
      tr = (float)t_rest;
      const float lpr = (r.m - x.m) * a.inv_temp + (logf(r.s) - log_s);
      pr = expf(lpr);
      ar = lpr - (float)log(t_rest);
      over = (float)(S64 + t_rest - 1.);
      total = (float)(S64 + t_rest);
    }
    // terms of either sign where a is far from 0, squares where it is near
    const bool near = fabsf(ak) <= 1.f, near_r = fabsf(ar) <= 1.f;
    const float f = !in ? 0.f : near ? tk * phi(ak) : p - tk - ta;
    const float q = !in ? 0.f : near ? p * phi(-ak) : tk - p + pa;
    F = group_total(f) + (near_r ? tr * phi(ar) : pr - tr - tr * ar) + over;
    R = group_total(q) + (near_r ? pr * phi(-ar) : tr - pr + (pr == 0.f ? 0.f : pr * ar)) - over;
    d = (1.f - b) * (p * total - tk) + b * (pa - p * R);
    o.outside = (1.f - b) * (pr * total - tr) + b * ((pr == 0.f ? 0.f : pr * ar) - pr * R);
  } else {
    F = group_total(-ta);
    R = group_total(pa);
    const float lpr = (r.m - x.m) * a.inv_temp + (logf(r.s) - log_s);
    pr = r.s == 0.f ? 0.f : expf(lpr);
    d = (1.f - b) * (p * total - tk) + b * (pa + p - p * (R + P));
    o.outside = pr * ((1.f - b) * total - b * (R + P));
  }
  if (!some) {  // every logit is -inf: no distribution
    F = S > 0.f ? __builtin_huge_valf() : 0.f;
    R = 0.f;
  }
  const float w = a.weight[t], scale = w * a.grad_scale * a.inv_temp;
  o.loss = (b < 1.f ? (1.f - b) * F : 0.f) + (b > 0.f ? b * R : 0.f);
  const float v[kTerms] = {o.loss, F, R, S, P, 1.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kTerms; ++i) o.terms[i] = w != 0.f ? w * v[i] : 0.f;
  o.zero = scale == 0.f || !some;
  o.m = r.m;
  o.log2_s = r.s == 0.f ? 0.f : logf(r.s) * kLog2e;
  o.outside *= scale;
  if (k < g.K) s.d[k] = d * scale;
  __syncthreads();
  return o;
}

// Bits of the listed words among first .. first + kWindow - 1.
__device__ __forceinline__ void mark(const List& s, int K, int first, uint32_t* bits) {
  __syncthreads();
  for (int i = (int)threadIdx.x; i < kWindow / 32; i += kPartThreads) bits[i] = 0;
  __syncthreads();
  for (int k = (int)threadIdx.x; k < K; k += kPartThreads) {
    const int at = s.id[k] - first;
    if (s.id[k] >= 0 && at >= 0 && at < kWindow) atomicOr(&bits[at / 32], 1u << (at % 32));
  }
  __syncthreads();
}

template <typename T>
__global__ __launch_bounds__(kPartThreads) void distill_kernel(DistillArgs g) {
  const LogitsArgs& a = g.z;
  __shared__ List list;
  __shared__ uint32_t bits[kWindow / 32];
  const int t = (int)blockIdx.x;
  const T* row = static_cast<const T*>(a.logits) + (int64_t)t * a.stride;
  T* out = static_cast<T*>(a.dlogits) + (int64_t)t * a.d_stride;
  const float c = a.inv_temp * kLog2e;
  load_list(g, t, row, list);
  Soft x = none();
  for (int first = 0; first < a.V; first += kWindow) {
    mark(list, g.K, first, bits);
    for (int i = (int)threadIdx.x; i < min(kWindow, a.V - first); i += kPartThreads)
      if (!(bits[i / 32] >> (i % 32) & 1)) add1(x, load1(row + first + i), c);
  }
  x = group_merge<kPartThreads>(x, c);
  const Row o = finish_row(g, t, x, list, c);
  if (threadIdx.x == 0) {
    write_terms(a, t, o.terms);
    if (g.losses) g.losses[t] = o.loss;
  }
  if (!a.dlogits) return;
  for (int first = 0; first < a.V; first += kWindow) {
    mark(list, g.K, first, bits);
    for (int i = (int)threadIdx.x; i < min(kWindow, a.V - first); i += kPartThreads)
      if (!(bits[i / 32] >> (i % 32) & 1)) {
        const float y = __builtin_amdgcn_exp2f(fmaf(load1(row + first + i) - o.m, c, -o.log2_s)) * o.outside;
        store1(out + first + i, o.zero ? 0.f : y);
      }
  }
  for (int k = (int)threadIdx.x; k < g.K; k += kPartThreads)
    if (list.id[k] >= 0) store1(out + list.id[k], o.zero ? 0.f : list.d[k]);
}

__global__ __launch_bounds__(1024) void distill_stats_kernel(LogitsArgs a) { sum_terms<1024, 8, kDistillStats>(a); }

template <typename T>
hipError_t distill_for(const DistillArgs& a, hipStream_t s) {
  DistillArgs args = a;
  void* params[] = {&args};
  if (!a.z.T) return hipSuccess;
  return hipLaunchKernel(reinterpret_cast<const void*>(&distill_kernel<T>), dim3((unsigned)a.z.T), dim3(kPartThreads), params, 0, s);
}

}  // namespace

hipError_t launch_distill_loss(const DistillArgs& a, hipStream_t s) {
  const hipError_t e = a.z.bf16 ? distill_for<uint16_t>(a, s) : distill_for<float>(a, s);
  if (e != hipSuccess) return e;
  LogitsArgs args = a.z;
  void* params[] = {&args};
  return hipLaunchKernel(reinterpret_cast<const void*>(&distill_stats_kernel), dim3(1), dim3(1024), params, 0, s);
}

}  // namespace pda
