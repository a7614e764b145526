// HIP kernels for the log-probabilities of given tokens and the clipped policy
// loss with its gradient at the logits, on MI355X (gfx950).
//
// For a row of logits l [V], z = l / temperature, target y:
//     lse = log sum exp z,  log p = z - lse,  lp = log p_y,  H = -sum p log p
// and with the rollout's lp0, a reference policy's lpr, advantage A, weight w,
// d = clamp(lp - lp0, +-20), ratio = e^d, u = clamp(lpr - lp, +-20):
//     policy = max(-A ratio, -A clip(ratio, 1 - low, 1 + high)), for A < 0 at most -A dual
//     kl = e^u - 1 - u,   loss = sum over rows of w (policy + kl_coef kl - ent_coef H)
//     dloss / dl_v = w / temperature ((1[v = y] - p_v) g + ent_coef p_v (log p_v + H)),
//     g = dpolicy / dlp + kl_coef (1 - e^u), a part being 0 where its clamp or clip holds.
//
// Everything about a row follows from its largest logit m, s = sum e^x and
// u = sum e^x (l - m), x = (l - m) / temperature: lp = x_y - log s,
// H = log s - u / (temperature s). Parts of a row are merged by rescaling to the
// larger m; s and u are float32. Logits are subtracted before they are scaled, so
// that a row of the type's lowest values is an even distribution.

#include "pda_rows.h"

namespace pda {
namespace {

constexpr float kClamp = 20.f;  // bound on log ratios

// x within +-20; NaN stays NaN.
__device__ __forceinline__ float clamped(float x) { return x < -kClamp ? -kClamp : x > kClamp ? kClamp : x; }

// A row's loss terms (times its weight) and the loss's derivative by lp.
__device__ __forceinline__ float policy_terms(const LogitsArgs& a, int t, const RowStats& r, float w, float (&out)[kTerms]) {
  const float A = a.adv[t], x = r.lp - a.old_logp[t];
  const float d = clamped(x), ratio = expf(d);
  const float plain = -A * ratio, cut = -A * fminf(fmaxf(ratio, 1.f - a.clip_low), 1.f + a.clip_high);
  bool held = cut > plain;
  float policy = held ? cut : plain;
  if (a.dual > 0.f && A < 0.f && policy > -A * a.dual) {
    policy = -A * a.dual;
    held = true;
  }
  float g = held || !(fabsf(x) <= kClamp) ? 0.f : plain, kl = 0.f;
  if (a.ref_logp) {
    const float y = a.ref_logp[t] - r.lp, u = clamped(y), em = expm1f(u);
    kl = em - u;
    if (fabsf(y) <= kClamp) g -= a.kl * em;
  }
  const float v[kTerms] = {policy + a.kl * kl - a.ent_coef * r.ent, policy, kl, r.ent, held ? 1.f : 0.f, ratio,
                           expm1f(-d) + d, 1.f};
#pragma unroll
  for (int i = 0; i < kTerms; ++i) out[i] = w != 0.f ? w * v[i] : 0.f;
  return g;
}

// dl_v = p_v (base + slope x), x = l_v - m, p_v = exp2(x c - log2 s); + at_y for the target.
// The exponent is rounded to float32, c and log2 s before it: p_v is off by some 2^-24 |x c|, 1e-6 where p_v
// is e^-20 (a division of the sums' own exponentials would keep 1e-7, and the exponentials a row long).
struct Grad {
  float m, c, log2_s, base, slope, at_y;
  bool zero;
};
__device__ __forceinline__ Grad row_grad(const LogitsArgs& a, const Soft& x, const RowStats& r, float g, float w, float c) {
#pragma clang fp contract(off)  // the products rounded: a target of probability 1 has gradient 0
  const float k = w * a.grad_scale * a.inv_temp;
  Grad d;
  d.zero = k == 0.f || x.s == 0.f;
  d.m = x.m;
  d.c = c;
  d.log2_s = r.log_s * kLog2e;
  d.base = k * (a.ent_coef * (r.ent - r.log_s) - g);
  d.slope = k * a.ent_coef * a.inv_temp;
  d.at_y = k * g;
  return d;
}
__device__ __forceinline__ float grad_of(const Grad& d, float l) {
  const float x = l - d.m;
  return __builtin_amdgcn_exp2f(fmaf(x, d.c, -d.log2_s)) * fmaf(d.slope, fmaxf(x, kFar), d.base);
}

// ------------------------------------------------------------- parts of rows

// Workgroup (row, part). A whole row's log-probability and entropy are written;
// of a part, or for policy_part_kernel, the sums. With counts the last part's
// workgroup of a row finishes it.
// 8192 x 131,072 bf16: 333 us, 6.4 TB/s, where the vector ALUs are busy for 97% of
// the cycles (9.4 instructions an element, an exponential of twice the cycles among
// them). Largest values of bf16 pairs by packed integer maxima, 5% fewer instructions, gave
// nothing.
template <typename T, int U, bool STREAM>
__global__ __launch_bounds__(kPartThreads) void sums_kernel(LogitsArgs a) {
  const int t = (int)(blockIdx.x / (uint32_t)a.splits), p = (int)(blockIdx.x - (uint32_t)t * a.splits);
  const int y = target_of(a, t);
  const bool whole = a.splits == 1 && !a.terms;
  if (y < 0) {
    if ((whole || (p == 0 && a.counts && !a.terms)) && threadIdx.x == 0) {
      a.logp[t] = 0.f;
      if (a.ent) a.ent[t] = 0.f;
    }
    return;
  }
  const T* row = static_cast<const T*>(a.logits) + (int64_t)t * a.stride;
  const Span sp = row_span(row, a.V);
  const int first = p * a.chunk, end = min(first + a.chunk, sp.vectors), odd = odd_of<T>(sp, a.V);
  const float c = a.inv_temp * kLog2e, ly = load1(row + y);
  Soft x = sum_vectors<T, U, STREAM>(row + sp.head, first, end, c);
  if (p == a.splits - 1 && odd >= 0) add1(x, load1(row + odd), c);
  x = group_merge<kPartThreads>(x, c);
  if (whole) {
    if (threadIdx.x) return;
    const RowStats r = row_stats(a, x, ly);
    a.logp[t] = r.lp;
    if (a.ent) a.ent[t] = r.ent;
    return;
  }
  uint64_t before = 0;
  if (threadIdx.x == 0) {
    float* part = reinterpret_cast<float*>(a.part + (int64_t)t * a.splits + p);
    store_part(part, x.m, x.s);
    store_part(part + 2, x.u, ly);
  }
  if (!a.counts || a.terms) return;
  if (threadIdx.x == 0) {
    parts_written();
    before = arrive(a.counts + t * kShortCountStride, a.epoch);
  }
  if (!last_of(before, a.epoch, a.splits) || threadIdx.x >= 64) return;
  x = merge_parts(a, t, c);
  if (threadIdx.x) return;
  const RowStats r = row_stats(a, x, ly);
  a.logp[t] = r.lp;
  if (a.ent) a.ent[t] = r.ent;
}

// A wave per row.
__global__ __launch_bounds__(kPartThreads) void finish_kernel(LogitsArgs a) {
  const int t = (int)(blockIdx.x * (kPartThreads / 64) + (threadIdx.x >> 6));
  if (t >= a.T) return;
  const int64_t y = a.targets64 ? static_cast<const int64_t*>(a.targets)[t] : static_cast<const int32_t*>(a.targets)[t];
  RowStats r = {0.f, 0.f, 0.f};
  if (y >= 0 && y < a.V) {
    const Soft x = merge_parts(a, t, a.inv_temp * kLog2e);
    r = row_stats(a, x, a.part[(int64_t)t * a.splits].w);
  }
  if ((threadIdx.x & 63) == 0) {
    a.logp[t] = r.lp;
    if (a.ent) a.ent[t] = r.ent;
  }
}

// The target's gradient, by the thread that wrote the others around it.
template <typename T>
__device__ __forceinline__ void store_target(T* out, int y, float ly, const Grad& d) {
  store1(out + y, grad_of(d, ly) + d.at_y);
}

// What thread 0 of a row writes beside the gradient; with counts also its arrival.
__device__ __forceinline__ uint64_t write_row(const LogitsArgs& a, int t, const RowStats& r, const float (&terms)[kTerms]) {
  write_terms(a, t, terms);
  if (a.logp) a.logp[t] = r.lp;
  if (a.ent) a.ent[t] = r.ent;
  if (!a.counts) return 0;
  parts_written();
  return arrive(a.counts, a.epoch);
}

// Workgroup (row, part), after sums_kernel: the loss's terms and the gradient.
// Returns thread 0's arrival.
template <typename T, bool STREAM>
__device__ __forceinline__ uint64_t policy_part(const LogitsArgs& a) {
  const int t = (int)(blockIdx.x / (uint32_t)a.splits), p = (int)(blockIdx.x - (uint32_t)t * a.splits);
  const int y = target_of(a, t);
  const T* row = static_cast<const T*>(a.logits) + (int64_t)t * a.stride;
  const Span sp = row_span(row, a.V);
  const int first = p * a.chunk, end = min(first + a.chunk, sp.vectors);
  const bool odds = p == a.splits - 1;
  T* out = static_cast<T*>(a.dlogits) + (int64_t)t * a.d_stride;
  float terms[kTerms] = {};
  uint64_t before = 0;
  if (y < 0) {
    if (p == 0 && threadIdx.x == 0) before = write_row(a, t, RowStats{0.f, 0.f, 0.f}, terms);
    if (a.dlogits) zero_vectors<STREAM>(out, sp, first, end, odds, a.V);
    return before;
  }
  const float c = a.inv_temp * kLog2e, w = a.weight[t], ly = a.part[(int64_t)t * a.splits].w;
  const Soft x = merge_parts(a, t, c);
  const RowStats r = row_stats(a, x, ly);
  const float g = policy_terms(a, t, r, w, terms);
  if (p == 0 && threadIdx.x == 0) before = write_row(a, t, r, terms);
  if (!a.dlogits) return before;
  const Grad d = row_grad(a, x, r, g, w, c);
  if (d.zero) {
    zero_vectors<STREAM>(out, sp, first, end, odds, a.V);
    return before;
  }
  for (int i = first + (int)threadIdx.x; i < end; i += kPartThreads) {
    const u32x4 v = load_vec<false>(row + sp.head, i);
    float o[kPer<T>];
#pragma unroll
    for (int e = 0; e < kPer<T>; ++e) o[e] = grad_of(d, element<T>(v, e));
    store_vec<STREAM>(out + sp.head, i, o);
    if (y >= sp.head && i == (y - sp.head) / kPer<T>) store_target(out, y, ly, d);
  }
  const int odd = odd_of<T>(sp, a.V);
  if (odds && odd >= 0) {
    store1(out + odd, grad_of(d, load1(row + odd)));
    if (odd == y) store_target(out, y, ly, d);
  }
  return before;
}

template <typename T, bool STREAM>
__global__ __launch_bounds__(kPartThreads) void policy_part_kernel(LogitsArgs a) {
  const uint64_t before = policy_part<T, STREAM>(a);
  // rows arrive with their first part
  if (a.counts && blockIdx.x % (uint32_t)a.splits == 0 && last_of(before, a.epoch, a.T)) sum_terms<kPartThreads, 1>(a);
}

// ------------------------------------------------------------- rows in registers

// Workgroup per row, whose vectors stay in its threads' registers (N of a thread)
// and LDS (L of a thread) between the sums and the gradient: one read and one
// write of the row.
// 4096 x 131,072 bf16: 418 us with the rows' sum, 5.1 TB/s (a 2 GiB device copy: 5.0). A long row's
// workgroup fills its compute unit, so its reads, sums and writes follow one another; the
// vector ALUs are busy for 69% of the cycles. The gradient without the entropy's
// instructions where its coefficient is 0 took 398 us instead of 416, but its second copy of
// the code took 428 us instead of 414 with a coefficient.
// Returns thread 0's arrival.
template <typename T, int NT, int N, int L, bool STREAM>
__device__ __forceinline__ uint64_t policy_row(const LogitsArgs& a) {
  const int t = (int)blockIdx.x, y = target_of(a, t);
  const T* row = static_cast<const T*>(a.logits) + (int64_t)t * a.stride;
  const Span sp = row_span(row, a.V);
  T* out = static_cast<T*>(a.dlogits) + (int64_t)t * a.d_stride;
  float terms[kTerms] = {};
  uint64_t before = 0;
  if (y < 0) {
    if (threadIdx.x == 0) before = write_row(a, t, RowStats{0.f, 0.f, 0.f}, terms);
    if (a.dlogits) zero_vectors<STREAM>(out, sp, 0, sp.vectors, true, a.V);
    return before;
  }
  const int odd = odd_of<T>(sp, a.V);
  const float c = a.inv_temp * kLog2e, ly = load1(row + y), w = a.weight[t];
  __shared__ u32x4 more[L ? L : 1][L ? NT : 1];
  static_assert(L % 3 == 0, "three at a time");
#pragma unroll
  for (int l = 0; l < L; ++l) {
    const int i = (int)threadIdx.x + (N + l) * NT;
    more[l][threadIdx.x] = i < sp.vectors ? load_vec<true>(row + sp.head, i) : nothing<T>();
  }
  u32x4 v[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int i = (int)threadIdx.x + n * NT;
    v[n] = i < sp.vectors ? load_vec<true>(row + sp.head, i) : nothing<T>();
  }
  const float lodd = odd >= 0 ? load1(row + odd) : -__builtin_huge_valf();
  Soft x = none();
  add<T>(x, v, c, (sp.vectors - __builtin_amdgcn_readfirstlane((int)threadIdx.x) + NT - 1) / NT);
  for (int l = 0; l < L; l += 3) {
    u32x4 m[3] = {more[l][threadIdx.x], more[l + 1][threadIdx.x], more[l + 2][threadIdx.x]};
    add<T>(x, m, c);
  }
  add1(x, lodd, c);
  x = group_merge<NT>(x, c);
  const RowStats r = row_stats(a, x, ly);
  const float g = policy_terms(a, t, r, w, terms);
  if (threadIdx.x == 0) before = write_row(a, t, r, terms);
  if (!a.dlogits) return before;
  const Grad d = row_grad(a, x, r, g, w, c);
  if (d.zero) {
    zero_vectors<STREAM>(out, sp, 0, sp.vectors, true, a.V);
    return before;
  }
  auto put = [&](int i, const u32x4& l) {
    float o[kPer<T>];
#pragma unroll
    for (int e = 0; e < kPer<T>; ++e) o[e] = grad_of(d, element<T>(l, e));
    store_vec<STREAM>(out + sp.head, i, o);
    if (y >= sp.head && i == (y - sp.head) / kPer<T>) store_target(out, y, ly, d);
  };
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int i = (int)threadIdx.x + n * NT;
    if (i >= sp.vectors) break;
    again(v[n]);
    put(i, v[n]);
  }
  for (int l = 0; l < L; ++l) {
    const int i = (int)threadIdx.x + (N + l) * NT;
    if (i < sp.vectors) put(i, more[l][threadIdx.x]);
  }
  if (odd >= 0) {
    store1(out + odd, grad_of(d, lodd));
    if (odd == y) store_target(out, y, ly, d);
  }
  return before;
}

// Only workgroups of this size finish a counted call's sums (few longer rows go in parts).
constexpr int kFinishThreads = 256;
template <typename T, int NT, int N, int L, bool STREAM>
__global__ __launch_bounds__(NT) void policy_row_kernel(LogitsArgs a) {
  const uint64_t before = policy_row<T, NT, N, L, STREAM>(a);
  if constexpr (NT == kFinishThreads) {
    if (a.counts && last_of(before, a.epoch, a.T)) sum_terms<NT, 1>(a);
  }
}

__global__ __launch_bounds__(1024) void stats_kernel(LogitsArgs a) { sum_terms<1024, 8>(a); }

hipError_t launch(const void* kernel, int64_t wgs, int threads, const LogitsArgs& a, hipStream_t s) {
  LogitsArgs args = a;
  void* params[] = {&args};
  return hipLaunchKernel(kernel, dim3((unsigned)wgs), dim3((unsigned)threads), params, 0, s);
}

// Eight 16-byte loads of a thread in flight, four where a part has no more for
// it (64 x 131072 bf16: 8.6 and 6.2 us). Long parts that are read once are streamed; short ones
// are not (8.5 us per call, 8.8 streamed).
template <typename T>
hipError_t sums_for(const LogitsArgs& a, hipStream_t s) {
  const void* k = a.chunk < 8 * kPartThreads ? reinterpret_cast<const void*>(&sums_kernel<T, 4, false>)
                  : a.terms ? reinterpret_cast<const void*>(&sums_kernel<T, 8, false>)
                            : reinterpret_cast<const void*>(&sums_kernel<T, 8, true>);
  return launch(k, (int64_t)a.T * a.splits, kPartThreads, a, s);
}

template <typename T>
hipError_t logprobs_for(const LogitsArgs& a, hipStream_t s) {
  hipError_t e = sums_for<T>(a, s);
  if (e != hipSuccess || a.splits == 1 || a.counts) return e;
  constexpr int rows = kPartThreads / 64;
  return launch(reinterpret_cast<const void*>(&finish_kernel), (a.T + rows - 1) / rows, kPartThreads, a, s);
}

// Bytes of a gradient from which it is stored past the caches, for the products that read
// it to find what they need of the rest. us, stored through them / past them, of the call
// alone, and with its logits' producer and the gradient's two products (by 1,024 hidden dims)
// around it; bf16: 1,024 x 4,000 11.0 / 10.9, 64 / 71; 256 x 8,000 9.6 / 9.6, 61 / 66; 300 x 20,000
// 14.1 / 13.5, 166 / 166; 2,048 x 4,000 16.1 / 15.0, 85 / 89; 1,024 x 8,000 13.6 / 12.8, 89 / 90; 1,024 x 16,000
// 19.8 / 16.9, 140 / 142; 512 x 131,072 60.5 / 59.4, 734 / 733; 4,096 x 131,072 427 / 435, 3,199 / 3,153;
// f32 2,048 x 110,000 377 / 356.
constexpr int64_t kStreamBytes = 10 << 20;

template <typename T>
bool streamed(const LogitsArgs& a) {
  return (int64_t)a.T * a.V * (int64_t)sizeof(T) >= kStreamBytes;
}

// Rows of more than kFinishThreads threads come in numbers that make 7 MB and more, and are always streamed.
template <typename T, int NT, int N, int L = 0>
hipError_t rows_for(const LogitsArgs& a, hipStream_t s) {
  const void* k = reinterpret_cast<const void*>(&policy_row_kernel<T, NT, N, L, true>);
  if constexpr (NT == kFinishThreads) {
    if (!streamed<T>(a)) k = reinterpret_cast<const void*>(&policy_row_kernel<T, NT, N, L, false>);
  }
  return launch(k, a.T, NT, a, s);
}

template <typename T>
hipError_t policy_for(LogitsArgs a, hipStream_t s) {
  hipError_t e = hipSuccess;
  if (!a.splits && a.V / kPer<T> > kFinishThreads * 16) a.counts = nullptr;  // the sums take a launch of their own
  if (a.splits) {
    const int64_t wgs = (int64_t)a.T * a.splits;
    e = sums_for<T>(a, s);
    const void* k = streamed<T>(a) ? reinterpret_cast<const void*>(&policy_part_kernel<T, true>)
                                   : reinterpret_cast<const void*>(&policy_part_kernel<T, false>);
    if (e == hipSuccess) e = launch(k, wgs, kPartThreads, a, s);
  } else if (a.T) {
    const int v = a.V / kPer<T>;
    e = v <= kFinishThreads * 4 ? rows_for<T, kFinishThreads, 4>(a, s)
        : v <= kFinishThreads * 8 ? rows_for<T, kFinishThreads, 8>(a, s)
        : v <= kFinishThreads * 16 ? rows_for<T, kFinishThreads, 16>(a, s)
        : v <= 512 * 16 ? rows_for<T, 512, 16>(a, s)
        : v <= 1024 * 16 ? rows_for<T, 1024, 16>(a, s)
        : v <= 1024 * 20 ? rows_for<T, 1024, 20>(a, s) : rows_for<T, 1024, 19, 9>(a, s);
  }
  if (e != hipSuccess || a.counts) return e;
  return launch(reinterpret_cast<const void*>(&stats_kernel), 1, 1024, a, s);
}

}  // namespace

hipError_t launch_token_logprobs(const LogitsArgs& a, hipStream_t s) {
  return a.bf16 ? logprobs_for<uint16_t>(a, s) : logprobs_for<float>(a, s);
}

hipError_t launch_policy_loss(const LogitsArgs& a, hipStream_t s) {
  return a.bf16 ? policy_for<uint16_t>(a, s) : policy_for<float>(a, s);
}

}  // namespace pda
