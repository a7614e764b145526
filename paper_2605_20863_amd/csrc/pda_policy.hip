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

#include "pda_arrive.h"
#include "pda_elem.h"
#include "pda_ops_internal.h"

namespace pda {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.402823466e38f;
constexpr float kFar = -1e25f;  // bound on differences in products with a zero: their exponential is 0 below temperatures of 1e23
constexpr float kClamp = 20.f;  // bound on log ratios
constexpr int kPartThreads = 256;

// Rows have the alignment of their elements only; vectors of the logits are taken
// from each row's first 16-byte boundary on, those of the gradient wherever that
// leaves them (8192 x 50,257 bf16, policy loss: 363 us per call with vectors from the
// rows' starts, 308 so).
typedef u32x4 __attribute__((aligned(2))) u32x4_any;

template <typename T>
constexpr int kPer = 16 / (int)sizeof(T);  // elements of a vector

// -inf in every element
template <typename T>
__device__ __forceinline__ u32x4 nothing() {
  const uint32_t w = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
  return u32x4{w, w, w, w};
}

template <typename T>
__device__ __forceinline__ float element(const u32x4& v, int i) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t w = v[i / 2];
    return as_f32(i & 1 ? w & 0xFFFF0000u : w << 16);
  } else {
    const uint32_t w = v[i];
    return as_f32(w);
  }
}

template <typename T>
__device__ __forceinline__ float load1(const T* p) {
  if constexpr (sizeof(T) == 2) return as_f32((uint32_t)*p << 16);
  else return *p;
}

// A row's whole vectors, behind its first `head` elements.
struct Span {
  int head, vectors;
};
template <typename T>
__device__ __forceinline__ Span row_span(const T* row, int V) {
  const int head = min((int)((0 - reinterpret_cast<uintptr_t>(row)) & 15) / (int)sizeof(T), V);
  return Span{head, (V - head) / kPer<T>};
}
// The element outside of the vectors that is this thread's, -1 if none is.
template <typename T>
__device__ __forceinline__ int odd_of(const Span& s, int V) {
  const int t = (int)threadIdx.x, in = s.vectors * kPer<T>;
  return t >= V - in ? -1 : t < s.head ? t : t + in;
}

// Vector i from `row` on, all of it in the row. STREAM: what is
// not read again soon, past the caches (log-probabilities of 8192 x 131072 bf16:
// 364 - 374 us per call without, 355 - 358 with).
template <bool STREAM, typename T>
__device__ __forceinline__ u32x4 load_vec(const T* row, int i) {
  const u32x4_any* p = reinterpret_cast<const u32x4_any*>(row + (int64_t)i * kPer<T>);
  return STREAM ? __builtin_nontemporal_load(p) : *p;
}

// STREAM as the launcher says (kStreamBytes).
template <bool STREAM, typename T>
__device__ __forceinline__ void store_vec(T* row, int i, const float (&y)[kPer<T>]) {
  u32x4 v;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = pack_bf16(y[2 * e], y[2 * e + 1]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = as_u32(y[e]);
  }
  u32x4_any* p = reinterpret_cast<u32x4_any*>(row + (int64_t)i * kPer<T>);
  if constexpr (STREAM) __builtin_nontemporal_store(v, p);
  else *p = v;
}

template <typename T>
__device__ __forceinline__ void store1(T* p, float y) {
  if constexpr (sizeof(T) == 2) *p = to_bf16(y);
  else *p = y;
}

struct Soft {
  float m, s, u;
};
__device__ __forceinline__ Soft none() { return Soft{kLowest, 0.f, 0.f}; }

// x's sums as of the larger maximum m.
__device__ __forceinline__ Soft rebase(const Soft& x, float m, float c) {
  const float d = x.m - m, f = __builtin_amdgcn_exp2f(d * c);
  return Soft{m, x.s * f, f * fmaf(x.s, fmaxf(d, kFar), x.u)};
}
__device__ __forceinline__ Soft merge(const Soft& a, const Soft& b, float c) {
  const float m = fmaxf(a.m, b.m);
  const Soft x = rebase(a, m, c), y = rebase(b, m, c);
  return Soft{m, x.s + y.s, x.u + y.u};
}

// Makes the compiler unpack a vector's elements again after this point, rather
// than keep them all in registers of their own (twice the vector's for bf16).
__device__ __forceinline__ void again(u32x4& v) { asm volatile("" : "+v"(v)); }

// Adds the first `live` of N vectors' elements to x (a number that is the same in
// the wave: 8192 x 17,000 bf16, with vectors for 32,768, 125 us per call with all of them, 104 so).
template <typename T, int N>
__device__ __forceinline__ void add(Soft& x, u32x4 (&v)[N], float c, int live = N) {
  float m = x.m;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (n >= live) continue;
#pragma unroll
    for (int e = 0; e < kPer<T>; ++e) m = fmaxf(m, element<T>(v[n], e));
  }
  x = rebase(x, m, c);
#pragma unroll
  for (int n = 0; n < N; ++n) again(v[n]);
  // these vectors' own sums: one chain of additions through a thread's whole part lost
  // digits (8192 x 131,072 bf16: 2.3e-7 from 64 bits, 6.7e-8 so, for 1% of the time)
  float s = 0.f, u = 0.f;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (n >= live) continue;
#pragma unroll
    for (int e = 0; e < kPer<T>; ++e) {
      const float d = element<T>(v[n], e) - m, p = __builtin_amdgcn_exp2f(d * c);
      s += p;
      u = fmaf(p, fmaxf(d, kFar), u);
    }
  }
  x.s += s;
  x.u += u;
}

// Adds one element.
__device__ __forceinline__ void add1(Soft& x, float l, float c) {
  const float m = fmaxf(x.m, l);
  x = rebase(x, m, c);
  const float d = l - m, p = __builtin_amdgcn_exp2f(d * c);
  x.s += p;
  x.u = fmaf(p, fmaxf(d, kFar), x.u);
}

// Over the aligned group of N lanes, in each of them.
template <int N>
__device__ __forceinline__ Soft lanes_merge(Soft x, float c) {
#pragma unroll
  for (int o = 1; o < N; o *= 2)
    x = merge(x, Soft{__shfl_xor(x.m, o, 64), __shfl_xor(x.s, o, 64), __shfl_xor(x.u, o, 64)}, c);
  return x;
}

// Over the workgroup, in every thread (and a barrier for all of them).
template <int NT>
__device__ __forceinline__ Soft group_merge(Soft x, float c) {
  constexpr int W = NT / 64;
  __shared__ Soft parts[W];
  x = lanes_merge<64>(x, c);
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = x;
  __syncthreads();
  return lanes_merge<W>(parts[threadIdx.x % W], c);
}

// Row t's target, or -1 for a row that takes no part.
__device__ __forceinline__ int target_of(const LogitsArgs& a, int t) {
  const int64_t y = a.targets64 ? static_cast<const int64_t*>(a.targets)[t] : static_cast<const int32_t*>(a.targets)[t];
  if (y >= a.V) {
    if (threadIdx.x == 0) atomicOr(a.status, kStatusBadTarget);
    return -1;
  }
  return y < 0 ? -1 : (int)y;
}

struct RowStats {
  float lp, ent, log_s;
};
// From a row's sums and its target's logit.
__device__ __forceinline__ RowStats row_stats(const LogitsArgs& a, const Soft& x, float ly) {
  RowStats r;
  if (x.s == 0.f) {  // every logit is -inf: no distribution
    r.lp = -__builtin_huge_valf();
    r.ent = r.log_s = 0.f;
    return r;
  }
  r.log_s = logf(x.s);
  r.lp = (ly - x.m) * a.inv_temp - r.log_s;
  r.ent = r.log_s - x.u / x.s * a.inv_temp;
  return r;
}

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

__device__ __forceinline__ void write_terms(const LogitsArgs& a, int t, const float (&v)[kTerms]) {
#pragma unroll
  for (int i = 0; i < kTerms; i += 2) store_part(a.terms + (int64_t)t * kTerms + i, v[i], v[i + 1]);
}

// The rows' terms summed in float64, in an order that no NT changes: row t goes to
// sum t % kSums, U rows of each at a time, and the sums are added as a tree.
constexpr int kSums = 128;
template <int NT, int U>
__device__ __forceinline__ void sum_terms(const LogitsArgs& a) {
  constexpr int S = kSums * kTerms / NT;  // sums of a thread
  __shared__ double sums[kSums][kTerms];
  const int k = (int)threadIdx.x % kTerms, r = (int)threadIdx.x / kTerms;
  double x[S] = {};
  for (int t0 = 0; t0 < a.T; t0 += U * kSums) {
    float v[S][U];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int t = t0 + i * kSums + r + s * (NT / kTerms);
        v[s][i] = load_part(a.terms + (int64_t)min(t, a.T - 1) * kTerms + k);
        if (t >= a.T) v[s][i] = 0.f;
      }
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int i = 0; i < U; ++i) x[s] += (double)v[s][i];
  }
#pragma unroll
  for (int s = 0; s < S; ++s) sums[r + s * (NT / kTerms)][k] = x[s];
  __syncthreads();
  for (int n = kSums / 2; n > 0; n /= 2) {
    for (int i = (int)threadIdx.x; i < n * kTerms; i += NT) sums[i / kTerms][i % kTerms] += sums[i / kTerms + n][i % kTerms];
    __syncthreads();
  }
  if (threadIdx.x < kTerms) a.stats[threadIdx.x] = (float)sums[0][threadIdx.x];
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

// Sums of vectors first .. end - 1 of a row, by the workgroup's threads; U
// vectors of a thread at a time.
template <typename T, int U, bool STREAM>
__device__ __forceinline__ Soft sum_vectors(const T* row, int first, int end, float c) {
  Soft x = none();
  int i = first + (int)threadIdx.x;
  for (; i + (U - 1) * kPartThreads < end; i += kPartThreads * U) {
    u32x4 v[U];
#pragma unroll
    for (int n = 0; n < U; ++n) v[n] = load_vec<STREAM>(row, i + n * kPartThreads);
    add<T>(x, v, c);
  }
  for (; i < end; i += kPartThreads) {
    u32x4 v[1] = {load_vec<STREAM>(row, i)};
    add<T>(x, v, c);
  }
  return x;
}

// A row's parts merged, in every lane of a wave.
__device__ __forceinline__ Soft merge_parts(const LogitsArgs& a, int t, float c) {
  const int l = (int)(threadIdx.x & 63);
  const float* q = reinterpret_cast<const float*>(a.part + (int64_t)t * a.splits + min(l, a.splits - 1));
  const Soft x = {load_part(q), load_part(q + 1), load_part(q + 2)};
  return lanes_merge<64>(l < a.splits ? x : none(), c);
}

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

// Zeros in vectors first .. end - 1, and with `odds` in the elements outside of the vectors.
template <bool STREAM, typename T>
__device__ __forceinline__ void zero_vectors(T* out, const Span& sp, int first, int end, bool odds, int V) {
  const float z[kPer<T>] = {};
  for (int i = first + (int)threadIdx.x; i < end; i += (int)blockDim.x) store_vec<STREAM>(out + sp.head, i, z);
  const int odd = odd_of<T>(sp, V);
  if (odds && odd >= 0) store1(out + odd, 0.f);
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
