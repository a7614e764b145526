// Rows of logits in the kernels that read them (pda_policy.hip, pda_top.hip,
// pda_distill.hip): their vectors, their sums as a running maximum with the sums of exponentials below it,
// and the rows' terms of a loss.
//
// Everything about a row follows from its largest logit m, s = sum e^x and
// u = sum e^x (l - m), x = (l - m) / temperature: the log-probability of word y is
// x_y - log s, the entropy log s - u / (temperature s).
#pragma once

#include "pda_arrive.h"
#include "pda_elem.h"
#include "pda_ops_internal.h"

namespace pda {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.402823466e38f;
constexpr float kFar = -1e25f;  // bound on differences in products with a zero: their exponential is 0 below temperatures of 1e23
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

// A row's loss terms.
__device__ __forceinline__ void write_terms(const LogitsArgs& a, int t, const float (&v)[kTerms]) {
#pragma unroll
  for (int i = 0; i < kTerms; i += 2) store_part(a.terms + (int64_t)t * kTerms + i, v[i], v[i + 1]);
}

// The rows' terms summed in float64, in an order that no NT changes: row t goes to
// sum t % kSums, U rows of each at a time, and the sums are added as a tree; the first OUT are written.
constexpr int kSums = 128;
template <int NT, int U, int OUT = kTerms>
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
  if (threadIdx.x < OUT) a.stats[threadIdx.x] = (float)sums[0][threadIdx.x];
}

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

// Zeros in vectors first .. end - 1, and with `odds` in the elements outside of the vectors.
template <bool STREAM, typename T>
__device__ __forceinline__ void zero_vectors(T* out, const Span& sp, int first, int end, bool odds, int V) {
  const float z[kPer<T>] = {};
  for (int i = first + (int)threadIdx.x; i < end; i += (int)blockDim.x) store_vec<STREAM>(out + sp.head, i, z);
  const int odd = odd_of<T>(sp, V);
  if (odds && odd >= 0) store1(out + odd, 0.f);
}

// Over the 64 lanes, in each of them (in one order of additions for all).
__device__ __forceinline__ float wave_total(float x) {
  x = group_sum<16>(x);
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}
__device__ __forceinline__ double wave_total(double x) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) x += __shfl_xor(x, o, 64);
  return x;
}
__device__ __forceinline__ float wave_top(float x) {
  x = group_max<16>(x);
  x = fmaxf(x, __shfl_xor(x, 16, 64));
  return fmaxf(x, __shfl_xor(x, 32, 64));
}

// ------------------------------------------------------------- sums in base 2

// For exponentials below a logit m, 2^(l c - k) with k = m c rounded, one instruction and one rounding before the
// exponential: sums of such terms are 2^off times those of 2^((l - m) c), off = m c - k exactly, so that the rounding of k
// costs nothing. Where k is so large that its rounding is not small (lowest values, temperatures near 0: FAR), logits are
// subtracted first, and off is 0.
struct Base2 {
  float c, k, m;
  bool far;
  template <bool FAR>
  __device__ __forceinline__ float of(float l) const {
    return FAR ? (l - m) * c : fmaf(l, c, -k);
  }
  __device__ __forceinline__ float of(float l) const { return far ? of<true>(l) : of<false>(l); }
  __device__ __forceinline__ float off() const { return far ? 0.f : fmaf(m, c, -k); }
};
// c for logits: 1 / temperature in base 2.
__device__ __forceinline__ float base2_rate(const LogitsArgs& a) { return fminf(a.inv_temp * kLog2e, -kLowest); }
__device__ __forceinline__ Base2 base2(float m, float c) {
  const float k = m * c;
  return Base2{c, k, m, !(fabsf(k) < 0x1p22f)};
}
// The exponent by which sums below `from` go on below m >= from.
__device__ __forceinline__ float exponent_to(float from, float m, float c) {
#pragma clang fp contract(off)  // rounded products, as in base2
  const Base2 a = base2(from, c), b = base2(m, c);
  return a.far || b.far ? (from - m) * c + (b.off() - a.off()) : a.k - b.k;
}
// Natural logarithm of a sum below m, had its terms been 2^((l - m) c).
__device__ __forceinline__ float log_below(float s, float m, float c) { return fmaf(base2(m, c).off(), -1.f / kLog2e, logf(s)); }

}  // namespace pda
