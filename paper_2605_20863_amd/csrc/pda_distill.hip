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
// one factor a row times a word's share of the rest. A bit in LDS for each of a row's words says which are listed: one
// LDS read for a vector of 16 bytes, whose listed words are made -inf as it is loaded. Their gradients are written
// over the vectors' by the threads that wrote these, after them.
//
// With rest, sum p + p_r = 1 turns the divergences into sums of terms that are not
// negative, which keeps their digits where teacher and student are close:
//     F = sum t (e^a - 1 - a) + (S + t_r - 1),  R = sum p (e^-a - 1 + a) - (S + t_r - 1).

#include "pda_lm_internal.h"
#include "pda_rows.h"

namespace pda {
namespace {

constexpr double kLeastRest = 0x1p-24;  // half a step of float32 below 1: what a sum of t can tell from it
constexpr int kListThreads = 256;       // the first threads of a workgroup hold a list's places
static_assert(kMaxTop <= kListThreads, "a place a thread");
static_assert(kPartThreads >= kListThreads, "in every workgroup");

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

// Largest logit and sum of exponentials below it.
struct Mass {
  float m, s;
};
__device__ __forceinline__ Mass no_mass() { return Mass{kLowest, 0.f}; }
__device__ __forceinline__ Mass rebase(const Mass& x, float m, float c) {
  return Mass{m, x.s * __builtin_amdgcn_exp2f((x.m - m) * c)};
}
__device__ __forceinline__ Mass merge(const Mass& a, const Mass& b, float c) {
#pragma clang fp contract(off)  // the same whichever side is which, so that all lanes agree
  const float m = fmaxf(a.m, b.m);
  return Mass{m, rebase(a, m, c).s + rebase(b, m, c).s};
}
__device__ __forceinline__ void add1(Mass& x, float l, float c) {
  const float m = fmaxf(x.m, l);
  x = rebase(x, m, c);
  x.s += __builtin_amdgcn_exp2f((l - m) * c);
}
// The first `live` of N vectors' elements (as for Soft).
template <typename T, int N>
__device__ __forceinline__ void add(Mass& x, u32x4 (&v)[N], float c, int live = N) {
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
  float s = 0.f;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (n >= live) continue;
#pragma unroll
    for (int e = 0; e < kPer<T>; ++e) s += __builtin_amdgcn_exp2f((element<T>(v[n], e) - m) * c);
  }
  x.s += s;
}
__device__ __forceinline__ Mass wave_merge(Mass x, float c) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) x = merge(x, Mass{__shfl_xor(x.m, o, 64), __shfl_xor(x.s, o, 64)}, c);
  return x;
}
template <typename X>
__device__ __forceinline__ X wave_total(X x) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) x += __shfl_xor(x, o, 64);
  return x;
}

// ------------------------------------------------------------- the list

// A place of a row's list, thread k's the k-th.
struct Place {
  int id;  // -1: no word
  float tau, l;
};
__device__ __forceinline__ Place load_place(const DistillArgs& g, int t) {
  Place p = {-1, 0.f, kLowest};
  const int k = (int)threadIdx.x;
  if (k >= g.K) return p;
  p.id = g.ids[(int64_t)t * g.K + k];
  p.tau = g.tau[(int64_t)t * g.K + k];
  if (p.id >= g.z.V) {
    atomicOr(g.z.status, kStatusBadTarget);
    p.id = -1;
  }
  if (p.id < 0 || p.tau == -__builtin_huge_valf()) p.id = -1;
  return p;
}

// Vectors first .. end - 1 of a row, and with `odds` the elements outside of all vectors.
struct Range {
  int first, end;
  bool odds;
};

// For a range of V vectors: which of its words are listed, and the places whose words each of NT threads writes.
template <typename T, int NT, int V>
struct Listed {
  static constexpr int kOdd = V * kPer<T>;  // bits of the elements outside of all vectors, from here on
  uint32_t bits[kOdd / 32 + 1];
  int head[NT], next[kListThreads];  // a thread's places, -1: no more
  int id[kListThreads];
  float d[kListThreads];  // gradients
  int twice;

  __device__ __forceinline__ void clear() {
    for (int i = (int)threadIdx.x; i < kOdd / 32 + 1; i += NT) bits[i] = 0;
    head[threadIdx.x] = -1;
    if (threadIdx.x == 0) twice = 0;
  }

  // Between two barriers, after clear(): this thread's place goes to the thread that writes its word, if that is in
  // the range. Returns the word's bit, or -1.
  __device__ __forceinline__ int chain(const Place& p, const Span& sp, const Range& r) {
    const int k = (int)threadIdx.x;
    if (k >= kListThreads) return -1;
    id[k] = p.id;
    if (p.id < 0) return -1;
    const int at = p.id - sp.head, in = sp.vectors * kPer<T>, i = at / kPer<T>;
    const bool odd = at < 0 || at >= in;
    if (odd ? !r.odds : i < r.first || i >= r.end) return -1;
    const int owner = odd ? (at < 0 ? p.id : p.id - in) : (i - r.first) % NT;
    next[k] = atomicExch(&head[owner], k);
    return odd ? kOdd + owner : at - r.first * kPer<T>;
  }
  // The same, and its bit is set.
  __device__ __forceinline__ bool enter(const Place& p, const Span& sp, const Range& r) {
    const int bit = chain(p, sp, r);
    if (bit < 0) return false;
    if (atomicOr(&bits[bit / 32], 1u << (bit % 32)) >> (bit % 32) & 1) twice = 1;
    return true;
  }
  // After the barrier behind enter(): a word's further places leave the list.
  __device__ __forceinline__ void drop_further(Place& p, int K, int32_t* status) {
    if (!twice) return;
    const int k = (int)threadIdx.x;
    bool further = false;
    if (k < kListThreads)
      for (int j = 0; j < k; ++j) further |= p.id >= 0 && id[j] == p.id;
    __syncthreads();
    if (further) {
      atomicOr(status, kStatusTwice);
      p.id = id[k] = -1;
    }
  }

  // Vector n (counted from the range's first) with its listed words made -inf.
  __device__ __forceinline__ void leave_out(u32x4& v, int n) const {
    const uint32_t byte = reinterpret_cast<const uint8_t*>(bits)[n * kPer<T> / 8];
    const uint32_t mask = kPer<T> == 8 ? byte : byte >> (4 * (n & 1)) & 15;
    if (mask) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if constexpr (kPer<T> == 8) {
          v[w] = mask >> (2 * w) & 1 ? (v[w] & 0xFFFF0000u) | 0xFF80u : v[w];
          v[w] = mask >> (2 * w + 1) & 1 ? (v[w] & 0xFFFFu) | 0xFF800000u : v[w];
        } else {
          v[w] = mask >> w & 1 ? 0xFF800000u : v[w];
        }
      }
    }
  }
  __device__ __forceinline__ bool odd_listed() const { return bits[kOdd / 32] >> (kOdd % 32 + threadIdx.x) & 1; }

  // This thread's places' gradients, over what it wrote before.
  __device__ __forceinline__ void write(T* out) const {
    for (int k = head[threadIdx.x]; k >= 0; k = next[k])
      if (id[k] >= 0) store1(out + id[k], d[k]);
  }
};

// ------------------------------------------------------------- a row's results

struct Row {
  float loss;
  float terms[kTerms];
  float m, c, log2_s, outside;  // gradient outside of the list: exp2((l - m) c - log2_s) outside
  bool zero;                    // no gradient, whatever the logits
};

// What the waves of a workgroup hand each other.
template <int NT>
struct Parts {
  Mass rest[NT / 64], list[kListThreads / 64];
  double S[kListThreads / 64];
  float P[kListThreads / 64], f[kListThreads / 64], r[kListThreads / 64];
};

// From the sums of the words outside of the list (`all`: the row's, otherwise this thread's part) and the
// places; *d: the gradient by this thread's place's logit. Two barriers.
template <int NT>
__device__ __forceinline__ Row finish_row(const DistillArgs& g, int t, Mass rest, bool all, const Place& place, Parts<NT>& s, float* d) {
  constexpr int LW = kListThreads / 64;
  const LogitsArgs& a = g.z;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const bool first = (threadIdx.x & 63) == 0, in = place.id >= 0;
  const float c = a.inv_temp * kLog2e, w = a.weight[t];
  double t64 = 0.;
  if (!all) {
    rest = wave_merge(rest, c);
    if (first) s.rest[wave] = rest;
  }
  if (wave < LW) {
    Mass x = no_mass();
    if (in) add1(x, place.l, c);
    x = wave_merge(x, c);
    t64 = in ? exp((double)place.tau) : 0.;
    const double S = wave_total(t64);
    if (first) {
      s.list[wave] = x;
      s.S[wave] = S;
    }
  }
  __syncthreads();
  if (!all) {
    rest = s.rest[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) rest = merge(rest, s.rest[i], c);
  }
  Mass x = rest;
  double S64 = 0.;
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    x = merge(x, s.list[i], c);
    S64 += s.S[i];
  }
  const bool some = x.s != 0.f;  // NaN too; else every logit is -inf: no distribution
  const bool others = g.rest && rest.s != 0.f;
  const float log_s = logf(x.s), b = g.rev;
  const float lpr = (rest.m - x.m) * a.inv_temp + (logf(rest.s) - log_s), pr = rest.s != 0.f ? expf(lpr) : 0.f;
  const double t_rest = others ? fmax(1. - S64, kLeastRest) : 0.;
  const float tr = (float)t_rest, ar = others ? lpr - (float)log(t_rest) : 0.f;
  const float total = (float)(S64 + t_rest), over = (float)(S64 + t_rest - 1.);
  // this thread's place
  float tk = 0.f, p = 0.f, ta = 0.f, pa = 0.f;
  if (wave < LW) {
    const float lp = some ? (place.l - x.m) * a.inv_temp - log_s : -__builtin_huge_valf();
    const float ak = in ? lp - place.tau : 0.f;
    tk = (float)t64;
    p = in ? expf(lp) : 0.f;
    ta = tk == 0.f ? 0.f : tk * ak;
    pa = p == 0.f ? 0.f : p * ak;
    float f = -ta, r = pa;
    if (g.rest) {  // squares where a is near to 0
      const bool near = fabsf(ak) <= 1.f;
      f = near ? tk * phi(ak) : p - tk - ta;
      r = near ? p * phi(-ak) : tk - p + pa;
    }
    const float P = wave_total(p), F = wave_total(f), R = wave_total(r);
    if (first) {
      s.P[wave] = P;
      s.f[wave] = F;
      s.r[wave] = R;
    }
  }
  __syncthreads();
  float P = 0.f, F = 0.f, R = 0.f;
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    P += s.P[i];
    F += s.f[i];
    R += s.r[i];
  }
  const float k = w * a.grad_scale * a.inv_temp;
  Row o;
  o.zero = k == 0.f || !some;
  if (g.rest) {
    const float par = pr == 0.f ? 0.f : pr * ar;
    const bool near = fabsf(ar) <= 1.f;
    F += (near ? tr * phi(ar) : pr - tr - tr * ar) + over;
    R += (near ? pr * phi(-ar) : tr - pr + par) - over;
    *d = (1.f - b) * (p * total - tk) + b * (pa - p * R);
    o.outside = (1.f - b) * (pr * total - tr) + b * (par - pr * R);
  } else {
    *d = (1.f - b) * (p * total - tk) + b * (pa + p - p * (R + P));
    o.outside = pr * ((1.f - b) * total - b * (R + P));
  }
  *d *= k;
  o.outside *= k;
  if (!some) {
    F = S64 > 0. ? __builtin_huge_valf() : 0.f;
    R = 0.f;
  }
  o.loss = (b < 1.f ? (1.f - b) * F : 0.f) + (b > 0.f ? b * R : 0.f);
  const float v[kTerms] = {o.loss, F, R, (float)S64, P, 1.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kTerms; ++i) o.terms[i] = w != 0.f ? w * v[i] : 0.f;
  o.m = rest.m;
  o.c = c;
  o.log2_s = rest.s == 0.f ? 0.f : logf(rest.s) * kLog2e;
  return o;
}

template <typename T>
__device__ __forceinline__ float outside_of(const Row& o, float l) {
  return __builtin_amdgcn_exp2f(fmaf(l - o.m, o.c, -o.log2_s)) * o.outside;
}

// What thread 0 of a row writes beside the gradient; with counts also its arrival.
__device__ __forceinline__ uint64_t write_result(const DistillArgs& g, int t, const Row& o) {
  write_terms(g.z, t, o.terms);
  if (g.losses) g.losses[t] = o.loss;
  if (!g.z.counts) return 0;
  parts_written();
  return arrive(g.z.counts, g.z.epoch);
}

// Whether row t takes no part at all: of weight 0, and its loss not wanted.
__device__ __forceinline__ bool idle(const DistillArgs& g, int t) { return g.z.weight[t] == 0.f && !g.losses; }
__device__ __forceinline__ uint64_t write_idle(const DistillArgs& g, int t) {
  Row o = {};
  return write_result(g, t, o);
}

// ------------------------------------------------------------- rows in registers

// Workgroup per row, whose vectors stay in its threads' registers (N of a thread)
// and LDS (L of a thread) between the sums and the gradient: one read and one
// write of the row. Returns thread 0's arrival.
template <typename T, int NT, int N, int L, bool STREAM>
__device__ __forceinline__ uint64_t distill_row(const DistillArgs& g) {
  const LogitsArgs& a = g.z;
  const int t = (int)blockIdx.x;
  const T* row = static_cast<const T*>(a.logits) + (int64_t)t * a.stride;
  const Span sp = row_span(row, a.V);
  T* out = static_cast<T*>(a.dlogits) + (int64_t)t * a.d_stride;
  uint64_t before = 0;
  if (idle(g, t)) {
    if (threadIdx.x == 0) before = write_idle(g, t);
    if (a.dlogits) zero_vectors<STREAM>(out, sp, 0, sp.vectors, true, a.V);
    return before;
  }
  __shared__ Listed<T, NT, NT * (N + L)> list;
  __shared__ Parts<NT> parts;
  __shared__ u32x4 more[L ? L : 1][L ? NT : 1];
  static_assert(L % 3 == 0, "three at a time");
  const float c = a.inv_temp * kLog2e;
  Place place = load_place(g, t);
  list.clear();
  u32x4 v[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int i = (int)threadIdx.x + n * NT;
    v[n] = i < sp.vectors ? load_vec<true>(row + sp.head, i) : nothing<T>();
  }
  const int odd = odd_of<T>(sp, a.V);
  float lodd = odd >= 0 ? load1(row + odd) : -__builtin_huge_valf();
  if (place.id >= 0) place.l = load1(row + place.id);
  __syncthreads();
  list.enter(place, sp, Range{0, sp.vectors, true});
  __syncthreads();
  list.drop_further(place, g.K, a.status);
  const int live = (sp.vectors - __builtin_amdgcn_readfirstlane((int)threadIdx.x) + NT - 1) / NT;
#pragma unroll
  for (int n = 0; n < N; ++n)
    if (n < live) list.leave_out(v[n], (int)threadIdx.x + n * NT);
  if (odd >= 0 && list.odd_listed()) lodd = -__builtin_huge_valf();
  Mass x = no_mass();
  add<T>(x, v, c, live);
  for (int l = 0; l < L; l += 3) {
    u32x4 m[3];
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      const int i = (int)threadIdx.x + (N + l + j) * NT;
      m[j] = i < sp.vectors ? load_vec<true>(row + sp.head, i) : nothing<T>();
    }
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      list.leave_out(m[j], (int)threadIdx.x + (N + l + j) * NT);
      more[l + j][threadIdx.x] = m[j];
    }
    add<T>(x, m, c);
  }
  add1(x, lodd, c);
  float d;
  const Row o = finish_row<NT>(g, t, x, false, place, parts, &d);
  if (threadIdx.x == 0) before = write_result(g, t, o);
  if (!a.dlogits) return before;
  if (o.zero) {
    zero_vectors<STREAM>(out, sp, 0, sp.vectors, true, a.V);
    return before;
  }
  if (threadIdx.x < kListThreads) list.d[threadIdx.x] = d;
  __syncthreads();
  auto put = [&](int i, const u32x4& l) {
    float y[kPer<T>];
#pragma unroll
    for (int e = 0; e < kPer<T>; ++e) y[e] = outside_of<T>(o, element<T>(l, e));
    store_vec<STREAM>(out + sp.head, i, y);
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
  if (odd >= 0) store1(out + odd, outside_of<T>(o, lodd));
  list.write(out);
  return before;
}

// Only workgroups of this size finish a counted call's sums (few longer rows go in parts).
constexpr int kFinishThreads = 256;
template <typename T, int NT, int N, int L, bool STREAM>
__global__ __launch_bounds__(NT) void distill_row_kernel(DistillArgs g) {
  const uint64_t before = distill_row<T, NT, N, L, STREAM>(g);
  if constexpr (NT == kFinishThreads) {
    if (g.z.counts && last_of(before, g.z.epoch, g.z.T)) sum_terms<NT, 1, kDistillStats>(g.z);
  }
}

// ------------------------------------------------------------- parts of rows

constexpr int kWindow = 4096;  // vectors whose bits LDS holds at a time

// Workgroup (row, part): the sums of its words that are not listed, and the listed words' logits.
template <typename T, int U, bool STREAM>
__global__ __launch_bounds__(kPartThreads) void distill_sums_kernel(DistillArgs g) {
  const LogitsArgs& a = g.z;
  const int t = (int)(blockIdx.x / (uint32_t)a.splits), p = (int)(blockIdx.x - (uint32_t)t * a.splits);
  if (idle(g, t)) return;
  __shared__ Listed<T, kPartThreads, kWindow> list;
  __shared__ Mass parts[kPartThreads / 64];
  const T* row = static_cast<const T*>(a.logits) + (int64_t)t * a.stride;
  const Span sp = row_span(row, a.V);
  const int first = p * a.chunk, end = min(first + a.chunk, sp.vectors), odd = odd_of<T>(sp, a.V);
  const bool odds = p == a.splits - 1;
  const float c = a.inv_temp * kLog2e;
  Place place = load_place(g, t);
  Mass x = no_mass();
  for (int w0 = first; w0 == first || w0 < end; w0 += kWindow) {
    const int w1 = min(w0 + kWindow, end);
    const bool last = w1 >= end;
    list.clear();
    __syncthreads();
    const bool mine = list.enter(place, sp, Range{w0, w1, odds && last});
    if (mine) place.l = load1(row + place.id);
    __syncthreads();
    Place kept = place;
    list.drop_further(kept, g.K, a.status);
    if (mine) reinterpret_cast<float2*>(g.listed)[(int64_t)t * g.K + threadIdx.x] = make_float2(place.l, kept.id >= 0 ? 1.f : 0.f);
    int i = w0 + (int)threadIdx.x;
    for (; i + (U - 1) * kPartThreads < w1; i += kPartThreads * U) {
      u32x4 v[U];
#pragma unroll
      for (int n = 0; n < U; ++n) v[n] = load_vec<STREAM>(row + sp.head, i + n * kPartThreads);
#pragma unroll
      for (int n = 0; n < U; ++n) list.leave_out(v[n], i + n * kPartThreads - w0);
      add<T>(x, v, c);
    }
    for (; i < w1; i += kPartThreads) {
      u32x4 v[1] = {load_vec<STREAM>(row + sp.head, i)};
      list.leave_out(v[0], i - w0);
      add<T>(x, v, c);
    }
    if (odds && last && odd >= 0 && !list.odd_listed()) add1(x, load1(row + odd), c);
    __syncthreads();
  }
  x = wave_merge(x, c);
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = x;
  __syncthreads();
  if (threadIdx.x) return;
#pragma unroll
  for (int i = 1; i < kPartThreads / 64; ++i) x = merge(x, parts[i], c);
  a.part[(int64_t)t * a.splits + p] = make_float4(x.m, x.s, 0.f, 0.f);
}

// Workgroup (row, part), after distill_sums_kernel: the row's results and the part's gradient.
// Returns thread 0's arrival.
template <typename T, bool STREAM>
__device__ __forceinline__ uint64_t distill_part(const DistillArgs& g) {
  const LogitsArgs& a = g.z;
  const int t = (int)(blockIdx.x / (uint32_t)a.splits), p = (int)(blockIdx.x - (uint32_t)t * a.splits);
  const T* row = static_cast<const T*>(a.logits) + (int64_t)t * a.stride;
  const Span sp = row_span(row, a.V);
  const int first = p * a.chunk, end = min(first + a.chunk, sp.vectors);
  const bool odds = p == a.splits - 1;
  T* out = static_cast<T*>(a.dlogits) + (int64_t)t * a.d_stride;
  uint64_t before = 0;
  if (idle(g, t)) {
    if (p == 0 && threadIdx.x == 0) before = write_idle(g, t);
    if (a.dlogits) zero_vectors<STREAM>(out, sp, first, end, odds, a.V);
    return before;
  }
  if (p > 0 && !a.dlogits) return before;
  __shared__ Listed<T, kPartThreads, 1> list;  // its bits are not needed
  __shared__ Parts<kPartThreads> parts;
  const float c = a.inv_temp * kLog2e;
  Place place = load_place(g, t);
  if (place.id >= 0) {
    const float2 x = reinterpret_cast<const float2*>(g.listed)[(int64_t)t * g.K + threadIdx.x];
    place.l = x.x;
    if (x.y == 0.f) place.id = -1;
  }
  const int lane = (int)(threadIdx.x & 63);
  Mass x = no_mass();
  if (lane < a.splits) {
    const float4 q = a.part[(int64_t)t * a.splits + lane];
    x = Mass{q.x, q.y};
  }
  list.head[threadIdx.x] = -1;
  __syncthreads();
  list.chain(place, sp, Range{first, end, odds});
  float d;
  const Row o = finish_row<kPartThreads>(g, t, wave_merge(x, c), true, place, parts, &d);
  if (p == 0 && threadIdx.x == 0) before = write_result(g, t, o);
  if (!a.dlogits) return before;
  if (o.zero) {
    zero_vectors<STREAM>(out, sp, first, end, odds, a.V);
    return before;
  }
  list.d[threadIdx.x] = d;
  __syncthreads();
  for (int i = first + (int)threadIdx.x; i < end; i += kPartThreads) {
    const u32x4 v = load_vec<false>(row + sp.head, i);
    float y[kPer<T>];
#pragma unroll
    for (int e = 0; e < kPer<T>; ++e) y[e] = outside_of<T>(o, element<T>(v, e));
    store_vec<STREAM>(out + sp.head, i, y);
  }
  const int odd = odd_of<T>(sp, a.V);
  if (odds && odd >= 0) store1(out + odd, outside_of<T>(o, load1(row + odd)));
  list.write(out);
  return before;
}

template <typename T, bool STREAM>
__global__ __launch_bounds__(kPartThreads) void distill_part_kernel(DistillArgs g) {
  const uint64_t before = distill_part<T, STREAM>(g);
  // rows arrive with their first part
  if (g.z.counts && blockIdx.x % (uint32_t)g.z.splits == 0 && last_of(before, g.z.epoch, g.z.T))
    sum_terms<kPartThreads, 1, kDistillStats>(g.z);
}

__global__ __launch_bounds__(1024) void distill_stats_kernel(LogitsArgs a) { sum_terms<1024, 8, kDistillStats>(a); }

// ------------------------------------------------------------- launches

template <typename A>
hipError_t launch(const void* kernel, int64_t wgs, int threads, const A& a, hipStream_t s) {
  A args = a;
  void* params[] = {&args};
  return hipLaunchKernel(kernel, dim3((unsigned)wgs), dim3((unsigned)threads), params, 0, s);
}

// Bytes of a gradient from which it is stored past the caches (see the policy loss).
constexpr int64_t kStreamBytes = 10 << 20;
template <typename T>
bool streamed(const LogitsArgs& a) {
  return (int64_t)a.T * a.V * (int64_t)sizeof(T) >= kStreamBytes;
}

// Rows of more than kFinishThreads threads come in numbers that make 7 MB and more, and are always streamed.
template <typename T, int NT, int N, int L = 0>
hipError_t rows_for(const DistillArgs& g, hipStream_t s) {
  const void* k = reinterpret_cast<const void*>(&distill_row_kernel<T, NT, N, L, true>);
  if constexpr (NT == kFinishThreads) {
    if (!streamed<T>(g.z)) k = reinterpret_cast<const void*>(&distill_row_kernel<T, NT, N, L, false>);
  }
  return launch(k, g.z.T, NT, g, s);
}

template <typename T>
hipError_t distill_for(DistillArgs g, hipStream_t s) {
  LogitsArgs& a = g.z;
  hipError_t e = hipSuccess;
  if (!a.splits && a.V / kPer<T> > kFinishThreads * 16) a.counts = nullptr;  // the sums take a launch of their own
  if (a.splits) {
    const int64_t wgs = (int64_t)a.T * a.splits;
    const void* k = a.chunk < 8 * kPartThreads ? reinterpret_cast<const void*>(&distill_sums_kernel<T, 4, false>)
                                               : reinterpret_cast<const void*>(&distill_sums_kernel<T, 8, false>);
    e = launch(k, wgs, kPartThreads, g, s);
    k = streamed<T>(a) ? reinterpret_cast<const void*>(&distill_part_kernel<T, true>)
                       : reinterpret_cast<const void*>(&distill_part_kernel<T, false>);
    if (e == hipSuccess) e = launch(k, wgs, kPartThreads, g, s);
  } else if (a.T) {
    const int v = a.V / kPer<T>;
    e = v <= kFinishThreads * 4 ? rows_for<T, kFinishThreads, 4>(g, s)
        : v <= kFinishThreads * 8 ? rows_for<T, kFinishThreads, 8>(g, s)
        : v <= kFinishThreads * 16 ? rows_for<T, kFinishThreads, 16>(g, s)
        : v <= 512 * 16 ? rows_for<T, 512, 16>(g, s)
        : v <= 1024 * 16 ? rows_for<T, 1024, 16>(g, s)
        : v <= 1024 * 20 ? rows_for<T, 1024, 20>(g, s) : rows_for<T, 1024, 19, 6>(g, s);
  }
  if (e != hipSuccess || a.counts) return e;
  return launch(reinterpret_cast<const void*>(&distill_stats_kernel), 1, 1024, a, s);
}

}  // namespace

hipError_t launch_distill_loss(const DistillArgs& a, hipStream_t s) {
  return a.z.bf16 ? distill_for<uint16_t>(a, s) : distill_for<float>(a, s);
}

}  // namespace pda
