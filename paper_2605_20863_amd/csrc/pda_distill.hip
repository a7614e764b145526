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
// one factor a row times a word's share of the rest. A byte in LDS for each of a row's vectors says which of its words are
// listed; these are made -inf when the vector has come. Their gradients are written
// over the vectors' by the threads that wrote these, after them.
//
// With rest, sum p + p_r = 1 turns the divergences into sums of terms that are not
// negative, which keeps their digits where teacher and student are close:
//     F = sum t (e^a - 1 - a) + (S + t_r - 1),  R = sum p (e^-a - 1 + a) - (S + t_r - 1).

#include "pda_lm_internal.h"
#include "pda_rows.h"

#include <type_traits>

namespace pda {
namespace {

constexpr double kLeastRest = 0x1p-24;  // half a step of float32 below 1: what a sum of t can tell from it

// A list's places are the first threads' of a workgroup of NT, one each up to 256, or all threads' in turn.
template <int NT>
constexpr int kPlaces = NT < kMaxTop ? kMaxTop / NT : 1;
template <int NT>
constexpr int kListWaves = (NT < kMaxTop ? NT : kMaxTop) / 64;

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

// Largest logit and sum of exponentials below it, as base2 has them.
struct Mass {
  float m, s;
};
__device__ __forceinline__ Mass no_mass() { return Mass{kLowest, 0.f}; }
__device__ __forceinline__ Mass rebase(const Mass& x, float m, float c) {
#pragma clang fp contract(off)  // a rounded product, whatever adds it: lanes that sum each other's agree
  return Mass{m, x.s * __builtin_amdgcn_exp2f(exponent_to(x.m, m, c))};
}
__device__ __forceinline__ Mass merge(const Mass& a, const Mass& b, float c) {
#pragma clang fp contract(off)  // the same whichever side is which, so that all lanes agree
  const float m = fmaxf(a.m, b.m);
  return Mass{m, rebase(a, m, c).s + rebase(b, m, c).s};
}
__device__ __forceinline__ void add1(Mass& x, float l, float c) {
  const float m = fmaxf(x.m, l);
  x = rebase(x, m, c);
  x.s += __builtin_amdgcn_exp2f(base2(m, c).of(l));
}
// N vectors' elements (as for Soft).
template <typename T, int N>
__device__ __forceinline__ void add(Mass& x, u32x4* v, float c) {
  float m = x.m;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int e = 0; e < kPer<T>; ++e) m = fmaxf(m, element<T>(v[n], e));
  const Base2 below = base2(m, c), before = base2(x.m, c);
  float s = 0.f;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    again(v[n]);
#pragma unroll
    for (int e = 0; e < kPer<T>; ++e) s += __builtin_amdgcn_exp2f(below.of<false>(element<T>(v[n], e)));
    asm volatile("" : "+v"(s));  // one vector's elements after another's
  }
#pragma unroll
  for (int n = 0; n < N; ++n) again(v[n]);
  // seldom, and apart, so that it costs the others a branch a batch
  if (__builtin_expect(__ballot(below.far || (before.far && x.s != 0.f)) != 0, 0)) {
    s = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n) {
#pragma unroll
      for (int e = 0; e < kPer<T>; ++e) s += __builtin_amdgcn_exp2f(below.of(element<T>(v[n], e)));
      asm volatile("" : "+v"(s));
    }
    x = rebase(x, m, c);
  } else {
#pragma clang fp contract(off)
    x = Mass{m, x.s * __builtin_amdgcn_exp2f(before.k - below.k)};
  }
  x.s += s;
}
__device__ __forceinline__ Mass wave_merge(const Mass& x, float c) {
  const float m = wave_top(x.m);
  return Mass{m, wave_total(rebase(x, m, c).s)};
}
// Over W waves' sums, in every thread.
template <int W>
__device__ __forceinline__ Mass waves_merge(const Mass* parts, float c) {
  static_assert(W <= 16, "a lane each");
  const int i = (int)threadIdx.x & 15;
  const Mass x = i < W ? parts[i] : no_mass();
  const float m = group_max<16>(x.m);
  return Mass{m, group_sum<16>(rebase(x, m, c).s)};
}

// ------------------------------------------------------------- the list

// A place of a row's list: thread t's n-th is the (t + n NT)-th.
struct Place {
  int id;  // -1: no word
  float tau, l, t;
};
template <int NT>
__device__ __forceinline__ void load_places(const DistillArgs& g, int t, Place (&p)[kPlaces<NT>]) {
#pragma unroll
  for (int n = 0; n < kPlaces<NT>; ++n) {
    p[n] = Place{-1, 0.f, kLowest, 0.f};
    const int k = (int)threadIdx.x + n * NT;
    if (k >= g.K) continue;
    p[n].id = g.ids[(int64_t)t * g.K + k];
    p[n].tau = g.tau[(int64_t)t * g.K + k];
    if (p[n].id >= g.z.V) {
      atomicOr(g.z.status, kStatusBadTarget);
      p[n].id = -1;
    }
    if (p[n].id < 0 || p[n].tau == -__builtin_huge_valf()) p[n].id = -1;
  }
}

// Vectors first .. end - 1 of a row, and with `odds` the elements outside of all vectors.
struct Range {
  int first, end;
  bool odds;
};

// For a range of up to V vectors of each of NT threads: which of its words are listed, and the places whose words each
// thread writes. Vector n of the range is thread n % NT's.
template <typename T, int NT, int V>
struct Listed {
  uint32_t bits[(V + 3) / 4][NT];  // a byte for each of a thread's vectors
  uint32_t odd;                    // of the elements outside of all vectors
  int head[NT], next[kMaxTop];  // a thread's places, -1: no more
  int id[kMaxTop];
  float p[kMaxTop], t[kMaxTop], pa[kMaxTop];  // see Row
  int twice;

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < (V + 3) / 4; ++i) bits[i][threadIdx.x] = 0;
    head[threadIdx.x] = -1;
    if (threadIdx.x == 0) odd = twice = 0;
  }

  // After clear() and a barrier: place k goes to the thread that writes its word, and the word's bit is set, if that is
  // in the range. A barrier later all can be read. MASK: the bits are wanted.
  template <bool MASK>
  __device__ __forceinline__ bool enter(const Place& place, int k, const Span& sp, const Range& r) {
    if (k >= kMaxTop) return false;
    id[k] = place.id;
    if (place.id < 0) return false;
    const int at = place.id - sp.head, in = sp.vectors * kPer<T>, n = at / kPer<T> - r.first;
    const bool outer = at < 0 || at >= in;
    if (outer ? !r.odds : n < 0 || n >= r.end - r.first) return false;
    const int owner = outer ? (at < 0 ? place.id : place.id - in) : n % NT;
    next[k] = atomicExch(&head[owner], k);
    if constexpr (MASK) {
      uint32_t* word = outer ? &odd : &bits[n / NT / 4][owner];
      const int bit = outer ? owner : n / NT % 4 * 8 + at % kPer<T>;
      if (atomicOr(word, 1u << bit) >> bit & 1) twice = 1;
    }
    return true;
  }
  // After that barrier: a word's further places leave the list.
  __device__ __forceinline__ void drop_further(Place (&place)[kPlaces<NT>], int32_t* status) {
    if (!twice) return;
    bool further[kPlaces<NT>];
#pragma unroll
    for (int n = 0; n < kPlaces<NT>; ++n) {
      const int k = (int)threadIdx.x + n * NT;
      further[n] = false;
      if (k < kMaxTop)
        for (int j = 0; j < k; ++j) further[n] |= place[n].id >= 0 && id[j] == place[n].id;
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kPlaces<NT>; ++n)
      if (further[n]) {
        atomicOr(status, kStatusTwice);
        place[n].id = id[(int)threadIdx.x + n * NT] = -1;
      }
  }

  // Vectors first .. first + N - 1 of this thread's, with their listed words made -inf.
  template <int N>
  __device__ __forceinline__ void leave_out(u32x4* v, int first) const {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const uint32_t mask = bits[(first + n) / 4][threadIdx.x] >> (first + n) % 4 * 8 & 255;
      if (!mask) continue;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        // all ones over a listed word's bits
        const auto ones = [&](int bit) { return (uint32_t)((int32_t)(mask << (31 - bit)) >> 31); };
        const uint32_t m = kPer<T> == 8 ? (ones(2 * w) & 0xFFFFu) | (ones(2 * w + 1) & 0xFFFF0000u) : ones(w);
        v[n][w] = (v[n][w] & ~m) | (m & (kPer<T> == 8 ? 0xFF80FF80u : 0xFF800000u));
      }
    }
  }
  __device__ __forceinline__ bool odd_listed() const { return odd >> threadIdx.x & 1; }
};

// ------------------------------------------------------------- a row's results

// A row's gradient, by the word's logit: outside of the list 2^below(l) outside, of a place's word
// f (p total - t) + b (pa - p R).
struct Row {
  Base2 below;
  float outside;
  float total, R, f, b;
  bool zero;  // no gradient, whatever the logits
};

// What the waves of a workgroup hand each other.
template <int NT>
struct Parts {
  Mass rest[NT / 64], list[kListWaves<NT>];
  double S[kListWaves<NT>];
  float P[kListWaves<NT>], F[kListWaves<NT>], R[kListWaves<NT>];
};

__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

// The list's own sums, by its waves: before the barrier in front of know_row.
template <int NT>
__device__ __forceinline__ void sum_list(Place (&place)[kPlaces<NT>], float c, Parts<NT>& s) {
  const int wave = wave_id();
  if (wave >= kListWaves<NT>) return;
  Mass x = no_mass();
  double S = 0.;
#pragma unroll
  for (int n = 0; n < kPlaces<NT>; ++n)
    if (place[n].id >= 0) {
      add1(x, place[n].l, c);
      const double t = exp((double)place[n].tau);
      place[n].t = (float)t;
      S += t;
    }
  x = wave_merge(x, c);
  S = wave_total(S);
  if ((threadIdx.x & 63) == 0) {
    s.list[wave] = x;
    s.S[wave] = S;
  }
}

// A row's quantities, from the sums of the words outside of the list, in every thread.
struct Known {
  Mass x;     // of all words
  bool some;  // a distribution: some logit is above -inf (or NaN)
  float log_s, pr, tr, ar, total, over;
  double S;
};
template <int NT>
__device__ __forceinline__ Known know_row(const DistillArgs& g, const Mass& rest, const Parts<NT>& s, float c) {
  Known q;
  q.x = rest;
  q.S = 0.;
#pragma unroll
  for (int i = 0; i < kListWaves<NT>; ++i) {
    q.x = merge(q.x, s.list[i], c);
    q.S += s.S[i];
  }
  q.some = q.x.s != 0.f;
  q.log_s = log_below(q.x.s, q.x.m, c);
  const float lpr = (rest.m - q.x.m) * g.z.inv_temp + (log_below(rest.s, rest.m, c) - q.log_s);
  q.pr = rest.s != 0.f ? expf(lpr) : 0.f;
  const bool others = g.rest && rest.s != 0.f;
  const double t_rest = others ? fmax(1. - q.S, kLeastRest) : 0.;
  q.tr = (float)t_rest;
  q.ar = others ? lpr - (float)log(t_rest) : 0.f;
  q.total = (float)(q.S + t_rest);
  q.over = (float)(q.S + t_rest - 1.);
  return q;
}

// This thread's places' part of the divergences, by the list's waves; what their gradients take goes to `list`.
template <int NT, typename List>
__device__ __forceinline__ void sum_places(const DistillArgs& g, const Known& q, const Place (&place)[kPlaces<NT>], List& list, Parts<NT>& s) {
  const int wave = wave_id();
  if (wave >= kListWaves<NT>) return;
  float P = 0.f, F = 0.f, R = 0.f;
#pragma unroll
  for (int n = 0; n < kPlaces<NT>; ++n) {
    const int k = (int)threadIdx.x + n * NT;
    if (place[n].id < 0) continue;
    const float lp = q.some ? (place[n].l - q.x.m) * g.z.inv_temp - q.log_s : -__builtin_huge_valf();
    const float a = lp - place[n].tau, t = place[n].t, p = expf(lp);
    const float ta = t == 0.f ? 0.f : t * a, pa = p == 0.f ? 0.f : p * a;
    if (g.rest) {  // squares where a is near to 0
      const bool near = fabsf(a) <= 1.f;
      F += near ? t * phi(a) : p - t - ta;
      R += near ? p * phi(-a) : t - p + pa;
    } else {
      F -= ta;
      R += pa;
    }
    P += p;
    list.p[k] = p;
    list.t[k] = t;
    list.pa[k] = pa;
  }
  P = wave_total(P);
  F = wave_total(F);
  R = wave_total(R);
  if ((threadIdx.x & 63) == 0) {
    s.P[wave] = P;
    s.F[wave] = F;
    s.R[wave] = R;
  }
}

// The divergences, a barrier after sum_places.
struct Sums {
  float P, F, R;
};
template <int NT>
__device__ __forceinline__ Sums sum_row(const DistillArgs& g, const Known& q, const Parts<NT>& s) {
  Sums o = {0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kListWaves<NT>; ++i) {
    o.P += s.P[i];
    o.F += s.F[i];
    o.R += s.R[i];
  }
  if (g.rest) {
    const bool near = fabsf(q.ar) <= 1.f;
    o.F += (near ? q.tr * phi(q.ar) : q.pr - q.tr - q.tr * q.ar) + q.over;
    o.R += (near ? q.pr * phi(-q.ar) : q.tr - q.pr + (q.pr == 0.f ? 0.f : q.pr * q.ar)) - q.over;
  }
  if (!q.some) {
    o.F = q.S > 0. ? __builtin_huge_valf() : 0.f;
    o.R = 0.f;
  }
  return o;
}

// With b = 0 the gradient takes none of the sums.
__device__ __forceinline__ Row row_grad(const DistillArgs& g, int t, const Mass& rest, const Known& q, const Sums& o, float c) {
  const float k = g.z.weight[t] * g.z.grad_scale * g.z.inv_temp, b = g.rev;
  Row r;
  r.zero = k == 0.f || !q.some;
  r.below = base2(rest.m, c);
  r.total = q.total;
  r.R = b == 0.f ? 0.f : g.rest ? o.R : o.R + o.P - 1.f;
  r.f = k * (1.f - b);
  r.b = k * b;
  const float away = g.rest ? (q.pr == 0.f ? 0.f : q.pr * q.ar) - q.pr * r.R : -q.pr * (r.R + 1.f);
  r.outside = rest.s == 0.f ? 0.f : (r.f * (q.pr * q.total - q.tr) + (b == 0.f ? 0.f : r.b * away)) / rest.s;
  return r;
}

__device__ __forceinline__ float outside_of(const Row& o, float l) { return __builtin_amdgcn_exp2f(o.below.of(l)) * o.outside; }
// The gradients of a vector's words as if none were listed.
template <bool STREAM, bool FAR, typename T>
__device__ __forceinline__ void put_vec(const Row& o, T* out, int i, const u32x4& l) {
  float y[kPer<T>];
#pragma unroll
  for (int e = 0; e < kPer<T>; ++e) y[e] = __builtin_amdgcn_exp2f(o.below.of<FAR>(element<T>(l, e))) * o.outside;
  store_vec<STREAM>(out, i, y);
}

// This thread's places' gradients, over what it wrote before.
template <typename T, typename List>
__device__ __forceinline__ void write_places(const List& s, const Row& r, T* out) {
  for (int k = s.head[threadIdx.x]; k >= 0; k = s.next[k])
    if (s.id[k] >= 0) store1(out + s.id[k], r.f * (s.p[k] * r.total - s.t[k]) + (r.b == 0.f ? 0.f : r.b * (s.pa[k] - s.p[k] * r.R)));
}

// What thread 0 of a row writes beside the gradient; with counts also its arrival.
__device__ __forceinline__ uint64_t write_result(const DistillArgs& g, int t, const Sums& o, double S, bool idle) {
  const float w = g.z.weight[t], b = g.rev;
  const float loss = (b < 1.f ? (1.f - b) * o.F : 0.f) + (b > 0.f ? b * o.R : 0.f);
  const float v[kTerms] = {loss, o.F, o.R, (float)S, o.P, 1.f, 0.f, 0.f};
  float terms[kTerms];
#pragma unroll
  for (int i = 0; i < kTerms; ++i) terms[i] = w != 0.f && !idle ? w * v[i] : 0.f;
  write_terms(g.z, t, terms);
  if (g.losses) g.losses[t] = loss;
  if (!g.z.counts) return 0;
  parts_written();
  return arrive(g.z.counts, g.z.epoch);
}

// Whether row t takes no part at all: of weight 0, and its loss not wanted.
__device__ __forceinline__ bool idle(const DistillArgs& g, int t) { return g.z.weight[t] == 0.f && !g.losses; }

// ------------------------------------------------------------- rows in registers

constexpr int kBatch = 4;  // vectors of a thread whose sums are made at a time

// Workgroup per row, whose vectors stay in its threads' registers (N of a thread)
// and LDS (L of a thread) between the sums and the gradient: one read and one
// write of the row. Of a longer row up to X more vectors of a thread are read again; few enough rows are on their way for the
// memory-side cache to hold them. Returns thread 0's arrival.
template <typename T, int NT, int N, int L, int X, bool STREAM>
__device__ __forceinline__ uint64_t distill_row(const DistillArgs& g) {
  const LogitsArgs& a = g.z;
  const int t = (int)blockIdx.x;
  const T* row = static_cast<const T*>(a.logits) + (int64_t)t * a.stride;
  const Span sp = row_span(row, a.V);
  T* out = static_cast<T*>(a.dlogits) + (int64_t)t * a.d_stride;
  uint64_t before = 0;
  if (idle(g, t)) {
    if (threadIdx.x == 0) before = write_result(g, t, Sums{}, 0., true);
    if (a.dlogits) zero_vectors<STREAM>(out, sp, 0, sp.vectors, true, a.V);
    return before;
  }
  __shared__ Listed<T, NT, N + L + X> list;
  __shared__ Parts<NT> parts;
  __shared__ u32x4 more[L ? L : 1][L ? NT : 1];
  static_assert(L % kBatch == 0 && N % kBatch == 0, "whole batches");
  const float c = base2_rate(a);
  // a list's waves ask for its words' logits before the row's vectors, and wait for no vector to have them
  Place place[kPlaces<NT>];
  load_places<NT>(g, t, place);
#pragma unroll
  for (int n = 0; n < kPlaces<NT>; ++n)
    if (place[n].id >= 0) place[n].l = load1(row + place[n].id);
  auto load = [&](int n) {
    const int i = (int)threadIdx.x + n * NT;
    return i < sp.vectors ? load_vec<true>(row + sp.head, i) : nothing<T>();
  };
#pragma unroll
  for (int l = 0; l < L; ++l) more[l][threadIdx.x] = load(N + l);
  u32x4 v[N];
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = load(n);
  const int odd = odd_of<T>(sp, a.V);
  float lodd = odd >= 0 ? load1(row + odd) : -__builtin_huge_valf();
  list.clear();
  __syncthreads();
#pragma unroll
  for (int n = 0; n < kPlaces<NT>; ++n)
    list.template enter<true>(place[n], (int)threadIdx.x + n * NT, sp, Range{0, sp.vectors, true});
  __syncthreads();
  list.drop_further(place, a.status);
  sum_list<NT>(place, c, parts);
  if (odd >= 0 && list.odd_listed()) lodd = -__builtin_huge_valf();
  Mass x = no_mass();
#pragma unroll
  for (int l = 0; l < L; l += kBatch) {
    u32x4 m[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) m[j] = more[l + j][threadIdx.x];
    list.template leave_out<kBatch>(m, N + l);
#pragma unroll
    for (int j = 0; j < kBatch; ++j) more[l + j][threadIdx.x] = m[j];
    add<T, kBatch>(x, m, c);
  }
  // a few vectors at a time, as they come
  const auto load_more = [&](int n, u32x4 (&m)[kBatch]) {
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int i = (int)threadIdx.x + (n + j) * NT;
      m[j] = i < sp.vectors ? load_vec<false>(row + sp.head, i) : nothing<T>();
    }
  };
  const int live = (sp.vectors - __builtin_amdgcn_readfirstlane((int)threadIdx.x) + NT - 1) / NT;
#pragma unroll
  for (int n = 0; n < N; n += kBatch) {
    if (n >= live) continue;
    list.template leave_out<kBatch>(v + n, n);
    add<T, kBatch>(x, v + n, c);
  }
  if constexpr (X > 0) {
    for (int n = N + L; n < live; n += kBatch) {
      u32x4 m[kBatch];
      load_more(n, m);
      list.template leave_out<kBatch>(m, n);
      add<T, kBatch>(x, m, c);
    }
  }
  add1(x, lodd, c);
  x = wave_merge(x, c);
  if ((threadIdx.x & 63) == 0) parts.rest[wave_id()] = x;
  __syncthreads();
  const Mass rest = waves_merge<NT / 64>(parts.rest, c);
  const Known q = know_row(g, rest, parts, c);
  sum_places<NT>(g, q, place, list, parts);
  // without a reverse part the gradient needs no more than this
  const bool late = g.rev == 0.f;
  Sums sums = {};
  if (!late) {
    __syncthreads();
    sums = sum_row(g, q, parts);
  }
  const Row o = row_grad(g, t, rest, q, sums, c);
  if (a.dlogits) {
    if (o.zero) {
      zero_vectors<STREAM>(out, sp, 0, sp.vectors, true, a.V);
    } else {
      // seldom: from the row itself again, so that the others have no second copy of what follows (447 us for 442, 4,096 x 131,072 bf16)
      const bool far = __builtin_amdgcn_readfirstlane(o.below.far);
#pragma unroll 1
      for (int i = (int)threadIdx.x; far && i < sp.vectors; i += NT)
        put_vec<STREAM, true>(o, out + sp.head, i, load_vec<false>(row + sp.head, i));
      if (!far) {
        auto put = [&](int i, const u32x4& l) { put_vec<STREAM, false>(o, out + sp.head, i, l); };
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
        if constexpr (X > 0) {
          for (int n = N + L; n < live; n += kBatch) {
            u32x4 m[kBatch];
            load_more(n, m);
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
              const int i = (int)threadIdx.x + (n + j) * NT;
              if (i < sp.vectors) put(i, m[j]);
            }
          }
        }
      }
      if (odd >= 0) store1(out + odd, outside_of(o, lodd));
    }
  }
  if (late) {
    __syncthreads();
    if (threadIdx.x == 0) sums = sum_row(g, q, parts);
  }
  if (threadIdx.x == 0) before = write_result(g, t, sums, q.S, false);
  if (a.dlogits && !o.zero) write_places(list, o, out);
  return before;
}

// 4,096 x 131,072 bf16, 64 places 432 us and 5 for the sums, 4.9 TB/s, what a copy of 2 GiB reaches; without its arithmetic it takes 395.
// Only workgroups of this size finish a counted call's sums (few longer rows go in parts).
constexpr int kFinishThreads = 256;
template <typename T, int NT, int N, int L, int X, bool STREAM>
__global__ __launch_bounds__(NT) void distill_row_kernel(DistillArgs g) {
  const uint64_t before = distill_row<T, NT, N, L, X, STREAM>(g);
  if constexpr (NT == kFinishThreads) {
    if (g.z.counts && last_of(before, g.z.epoch, g.z.T)) sum_terms<NT, 1, kDistillStats>(g.z);
  }
}

// ------------------------------------------------------------- parts of rows

constexpr int kWindow = 16;  // vectors of a thread whose bits LDS holds at a time

// Workgroup (row, part): the sums of its words that are not listed, and the listed words' logits. 37 x 50,001 f32, 100 places: 5.2 us, the
// parts' gradients 8.2 and the rows' sums 2.3, each a chain of dependent loads and barriers.
template <typename T, int U>
__global__ __launch_bounds__(kPartThreads) void distill_sums_kernel(DistillArgs g) {
  const LogitsArgs& a = g.z;
  const int t = (int)(blockIdx.x / (uint32_t)a.splits), p = (int)(blockIdx.x - (uint32_t)t * a.splits);
  if (idle(g, t)) return;
  static_assert(kWindow % U == 0 && U % 4 == 0, "whole batches, of whole words of bits");
  __shared__ Listed<T, kPartThreads, kWindow> list;
  __shared__ Mass parts[kPartThreads / 64];
  const T* row = static_cast<const T*>(a.logits) + (int64_t)t * a.stride;
  const Span sp = row_span(row, a.V);
  const int first = p * a.chunk, end = min(first + a.chunk, sp.vectors), odd = odd_of<T>(sp, a.V);
  const bool odds = p == a.splits - 1;
  const float c = base2_rate(a);
  Place place[1];
  load_places<kPartThreads>(g, t, place);
  Mass x = no_mass();
  int w0 = first;
  do {
    const int w1 = min(w0 + kWindow * kPartThreads, end);
    const bool last = w1 >= end;
    u32x4 v[U];
    auto load = [&](int i0) {
#pragma unroll
      for (int n = 0; n < U; ++n) {
        const int i = i0 + n * kPartThreads + (int)threadIdx.x;
        v[n] = i < w1 ? load_vec<false>(row + sp.head, i) : nothing<T>();
      }
    };
    load(w0);  // on its way while the list is entered
    list.clear();
    __syncthreads();
    const bool mine = list.template enter<true>(place[0], (int)threadIdx.x, sp, Range{w0, w1, odds && last});
    const float l = mine ? load1(row + place[0].id) : 0.f;
    __syncthreads();
    Place kept[1] = {place[0]};
    list.drop_further(kept, a.status);
    for (int n = 0;; n += U) {
      list.template leave_out<U>(v, n);
      add<T, U>(x, v, c);
      if (w0 + (n + U) * kPartThreads >= w1) break;
      load(w0 + (n + U) * kPartThreads);
    }
    if (mine) reinterpret_cast<float2*>(g.listed)[(int64_t)t * g.K + threadIdx.x] = make_float2(l, kept[0].id >= 0 ? 1.f : 0.f);
    if (odds && last && odd >= 0 && !list.odd_listed()) add1(x, load1(row + odd), c);
    __syncthreads();
    w0 = w1;
  } while (w0 < end);
  x = wave_merge(x, c);
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = x;
  __syncthreads();
  x = waves_merge<kPartThreads / 64>(parts, c);
  if (threadIdx.x == 0) a.part[(int64_t)t * a.splits + p] = make_float4(x.m, x.s, 0.f, 0.f);
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
    if (p == 0 && threadIdx.x == 0) before = write_result(g, t, Sums{}, 0., true);
    if (a.dlogits) zero_vectors<STREAM>(out, sp, first, end, odds, a.V);
    return before;
  }
  if (p > 0 && !a.dlogits) return before;
  __shared__ Listed<T, kPartThreads, 1> list;  // its bits are not used
  __shared__ Parts<kPartThreads> parts;
  const float c = base2_rate(a);
  Place place[1];
  load_places<kPartThreads>(g, t, place);
  const int lane = (int)(threadIdx.x & 63);
  Mass x = no_mass();
  if (lane < a.splits) {
    const float4 q = a.part[(int64_t)t * a.splits + lane];
    x = Mass{q.x, q.y};
  }
  if (place[0].id >= 0) {
    const float2 q = reinterpret_cast<const float2*>(g.listed)[(int64_t)t * g.K + threadIdx.x];
    place[0].l = q.x;
    if (q.y == 0.f) place[0].id = -1;
  }
  // the part's first vectors are on their way meanwhile
  constexpr int U = 4;
  u32x4 v[U];
  auto load = [&](int i0) {
#pragma unroll
    for (int n = 0; n < U; ++n) {
      const int i = i0 + n * kPartThreads + (int)threadIdx.x;
      if (i < end) v[n] = load_vec<false>(row + sp.head, i);
    }
  };
  if (a.dlogits) load(first);
  list.head[threadIdx.x] = -1;
  sum_list<kPartThreads>(place, c, parts);
  __syncthreads();
  list.template enter<false>(place[0], (int)threadIdx.x, sp, Range{first, end, odds});
  const Mass rest = wave_merge(x, c);
  const Known q = know_row(g, rest, parts, c);
  sum_places<kPartThreads>(g, q, place, list, parts);
  __syncthreads();
  const Sums sums = sum_row(g, q, parts);
  const Row o = row_grad(g, t, rest, q, sums, c);
  if (p == 0 && threadIdx.x == 0) before = write_result(g, t, sums, q.S, false);
  if (!a.dlogits) return before;
  if (o.zero) {
    zero_vectors<STREAM>(out, sp, first, end, odds, a.V);
    return before;
  }
  const auto write = [&](auto far) {
    for (int i0 = first; i0 < end;) {
#pragma unroll
      for (int n = 0; n < U; ++n) {
        const int i = i0 + n * kPartThreads + (int)threadIdx.x;
        if (i >= end) break;
        put_vec<STREAM, decltype(far)::value>(o, out + sp.head, i, v[n]);
      }
      i0 += U * kPartThreads;
      if (i0 < end) load(i0);
    }
  };
  if (o.below.far) write(std::true_type());
  else write(std::false_type());
  const int odd = odd_of<T>(sp, a.V);
  if (odds && odd >= 0) store1(out + odd, outside_of(o, load1(row + odd)));
  write_places(list, o, out);
  return before;
}

template <typename T, bool STREAM>
__global__ __launch_bounds__(kPartThreads) void distill_part_kernel(DistillArgs g) {
  const uint64_t before = distill_part<T, STREAM>(g);
  // rows arrive with their first part
  if (g.z.counts && blockIdx.x % (uint32_t)g.z.splits == 0 && last_of(before, g.z.epoch, g.z.T))
    sum_terms<kPartThreads, 1, kDistillStats>(g.z);
}

// U: rows' terms of a thread on their way at once.
template <int U>
__global__ __launch_bounds__(1024) void distill_stats_kernel(LogitsArgs a) {
  sum_terms<1024, U, kDistillStats>(a);
}

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

// Rows of 1,024 threads come in numbers that make 5 MB and more, and are always streamed.
template <typename T, int NT, int N, int L = 0, int X = 0>
hipError_t rows_for(const DistillArgs& g, hipStream_t s) {
  const void* k = reinterpret_cast<const void*>(&distill_row_kernel<T, NT, N, L, X, true>);
  if constexpr (NT <= 512) {
    if (!streamed<T>(g.z)) k = reinterpret_cast<const void*>(&distill_row_kernel<T, NT, N, L, X, false>);
  }
  return launch(k, g.z.T, NT, g, s);
}

// Rows from which short ones take a wave or two each: a workgroup's chain (places, listed logits, two barriers, sums,
// stores) is the same length for them, and more rows are on their way at once. us per call, 256 / 128 / 64 threads
// a row, 64 places, bf16: 8,192 x 1,000 51 / 38 / 30, x 2,000 57 / 41 / 34, x 4,000 62 / 48 / 45, x 8,000 78 / 68 / 73; 2,000 x 2,000 19.8 /
// 15.9 / 14.6; 1,000 x 4,000 15.0 / 13.4 / 13.6, x 8,000 17.8 / 17.3 / 17.9; 500 x 2,000 11.4 / 12.0 / 11.4; 300 x 4,000 11.3 / 11.6 / 13.2;
// f32 4,000 x 4,000 36.3 / 35.6 / 38.5.
constexpr int kManyRows = 600;

template <typename T>
hipError_t distill_for(DistillArgs g, hipStream_t s) {
  LogitsArgs& a = g.z;
  hipError_t e = hipSuccess;
  if (!a.splits && a.V / kPer<T> > kFinishThreads * 16) a.counts = nullptr;  // the sums take a launch of their own
  if (a.splits) {
    const int64_t wgs = (int64_t)a.T * a.splits;
    const void* k = a.chunk <= 4 * kPartThreads ? reinterpret_cast<const void*>(&distill_sums_kernel<T, 4>)
                                                : reinterpret_cast<const void*>(&distill_sums_kernel<T, 8>);
    e = launch(k, wgs, kPartThreads, g, s);
    k = streamed<T>(a) ? reinterpret_cast<const void*>(&distill_part_kernel<T, true>)
                       : reinterpret_cast<const void*>(&distill_part_kernel<T, false>);
    if (e == hipSuccess) e = launch(k, wgs, kPartThreads, g, s);
  } else if (a.T) {
    const int v = a.V / kPer<T>;
    e = a.T >= kManyRows && v <= 64 * 4 ? rows_for<T, 64, 4>(g, s)
        : a.T >= kManyRows && v <= 64 * 8 ? rows_for<T, 64, 8>(g, s)
        : a.T >= kManyRows && v <= 128 * 8 ? rows_for<T, 128, 8>(g, s)
        : v <= kFinishThreads * 4 ? rows_for<T, kFinishThreads, 4>(g, s)
        : v <= kFinishThreads * 8 ? rows_for<T, kFinishThreads, 8>(g, s)
        : v <= kFinishThreads * 16 ? rows_for<T, kFinishThreads, 16>(g, s)
        : v <= 512 * 16 ? rows_for<T, 512, 16>(g, s)
        : v <= 1024 * 16 ? rows_for<T, 1024, 16>(g, s)
        : v <= 1024 * 20 ? rows_for<T, 1024, 20>(g, s) : rows_for<T, 1024, 20, 4, kListedMore>(g, s);
  }
  if (e != hipSuccess || a.counts) return e;
  const void* k = a.T <= 8 * kSums ? reinterpret_cast<const void*>(&distill_stats_kernel<8>)
                                   : reinterpret_cast<const void*>(&distill_stats_kernel<32>);
  return launch(k, 1, 1024, a, s);
}

}  // namespace

hipError_t launch_distill_loss(const DistillArgs& a, hipStream_t s) {
  return a.z.bf16 ? distill_for<uint16_t>(a, s) : distill_for<float>(a, s);
}

}  // namespace pda
