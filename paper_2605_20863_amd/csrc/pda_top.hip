// HIP kernels for the most likely words of rows of logits, with their
// log-probabilities, on MI355X (gfx950).
//
// A row's words are in one order: by logit, equal ones by their place. A word's key
// is its logit's bits, made to compare as whole numbers do, over the complement of
// its place: all keys of a row differ, and the K largest are the answer.

#include "pda_lm_internal.h"
#include "pda_rows.h"

namespace pda {
namespace {

constexpr int kRoom = 2048;  // keys that a workgroup holds
constexpr int kStep = 4;     // words of a thread between two looks at the room left
static_assert(kRoom >= kMaxTop + kStep * kPartThreads, "a step fits behind the K kept");

// Whole numbers in the order of the logits; zeros of either sign are equal, NaN comes first.
__device__ __forceinline__ uint32_t rank_of(float l) {
  const uint32_t u = as_u32(l + 0.f);
  return l != l ? 0xFFFFFFFFu : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t rank) {
  return rank == 0xFFFFFFFFu ? __builtin_nanf("") : as_f32(rank & 0x80000000u ? rank ^ 0x80000000u : ~rank);
}
__device__ __forceinline__ uint64_t key_of(float l, int word) { return ((uint64_t)rank_of(l) << 32) | (uint32_t)~word; }

// Keys that may be among the K largest; n of them, in no order.
struct Pool {
  uint64_t keys[kRoom];
  uint64_t bar;      // after keep(): the K-th largest, 0 where there are fewer
  int count[3];      // of the keys that a batch adds, in turn
  uint32_t tops[2 * kPartThreads];
};

// This thread's number, for code that is seldom reached: the compiler works out what follows from it there, rather than
// once for all at the kernel's start and in registers of its own.
__device__ __forceinline__ int thread_here() {
  int t = (int)threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// A value that at least K of the n ranks are not below, and that is their K-th largest in its upper 16 bits (0 where there
// are fewer), the same in every lane: a wave settles bit after bit by counting. rank(i): the i-th; N * 64 >= n.
template <int N, typename F>
__device__ __forceinline__ uint32_t kth_of(int n, int K, F rank) {
  uint32_t v[N], c = 0;
  const int lane = thread_here() & 63;
#pragma unroll
  for (int j = 0; j < N; ++j) v[j] = lane + 64 * j < n ? rank(lane + 64 * j) : 0;
#pragma unroll 1
  for (uint32_t bit = 0x80000000u; bit >= 0x10000u; bit >>= 1) {
    int above = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) above += (int)__popcll(__ballot(v[j] >= (c | bit)));
    if (above >= K) c |= bit;
  }
  return c;
}
__device__ __forceinline__ uint32_t kth_in(const Pool& b, int n, int K) {
  const auto rank = [&](int i) { return (uint32_t)(b.keys[i] >> 32); };
  if (n <= 512) return kth_of<8>(n, K, rank);
  uint32_t c = 0;
  const int lane = thread_here() & 63;
#pragma unroll 1
  for (uint32_t bit = 0x80000000u; bit >= 0x10000u; bit >>= 1) {
    int above = 0;
#pragma unroll 4
    for (int i = 0; i < n; i += 64) above += (int)__popcll(__ballot(i + lane < n && rank(i + lane) >= (c | bit)));
    if (above >= K) c |= bit;
  }
  return c;
}

// Sorts the first `size` (a power of two) keys, the largest first.
__device__ __forceinline__ void sort_keys(Pool& b, int size) {
#pragma unroll 1
  for (int k = 2; k <= size; k *= 2)
#pragma unroll 1
    for (int j = k / 2; j > 0; j /= 2) {
      __syncthreads();
#pragma unroll 1
      for (int x = thread_here(); x < size / 2; x += kPartThreads) {
        const int lo = 2 * x - (x & (j - 1)), hi = lo + j;
        const uint64_t p = b.keys[lo], q = b.keys[hi];
        if ((p < q) == ((lo & k) == 0)) {
          b.keys[lo] = q;
          b.keys[hi] = p;
        }
      }
    }
  __syncthreads();
}

// Keeps the K largest of n keys, sorted; returns their number. For what the quicker ways below do not manage.
__device__ __forceinline__ int keep(Pool& b, int n, int K) {
  __syncthreads();
  int size = 2;
  while (size < n) size *= 2;
#pragma unroll 1
  for (int i = n + thread_here(); i < size; i += kPartThreads) b.keys[i] = 0;
  sort_keys(b, size);
  if (threadIdx.x == 0) b.bar = n >= K ? b.keys[K - 1] : 0;
  __syncthreads();
  return min(n, K);
}

// A logit that words of further batches have to pass: with key `bar` the K-th largest of earlier words, an equal one loses.
__device__ __forceinline__ float bar_of(uint64_t bar) { return bar ? logit_of((uint32_t)(bar >> 32)) : -__builtin_huge_valf(); }

// Leaves the keys whose rank is not below `least`; returns their number.
__device__ __forceinline__ int filter(Pool& b, int n, uint32_t least) {
  constexpr int N = kRoom / kPartThreads;
  uint64_t v[N];
  const int tid = thread_here();
  __syncthreads();
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int i = tid + j * kPartThreads;
    v[j] = i < n ? b.keys[i] : 0;
  }
  if (threadIdx.x == 0) b.count[0] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (v[j] && (uint32_t)(v[j] >> 32) >= least) b.keys[atomicAdd(&b.count[0], 1)] = v[j];
  __syncthreads();
  return b.count[0];
}

// The K largest of n keys, put(place, key) for each by some thread, 0 for places without.
template <typename F>
__device__ __forceinline__ void put_best(Pool& b, int n, int K, F put) {
  constexpr int kFew = 128, kRanked = 512;
  __syncthreads();
  if (n > kFew && n > K) n = filter(b, n, kth_in(b, n, K));
  if (n > kRanked) n = keep(b, n, K);
#pragma unroll 1
  for (int i = thread_here(); i < n; i += kPartThreads) {
    const uint64_t key = b.keys[i];
    int place = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) place += b.keys[j] > key;
    if (place < K) put(place, key);
  }
#pragma unroll 1
  for (int k = n + thread_here(); k < K; k += kPartThreads) put(k, (uint64_t)0);
}

// Offers vectors first .. end - 1 a few words of a thread at a time, looking at the room left in between; the n keys
// before them are all there. Returns the keys' number.
template <typename T>
__device__ __forceinline__ int offer_slowly(Pool& b, int n, int K, const T* row, const Span& sp, int first, int end) {
  constexpr int pieces = kPer<T> / kStep;
  const int tid = thread_here(), stop = end * pieces;
#pragma unroll 1
  for (int i0 = first * pieces;; i0 += kPartThreads) {
    if (n > kRoom - kStep * kPartThreads || i0 >= stop) n = keep(b, n, K);
    if (i0 >= stop) return n;
    __syncthreads();
    if (threadIdx.x == 0) b.count[0] = 0;
    __syncthreads();
    if (i0 + tid < stop) {
      const int word = sp.head + (i0 + tid) * kStep;
#pragma unroll 1
      for (int e = 0; e < kStep; ++e) {
        const float l = load1(row + word + e);
        const uint64_t key = key_of(l, word + e);
        if (l != -__builtin_huge_valf() && key > b.bar) b.keys[n + atomicAdd(&b.count[0], 1)] = key;
      }
    }
    __syncthreads();
    n += b.count[0];
  }
}

// The K largest words' keys of vectors first .. end - 1 of a row (and of the elements outside of the vectors, with `odds`),
// and the sums of these. A batch is U vectors of each thread; a word of it is taken if it passes the bar, a lower
// bound on the K-th largest so far: after the first batch from the largest of each thread's two halves of it, later, when
// the words seen have doubled, from the keys themselves. Batches go through the words in their order, so that an
// equal word of a later one loses.
template <typename T, int U, bool STREAM>
__device__ __forceinline__ int select_part(const T* row, const Span& sp, int V, int first, int end, bool odds, int K, float c,
                                           Pool& b, Soft& x) {
  const float low = -__builtin_huge_valf();
  const int odd = odds ? odd_of<T>(sp, V) : -1;
  const float lodd = odd >= 0 ? load1(row + odd) : low;
  x = none();
  if (odd >= 0) add1(x, lodd, c);
  if (threadIdx.x < 3) b.count[threadIdx.x] = 0;
  if (threadIdx.x == 0) b.bar = 0;
  __syncthreads();
  if (odd >= 0 && odd < sp.head && lodd != low) b.keys[atomicAdd(&b.count[2], 1)] = key_of(lodd, odd);
  __syncthreads();
  int n = b.count[2], turn = 0, batch = 0;
  float bar = low;
  for (int i0 = first; i0 < end; i0 += U * kPartThreads, ++batch) {
    u32x4 v[U];
    float vm[U];
    const int i = i0 + (int)threadIdx.x;
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = i + u * kPartThreads < end ? load_vec<STREAM>(row + sp.head, i + u * kPartThreads) : nothing<T>();
    float m = x.m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      vm[u] = low;
#pragma unroll
      for (int e = 0; e < kPer<T>; ++e) vm[u] = fmaxf(vm[u], element<T>(v[u], e));
      asm volatile("" : "+v"(vm[u]));
      m = fmaxf(m, vm[u]);
    }
    x = rebase(x, m, c);
    float s = 0.f, w = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      again(v[u]);
#pragma unroll
      for (int e = 0; e < kPer<T>; ++e) {
        const float d = element<T>(v[u], e) - m, p = __builtin_amdgcn_exp2f(d * c);
        s += p;
        w = fmaf(p, fmaxf(d, kFar), w);
      }
      asm volatile("" : "+v"(s), "+v"(w));  // one vector's elements after another's
    }
    x.s += s;
    x.u += w;
    if (batch == 0) {
      float lo = vm[0], hi = vm[U / 2];
#pragma unroll
      for (int u = 1; u < U / 2; ++u) {
        lo = fmaxf(lo, vm[u]);
        hi = fmaxf(hi, vm[U / 2 + u]);
      }
      b.tops[threadIdx.x] = rank_of(lo);
      b.tops[kPartThreads + threadIdx.x] = rank_of(hi);
      __syncthreads();
      const uint32_t r = kth_of<2 * kPartThreads / 64>(2 * kPartThreads, K, [&](int j) { return b.tops[j]; });
      // words of rank r pass (the rank below 0's is no number's)
      bar = r <= rank_of(low) ? low : r == rank_of(0.f) ? -1e-30f : logit_of(r - 1);
    }
    const bool all = x.s != x.s;  // a NaN, which the maxima pass over, or +inf
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (vm[u] > bar || all) {
        again(v[u]);
#pragma unroll
        for (int e = 0; e < kPer<T>; ++e) {
          const float l = element<T>(v[u], e);
          if (!(l <= bar)) {
            const int at = n + atomicAdd(&b.count[turn], 1);
            if (at < kRoom) b.keys[at] = key_of(l, sp.head + (i + u * kPartThreads) * kPer<T> + e);
          }
        }
      }
    __syncthreads();
    const int more = b.count[turn];
    const int next = turn == 2 ? 0 : turn + 1, last = turn == 0 ? 2 : turn - 1;
    if (threadIdx.x == 0) b.count[last] = 0;  // read before this barrier, added to after the next
    turn = next;
    if (n + more > kRoom) {
      n = offer_slowly(b, n, K, row, sp, i0, min(i0 + U * kPartThreads, end));
      bar = bar_of(b.bar);
      __syncthreads();
      if (threadIdx.x < 3) b.count[threadIdx.x] = 0;
      __syncthreads();
      continue;
    }
    n += more;
    if (n > kRoom / 2) {
      n = filter(b, n, kth_in(b, n, K));
      if (n > kRoom / 2) n = keep(b, n, K);
      if (n >= K) bar = logit_of(kth_in(b, n, K));
      __syncthreads();
      if (threadIdx.x < 3) b.count[threadIdx.x] = 0;
      __syncthreads();
    } else if (n >= K && (batch == 0 || (batch & (batch + 1)) == 0)) {
      bar = logit_of(kth_in(b, n, K));
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) b.count[0] = 0;
  __syncthreads();
  if (odd >= sp.head && lodd != low) b.keys[n + atomicAdd(&b.count[0], 1)] = key_of(lodd, odd);
  __syncthreads();
  return n + b.count[0];
}

// A row's results from its sums, its target's logit and its words' keys.
__device__ __forceinline__ void write_top(const TopArgs& g, int t, int k, uint64_t key, const Soft& x, const RowStats& r) {
  const int64_t at = (int64_t)t * g.K + k;
  g.ids[at] = key ? (int)~(uint32_t)key : -1;
  g.tops[at] = key ? (logit_of((uint32_t)(key >> 32)) - x.m) * g.z.inv_temp - r.log_s : -__builtin_huge_valf();
}
__device__ __forceinline__ void write_stats(const TopArgs& g, int t, const RowStats& r) {
  if (g.z.logp) g.z.logp[t] = r.lp;
  if (g.z.ent) g.z.ent[t] = r.ent;
}
// A row that takes no part.
__device__ __forceinline__ void write_none(const TopArgs& g, int t) {
  for (int k = (int)threadIdx.x; k < g.K; k += kPartThreads) write_top(g, t, k, 0, none(), RowStats{});
  if (threadIdx.x == 0) write_stats(g, t, RowStats{});
}

__device__ __forceinline__ uint64_t load_key(const uint64_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Joins row t's parts, whose lists are sorted: as each of S lists has K / S keys that are not below its own K / S-th, the
// smallest of these is a lower bound.
__device__ __forceinline__ void join_parts(const TopArgs& g, int t, Pool& b) {
  const LogitsArgs& a = g.z;
  const float c = a.inv_temp * kLog2e;
  const Soft x = first_lane(merge_parts(a, t, c));
  const RowStats r = row_stats(a, x, load_part(reinterpret_cast<const float*>(a.part + (int64_t)t * a.splits) + 3));
  if (threadIdx.x == 0) write_stats(g, t, r);
  const uint64_t* lists = g.keys + (int64_t)t * a.splits * g.K;
  const int each = (g.K + a.splits - 1) / a.splits, all = a.splits * g.K;
  uint64_t bar = ~(uint64_t)0;
  for (int s = (int)(threadIdx.x & 63); s < a.splits; s += 64) {
    const uint64_t key = load_key(lists + s * g.K + each - 1);
    bar = key < bar ? key : bar;
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const uint64_t y = __shfl_xor(bar, o, 64);
    bar = y < bar ? y : bar;
  }
  if (threadIdx.x == 0) b.count[0] = 0, b.count[1] = 0, b.bar = 0;
  __syncthreads();
  for (int i = (int)threadIdx.x; i < all; i += kPartThreads) {
    const uint64_t key = load_key(lists + i);
    if (!key || key < bar) continue;
    const int at = atomicAdd(&b.count[0], 1);
    if (at < kRoom) b.keys[at] = key;
  }
  __syncthreads();
  int n = b.count[0];
  if (n > kRoom) {
    n = 0;
    for (int i0 = 0; i0 < all; i0 += kPartThreads) {
      if (n > kRoom - kPartThreads) n = keep(b, n, g.K);
      __syncthreads();
      if (threadIdx.x == 0) b.count[1] = 0;
      __syncthreads();
      const int i = i0 + (int)threadIdx.x;
      const uint64_t key = i < all ? load_key(lists + i) : 0;
      if (key && key > b.bar) b.keys[n + atomicAdd(&b.count[1], 1)] = key;
      __syncthreads();
      n += b.count[1];
    }
  }
  put_best(b, n, g.K, [&](int k, uint64_t key) { write_top(g, t, k, key, x, r); });
}

// Workgroup (row, part): a whole row's results, or a part's sums and sorted keys, which the last part's workgroup joins
// where arrivals are counted.
template <typename T, int U, bool STREAM>
__global__ __launch_bounds__(kPartThreads) void top_kernel(TopArgs g) {
  const LogitsArgs& a = g.z;
  __shared__ Pool b;
  const int t = (int)(blockIdx.x / (uint32_t)a.splits), p = (int)(blockIdx.x - (uint32_t)t * a.splits);
  const int y = a.targets ? target_of(a, t) : 0;
  if (y < 0) {
    if (p == 0) write_none(g, t);
    return;
  }
  const T* row = static_cast<const T*>(a.logits) + (int64_t)t * a.stride;
  const Span sp = row_span(row, a.V);
  const int first = p * a.chunk, end = min(first + a.chunk, sp.vectors);
  const float c = a.inv_temp * kLog2e, ly = load1(row + y);
  Soft x;
  const int n = select_part<T, U, STREAM>(row, sp, a.V, first, end, p == a.splits - 1, g.K, c, b, x);
  x = first_lane(group_merge<kPartThreads>(x, c));
  if (a.splits == 1) {
    const RowStats r = row_stats(a, x, ly);
    if (threadIdx.x == 0) write_stats(g, t, r);
    put_best(b, n, g.K, [&](int k, uint64_t key) { write_top(g, t, k, key, x, r); });
    return;
  }
  if (threadIdx.x == 0) {
    float* part = reinterpret_cast<float*>(a.part + (int64_t)t * a.splits + p);
    store_part(part, x.m, x.s);
    store_part(part + 2, x.u, ly);
  }
  uint64_t* list = g.keys + ((int64_t)t * a.splits + p) * g.K;
  put_best(b, n, g.K, [&](int k, uint64_t key) { __hip_atomic_store(list + k, key, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); });
  if (!a.counts) return;
  parts_written();
  __syncthreads();
  uint64_t before = 0;
  if (threadIdx.x == 0) before = arrive(a.counts + t * kShortCountStride, a.epoch);
  if (last_of(before, a.epoch, a.splits)) join_parts(g, t, b);
}

__global__ __launch_bounds__(kPartThreads) void top_join_kernel(TopArgs g) {
  __shared__ Pool b;
  const int t = (int)blockIdx.x, y = g.z.targets ? target_of(g.z, t) : 0;
  if (y >= 0) join_parts(g, t, b);
}

hipError_t launch(const void* kernel, int64_t wgs, const TopArgs& a, hipStream_t s) {
  TopArgs args = a;
  void* params[] = {&args};
  return hipLaunchKernel(kernel, dim3((unsigned)wgs), dim3(kPartThreads), params, 0, s);
}

template <typename T>
hipError_t top_for(const TopArgs& a, hipStream_t s) {
  const void* k = a.z.chunk < 8 * kPartThreads ? reinterpret_cast<const void*>(&top_kernel<T, 4, false>)
                                               : reinterpret_cast<const void*>(&top_kernel<T, 8, true>);
  const hipError_t e = launch(k, (int64_t)a.z.T * a.z.splits, a, s);
  if (e != hipSuccess || a.z.splits == 1 || a.z.counts) return e;
  return launch(reinterpret_cast<const void*>(&top_join_kernel), a.z.T, a, s);
}

}  // namespace

hipError_t launch_top_logprobs(const TopArgs& a, hipStream_t s) {
  return a.z.bf16 ? top_for<uint16_t>(a, s) : top_for<float>(a, s);
}

}  // namespace pda
