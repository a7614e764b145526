// HIP kernels for the most likely words of rows of logits, with their
// log-probabilities, on MI355X (gfx950).
//
// A row's words are in one order: by logit, equal ones by their place. A word's key
// is its logit's bits, made to compare as whole numbers do, over the complement of
// its place: all keys of a row differ, and the K largest are the answer.

#include "pda_lm_internal.h"
#include "pda_rows.h"

#include <type_traits>

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

constexpr int kWaves = kPartThreads / 64;
constexpr int kRegion = kRoom / kWaves;  // keys that a wave holds by itself
constexpr int kRoomy = kRegion - 16;     // of them the vectors', the rest for the elements outside of all vectors

// Keys that may be among the K largest, in no order: while a row is read, each wave's in its own region, afterwards
// side by side.
struct Pool {
  uint64_t keys[kRoom];
  u32x4 queue[kWaves][64];  // vectors that hold a word above the bar, each wave's, to be looked through together
  int first[kWaves][64];    // their first words
  uint64_t bar;          // after keep(): the K-th largest, 0 where there are fewer
  int held[2][kWaves];   // of each wave's region, in turn
  int count;
  uint32_t floor;        // a bar on its way from the wave that settled it
  uint32_t tops[2 * kPartThreads];
};

__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }
// Bits of `mask` below this lane's.
__device__ __forceinline__ int lanes_before(uint64_t mask) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// Between a wave's writes to LDS and its other lanes' reads of them, or reads and the writes over them: its lanes go on together, and the
// compiler moves neither across (no instruction of its own).
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// This thread's number, for code that is seldom reached: the compiler works out what follows from it there, rather than
// once for all at the kernel's start and in registers of its own.
__device__ __forceinline__ int thread_here() {
  int t = (int)threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// Over the 64 lanes, in each of them.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, o, 64));
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}

// Of the ranks that the wave's lanes hold N each of (0: none): one that at least K are not below, and that is their K-th
// largest in its upper 16 bits, 0 where there are fewer; the same in every lane. Halves what is between `from`, which the
// K-th largest is not below, and the largest, by counting.
template <int N, int M>
__device__ __forceinline__ uint32_t kth_of(const uint32_t (&v)[M], int K, uint32_t from) {
  uint32_t top = v[0];
#pragma unroll
  for (int j = 1; j < N; ++j) top = max(top, v[j]);
  uint32_t lo = from >> 16, hi = wave_max(top) >> 16;
#pragma unroll 1
  while (lo < hi) {
    const uint32_t mid = (lo + hi + 1) / 2, least = mid << 16;
    int n = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) n += (int)__popcll(__ballot(v[j] >= least));
    if (n >= K) lo = mid;
    else hi = mid - 1;
  }
  return lo << 16;
}
// What the waves hold.
struct Held {
  int n[kWaves];
  __device__ __forceinline__ int all() const { return n[0] + n[1] + n[2] + n[3]; }
  __device__ __forceinline__ int most() const { return max(max(n[0], n[1]), max(n[2], n[3])); }
};
static_assert(kWaves == 4, "Held");
// Of the keys in the waves' regions, N in each lane from each region.
template <int N>
__device__ __forceinline__ uint32_t kth_held(const Pool& b, const Held& h, int K, uint32_t from) {
  const int lane = thread_here() & 63;
  uint32_t v[kWaves * N];
#pragma unroll
  for (int j = 0; j < kWaves * N; ++j) {
    const int w = j / N, i = lane + 64 * (j % N);
    v[j] = i < h.n[w] ? (uint32_t)(b.keys[w * kRegion + i] >> 32) : 0;
  }
  return kth_of<kWaves * N>(v, K, from);
}
__device__ __forceinline__ uint32_t kth_held(const Pool& b, const Held& h, int K, uint32_t from) {
  const int most = h.most();
  return most <= 128 ? kth_held<2>(b, h, K, from) : most <= 256 ? kth_held<4>(b, h, K, from) : kth_held<kRegion / 64>(b, h, K, from);
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

// This wave's keys of rank `least` and above to the front of its region; returns their number.
__device__ __forceinline__ int thin(Pool& b, int n, uint32_t least) {
  uint64_t* keys = b.keys + wave_id() * kRegion;
  const int lane = thread_here() & 63;
  int kept = 0;
#pragma unroll 1
  for (int i = 0; i < n; i += 64) {  // writes stay behind what has been read
    const uint64_t key = i + lane < n ? keys[i + lane] : 0;
    const bool stays = key && (uint32_t)(key >> 32) >= least;
    const uint64_t mask = __ballot(stays);
    wave_sync();
    if (stays) keys[kept + lanes_before(mask)] = key;
    kept += (int)__popcll(mask);
  }
  return kept;
}

// The waves' keys of rank `least` and above, side by side; returns their number. n: what this wave holds.
__device__ __forceinline__ int gather(Pool& b, int n, uint32_t least) {
  constexpr int N = kRegion / 64;
  const int wave = wave_id(), lane = thread_here() & 63;
  uint64_t v[N];
  int kept = 0;
  wave_sync();  // this wave's last keys
#pragma unroll
  for (int j = 0; j < N; ++j) {
    v[j] = lane + 64 * j < n ? b.keys[wave * kRegion + lane + 64 * j] : 0;
    if ((uint32_t)(v[j] >> 32) < least) v[j] = 0;
    kept += (int)__popcll(__ballot(v[j] != 0));
  }
  __syncthreads();  // earlier counts have been read
  if (lane == 0) b.held[0][wave] = kept;
  __syncthreads();
  int at = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    at += w < wave ? b.held[0][w] : 0;
    all += b.held[0][w];
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const uint64_t mask = __ballot(v[j] != 0);
    if (v[j]) b.keys[at + lanes_before(mask)] = v[j];
    at += (int)__popcll(mask);
  }
  __syncthreads();
  return all;
}

// The K largest of n keys that lie side by side, put(place, key) for each by some thread, 0 for places without. A key's
// place is the number of larger ones: counted by several threads for each key, or by one for two.
template <typename F>
__device__ __forceinline__ void put_best(Pool& b, int n, int K, F put) {
  __syncthreads();
  if (n > 2 * kPartThreads) n = keep(b, n, K);
  const int tid = thread_here();
  if (n > kPartThreads) {
    const uint64_t key = b.keys[tid], more = tid + kPartThreads < n ? b.keys[tid + kPartThreads] : 0;
    int place = 0, after = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) {
      const uint64_t other = b.keys[j];
      place += other > key;
      after += other > more;
    }
    if (place < K) put(place, key);
    if (more && after < K) put(after, more);
  } else {
    int each = 1;
    while (each < 16 && 2 * each * n <= kPartThreads) each *= 2;
    const int i = tid / each;
    const uint64_t key = i < n ? b.keys[i] : 0;
    int place = 0;
#pragma unroll 8
    for (int j = tid & (each - 1); j < n; j += each) place += b.keys[j] > key;
    for (int o = 1; o < each; o *= 2) place += __shfl_xor(place, o, 64);
    if (key && !(tid & (each - 1)) && place < K) put(place, key);
  }
#pragma unroll 1
  for (int k = n + tid; k < K; k += kPartThreads) put(k, (uint64_t)0);
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
    if (threadIdx.x == 0) b.count = 0;
    __syncthreads();
    if (i0 + tid < stop) {
      const int word = sp.head + (i0 + tid) * kStep;
#pragma unroll 1
      for (int e = 0; e < kStep; ++e) {
        const float l = load1(row + word + e);
        const uint64_t key = key_of(l, word + e);
        if (l != -__builtin_huge_valf() && key > b.bar) b.keys[n + atomicAdd(&b.count, 1)] = key;
      }
    }
    __syncthreads();
    n += b.count;
  }
}

// A row's largest logit m, and below it as base2 has them the sums of exponentials and of exponentials times exponents.
struct Mass {
  float m, s, u;
};
__device__ __forceinline__ Mass rebase(const Mass& x, float m, float c) {
#pragma clang fp contract(off)  // rounded products, whatever adds them: lanes that sum each other's agree
  const float k = exponent_to(x.m, m, c), f = __builtin_amdgcn_exp2f(k);
  return Mass{m, x.s * f, f * fmaf(x.s, fmaxf(k, kFar), x.u)};
}
__device__ __forceinline__ Mass merge(const Mass& a, const Mass& b, float c) {
  const float m = fmaxf(a.m, b.m);
  const Mass x = rebase(a, m, c), y = rebase(b, m, c);
  return Mass{m, x.s + y.s, x.u + y.u};
}
__device__ __forceinline__ void add1(Mass& x, float l, float c) {
  const float m = fmaxf(x.m, l);
  x = rebase(x, m, c);
  const float d = base2(m, c).of(l), p = __builtin_amdgcn_exp2f(d);
  x.s += p;
  x.u = fmaf(p, fmaxf(d, kFar), x.u);
}
// Over the 64 lanes, in each of them.
__device__ __forceinline__ Mass wave_merge(const Mass& x, float c) {
  const float m = wave_top(x.m);
  const Mass y = rebase(x, m, c);
  return Mass{m, wave_total(y.s), wave_total(y.u)};
}
// Over the workgroup, in every thread (and a barrier for all of them).
__device__ __forceinline__ Mass group_merge(Mass x, float c) {
  __shared__ Mass parts[kWaves];
  x = wave_merge(x, c);
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = x;
  __syncthreads();
  Mass y = parts[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) y = merge(y, parts[w], c);
  return y;
}
__device__ __forceinline__ RowStats row_stats(const LogitsArgs& a, const Mass& x, float ly) {
  RowStats r;
  if (x.s == 0.f) {  // every logit is -inf: no distribution
    r.lp = -__builtin_huge_valf();
    r.ent = r.log_s = 0.f;
    return r;
  }
  r.log_s = log_below(x.s, x.m, base2_rate(a));
  r.lp = fmaf(ly - x.m, a.inv_temp, -r.log_s);
  r.ent = fmaf(-x.u / x.s, 1.f / kLog2e, logf(x.s));
  return r;
}

// What the words of further batches have to pass.
struct Bar {
  float least;  // words above it pass; NaN does
  bool closed;  // none does
};
__device__ __forceinline__ Bar bar_at(uint32_t rank) {
  const float l = logit_of(rank);
  return l != l ? Bar{__builtin_huge_valf(), true} : Bar{l, false};
}

// The keys, side by side, of words among which the K largest of vectors first .. end - 1 of a row (and of the elements outside of
// the vectors, with `odds`) are, their number, and these words' sums. A batch is U vectors of each thread; a word of it is
// taken if it passes the bar, a lower bound on the K-th largest so far: in the first batch from the largest of
// each thread's words of it (or, for many places, of its even and odd vectors), later, when the batches read have doubled, from the keys themselves.
// Between these points the waves go on by themselves. Batches go through the words in their order, so that an equal word
// of a later one loses.
template <typename T, int U, bool STREAM>
__device__ __forceinline__ int select_part(const T* row, const Span& sp, int V, int first, int end, bool odds, int K, float c,
                                           Pool& b, Mass& x) {
  const float low = -__builtin_huge_valf();
  const int odd = odds ? odd_of<T>(sp, V) : -1, wave = wave_id(), lane = (int)(threadIdx.x & 63);
  const float lodd = odd >= 0 ? load1(row + odd) : low;
  x = Mass{kLowest, 0.f, 0.f};
  if (odd >= 0) add1(x, lodd, c);
  if (threadIdx.x == 0) b.bar = 0;  // read some barriers later
  uint64_t* keys = b.keys + wave * kRegion;
  int n = 0, turn = 0;  // n: of this wave's keys
  Held held = {};
  const auto take = [&](bool hit, float l, int word) {  // all lanes together
    const uint64_t mask = __ballot(hit);
    if (!mask) return;
    const int at = n + lanes_before(mask);
    if (hit && at < kRegion) keys[at] = key_of(l, word);
    n += (int)__popcll(mask);
  };
  int queued = 0;
  const auto look_through = [&](const float least) {
    wave_sync();
    const u32x4 w = b.queue[wave][lane];
    const int word = b.first[wave][lane];
    wave_sync();
#pragma unroll
    for (int e = 0; e < kPer<T>; ++e) {
      const float l = element<T>(w, e);
      take(lane < queued && !(l <= least), l, word + e);
    }
    queued = 0;
  };
  take(odd >= 0 && odd < sp.head && lodd != low, lodd, odd);
  const auto share = [&](int n) {
    if (lane == 0) b.held[turn][wave] = n;
    __syncthreads();
    Held h;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) h.n[w] = __builtin_amdgcn_readfirstlane(b.held[turn][w]);
    turn ^= 1;
    return h;
  };
  Bar bar = {low, false};
  // one wave of the workgroup, not always the same, settles the bars: the vector ALUs have no time for four
  const int settler = (int)blockIdx.x % kWaves;
  const bool few = K <= kPartThreads / 4;
  uint32_t floor = 0;  // the K-th largest rank so far is not below it
  int since = first, mine = n;  // the vectors that came after the last look at all keys; what this wave held then
  // 0 times -inf of a masked word is NaN: exponents have a least value (kFar), in longer parts from this wave's first batch with one
  // on (us per call, 20 alternatives of 131,072 words bf16, always / from the first on: 4,096 rows 206 / 199, half of the words
  // masked 186 / 195). Parts of few batches do not begin one twice (64 rows, half masked 15.6 / 16.9).
  bool masked = end - first <= 2 * U * kPartThreads;
  for (int i0 = first, batch = 0; i0 < end; i0 += U * kPartThreads, ++batch) {
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
    const Base2 below = base2(m, c);
    float s, w;
    const auto sums = [&](auto far, auto least) {
      s = w = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        again(v[u]);
#pragma unroll
        for (int e = 0; e < kPer<T>; ++e) {
          const float d = below.of<decltype(far)::value>(element<T>(v[u], e)), p = __builtin_amdgcn_exp2f(d);
          s += p;
          w = fmaf(p, decltype(least)::value ? fmaxf(d, kFar) : d, w);
        }
        asm volatile("" : "+v"(s), "+v"(w));  // one vector's elements after another's
      }
    };
    if (!masked) {
      sums(std::false_type(), std::false_type());
      masked = __ballot(below.far || w != w) != 0;
    }
    if (masked) {
      if (!below.far) sums(std::false_type(), std::true_type());
      else sums(std::true_type(), std::true_type());
    }
    x.s += s;
    x.u += w;
    if (batch == 0) {
      float lo = vm[0], hi = vm[1];
#pragma unroll
      for (int u = 2; u < U; u += 2) {
        lo = fmaxf(lo, vm[u]);
        hi = fmaxf(hi, vm[u + 1]);
      }
      if (few) lo = fmaxf(lo, hi);
      b.tops[threadIdx.x] = rank_of(lo);
      if (!few) b.tops[kPartThreads + threadIdx.x] = rank_of(hi);
      __syncthreads();
      if (wave == settler) {
        uint32_t t[2 * kWaves], r;
#pragma unroll
        for (int j = 0; j < kWaves; ++j) t[j] = b.tops[lane + 64 * j];
        if (few) {
          r = kth_of<kWaves>(t, K, 0);
        } else {
#pragma unroll
          for (int j = kWaves; j < 2 * kWaves; ++j) t[j] = b.tops[lane + 64 * j];
          r = kth_of<2 * kWaves>(t, K, 0);
        }
        if (lane == 0) b.floor = r;
      }
      __syncthreads();
      const uint32_t r = b.floor;
      // words of rank r pass (the rank below 0's is no number's)
      bar.least = r <= rank_of(low) ? low : r == rank_of(0.f) ? -1e-30f : logit_of(r - 1);
    }
    const bool all = x.s != x.s && !bar.closed;  // a NaN, which the maxima pass over, or +inf
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool hit = vm[u] > bar.least || all;
      const uint64_t mask = __ballot(hit);
      if (!mask) continue;
      const int more = (int)__popcll(mask);
      if (queued + more > 64) look_through(bar.least);
      if (hit) {
        const int at = queued + lanes_before(mask);
        b.queue[wave][at] = v[u];
        b.first[wave][at] = sp.head + (i + u * kPartThreads) * kPer<T>;
      }
      queued += more;
    }
    const int next = i0 + U * kPartThreads;
    const bool last = next >= end;
    if (!last && (batch & 63) != 63 && ((batch & (batch + 1)) != 0 || (batch == 0 && K <= kPartThreads / 2))) continue;
    if (queued) look_through(bar.least);
    Held now = share(n);
    if (now.most() > kRoomy) {  // some are lost: from the last look on again
      const int total = offer_slowly(b, gather(b, mine, 0), K, row, sp, since, min(next, end));
      floor = (uint32_t)(b.bar >> 32);
      bar = b.bar ? bar_at(floor) : Bar{low, false};
      now = Held{{total, 0, 0, 0}};
      n = wave == 0 ? total : 0;
      __syncthreads();
    } else if (!last && now.all() >= K) {
      if (wave == settler) {
        floor = kth_held(b, now, K, floor);
        if (lane == 0) b.floor = floor;
      }
      __syncthreads();
      floor = b.floor;
      bar = bar_at(floor);
      if (now.most() > kRegion / 2) {
        n = thin(b, n, floor);
        now = share(n);
      }
    }
    held = now;
    mine = n;
    since = next;
  }
  take(odd >= sp.head && lodd != low, lodd, odd);
  uint32_t least = 0;
  if (held.all() > kPartThreads / 2 && held.all() > K) {
    if (wave == settler) {
      least = kth_held(b, held, K, floor);
      if (lane == 0) b.floor = least;
    }
    __syncthreads();
    least = b.floor;
  }
  return gather(b, n, least);
}

// A row's results from its sums, its target's logit and its words' keys.
__device__ __forceinline__ void write_top(const TopArgs& g, int t, int k, uint64_t key, const Mass& x, const RowStats& r) {
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
  for (int k = (int)threadIdx.x; k < g.K; k += kPartThreads) write_top(g, t, k, 0, Mass{}, RowStats{});
  if (threadIdx.x == 0) write_stats(g, t, RowStats{});
}

__device__ __forceinline__ uint64_t load_key(const uint64_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Joins row t's parts, whose lists are sorted: as each of S lists has K / S keys that are not below its own K / S-th, the
// smallest of these is a lower bound. What is read is asked for at once.
__device__ __forceinline__ void join_parts(const TopArgs& g, int t, Pool& b) {
  constexpr int U = 4;
  const LogitsArgs& a = g.z;
  const uint64_t* lists = g.keys + (int64_t)t * a.splits * g.K;
  const int each = (g.K + a.splits - 1) / a.splits, all = a.splits * g.K;
  uint64_t keys[U];
  const auto load = [&](int i0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kPartThreads + (int)threadIdx.x;
      keys[u] = i < all ? load_key(lists + i) : 0;
    }
  };
  load(0);
  uint64_t bar = ~(uint64_t)0;
  static_assert(kMaxSplits <= 64, "a lane each");
  const int s = (int)(threadIdx.x & 63);
  if (s < a.splits) bar = load_key(lists + s * g.K + each - 1);
  const float ly = load_part(reinterpret_cast<const float*>(a.part + (int64_t)t * a.splits) + 3);
  const float* part = reinterpret_cast<const float*>(a.part + (int64_t)t * a.splits + min(s, a.splits - 1));
  const Mass mine = {load_part(part), load_part(part + 1), load_part(part + 2)};
  const Mass x = wave_merge(s < a.splits ? mine : Mass{kLowest, 0.f, 0.f}, base2_rate(a));
  const RowStats r = row_stats(a, x, ly);
  if (threadIdx.x == 0) write_stats(g, t, r);
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const uint64_t y = __shfl_xor(bar, o, 64);
    bar = y < bar ? y : bar;
  }
  if (threadIdx.x == 0) b.count = 0, b.bar = 0;
  __syncthreads();
  for (int i0 = 0;;) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (keys[u] && keys[u] >= bar) {
        const int at = atomicAdd(&b.count, 1);
        if (at < kRoom) b.keys[at] = keys[u];
      }
    i0 += U * kPartThreads;
    if (i0 >= all) break;
    load(i0);
  }
  __syncthreads();
  int n = b.count;
  if (n > kRoom) {  // as many at a time as fit behind the K largest
    n = 0;
    for (int i0 = 0; i0 < all; i0 += kPartThreads) {
      if (n > kRoom - kPartThreads) n = keep(b, n, g.K);
      __syncthreads();
      if (threadIdx.x == 0) b.count = 0;
      __syncthreads();
      const int i = i0 + (int)threadIdx.x;
      const uint64_t key = i < all ? load_key(lists + i) : 0;
      if (key && key > b.bar) b.keys[n + atomicAdd(&b.count, 1)] = key;
      __syncthreads();
      n += b.count;
    }
  }
  put_best(b, n, g.K, [&](int k, uint64_t key) { write_top(g, t, k, key, x, r); });
}

// Workgroup (row, part): a whole row's results, or a part's sums and sorted keys, which the last part's workgroup joins
// where arrivals are counted.
// Where rows are many the vector ALUs bound it (a word's sums take 8.5 instructions by their counters, with two conversions, a maximum, two
// multiply-adds, an addition and an exponential of four times the length; looking for words adds 2.3): 4,096 x 131,072 bf16,
// 64 alternatives 180-200 us, 8,192 rows 328 (6.5 TB/s). Where they are few, the chain of loads, bar, keys, arrival and
// join does: 64 rows, 20 alternatives 14 us.
// Six workgroups to a compute unit, as many as LDS holds: 4,096 x 131,072 bf16, 256 alternatives, 228 us, with the registers of five 243.
template <typename T, int U, bool STREAM>
__global__ __launch_bounds__(kPartThreads, 6) void top_kernel(TopArgs g) {
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
  const float c = base2_rate(a), ly = load1(row + y);
  Mass x;
  const int n = select_part<T, U, STREAM>(row, sp, a.V, first, end, p == a.splits - 1, g.K, c, b, x);
  x = group_merge(x, c);
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

// ------------------------------------------------------------- short rows

// M keys of each lane, key i = r 64 + lane in v[r], sorted, the largest first.
template <int M>
__device__ __forceinline__ void sort_wave(uint64_t (&v)[M]) {
  const int lane = (int)(threadIdx.x & 63);
#pragma unroll
  for (int k = 2; k <= 64 * M; k *= 2)
#pragma unroll
    for (int j = k / 2; j > 0; j /= 2) {
      if (j >= 64) {
#pragma unroll
        for (int r = 0; r < M; ++r) {
          const int q = r ^ (j / 64);
          if (q < r) continue;
          const bool down = (r * 64 & k) == 0;  // (k > 64: a lane's bits do not matter)
          const uint64_t a = v[r], b = v[q];
          const bool swap = (a < b) == down;
          v[r] = swap ? b : a;
          v[q] = swap ? a : b;
        }
      } else {
#pragma unroll
        for (int r = 0; r < M; ++r) {
          const uint64_t other = __shfl_xor(v[r], j, 64);
          const bool down = ((r * 64 + lane) & k) == 0, first = (lane & j) == 0;
          v[r] = (v[r] < other) == (down == first) ? other : v[r];
        }
      }
    }
}

// Writes the K largest of a wave's n <= 64 M keys.
template <int M>
__device__ __forceinline__ void sort_and_write(const TopArgs& g, int t, const uint64_t* keys, int n, const Mass& x, const RowStats& r) {
  const int lane = (int)(threadIdx.x & 63);
  uint64_t v[M];
#pragma unroll
  for (int j = 0; j < M; ++j) v[j] = lane + 64 * j < n ? keys[lane + 64 * j] : 0;
  sort_wave(v);
#pragma unroll
  for (int j = 0; j < M; ++j)
    if (lane + 64 * j < g.K) write_top(g, t, lane + 64 * j, v[j], x, r);
#pragma unroll 1
  for (int k = lane + 64 * M; k < g.K; k += 64) write_top(g, t, k, 0, x, r);
}

// A wave per row, whose N vectors of each lane stay in registers. A lower bound on the K-th largest comes from the lanes' vectors'
// largest; if too many words are above it, the K-th largest itself is found by halving over the words, and of words
// equal to it the first ones are taken.
template <typename T, int N>
__global__ __launch_bounds__(kPartThreads) void top_rows_kernel(TopArgs g) {
  constexpr int kHold = 256;  // keys of a wave
  __shared__ uint64_t pools[kWaves][kHold];
  const LogitsArgs& a = g.z;
  const int wave = wave_id(), lane = (int)(threadIdx.x & 63), t = (int)blockIdx.x * kWaves + wave;
  if (t >= a.T) return;
  uint64_t* keys = pools[wave];
  int64_t y = 0;
  if (a.targets) {
    y = a.targets64 ? static_cast<const int64_t*>(a.targets)[t] : static_cast<const int32_t*>(a.targets)[t];
    if (y >= a.V && lane == 0) atomicOr(a.status, kStatusBadTarget);
  }
  if (y < 0 || y >= a.V) {
    for (int k = lane; k < g.K; k += 64) write_top(g, t, k, 0, Mass{}, RowStats{});
    if (lane == 0) write_stats(g, t, RowStats{});
    return;
  }
  const float low = -__builtin_huge_valf(), c = base2_rate(a);
  const T* row = static_cast<const T*>(a.logits) + (int64_t)t * a.stride;
  const Span sp = row_span(row, a.V);
  u32x4 v[N];
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = lane + 64 * n < sp.vectors ? load_vec<false>(row + sp.head, lane + 64 * n) : nothing<T>();
  const int in = sp.vectors * kPer<T>, odd = lane >= a.V - in ? -1 : lane < sp.head ? lane : lane + in;
  const float lodd = odd >= 0 ? load1(row + odd) : low, ly = load1(row + y);
  // sums
  float vm[N], m = fmaxf(kLowest, lodd);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    vm[n] = low;
#pragma unroll
    for (int e = 0; e < kPer<T>; ++e) vm[n] = fmaxf(vm[n], element<T>(v[n], e));
    m = fmaxf(m, vm[n]);
  }
  Mass x = {m, 0.f, 0.f};
  {
    const Base2 below = base2(m, c);
    const auto sum = [&](float d) {
      const float p = __builtin_amdgcn_exp2f(d);
      x.s += p;
      x.u = fmaf(p, fmaxf(d, kFar), x.u);
    };
    if (!below.far) {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        again(v[n]);
#pragma unroll
        for (int e = 0; e < kPer<T>; ++e) sum(below.of<false>(element<T>(v[n], e)));
        asm volatile("" : "+v"(x.s), "+v"(x.u));
      }
    } else {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        again(v[n]);
#pragma unroll
        for (int e = 0; e < kPer<T>; ++e) sum(below.of<true>(element<T>(v[n], e)));
        asm volatile("" : "+v"(x.s), "+v"(x.u));
      }
    }
    sum(below.of(lodd));
  }
  x = wave_merge(x, c);
  const RowStats r = row_stats(a, x, ly);
  if (lane == 0) write_stats(g, t, r);

  // each(f): f(logit, word) for all words, all lanes together, a vector's e-th words at a time
  const auto each = [&](auto f) {
    f(lodd, odd);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      again(v[n]);
#pragma unroll
      for (int e = 0; e < kPer<T>; ++e) f(element<T>(v[n], e), sp.head + (lane + 64 * n) * kPer<T> + e);
      asm volatile("");
    }
  };
  const auto count = [&](float least) {  // words not below it, NaN among them
    int n = 0;
    each([&](float l, int) { n += (int)__popcll(__ballot(!(l < least))); });
    return n;
  };
  int held = 0;
  const auto take = [&](bool hit, float l, int word) {
    const uint64_t mask = __ballot(hit);
    if (!mask) return;
    const int at = held + lanes_before(mask);
    if (hit && at < kHold) keys[at] = key_of(l, word);
    held += (int)__popcll(mask);
  };
  uint32_t ranks[N];
#pragma unroll
  for (int n = 0; n < N; ++n) ranks[n] = vm[n] == low ? 0 : rank_of(vm[n]);
  const uint32_t least = kth_of<N>(ranks, g.K, 0);
  const float from = least ? logit_of(least) : low;
  each([&](float l, int word) { take(!(l < from) && l != low, l, word); });
  if (held > kHold) {
    // exactly: ranks in 16 bits for bf16, whose lower 16 are its sign's
    constexpr int shift = sizeof(T) == 2 ? 16 : 0;
    const auto value = [&](uint32_t rank) {
      const uint32_t k = shift ? rank << 16 | (rank & 0x8000u ? 0u : 0xFFFFu) : rank;
      return logit_of(k);
    };
    uint32_t lo = (least ? least : rank_of(-3.402823466e38f)) >> shift, hi = rank_of(__builtin_huge_valf()) >> shift;
#pragma unroll 1
    while (lo < hi) {
      const uint32_t mid = lo + (hi - lo + 1) / 2;
      if (count(value(mid)) >= g.K) lo = mid;
      else hi = mid - 1;
    }
    const float kth = value(lo);
    // NaN passes as larger than the K-th, or if these are enough is what the K-th is
    int above = 0;
    each([&](float l, int) { above += (int)__popcll(__ballot(!(l <= kth))); });
    const bool nan = above >= g.K;
    const auto larger = [&](float l) { return !nan && !(l <= kth); };
    const auto equal = [&](float l) { return nan ? l != l : l == kth; };
    held = 0;
    wave_sync();
    each([&](float l, int word) { take(larger(l) && l != low, l, word); });
    // of the equal ones the first in the order of words: head, vectors by lane and element, tail
    int room = g.K - held;
    const bool head = odd >= 0 && odd < sp.head;
    const auto first_of = [&](bool hit, float l, int word) {
      const uint64_t mask = __ballot(hit);
      if (room <= 0 || !mask) return;
      take(hit && lanes_before(mask) < room, l, word);
      room -= (int)__popcll(mask);
    };
    first_of(head && equal(lodd), lodd, odd);
#pragma unroll 1
    for (int n = 0; n < N && room > 0; ++n) {
      u32x4 w = v[0];
#pragma unroll
      for (int i = 1; i < N; ++i) w = i == n ? v[i] : w;
      int before = 0, all = 0;  // equal words of lower lanes, and of all
#pragma unroll
      for (int e = 0; e < kPer<T>; ++e) {
        const uint64_t mask = __ballot(equal(element<T>(w, e)));
        before += lanes_before(mask);
        all += (int)__popcll(mask);
      }
      if (!all) continue;
#pragma unroll
      for (int e = 0; e < kPer<T>; ++e) {
        const float l = element<T>(w, e);
        const bool hit = equal(l);
        take(hit && before < room, l, sp.head + (lane + 64 * n) * kPer<T> + e);
        before += hit;
      }
      room -= all;
    }
    first_of(odd >= 0 && !head && equal(lodd), lodd, odd);
  }
  wave_sync();
  if (held <= 64) sort_and_write<1>(g, t, keys, held, x, r);
  else if (held <= 128) sort_and_write<2>(g, t, keys, held, x, r);
  else sort_and_write<4>(g, t, keys, held, x, r);
}

// ------------------------------------------------------------- launches

hipError_t launch(const void* kernel, int64_t wgs, const TopArgs& a, hipStream_t s) {
  TopArgs args = a;
  void* params[] = {&args};
  return hipLaunchKernel(kernel, dim3((unsigned)wgs), dim3(kPartThreads), params, 0, s);
}

// Whether a wave takes each row: always where 4 vectors of a lane hold it, with 8 where the rows are many. us per call, a
// workgroup / a wave per row, bf16: 8,192 x 1,000, 20 alternatives 56 / 18, x 2,000 55 / 20, with 256 372 / 61, x 4,000, 20 54 / 28, 256 119 /
// 102; 300 x 2,000, 20 9.3 / 8.2; 300 x 4,000, 100 11.2 / 13.3; 8 x 4,000, 256 16 / 38; 1 x 2,000, 20 8.0 / 7.5, x 4,000 8.7 / 10.6; f32
// 4,000 x 1,000, 20 28 / 11, x 2,000, 100 35 / 18.
constexpr int kManyRows = 600;

template <typename T>
hipError_t top_for(const TopArgs& a, hipStream_t s) {
  const int v = a.z.V / kPer<T>;
  if (v <= 64 * 4 || (v <= 64 * 8 && a.z.T >= kManyRows)) {
    const void* k = v <= 64 * 4 ? reinterpret_cast<const void*>(&top_rows_kernel<T, 4>) : reinterpret_cast<const void*>(&top_rows_kernel<T, 8>);
    return launch(k, (a.z.T + kWaves - 1) / kWaves, a, s);
  }
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
