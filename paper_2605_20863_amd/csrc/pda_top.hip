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

// The n largest so far (n <= kRoom), and the key that a further one has to pass.
struct Best {
  uint64_t keys[kRoom];
  uint64_t bar;
  int n;
};

// Sorts b.keys' first `size` (a power of two), the largest first.
__device__ __forceinline__ void sort_keys(Best& b, int size) {
  for (int k = 2; k <= size; k *= 2)
    for (int j = k / 2; j > 0; j /= 2) {
      __syncthreads();
      for (int x = (int)threadIdx.x; x < size / 2; x += kPartThreads) {
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

// Keeps the K largest, sorted.
__device__ __forceinline__ void keep(Best& b, int K) {
  __syncthreads();
  const int n = b.n;
  int size = 2;
  while (size < n) size *= 2;
  for (int i = n + (int)threadIdx.x; i < size; i += kPartThreads) b.keys[i] = 0;
  sort_keys(b, size);
  if (threadIdx.x == 0) {
    b.n = min(n, K);
    b.bar = n >= K ? b.keys[K - 1] : 0;
  }
  __syncthreads();
}

__device__ __forceinline__ void offer(Best& b, uint64_t bar, float l, int word) {
  if (l == -__builtin_huge_valf()) return;
  const uint64_t key = key_of(l, word);
  if (key > bar) b.keys[atomicAdd(&b.n, 1)] = key;
}

template <typename T>
__global__ __launch_bounds__(kPartThreads) void top_kernel(TopArgs g) {
  const LogitsArgs& a = g.z;
  const int t = (int)blockIdx.x, y = a.targets ? target_of(a, t) : 0;
  if (y < 0) {
    for (int k = (int)threadIdx.x; k < g.K; k += kPartThreads) {
      g.ids[(int64_t)t * g.K + k] = -1;
      g.tops[(int64_t)t * g.K + k] = -__builtin_huge_valf();
    }
    if (threadIdx.x == 0 && a.logp) a.logp[t] = 0.f;
    if (threadIdx.x == 0 && a.ent) a.ent[t] = 0.f;
    return;
  }
  const T* row = static_cast<const T*>(a.logits) + (int64_t)t * a.stride;
  const Span sp = row_span(row, a.V);
  const int odd = odd_of<T>(sp, a.V);
  const float c = a.inv_temp * kLog2e, ly = load1(row + y);
  Soft x = sum_vectors<T, 4, false>(row + sp.head, 0, sp.vectors, c);
  if (odd >= 0) add1(x, load1(row + odd), c);
  x = group_merge<kPartThreads>(x, c);
  const RowStats r = row_stats(a, x, ly);
  if (threadIdx.x == 0 && a.logp) a.logp[t] = r.lp;
  if (threadIdx.x == 0 && a.ent) a.ent[t] = r.ent;

  __shared__ Best b;
  if (threadIdx.x == 0) b.n = 0, b.bar = 0;
  __syncthreads();
  for (int first = 0; first < a.V; first += kStep * kPartThreads) {
    const int n = b.n;
    __syncthreads();  // read by every thread before one adds to it
    if (n > kRoom - kStep * kPartThreads) keep(b, g.K);
    const uint64_t bar = b.bar;
#pragma unroll
    for (int i = 0; i < kStep; ++i) {
      const int word = first + i * kPartThreads + (int)threadIdx.x;
      if (word < a.V) offer(b, bar, load1(row + word), word);
    }
    __syncthreads();
  }
  keep(b, g.K);
  for (int k = (int)threadIdx.x; k < g.K; k += kPartThreads) {
    const bool some = k < b.n;
    const uint64_t key = b.keys[min(k, kRoom - 1)];
    g.ids[(int64_t)t * g.K + k] = some ? (int)~(uint32_t)key : -1;
    g.tops[(int64_t)t * g.K + k] = some ? (logit_of((uint32_t)(key >> 32)) - x.m) * a.inv_temp - r.log_s : -__builtin_huge_valf();
  }
}

template <typename T>
hipError_t top_for(const TopArgs& a, hipStream_t s) {
  TopArgs args = a;
  void* params[] = {&args};
  return hipLaunchKernel(reinterpret_cast<const void*>(&top_kernel<T>), dim3((unsigned)a.z.T), dim3(kPartThreads), params, 0, s);
}

}  // namespace

hipError_t launch_top_logprobs(const TopArgs& a, hipStream_t s) {
  return a.z.bf16 ? top_for<uint16_t>(a, s) : top_for<float>(a, s);
}

}  // namespace pda
