// HIP kernels for the residual stream's root-mean-square norm and its gradient
// on MI355X (gfx950).
//
// For a token's row x [H], weights w, h = x + residual rounded to the stream's type:
//     r = 1 / sqrt(mean h^2 + eps),  y = h w r
// out is y rounded once, or in fp8 y / s with s = max |y| / 448 of a row or of groups
// of neighbours. With g the gradient of y and q that of h from elsewhere:
//     dh = q + r (g w - h r^2 mean(g w h)),  dw = sum over rows of g h r.
//
// Both sums of a row (squares and, of the gradient, g w h; of a row's fp8 scale the
// largest |h w|, which is |y| before r) come from one read of it and one merge; the
// row stays in the registers of its RT threads, N vectors of 8 elements each, until
// it is written. Sums are float32, the weights' gradient over workgroups float64.

#include "pda_elem.h"
#include "pda_lm_internal.h"

namespace pda {
namespace {

// Threads of a workgroup: four rows of a wave each, or one row.
template <int RT>
constexpr int kGroup = RT == 64 ? 256 : RT;

struct Two {
  float a, b;
};

// Sum of x.a and, by MAX, largest or sum of x.b over the 64 lanes, in each of them.
template <bool MAX>
__device__ __forceinline__ Two wave_both(Two x) {
  x.a = group_sum<16>(x.a);
  x.b = MAX ? group_max<16>(x.b) : group_sum<16>(x.b);
#pragma unroll
  for (int o = 16; o < 64; o *= 2) {
    x.a += __shfl_xor(x.a, o, 64);
    const float y = __shfl_xor(x.b, o, 64);
    x.b = MAX ? fmaxf(x.b, y) : x.b + y;
  }
  return x;
}

// The same over a row's RT threads, M of each added up one after another's, so that RT threads' M give the bits of RT M threads' one;
// `turn` alternates between a workgroup's rows, so that one barrier a row does. SELDOM: in few registers rather than quickly, with an array
// of its own.
template <int RT, bool MAX, bool SELDOM = false, int M>
__device__ __forceinline__ Two row_both(Two (&x)[M], int turn) {
#pragma unroll
  for (int m = 0; m < M; ++m) x[m] = wave_both<MAX>(x[m]);
  const auto join = [](Two& a, const Two& b) {
    a.a += b.a;
    a.b = MAX ? fmaxf(a.b, b.b) : a.b + b.b;
  };
  Two all = x[0];
  if constexpr (RT > 64) {
    constexpr int W = RT / 64;
    __shared__ Two parts[2][M][W];
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int m = 0; m < M; ++m) parts[turn & 1][m][threadIdx.x / 64] = x[m];
    }
    __syncthreads();
    all = parts[turn & 1][0][0];
    // up to 16 in registers at once; of the 32 of 1,024 threads' two sums 8, so that two such rows' waves fit beside each other (2,048 x 16,384
    // bf16 into fp8 63 us with all of them, 48 so)
    constexpr int S = SELDOM ? 1 : M * W > 16 ? 8 : M * W;
    const Two* p = &parts[turn & 1][0][0];
#pragma unroll
    for (int i = 1; i < S; ++i) join(all, p[i]);
#pragma unroll 1
    for (int j = S; j < M * W; j += S)
#pragma unroll
      for (int i = 0; i < S; ++i) join(all, p[j + i]);
  } else {
#pragma unroll
    for (int m = 1; m < M; ++m) join(all, x[m]);
  }
  return all;
}

__device__ __forceinline__ void load_weight(const void* w, bool bf16, int at, float (&y)[8]) {
  if (bf16) unpack(load8<false, uint16_t>(w, at), y);
  else unpack(load8<false, float>(w, at), y);
}
// The same in two steps, so that what is loaded may be on its way.
struct RawWeight {
  Raw<uint16_t> half;
  Raw<float> full;
};
__device__ __forceinline__ void ask_weight(const void* w, bool bf16, int at, RawWeight& y) {
  if (bf16) y.half = load8<false, uint16_t>(w, at);
  else y.full = load8<false, float>(w, at);
}
__device__ __forceinline__ void have_weight(const RawWeight& w, bool bf16, float (&y)[8]) {
  if (bf16) unpack(w.half, y);
  else unpack(w.full, y);
}

// Makes the compiler unpack the elements again after this point, rather than keep them in registers of their own.
__device__ __forceinline__ void again(Raw<uint16_t>& x) { asm volatile("" : "+v"(x.a)); }
__device__ __forceinline__ void again(Raw<float>& x) { asm volatile("" : "+v"(x.a), "+v"(x.b)); }

// h = x + residual in the stream's type, as kept.
__device__ __forceinline__ void add_rounded(Raw<uint16_t>& x, const Raw<uint16_t>& r) {
  float a[8], b[8];
  unpack(x, a);
  unpack(r, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) x.a[i] = pack_bf16(a[2 * i] + b[2 * i], a[2 * i + 1] + b[2 * i + 1]);
}
__device__ __forceinline__ void add_rounded(Raw<float>& x, const Raw<float>& r) {
  float a[8], b[8];
  unpack(x, a);
  unpack(r, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x.a[i] = as_u32(a[i] + b[i]);
    x.b[i] = as_u32(a[4 + i] + b[4 + i]);
  }
}
// x times s, a power of two: exact but for what falls below the type's smallest numbers.
__device__ __forceinline__ void scale_raw(Raw<uint16_t>& x, float s) {
  float a[8];
  unpack(x, a);
#pragma unroll
  for (int i = 0; i < 4; ++i) x.a[i] = pack_bf16(a[2 * i] * s, a[2 * i + 1] * s);
}
__device__ __forceinline__ void scale_raw(Raw<float>& x, float s) {
  float a[8];
  unpack(x, a);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x.a[i] = as_u32(a[i] * s);
    x.b[i] = as_u32(a[4 + i] * s);
  }
}
template <bool STREAM>
__device__ __forceinline__ void store_raw(void* base, int64_t at, const Raw<uint16_t>& x) {
  put16<STREAM>(static_cast<uint16_t*>(base) + at, x.a);
}
template <bool STREAM>
__device__ __forceinline__ void store_raw(void* base, int64_t at, const Raw<float>& x) {
  float* p = static_cast<float*>(base) + at;
  put16<STREAM>(p, x.a);
  put16<STREAM>(p + 4, x.b);
}

// Codes of y / s; NaN stays NaN (a clamp by min and max would make a number of it), of either sign 0x7f.
__device__ __forceinline__ uint32_t encode4(const float* y, const Div& d) {
  float z[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    z[i] = quotient(y[i], d);
    z[i] = z[i] > kE4M3Max ? kE4M3Max : z[i] < -kE4M3Max ? -kE4M3Max : z[i];
  }
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(z[0], z[1], 0, false);
  const uint32_t codes = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(z[2], z[3], lo, true);
  return codes & ~(((codes & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u);  // the sign of a byte whose other bits are all ones
}
__device__ __forceinline__ float scale_of(float amax) { return fmaxf(__fdiv_rn(amax, kE4M3Max), kMinScale); }

__device__ __forceinline__ float inv_rms(float squares, const NormArgs& a) { return 1.f / sqrtf(squares / (float)a.H + a.eps); }

// A row whose squares sum past float32, where their mean need not: its sums are made again of the row times kDown, all of whose squares'
// sums float32 holds, and whose 1 / rms follows from them; 0 where the mean itself passes float32.
constexpr float kDown = 0x1p-72f;
__device__ __forceinline__ float inv_rms_down(float squares, const NormArgs& a) {
  const float mean = squares / (float)a.H + a.eps * kDown * kDown;
  return mean < 0x1p-16f ? 1.f / sqrtf(mean) : 0.f;  // 2^128 kDown^2
}

// Bound by its bytes where rows are many: 16,384 x 4,096 bf16 with residual 88 us, 6.1 TB/s (a copy of 256 MiB 5.3); 512 x 8,192 into fp8
// 8.8 us and 3 x 4,096 4, of which a launch with one load and one store takes most; 2,048 x 16,384 into fp8 47, 5.0 TB/s.
template <typename T, int RT, int N, bool FP8, bool STREAM>
__global__ __launch_bounds__(kGroup<RT>) void norm_kernel(NormArgs a) {
  constexpr int ROWS = kGroup<RT> / RT;
  const int t = (int)blockIdx.x * ROWS + (int)threadIdx.x / RT, lane = (int)threadIdx.x % RT, vecs = a.H / 8;
  if (t >= a.T) return;  // whole waves, and only where a row is one wave's
  Raw<T> x[N] = {}, r[N] = {};
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int i = lane + n * RT;
    if (i >= vecs) continue;
    x[n] = load8<STREAM, T>(a.x, t * a.x_stride + 8 * i);
    if (a.res) r[n] = load8<STREAM, T>(a.res, t * a.res_stride + 8 * i);
  }
  // Weights are asked for before the sum is stored, since a wait for a later load is one for the stores too (us per call, bf16, later /
  // before: 16,384 x 4,096 into fp8 of 128 85.2 / 81.4, 4,096 x 8,192 into fp8 48.1 / 45.7, 2,048 x 4,096 11.9 / 11.5, 32,768 x 1,024
  // 47.8 / 47.2; 512 x 4,096 5.1 / 5.5).
  constexpr bool EARLY = N == 2 || (N == 1 && (FP8 || RT < 512));
  RawWeight held[EARLY ? N : 1] = {};
  if constexpr (EARLY) {
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (lane + n * RT < vecs) ask_weight(a.w, a.w_bf16, 8 * (lane + n * RT), held[n]);
  }
  const auto weights = [&](int n, float (&w)[8]) {
    if constexpr (EARLY) have_weight(held[n], a.w_bf16, w);
    else load_weight(a.w, a.w_bf16, 8 * (lane + n * RT), w);
  };
  // up to 2 sums of a thread, for which the calls of few rows have a thread each: a row's results are the same in both
  constexpr int M = N <= 2 ? N : 1;
  Two sums[M] = {};
  const auto add_squares = [&](int n, Two& s) {
    float h[8];
    unpack(x[n], h);
    float q = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) q = fmaf(h[e], h[e], q);
    s.a += q;
    if (FP8 && !a.group) {
      float w[8];
      weights(n, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) s.b = fmaxf(s.b, fabsf(h[e] * w[e]));
    }
  };
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int i = lane + n * RT;
    if (i >= vecs) continue;
    Two& s = sums[n % M];
    if (a.res) {
      add_rounded(x[n], r[n]);
      if (a.sum) store_raw<STREAM>(a.sum, t * a.sum_stride + 8 * i, x[n]);
    }
    add_squares(n, s);
  }
  Two s = row_both<RT, true>(sums, 0);
  float rms = inv_rms(s.a, a);
  if (__builtin_expect(s.a == __builtin_huge_valf(), 0)) {  // all of a row's threads
    Two anew[M] = {};
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if (lane + n * RT >= vecs) continue;
      scale_raw(x[n], kDown);
      add_squares(n, anew[n % M]);
    }
    s = row_both<RT, true, true>(anew, 0);
    rms = inv_rms_down(s.a, a);
  }
  if (FP8 && !a.group) {
    s.b = scale_of(s.b * rms);
    if (lane == 0) a.scales[t] = s.b;
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int i = lane + n * RT;
    if (!FP8 && i >= vecs) continue;  // an fp8 group's lanes stay together
    float h[8], w[8] = {};
    unpack(x[n], h);
    if (i < vecs) weights(n, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = h[e] * w[e] * rms;
    if constexpr (FP8) {
      float scale = s.b;
      if (a.group) {
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(h[e]));
        scale = scale_of(a.group == 64 ? group_max<8>(m) : group_max<16>(m));
      }
      if (i >= vecs) continue;
      if (a.group && 8 * i % a.group == 0) a.scales[(int64_t)t * (a.H / a.group) + 8 * i / a.group] = scale;
      const Div d = make_div(scale);
      const u32x2 codes = {encode4(h, d), encode4(h + 4, d)};
      u32x2* p = reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.out) + t * a.out_stride + 8 * i);
      if constexpr (STREAM) __builtin_nontemporal_store(codes, p);
      else *p = codes;
    } else {
      store8<STREAM>(a.out, t * a.out_stride + 8 * i, a.type == OutType::BF16, h);
    }
  }
}

// Every workgroup takes rows in turn and keeps their part of the weights' gradient
// in registers. 16,384 x 4,096 bf16 92 us, 5.8 TB/s, of which the parts' sums take 5; a row's loads ahead of the row before's sums
// were slower (119 us where 110 without).
template <typename T, int RT, int N, bool STREAM>
__global__ __launch_bounds__(kGroup<RT>) void norm_backward_kernel(NormArgs a) {
  constexpr int ROWS = kGroup<RT> / RT;
  const int sub = (int)threadIdx.x / RT, lane = (int)threadIdx.x % RT, vecs = a.H / 8;
  float acc[N][8] = {}, held[N][8] = {};
  const auto load_weights = [&](int n, float (&w)[8]) {
    const int i = lane + n * RT;
    if (i < vecs) load_weight(a.w, a.w_bf16, 8 * i, w);
  };
  // Each thread's weights stay in registers where four waves a SIMD still fit, since a row's would be waited for twice (us per call,
  // bf16, loaded for each row / held: 16,384 x 4,096 110 / 94, 8,192 x 4,096 58.5 / 51.0, 2,000 x 16,384 67.3 / 62.8, 32,768 x 1,024
  // 54 / 52, 16,384 x 8,192 202 / 182, 4,096 x 8,192 63.5 / 57.0, 512 x 8,192 19.6 / 18.7).
  constexpr bool HOLD = N <= 2;
  if constexpr (HOLD) {
#pragma unroll
    for (int n = 0; n < N; ++n) load_weights(n, held[n]);
  }
  const auto weights = [&](int n, float (&w)[8]) {
    if constexpr (HOLD) {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = held[n][e];
    } else {
      load_weights(n, w);
    }
  };
  // of the longest rows grad_residual is loaded as it is used: beside the rest of the row it has no registers, and spills cost more (1,000 x
  // 32,768 f32 184 us, so 160 with 112 bytes of scratch left, bf16 none; 2,000 x 16,384 f32 117 / 114)
  constexpr bool LATE = N == 4 || (RT == 1024 && sizeof(T) == 4);
  int turn = 0;
  for (int t = (int)blockIdx.x * ROWS + sub; t < a.T; t += a.wgs * ROWS, ++turn) {
    Raw<T> x[N] = {}, g[N] = {}, q[LATE ? 1 : N] = {};
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = lane + n * RT;
      if (i >= vecs) continue;
      x[n] = load8<STREAM, T>(a.x, t * a.x_stride + 8 * i);
      g[n] = load8<STREAM, T>(a.out, t * a.out_stride + 8 * i);
      if (!LATE && a.res) q[LATE ? 0 : n] = load8<STREAM, T>(a.res, t * a.res_stride + 8 * i);
    }
    const auto sum_row = [&](float scale, Two (&sums)[1]) {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int i = lane + n * RT;
        if (i >= vecs) continue;
        float h[8], y[8], w[8];
        unpack(x[n], h);
        unpack(g[n], y);
        weights(n, w);
        float b = 0.f, c = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          h[e] *= scale;
          b = fmaf(h[e], h[e], b);
          c = fmaf(y[e] * w[e], h[e], c);
        }
        sums[0].a += b;
        sums[0].b += c;
      }
    };
    Two sums[1] = {};
    sum_row(1.f, sums);
    Two s = row_both<RT, false>(sums, turn);
    float rms = inv_rms(s.a, a), back = s.b / (float)a.H * rms * rms;
    if (__builtin_expect(s.a == __builtin_huge_valf(), 0)) {  // all of a row's threads
#pragma unroll
      for (int n = 0; n < N && N > 1; ++n) {
        again(x[n]);
        again(g[n]);
      }
      sums[0] = {};
      sum_row(kDown, sums);
      s = row_both<RT, false, true>(sums, 0);  // (a barrier lies between two rows' of these)
      rms = inv_rms_down(s.a, a);
      back = s.b / (float)a.H * rms * rms * kDown;
      rms *= kDown;
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = lane + n * RT;
      if (i >= vecs) continue;
      float h[8], y[8], w[8], o[8];
      unpack(x[n], h);
      unpack(g[n], y);
      weights(n, w);
      if (LATE && a.res) q[0] = load8<STREAM, T>(a.res, t * a.res_stride + 8 * i);
      unpack(q[LATE ? 0 : n], o);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        acc[n][e] = fmaf(y[e], h[e] * rms, acc[n][e]);
        o[e] = fmaf(rms, fmaf(-h[e], back, y[e] * w[e]), o[e]);
      }
      store8<STREAM>(a.sum, t * a.sum_stride + 8 * i, a.bf16, o);
    }
  }
  if (!a.dw) return;
  // waves of one row each: their parts to the first one's
  if constexpr (ROWS > 1) {
    __shared__ float sums[ROWS - 1][N][8][RT];
    if (sub > 0) {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[sub - 1][n][e][lane] = acc[n][e];
    }
    __syncthreads();
    if (sub > 0) return;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int r = 0; r < ROWS - 1; ++r) acc[n][e] += sums[r][n][e][lane];
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int i = lane + n * RT;
    if (i < vecs) store8<false>(a.dw_part, (int64_t)blockIdx.x * a.H + 8 * i, false, acc[n]);
  }
}

// Sums the workgroups' parts in a fixed order: a workgroup per 16 weights, a row of
// parts for each 16 of its threads, four loads of a thread in flight.
constexpr int kSumRows = 64;
__global__ __launch_bounds__(16 * kSumRows) void norm_weight_grad_kernel(NormArgs a) {
  __shared__ double sums[kSumRows][16];
  const int i = (int)threadIdx.x % 16, r = (int)threadIdx.x / 16, at = (int)blockIdx.x * 16 + i;
  const float* part = a.dw_part + min(at, a.H - 1);
  double x = 0.;
  int g = r;
  for (; g + 3 * kSumRows < a.wgs; g += 4 * kSumRows) {
    float v[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) v[n] = part[(int64_t)(g + n * kSumRows) * a.H];
    x += ((double)v[0] + (double)v[1]) + ((double)v[2] + (double)v[3]);
  }
  for (; g < a.wgs; g += kSumRows) x += (double)part[(int64_t)g * a.H];
  sums[r][i] = x;
  __syncthreads();
  for (int n = kSumRows / 2; n > 0; n /= 2) {
    if (r < n) sums[r][i] += sums[r + n][i];
    __syncthreads();
  }
  if (r == 0 && at < a.H) a.dw[at] = (float)sums[0][i];
}

// ------------------------------------------------------------- launches

template <typename K>
hipError_t launch(K kernel, int64_t wgs, int threads, const NormArgs& a, hipStream_t s) {
  NormArgs args = a;
  void* params[] = {&args};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((unsigned)wgs), dim3((unsigned)threads), params, 0, s);
}

// Whether the call loads and stores past the caches: from 2^28 bytes on (4 arrays of the stream's type), bf16 alone (a lane's 8 f32
// elements are two loads of half a cache line's pieces: 16,384 x 2,048 f32 gradient 102 us through, 113 past them). us through
// them / past them, alone and between the copy that makes x and a product that reads the result (by 1,024 columns):
//   tokens x width    16,384 x 4,096         8,192 x 4,096         32,768 x 1,024        4,096 x 8,192         2,048 x 16,384        6,144 x 4,096
//   norm        95.4 / 89.3, 248 / 241  40.1 / 44.6, 139 / 126 39.5 / 43.8, 131 / 125 40.9 / 44.8, 155 / 137 42.4 / 46.2, 210 / 175 30.1 / 33.4, 101 / 101
//   gradient  102.3 / 92.2, 261 / 238  46.3 / 50.8, 135 / 133 46.6 / 49.6, 137 / 137 58.5 / 63.2, 165 / 160 56.2 / 59.6, 216 / 191 35.5 / 40.0, 102 / 107
constexpr int64_t kStreamBytes = 1 << 28;

template <typename T>
bool streamed(const NormArgs& a) {
  return sizeof(T) == 2 && (int64_t)a.T * a.H * 2 * 4 >= kStreamBytes;
}

template <typename T, bool FP8, int RT, int N>
hipError_t norm_rows(const NormArgs& a, hipStream_t s) {
  constexpr int rows = kGroup<RT> / RT;
  const int64_t wgs = ((int64_t)a.T + rows - 1) / rows;
  if constexpr (sizeof(T) == 2 && !(N == 1 && RT >= 512))  // few rows' threads: below kStreamBytes
    if (streamed<T>(a)) return launch(&norm_kernel<T, RT, N, FP8, true>, wgs, kGroup<RT>, a, s);
  return launch(&norm_kernel<T, RT, N, FP8, false>, wgs, kGroup<RT>, a, s);
}

// Few rows take twice as many threads each (us per call, bf16, half / all of them: 3 x 4,096 5.2 / 4.3, 64 x 8,192 5.8 / 5.0, 512 x 8,192
// 10.6 / 10.0, 512 x 4,096 4.8 / 4.6; 2,048 x 4,096 12.0 / 13.0, 16,384 x 8,192 184 / 188).
constexpr int kFewRows = 1024;
static_assert((int64_t)kFewRows * kLongWidth * 8 < kStreamBytes, "few rows of one vector a thread are never streamed");

template <typename T, bool FP8>
hipError_t norm_for(const NormArgs& a, hipStream_t s) {
  const int v = a.H / 8;
  const bool few = a.T < kFewRows;
  return v <= 64 ? norm_rows<T, FP8, 64, 1>(a, s)
         : v <= 128 ? norm_rows<T, FP8, 128, 1>(a, s)
         : v <= 256 ? norm_rows<T, FP8, 128, 2>(a, s)
         : v <= 512 ? (few ? norm_rows<T, FP8, 512, 1>(a, s) : norm_rows<T, FP8, 256, 2>(a, s))
         : v <= kLongWidth / 8 ? (few ? norm_rows<T, FP8, 1024, 1>(a, s) : norm_rows<T, FP8, 512, 2>(a, s))
         : v <= 2048 ? norm_rows<T, FP8, 1024, 2>(a, s) : norm_rows<T, FP8, 1024, 4>(a, s);
}

template <typename T, int RT, int N>
hipError_t backward_rows(NormArgs a, hipStream_t s, int most) {
  constexpr int rows = kGroup<RT> / RT;
  const int64_t wgs = ((int64_t)a.T + rows - 1) / rows;
  if (a.wgs > most) a.wgs = most;
  if (wgs < a.wgs) a.wgs = (int32_t)wgs;
  hipError_t e = hipSuccess;
  if constexpr (sizeof(T) == 2) {
    if (streamed<T>(a)) e = launch(&norm_backward_kernel<T, RT, N, true>, a.wgs, kGroup<RT>, a, s);
    else if (a.wgs) e = launch(&norm_backward_kernel<T, RT, N, false>, a.wgs, kGroup<RT>, a, s);
  } else {
    if (a.wgs) e = launch(&norm_backward_kernel<T, RT, N, false>, a.wgs, kGroup<RT>, a, s);
  }
  if (e != hipSuccess || !a.dw) return e;
  return launch(&norm_weight_grad_kernel, (a.H + 15) / 16, 16 * kSumRows, a, s);
}

// A workgroup's part of the weights' gradient is as long as a row, written and read again: of long rows there are fewer workgroups,
// with more threads. us per call of 256 / 512 / 1,024 of them: 16,384 x 4,096 bf16 152 / 111 / 110 (a row by 256 threads), 8,192 x
// 8,192 121 / 114 / 120, 2,048 x 4,096 24 / 22 / 23, 2,000 x 16,384 73 / 81 / 95, 32,768 x 1,024 (a wave a row) 86 / 70 / 57; of 512 and
// a row by 512 threads 16,384 x 4,096 104 where 256 took 113, 2,048 x 4,096 20.4.
template <typename T>
hipError_t backward_for(const NormArgs& a, hipStream_t s) {
  const int v = a.H / 8;
  return v <= 64 ? backward_rows<T, 64, 1>(a, s, 1024)
         : v <= 128 ? backward_rows<T, 64, 2>(a, s, 1024)
         : v <= 256 ? backward_rows<T, 256, 1>(a, s, 512)
         : v <= 512 ? backward_rows<T, 512, 1>(a, s, 512)
         : v <= 1024 ? backward_rows<T, 512, 2>(a, s, 512)
         : v <= 2048 ? backward_rows<T, 1024, 2>(a, s, 256) : backward_rows<T, 1024, 4>(a, s, 256);
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  if (a.type == OutType::FP8) return a.bf16 ? norm_for<uint16_t, true>(a, s) : norm_for<float, true>(a, s);
  return a.bf16 ? norm_for<uint16_t, false>(a, s) : norm_for<float, false>(a, s);
}

hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s) {
  return a.bf16 ? backward_for<uint16_t>(a, s) : backward_for<float>(a, s);
}

}  // namespace pda
