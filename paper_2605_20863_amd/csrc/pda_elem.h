// Element types and wave helpers of the operators around attention
// (pda_rope.hip, pda_policy.hip, pda_norm.hip, pda_top.hip, pda_distill.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pda {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// By value: a bit cast of a vector's element in place reads the vector's first.
__device__ __forceinline__ float as_f32(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t as_u32(float f) { return __builtin_bit_cast(uint32_t, f); }

// Two floats as bf16 bits in one word (round to nearest even, one instruction).
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const f32x2 x = {lo, hi};
  const bf16x2 y = __builtin_convertvector(x, bf16x2);
  return __builtin_bit_cast(uint32_t, y);
}
__device__ __forceinline__ uint16_t to_bf16(float x) { return (uint16_t)pack_bf16(x, x); }

// Value of the lane that DPP control `ctrl` names (all lanes active).
template <int ctrl>
__device__ __forceinline__ float dpp(float x) {
  return as_f32((uint32_t)__builtin_amdgcn_update_dpp(0, (int)as_u32(x), ctrl, 0xF, 0xF, true));
}
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E;  // quad_perm [1,0,3,2], [2,3,0,1]
constexpr int kDppHalfMirror = 0x141, kDppMirror = 0x140;
constexpr int kDppRor8 = 0x128;  // lane i of a row of 16 takes lane (i + 8) % 16's value

// Sum over the aligned group of N = 8 or 16 lanes, in every lane of it.
template <int N>
__device__ __forceinline__ float group_sum(float x) {
  x += dpp<kDppXor1>(x);
  x += dpp<kDppXor2>(x);
  x += dpp<kDppHalfMirror>(x);
  if constexpr (N == 16) x += dpp<kDppMirror>(x);
  return x;
}

// Their largest.
template <int N>
__device__ __forceinline__ float group_max(float x) {
  x = fmaxf(x, dpp<kDppXor1>(x));
  x = fmaxf(x, dpp<kDppXor2>(x));
  x = fmaxf(x, dpp<kDppHalfMirror>(x));
  if constexpr (N == 16) x = fmaxf(x, dpp<kDppMirror>(x));
  return x;
}

__device__ __forceinline__ float wave_max_f(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o, 64));
  return x;
}

// fp8 (e4m3) scales: the largest code's value, and the smallest scale.
constexpr float kE4M3Max = 448.f;
constexpr float kMinScale = 0x1p-126f;

// Correctly rounded x / s for many x: with y the rounded reciprocal, q = x y and
// the exact remainder r = x - q s, the quotient is q + r y rounded once
// (Markstein). Where the remainder could leave float32's range the division is
// made as such.
struct Div {
  float s, y;
  bool plain;
};
__device__ __forceinline__ Div make_div(float s) { return Div{s, 1.f / s, s < 0x1p-90f || s > 0x1p90f}; }
__device__ __forceinline__ float quotient(float x, const Div& d) {
  if (d.plain) return __fdiv_rn(x, d.s);
  const float q = x * d.y, r = fmaf(-q, d.s, x);
  return r == 0.f ? q : fmaf(r, d.y, q);  // q as it is keeps the sign of a zero
}

// Eight neighbouring elements, as loaded.
template <typename T>
struct Raw;
template <>
struct Raw<uint16_t> {
  u32x4 a;
};
template <>
struct Raw<float> {
  u32x4 a, b;
};
// STREAM: past the caches.
template <bool STREAM, typename T>
__device__ __forceinline__ Raw<T> load8(const void* base, int64_t at) {
  const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const T*>(base) + at);
  Raw<T> r;
  r.a = STREAM ? __builtin_nontemporal_load(p) : *p;
  if constexpr (sizeof(T) == 4) r.b = STREAM ? __builtin_nontemporal_load(p + 1) : p[1];
  return r;
}
__device__ __forceinline__ void unpack(const Raw<uint16_t>& r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = r.a[i];
    x[2 * i] = as_f32(w << 16);
    x[2 * i + 1] = as_f32(w & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void unpack(const Raw<float>& r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t u = r.a[i], w = r.b[i];
    x[i] = as_f32(u);
    x[4 + i] = as_f32(w);
  }
}
template <bool STREAM>
__device__ __forceinline__ void put16(void* p, u32x4 v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, static_cast<u32x4*>(p));
  else *static_cast<u32x4*>(p) = v;
}
template <bool STREAM>
__device__ __forceinline__ void store8(void* base, int64_t at, bool bf16, const float (&y)[8]) {
  u32x4 o[2];
  if (bf16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[0][i] = pack_bf16(y[2 * i], y[2 * i + 1]);
    put16<STREAM>(static_cast<uint16_t*>(base) + at, o[0]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i / 4][i % 4] = as_u32(y[i]);
    float* p = static_cast<float*>(base) + at;
    put16<STREAM>(p, o[0]);
    put16<STREAM>(p + 4, o[1]);
  }
}

}  // namespace pda
