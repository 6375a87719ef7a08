// Elements of dense tensors (fp32, bf16, fp16) on the device: conversion, and
// eight of a row at a time as they lie in memory.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "polyq_fp4.h"

namespace polyq {

template <typename T>
struct Elem;
template <>
struct Elem<float> {
  static __device__ __forceinline__ float to(float v) { return v; }
  static __device__ __forceinline__ float from(float v) { return v; }
};
template <>
struct Elem<__nv_bfloat16> {
  static __device__ __forceinline__ float to(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ __nv_bfloat16 from(float v) { return __float2bfloat16_rn(v); }
};
template <>
struct Elem<__half> {
  static __device__ __forceinline__ float to(__half v) { return __half2float(v); }
  static __device__ __forceinline__ __half from(float v) { return __float2half_rn(v); }
};

// Two fp32 numbers in one instruction.
using F2 = unsigned long long;
__device__ __forceinline__ F2 f2(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 of(F2 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ float sum2(F2 v) {
  const float2 f = of(v);
  return f.x + f.y;
}

// 8 elements as they lie in memory.
template <typename T>
struct Raw8 {
  uint4 w[sizeof(T) * 8 / 16];
};
template <typename T>
__device__ __forceinline__ void to_float(const Raw8<T>& r, float (&v)[8]) {
  const T* e = reinterpret_cast<const T*>(r.w);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = Elem<T>::to(e[i]);
}

// Element i of an array of any type.
__device__ __forceinline__ float any_load(const void* p, int type, int64_t i) {
  if (type == POLYQ_F32) return __ldcg((const float*)p + i);
  const uint16_t h = __ldcg((const uint16_t*)p + i);
  return type == POLYQ_BF16 ? __uint_as_float((uint32_t)h << 16) : __half2float(__ushort_as_half(h));
}
__device__ __forceinline__ void any_store(void* p, int type, int64_t i, float v) {
  if (type == POLYQ_F32) ((float*)p)[i] = v;
  else if (type == POLYQ_BF16) ((__nv_bfloat16*)p)[i] = Elem<__nv_bfloat16>::from(v);
  else ((__half*)p)[i] = Elem<__half>::from(v);
}

// The 8 elements of a row that a thread holds.  VEC: eight neighbours from `col` on, of rows that
// start on 16 bytes.  Else every `step`-th from `col` on, so that a warp's accesses are of
// neighbours whatever the row starts on.  `mask` has a bit for each of the 8 that exists.
// Loads are ordinary ones through L2: a grid may be on its SM before the one that writes its
// inputs has begun, and the wait on it orders these with those writes.
template <bool VEC>
__device__ __forceinline__ uint32_t mask8(int col, int step, int K) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m |= (uint32_t)(col + i * (VEC ? 1 : step) < K) << i;
  return m;
}
template <bool VEC, typename T>
__device__ __forceinline__ void load8(const T* row, int col, int step, uint32_t mask, Raw8<T>& r) {
  constexpr int N16 = sizeof(T) * 8 / 16;
  if (VEC && mask == 0xFFu) {
#pragma unroll
    for (int i = 0; i < N16; ++i) r.w[i] = __ldcg(reinterpret_cast<const uint4*>(row + col) + i);
  } else {
    alignas(16) T e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      e[i] = mask >> i & 1 ? __ldcg(row + col + i * (VEC ? 1 : step)) : Elem<T>::from(0.f);
#pragma unroll
    for (int i = 0; i < N16; ++i) r.w[i] = reinterpret_cast<const uint4*>(e)[i];
  }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store8(T* row, int col, int step, uint32_t mask, const float (&v)[8]) {
  constexpr int N16 = sizeof(T) * 8 / 16;
  alignas(16) T e[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = Elem<T>::from(v[i]);
  if (VEC && mask == 0xFFu) {
#pragma unroll
    for (int i = 0; i < N16; ++i) reinterpret_cast<uint4*>(row + col)[i] = reinterpret_cast<const uint4*>(e)[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (mask >> i & 1) row[col + i * (VEC ? 1 : step)] = e[i];
  }
}

}  // namespace polyq
