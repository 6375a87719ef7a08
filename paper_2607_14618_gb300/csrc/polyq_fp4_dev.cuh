// The 4-bit floating-point formats on the device: block scales, element codes,
// and where a block's scale lies.  Also host checks shared by the entry points.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "polyq_fp4.h"

namespace polyq {
namespace fp4 {

__host__ __device__ constexpr int block_len(bool nv) { return nv ? 16 : 32; }
// Blocks of a row, and its 512-byte scale atoms (128 rows x 4 blocks).
__host__ __device__ inline int64_t blocks(int64_t K, bool nv) { return (K + block_len(nv) - 1) / block_len(nv); }
__host__ __device__ inline int64_t atoms(int64_t K, bool nv) { return (blocks(K, nv) + 3) / 4; }
// Byte of the scale of block b of row r; A atoms per row group.
__host__ __device__ __forceinline__ size_t scale_off(int64_t r, int64_t b, int64_t A) {
  return (size_t)((r >> 7) * A + (b >> 2)) * 512 + (size_t)((r & 31) * 16 + ((r >> 5) & 3) * 4 + (b & 3));
}

// Two / eight e2m1 codes, nearest even, saturating; the first element in the
// low bits.
__device__ __forceinline__ uint32_t codes8(const float (&v)[8]) {
  uint32_t r;
  asm("{\n .reg .b8 b0, b1, b2, b3;\n"
      " cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
      " cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
      " mov.b32 %0, {b0, b1, b2, b3};\n}\n"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}
// Two values of the codes in a byte (fp16 holds every e2m1 number).
__device__ __forceinline__ float2 values2(uint32_t byte) {
  uint32_t h;
  asm("{\n .reg .b8 b0, b1, b2, b3;\n mov.b32 {b0, b1, b2, b3}, %1;\n cvt.rn.f16x2.e2m1x2 %0, b0;\n}\n"
      : "=r"(h)
      : "r"(byte));
  const __half2 v = *reinterpret_cast<const __half2*>(&h);
  return __half22float2(v);
}
// e4m3 nearest even, saturating, and back.
__device__ __forceinline__ uint32_t to_e4m3(float v) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(v));
  return r & 0xFFu;
}
__device__ __forceinline__ float from_e4m3(uint32_t byte) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)byte));
  return __half2float(__ushort_as_half((uint16_t)(h & 0xFFFFu)));
}
__device__ __forceinline__ float from_e8m0(uint32_t byte) {
  return byte == 0 ? __uint_as_float(0x00400000u) : byte == 255 ? __uint_as_float(0x7FC00000u)
                                                                : __uint_as_float(byte << 23);
}

// a / d for a small integer or e4m3 d, from r = 1 / d to a unit: one residual
// step (Markstein 1990).  Its error, 2^-44, is far less than what a quotient that
// is not on a border of the next rounding (an e2m1 or e4m3 midpoint, at most 5
// significant bits) is away from it: a differs from border * d, which fp32
// holds, by a unit, so the quotient by 2^-31 more than half a unit, and the two
// roundings fall as one rounding of the exact quotient does.
__device__ __forceinline__ float quotient(float a, float d, float r) {
  const float q = a * r;
  return __fmaf_rn(__fmaf_rn(-q, d, a), r, q);
}
__device__ __forceinline__ float rcp_approx(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// A block's scale byte and how its elements are divided by the scale.
template <bool NV>
struct Scale {
  uint32_t byte;
  float s, r;  // NV: the scale and its reciprocal; MX: r = 2^-e
  bool zero;   // codes are 0: a block that is not finite (or, NV, a zero scale)
  // amax: bits of the largest |t|
  __device__ __forceinline__ explicit Scale(uint32_t amax) {
    const bool bad = amax >= 0x7F800000u;
    if (NV) {
      byte = bad ? 0x7Fu : to_e4m3(quotient(__uint_as_float(amax), 6.f, 1.f / 6.f));
      s = from_e4m3(byte);
      zero = bad || byte == 0;
      r = zero ? 0.f : rcp_approx(s);
    } else {
      const int e = (int)(amax >> 23) - 2;  // floor(log2) - 2, biased; at least 2^-127
      byte = bad ? 255u : (uint32_t)max(e, 0);
      zero = bad;
      r = bad ? 0.f : __uint_as_float((254u - byte) << 23);
      s = 0.f;
    }
  }
  // Codes of eight t.  MX: t / scale is exact, a power of two.
  __device__ __forceinline__ uint32_t codes(const float (&t)[8]) const {
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = NV ? quotient(t[i], s, r) : t[i] * r;
    return zero ? 0u : codes8(q);
  }
  // NV, eight elements v = t g of 16-bit types with r_g = 1 / (s g) to two units
  // (g a power of two): t has at most 11 significant bits, so a quotient that is
  // not on a border of two codes is 2^-13 or more from it, and rounding it to
  // a multiple of 2^-16 (the sum with 192) leaves it on its side and puts one that
  // is on the border there.
  __device__ __forceinline__ uint32_t codes_short(const float (&v)[8], float r_g) const {
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = __fadd_rn(__fmaf_rn(v[i], r_g, 192.f), -192.f);
    return zero ? 0u : codes8(q);
  }
};

}  // namespace fp4
}  // namespace polyq

// Checks a 4-bit tensor descriptor (host; `who` names the entry point, `what`
// the argument).
int polyq_check_fp4(const polyq_fp4* t, const char* who, const char* what);
// Checks a dense tensor of rows of `cols` elements.
int polyq_check_dense(const polyq_dense* d, int64_t cols, const char* who, const char* what);
