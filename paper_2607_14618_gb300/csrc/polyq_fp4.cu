// Microscaled 4-bit floating point: quantisation and its inverse.
//
//   MX  s = 2^(floor(log2 max|x|) - 2) per 32 elements,  q = e2m1(x / s)
//   NV  s = e4m3(max|x/g| / 6) per 16 elements,          q = e2m1(x / g / s)
//
// A lane holds 8 consecutive elements of a row, so a warp takes 256 elements:
// a block is four (MX) or two (NV) neighbouring lanes, its maximum two or one
// shuffles, and the 8 codes of a lane one 4-byte store (a warp stores 128
// consecutive bytes).  Bound by HBM for large tensors and by the launch for a
// token's.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "polyq_dev.cuh"
#include "polyq_fp4_dev.cuh"
#include "polyq_internal.h"

namespace {

using namespace polyq;

constexpr int kWarps = 4;  // of a CTA, side by side along a row: 1024 elements

struct QuantParams {
  const void* x;
  void* y;
  uint8_t* codes;
  uint8_t* scales;
  int64_t x_stride, y_stride, code_stride, rows, K, A;
  int64_t row_groups;     // of as many rows as a warp takes together
  float g, inv_g;         // tensor scale; its reciprocal where that is exact, else 0
  int mid_g;              // no product of it with a block scale leaves fp32's normal range
  float up;               // see scaled_to_odd
};

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

// 8 elements from k on as they lie in memory, and as floats; zeros past K.  VEC:
// rows start on 16 bytes.  (Two steps, so that the loads of several rows are in
// flight before the first is converted: 13824 x 5120 bf16 63 us with one.)
// Inputs are read once, through L2, by ordinary loads: a grid may be on its SM
// before the one that writes them has begun, and the grid dependency's wait orders
// these with those writes, but not loads through the read-only path.
template <typename T>
struct Raw8 {
  uint4 w[sizeof(T) * 8 / 16];
};
template <typename T, bool FULL>
__device__ __forceinline__ void load8(const T* __restrict__ row, int64_t k, int64_t K, Raw8<T>& r) {
  constexpr int N16 = sizeof(T) * 8 / 16;
  if (FULL || k + 8 <= K) {
#pragma unroll
    for (int i = 0; i < N16; ++i) r.w[i] = __ldcg(reinterpret_cast<const uint4*>(row + k) + i);
  } else {
    alignas(16) T e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = k + i < K ? __ldcg(row + k + i) : Elem<T>::from(0.f);
#pragma unroll
    for (int i = 0; i < N16; ++i) r.w[i] = reinterpret_cast<const uint4*>(e)[i];
  }
}
// The same for a row that starts anywhere: the warp's 256 elements in eight
// loads of 32 neighbours (strided_load), which go through shared memory to the
// lanes that hold eight in a row (strided_turn).  777 x 5003 fp16, both calls:
// 17.7 us with eight loads and stores per lane, two bytes every 16, 10.5 so.
template <typename T>
__device__ __forceinline__ void strided_load(const T* __restrict__ row, int64_t k0, int64_t K, T (&e)[8]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = k0 + 32 * i + lane < K ? __ldcg(row + k0 + 32 * i + lane) : Elem<T>::from(0.f);
}
template <typename T>
__device__ __forceinline__ void strided_turn(const T (&e)[8], T* buf, Raw8<T>& r) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < 8; ++i) buf[32 * i + lane] = e[i];
  __syncwarp();
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) * 8 / 16); ++i) r.w[i] = reinterpret_cast<const uint4*>(buf + 8 * lane)[i];
  __syncwarp();
}

// Bits of the largest |element| as a float's (NaN above infinity).
__device__ __forceinline__ uint32_t abs_max(const Raw8<float>& r) {
  const uint32_t* e = reinterpret_cast<const uint32_t*>(r.w);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, e[i] & 0x7FFFFFFFu);
  return m;
}
template <typename T>
__device__ __forceinline__ uint32_t abs_max(const Raw8<T>& r) {
  const uint32_t* e = reinterpret_cast<const uint32_t*>(r.w);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = __vmaxu2(m, e[i] & 0x7FFF7FFFu);
  const uint16_t h = (uint16_t)max(m & 0xFFFFu, m >> 16);
  return __float_as_uint(Elem<T>::to(*reinterpret_cast<const T*>(&h))) & 0x7FFFFFFFu;
}
template <typename T>
__device__ __forceinline__ void to_float(const Raw8<T>& r, float (&v)[8]) {
  const T* e = reinterpret_cast<const T*>(r.w);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = Elem<T>::to(e[i]);
}

// A CTA takes 1024 elements of ROWS consecutive rows, a warp 256, the loads of
// its rows in flight together.  FULL: all of a warp's elements exist (the
// checks took a third of the instructions, which bound 16-bit inputs: 13824 x
// 5120 bf16 MX 34 us with them, 29.5 without, 6.1 TB/s).  A flat index of
// (rows, chunk) pairs needs two 64-bit divisions a warp: 55 us.
template <typename T, bool NV, bool VEC, int ROWS, bool FULL>
__device__ __forceinline__ void quantize_rows(const QuantParams& P, int64_t r0, int64_t k, T* buf) {
  constexpr int LPB = NV ? 2 : 4;  // lanes of a block
  const int64_t b = k / (8 * LPB);
  const int n = FULL ? ROWS : (int)min((int64_t)ROWS, P.rows - r0);
  const bool scale = threadIdx.x % LPB == 0 && (FULL || (b >> 2) < P.A), code = FULL || k < P.K;
  Raw8<T> raw[ROWS];
  const T* x = (const T*)P.x + r0 * P.x_stride;
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {  // (a row past the last: the last one again, not stored)
      load8<T, FULL>(x, k, P.K, raw[i]);
      if (FULL || i + 1 < n) x += P.x_stride;
    }
  } else {
    T e[ROWS][8];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      strided_load(x, k - threadIdx.x % 32 * 8, P.K, e[i]);
      if (FULL || i + 1 < n) x += P.x_stride;
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) strided_turn(e[i], buf, raw[i]);
  }
  // ROWS consecutive rows from a multiple of ROWS lie in one group of 32: 16 bytes apart
  uint8_t* sp = P.scales + fp4::scale_off(r0, b, P.A);
  uint8_t* cp = P.codes + r0 * P.code_stride + k / 2;
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    if (!FULL && i >= n) break;  // the same for the whole warp
    uint32_t m = abs_max(raw[i]);
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    if (!NV) m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    float v[8];
    to_float(raw[i], v);
    // NV: dividing by the tensor scale keeps the order, the largest stays the largest
    if (NV) m = __float_as_uint(P.inv_g != 0.f ? __uint_as_float(m) * P.inv_g : __fdiv_rn(__uint_as_float(m), P.g));
    const fp4::Scale<NV> sc(m);
    uint32_t c;
    if (NV && sizeof(T) == 2 && P.inv_g != 0.f && P.mid_g) {
      c = sc.codes_short(v, sc.r * P.inv_g);
    } else {
      if (NV) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = P.inv_g != 0.f ? v[j] * P.inv_g : __fdiv_rn(v[j], P.g);
      }
      c = sc.codes(v);
    }
    if (code) *reinterpret_cast<uint32_t*>(cp) = c;
    if (scale) sp[16 * i] = (uint8_t)sc.byte;
    cp += P.code_stride;
  }
}
template <typename T, bool NV, bool VEC, int ROWS>
__global__ void __launch_bounds__(32 * kWarps) quantize_kernel(const __grid_constant__ QuantParams P) {
  const int64_t k = (int64_t)blockIdx.x * (256 * kWarps) + threadIdx.x * 8;
  const bool cols = k - threadIdx.x % 32 * 8 + 256 <= P.K;
  __shared__ __align__(16) T turn[VEC ? 1 : kWarps][VEC ? 8 : 256];
  T* buf = turn[VEC ? 0 : threadIdx.x / 32];
  pdl_trigger();
  pdl_wait();
  for (int64_t rg = blockIdx.y; rg < P.row_groups; rg += gridDim.y) {
    if (cols && (rg + 1) * ROWS <= P.rows) quantize_rows<T, NV, VEC, ROWS, true>(P, rg * ROWS, k, buf);
    else quantize_rows<T, NV, VEC, ROWS, false>(P, rg * ROWS, k, buf);
  }
}

// v g in fp32, rounded to odd: what fp32 does not hold of the product is kept in
// the last bit, so that rounding to a 16-bit type, two or more bits shorter,
// falls as one rounding of the product would (Boldo and Melquiond: Emulation of a
// FMA and correctly rounded sums, 2008).  v has at most six significant bits and
// is 2^-10 or more.  The remainder's sign is all that counts: `up` (2^40 for a g
// below 1, where v g < 2^12) keeps a subnormal product's from vanishing.
__device__ __forceinline__ float scaled_to_odd(float v, float g, float up) {
  const float p = v * g, rest = __fmaf_rn(v * up, g, -(p * up));
  int b = __float_as_int(p);
  if (rest != 0.f) b = (b - ((b ^ __float_as_int(rest)) < 0)) | 1;
  return __int_as_float(b);
}
// Codes of a block whose tensor scale g is not a power of two, as 16-bit values.
// The block's eight magnitudes are rounded once each and looked up by byte
// permutes.  They are 1 or 1.5 times a power of two, so two products rounded to
// odd serve all of them where no power of two leaves fp32's normal range (g from
// 2^-100 to 2^100).  13824 x 5120 to bf16: 36.9 us with these two chosen from and
// multiplied for each element, 33.1 us so, 30.5 us for a power of two.
template <typename T>
struct Magnitudes {
  uint32_t lo[2], hi[2];  // low and high bytes in the order of the codes
  __device__ __forceinline__ Magnitudes(float s, const QuantParams& P) {
    alignas(16) T m[8];
    if (P.mid_g) {
      const float one = scaled_to_odd(s, P.g, 1.f), more = scaled_to_odd(1.5f * s, P.g, 1.f);
      m[0] = Elem<T>::from(0.f * one);  // (a NaN of a block's NaN scale)
      m[1] = Elem<T>::from(0.5f * one);
#pragma unroll
      for (int i = 1; i < 4; ++i) {
        m[2 * i] = Elem<T>::from((float)(1 << (i - 1)) * one);
        m[2 * i + 1] = Elem<T>::from((float)(1 << (i - 1)) * more);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = i < 2 ? 0.5f * i : (float)(1 << (i / 2 - 1)) * (i % 2 ? 1.5f : 1.f);
        m[i] = Elem<T>::from(scaled_to_odd(v * s, P.g, P.up));
      }
    }
    const uint32_t* w = reinterpret_cast<const uint32_t*>(m);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      lo[i] = __byte_perm(w[2 * i], w[2 * i + 1], 0x6420);
      hi[i] = __byte_perm(w[2 * i], w[2 * i + 1], 0x7531);
    }
  }
  __device__ __forceinline__ void of(uint32_t codes, uint32_t (&out)[4]) const {
    const uint32_t odd = codes, even = codes << 4;  // byte i's top bit: sign of element 2 i + 1, of 2 i
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t at = (codes & 0x77777777u) >> (16 * i);
      const uint32_t l = __byte_perm(lo[0], lo[1], at), h = __byte_perm(hi[0], hi[1], at);
      out[2 * i] = __byte_perm(l, h, 0x5140) | (__byte_perm(even, odd, i ? 0x6020 : 0x4000) & 0x80008000u);
      out[2 * i + 1] = __byte_perm(l, h, 0x7362) | (__byte_perm(even, odd, i ? 0x7030 : 0x5010) & 0x80008000u);
    }
  }
};

template <typename T, bool NV, bool VEC, int ROWS>
__global__ void __launch_bounds__(32 * kWarps) dequantize_kernel(const __grid_constant__ QuantParams P) {
  const int64_t k = (int64_t)blockIdx.x * (256 * kWarps) + threadIdx.x * 8, b = k / fp4::block_len(NV);
  const int64_t k0 = k - threadIdx.x % 32 * 8;
  __shared__ __align__(16) T turn[VEC ? 1 : kWarps][VEC ? 8 : 256];
  T* buf = turn[VEC ? 0 : threadIdx.x / 32];
  pdl_trigger();
  pdl_wait();
  if (k0 >= P.K) return;  // the whole warp
  const bool in = k < P.K;
  for (int64_t rg = blockIdx.y; rg < P.row_groups; rg += gridDim.y) {
    const int64_t r0 = rg * ROWS;
    const uint8_t* sp = P.scales + fp4::scale_off(r0, b, P.A);
    const uint8_t* cp = P.codes + r0 * P.code_stride + k / 2;
    uint32_t c[ROWS], sb[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const int at = (int)min((int64_t)i, P.rows - 1 - r0);  // (past the last row: the last one again)
      c[i] = in ? __ldcg(reinterpret_cast<const uint32_t*>(cp + at * P.code_stride)) : 0u;  // (rows are padded)
      sb[i] = in ? __ldcg(sp + 16 * at) : 0u;
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      if (r0 + i >= P.rows) break;
      const float s = NV ? fp4::from_e4m3(sb[i]) : fp4::from_e8m0(sb[i]);
      alignas(16) T out[8];
      if (NV && sizeof(T) == 2 && P.inv_g == 0.f) {
        if constexpr (sizeof(T) == 2) {
          uint32_t w[4];
          Magnitudes<T>(s, P).of(c[i], w);
          *reinterpret_cast<uint4*>(out) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      } else {  // v s is exact, and v s g for a power of two
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 v = fp4::values2(c[i] >> (8 * j) & 0xFFu);
          out[2 * j] = Elem<T>::from(v.x * s * P.g);
          out[2 * j + 1] = Elem<T>::from(v.y * s * P.g);
        }
      }
      T* y = (T*)P.y + (r0 + i) * P.y_stride;
      if constexpr (VEC) {
        if (k + 8 <= P.K) {
#pragma unroll
          for (int j = 0; j < (int)(sizeof(T) * 8 / 16); ++j)
            reinterpret_cast<uint4*>(y + k)[j] = reinterpret_cast<const uint4*>(out)[j];
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (k + j < P.K) y[k + j] = out[j];
        }
      } else {  // eight stores of 32 neighbours
#pragma unroll
        for (int j = 0; j < (int)(sizeof(T) * 8 / 16); ++j)
          reinterpret_cast<uint4*>(buf + threadIdx.x % 32 * 8)[j] = reinterpret_cast<const uint4*>(out)[j];
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int at = 32 * j + threadIdx.x % 32;
          if (k0 + at < P.K) y[k0 + at] = buf[at];
        }
        __syncwarp();
      }
    }
  }
}

// Rows a warp takes together once there are enough of them: their loads in
// flight hide each other's latency (dequantising 13824 x 5120 to bf16: 33.0 us
// with 4, 31.2 with 8).
constexpr int kQuantRows = 4, kDequantRows = 8;

template <typename T, bool NV, bool VEC>
void* pick(bool quantize, bool many) {
  if (quantize) return many ? (void*)quantize_kernel<T, NV, VEC, kQuantRows> : (void*)quantize_kernel<T, NV, VEC, 1>;
  return many ? (void*)dequantize_kernel<T, NV, VEC, kDequantRows> : (void*)dequantize_kernel<T, NV, VEC, 1>;
}
template <typename T, bool NV>
void* pick(bool quantize, bool vec, bool many) {
  return vec ? pick<T, NV, true>(quantize, many) : pick<T, NV, false>(quantize, many);
}

int elem_bytes(int type) { return type == POLYQ_F32 ? 4 : 2; }

int launch(QuantParams& P, const polyq_fp4* t, const polyq_dense* d, bool quantize, void* stream,
           const char* who) {
  int sms = 0;
  int rc = polyq_sm_count(&sms);
  if (rc) return rc;
  const bool nv = t->format == POLYQ_FP4_NV;
  P.codes = t->codes;
  P.scales = t->scales;
  P.code_stride = t->code_stride;
  P.rows = t->rows;
  P.K = t->K;
  P.A = fp4::atoms(t->K, nv);
  P.g = t->tensor_scale;
  int e;
  P.inv_g = std::frexp(P.g, &e) == 0.5f ? 1.f / P.g : 0.f;
  if (!std::isfinite(P.inv_g)) P.inv_g = 0.f;
  P.up = P.g < 1.f ? 0x1p40f : 1.f;
  P.mid_g = P.g >= 0x1p-100f && P.g <= 0x1p100f;
  const int64_t chunks = (P.K + 255) / 256;
  // several rows a warp once that still gives every SM a full set of warps
  const bool many = P.rows * chunks >= (int64_t)sms * 64 * 4;
  const int rows = many ? (quantize ? kQuantRows : kDequantRows) : 1;
  P.row_groups = (P.rows + rows - 1) / rows;
  const int eb = elem_bytes(d->type);
  const bool vec = (uintptr_t)d->data % 16 == 0 && d->stride * eb % 16 == 0;
  void* f;
  if (d->type == POLYQ_F32) f = nv ? pick<float, true>(quantize, vec, many) : pick<float, false>(quantize, vec, many);
  else if (d->type == POLYQ_BF16)
    f = nv ? pick<__nv_bfloat16, true>(quantize, vec, many) : pick<__nv_bfloat16, false>(quantize, vec, many);
  else f = nv ? pick<__half, true>(quantize, vec, many) : pick<__half, false>(quantize, vec, many);
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = (cudaStream_t)stream;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3((unsigned)((chunks + kWarps - 1) / kWarps), (unsigned)std::min<int64_t>(P.row_groups, 65535));
  cfg.blockDim = dim3(32 * kWarps);
  void* args[] = {&P};
  cudaError_t ce = cudaLaunchKernelExC(&cfg, f, args);
  if (ce != cudaSuccess) return polyq_set_error(POLYQ_ECUDA, "%s: launch: %s", who, cudaGetErrorString(ce));
  return POLYQ_OK;
}

}  // namespace

int polyq_check_fp4(const polyq_fp4* t, const char* who, const char* what) {
  if (!t) return polyq_set_error(POLYQ_EINVAL, "%s: %s is NULL", who, what);
  if (t->format != POLYQ_FP4_MX && t->format != POLYQ_FP4_NV)
    return polyq_set_error(POLYQ_EINVAL, "%s: %s: format %d", who, what, t->format);
  if (t->rows < 1 || t->K < 1 || t->rows > (1 << 24) || t->K > (1 << 24))
    return polyq_set_error(POLYQ_EINVAL, "%s: %s: [%lld][%lld]", who, what, (long long)t->rows,
                           (long long)t->K);
  if (!t->codes || !t->scales || (uintptr_t)t->codes % 16 || (uintptr_t)t->scales % 16)
    return polyq_set_error(POLYQ_EINVAL, "%s: %s: codes and scales must be 16-byte aligned", who, what);
  if (t->code_stride % 16 || t->code_stride < (t->K + 1) / 2 || t->code_stride > (1ll << 30))
    return polyq_set_error(POLYQ_EINVAL, "%s: %s: code_stride %lld for K=%lld", who, what,
                           (long long)t->code_stride, (long long)t->K);
  if (!(t->tensor_scale > 0.f) || !std::isfinite(t->tensor_scale) ||
      (t->format == POLYQ_FP4_MX && t->tensor_scale != 1.f))
    return polyq_set_error(POLYQ_EINVAL, "%s: %s: tensor_scale %g", who, what, (double)t->tensor_scale);
  return POLYQ_OK;
}

int polyq_check_dense(const polyq_dense* d, int64_t cols, const char* who, const char* what) {
  if (!d || !d->data) return polyq_set_error(POLYQ_EINVAL, "%s: %s is NULL", who, what);
  if (d->type != POLYQ_F32 && d->type != POLYQ_BF16 && d->type != POLYQ_F16)
    return polyq_set_error(POLYQ_EINVAL, "%s: %s: type %d", who, what, d->type);
  if (d->stride < cols || d->stride > (1ll << 32))
    return polyq_set_error(POLYQ_EINVAL, "%s: %s: stride %lld for rows of %lld", who, what,
                           (long long)d->stride, (long long)cols);
  if ((uintptr_t)d->data % elem_bytes(d->type))
    return polyq_set_error(POLYQ_EINVAL, "%s: %s is not aligned to its elements", who, what);
  return POLYQ_OK;
}

extern "C" int polyq_fp4_bytes(int64_t rows, int64_t K, int32_t format, int64_t* code_stride,
                               int64_t* scale_bytes) {
  polyq_clear_error();
  if (!code_stride || !scale_bytes || rows < 1 || K < 1 || rows > (1 << 24) || K > (1 << 24) ||
      (format != POLYQ_FP4_MX && format != POLYQ_FP4_NV))
    return polyq_set_error(POLYQ_EINVAL, "polyq_fp4_bytes: [%lld][%lld] format %d", (long long)rows,
                           (long long)K, format);
  *code_stride = ((K + 1) / 2 + 15) / 16 * 16;
  *scale_bytes = (rows + 127) / 128 * fp4::atoms(K, format == POLYQ_FP4_NV) * 512;
  return POLYQ_OK;
}

extern "C" int polyq_fp4_quantize(const polyq_dense* x, const polyq_fp4* out, void* stream) {
  polyq_clear_error();
  int rc = polyq_check_fp4(out, "polyq_fp4_quantize", "out");
  if (!rc) rc = polyq_check_dense(x, out->K, "polyq_fp4_quantize", "x");
  if (rc) return rc;
  QuantParams P;
  memset(&P, 0, sizeof P);
  P.x = x->data;
  P.x_stride = x->stride;
  return launch(P, out, x, true, stream, "polyq_fp4_quantize");
}

extern "C" int polyq_fp4_dequantize(const polyq_fp4* t, const polyq_dense* y, void* stream) {
  polyq_clear_error();
  int rc = polyq_check_fp4(t, "polyq_fp4_dequantize", "t");
  if (!rc) rc = polyq_check_dense(y, t->K, "polyq_fp4_dequantize", "y");
  if (rc) return rc;
  QuantParams P;
  memset(&P, 0, sizeof P);
  P.y = y->data;
  P.y_stride = y->stride;
  return launch(P, t, y, false, stream, "polyq_fp4_dequantize");
}
