// Microscaled 4-bit floating point: quantisation and its inverse.
//
//   MX  s = 2^(floor(log2 max|x|) - 2) per 32 elements,  q = e2m1(x / s)
//   NV  s = e4m3(max|x/g| / 6) per 16 elements,          q = e2m1(x / g / s)
//
// A lane holds 8 consecutive elements of a row, so a warp takes 256 elements:
// a block is four (MX) or two (NV) neighbouring lanes, its maximum two or one
// shuffles, and the 8 codes of a lane one 4-byte store (a warp stores 128
// consecutive bytes).  The scales of four blocks are gathered into the 4-byte
// word that the tensor cores' scale layout keeps together.  Bound by HBM for
// large tensors and by the launch for a token's.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "polyq_dev.cuh"
#include "polyq_fp4_dev.cuh"
#include "polyq_internal.h"

namespace {

using namespace polyq;

constexpr int kWarps = 8;

struct QuantParams {
  const void* x;
  void* y;
  uint8_t* codes;
  uint8_t* scales;
  int64_t x_stride, y_stride, code_stride, rows, K, A;
  int64_t chunks, tasks;  // 256-element chunks of a row; (row group, chunk) pairs
  float g, inv_g;         // tensor scale; its reciprocal where that is exact, else 0
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

// 8 elements from k on; zeros past K.  VEC: rows start on 16 bytes.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* __restrict__ row, int64_t k, int64_t K, float (&v)[8]) {
  if (VEC && k + 8 <= K) {
    constexpr int N16 = sizeof(T) * 8 / 16;
    uint4 raw[N16];
#pragma unroll
    for (int i = 0; i < N16; ++i) raw[i] = __ldg(reinterpret_cast<const uint4*>(row + k) + i);
    const T* e = reinterpret_cast<const T*>(raw);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = Elem<T>::to(e[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + i < K ? Elem<T>::to(row[k + i]) : 0.f;
  }
}

// ROWS rows of a chunk per warp, their loads in flight together.
template <typename T, bool NV, bool VEC, int ROWS>
__global__ void __launch_bounds__(32 * kWarps) quantize_kernel(const __grid_constant__ QuantParams P) {
  const int lane = threadIdx.x & 31;
  pdl_trigger();
  pdl_wait();
  for (int64_t task = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); task < P.tasks;
       task += (int64_t)gridDim.x * kWarps) {
    const int64_t r0 = task / P.chunks * ROWS, k = (task % P.chunks) * 256 + lane * 8;
    float v[ROWS][8];
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
      if (r0 + i < P.rows) load8<T, VEC>((const T*)P.x + (r0 + i) * P.x_stride, k, P.K, v[i]);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const int64_t r = r0 + i;
      if (r >= P.rows) break;  // the same for the whole warp
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (NV) v[i][j] = P.inv_g != 0.f ? v[i][j] * P.inv_g : __fdiv_rn(v[i][j], P.g);
        m = max(m, __float_as_uint(v[i][j]) & 0x7FFFFFFFu);
      }
      m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
      if (!NV) m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
      const fp4::Scale<NV> sc(m);
      float q[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] = sc.div(v[i][j]);
      if (k < P.K) *reinterpret_cast<uint32_t*>(P.codes + r * P.code_stride + k / 2) = fp4::codes8(q);
      // the word of four blocks: byte b % 4 from each
      constexpr int LPB = NV ? 2 : 4;  // lanes of a block
      uint32_t w = sc.byte << (8 * (lane / LPB % 4));
      w |= __shfl_xor_sync(0xffffffffu, w, LPB);
      w |= __shfl_xor_sync(0xffffffffu, w, 2 * LPB);
      const int64_t b = k / (8 * LPB);
      if (lane % (4 * LPB) == 0 && (b >> 2) < P.A)
        *reinterpret_cast<uint32_t*>(P.scales + fp4::scale_off(r, b, P.A)) = w;
    }
  }
}

template <typename T, bool NV, bool VEC, int ROWS>
__global__ void __launch_bounds__(32 * kWarps) dequantize_kernel(const __grid_constant__ QuantParams P) {
  const int lane = threadIdx.x & 31;
  pdl_trigger();
  pdl_wait();
  for (int64_t task = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); task < P.tasks;
       task += (int64_t)gridDim.x * kWarps) {
    const int64_t r0 = task / P.chunks * ROWS, k = (task % P.chunks) * 256 + lane * 8;
    if (k >= P.K) continue;
    uint32_t c[ROWS], sb[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
      if (r0 + i < P.rows) {
        // rows are padded to 16 bytes, so a lane's 4 bytes exist
        c[i] = __ldg(reinterpret_cast<const uint32_t*>(P.codes + (r0 + i) * P.code_stride + k / 2));
        sb[i] = __ldg(P.scales + fp4::scale_off(r0 + i, k / fp4::block_len(NV), P.A));
      }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      if (r0 + i >= P.rows) break;
      const float s = NV ? fp4::from_e4m3(sb[i]) : fp4::from_e8m0(sb[i]);
      alignas(16) T out[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 v = fp4::values2(c[i] >> (8 * j) & 0xFFu);
        out[2 * j] = Elem<T>::from(v.x * s * P.g);
        out[2 * j + 1] = Elem<T>::from(v.y * s * P.g);
      }
      T* y = (T*)P.y + (r0 + i) * P.y_stride + k;
      if (VEC && k + 8 <= P.K) {
#pragma unroll
        for (int j = 0; j < (int)(sizeof(T) * 8 / 16); ++j)
          reinterpret_cast<uint4*>(y)[j] = reinterpret_cast<const uint4*>(out)[j];
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (k + j < P.K) y[j] = out[j];
      }
    }
  }
}

template <typename T, bool NV, bool VEC, int ROWS>
void* pick(bool quantize) {
  return quantize ? (void*)quantize_kernel<T, NV, VEC, ROWS> : (void*)dequantize_kernel<T, NV, VEC, ROWS>;
}
template <typename T, bool NV>
void* pick(bool quantize, bool vec, bool rows4) {
  return vec ? (rows4 ? pick<T, NV, true, 4>(quantize) : pick<T, NV, true, 1>(quantize))
             : (rows4 ? pick<T, NV, false, 4>(quantize) : pick<T, NV, false, 1>(quantize));
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
  P.chunks = (P.K + 255) / 256;
  // four rows a warp once that still gives every SM a full set of warps
  const bool rows4 = P.rows * P.chunks >= (int64_t)sms * 64 * 4;
  P.tasks = (P.rows + (rows4 ? 3 : 0)) / (rows4 ? 4 : 1) * P.chunks;
  const int eb = elem_bytes(d->type);
  const bool vec = (uintptr_t)d->data % 16 == 0 && d->stride * eb % 16 == 0;
  void* f;
  if (d->type == POLYQ_F32) f = nv ? pick<float, true>(quantize, vec, rows4) : pick<float, false>(quantize, vec, rows4);
  else if (d->type == POLYQ_BF16)
    f = nv ? pick<__nv_bfloat16, true>(quantize, vec, rows4) : pick<__nv_bfloat16, false>(quantize, vec, rows4);
  else f = nv ? pick<__half, true>(quantize, vec, rows4) : pick<__half, false>(quantize, vec, rows4);
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = (cudaStream_t)stream;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3((unsigned)std::min<int64_t>((P.tasks + kWarps - 1) / kWarps, 1 << 30));
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
