// Layer norm (or, without the mean, RMS norm) and its backward pass.
//
//   hat = (x - mean) rstd,  y = hat w + b
//   g = dy w,  dx = res + rstd (g - mean(g) - hat mean(g hat))
//   dw = sum over rows of dy hat,  db = sum over rows of dy
//
// Bound by HBM: x in and y out (forward), x, dy (and a residual gradient) in and
// dx out (backward), each once.  A row lies in the registers of a group of
// threads, eight elements each, so that the sums over it and its result need one
// reading; the next row's loads are in flight meanwhile.  A group keeps the
// weight, and in the backward pass its rows' sums for dw and db, in registers
// from row to row.  Rows wider than a thread block are shared by a cluster,
// whose blocks exchange the sums through distributed shared memory.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "polyq_dense_dev.cuh"
#include "polyq_dev.cuh"
#include "polyq_finetune.h"
#include "polyq_fp4_dev.cuh"
#include "polyq_internal.h"

namespace {

using namespace polyq;

constexpr int kMaxCluster = 8;
// Threads of a block at most (of eight columns each): the backward pass holds 24 sums
// and weights a thread beside its rows, and spills at the 64 registers of 1024 threads.
constexpr int kForwardThreads = 1024, kBackwardThreads = 768;
constexpr int kReduceCols = 32, kReduceRows = 8;

struct NormParams {
  const void* x;
  const void* dy;
  const void* res;
  void* y;  // y or dx
  const void* w;
  const void* b;
  float* stats;
  float* parts;  // [2][grid / cluster][K]: sums of dw and of db
  int64_t x_stride, dy_stride, res_stride, y_stride, rows, K;
  float eps, inv_k;
  int w_type, b_type, center, cluster, want_w, want_b;
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Sums over a row of two values per thread.  The order is fixed: a butterfly in
// each warp, a butterfly over the warps' sums, the cluster's blocks in order.
// One barrier a sum: `at` alternates between two places, and a place is written
// again only after the barrier of the sum between.
struct RowSum {
  float2 (*warps)[32];          // [2][32] of this row's threads
  float2 (*blocks)[kMaxCluster];  // [2][cluster]
  int nw, cluster, at;
  __device__ __forceinline__ float2 operator()(float2 v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
      v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o);
    }
    if (nw == 1 && cluster == 1) return v;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    at ^= 1;
    if (lane == 0) warps[at][warp] = v;
    __syncthreads();
    v = lane < nw ? warps[at][lane] : make_float2(0.f, 0.f);
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
      v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o);
    }
    if (cluster == 1) return v;
    if (threadIdx.x < (unsigned)cluster) {
      const uint32_t mine = smem_u32(&blocks[at][cluster_rank()]);
      uint32_t there;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine), "r"(threadIdx.x));
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(v.x), "f"(v.y) : "memory");
    }
    __syncwarp();
    cluster_sync();
    float2 s = make_float2(0.f, 0.f);
    for (int i = 0; i < cluster; ++i) {
      s.x += blocks[at][i].x;
      s.y += blocks[at][i].y;
    }
    return s;
  }
};

// threadIdx.x: a row's threads (whole warps), threadIdx.y: the rows that a block
// takes together (one in a cluster).
template <typename TX, typename TY, bool VEC>
__global__ void __launch_bounds__(kForwardThreads) norm_forward_kernel(const __grid_constant__ NormParams P) {
  __shared__ float2 warps[8][2][32];
  __shared__ float2 blocks[2][kMaxCluster];
  const int T = blockDim.x, R = blockDim.y;
  const int rank = P.cluster > 1 ? (int)cluster_rank() : 0;
  const int64_t c0 = (int64_t)rank * T * 8, col = c0 + (VEC ? threadIdx.x * 8 : threadIdx.x);
  const uint32_t mask = mask8<VEC>(col, T, P.K);
  RowSum sum{warps[threadIdx.y], blocks, T >> 5, P.cluster, 0};
  pdl_trigger();
  pdl_wait();
  if (P.cluster > 1) cluster_sync();  // (its blocks have begun: their shared memory may be written)
  const int64_t step = (int64_t)(gridDim.x / P.cluster) * R;
  int64_t base = (int64_t)(blockIdx.x / P.cluster) * R, row = base + threadIdx.y;
  const TX* x = (const TX*)P.x;
  Raw8<TX> next;
  load8<VEC>(x + row * P.x_stride, col, T, row < P.rows ? mask : 0u, next);
  float w[8], b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t k = col + i * (VEC ? 1 : T);
    const bool in = mask >> i & 1;
    w[i] = P.w && in ? any_load(P.w, P.w_type, k) : 1.f;
    b[i] = P.b && in ? any_load(P.b, P.b_type, k) : 0.f;
  }
  for (; base < P.rows; base += step, row += step) {
    float v[8];
    to_float(next, v);
    const int64_t then = row + step;
    load8<VEC>(x + then * P.x_stride, col, T, then < P.rows ? mask : 0u, next);
    float mean = 0.f;
    if (P.center) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[i];
      mean = sum(make_float2(s, 0.f)).x * P.inv_k;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = mask >> i & 1 ? v[i] - mean : 0.f;
    }
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) q = fmaf(v[i], v[i], q);
    const float rstd = __frsqrt_rn(fmaf(sum(make_float2(q, 0.f)).x, P.inv_k, P.eps));
    if (row >= P.rows) continue;
    if (P.stats && rank == 0 && threadIdx.x == 0) reinterpret_cast<float2*>(P.stats)[row] = make_float2(mean, rstd);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = fmaf(v[i] * rstd, w[i], b[i]);
    store8<VEC>((TY*)P.y + row * P.y_stride, col, T, mask, v);
  }
}

template <typename TX, typename TY, bool VEC>
__global__ void __launch_bounds__(kBackwardThreads) norm_backward_kernel(const __grid_constant__ NormParams P) {
  __shared__ float2 warps[8][2][32];
  __shared__ float2 blocks[2][kMaxCluster];
  __shared__ float rows_sum[2048];
  const int T = blockDim.x, R = blockDim.y;
  const int rank = P.cluster > 1 ? (int)cluster_rank() : 0;
  const int64_t c0 = (int64_t)rank * T * 8, col = c0 + (VEC ? threadIdx.x * 8 : threadIdx.x);
  const uint32_t mask = mask8<VEC>(col, T, P.K);
  RowSum sum{warps[threadIdx.y], blocks, T >> 5, P.cluster, 0};
  pdl_trigger();
  pdl_wait();
  if (P.cluster > 1) cluster_sync();
  const int64_t groups = gridDim.x / P.cluster, step = groups * R;
  const int64_t group = blockIdx.x / P.cluster;
  int64_t base = group * R, row = base + threadIdx.y;
  const TX* x = (const TX*)P.x;
  const TY* dy = (const TY*)P.dy;
  const TX* res = (const TX*)P.res;
  Raw8<TX> nx, nr;
  Raw8<TY> nd;
  float2 ns;
  {
    const uint32_t m = row < P.rows ? mask : 0u;
    load8<VEC>(x + row * P.x_stride, col, T, m, nx);
    load8<VEC>(dy + row * P.dy_stride, col, T, m, nd);
    if (P.res) load8<VEC>(res + row * P.res_stride, col, T, m, nr);
    ns = row < P.rows ? __ldcg(reinterpret_cast<const float2*>(P.stats) + row) : make_float2(0.f, 0.f);
  }
  float w[8], dw[8], db[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t k = col + i * (VEC ? 1 : T);
    w[i] = P.w && (mask >> i & 1) ? any_load(P.w, P.w_type, k) : 1.f;
    dw[i] = db[i] = 0.f;
  }
  for (; base < P.rows; base += step, row += step) {
    float h[8], d[8];
    to_float(nx, h);
    to_float(nd, d);
    const float mean = P.center ? ns.x : 0.f, rstd = ns.y;
    const int64_t then = row + step;
    const uint32_t m = then < P.rows ? mask : 0u;
    load8<VEC>(x + then * P.x_stride, col, T, m, nx);
    load8<VEC>(dy + then * P.dy_stride, col, T, m, nd);
    ns = then < P.rows ? __ldcg(reinterpret_cast<const float2*>(P.stats) + then) : make_float2(0.f, 0.f);
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      h[i] = (h[i] - mean) * rstd;
      if (row < P.rows) {  // (a row that is not there has no sums to add to)
        dw[i] = fmaf(d[i], h[i], dw[i]);
        db[i] += d[i];
      }
      d[i] *= w[i];
      if (mask >> i & 1) {
        s.x = fmaf(d[i], h[i], s.x);
        s.y += d[i];
      }
    }
    if (!P.y) continue;  // dx is not wanted
    s = sum(s);
    float a[8] = {};
    if (P.res) {
      to_float(nr, a);
      load8<VEC>(res + then * P.res_stride, col, T, m, nr);
    }
    if (row >= P.rows) continue;
    const float mgh = s.x * P.inv_k, mg = P.center ? s.y * P.inv_k : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) d[i] = fmaf(rstd, d[i] - mg - h[i] * mgh, a[i]);
    store8<VEC>((TX*)P.y + row * P.y_stride, col, T, mask, d);
  }
  // The block's rows are added in order; a group of blocks writes its sums once.
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (!(which ? P.want_b : P.want_w)) continue;
    float(&v)[8] = which ? db : dw;
    float* out = P.parts + ((int64_t)which * groups + group) * P.K;
    if (R > 1) {
      for (int r = 1; r < R; ++r) {  // (2048 floats hold one row's threads: 256 of eight)
        __syncthreads();
        if ((int)threadIdx.y == r)
#pragma unroll
          for (int i = 0; i < 8; ++i) rows_sum[i * T + threadIdx.x] = v[i];
        __syncthreads();
        if (threadIdx.y == 0)
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] += rows_sum[i * T + threadIdx.x];
      }
    }
    if (threadIdx.y == 0) store8<false>(out, col, VEC ? 1 : T, mask, v);
  }
}

// dw[k], db[k] = the sums over `groups` partial rows, in a fixed order.
struct ReduceParams {
  const float* parts;
  void* out[2];
  int type[2];
  int64_t groups, K;
};
__global__ void __launch_bounds__(kReduceCols* kReduceRows) norm_reduce_kernel(const __grid_constant__ ReduceParams P) {
  __shared__ float part[kReduceRows][kReduceCols];
  pdl_trigger();
  pdl_wait();
  if (!P.out[blockIdx.y]) return;
  const int64_t k = (int64_t)blockIdx.x * kReduceCols + threadIdx.x;
  const float* p = P.parts + (int64_t)blockIdx.y * P.groups * P.K + k;
  float s = 0.f;
  if (k < P.K) {
#pragma unroll 8
    for (int64_t g = threadIdx.y; g < P.groups; g += kReduceRows) s += __ldcg(p + g * P.K);
  }
  part[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.y != 0 || k >= P.K) return;
#pragma unroll
  for (int i = 1; i < kReduceRows; ++i) s += part[i][threadIdx.x];
  any_store(P.out[blockIdx.y], P.type[blockIdx.y], k, s);
}

// How rows are shared out.
struct Shape {
  int threads, rows, cluster;
  int64_t groups;
};
Shape shape_of(int64_t rows, int64_t K, int sms, bool backward) {
  Shape s;
  s.cluster = 1;
  while ((int64_t)s.cluster * 8 * (backward ? kBackwardThreads : kForwardThreads) < K) s.cluster *= 2;
  const int64_t cols = (K + s.cluster - 1) / s.cluster;
  s.threads = (int)((cols + 255) / 256 * 32);
  // small rows share a block once there is one for every SM
  s.rows = (int)std::min<int64_t>(std::max(1, 256 / s.threads), (rows + sms - 1) / sms);
  const int per_sm = std::max(1, (backward ? 1024 : 1536) / (s.threads * s.rows));
  s.groups = std::min<int64_t>((rows + s.rows - 1) / s.rows, std::max(1, sms * per_sm / s.cluster));
  return s;
}

template <typename TX, typename TY>
void* pick(bool backward, bool vec) {
  if (backward) return vec ? (void*)norm_backward_kernel<TX, TY, true> : (void*)norm_backward_kernel<TX, TY, false>;
  return vec ? (void*)norm_forward_kernel<TX, TY, true> : (void*)norm_forward_kernel<TX, TY, false>;
}
template <typename TX>
void* pick(int ty, bool backward, bool vec) {
  return ty == POLYQ_F32    ? pick<TX, float>(backward, vec)
         : ty == POLYQ_BF16 ? pick<TX, __nv_bfloat16>(backward, vec)
                            : pick<TX, __half>(backward, vec);
}
void* pick(int tx, int ty, bool backward, bool vec) {
  return tx == POLYQ_F32    ? pick<float>(ty, backward, vec)
         : tx == POLYQ_BF16 ? pick<__nv_bfloat16>(ty, backward, vec)
                            : pick<__half>(ty, backward, vec);
}

int launch(void* f, dim3 grid, dim3 block, int cluster, void* params, void* stream, const char* who) {
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = (cudaStream_t)stream;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  cfg.gridDim = grid;
  cfg.blockDim = block;
  void* args[] = {params};
  cudaError_t ce = cudaLaunchKernelExC(&cfg, f, args);
  if (ce != cudaSuccess) return polyq_set_error(POLYQ_ECUDA, "%s: launch: %s", who, cudaGetErrorString(ce));
  return POLYQ_OK;
}

int check_size(int64_t rows, int64_t K, const char* who) {
  if (rows < 1 || K < 1 || rows > (1 << 24) || K > (1 << 24))
    return polyq_set_error(POLYQ_EINVAL, "%s: [%lld][%lld]", who, (long long)rows, (long long)K);
  if (K > POLYQ_NORM_MAX_K)
    return polyq_set_error(POLYQ_EUNSUPPORTED, "%s: rows of %lld, at most %d", who, (long long)K, POLYQ_NORM_MAX_K);
  return POLYQ_OK;
}

bool rows_on_16(const polyq_dense* d) {
  const int eb = d->type == POLYQ_F32 ? 4 : 2;
  return (uintptr_t)d->data % 16 == 0 && d->stride * eb % 16 == 0;
}

// A weight or bias: K elements.
int check_vector(const polyq_dense* d, const char* who, const char* what) {
  polyq_dense one = *d;
  one.stride = 1;
  return polyq_check_dense(&one, 1, who, what);
}

}  // namespace

extern "C" int polyq_layernorm_forward(const polyq_dense* x, int64_t rows, int64_t K, const polyq_dense* weight,
                                       const polyq_dense* bias, float eps, int center, const polyq_dense* y,
                                       float* stats, void* stream) {
  static const char* who = "polyq_layernorm_forward";
  polyq_clear_error();
  int rc = check_size(rows, K, who);
  if (!rc) rc = polyq_check_dense(x, K, who, "x");
  if (!rc) rc = polyq_check_dense(y, K, who, "y");
  if (!rc && weight) rc = check_vector(weight, who, "weight");
  if (!rc && bias) rc = check_vector(bias, who, "bias");
  if (rc) return rc;
  if (!(eps >= 0.f) || !std::isfinite(eps)) return polyq_set_error(POLYQ_EINVAL, "%s: eps %g", who, (double)eps);
  if ((uintptr_t)stats % 8) return polyq_set_error(POLYQ_EINVAL, "%s: stats must be 8-byte aligned", who);
  int sms = 0;
  rc = polyq_sm_count(&sms);
  if (rc) return rc;
  const Shape s = shape_of(rows, K, sms, false);
  NormParams P;
  memset(&P, 0, sizeof P);
  P.x = x->data;
  P.x_stride = x->stride;
  P.y = y->data;
  P.y_stride = y->stride;
  if (weight) P.w = weight->data, P.w_type = weight->type;
  if (bias) P.b = bias->data, P.b_type = bias->type;
  P.stats = stats;
  P.rows = rows;
  P.K = K;
  P.eps = eps;
  P.inv_k = 1.f / (float)K;
  P.center = center != 0;
  P.cluster = s.cluster;
  return launch(pick(x->type, y->type, false, rows_on_16(x) && rows_on_16(y)), dim3((unsigned)(s.groups * s.cluster)),
                dim3(s.threads, s.rows), s.cluster, &P, stream, who);
}

extern "C" int polyq_layernorm_workspace_bytes(int64_t rows, int64_t K, size_t* bytes) {
  static const char* who = "polyq_layernorm_workspace_bytes";
  polyq_clear_error();
  if (!bytes) return polyq_set_error(POLYQ_EINVAL, "%s: NULL argument", who);
  int rc = check_size(rows, K, who);
  int sms = 0;
  if (!rc) rc = polyq_sm_count(&sms);
  if (rc) return rc;
  *bytes = (size_t)shape_of(rows, K, sms, true).groups * K * 2 * sizeof(float);
  return POLYQ_OK;
}

extern "C" int polyq_layernorm_backward(const polyq_dense* x, int64_t rows, int64_t K, const polyq_dense* weight,
                                        const float* stats, int center, const polyq_dense* dy,
                                        const polyq_dense* residual, const polyq_dense* dx, const polyq_dense* dweight,
                                        const polyq_dense* dbias, void* workspace, size_t workspace_bytes,
                                        void* stream) {
  static const char* who = "polyq_layernorm_backward";
  polyq_clear_error();
  int rc = check_size(rows, K, who);
  if (!rc) rc = polyq_check_dense(x, K, who, "x");
  if (!rc) rc = polyq_check_dense(dy, K, who, "dy");
  if (!rc && residual) rc = polyq_check_dense(residual, K, who, "residual");
  if (!rc && dx) rc = polyq_check_dense(dx, K, who, "dx");
  if (!rc && weight) rc = check_vector(weight, who, "weight");
  if (!rc && dweight) rc = check_vector(dweight, who, "dweight");
  if (!rc && dbias) rc = check_vector(dbias, who, "dbias");
  if (rc) return rc;
  if (!dx && !dweight && !dbias) return polyq_set_error(POLYQ_EINVAL, "%s: no gradient is wanted", who);
  if (dx && dx->type != x->type)
    return polyq_set_error(POLYQ_EINVAL, "%s: dx is of type %d, x of %d", who, dx->type, x->type);
  if (residual && (!dx || residual->type != dx->type))
    return polyq_set_error(POLYQ_EINVAL, "%s: a residual needs a dx of its type", who);
  if (!stats || (uintptr_t)stats % 8)
    return polyq_set_error(POLYQ_EINVAL, "%s: stats must be 8-byte aligned and not NULL", who);
  int sms = 0;
  rc = polyq_sm_count(&sms);
  if (rc) return rc;
  const Shape s = shape_of(rows, K, sms, true);
  const bool sums = dweight || dbias;
  if (sums && (!workspace || (uintptr_t)workspace % 16 ||
               workspace_bytes < (size_t)s.groups * K * 2 * sizeof(float)))
    return polyq_set_error(POLYQ_ENOMEM, "%s: workspace of %zu bytes, 16-byte aligned, needed", who,
                           (size_t)s.groups * K * 2 * sizeof(float));
  NormParams P;
  memset(&P, 0, sizeof P);
  P.x = x->data;
  P.x_stride = x->stride;
  P.dy = dy->data;
  P.dy_stride = dy->stride;
  if (residual) P.res = residual->data, P.res_stride = residual->stride;
  if (dx) P.y = dx->data, P.y_stride = dx->stride;
  if (weight) P.w = weight->data, P.w_type = weight->type;
  P.stats = const_cast<float*>(stats);
  P.parts = (float*)workspace;
  P.rows = rows;
  P.K = K;
  P.inv_k = 1.f / (float)K;
  P.center = center != 0;
  P.cluster = s.cluster;
  P.want_w = dweight != nullptr;
  P.want_b = dbias != nullptr;
  const bool vec = rows_on_16(x) && rows_on_16(dy) && (!residual || rows_on_16(residual)) && (!dx || rows_on_16(dx));
  rc = launch(pick(x->type, dy->type, true, vec), dim3((unsigned)(s.groups * s.cluster)), dim3(s.threads, s.rows),
              s.cluster, &P, stream, who);
  if (rc || !sums) return rc;
  ReduceParams Q;
  memset(&Q, 0, sizeof Q);
  Q.parts = P.parts;
  if (dweight) Q.out[0] = dweight->data, Q.type[0] = dweight->type;
  if (dbias) Q.out[1] = dbias->data, Q.type[1] = dbias->type;
  Q.groups = s.groups;
  Q.K = K;
  return launch((void*)norm_reduce_kernel, dim3((unsigned)((K + kReduceCols - 1) / kReduceCols), 2),
                dim3(kReduceCols, kReduceRows), 1, &Q, stream, who);
}
