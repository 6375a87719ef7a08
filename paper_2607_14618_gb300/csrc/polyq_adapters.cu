// Entry points of the low-rank adapters: checks, tiles and launches.
#include <algorithm>
#include <atomic>
#include <cstring>

#include "polyq_adapters_dev.cuh"
#include "polyq_fp4_dev.cuh"
#include "polyq_internal.h"

namespace polyq {
namespace lora {
extern template Kernel shrink_of<__nv_bfloat16>(int bm, int rn, bool trans, bool any);
extern template Kernel expand_of<__nv_bfloat16>(int bm, int rn, bool trans, bool f32);
extern template Kernel gradients_of<__nv_bfloat16>(int rn, bool any);
extern template Kernel shrink_of<__half>(int bm, int rn, bool trans, bool any);
extern template Kernel expand_of<__half>(int bm, int rn, bool trans, bool f32);
extern template Kernel gradients_of<__half>(int rn, bool any);
}  // namespace lora
}  // namespace polyq

namespace {

using namespace polyq;
using lora::Kernel;

constexpr int64_t kMaxSize = 1 << 24;

// Devices on which a kernel may use its shared memory (a bit each), by the kernel's tile.
std::atomic<uint64_t> g_ready[320];

int launch(const Kernel& k, int which, dim3 grid, int threads, int cluster, void* params, void* stream, const char* who) {
  int dev = 0;
  cudaError_t ce = cudaGetDevice(&dev);
  if (ce == cudaSuccess) {
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (!(g_ready[which].load(std::memory_order_acquire) & bit)) {
      ce = cudaFuncSetAttribute(k.f, cudaFuncAttributeMaxDynamicSharedMemorySize, k.smem);
      if (ce == cudaSuccess) g_ready[which].fetch_or(bit, std::memory_order_release);
    }
  }
  if (ce == cudaSuccess) {
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
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = k.smem;
    void* args[] = {params};
    ce = cudaLaunchKernelExC(&cfg, k.f, args);
  }
  if (ce != cudaSuccess) return polyq_set_error(POLYQ_ECUDA, "%s: launch: %s", who, cudaGetErrorString(ce));
  return POLYQ_OK;
}

// Rows of 16-bit elements that start on 16 bytes, as asynchronous copies want them.
bool rows_on_16(const polyq_dense* d) { return (uintptr_t)d->data % 16 == 0 && d->stride % 8 == 0; }

// Adapters, of `rows` rows each, that one tensor map describes: as the CUDA API documents its strides, an
// outer one is the inner one times the rows between, and below 2^40 bytes.  Others, as with one buffer
// of each adapter's a and b, are copied in the ordinary way in tiles of 16 rows (4096 rows of rank 64
// forward 97 us, 76 by the map; 6007 of rank 32: 114 and 70).  One matrix of all adapters (a stride of
// 0) is a map of one, see ShrinkParams.
bool mapped(const lora::Side& w, int64_t rows, int n) {
  return n == 1 || w.next == 0 || (w.next % w.stride == 0 && w.next / w.stride >= rows && w.next < (1ll << 39));
}

int rank_tile(int R) { return R <= 16 ? 16 : R <= 32 ? 32 : R <= 64 ? 64 : 128; }
int rank_index(int rn) { return rn == 16 ? 0 : rn == 32 ? 1 : rn == 64 ? 2 : 3; }

// Tiles of bm rows in any T rows of n segments: each has at most one that is not full.
int64_t most_tiles(int64_t T, int n, int bm) { return std::min<int64_t>(T, T / bm + n); }

// v [T][R] of x times one of the adapters' matrices.
int shrink(const polyq_dense* x, int64_t T, int64_t K, const polyq_adapters* ad, bool trans, const lora::Side& w,
           const float* scales, const lora::Segments& seg, float* v, int* status, int sms, void* stream,
           const char* who) {
  const int rn = rank_tile(ad->R);
  const int64_t mean = T / seg.n;
  const bool any = !rows_on_16(x);
  // Rows of a tile, by the segments' mean (us of whole calls with both).
  // 16 and 64: rank 16, 200 segments of 24 rows of 5120 columns 34 and 24, one of 8 7.7 and 6.7; rank 32, 48
  // of 13824 columns, of 8 rows 18.8 and 20.1, of 16 21.5 and 20.7, of 31 39 and 32; rank 64, 48 of 5120
  // columns, of 32 rows 33 and 37, of 48 41 and 36.
  // 64 and 128, worth it where 64-row tiles in clusters of eight are more than fit at once: rank 64, four of
  // 13824 columns, of 512 rows 24 and 33, of 1024 46 and 40; rank 128, 5120 columns, 512 rows 14 and 19, 1024
  // 25 and 21, 16 segments of 512 80 and 66 (but of 256 44 and 56).
  const bool few = mean <= (rn <= 32 ? 16 : 32);
  const bool many = rn >= 64 && mean >= 256 && T >= (rn == 64 ? 16 : 6) * (int64_t)sms;
  const int bm = any || !mapped(w, trans ? K : ad->R, ad->n) || few ? 16 : many ? 128 : 64;
  const bool half = ad->type == POLYQ_F16;
  const Kernel k = half ? lora::shrink_of<__half>(bm, rn, trans, any) : lora::shrink_of<__nv_bfloat16>(bm, rn, trans, any);
  const int64_t tiles = most_tiles(T, seg.n, bm), stages = K / (bm == 128 ? 64 : 128);
  int cluster = 1;
  while (cluster < lora::kMaxCluster && tiles * cluster < 2 * sms && stages >= 4 * cluster) cluster *= 2;
  lora::ShrinkParams P;
  memset(&P, 0, sizeof P);
  P.x = x->data;
  P.x_stride = x->stride;
  P.w = w;
  P.v = v;
  P.scales = scales;
  P.ranks = ad->ranks;
  P.seg = seg;
  P.K = K;
  P.R = ad->R;
  P.adapters = ad->n;
  P.cluster = cluster;
  P.status = status;
  if (bm != 16) {
    const uint64_t x_stride = (uint64_t)x->stride * 2;
    const int rc_x = polyq_tensor_map_3d(&P.x_map, x->data, (uint64_t)K, (uint64_t)T, 1, x_stride, x_stride * T, 64,
                                         (uint32_t)bm);
    if (rc_x) return rc_x;
    const uint64_t cols = trans ? ad->R : K, rows = trans ? K : ad->R, stride = (uint64_t)w.stride * 2;
    const bool one = ad->n == 1 || w.next == 0;
    P.map_next = !one;
    const int rc_w = polyq_tensor_map_3d(&P.w_map, w.w, cols, rows, one ? 1 : (uint64_t)ad->n, stride,
                                         one ? rows * stride : (uint64_t)w.next * 2,
                                         trans ? (uint32_t)std::min(rn, 64) : 64u,
                                         trans ? (uint32_t)(bm == 128 ? 64 : 128) : (uint32_t)rn);
    if (rc_w) return rc_w;
  }
  const int which = (((half * 2 + trans) * 4 + rank_index(rn)) * 4) + (any ? 3 : bm == 16 ? 0 : bm == 64 ? 1 : 2);
  return launch(k, which, dim3((unsigned)(tiles * cluster)), lora::kThreads + (bm != 16 ? 32 : 0), cluster, &P, stream,
                who);
}

// y = residual + v times one of the adapters' matrices.
int expand(const float* v, int64_t T, int64_t N, const polyq_adapters* ad, bool trans, const lora::Side& w,
           const float* scales, const lora::Segments& seg, const polyq_dense* residual, const polyq_dense* y, int sms,
           void* stream, const char* who) {
  // (Tiles of 16 against 64 rows, us: rank 64 onto 13824, 32 segments of 32 rows 40 and 42, of 48 50 and 50,
  // of 64 65 and 56; rank 16 onto 5120, of 32 17 and 20, of 64 26 and 25.)
  const int rn = rank_tile(ad->R), bm = T / seg.n <= 32 ? 16 : 64, bn = rn == 128 && bm == 64 ? 64 : 128;
  const bool half = ad->type == POLYQ_F16, f32 = y->type == POLYQ_F32;
  const Kernel k = half ? lora::expand_of<__half>(bm, rn, trans, f32) : lora::expand_of<__nv_bfloat16>(bm, rn, trans, f32);
  const int eb = f32 ? 4 : 2;
  lora::ExpandParams P;
  memset(&P, 0, sizeof P);
  P.v = v;
  P.w = w;
  if (residual) P.res = residual->data, P.res_stride = residual->stride;
  P.y = y->data;
  P.y_stride = y->stride;
  P.scales = scales;
  P.ranks = ad->ranks;
  P.seg = seg;
  P.N = N;
  P.R = ad->R;
  P.adapters = ad->n;
  P.tiles = (int32_t)most_tiles(T, seg.n, bm);
  P.vec = (uintptr_t)y->data % 16 == 0 && y->stride * eb % 16 == 0 &&
          (!residual || ((uintptr_t)residual->data % 16 == 0 && residual->stride * eb % 16 == 0));
  const int which = 128 + (((half * 2 + trans) * 4 + rank_index(rn)) * 2 + (bm == 64)) * 2 + f32;
  // Blocks of a row tile: two rounds of the SMs' blocks, one where rows are few.  (Tiles: one for
  // each segment at least, and half a tile more than full ones.)  4096 x 13824, rank 64: 67 us with 8, 60 with
  // 9; 6007 x 5120, rank 32: 46 us with 3, 31 with 5; 48 rows of rank 64: 21 us with 9, 23 with 16.
  const int64_t columns = (N + bn - 1) / bn, slots = (int64_t)sms * (bm != 16 ? 4 : rn <= 64 ? 3 : 2);
  const int64_t rows = std::min<int64_t>(P.tiles, std::max<int64_t>(seg.n, (T + bm - 1) / bm + seg.n / 2));
  const int64_t share = std::min(columns, std::max<int64_t>(1, slots / rows));
  return launch(k, which, dim3((unsigned)share, (unsigned)std::min(P.tiles, 65535)), lora::kThreads, 1, &P, stream,
                who);
}

// Blocks that share the rows of each of `used` adapters (at most), of `columns` tiles.  More of them
// are worth their exchange where each still has 512 rows of rank 16 or 1024 of a wider one and all of
// them fit at once; two of twice these rows also where they do not quite, as the adapters' rows are
// uneven, or (of one adapter) where one has a second round that is nearly empty.  us with one, two,
// four and eight:
//   5120 x 5120, rank 64 (80 blocks), 512 rows 28 30 44 84, 2048 rows 84 58 63 90;
//   1024 x 1024, rank 16 (16), 512 rows 12 11 10 10, 4096 rows 63 39 23 19;
//   four adapters of it, rank 64 (64), 1024 rows of each 46 38 46 71;
//   5120 x 5120, rank 128 (160 on 152 SMs), 1024 rows 72 75 94 165, 4096 rows 228 201 207 292;
//   5120 + 13824 of two adapters, rank 64 (296), 4096 rows, halves 110 124 184 319, uneven 141 136 196 322,
//   8192 uneven 232 205 270 412, 2048 83 91 151 280.
int gradient_cluster(int64_t T, int64_t used, int64_t columns, int rn, int sms) {
  const int64_t blocks = used * columns, slots = (int64_t)sms * (rn == 16 ? 3 : rn <= 64 ? 2 : 1);
  const int64_t each = T / used;
  const bool two = used > 1 ? 2 * blocks < 5 * sms : blocks > slots && 4 * blocks < 5 * slots;
  int c = two && each >= (rn <= 32 ? 1024 : 2048) ? 2 : 1;
  while (c < lora::kMaxCluster && each >= (rn == 16 ? 512 : 1024) * c && 2 * c * blocks <= slots) c *= 2;
  return c;
}

int check(const polyq_dense* x, int64_t T, const polyq_adapters* ad, const polyq_segments* s, const char* who) {
  if (!ad || !s) return polyq_set_error(POLYQ_EINVAL, "%s: adapters or segments are NULL", who);
  if (T < 1 || T > kMaxSize || ad->K < 1 || ad->K > kMaxSize || ad->N < 1 || ad->N > kMaxSize)
    return polyq_set_error(POLYQ_EINVAL, "%s: T=%lld K=%lld N=%lld", who, (long long)T, (long long)ad->K, (long long)ad->N);
  if (ad->type != POLYQ_BF16 && ad->type != POLYQ_F16)
    return polyq_set_error(POLYQ_EINVAL, "%s: adapters of type %d", who, ad->type);
  if (ad->R < 1 || ad->R % 8)
    return polyq_set_error(POLYQ_EINVAL, "%s: R=%d is not a multiple of 8", who, ad->R);
  if (ad->R > POLYQ_ADAPTERS_MAX_RANK)
    return polyq_set_error(POLYQ_EUNSUPPORTED, "%s: R=%d, at most %d", who, ad->R, POLYQ_ADAPTERS_MAX_RANK);
  if (ad->n < 1 || ad->n > kMaxSize) return polyq_set_error(POLYQ_EINVAL, "%s: %d adapters", who, ad->n);
  if (!ad->a || !ad->b || (uintptr_t)ad->a % 16 || (uintptr_t)ad->b % 16 || ad->a_stride < ad->K ||
      ad->b_stride < ad->R || ad->a_stride % 8 || ad->b_stride % 8 || ad->a_next < 0 || ad->b_next < 0 ||
      ad->a_next % 8 || ad->b_next % 8 || ad->a_stride > (1ll << 32) || ad->b_stride > (1ll << 32) ||
      ad->a_next > (1ll << 40) || ad->b_next > (1ll << 40))
    return polyq_set_error(POLYQ_EINVAL, "%s: a and b must be 16-byte aligned, with strides in multiples of 8 elements "
                           "that hold their rows", who);
  if ((uintptr_t)ad->scales % 4 || (uintptr_t)ad->ranks % 4)
    return polyq_set_error(POLYQ_EINVAL, "%s: scales and ranks must be aligned to their elements", who);
  if (!s->offsets || !s->ids || (uintptr_t)s->offsets % 4 || (uintptr_t)s->ids % 4 || s->n < 1 || s->n > kMaxSize)
    return polyq_set_error(POLYQ_EINVAL, "%s: %d segments; offsets and ids must be given and aligned", who, s->n);
  int rc = polyq_check_dense(x, ad->K, who, "x");
  if (rc) return rc;
  if (x->type != ad->type) return polyq_set_error(POLYQ_EINVAL, "%s: x must be of the adapters' type", who);
  return POLYQ_OK;
}

// An output of x's type or fp32 and what it is added to.
int check_sum(const polyq_dense* y, const polyq_dense* residual, int64_t cols, const polyq_adapters* ad, const char* who,
              const char* what) {
  int rc = polyq_check_dense(y, cols, who, what);
  if (rc) return rc;
  if (y->type != POLYQ_F32 && y->type != ad->type)
    return polyq_set_error(POLYQ_EINVAL, "%s: %s must be of the adapters' type or fp32", who, what);
  if (!residual) return POLYQ_OK;
  rc = polyq_check_dense(residual, cols, who, "residual");
  if (rc) return rc;
  if (residual->type != y->type)
    return polyq_set_error(POLYQ_EINVAL, "%s: the residual must be of %s's type", who, what);
  if (residual->data == y->data && residual->stride != y->stride)
    return polyq_set_error(POLYQ_EINVAL, "%s: a residual in %s's place must have its stride", who, what);
  return POLYQ_OK;
}

constexpr size_t kHead = 256;  // of the workspace: its status word
size_t workspace_size(int64_t T, int R) { return kHead + (size_t)T * R * sizeof(float); }

}  // namespace

extern "C" int polyq_adapters_workspace_bytes(int64_t T, int32_t R, size_t* bytes) {
  polyq_clear_error();
  if (!bytes || T < 1 || T > kMaxSize || R < 1 || R % 8 || R > POLYQ_ADAPTERS_MAX_RANK)
    return polyq_set_error(POLYQ_EINVAL, "polyq_adapters_workspace_bytes: T=%lld R=%d", (long long)T, R);
  *bytes = workspace_size(T, R);
  return POLYQ_OK;
}

extern "C" int polyq_adapters_forward(const polyq_dense* x, int64_t T, const polyq_adapters* adapters,
                                      const polyq_segments* segments, const polyq_dense* residual,
                                      const polyq_dense* y, float* saved, void* workspace, size_t workspace_bytes,
                                      void* stream) {
  static const char* who = "polyq_adapters_forward";
  polyq_clear_error();
  int rc = check(x, T, adapters, segments, who);
  if (!rc) rc = check_sum(y, residual, adapters->N, adapters, who, "y");
  if (rc) return rc;
  if ((uintptr_t)saved % 16 || (uintptr_t)workspace % 16)
    return polyq_set_error(POLYQ_EINVAL, "%s: saved and workspace must be 16-byte aligned", who);
  if (!workspace || workspace_bytes < workspace_size(T, adapters->R))
    return polyq_set_error(POLYQ_ENOMEM, "%s: workspace of %zu bytes needed", who, workspace_size(T, adapters->R));
  float* v = saved ? saved : (float*)((char*)workspace + kHead);
  int sms = 0;
  rc = polyq_sm_count(&sms);
  if (rc) return rc;
  const lora::Segments seg{segments->offsets, segments->ids, segments->n, (int32_t)T};
  rc = shrink(x, T, adapters->K, adapters, false, lora::Side{adapters->a, adapters->a_next, adapters->a_stride}, nullptr,
              seg, v, (int*)workspace, sms, stream, who);
  if (rc) return rc;
  return expand(v, T, adapters->N, adapters, false, lora::Side{adapters->b, adapters->b_next, adapters->b_stride},
                adapters->scales, seg, residual, y, sms, stream, who);
}

extern "C" int polyq_adapters_backward(const polyq_dense* x, int64_t T, const polyq_adapters* adapters,
                                       const polyq_segments* segments, const float* saved, const polyq_dense* dy,
                                       const polyq_dense* residual, const polyq_dense* dx, void* da, void* db,
                                       int32_t grad_type, void* workspace, size_t workspace_bytes, void* stream) {
  static const char* who = "polyq_adapters_backward";
  polyq_clear_error();
  int rc = check(x, T, adapters, segments, who);
  if (!rc) rc = polyq_check_dense(dy, adapters->N, who, "dy");
  if (rc) return rc;
  if (dy->type != adapters->type) return polyq_set_error(POLYQ_EINVAL, "%s: dy must be of the adapters' type", who);
  if (dx) rc = check_sum(dx, residual, adapters->K, adapters, who, "dx");
  if (rc) return rc;
  if (!dx && residual) return polyq_set_error(POLYQ_EINVAL, "%s: a residual needs a dx", who);
  if (!dx && !da && !db) return polyq_set_error(POLYQ_EINVAL, "%s: no gradient is wanted", who);
  if ((da || db) && grad_type != POLYQ_F32 && grad_type != adapters->type)
    return polyq_set_error(POLYQ_EINVAL, "%s: da and db must be of the adapters' type or fp32", who);
  const int eb = grad_type == POLYQ_F32 ? 4 : 2;
  if ((uintptr_t)da % eb || (uintptr_t)db % eb)
    return polyq_set_error(POLYQ_EINVAL, "%s: da and db must be aligned to their elements", who);
  if ((db && !saved) || (uintptr_t)saved % 16 || (uintptr_t)workspace % 16)
    return polyq_set_error(POLYQ_EINVAL, "%s: saved and workspace must be 16-byte aligned, and saved given for db", who);
  const bool needs_dv = dx || da;
  if (needs_dv && (!workspace || workspace_bytes < workspace_size(T, adapters->R)))
    return polyq_set_error(POLYQ_ENOMEM, "%s: workspace of %zu bytes needed", who, workspace_size(T, adapters->R));
  int sms = 0;
  rc = polyq_sm_count(&sms);
  if (rc) return rc;
  const int rn = rank_tile(adapters->R), bc = rn <= 64 ? 128 : 64;
  const bool half = adapters->type == POLYQ_F16;
  const lora::Segments seg{segments->offsets, segments->ids, segments->n, (int32_t)T};
  lora::GradParams G;
  memset(&G, 0, sizeof G);
  G.side[0] = lora::GradSide{(const float*)((const char*)workspace + kHead), x->data, x->stride, adapters->K, da, nullptr, grad_type, 0,
                             da ? (int32_t)((adapters->K + bc - 1) / bc) : 0};
  G.side[1] = lora::GradSide{saved, dy->data, dy->stride, adapters->N, db, adapters->scales, grad_type, 1,
                             db ? (int32_t)((adapters->N + bc - 1) / bc) : 0};
  const int64_t blocks = (int64_t)adapters->n * (G.side[0].tiles + G.side[1].tiles);
  if (blocks > 0x7FFFFFFF / lora::kMaxCluster)
    return polyq_set_error(POLYQ_EUNSUPPORTED, "%s: gradients of %d adapters at once", who, adapters->n);
  float* dv = (float*)((char*)workspace + kHead);
  if (needs_dv) {
    rc = shrink(dy, T, adapters->N, adapters, true, lora::Side{adapters->b, adapters->b_next, adapters->b_stride},
                adapters->scales, seg, dv, (int*)workspace, sms, stream, who);
    if (rc) return rc;
  }
  if (blocks) {
    G.ranks = adapters->ranks;
    G.seg = seg;
    G.R = adapters->R;
    G.cluster = gradient_cluster(T, std::min(adapters->n, segments->n), G.side[0].tiles + G.side[1].tiles, rn, sms);
    const bool any = (da && !rows_on_16(x)) || (db && !rows_on_16(dy));
    const Kernel k = half ? lora::gradients_of<__half>(rn, any) : lora::gradients_of<__nv_bfloat16>(rn, any);
    rc = launch(k, 256 + (any * 2 + half) * 4 + rank_index(rn), dim3((unsigned)(blocks * G.cluster)), lora::kThreads,
                G.cluster, &G, stream, who);
    if (rc) return rc;
  }
  if (!dx) return POLYQ_OK;
  return expand(dv, T, adapters->K, adapters, true, lora::Side{adapters->a, adapters->a_next, adapters->a_stride},
                nullptr, seg, residual, dx, sms, stream, who);
}
