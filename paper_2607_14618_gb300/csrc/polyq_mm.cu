// Products on the tcgen05 tensor cores with both operands as they lie in HBM:
// two 4-bit tensors with block scales (polyq_fp4_linear, polyq_fp4_ffn), or
// 16-bit tensors (polyq_ffn_forward, polyq_ffn_backward).
//
//   D[m][n] = sum_k A[m][k] B[n][k]
//
// Every kind moves 128 bytes of each operand row per stage, four MMAs: 256
// 4-bit or 64 16-bit elements of K.  Two kernels:
//   mm_pair  many rows: persistent CTA pairs (cta_group::2), 256 rows of A by 256
//            of B a tile, A the tokens, B the weights.
//   mm_few   few tokens: the weights are A (128 rows a CTA), the tokens B; the
//            CTAs of a cluster share the contraction and add their parts through
//            distributed shared memory, in rank order.
// GATED kernels hold gate and up side by side in tensor memory, so that one
// thread has both values of an output and applies the activation and the
// product in registers.  Every wait is bounded and reports through the
// workspace status word.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>

#include "polyq_dev.cuh"
#include "polyq_fp4_dev.cuh"
#include "polyq_internal.h"
#include "polyq_tc.cuh"

namespace {

using namespace polyq;
using namespace polyq::tc;

constexpr int k16 = 0, kMx = 1, kNv = 2;  // operand kinds
constexpr int kTileM = 256, kTileN = 256;  // rows of A and of B of a pair's tile
constexpr int kHalf = 128;                // of each of which a CTA holds half
constexpr int kRowBytes = 128;            // an operand row in a stage
constexpr int kOpBytes = kHalf * kRowBytes;
constexpr int kSmemMax = 227 * 1024 - 1024;  // less the static barriers
constexpr int kMaxDevices = 64;

// Division of 32-bit numbers by a d known at launch: n / d is the upper half of
// n * ceil(2^64 / d), exact for every n (Lemire, Kaser, Kurz: Faster remainder by
// direct computation, 2019).  mul is 0 for d = 1.
struct Divisor {
  uint64_t mul;
  __host__ void set(uint32_t d) { mul = d > 1 ? ~0ull / d + 1 : 0; }
  __device__ __forceinline__ int of(int n) const { return mul ? (int)__umul64hi(mul, (uint64_t)(uint32_t)n) : n; }
};

struct MmParams {
  CUtensorMap a[2], b[2];  // operand tiles (per segment, problem or matrix, see below)
  CUtensorMap sa, sb[2];   // scales, rows of one atom
  int M, N;                // output rows (A) and columns (B), of one problem
  int kt, k_last;          // stages of a segment, MMAs of its last stage
  int segs;                // segments of the contraction: a[s] with b[s]
  int probs;               // problems: a[p] with b[0]
  int tiles_m, tiles_n, tiles;
  Divisor per_prob, per_band, last_band;  // by tiles of a problem, of eight row tiles, by rows of the last band
  // mm_pair: the first sk_tiles tiles are shared along the contraction by the
  // pairs b < sk_pairs: sk_parts pairs a tile (even parts), or with sk_parts 0
  // all of their stages in tile order, sk_share a pair (the first sk_extra pairs
  // one more).  The other tiles are whole, strided over the pairs.
  int sk_tiles, sk_pairs, sk_parts, sk_share, sk_extra;
  int grid_pairs;
  float* parts;            // [2 pairs][64][256 rows][4 columns]: parts of shared tiles
  int* counters;           // [sk_tiles][2 CTAs][warps]: parts in place
  int a_mn, b_mn;          // operand has M (N) contiguous instead of K
  int atoms;               // scale atoms of a row group
  uint32_t idesc;
  float alpha[2];          // tensor scales of the result (GATED: of gate, of up)
  // outputs: y[p], of `type`; or 4 bits; and the saved gate and up values
  void* y[2];
  const void* res;
  int64_t y_stride, res_stride;
  int type, vec;           // vec: rows of y and res start on 8 (1), 16 (2) or 32 bytes (3)
  uint8_t *codes, *scales;
  int64_t code_stride, out_atoms;
  int qfmt;                // 0, kMx or kNv
  float g, inv_g;
  uint8_t* saved;          // see save_row32
  int64_t saved_stride;
  int* status;
};

__device__ __forceinline__ float silu(float a) { return __fdividef(a, 1.f + __expf(-a)); }

__device__ __forceinline__ uint32_t pack16(float lo, float hi, bool bf16) {
  if (bf16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ void from_f32(float v, float* p) { *p = v; }
__device__ __forceinline__ void from_f32(float v, __nv_bfloat16* p) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void from_f32(float v, __half* p) { *p = __float2half_rn(v); }
__device__ __forceinline__ float load_dense(const void* p, int64_t i, int type) {
  return type == POLYQ_F32    ? ((const float*)p)[i]
         : type == POLYQ_BF16 ? __bfloat162float(((const __nv_bfloat16*)p)[i])
                              : __half2float(((const __half*)p)[i]);
}
__device__ __forceinline__ void store_dense(void* p, int64_t i, float v, int type) {
  if (type == POLYQ_F32) ((float*)p)[i] = v;
  else if (type == POLYQ_BF16) ((__nv_bfloat16*)p)[i] = __float2bfloat16_rn(v);
  else ((__half*)p)[i] = __float2half_rn(v);
}
// Rows that start on 32 (vec = 3), 16 (2) or 8 bytes (1): a lane holds 32
// consecutive values of its row and stores whole sectors, or 8 bytes at a time.
__device__ __forceinline__ void store32(void* p, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
               "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
__device__ __forceinline__ void store32(void* p, const uint32_t (&w)[8], int vec) {
  if (vec == 3) {
    store32(p, w);
  } else if (vec == 2) {
    reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<uint2*>(p)[i] = make_uint2(w[2 * i], w[2 * i + 1]);
  }
}
__device__ __forceinline__ void store_row32(void* y, int64_t off, const float (&v)[32], int type, int vec) {
  uint32_t w[8];
  if (type == POLYQ_F32) {
#pragma unroll
    for (int i = 0; i < 32; i += 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[i + j]);
      store32((float*)y + off + i, w, vec);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; i += 16) {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = pack16(v[i + 2 * j], v[i + 2 * j + 1], type == POLYQ_BF16);
      store32((uint16_t*)y + off + i, w, vec);
    }
  }
}
// The lane's 32 consecutive residual values as they lie in memory (16-bit types:
// the first half of w), and their sum with v.  Ordinary loads, also where the
// launch before writes the residual: every thread that reads one has waited for
// that launch, and the wait makes its writes visible to them.
__device__ __forceinline__ void load_row32(const void* r, int64_t off, uint32_t (&w)[32], int type, int vec) {
  const uint8_t* p = (const uint8_t*)r + off * (type == POLYQ_F32 ? 4 : 2);
#pragma unroll
  for (int i = 0; i < 32; i += 8) {
    if (i == 16 && type != POLYQ_F32) break;
    if (vec == 3) {
      asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                   : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]), "=r"(w[i + 4]), "=r"(w[i + 5]),
                     "=r"(w[i + 6]), "=r"(w[i + 7])
                   : "l"(p + 4 * i)
                   : "memory");
    } else {
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        const uint2 u = *reinterpret_cast<const uint2*>(p + 4 * (i + j));
        w[i + j] = u.x;
        w[i + j + 1] = u.y;
      }
    }
  }
}
__device__ __forceinline__ void add_row32(const uint32_t (&w)[32], float (&v)[32], int type) {
  if (type == POLYQ_F32) {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] += __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float2 f;
      if (type == POLYQ_BF16) f = make_float2(bf16_lo(w[i]), bf16_hi(w[i]));
      else f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      v[2 * i] += f.x;
      v[2 * i + 1] += f.y;
    }
  }
}
// The values of gate and up that the backward pass needs are saved as 24 bits of
// fp32, rounded to nearest (16 significant bits, off by at most 2^-16 of the value,
// and fp32's range): with 16-bit types their rounding was most of the
// gradients' error (relative 0.0030, now 0.0024, where rounding the plain form's
// result once gives 0.0017).  Four planes of M rows of `stride` elements: the
// upper 16 bits of gate and of up, the next 8 of gate and of up; `which` is 0 for
// gate.  Rows are padded to 32 elements, so whole chunks of 32 always fit.
__device__ __forceinline__ uint8_t* saved_hi(const MmParams& P, int which, int64_t i) {
  return P.saved + 2 * ((int64_t)which * P.M * P.saved_stride + i);
}
__device__ __forceinline__ uint8_t* saved_lo(const MmParams& P, int which, int64_t i) {
  return P.saved + (4 + which) * (int64_t)P.M * P.saved_stride + i;
}
// Those 24 bits are the upper ones of this.  NaN and infinities stay as they are,
// and numbers next to the largest, which would become infinities.
__device__ __forceinline__ uint32_t round24(uint32_t v) {
  return fabsf(__uint_as_float(v)) < __uint_as_float(0x7F7FFF80u) ? v + 0x80u : v;
}
__device__ __forceinline__ void save_row32(const MmParams& P, int which, int64_t m, int n, const uint32_t (&r)[32]) {
  const int64_t at = m * P.saved_stride + n;
  uint32_t v[32], w[8];
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = round24(r[i]);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __byte_perm(v[16 * h + 2 * i], v[16 * h + 2 * i + 1], 0x7632);
    store32(saved_hi(P, which, at + 16 * h), w);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    w[i] = __byte_perm(__byte_perm(v[4 * i], v[4 * i + 1], 0x0051), __byte_perm(v[4 * i + 2], v[4 * i + 3], 0x0051), 0x5410);
  store32(saved_lo(P, which, at), w);
}

// The warp's 32 x 32 values transposed: v[r] of lane c becomes v[c] of lane r.
__device__ __forceinline__ void transpose32(float (&v)[32]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int d = 16; d >= 1; d /= 2)
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (!(i & d)) {
        const bool hi = lane & d;
        const float got = __shfl_xor_sync(0xffffffffu, hi ? v[i] : v[i | d], d);
        if (hi) v[i] = got;
        else v[i | d] = got;
      }
}
// The first `rows` values of a lane's column, of a matrix whose lanes' columns
// are neighbours.
template <typename T>
__device__ __forceinline__ void store_column(T* y, int64_t stride, const T* res, int64_t res_stride, int rows,
                                             const float (&v)[32]) {
#pragma unroll
  for (int r = 0; r < 32; ++r)
    if (r < rows) {
      const float f = res ? v[r] + to_f32(res[r * res_stride]) : v[r];
      from_f32(f, y + r * stride);
    }
}
// 32 values of each of the warp's 32 rows m.. from column n, of a matrix of M
// by N.  Whole chunks of aligned rows go lane by lane; others (rows of odd
// strides, the last columns) are transposed first, so that the lanes' elements
// are neighbours: 301 x 2731 fp16 took 31 us with a lane's 32 elements of two
// bytes stored one by one, 15 us so.
__device__ __forceinline__ void store_chunk(void* y, int64_t stride, const void* res, int64_t res_stride, int64_t m,
                                            int n, int64_t M, int64_t N, float (&v)[32], int type, int vec) {
  const int lane = threadIdx.x & 31;
  if (vec && n + 32 <= N) {  // (the residual has been added)
    if (m + lane < M) store_row32(y, (m + lane) * stride + n, v, type, vec);
  } else {
    transpose32(v);
    const int rows = n + lane < N ? (int)min((int64_t)32, M - m) : 0;
    const int64_t at = m * stride + n + lane, from = m * res_stride + n + lane;
    if (type == POLYQ_F32)
      store_column((float*)y + at, stride, res ? (const float*)res + from : nullptr, res_stride, rows, v);
    else if (type == POLYQ_BF16)
      store_column((__nv_bfloat16*)y + at, stride, res ? (const __nv_bfloat16*)res + from : nullptr, res_stride, rows, v);
    else
      store_column((__half*)y + at, stride, res ? (const __half*)res + from : nullptr, res_stride, rows, v);
  }
}

// 32 consecutive values of row m from column f0 (a multiple of 32) as one block
// of 32 or two of 16; values past the row's end are 0.
template <bool NV>
__device__ __forceinline__ void store_codes32(const MmParams& P, int64_t m, int64_t f0, float (&v)[32]) {
  uint32_t c[4];
  constexpr int BL = NV ? 16 : 32;
#pragma unroll
  for (int b = 0; b < 32 / BL; ++b) {
    uint32_t mx = 0;
#pragma unroll
    for (int i = 0; i < BL; ++i) {
      if (NV) v[BL * b + i] = P.inv_g != 0.f ? v[BL * b + i] * P.inv_g : __fdiv_rn(v[BL * b + i], P.g);
      mx = max(mx, __float_as_uint(v[BL * b + i]) & 0x7FFFFFFFu);
    }
    const fp4::Scale<NV> sc(mx);
#pragma unroll
    for (int i = 0; i < BL / 8; ++i) {
      float t[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) t[j] = v[BL * b + 8 * i + j];
      c[b * BL / 8 + i] = sc.codes(t);
    }
    const int64_t blk = f0 / BL + b;
    if (blk >> 2 < P.out_atoms) P.scales[fp4::scale_off(m, blk, P.out_atoms)] = (uint8_t)sc.byte;
  }
  // rows are padded to 16 bytes: a chunk that starts inside the row fits
  if (f0 < P.N) *reinterpret_cast<uint4*>(P.codes + m * P.code_stride + f0 / 2) = make_uint4(c[0], c[1], c[2], c[3]);
}

// ---------------------------------------------------------------------------
// many rows: CTA pairs
// ---------------------------------------------------------------------------
template <int KIND_, bool GATED_>
struct Pair {
  static constexpr int KIND = KIND_;
  static constexpr bool GATED = GATED_;
  static constexpr int MATS = GATED ? 2 : 1;
  static constexpr int ATOMS = KIND == k16 ? 0 : KIND == kNv ? 4 : 2;  // scale atoms of a stage
  static constexpr int kSa = ATOMS * 512, kSb = ATOMS * 1024;          // of A's 128 rows, of B's 256
  static constexpr int kStage = 2 * kOpBytes + kSa + kSb;
  static constexpr int STAGES = (kSmemMax - 1024) / kStage;
  static constexpr int kBOff = STAGES * kOpBytes, kSaOff = kBOff + STAGES * kOpBytes;
  static constexpr int kSbOff = kSaOff + STAGES * kSa;
  static constexpr size_t kSmem = (size_t)STAGES * kStage + 1024;
  // Tensor memory: two accumulators of 256 columns and SF stages' scales.  With
  // scales the accumulators share OV columns: the epilogue drains those first
  // and releases them for the next tile before the rest.
  static constexpr int SF = KIND == kNv ? 2 : 3;
  static constexpr int kSfStage = ATOMS * 4 * 3;
  static constexpr int kSfCols = (SF * kSfStage + 31) / 32 * 32;
  static constexpr int kSfCol = 512 - kSfCols;
  static constexpr int kAcc1 = kSfCol - kTileN;
  static constexpr int OV = kTileN - kAcc1;
  // EPI epilogue warps, EPQ to a quarter of the lanes, as measured with 12 / 8 / 4
  // (calls one after another over one set of operands): gradients of the weights
  // of 64 tokens with da and du, 5120 / 13824, 69.9 / 69.0 / 71.2 us, in fp32 129.9
  // / 130.9 / 131.1; 16-bit gated and saved, 1086 x 5504 x 384, 20.1 / 18.7 / 20.2;
  // gated 2048 x 13824 x 5120, NV 98.6 / 103.5 / 105.1, MX 90.7 / 95.6 / 96.4.
  static constexpr int kEpiWarp = 4, EPI = GATED && KIND != k16 ? 12 : 8, EPQ = EPI / 4;
  static constexpr int kThreads = 32 * (kEpiWarp + EPI);
  static_assert(OV % 32 == 0 && STAGES >= 4, "");
};
constexpr int kEpiWarps = 12;  // the most

// The pieces of work of a pair, in order: a tile and the stages [lo, hi) of its
// contraction; the pair's share of the shared tiles comes first.  Tiles of eight
// row tiles are taken together, rows fastest, so that the pairs at work share
// both operands through L2.
struct Tiles {
  int g, g_hi, t;         // shared stages; next whole tile
  int tile, lo, hi, prob, tm, tn;
  int shared, parts, own; // of a part: its tile, the tile's parts, which one it is; else shared is -1
  // The first shared stage of pair b, and the pair that has shared stage x.
  static __device__ __forceinline__ int share_of(const MmParams& P, int b) {
    if (P.sk_parts == 0) return b * P.sk_share + min(b, P.sk_extra);
    const int n_it = P.segs * P.kt, tile = b / P.sk_parts;
    return tile * n_it + (int)((int64_t)(b - tile * P.sk_parts) * n_it / P.sk_parts);
  }
  static __device__ __forceinline__ int pair_of(const MmParams& P, int x) {
    if (P.sk_parts == 0) {
      const int y = x - P.sk_extra * (P.sk_share + 1);
      return y < 0 ? x / (P.sk_share + 1) : P.sk_extra + y / P.sk_share;
    }
    const int n_it = P.segs * P.kt, tile = x / n_it;
    return tile * P.sk_parts + (int)(((int64_t)(x - tile * n_it + 1) * P.sk_parts - 1) / n_it);
  }
  __device__ __forceinline__ void init(const MmParams& P) {
    const int b = (int)(blockIdx.x >> 1);
    g = g_hi = 0;
    if (b < P.sk_pairs) {
      g = share_of(P, b);
      g_hi = share_of(P, b + 1);
    }
    t = P.sk_tiles + b;
  }
  __device__ __forceinline__ bool next(const MmParams& P) {
    const int n_it = P.segs * P.kt;
    lo = 0;
    hi = n_it;
    shared = -1;
    own = 0;
    if (g < g_hi) {
      tile = g / n_it;
      lo = g - tile * n_it;
      hi = min(n_it, lo + (g_hi - g));
      g += hi - lo;
      if (hi - lo < n_it) {
        const int p0 = pair_of(P, tile * n_it);
        shared = tile;
        parts = pair_of(P, tile * n_it + n_it - 1) - p0 + 1;
        own = (int)(blockIdx.x >> 1) - p0;
      }
    } else {
      if (t >= P.tiles) return false;
      tile = t;
      t += (int)(gridDim.x >> 1);
    }
    return true;
  }
  // Where the piece's tile lies.  (Each warp of the epilogue asks before it waits
  // for the tile, which is on the way where a tile has few stages.)
  __device__ __forceinline__ void place(const MmParams& P) {
    prob = P.per_prob.of(tile);
    const int r = tile - prob * (P.tiles_m * P.tiles_n);
    const int q = P.per_band.of(r), i = r - q * 8 * P.tiles_n;
    const bool whole = 8 * q + 8 <= P.tiles_m;
    tn = whole ? i >> 3 : P.last_band.of(i);
    tm = 8 * q + (i - tn * (whole ? 8 : P.tiles_m - 8 * q));
  }
  // Where part p of the tile lies: a pair has two slots, the second for a tile
  // that its share did not begin in.
  __device__ __forceinline__ int slot(const MmParams& P, int p) const {
    const int b = (int)(blockIdx.x >> 1) - own + p;
    return 2 * b + (share_of(P, b) < shared * (P.segs * P.kt));
  }
};

template <class C>
__global__ void __launch_bounds__(C::kThreads, 1) mm_pair(const __grid_constant__ MmParams P) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~(uintptr_t)1023);
  __shared__ uint64_t bar_full[C::STAGES];   // leader: both CTAs' copies of a stage have landed
  __shared__ uint64_t bar_empty[C::STAGES];  // a stage's MMAs are done
  __shared__ uint64_t bar_accf[2];           // an accumulator is complete
  __shared__ uint64_t bar_acce[2];           // leader: both CTAs have drained it (OV: what is shared)
  __shared__ uint64_t bar_done;              // every MMA is done
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int s_abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();

  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int s = 0; s < C::STAGES; ++s) {
      mbar_init(smem_u32(&bar_full[s]), 1);
      mbar_init(smem_u32(&bar_empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&bar_accf[b]), 1);
      mbar_init(smem_u32(&bar_acce[b]), 2 * C::EPI);
    }
    mbar_init(smem_u32(&bar_done), 1);
    mbar_fence_init();
  }
  if (warp == 1) {
    tmem_alloc<2>(smem_u32(&tmem_slot), 512);
    tmem_relinquish<2>();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_trigger();

  // A role gives up: both CTAs stop, and this one stays a thousand times the
  // time of a copy, so that none lands after its CTA has left.
  auto fail = [&](int code) {
    s_abort = 1;
    const uint32_t peer = mapa(smem_u32((const void*)&s_abort), rank ^ 1u);
    asm volatile("st.relaxed.cluster.shared::cluster.u32 [%0], %1;" ::"r"(peer), "r"(1) : "memory");
    atomicExch(P.status, code);
    for (const long long t0 = clock64(); clock64() - t0 < kStayCycles;) __nanosleep(1000);
  };
  Tiles T;
  T.init(P);

  if (warp == 0) {
    // ---------------- producer: this CTA's half of A, of B, and the scales ----------------
    if (elect_one()) {
      pdl_wait();
      int s = 0;
      uint32_t ph = 1;
      const uint32_t full0 = mapa(smem_u32(&bar_full[0]), 0);
      bool more = T.next(P);
      if (more) T.place(P);
      while (more && !s_abort) {
        const int m0 = T.tm * kTileM + (int)rank * kHalf, prob = T.prob, tn = T.tn, lo = T.lo, hi = T.hi;
        const int n0 = C::GATED ? tn * kHalf : tn * kTileN + (int)rank * kHalf;
        for (int i = lo; i < hi; ++i) {
          const int w = wait(smem_u32(&bar_empty[s]), ph, &s_abort);
          if (w != kOk) {
            if (w == kTimeout) fail(kStatusTimeoutEmpty);
            break;
          }
          const int seg = i >= P.kt, kt = seg ? i - P.kt : i;
          if (rank == 0) mbar_expect_tx(smem_u32(&bar_full[s]), 2 * C::kStage);
          const uint32_t bar = full0 + 8 * s;
          const uint32_t da = smem_u32(smem + s * kOpBytes);
          const uint32_t db = smem_u32(smem + C::kBOff + s * kOpBytes);
          const CUtensorMap* ma = &P.a[C::GATED ? 0 : seg + prob];
          const CUtensorMap* mb = &P.b[C::GATED ? (int)rank : seg];
          if (C::KIND == k16) {
            if (!P.a_mn) {
              tma_load_2d_pair(da, ma, kt * 64, m0, bar);
            } else {
              tma_load_2d_pair(da, ma, m0, kt * 64, bar);
              tma_load_2d_pair(da + 8192, ma, m0 + 64, kt * 64, bar);
            }
            if (!P.b_mn) {
              tma_load_2d_pair(db, mb, kt * 64, n0, bar);
            } else {
              tma_load_2d_pair(db, mb, n0, kt * 64, bar);
              tma_load_2d_pair(db + 8192, mb, n0 + 64, kt * 64, bar);
            }
          } else {
            tma_load_2d_pair(da, ma, kt * kRowBytes, m0, bar);
            tma_load_2d_pair(db, mb, kt * kRowBytes, n0, bar);
            const uint32_t sa = smem_u32(smem + C::kSaOff + s * C::kSa);
            const uint32_t sb = smem_u32(smem + C::kSbOff + s * C::kSb);
            tma_load_2d_pair(sa, &P.sa, 0, (m0 / 128) * P.atoms + kt * C::ATOMS, bar);
#pragma unroll
            for (int j = 0; j < 2; ++j)
              tma_load_2d_pair(sb + j * C::ATOMS * 512, &P.sb[C::GATED ? j : 0], 0,
                               (C::GATED ? tn : tn * 2 + j) * P.atoms + kt * C::ATOMS, bar);
          }
          if (++s == C::STAGES) {
            s = 0;
            ph ^= 1u;
          }
          if (i == lo) {
            more = T.next(P);
            if (more) T.place(P);
          }
        }
      }
    }
  } else if (warp == 1 && rank == 0) {
    // ---------------- MMA issuer (leader CTA) ----------------
    if (elect_one()) {
      int s = 0, tc = 0;
      bool ready = false;            // stage s is known to have landed
      int sf = 0, so = 0, held = 0;  // scales: next slot; the oldest stage in use, and how many are
      int freed = 0;                 // and how many of them were found done
      uint32_t ph = 0, so_ph = 0;
      const uint64_t a0 = desc_sw128(smem_u32(smem), P.a_mn ? 8192 : 16);
      const uint64_t b0 = desc_sw128(smem_u32(smem + C::kBOff), P.b_mn ? 8192 : 16);
      const uint64_t sa0 = desc_scales(smem_u32(smem + C::kSaOff));
      const uint64_t sb0 = desc_scales(smem_u32(smem + C::kSbOff));
      // K = 16 of 16-bit elements: 32 bytes on in a K-major row, 16 rows on otherwise
      const int a_step = P.a_mn ? 2048 >> 4 : 32 >> 4, b_step = P.b_mn ? 2048 >> 4 : 32 >> 4;
      for (; !s_abort && T.next(P); ++tc) {
        const int buf = tc & 1;
        int w = kOk, why = kStatusTimeoutEmpty;
        const uint32_t acc = tmem + (buf ? C::kAcc1 : 0);
        for (int i = T.lo; i < T.hi; ++i) {
          if (!ready) {
            w = wait(smem_u32(&bar_full[s]), ph, &s_abort);
            if (w != kOk) {
              why = kStatusTimeoutFull;
              break;
            }
          }
          tc_fence_after();
          // asked for here, needed when this stage's MMAs have been issued: a
          // poll's answer takes 250 to 300 cycles beside the tensor core's traffic
          const int s1 = s + 1 == C::STAGES ? 0 : s + 1;
          const uint32_t ph1 = s1 == 0 ? ph ^ 1u : ph;
          ready = mbar_test(smem_u32(&bar_full[s1]), ph1);
          auto release = [&](int n) {
            held -= n;
            so += n;
            if (so >= C::STAGES) {
              so -= C::STAGES;
              so_ph ^= 1u;
            }
          };
          if (C::KIND != k16) {
            if (C::SF > 2) release(freed);  // asked for a stage ago: the answer is not waited for
            freed = min(held, poll_ahead<2, C::STAGES>(smem_u32(&bar_empty[0]), so, so_ph));
            if (C::SF == 2) release(freed);
          }
          const int kt = i >= P.kt ? i - P.kt : i;
          const int n_mma = kt == P.kt - 1 ? P.k_last : 4;
          const uint64_t a = a0 + (uint64_t)((s * kOpBytes) >> 4), b = b0 + (uint64_t)((s * kOpBytes) >> 4);
          // the accumulator's columns, of a tile's first stage
          auto columns = [&]() {
            if (i != T.lo) return true;
            if (C::OV > 0) {
              if (tc >= 1) w = wait(smem_u32(&bar_acce[0]), (tc - 1) & 1, &s_abort);
            } else if (tc >= 2) {
              w = wait(smem_u32(&bar_acce[buf]), ((tc >> 1) - 1) & 1, &s_abort);
            }
            tc_fence_after();
            return w == kOk;
          };
          if constexpr (C::KIND == k16) {
            if (!columns()) break;
            for (int kk = 0; kk < n_mma; ++kk)
              mma_16<2>(acc, a + (uint64_t)(kk * a_step), b + (uint64_t)(kk * b_step), P.idesc, i > T.lo || kk > 0);
          } else {
            constexpr bool NV = C::KIND == kNv;
            const uint64_t sa = sa0 + (uint64_t)((s * C::kSa) >> 4), sb = sb0 + (uint64_t)((s * C::kSb) >> 4);
            if (held == C::SF) {  // a slot's scales stay until its stage's MMAs are done
              w = wait(smem_u32(&bar_empty[so]), so_ph, &s_abort);
              if (w != kOk) break;
              release(1);
              freed = 0;
            }
            const uint32_t c0 = tmem + C::kSfCol + sf * C::kSfStage;
#pragma unroll
            for (int q = 0; q < C::ATOMS; ++q) {
              const uint32_t c = c0 + q * 12;
              copy_scales<2>(c, sa + (uint64_t)(q * 32));
#pragma unroll
              for (int j = 0; j < 2; ++j)
                copy_scales<2>(c + 4 + 4 * j, sb + (uint64_t)((j * C::ATOMS + q) * 32));
            }
            if (!columns()) break;  // (the scales are on their way meanwhile)
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
              if (kk >= n_mma) break;
              const uint32_t c = c0 + (NV ? kk : kk >> 1) * 12;
              mma_fp4<2, NV>(acc, a + (uint64_t)(2 * kk), b + (uint64_t)(2 * kk),
                             NV || !(kk & 1) ? P.idesc : P.idesc | idesc_fp4(0, 0, false, 2), c, c + 4, i > T.lo || kk > 0);
            }
            if (++sf == C::SF) sf = 0;
            ++held;
          }
          commit<2>(smem_u32(&bar_empty[s]));
          s = s1;
          ph = ph1;
        }
        if (w == kTimeout) fail(why);
        commit<2>(smem_u32(&bar_accf[buf]));
      }
      // the pair's shared and tensor memory stay in use until the last MMA is done
      commit<2>(smem_u32(&bar_done));
      wait_stay(smem_u32(&bar_done), 0);
    }
  } else if (warp == 1) {
    // The leader's commits arrive in this CTA's shared memory too, where no
    // role waits for those of the last stages: stay for the last of all.
    if (elect_one()) wait_stay(smem_u32(&bar_done), 0);
  } else if (warp >= C::kEpiWarp) {
    // ---------------- epilogue: a lane owns a row of the tile ----------------
    const int q = warp & 3, e0 = (warp - C::kEpiWarp) >> 2;
    const uint32_t acce0 = mapa(smem_u32(&bar_acce[0]), 0);
    constexpr int kChunks = C::GATED ? kTileN / 64 : kTileN / 32;
    constexpr int kOvChunks = C::OV / 32;
    pdl_wait();
    for (int tc = 0; T.next(P); ++tc) {
      T.place(P);
      const int buf = tc & 1;
      const int64_t m = (int64_t)T.tm * kTileM + (int)rank * kHalf + 32 * q;  // the warp's first row
      const int n0 = C::GATED ? T.tn * kHalf : T.tn * kTileN;
      // A warp's i-th chunk (GATED: of gate, and of up): the columns that the
      // accumulators share are the first one's last and the second one's first.
      auto chunk = [&](int i) { return C::OV > 0 && buf == 0 && T.shared < 0 ? kChunks - 1 - i : i; };
      // A chunk's residual is asked for before its accumulator is complete, the
      // next chunk's before this one's stores (512 x 5120 x 13824 MX: 28.2 us with
      // loads of 8 bytes when they are needed, 23.5 so, 22.6 without a residual).
      constexpr bool RES = !C::GATED && C::KIND != k16;  // may have a residual
      uint32_t res[RES ? 32 : 1];
      auto fetch_res = [&](int c) {
        if constexpr (RES) {
          const int n = n0 + 32 * c;
          if (P.res && P.vec && n + 32 <= P.N && m + lane < P.M)
            load_row32(P.res, (m + lane) * P.res_stride + n, res, P.type, P.vec);
        }
      };
      fetch_res(chunk(e0));
      // The warp goes on or gives up as a whole, whatever its lanes' polls saw: the
      // loads of tensor memory, and its other steps together, are by all lanes.  (A
      // second vote, on s_abort at the loop's head: 8192 x 5120 x 13824 MX +1.8%.)
      const int w = wait(smem_u32(&bar_accf[buf]), (tc >> 1) & 1, &s_abort);
      if (!__all_sync(0xffffffffu, w == kOk)) {
        if (w == kTimeout) fail(kStatusTimeoutFull);
        break;
      }
      tc_fence_after();
      const uint32_t t0 = tmem + ((uint32_t)(32 * q) << 16) + (buf ? C::kAcc1 : 0);
      bool released = false;
      auto release = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(acce0 + (C::OV > 0 ? 0 : 8 * buf));
        released = true;
      };
      // a chunk's outputs from its accumulators (GATED: of gate and of up)
      auto finish = [&](int c, int next, uint32_t (&r0)[32], uint32_t (&r1)[C::GATED ? 32 : 1]) {
        const int n = n0 + 32 * c;
        float v[32];
        if constexpr (C::GATED) {
          if (C::KIND == k16 && P.saved && m + lane < P.M && n < P.N) {
            save_row32(P, 0, m + lane, n, r0);
            save_row32(P, 1, m + lane, n, r1);
          }
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 32; ++j)
            v[j] = silu(__uint_as_float(r0[j]) * P.alpha[0]) * (__uint_as_float(r1[j]) * P.alpha[1]);
          if (C::KIND != k16 && P.qfmt) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = n + j < P.N ? v[j] : 0.f;
            if (m + lane >= P.M) return;
            if (P.qfmt == kNv) store_codes32<true>(P, m + lane, n, v);
            else store_codes32<false>(P, m + lane, n, v);
            return;
          }
          store_chunk(P.y[0], P.y_stride, nullptr, 0, m, n, P.M, P.N, v, P.type, P.vec);
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r0[j]) * P.alpha[0];
          if constexpr (RES) {
            if (P.res && P.vec && n + 32 <= P.N) add_row32(res, v, P.type);
            if (next < kChunks) fetch_res(chunk(next));
          }
          store_chunk(P.y[T.prob], P.y_stride, RES ? P.res : nullptr, P.res_stride, m, n, P.M, P.N, v, P.type, P.vec);
        }
      };
      auto load = [&](int c, uint32_t (&r0)[32], uint32_t (&r1)[C::GATED ? 32 : 1]) {
        tc_ld_32x32b_x32(t0 + 32 * c, r0);
        if constexpr (C::GATED) tc_ld_32x32b_x32(t0 + kHalf + 32 * c, r1);
        tc_wait_ld();
        tc_regs_ready(r0);
        tc_regs_ready(r1);
      };
      // whether a chunk has an output (4 bits: a scale or a code) of this matrix
      auto inside = [&](int c) { return m < P.M && ((C::GATED && C::KIND != k16 && P.qfmt != 0) || n0 + 32 * c < P.N); };
      // A part goes into its slot; the warp that finds the other parts of its
      // chunks in place adds them all, in the order of the pairs.
      auto part = [&](int slot, int col) {  // 4 columns of the lane's row
        return reinterpret_cast<float4*>(P.parts) + ((int64_t)slot * (kTileN / 4) + col / 4) * kTileM +
               (int)rank * kHalf + 32 * q + lane;
      };
      auto put = [&](int slot, int col, const uint32_t (&r)[32]) {
        float4* d = part(slot, col);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          __stcg(d + j * kTileM, make_float4(__uint_as_float(r[4 * j]), __uint_as_float(r[4 * j + 1]),
                                             __uint_as_float(r[4 * j + 2]), __uint_as_float(r[4 * j + 3])));
      };
      auto add = [&](int slot, int col, uint32_t (&r)[32]) {
        const float4* d = part(slot, col);
        float4 f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = __ldcg(d + j * kTileM);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          r[4 * j] = __float_as_uint(__uint_as_float(r[4 * j]) + f[j].x);
          r[4 * j + 1] = __float_as_uint(__uint_as_float(r[4 * j + 1]) + f[j].y);
          r[4 * j + 2] = __float_as_uint(__uint_as_float(r[4 * j + 2]) + f[j].z);
          r[4 * j + 3] = __float_as_uint(__uint_as_float(r[4 * j + 3]) + f[j].w);
        }
      };
      const int slot0 = T.shared >= 0 ? T.slot(P, T.own) : 0;
      int mine = 1;
      if (T.shared >= 0) {
#pragma unroll 1
        for (int j = 0, i; (i = e0 + j / C::MATS * C::EPQ) < kChunks; ++j) {
          const int c = chunk(i), col = 32 * c + j % C::MATS * kHalf;
          if (!inside(c)) continue;
          uint32_t r[32];
          tc_ld_32x32b_x32(t0 + col, r);
          tc_wait_ld();
          tc_regs_ready(r);
          if (m + lane < P.M) put(slot0, col, r);
          __syncwarp();
        }
        __threadfence();
        __syncwarp();
        if (lane == 0) {
          int* counter = P.counters + (T.shared * 2 + (int)rank) * C::EPI + (warp - C::kEpiWarp);
          mine = atomicAdd(counter, 1) == T.parts - 1;
          if (mine) *counter = 0;  // for the next launch
        }
        mine = __shfl_sync(0xffffffffu, mine, 0);
        __threadfence();
        if (mine) {  // the sums back into tensor memory
#pragma unroll 1
          for (int j = 0, i; (i = e0 + j / C::MATS * C::EPQ) < kChunks; ++j) {
            const int c = chunk(i), col = 32 * c + j % C::MATS * kHalf;
            if (!inside(c)) continue;
            uint32_t r[32] = {};
#pragma unroll 1
            for (int p = 0; p < T.parts; ++p) {
              if (p != T.own) {
                if (m + lane < P.M) add(T.slot(P, p), col, r);
                __syncwarp();
              } else {
                uint32_t f[32];
                tc_ld_32x32b_x32(t0 + col, f);
                tc_wait_ld();
                tc_regs_ready(f);
#pragma unroll
                for (int k = 0; k < 32; ++k) r[k] = __float_as_uint(__uint_as_float(r[k]) + __uint_as_float(f[k]));
              }
            }
            tmem_st32(t0 + col, r);
          }
        }
      }
      if (mine) {
#pragma unroll 1
        for (int i = e0; i < kChunks; i += C::EPQ) {
          const int c = chunk(i);
          __syncwarp();  // (lanes without a row, or a residual, come on their own)
          uint32_t r0[32], r1[C::GATED ? 32 : 1];
          load(c, r0, r1);
          if (C::OV > 0 && !released && T.shared < 0 && i + C::EPQ >= kOvChunks) release();
          if (inside(c)) finish(c, i + C::EPQ, r0, r1);
          else if (i + C::EPQ < kChunks) fetch_res(chunk(i + C::EPQ));
        }
      }
      __syncwarp();
      if (!released) release();
    }
  }

  __syncthreads();
  cluster_sync();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc<2>(tmem, 512);
  }
  cluster_sync();
}

// ---------------------------------------------------------------------------
// few tokens: weights as the rows of A, the contraction shared by a cluster
// ---------------------------------------------------------------------------
constexpr int kMaxSplit = 8;

template <int KIND_, int NT_, bool GATED_>
struct Few {
  static constexpr int KIND = KIND_, NT = NT_;  // NT tokens
  static constexpr bool GATED = GATED_;
  static constexpr int MATS = GATED ? 2 : 1;
  static constexpr int ATOMS = KIND == k16 ? 0 : KIND == kNv ? 4 : 2;
  static constexpr int kB = NT * kRowBytes;
  static constexpr int kSa = ATOMS * 512 * MATS, kSb = ATOMS * 512;
  static constexpr int kStage = MATS * kOpBytes + kB + kSa + kSb;
  static constexpr int kFit = (kSmemMax - 1024) / kStage;
  static constexpr int STAGES = kFit < 12 ? kFit : 12;
  static constexpr int kBOff = STAGES * MATS * kOpBytes, kSaOff = kBOff + STAGES * kB;
  static constexpr int kSbOff = kSaOff + STAGES * kSa;
  static constexpr size_t kSmem = (size_t)STAGES * kStage + 1024;
  static constexpr int kSfStage = ATOMS * 4 * (MATS + 1);
  static constexpr int kSfCol = MATS * NT;
  static constexpr int SF = 4;  // stages' scales
  static constexpr int kCols = kSfCol + SF * kSfStage;
  static constexpr int kTmem = kCols <= 32 ? 32 : kCols <= 64 ? 64 : kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
  static constexpr int kThreads = 256;
  static_assert(MATS * NT * kHalf * 4 <= STAGES * kStage && STAGES >= SF && kCols <= 512, "parts where the stages were");
};

// A lane's four consecutive values of an output row.
__device__ __forceinline__ void store4(void* y, int64_t i, const float (&v)[4], int type) {
  if (type == POLYQ_F32) {
    reinterpret_cast<float2*>((float*)y + i)[0] = make_float2(v[0], v[1]);
    reinterpret_cast<float2*>((float*)y + i)[1] = make_float2(v[2], v[3]);
  } else *reinterpret_cast<uint2*>((uint16_t*)y + i) =
      make_uint2(pack16(v[0], v[1], type == POLYQ_BF16), pack16(v[2], v[3], type == POLYQ_BF16));
}
__device__ __forceinline__ void add4(const void* r, int64_t i, float (&v)[4], int type) {
  if (type == POLYQ_F32) {
    const float2 a = reinterpret_cast<const float2*>((const float*)r + i)[0];
    const float2 b = reinterpret_cast<const float2*>((const float*)r + i)[1];
    v[0] += a.x, v[1] += a.y, v[2] += b.x, v[3] += b.y;
  } else {
    const uint2 w = *reinterpret_cast<const uint2*>((const uint16_t*)r + i);
    if (type == POLYQ_BF16) {
      v[0] += bf16_lo(w.x), v[1] += bf16_hi(w.x), v[2] += bf16_lo(w.y), v[3] += bf16_hi(w.y);
    } else {
      const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&w.x));
      const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&w.y));
      v[0] += a.x, v[1] += a.y, v[2] += b.x, v[3] += b.y;
    }
  }
}
__device__ __forceinline__ void save4(const MmParams& P, int which, int64_t at, const float (&v)[4]) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = round24(__float_as_uint(v[e]));
  *reinterpret_cast<uint2*>(saved_hi(P, which, at)) =
      make_uint2(__byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632));
  *reinterpret_cast<uint32_t*>(saved_lo(P, which, at)) =
      __byte_perm(__byte_perm(w[0], w[1], 0x0051), __byte_perm(w[2], w[3], 0x0051), 0x5410);
}
// In 4 bits: a block is eight (MX) or four (NV) neighbouring lanes.  The whole
// warp calls; values past the row's end count as 0.
template <bool NV>
__device__ __forceinline__ void store_codes4(const MmParams& P, int64_t m, int n, const float (&v)[4]) {
  constexpr int BL = NV ? 16 : 32;
  float t[8] = {};
  uint32_t mx = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    t[e] = n + e < P.N ? v[e] : 0.f;
    if (NV) t[e] = P.inv_g != 0.f ? t[e] * P.inv_g : __fdiv_rn(t[e], P.g);
    mx = max(mx, __float_as_uint(t[e]) & 0x7FFFFFFFu);
  }
#pragma unroll
  for (int d = 1; d < BL / 4; d *= 2) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, d));
  const fp4::Scale<NV> sc(mx);
  if (n < P.N) *reinterpret_cast<uint16_t*>(P.codes + m * P.code_stride + n / 2) = (uint16_t)sc.codes(t);
  const int64_t blk = n / BL;
  if (n % BL == 0 && blk >> 2 < P.out_atoms) P.scales[fp4::scale_off(m, blk, P.out_atoms)] = (uint8_t)sc.byte;
}

template <class C>
__global__ void __launch_bounds__(C::kThreads, 1) mm_few(const __grid_constant__ MmParams P, int split) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~(uintptr_t)1023);
  __shared__ uint64_t bar_full[C::STAGES];
  __shared__ uint64_t bar_empty[C::STAGES];
  __shared__ uint64_t bar_acc;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int s_abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = split > 1 ? (int)cluster_ctarank() : 0;
  const int tile = (int)blockIdx.x / split;
  const int n0 = tile * kHalf, m0 = (int)blockIdx.y * C::NT;  // weight rows, tokens
  const int n_it = P.segs * P.kt;
  const int it0 = (int)((int64_t)rank * n_it / split), it1 = (int)((int64_t)(rank + 1) * n_it / split);

  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int s = 0; s < C::STAGES; ++s) {
      mbar_init(smem_u32(&bar_full[s]), 1);
      mbar_init(smem_u32(&bar_empty[s]), 1);
    }
    mbar_init(smem_u32(&bar_acc), 1);
    mbar_fence_init();
  }
  if (warp == 1) {
    tmem_alloc<1>(smem_u32(&tmem_slot), C::kTmem);
    tmem_relinquish<1>();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_trigger();
  auto fail = [&](int code) {
    s_abort = 1;
    atomicExch(P.status, code);
    for (const long long t0 = clock64(); clock64() - t0 < kStayCycles;) __nanosleep(1000);
  };

  if (warp == 0) {
    // ---------------- producer ----------------
    if (elect_one()) {
      pdl_wait();
      int s = 0;
      uint32_t ph = 1;
      for (int i = it0; i < it1; ++i) {
        const int w = wait(smem_u32(&bar_empty[s]), ph, &s_abort);
        if (w != kOk) {
          if (w == kTimeout) fail(kStatusTimeoutEmpty);
          break;
        }
        const uint32_t bar = smem_u32(&bar_full[s]);
        mbar_expect_tx(bar, C::kStage);
        const uint32_t da = smem_u32(smem + s * C::MATS * kOpBytes), db = smem_u32(smem + C::kBOff + s * C::kB);
        const int seg = i >= P.kt, kt = seg ? i - P.kt : i;
        const int k = C::KIND == k16 ? kt * 64 : kt * kRowBytes;
#pragma unroll
        for (int j = 0; j < C::MATS; ++j) {
          const CUtensorMap* map = &P.b[C::GATED ? j : seg];
          if (C::KIND == k16 && P.a_mn) {
            tma_load_2d(da + j * kOpBytes, map, n0, k, bar);
            tma_load_2d(da + j * kOpBytes + 8192, map, n0 + 64, k, bar);
          } else {
            tma_load_2d(da + j * kOpBytes, map, k, n0, bar);
          }
        }
        tma_load_2d(db, &P.a[C::GATED ? 0 : seg], k, m0, bar);
        if (C::KIND != k16) {
          const uint32_t sa = smem_u32(smem + C::kSaOff + s * C::kSa);
          const int row = kt * C::ATOMS;
#pragma unroll
          for (int j = 0; j < C::MATS; ++j)
            tma_load_2d(sa + j * C::ATOMS * 512, &P.sb[j], 0, tile * P.atoms + row, bar);
          tma_load_2d(smem_u32(smem + C::kSbOff + s * C::kSb), &P.sa, 0, (m0 / 128) * P.atoms + row, bar);
        }
        if (++s == C::STAGES) {
          s = 0;
          ph ^= 1u;
        }
      }
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer ----------------
    if (elect_one()) {
      int s = 0, sf = 0, so = 0, held = 0;  // as in mm_pair
      uint32_t ph = 0, so_ph = 0;
      bool ready = false;
      const uint64_t a0 = desc_sw128(smem_u32(smem), P.a_mn ? 8192 : 16), b0 = desc_sw128(smem_u32(smem + C::kBOff), 16);
      const int a_step = P.a_mn ? 2048 >> 4 : 32 >> 4;
      const uint32_t b_col = (uint32_t)(m0 & 127) >> 5;  // of the tokens' scales in their group of 128
      const uint64_t sa0 = desc_scales(smem_u32(smem + C::kSaOff)), sb0 = desc_scales(smem_u32(smem + C::kSbOff));
      for (int i = it0; i < it1; ++i) {
        const int kt = i >= P.kt ? i - P.kt : i;
        int w = kOk;
        if (!ready) w = wait(smem_u32(&bar_full[s]), ph, &s_abort);
        if (w != kOk) {
          if (w == kTimeout) fail(kStatusTimeoutFull);
          break;
        }
        tc_fence_after();
        const int s1 = s + 1 == C::STAGES ? 0 : s + 1;
        const uint32_t ph1 = s1 == 0 ? ph ^ 1u : ph;
        ready = mbar_test(smem_u32(&bar_full[s1]), ph1);
        const int n_mma = kt == P.kt - 1 ? P.k_last : 4;
        const uint64_t a = a0 + (uint64_t)((s * C::MATS * kOpBytes) >> 4), b = b0 + (uint64_t)((s * C::kB) >> 4);
        const uint32_t c0 = tmem + C::kSfCol + sf * C::kSfStage;
        if constexpr (C::KIND != k16) {
          auto release = [&](int n) {
            held -= n;
            so += n;
            if (so >= C::STAGES) {
              so -= C::STAGES;
              so_ph ^= 1u;
            }
          };
          if (held == C::SF) release(poll_ahead<2, C::STAGES>(smem_u32(&bar_empty[0]), so, so_ph));
          if (held == C::SF) {
            w = wait(smem_u32(&bar_empty[so]), so_ph, &s_abort);
            if (w != kOk) {
              if (w == kTimeout) fail(kStatusTimeoutEmpty);
              break;
            }
            release(1);
          }
          const uint64_t sa = sa0 + (uint64_t)((s * C::kSa) >> 4), sb = sb0 + (uint64_t)((s * C::kSb) >> 4);
#pragma unroll
          for (int q = 0; q < C::ATOMS; ++q) {
            const uint32_t c = c0 + q * 4 * (C::MATS + 1);
#pragma unroll
            for (int j = 0; j < C::MATS; ++j) copy_scales<1>(c + 4 * j, sa + (uint64_t)((j * C::ATOMS + q) * 32));
            copy_scales<1>(c + 4 * C::MATS, sb + (uint64_t)(q * 32));
          }
          if (++sf == C::SF) sf = 0;
          ++held;
        }
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          if (kk >= n_mma) break;
#pragma unroll
          for (int j = 0; j < C::MATS; ++j) {
            const uint64_t aj = a + (uint64_t)((j * kOpBytes) >> 4) + (uint64_t)(kk * a_step);
            const bool acc = i > it0 || kk > 0;
            if constexpr (C::KIND == k16) {
              mma_16<1>(tmem + j * C::NT, aj, b + (uint64_t)(2 * kk), P.idesc, acc);
            } else {
              constexpr bool NV = C::KIND == kNv;
              const uint32_t c = c0 + (NV ? kk : kk >> 1) * 4 * (C::MATS + 1);
              const uint32_t id = NV || !(kk & 1) ? P.idesc : P.idesc | idesc_fp4(0, 0, false, 2);
              mma_fp4<1, NV>(tmem + j * C::NT, aj, b + (uint64_t)(2 * kk), id, c + 4 * j, c + 4 * C::MATS + b_col, acc);
            }
          }
        }
        commit<1>(smem_u32(&bar_empty[s]));
        s = s1;
        ph = ph1;
      }
      commit<1>(smem_u32(&bar_acc));
      wait_stay(smem_u32(&bar_acc), 0);
    }
  }
  __syncthreads();  // every copy has landed and every MMA is done (or a role has given up)
  __syncwarp();
  tc_fence_after();

  // ---------------- epilogue ----------------
  // The CTA's part into shared memory, [column][weight row]; then CTA r of the
  // cluster adds the parts of the columns r, r + split, ... in rank order, a warp
  // a column, a lane four rows.
  float* part = reinterpret_cast<float*>(smem);
  {
    const int q = warp & 3;
#pragma unroll 1
    for (int c = (warp >> 2) * 16; c < C::MATS * C::NT; c += 32) {
      uint32_t r[16];
      tmem_ld16(tmem + ((uint32_t)(32 * q) << 16) + c, r);
      tc_wait_ld();
      tc_regs_ready(r);
#pragma unroll
      for (int j = 0; j < 16; ++j) part[(c + j) * kHalf + 32 * q + lane] = __uint_as_float(r[j]);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (split > 1) cluster_sync();
  pdl_wait();
  const int n = n0 + 4 * lane, cnt = min(4, P.N - n);  // the lane's columns of the output
  const uint32_t mine = smem_u32(part + 4 * lane);
  auto sum = [&](int col, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = 0.f;
#pragma unroll
    for (int r0 = 0; r0 < kMaxSplit; r0 += 4) {  // (four reads under way together)
      if (r0 >= split) break;
      float4 f[4];
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (r0 + r < split) f[r] = ld_cluster_f32x4(mapa(mine, r0 + r) + col * (kHalf * 4));
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (r0 + r < split) v[0] += f[r].x, v[1] += f[r].y, v[2] += f[r].z, v[3] += f[r].w;
    }
  };
  // two columns at a time, so that their reads from the peers are under way together
  constexpr int U = 2, kStep = C::kThreads / 32;
#pragma unroll 1
  for (int j0 = rank + split * warp; j0 < C::NT && m0 + j0 < P.M; j0 += U * kStep * split) {
    float vs[U][4], us[C::GATED ? U : 1][4];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int j = min(j0 + i * kStep * split, C::NT - 1);
      sum(j, vs[i]);
      if constexpr (C::GATED) sum(C::NT + j, us[i]);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int j = j0 + i * kStep * split;
      const int64_t m = m0 + j;
      if (j >= C::NT || m >= P.M) break;
      float (&v)[4] = vs[i];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= P.alpha[0];
      if constexpr (C::GATED) {
        float (&u)[4] = us[i];
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] *= P.alpha[1];
        if (C::KIND == k16 && P.saved && cnt > 0) {  // (rows are padded to 32)
          const int64_t at = m * P.saved_stride + n;
          save4(P, 0, at, v);
          save4(P, 1, at, u);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = silu(v[e]) * u[e];
        if (C::KIND != k16 && P.qfmt) {
          if (P.qfmt == kNv) store_codes4<true>(P, m, n, v);
          else store_codes4<false>(P, m, n, v);
          continue;
        }
      } else if (C::KIND != k16 && P.res && cnt > 0) {
        if (P.vec && cnt == 4) {
          add4(P.res, m * P.res_stride + n, v, P.type);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < cnt) v[e] += load_dense(P.res, m * P.res_stride + n + e, P.type);
        }
      }
      if (P.vec && cnt == 4) {
        store4(P.y[0], m * P.y_stride + n, v, P.type);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < cnt) store_dense(P.y[0], m * P.y_stride + n + e, v[e], P.type);
      }
    }
  }
  __syncthreads();
  if (split > 1) cluster_sync();  // a peer may still read this CTA's part
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc<1>(tmem, C::kTmem);
  }
}

// ---------------------------------------------------------------------------
// gradients of the activation and the product
// ---------------------------------------------------------------------------
// da = dh u s (1 + a (1 - s)), du = dh a s with s = 1 / (1 + exp(-a)); 8
// elements a thread.  One pass over a, u, dh; bound by HBM.  Read once, through L2
// (by ordinary loads, which the grid dependency's wait orders with the writes of
// the launch before).
struct ActParams {
  const uint8_t* saved;  // save_row32's planes
  const void* dh;
  void *da, *du;
  int64_t T, F, stride, dh_stride, items;  // stride: of a, u, da, du
  int vec;                                 // rows of dh start on 16 bytes
};
template <bool BF16>
__global__ void __launch_bounds__(256) act_backward(const __grid_constant__ ActParams P) {
  pdl_trigger();
  pdl_wait();
  const int64_t per = P.stride / 8, plane = P.T * P.stride;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < P.items; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / per, f = (i - t * per) * 8;
    if (f >= P.F) continue;
    const int64_t at = t * P.stride + f;
    uint4 hi[2];
    uint2 lo[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      hi[w] = __ldcg(reinterpret_cast<const uint4*>(P.saved + 2 * (w * plane + at)));
      lo[w] = __ldcg(reinterpret_cast<const uint2*>(P.saved + (4 + w) * plane + at));
    }
    uint32_t d[4], da[4], du[4];
    const uint16_t* dr = (const uint16_t*)P.dh + t * P.dh_stride + f;
    const int n = (int)(P.F - f < 8 ? P.F - f : 8);
    if (P.vec && n == 8) {
      const uint4 dv = __ldcg(reinterpret_cast<const uint4*>(dr));
      d[0] = dv.x, d[1] = dv.y, d[2] = dv.z, d[3] = dv.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        d[j] = (2 * j < n ? __ldcg(dr + 2 * j) : 0u) | (uint32_t)(2 * j + 1 < n ? __ldcg(dr + 2 * j + 1) : 0u) << 16;
    }
    auto value = [](const uint4& h, const uint2& l, int j) {  // element j of the eight
      const uint32_t hw = j < 2 ? h.x : j < 4 ? h.y : j < 6 ? h.z : h.w, lw = j < 4 ? l.x : l.y;
      // bytes: 0, the low byte, the two high bytes
      return __uint_as_float(__byte_perm(hw, __byte_perm(lw, 0, 0x4440 | (j & 3)), j & 1 ? 0x3245 : 0x1045));
    };
    auto grad = [](float x, float y, float g, float& ga, float& gu) {
      const float s = __fdividef(1.f, 1.f + __expf(-x)), xs = x * s;
      gu = g * xs;
      ga = g * y * (s + xs * (1.f - s));
    };
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float2 g, ga, gu;
      if (BF16) g = make_float2(bf16_lo(d[j]), bf16_hi(d[j]));
      else g = __half22float2(*reinterpret_cast<const __half2*>(&d[j]));
      grad(value(hi[0], lo[0], 2 * j), value(hi[1], lo[1], 2 * j), g.x, ga.x, gu.x);
      grad(value(hi[0], lo[0], 2 * j + 1), value(hi[1], lo[1], 2 * j + 1), g.y, ga.y, gu.y);
      da[j] = pack16(ga.x, ga.y, BF16);
      du[j] = pack16(gu.x, gu.y, BF16);
    }
    // columns past F of a row's last 8 are padding that nothing reads
    *reinterpret_cast<uint4*>((uint16_t*)P.da + at) = make_uint4(da[0], da[1], da[2], da[3]);
    *reinterpret_cast<uint4*>((uint16_t*)P.du + at) = make_uint4(du[0], du[1], du[2], du[3]);
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
int device_index(int* dev, const char* who) {
  *dev = 0;
  cudaGetDevice(dev);
  if (*dev < 0 || *dev >= kMaxDevices)
    return polyq_set_error(POLYQ_EUNSUPPORTED, "%s: device %d >= %d", who, *dev, kMaxDevices);
  return POLYQ_OK;
}

#ifdef POLYQ_DEBUG
std::atomic<int> g_largest_cluster{kMaxSplit};
#endif

// Clusters of `size` CTAs of a kernel that fit on the device at once: 0 where
// none does, as in a context of few SMs.  `cached` holds one more, 0 until asked.
int resident_clusters(const void* f, int threads, size_t smem, int size, std::atomic<int>* cached, int* out,
                      const char* who) {
  int n = cached->load(std::memory_order_acquire) - 1;
  if (n < 0) {
    cudaError_t e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = size;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(size);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&n, f, &cfg);
    if (e != cudaSuccess)
      return polyq_set_error(POLYQ_ECUDA, "%s: clusters of %d that fit: %s", who, size, cudaGetErrorString(e));
    n = std::max(n, 0);
    cached->store(n + 1, std::memory_order_release);
  }
#ifdef POLYQ_DEBUG
  if (size > g_largest_cluster.load()) n = 0;
#endif
  *out = n;
  return POLYQ_OK;
}

int launch_cluster(const void* f, dim3 grid, int threads, size_t smem, int cluster, void** args, void* stream,
                   const char* who) {
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = (cudaStream_t)stream;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  const cudaError_t e = cudaLaunchKernelExC(&cfg, f, args);
  if (e != cudaSuccess) return polyq_set_error(POLYQ_ECUDA, "%s: launch: %s", who, cudaGetErrorString(e));
  return POLYQ_OK;
}

// The workspace: the status word, the counters of shared tiles' parts, and two
// parts (256 x 256 fp32) for each pair of SMs.
constexpr size_t kCountersOff = POLYQ_FP4_WORKSPACE_ZERO - 16384, kPartsOff = POLYQ_FP4_WORKSPACE_ZERO;
constexpr int kMaxPairs = 16384 / (2 * kEpiWarps * 4);
size_t workspace_bytes_of(int sms) { return kPartsOff + (size_t)sms * kTileM * kTileN * 4; }

// How a pair launch shares its tiles (P.tiles, P.segs, P.kt are set): whole tiles
// in whole waves; the last wave's along the contraction where pairs would be
// idle and that is shorter.  In stages (0.3 us): writing a part and finding the
// others in place cost kShareCost, each part that the last of a tile's pairs
// adds kPartCost; where shares do not end with tiles a pair has two parts.
// Returns the last wave's stages.
// (256 x 1024 x 13824 4 bits, 4 tiles: 19.9 us whole, 18.0 / 17.0 / 18.6 in 2 / 3 / 6
// parts; 5120 instead of 13824 11.1, 13.7 in 2.  16-bit, 4 tiles of 160 stages
// beside 76 whole ones 105 us, 72 in 4; 24 tiles of 48 stages 21 us, 25 in 3.)
constexpr double kShareCost = 13, kPartCost = 4.5;
double plan_tiles(MmParams& P, int pairs) {
  const int n_it = P.segs * P.kt, rest = P.tiles % pairs;
  P.sk_tiles = P.sk_pairs = P.sk_parts = P.sk_share = P.sk_extra = 0;
  if (rest == 0) return 0;
  double best = 0.85 * n_it, last = n_it;
  for (int s = 2; s * rest <= pairs && s <= n_it; ++s) {
    const double t = (n_it + s - 1) / s + kShareCost + kPartCost * s;
    if (t < best) {
      best = last = t;
      P.sk_tiles = rest;
      P.sk_parts = s;
      P.sk_pairs = s * rest;
    }
  }
  const double share = (double)rest * n_it / pairs;
  const double t = share + 2 * kShareCost + kPartCost * (std::ceil(n_it / share) + 1);
  if (share >= 2 && t < 0.95 * best) {
    last = t;
    P.sk_tiles = rest;
    P.sk_parts = 0;
    P.sk_pairs = pairs;
    P.sk_share = (int)((int64_t)rest * n_it / pairs);
    P.sk_extra = (int)((int64_t)rest * n_it % pairs);
  }
  return last;
}

// What a call launches: mm_few with a token tile and a split of the
// contraction, or mm_pair (tokens 0), whichever the model below says is
// shorter.  Times in us, of products whose operands lie in L2, both sides as
// measured (MX; gated after the stroke), few with 64 tokens a tile / few with
// 128 / pair:
//   13824 x 5120, 128 tokens  19.2/26.6  11.5/17.6  11.6/19.0
//   5120 x 5120, 192 tokens    9.8/13.2  11.3/16.9  11.3/11.8
//   5120 x 13824, 96 tokens   19.5/25.6  10.8/15.4  18.3/21.4
//   1024 x 5120, 1024 tokens   9.8/13.2   9.2/13.2  11.2/11.6
//   4096 x 512, 256 tokens     4.6/6.6    6.1/9.3    6.3/6.5
// Weights from HBM add 0 to 2 us to all three (5 where gate and up of 13824 x 5120
// bind few tokens), so the order stays: at ten sizes of 48 to 1024 tokens, MX and
// NV, plain and gated, the choice is at most 5% from the fastest with weights that
// rotate through 400 MB.
constexpr int kFewTokens = 2048;
struct Plan {
  int tokens, split;
  double us;
};

// A wave of mm_few's CTAs: launch, first loads and epilogue, and a stage.
template <class C>
constexpr double few_base() {
  return C::GATED ? (C::NT == 16 ? 4.2 : C::NT == 32 ? 4.6 : C::NT == 64 ? 5.5 : 8.0)
                  : (C::NT == 16 ? 3.3 : C::NT == 32 ? 3.5 : C::NT == 64 ? 3.8 : 5.6);
}
template <class C>
constexpr double few_stage() {
  if (C::KIND == k16) return C::GATED ? (C::NT == 128 ? 0.50 : 0.36) : (C::NT == 128 ? 0.38 : 0.28);
  return C::GATED ? (C::NT == 128 ? 0.55 : C::NT == 64 ? 0.385 : 0.35) : (C::NT == 128 ? 0.30 : 0.28);
}
// A cluster's exchange; a pair launch, its stages and each further wave; what
// saved values and rows that start on 8 or fewer bytes (16-bit outputs of N % 8
// columns) add to its epilogue; the weights from HBM, bytes a us.  The plan goes
// by formats and sizes alone: outputs of another type or stride, or in 4 bits,
// and a call without saved values are the same sums in the same order.
constexpr double kFewSplit = 0.5, kPairBase = 5.4, kPairStage = 0.27, kPairStage16 = 0.30, kPairWave = 1.6;
constexpr double kPairSaved = 1.5, kPairRows8 = 1.5, kPairRowsOdd = 3.0, kHbm = 6.4e6;

// Bytes of the weights: P.N rows of every matrix or segment.
template <class C>
double weight_bytes(const MmParams& P) {
  return (double)P.N * P.kt * P.segs * C::MATS * kRowBytes;
}

// P.M tokens, P.N weight rows, P.segs and P.kt are set.
template <class C>
int consider_few(const MmParams& P, int dev, Plan* best, const char* who) {
  static std::atomic<int> cached[kMaxDevices][kMaxSplit];
  const int64_t tiles = (int64_t)((P.N + kHalf - 1) / kHalf) * ((P.M + C::NT - 1) / C::NT);
  const int n_it = P.segs * P.kt;
  for (int s = 1; s <= kMaxSplit && s <= n_it; ++s) {
    int fit = 0;
    const int rc = resident_clusters((const void*)mm_few<C>, C::kThreads, C::kSmem, s, &cached[dev][s - 1], &fit, who);
    if (rc) return rc;
    if (fit == 0) continue;
    const double us = std::max((double)((tiles + fit - 1) / fit) * (few_base<C>() + few_stage<C>() * ((n_it + s - 1) / s) +
                                                                    (s > 1 ? kFewSplit : 0.0)),
                               few_base<C>() + weight_bytes<C>(P) / kHbm);
    if (us < 0.98 * best->us) *best = {C::NT, s, us};
  }
  return POLYQ_OK;
}

// P.probs is set too; fills in the tiles and how they are shared, where a pair
// fits on the device.
template <class C>
int consider_pair(MmParams& P, int dev, Plan* best, const char* who) {
  static std::atomic<int> cached[kMaxDevices];
  int pairs = 0;
  const int rc = resident_clusters((const void*)mm_pair<C>, C::kThreads, C::kSmem, 2, &cached[dev], &pairs, who);
  if (rc || pairs == 0) return rc;
  pairs = std::min(pairs, kMaxPairs);
  const int cols = C::GATED ? kHalf : kTileN;
  P.tiles_m = (P.M + kTileM - 1) / kTileM;
  P.tiles_n = (P.N + cols - 1) / cols;
  const int64_t tiles = (int64_t)P.tiles_m * P.tiles_n * P.probs;
  if (tiles >= 1ll << 31) return polyq_set_error(POLYQ_EUNSUPPORTED, "%s: %lld tiles", who, (long long)tiles);
  P.tiles = (int)tiles;
  P.per_prob.set((uint32_t)(P.tiles_m * P.tiles_n));
  P.per_band.set(8u * (uint32_t)P.tiles_n);
  P.last_band.set((uint32_t)(P.tiles_m % 8 ? P.tiles_m % 8 : 8));
  const double last = plan_tiles(P, pairs);
  P.grid_pairs = P.tiles > pairs ? pairs : std::max(P.tiles, P.sk_pairs);
  const double waves = (double)(P.tiles / pairs);
  const double epilogue = (C::KIND == k16 && C::GATED ? kPairSaved : 0.0) + (P.N % 8 == 0 ? 0.0 : P.N % 4 == 0 ? kPairRows8 : kPairRowsOdd);
  const double us = kPairBase + epilogue + (C::KIND == k16 ? kPairStage16 : kPairStage) * (waves * P.segs * P.kt + last) +
                    kPairWave * (waves + (last > 0) - 1);
  if (us < best->us) *best = {0, 1, us};
  return POLYQ_OK;
}

constexpr double kNoPlan = 1e30;
int check_plan(const Plan& plan, const char* who) {
  if (plan.us < kNoPlan) return POLYQ_OK;
  return polyq_set_error(POLYQ_EUNSUPPORTED, "%s: no cluster of a kernel's thread blocks fits on the device", who);
}

template <int KIND, bool GATED>
int plan_product(MmParams& P, int dev, Plan* plan, const char* who) {
  *plan = {0, 1, kNoPlan};
  int rc = consider_pair<Pair<KIND, GATED>>(P, dev, plan, who);
  if (!rc && P.M <= 16) rc = consider_few<Few<KIND, 16, GATED>>(P, dev, plan, who);
  if (!rc && P.M > 16 && P.M <= 32) rc = consider_few<Few<KIND, 32, GATED>>(P, dev, plan, who);
  // (with more tokens than fill every SM's tile the pairs are far ahead)
  if (!rc && P.M > 32 && P.M <= kFewTokens) rc = consider_few<Few<KIND, 64, GATED>>(P, dev, plan, who);
  if (!rc && P.M > 32 && P.M <= kFewTokens) rc = consider_few<Few<KIND, 128, GATED>>(P, dev, plan, who);
  return rc ? rc : check_plan(*plan, who);
}

template <class C>
int launch_few(MmParams& P, const Plan& plan, void* stream, const char* who) {
  int split = plan.split;
  void* args[] = {&P, &split};
  const unsigned tiles = (unsigned)((P.N + kHalf - 1) / kHalf), ty = (unsigned)((P.M + C::NT - 1) / C::NT);
  return launch_cluster((const void*)mm_few<C>, dim3(tiles * split, ty), C::kThreads, C::kSmem, split, args, stream, who);
}
template <class C>
int launch_pair(MmParams& P, void* workspace, void* stream, const char* who) {
  P.counters = (int*)((uint8_t*)workspace + kCountersOff);
  P.parts = (float*)((uint8_t*)workspace + kPartsOff);
  void* args[] = {&P};
  return launch_cluster((const void*)mm_pair<C>, dim3(2u * (unsigned)P.grid_pairs), C::kThreads, C::kSmem, 2, args,
                        stream, who);
}
template <int KIND, bool GATED>
int launch_product(MmParams& P, const Plan& plan, void* workspace, void* stream, const char* who) {
  switch (plan.tokens) {
    case 16: return launch_few<Few<KIND, 16, GATED>>(P, plan, stream, who);
    case 32: return launch_few<Few<KIND, 32, GATED>>(P, plan, stream, who);
    case 64: return launch_few<Few<KIND, 64, GATED>>(P, plan, stream, who);
    case 128: return launch_few<Few<KIND, 128, GATED>>(P, plan, stream, who);
    default: return launch_pair<Pair<KIND, GATED>>(P, workspace, stream, who);
  }
}

int check_workspace(const void* ws, size_t bytes, size_t more, const char* who) {
  if (!ws) return polyq_set_error(POLYQ_ENOMEM, "%s: workspace is NULL", who);
  if ((uintptr_t)ws % 256) return polyq_set_error(POLYQ_EINVAL, "%s: workspace must be 256-byte aligned", who);
  size_t need = 0;
  const int rc = polyq_fp4_workspace_bytes(&need);
  if (rc) return rc;
  need += more;
  if (bytes < need)
    return polyq_set_error(POLYQ_ENOMEM, "%s: workspace needs %zu bytes, got %zu", who, need, bytes);
  return POLYQ_OK;
}

int elem_bytes(int type) { return type == POLYQ_F32 ? 4 : 2; }
// Whether rows start on 32 (3), 16 (2), 8 (1) or fewer bytes (0).
int vec_rows(const void* p, int64_t stride, int type) {
  const uint64_t a = (uint64_t)(uintptr_t)p | (uint64_t)(stride * elem_bytes(type));
  return a % 32 == 0 ? 3 : a % 16 == 0 ? 2 : a % 8 == 0 ? 1 : 0;
}
int vec_rows(const polyq_dense* d) { return vec_rows(d->data, d->stride, d->type); }

// Tensor maps of a 4-bit operand: its code tiles of `rows` rows, and its scales.
int map_fp4(CUtensorMap* codes, CUtensorMap* scales, const polyq_fp4* t, int rows, const char* who) {
  const bool nv = t->format == POLYQ_FP4_NV;
  const int64_t atom_rows = (t->rows + 127) / 128 * fp4::atoms(t->K, nv);
  if (atom_rows >= 1ll << 30)
    return polyq_set_error(POLYQ_EUNSUPPORTED, "%s: [%lld][%lld]", who, (long long)t->rows, (long long)t->K);
  int rc = polyq_tensor_map_2d(codes, t->codes, 1, (uint64_t)(t->K + 1) / 2, (uint64_t)t->rows,
                               (uint64_t)t->code_stride, kRowBytes, (uint32_t)rows, 128);
  if (!rc) rc = polyq_tensor_map_2d(scales, t->scales, 4, 128, (uint64_t)atom_rows, 512, 128, nv ? 4 : 2);
  return rc;
}
// A 16-bit matrix [rows][cols] as an operand: K-major tiles (box of 64 columns)
// or, with `mn`, tiles of 64 K rows by 64 columns.
int map_16(CUtensorMap* m, const void* data, int64_t stride, int64_t rows, int64_t cols, bool mn, int box_rows) {
  return polyq_tensor_map_2d(m, data, 2, (uint64_t)cols, (uint64_t)rows, (uint64_t)stride * 2, 64,
                             mn ? 64u : (uint32_t)box_rows, 128);
}

void set_quant_out(MmParams& P, const polyq_fp4* q) {
  const bool nv = q->format == POLYQ_FP4_NV;
  P.codes = q->codes;
  P.scales = q->scales;
  P.code_stride = q->code_stride;
  P.out_atoms = fp4::atoms(q->K, nv);
  P.qfmt = nv ? kNv : kMx;
  P.g = q->tensor_scale;
  int e;
  P.inv_g = std::frexp(P.g, &e) == 0.5f && std::isfinite(1.f / P.g) ? 1.f / P.g : 0.f;
}

// The product's tensor scale, which has to be a normal fp32 number.
float product_scale(const polyq_fp4* a, const polyq_fp4* b) {
  return (float)((double)a->tensor_scale * (double)b->tensor_scale);
}

// The product of 4-bit operands: x [M][K] with w0 (and w1) [N][K].
template <int KIND, bool GATED>
int run_fp4(MmParams& P, const polyq_fp4* x, const polyq_fp4* w0, const polyq_fp4* w1, void* workspace,
            void* stream, const char* who) {
  int dev = 0;
  int rc = device_index(&dev, who);
  if (rc) return rc;
  const bool nv = KIND == kNv;
  P.M = (int)x->rows;
  P.N = (int)w0->rows;
  P.segs = P.probs = 1;
  P.kt = (int)((x->K + 255) / 256);
  P.k_last = (int)((x->K - (int64_t)(P.kt - 1) * 256 + 63) / 64);
  P.atoms = (int)fp4::atoms(x->K, nv);
  P.alpha[0] = product_scale(x, w0);
  P.alpha[1] = GATED ? product_scale(x, w1) : 1.f;
  Plan plan;
  rc = plan_product<KIND, GATED>(P, dev, &plan, who);
  if (rc) return rc;
  P.idesc = plan.tokens ? idesc_fp4(kHalf, plan.tokens, !nv, 0) : idesc_fp4(kTileM, kTileN, !nv, 0);
  rc = map_fp4(&P.a[0], &P.sa, x, plan.tokens ? plan.tokens : kHalf, who);
  if (!rc) rc = map_fp4(&P.b[0], &P.sb[0], w0, kHalf, who);
  if (!rc && GATED) rc = map_fp4(&P.b[1], &P.sb[1], w1, kHalf, who);
  return rc ? rc : launch_product<KIND, GATED>(P, plan, workspace, stream, who);
}

int check_same(const polyq_fp4* x, const polyq_fp4* w, const char* who, const char* what) {
  if (w->K != x->K || w->format != x->format)
    return polyq_set_error(POLYQ_EINVAL, "%s: %s [%lld][%lld] format %d against x [%lld][%lld] format %d", who,
                           what, (long long)w->rows, (long long)w->K, w->format, (long long)x->rows,
                           (long long)x->K, x->format);
  if (!std::isnormal(product_scale(x, w)))
    return polyq_set_error(POLYQ_EINVAL, "%s: %s: tensor scales %g and %g", who, what, (double)x->tensor_scale,
                           (double)w->tensor_scale);
  return POLYQ_OK;
}

// A 16-bit operand of the training block.
int check_16(const polyq_dense* d, int64_t cols, int type, const char* who, const char* what) {
  int rc = polyq_check_dense(d, cols, who, what);
  if (rc) return rc;
  if (d->type != type || type == POLYQ_F32)
    return polyq_set_error(POLYQ_EINVAL, "%s: %s: type %d (all bf16 or all f16)", who, what, d->type);
  return POLYQ_OK;
}
int check_operand(const polyq_dense* d, int64_t cols, int type, const char* who, const char* what) {
  int rc = check_16(d, cols, type, who, what);
  if (rc) return rc;
  if (vec_rows(d) < 2)
    return polyq_set_error(POLYQ_EINVAL, "%s: %s: rows must start on 16 bytes (address and stride)", who, what);
  return POLYQ_OK;
}
// Row length of the saved values and of the gradients of a and u, and the bytes
// of the latter.
int64_t saved_stride(int64_t F) { return (F + 31) / 32 * 32; }
size_t grad_bytes(int64_t T, int64_t F) { return (size_t)T * (size_t)saved_stride(F) * 4; }
int check_sizes(int64_t T, int64_t F, int64_t K, const char* who) {
  if (T < 1 || F < 1 || K < 1 || T > (1 << 24) || F > (1 << 24) || K > (1 << 24))
    return polyq_set_error(POLYQ_EINVAL, "%s: T=%lld F=%lld K=%lld", who, (long long)T, (long long)F, (long long)K);
  return POLYQ_OK;
}

}  // namespace

extern "C" int polyq_fp4_workspace_bytes(size_t* bytes) {
  polyq_clear_error();
  if (!bytes) return polyq_set_error(POLYQ_EINVAL, "polyq_fp4_workspace_bytes: bytes is NULL");
  int sms = 0;
  const int rc = polyq_sm_count(&sms);
  if (!rc) *bytes = workspace_bytes_of(sms);
  return rc;
}

extern "C" int polyq_fp4_linear(const polyq_fp4* x, const polyq_fp4* w, const polyq_dense* residual,
                                const polyq_dense* y, void* workspace, size_t workspace_bytes, void* stream) {
  polyq_clear_error();
  const char* who = "polyq_fp4_linear";
  int rc = polyq_check_fp4(x, who, "x");
  if (!rc) rc = polyq_check_fp4(w, who, "w");
  if (!rc) rc = check_same(x, w, who, "w");
  if (!rc) rc = polyq_check_dense(y, w->rows, who, "y");
  if (!rc && residual) rc = polyq_check_dense(residual, w->rows, who, "residual");
  if (rc) return rc;
  if (residual && residual->type != y->type)
    return polyq_set_error(POLYQ_EINVAL, "%s: residual has type %d, y %d", who, residual->type, y->type);
  if (residual && residual->data == y->data && residual->stride != y->stride)
    return polyq_set_error(POLYQ_EINVAL, "%s: residual is y with another stride", who);
  rc = check_workspace(workspace, workspace_bytes, 0, who);
  if (rc) return rc;
  MmParams P;
  memset(&P, 0, sizeof P);
  P.y[0] = y->data;
  P.y_stride = y->stride;
  P.type = y->type;
  P.vec = std::min(vec_rows(y), residual ? vec_rows(residual) : 3);
  P.res = residual ? residual->data : nullptr;
  P.res_stride = residual ? residual->stride : 0;
  P.status = (int*)workspace;
  return x->format == POLYQ_FP4_NV ? run_fp4<kNv, false>(P, x, w, nullptr, workspace, stream, who)
                                   : run_fp4<kMx, false>(P, x, w, nullptr, workspace, stream, who);
}

extern "C" int polyq_fp4_ffn(const polyq_fp4* x, const polyq_fp4* gate, const polyq_fp4* up, const polyq_dense* h,
                             const polyq_fp4* hq, void* workspace, size_t workspace_bytes, void* stream) {
  polyq_clear_error();
  const char* who = "polyq_fp4_ffn";
  int rc = polyq_check_fp4(x, who, "x");
  if (!rc) rc = polyq_check_fp4(gate, who, "gate");
  if (!rc) rc = polyq_check_fp4(up, who, "up");
  if (!rc) rc = check_same(x, gate, who, "gate");
  if (!rc) rc = check_same(x, up, who, "up");
  if (rc) return rc;
  if (gate->rows != up->rows || !h == !hq)
    return polyq_set_error(POLYQ_EINVAL, "%s: gate has %lld rows, up %lld; one of h and hq is wanted", who,
                           (long long)gate->rows, (long long)up->rows);
  if (h) rc = polyq_check_dense(h, gate->rows, who, "h");
  else rc = polyq_check_fp4(hq, who, "hq");
  if (!rc && hq && (hq->rows != x->rows || hq->K != gate->rows))
    rc = polyq_set_error(POLYQ_EINVAL, "%s: hq is [%lld][%lld]", who, (long long)hq->rows, (long long)hq->K);
  if (!rc) rc = check_workspace(workspace, workspace_bytes, 0, who);
  if (rc) return rc;
  MmParams P;
  memset(&P, 0, sizeof P);
  if (h) {
    P.y[0] = h->data;
    P.y_stride = h->stride;
    P.type = h->type;
    P.vec = vec_rows(h);
  } else {
    set_quant_out(P, hq);
  }
  P.status = (int*)workspace;
  return x->format == POLYQ_FP4_NV ? run_fp4<kNv, true>(P, x, gate, up, workspace, stream, who)
                                   : run_fp4<kMx, true>(P, x, gate, up, workspace, stream, who);
}

extern "C" int polyq_ffn_saved_bytes(int64_t T, int64_t F, size_t* bytes) {
  polyq_clear_error();
  const int rc = check_sizes(T, F, 1, "polyq_ffn_saved_bytes");
  if (rc) return rc;
  if (!bytes) return polyq_set_error(POLYQ_EINVAL, "polyq_ffn_saved_bytes: bytes is NULL");
  *bytes = (size_t)T * (size_t)saved_stride(F) * 6;
  return POLYQ_OK;
}

extern "C" int polyq_ffn_forward(const polyq_dense* x, const polyq_dense* gate, const polyq_dense* up, int64_t T,
                                 int64_t F, int64_t K, const polyq_dense* h, void* saved, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  polyq_clear_error();
  const char* who = "polyq_ffn_forward";
  int rc = check_sizes(T, F, K, who);
  if (!rc) rc = polyq_check_dense(x, K, who, "x");
  if (!rc) rc = check_operand(x, K, x->type, who, "x");
  if (!rc) rc = check_operand(gate, K, x->type, who, "gate");
  if (!rc) rc = check_operand(up, K, x->type, who, "up");
  if (!rc) rc = check_16(h, F, x->type, who, "h");
  if (rc) return rc;
  if ((uintptr_t)saved % 32) return polyq_set_error(POLYQ_EINVAL, "%s: saved must be 32-byte aligned", who);
  rc = check_workspace(workspace, workspace_bytes, 0, who);
  int dev = 0;
  if (!rc) rc = device_index(&dev, who);
  if (rc) return rc;
  MmParams P;
  memset(&P, 0, sizeof P);
  P.M = (int)T;
  P.N = (int)F;
  P.segs = P.probs = 1;
  P.kt = (int)((K + 63) / 64);
  P.k_last = (int)((K - (int64_t)(P.kt - 1) * 64 + 15) / 16);
  P.alpha[0] = P.alpha[1] = 1.f;
  P.y[0] = h->data;
  P.y_stride = h->stride;
  P.type = h->type;
  P.vec = vec_rows(h);
  P.saved = (uint8_t*)saved;
  P.saved_stride = saved_stride(F);
  P.status = (int*)workspace;
  const bool bf16 = x->type == POLYQ_BF16;
  Plan plan;
  rc = plan_product<k16, true>(P, dev, &plan, who);
  if (rc) return rc;
  P.idesc = plan.tokens ? idesc_16(kHalf, plan.tokens, bf16, false, false) : idesc_16(kTileM, kTileN, bf16, false, false);
  rc = map_16(&P.a[0], x->data, x->stride, T, K, false, plan.tokens ? plan.tokens : kHalf);
  if (!rc) rc = map_16(&P.b[0], gate->data, gate->stride, F, K, false, kHalf);
  if (!rc) rc = map_16(&P.b[1], up->data, up->stride, F, K, false, kHalf);
  return rc ? rc : launch_product<k16, true>(P, plan, workspace, stream, who);
}

extern "C" int polyq_ffn_backward_workspace_bytes(int64_t T, int64_t F, size_t* bytes) {
  polyq_clear_error();
  int rc = check_sizes(T, F, 1, "polyq_ffn_backward_workspace_bytes");
  if (rc) return rc;
  if (!bytes) return polyq_set_error(POLYQ_EINVAL, "polyq_ffn_backward_workspace_bytes: bytes is NULL");
  rc = polyq_fp4_workspace_bytes(bytes);
  if (!rc) *bytes += grad_bytes(T, F);
  return rc;
}

extern "C" int polyq_ffn_backward(const polyq_dense* x, const polyq_dense* gate, const polyq_dense* up, int64_t T,
                                  int64_t F, int64_t K, const void* saved, const polyq_dense* dh,
                                  const polyq_dense* dx, const polyq_dense* dgate, const polyq_dense* dup,
                                  void* workspace, size_t workspace_bytes, void* stream) {
  polyq_clear_error();
  const char* who = "polyq_ffn_backward";
  int rc = check_sizes(T, F, K, who);
  if (!rc) rc = polyq_check_dense(x, K, who, "x");
  if (!rc) rc = check_operand(x, K, x->type, who, "x");
  if (!rc) rc = check_operand(gate, K, x->type, who, "gate");
  if (!rc) rc = check_operand(up, K, x->type, who, "up");
  if (!rc) rc = check_16(dh, F, x->type, who, "dh");
  if (rc) return rc;
  if (!saved || (uintptr_t)saved % 32)
    return polyq_set_error(POLYQ_EINVAL, "%s: saved must be given, 32-byte aligned", who);
  if (!dgate != !dup || (!dx && !dgate))
    return polyq_set_error(POLYQ_EINVAL, "%s: dx, or dgate and dup, or all three are wanted", who);
  if (dx) rc = polyq_check_dense(dx, K, who, "dx");
  if (!rc && dgate) rc = polyq_check_dense(dgate, K, who, "dgate");
  if (!rc && dup) rc = polyq_check_dense(dup, K, who, "dup");
  if (rc) return rc;
  for (const polyq_dense* d : {dx, dgate, dup})
    if (d && d->type != x->type && d->type != POLYQ_F32)
      return polyq_set_error(POLYQ_EINVAL, "%s: a gradient of type %d", who, d->type);
  if (dgate && (dgate->type != dup->type || dgate->stride != dup->stride))
    return polyq_set_error(POLYQ_EINVAL, "%s: dgate and dup must have one type and stride", who);
  int dev = 0;
  size_t head = 0;
  rc = check_workspace(workspace, workspace_bytes, grad_bytes(T, F), who);
  if (!rc) rc = device_index(&dev, who);
  if (!rc) rc = polyq_fp4_workspace_bytes(&head);
  if (rc) return rc;

  const bool bf16 = x->type == POLYQ_BF16;
  const int64_t fs = saved_stride(F);
  uint16_t* da = (uint16_t*)((uint8_t*)workspace + head);
  uint16_t* du = da + T * fs;
  {
    ActParams A;
    A.saved = (const uint8_t*)saved;
    A.dh = dh->data;
    A.da = da;
    A.du = du;
    A.T = T;
    A.F = F;
    A.stride = fs;
    A.dh_stride = dh->stride;
    A.items = T * (fs / 8);
    A.vec = vec_rows(dh) >= 2;
    void* args[] = {&A};
    rc = launch_cluster(bf16 ? (const void*)act_backward<true> : (const void*)act_backward<false>,
                        dim3((unsigned)std::min<int64_t>((A.items + 255) / 256, 1 << 30)), 256, 0, 1, args, stream, who);
    if (rc) return rc;
  }
  MmParams P;
  memset(&P, 0, sizeof P);
  P.alpha[0] = 1.f;
  P.status = (int*)workspace;
  if (dx) {
    // dx [T][K]: A = da, du [T][F], B = gate, up [F][K] with K contiguous
    P.M = (int)T;
    P.N = (int)K;
    P.segs = 2;
    P.probs = 1;
    P.kt = (int)((F + 63) / 64);
    P.k_last = (int)((F - (int64_t)(P.kt - 1) * 64 + 15) / 16);
    P.y[0] = dx->data;
    P.y_stride = dx->stride;
    P.type = dx->type;
    P.vec = vec_rows(dx);
    Plan plan;
    rc = plan_product<k16, false>(P, dev, &plan, who);
    if (rc) return rc;
    // mm_few: the weights are the MMAs' A, else their B
    P.a_mn = plan.tokens != 0;
    P.b_mn = plan.tokens == 0;
    P.idesc = plan.tokens ? idesc_16(kHalf, plan.tokens, bf16, true, false) : idesc_16(kTileM, kTileN, bf16, false, true);
    const int rows = plan.tokens ? plan.tokens : kHalf;
    rc = map_16(&P.a[0], da, fs, T, F, false, rows);
    if (!rc) rc = map_16(&P.a[1], du, fs, T, F, false, rows);
    if (!rc) rc = map_16(&P.b[0], gate->data, gate->stride, F, K, true, 0);
    if (!rc) rc = map_16(&P.b[1], up->data, up->stride, F, K, true, 0);
    if (!rc) rc = launch_product<k16, false>(P, plan, workspace, stream, who);
    if (rc) return rc;
  }
  if (dgate) {
    // dgate, dup [F][K]: A = da, du with F contiguous, B = x with K contiguous, over T
    P.M = (int)F;
    P.N = (int)K;
    P.segs = 1;
    P.probs = 2;
    P.kt = (int)((T + 63) / 64);
    P.k_last = (int)((T - (int64_t)(P.kt - 1) * 64 + 15) / 16);
    P.a_mn = P.b_mn = 1;
    P.y[0] = dgate->data;
    P.y[1] = dup->data;
    P.y_stride = dgate->stride;
    P.type = dgate->type;
    P.vec = std::min(vec_rows(dgate), vec_rows(dup));
    P.idesc = idesc_16(kTileM, kTileN, bf16, true, true);
    rc = map_16(&P.a[0], da, fs, T, F, true, 0);
    if (!rc) rc = map_16(&P.a[1], du, fs, T, F, true, 0);
    if (!rc) rc = map_16(&P.b[0], x->data, x->stride, T, K, true, 0);
    P.b[1] = P.b[0];
    Plan plan = {0, 1, kNoPlan};
    if (!rc) rc = consider_pair<Pair<k16, false>>(P, dev, &plan, who);
    if (!rc) rc = check_plan(plan, who);
    if (!rc) rc = launch_pair<Pair<k16, false>>(P, workspace, stream, who);
  }
  return rc;
}

#ifdef POLYQ_DEBUG
#include "polyq_debug_mm.h"
extern "C" void polyq_debug_mm_largest_cluster(int size) { g_largest_cluster = size; }
#endif
