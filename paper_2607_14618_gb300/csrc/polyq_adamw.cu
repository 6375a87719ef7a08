// AdamW over many tensors in one launch, with the moments in 32 or in 8 bits.
//
//   m = b1 m + (1-b1) g,  v = b2 v + (1-b2) g^2
//   p = p (1 - lr decay) - lr / (1-b1^t) m / (sqrt(v / (1-b2^t)) + eps)
//
// Bound by HBM: parameters and moments in and out, gradients in.  A warp takes
// 256 elements of one tensor, eight a lane, which are a block of an 8-bit state:
// its largest magnitude is one reduction over the warp.  The tensors' pointers
// are parameters of the kernel, so that a step needs no copy to the device; a
// thread block finds its tensor by bisection.
//
// Measured: 212 M elements, fp32 with bf16 gradients and copies, 32-bit states 850 us, 7.0 TB/s;
// the same with 8-bit states 740 us, bound by instructions, 92 an element (81% of the issue slots),
// in packed pairs where the order of roundings allows (760 us one by one); 560 tensors, 62 M
// elements, 258 us; 81 vectors of 5120 6 us, a launch.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>

#include "polyq_dense_dev.cuh"
#include "polyq_dev.cuh"
#include "polyq_finetune.h"
#include "polyq_fp4_dev.cuh"
#include "polyq_internal.h"

namespace {

using namespace polyq;

constexpr int kBlock = POLYQ_ADAMW_BLOCK;
constexpr int kWarps = 8;  // of a thread block
// Tensors of a launch: 4 KB of parameters for few of them, else what a kernel
// may have (32 764 bytes).
constexpr int kFew = 64, kMany = 640;

struct Tensor {
  void* p;
  const void* grad;
  void* copy;
  int64_t n;
  uint32_t at;     // first block of its state
  uint32_t first;  // first block among the launch's
  float decay, rate;
};
template <int N>
struct AdamParams {
  void* m;
  void* v;
  uint8_t* ms;
  uint8_t* vs;
  const float* lr_dev;
  const int64_t* step_dev;
  const float* grad_scale;
  uint64_t seed;
  float lr, inv_bc1, inv_root_bc2, b1, c1, b2, c2, eps, log_b1, log_b2;
  uint32_t blocks;
  int32_t n, copy_type;
  Tensor t[N];
};
static_assert(sizeof(AdamParams<kMany>) <= 32764, "parameters of a kernel");

__device__ __forceinline__ uint32_t mix(uint32_t h) {
  h = (h ^ h >> 16) * 0x9E2D58A5u;
  return (h ^ h >> 15) * 0x6C62272Du;
}

// A magnitude with MANT mantissa bits, whose smallest normal number is 1, is, scaled by
// 2^-126, an fp32 number of the same exponent field, subnormal ones included: its code is
// that number's upper bits.  Between it and the block's scale, 2^(scale-127), lies the power
// 2^(scale-1): fp32 holds it or its reciprocal for scales up to 127, which one product then
// takes; others take two.  Both are exact but for numbers that fp32 holds as subnormal.
struct Scale {
  float one, rest;  // the power of two, as two factors
  bool two;
  static __device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
  // 2^(s-1), codes to values
  static __device__ __forceinline__ Scale up(int s) { return Scale{pow2(min(s, 128) - 1), pow2(max(s - 128, 0)), s > 128}; }
  // 2^(1-s), values to codes
  static __device__ __forceinline__ Scale down(int s) {
    return Scale{pow2(1 - min(s, 127)), pow2(min(127 - s, 0)), s > 127};
  }
  __device__ __forceinline__ void apply(F2 (&v)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], f2(one, one));
    if (two)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], f2(rest, rest));
  }
};
// Values of eight codes (a byte each): MANT 3 with a sign in bit 7, MANT 4 without.
template <int MANT>
__device__ __forceinline__ void decode(uint2 codes, int scale, F2 (&v)[4]) {
  constexpr uint32_t MASK = (MANT == 3 ? 0x7Fu : 0xFFu) << (23 - MANT);
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t w = i < 4 ? codes.x : codes.y;
    const int at = 23 - MANT - 8 * (i & 3);  // from a byte's place to the code's
    uint32_t b = (at >= 0 ? w << at : w >> -at) & MASK;
    if (MANT == 3) b |= w << (24 - 8 * (i & 3)) & 0x80000000u;
    f[i] = __uint_as_float(b);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = f2(f[2 * i], f[2 * i + 1]);
  if (scale == 255) {
    const float nan = __uint_as_float(0x7FC00000u);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = f2(nan, nan);
  } else {
    Scale::up(scale).apply(v);
  }
}
// The smallest scale with which the largest magnitude `top` is within the codes (so
// that none is cut off, which would bias the largest ones): the one that brings it to
// 2^14 .. 2^15, or the next where it lies above the last code there.
template <int MANT>
__device__ __forceinline__ int scale_of(uint32_t top) {
  const uint32_t past = top + (1u << (23 - MANT)) - 1;
  return top >= 0x7F800000u ? 255 : max((int)(past >> 23) - 14, 0);
}
// The largest magnitude of three; NaN where one is.
__device__ __forceinline__ float most(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// a + b, each sum by itself: of a packed sum and a product that it adds, the compiler makes one
// rounding.
__device__ __forceinline__ F2 sum_rn(F2 a, F2 b) {
  const float2 x = of(a), y = of(b);
  return f2(__fadd_rn(x.x, y.x), __fadd_rn(x.y, y.y));
}
__device__ __forceinline__ void flat(const F2 (&v)[4], float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 a = of(v[i]);
    f[2 * i] = a.x;
    f[2 * i + 1] = a.y;
  }
}
template <typename T>
__device__ __forceinline__ void pairs(const Raw8<T>& r, F2 (&v)[4]) {
  float f[8];
  to_float(r, f);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = f2(f[2 * i], f[2 * i + 1]);
}
__device__ __forceinline__ uint32_t pack4(const uint32_t (&c)[8], int i) {
  return c[i] | c[i + 1] << 8 | c[i + 2] << 16 | c[i + 3] << 24;
}

// What is the same for all elements of a tensor.
struct Rates {
  float gs, keep, step, inv_root_bc2;
  uint32_t seed_key, seed_high;
};

// The whole blocks of an 8-bit state come through shared memory, a place for each block that a
// warp has asked for: p, the gradient and the two moments' codes.  (Loads to registers waited:
// 10 cycles of a warp for each that it issued; 212 M elements 795 us, 760 this way.)
template <typename TP, typename TG>
struct Staged {
  static constexpr int P_BYTES = kBlock * sizeof(TP), G_BYTES = kBlock * sizeof(TG), STAGE = P_BYTES + G_BYTES + 2 * kBlock;
  static constexpr int STAGES = STAGE <= 2048 ? 3 : 2;  // (48 KB of a thread block)
  // Where the 16-byte piece j of a tensor's elements lies: a lane's pieces of fp32 lie in different banks.
  template <typename T>
  static __device__ __forceinline__ uint32_t piece(int j) {
    return (sizeof(T) == 4 ? j ^ (j >> 3 & 1) : j) * 16u;
  }
  static __device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  }
  template <typename T>
  static __device__ __forceinline__ void ask(uint32_t place, const void* data, uint32_t block) {
    const int lane = threadIdx.x & 31;
    const char* from = (const char*)data + (int64_t)block * (kBlock * sizeof(T));
#pragma unroll
    for (int j = lane; j < (int)sizeof(T) * kBlock / 16; j += 32) copy16(place + piece<T>(j), from + 16 * j);
  }
  template <typename T>
  static __device__ __forceinline__ void get(uint32_t place, Raw8<T>& r) {
    constexpr int N16 = sizeof(T) * 8 / 16;
#pragma unroll
    for (int i = 0; i < N16; ++i)
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(r.w[i].x), "=r"(r.w[i].y), "=r"(r.w[i].z), "=r"(r.w[i].w)
                   : "r"(place + piece<T>((threadIdx.x & 31) * N16 + i))
                   : "memory");
  }
  static __device__ __forceinline__ uint2 codes(uint32_t place) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(place + (threadIdx.x & 31) * 8u) : "memory");
    return v;
  }
};

// One block: elements i of the tensor from e0 on.  FULL: 256 of them, on 16 bytes, which with 8
// bits lie at `place`.  sm_was, sv_was: the scales of 8 bits.
template <typename TP, typename TG, int BITS, bool FULL, int N>
__device__ __forceinline__ void update_block(const AdamParams<N>& P, const Tensor& t, uint32_t block, const Rates& c,
                                             uint32_t place, int sm_was, int sv_was) {
  using S = Staged<TP, TG>;
  const int lane = threadIdx.x & 31;
  const int64_t e0 = (int64_t)block * kBlock, s0 = (int64_t)(t.at + block) * kBlock;
  // the eight elements of a lane: neighbours, or every 32nd (see load8)
  const int col = FULL ? 8 * lane : lane;
  const uint32_t mask = FULL ? 0xFFu : mask8<false>(col, 32, (int)min(t.n - e0, (int64_t)kBlock));
  Raw8<TP> rp;
  Raw8<TG> rg;
  if constexpr (FULL && BITS == 8) {
    S::get(place, rp);
    S::get(place + S::P_BYTES, rg);
  } else {
    load8<FULL>((const TP*)t.p + e0, col, 32, mask, rp);
    load8<FULL>((const TG*)t.grad + e0, col, 32, mask, rg);
  }
  F2 m[4], v[4];
  if constexpr (BITS == 32) {
    Raw8<float> rm, rv;
    load8<FULL>((const float*)P.m + s0, col, 32, mask, rm);
    load8<FULL>((const float*)P.v + s0, col, 32, mask, rv);
    pairs(rm, m);
    pairs(rv, v);
  } else {
    uint2 cm, cv;
    if constexpr (FULL) {
      cm = S::codes(place + S::P_BYTES + S::G_BYTES);
      cv = S::codes(place + S::P_BYTES + S::G_BYTES + kBlock);
    } else {
      const uint8_t *pm = (const uint8_t*)P.m + s0, *pv = (const uint8_t*)P.v + s0;
      uint32_t bm[8], bv[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        bm[i] = mask >> i & 1 ? __ldcg(pm + col + 32 * i) : 0u;
        bv[i] = mask >> i & 1 ? __ldcg(pv + col + 32 * i) : 0u;
      }
      cm = make_uint2(pack4(bm, 0), pack4(bm, 4));
      cv = make_uint2(pack4(bv, 0), pack4(bv, 4));
    }
    decode<3>(cm, sm_was, m);
    decode<4>(cv, sv_was, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], v[i]);
  }
  F2 p2[4], g[4];
  pairs(rp, p2);
  pairs(rg, g);
  const F2 gs = f2(c.gs, c.gs), b1 = f2(P.b1, P.b1), c1 = f2(P.c1, P.c1), b2 = f2(P.b2, P.b2), c2 = f2(P.c2, P.c2);
  const F2 keep = f2(c.keep, c.keep), step = f2(-c.step, -c.step), eps = f2(P.eps, P.eps);
  const F2 inv = f2(c.inv_root_bc2, c.inv_root_bc2);
  float top_m = 0.f, top_r = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // each operation rounded by itself: the codes of an 8-bit state follow from this order
    const F2 s = mul2(g[i], gs);
    m[i] = sum_rn(mul2(b1, m[i]), mul2(c1, s));
    v[i] = sum_rn(mul2(b2, v[i]), mul2(mul2(c2, s), s));
    const float2 vs = of(v[i]), roots = make_float2(__fsqrt_rn(vs.x), __fsqrt_rn(vs.y));
    const F2 root = f2(roots.x, roots.y);
    // (the denominator is eps or more, a normal number, and at most 2^65 / (1 - b2^t): within the
    // reciprocal's range, which takes subnormal numbers for 0)
    const float2 below = of(fma2(root, inv, eps));
    p2[i] = fma2(mul2(step, m[i]), f2(fp4::rcp_approx(below.x), fp4::rcp_approx(below.y)), mul2(p2[i], keep));
    if (BITS == 8) {
      v[i] = root;
      if (!FULL) {
        const bool x = mask >> (2 * i) & 1, y = mask >> (2 * i + 1) & 1;
        const float2 ms = of(m[i]);
        m[i] = f2(x ? ms.x : 0.f, y ? ms.y : 0.f);
        v[i] = f2(x ? roots.x : 0.f, y ? roots.y : 0.f);
      }
      const float2 ms = of(m[i]), rs = of(v[i]);
      top_m = most(ms.x, ms.y, top_m);
      top_r = most(rs.x, rs.y, top_r);
    }
  }
  float p[8];
  flat(p2, p);
  store8<FULL>((TP*)t.p + e0, col, 32, mask, p);
  if (t.copy) {
    if (sizeof(TP) < 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = Elem<TP>::to(Elem<TP>::from(p[i]));  // once from p
    }
    const bool on16 = FULL && (uintptr_t)t.copy % 16 == 0;
    if (FULL && !on16) {
#pragma unroll
      for (int i = 0; i < 8; ++i) any_store(t.copy, P.copy_type, e0 + col + i, p[i]);
    } else if (P.copy_type == POLYQ_F32) {
      store8<FULL>((float*)t.copy + e0, col, 32, mask, p);
    } else if (P.copy_type == POLYQ_BF16) {
      store8<FULL>((__nv_bfloat16*)t.copy + e0, col, 32, mask, p);
    } else {
      store8<FULL>((__half*)t.copy + e0, col, 32, mask, p);
    }
  }
  if constexpr (BITS == 32) {
    float fm[8], fv[8];
    flat(m, fm);
    flat(v, fv);
    store8<FULL>((float*)P.m + s0, col, 32, mask, fm);
    store8<FULL>((float*)P.v + s0, col, 32, mask, fv);
  } else {
    const int sm = scale_of<3>(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top_m)));
    const int sr = scale_of<4>(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top_r)));
    const uint64_t b64 = (uint64_t)t.at + block;
    const uint32_t key = mix(mix((uint32_t)b64 ^ c.seed_key) ^ (uint32_t)(b64 >> 32) ^ c.seed_high);
    uint32_t cm[8] = {}, cv[8] = {};
    uint32_t some[8];  // 1 where the root is not 0
    float fm[8], fr[8];
    flat(v, fr);
#pragma unroll
    for (int i = 0; i < 8; ++i) some[i] = min(__float_as_uint(fr[i]), 1u);
    Scale::down(sm).apply(m);
    Scale::down(sr).apply(v);
    flat(m, fm);
    flat(v, fr);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t e = FULL ? (uint32_t)(col + i) : (uint32_t)(col + 32 * i);
      // 16 bits for the root, and 16 for m
      const uint32_t h = mix(key + 0x9E3779B1u * e), high = h >> 16;
      // (the sign stays above: no magnitude of the block carries into it)
      const uint32_t a = __float_as_uint(fm[i]) + (((h ^ high) & 0xFFFFu) << 4);
      cm[i] = (a >> 20 & 0x7Fu) | (a >> 24 & ~0x7Fu);
      cv[i] = max((__float_as_uint(fr[i]) + (high << 3)) >> 19, some[i]);
    }
    if (sm == 255 || sr == 255)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (sm == 255) cm[i] = 0u;
        if (sr == 255) cv[i] = 0u;
      }
    uint8_t *pm = (uint8_t*)P.m + s0, *pv = (uint8_t*)P.v + s0;
    if constexpr (FULL) {
      *reinterpret_cast<uint2*>(pm + col) = make_uint2(pack4(cm, 0), pack4(cm, 4));
      *reinterpret_cast<uint2*>(pv + col) = make_uint2(pack4(cv, 0), pack4(cv, 4));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {  // (the whole block is the tensor's)
        pm[col + 32 * i] = (uint8_t)cm[i];
        pv[col + 32 * i] = (uint8_t)cv[i];
      }
    }
    __syncwarp();  // every lane has read the block's scales, and its place in shared memory
    if (lane == 0) {
      P.ms[t.at + block] = (uint8_t)sm;
      P.vs[t.at + block] = (uint8_t)sr;
    }
  }
}

// Thread blocks of an SM.  32 bits: bound by HBM, and nearest to it with short ones that the
// SMs take as they come (212 M elements: 996 us with 8 an SM, 870 with 64, 848 with 256: 7.0
// TB/s).  8 bits: bound by instructions (as many as fit at once: 833 us with 4, 939 with 8, with
// loads to registers; a warp that asks for its next block ahead into them has room for 3: 893).
constexpr int kBlocks32 = 256, kBlocks8 = 4;

template <typename TP, typename TG, int BITS, int N>
__global__ void __launch_bounds__(32 * kWarps, 4)
    adamw_kernel(const __grid_constant__ AdamParams<N> P) {
  pdl_trigger();
  pdl_wait();
  Rates c;
  c.gs = 1.f;
  if (P.grad_scale) {
    c.gs = __ldcg(P.grad_scale);
    if (!(fabsf(c.gs) < INFINITY)) return;
  }
  const float lr = P.lr_dev ? __ldcg(P.lr_dev) : P.lr;
  float inv_bc1 = P.inv_bc1;
  c.inv_root_bc2 = P.inv_root_bc2;
  uint64_t seed = P.seed;
  if (P.step_dev) {  // 1 - b^t = -expm1(t log b)
    const int64_t t = max(__ldcg(P.step_dev), (int64_t)1);
    seed += (uint64_t)t;
    inv_bc1 = -1.f / expm1f((float)t * P.log_b1);
    c.inv_root_bc2 = rsqrtf(-expm1f((float)t * P.log_b2));
  }
  c.seed_key = mix((uint32_t)seed + 1u);
  c.seed_high = (uint32_t)(seed >> 32);
  const uint32_t stride = gridDim.x * kWarps;
  struct Place {
    int which;  // tensor
    uint32_t block;
    bool full;
    int sm, sv;
  };
  auto find = [&](uint32_t b) {  // the last tensor whose first block is b or before it
    int lo = 0, hi = P.n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (P.t[mid].first <= b) lo = mid;
      else hi = mid - 1;
    }
    const Tensor& t = P.t[lo];
    Place a{lo, b - t.first, false, 0, 0};
    a.full = ((int64_t)a.block + 1) * kBlock <= t.n && (((uintptr_t)t.p | (uintptr_t)t.grad) & 15) == 0;
    return a;
  };
  auto update = [&](const Place& a, uint32_t place) {
    const Tensor& t = P.t[a.which];
    const float rate = lr * t.rate;
    c.keep = 1.f - rate * t.decay;
    c.step = rate * inv_bc1;
    if (a.full) update_block<TP, TG, BITS, true>(P, t, a.block, c, place, a.sm, a.sv);
    else update_block<TP, TG, BITS, false>(P, t, a.block, c, place, a.sm, a.sv);
  };
  uint32_t b = blockIdx.x * kWarps + (threadIdx.x >> 5);
  if constexpr (BITS == 32) {
    for (; b < P.blocks; b += stride) update(find(b), 0);
  } else {
    using S = Staged<TP, TG>;
    __shared__ __align__(16) uint8_t smem[kWarps * S::STAGES * S::STAGE];
    const uint32_t ring = smem_u32(smem) + (threadIdx.x >> 5) * (S::STAGES * S::STAGE);
    const int lane = threadIdx.x & 31;
    auto ask = [&](uint32_t b, uint32_t place) {
      Place a{0, 0, false, 0, 0};
      if (b < P.blocks) {
        a = find(b);
        const Tensor& t = P.t[a.which];
        a.sm = __ldcg(P.ms + t.at + a.block);
        a.sv = __ldcg(P.vs + t.at + a.block);
        if (a.full) {
          S::template ask<TP>(place, t.p, a.block);
          S::template ask<TG>(place + S::P_BYTES, t.grad, a.block);
          const int64_t s0 = (int64_t)(t.at + a.block) * kBlock;
          const uint8_t* codes = (const uint8_t*)(lane < 16 ? P.m : P.v) + s0 + (lane & 15) * 16;
          S::copy16(place + S::P_BYTES + S::G_BYTES + lane * 16, codes);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      return a;
    };
    // this block, and those on their way
    Place at[S::STAGES];
#pragma unroll
    for (int i = 0; i < S::STAGES - 1; ++i) at[i] = ask(b + i * stride, ring + i * S::STAGE);
    for (uint32_t slot = 0; b < P.blocks; b += stride) {
      const uint32_t last = slot == 0 ? S::STAGES - 1 : slot - 1;
      at[S::STAGES - 1] = ask(b + (S::STAGES - 1) * stride, ring + last * S::STAGE);
      asm volatile("cp.async.wait_group %0;" ::"n"(S::STAGES - 1) : "memory");
      __syncwarp();
      update(at[0], ring + slot * S::STAGE);
#pragma unroll
      for (int i = 0; i < S::STAGES - 1; ++i) at[i] = at[i + 1];
      if (++slot == S::STAGES) slot = 0;
    }
  }
}

struct ValuesParams {
  const uint8_t* m;
  const uint8_t* v;
  const uint8_t* ms;
  const uint8_t* vs;
  void* out[2];
  int type[2];
  uint32_t blocks;
};
template <int MANT>
__device__ __forceinline__ void values_block(const uint8_t* codes, const uint8_t* scales, void* out, int type,
                                             uint32_t b) {
  const int lane = threadIdx.x & 31;
  const int64_t e = (int64_t)b * kBlock + 8 * lane;
  F2 pairs_of[4];
  decode<MANT>(__ldcg(reinterpret_cast<const uint2*>(codes + e)), __ldcg(scales + b), pairs_of);
  float v[8];
  flat(pairs_of, v);
  if ((uintptr_t)out % 16) {
#pragma unroll
    for (int i = 0; i < 8; ++i) any_store(out, type, e + i, v[i]);
  } else if (type == POLYQ_F32) {
    store8<true>((float*)out + e, 0, 1, 0xFFu, v);
  } else if (type == POLYQ_BF16) {
    store8<true>((__nv_bfloat16*)out + e, 0, 1, 0xFFu, v);
  } else {
    store8<true>((__half*)out + e, 0, 1, 0xFFu, v);
  }
}
__global__ void __launch_bounds__(32 * kWarps) adamw_values_kernel(const __grid_constant__ ValuesParams P) {
  pdl_trigger();
  pdl_wait();
  for (uint32_t b = blockIdx.x * kWarps + (threadIdx.x >> 5); b < P.blocks; b += gridDim.x * kWarps) {
    if (P.out[0]) values_block<3>(P.m, P.ms, P.out[0], P.type[0], b);
    if (P.out[1]) values_block<4>(P.v, P.vs, P.out[1], P.type[1], b);
  }
}

template <int N, int BITS, typename TP>
void* pick(int tg) {
  return tg == POLYQ_F32    ? (void*)adamw_kernel<TP, float, BITS, N>
         : tg == POLYQ_BF16 ? (void*)adamw_kernel<TP, __nv_bfloat16, BITS, N>
                            : (void*)adamw_kernel<TP, __half, BITS, N>;
}
template <int N, int BITS>
void* pick(int tp, int tg) {
  return tp == POLYQ_F32    ? pick<N, BITS, float>(tg)
         : tp == POLYQ_BF16 ? pick<N, BITS, __nv_bfloat16>(tg)
                            : pick<N, BITS, __half>(tg);
}

int launch(void* f, uint32_t blocks, int per_sm, void* params, void* stream, const char* who) {
  int sms = 0;
  int rc = polyq_sm_count(&sms);
  if (rc) return rc;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.stream = (cudaStream_t)stream;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3((unsigned)std::min<int64_t>(((int64_t)blocks + kWarps - 1) / kWarps, (int64_t)sms * per_sm));
  cfg.blockDim = dim3(32 * kWarps);
  void* args[] = {params};
  cudaError_t ce = cudaLaunchKernelExC(&cfg, f, args);
  if (ce != cudaSuccess) return polyq_set_error(POLYQ_ECUDA, "%s: launch: %s", who, cudaGetErrorString(ce));
  return POLYQ_OK;
}

template <int N>
int run_step(const polyq_adamw_tensor* tensors, int n, int p_type, int grad_type, int copy_type,
             const polyq_adamw_state* state, const polyq_adamw_hyper* h, void* stream, const char* who) {
  AdamParams<N> P;
  P.m = state->m;
  P.v = state->v;
  P.ms = state->m_scales;
  P.vs = state->v_scales;
  P.lr_dev = h->lr_dev;
  P.step_dev = h->step_dev;
  P.grad_scale = h->grad_scale;
  P.seed = h->seed;
  P.lr = (float)h->lr;
  P.inv_bc1 = (float)(1.0 / (1.0 - std::pow(h->beta1, (double)h->step)));
  P.inv_root_bc2 = (float)(1.0 / std::sqrt(1.0 - std::pow(h->beta2, (double)h->step)));
  P.b1 = (float)h->beta1;
  P.c1 = (float)(1.0 - h->beta1);
  P.b2 = (float)h->beta2;
  P.c2 = (float)(1.0 - h->beta2);
  P.eps = (float)h->eps;
  P.log_b1 = (float)std::log(h->beta1);
  P.log_b2 = (float)std::log(h->beta2);
  P.copy_type = copy_type;
  for (int i0 = 0; i0 < n;) {
    int64_t blocks = 0;
    int k = 0;
    for (; k < N && i0 + k < n; ++k) {
      const polyq_adamw_tensor& t = tensors[i0 + k];
      const int64_t b = (t.n + kBlock - 1) / kBlock;
      if (k && blocks + b > 0x7FFFFFFF) break;
      P.t[k] = Tensor{t.p, t.grad, t.copy, t.n, (uint32_t)(t.at / kBlock), (uint32_t)blocks, t.decay, t.rate};
      blocks += b;
    }
    P.n = k;
    P.blocks = (uint32_t)blocks;
    void* f = state->bits == 8 ? pick<N, 8>(p_type, grad_type) : pick<N, 32>(p_type, grad_type);
    const int rc = launch(f, P.blocks, state->bits == 8 ? kBlocks8 : kBlocks32, &P, stream, who);
    if (rc) return rc;
    i0 += k;
  }
  return POLYQ_OK;
}

bool good_type(int t) { return t == POLYQ_F32 || t == POLYQ_BF16 || t == POLYQ_F16; }
bool misaligned(const void* p, int type) { return (uintptr_t)p % (type == POLYQ_F32 ? 4 : 2) != 0; }

int check_state(const polyq_adamw_state* s, const char* who) {
  if (!s || !s->m || !s->v || (uintptr_t)s->m % 16 || (uintptr_t)s->v % 16)
    return polyq_set_error(POLYQ_EINVAL, "%s: the state's m and v must be 16-byte aligned and not NULL", who);
  if (s->bits != 8 && s->bits != 32) return polyq_set_error(POLYQ_EINVAL, "%s: a state of %d bits", who, s->bits);
  if (s->bits == 8 && (!s->m_scales || !s->v_scales))
    return polyq_set_error(POLYQ_EINVAL, "%s: a state of 8 bits needs scales", who);
  if (s->n < 1 || s->n % kBlock || s->n > (1ll << 38))
    return polyq_set_error(POLYQ_EINVAL, "%s: a state of %lld elements", who, (long long)s->n);
  return POLYQ_OK;
}

}  // namespace

extern "C" int polyq_adamw_step(const polyq_adamw_tensor* tensors, int32_t n_tensors, int32_t p_type,
                                int32_t grad_type, int32_t copy_type, const polyq_adamw_state* state,
                                const polyq_adamw_hyper* hyper, void* stream) {
  static const char* who = "polyq_adamw_step";
  polyq_clear_error();
  if (!tensors || n_tensors < 1 || !hyper)
    return polyq_set_error(POLYQ_EINVAL, "%s: no tensors or no rates", who);
  int rc = check_state(state, who);
  if (rc) return rc;
  if (!good_type(p_type) || !good_type(grad_type))
    return polyq_set_error(POLYQ_EINVAL, "%s: types %d and %d", who, p_type, grad_type);
  const polyq_adamw_hyper& h = *hyper;
  if (!(h.lr >= 0.0) || !std::isfinite((float)h.lr) || !(h.beta1 >= 0.0 && h.beta1 < 1.0) ||
      !(h.beta2 >= 0.0 && h.beta2 < 1.0) || !((float)h.eps >= FLT_MIN) || !(h.eps <= 1e30) || h.step < 1)
    return polyq_set_error(POLYQ_EINVAL, "%s: lr %g, betas %g and %g, eps %g, step %lld", who, h.lr, h.beta1, h.beta2,
                           h.eps, (long long)h.step);
  if ((uintptr_t)h.lr_dev % 4 || (uintptr_t)h.step_dev % 8 || (uintptr_t)h.grad_scale % 4)
    return polyq_set_error(POLYQ_EINVAL, "%s: device values must be aligned to their size", who);
  for (int i = 0; i < n_tensors; ++i) {
    const polyq_adamw_tensor& t = tensors[i];
    if (!t.p || !t.grad || misaligned(t.p, p_type) || misaligned(t.grad, grad_type))
      return polyq_set_error(POLYQ_EINVAL, "%s: tensor %d: p and grad must be aligned to their elements", who, i);
    if (t.copy && (!good_type(copy_type) || misaligned(t.copy, copy_type)))
      return polyq_set_error(POLYQ_EINVAL, "%s: tensor %d: copy of type %d", who, i, copy_type);
    if (t.n < 1 || t.n > (1ll << 38) || t.at < 0 || t.at % kBlock || t.at > state->n ||
        (t.n + kBlock - 1) / kBlock * kBlock > state->n - t.at)
      return polyq_set_error(POLYQ_EINVAL, "%s: tensor %d: %lld elements at %lld of a state of %lld", who, i,
                             (long long)t.n, (long long)t.at, (long long)state->n);
    if (!(t.decay >= 0.f) || !std::isfinite(t.decay) || !(t.rate >= 0.f) || !std::isfinite(t.rate))
      return polyq_set_error(POLYQ_EINVAL, "%s: tensor %d: decay %g, rate %g", who, i, (double)t.decay, (double)t.rate);
  }
  return n_tensors <= kFew ? run_step<kFew>(tensors, n_tensors, p_type, grad_type, copy_type, state, hyper, stream, who)
                           : run_step<kMany>(tensors, n_tensors, p_type, grad_type, copy_type, state, hyper, stream, who);
}

extern "C" int polyq_adamw_values(const polyq_adamw_state* state, const polyq_dense* m, const polyq_dense* root,
                                  void* stream) {
  static const char* who = "polyq_adamw_values";
  polyq_clear_error();
  int rc = check_state(state, who);
  if (rc) return rc;
  if (state->bits != 8) return polyq_set_error(POLYQ_EINVAL, "%s: a state of %d bits", who, state->bits);
  if (!m && !root) return polyq_set_error(POLYQ_EINVAL, "%s: neither m nor root is wanted", who);
  ValuesParams P;
  memset(&P, 0, sizeof P);
  const polyq_dense* d[2] = {m, root};
  for (int i = 0; i < 2; ++i) {
    if (!d[i]) continue;
    if (!d[i]->data || !good_type(d[i]->type) || misaligned(d[i]->data, d[i]->type))
      return polyq_set_error(POLYQ_EINVAL, "%s: %s must be aligned to its elements", who, i ? "root" : "m");
    P.out[i] = d[i]->data;
    P.type[i] = d[i]->type;
  }
  P.m = (const uint8_t*)state->m;
  P.v = (const uint8_t*)state->v;
  P.ms = state->m_scales;
  P.vs = state->v_scales;
  P.blocks = (uint32_t)(state->n / kBlock);
  return launch((void*)adamw_values_kernel, P.blocks, 8, &P, stream, who);
}
