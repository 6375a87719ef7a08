// Layer norm (or, without the mean, RMS norm) and its backward pass.
//
//   hat = (x - mean) rstd,  y = hat w + b
//   g = dy w,  dx = res + rstd (g - mean(g) - hat mean(g hat))
//   dw = sum over rows of dy hat,  db = sum over rows of dy
//
// What has to move is x in and y out (forward), x, dy (and a residual gradient) in and dx
// out (backward), each once: 8192 x 5120 bf16 are 25 and 37 us of HBM.  A row's elements
// stay in registers or shared memory between the sums over them and its result, so that they
// are read once; the next rows are on their way meanwhile.  Forward and backward share rows
// out differently (see the kernels): the forward keeps a row in registers, the weight in
// shared memory; the backward keeps the rows' sums for dw and db in registers, and rows and
// weight in shared memory.  Rows that start anywhere come as the 16-byte pieces that hold
// them (fp32 3551 x 11811, training: 330 us, 508 with element loads).
//
// Measured, forward and backward with the residual gradient (by the profiler, operands from
// HBM): RMS norm of 8192 x 5120 bf16 33 + 64 + 4.5 us, 5.1 and 5.2 TB/s, bound by latency at the
// warps that registers leave room for: 38 instructions for an element backward, in packed fp32
// pairs, by 20 warps an SM that fill 66% of the issue slots; 17 forward (with mean and bias), by 28
// warps that fill 57% (shared memory, the row's barrier).  777 x 5003 fp16: 12.6 + 16.7 + 4.7 us, bound by the latency of three launches.  One row:
// 3.2 us, a launch.
#include <algorithm>
#include <atomic>
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
// Backward: warps of an SM, whose four parts have 16384 registers each.  Rows that a thread takes
// together once there are enough.
constexpr int kBackwardRegs = 96, kBackwardWarps = 4 * (16384 / (32 * kBackwardRegs)), kTogether = 2;
// Rows that these warps hold with eight columns a thread take eight, wider ones sixteen, in up to
// kWideThreads, which read hat and dy w twice (with a residual, as wide as 42 M elements of bf16, eight
// and sixteen: 1024, 2048, 4096 and 4608 columns 69 to 72 and 107 to 110 us, 5120 68 and 102; fp32 97 to 102 and
// 104 to 108; 21 warps, for 5376 columns, do not launch); small rows share up to kNarrowThreads.
constexpr int kNarrow = 8 * 32 * kBackwardWarps, kNarrowThreads = 256, kWideThreads = 512;
constexpr int kReduceCols = 32, kReduceRows = 16;
constexpr int kBackwardPerSm = 32 * kBackwardWarps;
constexpr int kMostSmem = 200 << 10;
constexpr int kSmSmem = 226 << 10, kStaticSmem = 14 << 10;  // of an SM; of a backward block, beside its rows

struct NormParams {
  const void* x;
  const void* dy;
  const void* res;
  void* y;  // y or dx
  const void* w;
  const void* b;
  float* stats;
  float* parts;  // [2][groups][K]: sums of dw and of db
  int64_t x_stride, dy_stride, res_stride, y_stride;
  int rows, K;
  float eps, inv_k;
  int w_type, b_type, vec_w, vec_b;  // vec: on 16 bytes
  int center, cluster, depth, staged, want_w, want_b;
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Sums over a row's threads of M values each (M a power of two; several rows' at once,
// so that their latencies are one).  The order is fixed: a butterfly in each warp, in
// which every step halves the values that a lane still holds; the warps' sums, which as
// many lanes per value as there are add in turn and by a butterfly; the cluster's blocks
// in order.  One barrier: `at` alternates between two places, and a place is written
// again only after the barrier of the sums between.
template <int M>
struct RowSums {
  static constexpr int S = 32 / M;  // lanes of a value
  float* warps;                     // [2][32][M] of this row's threads
  float* blocks;                    // [2][kMaxCluster][M]
  int nw, cluster, at;
  __device__ __forceinline__ void operator()(float (&v)[M]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, which = lane / S, part = lane % S;
    int n = M;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      if (n > 1) {
        n >>= 1;
#pragma unroll
        for (int i = 0; i < M / 2; ++i) {
          if (i >= n) break;
          const bool up = lane & o;
          const float keep = up ? v[i + n] : v[i], give = up ? v[i] : v[i + n];
          v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, o);
        }
      } else {
        v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], o);
      }
    }
    float s = v[0];
    if (nw > 1 || cluster > 1) {
      at ^= 1;
      float* w = warps + at * 32 * M;
      if (part == 0) w[warp * M + which] = s;
      __syncthreads();
      s = 0.f;
      for (int i = part; i < nw; i += S) s += w[i * M + which];
#pragma unroll
      for (int o = S / 2; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
      if (cluster > 1) {
        float* b = blocks + at * kMaxCluster * M;
        if (warp == 0 && part == 0) {
          const uint32_t mine = smem_u32(b + cluster_rank() * M + which);
          for (int r = 0; r < cluster; ++r) {
            uint32_t there;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine), "r"(r));
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there), "f"(s) : "memory");
          }
        }
        __syncwarp();
        cluster_sync();
        s = 0.f;
        for (int r = 0; r < cluster; ++r) s += b[r * M + which];
      }
    }
#pragma unroll
    for (int i = 0; i < M; ++i) v[i] = __shfl_sync(0xFFFFFFFFu, s, i * S);
  }
};

template <typename T>
__device__ __forceinline__ void pairs(const Raw8<T>& r, F2 (&v)[4]) {
  float f[8];
  to_float(r, f);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = f2(f[2 * i], f[2 * i + 1]);
}
template <bool VEC, typename T>
__device__ __forceinline__ void store_pairs(T* row, int col, int step, uint32_t mask, const F2 (&v)[4]) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 p = of(v[i]);
    f[2 * i] = p.x;
    f[2 * i + 1] = p.y;
  }
  store8<VEC>(row, col, step, mask, f);
}
// Zeros in the pairs of elements that are not there.
__device__ __forceinline__ void clear(F2 (&v)[4], uint32_t mask) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 p = of(v[i]);
    v[i] = f2(mask >> (2 * i) & 1 ? p.x : 0.f, mask >> (2 * i + 1) & 1 ? p.y : 0.f);
  }
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {  // the rest of 16: zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// A thread's eight elements of a row, on their way to its own place in shared memory (VEC; no
// other thread reads it, so that no barrier is needed).
template <typename T>
struct Rows {
  uint32_t at, piece;  // this thread's place, and bytes from one 16-byte piece to the next
  static constexpr int N16 = sizeof(T) * 8 / 16;
  __device__ __forceinline__ void ask(const T* row, int col, uint32_t mask, uint32_t slot) const {
    const int have = __popc(mask) * (int)sizeof(T);  // (the row's end: the rest is zeros)
#pragma unroll
    for (int i = 0; i < N16; ++i) {
      const int bytes = min(max(have - 16 * i, 0), 16);
      copy16(at + slot + i * piece, bytes ? row + col + i * (16 / (int)sizeof(T)) : row, bytes);
    }
  }
  __device__ __forceinline__ void get(uint32_t slot, F2 (&v)[4]) const {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < N16; ++i)
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(r.w[i].x), "=r"(r.w[i].y), "=r"(r.w[i].z), "=r"(r.w[i].w)
                   : "r"(at + slot + i * piece)
                   : "memory");
    pairs(r, v);
  }
  __device__ __forceinline__ void put(uint32_t slot, const F2 (&v)[4]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float2 a = of(v[2 * i]), b = of(v[2 * i + 1]);
      asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at + slot + i * piece), "f"(a.x), "f"(a.y), "f"(b.x),
                   "f"(b.y)
                   : "memory");
    }
  }
};
// A row that starts anywhere (not VEC): the 16-byte pieces of memory that hold it, copied by the
// row's threads together, of which each reads every T-th element; a barrier of theirs lies
// between.  A row begins up to 15 bytes into its place.  Nothing outside the tensor is read:
// before its first element (`first`) the piece is copied by elements, and none goes past the row.
template <typename T>
struct AnyRow {
  static __host__ __device__ constexpr uint32_t bytes(int cols) { return (cols * (uint32_t)sizeof(T) + 30) / 16 * 16; }
  static __device__ __forceinline__ void ask(const T* row, int cols, const void* first, uint32_t place) {
    const uintptr_t from = (uintptr_t)row, to = from + cols * sizeof(T), base = from & ~(uintptr_t)15;
    for (int i = threadIdx.x; base + 16 * i < to; i += blockDim.x) {
      const uintptr_t src = base + 16 * i;
      if (src >= (uintptr_t)first) {
        copy16(place + 16 * i, (const void*)src, (int)min((uintptr_t)16, to - src));
      } else {
        for (uintptr_t q = from; q < min(src + 16, to); q += sizeof(T)) {
          const uint32_t dst = place + (uint32_t)(q - base);
          if (sizeof(T) == 4) asm volatile("st.shared.u32 [%0], %1;" ::"r"(dst), "r"(__ldcg((const uint32_t*)q)) : "memory");
          else asm volatile("st.shared.u16 [%0], %1;" ::"r"(dst), "h"(__ldcg((const uint16_t*)q)) : "memory");
        }
      }
    }
  }
  // Elements col, col + step, ... of the row (those of `mask`).
  static __device__ __forceinline__ void get(const T* row, uint32_t place, int col, int step, uint32_t mask, F2 (&v)[4]) {
    const uint32_t at = place + (uint32_t)((uintptr_t)row & 15);
    Raw8<T> r;
    T* e = reinterpret_cast<T*>(r.w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t src = at + (mask >> i & 1 ? (uint32_t)(col + i * step) * (uint32_t)sizeof(T) : 0u);
      if constexpr (sizeof(T) == 4) {
        float f;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f) : "r"(src) : "memory");
        e[i] = mask >> i & 1 ? f : 0.f;
      } else {
        uint16_t h;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(src) : "memory");
        h = mask >> i & 1 ? h : (uint16_t)0;
        e[i] = *reinterpret_cast<const T*>(&h);
      }
    }
    pairs(r, v);
  }
};

// Waits for all but the last `left` (0 to 3) stages that have been asked for.
__device__ __forceinline__ void wait_stages(int left) {
  if (left == 0) asm volatile("cp.async.wait_group 0;" ::: "memory");
  else if (left == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else if (left == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else asm volatile("cp.async.wait_group 3;" ::: "memory");
}

// Eight elements of a weight or bias; the loads of each type are in flight together, and 16
// bytes wide where rows are VEC and the vector lies so (4 bytes of every 32 each time: 99 MB
// from L2 for 304 blocks, 10 us).
template <bool VEC, typename T>
__device__ __forceinline__ void vector8(const T* p, int vec, int col, int step, uint32_t mask, F2 (&v)[4]) {
  Raw8<T> r;
  if (VEC && vec) load8<true>(p, col, step, mask, r);
  else load8<false>(p, col, VEC ? 1 : step, mask, r);
  pairs(r, v);
}
template <bool VEC>
__device__ __forceinline__ void vector8(const void* p, int type, int vec, int col, int step, uint32_t mask,
                                        F2 (&v)[4]) {
  if (type == POLYQ_F32) vector8<VEC>((const float*)p, vec, col, step, mask, v);
  else if (type == POLYQ_BF16) vector8<VEC>((const __nv_bfloat16*)p, vec, col, step, mask, v);
  else vector8<VEC>((const __half*)p, vec, col, step, mask, v);
}

// A thread's groups of eight columns.
template <int G, bool VEC>
struct Columns {
  int col[G], step;
  uint32_t mask[G];
  __device__ __forceinline__ Columns(int c0, int T, int K) : step(T) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      col[g] = c0 + (VEC ? (g * T + (int)threadIdx.x) * 8 : g * 8 * T + (int)threadIdx.x);
      mask[g] = mask8<VEC>(col[g], T, K);
    }
  }
};

// Forward: W warps hold a row in registers as fp32 (threadIdx.x), C pieces of eight columns
// a lane; rows side by side (threadIdx.y) share a block, which keeps the weight and bias in
// shared memory as fp32 (from L2 for each row they were the L2's bound: 2048 x 5120 RMS norm
// 42 us, 37 now).  The next row is on its way to shared memory meanwhile.  The variance is of
// the differences from the mean, not of squares: nothing cancels.  All
// pieces but a lane's last are whole (W follows from that), so that the others need no checks.
constexpr int kForwardWarps = 24, kForwardRegs = 64;

template <typename TX, typename TY, bool VEC, int C>
__global__ void __maxnreg__(kForwardRegs) norm_forward_kernel(const __grid_constant__ NormParams P) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float parts[15][2][kForwardWarps];  // of rows side by side, in turns, of warps
  const int W = blockDim.x >> 5, R = blockDim.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, K = P.K;
  const int c0 = VEC ? 8 * (int)threadIdx.x : 256 * warp + lane, next = 256 * W;
  const uint32_t last = mask8<VEC>(c0 + (C - 1) * next, 32, K);
  pdl_trigger();
  pdl_wait();
  const int plane = (K + 7) / 8;
  const uint32_t ring = smem_u32(smem) + (VEC || P.staged ? ((P.w ? 2 : 0) + (P.b ? 2 : 0)) * plane * 16u : 0u);
  const uint32_t slot = blockDim.x * R * 8 * sizeof(TX);  // of a piece of all threads
  const Rows<TX> mine{ring + (threadIdx.y * blockDim.x + threadIdx.x) * 16u, (uint32_t)(blockDim.x * R * 16)};
  const uint32_t any_slot = AnyRow<TX>::bytes(K);
  auto any_place = [&](int stage) { return ring + (uint32_t)(stage * R + threadIdx.y) * any_slot; };
  auto ask = [&](int row, int stage) {
    if (row < P.rows) {
      const TX* x = (const TX*)P.x + (int64_t)row * P.x_stride;
      if constexpr (VEC) {
#pragma unroll
        for (int j = 0; j < C; ++j) mine.ask(x, c0 + j * next, j < C - 1 ? 0xFFu : last, (stage * C + j) * slot);
      } else {
        AnyRow<TX>::ask(x, K, P.x, any_place(stage));
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int row = blockIdx.x * R + threadIdx.y;
  ask(row, 0);
  // The weight and the bias: two planes each, the first and the second four of every eight columns.
  float4 *sw = reinterpret_cast<float4*>(smem), *sb = sw + (P.w ? 2 * plane : 0);
#pragma unroll 1
  for (int which = 0; which < 2; ++which) {
    const void* p = which ? P.b : P.w;
    if (!p || (!VEC && !P.staged)) continue;
    float4* to = which ? sb : sw;
    for (int i = threadIdx.y * blockDim.x + threadIdx.x; i < plane; i += blockDim.x * R) {
      F2 v[4];
      vector8<true>(p, which ? P.b_type : P.w_type, which ? P.vec_b : P.vec_w, 8 * i, 1, mask8<true>(8 * i, 1, K), v);
      const float2 q0 = of(v[0]), q1 = of(v[1]), q2 = of(v[2]), q3 = of(v[3]);
      to[i] = make_float4(q0.x, q0.y, q1.x, q1.y);
      to[plane + i] = make_float4(q2.x, q2.y, q3.x, q3.y);
    }
  }
  __syncthreads();
  // Four columns of a piece (its half h) from a staged vector (or, not VEC, of rows so wide that
  // it has no room beside them, from L2).
  auto staged4 = [&](const float4* at, const void* p, int type, int col, int h, F2& v0, F2& v1) {
    if (!VEC && !P.staged) {
      float f[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = col + 32 * (4 * h + e);
        f[e] = c < K ? any_load(p, type, c) : 0.f;
      }
      v0 = f2(f[0], f[1]), v1 = f2(f[2], f[3]);
    } else if (VEC) {
      const float4 x = at[h * plane + col / 8];
      v0 = f2(x.x, x.y), v1 = f2(x.z, x.w);
    } else {
      float f[4];
      const float* q = reinterpret_cast<const float*>(at);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = min(col + 32 * (4 * h + e), 8 * plane - 1);
        f[e] = q[((c >> 2 & 1) * plane + (c >> 3)) * 4 + (c & 3)];
      }
      v0 = f2(f[0], f[1]), v1 = f2(f[2], f[3]);
    }
  };
  int turn = 0;
  // A row's sum: the warp's butterfly, then a butterfly over its warps' sums.
  auto sum = [&](float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if (W == 1) return v;
    turn ^= 1;
    float* p = parts[threadIdx.y][turn];
    if (lane == 0) p[warp] = v;
    asm volatile("bar.sync %0, %1;" ::"r"((int)threadIdx.y + 1), "r"((int)blockDim.x) : "memory");
    v = lane < W ? p[lane] : 0.f;
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
  };
  for (int stage = 0; row < P.rows; row += gridDim.x * R, stage ^= 1) {
    ask(row + gridDim.x * R, stage ^ 1);
    wait_stages(1);
    if (!VEC) {  // (the row's pieces come from all of its threads)
      if (W == 1) __syncwarp();
      else asm volatile("bar.sync %0, %1;" ::"r"((int)threadIdx.y + 1), "r"((int)blockDim.x) : "memory");
    }
    F2 v[C][4];
#pragma unroll
    for (int j = 0; j < C; ++j) {
      if constexpr (VEC) mine.get((stage * C + j) * slot, v[j]);
      else
        AnyRow<TX>::get((const TX*)P.x + (int64_t)row * P.x_stride, any_place(stage), c0 + j * next, 32,
                        j < C - 1 ? 0xFFu : last, v[j]);
    }
    if (!VEC && W == 1) __syncwarp();  // (read before the next but one is asked for)
    float mean = 0.f;
    if (P.center) {
      F2 s = v[0][0];
#pragma unroll
      for (int i = 1; i < 4 * C; ++i) s = add2(s, v[i / 4][i % 4]);
      mean = sum(sum2(s)) * P.inv_k;
      const F2 minus = f2(-mean, -mean);
#pragma unroll
      for (int j = 0; j < C; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[j][e] = add2(v[j][e], minus);
      if (last != 0xFFu) clear(v[C - 1], last);
    }
    F2 q = mul2(v[0][0], v[0][0]);
#pragma unroll
    for (int i = 1; i < 4 * C; ++i) q = fma2(v[i / 4][i % 4], v[i / 4][i % 4], q);
    const float rstd = __frsqrt_rn(fmaf(sum(sum2(q)), P.inv_k, P.eps));
    if (P.stats && threadIdx.x == 0) reinterpret_cast<float2*>(P.stats)[row] = make_float2(mean, rstd);
    const F2 r = f2(rstd, rstd);
    TY* y = (TY*)P.y + (int64_t)row * P.y_stride;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int col = c0 + j * next;
      const uint32_t mask = j < C - 1 ? 0xFFu : last;
      if (!mask) break;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        F2 &x0 = v[j][2 * h], &x1 = v[j][2 * h + 1], w0, w1, b0, b1;
        x0 = mul2(x0, r), x1 = mul2(x1, r);
        if (P.w) staged4(sw, P.w, P.w_type, col, h, w0, w1);
        if (P.b) staged4(sb, P.b, P.b_type, col, h, b0, b1);
        if (P.w && P.b) x0 = fma2(x0, w0, b0), x1 = fma2(x1, w1, b1);
        else if (P.w) x0 = mul2(x0, w0), x1 = mul2(x1, w1);
        else if (P.b) x0 = add2(x0, b0), x1 = add2(x1, b1);
      }
      store_pairs<VEC>(y, col, 32, mask, v[j]);
    }
  }
}

// Backward: threadIdx.x: a row's threads (whole warps), threadIdx.y: rows side by side (one
// in a cluster); each takes NR rows together, blockDim.y apart.  Registers hold the sums over
// rows, and, with one group of columns (G), hat and dy w of the rows at hand until the sums
// over them are there; with two they are read from shared memory again.  A row's statistics
// are asked for a round ahead (8192 x 5120 bf16 with a residual: 78 us without that, 64 with it).
template <typename TX, typename TY, bool VEC, int NR, int G>
__global__ void __maxnreg__(kBackwardRegs) norm_backward_kernel(
    const __grid_constant__ NormParams P) {
  constexpr bool KEEP = G == 1;
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float warps[8][2 * 32 * 2 * NR];
  __shared__ float blocks[2 * kMaxCluster * 2 * NR];
  __shared__ float rows_sum[1024];
  const int T = blockDim.x, R = blockDim.y, me = threadIdx.y * T + threadIdx.x;
  const int rank = P.cluster > 1 ? (int)cluster_rank() : 0;
  const Columns<G, VEC> at(rank * T * 8 * G, T, P.K);
  RowSums<2 * NR> sums{warps[threadIdx.y], blocks, T >> 5, P.cluster, 0};
  pdl_trigger();
  pdl_wait();
  if (P.cluster > 1) cluster_sync();
  const int blocks_all = gridDim.x / P.cluster, mine = blockIdx.x / P.cluster, step = blocks_all * R * NR;
  int row0 = mine * R * NR + threadIdx.y;
  // VEC: groups of x, of dy and of the residual, of all threads; else rows, R of each
  const int c0 = rank * T * 8 * G, cols = min(T * 8 * G, P.K - c0);  // this block's columns
  const uint32_t x_group = VEC ? T * R * 8 * sizeof(TX) : AnyRow<TX>::bytes(T * 8 * G);
  const uint32_t d_group = VEC ? T * R * 8 * sizeof(TY) : AnyRow<TY>::bytes(T * 8 * G);
  const uint32_t d_at = (VEC ? G : R) * x_group, r_at = d_at + (VEC ? G : R) * d_group;
  const uint32_t slots = r_at + (P.res ? (VEC ? G : R) * x_group : 0);
  const Rows<TX> x{smem_u32(ring) + me * 16u, (uint32_t)(T * R * 16)};
  const Rows<TY> dy{x.at, x.piece};
  auto x_row = [&](int row) { return (const TX*)P.x + (int64_t)row * P.x_stride + (VEC ? 0 : c0); };
  auto d_row = [&](int row) { return (const TY*)P.dy + (int64_t)row * P.dy_stride + (VEC ? 0 : c0); };
  auto r_row = [&](int row) { return (const TX*)P.res + (int64_t)row * P.res_stride + (VEC ? 0 : c0); };
  auto any_place = [&](uint32_t slot, uint32_t part, uint32_t size) { return smem_u32(ring) + slot + part + threadIdx.y * size; };
  auto ask = [&](int from, int stage) {
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int row = from + i * R;
      if (row < P.rows) {
        const uint32_t slot = (stage * NR + i) * slots;
        if constexpr (VEC) {
#pragma unroll
          for (int g = 0; g < G; ++g) {
            x.ask(x_row(row), at.col[g], at.mask[g], slot + g * x_group);
            dy.ask(d_row(row), at.col[g], at.mask[g], slot + d_at + g * d_group);
            if (P.res) x.ask(r_row(row), at.col[g], at.mask[g], slot + r_at + g * x_group);
          }
        } else {
          AnyRow<TX>::ask(x_row(row), cols, P.x, any_place(slot, 0, x_group));
          AnyRow<TY>::ask(d_row(row), cols, P.dy, any_place(slot, d_at, d_group));
          if (P.res) AnyRow<TX>::ask(r_row(row), cols, P.res, any_place(slot, r_at, x_group));
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int i = 0; i < P.depth - 1; ++i) ask(row0 + i * step, i);
  F2 dw[G][4], db[G][4];
  const Rows<float> weight{x.at + P.depth * NR * slots, x.piece};  // this thread's eight of each group
#pragma unroll
  for (int g = 0; g < G; ++g) {
    F2 w[4] = {f2(1.f, 1.f), f2(1.f, 1.f), f2(1.f, 1.f), f2(1.f, 1.f)};
    if (P.w) vector8<VEC>(P.w, P.w_type, P.vec_w, at.col[g], T, at.mask[g], w);
    weight.put(g * T * R * 32, w);
#pragma unroll
    for (int e = 0; e < 4; ++e) dw[g][e] = db[g][e] = f2(0.f, 0.f);
  }
  float2 stat[NR], next[NR];  // (the next rows' are asked for before these rows are)
  auto stats_of = [&](int from) {
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int row = from + i * R;
      next[i] = row < P.rows ? __ldcg(reinterpret_cast<const float2*>(P.stats) + row) : make_float2(0.f, 0.f);
    }
  };
  stats_of(row0);
  for (int stage = 0; row0 - (int)threadIdx.y < P.rows; row0 += step) {
    const int there = stage == 0 ? P.depth - 1 : stage - 1;
#pragma unroll
    for (int i = 0; i < NR; ++i) stat[i] = make_float2(P.center ? next[i].x : 0.f, next[i].y);
    stats_of(row0 + step);
    if (VEC) {
      ask(row0 + (P.depth - 1) * step, there);
      wait_stages(P.depth - 1);
    } else {
      wait_stages(P.depth - 2);
      __syncthreads();  // the pieces of all threads are here, and the rows before have been read
      ask(row0 + (P.depth - 1) * step, there);
    }
    // hat and the gradient of a row's columns, zeros where there is no element (what the loads
    // give there is anything).
    auto read = [&](int i, int g, F2(&h)[4], F2(&d)[4]) {
      const uint32_t slot = (stage * NR + i) * slots;
      if constexpr (VEC) {
        x.get(slot + g * x_group, h);
        dy.get(slot + d_at + g * d_group, d);
      } else {
        const int row = row0 + i * R;
        AnyRow<TX>::get(x_row(row), any_place(slot, 0, x_group), at.col[g] - c0, T, at.mask[g], h);
        AnyRow<TY>::get(d_row(row), any_place(slot, d_at, d_group), at.col[g] - c0, T, at.mask[g], d);
      }
      const F2 minus = f2(-stat[i].x, -stat[i].x), r = f2(stat[i].y, stat[i].y);
#pragma unroll
      for (int e = 0; e < 4; ++e) h[e] = mul2(add2(h[e], minus), r);
      if (at.mask[g] != 0xFFu) {
        clear(h, at.mask[g]);
        clear(d, at.mask[g]);
      }
    };
    F2 hat[KEEP ? NR : 1][4], gw[KEEP ? NR : 1][4];  // hat and dy w
    float s[2 * NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      s[2 * i] = s[2 * i + 1] = 0.f;
      if (row0 + i * R >= P.rows) continue;  // (all threads of the row)
      F2 sh = f2(0.f, 0.f), sg = sh;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        F2(&h)[4] = hat[KEEP ? i : 0];
        F2(&d)[4] = gw[KEEP ? i : 0];
        F2 w[4];
        read(i, g, h, d);
        weight.get(g * T * R * 32, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          dw[g][e] = fma2(d[e], h[e], dw[g][e]);
          db[g][e] = add2(db[g][e], d[e]);
          d[e] = mul2(d[e], w[e]);
          sh = fma2(d[e], h[e], sh);
          sg = add2(sg, d[e]);
        }
      }
      s[2 * i] = sum2(sh);
      s[2 * i + 1] = sum2(sg);
    }
    if (P.y) {
      sums(s);
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const int row = row0 + i * R;
        if (row >= P.rows) continue;
        const float mgh = -s[2 * i] * P.inv_k, mg = P.center ? -s[2 * i + 1] * P.inv_k : 0.f;
        const F2 mgh2 = f2(mgh, mgh), mg2 = f2(mg, mg), r = f2(stat[i].y, stat[i].y);
#pragma unroll
        for (int g = 0; g < G; ++g) {
          F2(&h)[4] = hat[KEEP ? i : 0];
          F2(&d)[4] = gw[KEEP ? i : 0];
          F2 a[4] = {f2(0.f, 0.f), f2(0.f, 0.f), f2(0.f, 0.f), f2(0.f, 0.f)};
          if constexpr (!KEEP) {
            F2 w[4];
            read(i, g, h, d);
            weight.get(g * T * R * 32, w);
#pragma unroll
            for (int e = 0; e < 4; ++e) d[e] = mul2(d[e], w[e]);
          }
          if (P.res) {
            const uint32_t slot = (stage * NR + i) * slots;
            if constexpr (VEC) x.get(slot + r_at + g * x_group, a);
            else AnyRow<TX>::get(r_row(row), any_place(slot, r_at, x_group), at.col[g] - c0, T, at.mask[g], a);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) d[e] = fma2(r, fma2(h[e], mgh2, add2(d[e], mg2)), a[e]);
          store_pairs<VEC>((TX*)P.y + (int64_t)row * P.y_stride, at.col[g], T, at.mask[g], d);
        }
      }
    }
    if (++stage == P.depth) stage = 0;
  }
  // The rows side by side are added in order; a group of blocks writes its sums once.
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (!(which ? P.want_b : P.want_w)) continue;
    float* out = P.parts + ((int64_t)which * blocks_all + mine) * P.K;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      F2(&v)[4] = which ? db[g] : dw[g];
      for (int r = 1; r < R; ++r) {  // (two rows side by side have at most 128 threads each)
        F2* other = reinterpret_cast<F2*>(rows_sum) + threadIdx.x;
        __syncthreads();
        if ((int)threadIdx.y == r)
#pragma unroll
          for (int i = 0; i < 4; ++i) other[i * T] = v[i];
        __syncthreads();
        if (threadIdx.y == 0)
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = add2(v[i], other[i * T]);
      }
      if (threadIdx.y == 0) store_pairs<false>(out, at.col[g], VEC ? 1 : T, at.mask[g], v);
    }
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
  int groups, threads, rows, cluster, nr;  // of columns a thread; of a row; side by side; blocks of a row; together
  int64_t blocks;  // (clusters of them)
};
// `bytes`: of a column's x, dy and residual; two rows of a block and the weight fit into its
// shared memory.  (Fewer bytes never make for fewer blocks.)
Shape backward_shape(int64_t rows, int64_t K, int bytes, int sms) {
  Shape s;
  s.groups = K <= kNarrow ? 1 : 2;
  s.cluster = 1;
  const int most_cols = std::min(16 * kWideThreads, (kMostSmem - 512) / (2 * bytes + 4) / 512 * 512);
  while ((int64_t)s.cluster * most_cols < K) s.cluster *= 2;
  const int64_t cols = (K + s.cluster - 1) / s.cluster, warp = 256 * s.groups;
  s.threads = (int)((cols + warp - 1) / warp * 32);
  // small rows share a block once there is one for every SM
  s.rows = (int)std::min<int64_t>(std::max(1, kNarrowThreads / s.threads), (rows + sms - 1) / sms);
  const int64_t most = std::max(1, sms * std::max(1, kBackwardPerSm / (s.threads * s.rows)) / s.cluster);
  s.nr = rows >= kTogether * most * s.rows ? kTogether : 1;
  s.blocks = std::min<int64_t>((rows + s.rows * s.nr - 1) / (s.rows * s.nr), most);
  return s;
}
// Forward: pieces of a lane (1, 2 or 4), warps of a row, rows of a block.
struct ForwardShape {
  int c, warps, rows;
  int64_t blocks;
};
ForwardShape forward_shape(int64_t rows, int64_t K, bool vec, int sms) {
  ForwardShape s;
  const int n = (int)((K + 255) / 256), full = (int)(K / 256);  // a warp's pieces of 256 columns, whole ones
  // Many rows: the most pieces of which all but a lane's last are whole (two where rows start
  // anywhere: their addresses take the registers).  Few: as many warps as there are, for their latency.
  const int few = n <= kForwardWarps ? 1 : n <= 2 * kForwardWarps ? 2 : 4;
  s.c = rows < sms ? few : vec ? 4 : std::max(few, 2);
  while (s.c > 1 && (s.c - 1) * ((n + s.c - 1) / s.c) > full) s.c /= 2;
  s.warps = (n + s.c - 1) / s.c;
  const int fit = 65536 / kForwardRegs / 32;  // warps of an SM
  s.rows = (int)std::min<int64_t>(std::max(1, std::min(15, fit / s.warps)), (rows + sms - 1) / sms);
  s.blocks = std::min<int64_t>((rows + s.rows - 1) / s.rows, (int64_t)sms * std::max(1, fit / (s.warps * s.rows)));
  return s;
}

struct Variant {  // size: pieces of a lane (forward), groups of a thread (backward)
  bool backward, vec;
  int nr, size;
  int index(int tx, int ty) const {
    return ((tx * 3 + ty) * 2 + vec) * 7 + (backward ? 3 + (nr > 1) * 2 + size - 1 : size / 2);
  }
};
template <typename TX, typename TY, bool VEC>
void* pick(const Variant& v) {
  if (!v.backward)
    return v.size == 1   ? (void*)norm_forward_kernel<TX, TY, VEC, 1>
           : v.size == 2 ? (void*)norm_forward_kernel<TX, TY, VEC, 2>
                         : (void*)norm_forward_kernel<TX, TY, VEC, 4>;
  if (v.nr > 1)
    return v.size == 1 ? (void*)norm_backward_kernel<TX, TY, VEC, kTogether, 1> : (void*)norm_backward_kernel<TX, TY, VEC, kTogether, 2>;
  return v.size == 1 ? (void*)norm_backward_kernel<TX, TY, VEC, 1, 1> : (void*)norm_backward_kernel<TX, TY, VEC, 1, 2>;
}
template <typename TX, typename TY>
void* pick(const Variant& v) {
  return v.vec ? pick<TX, TY, true>(v) : pick<TX, TY, false>(v);
}
template <typename TX>
void* pick(int ty, const Variant& v) {
  return ty == POLYQ_F32 ? pick<TX, float>(v) : ty == POLYQ_BF16 ? pick<TX, __nv_bfloat16>(v) : pick<TX, __half>(v);
}
void* pick(int tx, int ty, const Variant& v) {
  return tx == POLYQ_F32 ? pick<float>(ty, v) : tx == POLYQ_BF16 ? pick<__nv_bfloat16>(ty, v) : pick<__half>(ty, v);
}

// Kernels whose shared memory has been allowed, by type, direction and rows, a bit for each device.
std::atomic<uint64_t> g_ready[128];

int allow_smem(void* f, int which, const char* who) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) {
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (g_ready[which].load(std::memory_order_acquire) & bit) return POLYQ_OK;
    e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem);
    if (e == cudaSuccess) g_ready[which].fetch_or(bit, std::memory_order_release);
  }
  if (e != cudaSuccess) return polyq_set_error(POLYQ_ECUDA, "%s: shared memory: %s", who, cudaGetErrorString(e));
  return POLYQ_OK;
}

int launch(void* f, dim3 grid, dim3 block, int smem, int cluster, void* params, void* stream, const char* who) {
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
  cfg.dynamicSmemBytes = smem;
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

// An output in the place of what it is made of: each row has to lie where its own input does, or a
// block overwrites rows that another has yet to read.
int check_in_place(const polyq_dense* out, const polyq_dense* in, int64_t rows, const char* who, const char* what) {
  if (out && in && out->data == in->data && (out->type != in->type || (rows > 1 && out->stride != in->stride)))
    return polyq_set_error(POLYQ_EINVAL, "%s: %s, in place, must have one type and stride", who, what);
  return POLYQ_OK;
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
  if (!rc) rc = check_in_place(y, x, rows, who, "x and y");
  if (rc) return rc;
  if (!(eps >= 0.f) || !std::isfinite(eps)) return polyq_set_error(POLYQ_EINVAL, "%s: eps %g", who, (double)eps);
  if ((uintptr_t)stats % 8) return polyq_set_error(POLYQ_EINVAL, "%s: stats must be 8-byte aligned", who);
  int sms = 0;
  rc = polyq_sm_count(&sms);
  if (rc) return rc;
  NormParams P;
  memset(&P, 0, sizeof P);
  P.x = x->data;
  P.x_stride = x->stride;
  P.y = y->data;
  P.y_stride = y->stride;
  if (weight) P.w = weight->data, P.w_type = weight->type, P.vec_w = (uintptr_t)weight->data % 16 == 0;
  if (bias) P.b = bias->data, P.b_type = bias->type, P.vec_b = (uintptr_t)bias->data % 16 == 0;
  P.stats = stats;
  P.rows = (int)rows;
  P.K = (int)K;
  P.eps = eps;
  P.inv_k = 1.f / (float)K;
  P.center = center != 0;
  bool vec = rows_on_16(x) && rows_on_16(y);
  ForwardShape s = forward_shape(rows, K, vec, sms);
  int smem = (int)(K + 7) / 8 * 32 * ((weight != nullptr) + (bias != nullptr));
  {  // two rows of each that lie side by side, on their way
    const int xb = x->type == POLYQ_F32 ? 4 : 2, any = ((int)K * xb + 30) / 16 * 16;
    if (vec && smem + 2 * s.warps * s.c * 256 * xb > kMostSmem) vec = false, s = forward_shape(rows, K, vec, sms);
    const int row = 2 * (vec ? s.warps * s.c * 256 * xb : any);  // (at most 196 640 bytes)
    P.staged = smem + row <= kMostSmem;
    if (!P.staged) smem = 0;
    s.rows = std::min(s.rows, (kMostSmem - smem) / row), smem += s.rows * row;
  }
  const Variant v{false, vec, 1, s.c};
  void* f = pick(x->type, y->type, v);
  if (smem > 32 << 10) rc = allow_smem(f, v.index(x->type, y->type), who);
  if (rc) return rc;
  return launch(f, dim3((unsigned)s.blocks), dim3(32 * s.warps, s.rows), smem, 1, &P, stream, who);
}

extern "C" int polyq_layernorm_workspace_bytes(int64_t rows, int64_t K, size_t* bytes) {
  static const char* who = "polyq_layernorm_workspace_bytes";
  polyq_clear_error();
  if (!bytes) return polyq_set_error(POLYQ_EINVAL, "%s: NULL argument", who);
  int rc = check_size(rows, K, who);
  int sms = 0;
  if (!rc) rc = polyq_sm_count(&sms);
  if (rc) return rc;
  *bytes = (size_t)backward_shape(rows, K, 4, sms).blocks * K * 2 * sizeof(float);
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
  if (!rc) rc = check_in_place(dx, dy, rows, who, "dy and dx");
  if (!rc) rc = check_in_place(dx, residual, rows, who, "the residual and dx");
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
  const int xb = x->type == POLYQ_F32 ? 4 : 2, yb = dy->type == POLYQ_F32 ? 4 : 2;
  const int bytes = xb * (residual ? 2 : 1) + yb;
  const Shape s = backward_shape(rows, K, bytes, sms);
  const bool sums = dweight || dbias;
  if (sums && (!workspace || (uintptr_t)workspace % 16 ||
               workspace_bytes < (size_t)s.blocks * K * 2 * sizeof(float)))
    return polyq_set_error(POLYQ_ENOMEM, "%s: workspace of %zu bytes, 16-byte aligned, needed", who,
                           (size_t)s.blocks * K * 2 * sizeof(float));
  NormParams P;
  memset(&P, 0, sizeof P);
  P.x = x->data;
  P.x_stride = x->stride;
  P.dy = dy->data;
  P.dy_stride = dy->stride;
  if (residual) P.res = residual->data, P.res_stride = residual->stride;
  if (dx) P.y = dx->data, P.y_stride = dx->stride;
  if (weight) P.w = weight->data, P.w_type = weight->type, P.vec_w = (uintptr_t)weight->data % 16 == 0;
  P.stats = const_cast<float*>(stats);
  P.parts = (float*)workspace;
  P.rows = (int)rows;
  P.K = (int)K;
  P.inv_k = 1.f / (float)K;
  P.center = center != 0;
  P.cluster = s.cluster;
  P.want_w = dweight != nullptr;
  P.want_b = dbias != nullptr;
  const bool vec = rows_on_16(x) && rows_on_16(dy) && (!residual || rows_on_16(residual)) && (!dx || rows_on_16(dx));
  const int cols = s.threads * s.rows * s.groups * 8;
  const int slack = 32 * 3 * s.rows;  // of rows that start anywhere
  int nr = s.nr, stage = (cols * bytes + (vec ? 0 : slack)) * nr;
  if (2 * stage + cols * 4 > kMostSmem) stage /= nr, nr = 1;
  const Variant v{true, vec, nr, s.groups};
  void* f = pick(x->type, dy->type, v);
  // As many rows on their way as the SM's blocks have room for (10817 x 1728 fp32 with two
  // stages 70 us, with three 64; 8192 x 5120 bf16 the same with both).
  const int share = std::min(kMostSmem, kSmSmem / std::max(1, kBackwardPerSm / (s.threads * s.rows)) - kStaticSmem);
  P.depth = std::max(2, std::min(4, (share - cols * 4) / stage));
  const int smem = stage * P.depth + cols * 4;
  if (smem > 32 << 10) rc = allow_smem(f, v.index(x->type, dy->type), who);
  if (rc) return rc;
  rc = launch(f, dim3((unsigned)(s.blocks * s.cluster)), dim3(s.threads, s.rows), smem, s.cluster, &P, stream, who);
  if (rc || !sums) return rc;
  ReduceParams Q;
  memset(&Q, 0, sizeof Q);
  Q.parts = P.parts;
  if (dweight) Q.out[0] = dweight->data, Q.type[0] = dweight->type;
  if (dbias) Q.out[1] = dbias->data, Q.type[1] = dbias->type;
  Q.groups = s.blocks;
  Q.K = K;
  return launch((void*)norm_reduce_kernel, dim3((unsigned)((K + kReduceCols - 1) / kReduceCols), 2),
                dim3(kReduceCols, kReduceRows), 0, 1, &Q, stream, who);
}
