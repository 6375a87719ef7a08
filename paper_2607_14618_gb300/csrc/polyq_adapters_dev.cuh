// Low-rank adapters of many requests beside a shared projection, on operands of
// one 16-bit type T.  For the rows of a segment with adapter i:
//
//   v = x A_i^T,  y = res + s_i v B_i^T              (forward)
//   dv = s_i dy B_i,  dx = res + dv A_i              (backward)
//   dA_i = dv^T x,  dB_i = s_i dy^T v                (sums over the adapter's rows)
//
// A rank is a few dozen, so that all of it is bound by HBM: x and dy in, y and dx
// in and out, the adapters in.  Three kernels: `shrink` (a long row times a thin
// matrix: v and dv), `expand` (a thin row times a wide matrix onto the residual: y
// and dx) and `gradients` (a product over the rows: dA and dB).  Operands come
// through shared memory by asynchronous copies, the products are mma.sync of
// 16-bit operands with fp32 sums: at these ranks the legacy tensor path keeps up
// with HBM, and needs no tensor memory, so that several small thread blocks share
// an SM and cover each other's latency.
//
// v and dv are in fp32 between the kernels.  As an operand each is the sum of two
// 16-bit numbers, v = h + l + O(2^-17 v) (bf16) or O(2^-22) (fp16), and both are
// multiplied: rounded once to 16 bits it would be off by 2^-9 of what an adapter
// adds.  fp16 has too few exponents for fp32's range: there v is scaled by a power
// of two, of a row's largest magnitude (expand) or of 64 rows' (gradients).
#pragma once
#include <type_traits>

#include "polyq_dense_dev.cuh"
#include "polyq_dev.cuh"
#include "polyq_finetune.h"

namespace polyq {
namespace lora {

constexpr int kThreads = 256;
constexpr int kMaxCluster = 8;

struct Segments {
  const int32_t* offsets;
  const int32_t* ids;
  int32_t n, rows;  // of segments, of the tensors' rows
};

// ---- instructions ----
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t bytes) {  // the rest of 16: zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
template <bool TRANS>
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
  if (TRANS)
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
  else
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
template <typename T>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (sizeof(T) == 2 && std::is_same<T, __half>::value)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// The sum over a cluster's blocks, in their order, of what lies at one place in their shared
// memory; all loads are under way before the first is added (one after another, eight blocks
// cost 0.3 us each for every number of a thread).
__device__ __forceinline__ uint32_t mapa(uint32_t addr, uint32_t rank) {
  uint32_t there;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(addr), "r"(rank));
  return there;
}
__device__ __forceinline__ float sum_cluster(uint32_t addr, int blocks) {
  float v[kMaxCluster], s = 0.f;
#pragma unroll
  for (int r = 0; r < kMaxCluster; ++r) {
    v[r] = 0.f;
    if (r < blocks) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[r]) : "r"(mapa(addr, r)) : "memory");
  }
#pragma unroll
  for (int r = 0; r < kMaxCluster; ++r) s += v[r];
  return s;
}
__device__ __forceinline__ float4 sum_cluster4(uint32_t addr, int blocks) {
  float4 v[kMaxCluster], s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int r = 0; r < kMaxCluster; ++r) {
    v[r] = s;
    if (r < blocks)
      asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                   : "=f"(v[r].x), "=f"(v[r].y), "=f"(v[r].z), "=f"(v[r].w)
                   : "r"(mapa(addr, r))
                   : "memory");
  }
#pragma unroll
  for (int r = 0; r < kMaxCluster; ++r) s.x += v[r].x, s.y += v[r].y, s.z += v[r].z, s.w += v[r].w;
  return s;
}

// ---- tiles in shared memory ----
// Rows of C 16-byte pieces, of which eight in a row of ldmatrix lie in different
// banks: the pieces of rows that start in the same bank are permuted.
template <int C>
__device__ __forceinline__ uint32_t piece(int row, int c) {
  const int s = C >= 8 ? row & 7 : (row / (8 / C)) & (C - 1);
  return (uint32_t)(row * C + (c ^ s)) * 16u;
}
// A operand (16 rows m, 16 of the contraction k) from rows [m][k], or TRANS [k][m].
template <int C, bool TRANS>
__device__ __forceinline__ void frag_a(uint32_t tile, int m, int k, uint32_t (&r)[4]) {
  const int lane = threadIdx.x & 31, i = lane >> 3, j = lane & 7;
  if (TRANS) ldmatrix4<true>(tile + piece<C>(k + (i >> 1) * 8 + j, m / 8 + (i & 1)), r);
  else ldmatrix4<false>(tile + piece<C>(m + (i & 1) * 8 + j, k / 8 + (i >> 1)), r);
}
// B operand of two tiles (8 columns n each; r[0..1], r[2..3]) from rows [n][k], or TRANS [k][n].
template <int C, bool TRANS>
__device__ __forceinline__ void frag_b(uint32_t tile, int n, int k, uint32_t (&r)[4]) {
  const int lane = threadIdx.x & 31, i = lane >> 3, j = lane & 7;
  if (TRANS) ldmatrix4<true>(tile + piece<C>(k + (i & 1) * 8 + j, n / 8 + (i >> 1)), r);
  else ldmatrix4<false>(tile + piece<C>(n + (i >> 1) * 8 + j, k / 8 + (i & 1)), r);
}
// A thread's pieces of a tile of ROWS x C pieces that comes from rows of `stride`
// elements: the same piece of every kThreads / C-th row, so that one pointer, one place and
// one length serve them all (with an address, a bound and a swizzle computed for each
// piece, copies took 60 instructions and bound the kernels).  Elements from `cols` on
// (counted from the tile's first) and rows from `rows` on are zeros.
template <int ROWS, int C, int ELEM = 2>
struct Mover {
  static constexpr int E = 16 / ELEM, EACH = kThreads / C;  // elements of a piece; rows from one to the next
  const char* p;
  int64_t step;  // bytes of EACH rows
  uint32_t dst, bytes;
  int row;
  __device__ __forceinline__ Mover(const void* src, int64_t stride, int cols, uint32_t place) {
    const int c = threadIdx.x % C;
    row = threadIdx.x / C;
    p = (const char*)src + ((int64_t)row * stride + c * E) * ELEM;
    step = stride * EACH * ELEM;
    dst = place;
    limit(cols);
  }
  __device__ __forceinline__ void limit(int cols) {
    bytes = (uint32_t)(min(max(cols - (int)(threadIdx.x % C) * E, 0), E) * ELEM);
  }
  // The tile that begins `off` bytes after src.
  __device__ __forceinline__ void copy(uint32_t tile, int64_t off, int rows) const {
    if (ROWS * C < kThreads && threadIdx.x >= ROWS * C) return;
    const char* q = p + off;
#pragma unroll
    for (int i = 0; i < (ROWS * C + kThreads - 1) / kThreads; ++i) {
      const bool in = row + i * EACH < rows && bytes;
      cp_async16(tile + dst + i * kThreads * 16, in ? q : p, in ? bytes : 0u);
      q += step;
    }
  }
};
// The same of rows that start anywhere: neighbouring elements by neighbouring threads, through
// registers (asynchronous copies want 16 bytes, and eight loads of a piece by one thread would
// ask L2 for its sector eight times).
template <int ROWS, int C>
__device__ __forceinline__ void copy_any(uint8_t* tile, const void* src, int64_t stride, int rows, int cols) {
  constexpr int COLS = 8 * C, EACH = ROWS * COLS / kThreads, PART = EACH < 16 ? EACH : 16;
#pragma unroll 1
  for (int i0 = 0; i0 < EACH; i0 += PART) {
    uint16_t v[PART];
#pragma unroll
    for (int i = 0; i < PART; ++i) {
      const int e = (i0 + i) * kThreads + threadIdx.x, row = e / COLS, c = e % COLS;
      v[i] = row < rows && c < cols ? __ldcg((const uint16_t*)src + row * stride + c) : (uint16_t)0;
    }
#pragma unroll
    for (int i = 0; i < PART; ++i) {
      const int e = (i0 + i) * kThreads + threadIdx.x, row = e / COLS, c = e % COLS;
      *reinterpret_cast<uint16_t*>(tile + piece<C>(row, c / 8) + c % 8 * 2) = v[i];
    }
  }
}
template <int C>
__device__ __forceinline__ uint32_t my_piece() {
  return piece<C>(threadIdx.x / C, threadIdx.x % C);
}

// ---- which rows ----
// A tile of at most bm rows of one segment.
struct Tile {
  int32_t id, row, rows;
};
// Tile number `tile` of all segments' in turn (the whole block calls; false: there are
// fewer).  Offsets outside the tensors' rows are held at their ends.  One warp looks: every
// block reads the same few lines (48 rows of rank 64 27 us; 29 where every warp looks for itself,
// and 41 with four neighbouring segments a lane of those).
__device__ __forceinline__ bool find_tile(const Segments& s, int bm, int tile, Tile& t) {
  __shared__ Tile found;
  const int lane = threadIdx.x & 31;
  if (threadIdx.x < 32) {
    int before = 0;
    bool there = false;
    for (int s0 = 0; s0 < s.n && !there; s0 += 128) {  // four segments a lane, all loads under way together
      int from[4], to[4], id[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = s0 + 32 * k + lane;
        from[k] = to[k] = 0, id[k] = -1;
        if (i < s.n) {
          id[k] = __ldcg(s.ids + i);
          from[k] = min(max(__ldcg(s.offsets + i), 0), s.rows);
          to[k] = min(max(__ldcg(s.offsets + i + 1), 0), s.rows);
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int n = to[k] > from[k] ? (to[k] - from[k] - 1) / bm + 1 : 0;
        int sum = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(0xFFFFFFFFu, sum, o);
          if (lane >= o) sum += v;
        }
        const int first = before + sum - n;
        if (first <= tile && tile < first + n) {
          const int row = from[k] + (tile - first) * bm;
          found = Tile{id[k], row, min(bm, to[k] - row)};
        }
        before += __shfl_sync(0xFFFFFFFFu, sum, 31);
        there = there || tile < before;
      }
    }
    if (lane == 0 && !there) found.rows = 0;
  }
  __syncthreads();
  t = found;
  return t.rows > 0;
}
// The tiles of all segments of one adapter, every `stride`-th from `first` on.
struct AdapterTiles {
  int s0, from, to, row, end, skip;
  uint32_t mine;  // segments of the 32 from s0 on
  __device__ __forceinline__ void begin(int first) {
    s0 = -32;
    mine = 0;
    row = end = 0;
    skip = first;
  }
  __device__ __forceinline__ bool next(const Segments& s, int id, int bm, int stride, int& at, int& rows) {
    const int lane = threadIdx.x & 31;
    for (;;) {
      while (row >= end) {
        while (!mine) {
          s0 += 32;
          if (s0 >= s.n) return false;
          const int i = s0 + lane;
          int whose = -1;
          from = to = 0;
          if (i < s.n) {
            whose = __ldcg(s.ids + i);
            from = min(max(__ldcg(s.offsets + i), 0), s.rows);
            to = min(max(__ldcg(s.offsets + i + 1), 0), s.rows);
          }
          mine = __ballot_sync(0xFFFFFFFFu, whose == id && to > from);
        }
        const int src = __ffs(mine) - 1;
        mine &= mine - 1;
        row = __shfl_sync(0xFFFFFFFFu, from, src);
        end = __shfl_sync(0xFFFFFFFFu, to, src);
      }
      at = row;
      rows = min(bm, end - row);
      row += bm;
      if (skip-- == 0) {
        skip = stride - 1;
        return true;
      }
    }
  }
};

// ---- v as two 16-bit numbers ----
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {  // a in the lower half
  uint32_t r;
  if constexpr (std::is_same<T, __half>::value) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if constexpr (std::is_same<T, __half>::value) return __half22float2(*reinterpret_cast<const __half2*>(&w));
  return make_float2(bf16_lo(w), bf16_hi(w));
}
template <typename T>
__device__ __forceinline__ void split8(const float (&v)[8], float scale, uint4& h, uint4& l) {
  constexpr uint32_t INF = std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u;
  uint32_t eh[4], el[4], top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = v[2 * i] * scale, b = v[2 * i + 1] * scale;
    eh[i] = pack2<T>(a, b);
    const float2 f = unpack2<T>(eh[i]);
    el[i] = pack2<T>(a - f.x, b - f.y);
    top = __vmaxu2(top, eh[i] & 0x7FFF7FFFu);
  }
  if (max(top & 0xFFFFu, top >> 16) >= INF) {  // what is not finite is so once
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if ((eh[i] & 0x7FFFu) >= INF) el[i] &= 0xFFFF0000u;
      if ((eh[i] >> 16 & 0x7FFFu) >= INF) el[i] &= 0xFFFFu;
    }
  }
  h = make_uint4(eh[0], eh[1], eh[2], eh[3]);
  l = make_uint4(el[0], el[1], el[2], el[3]);
}
// 2^e and 2^-e that bring the largest magnitude (its bits) to 2^14 .. 2^15, both normal numbers.
__device__ __forceinline__ uint32_t scale_bits(uint32_t top) {
  return (uint32_t)min(max(127 + 14 + 127 - (int)(top >> 23), 1), 253);
}
__device__ __forceinline__ float scale_down(uint32_t top) { return __uint_as_float(scale_bits(top) << 23); }
__device__ __forceinline__ float scale_up(uint32_t top) { return __uint_as_float((254u - scale_bits(top)) << 23); }
// The bits of the largest magnitude that is finite (one rank's infinity scales no other's away).
__device__ __forceinline__ uint32_t abs_bits(const float (&v)[8]) {
  constexpr uint32_t INF = 0x7F800000u;
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  if (m >= INF) {
    m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t b = __float_as_uint(v[i]) & 0x7FFFFFFFu;
      m = max(m, b < INF ? b : 0u);
    }
  }
  return m;
}
__device__ __forceinline__ void load_v8(const float* p, bool there, float (&v)[8]) {
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
  if (there) {
    a = __ldcg(reinterpret_cast<const float4*>(p));
    b = __ldcg(reinterpret_cast<const float4*>(p) + 1);
  }
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
  v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}

struct Side {  // an adapter's matrix: `next` elements from one to the next, rows of `stride`
  const void* w;
  int64_t next, stride;
};

// ---------------------------------------------------------------------------
// v[t][j] = s sum_k x[t][k] W[j][k]   (TRANS: W[k][j])
// ---------------------------------------------------------------------------
struct ShrinkParams {
  const void* x;
  Side w;
  float* v;  // [rows][R]
  const float* scales;  // NULL: s = 1
  const int32_t* ranks;
  int* status;
  Segments seg;
  int64_t x_stride, K;
  int32_t R, adapters, cluster;
  int32_t map_next;          // 1; 0: all adapters are w_map's first
  CUtensorMap x_map, w_map;  // (shrink_tiled_kernel)
};

// A cluster's blocks share the contraction of one tile of BM rows and add their
// sums through distributed shared memory, each a part of the tile, in the blocks'
// order.  Few rows (BM = 16): the adapters' bytes, which each row or few rows read anew: 48
// requests of rank 64 on 5120 columns 12.8 us, 31 MB at 2.5 TB/s, half of it launch, offsets
// and the cluster's exchange.
template <typename T, int BM, int RN, bool TRANS>
struct Shrink {
  static_assert(BM == 16, "tiles of few rows");
  static constexpr int KC = 128;                  // contraction of a stage
  static constexpr int STAGES = RN == 64 ? 3 : 4;  // (three blocks to an SM)
  static constexpr int WN = RN / 16, WK = 8 / WN;  // warps along the rank (16 each) and the contraction of a stage
  static constexpr int X_BYTES = BM * KC * 2, W_BYTES = RN * KC * 2;
  static constexpr int RED_BYTES = WK * BM * RN * 4;
  static constexpr int SMEM = STAGES * (X_BYTES + W_BYTES) > RED_BYTES ? STAGES * (X_BYTES + W_BYTES) : RED_BYTES;
};

// Adds the tile's sums [WK][BM][RN] of the cluster's blocks, each block a part of the tile.
template <int BM, int RN, int WK>
__device__ __forceinline__ void shrink_finish(const ShrinkParams& P, const Tile& t, uint32_t base, const uint8_t* smem,
                                              int rank) {
  const int own = P.ranks ? min(max(__ldcg(P.ranks + t.id), 0), P.R) : P.R;
  const float s = P.scales ? __ldcg(P.scales + t.id) : 1.f;
  if (P.cluster > 1) cluster_sync();
  else __syncthreads();
  const int part = BM * RN / 4 / P.cluster;  // four columns each
  for (int i = rank * part + threadIdx.x; i < (rank + 1) * part; i += blockDim.x) {
    const int row = 4 * i / RN, col = 4 * i % RN;
    if (row >= t.rows) break;
    if (col >= P.R) continue;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int q = 0; q < WK; ++q) {
      const int at = q * BM * RN + 4 * i;
      const float4 w = P.cluster > 1 ? sum_cluster4(base + at * 4, P.cluster)
                                     : *reinterpret_cast<const float4*>(smem + at * 4);
      v.x += w.x, v.y += w.y, v.z += w.z, v.w += w.w;
    }
    v.x = col < own ? v.x * s : 0.f;
    v.y = col + 1 < own ? v.y * s : 0.f;
    v.z = col + 2 < own ? v.z * s : 0.f;
    v.w = col + 3 < own ? v.w * s : 0.f;
    *reinterpret_cast<float4*>(P.v + (int64_t)(t.row + row) * P.R + col) = v;  // (R is a multiple of 8)
  }
  if (P.cluster > 1) cluster_sync();  // (another block may still read this one's sums)
}

// ANY: rows of x start anywhere.
template <typename T, int BM, int RN, bool TRANS, bool ANY>
__global__ void __launch_bounds__(kThreads) shrink_kernel(const __grid_constant__ ShrinkParams P) {
  using S = Shrink<T, BM, RN, TRANS>;
  constexpr int KC = S::KC, CX = KC / 8, CW = TRANS ? RN / 8 : KC / 8;
  extern __shared__ __align__(128) uint8_t smem[];
  const uint32_t base = smem_u32(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = P.cluster > 1 ? (int)cluster_rank() : 0;
  pdl_wait();
  pdl_trigger();  // (not before the wait: what follows reads what this grid has waited for)
  Tile t;
  if (!find_tile(P.seg, BM, blockIdx.x / P.cluster, t)) return;  // the whole cluster
  if (t.id < 0 || t.id >= P.adapters) return;
  const int rank_of = P.ranks ? __ldcg(P.ranks + t.id) : P.R;  // (used once the copies of x are under way)
  const T* x = (const T*)P.x + (int64_t)t.row * P.x_stride;
  const T* w = (const T*)P.w.w + (int64_t)t.id * P.w.next;
  const int64_t chunks = (P.K + KC - 1) / KC;
  const int64_t c0 = chunks * rank / P.cluster, c1 = chunks * (rank + 1) / P.cluster;

  Mover<BM, CX> mx(x, P.x_stride, KC, my_piece<CX>());
  auto copy_x = [&](int64_t c, int stage) {
    const int left = (int)min(P.K - c * KC, (int64_t)KC);
    if constexpr (ANY) {
      copy_any<BM, CX>(smem + stage * (S::X_BYTES + S::W_BYTES), x + c * KC, P.x_stride, t.rows, left);
    } else {
      if (left < KC) mx.limit(left);  // the contraction's end
      mx.copy(base + stage * (S::X_BYTES + S::W_BYTES), c * (KC * 2), t.rows);
    }
  };
  for (int i = 0; i < S::STAGES - 1; ++i)
    if (c0 + i < c1) copy_x(c0 + i, i);
  const int own = min(max(rank_of, 0), P.R);
  Mover<TRANS ? KC : RN, CW> mw(w, P.w.stride, TRANS ? own : KC, my_piece<CW>());
  auto copy_w = [&](int64_t c, int stage) {
    const int left = (int)min(P.K - c * KC, (int64_t)KC);
    if (!TRANS && left < KC) mw.limit(left);
    mw.copy(base + stage * (S::X_BYTES + S::W_BYTES) + S::X_BYTES, c * (TRANS ? P.w.stride * KC * 2 : KC * 2),
            TRANS ? left : own);
  };
  float acc[2][4] = {};
  const int wn = warp % S::WN, wk = warp / S::WN;
  for (int i = 0; i < S::STAGES - 1; ++i) {
    if (c0 + i < c1) copy_w(c0 + i, i);
    cp_commit();  // (the first with all that x has asked for)
  }
  int stage = 0;
  for (int64_t c = c0; c < c1; ++c) {
    cp_wait<S::STAGES - 2>();
    __syncthreads();
    if (c + S::STAGES - 1 < c1) {
      const int there = stage == 0 ? S::STAGES - 1 : stage - 1;
      copy_x(c + S::STAGES - 1, there);
      copy_w(c + S::STAGES - 1, there);
    }
    cp_commit();
    const uint32_t at = base + stage * (S::X_BYTES + S::W_BYTES);
    if (++stage == S::STAGES) stage = 0;
    float sum[2][4] = {};  // of the stage: the tensor cores cut running sums off
#pragma unroll
    for (int k = wk * 16; k < KC; k += 16 * S::WK) {
      uint32_t a[4], b[4];
      frag_a<CX, false>(at, 0, k, a);
      frag_b<CW, TRANS>(at + S::X_BYTES, wn * 16, k, b);
      mma<T>(sum[0], a, b[0], b[1]);
      mma<T>(sum[1], a, b[2], b[3]);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[j][e] += sum[j][e];
  }
  cp_wait<0>();
  __syncthreads();
  float* red = reinterpret_cast<float*>(smem) + wk * BM * RN;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int row = lane / 4, col = wn * 16 + j * 8 + lane % 4 * 2;
    *reinterpret_cast<float2*>(red + row * RN + col) = make_float2(acc[j][0], acc[j][1]);
    *reinterpret_cast<float2*>(red + (row + 8) * RN + col) = make_float2(acc[j][2], acc[j][3]);
  }
  shrink_finish<BM, RN, S::WK>(P, t, base, smem, rank);
}

// The same for tiles of 64 or 128 rows: a ninth warp asks the TMA unit for whole stages, whose
// barriers the eight others wait on, each by itself.  (With copies by all threads and a barrier
// of the block for every stage, half of the instructions were the copies'.)  A tile's rows past
// its segment, and columns past its rank, are what lies there: their sums are not used.
// 6007 rows of 13824 columns, ranks to 32: 33 us, 5.0 TB/s; 4096 of 5120 and of 13824, rank 64:
// 20 and 32 us (2.1 and 3.6 TB/s: one wave of tiles, which fill and finish together).
template <typename T, int BM, int RN, bool TRANS>
struct Tiled {
  static constexpr int KC = BM == 128 ? 64 : 128;  // contraction of a stage, in panels of 64
  static constexpr int PANELS = KC / 64;
  static constexpr int WM = 4, WN = RN == 16 ? 1 : 2, WK = 8 / (WM * WN);
  static constexpr int MT = BM / 64, NT = RN / 8 / WN;
  static constexpr int X_BYTES = BM * KC * 2, W_BYTES = RN * KC * 2, STAGE = X_BYTES + W_BYTES;
  static constexpr int STAGES = BM == 128 ? (RN == 64 ? 4 : 3) : RN == 128 ? 2 : 3;  // (two or three blocks to an SM)
  static constexpr int RED_BYTES = WK * BM * RN * 4;
  static constexpr int SMEM = 1024 + (STAGES * STAGE > RED_BYTES ? STAGES * STAGE : RED_BYTES);
};

template <typename T, int BM, int RN, bool TRANS>
__global__ void __launch_bounds__(kThreads + 32, RN == 128 ? 1 : BM == 64 && RN <= 32 ? 3 : 2) shrink_tiled_kernel(const __grid_constant__ ShrinkParams P) {
  using S = Tiled<T, BM, RN, TRANS>;
  constexpr int KC = S::KC, CW = TRANS && RN < 64 ? RN / 8 : 8;
  extern __shared__ uint8_t raw_smem[];
  __shared__ __align__(8) uint64_t bars[2 * S::STAGES];
  const uint32_t base = (smem_u32(raw_smem) + 1023u) & ~1023u, full = smem_u32(bars), empty = full + 8 * S::STAGES;
  uint8_t* smem = raw_smem + (base - smem_u32(raw_smem));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = P.cluster > 1 ? (int)cluster_rank() : 0;
  if (threadIdx.x == 0) {
    for (int i = 0; i < S::STAGES; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 8);
    }
    mbar_fence_init();
  }
  if (warp == 8 && elect_one()) {
    prefetch_tmap(&P.x_map);
    prefetch_tmap(&P.w_map);
  }
  pdl_wait();
  pdl_trigger();  // (not before the wait: what follows reads what this grid has waited for)
  Tile t;
  if (!find_tile(P.seg, BM, blockIdx.x / P.cluster, t)) return;  // the whole cluster
  if (t.id < 0 || t.id >= P.adapters) return;
  const int chunks = (int)((P.K + KC - 1) / KC);
  const int c0 = (int)((int64_t)chunks * rank / P.cluster), c1 = (int)((int64_t)chunks * (rank + 1) / P.cluster);
  float acc[S::MT][S::NT][4] = {};
  const int wm = warp % S::WM, wn = warp / S::WM % S::WN, wk = warp / (S::WM * S::WN);
  if (warp == 8) {
    if (elect_one()) {
      int asked = 0;
      for (int c = c0; c < c1; ++c, ++asked) {
        const int stage = asked % S::STAGES;
        const uint32_t bar = full + 8 * stage, at = base + stage * S::STAGE;
        if (asked >= S::STAGES && !mbar_wait(empty + 8 * stage, (asked / S::STAGES - 1) & 1)) {
          atomicExch(P.status, kStatusTimeoutEmpty);
          break;
        }
        mbar_expect_tx(bar, S::STAGE);
#pragma unroll
        for (int q = 0; q < S::PANELS; ++q) {
          tma_load_3d(at + q * BM * 128, &P.x_map, c * KC + q * 64, t.row, 0, bar);
          if (!TRANS) tma_load_3d(at + S::X_BYTES + q * RN * 128, &P.w_map, c * KC + q * 64, 0, t.id * P.map_next, bar);
        }
        if (TRANS)
#pragma unroll
          for (int q = 0; q < (RN + 63) / 64; ++q)
            tma_load_3d(at + S::X_BYTES + q * KC * 128, &P.w_map, q * 64, c * KC, t.id * P.map_next, bar);
      }
      // no copy is under way when the block ends, whether its stages were awaited or not
      for (int i = asked > S::STAGES ? asked - S::STAGES : 0; i < asked; ++i)
        if (!mbar_wait(full + 8 * (i % S::STAGES), (i / S::STAGES) & 1)) break;
    }
    __syncwarp();
  } else {
    bool ok = true;
    for (int i = 0; i < c1 - c0; ++i) {
      const int stage = i % S::STAGES;
      const uint32_t at = base + stage * S::STAGE;
      if (ok && !mbar_wait(full + 8 * stage, (i / S::STAGES) & 1)) {
        ok = false;
        atomicExch(P.status, kStatusTimeoutFull);
      }
      if (!ok) continue;
      float sum[S::MT][S::NT][4] = {};  // of the stage: the tensor cores cut running sums off
#pragma unroll
      for (int k = wk * 16; k < KC; k += 16 * S::WK) {
        const uint32_t xt = at + k / 64 * (BM * 128), wt = at + S::X_BYTES + (TRANS ? 0 : k / 64 * (RN * 128));
        uint32_t a[S::MT][4];
#pragma unroll
        for (int m = 0; m < S::MT; ++m) frag_a<8, false>(xt, (wm * S::MT + m) * 16, k % 64, a[m]);
#pragma unroll
        for (int j = 0; j < S::NT; j += 2) {
          const int n = (wn * S::NT + j) * 8;
          uint32_t b[4];
          if (TRANS) frag_b<CW, true>(wt + n / 64 * (KC * 128), n % 64, k, b);
          else frag_b<8, false>(wt, n, k % 64, b);
#pragma unroll
          for (int m = 0; m < S::MT; ++m) {
            mma<T>(sum[m][j], a[m], b[0], b[1]);
            mma<T>(sum[m][j + 1], a[m], b[2], b[3]);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty + 8 * stage);
#pragma unroll
      for (int m = 0; m < S::MT; ++m)
#pragma unroll
        for (int j = 0; j < S::NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[m][j][e] += sum[m][j][e];
    }
  }
  __syncthreads();
  if (warp < 8) {
    float* red = reinterpret_cast<float*>(smem) + wk * BM * RN;
#pragma unroll
    for (int i = 0; i < S::MT; ++i)
#pragma unroll
      for (int j = 0; j < S::NT; ++j) {
        const int row = (wm * S::MT + i) * 16 + lane / 4, col = (wn * S::NT + j) * 8 + lane % 4 * 2;
        *reinterpret_cast<float2*>(red + row * RN + col) = make_float2(acc[i][j][0], acc[i][j][1]);
        *reinterpret_cast<float2*>(red + (row + 8) * RN + col) = make_float2(acc[i][j][2], acc[i][j][3]);
      }
  }
  shrink_finish<BM, RN, S::WK>(P, t, base, smem, rank);
}

// ---------------------------------------------------------------------------
// y[t][n] = res[t][n] + s sum_j v[t][j] W[n][j]   (TRANS: W[j][n])
// ---------------------------------------------------------------------------
struct ExpandParams {
  const float* v;
  Side w;
  const void* res;
  void* y;
  const float* scales;
  const int32_t* ranks;
  Segments seg;
  int64_t res_stride, y_stride, N;
  int32_t R, adapters, tiles, vec;
};

// A block takes BM rows of a segment and every G-th tile of BN columns.  v is held in
// registers as two operands; the tiles' weights and residuals are on their way to shared
// memory STAGES - 1 tiles ahead.  A warp's sums are added to the residual in its place
// there, and go out in whole 128-byte lines (BM = 64): without a barrier, as no other
// warp touches them.  6007 rows onto 5120 columns, ranks to 32: 35 us, 3.5 TB/s; 4096 onto
// 13824 and 5120, rank 64: 61 and 29 us (3.7 and 2.9 TB/s), where the two products alone are
// 12 and 4.5 us each of mma.sync's 598 TFLOP/s (measured).  Stages by the TMA unit with barriers were slower
// (60 -> 82 us): copies and sums share the shared memory's bandwidth either way.
template <typename T, int BM, int RN, bool TRANS, typename TY>
struct Expand {
  static constexpr int BN = RN == 128 && BM == 64 ? 64 : 128;
  static constexpr int WM = BM / 16, WN = 8 / WM, NW = BN / WN, NT = NW / 8;  // warps; columns of a warp
  static constexpr int STAGES = sizeof(TY) == 4 && BM == 64 ? 2 : 3;
  static constexpr int V_BYTES = BM * RN * 2, W_BYTES = BN * RN * 2, Y_BYTES = BM * BN * (int)sizeof(TY);
  static constexpr int SMEM = 2 * V_BYTES + STAGES * (W_BYTES + Y_BYTES);
};

// The 16-byte piece of a tile of outputs (rows of C pieces) in which column c of a row
// lies: those that a warp's accumulators go to are in different banks.
template <typename TY, int C>
__device__ __forceinline__ uint32_t out_piece(int row, int p) {
  const int s = (sizeof(TY) == 4 ? 2 * row : row) & (C >= 8 ? 7 : C - 1);
  return (uint32_t)(row * C + (p ^ s)) * 16u;
}

// `rows` rows of `cols` columns from src to dst as the whole block (rows without an adapter).
template <typename TY, bool VEC>
__device__ __forceinline__ void copy_rows(const TY* src, int64_t src_stride, TY* dst, int64_t dst_stride, int rows,
                                          int cols) {
  constexpr int E = VEC ? 8 : 1;
  const int per = (cols + E - 1) / E;
  for (int i = threadIdx.x; i < rows * per; i += kThreads) {
    const int row = i / per, c = i % per * E;
    if constexpr (VEC) {
      const uint32_t mask = mask8<true>(c, 1, cols);
      Raw8<TY> r;
      float v[8];
      load8<true>(src + row * src_stride, c, 1, src ? mask : 0u, r);
      to_float(r, v);
      store8<true>(dst + row * dst_stride, c, 1, mask, v);
    } else {
      dst[row * dst_stride + c] = src ? __ldcg(src + row * src_stride + c) : Elem<TY>::from(0.f);
    }
  }
}

template <typename T, int BM, int RN, bool TRANS, typename TY, bool VEC>
__device__ __forceinline__ void expand_tile(const ExpandParams& P, const Tile& t, uint8_t* smem, float* row_scale,
                                            bool first) {
  using E = Expand<T, BM, RN, TRANS, TY>;
  constexpr int CV = RN / 8, CW = TRANS ? E::BN / 8 : RN / 8, EP = 16 / sizeof(TY), CY = E::BN / EP;
  const uint32_t base = smem_u32(smem), ring = base + 2 * E::V_BYTES;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, N = (int)P.N;
  const int tiles = (N + E::BN - 1) / E::BN, G = gridDim.x;
  const TY* res = (const TY*)P.res + (int64_t)t.row * P.res_stride;
  TY* y = (TY*)P.y + (int64_t)t.row * P.y_stride;
  if (t.id < 0 || t.id >= P.adapters) {
    if (first) pdl_wait();
    if (P.res == P.y) return;  // nothing to add
    for (int n0 = blockIdx.x * E::BN; n0 < N; n0 += G * E::BN)
      copy_rows<TY, VEC>(P.res ? res + n0 : nullptr, P.res_stride, y + n0, P.y_stride, t.rows, min(E::BN, N - n0));
    return;
  }
  const int rank_of = P.ranks ? __ldcg(P.ranks + t.id) : P.R;  // (used once the residuals are under way)
  float s0 = P.scales ? __ldcg(P.scales + t.id) : 1.f, s1;
  const T* w = (const T*)P.w.w + (int64_t)t.id * P.w.next;
  Mover<BM, CY, (int)sizeof(TY)> mr(P.res ? res : y, P.res_stride, E::BN,
                                    out_piece<TY, CY>(threadIdx.x / CY, threadIdx.x % CY));
  auto ask_res = [&](int tile, int stage) {
    if (!VEC || !P.res || tile >= tiles) return;
    const int left = N - tile * E::BN;
    if (left < E::BN) mr.limit(left);  // the columns' end
    mr.copy(ring + stage * (E::W_BYTES + E::Y_BYTES) + E::W_BYTES, (int64_t)tile * E::BN * (int)sizeof(TY), t.rows);
  };
  int tile = blockIdx.x;
#pragma unroll
  for (int i = 0; i < E::STAGES - 1; ++i) ask_res(tile + i * G, i);
  const int own = min(max(rank_of, 0), P.R);
  Mover<TRANS ? RN : E::BN, CW> mw(w, P.w.stride, TRANS ? E::BN : own, my_piece<CW>());
  auto ask_w = [&](int tile, int stage) {
    if (tile >= tiles) return;
    const int left = min(N - tile * E::BN, E::BN);
    if (TRANS && left < E::BN) mw.limit(left);
    mw.copy(ring + stage * (E::W_BYTES + E::Y_BYTES), (int64_t)tile * E::BN * 2 * (TRANS ? 1 : P.w.stride),
            TRANS ? own : left);
  };
#pragma unroll
  for (int i = 0; i < E::STAGES - 1; ++i) {
    ask_w(tile + i * G, i);
    cp_commit();  // (the first with all residuals that have been asked for)
  }
  if (first) pdl_wait();  // v comes from the launch before
#pragma unroll
  for (int i0 = 0; i0 < BM * CV; i0 += kThreads) {
    const int i = i0 + threadIdx.x;
    if (BM * CV % kThreads && i >= BM * CV) break;  // (whole warps)
    const int row = i / CV, c = i % CV;
    float v[8];
    load_v8(P.v + (int64_t)(t.row + row) * P.R + 8 * c, row < t.rows && 8 * c < P.R, v);
    float scale = 1.f;
    if constexpr (std::is_same<T, __half>::value) {
      uint32_t top = abs_bits(v);
#pragma unroll
      for (int o = CV / 2; o; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
      scale = scale_down(top);
      if (c == 0) row_scale[row] = scale_up(top);
    }
    uint4 h, l;
    split8<T>(v, scale, h, l);
    *reinterpret_cast<uint4*>(smem + piece<CV>(row, c)) = h;
    *reinterpret_cast<uint4*>(smem + E::V_BYTES + piece<CV>(row, c)) = l;
  }
  __syncthreads();
  const int wm = warp % E::WM, wn = warp / E::WM, r0 = wm * 16 + lane / 4;
  uint32_t h[RN / 16][4], l[RN / 16][4];
#pragma unroll
  for (int k = 0; k < RN / 16; ++k) {
    frag_a<CV, false>(base, wm * 16, k * 16, h[k]);
    frag_a<CV, false>(base + E::V_BYTES, wm * 16, k * 16, l[k]);
  }
  s1 = s0;
  if constexpr (std::is_same<T, __half>::value) s0 *= row_scale[r0], s1 *= row_scale[r0 + 8];
  for (int stage = 0; tile < tiles; tile += G) {
    cp_wait<E::STAGES - 2>();
    __syncthreads();
    const int there = stage == 0 ? E::STAGES - 1 : stage - 1;
    ask_res(tile + (E::STAGES - 1) * G, there);
    ask_w(tile + (E::STAGES - 1) * G, there);
    cp_commit();
    const uint32_t at = ring + stage * (E::W_BYTES + E::Y_BYTES);
    uint8_t* out = smem + (at - base) + E::W_BYTES;
    float acc[E::NT][4] = {};
#pragma unroll
    for (int k = 0; k < RN / 16; ++k)
#pragma unroll
      for (int j = 0; j < E::NT; j += 2) {
        uint32_t b[4];
        frag_b<CW, TRANS>(at, wn * E::NW + j * 8, k * 16, b);
        mma<T>(acc[j], l[k], b[0], b[1]);
        mma<T>(acc[j + 1], l[k], b[2], b[3]);
        mma<T>(acc[j], h[k], b[0], b[1]);
        mma<T>(acc[j + 1], h[k], b[2], b[3]);
      }
    const int n0 = tile * E::BN + wn * E::NW;  // this warp's first column
#pragma unroll
    for (int j = 0; j < E::NT; ++j)
#pragma unroll
      for (int q = 0; q < 2; ++q) {  // a row of the accumulators' two
        const int row = r0 + 8 * q, c = wn * E::NW + j * 8 + lane % 4 * 2;
        TY* o = reinterpret_cast<TY*>(out + out_piece<TY, CY>(row, c / EP)) + c % EP;
        float a = acc[j][2 * q] * (q ? s1 : s0), b = acc[j][2 * q + 1] * (q ? s1 : s0);
        if (VEC && P.res) {
          a += Elem<TY>::to(o[0]);
          b += Elem<TY>::to(o[1]);
        } else if (!VEC && P.res && row < t.rows) {
          const int n = tile * E::BN + c;
          if (n < N) a += Elem<TY>::to(__ldcg(res + row * P.res_stride + n));
          if (n + 1 < N) b += Elem<TY>::to(__ldcg(res + row * P.res_stride + n + 1));
        }
        o[0] = Elem<TY>::from(a);
        o[1] = Elem<TY>::from(b);
      }
    __syncwarp();
    if constexpr (VEC) {
      constexpr int PW = E::NW / EP;  // pieces of the warp's part of a row
#pragma unroll
      for (int i = lane; i < 16 * PW; i += 32) {
        const int row = wm * 16 + i / PW, c = i % PW;
        if (row >= t.rows) continue;
        const uint4 v = *reinterpret_cast<const uint4*>(out + out_piece<TY, CY>(row, wn * E::NW / EP + c));
        const int n = n0 + c * EP, left = N - n;
        TY* to = y + row * P.y_stride + n;
        if (left >= EP) {
          *reinterpret_cast<uint4*>(to) = v;
        } else {
          const TY* e = reinterpret_cast<const TY*>(&v);
#pragma unroll
          for (int k = 0; k < EP - 1; ++k)
            if (k < left) to[k] = e[k];
        }
      }
    } else {
#pragma unroll 4
      for (int i = lane; i < 16 * E::NW; i += 32) {
        const int row = wm * 16 + i / E::NW, c = wn * E::NW + i % E::NW;
        if (row < t.rows && tile * E::BN + c < N)
          y[row * P.y_stride + tile * E::BN + c] =
              reinterpret_cast<const TY*>(out + out_piece<TY, CY>(row, c / EP))[c % EP];
      }
    }
    if (++stage == E::STAGES) stage = 0;
  }
  cp_wait<0>();
}

template <typename T, int BM, int RN, bool TRANS, typename TY>
__global__ void __launch_bounds__(kThreads, BM == 16 && RN <= 64 ? 3 : 2) expand_kernel(const __grid_constant__ ExpandParams P) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float row_scale[BM];
  bool first = true;
  for (int tile = blockIdx.y; tile < P.tiles; tile += gridDim.y) {
    Tile t;
    if (!first) __syncthreads();  // (the tile before has been read)
    if (!find_tile(P.seg, BM, tile, t)) break;
    if (P.vec) expand_tile<T, BM, RN, TRANS, TY, true>(P, t, smem, row_scale, first);
    else expand_tile<T, BM, RN, TRANS, TY, false>(P, t, smem, row_scale, first);
    first = false;
  }
  if (first) pdl_wait();
  pdl_trigger();
}

// ---------------------------------------------------------------------------
// out[j][c] = s sum_t v[t][j] x[t][c] over the rows t of an adapter (dA), or
// out[c][j] (dB)
// ---------------------------------------------------------------------------
struct GradSide {
  const float* v;       // [rows][R]
  const void* x;
  int64_t x_stride, C;  // columns
  void* out;            // of adapter i from element i * R * C on
  const float* scales;
  int32_t type, by_column;  // by_column: out[c][j]
  int32_t tiles;            // of columns, 0: not wanted
};
struct GradParams {
  GradSide side[2];
  const int32_t* ranks;
  Segments seg;
  int32_t R, cluster;
};

template <typename T, int RN>
struct Grad {
  static constexpr int BT = 64;                    // rows of a stage
  static constexpr int BC = RN <= 64 ? 128 : 64;   // columns of a block
  static constexpr int WR = RN <= 32 ? 1 : RN / 32, WC = 8 / WR;
  static constexpr int MT = RN / 16 / WR, NT = BC / 8 / WC;
  // x of three stages (multiplied, here, on its way), v of two as it lies and of two split
  static constexpr int X_BYTES = BT * BC * 2, F_BYTES = BT * RN * 4, V_BYTES = BT * RN * 2;
  static constexpr int PITCH = BC + 1;
  static constexpr int RED_BYTES = RN * PITCH * 4;
  static constexpr int MAIN = 3 * X_BYTES + 2 * F_BYTES + 4 * V_BYTES;
  static constexpr int SMEM = MAIN > RED_BYTES ? MAIN : RED_BYTES;
};

// A block holds an adapter's sums for BC columns and all ranks over the rows that it takes (a
// cluster's blocks share an adapter's rows and add their sums in order: no atomics).  4096 rows of rank
// 64, 5120 + 13824 columns: 86 us for 20 GFLOP (v as two numbers), 33 us of mma.sync's rate, and
// 155 MB, 23 us of HBM; with 16 warps on an SM the rest is latency of shared memory and MMAs.
//
// The sums of 128 rows (fp16: of a stage's 64, which have a scale of their own) start anew and are
// added to the block's in fp32: the tensor cores cut their running sums off, and over thousands of
// rows that adds up (4096 rows of two adapters: 5e-6 off without it, 2.4e-6 with it).
template <typename T, int RN, bool ANY>
__global__ void __launch_bounds__(kThreads, RN <= 64 ? 2 : 1) gradients_kernel(const __grid_constant__ GradParams P) {
  using G = Grad<T, RN>;
  constexpr int CX = G::BC / 8, CV = RN / 8, CF = RN / 4, BT = G::BT;
  constexpr bool SCALED = std::is_same<T, __half>::value;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint32_t tops[8];
  constexpr int F_AT = 3 * G::X_BYTES, V_AT = F_AT + 2 * G::F_BYTES;
  const uint32_t base = smem_u32(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = P.cluster > 1 ? (int)cluster_rank() : 0;
  const int per = P.side[0].tiles + P.side[1].tiles, block = blockIdx.x / P.cluster;
  const int id = block / per, which = block % per >= P.side[0].tiles;
  const GradSide& D = P.side[which];
  const int64_t n0 = (int64_t)(block % per - (which ? P.side[0].tiles : 0)) * G::BC;
  pdl_wait();
  pdl_trigger();
  const int rank_of = P.ranks ? __ldcg(P.ranks + id) : P.R;
  const float s = D.scales ? __ldcg(D.scales + id) : 1.f;
  AdapterTiles ahead;
  ahead.begin(rank);
  const Mover<BT, CX> mx((const T*)D.x + n0, D.x_stride, (int)min(D.C - n0, (int64_t)G::BC), my_piece<CX>());
  const Mover<BT, CF, 4> mv(D.v, P.R, P.R, threadIdx.x * 16u);  // (rows as they lie)
  int asked = 0;  // stages that have been asked for
  bool any = true;
  auto copy = [&](int stage) {
    int row, rows;
    any = any && ahead.next(P.seg, id, BT, P.cluster, row, rows);
    if (any) {
      if constexpr (ANY)
        copy_any<BT, CX>(smem + stage % 3 * G::X_BYTES, (const T*)D.x + (int64_t)row * D.x_stride + n0, D.x_stride, rows,
                         (int)min(D.C - n0, (int64_t)G::BC));
      else
        mx.copy(base + stage % 3 * G::X_BYTES, (int64_t)row * D.x_stride * 2, rows);
      mv.copy(base + F_AT + stage % 2 * G::F_BYTES, (int64_t)row * P.R * 4, rows);
      ++asked;
    }
    cp_commit();
  };
  float down = 1.f, up = 1.f;
  // v of a stage as two numbers; `up` is what undoes its scale.
  auto split = [&](int stage) {
    const float4* f = reinterpret_cast<const float4*>(smem + F_AT + stage % 2 * G::F_BYTES);
    uint8_t* to = smem + V_AT + stage % 2 * 2 * G::V_BYTES;
    auto v8 = [&](int g, float(&v)[8]) {
      const float4 a = f[2 * g], b = f[2 * g + 1];
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    };
    if constexpr (SCALED) {
      uint32_t top = 0;
#pragma unroll
      for (int g = threadIdx.x; g < BT * CV; g += kThreads) {
        float v[8];
        v8(g, v);
        top = max(top, abs_bits(v));
      }
      top = __reduce_max_sync(0xFFFFFFFFu, top);
      if (lane == 0) tops[warp] = top;
      __syncthreads();
      top = __reduce_max_sync(0xFFFFFFFFu, tops[lane & 7]);
      down = scale_down(top);
      up = scale_up(top);
    }
#pragma unroll
    for (int g = threadIdx.x; g < BT * CV; g += kThreads) {
      float v[8];
      uint4 h, l;
      v8(g, v);
      split8<T>(v, down, h, l);
      *reinterpret_cast<uint4*>(to + piece<CV>(g / CV, g % CV)) = h;
      *reinterpret_cast<uint4*>(to + G::V_BYTES + piece<CV>(g / CV, g % CV)) = l;
    }
  };
  float acc[G::MT][G::NT][4] = {}, part[G::MT][G::NT][4] = {};
  const int wr = warp % G::WR, wc = warp / G::WR;
  copy(0);
  copy(1);
  if (asked) {
    cp_wait<1>();
    __syncthreads();
    split(0);
  }
  for (int done = 0; done < asked; ++done) {
    cp_wait<0>();
    __syncthreads();  // the next stage is here, this one is split, the one before has been read
    copy(done + 2);
    const uint32_t at = base + done % 3 * G::X_BYTES, vt = base + V_AT + done % 2 * 2 * G::V_BYTES;
#pragma unroll
    for (int k = 0; k < BT; k += 16) {
      uint32_t h[G::MT][4], l[G::MT][4];
#pragma unroll
      for (int i = 0; i < G::MT; ++i) {
        frag_a<CV, true>(vt, (wr * G::MT + i) * 16, k, h[i]);
        frag_a<CV, true>(vt + G::V_BYTES, (wr * G::MT + i) * 16, k, l[i]);
      }
#pragma unroll
      for (int j = 0; j < G::NT; j += 2) {
        uint32_t b[4];
        frag_b<CX, true>(at, (wc * G::NT + j) * 8, k, b);
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
          for (int i = 0; i < G::MT; ++i) mma<T>(part[i][j + q], l[i], b[2 * q], b[2 * q + 1]);
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
          for (int i = 0; i < G::MT; ++i) mma<T>(part[i][j + q], h[i], b[2 * q], b[2 * q + 1]);
      }
    }
    const float mine = up;
    if (done + 1 < asked) split(done + 1);
    if (SCALED || (done & 1) || done + 1 == asked) {
#pragma unroll
      for (int i = 0; i < G::MT; ++i)
#pragma unroll
        for (int j = 0; j < G::NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            acc[i][j][e] = fmaf(part[i][j][e], mine, acc[i][j][e]);
            part[i][j][e] = 0.f;
          }
    }
  }
  const int own = min(max(rank_of, 0), P.R);
  cp_wait<0>();
  __syncthreads();
  float* red = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int i = 0; i < G::MT; ++i)
#pragma unroll
    for (int j = 0; j < G::NT; ++j) {
      const int row = (wr * G::MT + i) * 16 + lane / 4, col = (wc * G::NT + j) * 8 + lane % 4 * 2;
      red[row * G::PITCH + col] = acc[i][j][0];
      red[row * G::PITCH + col + 1] = acc[i][j][1];
      red[(row + 8) * G::PITCH + col] = acc[i][j][2];
      red[(row + 8) * G::PITCH + col + 1] = acc[i][j][3];
    }
  if (P.cluster > 1) cluster_sync();
  else __syncthreads();
  const int share = RN * G::BC / P.cluster;
  for (int i = rank * share + threadIdx.x; i < (rank + 1) * share; i += kThreads) {
    const int j = D.by_column ? i % RN : i / G::BC, c = D.by_column ? i / RN : i % G::BC;
    if (j >= P.R || n0 + c >= D.C) continue;
    const int at = j * G::PITCH + c;
    const float sum = P.cluster > 1 ? sum_cluster(base + at * 4, P.cluster) : red[at];
    const int64_t o = (int64_t)id * P.R * D.C + (D.by_column ? (n0 + c) * P.R + j : j * D.C + n0 + c);
    any_store(D.out, D.type, o, j < own ? sum * s : 0.f);
  }
  if (P.cluster > 1) cluster_sync();
}

// ---------------------------------------------------------------------------
// host: kernels by their tile
// ---------------------------------------------------------------------------
struct Kernel {
  void* f;
  int smem;
};
// rn: the rank rounded up to 16, 32, 64 or 128; bm: 16, 64 or (shrink, rn >= 64) 128; any: rows of
// x start anywhere (shrink: bm 16).
template <typename T>
Kernel shrink_of(int bm, int rn, bool trans, bool any);
template <typename T>
Kernel expand_of(int bm, int rn, bool trans, bool f32);
template <typename T>
Kernel gradients_of(int rn, bool any);

template <typename T, int RN, bool TRANS>
Kernel shrink_for(int bm, bool any) {
  if constexpr (RN >= 64) {
    if (bm == 128) return Kernel{(void*)shrink_tiled_kernel<T, 128, RN, TRANS>, Tiled<T, 128, RN, TRANS>::SMEM};
  }
  if (bm == 64) return Kernel{(void*)shrink_tiled_kernel<T, 64, RN, TRANS>, Tiled<T, 64, RN, TRANS>::SMEM};
  return Kernel{any ? (void*)shrink_kernel<T, 16, RN, TRANS, true> : (void*)shrink_kernel<T, 16, RN, TRANS, false>,
                Shrink<T, 16, RN, TRANS>::SMEM};
}
template <typename T, int RN>
Kernel shrink_for(int bm, bool trans, bool any) {
  return trans ? shrink_for<T, RN, true>(bm, any) : shrink_for<T, RN, false>(bm, any);
}
template <typename T, int BM, int RN, bool TRANS>
Kernel expand_at(bool f32) {
  return f32 ? Kernel{(void*)expand_kernel<T, BM, RN, TRANS, float>, Expand<T, BM, RN, TRANS, float>::SMEM}
             : Kernel{(void*)expand_kernel<T, BM, RN, TRANS, T>, Expand<T, BM, RN, TRANS, T>::SMEM};
}
template <typename T, int RN>
Kernel expand_for(int bm, bool trans, bool f32) {
  if (bm == 16) return trans ? expand_at<T, 16, RN, true>(f32) : expand_at<T, 16, RN, false>(f32);
  return trans ? expand_at<T, 64, RN, true>(f32) : expand_at<T, 64, RN, false>(f32);
}
template <typename T>
Kernel shrink_of(int bm, int rn, bool trans, bool any) {
  return rn == 16   ? shrink_for<T, 16>(bm, trans, any)
         : rn == 32 ? shrink_for<T, 32>(bm, trans, any)
         : rn == 64 ? shrink_for<T, 64>(bm, trans, any)
                    : shrink_for<T, 128>(bm, trans, any);
}
template <typename T>
Kernel expand_of(int bm, int rn, bool trans, bool f32) {
  return rn == 16   ? expand_for<T, 16>(bm, trans, f32)
         : rn == 32 ? expand_for<T, 32>(bm, trans, f32)
         : rn == 64 ? expand_for<T, 64>(bm, trans, f32)
                    : expand_for<T, 128>(bm, trans, f32);
}
template <typename T, int RN>
Kernel gradients_at(bool any) {
  return Kernel{any ? (void*)gradients_kernel<T, RN, true> : (void*)gradients_kernel<T, RN, false>, Grad<T, RN>::SMEM};
}
template <typename T>
Kernel gradients_of(int rn, bool any) {
  return rn == 16   ? gradients_at<T, 16>(any)
         : rn == 32 ? gradients_at<T, 32>(any)
         : rn == 64 ? gradients_at<T, 64>(any)
                    : gradients_at<T, 128>(any);
}

}  // namespace lora
}  // namespace polyq
