// Device helpers of the kernels that multiply on CTA pairs or with block
// scales (tcgen05 of sm_103a): cluster addressing, tensor memory, bounded
// waits, operand descriptors and the MMA forms.  CG is the CTA group: 1 (one
// CTA's tensor core) or 2 (the pair of a cluster of two).
#pragma once
#include "polyq_dev.cuh"

namespace polyq {
namespace tc {

__device__ __forceinline__ uint32_t cluster_ctarank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t mapa(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ float4 ld_cluster_f32x4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(addr)
               : "memory");
  return v;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// ---- tensor memory ----
template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t dst_smem, uint32_t ncols) {
  if (CG == 2)
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem),
                 "r"(ncols)
                 : "memory");
  else
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem),
                 "r"(ncols)
                 : "memory");
}
template <int CG>
__device__ __forceinline__ void tmem_relinquish() {
  if (CG == 2) asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  else asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
template <int CG>
__device__ __forceinline__ void tmem_dealloc(uint32_t taddr, uint32_t ncols) {
  if (CG == 2)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols)
                 : "memory");
  else
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols)
                 : "memory");
}

// 16 consecutive fp32 columns of this thread's lane.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,"
      "%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}

// 32 consecutive columns of this thread's lane set, and waited for.
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,"
      "%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};\n"
      " tcgen05.wait::st.sync.aligned;" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]),
      "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
      "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}

// ---- copies ----
// 2-D tiled TMA load into this CTA's shared memory that completes on `bar`, an
// address of either CTA of the pair (mapa).
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, int32_t x,
                                                 int32_t y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
      : "memory");
}

// ---- bounded waits ----
// They give up after a few seconds, or once `abort` was raised by another role;
// the flag is read only after a poll has failed.  A poll suspends the thread
// for up to a microsecond, so that lone roles take no issue slots from the rest.
constexpr uint32_t kSleepLimit = 1u << 22;
constexpr uint32_t kSleepNs = 1000;
constexpr long long kStayCycles = 1 << 21;  // a millisecond
constexpr int kOk = 0, kTimeout = 1, kAborted = 2;
__device__ __forceinline__ bool mbar_try_wait_hint(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n"
      " selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity), "r"(kSleepNs)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ int wait(uint32_t bar, uint32_t parity, const volatile int* abort) {
  for (uint32_t it = 0; it < kSleepLimit; ++it) {
    if (mbar_try_wait_hint(bar, parity)) return kOk;
    if (*abort) return kAborted;
  }
  return kTimeout;
}
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n"
      " selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// How many phases in a row, of the B slots from `s` on in a ring of N (parity
// `ph` up to the ring's end, the other after it), have completed.  A poll's
// answer takes 250 to 300 cycles beside the tensor core's shared-memory
// traffic, but polls follow each other every few: a lone thread that asks for
// several slots at once pays that once for all that are ready.
template <int B, int N>
__device__ __forceinline__ int poll_ahead(uint32_t bar0, int s, uint32_t ph) {
  static_assert(B <= N, "one phase per slot");
  uint32_t ok = 0;
#pragma unroll
  for (int i = 0; i < B; ++i) {
    int k = s + i;
    uint32_t p = ph;
    if (k >= N) {
      k -= N;
      p ^= 1u;
    }
    ok |= (mbar_test(bar0 + 8 * k, p) ? 1u : 0u) << i;
  }
  return __ffs(~ok) - 1;
}
__device__ __forceinline__ void wait_stay(uint32_t bar, uint32_t parity) {
  for (uint32_t it = 0; it < kSleepLimit && !mbar_try_wait_hint(bar, parity); ++it) {
  }
}

// ---- descriptors ----
// Shared-memory descriptor of an operand tile of 128-byte rows in the 128-byte
// swizzle.  K-major: rows are the operand's rows, 128 bytes of K each; 8-row
// atoms lie 1024 bytes apart and the leading offset is unused.  MN-major: rows
// are K indices of 64 two-byte elements; groups of 8 K rows lie 1024 bytes
// apart, the next 64 elements of M or N `lead` bytes on.
__device__ __forceinline__ uint64_t desc_sw128(uint32_t smem_addr, uint32_t lead) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr >> 4) & 0x3FFFu);
  d |= (uint64_t)((lead >> 4) & 0x3FFFu) << 16;
  d |= (uint64_t)(1024u >> 4) << 32;
  d |= (uint64_t)1u << 46;  // descriptor version (sm_100)
  d |= (uint64_t)2u << 61;  // 128-byte swizzle
  return d;
}
// A scale atom: 32 lanes of 16 bytes, contiguous, no swizzle (8 lanes 128 bytes).
__device__ __forceinline__ uint64_t desc_scales(uint32_t smem_addr) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr >> 4) & 0x3FFFu);
  d |= (uint64_t)(128u >> 4) << 32;
  d |= (uint64_t)1u << 46;
  return d;
}
// Instruction descriptors, fp32 accumulators.  kind::f16: operand types f16 or
// bf16, each operand K-major or MN-major.
__host__ __device__ constexpr uint32_t idesc_16(int M, int N, bool bf16, bool a_mn, bool b_mn) {
  return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((a_mn ? 1u : 0u) << 15) |
         ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// e2m1 operands with block scales: e8m0 (32 elements) or e4m3 (16).  sf: which
// of a scale word's bytes the instruction's K = 64 starts at (0 or 2).
__host__ __device__ constexpr uint32_t idesc_fp4(int M, int N, bool e8m0, int sf) {
  return ((uint32_t)sf << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) |
         ((e8m0 ? 1u : 0u) << 23) | ((uint32_t)(M >> 4) << 24) | ((uint32_t)sf << 29);
}

// ---- tensor core ----
template <int CG>
__device__ __forceinline__ void mma_16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                       uint32_t accumulate) {
  if (CG == 2)
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
#define POLYQ_MMA_FP4(CGS, KIND)                                                            \
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n tcgen05.mma.cta_group::" CGS     \
               ".kind::" KIND " [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),             \
               "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)              \
               : "memory")
// K = 64.  NV: e4m3 scales of 16 elements, else e8m0 scales of 32.
template <int CG, bool NV>
__device__ __forceinline__ void mma_fp4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                        uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  if (CG == 2) {
    if (NV) POLYQ_MMA_FP4("2", "mxf4nvf4.block_scale.scale_vec::4X");
    else POLYQ_MMA_FP4("2", "mxf4.block_scale.scale_vec::2X");
  } else {
    if (NV) POLYQ_MMA_FP4("1", "mxf4nvf4.block_scale.scale_vec::4X");
    else POLYQ_MMA_FP4("1", "mxf4.block_scale.scale_vec::2X");
  }
}
#undef POLYQ_MMA_FP4
// A scale atom (512 bytes of shared memory) into four columns of tensor
// memory, the 32 lanes repeated for each quarter; CG = 2: in both CTAs, each
// from its own shared memory.
template <int CG>
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
  if (CG == 2)
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
  else
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// Arrive (once) on the barrier (CG = 2: at this offset in both CTAs) when all
// tcgen05 operations issued so far by this thread have completed.
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar) {
  if (CG == 2)
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64"
        " [%0], %1;" ::"r"(bar),
        "h"((uint16_t)3)
        : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar)
                 : "memory");
}

}  // namespace tc
}  // namespace polyq
