// Thin wrappers over the 5th-generation tensor-core PTX (tcgen05, sm_100a): tensor-memory
// allocation, the single-thread MMA with shared-memory operand descriptors, commit to an mbarrier,
// and the 32-lane x 32-bit tensor-memory loads / stores of the epilogue warps.
//
// Formats used here (bf16 operands, fp32 accumulators, one CTA per MMA):
//  * instruction descriptor (32 bit): accumulator format at bit 4 (1 = f32), A / B element format at
//    bits 7 / 10 (1 = bf16), A / B major-ness at bits 15 / 16 (0 = K-major, 1 = MN-major), N / 8 at
//    bit 17, M / 16 at bit 24;
//  * shared-memory matrix descriptor (64 bit): start address / 16 in bits 0-13, leading byte offset
//    / 16 in bits 16-29, stride byte offset / 16 in bits 32-45, descriptor version 1 at bit 46,
//    swizzle mode at bits 61-63 (2 = 128-byte swizzle).  With the 128-byte swizzle an operand tile
//    is a stack of 1024-byte atoms of 8 rows x 128 bytes; a K-major operand steps 32 bytes along
//    its rows per 16-element MMA step, an MN-major one steps two atoms.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "ngc_common.cuh"
#include "ptx.cuh"

namespace ngc {
namespace umma {

constexpr uint32_t kF32Acc = 1u << 4, kBf16A = 1u << 7, kBf16B = 1u << 10, kAMajorMN = 1u << 15, kBMajorMN = 1u << 16;
__host__ __device__ constexpr uint32_t instr_desc(uint32_t M, uint32_t N, bool b_mn_major, bool a_mn_major = false) {
  return kF32Acc | kBf16A | kBf16B | (a_mn_major ? kAMajorMN : 0u) | (b_mn_major ? kBMajorMN : 0u) | ((N >> 3) << 17) | ((M >> 4) << 24);
}

// 128-byte-swizzled operand at shared address `saddr` (the tile it belongs to is 1024-byte aligned).
__device__ __forceinline__ uint64_t smem_desc_sw128(uint32_t saddr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
  const uint32_t lo = ((saddr >> 4) & 0x3FFFu) | (((lbo_bytes >> 4) & 0x3FFFu) << 16);
  const uint32_t hi = ((sbo_bytes >> 4) & 0x3FFFu) | (1u << 14) | (2u << 29);
  return ((uint64_t)hi << 32) | lo;
}

// True in exactly one lane of a converged warp.  The compiler knows that the branch it guards runs in one thread: the
// operands of the instructions inside stay in uniform registers (a plain `lane == 0` costs a move out of the vector
// registers for every descriptor).
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}

// Tensor memory: `cols` columns (a power of two, 32..512) of 128 lanes x 32 bit.  Warp-collective; the
// base address lands in *slot (shared memory).  The same warp frees it.
__device__ __forceinline__ void tmem_alloc(uint32_t* slot, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(ptx::smem_u32(slot)), "r"(cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc(uint32_t taddr, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols) : "memory");
}
__device__ __forceinline__ void fence_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// D[tmem] (+)= A[smem] * B[smem]; issued by ONE thread.  accumulate == 0 overwrites D.
__device__ __forceinline__ void mma_bf16(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// The same with the A operand in tensor memory: lane = row, one 32-bit column = two consecutive K elements (bf16).
__device__ __forceinline__ void mma_bf16_a_tmem(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// The mbarrier gets one arrival when every MMA this thread issued so far has completed.
__device__ __forceinline__ void commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(ptx::smem_u32(bar)) : "memory");
}

// 32 consecutive columns of this thread's lane (lane = 32 * (warp % 4) + lane id, encoded in taddr bits 16+).
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
// 16 consecutive columns of this thread's lane.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
        "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Arithmetic of the softmax warps.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// two floats in one 64-bit register for the packed fp32 instructions (fma / add on both halves at once)
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// Bounded wait that also gives up as soon as another thread of the CTA has given up (*abort, in shared memory).  The
// clock is first read after 64 tries: reading it takes longer than most waits last.
__device__ __forceinline__ bool wait_or_abort(uint64_t* bar, uint32_t parity, int* abort, int32_t* dev_status) {
  uint64_t t0 = 0;
  for (uint32_t spins = 0;; ++spins) {
    if (ptx::mbar_try_wait(bar, parity)) return true;
    if ((spins & 63u) == 63u) {
      if (*(volatile int*)abort) return false;
      const uint64_t t = ptx::globaltimer_ns();
      if (t0 == 0) t0 = t;
      if (t - t0 > ptx::kWaitLimitNs) {
        *(volatile int*)abort = 1;
        set_dev_status(dev_status, NGC_DEV_TIMEOUT);
        return false;
      }
    }
  }
}
// The same for a thread whose every instruction counts (one that issues MMAs beside busy warps): the first look is all that is
// inlined.
static __device__ __noinline__ bool wait_long(uint64_t* bar, uint32_t parity, int* abort, int32_t* dev_status) {
  return wait_or_abort(bar, parity, abort, dev_status);
}
__device__ __forceinline__ bool wait_quick(uint64_t* bar, uint32_t parity, int* abort, int32_t* dev_status) {
  return ptx::mbar_try_wait(bar, parity) || wait_long(bar, parity, abort, dev_status);
}
// The limit of a thread's turns round a loop in which it looks at barriers without waiting at any.
struct Patience {
  uint32_t turns = 0;
  uint64_t since = 0;
  __device__ __forceinline__ void moved() { since = 0; }
  // One more turn without anything to do; false when it is time to leave.
  __device__ __forceinline__ bool more(int* abort, int32_t* dev_status) {
    if ((++turns & 255u) != 0) return true;
    if (*(volatile int*)abort) return false;
    const uint64_t now = ptx::globaltimer_ns();
    if (since == 0) since = now;
    if (now - since <= ptx::kWaitLimitNs) return true;
    *(volatile int*)abort = 1;
    set_dev_status(dev_status, NGC_DEV_TIMEOUT);
    return false;
  }
};
// Bounded wait of a whole warp: every lane gets the same answer.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, int* abort, int32_t* dev_status) {
  return __all_sync(0xffffffffu, wait_or_abort(bar, parity, abort, dev_status));
}

}  // namespace umma
}  // namespace ngc
