// sm_103a primitives for the tcgen05 kernels: mbarriers with bounded waits,
// bulk global->shared copies, tensor-memory allocation, tcgen05.mma with the
// A operand in tensor memory, and tensor-memory loads/stores.
//
// Shared-memory matrix descriptor (no swizzle, K-major): bits [0,14) start
// address >> 4, [16,30) leading-dimension byte offset >> 4 (distance between
// the 8x16-byte core matrices adjacent along K), [32,46) stride byte offset
// >> 4 (distance between core matrices adjacent along M/N), bits [46,48) =
// 1 (descriptor version), layout type 0 (no swizzle) in bits [61,64).
// Instruction descriptor (kind::f16): bits [4,6) = 1 (f32 accumulator),
// [7,10) / [10,13) = A and B type (0 f16, 1 bf16), bits 15 / 16 = 0 (A and B K-major),
// [17,23) = N >> 3, [24,29) = M >> 4.
#pragma once

#include <stdint.h>

namespace optr {
namespace tc05 {

__device__ __forceinline__ uint32_t smem_addr(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

__device__ __forceinline__ uint64_t smem_desc(uint32_t saddr, uint32_t lbo,
                                              uint32_t sbo) {
  return (uint64_t)((saddr >> 4) & 0x3FFFu) |
         ((uint64_t)((lbo >> 4) & 0x3FFFu) << 16) |
         ((uint64_t)((sbo >> 4) & 0x3FFFu) << 32) | ((uint64_t)1 << 46);
}

// The same with the 128-byte swizzle (layout type 2: 16-byte piece c of a
// 128-byte row r at piece c ^ (r % 8), rows 128 B apart, 1024-byte aligned;
// what TMA writes).  K-major: rows along M/N, 8 of them SBO = 1024 B; a K step
// of 16 starts 32 B further.  MN-major (bit 15 or 16 of the instruction
// descriptor): rows along K, 8 of them SBO = 1024 B; LBO from 64 elements of
// M/N to the next 64; a K step of 16 starts 2048 B further.
__device__ __forceinline__ uint64_t smem_desc_sw128(uint32_t saddr, uint32_t lbo) {
  return smem_desc(saddr, lbo, 1024) | ((uint64_t)2 << 61);
}

constexpr uint32_t kIdescBf16 = (1u << 7) | (1u << 10);  // A and B bf16
constexpr uint32_t kIdescMajorMnB = 1u << 16;

__host__ __device__ constexpr uint32_t idesc_f16(int M, int N) {
  return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

__device__ __forceinline__ void bar_init(uint64_t* bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)),
               "r"(count));
}

__device__ __forceinline__ void bar_init_fence() {
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}

__device__ __forceinline__ void bar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar))
               : "memory");
}

// Arrives once this thread's cp.async copies so far have landed.
__device__ __forceinline__ void bar_arrive_copies(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}

__device__ __forceinline__ void bar_arrive_expect_tx(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.release.cta.shared::cta.b64 _, [%0], %1;"
               ::"r"(smem_addr(bar)), "r"(bytes) : "memory");
}

__device__ __forceinline__ bool bar_try_wait(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n"
      " mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\n"
      " selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok) : "r"(smem_addr(bar)), "r"(parity) : "memory");
  return ok != 0;
}

// Wait for the phase of the given parity to complete.  Gives up after
// limit_ns nanoseconds (about two seconds unless given), or as soon as
// *abort is set; returns false then (and sets *abort itself on its own
// timeout), so that no wait can hang the GPU.
__device__ __forceinline__ bool bar_wait(uint64_t* bar, uint32_t parity,
                                         volatile int* abort,
                                         uint64_t limit_ns = 2000000000ull) {
  if (bar_try_wait(bar, parity)) return true;
  uint64_t t0;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
  uint32_t ns = 32;  // back off: a sleeping warp leaves its issue slots to others
  for (uint32_t it = 1;; ++it) {
    __nanosleep(ns);
    if (bar_try_wait(bar, parity)) return true;
    ns = ns < 256 ? 2 * ns : 256;
    if ((it & 15u) == 0) {
      if (*abort) return false;
      uint64_t t;
      asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
      if (t - t0 > limit_ns) {
        *abort = 1;
        return false;
      }
    }
  }
}

// Wait for the phase of the given parity for at most about two seconds,
// whatever *abort says (for draining copies and MMAs before the CTA exits).
__device__ __forceinline__ bool bar_wait_drain(uint64_t* bar, uint32_t parity) {
  uint64_t t0;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
  for (uint32_t it = 0;; ++it) {
    if (bar_try_wait(bar, parity)) return true;
    if ((it & 63u) == 63u) {
      uint64_t t;
      asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
      if (t - t0 > 2000000000ull) return false;
    }
  }
}

// bar_wait without sleeping between the polls (each of which the hardware
// suspends for a while itself): for waits of a few hundred cycles on the
// critical path.
__device__ __forceinline__ bool bar_wait_spin(uint64_t* bar, uint32_t parity, volatile int* abort) {
  if (bar_try_wait(bar, parity)) return true;
  uint64_t t0;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
  for (uint32_t it = 1;; ++it) {
    if (bar_try_wait(bar, parity)) return true;
    if ((it & 63u) == 0) {
      if (*abort) return false;
      uint64_t t;
      asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
      if (t - t0 > 2000000000ull) {
        *abort = 1;
        return false;
      }
    }
  }
}

// Bulk copy of `bytes` (multiple of 16; both addresses 16-byte aligned)
// from global to shared memory, completing on bar's transaction count.
__device__ __forceinline__ void bulk_g2s(void* dst, const void* src,
                                         uint32_t bytes, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes "
      "[%0], [%1], %2, [%3];"
      ::"r"(smem_addr(dst)), "l"(src), "r"(bytes), "r"(smem_addr(bar))
      : "memory");
}

// TMA tiled load of one box at coordinates (c0, c1, c2) of the tensor map
// (a __grid_constant__ kernel parameter) into shared memory, completing on
// bar's transaction count.  c0 * element size must be a multiple of 16.
__device__ __forceinline__ void tma_load_3d(void* dst, const void* tmap, int c0,
                                            int c1, int c2, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(smem_addr(dst)), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(c0), "r"(c1),
        "r"(c2), "r"(smem_addr(bar))
      : "memory");
}

// Whole warpgroup: take registers from (inc) or give them to (dec) the CTA's
// launch total.  What the warpgroups hold afterwards must add up to no more
// than the launch gave them, or inc waits for ever.
template <int kRegs>
__device__ __forceinline__ void reg_inc() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs));
}
template <int kRegs>
__device__ __forceinline__ void reg_dec() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs));
}

__device__ __forceinline__ void fence_proxy_async() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

__device__ __forceinline__ void fence_before() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}

__device__ __forceinline__ void fence_after() {
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}

// Whole warp: allocate `cols` tensor-memory columns (a power of two >= 32),
// base address to *dst (shared memory).
__device__ __forceinline__ void tmem_alloc(uint32_t* dst, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
               ::"r"(smem_addr(dst)), "r"(cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_dealloc(uint32_t base, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base),
               "r"(cols) : "memory");
}

// D[tmem d] (+)= A[tmem a] * B[smem desc b]^T, M x N x 16, f16 -> f32.
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b,
                                       uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

// Arrive on bar once every tcgen05.mma issued so far by this thread is done.
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];"
      ::"r"(smem_addr(bar)) : "memory");
}

// D (+)= A B^T over 128 of the inner dimension: eight MMAs, issued by one elected
// thread of a whole converged warp.  One block of code for all eight, so that only
// the bases have to be brought into uniform registers and the steps are added
// there: one by one, from operands that the compiler cannot prove uniform, each
// MMA took about 120 cycles to issue, against the 64 that a 128 x 128 x 16 takes.
// kA, kB: how far apart the steps lie, in units of 16 bytes (descriptors) or
// columns (A in tensor memory); kWrap: 64 of the inner dimension fill 128-byte rows,
// and the other 64 lie 16 KB on (K-major, 128-byte swizzle, 128 rows).
template <int kA, int kB, bool kWrapA, bool kWrapB>
__device__ __forceinline__ void mma128_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                          uint32_t accumulate) {
  constexpr int kHalfOff = 1024 - 4 * 2;  // 16 KB instead of four steps of 32 B
  constexpr int wa = kWrapA ? kHalfOff : 0, wb = kWrapB ? kHalfOff : 0;
  asm volatile(
      "{\n .reg .pred p, t, e;\n .reg .b64 x<8>, y<8>;\n"
      " setp.ne.b32 p, %4, 0;\n setp.eq.u32 t, 0, 0;\n elect.sync _|e, 0xffffffff;\n"
      " add.s64 x1, %1, %5;\n add.s64 y1, %2, %12;\n"
      " add.s64 x2, %1, %6;\n add.s64 y2, %2, %13;\n"
      " add.s64 x3, %1, %7;\n add.s64 y3, %2, %14;\n"
      " add.s64 x4, %1, %8;\n add.s64 y4, %2, %15;\n"
      " add.s64 x5, %1, %9;\n add.s64 y5, %2, %16;\n"
      " add.s64 x6, %1, %10;\n add.s64 y6, %2, %17;\n"
      " add.s64 x7, %1, %11;\n add.s64 y7, %2, %18;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], x1, y1, %3, t;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], x2, y2, %3, t;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], x3, y3, %3, t;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], x4, y4, %3, t;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], x5, y5, %3, t;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], x6, y6, %3, t;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], x7, y7, %3, t;\n}\n"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "n"(kA), "n"(2 * kA), "n"(3 * kA),
        "n"(4 * kA + wa), "n"(5 * kA + wa), "n"(6 * kA + wa), "n"(7 * kA + wa), "n"(kB), "n"(2 * kB),
        "n"(3 * kB), "n"(4 * kB + wb), "n"(5 * kB + wb), "n"(6 * kB + wb), "n"(7 * kB + wb)
      : "memory");
}

template <int kB>
__device__ __forceinline__ void mma128_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc,
                                          uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p, t, e;\n .reg .b32 x<8>;\n .reg .b64 y<8>;\n"
      " setp.ne.b32 p, %4, 0;\n setp.eq.u32 t, 0, 0;\n elect.sync _|e, 0xffffffff;\n"
      " add.u32 x1, %1, 8;\n add.s64 y1, %2, %5;\n"
      " add.u32 x2, %1, 16;\n add.s64 y2, %2, %6;\n"
      " add.u32 x3, %1, 24;\n add.s64 y3, %2, %7;\n"
      " add.u32 x4, %1, 32;\n add.s64 y4, %2, %8;\n"
      " add.u32 x5, %1, 40;\n add.s64 y5, %2, %9;\n"
      " add.u32 x6, %1, 48;\n add.s64 y6, %2, %10;\n"
      " add.u32 x7, %1, 56;\n add.s64 y7, %2, %11;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [x1], y1, %3, t;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [x2], y2, %3, t;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [x3], y3, %3, t;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [x4], y4, %3, t;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [x5], y5, %3, t;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [x6], y6, %3, t;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [x7], y7, %3, t;\n}\n"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "n"(kB), "n"(2 * kB), "n"(3 * kB),
        "n"(4 * kB), "n"(5 * kB), "n"(6 * kB), "n"(7 * kB)
      : "memory");
}

// One step of that.
__device__ __forceinline__ void mma16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc,
                                         uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p, e;\n setp.ne.b32 p, %4, 0;\n elect.sync _|e, 0xffffffff;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

__device__ __forceinline__ void mma_commit_warp(uint64_t* bar) {
  asm volatile(
      "{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n"
      " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n"
      ::"r"(smem_addr(bar)) : "memory");
}

// 32 consecutive columns of the warp's 32 lanes: register j <-> column c + j
// of lane (32 * (warp % 4) + lane), taddr = base + (lane quarter << 21) + c.
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,"
      "%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,"
      "%27,%28,%29,%30,%31,%32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]),
        "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]),
        "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
        "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
        "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,"
      "%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,"
      "%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]),
        "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]),
        "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
        "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,"
      "%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
        "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,"
      "%9,%10,%11,%12,%13,%14,%15,%16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]),
        "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]),
                 "r"(r[6]), "r"(r[7])
               : "memory");
}

__device__ __forceinline__ void tmem_wait_st() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_wait_ld() {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

}  // namespace tc05
}  // namespace optr
