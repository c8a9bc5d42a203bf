// What the two attention kernels over the 8-bit cache share of the tensor cores: e4m3 products and their operands' layouts.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "kv8.cuh"
#include "ptx.cuh"

namespace hsa {

constexpr float kNone = -3.402823466e38f; // reference of a row that has seen nothing: no score of fp32 is below it

struct PageMeta {
  int pos;      // position of the page's first token; < 0: nothing to see
  float ks, vs; // scales; vs 0: no page
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// mbar_wait in a handful of instructions: the roles of these kernels share the instruction caches of their SM, and the
// unrolled loop, at every wait, costs more than the waits do.  `tries` is where the count of polls begins, or, after a wait that ran
// out, kMaxPolls, with which all later ones give up at once.  Returns the new one.  A poll may sleep for some 20 us (without that
// the waiting warps' polls take issue slots from the others).
//
// A thread whose wait ran out goes on, because its warp and others meet it at barriers of the CTA, but hands nothing on: it neither
// arrives at an mbarrier nor issues a product, so that those behind it run out too, and no place is given back to the loads whose
// last copy may still be in flight.  (A word in shared memory that the loads look at instead: 1437 us for a chunk of 1345.)
__device__ __forceinline__ uint32_t mbar_poll(uint64_t* bar, uint32_t parity, uint32_t tries) {
  uint32_t after;
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      ".reg .u32 n;\n"
      "mov.u32 n, %3;\n"
      "AGAIN:\n"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 20000;\n"
      "@p bra DONE;\n"
      "add.u32 n, n, 1;\n"
      "setp.lt.u32 q, n, %4;\n"
      "@q bra AGAIN;\n"
      "DONE:\n"
      "selp.u32 %0, %3, %4, p;\n"
      "}\n"
      : "=r"(after)
      : "r"(smem_u32(bar)), "r"(parity), "r"(tries), "n"(kMaxPolls)
      : "memory");
  return after;
}
// What is in flight at the end (copies, products) is waited for with all patience, whatever ran out before: it must not outlive the CTA.
__device__ __forceinline__ bool mbar_drain(uint64_t* bar, uint32_t parity) { return mbar_poll(bar, parity, 0) == 0; }
// The same for a bound below a poll's sleep: looks for that many cycles.  (In instances of their own: a look ahead of the polls takes
// 2 % of a chunk.)
__device__ __forceinline__ uint32_t mbar_look(uint64_t* bar, uint32_t parity, uint32_t tries, uint32_t cycles) {
  const uint32_t t0 = static_cast<uint32_t>(clock64());
  while (tries != kMaxPolls && !mbar_test_wait(bar, parity))
    if (static_cast<uint32_t>(clock64()) - t0 >= cycles) tries = kMaxPolls;
  return tries;
}
// an arrival by some threads or sometimes, without a branch
__device__ __forceinline__ void mbar_arrive_if(uint64_t* bar, bool yes) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %1, 0;\n@p mbarrier.arrive.shared::cta.b64 _, [%0];\n}\n" ::"r"(smem_u32(bar)), "r"(static_cast<uint32_t>(yes)) : "memory");
}
// the bytes alone: the arrival comes later
__device__ __forceinline__ void mbar_expect_tx_only(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
// kind::f8f6f4, e4m3 operands (format 0), fp32 accumulator; bits as idesc_bf16_f32
__host__ __device__ constexpr uint32_t idesc_e4m3(uint32_t M, uint32_t N, uint32_t a_mn, uint32_t b_mn) {
  return (1u << 4) | (a_mn << 15) | (b_mn << 16) | ((N >> 3) << 17) | ((M >> 4) << 24);
}
// kind::f16, fp16 operands (format 0)
__host__ __device__ constexpr uint32_t idesc_fp16(uint32_t M, uint32_t N, uint32_t a_mn, uint32_t b_mn) { return idesc_e4m3(M, N, a_mn, b_mn); }
// lane 0's value; what comes of it is the same for the whole warp, which the compiler knows
__device__ __forceinline__ uint32_t warp_uniform(uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); }
// Descriptors of rows of D bytes in the swizzle that spans a row (128 bytes: layout 2, 64 bytes: layout 4); eight rows are 8 * D
// bytes.  The low word is without a leading offset.
__device__ __forceinline__ uint32_t row_desc_lo(uint32_t addr) { return (addr & 0x3FFFFu) >> 4; }
template <int D>
__host__ __device__ constexpr uint32_t row_desc_hi() {
  return ((8 * D) >> 4) | 1u << 14 | (D == 128 ? 2u : 4u) << 29;
}
__device__ __forceinline__ void mma_f8_lo(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t a_hi, uint32_t b_hi, uint32_t idesc,
                                          uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      ".reg .b64 da, db;\n"
      "setp.ne.b32 p, %6, 0;\n"
      "mov.b64 da, {%1, %3};\n"
      "mov.b64 db, {%2, %4};\n"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %5, p;\n"
      "}\n" ::"r"(d_tmem),
      "r"(a_lo), "r"(b_lo), "r"(a_hi), "r"(b_hi), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Byte of (row, byte in the row) in such a tile.
template <int D>
__device__ __forceinline__ int swizzled(int row, int byte) {
  return row * D + ((byte >> 4) ^ (D == 128 ? row & 7 : (row >> 1) & 3)) * 16 + (byte & 15);
}

}  // namespace hsa
