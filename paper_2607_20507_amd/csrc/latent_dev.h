// Device helpers of the absorbed latent attention: products in place, and the order they
// are issued in.
#pragma once

#include "common.h"

namespace spec {
namespace {

// A product whose sum stays in accumulation registers, in place: left to itself the
// compiler keeps a second copy of the sums, and there are no registers for one.  It
// does not see that this is an MFMA, so the waits that one needs are written out:
// two states after a vector instruction that wrote an operand, sums_ready() before
// anything but such a product reads the sums.
__device__ __forceinline__ void mfma_in_place(const uint4& a, const uint4& b, f32x4& c) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0"
               : "+a"(c)
               : "v"(__builtin_bit_cast(u32x4, a)), "v"(__builtin_bit_cast(u32x4, b)));
}
// The same on vector registers, and a first product (sum 0).
__device__ __forceinline__ void mfma_in_place_v(const uint4& a, const uint4& b, f32x4& c) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0"
               : "+v"(c)
               : "v"(__builtin_bit_cast(u32x4, a)), "v"(__builtin_bit_cast(u32x4, b)));
}
__device__ __forceinline__ f32x4 mfma_first_v(const uint4& a, const uint4& b) {
  f32x4 c;
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, 0"
               : "=&v"(c)
               : "v"(__builtin_bit_cast(u32x4, a)), "v"(__builtin_bit_cast(u32x4, b)));
  return c;
}
// x ^ k, computed where it stands: the compiler would have every step's address ready
// ahead, and there are no registers for that.
__device__ __forceinline__ uint32_t xor_here(uint32_t x, uint32_t k) {
  asm volatile("v_xor_b32 %0, %1, %2" : "=v"(x) : "s"(k), "v"(x));
  return x;
}
// c *= x for such a sum, which stays where it is.
__device__ __forceinline__ void scale_in_place(f32x4& c, float x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float v = c[i], w;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(w) : "a"(v));
    w *= x;
    asm volatile("v_accvgpr_write_b32 %0, %1" : "=a"(v) : "v"(w));
    c[i] = v;
  }
}
__device__ __forceinline__ void operands_ready() { asm volatile("s_nop 1"); }
// (Keeps its place among the statements of asm only: what else reads a sum takes it from one behind this wait, or is
// moved ahead of it.)
__device__ __forceinline__ void sums_ready() { asm volatile("s_nop 15\n\ts_nop 7"); }
template <int N>
__device__ __forceinline__ void sums_ready(f32x4 (&acc)[N]) {
  sums_ready();
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+a"(acc[i]));
}

__device__ __forceinline__ void wave_fence() {
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __builtin_amdgcn_sched_barrier(0);
}
__device__ __forceinline__ void block_sync() {
  wave_fence();
  __builtin_amdgcn_s_barrier();
  wave_fence();
}

}  // namespace
}  // namespace spec
