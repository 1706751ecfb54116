// Device helpers of the two attention kernels (attn_tc.cu, attn_var.cu):
// paired fp32 arithmetic, the exponential, row maxima, waits on two barriers.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"

namespace hilo {

// Pairs of fp32 values in one 64-bit register pair: Blackwell's paired fp32
// instructions (fma/mul/add .f32x2) apply the same IEEE operation to both
// halves at one issue slot per pair.
__device__ __forceinline__ uint64_t f2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void f2_split(uint64_t v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// mbar_wait_warp on two barriers: both phases must complete. The common case
// (both already complete) costs two try_waits and one warp vote.
__device__ __forceinline__ bool mbar_wait2_warp(uint64_t* a, uint32_t pa, uint64_t* b, uint32_t pb,
                                                volatile int* abort, int* err, int code_a, int code_b) {
  bool ok = mbar_try_wait(smem_u32(a), pa) && mbar_try_wait(smem_u32(b), pb);
  if (!ok) ok = mbar_wait(a, pa, abort, err, code_a) && mbar_wait(b, pb, abort, err, code_b);
  return __all_sync(0xffffffffu, ok);
}

// The largest of three floats in one instruction (three-input max.f32). A
// maximum is exact, so grouping the row's values by threes gives the same
// result as any other order.
__device__ __forceinline__ float fmax3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

__device__ __forceinline__ int warp_incl_scan(int v) {
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int n = __shfl_up_sync(0xffffffffu, v, off);
    if (lane_id() >= off) v += n;
  }
  return v;
}

}  // namespace hilo
