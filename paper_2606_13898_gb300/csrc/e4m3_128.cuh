// e4m3 codes with an fp32 scale for each block of 128 (quant128.cu,
// gemm128_tc.cu): the block's scale and the codes' values.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"

namespace hilo {

constexpr int QBLOCK = 128;

// What a block of largest magnitude `amax` is multiplied by before its rounding to e4m3, and
// its scale: 448 / amax and amax / 448, both correctly rounded; 1 and 1 for a block of zeros. Below 2^-100 amax
// counts as 2^-100, so that neither leaves fp32's normal range (the codes then end below 448).
__device__ __forceinline__ void block_scale(float amax, float& inv, float& scale) {
  const float m = amax > 0.f ? fmaxf(amax, 0x1p-100f) : 448.f;
  inv = __fdiv_rn(448.f, m);
  scale = __fdiv_rn(m, 448.f);
}

// Eight codes of eight values.
__device__ __forceinline__ uint2 block_codes(const float* f, float inv) {
  return make_uint2(pack_e4m3x4(__fmul_rn(f[0], inv), __fmul_rn(f[1], inv), __fmul_rn(f[2], inv), __fmul_rn(f[3], inv)),
                    pack_e4m3x4(__fmul_rn(f[4], inv), __fmul_rn(f[5], inv), __fmul_rn(f[6], inv), __fmul_rn(f[7], inv)));
}

// The first min(*n_rows, rows) rows are there, all where n_rows is null.
__device__ __forceinline__ int rows_there(const int32_t* n_rows, int rows) {
  return n_rows ? max(0, min(__ldg(n_rows), rows)) : rows;
}

}  // namespace hilo
