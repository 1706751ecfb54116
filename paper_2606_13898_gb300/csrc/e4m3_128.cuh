// Device helpers of the 8-bit operators with an fp32 scale for each block of 128
// (quant128.cu, gemm128_tc.cu, group_norm.cu): the block's scale and codes,
// eight elements of a row, activations, stores.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "attn_common.cuh"
#include "common.cuh"
#include "../../include/hilo.h"

namespace hilo {

constexpr int QBLOCK = 128;

// What a block of largest magnitude `amax` is multiplied by before its rounding to e4m3, and
// its scale: 448 / amax and amax / 448, both correctly rounded; 1 and 1 for a block of zeros. Below 2^-100 amax
// counts as 2^-100, so that neither leaves fp32's normal range (the codes then end below 448).
__device__ __forceinline__ void block_scale(float amax, float& inv, float& scale) {
  const float m = amax > 0.f ? fmaxf(amax, 0x1p-100f) : 448.f;
  inv = __fdiv_rn(448.f, m);
  // m / 448 by Markstein's correction of a quotient within an ulp by its remainder, which is exact here (IBM J. Res. Dev. 34,
  // 1990): correctly rounded, as 1 / 448 is. An infinity stays one.
  constexpr float R = 1.f / 448.f;
  const float q = __fmul_rn(m, R);
  scale = m < INFINITY ? __fmaf_rn(__fmaf_rn(-448.f, q, m), R, q) : m;
}

// Eight codes of eight values.
__device__ __forceinline__ uint2 block_codes(const float* f, float inv) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; i += 2) f2_split(f2_mul(f2(f[i], f[i + 1]), f2(inv, inv)), v[i], v[i + 1]);
  return make_uint2(pack_e4m3x4(v[0], v[1], v[2], v[3]), pack_e4m3x4(v[4], v[5], v[6], v[7]));
}

// Eight neighbouring elements in 16-byte aligned memory, as they are there (TYPE 0 bf16, 1 fp16, 2 fp32).
template <int TYPE>
struct Eight {
  uint4 q[TYPE == 2 ? 2 : 1];
  __device__ __forceinline__ void clear() {
    for (auto& v : q) v = make_uint4(0u, 0u, 0u, 0u);
  }
  __device__ __forceinline__ void load(const unsigned char* p) {
#pragma unroll
    for (int i = 0; i < (TYPE == 2 ? 2 : 1); ++i) q[i] = *(reinterpret_cast<const uint4*>(p) + i);
  }
  // of what is read once
  __device__ __forceinline__ void load_once(const unsigned char* p) {
#pragma unroll
    for (int i = 0; i < (TYPE == 2 ? 2 : 1); ++i) q[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
  }
  __device__ __forceinline__ void widen(uint64_t* f) const {
    float v[8];
    widen(v);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = f2(v[2 * i], v[2 * i + 1]);
  }
  __device__ __forceinline__ void widen(float* f) const {
    const uint32_t w[8] = {q[0].x, q[0].y, q[0].z, q[0].w, q[TYPE == 2 ? 1 : 0].x, q[TYPE == 2 ? 1 : 0].y,
                           q[TYPE == 2 ? 1 : 0].z, q[TYPE == 2 ? 1 : 0].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (TYPE == 2) f[i] = __uint_as_float(w[i]);
      else if (TYPE == 0) f[i] = __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
      else f[i] = __half2float(__ushort_as_half(static_cast<unsigned short>(i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xFFFFu)));
    }
  }
};

__device__ __forceinline__ float amax8(const float* f, float m) {
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(f[i]));
  return m;
}

// SiLU z / (1 + e^-z); GELU in its tanh form, z / (1 + 2^(-2u log2(e))) with u = sqrt(2 / pi) (z + 0.044715 z^3),
// the same function.
template <int ACT>
__device__ __forceinline__ float activation(float z) {
  constexpr float LOG2E = 1.4426950408889634f;
  if (ACT == HILO_ACT_NONE) return z;
  const float t = ACT == HILO_ACT_SILU ? -LOG2E * z : -2.f * LOG2E * 0.7978845608028654f * (z + 0.044715f * z * z * z);
  float inv;  // (within 1 ulp; of infinity 0)
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(1.f + ex2(t)));
  return z * inv;
}
// Of two values in a register pair: half the instructions.
template <int ACT>
__device__ __forceinline__ uint64_t activation2(uint64_t z) {
  constexpr float LOG2E = 1.4426950408889634f, G = -2.f * LOG2E * 0.7978845608028654f;
  if (ACT == HILO_ACT_NONE) return z;
  const uint64_t t = ACT == HILO_ACT_SILU ? f2_mul(z, f2(-LOG2E, -LOG2E))
                                          : f2_mul(z, f2_fma(f2_mul(z, z), f2(0.044715f * G, 0.044715f * G), f2(G, G)));
  float lo, hi;
  f2_split(t, lo, hi);
  const uint64_t under = f2_add(f2(ex2(lo), ex2(hi)), f2(1.f, 1.f));
  f2_split(under, lo, hi);
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(lo));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(hi));
  return f2_mul(z, f2(lo, hi));
}
// f(Act<..>) for the activation `act`: one branch around all of a row's values.
template <int ACT>
struct Act {
  static constexpr int value = ACT;
};
template <typename F>
__device__ __forceinline__ void with_activation(int act, F f) {
  if (act == HILO_ACT_SILU) f(Act<HILO_ACT_SILU>());
  else if (act == HILO_ACT_GELU) f(Act<HILO_ACT_GELU>());
  else f(Act<HILO_ACT_NONE>());
}

// Four values of a row, rounded once (fp16 saturating), at an element offset that is a multiple of four.
__device__ __forceinline__ void store4(void* out, int type, long long at, const float* v) {
  if (type == HILO_F32) {
    *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
    const bool f16 = type == HILO_F16;
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) =
        f16 ? make_uint2(pack_f16x2_sat(v[0], v[1]), pack_f16x2_sat(v[2], v[3]))
            : make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  }
}

// Eight values of a row, likewise.
__device__ __forceinline__ void store8(void* out, int type, long long at, const float* v) {
  if (type == HILO_F32) {
    store4(out, type, at, v);
    store4(out, type, at + 4, v + 4);
  } else {
    const bool f16 = type == HILO_F16;
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = f16 ? pack_f16x2_sat(v[2 * j], v[2 * j + 1]) : pack_bf16x2(v[2 * j], v[2 * j + 1]);
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + at) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// The first min(*n_rows, rows) rows are there, all where n_rows is null.
__device__ __forceinline__ int rows_there(const int32_t* n_rows, int rows) {
  return n_rows ? max(0, min(__ldg(n_rows), rows)) : rows;
}

}  // namespace hilo
