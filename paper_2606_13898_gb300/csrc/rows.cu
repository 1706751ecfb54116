// Rows of the conditioned block: the fused norm, gate and modulation between
// its sub-layers (gate_norm_kernel) and the rotary positions of the q and k
// heads (rope_kernel). The DiT they belong to is paper Sec. 2.1; the formulas
// are given in include/hilo.h. All arithmetic is fp32.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>

#include "common.cuh"
#include "internal.h"

namespace hilo {

namespace {

// ------------------------------------------------- eight elements of a row --
// A thread moves eight neighbouring elements at a time: 16 bytes of a 16-bit
// type, 32 of fp32.

// The elements as they are in memory.
template <bool F32>
struct Raw {
  uint4 a, b;  // b: fp32 only
};

template <bool F32>
__device__ __forceinline__ Raw<F32> load8(const void* base, long long i) {
  Raw<F32> r;
  if (F32) {
    const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(base) + i);
    r.a = p[0];
    r.b = p[1];
  } else {
    r.a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + i);
  }
  return r;
}

__device__ __forceinline__ void widen_bf16(const uint4& a, float* v) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}

__device__ __forceinline__ void widen_f16(const uint4& a, float* v) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}

template <bool F32>
__device__ __forceinline__ void widen(const Raw<F32>& r, float* v) {
  if (F32) {
    const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
  } else {
    widen_bf16(r.a, v);
  }
}

__device__ __forceinline__ void store8_f32(void* base, long long i, const float* v) {
  float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + i);
  p[0] = make_float4(v[0], v[1], v[2], v[3]);
  p[1] = make_float4(v[4], v[5], v[6], v[7]);
}

__device__ __forceinline__ void store8_bf16(void* base, long long i, const float* v) {
  *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + i) = make_uint4(
      pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}

// ------------------------------------------------- sums over a row's threads --
// Over the CTA's W warps (one row at a time), or over a warp (W = 0). `red` is two
// arrays of 16 floats that take turns (`turn`): a slot is written again only
// after the reduction in between, whose barrier every thread passes after its
// last read of the slot.
template <bool WARP, bool MAX>
__device__ __forceinline__ float row_reduce(float v, float (*red)[16], int& turn, int warps) {
  auto join = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) v = join(v, __shfl_xor_sync(0xffffffffu, v, off));
  if (WARP) return v;
  float* r = red[turn];
  turn ^= 1;
  if (lane_id() == 0) r[warp_id()] = v;
  __syncthreads();
  // (the slots past the last warp stay 0, which neither a sum nor a maximum of
  // magnitudes changes)
  float4 s = *reinterpret_cast<const float4*>(r);
  v = join(join(s.x, s.y), join(s.z, s.w));
  for (int w = 4; w < warps; w += 4) {
    s = *reinterpret_cast<const float4*>(r + w);
    v = join(v, join(join(s.x, s.y), join(s.z, s.w)));
  }
  return v;
}

// The image that packed row r belongs to: the last one that begins at or
// before it (in [0, B), whatever the offsets).
__device__ __forceinline__ int image_of(const int32_t* cu, int B, int r) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (__ldg(cu + mid) <= r) lo = mid;
    else hi = mid;
  }
  return lo;
}

// ========================================================== gate and norm ===
//
// z = norm_branch(y) w_branch; u' = rs u + gate z; h = (norm(u') w + b)(1 + scale) + shift.
//
// With A = gate w_branch, S = w (1 + scale) and C = b (1 + scale) + shift that is
// u' = rs u + A norm_branch(y) and h = S norm(u') + C.
//
// Eight elements of a row per thread: a row is a CTA of d / 8 threads (whole
// warps), of up to 256 elements a warp. The row is in registers from its one read
// to its writes, and the variance is a second pass over them. A CTA goes through
// a range of neighbouring rows and keeps A, S and C of their image in registers.
// Bound by HBM for many rows, by the chain load, reductions, store for few. What
// hides the chain is rows in flight: each row is asked for before the one ahead of
// it is reduced. (More elements per thread, as a warpgroup per row, take more
// registers and leave fewer threads on the SM: 2389 rows of 3072 30.9 us, 8586 rows
// of 1152 with both norms 65.6. Vectors read again for every row: 25.9 and 43.7,
// half of the issue slots and a third of the loads' pipe spent on them. So: 19.3 =
// 4.6 TB/s, and 17.5. Rows copied two to four ahead into shared memory or registers, sixteen
// elements per thread, or rows dealt one by one to the CTAs: 20 to 28 and 18 to 30.)

constexpr int GN_WARP_ROWS = 8;  // rows of up to 256 elements: warps per CTA

enum { Y_NONE = 0, Y_BF16 = 1, Y_F32 = 2 };

// Registers per thread, and with them the threads on an SM: three rows of 3072 at 56, two
// at 64 (with gate and norm, 15000 rows 111 us, 120 at 64); fp32 branch rows spill at 56
// (6000 rows of 2048: 35.4 us, 31.8 at 64), rows of a warp gain nothing (30000 of 256:
// 19.7 and 19.1).
__host__ __device__ constexpr int gn_regs(bool warp, int y) { return warp || y == Y_F32 ? 64 : 56; }

// Eight elements of a vector, `none` where there is no vector.
__device__ __forceinline__ void vector8(const void* v, bool f32, long long i, float none, float* out) {
  if (v == nullptr) {
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = none;
  } else if (f32) {
    widen<true>(load8<true>(v, i), out);
  } else {
    widen<false>(load8<false>(v, i), out);
  }
}

template <bool WARP>
__device__ __forceinline__ void row_norm(float (&v)[8], int kind, float eps, float inv_d, bool in, float (*red)[16],
                                         int& turn, int warps) {
  if (kind == HILO_NORM_NONE) return;
  if (kind == HILO_NORM_LAYER) {
    const float sum = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    const float mean = row_reduce<WARP, false>(sum, red, turn, warps) * inv_d;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = in ? v[i] - mean : 0.f;
  }
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) sq = fmaf(v[i], v[i], sq);
  const float r = rsqrtf(row_reduce<WARP, false>(sq, red, turn, warps) * inv_d + eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] *= r;
}

template <bool WARP, bool UF32, int YM>
__global__ void __maxnreg__((gn_regs(WARP, YM)))
    gate_norm_kernel(const __grid_constant__ NormArgs a) {
  pdl_wait();
  pdl_trigger();
  __shared__ __align__(16) float red[2][16];
  int turn = 0;
  const int warps = blockDim.x / 32;
  if (!WARP) {
    if (threadIdx.x < 32) red[threadIdx.x >> 4][threadIdx.x & 15] = 0.f;
    __syncthreads();
  }
  const int d = a.s.d, k = 8 * (WARP ? lane_id() : static_cast<int>(threadIdx.x));
  const bool in = k < d;
  const int n_txt = a.s.B * a.s.T;
  const int rows = n_txt + max(0, min(a.cu_img[a.s.B], a.s.cap));
  const float inv_d = 1.0f / static_cast<float>(d);
  // this group's range of rows
  const int groups = WARP ? gridDim.x * GN_WARP_ROWS : gridDim.x;
  const int group = WARP ? blockIdx.x * GN_WARP_ROWS + warp_id() : blockIdx.x;
  const int each = rows / groups, more = rows - each * groups;
  int r = group * each + min(group, more);
  const int end = r + each + (group < more ? 1 : 0);
  Raw<UF32> u_raw;
  Raw<YM == Y_F32> y_raw;
  auto load = [&](int row) {
    const long long off = static_cast<long long>(row < n_txt ? row : row - n_txt) * d + k;
    u_raw = load8<UF32>(row < n_txt ? a.u_txt : a.u_img, off);
    if (YM != Y_NONE) y_raw = load8<YM == Y_F32>(a.y, static_cast<long long>(row) * d + k);
  };
  if (r < end && in) load(r);
  float A[8], S[8], C[8];
  int change = r;  // the row from which on they are another image's
  for (; r < end; ++r) {
    if (r >= change) {
      const int stream = r >= n_txt;
      const int image = stream ? image_of(a.cu_img, a.s.B, r - n_txt) : r / a.s.T;
      change = !stream ? (image + 1) * a.s.T : image + 1 < a.s.B ? max(r + 1, n_txt + __ldg(a.cu_img + image + 1)) : rows;
      const hilo_norm_vectors& v = a.vec[stream];
      const long long vk = static_cast<long long>(image) * a.s.vec_row + k;
      const bool f32 = a.s.vec_dtype == HILO_F32;
      if (in) {
        float w[8];
        if (YM != Y_NONE) {
          vector8(v.gate, f32, vk, 1.0f, A);
          vector8(v.w_branch, f32, k, 1.0f, w);
#pragma unroll
          for (int i = 0; i < 8; ++i) A[i] *= w[i];
        }
        if (a.h) {
          vector8(v.scale, f32, vk, 0.0f, w);
          vector8(v.w_norm, f32, k, 1.0f, S);
          vector8(v.b_norm, f32, k, 0.0f, C);
#pragma unroll
          for (int i = 0; i < 8; ++i) S[i] *= 1.0f + w[i], C[i] *= 1.0f + w[i];
          vector8(v.shift, f32, vk, 0.0f, w);
#pragma unroll
          for (int i = 0; i < 8; ++i) C[i] += w[i];
        }
      }
    }
    const long long at = static_cast<long long>(r) * d + k;
    float u[8], z[8];
    widen<UF32>(u_raw, u);
    if (YM != Y_NONE) widen<YM == Y_F32>(y_raw, z);
    if (!in) {
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = z[i] = 0.f;
    } else if (r + 1 < end) {
      load(r + 1);
    }
    if (YM != Y_NONE) {
      row_norm<WARP>(z, a.s.norm_branch, a.s.eps, inv_d, in, red, turn, warps);
      if (in) {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = fmaf(A[i], z[i], a.s.resid_scale * u[i]);
        if (a.u_out) {
          if (a.s.u_out_dtype == HILO_F32) store8_f32(a.u_out, at, u);
          else store8_bf16(a.u_out, at, u);
        }
      }
    }
    if (!a.h) continue;
    row_norm<WARP>(u, a.s.norm, a.s.eps, inv_d, in, red, turn, warps);
    float am = 0.f;
    if (in) {
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = fmaf(u[i], S[i], C[i]);
      if (a.s.h_dtype == HILO_BF16) {
        store8_bf16(a.h, at, u);
      } else if (a.s.h_dtype == HILO_F32) {
        store8_f32(a.h, at, u);
      } else if (a.s.h_dtype == HILO_F16) {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.h) + at) =
            make_uint4(pack_f16x2_sat(u[0], u[1]), pack_f16x2_sat(u[2], u[3]), pack_f16x2_sat(u[4], u[5]),
                       pack_f16x2_sat(u[6], u[7]));
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) am = fmaxf(am, fabsf(u[i]));
      }
    }
    if (a.s.h_dtype == HILO_E4M3) {  // quantised by the row's largest magnitude
      am = row_reduce<WARP, true>(am, red, turn, warps);
      const float inv = am > 0.f ? __fdiv_rn(448.0f, am) : 1.0f;
      if (in) {
        float q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = __fmul_rn(u[i], inv);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.h) + at) =
            make_uint2(pack_e4m3x4(q[0], q[1], q[2], q[3]), pack_e4m3x4(q[4], q[5], q[6], q[7]));
      }
      if (k == 0) a.h_scale[r] = am > 0.f ? __fdiv_rn(am, 448.0f) : 1.0f;
    }
  }
}

// ================================================================= rotary ===
//
// (a, b) -> (a cos t - b sin t, a sin t + b cos t), t = pos * theta^-p.
//
// A row per group of 128 threads (a warp where a row is at most 64 pieces of
// 16 bytes). The row's pieces are on their way while the group's threads form
// the row's angles, one pair each, into shared memory; all heads of the row
// share them. Bound by HBM, each element read and written once: 2389 interleaved
// rows of 48 heads of 128 (bf16) 10.6 us = 5.5 TB/s, 18001 split fp32 rows of 16 heads
// of 64 24.8 us = 5.9 TB/s.
//
// How many pieces a thread has in flight decides with how many CTAs an SM holds:
// interleaved, six pieces and 8 CTAs (four and 10 take 12.4 us for the first rows above);
// split, two pieces of each half and 9 CTAs (three of each half take 27.4 us for the
// second rows, one and 16 CTAs 26.4; two and 12 spill, and 1415 rows of 16 heads of 128
// take 5.3 us instead of 4.7; rows of a warp spill a little at 9 already, 4 to 16 bytes). A thread steps through heads and pieces by addition: one
// division per row and piece took 11.5 us for the first rows, and 5.1 us instead of 2.9
// for 16 rows of 48 heads of 256.
//
// The angle in turns is pos * f, f = theta^-p / 2 pi as the sum of two floats
// (fh, fl): pos * fh is formed exactly as a product and its error, whole turns
// are taken off the product (exact), then the error and pos * fl are added.
// What is left is below one turn, with an error below 2^-24 turns up to |pos| = 2^24, the last
// whole numbers that fp32 tells apart; a plain fp32 product at position 30000 is off by 2e-3
// radians. Beyond, the error grows with the position: f is known to 2^-46, and the two
// terms added are no longer small (1e-6 turns at 2^30, 1e-3 at 1e12).

constexpr int RP_MAX_PAIRS = 128;
constexpr int RP_THREADS = 128;
constexpr int rp_ctas(bool interleaved) { return interleaved ? 8 : 9; }  // resident per SM

struct RopeArgs {
  const void* x;
  void* y;
  const float* pos;
  const int32_t* n_rows;
  long long x_row, x_head, y_row, y_head;
  int rows, row_base, heads, axes;
  int pairs;      // D / 2
  int per_head;   // pieces of a head that are rotated: interleaved one piece, else two (i and i + D/2)
  int rest;       // pieces of a head that are copied (0 in place)
  int rest_from;  // the first of them, in elements
  float fh[RP_MAX_PAIRS], fl[RP_MAX_PAIRS];
  uint8_t axis[RP_MAX_PAIRS];
};

// 16 bytes of the dtype as fp32: EV = 8 (16-bit types) or 4 elements.
template <int DT>
struct Piece {
  static constexpr int EV = DT == HILO_F32 ? 4 : 8;
  static constexpr int ES = DT == HILO_F32 ? 4 : 2;
};

template <int DT>
__device__ __forceinline__ void piece_widen(const uint4& a, float* v) {
  if (DT == HILO_F32) {
    v[0] = __uint_as_float(a.x), v[1] = __uint_as_float(a.y), v[2] = __uint_as_float(a.z), v[3] = __uint_as_float(a.w);
  } else if (DT == HILO_BF16) {
    widen_bf16(a, v);
  } else {
    widen_f16(a, v);
  }
}

template <int DT>
__device__ __forceinline__ uint4 piece_pack(const float* v) {
  if (DT == HILO_F32)
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (DT == HILO_BF16) {
      w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    } else {
      const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int DT, bool INTERLEAVED, int GROUP>
__global__ void __launch_bounds__(RP_THREADS, rp_ctas(INTERLEAVED)) rope_kernel(const __grid_constant__ RopeArgs a) {
  pdl_wait();
  pdl_trigger();
  constexpr int GROUPS = RP_THREADS / GROUP;
  constexpr int EV = Piece<DT>::EV;
  constexpr int PT = (RP_MAX_PAIRS + GROUP - 1) / GROUP;  // pairs per thread
  constexpr int BATCH = INTERLEAVED ? 6 : 2;              // units in flight per thread
  // cosines and sines of a group's row, of two rows in turn
  __shared__ __align__(16) float cs_s[GROUPS][2][RP_MAX_PAIRS], sn_s[GROUPS][2][RP_MAX_PAIRS];
  const int group = threadIdx.x / GROUP, tid = threadIdx.x % GROUP;
  float fh[PT], fl[PT];
  int ax[PT];
#pragma unroll
  for (int i = 0; i < PT; ++i) {
    const int p = min(tid + GROUP * i, RP_MAX_PAIRS - 1);
    fh[i] = a.fh[p];
    fl[i] = a.fl[p];
    ax[i] = a.axis[p];
  }
  const int rows = a.n_rows ? static_cast<int>(min(static_cast<long long>(a.rows),
                                                   static_cast<long long>(a.row_base) + max(0, *a.n_rows)))
                            : a.rows;
  const int per = a.per_head, units = a.heads * per, rest = a.heads * a.rest;
  const int head0 = tid / per, piece0 = tid - head0 * per, step_h = GROUP / per, step_e = GROUP - step_h * per;
  const char* x = static_cast<const char*>(a.x);
  char* y = static_cast<char*>(a.y);
  constexpr int ES = Piece<DT>::ES;
  int turn = 0;
  const long long step = static_cast<long long>(gridDim.x) * GROUPS;
  for (long long r = blockIdx.x + static_cast<long long>(gridDim.x) * group; r < rows; r += step) {
    const char* xr = x + r * a.x_row * ES;
    char* yr = y + r * a.y_row * ES;
    // unit u: piece u % per of head u / per; the thread's next unit is step_h heads and
    // step_e pieces on
    uint4 lo[BATCH], hi[BATCH];
    int hl = head0, el = piece0, hs = head0, es = piece0;  // of the loads, of the stores
    auto next = [&](int& h, int& e) {
      h += step_h;
      e += step_e;
      if (e >= per) {
        e -= per;
        ++h;
      }
    };
    auto load = [&](int u0) {
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        if (u0 + GROUP * i < units) {
          const char* p = xr + (hl * a.x_head + el * EV) * ES;
          lo[i] = *reinterpret_cast<const uint4*>(p);
          if (!INTERLEAVED) hi[i] = *reinterpret_cast<const uint4*>(p + a.pairs * ES);
          next(hl, el);
        }
      }
    };
    load(tid);
    float* cs = cs_s[group][turn];
    float* sn = sn_s[group][turn];
    turn ^= 1;
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int p = tid + GROUP * i;
      if (p < a.pairs) {
        const float at = __ldg(a.pos + r * a.axes + ax[i]);
        const float t = __fmul_rn(at, fh[i]);
        const float err = fmaf(at, fh[i], -t);
        const float turns = (t - rintf(t)) + fmaf(at, fl[i], err);
        float s, c;
        sincospif(2.0f * turns, &s, &c);
        cs[p] = c;
        sn[p] = s;
      }
    }
    if (GROUP == 32) __syncwarp();
    else named_bar_sync(1 + group, GROUP);
    for (int u0 = tid; u0 < units; u0 += GROUP * BATCH) {
      if (u0 != tid) load(u0);
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        if (u0 + GROUP * i >= units) break;
        const int e = es * EV;
        char* p = yr + (hs * a.y_head + e) * ES;
        next(hs, es);
        float v[EV], w[EV];
        piece_widen<DT>(lo[i], v);
        if constexpr (INTERLEAVED) {
          float o[EV];
#pragma unroll
          for (int j = 0; j < EV / 2; ++j) {
            const float c = cs[e / 2 + j], s = sn[e / 2 + j];
            o[2 * j] = fmaf(v[2 * j], c, -(v[2 * j + 1] * s));
            o[2 * j + 1] = fmaf(v[2 * j], s, v[2 * j + 1] * c);
          }
          *reinterpret_cast<uint4*>(p) = piece_pack<DT>(o);
        } else {
          piece_widen<DT>(hi[i], w);
          float oa[EV], ob[EV];
#pragma unroll
          for (int j = 0; j < EV; ++j) {
            const float c = cs[e + j], s = sn[e + j];
            oa[j] = fmaf(v[j], c, -(w[j] * s));
            ob[j] = fmaf(v[j], s, w[j] * c);
          }
          *reinterpret_cast<uint4*>(p) = piece_pack<DT>(oa);
          *reinterpret_cast<uint4*>(p + a.pairs * ES) = piece_pack<DT>(ob);
        }
      }
    }
    for (int u = tid; u < rest; u += GROUP) {
      const int h = u / a.rest, e = a.rest_from + (u - h * a.rest) * EV;
      *reinterpret_cast<uint4*>(yr + (h * a.y_head + e) * ES) =
          *reinterpret_cast<const uint4*>(xr + (h * a.x_head + e) * ES);
    }
  }
}

int grid_for(long long items, int per_block, int num_sms, int blocks_per_sm) {
  const long long g = (items + per_block - 1) / per_block, most = static_cast<long long>(num_sms) * blocks_per_sm;
  return static_cast<int>(g < 1 ? 1 : g < most ? g : most);
}

template <bool WARP, bool UF32, int YM>
cudaError_t gate_norm_of(const NormArgs& a, int num_sms, cudaStream_t st) {
  const long long R = static_cast<long long>(a.s.B) * a.s.T + a.s.cap;
  const int threads = WARP ? 32 * GN_WARP_ROWS : (a.s.d / 8 + 31) / 32 * 32;
  const dim3 grid(grid_for(R, WARP ? GN_WARP_ROWS : 1, num_sms, 65536 / gn_regs(WARP, YM) / threads));
  return launch_pdl(gate_norm_kernel<WARP, UF32, YM>, grid, dim3(threads), 0, st, a);
}

template <bool WARP>
cudaError_t gate_norm_by_type(const NormArgs& a, int num_sms, cudaStream_t st) {
  const bool uf = a.s.u_dtype == HILO_F32;
  if (!a.y) return uf ? gate_norm_of<WARP, true, Y_NONE>(a, num_sms, st) : gate_norm_of<WARP, false, Y_NONE>(a, num_sms, st);
  if (a.s.y_dtype == HILO_BF16)
    return uf ? gate_norm_of<WARP, true, Y_BF16>(a, num_sms, st) : gate_norm_of<WARP, false, Y_BF16>(a, num_sms, st);
  return uf ? gate_norm_of<WARP, true, Y_F32>(a, num_sms, st) : gate_norm_of<WARP, false, Y_F32>(a, num_sms, st);
}

}  // namespace

cudaError_t launch_gate_norm(const NormArgs& a, int num_sms, cudaStream_t st) {
  return a.s.d <= 256 ? gate_norm_by_type<true>(a, num_sms, st) : gate_norm_by_type<false>(a, num_sms, st);
}

cudaError_t launch_rope(const hilo_rope_shape& s, const void* x, const float* pos, int row_base,
                        const int32_t* n_rows, void* y, int num_sms, cudaStream_t st) {
  RopeArgs a = {};
  const int ev = s.dtype == HILO_F32 ? 4 : 8;
  int D = 0;
  for (int k = 0; k < s.rot.axes; ++k) D += s.rot.axis_dims[k];
  // each frequency from the one before it: 128 products of doubles are off by 2^-46, and
  // a power per pair is half of the call's time on the host
  int p = 0;
  double f = 0.15915494309189535;  // 1 / (2 pi)
  double step = pow(s.rot.theta, -2.0 / D);
  for (int k = 0; k < s.rot.axes; ++k) {
    if (s.rot.per_axis) {
      f = 0.15915494309189535;
      step = pow(s.rot.theta, -2.0 / s.rot.axis_dims[k]);
    }
    for (int j = 0; j < s.rot.axis_dims[k] / 2; ++j, ++p, f *= step) {
      a.fh[p] = static_cast<float>(f);
      a.fl[p] = static_cast<float>(f - static_cast<double>(a.fh[p]));
      a.axis[p] = static_cast<uint8_t>(k);
    }
  }
  a.x = x;
  a.y = y;
  a.pos = pos;
  a.n_rows = n_rows;
  a.x_row = s.x_row;
  a.x_head = s.x_head;
  a.y_row = s.y_row;
  a.y_head = s.y_head;
  a.rows = s.rows;
  a.row_base = row_base;
  a.heads = s.heads;
  a.axes = s.rot.axes;
  a.pairs = D / 2;
  a.per_head = (s.rot.interleaved ? D : D / 2) / ev;
  a.rest = x == y ? 0 : (s.head_dim - D) / ev;
  a.rest_from = D;
  // a warp per row where the row gives its lanes at most two units each
  const bool small = a.heads * (a.per_head + a.rest) <= 64;
  const dim3 grid(grid_for(s.rows, small ? RP_THREADS / 32 : 1, num_sms, rp_ctas(s.rot.interleaved)));
#define HILO_ROPE(DT)                                                                        \
  (s.rot.interleaved ? (small ? rope_kernel<DT, true, 32> : rope_kernel<DT, true, 128>)      \
                     : (small ? rope_kernel<DT, false, 32> : rope_kernel<DT, false, 128>))
  auto* kern = s.dtype == HILO_BF16 ? HILO_ROPE(HILO_BF16) : s.dtype == HILO_F16 ? HILO_ROPE(HILO_F16) : HILO_ROPE(HILO_F32);
#undef HILO_ROPE
  return launch_pdl(kern, grid, dim3(RP_THREADS), 0, st, a);
}

}  // namespace hilo
