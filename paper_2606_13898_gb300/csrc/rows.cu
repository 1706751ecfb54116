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

// Eight elements of a vector that many rows read (bf16 or fp32).
__device__ __forceinline__ void vec8(const void* base, bool f32, long long i, float* v) {
  if (f32) {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(base) + i);
    const float4 a = __ldg(p), b = __ldg(p + 1);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else {
    widen_bf16(__ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + i)), v);
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
// `red` is two arrays of four floats that take turns (`turn`): a slot is
// written again only after the reduction in between, whose barrier every
// thread passes after its last read of the slot.
template <int GROUP, bool MAX>
__device__ __forceinline__ float group_reduce(float v, float (*red)[4], int& turn) {
  auto join = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) v = join(v, __shfl_xor_sync(0xffffffffu, v, off));
  if (GROUP == 32) return v;
  float* r = red[turn];
  turn ^= 1;
  if ((threadIdx.x & 31) == 0) r[(threadIdx.x >> 5) % (GROUP / 32)] = v;
  named_bar_sync(1 + static_cast<int>(threadIdx.x) / GROUP, GROUP);
  return GROUP == 64 ? join(r[0], r[1]) : join(join(r[0], r[1]), join(r[2], r[3]));
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
// A row per group of 128 threads (64 up to 512 elements, a warp up to 256),
// 384 threads per CTA. Thread t of a group of G holds the chunks of eight
// elements t, t + G, ..: the whole row is in registers from its one read to
// its writes, and the variance is a second pass over them. The vectors are
// read for every row again: an image's rows are neighbours, so that all but
// the first read of a CTA hit its L1.
// Bound by HBM for many rows, by the chain load, reductions, store for few, so
// each group loads its next row before it reduces the present one.

constexpr int GN_THREADS = 384;
constexpr int gn_group(int d) { return d <= 256 ? 32 : d <= 512 ? 64 : 128; }

enum { Y_NONE = 0, Y_BF16 = 1, Y_F32 = 2 };

template <int NC, int GROUP>
__device__ __forceinline__ void row_norm(float (&v)[NC][8], int kind, float eps, float inv_d, int tid, int nchunk,
                                         float (*red)[4], int& turn) {
  if (kind == HILO_NORM_NONE) return;
  if (kind == HILO_NORM_LAYER) {
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += v[c][i];
    const float mean = group_reduce<GROUP, false>(sum, red, turn) * inv_d;
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (tid + GROUP * c < nchunk)  // (the chunks past the row stay zero)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] -= mean;
  }
  float sq = 0.f;
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) sq = fmaf(v[c][i], v[c][i], sq);
  const float r = rsqrtf(group_reduce<GROUP, false>(sq, red, turn) * inv_d + eps);
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[c][i] *= r;
}

template <int NC, int GROUP, bool UF32, int YM>
__global__ void __launch_bounds__(GN_THREADS) gate_norm_kernel(const __grid_constant__ NormArgs a) {
  pdl_wait();
  pdl_trigger();
  constexpr int GROUPS = GN_THREADS / GROUP;
  __shared__ float red_s[GROUPS][2][4];
  const int group = threadIdx.x / GROUP, tid = threadIdx.x % GROUP;
  float(*red)[4] = red_s[group];
  int turn = 0;
  const int d = a.s.d, nchunk = d / 8, n_txt = a.s.B * a.s.T;
  const int rows = n_txt + max(0, min(a.cu_img[a.s.B], a.s.cap));
  const float inv_d = 1.0f / static_cast<float>(d);
  const bool vf32 = a.s.vec_dtype == HILO_F32;
  const long long step = static_cast<long long>(gridDim.x) * GROUPS;
  Raw<UF32> u_raw[NC];
  Raw<YM == Y_F32> y_raw[NC];
  int stream = 0, image = 0;  // of the row loaded last
  auto load = [&](int r) {
    const long long off = static_cast<long long>(r < n_txt ? r : r - n_txt) * d;
    const void* u = r < n_txt ? a.u_txt : a.u_img;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int k = tid + GROUP * c;
      if (k < nchunk) {
        u_raw[c] = load8<UF32>(u, off + 8 * k);
        if (YM != Y_NONE) y_raw[c] = load8<YM == Y_F32>(a.y, static_cast<long long>(r) * d + 8 * k);
      }
    }
    stream = r >= n_txt;
    image = stream ? image_of(a.cu_img, a.s.B, r - n_txt) : r / a.s.T;
  };
  long long r = blockIdx.x + static_cast<long long>(gridDim.x) * group;
  if (r < rows) load(static_cast<int>(r));
  for (; r < rows; r += step) {
    const hilo_norm_vectors& vec = a.vec[stream];
    const long long vrow = static_cast<long long>(image) * a.s.vec_row;
    const long long at = r * d;
    float u[NC][8], z[NC][8];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const bool in = tid + GROUP * c < nchunk;
      float t[8];
      widen<UF32>(u_raw[c], t);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[c][i] = in ? t[i] : 0.f;
      if (YM != Y_NONE) {
        widen<YM == Y_F32>(y_raw[c], t);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[c][i] = in ? t[i] : 0.f;
      }
    }
    if (r + step < rows) load(static_cast<int>(r + step));
    if (YM != Y_NONE) {
      row_norm<NC, GROUP>(z, a.s.norm_branch, a.s.eps, inv_d, tid, nchunk, red, turn);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int k = tid + GROUP * c;
        if (k >= nchunk) continue;
        float w[8];
        if (vec.w_branch) {
          vec8(vec.w_branch, vf32, 8 * k, w);
#pragma unroll
          for (int i = 0; i < 8; ++i) z[c][i] *= w[i];
        }
        if (vec.gate) {
          vec8(vec.gate, vf32, vrow + 8 * k, w);
#pragma unroll
          for (int i = 0; i < 8; ++i) u[c][i] = fmaf(w[i], z[c][i], a.s.resid_scale * u[c][i]);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) u[c][i] = fmaf(a.s.resid_scale, u[c][i], z[c][i]);
        }
        if (a.u_out) {
          if (a.s.u_out_dtype == HILO_F32) store8_f32(a.u_out, at + 8 * k, u[c]);
          else store8_bf16(a.u_out, at + 8 * k, u[c]);
        }
      }
    }
    if (!a.h) continue;
    row_norm<NC, GROUP>(u, a.s.norm, a.s.eps, inv_d, tid, nchunk, red, turn);
    float am = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int k = tid + GROUP * c;
      if (k >= nchunk) continue;
      float w[8];
      if (vec.w_norm) {
        vec8(vec.w_norm, vf32, 8 * k, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[c][i] *= w[i];
      }
      if (vec.b_norm) {
        vec8(vec.b_norm, vf32, 8 * k, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[c][i] += w[i];
      }
      if (vec.scale) {
        vec8(vec.scale, vf32, vrow + 8 * k, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[c][i] *= 1.0f + w[i];
      }
      if (vec.shift) {
        vec8(vec.shift, vf32, vrow + 8 * k, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[c][i] += w[i];
      }
      if (a.s.h_dtype == HILO_BF16) {
        store8_bf16(a.h, at + 8 * k, u[c]);
      } else if (a.s.h_dtype == HILO_F32) {
        store8_f32(a.h, at + 8 * k, u[c]);
      } else if (a.s.h_dtype == HILO_F16) {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.h) + at + 8 * k) =
            make_uint4(pack_f16x2_sat(u[c][0], u[c][1]), pack_f16x2_sat(u[c][2], u[c][3]),
                       pack_f16x2_sat(u[c][4], u[c][5]), pack_f16x2_sat(u[c][6], u[c][7]));
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) am = fmaxf(am, fabsf(u[c][i]));
      }
    }
    if (a.s.h_dtype == HILO_E4M3) {  // quantised by the row's largest magnitude
      am = group_reduce<GROUP, true>(am, red, turn);
      const float inv = am > 0.f ? __fdiv_rn(448.0f, am) : 1.0f;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int k = tid + GROUP * c;
        if (k >= nchunk) continue;
        float q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = __fmul_rn(u[c][i], inv);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.h) + at + 8 * k) =
            make_uint2(pack_e4m3x4(q[0], q[1], q[2], q[3]), pack_e4m3x4(q[4], q[5], q[6], q[7]));
      }
      if (tid == 0) a.h_scale[r] = am > 0.f ? __fdiv_rn(am, 448.0f) : 1.0f;
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
// share them. Bound by HBM, each element read and written once.
//
// The angle in turns is pos * f, f = theta^-p / 2 pi as the sum of two floats
// (fh, fl): pos * fh is formed exactly as a product and its error, whole turns
// are taken off the product (exact), then the error and pos * fl are added.
// What is left is below one turn with an error of a few 1e-8, however far the
// position; a plain fp32 product at position 30000 is off by 2e-3 radians.

constexpr int RP_MAX_PAIRS = 128;
constexpr int RP_THREADS = 128;

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
__global__ void __launch_bounds__(RP_THREADS) rope_kernel(const __grid_constant__ RopeArgs a) {
  pdl_wait();
  pdl_trigger();
  constexpr int GROUPS = RP_THREADS / GROUP;
  constexpr int EV = Piece<DT>::EV;
  constexpr int PT = (RP_MAX_PAIRS + GROUP - 1) / GROUP;  // pairs per thread
  constexpr int BATCH = INTERLEAVED ? 4 : 2;              // units in flight per thread
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
  const char* x = static_cast<const char*>(a.x);
  char* y = static_cast<char*>(a.y);
  constexpr int ES = Piece<DT>::ES;
  int turn = 0;
  const long long step = static_cast<long long>(gridDim.x) * GROUPS;
  for (long long r = blockIdx.x + static_cast<long long>(gridDim.x) * group; r < rows; r += step) {
    const char* xr = x + r * a.x_row * ES;
    char* yr = y + r * a.y_row * ES;
    // unit u: piece u % per of head u / per
    auto head_of = [&](int u) { return static_cast<int>(static_cast<uint32_t>(u) / static_cast<uint32_t>(per)); };
    uint4 lo[BATCH], hi[BATCH];
    auto load = [&](int u0) {
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int u = u0 + GROUP * i;
        if (u < units) {
          const int h = head_of(u), e = (u - h * per) * EV;
          const char* p = xr + (h * a.x_head + e) * ES;
          lo[i] = *reinterpret_cast<const uint4*>(p);
          if (!INTERLEAVED) hi[i] = *reinterpret_cast<const uint4*>(p + a.pairs * ES);
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
        const int u = u0 + GROUP * i;
        if (u >= units) break;
        const int h = head_of(u), e = (u - h * per) * EV;
        char* p = yr + (h * a.y_head + e) * ES;
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

template <int NC, int GROUP>
cudaError_t gate_norm_of(const NormArgs& a, int num_sms, cudaStream_t st) {
  const long long R = static_cast<long long>(a.s.B) * a.s.T + a.s.cap;
  const dim3 grid(grid_for(R, GN_THREADS / GROUP, num_sms, 2));
  const bool uf = a.s.u_dtype == HILO_F32;
  auto* kern = !a.y                         ? (uf ? gate_norm_kernel<NC, GROUP, true, Y_NONE> : gate_norm_kernel<NC, GROUP, false, Y_NONE>)
               : a.s.y_dtype == HILO_BF16 ? (uf ? gate_norm_kernel<NC, GROUP, true, Y_BF16> : gate_norm_kernel<NC, GROUP, false, Y_BF16>)
                                          : (uf ? gate_norm_kernel<NC, GROUP, true, Y_F32> : gate_norm_kernel<NC, GROUP, false, Y_F32>);
  return launch_pdl(kern, grid, dim3(GN_THREADS), 0, st, a);
}

}  // namespace

cudaError_t launch_gate_norm(const NormArgs& a, int num_sms, cudaStream_t st) {
  const int group = gn_group(a.s.d);
  if (group == 32) return gate_norm_of<1, 32>(a, num_sms, st);
  if (group == 64) return gate_norm_of<1, 64>(a, num_sms, st);
  switch ((a.s.d + 1023) / 1024) {
    case 1: return gate_norm_of<1, 128>(a, num_sms, st);
    case 2: return gate_norm_of<2, 128>(a, num_sms, st);
    case 3: return gate_norm_of<3, 128>(a, num_sms, st);
    case 4: return gate_norm_of<4, 128>(a, num_sms, st);
    default: return cudaErrorInvalidValue;
  }
}

cudaError_t launch_rope(const hilo_rope_shape& s, const void* x, const float* pos, int row_base,
                        const int32_t* n_rows, void* y, int num_sms, cudaStream_t st) {
  RopeArgs a = {};
  const int ev = s.dtype == HILO_F32 ? 4 : 8;
  int D = 0;
  for (int k = 0; k < s.rot.axes; ++k) D += s.rot.axis_dims[k];
  int p = 0;
  for (int k = 0; k < s.rot.axes; ++k) {
    for (int j = 0; j < s.rot.axis_dims[k] / 2; ++j, ++p) {
      const double e = s.rot.per_axis ? 2.0 * j / s.rot.axis_dims[k] : 2.0 * p / D;
      const double f = pow(s.rot.theta, -e) * 0.15915494309189535;  // 1 / (2 pi)
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
  const dim3 grid(grid_for(s.rows, small ? RP_THREADS / 32 : 1, num_sms, 16));
#define HILO_ROPE(DT)                                                                        \
  (s.rot.interleaved ? (small ? rope_kernel<DT, true, 32> : rope_kernel<DT, true, 128>)      \
                     : (small ? rope_kernel<DT, false, 32> : rope_kernel<DT, false, 128>))
  auto* kern = s.dtype == HILO_BF16 ? HILO_ROPE(HILO_BF16) : s.dtype == HILO_F16 ? HILO_ROPE(HILO_F16) : HILO_ROPE(HILO_F32);
#undef HILO_ROPE
  return launch_pdl(kern, grid, dim3(RP_THREADS), 0, st, a);
}

}  // namespace hilo
