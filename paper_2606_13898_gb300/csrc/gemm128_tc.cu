// Products of e4m3 rows and weights with an fp32 scale for each block of 128, and
// the gated feed-forward's first half built on them (hilo_gemm_e4m3_128,
// hilo_gated_e4m3_128, include/hilo.h; paper Sec. 3.3 reports FP8 on top of
// HiLo-Token, the scaling scheme is the library's):
//   y[r][n] = sum_b sa[b][r] sw[n / 128][b] sum_{k in block b} a[r][k] w[n][k]   (+ bias)
//   h[r][n] = act(gate[r][n]) * up[r][n],   gate and up two such products of the same rows.
//
// The scales change along K, so the tensor core cannot sum past a block: it
// forms each block's product of 128 (four tcgen05.mma kind::f8f6f4) in a tensor memory buffer of its
// own, and eight warps add it, scaled, to sums in their registers while the next
// block's is formed. The codes' products are exact in fp32.
//
// Two kernels:
//   few128   few rows: features on the lanes (M), rows on the columns (N = NT). A CTA has 128
//            features; a cluster of up to eight shares them along K and adds its sums up through
//            distributed shared memory in a fixed order. Bound by reading the weights.
//   many128  CTA pairs (cta_group::2): 256 rows on the lanes, 256 features (or 128 of gate and 128
//            of up) on the columns, a persistent grid. Bound by the tensor pipe and by shared memory, which
//            takes each operand byte twice.
//
// Every mbarrier wait is bounded (error latched, TMEM freed, CTA returns).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "attn_common.cuh"
#include "common.cuh"
#include "e4m3_128.cuh"
#include "internal.h"

namespace hilo {

__device__ int g_gemm128_err;

namespace {

constexpr int BK = 128;  // K of a stage: a block, a 128-byte swizzled row
constexpr int PIECE = 128 * BK;  // bytes of 128 rows of a stage

struct Params128 {
  const float* a_scale;      // [k / 128][a_scale_ld]
  const float* w_scale[2];   // [n / 128][w_scale_ld]
  const __nv_bfloat16* bias[2];
  const int32_t* n_rows;
  void* out;
  float* out_scale;          // [n / 128][out_scale_ld]
  long long a_scale_ld, w_scale_ld, out_row, out_scale_ld;
  int rows, n, kblocks;
  int out_type, act;
  int out_wide;  // out's rows begin on 32 bytes
};

// ------------------------------------------------------------------ tcgen05 --

// D[tmem] (+)= A[smem] * B[smem], e4m3 inputs, fp32 accumulator: 32 elements of K.
__device__ __forceinline__ void umma_e4m3(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc,
                                          uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "mov.b64 da, {%1, %3};\n\t"
      "mov.b64 db, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %4, p;\n\t}" ::"r"(d_tmem),
      "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(acc)
      : "memory");
}

__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float* v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32"
      " {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(taddr));
}
template <int N>
__device__ __forceinline__ void tmem_ldn(uint32_t taddr, float* v) {
  static_assert(N == 8 || N == 16 || N == 32, "columns of a load");
  if constexpr (N == 8) tmem_ld8(taddr, v);
  else if constexpr (N == 16) tmem_ld16(taddr, v);
  else tmem_ld32(taddr, v);
}
// tcgen05.wait::ld that marks N registers as written here (tmem_ld_wait_regs).
template <int N>
__device__ __forceinline__ void tmem_ld_wait_n(float* v) {
  if constexpr (N == 32) {
    tmem_ld_wait_regs(v);
  } else {
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < N; i += 8)
      asm volatile("" : "+f"(v[i]), "+f"(v[i + 1]), "+f"(v[i + 2]), "+f"(v[i + 3]), "+f"(v[i + 4]), "+f"(v[i + 5]),
                        "+f"(v[i + 6]), "+f"(v[i + 7]));
  }
}

// ----------------------------------------------------------- scales in flight --
// A warp's scales of the blocks to come, through its own ring in shared memory: four bytes
// a lane and copy, so any row offset will do; no other warp is waited for.

__device__ __forceinline__ void copy4(void* dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

constexpr int SCALES_AHEAD = 4;

__device__ __forceinline__ float bias_at(const __nv_bfloat16* b, int n) { return b ? __bfloat162float(__ldg(b + n)) : 0.f; }

// ------------------------------------------------------------------- few rows --

constexpr int FEW_THREADS = 320;  // eight warps for the sums, one for the copies, one for the products
constexpr int FEW_SPLIT = 8;      // CTAs of a cluster at most

template <int NT, bool GATED>
struct Few {
  static constexpr int PARTS = GATED ? 2 : 1;
  static constexpr int STAGE = PARTS * PIECE + NT * BK;
  static constexpr int CTAS = NT * PARTS <= 64 ? 2 : 1;  // per SM
  static constexpr int STAGES = CTAS == 2 ? (104 * 1024) / STAGE : (200 * 1024) / STAGE;
  static constexpr int BUFS = NT * PARTS <= 64 ? 4 : 2;
  static constexpr int NEED = BUFS * PARTS * NT;
  static constexpr uint32_t TMEM_COLS = NEED <= 64 ? 64 : NEED <= 128 ? 128 : NEED <= 256 ? 256 : 512;
  static constexpr int COLS = NT / 2;  // of a warp
  static constexpr int SLOT = COLS + 4;  // floats of a warp's scales of a block: its rows', its weights'
  static constexpr int OFF_BARS = STAGES * STAGE;
  static constexpr int OFF_SCALES = OFF_BARS + 256;
  static constexpr int SMEM_BYTES = OFF_SCALES + 8 * SCALES_AHEAD * SLOT * 4 + 1024;
  static_assert(STAGES * STAGE >= PARTS * NT * 128 * 4, "the sums take the stages' place");
  static_assert((2 * STAGES + 2 * BUFS + 3) * 8 <= 256, "room for the barriers");
  static_assert(SMEM_BYTES <= (CTAS == 2 ? 112 : 226) * 1024, "shared memory");
};

template <int NT, bool GATED>
__global__ void __launch_bounds__(FEW_THREADS, Few<NT, GATED>::CTAS)
    few128_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w0,
                  const __grid_constant__ CUtensorMap tm_w1, const __grid_constant__ Params128 p, int split) {
  using C = Few<NT, GATED>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::OFF_BARS);
  uint64_t* empty = full + C::STAGES;
  uint64_t* tfull = empty + C::STAGES;
  uint64_t* tempty = tfull + C::BUFS;
  uint64_t* drain = tempty + C::BUFS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* err = &g_gemm128_err;
  const int warp = warp_id(), lane = lane_id();

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < C::BUFS; ++b) {
      mbar_init(&tfull[b], 1);
      mbar_init(&tempty[b], 8);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 8 && lane == 0) {
    tma_prefetch_desc(&tm_a);
    tma_prefetch_desc(&tm_w0);
    if (GATED) tma_prefetch_desc(&tm_w1);
  }
  if (warp == 9) {
    tmem_alloc(tmem_slot, C::TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();  // all threads, ahead of the roles
  pdl_trigger();

  const int rank = blockIdx.x % split, f0 = (blockIdx.x / split) * 128, r0 = blockIdx.y * NT;
  const int rows = min(NT, rows_there(p.n_rows, p.rows) - r0);
  if (rows <= 0) {  // (the same for the whole cluster)
    if (warp == 9) tmem_dealloc(tmem, C::TMEM_COLS);
    return;
  }
  const int kb0 = static_cast<int>(static_cast<long long>(p.kblocks) * rank / split);
  const int nkb = static_cast<int>(static_cast<long long>(p.kblocks) * (rank + 1) / split) - kb0;

  if (warp == 8) {
    // ---------------- copies
    const bool issuer = elect_one();
    uint32_t armed = 0, par = 0;
    bool ok = true;
    for (int i = 0, st = 0, ph = 0; i < nkb; ++i) {
      if (!mbar_wait_warp(&empty[st], ph ^ 1u, abort_flag, err, DEV_TIMEOUT_GEMM + 256 * 11)) {
        ok = false;
        break;
      }
      if (issuer) {
        unsigned char* dst = smem + st * C::STAGE;
        const int k = (kb0 + i) * BK;
        mbar_arrive_expect_tx(&full[st], C::STAGE);
        tma_load_2d(dst, &tm_w0, &full[st], k, f0);
        if (GATED) tma_load_2d(dst + PIECE, &tm_w1, &full[st], k, f0);
        tma_load_2d(dst + C::PARTS * PIECE, &tm_a, &full[st], k, r0);
      }
      __syncwarp();
      armed |= 1u << st;
      par = (par & ~(1u << st)) | (static_cast<uint32_t>(ph) << st);
      if (++st == C::STAGES) {
        st = 0;
        ph ^= 1;
      }
    }
    if (!ok) {  // the copies in flight, before the CTA exits
      const uint64_t g0 = globaltimer_ns();
      for (int st = 0; st < C::STAGES; ++st)
        if (armed >> st & 1u)
          while (!mbar_try_wait(smem_u32(&full[st]), par >> st & 1u) && globaltimer_ns() - g0 < HILO_WAIT_LIMIT_NS / 4) {
          }
    }
    __syncwarp();
  } else if (warp == 9) {
    // ---------------- products
    const bool issuer = elect_one();
    constexpr uint32_t idesc = idesc_kind_f16(128, NT, 0, 0, 0);  // (format code 0 is E4M3)
    constexpr uint32_t hi = sw128_hi(1024);
    const uint32_t base = (smem_u32(smem) >> 4) + sw128_lo_lbo(16);
    for (int i = 0, st = 0, ph = 0; i < nkb; ++i) {
      const int b = i % C::BUFS;
      if (!mbar_wait_warp(&tempty[b], (static_cast<uint32_t>(i / C::BUFS) & 1u) ^ 1u, abort_flag, err,
                          DEV_TIMEOUT_GEMM + 256 * 12) ||
          !mbar_wait_warp(&full[st], static_cast<uint32_t>(ph), abort_flag, err, DEV_TIMEOUT_GEMM + 256 * 13))
        break;
      tc_fence_after();
      if (issuer) {
        const uint32_t w = base + static_cast<uint32_t>(st * C::STAGE >> 4), a = w + (C::PARTS * PIECE >> 4);
#pragma unroll
        for (int g = 0; g < C::PARTS; ++g)
#pragma unroll
          for (int k = 0; k < BK / 32; ++k)
            umma_e4m3(tmem + (b * C::PARTS + g) * NT, w + g * (PIECE >> 4) + 2 * k, a + 2 * k, hi, idesc, k > 0 ? 1u : 0u);
        umma_commit(&empty[st]);
        umma_commit(&tfull[b]);
      }
      __syncwarp();
      if (++st == C::STAGES) {
        st = 0;
        ph ^= 1;
      }
    }
    if (issuer) umma_commit(drain);
    __syncwarp();
    const uint64_t g0 = globaltimer_ns();
    while (!mbar_try_wait(smem_u32(drain), 0u)) {
      if (globaltimer_ns() - g0 > HILO_WAIT_LIMIT_NS) {
        if (issuer) atomicExch(err, DEV_TIMEOUT_GEMM + 256 * 14);
        break;
      }
    }
    __syncwarp();
  } else {
    // ---------------- sums: lane quarter warp % 4 (32 features), half of the columns
    const int q = warp & 3, col0 = (warp >> 2) * C::COLS;
    float* ring = reinterpret_cast<float*>(smem + C::OFF_SCALES) + warp * SCALES_AHEAD * C::SLOT;
    const float* ws0 = p.w_scale[0] + (f0 >> 7) * p.w_scale_ld + kb0;
    const float* ws1 = GATED ? p.w_scale[1] + (f0 >> 7) * p.w_scale_ld + kb0 : ws0;
    const float* as = p.a_scale + kb0 * p.a_scale_ld + r0 + col0;
    auto fetch = [&](int i) {
      if (i < nkb) {
        float* slot = ring + (i % SCALES_AHEAD) * C::SLOT;
#pragma unroll
        for (int c = 0; c < C::COLS; c += 32) {
          const bool in = col0 + c + lane < rows;
          if (c + lane < C::COLS) copy4(slot + c + lane, in ? as + i * p.a_scale_ld + c + lane : p.a_scale, in);
        }
        if (lane < C::PARTS) copy4(slot + C::COLS + lane, (lane ? ws1 : ws0) + i, true);
      }
      copies_commit();
    };
    for (int i = 0; i < SCALES_AHEAD - 1; ++i) fetch(i);
    uint64_t acc[C::PARTS][C::COLS / 2] = {};
    const uint32_t taddr = tmem + (static_cast<uint32_t>(q * 32) << 16) + col0;
    bool ok = true;
    for (int i = 0; i < nkb; ++i) {
      __syncwarp();  // (the slot that is fetched into was read by all lanes)
      fetch(i + SCALES_AHEAD - 1);
      const int b = i % C::BUFS;
      if (!mbar_wait_warp(&tfull[b], static_cast<uint32_t>(i / C::BUFS) & 1u, abort_flag, err, DEV_TIMEOUT_GEMM + 256 * 15)) {
        ok = false;
        break;
      }
      tc_fence_after();
      constexpr int STEP = C::COLS < 32 ? C::COLS : 32, LOADS = C::PARTS * C::COLS / STEP;
      float v[LOADS][STEP];
#pragma unroll
      for (int l = 0; l < LOADS; ++l)
        tmem_ldn<STEP>(taddr + b * C::PARTS * NT + (l * STEP / C::COLS) * NT + l * STEP % C::COLS, v[l]);
      copies_wait<SCALES_AHEAD - 1>();
      __syncwarp();  // every lane's copies of block i have arrived
#pragma unroll
      for (int l = 0; l < LOADS; ++l) tmem_ld_wait_n<STEP>(v[l]);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&tempty[b]);
      const float* slot = ring + (i % SCALES_AHEAD) * C::SLOT;
#pragma unroll
      for (int l = 0; l < LOADS; ++l) {
        const int g = l * STEP / C::COLS, c0 = l * STEP % C::COLS;
        const float w = slot[C::COLS + g];
        const uint64_t w2 = f2(w, w);
#pragma unroll
        for (int c = 0; c < STEP; c += 4) {
          const float4 s = *reinterpret_cast<const float4*>(slot + c0 + c);
          uint64_t* o = &acc[g][(c0 + c) / 2];
          o[0] = f2_fma(f2(v[l][c], v[l][c + 1]), f2_mul(f2(s.x, s.y), w2), o[0]);
          o[1] = f2_fma(f2(v[l][c + 2], v[l][c + 3]), f2_mul(f2(s.z, s.w), w2), o[1]);
        }
      }
    }
    copies_wait<0>();
    if (ok) {
      // [part][row][feature], over the stages: every product has been waited for. (After a given-up wait
      // copies may still arrive there; nothing is written then, and what is read below is not meant to be right.)
      float* sums = reinterpret_cast<float*>(smem) + q * 32 + lane;
#pragma unroll
      for (int g = 0; g < C::PARTS; ++g)
#pragma unroll
        for (int c = 0; c < C::COLS; c += 2) {
          float lo, hi;
          f2_split(acc[g][c / 2], lo, hi);
          sums[(g * NT + col0 + c) * 128] = lo;
          sums[(g * NT + col0 + c + 1) * 128] = hi;
        }
    }
  }
  __syncthreads();
  if (split > 1) cluster_sync();
  // ---- rows rank, rank + split, ..: a warp each, four features a lane, the CTAs' sums in the order of K
  const bool good = *abort_flag == 0;
  const int f = f0 + 4 * lane;
  const uint32_t mine = smem_u32(smem) + 16 * lane;
  for (int t = rank + split * warp; good && t < rows; t += split * (FEW_THREADS / 32)) {
    float y[C::PARTS][4] = {};
    for (int s = 0; s < split; ++s)
#pragma unroll
      for (int g = 0; g < C::PARTS; ++g) {
        float4 v;
        const uint32_t at = mapa_shared(mine + (g * NT + t) * 512, split > 1 ? s : 0);
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                     : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                     : "r"(at)
                     : "memory");
        y[g][0] += v.x;
        y[g][1] += v.y;
        y[g][2] += v.z;
        y[g][3] += v.w;
      }
    const bool in = f < p.n;  // (n is a multiple of 16)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      y[0][j] += in ? bias_at(p.bias[0], f + j) : 0.f;
      if (GATED) y[0][j] = activation(y[0][j], p.act) * (y[C::PARTS - 1][j] + (in ? bias_at(p.bias[1], f + j) : 0.f));
    }
    if (GATED && p.out_type == HILO_E4M3) {
      float m = 0.f, inv, sc;
#pragma unroll
      for (int j = 0; j < 4; ++j) m = fmaxf(m, in ? fabsf(y[0][j]) : 0.f);
#pragma unroll
      for (int off = 16; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
      block_scale(m, inv, sc);
      if (in)
        *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(p.out) + (r0 + t) * p.out_row + f) =
            pack_e4m3x4(__fmul_rn(y[0][0], inv), __fmul_rn(y[0][1], inv), __fmul_rn(y[0][2], inv), __fmul_rn(y[0][3], inv));
      if (lane == 0) p.out_scale[(f0 >> 7) * p.out_scale_ld + r0 + t] = sc;
    } else if (in) {
      store4(p.out, p.out_type, (r0 + t) * p.out_row + f, y[0]);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (split > 1) cluster_sync();  // no CTA leaves while another reads its sums
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, C::TMEM_COLS);
  }
}

// ------------------------------------------------------------------ many rows --

constexpr int MANY_THREADS = 384;  // two warpgroups for the sums, one for copies and products
constexpr uint32_t SUM_REGS = 216, CONTROL_REGS = 72;
static_assert(256 * SUM_REGS + 128 * CONTROL_REGS <= 65536, "registers of an SM");
constexpr int MANY_STAGES = 6;
constexpr int MANY_STAGE = 2 * PIECE;  // 128 rows of A, 128 features: half of the pair's
constexpr int MANY_BARS = MANY_STAGES * MANY_STAGE;
constexpr int MANY_SLOT = 36;  // floats of a warp's scales of a block: its rows', the weights' two
constexpr int MANY_SCALES = MANY_BARS + 256;
constexpr int MANY_MOST = MANY_SCALES + 8 * SCALES_AHEAD * MANY_SLOT * 4;  // [2][128] row maxima
constexpr int MANY_SMEM = MANY_MOST + 2 * 128 * 4 + 1024;
static_assert(MANY_SMEM <= 227 * 1024, "shared memory of a CTA");
constexpr int PANEL = 8;  // row tiles that are taken together along the features

template <bool GATED>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(MANY_THREADS, 1)
    many128_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w0,
                   const __grid_constant__ CUtensorMap tm_w1, const __grid_constant__ Params128 p) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + MANY_BARS);
  uint64_t* empty = full + MANY_STAGES;
  uint64_t* tfull = empty + MANY_STAGES;
  uint64_t* tempty = tfull + 2;
  uint64_t* drain = tempty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* err = &g_gemm128_err;
  const int warp = warp_id(), lane = lane_id();
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < MANY_STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&tfull[b], 1);
      mbar_init(&tempty[b], 16);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 8 && lane == 0) {
    tma_prefetch_desc(&tm_a);
    tma_prefetch_desc(&tm_w0);
    tma_prefetch_desc(&tm_w1);
  }
  if (warp == 9) {
    tmem_alloc_pair(tmem_slot, 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // both CTAs' barriers are initialised before any remote use
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();  // all threads, ahead of the roles
  pdl_trigger();

  // The pair's tiles: panels of PANEL row tiles, within one the row tiles of a feature tile after one another, so that the
  // pairs at work at a time read few rows and few features.
  constexpr int TF = GATED ? 128 : 256;  // features of a tile
  const int rows = rows_there(p.n_rows, p.rows);
  const int row_tiles = (rows + 255) / 256, f_tiles = (p.n + TF - 1) / TF;
  const int tiles = row_tiles * f_tiles, step = gridDim.x >> 1;
  auto place = [&](int t, int& r0, int& f0) {
    const int panel = t / (PANEL * f_tiles), in = t - panel * PANEL * f_tiles;
    const int high = min(PANEL, row_tiles - panel * PANEL), f = in / high;
    r0 = (panel * PANEL + in - f * high) * 256;
    f0 = f * TF;
  };

  if (warp >= 8) {
    setmaxnreg_dec<CONTROL_REGS>();
    if (warp == 8) {
      // ---------------- copies (both CTAs)
      const bool issuer = elect_one();
      uint32_t armed = 0, par = 0;
      bool ok = true;
      int st = 0;
      uint32_t ph = 0;
      const uint32_t full0 = mapa_shared(smem_u32(full), 0);
      for (int t = blockIdx.x >> 1; ok && t < tiles; t += step) {
        int r0, f0;
        place(t, r0, f0);
        const CUtensorMap* tm_w = GATED && rank ? &tm_w1 : &tm_w0;
        const int fw = GATED ? f0 : f0 + 128 * static_cast<int>(rank), rw = r0 + 128 * static_cast<int>(rank);
        for (int kb = 0; kb < p.kblocks; ++kb) {
          if (!mbar_wait_warp(&empty[st], ph ^ 1u, abort_flag, err, DEV_TIMEOUT_GEMM + 256 * 16)) {
            ok = false;
            break;
          }
          if (issuer) {
            unsigned char* dst = smem + st * MANY_STAGE;
            if (leader) mbar_arrive_expect_tx(&full[st], 2 * MANY_STAGE);
            tma_load_2d_pair(dst, &tm_a, full0 + 8u * st, kb * BK, rw);
            tma_load_2d_pair(dst + PIECE, tm_w, full0 + 8u * st, kb * BK, fw);
          }
          __syncwarp();
          armed |= 1u << st;
          par = (par & ~(1u << st)) | (ph << st);
          if (++st == MANY_STAGES) {
            st = 0;
            ph ^= 1u;
          }
        }
      }
      if (!ok) {  // the copies in flight, before the CTA can exit
        const uint64_t g0 = globaltimer_ns();
        if (leader) {
          for (int s = 0; s < MANY_STAGES; ++s)
            if (armed >> s & 1u)
              while (!mbar_try_wait(smem_u32(&full[s]), par >> s & 1u) && globaltimer_ns() - g0 < HILO_WAIT_LIMIT_NS / 4) {
              }
        } else {
          while (globaltimer_ns() - g0 < 50000ull) {
          }
        }
      }
      __syncwarp();
    } else if (warp == 9 && leader) {
      // ---------------- products (the even CTA)
      const bool issuer = elect_one();
      constexpr uint32_t idesc = idesc_kind_f16(256, 256, 0, 0, 0);  // (format code 0 is E4M3)
      constexpr uint32_t hi = sw128_hi(1024);
      const uint32_t base = (smem_u32(smem) >> 4) + sw128_lo_lbo(16);
      int st = 0;
      uint32_t ph = 0, i = 0;
      bool ok = true;
      for (int t = blockIdx.x >> 1; ok && t < tiles; t += step) {
        for (int kb = 0; kb < p.kblocks; ++kb, ++i) {
          const uint32_t b = i & 1u;
          if (!mbar_wait_warp(&tempty[b], ((i >> 1) & 1u) ^ 1u, abort_flag, err, DEV_TIMEOUT_GEMM + 256 * 17) ||
              !mbar_wait_warp(&full[st], ph, abort_flag, err, DEV_TIMEOUT_GEMM + 256 * 18)) {
            ok = false;
            break;
          }
          tc_fence_after();
          if (issuer) {
            const uint32_t a = base + static_cast<uint32_t>(st * MANY_STAGE >> 4), w = a + (PIECE >> 4);
#pragma unroll
            for (int k = 0; k < BK / 32; ++k) umma_pair_w<true>(tmem + 256 * b, a + 2 * k, w + 2 * k, hi, idesc, k > 0 ? 1u : 0u);
            umma_commit_pair(&empty[st], 0x3);
            umma_commit_pair(&tfull[b], 0x3);
          }
          __syncwarp();
          if (++st == MANY_STAGES) {
            st = 0;
            ph ^= 1u;
          }
        }
      }
      if (issuer) umma_commit_pair(drain, 0x1);
      __syncwarp();
      const uint64_t g0 = globaltimer_ns();
      while (!mbar_try_wait(smem_u32(drain), 0u)) {
        if (globaltimer_ns() - g0 > HILO_WAIT_LIMIT_NS) {
          if (issuer) atomicExch(err, DEV_TIMEOUT_GEMM + 256 * 19);
          break;
        }
      }
      __syncwarp();
    }
  } else {
    setmaxnreg_inc<SUM_REGS>();
    // ---------------- sums: lane quarter warp % 4 (32 rows), and of both halves of the columns (gate and up) the
    // half of the warpgroup
    const int q = warp & 3, h = warp >> 2, r = 32 * q + lane;
    float* ring = reinterpret_cast<float*>(smem + MANY_SCALES) + warp * SCALES_AHEAD * MANY_SLOT;
    float* most = reinterpret_cast<float*>(smem + MANY_MOST);
    const uint32_t taddr = tmem + (static_cast<uint32_t>(32 * q) << 16) + 64 * h;
    const uint32_t tempty0 = mapa_shared(smem_u32(tempty), 0);
    uint32_t i = 0;
    bool ok = true;
    for (int t = blockIdx.x >> 1; t < tiles; t += step) {
      int r0, f0;
      place(t, r0, f0);
      const int row = r0 + 128 * static_cast<int>(rank) + r;
      const int nb = f0 >> 7, nb_last = (p.n - 1) >> 7;
      const float* ws = GATED && (lane & 1) ? p.w_scale[1] + nb * p.w_scale_ld
                                            : p.w_scale[0] + (GATED ? nb : min(nb + (lane & 1), nb_last)) * p.w_scale_ld;
      const float* as = p.a_scale + min(row, p.rows - 1);
      auto fetch = [&](int kb) {
        if (kb < p.kblocks) {
          float* slot = ring + (kb % SCALES_AHEAD) * MANY_SLOT;
          copy4(slot + lane, as + kb * p.a_scale_ld, true);
          if (lane < 2) copy4(slot + 32 + lane, ws + kb, true);
        }
        copies_commit();
      };
      __syncwarp();
      for (int kb = 0; kb < SCALES_AHEAD - 1; ++kb) fetch(kb);
      uint64_t acc[2][32];
#pragma unroll
      for (int j = 0; j < 32; ++j) acc[0][j] = acc[1][j] = 0ull;
#pragma unroll 1
      for (int kb = 0; kb < p.kblocks; ++kb, ++i) {
        __syncwarp();  // (the slot that is fetched into was read by all lanes)
        fetch(kb + SCALES_AHEAD - 1);
        const uint32_t b = i & 1u;
        if (!mbar_wait_warp(&tfull[b], (i >> 1) & 1u, abort_flag, err, DEV_TIMEOUT_GEMM + 256 * 20)) {
          ok = false;
          break;
        }
        tc_fence_after();
        float v[2][32];
        const uint32_t at = taddr + 256 * b;
        tmem_ld32(at, v[0]);
        copies_wait<SCALES_AHEAD - 1>();
        __syncwarp();
        const float* slot = ring + (kb % SCALES_AHEAD) * MANY_SLOT;
        const float s0 = slot[lane] * slot[32], s1 = slot[lane] * slot[33];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          tmem_ld_wait_regs(v[c & 1]);
          if (c < 3) {
            tmem_ld32(at + ((c + 1) >> 1) * 128 + ((c + 1) & 1) * 32, v[(c + 1) & 1]);
          } else {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(tempty0 + 8u * b);
          }
          const float s = c < 2 ? s0 : s1;
          const uint64_t s2 = f2(s, s);
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            uint64_t& o = acc[c >> 1][(c & 1) * 16 + j];
            o = f2_fma(f2(v[c & 1][2 * j], v[c & 1][2 * j + 1]), s2, o);
          }
        }
      }
      copies_wait<0>();
      if (!ok && !(GATED && p.out_type == HILO_E4M3)) break;
      // ---- the tile's rows
      const bool there = row < rows;
      if (GATED) {
        float y[64], m = 0.f;
        const int f1 = f0 + 64 * h;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          float g0, g1, u0, u1;
          f2_split(acc[0][j], g0, g1);
          f2_split(acc[1][j], u0, u1);
          const int f = f1 + 2 * j;
          const bool in = f < p.n;
          y[2 * j] = in ? activation(g0 + bias_at(p.bias[0], f), p.act) * (u0 + bias_at(p.bias[1], f)) : 0.f;
          y[2 * j + 1] = in ? activation(g1 + bias_at(p.bias[0], f + 1), p.act) * (u1 + bias_at(p.bias[1], f + 1)) : 0.f;
          m = fmaxf(m, fmaxf(fabsf(y[2 * j]), fabsf(y[2 * j + 1])));
        }
        if (p.out_type == HILO_E4M3) {
          most[128 * h + r] = m;
          // the two warps of these rows go on together or not at all
          ok = !bar_red_or(1 + q, 64, !ok);
          if (!ok) break;
          m = fmaxf(m, most[128 * (1 - h) + r]);
          named_bar_sync(1 + q, 64);  // (read before the next tile's are written)
          float inv, sc;
          block_scale(m, inv, sc);
          if (there) {
            uint8_t* dst = static_cast<uint8_t*>(p.out) + row * p.out_row + f1;
#pragma unroll
            for (int c = 0; c < 64; c += 16)
              if (f1 + c < p.n) {
                const uint2 lo = block_codes(y + c, inv), hi = block_codes(y + c + 8, inv);
                *reinterpret_cast<uint4*>(dst + c) = make_uint4(lo.x, lo.y, hi.x, hi.y);
              }
            if (h == 0) p.out_scale[nb * p.out_scale_ld + row] = sc;
          }
        } else if (there) {
#pragma unroll
          for (int c = 0; c < 64; c += 4)
            if (f1 + c < p.n) store4(p.out, p.out_type, row * p.out_row + f1 + c, y + c);
        }
      } else if (there) {
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int c = 0; c < 64; c += 4) {
            const int f = f0 + 128 * g + 64 * h + c;
            if (f >= p.n) continue;
            float y[4];
            f2_split(acc[g][c / 2], y[0], y[1]);
            f2_split(acc[g][c / 2 + 1], y[2], y[3]);
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] += bias_at(p.bias[0], f + j);
            store4(p.out, p.out_type, row * p.out_row + f, y);
          }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync();  // no remote arrivals / copies into the peer after this point
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 512);
  }
}

// --------------------------------------------------------------------- launch --

bool encode(CUtensorMap* m, const void* base, long long rows, long long k, long long row, int box) {
  return encode_tmap_2d(m, TMAP_U8, base, static_cast<uint64_t>(k), static_cast<uint64_t>(rows), static_cast<uint64_t>(row),
                        BK, static_cast<uint32_t>(box));
}

template <int NT, bool GATED>
cudaError_t launch_few(const Gemm128Args& a, const Params128& p, int split, cudaStream_t st) {
  using C = Few<NT, GATED>;
  CUtensorMap ta, tw[2];
  const hilo_gemm128_shape& s = a.s;
  if (!encode(&ta, a.a, s.rows, s.k, s.a_row, NT)) return cudaErrorInvalidValue;
  for (int g = 0; g < C::PARTS; ++g)
    if (!encode(&tw[g], a.w[g], s.n, s.k, s.w_row, 128)) return cudaErrorInvalidValue;
  if (!GATED) tw[1] = tw[0];
  auto* kern = few128_kernel<NT, GATED>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM_BYTES);
  if (e != cudaSuccess) return e;
  const dim3 grid(static_cast<unsigned>((s.n + 127) / 128 * split), static_cast<unsigned>((s.rows + NT - 1) / NT));
  return launch_pdl_cluster(kern, split, grid, dim3(FEW_THREADS), C::SMEM_BYTES, st, ta, tw[0], tw[1], p, split);
}

template <bool GATED>
int resident_pairs(int device, int num_sms) {
  static PerDevice pairs;
  const int n = pairs.get(device, [&] {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * (num_sms / 2), 1, 1);
    cfg.blockDim = dim3(MANY_THREADS, 1, 1);
    cfg.dynamicSmemBytes = MANY_SMEM;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int found = 0;
    if (cudaOccupancyMaxActiveClusters(&found, many128_kernel<GATED>, &cfg) != cudaSuccess) {
      cudaGetLastError();
      found = 0;
    }
    return found;
  });
  return n > 0 ? n : num_sms / 2;
}

template <bool GATED>
cudaError_t launch_many(const Gemm128Args& a, const Params128& p, int device, int num_sms, cudaStream_t st) {
  CUtensorMap ta, tw[2];
  const hilo_gemm128_shape& s = a.s;
  if (!encode(&ta, a.a, s.rows, s.k, s.a_row, 128)) return cudaErrorInvalidValue;
  for (int g = 0; g < (GATED ? 2 : 1); ++g)
    if (!encode(&tw[g], a.w[g], s.n, s.k, s.w_row, 128)) return cudaErrorInvalidValue;
  if (!GATED) tw[1] = tw[0];
  auto* kern = many128_kernel<GATED>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, MANY_SMEM);
  if (e != cudaSuccess) return e;
  // the register split must fit what the CTA is launched with (setmaxnreg.inc would wait forever)
  static std::atomic<int> known{0};
  int regs = known.load(std::memory_order_relaxed);
  if (regs == 0) {
    cudaFuncAttributes fa;
    e = cudaFuncGetAttributes(&fa, kern);
    if (e != cudaSuccess) return e;
    regs = fa.numRegs;
    known.store(regs, std::memory_order_relaxed);
  }
  if (static_cast<long long>(regs) * MANY_THREADS < 256LL * SUM_REGS + 128LL * CONTROL_REGS) return cudaErrorInvalidConfiguration;
  const long long tiles = static_cast<long long>((s.rows + 255) / 256) * ((s.n + (GATED ? 127 : 255)) / (GATED ? 128 : 256));
  if (tiles > 0x7fffffff / 2) return cudaErrorInvalidValue;
  const int pairs = resident_pairs<GATED>(device, num_sms);
  return launch_pdl_cluster(kern, 1, dim3(2 * static_cast<unsigned>(tiles < pairs ? tiles : pairs)), dim3(MANY_THREADS), MANY_SMEM,
                            st, ta, tw[0], tw[1], p);
}

template <bool GATED>
cudaError_t launch_kind(const Gemm128Args& a, const Params128& p, int device, int num_sms, cudaStream_t st) {
  const int rows = a.s.rows;
  if (rows > 512) return launch_many<GATED>(a, p, device, num_sms, st);
  const int nt = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  // as many CTAs along K as fill the device
  const long long tiles = static_cast<long long>((a.s.n + 127) / 128) * ((rows + nt - 1) / nt);
  int split = 1;
  while (2 * split <= FEW_SPLIT && 2 * split <= p.kblocks && tiles * split < num_sms) split *= 2;
  switch (nt) {
    case 16: return launch_few<16, GATED>(a, p, split, st);
    case 32: return launch_few<32, GATED>(a, p, split, st);
    case 64: return launch_few<64, GATED>(a, p, split, st);
    default: return launch_few<128, GATED>(a, p, split, st);
  }
}

}  // namespace

cudaError_t launch_gemm128(const Gemm128Args& a, int device, int num_sms, cudaStream_t st) {
  Params128 p;
  const hilo_gemm128_shape& s = a.s;
  const bool two = s.act != HILO_ACT_NONE;
  p.a_scale = a.a_scale;
  for (int g = 0; g < 2; ++g) {
    p.w_scale[g] = a.w_scale[g];
    p.bias[g] = static_cast<const __nv_bfloat16*>(a.bias[g]);
  }
  p.n_rows = a.n_rows;
  p.out = a.out;
  p.out_scale = a.out_scale;
  p.a_scale_ld = s.a_scale_ld;
  p.w_scale_ld = s.w_scale_ld;
  p.out_row = s.out_row;
  p.out_scale_ld = s.out_scale_ld;
  p.rows = s.rows;
  p.n = s.n;
  p.kblocks = (s.k + BK - 1) / BK;
  p.out_type = s.out_dtype;
  p.act = s.act;
  p.out_wide = 0;
  return two ? launch_kind<true>(a, p, device, num_sms, st) : launch_kind<false>(a, p, device, num_sms, st);
}

int gemm128_take_device_error() {
  int v = 0, z = 0;
  if (cudaMemcpyFromSymbol(&v, g_gemm128_err, sizeof(int)) != cudaSuccess) return -1;
  if (v) cudaMemcpyToSymbol(g_gemm128_err, &z, sizeof(int));
  return v;
}

}  // namespace hilo
