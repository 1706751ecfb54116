// Products of e4m3 rows and weights with an fp32 scale for each block of 128, and
// the gated feed-forward's first half built on them (hilo_gemm_e4m3_128,
// hilo_gated_e4m3_128, include/hilo.h; paper Sec. 3.3 reports FP8 on top of
// HiLo-Token, the scaling scheme is the library's):
//   y[r][n] = sum_b sa[b][r] sw[n / 128][b] sum_{k in block b} a[r][k] w[n][k]   (+ bias)
//   h[r][n] = act(gate[r][n]) * up[r][n],   gate and up two such products of the same rows.
//
// The scales change along K, so the tensor core cannot sum past a block: it forms each block's product of 128 (four
// tcgen05.mma kind::f8f6f4) in a tensor memory buffer of its own, and other warps add it, scaled, to sums
// in their registers while the next block's is formed. The codes' products are exact in fp32.
//
// Two kernels, chosen by cost (gemm128_choice.h):
//   few128   few rows: features on the lanes (M), rows on the columns (N = NT). A CTA has 128 features; a cluster of up
//            to eight shares them along K and adds its sums up through distributed shared memory in a fixed order.
//            Bound by reading the weights, and for small ones by a launch and the chain first copy, product, sums,
//            cluster, rows (about 4 us).
//   many128  CTA pairs (cta_group::2): 256 rows on the lanes, NT columns: features, or half of them gate and half up;
//            a persistent grid. Bound by the chain product, sums, next product in the same buffer, of which tensor memory
//            holds 512 / NT (a block takes 780 cycles with 256 columns, its product 512), by a tile's rows, which leave while
//            the tensor core waits (2 to 3 us a tile), and at full load by the chip's power besides: 4864 rows of 16384, 4096
//            features 224 to 239 us, 2.7 to 2.9 PFLOP/s, 71 to 76% of twice the measured bf16 rate; of 4096 columns the tensor pipe
//            is active 51% of the time.
//
// Every mbarrier wait is bounded (error latched, TMEM freed, CTA returns).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "attn_common.cuh"
#include "common.cuh"
#include "e4m3_128.cuh"
#include "gemm128_choice.h"
#include "internal.h"

namespace hilo {

__device__ int g_gemm128_err;

namespace {

constexpr int BK = 128;  // K of a stage: a block, a 128-byte swizzled row
constexpr int PIECE = GEMM128_PIECE;  // bytes of 128 rows of a stage

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

// Whether the phase is complete, without waiting for it (try_wait may stay for microseconds).
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}

// Arrivals of lane 0, without a branch, on a barrier of the cluster and on one of this CTA. The first says only that
// tensor memory was read, which tcgen05.wait::ld and tcgen05's fences order. (One that releases the thread's other
// memory accesses to the cluster waits for all of them: 8192 rows of 10240, 4096 features, 718 us and 337 so.)
__device__ __forceinline__ void arrive2_lane0(uint32_t cluster_addr, uint32_t addr, int lane) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.eq.u32 p, %2, 0;\n\t"
      "@p mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];\n\t"
      "@p mbarrier.arrive.shared::cta.b64 _, [%1];\n\t}" ::"r"(cluster_addr),
      "r"(addr), "r"(lane)
      : "memory");
}

// ----------------------------------------------------------------- scales --
// One warp copies each block's scales, of the rows and of the weights' parts, into a ring of SLOTS slots in
// shared memory, asynchronously and four bytes at a time, so that any row offset will do; the copies arrive on
// the slot's barrier themselves. (4864 rows of 16384, 4096 features: 431 us where the sums' warps loaded their scales
// four blocks ahead, 270 where one warp loaded two blocks' and then wrote them: its loads' latency.)
constexpr int SLOTS = 8;

struct ScaleRing {
  float* slots;
  uint64_t *full, *empty;  // [SLOTS]: copied (an arrival per lane); read by the sums' warps
  int size;                // floats of a slot
};

__device__ __forceinline__ void copy4(void* dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copies_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// A slot: the scales of ROWS rows (0 behind `rows`), then the weights' PARTS. as, ws: of the first block; as is this lane's.
template <int ROWS, int PARTS>
__device__ __forceinline__ bool fill_scales(const ScaleRing& ring, uint32_t& n, int nkb, int rows, const float* as, long long a_step,
                                            const float* w0, const float* w1, const float* w2, volatile int* abort_flag, int* err,
                                            int code) {
  const int lane = lane_id();
  const float* ws = lane == 0 ? w0 : lane == 1 ? w1 : w2;
  for (int i = 0; i < nkb; ++i, ++n) {
    const uint32_t k = n % SLOTS;
    if (!mbar_wait_warp(&ring.empty[k], ((n / SLOTS) & 1u) ^ 1u, abort_flag, err, code)) return false;
    float* to = ring.slots + k * ring.size;
#pragma unroll
    for (int j = 0; j < ROWS; j += 32)
      if (ROWS >= 32 || lane < ROWS) copy4(to + j + lane, j + lane < rows ? as + j : w0, j + lane < rows);
    if (lane < PARTS) copy4(to + ROWS + lane, ws, true);
    copies_arrive(&ring.full[k]);
    as += a_step;
    ++ws;
  }
  return true;
}

// The warp's number, known to be the same for its lanes: addresses in tensor memory and of barriers then take one register a
// warp (8192 rows of 4096, 10240 features gated 619 us, 581 so; one row of 2048, 5504 features 7.3 and 6.9).
__device__ __forceinline__ int one_warp() { return __shfl_sync(0xffffffffu, warp_id(), 0); }

// Biases of features n and n + 1 (n even).
__device__ __forceinline__ float2 bias2(const __nv_bfloat16* b, int n) {
  return make_float2(__bfloat162float(__ldg(b + n)), __bfloat162float(__ldg(b + n + 1)));
}

__device__ __forceinline__ void st_32bytes(void* p, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
               "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "l"(p)
               : "memory");
}
// 32 bytes of a lane's own row: a whole sector where the row begins on one.
__device__ __forceinline__ void store32(void* p, const uint32_t* w, bool wide) {
  if (wide) {
    st_32bytes(p, w);
  } else {
    reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}
// 16 values of a row, rounded once (fp16 saturating).
__device__ __forceinline__ void store16(void* out, int type, long long at, const float* v, bool wide) {
  uint32_t w[8];
  if (type == HILO_F32) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[8 * h + j]);
      store32(static_cast<float*>(out) + at + 8 * h, w, wide);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = type == HILO_F16 ? pack_f16x2_sat(v[2 * j], v[2 * j + 1]) : pack_bf16x2(v[2 * j], v[2 * j + 1]);
    store32(static_cast<uint16_t*>(out) + at, w, wide);
  }
}

// Where a CTA has the SM to itself: sixteen warps for the sums (four warpgroups), one each for copies, products and
// scales, and one to make a warpgroup of them; the registers of a thread, which are shared out anew.
constexpr int SUM_WARPS = 16;
constexpr int WHOLE_THREADS = 32 * (SUM_WARPS + 4);
constexpr uint32_t SUM_REGS = 112, CONTROL_REGS = 32;
constexpr int SPLIT_REGS = 32 * SUM_WARPS * SUM_REGS + 128 * CONTROL_REGS;  // what the kernel's launch must have
static_assert(SPLIT_REGS <= 65536, "registers of an SM");

// ------------------------------------------------------------------- few rows --

template <int NT, bool GATED>
struct Few {
  static constexpr int PARTS = GATED ? 2 : 1;
  static constexpr int CTAS = NT * PARTS <= 64 ? 2 : 1;  // per SM
  static constexpr int SUMS = CTAS == 2 ? 8 : SUM_WARPS;
  static constexpr int THREADS = CTAS == 2 ? 32 * (SUMS + 3) : WHOLE_THREADS;
  static constexpr int COLS = NT / (SUMS / 4);           // of a warp
  static constexpr int STEP = COLS < 16 ? COLS : 16;     // columns read at a time
  // The cluster's sums: where there is room for them beside the stages, each CTA stores its sums where they are added up
  // (PUSH); else they take its own stages' place and are fetched.
  static constexpr bool PUSH = CTAS == 2 && !GATED;  // (gated, two stages would be left: 16 rows of 4096, 10240 features, 19.3 us, 17.2 so)
  static constexpr int SUMS_BYTES = PARTS * NT * 128 * 4;
  static constexpr int STAGE = PARTS * PIECE + NT * BK;
  static constexpr int STAGES = CTAS == 2 ? (106 * 1024 - (PUSH ? SUMS_BYTES : 0)) / STAGE : (200 * 1024) / STAGE;
  static constexpr int BUFS = NT * PARTS <= 128 ? 4 : 2;  // of tensor memory
  static constexpr int NEED = BUFS * PARTS * NT;
  static constexpr uint32_t TMEM_COLS = NEED <= 64 ? 64 : NEED <= 128 ? 128 : NEED <= 256 ? 256 : 512;
  static constexpr int SLOT = NT + 4;  // floats of a block's scales
  static constexpr int OFF_SUMS = PUSH ? STAGES * STAGE : 0;
  static constexpr int OFF_BARS = STAGES * STAGE + (PUSH ? SUMS_BYTES : 0);
  static constexpr int OFF_SCALES = OFF_BARS + 384;
  static constexpr int SMEM_BYTES = OFF_SCALES + SLOTS * SLOT * 4 + 1024;
  static_assert(STAGES >= 2 && (PUSH || STAGES * STAGE >= SUMS_BYTES), "the sums take the stages' place");
  static_assert((2 * STAGES + 2 * BUFS + 2 * SLOTS + 3) * 8 <= 384, "room for the barriers");
  static_assert(SMEM_BYTES <= (CTAS == 2 ? 112 : 226) * 1024, "shared memory");
};

template <int NT, bool GATED>
__global__ void __launch_bounds__(Few<NT, GATED>::THREADS, Few<NT, GATED>::CTAS)
    few128_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w0,
                  const __grid_constant__ CUtensorMap tm_w1, const __grid_constant__ Params128 p, int split) {
  using C = Few<NT, GATED>;
  constexpr int COPY_WARP = C::SUMS, MMA_WARP = C::SUMS + 1, SCALE_WARP = C::SUMS + 2;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::OFF_BARS);
  uint64_t* empty = full + C::STAGES;
  uint64_t* tfull = empty + C::STAGES;
  uint64_t* tempty = tfull + C::BUFS;
  const ScaleRing ring = {reinterpret_cast<float*>(smem + C::OFF_SCALES), tempty + C::BUFS, tempty + C::BUFS + SLOTS, C::SLOT};
  uint64_t* drain = ring.empty + SLOTS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* err = &g_gemm128_err;
  const int warp = one_warp(), lane = lane_id();

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < C::BUFS; ++b) {
      mbar_init(&tfull[b], 1);
      mbar_init(&tempty[b], C::SUMS);
    }
    for (int k = 0; k < SLOTS; ++k) {
      mbar_init(&ring.full[k], 32);
      mbar_init(&ring.empty[k], C::SUMS);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == COPY_WARP && lane == 0) {
    tma_prefetch_desc(&tm_a);
    tma_prefetch_desc(&tm_w0);
    if (GATED) tma_prefetch_desc(&tm_w1);
  }
  if (warp == MMA_WARP) {
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
  // The first rows' copies do not wait for the row count (most of a microsecond). The whole cluster has the same rows.
  if (blockIdx.y > 0 && rows_there(p.n_rows, p.rows) <= r0) {
    if (warp == MMA_WARP) tmem_dealloc(tmem, C::TMEM_COLS);
    return;
  }
  if (C::PUSH && split > 1) cluster_arrive_relaxed();  // this CTA has begun: the others may store into it
  const int kb0 = static_cast<int>(static_cast<long long>(p.kblocks) * rank / split);
  const int nkb = static_cast<int>(static_cast<long long>(p.kblocks) * (rank + 1) / split) - kb0;

  if (C::CTAS == 1 && warp >= C::SUMS) setmaxnreg_dec<CONTROL_REGS>();
  if (warp == COPY_WARP) {
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
  } else if (warp == MMA_WARP) {
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
  } else if (warp == SCALE_WARP) {
    // ---------------- scales (of the rows that the buffers have: more may be read than count)
    const long long w = (f0 >> 7) * p.w_scale_ld + kb0;
    uint32_t n = 0;
    fill_scales<NT, C::PARTS>(ring, n, nkb, p.rows - r0, p.a_scale + kb0 * p.a_scale_ld + r0 + lane, p.a_scale_ld, p.w_scale[0] + w,
                              p.w_scale[C::PARTS - 1] + w, nullptr, abort_flag, err, DEV_TIMEOUT_GEMM + 256 * 22);
    copies_done();
    __syncwarp();
  } else if (warp < C::SUMS) {
    if (C::CTAS == 1) setmaxnreg_inc<SUM_REGS>();
    // ---------------- sums: lane quarter warp % 4 (32 features), a part of the columns
    const int rows = min(NT, rows_there(p.n_rows, p.rows) - r0);
    const int q = warp & 3, col0 = (warp >> 2) * C::COLS;
    uint64_t acc[C::PARTS][C::COLS / 2] = {};
    const uint32_t taddr = tmem + (static_cast<uint32_t>(q * 32) << 16) + col0;
    const uint32_t ring_full = smem_u32(ring.full), tfull0 = smem_u32(tfull);
    constexpr int STEP = C::STEP, LOADS = C::PARTS * C::COLS / STEP;
    bool ok = true, there_already = false;  // block i's products and scales
#pragma unroll 1
    for (uint32_t i = 0; i < static_cast<uint32_t>(nkb); ++i) {
      const uint32_t b = i % C::BUFS, k = i % SLOTS;
      if (!there_already && (!mbar_wait_warp(&ring.full[k], (i / SLOTS) & 1u, abort_flag, err, DEV_TIMEOUT_GEMM + 256 * 21) ||
                             !mbar_wait_warp(&tfull[b], (i / C::BUFS) & 1u, abort_flag, err, DEV_TIMEOUT_GEMM + 256 * 15))) {
        ok = false;
        break;
      }
      tc_fence_after();
      auto column = [&](int l) { return taddr + (b * C::PARTS + l * STEP / C::COLS) * NT + l * STEP % C::COLS; };
      const float* slot = ring.slots + k * C::SLOT;
      float v[2][STEP];
      tmem_ldn<STEP>(column(0), v[0]);
#pragma unroll
      for (int l = 0; l < LOADS; ++l) {
        tmem_ld_wait_n<STEP>(v[l & 1]);
        if (l + 1 < LOADS) {
          tmem_ldn<STEP>(column(l + 1), v[(l + 1) & 1]);
        } else {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&tempty[b]);
          // asked beside the last sums: a wait takes a hundred cycles where it has nothing to wait for
          const uint32_t n = i + 1;
          there_already = __all_sync(0xffffffffu, mbar_test(ring_full + 8u * (n % SLOTS), (n / SLOTS) & 1u) &&
                                                      mbar_test(tfull0 + 8u * (n % C::BUFS), (n / C::BUFS) & 1u));
        }
        const int g = l * STEP / C::COLS, c0 = l * STEP % C::COLS;
        const uint64_t w2 = f2(slot[NT + g], slot[NT + g]);
#pragma unroll
        for (int c = 0; c < STEP; c += 4) {
          const float4 s = *reinterpret_cast<const float4*>(slot + col0 + c0 + c);
          uint64_t* o = &acc[g][(c0 + c) / 2];
          o[0] = f2_fma(f2(v[l & 1][c], v[l & 1][c + 1]), f2_mul(f2(s.x, s.y), w2), o[0]);
          o[1] = f2_fma(f2(v[l & 1][c + 2], v[l & 1][c + 3]), f2_mul(f2(s.z, s.w), w2), o[1]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&ring.empty[k]);
    }
    // The sums of row t are added up by CTA t % split: [CTA][part][t / split][feature] (PUSH), or [part][t][feature]
    // where they are fetched from, over the stages: every product has been waited for. (After a given-up wait
    // copies may still arrive there; nothing is stored then, and what is read below is not meant to be right.)
    const int shift = 31 - __clz(split), per = NT >> shift;  // (a power of two)
    const uint32_t sums = smem_u32(smem) + C::OFF_SUMS;
    if (C::PUSH && split > 1) cluster_wait();
    if (ok) {
#pragma unroll
      for (int g = 0; g < C::PARTS; ++g)
#pragma unroll
        for (int c = 0; c < C::COLS; ++c) {
          float lo, hi;
          f2_split(acc[g][c / 2], lo, hi);
          const int t = col0 + c;
          if (t >= rows) continue;
          uint32_t at = sums + ((g * NT + t) * 128 + q * 32 + lane) * 4;
          if (C::PUSH) {
            at = sums + (((rank * C::PARTS + g) * per + (t >> shift)) * 128 + q * 32 + lane) * 4;
            if (split > 1) at = mapa_shared(at, t & (split - 1));
          }
          const float x = c & 1 ? hi : lo;
          if (C::PUSH && split > 1) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(x) : "memory");
          else asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(x) : "memory");
        }
    }
    if (split > 1) cluster_sync();
    else named_bar_sync(1, 32 * C::SUMS);
    // ---- rows rank, rank + split, ..: a warp each, four features a lane, the CTAs' sums in the order of K
    const bool good = *abort_flag == 0;
    const int f = f0 + 4 * lane;
    const bool in = f < p.n;  // (n is a multiple of 16)
    auto finish = [&](int t, float (*y)[4]) {
#pragma unroll
      for (int g = 0; g < C::PARTS; ++g)
        if (p.bias[g] && in)
#pragma unroll
          for (int j = 0; j < 4; j += 2) {
            const float2 v = bias2(p.bias[g], f + j);
            y[g][j] += v.x;
            y[g][j + 1] += v.y;
          }
      if (GATED)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          y[0][j] = (p.act == HILO_ACT_SILU ? activation<HILO_ACT_SILU>(y[0][j]) : activation<HILO_ACT_GELU>(y[0][j])) * y[C::PARTS - 1][j];
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
    };
    // TOGETHER rows of a warp at a time, and of each four CTAs' sums, are on their way before the first is added
    constexpr int TOGETHER = C::PUSH ? 1 : 2;
    const int step = split * C::SUMS;
    for (int t0 = rank + split * warp; good && t0 < rows; t0 += TOGETHER * step) {
      float y[TOGETHER][C::PARTS][4] = {};
      for (int s0 = 0; s0 < split; s0 += 4) {
        float4 v[TOGETHER][4][C::PARTS];
#pragma unroll
        for (int u = 0; u < TOGETHER; ++u)
#pragma unroll
          for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int g = 0; g < C::PARTS; ++g) {
              float4& x = v[u][s][g];
              x = make_float4(0.f, 0.f, 0.f, 0.f);
              const int t = t0 + u * step;
              if (s0 + s >= split || t >= rows) continue;
              if (C::PUSH) {
                const uint32_t at = sums + ((((s0 + s) * C::PARTS + g) * per + (t >> shift)) * 128 + 4 * lane) * 4;
                asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(at) : "memory");
              } else {
                const uint32_t at = mapa_shared(sums + ((g * NT + t) * 128 + 4 * lane) * 4, s0 + s);
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                             : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w)
                             : "r"(at)
                             : "memory");
              }
            }
#pragma unroll
        for (int u = 0; u < TOGETHER; ++u)
#pragma unroll
          for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int g = 0; g < C::PARTS; ++g) {
              y[u][g][0] += v[u][s][g].x;
              y[u][g][1] += v[u][s][g].y;
              y[u][g][2] += v[u][s][g].z;
              y[u][g][3] += v[u][s][g].w;
            }
      }
#pragma unroll
      for (int u = 0; u < TOGETHER; ++u)
        if (t0 + u * step < rows) finish(t0 + u * step, y[u]);
    }
  }
  // (the other warps come to the cluster's meetings, too)
  if (split > 1 && warp >= C::SUMS) {
    if (C::PUSH) cluster_wait();
    cluster_sync();
  }
  tc_fence_before();
  __syncthreads();
  if (!C::PUSH && split > 1) cluster_sync();  // no CTA leaves while another fetches its sums
  if (warp == MMA_WARP) {
    tc_fence_after();
    tmem_dealloc(tmem, C::TMEM_COLS);
  }
}

// ------------------------------------------------------------------ many rows --

constexpr int MANY_SMEM = 222 * 1024;

// A pair's tile: 256 rows, NT columns of the product: NT features, or NT / 2 of gate and NT / 2 of up.
template <int NT, bool GATED>
struct Many {
  static constexpr int TF = GATED ? NT / 2 : NT;     // features
  static constexpr int STAGE = PIECE + NT / 2 * BK;  // 128 rows, and half of the columns
  static constexpr int BUFS = 512 / NT;              // of tensor memory
  // The columns' parts, each with one scale of the weights (gate and up; halves; of 192 columns, whose tiles begin anywhere
  // on 64, thirds).
  static constexpr int PARTS = NT == 192 ? 3 : 2, SPAN = NT / PARTS;
  static constexpr int COLS = SPAN / 4;              // of a warp, in each part
  static_assert(128 % SPAN == 0 && (!GATED || PARTS == 2), "a scale for each part");
  static constexpr int LOAD = 16;                    // columns read at a time, into one of two sets of registers
  static constexpr int SLOT = 128 + 4;                      // floats of a block's scales: its rows', the weights' parts'
  static constexpr int SCALES_BYTES = SLOTS * SLOT * 4, MOST_BYTES = 4 * 128 * 4;  // [4][128] row maxima
  static constexpr int STAGES = (MANY_SMEM - 1024 - 384 - SCALES_BYTES - MOST_BYTES) / STAGE;
  static constexpr int OFF_BARS = STAGES * STAGE, OFF_SCALES = OFF_BARS + 384, OFF_MOST = OFF_SCALES + SCALES_BYTES;
  static_assert(OFF_MOST + MOST_BYTES + 1024 <= MANY_SMEM, "shared memory of a CTA");
  static_assert((2 * STAGES + 2 * BUFS + 2 * SLOTS + 3) * 8 <= 384, "room for the barriers");
};
constexpr int PANEL = 8;  // row tiles that are taken together along the features

template <int NT, bool GATED>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(WHOLE_THREADS, 1)
    many128_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w0,
                   const __grid_constant__ CUtensorMap tm_w1, const __grid_constant__ Params128 p) {
  using C = Many<NT, GATED>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::OFF_BARS);
  uint64_t* empty = full + C::STAGES;
  uint64_t* tfull = empty + C::STAGES;
  uint64_t* tempty = tfull + C::BUFS;
  const ScaleRing ring = {reinterpret_cast<float*>(smem + C::OFF_SCALES), tempty + C::BUFS, tempty + C::BUFS + SLOTS, C::SLOT};
  uint64_t* drain = ring.empty + SLOTS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* err = &g_gemm128_err;
  const int warp = one_warp(), lane = lane_id();
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < C::BUFS; ++b) {
      mbar_init(&tfull[b], 1);
      mbar_init(&tempty[b], 2 * SUM_WARPS);
    }
    for (int k = 0; k < SLOTS; ++k) {
      mbar_init(&ring.full[k], 32);
      mbar_init(&ring.empty[k], SUM_WARPS);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == SUM_WARPS && lane == 0) {
    tma_prefetch_desc(&tm_a);
    tma_prefetch_desc(&tm_w0);
    tma_prefetch_desc(&tm_w1);
  }
  if (warp == SUM_WARPS + 1) {
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
  constexpr int TF = C::TF;
  const int rows = rows_there(p.n_rows, p.rows);
  const int row_tiles = (rows + 255) / 256, f_tiles = (p.n + TF - 1) / TF;
  const int tiles = row_tiles * f_tiles, step = gridDim.x >> 1;
  auto place = [&](int t, int& r0, int& f0) {
    const int panel = t / (PANEL * f_tiles), in = t - panel * PANEL * f_tiles;
    const int high = min(PANEL, row_tiles - panel * PANEL), f = in / high;
    r0 = (panel * PANEL + in - f * high) * 256;
    f0 = f * TF;
  };

  if (warp >= SUM_WARPS) {
    setmaxnreg_dec<CONTROL_REGS>();
    if (warp == SUM_WARPS) {
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
        const int fw = GATED ? f0 : f0 + NT / 2 * static_cast<int>(rank), rw = r0 + 128 * static_cast<int>(rank);
        for (int kb = 0; kb < p.kblocks; ++kb) {
          if (!mbar_wait_warp(&empty[st], ph ^ 1u, abort_flag, err, DEV_TIMEOUT_GEMM + 256 * 16)) {
            ok = false;
            break;
          }
          if (issuer) {
            unsigned char* dst = smem + st * C::STAGE;
            if (leader) mbar_arrive_expect_tx(&full[st], 2 * C::STAGE);
            tma_load_2d_pair(dst, &tm_a, full0 + 8u * st, kb * BK, rw);
            tma_load_2d_pair(dst + PIECE, tm_w, full0 + 8u * st, kb * BK, fw);
          }
          __syncwarp();
          armed |= 1u << st;
          par = (par & ~(1u << st)) | (ph << st);
          if (++st == C::STAGES) {
            st = 0;
            ph ^= 1u;
          }
        }
      }
      if (!ok) {  // the copies in flight, before the CTA can exit
        const uint64_t g0 = globaltimer_ns();
        if (leader) {
          for (int s = 0; s < C::STAGES; ++s)
            if (armed >> s & 1u)
              while (!mbar_try_wait(smem_u32(&full[s]), par >> s & 1u) && globaltimer_ns() - g0 < HILO_WAIT_LIMIT_NS / 4) {
              }
        } else {
          while (globaltimer_ns() - g0 < 50000ull) {
          }
        }
      }
      __syncwarp();
    } else if (warp == SUM_WARPS + 1 && leader) {
      // ---------------- products (the even CTA)
      const bool issuer = elect_one();
      constexpr uint32_t idesc = idesc_kind_f16(256, NT, 0, 0, 0);  // (format code 0 is E4M3)
      constexpr uint32_t hi = sw128_hi(1024);
      const uint32_t base = (smem_u32(smem) >> 4) + sw128_lo_lbo(16);
      int st = 0;
      uint32_t ph = 0, i = 0;
      bool ok = true;
      for (int t = blockIdx.x >> 1; ok && t < tiles; t += step) {
        for (int kb = 0; kb < p.kblocks; ++kb, ++i) {
          const uint32_t b = i % C::BUFS;
          if (!mbar_wait_warp(&full[st], ph, abort_flag, err, DEV_TIMEOUT_GEMM + 256 * 17)) {
            ok = false;
            break;
          }
          if (!mbar_wait_warp(&tempty[b], ((i / C::BUFS) & 1u) ^ 1u, abort_flag, err, DEV_TIMEOUT_GEMM + 256 * 18)) {
            ok = false;
            break;
          }
          tc_fence_after();
          if (issuer) {
            const uint32_t a = base + static_cast<uint32_t>(st * C::STAGE >> 4), w = a + (PIECE >> 4);
#pragma unroll
            for (int k = 0; k < BK / 32; ++k) umma_pair_w<true>(tmem + NT * b, a + 2 * k, w + 2 * k, hi, idesc, k > 0 ? 1u : 0u);
            umma_commit_pair(&tfull[b], 0x3);
            umma_commit_pair(&empty[st], 0x3);
          }
          __syncwarp();
          if (++st == C::STAGES) {
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
    } else if (warp == SUM_WARPS + 2) {
      // ---------------- scales of this CTA's rows and the tile's two parts of the features
      uint32_t n = 0;
      for (int t = blockIdx.x >> 1; t < tiles; t += step) {
        int r0, f0;
        place(t, r0, f0);
        const int row = r0 + 128 * static_cast<int>(rank);
        const float* w0 = p.w_scale[0] + (f0 >> 7) * p.w_scale_ld;
        auto later = [&](int g) { return p.w_scale[0] + (min(f0 + g * C::SPAN, p.n - 1) >> 7) * p.w_scale_ld; };
        const float* w1 = GATED ? p.w_scale[1] + (f0 >> 7) * p.w_scale_ld : later(1);
        if (!fill_scales<128, C::PARTS>(ring, n, p.kblocks, rows - row, p.a_scale + row + lane, p.a_scale_ld, w0, w1, later(2), abort_flag,
                                        err, DEV_TIMEOUT_GEMM + 256 * 24))
          break;
      }
      copies_done();
      __syncwarp();
    }
  } else {
    setmaxnreg_inc<SUM_REGS>();
    // ---------------- sums: lane quarter warp % 4 (32 rows), and of each part of the columns the quarter warp / 4
    const int q = warp & 3, h = warp >> 2, r = 32 * q + lane;
    float* most = reinterpret_cast<float*>(smem + C::OFF_MOST);
    const uint32_t taddr = tmem + (static_cast<uint32_t>(32 * q) << 16) + C::COLS * h;
    const uint32_t tempty0 = mapa_shared(smem_u32(tempty), 0), tfull0 = smem_u32(tfull);
    const uint32_t ring_full = smem_u32(ring.full), ring_empty = smem_u32(ring.empty);
    uint32_t i = 0;
    bool ok = true, there_already = false;  // block i's products and scales
    for (int t = blockIdx.x >> 1; t < tiles; t += step) {
      int r0, f0;
      place(t, r0, f0);
      const int row = r0 + 128 * static_cast<int>(rank) + r;
      uint64_t acc[C::PARTS][C::COLS / 2];
#pragma unroll
      for (int j = 0; j < C::PARTS * C::COLS / 2; ++j) acc[j / (C::COLS / 2)][j % (C::COLS / 2)] = 0ull;
#pragma unroll 1
      for (int kb = 0; kb < p.kblocks; ++kb, ++i) {
        if (!there_already) {
          const uint32_t b = i % C::BUFS, k = i % SLOTS;
          if (!mbar_wait_warp(&ring.full[k], (i / SLOTS) & 1u, abort_flag, err, DEV_TIMEOUT_GEMM + 256 * 23) ||
              !mbar_wait_warp(&tfull[b], (i / C::BUFS) & 1u, abort_flag, err, DEV_TIMEOUT_GEMM + 256 * 20)) {
            ok = false;
            break;
          }
        }
        tc_fence_after();
        const uint32_t at = taddr + (i % C::BUFS) * NT;
        const float* slot = ring.slots + i % SLOTS * C::SLOT;
        constexpr int LOADS = C::PARTS * C::COLS / C::LOAD;  // part by part
        auto column = [&](int c) { return at + (c * C::LOAD / C::COLS) * C::SPAN + c * C::LOAD % C::COLS; };
        float v[2][C::LOAD];
        tmem_ldn<C::LOAD>(column(0), v[0]);
        float sc[C::PARTS];
#pragma unroll
        for (int g = 0; g < C::PARTS; ++g) sc[g] = slot[r] * slot[128 + g];
#pragma unroll
        for (int c = 0; c < LOADS; ++c) {
          tmem_ld_wait_n<C::LOAD>(v[c & 1]);
          if (c + 1 < LOADS) {
            tmem_ldn<C::LOAD>(column(c + 1), v[(c + 1) & 1]);
          } else {
            tc_fence_before();
            __syncwarp();
            arrive2_lane0(tempty0 + 8u * (i % C::BUFS), ring_empty + 8u * (i % SLOTS), lane);
            // asked beside the last sums: a wait takes a hundred cycles where it has nothing to wait for
            const uint32_t n = i + 1;
            there_already = __all_sync(0xffffffffu, mbar_test(ring_full + 8u * (n % SLOTS), (n / SLOTS) & 1u) &&
                                                        mbar_test(tfull0 + 8u * (n % C::BUFS), (n / C::BUFS) & 1u));
          }
          const int g = c * C::LOAD / C::COLS, c0 = c * C::LOAD % C::COLS;
          const uint64_t s2 = f2(sc[g], sc[g]);
#pragma unroll
          for (int j = 0; j < C::LOAD; j += 2) {
            uint64_t& o = acc[g][(c0 + j) / 2];
            o = f2_fma(f2(v[c & 1][j], v[c & 1][j + 1]), s2, o);
          }
        }
      }
      if (!ok && !(GATED && NT == 256 && p.out_type == HILO_E4M3)) break;
      // ---- the tile's rows
      const bool there = row < rows;
      // part g's features of this thread, from f on
      auto feature = [&](int g) { return f0 + (GATED ? 0 : C::SPAN * g) + C::COLS * h; };
#pragma unroll
      for (int g = 0; g < C::PARTS; ++g)
        if (const __nv_bfloat16* bias = p.bias[GATED ? g : 0]) {
#pragma unroll
          for (int j = 0; j < C::COLS; j += 2)
            if (feature(g) + j < p.n) {
              const float2 v = bias2(bias, feature(g) + j);
              acc[g][j / 2] = f2_add(acc[g][j / 2], f2(v.x, v.y));
            }
        }
      if (GATED) {
        const int f = feature(0);
        float y[C::COLS], m = 0.f;
        auto combine = [&](auto act) {
#pragma unroll
          for (int j = 0; j < C::COLS; j += 2) {
            float g0, g1, u0, u1;
            f2_split(acc[0][j / 2], g0, g1);
            f2_split(acc[1][j / 2], u0, u1);
            y[j] = activation<decltype(act)::value>(g0) * u0;
            y[j + 1] = activation<decltype(act)::value>(g1) * u1;
            m = fmaxf(m, fmaxf(fabsf(y[j]), fabsf(y[j + 1])));  // (features that are not there are 0)
          }
        };
        if (p.act == HILO_ACT_SILU) combine(Act<HILO_ACT_SILU>());
        else combine(Act<HILO_ACT_GELU>());
        if (NT == 256 && p.out_type == HILO_E4M3) {  // (a tile's features are a block)
          most[128 * h + r] = m;
          // the four warps of these rows go on together or not at all
          ok = !bar_red_or(1 + q, 128, !ok);
          if (!ok) break;
#pragma unroll
          for (int o = 0; o < 4; ++o) m = fmaxf(m, most[128 * o + r]);
          named_bar_sync(1 + q, 128);  // (read before the next tile's are written)
          float inv, sc;
          block_scale(m, inv, sc);
          if (there) {
            const int nb = f0 >> 7;
            uint8_t* dst = static_cast<uint8_t*>(p.out) + row * p.out_row + f;
            uint32_t w[8] = {};
#pragma unroll
            for (int j = 0; j < C::COLS; j += 8) {
              const uint2 c = block_codes(y + j, inv);
              w[j / 4] = c.x;
              w[j / 4 + 1] = c.y;
            }
            if (f + 16 < p.n)
              store32(dst, w, p.out_wide);
            else if (f < p.n)
              *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
            if (h == 0) p.out_scale[nb * p.out_scale_ld + row] = sc;
          }
        } else if (there) {
#pragma unroll
          for (int c = 0; c < C::COLS; c += 16)
            if (f + c < p.n) store16(p.out, p.out_type, row * p.out_row + f + c, y + c, p.out_wide);
        }
      } else if (there) {
#pragma unroll
        for (int g = 0; g < C::PARTS; ++g)
#pragma unroll
          for (int c = 0; c < C::COLS; c += 16) {
            const int f = feature(g);
            if (f + c >= p.n) continue;
            float y[16];
#pragma unroll
            for (int j = 0; j < 16; j += 2) f2_split(acc[g][(c + j) / 2], y[j], y[j + 1]);
            store16(p.out, p.out_type, row * p.out_row + f + c, y, p.out_wide);
          }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync();  // no remote arrivals / copies into the peer after this point
  if (warp == SUM_WARPS + 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 512);
  }
}

// --------------------------------------------------------------------- launch --

bool encode(CUtensorMap* m, const void* base, long long rows, long long k, long long row, int box) {
  return encode_tmap_2d(m, TMAP_U8, base, static_cast<uint64_t>(k), static_cast<uint64_t>(rows), static_cast<uint64_t>(row),
                        BK, static_cast<uint32_t>(box));
}

// The register split must fit what the CTA is launched with, or setmaxnreg.inc would wait forever. (One number for every
// device: the library holds one binary.)
template <auto KERNEL>
cudaError_t registers_fit() {
  static std::atomic<int> known{0};
  int regs = known.load(std::memory_order_relaxed);
  if (regs == 0) {
    cudaFuncAttributes fa;
    const cudaError_t e = cudaFuncGetAttributes(&fa, KERNEL);
    if (e != cudaSuccess) return e;
    regs = fa.numRegs;
    known.store(regs, std::memory_order_relaxed);
  }
  return regs * WHOLE_THREADS < SPLIT_REGS ? cudaErrorInvalidConfiguration : cudaSuccess;
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
  if (C::CTAS == 1 && (e = registers_fit<few128_kernel<NT, GATED>>()) != cudaSuccess) return e;
  const dim3 grid(static_cast<unsigned>((s.n + 127) / 128 * split), static_cast<unsigned>((s.rows + NT - 1) / NT));
  return launch_pdl_cluster(kern, split, grid, dim3(C::THREADS), C::SMEM_BYTES, st, ta, tw[0], tw[1], p, split);
}

template <int NT, bool GATED>
int resident_pairs(int device, int num_sms) {
  static PerDevice pairs;
  const int n = pairs.get(device, [&] {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * (num_sms / 2), 1, 1);
    cfg.blockDim = dim3(WHOLE_THREADS, 1, 1);
    cfg.dynamicSmemBytes = MANY_SMEM;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int found = 0;
    if (cudaOccupancyMaxActiveClusters(&found, many128_kernel<NT, GATED>, &cfg) != cudaSuccess) {
      cudaGetLastError();
      found = 0;
    }
    return found;
  });
  return n > 0 ? n : num_sms / 2;
}

template <int NT, bool GATED>
cudaError_t launch_many(const Gemm128Args& a, const Params128& p, int device, int num_sms, cudaStream_t st) {
  CUtensorMap ta, tw[2];
  const hilo_gemm128_shape& s = a.s;
  if (!encode(&ta, a.a, s.rows, s.k, s.a_row, 128)) return cudaErrorInvalidValue;
  for (int g = 0; g < (GATED ? 2 : 1); ++g)
    if (!encode(&tw[g], a.w[g], s.n, s.k, s.w_row, NT / 2)) return cudaErrorInvalidValue;
  if (!GATED) tw[1] = tw[0];
  auto* kern = many128_kernel<NT, GATED>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, MANY_SMEM);
  if (e != cudaSuccess) return e;
  if ((e = registers_fit<many128_kernel<NT, GATED>>()) != cudaSuccess) return e;
  const long long tiles = static_cast<long long>((s.rows + 255) / 256) * ((s.n + Many<NT, GATED>::TF - 1) / Many<NT, GATED>::TF);
  if (tiles > 0x7fffffff / 2) return cudaErrorInvalidValue;
  const int pairs = resident_pairs<NT, GATED>(device, num_sms);
  return launch_pdl_cluster(kern, 1, dim3(2 * static_cast<unsigned>(tiles < pairs ? tiles : pairs)), dim3(WHOLE_THREADS), MANY_SMEM,
                            st, ta, tw[0], tw[1], p);
}

template <bool GATED>
cudaError_t launch_kind(const Gemm128Args& a, const Params128& p, int device, int num_sms, cudaStream_t st) {
  const Gemm128Choice c = gemm128_choice<GATED>(a.s.rows, a.s.n, p.kblocks, p.out_type == HILO_E4M3, num_sms);
  if (c.many) {
    if constexpr (!GATED)
      if (c.nt == 192) return launch_many<192, false>(a, p, device, num_sms, st);
    return c.nt == 128 ? launch_many<128, GATED>(a, p, device, num_sms, st) : launch_many<256, GATED>(a, p, device, num_sms, st);
  }
  switch (c.nt) {
    case 16: return launch_few<16, GATED>(a, p, c.split, st);
    case 32: return launch_few<32, GATED>(a, p, c.split, st);
    case 64: return launch_few<64, GATED>(a, p, c.split, st);
    default: return launch_few<128, GATED>(a, p, c.split, st);
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
  const int bytes = s.out_dtype == HILO_F32 ? 4 : s.out_dtype == HILO_E4M3 ? 1 : 2;
  p.out_wide = reinterpret_cast<uintptr_t>(a.out) % 32 == 0 && s.out_row * bytes % 32 == 0;
  return two ? launch_kind<true>(a, p, device, num_sms, st) : launch_kind<false>(a, p, device, num_sms, st);
}

int gemm128_take_device_error() {
  int v = 0, z = 0;
  if (cudaMemcpyFromSymbol(&v, g_gemm128_err, sizeof(int)) != cudaSuccess) return -1;
  if (v) cudaMemcpyToSymbol(g_gemm128_err, &z, sizeof(int));
  return v;
}

}  // namespace hilo
