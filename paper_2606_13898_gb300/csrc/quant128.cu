// Rows and weights to e4m3 codes with an fp32 scale for each block of 128
// (hilo_quantize_e4m3_128, include/hilo.h; paper Sec. 3.3 reports FP8 on top of
// HiLo-Token, the scaling scheme is the library's):
//   m = max |x| over the block,  scale = m / 448,  code = e4m3(x * (448 / m)),
// the block being 128 columns of one row, or 128 rows x 128 columns.
//
// Bound by HBM: each element is read once, stays in registers for both the
// maximum and the rounding, and leaves as one byte. Of bf16 nearly as much by the work of a block: 8192 rows of
// 4096 18.8 us (81% of a copy's rate), of fp32 26.5 (95%); one row 1.3 to 1.5.
#include "e4m3_128.cuh"
#include "internal.h"

namespace hilo {

namespace {

constexpr int THREADS = 256;

struct QuantParams {
  const unsigned char* src;
  uint8_t* dst;
  float* scale;
  const int32_t* n_rows;
  long long src_row, dst_row, scale_ld;  // src_row in bytes
  int rows, cols, blocks;                // blocks: of a row, ceil(cols / 128)
  int step_rows, step_pairs;             // THREADS / 32 pairs of blocks on
};

// A scale per row and 128 columns. A half warp has a block, eight columns a lane; a warp has
// two neighbouring blocks of a row at a time, and U of these on their way at once: four where there are more than the
// device holds at once, one otherwise (bf16 rows of 4096, one and four: 64 rows 1.57 and 2.05 us, 600 rows 2.67 and 2.68, 8192
// rows 23.7 and 19.6).
template <int TYPE, int U>
__global__ void __launch_bounds__(THREADS) quant128_rows_kernel(const __grid_constant__ QuantParams p) {
  pdl_wait();
  pdl_trigger();
  const int rows = rows_there(p.n_rows, p.rows);
  const int pairs = (p.blocks + 1) >> 1, lane = lane_id(), half = lane >> 4;
  const long long total = static_cast<long long>(rows) * pairs;
  const long long first = (static_cast<long long>(blockIdx.x) * U) * (THREADS / 32) + warp_id();
  Eight<TYPE> x[U];
  int row[U], col[U];
  // the first's row and pair (a 64-bit division is as much work as the rest of a block), from there on by steps
  int at = first >> 32 ? static_cast<int>(first / pairs) : static_cast<int>(static_cast<uint32_t>(first) / static_cast<uint32_t>(pairs));
  int pair = static_cast<int>(first - static_cast<long long>(at) * pairs);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    row[u] = at;
    col[u] = first + u * (THREADS / 32) < total ? pair * 256 + lane * 8 : p.cols;
    at += p.step_rows;
    pair += p.step_pairs;
    if (pair >= pairs) {
      pair -= pairs;
      ++at;
    }
    x[u].clear();
    if (col[u] < p.cols) x[u].load_once(p.src + row[u] * p.src_row + static_cast<long long>(col[u]) * (TYPE == 2 ? 4 : 2));
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float f[8], inv, sc;
    x[u].widen(f);
    float m = amax8(f, 0.f);
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
    block_scale(m, inv, sc);
    if (col[u] >= p.cols) continue;
    *reinterpret_cast<uint2*>(p.dst + row[u] * p.dst_row + col[u]) = block_codes(f, inv);
    if (lane == 16 * half) p.scale[(col[u] >> 7) * p.scale_ld + row[u]] = sc;
  }
}

// A scale per 128 rows x 128 columns: a CTA each, all of the tile in registers, three CTAs on an SM. (10240 rows of 4096 in
// bf16 21.6 us, 5.8 TB/s; two 25.1, four as three, but of fp32 the tile spills: 32.6 us, four 41.6.)
template <int TYPE>
__global__ void __launch_bounds__(THREADS, 3) quant128_tiles_kernel(const __grid_constant__ QuantParams p) {
  pdl_wait();
  pdl_trigger();
  __shared__ float most[THREADS / 32];
  const int rows = rows_there(p.n_rows, p.rows);
  const int down = blockIdx.x / p.blocks, across = blockIdx.x - down * p.blocks;
  if (down * QBLOCK >= rows) return;
  const int col = across * QBLOCK + (threadIdx.x & 15) * 8, row0 = down * QBLOCK + (threadIdx.x >> 4);
  Eight<TYPE> x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = row0 + 16 * i;
    x[i].clear();
    if (row < rows && col < p.cols) x[i].load_once(p.src + row * p.src_row + static_cast<long long>(col) * (TYPE == 2 ? 4 : 2));
  }
  float m = 0.f, inv, sc;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float f[8];
    x[i].widen(f);
    m = amax8(f, m);
  }
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
  if (lane_id() == 0) most[warp_id()] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) m = fmaxf(m, most[w]);
  block_scale(m, inv, sc);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = row0 + 16 * i;
    float f[8];
    x[i].widen(f);
    if (row < rows && col < p.cols) *reinterpret_cast<uint2*>(p.dst + row * p.dst_row + col) = block_codes(f, inv);
  }
  if (threadIdx.x == 0) p.scale[down * p.scale_ld + across] = sc;
}

template <int TYPE>
cudaError_t launch_type(const QuantParams& p, bool tile, int num_sms, cudaStream_t st) {
  if (tile) {
    const long long tiles = static_cast<long long>((p.rows + QBLOCK - 1) / QBLOCK) * p.blocks;
    if (tiles > 0x7fffffffLL) return cudaErrorInvalidValue;
    return launch_pdl(quant128_tiles_kernel<TYPE>, dim3(static_cast<unsigned>(tiles)), dim3(THREADS), 0, st, p);
  }
  constexpr int WARPS = THREADS / 32;
  const long long chunks = static_cast<long long>(p.rows) * ((p.blocks + 1) / 2);
  const bool many = chunks > static_cast<long long>(num_sms) * 8 * WARPS;  // more than the device holds at once
  const long long per = many ? 4 * WARPS : WARPS, grid = (chunks + per - 1) / per;
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  return launch_pdl(many ? quant128_rows_kernel<TYPE, 4> : quant128_rows_kernel<TYPE, 1>, dim3(static_cast<unsigned>(grid)),
                    dim3(THREADS), 0, st, p);
}

}  // namespace

cudaError_t launch_quant128(const hilo_quant128_shape& s, const void* src, const int32_t* n_rows, uint8_t* dst, float* scale,
                            int num_sms, cudaStream_t st) {
  QuantParams p;
  p.src = static_cast<const unsigned char*>(src);
  p.dst = dst;
  p.scale = scale;
  p.n_rows = n_rows;
  p.src_row = s.src_row * (s.dtype == HILO_F32 ? 4 : 2);
  p.dst_row = s.dst_row;
  p.scale_ld = s.scale_ld;
  p.rows = s.rows;
  p.cols = s.cols;
  p.blocks = (s.cols + QBLOCK - 1) / QBLOCK;
  const int pairs = (p.blocks + 1) / 2;
  p.step_rows = THREADS / 32 / pairs;
  p.step_pairs = THREADS / 32 % pairs;
  return s.dtype == HILO_BF16 ? launch_type<0>(p, s.tile, num_sms, st)
         : s.dtype == HILO_F16 ? launch_type<1>(p, s.tile, num_sms, st)
                               : launch_type<2>(p, s.tile, num_sms, st);
}

}  // namespace hilo
