// Group norm of images, channels last, with its weights, a scale and a shift per
// image and an activation (hilo_group_norm, include/hilo.h; the levels of the image encoder
// and decoder around the block, paper Sec. 2.1):
//   y = act(((x - mean) / sqrt(var + eps) w + b) (1 + scale) + shift)
// with mean and variance over all rows of an image and the channels of a group.
//
// Statistics are pairs (mean, sum of squares about it), joined by
//   n = na + nb,  mean = (na ma + nb mb) / n,  M = Ma + Mb + na (ma - mean)^2 + nb (mb - mean)^2,
// so that no step subtracts large sums from one another. Every order is fixed.
//
// Two kernels over the same chunks of rows: the first leaves each chunk's pairs in the
// workspace, the second joins an image's pairs and writes its chunk, from the last row to the
// first, as the rows read last are the ones still in L2. Bound by HBM: x is read once, and
// again as far as it is not in L2, y is written once.
#include "e4m3_128.cuh"
#include "internal.h"

namespace hilo {

namespace {

constexpr int MAX_THREADS = 512;
constexpr int MAX_CHUNKS = 320;  // of a call, but for one per image

struct NormParams {
  const unsigned char* x;
  void* y;
  float* y_scale;
  float2* part;  // [image][chunk][group]: mean, sum of squares about it
  const void *scale, *shift, *w, *b;
  long long x_row, y_row, vec_row, y_scale_ld;  // x_row in bytes
  int rows, d, groups, per, act;                // per: channels of a group
  int y_type, vec_f32;
  int across, down;  // threads along the channels (eight each, a multiple of 16 of them), along the rows
  int passes;        // of the channels: across * passes * 8 >= d
  int chunks, chunk; // of an image, and rows of each
  float eps;
};

// Mean and sum of squares about it of n values.
struct Pair {
  float mean, sq;
};

__device__ __forceinline__ float vec_at(const void* v, int f32, long long i, float none) {
  if (!v) return none;
  return f32 ? __ldg(static_cast<const float*>(v) + i) : __bfloat162float(__ldg(static_cast<const __nv_bfloat16*>(v) + i));
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  return v;
}

// Rows of a thread at a time: their mean and squares from registers, joined with what there was.
constexpr int BATCH = 8;

template <int TYPE>
__global__ void __launch_bounds__(MAX_THREADS) group_stats_kernel(const __grid_constant__ NormParams p) {
  extern __shared__ float shared[];  // [down][d] means, then [down][d] squares
  pdl_wait();
  pdl_trigger();
  const int image = blockIdx.x / p.chunks, chunk = blockIdx.x - image * p.chunks, r0 = chunk * p.chunk, r1 = min(p.rows, r0 + p.chunk);
  const int tx = threadIdx.x % p.across, ty = threadIdx.x / p.across;
  const unsigned char* x = p.x + (static_cast<long long>(image) * p.rows) * p.x_row;
  float* means = shared;
  float* squares = shared + p.down * p.d;
  constexpr int ESIZE = TYPE == 2 ? 4 : 2;
  for (int c = tx * 8; c < p.d && ty < p.down; c += p.across * 8) {
    float mean[8], sq[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) mean[j] = sq[j] = 0.f;
    int n = 0;
    for (int r = r0 + ty; r < r1; r += p.down * BATCH) {
      Eight<TYPE> e[BATCH];
      const int m = min(BATCH, (r1 - r + p.down - 1) / p.down);
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        e[i].clear();
        if (i < m) e[i].load(x + (r + i * p.down) * p.x_row + c * ESIZE);
      }
      float sum[8], two[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] = two[j] = 0.f;
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        float f[8];
        e[i].widen(f);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += f[j];  // (rows that are not there are zeros)
      }
      const float inv = __fdividef(1.f, static_cast<float>(m));
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] *= inv;
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        float f[8];
        e[i].widen(f);
        if (i < m)
#pragma unroll
          for (int j = 0; j < 8; ++j) two[j] = fmaf(f[j] - sum[j], f[j] - sum[j], two[j]);
      }
      // joined: the new mean lies wb of the way to the batch's
      const float wb = __fdividef(static_cast<float>(m), static_cast<float>(n + m));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float gap = sum[j] - mean[j];
        mean[j] = fmaf(gap, wb, mean[j]);
        sq[j] += fmaf(gap * gap, wb * static_cast<float>(n), two[j]);
      }
      n += m;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      means[ty * p.d + c + j] = mean[j];
      squares[ty * p.d + c + j] = sq[j];
    }
  }
  __syncthreads();
  // a warp per group: the pairs of its channels and of the threads along the rows
  const int lane = lane_id(), warps = blockDim.x >> 5;
  for (int g = warp_id(); g < p.groups; g += warps) {
    const int entries = p.down * p.per;
    auto each = [&](auto f) {
      for (int e = lane; e < entries; e += 32) {
        const int t = e / p.per, at = t * p.d + g * p.per + (e - t * p.per);
        const int n = max(0, (r1 - r0 - t + p.down - 1) / p.down);  // rows of thread t
        f(static_cast<float>(n), means[at], squares[at]);
      }
    };
    float sum = 0.f, sq = 0.f;
    each([&](float n, float m, float) { sum = fmaf(n, m, sum); });
    const float mean = warp_sum(sum) / (static_cast<float>(r1 - r0) * static_cast<float>(p.per));
    each([&](float n, float m, float s) { sq += n > 0.f ? fmaf(n * (m - mean), m - mean, s) : 0.f; });
    sq = warp_sum(sq);
    if (lane == 0) p.part[(static_cast<long long>(image) * p.chunks + chunk) * p.groups + g] = make_float2(mean, sq);
  }
}

template <int TYPE>
__global__ void __launch_bounds__(MAX_THREADS) group_apply_kernel(const __grid_constant__ NormParams p) {
  extern __shared__ float shared[];  // [groups] means, then [groups] 1 / deviation
  pdl_wait();
  pdl_trigger();
  const int image = blockIdx.x / p.chunks, chunk = blockIdx.x - image * p.chunks, r0 = chunk * p.chunk, r1 = min(p.rows, r0 + p.chunk);
  float* means = shared;
  float* invs = shared + p.groups;
  // the image's pairs, a warp per group
  const int lane = lane_id(), warps = blockDim.x >> 5;
  const float2* part = p.part + static_cast<long long>(image) * p.chunks * p.groups;
  for (int g = warp_id(); g < p.groups; g += warps) {
    float sum = 0.f, sq = 0.f;
    auto rows_of = [&](int k) { return static_cast<float>(min(p.rows, (k + 1) * p.chunk) - k * p.chunk); };
    for (int k = lane; k < p.chunks; k += 32) sum = fmaf(rows_of(k), part[static_cast<long long>(k) * p.groups + g].x, sum);
    const float mean = warp_sum(sum) / static_cast<float>(p.rows);
    for (int k = lane; k < p.chunks; k += 32) {
      const float2 q = part[static_cast<long long>(k) * p.groups + g];
      sq += fmaf(rows_of(k) * static_cast<float>(p.per) * (q.x - mean), q.x - mean, q.y);
    }
    const float var = warp_sum(sq) / (static_cast<float>(p.rows) * static_cast<float>(p.per));
    if (lane == 0) {
      means[g] = mean;
      invs[g] = 1.f / sqrtf(var + p.eps);
    }
  }
  __syncthreads();
  const int tx = threadIdx.x % p.across, ty = threadIdx.x / p.across;
  const long long row0 = static_cast<long long>(image) * p.rows;
  const unsigned char* x = p.x + row0 * p.x_row;
  constexpr int ESIZE = TYPE == 2 ? 4 : 2;
  // (all lanes of a half warp stay together: its 128 channels are a block of codes)
  for (int pass = 0; pass < p.passes; ++pass) {
    const int c = (tx + pass * p.across) * 8;
    const bool in = c < p.d && ty < p.down;
    float mean[8], a[8], b[8];
    if (in)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int g = (c + j) / p.per;
        const long long v = image * p.vec_row + c + j;
        const float up = 1.f + vec_at(p.scale, p.vec_f32, v, 0.f);
        mean[j] = means[g];
        a[j] = invs[g] * vec_at(p.w, p.vec_f32, c + j, 1.f) * up;
        b[j] = fmaf(vec_at(p.b, p.vec_f32, c + j, 0.f), up, vec_at(p.shift, p.vec_f32, v, 0.f));
      }
    const int n = r1 - r0, steps = (n + p.down - 1) / p.down;
    constexpr int AHEAD = 4;
    for (int s = (steps - 1) / AHEAD; s >= 0; --s) {
      Eight<TYPE> e[AHEAD];
      int row[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        row[i] = r0 + ty + (s * AHEAD + i) * p.down;
        if (!in || row[i] >= r1) row[i] = -1;
        e[i].clear();
        if (row[i] >= 0) e[i].load(x + row[i] * p.x_row + c * ESIZE);
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        float f[8];
        e[i].widen(f);
        if (in)
          with_activation(p.act, [&](auto act) {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = activation<decltype(act)::value>(fmaf(f[j] - mean[j], a[j], b[j]));
          });
        if (p.y_type == HILO_E4M3) {
          float m = row[i] >= 0 ? amax8(f, 0.f) : 0.f, inv, sc;
#pragma unroll
          for (int off = 8; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
          block_scale(m, inv, sc);
          if (row[i] < 0) continue;
          __stcs(reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.y) + (row0 + row[i]) * p.y_row + c), block_codes(f, inv));
          if ((tx & 15) == 0) p.y_scale[(c >> 7) * p.y_scale_ld + row0 + row[i]] = sc;
        } else if (row[i] >= 0) {
          store4(p.y, p.y_type, (row0 + row[i]) * p.y_row + c, f);
          store4(p.y, p.y_type, (row0 + row[i]) * p.y_row + c + 4, f + 4);
        }
      }
    }
  }
}

// Threads and chunks of a shape.
void lay_out(const hilo_group_norm_shape& s, NormParams& p) {
  const int vectors = s.d / 8, wide = (vectors + 15) / 16 * 16;
  p.across = wide < MAX_THREADS ? wide : MAX_THREADS;
  p.passes = (vectors + p.across - 1) / p.across;
  p.down = MAX_THREADS / p.across;
  if (p.down > s.rows && s.rows > 0) p.down = s.rows;
  const int most = MAX_CHUNKS / s.B > 1 ? MAX_CHUNKS / s.B : 1;
  const int unit = p.down * BATCH;
  int chunks = (s.rows + unit - 1) / unit;
  if (chunks > most) chunks = most;
  if (chunks < 1) chunks = 1;
  p.chunk = ((s.rows + chunks - 1) / chunks + p.down - 1) / p.down * p.down;
  p.chunks = p.chunk ? (s.rows + p.chunk - 1) / p.chunk : 1;
}

template <int TYPE>
cudaError_t launch_type(const NormParams& p, int B, int* launches, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>(p.chunks) * static_cast<unsigned>(B));
  const dim3 block(static_cast<unsigned>((p.across * p.down + 31) / 32 * 32));
  const size_t stats = static_cast<size_t>(p.down) * p.d * 2 * sizeof(float);
  auto* kern = group_stats_kernel<TYPE>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 72 * 1024);
  if (e != cudaSuccess) return e;
  e = launch_pdl(kern, grid, block, stats, st, p);
  if (e != cudaSuccess) return e;
  *launches = 1;
  auto* apply = group_apply_kernel<TYPE>;
  e = cudaFuncSetAttribute(apply, cudaFuncAttributeMaxDynamicSharedMemorySize, 72 * 1024);
  if (e != cudaSuccess) return e;
  e = launch_pdl(apply, grid, block, static_cast<size_t>(p.groups) * 2 * sizeof(float), st, p);
  if (e == cudaSuccess) *launches = 2;
  return e;
}

}  // namespace

size_t group_norm_workspace_bytes(const hilo_group_norm_shape& s) {
  NormParams p;
  lay_out(s, p);
  return static_cast<size_t>(s.B) * p.chunks * s.groups * sizeof(float2);
}

cudaError_t launch_group_norm(const GroupNormArgs& a, int device, int num_sms, int* launches, cudaStream_t st) {
  (void)device;
  (void)num_sms;
  *launches = 0;
  const hilo_group_norm_shape& s = a.s;
  NormParams p;
  p.x = static_cast<const unsigned char*>(a.x);
  p.y = a.y;
  p.y_scale = a.y_scale;
  p.part = static_cast<float2*>(a.ws);
  p.scale = a.vec.scale;
  p.shift = a.vec.shift;
  p.w = a.vec.w_norm;
  p.b = a.vec.b_norm;
  p.x_row = s.x_row * (s.x_dtype == HILO_F32 ? 4 : 2);
  p.y_row = s.y_row;
  p.vec_row = s.vec_row;
  p.y_scale_ld = s.y_scale_ld;
  p.rows = s.rows;
  p.d = s.d;
  p.groups = s.groups;
  p.per = s.d / s.groups;
  p.act = s.act;
  p.y_type = s.y_dtype;
  p.vec_f32 = s.vec_dtype == HILO_F32;
  p.eps = s.eps;
  lay_out(s, p);
  return s.x_dtype == HILO_BF16  ? launch_type<0>(p, s.B, launches, st)
         : s.x_dtype == HILO_F16 ? launch_type<1>(p, s.B, launches, st)
                                 : launch_type<2>(p, s.B, launches, st);
}

}  // namespace hilo
