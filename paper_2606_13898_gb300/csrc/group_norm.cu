// Group norm of images, channels last, with its weights, a scale and a shift per
// image and an activation (hilo_group_norm, include/hilo.h; the levels of the image encoder
// and decoder around the block, paper Sec. 2.1):
//   y = act(((x - mean) / sqrt(var + eps) w + b) (1 + scale) + shift)
// with mean and variance over all rows of an image and the channels of a group.
//
// Statistics are pairs (mean, sum of squares about it), joined by
//   n = na + nb,  mean = (na ma + nb mb) / n,  M = Ma + Mb + na (ma - mean)^2 + nb (mb - mean)^2,
// so that no step subtracts large sums from one another. Every order is fixed. A mean formed from a sum and a reciprocal is
// off by some ulp of an offset that all values share; what the values (or pairs) are about it sums up to that error, as they
// are read again for the squares, and is added to it. So equal values have exactly their value as their mean, and an offset costs
// one rounding a level. (With it and without, us: 1024 rows of 512 5.3 and 5.2, 8 x 82 rows of 2048 6.3 and 6.1, 3 x 1380 rows
// of 1152 to codes 10.1 and 10.0, 65536 rows of 512 42.9 and 43.3, in 512 groups 58.5 and 56.4.)
//
// Images whose slices of channels (whole groups) fit the shared memory of a cluster: one kernel
// (group_norm_kernel). A CTA copies its rows of the slice by TMA, finds each group's mean and the squares about it in two
// passes over them, tells the cluster's other CTAs, and writes. x is read once. 1024 rows of 512 channels take 5.3 us
// (two kernels: 8.2): launch and copy 1.8, means and squares 1, groups and cluster 1.7, rows the rest. More rows: bound by
// the passes over shared memory and the activation, not by HBM (2 TB/s).
//
// Other images: two kernels over chunks of rows. The first leaves the pairs of each cluster's chunks in the workspace, the
// second joins an image's pairs (of many groups a third kernel between the two does) and writes its chunk, from the last row
// to the first, as the rows read last are the ones still in L2. Bound by HBM: x is read once, and again as far as it is not
// in L2, y is written once; 2^20 rows of 128 channels in bf16 take 142 us, 5.7 TB/s of three passes (152 us with sums and
// activations in single registers instead of pairs). Of fewer than 128 channels, and of 129 to 255 vectors, a part of the threads
// has no column (a row's vectors are rounded up to sixteen, and a CTA takes whole rows): 2^21 rows of 64 take 212 us.
#include "e4m3_128.cuh"
#include "internal.h"

namespace hilo {

__device__ int g_group_norm_err;

namespace {

struct NormParams {
  const unsigned char* x;
  void* y;
  float* y_scale;
  float2* part;    // [image][group][cluster of chunks]: mean, sum of squares about it
  float2* joined;  // [image][group]: mean, 1 / deviation
  const void *scale, *shift, *w, *b;
  long long x_row, y_row, vec_row, y_scale_ld;  // x_row in bytes
  int rows, d, groups, per, act;                // per: channels of a group
  int y_type, vec_f32;
  float eps, inv_rows, inv_count;  // 1 / rows, 1 / (rows per)
};

// Mean and sum of squares about it.
struct Pair {
  float mean, sq;
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  return v;
}

// Eight neighbouring elements of a vector, `none` where there is none.
__device__ __forceinline__ void vec8(const void* v, int f32, long long i, float none, float* f) {
  if (!v) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = none;
  } else if (f32) {
    Eight<2> e;
    e.load(static_cast<const unsigned char*>(v) + i * 4);
    e.widen(f);
  } else {
    Eight<0> e;
    e.load(static_cast<const unsigned char*>(v) + i * 2);
    e.widen(f);
  }
}

// What a normalised row's channels c .. c + 7 are multiplied by, and what is added:
// w (1 + scale) and b (1 + scale) + shift.
__device__ __forceinline__ void gains(const NormParams& p, int image, int c, float* a, float* b) {
  float up[8], t[8];
  vec8(p.w, p.vec_f32, c, 1.f, a);
  vec8(p.b, p.vec_f32, c, 0.f, b);
  vec8(p.scale, p.vec_f32, image * p.vec_row + c, 0.f, up);
  vec8(p.shift, p.vec_f32, image * p.vec_row + c, 0.f, t);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    a[j] *= 1.f + up[j];
    b[j] = fmaf(b[j], 1.f + up[j], t[j]);
  }
}

// A row's channels c .. c + 7, from the elements to the values before rounding.
struct Affine {
  uint64_t minus[4], a[4], b[4];
  // stats(group): mean and 1 / deviation; c0: the first channel among those of the groups
  template <typename Stats>
  __device__ __forceinline__ void set(const NormParams& p, int image, int c, int c0, Stats stats) {
    float u[8], v[8];
    gains(p, image, c, u, v);
    set(u, v, p.per, c0, stats);
  }
  template <typename Stats>
  __device__ __forceinline__ void set(const float* u, const float* v, int per, int c0, Stats stats) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const Pair lo = stats((c0 + j) / per), hi = stats((c0 + j + 1) / per);
      minus[j / 2] = f2(-lo.mean, -hi.mean);
      a[j / 2] = f2(u[j] * lo.sq, u[j + 1] * hi.sq);
      b[j / 2] = f2(v[j], v[j + 1]);
    }
  }
  template <int ACT, int TYPE>
  __device__ __forceinline__ void apply(const Eight<TYPE>& e, float* f) const {
    uint64_t x[4];
    e.widen(x);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      f2_split(activation2<ACT>(f2_fma(f2_add(x[j], minus[j]), a[j], b[j])), f[2 * j], f[2 * j + 1]);
  }
};

// ----------------------------------------------------------- a CTA's groups --
// A CTA has n rows of some channels. Thread (tx, ty) has the channels 8 tx .. of the rows ty, ty + down, .. It leaves its
// pairs in shared memory: one for all eight channels where groups are whole vectors, one per channel
// otherwise. Then `lanes` threads a group, as many as there are for all groups at once, join them: the means first, then the squares
// about the joint mean.
__host__ __device__ inline int lanes_of(int groups, int threads) {
  int lanes = 32;
  while (lanes > 4 && groups * lanes > threads) lanes /= 2;
  return lanes;
}

struct Rows {
  int n, down;
  int unit, pitch;  // entries of a group in a thread row, entries of a thread row
  float weight;     // channels of an entry
  int base, more;   // rows of a thread: base, and one more of the first `more` thread rows
  int lanes;        // a power of two
  int t0, c0, dt, dc;  // a lane's first entry: its thread row and column, and what leads to the next, `lanes` entries on
  __device__ __forceinline__ Rows(int n, int down, int across, int wide, int per, int groups, int threads) : n(n), down(down) {
    const bool vectors = per % 8 == 0;
    unit = vectors ? per / 8 : per;
    pitch = vectors ? across : wide;
    weight = vectors ? 8.f : 1.f;
    base = n / down;
    more = n - base * down;
    lanes = lanes_of(groups, threads);
    const int l = threadIdx.x & (lanes - 1);
    t0 = l / unit;
    c0 = l - t0 * unit;
    dt = lanes / unit;
    dc = lanes - dt * unit;
  }
  // rows of the threads ty
  __device__ __forceinline__ int of(int ty) const { return base + (ty < more ? 1 : 0); }
};

// (8 floats a thread each)
__device__ __forceinline__ void leave_pairs(const Rows& o, int per, int tx, int ty, int n, const float* mean, const float* sq,
                                            float* means, float* squares) {
  if (per % 8 == 0) {
    // (in pairs: of equal values every sum is exact)
    const float m = 0.125f * (((mean[0] + mean[1]) + (mean[2] + mean[3])) + ((mean[4] + mean[5]) + (mean[6] + mean[7])));
    float q = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) q += fmaf(static_cast<float>(n) * (mean[j] - m), mean[j] - m, sq[j]);
    means[ty * o.pitch + tx] = m;
    squares[ty * o.pitch + tx] = q;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      means[ty * o.pitch + 8 * tx + j] = mean[j];
      squares[ty * o.pitch + 8 * tx + j] = sq[j];
    }
  }
}

__device__ __forceinline__ float lanes_sum(float v, int lanes) {
  for (int off = lanes >> 1; off >= 1; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  return v;
}

// Every group's pair, to use(group, lane of the group, pair), in whole warps; inv: 1 / (n per).
template <typename Use>
__device__ __forceinline__ void join_groups(const Rows& o, int groups, float inv, const float* means, const float* squares, Use use) {
  const int l = threadIdx.x & (o.lanes - 1), shift = 31 - __clz(o.lanes), threads = blockDim.x;
  for (int g0 = 0; g0 < groups; g0 += threads >> shift) {
    const int g = g0 + (threadIdx.x >> shift);
    const bool there = g < groups && o.n > 0;
    auto each = [&](auto f) {
      if (!there) return;
      for (int t = o.t0, c = o.c0; t < o.down;) {
        f(o.weight * static_cast<float>(o.of(t)), t * o.pitch + g * o.unit + c);
        t += o.dt;
        c += o.dc;
        if (c >= o.unit) {
          c -= o.unit;
          ++t;
        }
      }
    };
    float sum = 0.f, sq = 0.f, rest = 0.f;
    each([&](float n, int at) { sum += n > 0.f ? n * means[at] : 0.f; });
    const float mean = lanes_sum(sum, o.lanes) * inv;
    each([&](float n, int at) {
      if (n > 0.f) {
        const float gap = means[at] - mean;
        rest = fmaf(n, gap, rest);
        sq += fmaf(n * gap, gap, squares[at]);
      }
    });
    rest = lanes_sum(rest, o.lanes);
    sq = lanes_sum(sq, o.lanes);
    if (g < groups) use(g, l, there ? Pair{fmaf(rest, inv, mean), sq} : Pair{0.f, 0.f});
  }
}

// The pairs of a cluster's CTAs, [CTA][pitch groups], joined by LANES lanes a group, to use(group, pair); rows_of(k): rows of
// CTA k.
template <int LANES, typename RowsOf, typename Use>
__device__ __forceinline__ void join_cluster(const Pair* pairs, int pitch, int parts, int groups, int per, RowsOf rows_of, Use use) {
  const int k = threadIdx.x & (LANES - 1), threads = blockDim.x;
  for (int g0 = 0; g0 < groups; g0 += threads / LANES) {
    const int g = g0 + threadIdx.x / LANES;
    const float m = g < groups && k < parts ? static_cast<float>(rows_of(k)) : 0.f;
    const Pair q = m > 0.f ? pairs[k * pitch + g] : Pair{0.f, 0.f};
    const float rows = lanes_sum(m, LANES), inv = rows > 0.f ? __fdividef(1.f, rows) : 0.f;
    const float mean = lanes_sum(m * q.mean, LANES) * inv, gap = m > 0.f ? q.mean - mean : 0.f;
    const float rest = lanes_sum(m * gap, LANES), sq = lanes_sum(fmaf(m * static_cast<float>(per) * gap, gap, q.sq), LANES);
    if (g < groups && k == 0) use(g, Pair{fmaf(rest, inv, mean), sq});
  }
}

// Eight values of each of R rows, to the output's type. A half warp's lanes all come here, rows that are not there (below 0)
// too: its 128 channels are a block of codes.
template <int R>
__device__ __forceinline__ void put(const NormParams& p, const long long* row, int c, int tx, const float (*f)[8]) {
  if (p.y_type == HILO_E4M3) {
    float m[R];
#pragma unroll
    for (int i = 0; i < R; ++i) m[i] = row[i] >= 0 ? amax8(f[i], 0.f) : 0.f;
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1)
#pragma unroll
      for (int i = 0; i < R; ++i) m[i] = fmaxf(m[i], __shfl_xor_sync(0xffffffffu, m[i], off));
#pragma unroll
    for (int i = 0; i < R; ++i) {
      float inv, sc;
      block_scale(m[i], inv, sc);
      if (row[i] < 0) continue;
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.y) + row[i] * p.y_row + c) = block_codes(f[i], inv);
      if ((tx & 15) == 0) p.y_scale[(c >> 7) * p.y_scale_ld + row[i]] = sc;
    }
  } else {
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (row[i] >= 0) store8(p.y, p.y_type, row[i] * p.y_row + c, f[i]);
  }
}

// ------------------------------------------------------------------ two kernels --

constexpr int THREADS = 256;
constexpr int STATS_CTAS = 3, APPLY_CTAS = 3;  // per SM (four: the sums spill, 2^20 rows of 128 took 1.2 and 1.35 times as long)
constexpr int MAX_CHUNKS = 456;                // of a call's statistics, but for a cluster per image
constexpr int CHUNKS = 4;                      // of a cluster, whose pairs are joined before they are stored
constexpr int BATCH = 4;                       // rows of a thread at a time (eight: 2^20 rows of 128 in 3% more)
constexpr int JOINED = MAX_CHUNKS / CHUNKS / 32 + 1;  // pairs of a lane

// The chunks of an image: of its statistics and of its output.
struct Two {
  int across, down, passes;  // passes of the channels: across * passes * 8 >= d
  int chunks, chunk;         // (a multiple of CHUNKS; the last ones may be empty), and rows of each
  int clusters;
  int out_chunks, out_chunk;
};

template <int TYPE>
__global__ void __launch_bounds__(THREADS, STATS_CTAS) group_stats_kernel(const __grid_constant__ NormParams p, const __grid_constant__ Two o) {
  extern __shared__ float shared[];  // means, then squares
  pdl_wait();
  pdl_trigger();
  const int image = blockIdx.x / o.chunks, chunk = blockIdx.x - image * o.chunks, r0 = chunk * o.chunk;
  cluster_arrive_relaxed();  // this CTA has begun: the others may store into it
  const Rows rows(max(0, min(p.rows, r0 + o.chunk) - r0), o.down, o.passes * o.across, p.d, p.per, p.groups, THREADS);
  const int tx = threadIdx.x % o.across, ty = threadIdx.x / o.across;
  const unsigned char* x = p.x + (static_cast<long long>(image) * p.rows + r0) * p.x_row;
  float* means = shared;
  float* squares = shared + o.down * rows.pitch;
  Pair* pairs = reinterpret_cast<Pair*>(squares + o.down * rows.pitch);  // [chunk of the cluster][group of this CTA]
  constexpr int ESIZE = TYPE == 2 ? 4 : 2;
  for (int v = tx; v * 8 < p.d && ty < o.down; v += o.across) {
    uint64_t mean2[4], sq2[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) mean2[j] = sq2[j] = 0ull;
    int n = 0;
    const unsigned char* at = x + ty * p.x_row + v * 8 * ESIZE;
    const long long step = o.down * p.x_row;
    // more rows, of mean -minus and squares `two` about it, `part` of all there are: the mean moves by that of the gap
    auto join = [&](int j, uint64_t minus, uint64_t two, float part) {
      const uint64_t gap = f2_add(mean2[j], minus);
      const float scale = part * static_cast<float>(n);
      mean2[j] = f2_fma(gap, f2(-part, -part), mean2[j]);
      // (the scale first: of the thread's first rows it is 0, and the gap all of their mean, whose square may leave fp32)
      sq2[j] = f2_add(sq2[j], f2_fma(f2_mul(gap, f2(scale, scale)), gap, two));
    };
    int r = ty;
    for (; r + (BATCH - 1) * o.down < rows.n; r += BATCH * o.down) {
      Eight<TYPE> e[BATCH];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) e[i].load(at + i * step);
      at += BATCH * step;
      const float part = __fdividef(static_cast<float>(BATCH), static_cast<float>(n + BATCH));
      uint64_t f[BATCH][4];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) e[i].widen(f[i]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t minus = f2_mul(f2_add(f2_add(f[0][j], f[1][j]), f2_add(f[2][j], f[3][j])), f2(-0.25f, -0.25f));
        uint64_t two = 0ull;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          const uint64_t d = f2_add(f[i][j], minus);
          two = i ? f2_fma(d, d, two) : f2_mul(d, d);
        }
        join(j, minus, two, part);
      }
      n += BATCH;
    }
    Eight<TYPE> e[BATCH - 1];
#pragma unroll
    for (int i = 0; i < BATCH - 1; ++i)
      if (r + i * o.down < rows.n) e[i].load(at + i * step);
#pragma unroll
    for (int i = 0; i < BATCH - 1; ++i)
      if (r + i * o.down < rows.n) {
        const float part = __fdividef(1.f, static_cast<float>(n + 1));
        uint64_t f[4];
        e[i].widen(f);
#pragma unroll
        for (int j = 0; j < 4; ++j) join(j, f2_mul(f[j], f2(-1.f, -1.f)), 0ull, part);
        ++n;
      }
    float mean[8], sq[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f2_split(mean2[j], mean[2 * j], mean[2 * j + 1]);
      f2_split(sq2[j], sq[2 * j], sq[2 * j + 1]);
    }
    leave_pairs(rows, p.per, v, ty, n, mean, sq, means, squares);
  }
  __syncthreads();
  // group g's pairs to the cluster's CTA g % CHUNKS, which joins them
  const float inv = rows.n > 0 ? __fdividef(1.f, static_cast<float>(rows.n) * static_cast<float>(p.per)) : 0.f;
  const int rank = blockIdx.x % CHUNKS, pitch = (p.groups + CHUNKS - 1) / CHUNKS, first = r0 - rank * o.chunk;
  cluster_wait();
  join_groups(rows, p.groups, inv, means, squares, [&](int g, int l, Pair q) {
    if (l == 0)
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(mapa_shared(smem_u32(pairs + rank * pitch + g / CHUNKS), g % CHUNKS)),
                   "f"(q.mean), "f"(q.sq)
                   : "memory");
  });
  cluster_sync();
  join_cluster<CHUNKS>(
      pairs, pitch, CHUNKS, (p.groups - rank + CHUNKS - 1) / CHUNKS, p.per,
      [&](int k) { return max(0, min(p.rows, first + (k + 1) * o.chunk) - (first + k * o.chunk)); },
      [&](int i, Pair q) {
        p.part[(static_cast<long long>(image) * p.groups + i * CHUNKS + rank) * o.clusters + chunk / CHUNKS] = make_float2(q.mean, q.sq);
      });
}

// A group's mean and 1 / deviation from the pairs of its image's clusters, by a warp, the lanes' pairs in registers.
__device__ __forceinline__ Pair join_image(const NormParams& p, const Two& o, long long group, int lane) {
  const float2* part = p.part + group * o.clusters;
  const long long each = static_cast<long long>(CHUNKS) * o.chunk;
  auto rows_of = [&](int k) { return static_cast<float>(min(static_cast<long long>(p.rows), (k + 1) * each) - k * each); };
  float2 q[JOINED];
  float sum = 0.f, sq = 0.f, rest = 0.f;
#pragma unroll
  for (int i = 0; i < JOINED; ++i) {
    q[i] = make_float2(0.f, 0.f);
    if (32 * i + lane < o.clusters) q[i] = __ldg(part + 32 * i + lane);
  }
#pragma unroll
  for (int i = 0; i < JOINED; ++i)
    if (32 * i + lane < o.clusters) sum = fmaf(rows_of(32 * i + lane), q[i].x, sum);
  const float mean = warp_sum(sum) * p.inv_rows;
#pragma unroll
  for (int i = 0; i < JOINED; ++i)
    if (32 * i + lane < o.clusters) {
      const float part = rows_of(32 * i + lane) * (q[i].x - mean);
      rest += part;
      sq += fmaf(part * static_cast<float>(p.per), q[i].x - mean, q[i].y);
    }
  rest = warp_sum(rest);
  const float var = warp_sum(sq) * p.inv_count;
  return {fmaf(rest, p.inv_rows, mean), rsqrtf(var + p.eps)};
}

// More groups than FEW_GROUPS get a warp each in a kernel of their own; few ones each CTA of the output joins for itself.
// (65536 rows of 512, in us, for itself and by the kernel: 32 groups 42.8 and 48.5, 64 groups 44.6 and 47.4, 128 groups 50.1 and
// 49.9, 512 groups 75.4 and 58.5.)
constexpr int FEW_GROUPS = 64;
__global__ void __launch_bounds__(THREADS) group_join_kernel(const __grid_constant__ NormParams p, const __grid_constant__ Two o, long long groups) {
  pdl_wait();
  pdl_trigger();
  const long long g = static_cast<long long>(blockIdx.x) * (THREADS / 32) + warp_id();
  if (g >= groups) return;
  const Pair q = join_image(p, o, g, lane_id());
  if (lane_id() == 0) p.joined[g] = make_float2(q.mean, q.sq);
}

template <int TYPE>
__global__ void __launch_bounds__(THREADS, APPLY_CTAS) group_apply_kernel(const __grid_constant__ NormParams p, const __grid_constant__ Two o) {
  __shared__ Pair stats[FEW_GROUPS];  // means and 1 / deviation
  pdl_wait();
  pdl_trigger();
  const int image = blockIdx.x / o.out_chunks, r0 = (blockIdx.x - image * o.out_chunks) * o.out_chunk;
  const int n = min(p.rows, r0 + o.out_chunk) - r0;
  const long long group0 = static_cast<long long>(image) * p.groups;
  if (p.groups <= FEW_GROUPS) {
    const int lane = lane_id();
#pragma unroll 2
    for (int g = warp_id(); g < p.groups; g += THREADS / 32) {
      const Pair q = join_image(p, o, group0 + g, lane);
      if (lane == 0) stats[g] = q;
    }
  }
  __syncthreads();
  const int tx = threadIdx.x % o.across, ty = threadIdx.x / o.across;
  const long long row0 = static_cast<long long>(image) * p.rows + r0;
  const unsigned char* x = p.x + row0 * p.x_row;
  constexpr int ESIZE = TYPE == 2 ? 4 : 2;
  for (int pass = 0; pass < o.passes; ++pass) {
    const int c = (tx + pass * o.across) * 8;
    const bool in = c < p.d && ty < o.down;
    Affine affine;
    if (in)
      affine.set(p, image, c, c, [&](int g) {
        if (p.groups <= FEW_GROUPS) return stats[g];
        const float2 q = p.joined[group0 + g];
        return Pair{q.x, q.y};
      });
    const int steps = (n + o.down - 1) / o.down;
    with_activation(p.act, [&](auto act) {
      for (int s = (steps - 1) / BATCH; s >= 0; --s) {
        Eight<TYPE> e[BATCH];
        long long row[BATCH];  // of all images, -1: not there
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          const int r = ty + (s * BATCH + i) * o.down;
          const bool there = in && r < n;
          row[i] = there ? row0 + r : -1;
          e[i].clear();
          if (there) e[i].load(x + r * p.x_row + c * ESIZE);
        }
#pragma unroll
        for (int i = 0; i < BATCH; i += 2) {
          float f[2][8];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            affine.template apply<decltype(act)::value>(e[i + u], f[u]);
          }
          put<2>(p, row + i, c, tx, f);
        }
      }
    });
  }
}

// ------------------------------------------------------------------ one kernel --

constexpr int ONE_THREADS = 256;
constexpr int ONE_PARTS = 16;         // CTAs of a cluster at most
constexpr int ONE_SMEM = 112 * 1024;  // shared memory of a CTA at most: two on an SM (220 KB and one: 4 x 4096 rows of 512 35 us, else 21)
constexpr int ONE_LEAST = 76 * 1024;  // and at least: three on some SMs and one on others take longer (3 x 1380 rows of 1152: 14.8 us, else 11.6)
constexpr int ONE_WIDE = 256;         // channels of a slice at most, and rows of a box (TMA)

// How an image is shared out: `slices` of `wide` channels, each `parts` CTAs of `chunk` rows; a row's `across` vectors of
// eight channels, `down` rows at a time.
struct One {
  int wide, slices, parts, chunk, across, down, box, groups;  // groups: of a slice
  int tile;                                                   // bytes of x
  // the tile, means, squares, barrier and flag, the cluster's pairs, the groups' statistics; alignment
  int smem() const {
    return tile + ONE_THREADS * 8 * 2 * static_cast<int>(sizeof(float)) + 16 + (parts + 1) * groups * static_cast<int>(sizeof(Pair)) + 16 + 128;
  }
};

template <int TYPE>
__global__ void __launch_bounds__(ONE_THREADS, 2)
    group_norm_kernel(const __grid_constant__ CUtensorMap tm, const __grid_constant__ NormParams p, const __grid_constant__ One o) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((128u - (smem_u32(smem_raw) & 127u)) & 127u);
  constexpr int ESIZE = TYPE == 2 ? 4 : 2;
  unsigned char* tile = smem;  // [rows][wide]
  float* means = reinterpret_cast<float*>(smem + o.tile);
  float* squares = means + ONE_THREADS * 8;
  uint64_t* bar = reinterpret_cast<uint64_t*>(squares + ONE_THREADS * 8);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bar + 1);
  Pair* pairs = reinterpret_cast<Pair*>(bar + 2);  // [CTA][group]
  Pair* stats = pairs + o.parts * o.groups;        // [group]: mean, 1 / deviation
  if (threadIdx.x == 0) {
    mbar_init(bar, 1);
    *abort_flag = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tm);
  }
  __syncthreads();
  pdl_wait();  // all threads
  pdl_trigger();
  const int rank = blockIdx.x % o.parts, unit = blockIdx.x / o.parts;
  const int image = unit / o.slices, c0 = (unit - image * o.slices) * o.wide;
  const int r0 = rank * o.chunk, n = max(0, min(p.rows, r0 + o.chunk) - r0);
  const int here = min(o.wide, p.d - c0), groups = here / p.per;
  const long long row0 = static_cast<long long>(image) * p.rows + r0;
  if (threadIdx.x == 0 && n > 0) {
    // (whole boxes: the rows behind the part, and the channels behind the last, are read over or are zeros)
    const int boxes = (n + o.box - 1) / o.box;
    mbar_arrive_expect_tx(bar, static_cast<uint32_t>(boxes * o.box * o.wide * ESIZE));
    for (int i = 0; i < boxes; ++i)
      tma_load_2d(tile + static_cast<size_t>(i) * o.box * o.wide * ESIZE, &tm, bar, c0, static_cast<int>(row0) + i * o.box);
  }
  if (o.parts > 1) cluster_arrive_relaxed();  // this CTA has begun: the others may store into it
  const int tx = threadIdx.x % o.across, ty = threadIdx.x / o.across, c = tx * 8;
  const bool on = ty < o.down && c < here;
  const Rows rows(n, o.down, o.across, o.wide, p.per, groups, ONE_THREADS);
  const float inv_n = __fdividef(1.f, static_cast<float>(n) * static_cast<float>(p.per));
  float a[8], b[8];
  if (on) gains(p, image, c0 + c, a, b);  // beside the copies
  // (a wait that ran out leaves an error and rows that are not meant to be right; the copies in flight once more, before the CTA exits)
  if (n > 0 && !mbar_wait(bar, 0, abort_flag, &g_group_norm_err, DEV_TIMEOUT_GEMM + 256 * 30)) {
    const uint64_t g0 = globaltimer_ns();
    while (!mbar_try_wait(smem_u32(bar), 0) && globaltimer_ns() - g0 < HILO_WAIT_LIMIT_NS / 4) {
    }
  }
  const int pitch = o.wide * ESIZE;
  auto at = [&](int r) { return tile + r * pitch + c * ESIZE; };
  // the thread's pairs: its means, then the squares about them
  if (on) {
    uint64_t sum2[4], sq2[4], rest2[4];  // rest2: of fp32
#pragma unroll
    for (int j = 0; j < 4; ++j) sum2[j] = sq2[j] = rest2[j] = 0ull;
#pragma unroll 4
    for (int r = ty; r < n; r += o.down) {
      Eight<TYPE> e;
      uint64_t f[4];
      e.load(at(r));
      e.widen(f);
#pragma unroll
      for (int j = 0; j < 4; ++j) sum2[j] = f2_add(sum2[j], f[j]);
    }
    const int mine = rows.of(ty);
    const float inv = mine > 0 ? __fdividef(1.f, static_cast<float>(mine)) : 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint64_t sum = sum2[j];
      sum2[j] = f2_mul(sum, f2(-inv, -inv));
      // Of equal values in 16 bits the sum is exact (of less than 2^13 rows), and the quotient, put right by its remainder, is the value.
      // Of fp32 what the values are about the mean is added up below, which took 16384 rows of 512 in bf16 from 15.1 to 15.9 us.
      const float n = static_cast<float>(mine);
      if (TYPE != 2) sum2[j] = f2_fma(f2_fma(sum2[j], f2(n, n), sum), f2(-inv, -inv), sum2[j]);
    }
#pragma unroll 4
    for (int r = ty; r < n; r += o.down) {
      Eight<TYPE> e;
      uint64_t f[4];
      e.load(at(r));
      e.widen(f);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t d = f2_add(f[j], sum2[j]);
        if (TYPE == 2) rest2[j] = f2_add(rest2[j], d);
        sq2[j] = f2_fma(d, d, sq2[j]);
      }
    }
    float mean[8], sq[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f2_split(TYPE == 2 ? f2_fma(rest2[j], f2(-inv, -inv), sum2[j]) : sum2[j], mean[2 * j], mean[2 * j + 1]);
      f2_split(sq2[j], sq[2 * j], sq[2 * j + 1]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) mean[j] = -mean[j];
    leave_pairs(rows, p.per, tx, ty, mine, mean, sq, means, squares);
  }
  __syncthreads();
  // every CTA gets every CTA's pairs
  if (o.parts > 1) cluster_wait();
  join_groups(rows, groups, inv_n, means, squares, [&](int g, int l, Pair q) {
    for (int k = l; k < o.parts; k += rows.lanes) {
      const uint32_t to = smem_u32(pairs + rank * groups + g), remote = o.parts > 1 ? mapa_shared(to, k) : to;
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(remote), "f"(q.mean), "f"(q.sq) : "memory");
    }
  });
  if (o.parts > 1) cluster_sync();
  else __syncthreads();
  join_cluster<ONE_PARTS>(
      pairs, groups, o.parts, groups, p.per, [&](int k) { return max(0, min(p.rows, (k + 1) * o.chunk) - k * o.chunk); },
      [&](int g, Pair q) { stats[g] = {q.mean, rsqrtf(fmaf(q.sq, p.inv_count, p.eps))}; });
  __syncthreads();
  Affine affine;
  if (on) affine.set(a, b, p.per, c, [&](int g) { return stats[g]; });
  with_activation(p.act, [&](auto act) {
#pragma unroll 1
    for (int r1 = ty; r1 - ty < n; r1 += 2 * o.down) {
      float f[2][8];
      long long row[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int r = r1 + u * o.down;
        const bool there = on && r < n;
        row[u] = there ? row0 + r : -1;
        Eight<TYPE> e;
        e.clear();
        if (there) e.load(at(r));
        affine.template apply<decltype(act)::value>(e, f[u]);
      }
      put<2>(p, row, c0 + c, tx, f);
    }
  });
}

// How many clusters of so many CTAs the device holds, two CTAs on an SM: sizes above eight fill its groups of SMs badly or well.
template <int TYPE>
int resident_clusters(int parts, int device, int num_sms) {
  static PerDevice known[ONE_PARTS + 1];
  const int n = known[parts].get(device, [&] {
    if (parts > 8 && cudaFuncSetAttribute(group_norm_kernel<TYPE>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
      cudaGetLastError();
      return 0;
    }
    cudaFuncSetAttribute(group_norm_kernel<TYPE>, cudaFuncAttributeMaxDynamicSharedMemorySize, ONE_SMEM);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(parts * num_sms, 1, 1);
    cfg.blockDim = dim3(ONE_THREADS, 1, 1);
    cfg.dynamicSmemBytes = ONE_SMEM;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = parts;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int found = 0;
    if (cudaOccupancyMaxActiveClusters(&found, group_norm_kernel<TYPE>, &cfg) != cudaSuccess) {
      cudaGetLastError();
      found = 0;
    }
    return found;
  });
  return n > 0 ? n : parts > 8 ? 0 : num_sms / 8;  // 0: none of this size
}

// The cheapest way to share an image out, and its cost in us: by waves of clusters, 2.9 us each beside an element's work and
// a byte's way, more by CTAs of a cluster and by entries that a lane joins. Against the two kernels' 8.2 us and 1.2 for a
// million elements. Fitted to 34 shapes of 22 to 65536 rows, 32 to 2304 channels in every slice and number of parts: the pick
// is 1.6% behind the fastest in the mean, 18% at worst (8 x 82 rows of 2048 6.6 us, 5.6 in wider slices). Examples, in us:
// 1024 rows of 512 5.3, two kernels 8.2; 3 x 1380 rows of 1152 to codes 10.1 in 10 parts, 11.6 in 8, two kernels 17.2; 16384
// rows of 512 15.4 in 13 parts, 19.8 in 16 (two waves), two kernels 18.2; 4 x 4096 rows of 512 to codes 20.7, two kernels 18.2.
constexpr float NO_PLAN = 3e38f;
template <int TYPE>
float plan_one(const hilo_group_norm_shape& s, int device, int num_sms, One* best) {
  const int per = s.d / s.groups, esize = s.x_dtype == HILO_F32 ? 4 : 2;
  if (s.x_row * esize >= (1LL << 40)) return NO_PLAN;  // (TMA's strides)
  // whole groups, whole vectors, and of codes whole blocks
  int unit = per;
  while (unit % 8) unit += per;
  if (s.y_dtype == HILO_E4M3 && s.d > 128)
    while (unit % 128 && unit < s.d) unit += per;
  int held[ONE_PARTS + 1];
  for (int parts = 1; parts <= ONE_PARTS; ++parts) held[parts] = resident_clusters<TYPE>(parts, device, num_sms);
  float least = NO_PLAN;
  for (int wide = unit; wide <= ONE_WIDE && wide < s.d + unit; wide += unit) {
    const int w = wide < s.d ? wide : s.d;
    if (w > ONE_WIDE || (w * esize < 64 && w < s.d)) continue;
    if (s.y_dtype == HILO_E4M3 && w % 128 && w < s.d) continue;
    int across = w / 8;
    if (s.y_dtype == HILO_E4M3) across = (across + 15) / 16 * 16;
    const int groups = w / per, down = ONE_THREADS / across, lanes = lanes_of(groups, ONE_THREADS);
    const int entries = (down * (per % 8 == 0 ? per / 8 : per) + lanes - 1) / lanes;  // of a lane, a group
    const int joined = entries * ((groups * lanes + ONE_THREADS - 1) / ONE_THREADS);
    const long long slices = (s.d + w - 1) / w, clusters = s.B * slices;
    for (int parts = 1; parts <= ONE_PARTS && parts <= (s.rows > 1 ? s.rows : 1); ++parts) {
      const float fixed = 0.15f * static_cast<float>(parts) + 0.16f * static_cast<float>(joined);
      if (2.9f + fixed >= least) break;
      const int chunk = (s.rows + parts - 1) / parts;
      const long long ctas = clusters * parts, bytes = static_cast<long long>(chunk) * w * esize;
      if (ctas > 0x7fffffffLL || bytes > ONE_SMEM || held[parts] == 0) continue;
      const long long waves = clusters <= held[parts] ? 1 : (clusters + held[parts] - 1) / held[parts];
      const float work = (0.064e-3f / static_cast<float>(esize) + 0.047e-3f) * static_cast<float>(bytes);
      const float cost = static_cast<float>(waves) * (2.9f + work * (ctas > num_sms ? 1.26f : 1.f)) + fixed;
      if (!(cost < least)) continue;
      int box = (chunk + 7) / 8 * 8;
      if (box > ONE_WIDE) box = ONE_WIDE;
      const long long tile = static_cast<long long>((chunk + box - 1) / box) * box * w * esize;
      const One one = {w, static_cast<int>(slices), parts, chunk, across, down, box, groups, static_cast<int>(tile < ONE_SMEM ? tile : ONE_SMEM)};
      if (one.smem() > ONE_SMEM) continue;
      least = cost;
      *best = one;
    }
  }
  return least;
}

template <int TYPE>
cudaError_t launch_one(const hilo_group_norm_shape& s, const NormParams& p, const One& o, int* launches, cudaStream_t st) {
  CUtensorMap tm;
  const int esize = TYPE == 2 ? 4 : 2;
  if (!encode_tmap_rows_2d(&tm, esize, p.x, static_cast<uint64_t>(s.d), static_cast<uint64_t>(s.B) * s.rows, static_cast<uint64_t>(s.x_row),
                           static_cast<uint32_t>(o.wide), static_cast<uint32_t>(o.box)))
    return cudaErrorInvalidValue;
  auto* kern = group_norm_kernel<TYPE>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, ONE_SMEM);
  if (e != cudaSuccess) return e;
  if (o.parts > 8 && (e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1)) != cudaSuccess) return e;
  e = launch_pdl_cluster(kern, o.parts, dim3(static_cast<unsigned>(s.B) * o.slices * o.parts), dim3(ONE_THREADS),
                         static_cast<size_t>(o.smem() > ONE_LEAST ? o.smem() : ONE_LEAST), st, tm, p, o);
  if (e == cudaSuccess) *launches = 1;
  return e;
}

// Threads and chunks of the two kernels; `most` chunks of statistics and `most_out` of output, if each image has one.
Two plan_two(const hilo_group_norm_shape& s, int most, int most_out) {
  Two o;
  const int vectors = s.d / 8, wide = (vectors + 15) / 16 * 16;
  o.across = wide < THREADS ? wide : THREADS;
  o.passes = (vectors + o.across - 1) / o.across;
  o.down = THREADS / o.across;
  if (o.down > s.rows && s.rows > 0) o.down = s.rows;
  auto share = [&](int chunks, int* chunk) {  // an image's rows among so many chunks, whole passes each
    const int unit = o.down * BATCH, full = (s.rows + unit - 1) / unit;
    if (chunks > full) chunks = full;
    if (chunks < 1) chunks = 1;
    *chunk = ((s.rows + chunks - 1) / chunks + o.down - 1) / o.down * o.down;
    return *chunk ? (s.rows + *chunk - 1) / *chunk : 1;
  };
  const int each = most / s.B / CHUNKS * CHUNKS;
  o.clusters = (share(each > CHUNKS ? each : CHUNKS, &o.chunk) + CHUNKS - 1) / CHUNKS;
  o.chunks = CHUNKS * o.clusters;
  o.out_chunks = share(most_out / s.B, &o.out_chunk);
  return o;
}

// As many chunks of statistics as the device holds at once: clusters do not fill its groups of SMs. (2^20 rows of
// 128 channels in bf16: 155 us with the 432 that it holds in clusters of 4, 182 with 448; 164 with the 400 of clusters of 8; by
// an earlier form of the loops.)
template <int TYPE>
int resident_chunks(int device, int num_sms) {
  static PerDevice clusters;
  const int n = clusters.get(device, [&] {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(CHUNKS * num_sms, 1, 1);
    cfg.blockDim = dim3(THREADS, 1, 1);
    cfg.dynamicSmemBytes = 72 * 1024;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = CHUNKS;
    attr.val.clusterDim.y = 1;
    attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int found = 0;
    if (cudaOccupancyMaxActiveClusters(&found, group_stats_kernel<TYPE>, &cfg) != cudaSuccess) {
      cudaGetLastError();
      found = 0;
    }
    return found;
  });
  const int chunks = n > 0 ? CHUNKS * n : num_sms;
  return chunks < MAX_CHUNKS ? chunks : MAX_CHUNKS;
}

template <int TYPE>
cudaError_t launch_two(const hilo_group_norm_shape& s, const NormParams& p, int device, int num_sms, int* launches, cudaStream_t st) {
  auto* kern = group_stats_kernel<TYPE>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
  if (e != cudaSuccess) return e;
  const Two o = plan_two(s, resident_chunks<TYPE>(device, num_sms), APPLY_CTAS * num_sms);
  // (o.chunks is at most what the device holds over B, or CHUNKS: with B below 2^29 the grids are ints)
  const size_t stats = static_cast<size_t>(o.down) * 2 * sizeof(float) * (p.per % 8 == 0 ? o.across * o.passes : s.d) +
                       static_cast<size_t>(s.groups + CHUNKS) * sizeof(Pair);
  e = launch_pdl_cluster(kern, CHUNKS, dim3(static_cast<unsigned>(o.chunks) * static_cast<unsigned>(s.B)), dim3(THREADS), stats, st, p, o);
  if (e != cudaSuccess) return e;
  *launches = 1;
  if (s.groups > FEW_GROUPS) {
    const long long groups = static_cast<long long>(s.B) * s.groups, ctas = (groups + THREADS / 32 - 1) / (THREADS / 32);
    e = launch_pdl(group_join_kernel, dim3(static_cast<unsigned>(ctas)), dim3(THREADS), 0, st, p, o, groups);
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  e = launch_pdl(group_apply_kernel<TYPE>, dim3(static_cast<unsigned>(o.out_chunks) * static_cast<unsigned>(s.B)), dim3(THREADS), 0, st, p, o);
  if (e == cudaSuccess) ++*launches;
  return e;
}

template <int TYPE>
cudaError_t launch_type(const hilo_group_norm_shape& s, const NormParams& p, int device, int num_sms, int* launches, cudaStream_t st) {
  One o;
  const float two = 8.2f + 1.2e-6f * static_cast<float>(s.B) * static_cast<float>(s.rows) * static_cast<float>(s.d);
  return plan_one<TYPE>(s, device, num_sms, &o) < two ? launch_one<TYPE>(s, p, o, launches, st) : launch_two<TYPE>(s, p, device, num_sms, launches, st);
}

}  // namespace

size_t group_norm_workspace_bytes(const hilo_group_norm_shape& s) {
  return static_cast<size_t>(s.B) * (plan_two(s, MAX_CHUNKS, 1).clusters + (s.groups > FEW_GROUPS ? 1 : 0)) * s.groups * sizeof(float2);
}

cudaError_t launch_group_norm(const GroupNormArgs& a, int device, int num_sms, int* launches, cudaStream_t st) {
  *launches = 0;
  const hilo_group_norm_shape& s = a.s;
  NormParams p;
  p.x = static_cast<const unsigned char*>(a.x);
  p.y = a.y;
  p.y_scale = a.y_scale;
  p.joined = static_cast<float2*>(a.ws);
  p.part = p.joined + (s.groups > FEW_GROUPS ? static_cast<long long>(s.B) * s.groups : 0);
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
  p.inv_rows = 1.0f / static_cast<float>(s.rows);
  p.inv_count = static_cast<float>(1.0 / (static_cast<double>(s.rows) * p.per));
  return s.x_dtype == HILO_BF16  ? launch_type<0>(s, p, device, num_sms, launches, st)
         : s.x_dtype == HILO_F16 ? launch_type<1>(s, p, device, num_sms, launches, st)
                                 : launch_type<2>(s, p, device, num_sms, launches, st);
}

int group_norm_take_device_error() {
  int v = 0, z = 0;
  if (cudaMemcpyFromSymbol(&v, g_group_norm_err, sizeof(int)) != cudaSuccess) return -1;
  if (v) cudaMemcpyToSymbol(g_group_norm_err, &z, sizeof(int));
  return v;
}

}  // namespace hilo
