// The choice among the kernels of the products with a scale per 128 (gemm128_tc.cu), by sizes alone: plain C++,
// so that the host's tests can ask it, too.
#pragma once

namespace hilo {

constexpr int GEMM128_PIECE = 128 * 128;  // bytes of 128 rows of a block of 128 along K
constexpr int GEMM128_SPLIT = 8;          // CTAs of a cluster of few128 at most

// Which kernel, by its cost in microseconds. A launch is 2.2 of them; then
//   few128<NT>    per wave of CTAs (as many as the device holds of clusters of `split`) an `each` and, per block of
//                 128 along K, the longer of `block`, the chain from a block's copy to its sums, and of what the wave's CTAs
//                 read of the weights at 8 TB/s (L2 and HBM)
//   many128<NT>   the first tile of a pair and each further one: an `each` and a `block` of their own (at full load
//                 the chip is at its power limit)
// fitted to 252 shapes of 1 to 8192 rows, 512 to 6080 columns, 128 to 16384 features, each with every choice: its pick is 0.5%
// behind the fastest in the mean, 31% at worst (64 rows of 4096, 1024 features gated: 8.8 us, 6.7 in four tiles of 16
// rows, cut in four). Examples, in us: 64 rows of 4096, 4096 features: few128<64> cut in four 6.6, few128<16> in two 8.7; 512
// rows: few128<128> 16.9, many128<128> 12.7, many128<256> 17.6; 1024 rows: many128<128> 22.3, many128<256> 19.4; 1300 rows
// of 6080, 512 features: few128<128> in two 14.1, many128<128> 15.5. 192 columns are for what fills a round with them and leaves
// a part of one idle with 256: 700 rows of 4096, 4096 features: 16.6, 128 columns 22.0, 256 18.9; 2389 rows: 41.1, 49.5 and 48.6;
// 8192 rows: 125, 136 and 109. (Of 18 shapes with all three timed each pick was the fastest.)
struct Gemm128Choice {
  int many;  // few128 otherwise
  int nt, split;
};
template <bool GATED>
Gemm128Choice gemm128_choice(int rows, int n, int kblocks, bool codes, int num_sms) {
  struct Cost {
    float each, block;
  };
  constexpr Cost FEW[2][4] = {{{1.14f, .203f}, {1.78f, .202f}, {3.14f, .263f}, {3.52f, .292f}},
                              {{1.37f, .325f}, {2.58f, .326f}, {4.27f, .326f}, {6.16f, .655f}}};
  constexpr Cost FIRST[2][3] = {{{1.92f, .245f}, {2.52f, .327f}, {2.8f, .41f}}, {{1.91f, .244f}, {}, {3.12f, .398f}}};
  constexpr Cost NEXT[2][3] = {{{1.2f, .274f}, {2.05f, .349f}, {3.24f, .399f}}, {{.77f, .26f}, {}, {2.29f, .416f}}};
  constexpr int PARTS = GATED ? 2 : 1;
  auto ceil_div = [](long long a, long long b) { return (a + b - 1) / b; };
  Gemm128Choice best = {1, 256, 1};
  float least = 3e38f;
  auto offer = [&](float cost, Gemm128Choice c) {
    if (cost < least) {
      least = cost;
      best = c;
    }
  };
  for (int i = 0; i < 4; ++i) {
    const int nt = 16 << i;
    if (rows > 32 * nt || (nt > 16 && rows <= nt / 2)) continue;
    const long long row_tiles = ceil_div(rows, nt), tiles = ceil_div(n, 128) * row_tiles;
    const int per_sm = nt * PARTS <= 64 ? 2 : 1;
    for (int split = 1; split <= GEMM128_SPLIT && split <= kblocks; split *= 2) {
      // (clusters stay within a group of SMs, whose number eight does not divide)
      const int held = per_sm * num_sms * (split <= 2 ? 38 : split == 4 ? 36 : per_sm == 2 ? 32 : 26) / 38;
      const long long ctas = tiles * split, waves = ceil_div(ctas, held);
      const float reads = static_cast<float>(ctas < held ? ctas : held) * (PARTS * GEMM128_PIECE) / (row_tiles == 1 ? 8.18e6f : 8.06e6f);
      const Cost c = FEW[GATED][i];
      offer(0.05f * split + static_cast<float>(waves) * (c.each + static_cast<float>(ceil_div(kblocks, split)) * (reads > c.block ? reads : c.block)),
            {0, nt, split});
    }
  }
  for (int i = codes ? 2 : 0; i < 3; i += GATED ? 2 : 1) {  // (gated to codes: a tile has whole blocks)
    const int nt = 128 + 64 * i;
    const long long rounds = ceil_div(ceil_div(rows, 256) * ceil_div(n, nt / PARTS), num_sms / 2 > 0 ? num_sms / 2 : 1);
    const Cost f = FIRST[GATED][i], x = NEXT[GATED][i];
    offer(f.each + static_cast<float>(kblocks) * f.block + static_cast<float>(rounds - 1) * (x.each + static_cast<float>(kblocks) * x.block),
          {1, nt, 1});
  }
  return best;
}

}  // namespace hilo
