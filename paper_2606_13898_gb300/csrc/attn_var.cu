// Softmax attention of packed sequences with grouped heads on tcgen05: whole
// prompts, chunks of new tokens over earlier ones, single tokens; causal or
// not (hilo_attention, include/hilo.h). It serves the transformer that makes
// the text rows of the block's joint attention (paper Sec. 2.1) and any other
// attention over sequences whose lengths only the device knows.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(scale q_i.k_j - m_i), over the keys j that query i sees,
//
// in one pass over the keys with the running maximum m_i and sum.
//
// Tiles. The g query heads of one key head share its keys, so a tile of 128
// rows of the matrix product is floor(128 / g) neighbouring tokens with their
// g heads each (row = token * g + head): one box of a three-axis tensor map.
// A single token therefore costs one pass over the keys per key head, not per
// query head, and a tile's rows see nearly the same keys.
//
// Jobs. Two neighbouring tiles of one key head are a job (pair): each softmax
// warpgroup has one of them, and both share every K/V tile. A tile without a
// partner is a job of its own (single), whose key tiles alternate between the
// two warpgroups; the second then hands its maxima, sums and accumulator to
// the first. A job whose steps are more than a CTA's fair share is cut along
// the keys into pieces, each of which leaves unnormalised fp32 rows with their
// maxima and sums in the workspace; a second kernel joins them. That is how a
// few long sequences of single tokens get the whole device.
//
// Plan. Only the device knows the lengths, so every CTA makes the same plan
// (plan_build): the jobs of all sequences, the fair share, the cuts, longest
// first. CTA x of G takes items x, 2G-1-x, ..: the longest with the
// shortest. One warp walks the CTA's items ahead of the others and hands them
// on through a ring of four in shared memory.
//
// A CTA is three warpgroups, as in attn_tc.cu: two for the softmax (a row per
// thread, S and P in tensor memory, P the A operand of the second product),
// one for the Q/K copies, the V copies, the MMAs and the items.
//
// What a query does not see never reaches its result: masked logits are
// replaced, not computed with, and a value tile that some row of the job sees
// only in part is looked through for infinities and NaNs, whose product with
// a probability of 0 would be NaN. They are taken out of the tile, and rows
// that do see them get them back at the end (take_out, give_back).
//
// Every mbarrier wait is bounded (error latched, TMEM freed, CTA returns).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>

#include <atomic>

#include "attn_common.cuh"
#include "common.cuh"
#include "internal.h"

namespace hilo {

__device__ int g_attn_var_err;

namespace {

constexpr int BQ = 128;
constexpr int BKV = 128;
constexpr int THREADS = 384;
constexpr int PRODUCER_WARP = 8;     // Q and K copies
constexpr int MMA_WARP = 9;
constexpr int V_PRODUCER_WARP = 10;  // V copies
constexpr int ITEM_WARP = 11;
// (The softmax spills with 216 registers: prompts of 8192 tokens 357 us, 355 with 232;
// of 1 to 1021 24.1 and 23.1.)
constexpr uint32_t SOFTMAX_REGS = 232;
constexpr uint32_t CONTROL_REGS = 40;
constexpr float RESCALE_LOG2 = 8.0f;
// Probabilities are 2^(x - m), m the running maximum less this: fp16 ones begin at 2^7, so that
// with the 2^8 which the maximum may lag behind they end at 2^15, and what is lost below fp16's
// smallest number is 2^-32 of the largest one, not 2^-25. bf16 has fp32's exponents.
template <bool F16>
constexpr float P_ABOVE_LOG2 = F16 ? 7.0f : 0.0f;

struct VarParams {
  const int32_t *cu_q, *cu_k;
  const void* v;
  void* out;
  float* part;      // pieces' rows: [slot][tile 0, 1][HD / 8][row][8], so that a warp's stores join up
  float2* part_ml;  // their maxima and sums: [slot][tile][row]
  struct Joints* joints;  // the cut jobs
  long long v_row, v_head, out_row, out_head;
  int B, kv_heads, group, tpt;  // tpt: tokens per tile
  unsigned long long tpt_mul;   // n / tpt = n * tpt_mul >> tpt_shift, n < 2^31
  int tpt_shift;
  int causal, rows_q, rows_k;
  int grid;  // CTAs of the main kernel
  int may_cut;
  int out_wide;  // out's rows and heads begin on 32 bytes
  float scale_log2;  // log2(e) * scale
};

// ---------------------------------------------------------------- sequences --

struct Seq {
  int q0, lq, k0, lk;
  // Keys that token i sees.
  __device__ __forceinline__ int seen(const VarParams& p, int i) const {
    return p.causal ? min(lk, max(0, i + 1 + (lk - lq))) : lk;
  }
  __device__ __forceinline__ int tiles(const VarParams& p) const {
    return static_cast<int>(static_cast<unsigned long long>(lq + p.tpt - 1) * p.tpt_mul >> p.tpt_shift);
  }
  // Key tiles of query tile j: those its last token sees (one, all of it
  // masked, where it sees none: the zeros of such rows are written too).
  __device__ __forceinline__ int key_tiles(const VarParams& p, int j) const {
    return max(1, (seen(p, min(lq, (j + 1) * p.tpt) - 1) + BKV - 1) / BKV);
  }
  // Row jobs of up to `width` tiles, and the steps of job i of a sequence of nt tiles: a
  // pair's key tiles, half of a single's.
  __device__ __forceinline__ int row_jobs(const VarParams& p, int width) const {
    const int nt = tiles(p);
    return width == 1 ? nt : (nt + 1) / 2;
  }
  __device__ __forceinline__ int steps(const VarParams& p, int width, int nt, int i) const {
    const int last = width * (i + 1) - 1;
    return width == 2 && last < nt ? key_tiles(p, last) : (key_tiles(p, min(last, nt - 1)) + 1) / 2;
  }
};

__device__ __forceinline__ Seq sequence(const VarParams& p, int b) {
  auto at = [](const int32_t* cu, int rows) { return min(max(*cu, 0), rows); };
  const int q0 = at(p.cu_q + b, p.rows_q), q1 = at(p.cu_q + b + 1, p.rows_q);
  const int k0 = at(p.cu_k + b, p.rows_k), k1 = at(p.cu_k + b + 1, p.rows_k);
  return {q0, max(0, q1 - q0), k0, max(0, k1 - k0)};
}

// --------------------------------------------------------------------- plan --
//
// A row job is a job of one sequence for all its key heads. Up to MAX_TABLE
// row jobs are listed; the items of an entry are its key heads' jobs, or their
// pieces. More row jobs than that are taken as they come, the last of each
// sequence first: MAX_TABLE * kv_heads / G items per CTA and more, which is 6 with
// one key head. So of them, too, those that are longer than a share are listed, their pieces
// ahead of all others (cut_longest: 1100 single tokens, one over 131072 keys and the
// others over up to 200, 784 us without, 82 so).
//
// Cutting: J jobs of T steps together on G CTAs, pieces of at most `share`
// steps. An item costs about ITEM_STEPS more than its steps (copies to wait for,
// the last product, the output rows).
//   J < G   the smallest share, of one per warp between ceil(T / G) and the smaller
//           of ceil(T / (G - J)) and the longest job in floor(G / J) pieces, that makes at
//           most G items: one for each CTA. (The last two do: sum(c / share + 1)
//           <= G, and each job of at most floor(G / J) pieces.)
//           Not so single tokens whose jobs are too many for that (deal_few).
//   J >= G  ceil((T + J ITEM_STEPS) / G) - ITEM_STEPS, and only jobs that are
//           longer by more than ITEM_STEPS are cut. Listed longest first, to a
//           sixteenth of the longest, the cut ones ahead of the others: fewer than
//           2G pieces. (One of k pieces has more than (k - 1) share steps, of two at least
//           share + 3, and T < G (share + 2) - 2J: so too with J >= G / 2.)
// Pieces of fewer steps than min_steps would cost more in their epilogues and in the second
// kernel than they save.
//
// Singles or pairs: both take two tiles' products per step, a pair reads the keys once
// for both. Every tile is a job of its own where that makes shorter jobs for idle CTAs or
// evens out a causal triangle (job_width): one prompt of 985 tokens, 8 heads, 23.4 us
// in pairs and 15.3 in singles; prompts of up to 2235 tokens, 6 heads on one, 49.3 and 25.7.

constexpr int MAX_SEQ = ATTN_MAX_SEQUENCES;
constexpr int MAX_TABLE = 1024;
constexpr int MIN_STEPS = 4;       // of a piece
constexpr int MIN_STEPS_ROWS = 2;  // of jobs of up to FEW_ROWS rows, which are joined at once
constexpr int FEW_ROWS = 32;
constexpr int ITEM_STEPS = 2;
constexpr int SLOTS_PER_CTA = 2;
constexpr int BUCKETS = 32;  // 16 of cut jobs, 16 of whole ones

struct Plan {
  int first[MAX_SEQ + 1];  // row jobs before sequence b
  int seq[MAX_TABLE];      // entry: sequence << 16 | row job of it (of more than MAX_TABLE: counted from its last)
  int steps[MAX_TABLE];
  int items[MAX_TABLE];    // items before the entry
  int width;  // tiles of a job at most
  int jobs, n_items, n_cut, share, cut_above;  // row jobs, items, entries that may be cut (the first ones)
  // Entries and their items, the first ones. More row jobs than MAX_TABLE: what is listed of them, and behind
  // it an item for every key head of every row job, nothing to do where that is listed.
  __device__ __forceinline__ bool whole() const { return jobs <= MAX_TABLE; }
  __device__ __forceinline__ int entries() const { return whole() ? jobs : n_cut; }
  __device__ __forceinline__ int entry_items(const VarParams& p) const { return whole() ? n_items : n_items - jobs * p.kv_heads; }
  __device__ __forceinline__ int row_job(const VarParams& p, const Seq& s, int entry) const {
    const int i = seq[entry] & 0xffff;
    return whole() ? i : s.row_jobs(p, width) - 1 - i;
  }
};
static_assert(2 * MIN_STEPS_ROWS >= MIN_STEPS, "may_cut goes by the key tiles of a pair");
static_assert(MAX_SEQ <= 1 << 15 && MAX_TABLE <= 1 << 16, "an entry's sequence and row job share a word");

// Pieces of a job of so many steps, at most `share` each but for a rounding: in fp32, a
// share above a thousand steps may be passed by one. The same numbers everywhere.
__device__ __forceinline__ int pieces_of(int steps, int share, int cut_above) {
  return steps > cut_above
             ? static_cast<int>(ceilf(__fdividef(static_cast<float>(steps), static_cast<float>(share)) - 1e-3f))
             : 1;
}
__device__ __forceinline__ int pieces_of(const Plan& pl, int steps) { return pieces_of(steps, pl.share, pl.cut_above); }

// The plan's larger parts (block_excl_scan, count_jobs, cut_longest, plan_sort, list_joints) are calls of their own,
// made before the warpgroups share out their registers only: setmaxnreg does not know
// a callee's need.

// A CTA's unit of work: query tiles j0 (and j0 + 1 of a pair) of a sequence and
// a key head over the key tiles [t0, t1).
struct Item {
  int more;  // 0: the CTA has no further item
  int q0, lq, k0, lk;
  int hk, j0, pair;
  int t0, t1;
  int n0, n1;  // steps of the two warpgroups
  int slot;    // of a piece; -1: the whole job
};

// The key tile of step s of warpgroup i.
__device__ __forceinline__ int item_tile(int pair, int t0, int i, int s) { return pair ? t0 + s : t0 + 2 * s + i; }

// Item t: of the items of row job i of a sequence (c steps, `pieces` pieces), number r.
__device__ __forceinline__ void make_item(const VarParams& p, Item* out, const Seq& s, int width, int i, int c, int pieces,
                                          int r, int t) {
  Item it;
  it.hk = pieces == 1 ? r : static_cast<int>(static_cast<uint32_t>(r) / static_cast<uint32_t>(pieces));
  const int piece = r - it.hk * pieces;
  it.more = 1;
  it.q0 = s.q0;
  it.lq = s.lq;
  it.k0 = s.k0;
  it.lk = s.lk;
  it.j0 = width * i;
  it.pair = width == 2 && 2 * i + 1 < s.tiles(p);
  int u0 = 0, u1 = c;
  if (pieces > 1) {  // (a piece begins where the one before it ends: the same product)
    const float each = __fdividef(static_cast<float>(c), static_cast<float>(pieces));
    u0 = static_cast<int>(static_cast<float>(piece) * each);
    if (piece + 1 < pieces) u1 = static_cast<int>(static_cast<float>(piece + 1) * each);
  }
  const int nkv0 = s.key_tiles(p, it.j0);
  if (it.pair) {
    it.t0 = u0;
    it.t1 = u1;
    it.n0 = max(0, min(u1, nkv0) - u0);
    it.n1 = u1 - u0;
  } else {
    it.t0 = 2 * u0;
    it.t1 = min(nkv0, 2 * u1);
    it.n1 = (it.t1 - it.t0) / 2;
    it.n0 = it.t1 - it.t0 - it.n1;
  }
  it.slot = pieces > 1 ? t : -1;
  *out = it;
}

// Sum of v over the CTA's threads before this one, and of all (*total): `tot` is a word per
// warp that no other call is using.
__device__ __noinline__ int block_excl_scan(int v, int* tot, int* total) {
  const int incl = warp_incl_scan(v), w = warp_id();
  if (lane_id() == 31) tot[w] = incl;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < THREADS / 32; ++i) {
    const int t = tot[i];
    before += i < w ? t : 0;
    all += t;
  }
  *total = all;
  return before + incl - v;
}

// Between which shares of few jobs (J < G) the one is looked for; the share of many.
struct Shares {
  int lo, hi;
};
__device__ __forceinline__ Shares shares_of_few(float T, int most, int J, int G, int least_piece) {
  const int each = static_cast<int>(__fdividef(static_cast<float>(G), static_cast<float>(J)) + 1e-3f);  // floor(G / J)
  const int hi = max(least_piece, min(static_cast<int>(__fdividef(T, static_cast<float>(G - J))) + 1,
                                    static_cast<int>(__fdividef(static_cast<float>(most), static_cast<float>(each))) + 1));
  return {max(least_piece, min(hi, static_cast<int>(__fdividef(T, static_cast<float>(G))) + 1)), hi};
}
__device__ __forceinline__ int share_of_many(float T, float J, int G, int least_piece) {
  return max(least_piece, static_cast<int>(__fdividef(T + J * ITEM_STEPS, static_cast<float>(G))) + 1 - ITEM_STEPS);
}

// Whether few jobs (J < G) are dealt out like many: where they are at least half of the CTAs, one
// item for each may leave too few pieces for the longest. Of single tokens only, whose
// items cost little beside their steps: 16 of them over 1 to 32768 keys, 8 key heads of 64,
// 97 us and 69 so, 10 over 64 to 16000 keys, whose share is near the even one,
// 39 us and 49; prompts of 8 to 2500 tokens 24 us and 39.
__device__ __forceinline__ bool deal_few(float T, int share, int J, int G, int least_piece) {
  return least_piece == MIN_STEPS_ROWS && 2 * J >= G && static_cast<float>(share) * static_cast<float>(G) > 1.2f * T + static_cast<float>(2 * ITEM_STEPS * G);
}

// Tiles per job at most, for so many tiles (of one head; counted up to MANY_TILES per
// sequence or thread) whose longest sequence has lk keys. Jobs without a causal order
// are of one length: singles only fill idle CTAs there. (Up to four tiles per CTA: prompts
// of up to 2251 tokens 55 us in pairs and 51 in singles, but of up to 1021, where the
// items' own time counts, 24 and 31.)
constexpr int MANY_TILES = 1 << 16;
__device__ __forceinline__ int job_width(const VarParams& p, int tiles, int lk) {
  const int per_cta = !p.causal ? 1 : lk >= 16 * BKV ? 4 : 2;
  return static_cast<long long>(tiles) * p.kv_heads <= per_cta * p.grid ? 1 : 2;
}
__device__ __forceinline__ int min_steps(const VarParams& p, int lq) {
  return lq * static_cast<long long>(p.group) <= FEW_ROWS ? MIN_STEPS_ROWS : MIN_STEPS;
}

// What plan_build needs for itself.
constexpr int PLAN_PER = (MAX_TABLE + THREADS - 1) / THREADS;
struct PlanScratch {
  Seq of[32];       // up to 32 sequences
  int least_piece;  // of theirs
  int lk;           // the longest one's keys
  int tot[4][THREADS / 32];
  int sum[THREADS / 32], most[THREADS / 32], least[THREADS / 32], count[THREADS / 32], cut[THREADS / 32];
  int seq[MAX_TABLE], steps[MAX_TABLE], rank[MAX_TABLE];  // in the order of the sequences
  int hist[BUCKETS * PLAN_PER * (THREADS / 32)];          // [bucket][round, warp]
};

// The plan of up to 32 row jobs of up to 32 sequences, by one warp without a barrier: a lane per
// sequence, then per row job. (The CTA's way to the same plan takes barriers and shared memory:
// 32 single tokens over 100 keys each, one key head of 128, 8.0 us, 33 of them 10.5.) More row
// jobs than that: it leaves what it knows of the sequences.
constexpr int MANY_JOBS = 1 << 25;  // of a sequence: not counted exactly here
__device__ __forceinline__ void plan_small(const VarParams& p, Plan& pl, PlanScratch& sc, Item* own, int t_own) {
  constexpr uint32_t ALL = 0xffffffffu;
  const int lane = lane_id();
  Seq s = {0, 0, 0, 0};
  if (lane < p.B) s = sequence(p, lane);
  const int lk = __reduce_max_sync(ALL, s.lk);
  const int width = job_width(p, __reduce_add_sync(ALL, min(s.tiles(p), MANY_TILES)), lk);
  const int least_piece = min_steps(p, __reduce_max_sync(ALL, s.lq));
  const int mine = min(s.row_jobs(p, width), MANY_JOBS), incl = warp_incl_scan(mine), first = incl - mine;
  const int U = __shfl_sync(ALL, incl, 31);
  if (lane == 0) {
    pl.jobs = U;
    pl.width = width;
  }
  if (U > 32) {
    if (lane < p.B) {
      pl.first[lane] = first;
      sc.of[lane] = s;
    }
    if (lane == 0) {
      sc.least_piece = least_piece;
      sc.lk = lk;
      pl.first[p.B] = U;
      pl.n_items = U * p.kv_heads;  // (of a plan without a table)
      pl.n_cut = 0;
      pl.share = pl.cut_above = 0x7fffffff;
    }
    return;
  }
  int b = 0;  // the sequence of row job `lane`: the sequences that end at or before it
#pragma unroll
  for (int step = 16; step >= 1; step >>= 1)
    if (__shfl_sync(ALL, incl, b + step - 1) <= lane) b += step;
  b = min(b, 31);
  const int i = lane - __shfl_sync(ALL, first, b);
  const Seq q = {__shfl_sync(ALL, s.q0, b), __shfl_sync(ALL, s.lq, b), __shfl_sync(ALL, s.k0, b),
                 __shfl_sync(ALL, s.lk, b)};
  const bool in = lane < U;
  const int c = in ? q.steps(p, width, q.tiles(p), i) : 0;
  const float T = static_cast<float>(__reduce_add_sync(ALL, c)) * static_cast<float>(p.kv_heads);
  const int most = __reduce_max_sync(ALL, c), least = __reduce_min_sync(ALL, in ? c : 0x7fffffff);
  const int G = p.grid;
  bool few = U * static_cast<long long>(p.kv_heads) < G;
  int share = most, cut_above = most;
  if (p.may_cut && few && most > least_piece) {
    const Shares r = shares_of_few(T, most, U * p.kv_heads, G, least_piece);
    const int tried = r.lo + (r.hi - r.lo) * lane / 31;
    const float inv = __fdividef(1.0f, static_cast<float>(tried));
    const float cf = static_cast<float>(c);
    float n = 0.f;
#pragma unroll 8
    for (int j = 0; j < U; ++j) n += ceilf(fmaf(__shfl_sync(ALL, cf, j), inv, -1e-3f));
    share = cut_above = min(most, __reduce_min_sync(ALL, n * static_cast<float>(p.kv_heads) <= static_cast<float>(G) ? tried : r.hi));
    few = !deal_few(T, share, U * p.kv_heads, G, least_piece);
  }
  if (p.may_cut && !few) {
    share = min(most, share_of_many(T, static_cast<float>(U) * static_cast<float>(p.kv_heads), G, least_piece));
    cut_above = min(most, share + ITEM_STEPS);
  }
  const int pieces = pieces_of(c, share, cut_above), n = in ? pieces * p.kv_heads : 0;
  int at = lane, run = 0;  // the entry, and the items before it
  if (!few && most > least) {
    at = 0;
#pragma unroll 8
    for (int j = 0; j < U; ++j) {
      const int cj = __shfl_sync(ALL, c, j), nj = __shfl_sync(ALL, n, j);
      const bool before = cj > c || (cj == c && j < lane);
      at += before;
      run += before ? nj : 0;
    }
  } else {
    run = warp_incl_scan(n) - n;
  }
  if (in) {
    pl.seq[at] = b << 16 | i;
    pl.steps[at] = c;
    pl.items[at] = run;
    if (t_own >= run && t_own < run + n) make_item(p, own, q, width, i, c, pieces, t_own - run, t_own);
  }
  const int total = __reduce_add_sync(ALL, n), cut = __reduce_max_sync(ALL, pieces > 1 ? at + 1 : 0);
  if (lane == 0) {
    pl.n_items = total;
    pl.n_cut = cut;
    pl.share = share;
    pl.cut_above = cut_above;
  }
}

// Longest first by bucket, in the sequences' order within one: the rank among a
// warp's lanes, then a scan over all warps' counts.
__device__ __noinline__ void plan_sort(Plan& pl, PlanScratch& s, int U, int most, int cut_above) {
  constexpr int WARPS = THREADS / 32;
  static_assert(BUCKETS * WARPS == THREADS, "a count per thread and round");
  const int tid = threadIdx.x, warp = warp_id(), lane = lane_id();
  const int rounds = (U + THREADS - 1) / THREADS, rows = rounds * WARPS;
#pragma unroll 1
  for (int k = 0; k < rounds; ++k) s.hist[k * THREADS + tid] = 0;
  __syncthreads();
  auto bucket_of = [&](int c) {
    const bool cut = c > cut_above;
    const float top = static_cast<float>(cut ? most : cut_above);
    return (cut ? 15 : 31) - min(15, static_cast<int>(static_cast<float>(c - 1) * __fdividef(16.0f, top)));
  };
#pragma unroll 1
  for (int k = 0; k * THREADS < U; ++k) {
    const int u = k * THREADS + tid;
    const int bucket = u < U ? bucket_of(s.steps[u]) : BUCKETS;
    const uint32_t same = __match_any_sync(0xffffffffu, bucket);
    const int rank = __popc(same & ((1u << lane) - 1u));
    if (u < U) s.rank[u] = rank;
    if (u < U && rank == 0) s.hist[bucket * rows + k * WARPS + warp] = __popc(same);
  }
  __syncthreads();
  int mine = 0, total;  // thread i has the counts [i * rounds, (i + 1) * rounds)
#pragma unroll 1
  for (int i = 0; i < rounds; ++i) mine += s.hist[tid * rounds + i];
  int run = block_excl_scan(mine, s.tot[2], &total);
#pragma unroll 1
  for (int i = 0; i < rounds; ++i) {
    const int h = s.hist[tid * rounds + i];
    s.hist[tid * rounds + i] = run;
    run += h;
  }
  __syncthreads();
#pragma unroll 1
  for (int k = 0; k * THREADS < U; ++k) {
    const int u = k * THREADS + tid;
    if (u >= U) break;
    const int at = s.hist[bucket_of(s.steps[u]) * rows + k * WARPS + warp] + s.rank[u];
    pl.seq[at] = s.seq[u];
    pl.steps[at] = s.steps[u];
  }
  __syncthreads();
}

// The sequences' row jobs, counted by all threads: pl.first, pl.jobs, pl.width; the plan without a table. False
// where the offsets make no sense; ends with a barrier.
__device__ __noinline__ bool count_jobs(const VarParams& p, Plan& pl, PlanScratch& s) {
  constexpr int WARPS = THREADS / 32;
  const int tid = threadIdx.x, warp = warp_id(), lane = lane_id();
  // row jobs before each sequence
  int before = 0, total, tiles = 0, lk = 0, lq = 0;
  long long all = 0;
#pragma unroll 1
  for (int b = tid; b < p.B; b += THREADS) {
    const Seq q = sequence(p, b);
    all += q.tiles(p);
    tiles = min(tiles + min(q.tiles(p), MANY_TILES), MANY_TILES);
    lk = max(lk, q.lk);
    lq = max(lq, q.lq);
  }
  constexpr uint32_t ALL = 0xffffffffu;
  lk = __reduce_max_sync(ALL, lk);
  lq = __reduce_max_sync(ALL, lq);
  tiles = __reduce_add_sync(ALL, tiles);
  int many = __reduce_add_sync(ALL, static_cast<int>(all >> 12));
  if (lane == 0) {
    s.sum[warp] = lk;
    s.most[warp] = lq;
    s.count[warp] = tiles;
    s.cut[warp] = many;
  }
  __syncthreads();
  // (lane w of each warp has warp w's)
  lk = __reduce_max_sync(ALL, lane < WARPS ? s.sum[lane] : 0);
  lq = __reduce_max_sync(ALL, lane < WARPS ? s.most[lane] : 0);
  tiles = __reduce_add_sync(ALL, lane < WARPS ? s.count[lane] : 0);
  many = __reduce_add_sync(ALL, lane < WARPS ? s.cut[lane] : 0);
  // Offsets that fall and rise again can name every row thousands of times, more jobs than an
  // int counts: then there are none. (In order they make at most a tile per row and one per
  // sequence. Counted in 4096s: the threads' sums are below 2^34, what is let through below 2^31.)
  if (many > static_cast<int>((static_cast<long long>(p.rows_q) + p.B) >> 12)) {
    if (tid == 0) pl.jobs = pl.n_items = pl.n_cut = 0;
    __syncthreads();
    return false;
  }
  const int width = job_width(p, tiles, lk), least_piece = min_steps(p, lq);
#pragma unroll 1
  for (int b0 = 0; b0 < p.B; b0 += THREADS) {
    const int b = b0 + tid;
    int n = 0;
    if (b < p.B) n = sequence(p, b).row_jobs(p, width);
    const int at = block_excl_scan(n, s.tot[(b0 / THREADS) & 1], &total);
    if (b < p.B) pl.first[b] = before + at;
    before += total;
  }
  const int U = before;
  if (tid == 0) {
    s.least_piece = least_piece;
    s.lk = lk;
    pl.first[p.B] = U;
    pl.jobs = U;
    pl.width = width;
    pl.n_items = U * p.kv_heads;  // (of a plan without a table)
    pl.n_cut = 0;
    pl.share = pl.cut_above = 0x7fffffff;
  }
  __syncthreads();
  return true;
}

// Of more row jobs than MAX_TABLE, those that are longer than a CTA's share by more than
// ITEM_STEPS: listed with their pieces. A sequence's jobs are of one length, or grow evenly
// towards its last one, which gives the steps of all of them closely enough for a share; the
// long ones are looked for from the last (which may be a single of half the steps of the pair
// before it). By all threads; ends with a barrier.
__device__ __noinline__ void cut_longest(const VarParams& p, Plan& pl, PlanScratch& s) {
  constexpr int WARPS = THREADS / 32;
  constexpr uint32_t ALL = 0xffffffffu;
  const int tid = threadIdx.x, warp = warp_id(), lane = lane_id(), width = pl.width, G = p.grid;
  const float J = static_cast<float>(pl.jobs) * static_cast<float>(p.kv_heads);
  // (what nothing can be longer than, if each had a single step: 1100 tokens over up to 200 keys 39.6 us without, 38.8 so)
  if ((s.lk + BKV - 1) / BKV <= share_of_many(J, J, G, s.least_piece) + ITEM_STEPS) return;
  float T = 0.f;
  int most = 0;
#pragma unroll 1
  for (int b = tid; b < p.B; b += THREADS) {
    const Seq q = sequence(p, b);
    const int nt = q.tiles(p), n = q.row_jobs(p, width);
    if (n == 0) continue;
    const int last = q.steps(p, width, nt, n - 1);
    most = max(most, last);
    T += static_cast<float>(last);
    if (n == 1) continue;
    const int before = q.steps(p, width, nt, n - 2);
    most = max(most, before);
    // (the first ones of more queries than keys see nothing, and are of one step)
    const int none = p.causal ? min(n - 2, max(0, q.lq - q.lk) / (width * p.tpt)) : 0;
    T += static_cast<float>(none) + 0.5f * static_cast<float>(n - 1 - none) * static_cast<float>(q.steps(p, width, nt, none) + before);
  }
#pragma unroll
  for (int off = 16; off >= 1; off >>= 1) T += __shfl_xor_sync(ALL, T, off);
  most = __reduce_max_sync(ALL, most);
  if (lane == 0) {
    s.sum[warp] = __float_as_int(T);
    s.most[warp] = most;
  }
  __syncthreads();
  T = lane < WARPS ? __int_as_float(s.sum[lane]) : 0.f;
#pragma unroll
  for (int off = 8; off >= 1; off >>= 1) T += __shfl_xor_sync(ALL, T, off);
  T = fminf(__shfl_sync(ALL, T, 0) * static_cast<float>(p.kv_heads), 1e9f * static_cast<float>(G));
  most = __reduce_max_sync(ALL, lane < WARPS ? s.most[lane] : 0);
  const int share = share_of_many(T, J, G, s.least_piece), cut_above = share + ITEM_STEPS;
  if (most <= cut_above) return;  // (the plan is written by no thread, and s by none behind the barrier)
  int listed = 0, total;
#pragma unroll 1
  for (int b0 = 0; b0 < p.B; b0 += THREADS) {
    const int b = b0 + tid;
    Seq q = {0, 0, 0, 0};
    if (b < p.B) q = sequence(p, b);
    const int nt = q.tiles(p), n = q.row_jobs(p, width);
    const int skip = n > 0 && q.steps(p, width, nt, n - 1) <= cut_above ? 1 : 0;
    int longs = 0;
#pragma unroll 1
    while (longs + skip < n && longs <= MAX_TABLE && q.steps(p, width, nt, n - 1 - skip - longs) > cut_above) ++longs;
    const int at = listed + block_excl_scan(longs, s.tot[(b0 / THREADS) & 1], &total);
    listed += total;
#pragma unroll 1
    for (int e = 0; e < longs && at + e < MAX_TABLE; ++e) {
      pl.seq[at + e] = b << 16 | (skip + e);
      pl.steps[at + e] = q.steps(p, width, nt, n - 1 - skip - e);
    }
  }
  if (listed > MAX_TABLE) return;
  __syncthreads();
  int mine = 0;
  const int at0 = min(listed, tid * PLAN_PER), at1 = min(listed, at0 + PLAN_PER);
#pragma unroll 1
  for (int at = at0; at < at1; ++at) mine += pieces_of(pl.steps[at], share, cut_above) * p.kv_heads;
  int run = block_excl_scan(mine, s.tot[3], &total);
#pragma unroll 1
  for (int at = at0; at < at1; ++at) {
    pl.items[at] = run;
    run += pieces_of(pl.steps[at], share, cut_above) * p.kv_heads;
  }
  // (as in the table fewer than 2G, T being what it is, but the workspace has no more)
  if (tid == 0 && total <= SLOTS_PER_CTA * G) {
    pl.n_items = total + pl.jobs * p.kv_heads;
    pl.n_cut = listed;
    pl.share = share;
    pl.cut_above = cut_above;
  }
  __syncthreads();
}

// By all threads; ends with a barrier. The thread that finds item t_own among the listed
// ones writes it to *own. The warp that makes a plan of up to 32 jobs calls `made` before the others
// go on and `ahead` beside them, lane 0 both; then the result is true.
template <typename Made, typename Ahead>
__device__ __forceinline__ bool plan_build(const VarParams& p, Plan& pl, PlanScratch& s, Item* own, int t_own, Made made, Ahead ahead) {
  constexpr int WARPS = THREADS / 32;
  const int tid = threadIdx.x, warp = warp_id(), lane = lane_id();
  bool known = false;  // the sequences' row jobs are counted
  if (p.B <= 32) {
    if (warp == PRODUCER_WARP) {
      plan_small(p, pl, s, own, t_own);
      __syncwarp();
      if (lane == 0 && pl.jobs <= 32) made();
      __syncwarp();
      asm volatile("bar.arrive 3, %0;" ::"n"(THREADS) : "memory");
      if (pl.jobs <= 32) {
        if (lane == 0) ahead();
        __syncwarp();
        return true;
      }
    } else {
      asm volatile("bar.sync 3, %0;" ::"n"(THREADS) : "memory");
      if (pl.jobs <= 32) return true;
    }
    known = pl.jobs < MANY_JOBS;
  }
  if (!known) {
    __syncthreads();  // (pl.jobs is written again)
    if (!count_jobs(p, pl, s)) return false;
  }
  const int U = pl.jobs, width = pl.width, least_piece = s.least_piece;
  if (U > MAX_TABLE && p.may_cut) cut_longest(p, pl, s);
  if (U > MAX_TABLE || U == 0) return false;
  int total;
  // the row jobs' steps
  int sum = 0, most = 0, least = 0x7fffffff;
#pragma unroll 1
  for (int u = tid; u < U; u += THREADS) {
    int lo = 0, hi = p.B;  // the last sequence that begins at or before u
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (pl.first[mid] <= u) lo = mid;
      else hi = mid;
    }
    const int i = u - pl.first[lo];
    const Seq q = known ? s.of[lo] : sequence(p, lo);
    const int c = q.steps(p, width, q.tiles(p), i);
    s.seq[u] = lo << 16 | i;
    s.steps[u] = c;
    sum += c;
    most = max(most, c);
    least = min(least, c);
  }
  sum = __reduce_add_sync(0xffffffffu, sum);  // (steps are below 2^24)
  most = __reduce_max_sync(0xffffffffu, most);
  least = __reduce_min_sync(0xffffffffu, least);
  if (lane == 0) {
    s.sum[warp] = sum;
    s.most[warp] = most;
    s.least[warp] = least;
  }
  __syncthreads();
  // (lane w of each warp has warp w's: fp32, a share that is off by its rounding is as good)
  float T = lane < WARPS ? static_cast<float>(s.sum[lane]) : 0.f;
#pragma unroll
  for (int off = 8; off >= 1; off >>= 1) T += __shfl_xor_sync(0xffffffffu, T, off);
  T = __shfl_sync(0xffffffffu, T, 0) * static_cast<float>(p.kv_heads);
  most = __reduce_max_sync(0xffffffffu, lane < WARPS ? s.most[lane] : 0);
  least = __reduce_min_sync(0xffffffffu, lane < WARPS ? s.least[lane] : 0x7fffffff);
  const int G = p.grid;
  bool few = U * static_cast<long long>(p.kv_heads) < G;
  int share = most, cut_above = most;
  if (p.may_cut && few && most > least_piece) {
    const int J = U * p.kv_heads;
    const Shares r = shares_of_few(T, most, J, G, least_piece);
    const int lo = r.lo, hi = r.hi;
    const int tried = lo + (hi - lo) * warp / (WARPS - 1);  // (the last one is hi)
    const float inv = __fdividef(1.0f, static_cast<float>(tried));
    int n = 0;
    for (int u = lane; u < U; u += 32) n += static_cast<int>(ceilf(static_cast<float>(s.steps[u]) * inv - 1e-3f));
    n = __reduce_add_sync(0xffffffffu, n) * p.kv_heads;
    if (lane == 0) s.count[warp] = n <= G ? tried : hi;
    __syncthreads();
    share = __reduce_min_sync(0xffffffffu, lane < WARPS ? s.count[lane] : hi);
    share = min(share, most);
    cut_above = share;
    few = !deal_few(T, share, J, G, least_piece);
  }
  if (p.may_cut && !few) {
    const float J = static_cast<float>(U) * static_cast<float>(p.kv_heads);
    share = min(most, share_of_many(T, J, G, least_piece));
    cut_above = min(most, share + ITEM_STEPS);
  }
  const bool sorted = !few && most > least;
  if (sorted) plan_sort(pl, s, U, most, cut_above);
  // items before each entry
  const int* steps = sorted ? pl.steps : s.steps;
  int mine = 0, cut = 0;
  const int per = U <= THREADS ? 1 : PLAN_PER, at0 = tid * per, at1 = min(U, at0 + per);
#pragma unroll 1
  for (int at = at0; at < at1; ++at) {
    const int c = steps[at], n = pieces_of(c, share, cut_above);
    if (n > 1) cut = at + 1;
    mine += n * p.kv_heads;
  }
  cut = __reduce_max_sync(0xffffffffu, cut);
  if (lane == 0) s.cut[warp] = cut;
  int run = block_excl_scan(mine, s.tot[3], &total);
#pragma unroll 1
  for (int at = at0; at < at1; ++at) {
    const int c = steps[at], n = pieces_of(c, share, cut_above);
    const int job = sorted ? pl.seq[at] : s.seq[at];
    pl.items[at] = run;
    if (!sorted) {
      pl.seq[at] = job;
      pl.steps[at] = c;
    }
    if (t_own >= run && t_own < run + n * p.kv_heads)
      make_item(p, own, known ? s.of[job >> 16] : sequence(p, job >> 16), width, job & 0xffff, c, n, t_own - run, t_own);
    run += n * p.kv_heads;
  }
  cut = __reduce_max_sync(0xffffffffu, lane < WARPS ? s.cut[lane] : 0);
  if (tid == 0) {
    pl.n_items = total;
    pl.n_cut = cut;
    pl.share = share;
    pl.cut_above = cut_above;
  }
  __syncthreads();
  return false;
}

// A cut job for the second kernel.
struct Joint {
  int q0, lq, lk, hk, tok0;  // tok0: the job's first token
  int slot, pieces;          // of the first piece
  int width;                 // tiles at most
};
struct Joints {
  int n;
  int unused[7];
  Joint job[SLOTS_PER_CTA * ATTN_MAX_CTAS];
};

// The cut jobs, listed for the second kernel by one CTA. (Each has at least two pieces.)
__device__ __noinline__ void list_joints(const VarParams& p, const Plan& pl) {
  if (threadIdx.x == 0) p.joints->n = 0;
  __syncthreads();
#pragma unroll 1
  for (int e = threadIdx.x; e < pl.n_cut * p.kv_heads; e += THREADS) {
    const int at = e / p.kv_heads, hk = e - at * p.kv_heads, n = pieces_of(pl, pl.steps[at]);
    if (n == 1) continue;
    const Seq s = sequence(p, pl.seq[at] >> 16);
    p.joints->job[atomicAdd(&p.joints->n, 1)] = {s.q0, s.lq, s.lk, hk, pl.width * pl.row_job(p, s, at) * p.tpt,
                                                 pl.items[at] + hk * n, n, pl.width};
  }
}

// ------------------------------------------------------------------- items --

// False where item t is nothing to do.
__device__ __forceinline__ bool item_at(const VarParams& p, const Plan& pl, int t, Item* out) {
  if (t >= pl.n_items) {
    out->more = 0;
    return true;
  }
  const int in_entries = pl.entry_items(p);
  if (t < in_entries) {
    int lo = 0, hi = pl.entries();
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (pl.items[mid] <= t) lo = mid;
      else hi = mid;
    }
    const int steps = pl.steps[lo];
    const Seq s = sequence(p, pl.seq[lo] >> 16);
    make_item(p, out, s, pl.width, pl.row_job(p, s, lo), steps, pieces_of(pl, steps), t - pl.items[lo], t);
    return true;
  }
  const int r = t - in_entries, v = r / p.kv_heads, u = pl.jobs - 1 - v;
  int lo = 0, hi = p.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pl.first[mid] <= u) lo = mid;
    else hi = mid;
  }
  const int i = u - pl.first[lo];
  const Seq s = sequence(p, lo);
  const int steps = s.steps(p, pl.width, s.tiles(p), i);
  if (steps > pl.cut_above) return false;
  make_item(p, out, s, pl.width, i, steps, 1, r - v * p.kv_heads, t);
  return true;
}

// Item k of CTA x of G, of n: every other round in reverse order; of few rounds the third
// instead of the fourth, as the first round's items differ the most. (Prompts of 64 to 4000
// tokens, 8 heads on 2, 2.4 rounds, 80 us and 73; one of 8192, 6.7 rounds, 365 and 374.)
__device__ __forceinline__ int item_index(int k, int x, int G, int n) {
  const bool forward = n <= 4 * G ? k == 0 || k == 3 : (k & 1) == 0;
  return forward ? k * G + x : (k + 1) * G - 1 - x;
}

// mbar_wait for what may take as long as whole items (up to 2^23 steps of 2 us each, of
// a sequence of 2^30 keys): the other roles' waits are of single steps, and raise `abort`
// within a second where something is wrong.
__device__ __forceinline__ bool mbar_wait_items(uint64_t* bar, uint32_t parity, volatile int* abort, int* err, int code) {
  const uint32_t a = smem_u32(bar);
  const uint64_t g0 = globaltimer_ns();
  while (!mbar_try_wait(a, parity)) {
    if (*abort) return false;
    if (globaltimer_ns() - g0 > 100 * HILO_WAIT_LIMIT_NS) {
      atomicExch(err, code);
      *abort = 1;
      return false;
    }
  }
  return true;
}

// -------------------------------------------------------------- 16-bit types --

template <bool F16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  if (F16) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  return pack_bf16x2(lo, hi);
}

// The exponent bits of both halves, and what carries an exponent of all ones (an
// infinity or a NaN) into the half's sign bit.
template <bool F16>
__device__ __forceinline__ uint32_t special16(uint32_t w) {
  return F16 ? ((w & 0x7C007C00u) + 0x04000400u) & 0x80008000u : ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
}

template <bool F16>
__device__ __forceinline__ float widen16(uint32_t half) {
  return F16 ? __half2float(__ushort_as_half(static_cast<unsigned short>(half))) : __uint_as_float(half << 16);
}

__device__ __forceinline__ void st_f32x8(float* p, const float* v) {
  asm volatile("st.global.v8.f32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
               "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "l"(p)
               : "memory");
}

__device__ __forceinline__ void st_b32x8(void* p, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
               "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "l"(p)
               : "memory");
}

// The first key tile that some row of the item does not see whole.
__device__ __forceinline__ int part_tile(const VarParams& p, const Item& it) {
  return (p.causal ? min(it.lk, max(0, it.j0 * p.tpt + it.lk - it.lq + 1)) : it.lk) / BKV;
}

constexpr int RING = 4;

// What the softmax warpgroups hand over, and the items.
struct Shared {
  float m1[BQ], l1[BQ];
  Item ring[RING];
  int ahead;       // K tiles of the first item that are on their way
  int special[2];  // an infinity or NaN was taken out of a value tile of the item (by its parity)
};

template <int HD>
struct Cfg {
  static constexpr int NBOX = HD / 64;               // boxes of 64 columns
  static constexpr int Q_BOX = BQ * 128, KV_BOX = BKV * 128;
  static constexpr int Q_BYTES = NBOX * Q_BOX, KV_BYTES = NBOX * KV_BOX;
  // Stages of K and of V. (Heads of 64, 32 single tokens over 8192 keys each, 8 key heads:
  // 103 us with two, 98 with four, 81% of HBM's rate.)
  static constexpr int STAGES = HD == 64 ? 4 : 2;
  // Q0 | Q1 | K.. | V.. (the plan's scratch before the first copy)
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_K = 2 * Q_BYTES;
  static constexpr int OFF_V = OFF_K + STAGES * KV_BYTES;
  static constexpr int DATA_BYTES = OFF_V + STAGES * KV_BYTES;
  static constexpr int OFF_X = DATA_BYTES + 384;  // barriers before it
  static constexpr int OFF_PLAN = OFF_X + static_cast<int>(sizeof(Shared));
  static constexpr int SMEM_BYTES = OFF_PLAN + static_cast<int>(sizeof(Plan)) + 1024;  // + alignment of the base
  // Tensor memory: S0 | S1 | O0 | O1, P_i over the first half of S_i; of heads of 64
  // there is room for a P_i of its own (S0 | S1 | P0 | P1 | O0 | O1).
  static constexpr bool OWN_P = HD == 64;
  static constexpr uint32_t COL_P = OWN_P ? 2 * BKV : 0, P_STEP = OWN_P ? BKV / 2 : BKV;
  static constexpr uint32_t COL_O = 2 * BKV + (OWN_P ? BKV : 0);
  static constexpr uint32_t TMEM_COLS = 512;
  static_assert(COL_O + 2 * HD <= TMEM_COLS, "tensor memory");
  static_assert(SMEM_BYTES <= 227 * 1024, "shared memory of a CTA");
  static_assert(sizeof(PlanScratch) <= DATA_BYTES, "the plan's scratch");
};

template <int HD, bool F16>
__global__ void __launch_bounds__(THREADS, 1)
    attn_var_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                    const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ VarParams p) {
  using C = Cfg<HD>;
  extern __shared__ unsigned char smem_raw[];
  // (an offset from smem_raw, so that accesses stay 32-bit shared-memory ones)
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::DATA_BYTES);
  uint64_t* q_full = bars + 0;
  uint64_t* s_full = bars + 1;    // [2] per softmax warpgroup
  uint64_t* p_full = bars + 3;    // [2] per softmax warpgroup
  uint64_t* o_done = bars + 5;    // [2] per softmax warpgroup
  uint64_t* s_free = bars + 7;    // [2] OWN_P: S_i is in registers, the next one may be formed
  uint64_t* drain = bars + 9;
  uint64_t* q_empty = bars + 10;  // every S product of an item done: Q may be reloaded
  uint64_t* it_full = bars + 11;  // [RING]
  uint64_t* it_empty = it_full + RING;
  uint64_t* k_full = it_empty + RING;
  uint64_t* k_empty = k_full + C::STAGES;
  uint64_t* v_full = k_empty + C::STAGES;
  uint64_t* v_empty = v_full + C::STAGES;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(v_empty + C::STAGES);
  static_assert((11 + 2 * RING + 4 * C::STAGES + 1) * 8 <= C::OFF_X - C::DATA_BYTES, "room for the barriers");
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  Shared& shr = *reinterpret_cast<Shared*>(smem + C::OFF_X);
  Plan& plan = *reinterpret_cast<Plan*>(smem + C::OFF_PLAN);
  int* err = &g_attn_var_err;
  auto sK = [&](int st) { return smem + C::OFF_K + st * C::KV_BYTES; };
  auto sV = [&](int st) { return smem + C::OFF_V + st * C::KV_BYTES; };
  auto sQ = [&](int i) { return smem + C::OFF_Q + i * C::Q_BYTES; };

  const int warp = warp_id(), lane = lane_id();
  if (warp == V_PRODUCER_WARP && lane == 0) {
    tma_prefetch_desc(&tm_q);
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  if (warp == PRODUCER_WARP && lane == 0) {
    mbar_init(q_full, 1);
    for (int i = 0; i < C::STAGES; ++i) {
      mbar_init(&k_full[i], 1);
      mbar_init(&k_empty[i], 1);
      mbar_init(&v_full[i], 1);
      mbar_init(&v_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&p_full[i], 4);
      mbar_init(&o_done[i], 1);
      mbar_init(&s_free[i], 4);
    }
    mbar_init(drain, 1);
    mbar_init(q_empty, 1);
    for (int i = 0; i < RING; ++i) {
      mbar_init(&it_full[i], 1);
      mbar_init(&it_empty[i], 3 + 8);  // two copy warps, the MMA warp, the softmax warps
    }
    *abort_flag = 0;
    shr.special[0] = shr.special[1] = 0;
    fence_mbar_init();
  }
  // the lengths may be the previous kernel's
  pdl_wait();
  pdl_trigger();
  if (warp == MMA_WARP) {  // (the others go on to the plan)
    tmem_alloc(tmem_slot, C::TMEM_COLS);
    tmem_relinquish();
  }
  auto copy_q = [&](const Item& it) {
    const int row0 = it.q0 + it.j0 * p.tpt, h0 = it.hk * p.group;
    mbar_arrive_expect_tx(q_full, static_cast<uint32_t>((it.pair ? 2 : 1) * C::NBOX * 128 * p.tpt * p.group));
#pragma unroll
    for (int j = 0; j < C::NBOX; ++j) {
      tma_load_3d(sQ(0) + j * C::Q_BOX, &tm_q, q_full, 64 * j, h0, row0);
      if (it.pair) tma_load_3d(sQ(1) + j * C::Q_BOX, &tm_q, q_full, 64 * j, h0, row0 + p.tpt);
    }
  };
  auto copy_tile = [&](const CUtensorMap* tm, unsigned char* dst, uint64_t* full, int hk, int row) {
    mbar_arrive_expect_tx(full, C::KV_BYTES);
#pragma unroll
    for (int j = 0; j < C::NBOX; ++j) tma_load_3d(dst + j * C::KV_BOX, tm, full, 64 * j, hk, row);
  };
  // The first item's Q and first K tiles leave as soon as a small plan is made, by the thread
  // that goes on with the Q and K copies (the plan has not used their shared memory then), and
  // nothing else waits for that: prompts of 1 to 1021 tokens 24.4 us and 23.4, a chunk of 113
  // and fewer tokens 9.0 and 8.6; plans of more jobs, which gain nothing, 0.5 more.
  tc_fence_before();
  const bool small = plan_build(p, plan, *reinterpret_cast<PlanScratch*>(smem), &shr.ring[0], blockIdx.x, [&] {
    mbar_arrive(&it_full[0]);  // the plan has left the first item in the ring
  }, [&] {
    shr.ahead = 0;
    if (static_cast<int>(blockIdx.x) >= plan.n_items) return;
    const Item& it = shr.ring[0];
    fence_proxy_async_smem();
    copy_q(it);
    const int n = min(it.t1 - it.t0, C::STAGES);
    for (int t = 0; t < n; ++t) copy_tile(&tm_k, sK(t), &k_full[t], it.hk, it.k0 + (it.t0 + t) * BKV);
    shr.ahead = n;
  });
  if (p.may_cut && blockIdx.x == gridDim.x - 1) list_joints(p, plan);  // (the CTA that is idle or has the least)
  const bool idle = static_cast<int>(blockIdx.x) >= plan.n_items;  // (uniform)
  if (!small) {
    if (threadIdx.x == 0 && plan.whole()) mbar_arrive(&it_full[0]);
    // the plan's scratch (generic proxy) before the first copy over it (async proxy)
    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
  }
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  if (idle) {
    if (warp == MMA_WARP) tmem_dealloc(tmem, C::TMEM_COLS);
    return;
  }
  // key tile number kt of the CTA: its stage and the parity of that stage's use
  auto kv_stage = [](uint32_t kt) { return static_cast<int>(kt & (C::STAGES - 1u)); };
  auto kv_phase = [](uint32_t kt) { return (kt / C::STAGES) & 1u; };
  auto it_wait = [&](uint32_t jn, int code) {
    return mbar_wait(&it_full[jn & (RING - 1)], (jn / RING) & 1u, abort_flag, err, DEV_TIMEOUT_ATTN + 256 * code);
  };
  if (warp >= 8) {
    setmaxnreg_dec<CONTROL_REGS>();
    if (warp == PRODUCER_WARP || warp == V_PRODUCER_WARP) {
      if (lane == 0) {
        // ---------------- TMA producers: Q and K tiles (warp 8), V tiles
        // (warp 10). Two threads, so that a K copy never queues behind a V
        // stage that is still being read, and the other way round.
        const bool kq = warp == PRODUCER_WARP;
        const int ahead = kq && small ? shr.ahead : 0;  // K tiles on their way
        const CUtensorMap* tm = kq ? &tm_k : &tm_v;
        // per stage (bit st): armed at least once, and the parity of the last arming
        uint32_t armed = (1u << ahead) - 1u, par = 0;
        bool q_armed = ahead > 0;
        uint32_t q_par = 0;
        bool ok = true;
        uint32_t kt = 0;
        uint64_t* full = kq ? k_full : v_full;
        uint64_t* empty = kq ? k_empty : v_empty;
        for (uint32_t jn = 0;; ++jn) {
          if (!it_wait(jn, 18)) {
            ok = false;
            break;
          }
          const Item& it = shr.ring[jn & (RING - 1)];
          if (!it.more) break;
          const int hk = it.hk, k0 = it.k0, t0 = it.t0, n = it.t1 - it.t0;
          if (kq && (jn > 0 || ahead == 0)) {
            // Q once the previous item's S products are done with it
            if (jn > 0 && !mbar_wait_items(q_empty, (jn - 1) & 1u, abort_flag, err, DEV_TIMEOUT_ATTN + 256 * 17)) {
              ok = false;
              break;
            }
            copy_q(it);
            q_armed = true;
            q_par = jn & 1u;
          }
          mbar_arrive(&it_empty[jn & (RING - 1)]);
          for (int t = jn == 0 ? ahead : 0; t < n; ++t) {
            const int st = kv_stage(kt + t);
            const uint32_t ph = kv_phase(kt + t);
            if (!mbar_wait(&empty[st], ph ^ 1u, abort_flag, err, DEV_TIMEOUT_ATTN + 256 * (kq ? 1 : 2))) {
              ok = false;
              break;
            }
            copy_tile(tm, kq ? sK(st) : sV(st), &full[st], hk, k0 + (t0 + t) * BKV);
            armed |= 1u << st;
            par = (par & ~(1u << st)) | (ph << st);
          }
          if (!ok) break;
          kt += static_cast<uint32_t>(n);
        }
        if (!ok) {
          // wait (bounded) for this thread's bulk copies in flight before the
          // CTA exits
          const uint64_t g0 = globaltimer_ns();
          const uint64_t lim = HILO_WAIT_LIMIT_NS / 4;
          if (q_armed)
            while (!mbar_try_wait(smem_u32(q_full), q_par) && globaltimer_ns() - g0 < lim) {
            }
          for (int st = 0; st < C::STAGES; ++st)
            if ((armed >> st) & 1u)
              while (!mbar_try_wait(smem_u32(&full[st]), (par >> st) & 1u) && globaltimer_ns() - g0 < lim) {
              }
        }
      }
    } else if (warp == MMA_WARP) {
      // ---------------- MMA issuer: the whole warp walks the schedule and
      // waits (descriptor words stay warp-uniform), one elected lane issues.
      const bool leader = elect_one();
      constexpr int FMT = F16 ? 0 : 1;
      constexpr uint32_t idesc_s = idesc_kind_f16(BQ, BKV, 0, 0, FMT);
      constexpr uint32_t idesc_o = idesc_kind_f16(BQ, HD, 0, 1, FMT);
      constexpr uint32_t Q16 = C::Q_BYTES >> 4, KV16 = C::KV_BYTES >> 4;
      const uint32_t base16 = smem_u32(smem) >> 4;
      const uint32_t q_lo = base16 + (C::OFF_Q >> 4) + sw128_lo_lbo(16);
      const uint32_t k_lo = base16 + (C::OFF_K >> 4) + sw128_lo_lbo(16);
      const uint32_t v_lo = base16 + (C::OFF_V >> 4) + sw128_lo_lbo(C::KV_BOX);
      constexpr uint32_t hi = sw128_hi(1024);
      // S_i = Q_qb K^T (K from stage kst)
      auto issue_s = [&](int i, int qb, int kst) {
        if (leader) {
          const uint32_t a = q_lo + static_cast<uint32_t>(qb) * Q16, b = k_lo + static_cast<uint32_t>(kst) * KV16;
#pragma unroll
          for (int k = 0; k < HD / 16; ++k) {
            const uint32_t qo = static_cast<uint32_t>((k >> 2) * C::Q_BOX + (k & 3) * 32) >> 4;
            const uint32_t ko = static_cast<uint32_t>((k >> 2) * C::KV_BOX + (k & 3) * 32) >> 4;
            umma_f16_w(tmem + BKV * i, a + qo, b + ko, hi, idesc_s, k > 0 ? 1u : 0u);
          }
          umma_commit(&s_full[i]);
        }
        __syncwarp();
      };
      // O_i (+)= P_i V: P_i from the first half of S_i's columns, V from stage vst
      auto issue_pv = [&](int i, int vst, bool acc, bool last) {
        if (leader) {
          const uint32_t b = v_lo + static_cast<uint32_t>(vst) * KV16;
#pragma unroll
          for (int k = 0; k < BKV / 16; ++k)
            umma_f16_tmem_a_w(tmem + C::COL_O + HD * i, tmem + C::COL_P + C::P_STEP * i + 8u * k, b + ((k * 2048) >> 4), hi, idesc_o,
                              (acc || k > 0) ? 1u : 0u);
          if (C::OWN_P || last) umma_commit(&o_done[i]);
        }
        __syncwarp();
      };
      auto commit = [&](uint64_t* bar) {
        if (leader) umma_commit(bar);
        __syncwarp();
      };
      bool ok = true;
      uint32_t kt = 0, sc0 = 0, sc1 = 0;
      for (uint32_t jn = 0;; ++jn) {
        if (!__all_sync(0xffffffffu, it_wait(jn, 19))) {
          ok = false;
          break;
        }
        const Item& it = shr.ring[jn & (RING - 1)];
        if (!it.more) break;
        const bool pair = it.pair;
        const int n0 = it.n0, n1 = it.n1, n = it.t1 - it.t0;
        __syncwarp();
        if (lane == 0) mbar_arrive(&it_empty[jn & (RING - 1)]);
        const int qb1 = pair ? 1 : 0;  // the Q buffer of warpgroup 1
        // key tile of step s of warpgroup i, counted from the CTA's first
        auto tile = [&](int i, int s) { return kt + static_cast<uint32_t>(pair ? s : 2 * s + i); };
        auto wait_k = [&](uint32_t t) {
          return mbar_wait_warp(&k_full[kv_stage(t)], kv_phase(t), abort_flag, err, DEV_TIMEOUT_ATTN + 256 * 4);
        };
        auto wait_v = [&](uint32_t t) {
          return mbar_wait_warp(&v_full[kv_stage(t)], kv_phase(t), abort_flag, err, DEV_TIMEOUT_ATTN + 256 * 6);
        };
        if (!mbar_wait_warp(q_full, jn & 1u, abort_flag, err, DEV_TIMEOUT_ATTN + 256 * 3) || !wait_k(kt)) {
          ok = false;
          break;
        }
        tc_fence_after();
        // the first S of each warpgroup; a pair shares its first key tile, a
        // single gives warpgroup 1 the second one
        if (n0 > 0) issue_s(0, 0, kv_stage(kt));
        if (pair) {
          issue_s(1, 1, kv_stage(kt));
          commit(&k_empty[kv_stage(kt)]);
        } else {
          commit(&k_empty[kv_stage(kt)]);
          if (n1 > 0) {
            if (!wait_k(kt + 1)) {
              ok = false;
              break;
            }
            tc_fence_after();
            issue_s(1, 0, kv_stage(kt + 1));
            commit(&k_empty[kv_stage(kt + 1)]);
          }
        }
        // S_i(s + 1) of a step whose S_i(s) has been taken
        auto next_s = [&](int i, int qb, int s, int n, uint32_t sc, bool waited) {
          if (s + 1 >= n) return true;
          const uint32_t t2 = tile(i, s + 1);
          if (!waited && !wait_k(t2)) return false;
          if (C::OWN_P) {
            if (!mbar_wait_warp(&s_free[i], (sc + s) & 1u, abort_flag, err, DEV_TIMEOUT_ATTN + 256 * 7)) return false;
            tc_fence_after();
          }
          // (without OWN_P no tcgen05 fence here: S reads only TMA-written Q and K, ordered
          // by their mbarrier, and it follows the PV block before it, whose fence
          // already ordered the softmax's TMEM accesses, in issue order)
          issue_s(i, qb, kv_stage(t2));
          if (!pair || i == 1) commit(&k_empty[kv_stage(t2)]);
          return true;
        };
        // P_i over S_i: PV_0(s), S_0(s+1), PV_1(s), S_1(s+1), where S_i(s+1) overwrites
        // P_i(s) only after PV_i(s), in issue order. P_i of its own: S_i(s+1) before
        // PV_i(s), as soon as S_i(s) is in registers, so that the softmax never waits
        // for two products in a row (images of 1111 to 4096 tokens, 16 heads of 64:
        // 132 us with P over S).
        const int nmax = n0 > n1 ? n0 : n1;
        if (nmax == 1) commit(q_empty);
        for (int s = 0; s < nmax && ok; ++s) {
          if (s < n0) {
            if (C::OWN_P && !next_s(0, 0, s, n0, sc0, false)) {
              ok = false;
              break;
            }
            const uint32_t t = tile(0, s);
            if (!mbar_wait2_warp(&p_full[0], (sc0 + s) & 1u, &v_full[kv_stage(t)], kv_phase(t), abort_flag, err,
                                 DEV_TIMEOUT_ATTN + 256 * 5, DEV_TIMEOUT_ATTN + 256 * 6)) {
              ok = false;
              break;
            }
            tc_fence_after();
            issue_pv(0, kv_stage(t), s > 0, s + 1 == n0);
            if (!pair) commit(&v_empty[kv_stage(t)]);
            if (!C::OWN_P && !next_s(0, 0, s, n0, sc0, false)) {
              ok = false;
              break;
            }
          }
          if (s < n1) {
            // a pair's second tile has at least the first one's steps, and where both
            // have one its key tiles are those that were waited for above
            if (C::OWN_P && !next_s(1, qb1, s, n1, sc1, pair && s + 1 < n0)) {
              ok = false;
              break;
            }
            const uint32_t t = tile(1, s);
            if (!mbar_wait_warp(&p_full[1], (sc1 + s) & 1u, abort_flag, err, DEV_TIMEOUT_ATTN + 256 * 8) ||
                ((!pair || s >= n0) && !wait_v(t))) {
              ok = false;
              break;
            }
            tc_fence_after();
            issue_pv(1, kv_stage(t), s > 0, s + 1 == n1);
            commit(&v_empty[kv_stage(t)]);
            if (!C::OWN_P && !next_s(1, qb1, s, n1, sc1, pair && s + 1 < n0)) {
              ok = false;
              break;
            }
          }
          if (s + 2 == nmax) commit(q_empty);  // the item's last S products are issued
        }
        if (!ok) break;
        sc0 += static_cast<uint32_t>(n0);
        sc1 += static_cast<uint32_t>(n1);
        kt += static_cast<uint32_t>(n);
      }
      // every issued MMA has completed before TMEM is freed, also after an
      // abort (so this wait ignores the abort flag; it is bounded by time)
      commit(drain);
      const uint64_t g0 = globaltimer_ns();
      while (!mbar_try_wait(smem_u32(drain), 0u)) {
        if (globaltimer_ns() - g0 > HILO_WAIT_LIMIT_NS) {
          if (leader) atomicExch(err, DEV_TIMEOUT_ATTN + 256 * 9);
          break;
        }
      }
      __syncwarp();
    } else if (warp == ITEM_WARP && lane == 0) {
      // ---------------- warp 11, one lane: the CTA's items, ahead of their use
      int k = plan.whole() ? 1 : 0;  // (of a whole table item 0 is there already)
      for (uint32_t jn = static_cast<uint32_t>(k);; ++jn) {
        const int slot = jn & (RING - 1);
        if (jn >= RING &&
            !mbar_wait_items(&it_empty[slot], ((jn - RING) / RING) & 1u, abort_flag, err, DEV_TIMEOUT_ATTN + 256 * 20))
          break;
        while (!item_at(p, plan, item_index(k, blockIdx.x, gridDim.x, plan.n_items), &shr.ring[slot])) ++k;
        ++k;
        mbar_arrive(&it_full[slot]);
        if (!shr.ring[slot].more) break;
      }
    }
  } else {
    setmaxnreg_inc<SOFTMAX_REGS>();
    // ---------------- softmax: warpgroup i = warps 4i..4i+3, TMEM lane quarter warp % 4
    const int i = warp >> 2;
    const int row = (warp & 3) * 32 + lane;
    const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + BKV * i + lane_off;
    const uint32_t tP = tmem + C::COL_P + C::P_STEP * i + lane_off;
    const uint32_t tO = tmem + C::COL_O + HD * i + lane_off;
    const uint32_t tO1 = tmem + C::COL_O + HD + lane_off;  // warpgroup 1's accumulator (single's merge)
    const int row_tok = row / p.group;            // the row's token in its tile
    bool ok = true;
    // sc: S phases of this warpgroup so far (one per step); oc*: o_done phases so
    // far (one per item in which a warpgroup has steps, or with OWN_P one per step);
    // kt: the running key tile
    uint32_t kt = 0, sc = 0, oc0 = 0, oc1 = 0;
    // the phase of o_done after a warpgroup's n steps of the item
    auto o_phase = [](uint32_t oc, int n) { return (C::OWN_P ? oc + static_cast<uint32_t>(n) - 1u : oc) & 1u; };
    // All softmax warps go on to an item together or not at all: a warp that gave up
    // a wait still meets the others at the barriers of its item.
    bool go = !bar_red_or(2, 256, !it_wait(0, 21));
    for (uint32_t jn = 0; go; ++jn) {
      const Item& it = shr.ring[jn & (RING - 1)];
      if (!it.more) break;
      const bool pair = it.pair;
      const int n = i ? it.n1 : it.n0, n1 = it.n1, t0 = it.t0, lk = it.lk;
      const int tok0 = (it.j0 + (pair ? i : 0)) * p.tpt;  // the tile's first token
      // keys that the row sees (rows without a token: as if all), the fewest that
      // a row of the warp sees, and the first key that some row of the tile does not
      int lim = lk, lim_warp, part0 = lk;
      if (p.causal) {
        const int off1 = lk - it.lq + 1;
        if (row_tok < p.tpt && tok0 + row_tok < it.lq) lim = min(lk, max(0, tok0 + row_tok + off1));
        part0 = min(lk, max(0, tok0 + off1));
      }
      lim_warp = __reduce_min_sync(0xffffffffu, lim);
      // Steps below `owned` use a value tile that the other warpgroup takes care of.
      const int owned = pair && i == 1 ? it.n0 : 0;
      float m = -INFINITY, l = 0.f;
      // Value tile t in shared memory: rows past the sequence (other tokens or stale data)
      // become zero, so that their zero probabilities add exactly 0; so do, a thread per
      // row, infinities and NaNs of keys that some row of the tile does not see, and the item
      // is marked. False when the wait for V gave up.
      auto take_out = [&](int t, uint32_t ktile) -> bool {
        if (!mbar_wait_warp(&v_full[kv_stage(ktile)], kv_phase(ktile), abort_flag, err, DEV_TIMEOUT_ATTN + 256 * 11))
          return false;
        unsigned char* vr = sV(kv_stage(ktile)) + row * 128;
        const int end = lk - t * BKV;  // rows past the sequence, eight lanes each
        if (end < (warp & 3) * 32 + 32) {
          unsigned char* v = sV(kv_stage(ktile)) + (lane & 7) * 16;
          const int r0 = (warp & 3) * 32 + (lane >> 3);
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (r0 + 4 * k >= end)
#pragma unroll
              for (int j = 0; j < C::NBOX; ++j)
                *reinterpret_cast<uint4*>(v + j * C::KV_BOX + (r0 + 4 * k) * 128) = make_uint4(0, 0, 0, 0);
          fence_proxy_async_smem();  // before the tensor core reads the tile
        }
        if (row < end && t * BKV + row >= part0) {
          auto word = [&](int c16) { return reinterpret_cast<uint4*>(vr + (c16 >> 3) * C::KV_BOX + (c16 & 7) * 16); };
          uint32_t any = 0;
#pragma unroll 4
          for (int c16 = 0; c16 < 8 * C::NBOX; ++c16) {
            const uint4 q = *word(c16);
            any |= (special16<F16>(q.x) | special16<F16>(q.y)) | (special16<F16>(q.z) | special16<F16>(q.w));
          }
          if (any) {
            shr.special[jn & 1u] = 1;
#pragma unroll 1
            for (int c16 = 0; c16 < 8 * C::NBOX; ++c16) {
              uint4 q = *word(c16);
              uint32_t* w = &q.x;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t bad = special16<F16>(w[e]);
                w[e] &= ~((bad & 0x8000u ? 0xFFFFu : 0u) | (bad & 0x80000000u ? 0xFFFF0000u : 0u));
              }
              *word(c16) = q;
            }
            fence_proxy_async_smem();
          }
        }
        return true;
      };
      // With P_i over S_i, S_i complete means every earlier MMA is too (PV_i of the
      // previous step included), so O_i can be rescaled and P_i written
      // without another wait. tcgen05.ld / tcgen05.st are warp-collective:
      // the whole warp rescales when any of its rows needs it (rows that do
      // not use alpha = 1)
      auto rescale_o = [&](bool rescale, float m_use) {
        if (__any_sync(0xffffffffu, rescale)) {
          const float alpha = rescale ? ex2(m - m_use) : 1.0f;
#pragma unroll 1
          for (int c = 0; c < HD / 32; ++c) {
            float o[32];
            tmem_ld32(tO + c * 32, o);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] *= alpha;
            tmem_st32(tO + c * 32, o);
          }
          l *= alpha;
        }
      };
      for (int s = 0; s < n && ok; ++s) {
        const int t = item_tile(pair, t0, i, s);
        const uint32_t ktile = kt + static_cast<uint32_t>(t - t0);
        // The wait for a value tile tells its arrival from the next but one only: the one
        // before it in its stage has to be there already. In a pair that is the tile
        // of two steps ago, whose PV is done: while the tensor core forms S, as in an item's first
        // step. In a single's others it is the step before's, whose PV is done once S is complete:
        // last of all, as V may come later than P (64 single tokens over 400 keys
        // 42.0 us with the wait ahead of P, 40.3 so, 37.1 with rows cleared by eight lanes each).
        const bool take = s >= owned && (t + 1) * BKV > part0, early = pair || s == 0;
        if (take && early && !take_out(t, ktile)) {
          ok = false;
          break;
        }
        if (!mbar_wait_warp(&s_full[i], (sc + s) & 1u, abort_flag, err, DEV_TIMEOUT_ATTN + 256 * 10)) {
          ok = false;
          break;
        }
        tc_fence_after();
        float sv[BKV];
#pragma unroll
        for (int c = 0; c < BKV / 32; ++c) tmem_ld32(tS + c * 32, sv + c * 32);
        tmem_ld_wait();
        if (C::OWN_P) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&s_free[i]);
        }
        // the keys that the row does not see, whatever their logits
        if ((t + 1) * BKV > lim_warp) {
          const int valid = lim - t * BKV;
#pragma unroll
          for (int j = 0; j < BKV; ++j) sv[j] = j < valid ? sv[j] : -INFINITY;
        }
        // row max and row sum with 8 independent partials combined by a tree
        float mx8[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) mx8[u] = -INFINITY;
#pragma unroll
        for (int j = 0; j < BKV; j += 16)
#pragma unroll
          for (int u = 0; u < 8; ++u) mx8[u] = fmax3(mx8[u], sv[j + u], sv[j + 8 + u]);
        const float mx = fmax3(fmax3(mx8[0], mx8[1], mx8[2]), fmax3(mx8[3], mx8[4], mx8[5]),
                               fmaxf(mx8[6], mx8[7]));
        const float m_tile = mx * p.scale_log2 - P_ABOVE_LOG2<F16>;
        bool rescale = false;
        float m_use = m;
        if (s == 0) {
          m_use = m_tile;
        } else if (m_tile > m + RESCALE_LOG2) {
          m_use = m_tile;
          rescale = true;
        }
        // a row that has seen nothing but -inf: its probabilities are exp(-inf) = 0
        const float shift = m_use == -INFINITY ? 0.f : -m_use;
        float ls8[8];
        const uint64_t sc2 = f2(p.scale_log2, p.scale_log2), nm2 = f2(shift, shift);
        uint64_t ls4[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) ls4[u] = 0ull;
#pragma unroll
        for (int c = 0; c < BKV / 2; ++c) {
          float a, a1;
          f2_split(f2_fma(f2(sv[2 * c], sv[2 * c + 1]), sc2, nm2), a, a1);
          a = ex2(a);
          a1 = ex2(a1);
          sv[2 * c] = a;
          sv[2 * c + 1] = a1;
          ls4[c & 3] = f2_add(ls4[c & 3], f2(a, a1));
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) f2_split(ls4[u], ls8[2 * u], ls8[2 * u + 1]);
        const float lsum =
            ((ls8[0] + ls8[1]) + (ls8[2] + ls8[3])) + ((ls8[4] + ls8[5]) + (ls8[6] + ls8[7]));
        // (OWN_P: the previous step's PV may still read P_i and write O_i)
        if (C::OWN_P && s > 0) {
          if (!mbar_wait_warp(&o_done[i], o_phase(i ? oc1 : oc0, s), abort_flag, err, DEV_TIMEOUT_ATTN + 256 * 12)) {
            ok = false;
            break;
          }
          tc_fence_after();
        }
        rescale_o(rescale, m_use);
        m = m_use;
        l += lsum;
        // P_i as 16-bit pairs (keys 2c, 2c+1 in column c), the A operand of the PV product: one
        // rounding each, which the product's operands cannot do without; the sum keeps 32 bits
#pragma unroll
        for (int h2 = 0; h2 < BKV / 64; ++h2) {
          float pk[32];
#pragma unroll
          for (int c = 0; c < 32; ++c)
            pk[c] = __uint_as_float(pack16<F16>(sv[64 * h2 + 2 * c], sv[64 * h2 + 2 * c + 1]));
          tmem_st32(tP + 32 * h2, pk);
        }
        if (take && !early && !take_out(t, ktile)) {
          ok = false;
          break;
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[i]);
      }
      // ---- output rows. A pair: warpgroup i writes its tile. A single:
      // warpgroup 1 hands its row maximum and sum to warpgroup 0, which merges
      // the two accumulators (each relative to its own maximum) and writes.
      const bool writer = pair || i == 0;
      const bool merge = !pair && n1 > 0;
      if (!pair) {
        if (i == 1) {
          shr.m1[row] = m;
          shr.l1[row] = l;
        }
        named_bar_sync(1, 256);
      }
      if (ok && writer) {
        bool done = n == 0 || mbar_wait_warp(&o_done[i], o_phase(i ? oc1 : oc0, n), abort_flag, err, DEV_TIMEOUT_ATTN + 256 * 14);
        if (merge)
          done = done && mbar_wait_warp(&o_done[1], o_phase(oc1, n1), abort_flag, err, DEV_TIMEOUT_ATTN + 256 * 15);
        ok = done;
        if (ok) {
          tc_fence_after();
          float a0 = 1.f, a1 = 0.f;
          if (merge) {
            const float m1 = shr.m1[row], l1 = shr.l1[row];
            const float mm = fmaxf(m, m1);
            a0 = m == mm ? 1.f : ex2(m - mm);  // (both -inf: 1)
            a1 = m1 == mm ? 1.f : ex2(m1 - mm);
            l = l * a0 + l1 * a1;
            m = mm;
          }
          const bool special = shr.special[jn & 1u] != 0;
          // The infinities and NaNs that were taken out of the value tiles, added to
          // 32 columns of the rows that see them.
          auto give_back = [&](int c, float* o) {
            const int first = max(t0, part_tile(p, it)) * BKV, last = min(lim, it.t1 * BKV);
            const uint16_t* v = static_cast<const uint16_t*>(p.v) + static_cast<long long>(it.hk) * p.v_head + 32 * c;
            for (int j = first; j < last; ++j) {
              const uint4* src = reinterpret_cast<const uint4*>(v + static_cast<long long>(it.k0 + j) * p.v_row);
#pragma unroll
              for (int u = 0; u < 4; ++u) {
                const uint4 q = __ldg(src + u);
                const uint32_t qs[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const uint32_t bad = special16<F16>(qs[e]);
                  if (bad & 0x8000u) o[8 * u + 2 * e] += widen16<F16>(qs[e] & 0xFFFFu);
                  if (bad & 0x80000000u) o[8 * u + 2 * e + 1] += widen16<F16>(qs[e] >> 16);
                }
              }
            }
          };
          if (it.slot >= 0) {
            // a piece: unnormalised rows, their maxima and sums
            const long long at = (static_cast<long long>(it.slot) * 2 + (pair ? i : 0)) * BQ + row;
            p.part_ml[at] = make_float2(m, n > 0 ? l : -1.f);  // -1: no rows (a sum is not below 0)
            if (n > 0) {
#pragma unroll 1
              for (int c = 0; c < HD / 32; ++c) {
                float o[32];
                tmem_ld32(tO + c * 32, o);
                if (merge) {
                  float o1[32];
                  tmem_ld32(tO1 + c * 32, o1);
                  tmem_ld_wait_regs(o);
                  tmem_ld_wait_regs(o1);
#pragma unroll
                  for (int j = 0; j < 32; ++j) o[j] = o[j] * a0 + o1[j] * a1;
                } else {
                  tmem_ld_wait_regs(o);
                }
                if (special) give_back(c, o);
                float* dst = p.part + ((at - row) * HD + (32 * c * BQ + 8 * row));
#pragma unroll
                for (int j = 0; j < 32; j += 8) st_f32x8(dst + j * BQ, o + j);
              }
            }
          } else {
            const float inv = lim == 0 ? 0.f : 1.0f / l;
            // normalised rows to 16 bits, each lane its own row, 32 bytes (whole sectors)
            // at a time. (Staged through shared memory for whole lines the rows left no
            // sooner, and Q, in whose place they were staged, could not be
            // loaded for the next item meanwhile: 2000 to 3000 cycles an item.)
            const bool token = row_tok < p.tpt && tok0 + row_tok < it.lq;
            uint16_t* dst = static_cast<uint16_t*>(p.out) + static_cast<long long>(it.q0 + tok0 + row_tok) * p.out_row +
                            static_cast<long long>(it.hk * p.group + (row - row_tok * p.group)) * p.out_head;
            auto store_chunk = [&](int c, const float* o) {
              uint32_t w[16];
#pragma unroll
              for (int j = 0; j < 16; ++j) w[j] = pack16<F16>(o[2 * j] * inv, o[2 * j + 1] * inv);
              if (!token) return;
              if (p.out_wide) {
                st_b32x8(dst + 32 * c, w);
                st_b32x8(dst + 32 * c + 16, w + 8);
              } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  reinterpret_cast<uint4*>(dst + 32 * c)[j] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
              }
            };
            if (!merge && !special) {
              // all of O's columns in flight before one wait (the softmax's
              // registers are free here)
              float o[HD];
#pragma unroll
              for (int c = 0; c < HD / 32; ++c) tmem_ld32(tO + c * 32, o + c * 32);
#pragma unroll
              for (int c = 0; c < HD / 32; ++c) tmem_ld_wait_regs(o + c * 32);
#pragma unroll
              for (int c = 0; c < HD / 32; ++c) store_chunk(c, o + c * 32);
            } else {
#pragma unroll 1
              for (int c = 0; c < HD / 32; ++c) {
                float o[32];
                tmem_ld32(tO + c * 32, o);
                if (merge) {
                  float o1[32];
                  tmem_ld32(tO1 + c * 32, o1);
                  tmem_ld_wait_regs(o);
                  tmem_ld_wait_regs(o1);
#pragma unroll
                  for (int j = 0; j < 32; ++j) o[j] = o[j] * a0 + o1[j] * a1;
                } else {
                  tmem_ld_wait_regs(o);
                }
                if (special) give_back(c, o);
                store_chunk(c, o);
              }
            }
          }
        }
      }
      // end of the item: in a single, warpgroup 1's accumulator has been read before
      // its next PV may overwrite it
      const int n0_all = it.n0, len = it.t1 - t0;
      if (threadIdx.x == 0) shr.special[(jn + 1) & 1u] = 0;  // (last read before the previous item's end)
      tc_fence_before();
      ok = ok && it_wait(jn + 1, 21);
      go = !bar_red_or(2, 256, !ok);
      if (!go) break;
      if (lane == 0) mbar_arrive(&it_empty[jn & (RING - 1)]);
      sc += static_cast<uint32_t>(n);
      oc0 += C::OWN_P ? static_cast<uint32_t>(n0_all) : n0_all > 0 ? 1u : 0u;
      oc1 += C::OWN_P ? static_cast<uint32_t>(n1) : n1 > 0 ? 1u : 0u;
      kt += static_cast<uint32_t>(len);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == MMA_WARP) {
    tc_fence_after();
    tmem_dealloc(tmem, C::TMEM_COLS);
  }
}

// -------------------------------------------------------------------- join --
//
// The pieces of the cut jobs, joined: o = sum_p 2^(m_p - M) O_p / sum_p 2^(m_p - M) l_p with
// M the largest m_p. As many CTAs per job as there are, a warp per row, a lane
// per four (two) columns; the pieces' maxima and sums are read 32 at a time, a
// lane each. Bound by the chain job, maxima, rows for single tokens, by L2 for whole tiles.

constexpr int JOIN_THREADS = 256;

template <int HD, bool F16>
__global__ void __launch_bounds__(JOIN_THREADS) attn_join_kernel(const __grid_constant__ VarParams p) {
  pdl_wait();
  pdl_trigger();
  constexpr int COLS = HD / 32;
  constexpr int WARPS = JOIN_THREADS / 32;
  const int warp = warp_id(), lane = lane_id();
  const int jobs = p.joints->n;
  if (jobs == 0) return;
  const int slices = max(1, static_cast<int>(gridDim.x) / jobs);
  for (int w = blockIdx.x; w < jobs * slices; w += gridDim.x) {
    const int job = w / slices, slice = w - job * slices;
    const Joint j = p.joints->job[job];
    const int rows = min(j.lq - j.tok0, j.width * p.tpt) * p.group;  // tokens with their heads
    for (int g = slice * WARPS + warp; g < rows; g += slices * WARPS) {
      const int tok = j.tok0 + g / p.group, h = g % p.group;
      const int tile = tok >= j.tok0 + p.tpt, r = g - tile * p.tpt * p.group;
      auto row_of = [&](int q) { return (static_cast<long long>(j.slot + q) * 2 + tile) * BQ + r; };
      float M = -INFINITY;
      for (int q = lane; q < j.pieces; q += 32) M = fmaxf(M, p.part_ml[row_of(q)].x);
#pragma unroll
      for (int off = 16; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
      float o[COLS] = {}, total = 0.f;
      for (int q0 = 0; q0 < j.pieces; q0 += 32) {
        float a = 0.f;
        bool there = false;  // the piece left rows; their weight may be 0, which leaves an infinity or a NaN a NaN
        if (q0 + lane < j.pieces) {
          const float2 ml = p.part_ml[row_of(q0 + lane)];
          there = !(ml.y < 0.f);
          if (there) {
            a = ml.x == M ? 1.f : ex2(ml.x - M);
            total = fmaf(a, ml.y, total);
          }
        }
        const uint32_t left = __ballot_sync(0xffffffffu, there);
        const int most = min(32, j.pieces - q0);
#pragma unroll 4
        for (int q = 0; q < most; ++q) {
          const float f = __shfl_sync(0xffffffffu, a, q);
          if (!(left >> q & 1u)) continue;
          const float* src = p.part + (row_of(q0 + q) - r) * HD + (lane * COLS / 8 * (8 * BQ) + 8 * r + lane * COLS % 8);
          if (COLS == 4) {
            const float4 v = *reinterpret_cast<const float4*>(src);
            o[0] = fmaf(f, v.x, o[0]);
            o[1] = fmaf(f, v.y, o[1]);
            o[COLS - 2] = fmaf(f, v.z, o[COLS - 2]);
            o[COLS - 1] = fmaf(f, v.w, o[COLS - 1]);
          } else {
            const float2 v = *reinterpret_cast<const float2*>(src);
            o[0] = fmaf(f, v.x, o[0]);
            o[1] = fmaf(f, v.y, o[1]);
          }
        }
      }
#pragma unroll
      for (int off = 16; off >= 1; off >>= 1) total += __shfl_xor_sync(0xffffffffu, total, off);
      const Seq s = {j.q0, j.lq, 0, j.lk};
      const float inv = s.seen(p, tok) == 0 ? 0.f : 1.0f / total;
      uint16_t* dst = static_cast<uint16_t*>(p.out) + static_cast<long long>(j.q0 + tok) * p.out_row +
                      static_cast<long long>(j.hk * p.group + h) * p.out_head + COLS * lane;
      if (COLS == 4)
        *reinterpret_cast<uint2*>(dst) =
            make_uint2(pack16<F16>(o[0] * inv, o[1] * inv), pack16<F16>(o[COLS - 2] * inv, o[COLS - 1] * inv));
      else
        *reinterpret_cast<uint32_t*>(dst) = pack16<F16>(o[0] * inv, o[1] * inv);
    }
  }
}

template <int HD, bool F16>
cudaError_t launch_hd(const hilo_attn_shape& s, const VarParams& p, const void* q, const void* k, const void* v,
                      int* launches, cudaStream_t st) {
  // k and v of no rows: any address will do, all keys are masked
  const bool none = s.rows_k == 0;
  const uint64_t rows_k = none ? 1 : s.rows_k;
  CUtensorMap tm_q, tm_k, tm_v;
  const uint64_t hd = HD;
  if (!encode_tmap_16bit_3d(&tm_q, q, hd, s.heads, s.rows_q, s.q_head, s.q_row, 64, p.group, p.tpt) ||
      !encode_tmap_16bit_3d(&tm_k, none ? q : k, hd, none ? 1 : s.kv_heads, rows_k, s.k_head, s.k_row, 64, 1, BKV) ||
      !encode_tmap_16bit_3d(&tm_v, none ? q : v, hd, none ? 1 : s.kv_heads, rows_k, s.v_head, s.v_row, 64, 1, BKV))
    return cudaErrorInvalidValue;
  auto* kern = attn_var_kernel<HD, F16>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<HD>::SMEM_BYTES);
  if (e != cudaSuccess) return e;
  // the register split must fit what the CTA is launched with, or the
  // softmax warpgroups' setmaxnreg.inc would wait for registers forever
  // (one number for every device: the library holds one binary)
  static std::atomic<int> known{0};
  int regs = known.load(std::memory_order_relaxed);
  if (regs == 0) {
    cudaFuncAttributes fa;
    e = cudaFuncGetAttributes(&fa, kern);
    if (e != cudaSuccess) return e;
    regs = fa.numRegs;
    known.store(regs, std::memory_order_relaxed);
  }
  if (static_cast<long long>(regs) * THREADS < 256LL * SOFTMAX_REGS + 128LL * CONTROL_REGS)
    return cudaErrorInvalidConfiguration;
  e = launch_pdl(kern, dim3(p.grid), dim3(THREADS), Cfg<HD>::SMEM_BYTES, st, tm_q, tm_k, tm_v, p);
  if (e != cudaSuccess) return e;
  *launches = 1;
  if (!p.may_cut) return cudaSuccess;
  auto* join = attn_join_kernel<HD, F16>;
  e = launch_pdl(join, dim3(p.grid), dim3(JOIN_THREADS), 0, st, p);
  if (e == cudaSuccess) *launches = 2;
  return e;
}

// Whether a job could have more steps than the smallest piece: a pair a step per key tile, a
// single half of that.
bool may_cut(const hilo_attn_shape& s) { return (s.rows_k + BKV - 1) / BKV > MIN_STEPS; }
constexpr size_t SLOTS = static_cast<size_t>(SLOTS_PER_CTA) * ATTN_MAX_CTAS;

}  // namespace

size_t attn_var_workspace_bytes(const hilo_attn_shape& s) {
  // (32 bytes to bring the rows onto the boundary that they are stored from)
  return may_cut(s) ? SLOTS * 2 * BQ * (static_cast<size_t>(s.head_dim) * sizeof(float) + sizeof(float2)) +
                          sizeof(Joints) + 32
                    : 32;
}

cudaError_t launch_attention_var(const hilo_attn_shape& s, const int32_t* cu_q, const int32_t* cu_k, const void* q,
                                 const void* k, const void* v, void* out, void* ws, int num_sms, int* launches,
                                 cudaStream_t st) {
  *launches = 0;
  VarParams p;
  p.cu_q = cu_q;
  p.cu_k = cu_k;
  p.v = v;
  p.out = out;
  p.part = reinterpret_cast<float*>((reinterpret_cast<uintptr_t>(ws) + 31) & ~static_cast<uintptr_t>(31));
  p.part_ml = reinterpret_cast<float2*>(p.part + SLOTS * 2 * BQ * s.head_dim);
  p.joints = reinterpret_cast<Joints*>(p.part_ml + SLOTS * 2 * BQ);
  p.v_row = s.v_row;
  p.v_head = s.v_head;
  p.out_row = s.out_row;
  p.out_head = s.out_head;
  p.B = s.B;
  p.kv_heads = s.kv_heads;
  p.group = s.heads / s.kv_heads;
  p.tpt = BQ / p.group;
  p.causal = s.causal;
  p.rows_q = s.rows_q;
  p.rows_k = s.rows_k;
  int log2 = 0;
  while ((1 << log2) < p.tpt) ++log2;
  p.tpt_shift = 31 + log2;  // 2^31 / 2^shift <= 1 / tpt: exact below 2^31
  p.tpt_mul = ((1ull << p.tpt_shift) + p.tpt - 1) / p.tpt;
  // a persistent grid: one CTA per SM; each takes its share of the items, whose
  // number is known on the device only
  p.grid = num_sms < 1 ? 1 : num_sms < ATTN_MAX_CTAS ? num_sms : ATTN_MAX_CTAS;
  p.may_cut = may_cut(s);
  p.out_wide = reinterpret_cast<uintptr_t>(out) % 32 == 0 && s.out_row % 16 == 0 && s.out_head % 16 == 0;
  const double scale = s.scale > 0.f ? s.scale : 1.0 / sqrt(static_cast<double>(s.head_dim));
  p.scale_log2 = static_cast<float>(1.4426950408889634 * scale);
  const bool f16 = s.dtype == HILO_F16;
  if (s.head_dim == 128)
    return f16 ? launch_hd<128, true>(s, p, q, k, v, launches, st) : launch_hd<128, false>(s, p, q, k, v, launches, st);
  return f16 ? launch_hd<64, true>(s, p, q, k, v, launches, st) : launch_hd<64, false>(s, p, q, k, v, launches, st);
}

int attn_var_take_device_error() {
  int v = 0, z = 0;
  if (cudaMemcpyFromSymbol(&v, g_attn_var_err, sizeof(int)) != cudaSuccess) return -1;
  if (v) cudaMemcpyToSymbol(g_attn_var_err, &z, sizeof(int));
  return v;
}

}  // namespace hilo
