// A projection shared by all rows with a low-rank adapter for each segment of them:
//   y = x W^T + bias + scale_e (x A_e^T) B_e^T,  e the adapter of the row's segment
//   out = act(y), or resid + gate * act(y)
//
// Segments of some length: t = scale_e x A_e^T is formed first (adapter_tc_kernel<true, ..>), and
// the product takes it as further K blocks, x W^T + t B_e^T in one accumulator
// (adapter_tc_kernel<false, ..>): two more K blocks for a rank of 64, no extra pass over the
// results. The tensor cores take bf16, so t enters as a sum of bf16 terms, each the rounding of what
// the ones before leave: two of them (2^-16 of t) for bf16 results, three (2^-24) for fp32 ones. A
// rank of 16 or 32 has its terms side by side in one K block, against the same columns of B_e.
// Many short segments (a token or a few rows each): padding every one to a tile's 16 rows and reading
// W's tiles from L2 once more for each would cost more than the adapters, so their part is formed by
// itself in fp32 (adapter_delta_kernel) while the product of all rows begins, whose epilogue adds it.
//
// Product in tiles, a cluster of two CTAs per tile of 256 weight rows x w rows of x of one segment
// (tcgen05, cta_group::2; weight rows are the MMA's M side, rows of x its N side, any multiple of 16
// up to 256): the scheme of the products grouped by expert, with the segments as groups.
//  * warp 0 loads weights, one TMA box of 128 rows x 64 k: W, then B_e (or A_e).
//  * warp 1 issues the MMAs, warps 2 and up of both CTAs run the epilogue.
//  * the last two warps load rows of x, then of t, a K block each by turns.
// fp32 results take K in parts of 4 blocks, each in an accumulator of its own, which the epilogue
// adds up (the tensor core's sums lose about 6e-8 of the result per K block of 64). So do results of
// a K past 2^17.
// Bounds: with many rows the tensor pipe under the power cap (24960 rows, 8960 x 1536, rank 64: 421 us, 1.7
// PFLOP/s, t's 26 among them). With one round of tiles a K block of 256 x 192 takes 590 clocks (1560 rows,
// 1536 x 8960, rank 32, fp32: 58 us), where the tensor pipe needs 384 and operands, 256 + 192 clocks, 448;
// what the others go to is not known, and other widths took no less in all. With few rows latency (see
// adapter_delta_kernel).
// Every wait is bounded (mbar_wait): a role that gives up records it and the kernel ends.
#include <atomic>
#include <climits>
#include <type_traits>

#include "grouped.cuh"
#include "kernels.h"

namespace {

constexpr int TMEM_COLS = 512;
constexpr int MAX_STAGES = 8, MAX_ACCS = 8;
// Warps: weight loader, MMA, epilogue, two row loaders. Sums in parts wait in the epilogue's registers,
// 64 a thread, so that twelve warps hold a tile of 192 rows (a K block costs 256 + w clocks of
// operands: the wider the better), where 128 registers are left to a thread.
template <bool PARTS>
struct Warps {
  static constexpr int EPI = PARTS ? 12 : 8, GROUPS = EPI / 4, LOAD = 2 + EPI, THREADS = 32 * (4 + EPI);
};
constexpr int MAX_S = FB_ADAPTER_MAX_SEGMENTS;
constexpr int SMEM_BYTES = 229888;  // of 232448 that a block may have
constexpr int EPI_TILE = 2048;      // an epilogue warp's tile: 32 tokens x 32 rows, bf16
constexpr int EPI_BYTES = 8 * 2 * EPI_TILE;
constexpr int TABLE_BYTES = (3 * (MAX_S + 8) * 4 + 127) / 128 * 128;
constexpr int BAR_BYTES = 512;
__host__ __device__ constexpr int ring_bytes(bool tiles) {
  return SMEM_BYTES - BAR_BYTES - TABLE_BYTES - (tiles ? EPI_BYTES : 0);
}
static_assert(ring_bytes(true) % 128 == 0, "TMA tiles lie on 128-byte boundaries");
constexpr int64_t BAND_BYTES = 16ll << 20;  // of weights before a segment's next rows (they stay in L2)
constexpr int PART_BLOCKS = 4;              // K blocks of one accumulator, for sums in parts
constexpr int F32_T = 192;                  // widest tile then
constexpr int LONG_K = 1 << 17;
bool in_parts(const AdapterArgs& g) { return g.out_type == FB_F32 || g.k > LONG_K; }

// How t's terms lie in a row of the scratch. Ranks up to 64 are rounded up to 16, the terms side by
// side; larger ones to 64, 64 columns of each term by turns. Either way K block i of t is columns 64 i
// and up, chunk j (16 columns) of it meets chunk (4 i + j) % chunks of B_e's box of 64 columns, and
// the box is i / terms (the only one for ranks up to 64). Chunks behind the last term are zeros, and meet
// the zeros behind B_e's last column.
struct Terms {
  int terms, rp, cols;  // rank as rounded up, columns of a row of t (whole K blocks)
  __host__ __device__ Terms(int rank, bool parts)
      : terms(parts ? 3 : 2), rp(rank > 64 ? (rank + 63) / 64 * 64 : (rank + 15) / 16 * 16),
        cols((terms * rp + 63) / 64 * 64) {}
  __host__ __device__ int blocks() const { return cols / 64; }
  __host__ __device__ int column(int term, int r) const {
    return rp <= 64 ? term * rp + r : (r / 64 * terms + term) * 64 + r % 64;
  }
};

// Tensor maps: W (or A_e) and B_e in boxes of 128 rows, x and t in boxes of 64, 32, 16 and 8 rows (a
// tile's half is a multiple of 8), results in boxes of 16 tokens.
struct Maps {
  CUtensorMap w, b, x[4], t[4], o;
};
struct TcArgs {
  int groups;               // segments, or (offsets null) one group of the first *end rows
  const int32_t *offsets, *end, *adapter;
  int adapters, rows, n, k; // n: weight rows
  int rank;
  bf16* t;                  // DOWN
  const float* scale;       // DOWN
  float* ws;                // parts of cut tiles (null: whole tiles only): two slots a cluster
  int* counters;            // [clusters][ADAPTER_COUNTERS], zero between launches
  const float *bias, *delta, *resid, *gate;
  int64_t ldr, ldo;
  int act, out_type;
  void* out;
};

// Tiles cut between clusters, where whole ones would leave clusters idle in the last round (t alone
// has few tiles): the clusters take equal stretches of the row of all tiles' K blocks, each weighted
// by its tile's clocks, and a stretch may begin within a tile, four blocks from its ends at least.
// Each cluster of a cut tile leaves its sums in the scratch; a counter tells who comes last, and
// that one adds them up, in cluster order. Nobody waits.
constexpr int MIN_BLOCKS = 4;
struct Cut {
  int on, clusters;         // clusters that work
  int t0, k0, t1, k1;       // this cluster's stretch: from block k0 of tile t0 to block k1 of tile t1
  unsigned u0, u1, units;   // where those tiles begin, all units
};
constexpr int WS_WARP = MAX_T / 2 * 32;  // floats of an epilogue warp's part, at most
constexpr size_t WS_SLOT = 2 * 12 * (size_t)WS_WARP;
constexpr int ADAPTER_COUNTERS = 2 * 12;  // of a cluster

// DOWN: t = scale x A_e^T (n = rank), else the product.
template <bool DOWN, bool PARTS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Warps<PARTS>::THREADS, 1)
    adapter_tc_kernel(const __grid_constant__ Maps maps, const TcArgs g, int* err) {
  constexpr int THREADS = Warps<PARTS>::THREADS, EPI = Warps<PARTS>::EPI, GROUPS = Warps<PARTS>::GROUPS;
  constexpr int LOAD = Warps<PARTS>::LOAD;
  constexpr bool TILES = !DOWN && !PARTS;  // results leave through shared-memory tiles
  extern __shared__ __align__(1024) uint8_t smem[];  // (operand tiles need the alignment)
  if ((smem_u32(smem) & 1023u) != 0) {
    if (threadIdx.x == 0) fb_report(err, FB_DEVERR_BAD_ARG);
    return;
  }
  constexpr int RING_BYTES = ring_bytes(TILES);
  uint8_t* epi_smem = smem + RING_BYTES;
  int* off = reinterpret_cast<int*>(smem + SMEM_BYTES - BAR_BYTES - TABLE_BYTES);
  int* first = off + MAX_S + 8;
  int* who = first + MAX_S + 8;  // a group's adapter
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + SMEM_BYTES - BAR_BYTES);
  uint64_t* empty = full + MAX_STAGES;
  uint64_t* tmem_full = empty + MAX_STAGES;
  uint64_t* tmem_empty = tmem_full + MAX_ACCS;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(tmem_empty + MAX_ACCS);
  uint32_t* gave_up = tmem_holder + 1;  // a role of this CTA gave up a wait
  int* bad = reinterpret_cast<int*>(tmem_holder + 2);
  int* width = bad + 1;
  unsigned* cost = reinterpret_cast<unsigned*>(width + 1);  // of each width, and its token tiles
  unsigned* count = cost + WIDTHS;
  __shared__ Cut cut;

  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t rank = cluster_ctarank();
  const int cluster = blockIdx.x >> 1, n_clusters = gridDim.x >> 1;
  const int n_ft = (g.n + 2 * W_ROWS - 1) / (2 * W_ROWS);  // (DOWN: 1)
  const int nk = (g.k + BK - 1) / BK, E = g.groups;
  const Terms terms(g.rank, PARTS);
  const int ext = g.adapter ? terms.blocks() : 0;
  const int chunks = terms.rp <= 64 ? terms.rp / 16 : 4, all_chunks = terms.terms * terms.rp / 16;
  bool failed = false;

  if (threadIdx.x == 0) {
    *gave_up = 0;
    *bad = 0;
    for (int s = 0; s < MAX_STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < MAX_ACCS; ++a) {
      mbar_init(&tmem_full[a], 1);
      mbar_init(&tmem_empty[a], 2 * EPI);  // the epilogue warps of both CTAs
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_desc(&maps.w);
    tma_prefetch_desc(&maps.x[0]);
    if (TILES) tma_prefetch_desc(&maps.o);
  }
  if (threadIdx.x >= 64 && threadIdx.x < 64 + 2 * WIDTHS) cost[threadIdx.x - 64] = 0;
  if (warp == 1) tmem_alloc_cg2(tmem_holder, TMEM_COLS);
  // (The product: all but t and the low-rank part was there before the kernel that forms them
  // began; whoever reads those waits for it. DOWN is the first of a call's kernels and overwrites
  // what the last call's read.)
  if (DOWN) griddep_wait();
  griddep_launch();
  // ---- the groups and the tile width ----
  __syncthreads();
  for (int i = threadIdx.x; i <= E; i += THREADS) {
    const int o = g.offsets ? g.offsets[i] : i ? *g.end : 0, p = i && g.offsets ? g.offsets[i - 1] : 0;
    off[i] = o;
    const int e = i < E && g.adapter ? g.adapter[i] : -1;
    who[i] = e;
    if (o < p || o > g.rows || (i == 0 && o != 0) || e < -1 || e >= g.adapters) *bad = 1;
  }
  __syncthreads();
  if (*bad) {  // (every CTA sees the same)
    if (threadIdx.x == 0) fb_report(err, FB_DEVERR_BAD_INDEX);
    for (int i = threadIdx.x; i <= E; i += THREADS) off[i] = 0;
    __syncthreads();
  }
  auto rows_of = [&](int e) { return DOWN && who[e] < 0 ? 0 : off[e + 1] - off[e]; };
  const int all_blocks = nk + (DOWN ? 0 : ext);  // K blocks of a tile whose rows have an adapter
  // a K block of group e's tiles in units of 32 clocks
  auto weight = [&](int e) -> unsigned {
    const int nt = first[e + 1] - first[e], w = nt ? (rows_of(e) + nt - 1) / nt : 0;
    return (unsigned)(256 + w > 313 ? 256 + w : 313) / 32;
  };
  auto units_of = [&](int e) { return (unsigned)((first[e + 1] - first[e]) * n_ft) * all_blocks * weight(e); };
  // where cluster c's stretch of `all` units begins: floor(c all / n)
  auto stretch = [](unsigned c, unsigned all, unsigned n) { return all / n * c + all % n * c / n; };
  {
    // (nt tiles of widths that add up to r: 256 nt + r, see below)
    const int c = threadIdx.x % WIDTHS, T = T_STEP * (c + 1);
    unsigned tiles = 0, clocks = 0;
    for (int e = threadIdx.x / WIDTHS; e < E; e += THREADS / WIDTHS) {
      const int r = rows_of(e), nt = (r + T - 1) / T;
      tiles += nt;
      clocks += 256 * nt + r > 313 * nt ? 256 * nt + r : 313 * nt;
    }
    if (tiles) {
      atomicAdd(&count[c], tiles);
      atomicAdd(&cost[c], clocks);
    }
  }
  __syncthreads();
  if (warp == 0) {
    // The width of the least estimated time in SM clocks: 256 + w clocks of operands, or 313 of
    // issue, per K block; in the fullest cluster each tile but the first takes its mainloop or its
    // epilogue. Lanes 16 and up: the same with tiles cut into equal stretches, at least 12 K blocks
    // a cluster, and what storing and adding up the last tile's parts takes.
    const int T = T_STEP * (lane % WIDTHS + 1);
    float est = 3e38f, ctas = n_clusters;
    if (!PARTS || T <= F32_T) {
      const float n = (float)count[lane % WIDTHS] * n_ft, rounds = ceilf(n / n_clusters);
      const float main = n > 0.f ? (float)cost[lane % WIDTHS] / count[lane % WIDTHS] * all_blocks : 0.f;
      const float epi = TILES ? 2900.f + 12.f * T : 3300.f + 30.f * T;
      const float last = (TILES ? 16.f : 28.f) * T;
      if (lane < WIDTHS) {
        est = main + (rounds - 1.f) * fmaxf(main, epi) + last;
      } else if (g.ws && all_blocks >= 4 * MIN_BLOCKS) {
        ctas = fminf(ctas, fmaxf(1.f, floorf(n * all_blocks / 12.f)));
        est = fmaxf(main, epi) * n / ctas + last + (DOWN ? 5000.f : 6000.f + 100.f * T);
      }
    }
    float best = est;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = fminf(best, __shfl_xor_sync(0xffffffffu, best, o));
    const int winner = __ffs(__ballot_sync(0xffffffffu, est == best)) - 1, Tb = T_STEP * (winner % WIDTHS + 1);
    ctas = __shfl_sync(0xffffffffu, ctas, winner);
    int sum = 0;
    for (int e0 = 0; e0 <= E; e0 += 32) {
      const int e = e0 + lane;
      int n = e < E ? (rows_of(e) + Tb - 1) / Tb : 0, s = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += v;
      }
      if (e <= E) first[e] = sum + s - n;
      sum += __shfl_sync(0xffffffffu, s, 31);
    }
    __syncwarp();
    if (lane == 0) {
      *width = Tb;
      cut.on = winner >= WIDTHS;
      cut.clusters = (int)ctas;
    }
    if (winner >= WIDTHS) {
      // all units, then the groups in which this cluster's stretch and the next one's begin
      unsigned all = 0;
      for (int e = lane; e < E; e += 32) all += units_of(e);
      all = __reduce_add_sync(0xffffffffu, all);
      if (lane == 0) cut.units = all;
      const unsigned x0 = stretch(cluster, all, (unsigned)ctas), x1 = stretch(cluster + 1, all, (unsigned)ctas);
      unsigned before = 0;
      bool have0 = false, have1 = false;
      if (lane == 0) {  // (behind the last tile)
        cut.t0 = cut.t1 = first[E] * n_ft;
        cut.k0 = cut.k1 = 0;
      }
      __syncwarp();
      for (int e0 = 0; e0 < E && !(have0 && have1); e0 += 32) {
        const int e = e0 + lane;
        const unsigned mine = e < E ? units_of(e) : 0;
        unsigned upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const unsigned v = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += v;
        }
        const unsigned u = before + upto - mine;
        // the lane whose group a position lies in works it out
        auto place = [&](unsigned x, int& t, int& kb, unsigned& u_t) {
          const bool here = x >= u && x - u < mine;
          if (here) {
            const unsigned wt = weight(e), per = all_blocks * wt, v = x - u, q = v / per;
            u_t = u + q * per;
            kb = (int)((v - q * per) / wt);
            t = first[e] * n_ft + (int)q;
            if (kb < MIN_BLOCKS) {
              kb = 0;
            } else if (all_blocks - kb < MIN_BLOCKS) {
              kb = 0;
              ++t;
            }
          }
          return __any_sync(0xffffffffu, here);
        };
        have0 = place(x0, cut.t0, cut.k0, cut.u0) || have0;
        have1 = place(x1, cut.t1, cut.k1, cut.u1) || have1;
        before += __shfl_sync(0xffffffffu, upto, 31);
      }
    }
  }
  tc_fence_before();
  cluster_sync();  // barriers initialised, TMEM allocated, tables written
  tc_fence_after();
  const uint32_t tmem_base = *tmem_holder;
  const int T = *width;
  const int stage_bytes = W_BYTES + T / 2 * BK * 2;
  const int stages = RING_BYTES / stage_bytes < MAX_STAGES ? RING_BYTES / stage_bytes : MAX_STAGES;
  const int acc_cols = acc_cols_of(T);
  const int n_accs = TMEM_COLS / acc_cols < MAX_ACCS ? TMEM_COLS / acc_cols : MAX_ACCS;
  const int fit = (int)(BAND_BYTES / ((int64_t)2 * W_ROWS * g.k * sizeof(bf16)));
  const bool split = cut.on != 0;
  TileIter ti(off, first, split ? cluster < cut.clusters ? cut.t0 : INT_MAX - (1 << 20) : cluster,
              split ? 1 : n_clusters, n_ft, fit < 1 ? 1 : fit < n_ft ? fit : n_ft, E);
  Tile k;
  int kb0, blocks;
  // The next tile, and the K blocks kb0 .. kb0 + blocks - 1 of it that are this cluster's (t's behind
  // x's; none where they are all t's and the tile has no adapter).
  auto next_tile = [&](Tile& q, int& from, int& n) {
    if (split && (ti.t > cut.t1 || (ti.t == cut.t1 && cut.k1 == 0))) return false;
    const int t = ti.t;
    if (!ti.next(q)) return false;
    const int all = DOWN || who[q.e] < 0 ? nk : nk + ext;
    const int a = split && t == cut.t0 ? cut.k0 : 0, b = split && t == cut.t1 ? cut.k1 : all;
    from = a < all ? a : all;
    n = (b < all ? b : all) - from;
    return true;
  };

  // The clusters lo .. hi that hold parts of tile t of group e (cut.t0 or cut.t1): a stretch begins
  // within it at least MIN_BLOCKS from its ends.
  auto holders = [&](int t, int e, int& lo, int& hi) {
    const unsigned wt = weight(e), u = t == cut.t0 && cut.k0 > 0 ? cut.u0 : cut.u1;
    const unsigned most = cut.units / cut.clusters + 1;
    auto from = [&](unsigned y) {  // the first cluster whose stretch begins at y or behind
      unsigned c = y / most;
      while (stretch(c, cut.units, cut.clusters) < y) ++c;
      return (int)c;
    };
    lo = from(u + MIN_BLOCKS * wt) - 1;
    hi = from(u + (all_blocks - MIN_BLOCKS + 1) * wt) - 1;
  };

  if (warp == 0) {
    // ---------------- weights (both CTAs) ----------------
    int stage = 0;
    uint32_t phase = 0;
    while (!failed && next_tile(k, kb0, blocks)) {
      const uint32_t bytes = 2 * (W_BYTES + k.w / 2 * BK * 2);
      const int e = who[k.e];
      for (int i = kb0; i < kb0 + blocks; ++i) {
        if (!mbar_wait_warp(&empty[stage], phase ^ 1u, err)) { failed = true; break; }
        if (elect_one()) {
          const uint32_t dst = smem_u32(smem) + stage * stage_bytes;
          const uint32_t fb = mapa_shared(smem_u32(&full[stage]), 0);
          if (rank == 0) mbar_expect_tx(&full[stage], bytes);
          if (DOWN)
            tma_load_3d_cg2(dst, &maps.w, fb, i * BK, (int)rank * W_ROWS, e);
          else if (i < nk)
            tma_load_3d_cg2(dst, &maps.w, fb, i * BK, (2 * k.f + (int)rank) * W_ROWS, 0);
          else
            tma_load_3d_cg2(dst, &maps.b, fb, terms.rp <= 64 ? 0 : (i - nk) / terms.terms * BK,
                            (2 * k.f + (int)rank) * W_ROWS, e);
        }
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp >= LOAD) {
    // ---------------- rows of x and t (both CTAs) ----------------
    int stage = 0;
    uint32_t phase = 0;
    int turn = warp - LOAD;  // K blocks until this warp's next: they go round the two
    bool waited = DOWN;
    while (!failed && next_tile(k, kb0, blocks)) {
      const int half = k.w / 2, a0 = k.r0 + half * (int)rank;
      for (int i = kb0; i < kb0 + blocks; ++i) {
        if (turn-- == 0) {
          turn = 1;
          if (!mbar_wait_warp(&empty[stage], phase ^ 1u, err)) { failed = true; break; }
          const bool of_t = !DOWN && i >= nk;
          if (of_t && !waited) {
            griddep_wait();
            waited = true;
          }
          if (elect_one()) {
            const uint32_t dst = smem_u32(smem) + stage * stage_bytes + W_BYTES;
            const uint32_t fb = mapa_shared(smem_u32(&full[stage]), 0);
            const CUtensorMap* m = of_t ? maps.t : maps.x;
            const int x = (of_t ? i - nk : i) * BK;
            int r = 0;
            for (; r + 64 <= half; r += 64) tma_load_rows_cg2(dst + r * (BK * 2), m, fb, x, a0 + r);
#pragma unroll
            for (int b = 32, j = 1; b >= 8; b /= 2, ++j)
              if (half & b) {
                tma_load_rows_cg2(dst + r * (BK * 2), m + j, fb, x, a0 + r);
                r += b;
              }
          }
        }
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
    }
    if (!waited) griddep_wait();
  } else if (warp == 1) {
    if (rank == 0) {
      // ---------------- MMA issuer (even CTA) ----------------
      const uint32_t ring_lo = desc_lo_k(smem_u32(smem));
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      while (!failed && next_tile(k, kb0, blocks)) {
        const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(k.w >> 3) << 17) |
                               ((uint32_t)(2 * W_ROWS >> 4) << 24);
        // The tile's K parts, each in the ring's next accumulator. All control flow goes by votes: the
        // K range comes from shared memory, and what the compiler does not see to be the same in all
        // lanes costs the MMAs' operands a move to a uniform register each (one K block 550 clocks
        // whatever its width; see elect_one).
        const int stop = kb0 + blocks;
        int i = kb0, end = i;
        bool more = __all_sync(0xffffffffu, i < stop);
        while (!failed && more) {
          if (!mbar_wait_warp(&tmem_empty[acc], acc_phase ^ 1u, err)) { failed = true; break; }
          tc_fence_after();
          const uint32_t d_tmem = tmem_base + acc * acc_cols;
          end = PARTS && stop - i > PART_BLOCKS ? i + PART_BLOCKS : stop;
          bool first = true, last = false;
          while (!last) {
            last = __all_sync(0xffffffffu, i + 1 >= end);
            const bool straight = DOWN || terms.rp >= 64 || __all_sync(0xffffffffu, i < nk);
            uint32_t cols = 0;  // t's chunks against B_e's: columns of each, 16 to a unit (see Terms)
            if (!straight) {
              int c = 4 * (i - nk);
#pragma unroll
              for (int j = 0; j < 4; ++j, ++c) cols |= (uint32_t)(c < all_chunks ? c % chunks : 3) << (8 * j);
            }
            if (!mbar_wait_warp(&full[stage], phase, err)) { failed = true; break; }
            tc_fence_after();
            const uint32_t wlo = ring_lo + (uint32_t)(stage * (stage_bytes >> 4));
            const uint32_t alo = wlo + (W_BYTES >> 4);
            if (straight) {
              if (elect_one()) {
#pragma unroll
                for (int j = 0; j < BK / 16; ++j)
                  tc_mma_cg2_lo(d_tmem, wlo + 2 * j, alo + 2 * j, DESC_HI, idesc,
                                (!first || j > 0) ? 1u : 0u);
                tc_commit_mc(&empty[stage], 0x3);
                if (last) tc_commit_mc(&tmem_full[acc], 0x3);
              }
            } else if (elect_one()) {
#pragma unroll
              for (int j = 0; j < BK / 16; ++j)
                tc_mma_cg2_lo(d_tmem, wlo + 2 * ((cols >> (8 * j)) & 3), alo + 2 * j, DESC_HI, idesc,
                              (!first || j > 0) ? 1u : 0u);
              tc_commit_mc(&empty[stage], 0x3);
              if (last) tc_commit_mc(&tmem_full[acc], 0x3);
            }
            first = false;
            ++i;
            if (++stage == stages) { stage = 0; phase ^= 1u; }
          }
          if (++acc == n_accs) { acc = 0; acc_phase ^= 1u; }
          more = __all_sync(0xffffffffu, i < stop);
        }
      }
    }
  } else {
    // ---------------- epilogue (warps 2..9 of both CTAs) ----------------
    // warp: weight rows quarter * 32 .. + 31 of this CTA's 128 (its TMEM lanes), every GROUPS-th
    // CH-token chunk of the tile
    constexpr int CH = PARTS ? 16 : 32;
    const int quarter = warp & 3, we = warp - 2;
    int group = we >> 2;  // a tile's first chunk goes to each group of four warps by turns
    const uint32_t te_remote = mapa_shared(smem_u32(&tmem_empty[0]), 0);
    uint8_t* tiles = epi_smem + we * 2 * EPI_TILE;
    int acc = 0, buf = 0;
    uint32_t acc_phase = 0;
    auto first_feature = [&](const Tile& q) {
      return ((DOWN ? 0 : 2 * q.f) + (int)rank) * W_ROWS + quarter * 32;
    };
    // the bias of this lane's weight row; DOWN: the adapter's scale
    auto bias_of = [&](const Tile& q) {
      if (DOWN) return g.scale ? __ldg(g.scale + who[q.e]) : 1.f;
      const int feature = first_feature(q) + lane;
      return g.bias && feature < g.n ? __ldg(g.bias + feature) : 0.f;
    };
    const int limit = DOWN ? terms.rp : g.n;  // features that are stored
    Tile after;
    int kb_after = 0, blocks_after = 0, t_after = ti.t, t = 0;
    bool more = next_tile(k, kb0, blocks);
    float bias = more ? bias_of(k) : 0.f;
    for (; !failed && more; k = after, kb0 = kb_after, blocks = blocks_after) {
      t = t_after;  // the tile's number
      t_after = ti.t;
      more = next_tile(after, kb_after, blocks_after);
      const float bias_after = more ? bias_of(after) : 0.f;  // (it may come from memory)
      const int f0 = first_feature(k), feature = f0 + lane;
      const int col0 = terms.column(0, feature), col1 = terms.column(1, feature), col2 = terms.column(2, feature);
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16);
      // a part of a cut tile: its first K block, or its last, is another cluster's
      const bool partly = split && ((t == cut.t0 && cut.k0 > 0) || (t == cut.t1 && cut.k1 > 0));
      // (the kernel before forms the low-rank part, or t, whose cut tiles' parts and counters lie in
      // the same place)
      if (!DOWN && (g.delta || partly)) griddep_wait();
      if (partly) group = we >> 2;  // (every cluster's warps take the same chunks)
      // sums in parts: added up here as they are done, a part's accumulator going back at once
      float sum[PARTS ? F32_T / GROUPS : 1];
      bool ok = true;
      const int parts = PARTS ? (blocks + PART_BLOCKS - 1) / PART_BLOCKS : blocks > 0;
      if (PARTS && !DOWN && g.resid && f0 < limit) {  // its residual rows on their way into L2, a lane a row
        for (int c = 0; c < F32_T / (GROUPS * CH); c += 2) {
          const int row = (group + GROUPS * (c + lane / CH)) * CH + lane % CH;
          if (row < k.nv)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(g.resid + (size_t)(k.r0 + row) * g.ldr + f0));
        }
      }
      for (int p = 0; p < parts; ++p) {
        ok = __all_sync(0xffffffffu, mbar_wait(&tmem_full[acc], acc_phase, err));
        if (!ok) break;
        tc_fence_after();
        if constexpr (PARTS) {
#pragma unroll
          for (int c = 0; c < F32_T / (GROUPS * CH); ++c) {
            const int t0 = (group + GROUPS * c) * CH;
            if (t0 >= k.nv || f0 >= limit) break;
            uint32_t r[16];
            tmem_ld16(taddr + acc * acc_cols + t0, r);
            tmem_ld_wait();
            reg_fence16(r);
#pragma unroll
            for (int j = 0; j < 16; ++j)
              sum[c * CH + j] = __uint_as_float(r[j]) + (p == 0 ? 0.f : sum[c * CH + j]);
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_relaxed_cluster(te_remote + acc * (uint32_t)sizeof(uint64_t));
          if (++acc == n_accs) { acc = 0; acc_phase ^= 1u; }
        }
      }
      if (!ok) { failed = true; break; }
      int lo = 0, hi = 0;  // the clusters that hold the tile's parts
      bool adds = false;   // this warp comes last and adds them up
      auto part_of = [&](int c) {  // (a cluster holds two at most, one of them of a tile that begins with it)
        return g.ws + (size_t)(c == lo ? 2 * c + 1 : 2 * c) * WS_SLOT + ((size_t)rank * EPI + we) * WS_WARP + lane;
      };
      if (partly) {
        holders(t, k.e, lo, hi);
        float* to = part_of(cluster);
        if (f0 < limit) {
          constexpr int UN = PARTS ? F32_T / (GROUPS * CH) : 1;
#pragma unroll UN
          for (int c = 0; c < (PARTS ? F32_T : MAX_T) / (GROUPS * CH); ++c) {
            const int t0 = (group + GROUPS * c) * CH;
            if (t0 >= k.nv) break;
            if constexpr (PARTS) {
#pragma unroll
              for (int j = 0; j < CH; ++j) to[(c * CH + j) * 32] = blocks ? sum[c * CH + j] : 0.f;
            } else {
              uint32_t r[32];
              tmem_ld32(taddr + acc * acc_cols + t0, r);
              tmem_ld_wait();
              reg_fence32(r);
#pragma unroll
              for (int j = 0; j < CH; ++j) to[(c * CH + j) * 32] = blocks ? __uint_as_float(r[j]) : 0.f;
            }
          }
        }
        if (!PARTS && blocks) {  // the accumulator is read
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_relaxed_cluster(te_remote + acc * (uint32_t)sizeof(uint64_t));
          if (++acc == n_accs) { acc = 0; acc_phase ^= 1u; }
        }
        __threadfence();
        __syncwarp();
        int* counter = g.counters + lo * ADAPTER_COUNTERS + (int)rank * EPI + we;
        int came = 0;
        if (lane == 0) came = atomicAdd(counter, 1);
        adds = __shfl_sync(0xffffffffu, came, 0) == hi - lo;
        if (adds) {
          __threadfence();
          if (lane == 0) *counter = 0;
        }
      }
      // The results of CH tokens from t0 on. ALL: every token and every lane's feature exists.
      auto finish_as = [&](auto all, float* v, int t0) {
        constexpr bool ALL = decltype(all)::value;
        const int n = ALL || k.nv - t0 > CH ? CH : k.nv - t0;  // tokens of the chunk that exist
        const size_t row = k.r0 + t0;
        const bool in = ALL || feature < g.n;
        if constexpr (DOWN) {  // (columns behind the rank, and behind the last term, are zeros)
          const int pad = terms.cols - terms.terms * terms.rp;
          bf16* at = g.t + row * terms.cols;
#pragma unroll
          for (int j = 0; j < CH; ++j, at += terms.cols) {
            if (!ALL && j >= n) break;
            if (feature < terms.rp) {
              float x = in ? v[j] * bias : 0.f;
              bf16 b = __float2bfloat16(x);
              at[col0] = b;
              x -= __bfloat162float(b);
              b = __float2bfloat16(x);
              at[col1] = b;
              if (PARTS) at[col2] = __float2bfloat16(x - __bfloat162float(b));
            }
            if (feature < pad) at[terms.cols - pad + feature] = __float2bfloat16(0.f);
          }
          return;
        }
        if (g.delta) {  // the low-rank part, formed by itself
          const float* from = g.delta + row * g.n + feature;
          float d[CH];
#pragma unroll
          for (int j = 0; j < CH; ++j, from += g.n) d[j] = ALL || (in && j < n) ? *from : 0.f;
#pragma unroll
          for (int j = 0; j < CH; ++j) v[j] += d[j];
        }
        if constexpr (PARTS) {
          // straight to memory, 32 features of a token
          float rs[CH];
          if (g.resid) {
            const float* from = g.resid + row * g.ldr + feature;
#pragma unroll
            for (int j = 0; j < CH; ++j, from += g.ldr) rs[j] = ALL || (in && j < n) ? *from : 0.f;
          }
#pragma unroll
          for (int j = 0; j < CH; ++j) v[j] += bias;
          if (g.act == FB_ACT_GELU) {
#pragma unroll
            for (int j = 0; j < CH; ++j) v[j] = gelu_f<true>(v[j]);
          }
          if (g.gate) {
            const float gate = in ? __ldg(g.gate + feature) : 0.f;
#pragma unroll
            for (int j = 0; j < CH; ++j) v[j] *= gate;
          }
          if (g.resid) {
#pragma unroll
            for (int j = 0; j < CH; ++j) v[j] += rs[j];
          }
          if (g.out_type == FB_F32) {
            float* at = reinterpret_cast<float*>(g.out) + row * g.ldo + feature;
#pragma unroll
            for (int j = 0; j < CH; ++j, at += g.ldo)
              if (ALL || (in && j < n)) *at = v[j];
          } else {
            bf16* at = reinterpret_cast<bf16*>(g.out) + row * g.ldo + feature;
#pragma unroll
            for (int j = 0; j < CH; ++j, at += g.ldo)
              if (ALL || (in && j < n)) *at = __float2bfloat16(v[j]);
          }
        } else {
          uint8_t* tile = tiles + buf * EPI_TILE;
          buf ^= 1;
          if (elect_one()) bulk_wait_read<1>();  // the store from this tile two chunks ago
          __syncwarp();
#pragma unroll
          for (int j = 0; j < CH; ++j) v[j] += bias;
          if (g.act == FB_ACT_GELU) {
#pragma unroll
            for (int j = 0; j < CH; j += 2) gelu_f2(v[j], v[j + 1]);
          }
          // two tokens' values of each lane's feature as one 4-byte store per lane: lanes
          // exchange with their neighbour, even lanes then hold two features of token j, odd
          // lanes of token j + 1
          uint32_t* tw = reinterpret_cast<uint32_t*>(tile) + (lane & 1) * 16 + (lane >> 1);
#pragma unroll
          for (int j = 0; j < CH; j += 2) {
            const float got = __shfl_xor_sync(0xffffffffu, (lane & 1) ? v[j] : v[j + 1], 1);
            tw[j * 16] = (lane & 1) ? pack_bf16x2(got, v[j + 1]) : pack_bf16x2(v[j], got);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (elect_one()) {
#pragma unroll
            for (int b = 0; b < CH; b += 16)
              if (ALL || b + 16 <= n) tma_store_2d(&maps.o, smem_u32(tile) + b * 64, f0, (int)row + b);
            bulk_commit();
          }
          if (!ALL && n % 16) {  // 16 bytes at a time: n is a multiple of 8 features
            const int b = n / 16 * 16;
#pragma unroll 1
            for (int i = lane; i < (n - b) * 4; i += 32) {
              const int tok = b + i / 4, q = i % 4;
              if (f0 + q * 8 < g.n)
                *reinterpret_cast<uint4*>(reinterpret_cast<bf16*>(g.out) + (row + tok) * g.ldo + f0 +
                                          q * 8) = *reinterpret_cast<const uint4*>(tile + tok * 64 + q * 16);
            }
            __syncwarp();
          }
        }
      };
      auto finish = [&](float* v, int t0) {
        if (t0 + CH <= k.nv && f0 + 32 <= g.n)
          finish_as(std::true_type{}, v, t0);
        else
          finish_as(std::false_type{}, v, t0);
      };
      // The chunks one after the other, the code of one for all of them (unrolled it would not fit the
      // instruction caches); sums in registers move up by a chunk each time.
      constexpr int CHUNKS = (PARTS ? F32_T : MAX_T) / (GROUPS * CH);
      if (partly) {
#pragma unroll 1
        for (int c = 0; adds && c < CHUNKS; ++c) {
          const int t0 = (group + GROUPS * c) * CH;
          if (t0 >= k.nv || f0 >= limit) break;
          float v[CH] = {};
#pragma unroll 2
          for (int b = lo; b <= hi; ++b) {
            const float* from = part_of(b) + c * CH * 32;
            float w[CH];
#pragma unroll
            for (int j = 0; j < CH; ++j) w[j] = __ldcg(from + j * 32);
#pragma unroll
            for (int j = 0; j < CH; ++j) v[j] += w[j];
          }
          finish(v, t0);
        }
      } else {
#pragma unroll 1
        for (int c = 0; c < CHUNKS; ++c) {
          const int t0 = (group + GROUPS * c) * CH;
          if (t0 >= k.nv || f0 >= limit) break;
          float v[CH];
          if constexpr (PARTS) {
#pragma unroll
            for (int j = 0; j < CH; ++j) v[j] = sum[j];
#pragma unroll
            for (int j = 0; j + CH < F32_T / GROUPS; ++j) sum[j] = sum[j + CH];
          } else {
            uint32_t r[32];
            tmem_ld32(taddr + acc * acc_cols + t0, r);
            tmem_ld_wait();
            reg_fence32(r);
#pragma unroll
            for (int j = 0; j < CH; ++j) v[j] = __uint_as_float(r[j]);
          }
          finish(v, t0);
        }
      }
      if (!PARTS && !partly) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_relaxed_cluster(te_remote + acc * (uint32_t)sizeof(uint64_t));
        if (++acc == n_accs) { acc = 0; acc_phase ^= 1u; }
      }
      bias = bias_after;
      group = group + 1 == GROUPS ? 0 : group + 1;
    }
    if (TILES && elect_one()) bulk_wait<0>();  // own TMA stores complete (one lane issued them all)
  }

  if (failed) *gave_up = 1;
  tc_fence_before();
  cluster_sync();
  if (*gave_up != 0) {
    // After a timeout, give TMA loads that may still be in flight time to land before the
    // shared memory they target is released (they complete within microseconds).
    const uint64_t t0 = fb_globaltimer();
    while (fb_globaltimer() - t0 < 100000ull) __nanosleep(1000);
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_cg2(tmem_base, TMEM_COLS);
  }
}

// ---- short segments ---------------------------------------------------------------------
// The low-rank part of up to 16 rows of a segment, scale (x A_e^T) B_e^T in fp32, by a cluster of
// eight CTAs: each forms its eighth of K's sums of t (mma.sync, A_e and x straight from memory into the
// operand registers, A_e the M side), all of them add the eighths up in CTA order through distributed
// shared memory, and each multiplies t with its eighth of B_e's rows (a feature per thread). Rows without
// an adapter get zeros. Latency bounds it: 64 segments of a row, 9216 x 1536, rank 16 (22 MB) take 7 us of
// the call's 22.5, of which 1.5 find the segment, 1.5 form the sums, 2 join them and 2 multiply. So B_e's rows
// come by one bulk copy meanwhile (read when t is there, or by copies of single threads, which wait behind
// A_e's in the load units: 25 to 27 us a call), and a row's features share the reads of t.
constexpr int D_CTAS = 8, D_WARPS = 8, D_THREADS = 32 * D_WARPS, D_ROWS = 16;
constexpr int D_STAGE = 40 << 10;  // of B_e's rows in shared memory (four blocks of rank 16 on an SM)
// Features of a block whose rows of B_e wait in shared memory, the others come from L2. (Ranks above 32
// have their rows on too few banks.)
__host__ __device__ inline int delta_staged(int features, int rank) {
  const int fit = rank > 32 ? 0 : D_STAGE / (rank * 2);
  return features < fit ? features : fit;
}
// MT: 16 of the rank each, in one pass over K.
template <int MT>
size_t delta_smem(int n, int rank) {
  return (size_t)(D_WARPS * 16 * MT + 2 * rank) * D_ROWS * sizeof(float) +
         (size_t)delta_staged(n / D_CTAS + 1, rank) * rank * sizeof(bf16);
}

__device__ __forceinline__ float ld_cluster(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}
// bytes (a multiple of 16) into this CTA's shared memory
__device__ __forceinline__ void bulk_load(void* to, const void* from, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                   smem_u32(to)),
               "l"(from), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

template <int MT>
__global__ void __cluster_dims__(D_CTAS, 1, 1) __launch_bounds__(D_THREADS, MT == 1 ? 4 : MT == 2 ? 3 : 2)
    adapter_delta_kernel(const AdapterArgs g, float* delta, int* err) {
  griddep_wait();
  griddep_launch();
  constexpr int D_RANKS = 16 * MT;
  extern __shared__ __align__(16) float sm[];
  float* part = sm;                                // [warp][D_RANKS of the rank][16 rows]
  float* own = part + D_WARPS * D_RANKS * D_ROWS;  // [rank][16]: this CTA's sums
  float* t = own + g.rank * D_ROWS;                // [rank][16]: all of them
  bf16* stage = reinterpret_cast<bf16*>(t + g.rank * D_ROWS);  // rows of B_e
  __shared__ int found[4], scan[D_WARPS];
  __shared__ uint64_t landed;
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  const uint32_t c = cluster_ctarank();
  const int want = blockIdx.x / D_CTAS;
  // ---- the want-th chunk of 16 rows: each thread up to four segments ----
  if (tid == 0) {
    found[0] = -2;
    mbar_init(&landed, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  int a[4], b[4], of[4], sum = 0;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int s = 4 * tid + i;
    const bool in = s < g.segments;
    a[i] = in ? g.offsets[s] : 0;
    b[i] = in ? g.offsets[s + 1] : 0;
    of[i] = in ? g.adapter[s] : -1;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bad = bad || a[i] < 0 || b[i] < a[i] || b[i] > g.rows || (tid == 0 && i == 0 && a[i] != 0) || of[i] < -1 ||
          of[i] >= g.adapters;
    sum += (b[i] - a[i] + D_ROWS - 1) / D_ROWS;
  }
  static_assert(FB_ADAPTER_MAX_SEGMENTS <= 4 * D_THREADS, "segments of a thread");
  int upto = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) scan[warp] = upto;
  if (__syncthreads_or(bad)) {  // (every CTA sees the same)
    if (tid == 0) fb_report(err, FB_DEVERR_BAD_INDEX);
    return;
  }
  int at = upto - sum;
  for (int w = 0; w < warp; ++w) at += scan[w];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int chunks = (b[i] - a[i] + D_ROWS - 1) / D_ROWS;
    if (want >= at && want < at + chunks) {
      found[0] = of[i];
      found[1] = a[i] + (want - at) * D_ROWS;
      found[2] = b[i];
    }
    at += chunks;
  }
  __syncthreads();
  const int e = found[0], r0 = found[1];
  if (e == -2) return;  // (the whole cluster)
  const int rows = found[2] - r0 < D_ROWS ? found[2] - r0 : D_ROWS;
  const int fa = (int)((int64_t)g.n * c / D_CTAS), fb = (int)((int64_t)g.n * (c + 1) / D_CTAS);
  // B_e's rows on their way meanwhile: as many as fit into shared memory, the others into L2, an eighth of
  // them a thread
  const int staged = delta_staged(fb - fa, g.rank);
  if (e >= 0 && tid < D_WARPS) {
    const bf16* b = (const bf16*)g.b + ((size_t)e * g.n + fa) * g.rank;
    if (tid == 0 && staged > 0) {
      const uint32_t bytes = (uint32_t)(staged * g.rank * sizeof(bf16));
      mbar_expect_tx(&landed, bytes);
      bulk_load(stage, b, bytes, &landed);
    }
    const int64_t first = (int64_t)staged * g.rank / 8, pieces = (int64_t)(fb - fa) * g.rank / 8 - first;
    const int64_t p0 = first + pieces * tid / D_WARPS, p1 = first + pieces * (tid + 1) / D_WARPS;
    if (p1 > p0 && p1 - p0 < (1 << 20)) prefetch_l2_bulk(b + p0 * 8, (uint32_t)(p1 - p0) * 16);
  }
  // ---- t: this CTA's part of K ----
  if (e >= 0) {
    const int gr = lane / 4, q = lane % 4;
    const int steps = (g.k + 31) / 32;
    const int s0 = steps * (int)c / D_CTAS, s1 = steps * ((int)c + 1) / D_CTAS;
    const bf16* x0 = (const bf16*)g.x + (size_t)(r0 + (gr < rows ? gr : 0)) * g.ldx + 8 * q;
    const bf16* x1 = (const bf16*)g.x + (size_t)(r0 + (8 + gr < rows ? 8 + gr : 0)) * g.ldx + 8 * q;
    const bool two = rows > 8;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    for (int f0 = 0; f0 < g.rank; f0 += D_RANKS) {
      const bf16* a = (const bf16*)g.a + ((size_t)e * g.rank + f0) * g.k + 8 * q;
      const int tiles = (g.rank - f0 + 15) / 16 < D_RANKS / 16 ? (g.rank - f0 + 15) / 16 : D_RANKS / 16;
      float acc[D_RANKS / 16][2][4] = {};
#pragma unroll 2
      for (int s = s0 + warp; s < s1; s += D_WARPS) {
        const int kk = 32 * s;
        const bool in = kk + 8 * q < g.k;
        const uint4 u0 = in && gr < rows ? *reinterpret_cast<const uint4*>(x0 + kk) : zero;
        const uint4 u1 = in && 8 + gr < rows ? *reinterpret_cast<const uint4*>(x1 + kk) : zero;
#pragma unroll
        for (int m = 0; m < D_RANKS / 16; ++m) {
          if (m >= tiles) break;
          const int ra = 16 * m + gr, rb = ra + 8;
          const uint4 va = in && f0 + ra < g.rank ? __ldg(reinterpret_cast<const uint4*>(a + (size_t)ra * g.k + kk)) : zero;
          const uint4 vb = in && f0 + rb < g.rank ? __ldg(reinterpret_cast<const uint4*>(a + (size_t)rb * g.k + kk)) : zero;
          // (fp32 sums outside the instruction: its own cut a bit off per step)
          float d[2][4] = {};
          mma_16816(d[0], va.x, vb.x, va.y, vb.y, u0.x, u0.y);
          mma_16816(d[0], va.z, vb.z, va.w, vb.w, u0.z, u0.w);
          if (two) {
            mma_16816(d[1], va.x, vb.x, va.y, vb.y, u1.x, u1.y);
            mma_16816(d[1], va.z, vb.z, va.w, vb.w, u1.z, u1.w);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            acc[m][0][i] += d[0][i];
            acc[m][1][i] += d[1][i];
          }
        }
      }
      // d[i][0..1]: rank row gr, rows 8 i + 2 q and + 1 of x; d[i][2..3]: rank row gr + 8
      float* mine = part + warp * D_RANKS * D_ROWS;
#pragma unroll
      for (int m = 0; m < D_RANKS / 16; ++m)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          *reinterpret_cast<float2*>(mine + (16 * m + gr) * D_ROWS + 8 * i + 2 * q) =
              make_float2(acc[m][i][0], acc[m][i][1]);
          *reinterpret_cast<float2*>(mine + (16 * m + gr + 8) * D_ROWS + 8 * i + 2 * q) =
              make_float2(acc[m][i][2], acc[m][i][3]);
        }
      __syncthreads();
      for (int i = tid; i < D_RANKS * D_ROWS; i += D_THREADS) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < D_WARPS; ++w) v += part[w * D_RANKS * D_ROWS + i];
        if (f0 + i / D_ROWS < g.rank) own[f0 * D_ROWS + i] = v;
      }
      __syncthreads();
    }
    const float scale = g.scale ? g.scale[e] : 1.f;
    cluster_sync();
    for (int i = tid; i < g.rank * D_ROWS; i += D_THREADS) {
      float v = 0.f, w[D_CTAS];
      if (i % D_ROWS < rows) {
#pragma unroll
        for (uint32_t p = 0; p < D_CTAS; ++p) w[p] = ld_cluster(mapa_shared(smem_u32(own + i), p));
#pragma unroll
        for (int p = 0; p < D_CTAS; ++p) v += w[p];
      }
      t[i] = v * scale;
    }
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  }
  // ---- the product with this CTA's rows of B_e ----
  if (e >= 0 && staged > 0 && !mbar_wait(&landed, 0, err)) {  // (reported; the copy lands before the block ends)
    const uint64_t t0 = fb_globaltimer();
    while (fb_globaltimer() - t0 < 100000ull) __nanosleep(1000);
  }
  // F of a thread's features at a time, so that each reads t only once for all of them
  auto product = [&](auto features, auto of_rows) {
    constexpr int F = decltype(features)::value, R = decltype(of_rows)::value;
#pragma unroll 1
    for (int f = fa + tid; f < fb; f += F * D_THREADS) {
      float y[F][R] = {};
#pragma unroll 1
      for (int r = 0; e >= 0 && r < g.rank; r += 8) {
        float w[F][8];
#pragma unroll
        for (int j = 0; j < F; ++j) {
          const int at = min(f + j * D_THREADS, fb - 1) - fa;
          const bf16* from = stage + at * g.rank + r;
          if (at >= staged) from = (const bf16*)g.b + ((size_t)e * g.n + fa + at) * g.rank + r;
          load_bf16x8(from, w[j]);
        }
        if constexpr (R == 1) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float v = t[(r + i) * D_ROWS];
#pragma unroll
            for (int j = 0; j < F; ++j) y[j][0] = fmaf(w[j][i], v, y[j][0]);
          }
        } else {
#pragma unroll
          for (int k = 0; k < R; k += 4) {
            if (k >= rows) break;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float4 v = *reinterpret_cast<const float4*>(t + (r + i) * D_ROWS + k);
#pragma unroll
              for (int j = 0; j < F; ++j) {
                y[j][k] = fmaf(w[j][i], v.x, y[j][k]);
                y[j][k + 1] = fmaf(w[j][i], v.y, y[j][k + 1]);
                y[j][k + 2] = fmaf(w[j][i], v.z, y[j][k + 2]);
                y[j][k + 3] = fmaf(w[j][i], v.w, y[j][k + 3]);
              }
            }
          }
        }
      }
#pragma unroll
      for (int j = 0; j < F; ++j)
#pragma unroll
        for (int k = 0; k < R; ++k)
          if (k < rows && f + j * D_THREADS < fb) delta[(size_t)(r0 + k) * g.n + f + j * D_THREADS] = y[j][k];
    }
  };
  if (rows == 1)
    product(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
  else
    product(std::integral_constant<int, 1>{}, std::integral_constant<int, D_ROWS>{});
  if (e >= 0) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");  // (no CTA leaves while its sums are read)
}

// ---- few rows ---------------------------------------------------------------------------
// Up to 32 rows read every weight once, up to 64 in two halves: a block takes 16 weight rows, its warps split K,
// and the weights go straight from memory into the operand registers of mma.sync (the weights are the M
// side, eight rows of x the N side), as in the products grouped by expert. The weights do not wait
// for the low-rank part; the epilogue does. One row, 1536 x 1536, rank 16: 6.0 us with the low-rank part's
// kernel (in tiles 12), whose latency and its own are all there is. 32 rows at a time with two steps of K
// on their way, two blocks an SM, against 16 with four: 5120 x 5120 21.0 us for 26.1; 16 rows with three
// steps, three blocks, 11.5 for 15.6.
constexpr int FEW_WARPS = 8, FEW_THREADS = FEW_WARPS * 32, FEW_LONG_K = 2048;

template <bool EXACT, int NT, int UN, int BLOCKS>
__global__ void __launch_bounds__(FEW_THREADS, BLOCKS)
    adapter_few_kernel(const AdapterArgs g, const float* delta) {
  griddep_launch();
  __shared__ float part[FEW_WARPS][16][8 * NT + 1];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, gr = lane / 4, t = lane % 4;
  const int f0 = blockIdx.x * 16;
  // (the low-rank part's kernel checks the offsets; what it refuses is not used)
  const int end = g.offsets[g.segments], rows = end < 0 ? 0 : end < g.rows ? end : g.rows;
  const bf16* wa = (const bf16*)g.w + (size_t)min(f0 + gr, g.n - 1) * g.k + 8 * t;
  const bf16* wb = (const bf16*)g.w + (size_t)min(f0 + 8 + gr, g.n - 1) * g.k + 8 * t;
  const int steps = (g.k + 31) / 32;
  const int s0 = steps * warp / FEW_WARPS, s1 = steps * (warp + 1) / FEW_WARPS;
  bool waited = false;
  for (int p0 = 8 * NT * blockIdx.y; p0 < rows; p0 += 8 * NT * gridDim.y) {
    const bf16* x[NT];
    bool have[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int row = p0 + 8 * i + gr;
      have[i] = row < rows;
      x[i] = (const bf16*)g.x + (size_t)(have[i] ? row : 0) * g.ldx + 8 * t;
    }
    float c[NT][4] = {}, sum[NT][4] = {};
    const uint4 zero = make_uint4(0, 0, 0, 0);
    for (int s = s0; s < s1; s += UN) {
      uint4 a[UN], b[UN], v[UN][NT];
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        const int kk = 32 * (s + u);
        const bool in = s + u < s1 && kk + 8 * t < g.k;
        a[u] = in ? __ldg(reinterpret_cast<const uint4*>(wa + kk)) : zero;
        b[u] = in ? __ldg(reinterpret_cast<const uint4*>(wb + kk)) : zero;
#pragma unroll
        for (int i = 0; i < NT; ++i)
          v[u][i] = in && have[i] ? *reinterpret_cast<const uint4*>(x[i] + kk) : zero;
      }
#pragma unroll
      for (int u = 0; u < UN; ++u)
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          mma_16816(c[i], a[u].x, b[u].x, a[u].y, b[u].y, v[u][i].x, v[u][i].y);
          mma_16816(c[i], a[u].z, b[u].z, a[u].w, b[u].w, v[u][i].z, v[u][i].w);
        }
      if constexpr (EXACT) {  // (the instruction's own sums cut a bit off per step)
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            sum[i][j] += c[i][j];
            c[i][j] = 0.f;
          }
      }
    }
    if constexpr (EXACT) {
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) c[i][j] = sum[i][j];
    }
    // c[i][0..1]: weight row gr, rows 2 t and 2 t + 1 of part i; c[i][2..3]: row gr + 8
    __syncthreads();  // (the last pass's sums are read)
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        part[warp][gr][8 * i + 2 * t + j] = c[i][j];
        part[warp][gr + 8][8 * i + 2 * t + j] = c[i][2 + j];
      }
    if (!waited) griddep_wait();
    waited = true;
    __syncthreads();
    for (int o = threadIdx.x; o < 16 * 8 * NT; o += FEW_THREADS) {
      const int f = o % 16, row = p0 + o / 16, feature = f0 + f;
      if (feature >= g.n || row >= rows) continue;
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < FEW_WARPS; ++w) v += part[w][f][o / 16];
      if (g.bias) v += g.bias[feature];
      v += delta[(size_t)row * g.n + feature];
      if (g.act == FB_ACT_GELU) v = gelu_f<EXACT>(v);
      if (g.out_type == FB_F32) {
        if (g.gate) v *= g.gate[feature];
        if (g.resid) v += g.resid[(size_t)row * g.ldr + feature];
        put((float*)g.out + (size_t)row * g.ldo + feature, v);
      } else {
        put((bf16*)g.out + (size_t)row * g.ldo + feature, v);
      }
    }
  }
  if (!waited) griddep_wait();
}

// ---- host -------------------------------------------------------------------------------
// Clusters that the current device can hold at once, asked once per device.
template <bool DOWN, bool PARTS>
int resident_clusters(int num_sms) {
  constexpr int DEVICES = 64;
  static std::atomic<int> known[DEVICES];  // zero until a launch has asked (any thread)
  int dev = 0, sms = 0, n = 0;
  if (cudaGetDevice(&dev) == cudaSuccess && dev < DEVICES) {
    n = known[dev].load(std::memory_order_relaxed);
    if (n > 0) return n;
  }
  cudaLaunchConfig_t cfg = {};
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess) {
    cfg.gridDim = dim3(sms / 2 * 2, 1, 1);
    cfg.blockDim = dim3(Warps<PARTS>::THREADS, 1, 1);
    cfg.dynamicSmemBytes = SMEM_BYTES;
    if (cudaOccupancyMaxActiveClusters(&n, adapter_tc_kernel<DOWN, PARTS>, &cfg) == cudaSuccess && n > 0) {
      if (dev < DEVICES) known[dev].store(n, std::memory_order_relaxed);
      return n;
    }
  }
  cudaGetLastError();
  return num_sms / 2;
}

typedef cuuint64_t u64;
// rows of x or t, in boxes of 64, 32, 16 and 8
bool row_maps(CUtensorMap (&m)[4], const void* p, u64 cols, u64 rows, u64 ld) {
  for (int i = 0; i < 4; ++i)
    if (!make_map<2>(&m[i], p, {cols, rows}, {ld}, {BK, 64u >> i}, true)) return false;
  return true;
}

template <bool DOWN, bool PARTS>
cudaError_t launch_tc(const AdapterArgs& g, TcArgs a, const bf16* t, int most, int* err, int num_sms,
                      cudaStream_t st) {
  auto kern = adapter_tc_kernel<DOWN, PARTS>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES);
  if (e != cudaSuccess) return e;
  const u64 K = g.k, N = g.n, R = g.rank, E = g.adapters, rows = g.rows;
  const Terms terms(g.rank, PARTS);
  Maps m{};  // (zero: not used by this form)
  bool ok = row_maps(m.x, g.x, K, rows, g.ldx);
  if (DOWN) {
    ok = ok && make_map<3>(&m.w, g.a, {K, R, E}, {K, R * K}, {BK, W_ROWS, 1}, true);
  } else {
    ok = ok && make_map<3>(&m.w, g.w, {K, N, 1}, {K, N * K}, {BK, W_ROWS, 1}, true);
    if (a.adapter)
      ok = ok && make_map<3>(&m.b, g.b, {R, N, E}, {R, N * R}, {BK, W_ROWS, 1}, true) &&
           row_maps(m.t, t, terms.cols, rows, terms.cols);
    if (!PARTS) ok = ok && make_map<2>(&m.o, g.out, {N, rows}, {(u64)g.ldo}, {32, 16}, false);
  }
  if (!ok) return cudaErrorInvalidValue;
  const int occ = resident_clusters<DOWN, PARTS>(num_sms);
  const int mc = occ < most ? occ : most;
  // no more clusters than there can be tiles: 16 rows at least each but a segment's last
  const int n_ft = (a.n + 2 * W_ROWS - 1) / (2 * W_ROWS);
  const long long groups = a.groups < g.rows ? a.groups : g.rows;
  const long long tiles = (g.rows / T_STEP + groups) * n_ft * (a.ws ? 32 : 1);  // (cut ones in parts)
  const int clusters = tiles < mc ? (int)tiles : mc;
  return launch_k(kern, dim3(2 * clusters), dim3(Warps<PARTS>::THREADS), SMEM_BYTES, st, m, a, err);
}

template <int MT>
cudaError_t launch_delta(const AdapterArgs& g, float* delta, int* err, cudaStream_t st) {
  auto kern = adapter_delta_kernel<MT>;
  const size_t smem = delta_smem<MT>(g.n, g.rank);
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)(delta_smem<MT>(0, FB_ADAPTER_MAX_RANK) + D_STAGE));
  if (e != cudaSuccess) return e;
  const long long chunks = g.rows / D_ROWS + (g.segments < g.rows ? g.segments : g.rows);
  return launch_k(kern, dim3((unsigned)(chunks * D_CTAS)), dim3(D_THREADS), smem, st, g, delta, err);
}

// How a call is computed.
struct Plan {
  bool parts;   // sums in parts (fp32 results, very long K)
  bool by_row;  // the low-rank part formed by itself and added in the epilogue
  bool few;     // (then) the product by streamed weights
  bool cut, cut_t;  // the product's tiles, or t's, may be cut
  int down_clusters, clusters;  // of t's kernel and the product's
  size_t t_bytes, ws_bytes, delta_bytes;
};
size_t padded(size_t n) { return (n + 255) / 256 * 256; }
// Whether forming the low-rank part by itself is faster. In us, fitted to the figures below: it costs
// reading A_e and B_e for every 16 rows, multiplying them by CUDA cores, and writing and reading the
// part, and something to begin with; the K blocks of t cost every segment tiles of its own, which
// take 313 clocks a K block however few rows they have. us by itself / as K blocks (segments x
// rows, n x k, rank): 1536 x 1536, 16: 64 x 4 19.2 / 48.6, 64 x 32 32.5 / 50.4, 64 x 64 53.3 / 51.2,
// 16 x 32 20.8 / 23.6, 16 x 128 31.3 / 31.5, 4 x 256 23.7 / 19.4, 1 x 1560 29.4 / 22.3; rank 64: 64 x 16
// 42.4 / 52.2, 64 x 32 69.5 / 46.8, 1 x 64 17.9 / 14.4; 1536 x 4096, 16: 64 x 64 78.4 / 110, 16 x 128
// 42.0 / 46.6, 1 x 256 27.0 / 22.6 (taken by itself all the same), 1 x 1560 39.0 / 29.5; 8960 x 1536, 16:
// 64 x 64 159 / 208, 16 x 128 88.7 / 70.2, 1 x 64 26.3 / 14.8; 1536 x 8960, 32, fp32: 16 x 128 107 / 120,
// 4 x 1024 198 / 150.
bool short_segments(const AdapterArgs& g, int n_ft) {
  const double n = g.n, k = g.k, r = g.rank, blocks = (k + BK - 1) / BK;
  const double row = 1.1e-7 * r * n + 4e-8 * r * k + 0.003, first = n / 850 * (r / 32 + 0.5);
  const double segment = 1.45 * n_ft * blocks * 313 / 144400;
  return g.rows * row + first < g.segments * segment + 3.5 && g.rows * n < 1 << 28;  // (1 GB of scratch)
}
// Where the product's tiles fit into one round with clusters to spare, those form t meanwhile: the
// product needs it for its last K blocks only, and its launch does not wait for t's. Both together
// have no more clusters than are resident at once. us of a call's launches one after the other / side
// by side: 1560 rows, 1536 x 1536, rank 16 28.8 / 22.8, fp32 34.9 / 26.3; 1536 x 4096 40.4 / 29.5, fp32
// 58.5 / 33.2; 1536 x 8960, rank 32, fp32 72.1 / 51.9; 2200 rows, 1536 x 1536, rank 64 27.2 / 23.7.
void side_by_side(const AdapterArgs& g, int n_ft, Plan* p) {
  if (p->by_row) return;
  const int all = p->clusters;
  for (int T = 128; T <= (p->parts ? F32_T : MAX_T); T += T_STEP) {
    const long long tiles = (long long)(g.rows / T + g.segments) * n_ft;
    if (tiles > all - (all < 8 ? 1 : all / 8)) continue;  // (at least one is left for t)
    p->clusters = (int)tiles;
    p->down_clusters = all - (int)tiles;
    return;
  }
}
// Whether the K blocks of all tiles, 16 units each at most, can be counted in 32 bits.
bool fits(const AdapterArgs& g, int n_ft, const Plan& p) {
  const double tiles = (double)(g.rows / T_STEP + g.segments) * n_ft;
  return tiles * ((g.k + BK - 1) / BK + Terms(g.rank, p.parts).blocks()) * 16 < 4e9;
}
Plan plan_of(const AdapterArgs& g, int num_sms) {
  Plan p{};
  p.parts = in_parts(g);
  const int n_ft = (g.n + 2 * W_ROWS - 1) / (2 * W_ROWS);
  // Streamed weights: up to 8 rows at any rate, up to 32 unless there are tiles for all clusters, and up to
  // 64 (by two blocks a weight row, which both read it) where the tiles leave most SMs without work and the
  // weights are not many. us streamed / in tiles: 32 rows 9216 x 1536 17.7 / 20.7, 1536 x 8960 18.1 / 29.2;
  // 64 rows 1536 x 1536 12.1 / 18.4, 4608 x 1536 17.3 / 21.4, 4096 x 4096 25.5 / 28.2, 1536 x 8960 31.8 / 39.9,
  // 4864 x 8960 52.2 / 41.9, 9216 x 1536 27.5 / 22.4; 40 rows 2048 x 16384 37.8 / 35.5.
  p.few = (g.rows <= 32 && n_ft <= num_sms / 2 * (g.rows <= 8 ? 2 : 1)) ||
          (g.rows <= 64 && n_ft <= num_sms / 8 && (long long)g.n * g.k <= 20 << 20);
  p.by_row = p.few || short_segments(g, n_ft);
  if (p.by_row)
    p.delta_bytes = padded((size_t)g.rows * g.n * sizeof(float));
  else
    p.t_bytes = padded((size_t)g.rows * Terms(g.rank, p.parts).cols * sizeof(bf16));
  p.down_clusters = p.clusters = num_sms / 2;
  side_by_side(g, n_ft, &p);
  // parts of cut tiles: of t, and of the product where the tiles make few rounds
  const long long tiles = (long long)(g.rows / MAX_T) * n_ft;
  p.cut = !p.few && p.clusters == num_sms / 2 && tiles < 4ll * num_sms && fits(g, n_ft, p);
  p.cut_t = !p.by_row && fits(g, 1, p);
  if (p.cut || p.cut_t) p.ws_bytes = num_sms / 2 * 2 * WS_SLOT * sizeof(float);
  return p;
}

template <bool PARTS>
cudaError_t run(const AdapterArgs& g, const Plan& p, uint8_t* ws, int* counters, int* err, int num_sms,
                cudaStream_t st) {
  TcArgs a{};
  a.rows = g.rows;
  a.k = g.k;
  a.rank = g.rank;
  a.adapters = g.adapters;
  a.act = g.act;
  a.bias = g.bias;
  a.resid = g.resid;
  a.ldr = g.ldr;
  a.gate = g.gate;
  a.out = g.out;
  a.out_type = g.out_type;
  a.ldo = g.ldo;
  a.n = g.n;
  a.counters = counters;
  float* parts = (float*)(ws + p.t_bytes + p.delta_bytes);
  a.ws = p.cut ? parts : nullptr;
  cudaError_t e;
  if (p.by_row) {
    float* delta = (float*)ws;
    e = g.rank <= 16   ? launch_delta<1>(g, delta, err, st)
        : g.rank <= 32 ? launch_delta<2>(g, delta, err, st)
                       : launch_delta<4>(g, delta, err, st);
    if (e != cudaSuccess) return e;
    if (p.few) {
      auto kern = g.rows > 16        ? adapter_few_kernel<PARTS, 4, 2, 2>
                  : g.rows > 8       ? adapter_few_kernel<PARTS, 2, 3, 3>
                  : g.k > FEW_LONG_K ? adapter_few_kernel<PARTS, 1, 6, 2>
                                     : adapter_few_kernel<PARTS, 1, 4, 3>;
      return launch_k(kern, dim3((g.n + 15) / 16, g.rows > 32 ? 2 : 1), dim3(FEW_THREADS), 0, st, g, (const float*)delta);
    }
    a.groups = 1;
    a.end = g.offsets + g.segments;
    a.delta = delta;
    return launch_tc<false, PARTS>(g, a, nullptr, num_sms / 2, err, num_sms, st);
  }
  a.groups = g.segments;
  a.offsets = g.offsets;
  a.adapter = g.adapter;
  a.t = (bf16*)ws;
  a.scale = g.scale;
  a.n = g.rank;
  a.ws = p.cut_t ? parts : nullptr;
  e = launch_tc<true, PARTS>(g, a, nullptr, p.down_clusters, err, num_sms, st);
  if (e != cudaSuccess) return e;
  a.n = g.n;
  a.ws = p.cut ? parts : nullptr;
  return launch_tc<false, PARTS>(g, a, a.t, p.clusters, err, num_sms, st);
}

}  // namespace

cudaError_t adapter_set_wait_limit(unsigned long long ns) { return fb_set_wait_limit_tu(ns); }

size_t adapter_ws_bytes(const AdapterArgs& g, int num_sms) {
  const Plan p = plan_of(g, num_sms);
  return p.t_bytes + p.ws_bytes + p.delta_bytes;
}

cudaError_t adapter_gemm(const AdapterArgs& g, void* ws, int* counters, int* err, int num_sms,
                         cudaStream_t st) {
  if (num_sms < 2) return cudaErrorInvalidValue;
  const Plan p = plan_of(g, num_sms);
  return p.parts ? run<true>(g, p, (uint8_t*)ws, counters, err, num_sms, st)
                 : run<false>(g, p, (uint8_t*)ws, counters, err, num_sms, st);
}
