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
//  * warps 10 and 11 load rows of x, then of t, a K block each by turns.
//  * warp 1 issues the MMAs, warps 2-9 of both CTAs run the epilogue.
// fp32 results take K in parts of 4 blocks, each in an accumulator of its own, which the epilogue
// adds up (the tensor core's sums lose about 6e-8 of the result per K block of 64). So do results of
// a K past 2^17.
// Every wait is bounded (mbar_wait): a role that gives up records it and the kernel ends.
#include <atomic>

#include "grouped.cuh"
#include "kernels.h"

namespace {

constexpr int TMEM_COLS = 512;
constexpr int MAX_STAGES = 8, MAX_ACCS = 8;
constexpr int THREADS = 384;
constexpr int MAX_S = FB_ADAPTER_MAX_SEGMENTS;
constexpr int SMEM_BYTES = 229888;  // (room for a block of the low-rank part beside it)
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
constexpr int F32_T = 128;                  // widest tile then (its sums wait in registers)
constexpr int LONG_K = 1 << 17;
bool in_parts(const AdapterArgs& g) { return g.out_type == FB_F32 || g.k > LONG_K; }

// How t's terms lie in a row of the scratch. Ranks up to 64 are rounded up to 16, the terms side by
// side; larger ones to 64, 64 columns of each term by turns. Either way K block i of t is columns 64 i
// and up, chunk j (16 columns) of it meets chunk (4 i + j) % chunks of B_e's box of 64 columns, and
// the box is i / terms (the only one for ranks up to 64).
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

struct TcArgs {
  int groups;               // segments, or (offsets null) one group of the first *end rows
  const int32_t *offsets, *end, *adapter;
  int adapters, rows, n, k; // n: weight rows
  int rank;
  int slices;               // of K, DOWN: each forms a sum of its own
  bf16* t;                  // DOWN with one slice: its terms
  float* part;              // DOWN: [slice][rows][rp]
  const float* scale;       // DOWN
  const float *bias, *delta, *resid, *gate;
  int64_t ldr, ldo;
  int act, out_type;
  void* out;
};

// DOWN: t = scale x A_e^T (n = rank), else the product.
template <bool DOWN, bool PARTS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1)
    adapter_tc_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmB,
                      const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmX8,
                      const __grid_constant__ CUtensorMap tmT, const __grid_constant__ CUtensorMap tmT8,
                      const __grid_constant__ CUtensorMap tmO, const TcArgs g, int* err) {
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

  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t rank = cluster_ctarank();
  const int cluster = blockIdx.x >> 1, n_clusters = gridDim.x >> 1;
  // DOWN: one tile of weight rows, its K slices stand in the tile's place
  const int n_ft = DOWN ? g.slices : (g.n + 2 * W_ROWS - 1) / (2 * W_ROWS);
  const int nk = (g.k + BK - 1) / BK, E = g.groups;
  const Terms terms(g.rank, PARTS);
  const int ext = g.adapter ? terms.blocks() : 0;
  const int chunks = terms.rp <= 64 ? terms.rp / 16 : 4, all_chunks = terms.terms * terms.rp / 16;
  // K blocks kb0 .. of a tile, and how many; the ones of t behind those of x
  auto k_range = [&](const Tile& q, int& kb0, int& blocks) {
    if (DOWN) {
      kb0 = (int)((int64_t)nk * q.f / g.slices);
      blocks = (int)((int64_t)nk * (q.f + 1) / g.slices) - kb0;
    } else {
      kb0 = 0;
      blocks = nk + (who[q.e] >= 0 ? ext : 0);
    }
  };
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
      mbar_init(&tmem_empty[a], 16);  // 8 epilogue warps x 2 CTAs
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_desc(&tmW);
    tma_prefetch_desc(&tmX);
    tma_prefetch_desc(&tmX8);
    if (!DOWN) tma_prefetch_desc(&tmB);
    if (TILES) tma_prefetch_desc(&tmO);
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
    // the width of the least estimated time in SM clocks: 256 + w clocks of operands, or 313 of
    // issue, per K block; in the fullest cluster each tile but the first takes its mainloop or its
    // epilogue
    const int T = T_STEP * (lane + 1);
    const float blocks = DOWN ? (float)nk / g.slices : (float)(nk + ext);
    float est = 3e38f;
    if (lane < WIDTHS && (!PARTS || T <= F32_T)) {
      const float n = (float)count[lane] * n_ft, rounds = ceilf(n / n_clusters);
      const float main = count[lane] ? (float)cost[lane] / count[lane] * blocks : 0.f;
      const float epi = TILES ? 2900.f + 12.f * T : 3300.f + 30.f * T;
      est = main + (rounds - 1.f) * fmaxf(main, epi) + (TILES ? 16.f : 28.f) * T;
    }
    float best = est;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = fminf(best, __shfl_xor_sync(0xffffffffu, best, o));
    const int Tb = T_STEP * __ffs(__ballot_sync(0xffffffffu, est == best));
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
    if (lane == 0) *width = Tb;
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
  const int fit = DOWN ? n_ft : (int)(BAND_BYTES / ((int64_t)2 * W_ROWS * g.k * sizeof(bf16)));
  TileIter ti(off, first, cluster, n_clusters, n_ft, fit < 1 ? 1 : fit < n_ft ? fit : n_ft, E);
  Tile k;
  int kb0, blocks;

  if (warp == 0) {
    // ---------------- weights (both CTAs) ----------------
    int stage = 0;
    uint32_t phase = 0;
    while (!failed && ti.next(k)) {
      const uint32_t bytes = 2 * (W_BYTES + k.w / 2 * BK * 2);
      const int e = who[k.e];
      k_range(k, kb0, blocks);
      for (int i = 0; i < blocks; ++i) {
        if (!mbar_wait_warp(&empty[stage], phase ^ 1u, err)) { failed = true; break; }
        if (elect_one()) {
          const uint32_t dst = smem_u32(smem) + stage * stage_bytes;
          const uint32_t fb = mapa_shared(smem_u32(&full[stage]), 0);
          if (rank == 0) mbar_expect_tx(&full[stage], bytes);
          if (DOWN)
            tma_load_3d_cg2(dst, &tmW, fb, (kb0 + i) * BK, (int)rank * W_ROWS, e);
          else if (i < nk)
            tma_load_3d_cg2(dst, &tmW, fb, i * BK, (2 * k.f + (int)rank) * W_ROWS, 0);
          else
            tma_load_3d_cg2(dst, &tmB, fb, terms.rp <= 64 ? 0 : (i - nk) / terms.terms * BK,
                            (2 * k.f + (int)rank) * W_ROWS, e);
        }
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp >= 10) {
    // ---------------- rows of x and t (both CTAs) ----------------
    int stage = 0;
    uint32_t phase = 0;
    int turn = warp - 10;  // K blocks until this warp's next: they go round the two
    bool waited = DOWN;
    while (!failed && ti.next(k)) {
      const int half = k.w / 2, a0 = k.r0 + half * (int)rank;
      k_range(k, kb0, blocks);
      for (int i = 0; i < blocks; ++i) {
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
            const CUtensorMap *m64 = of_t ? &tmT : &tmX, *m8 = of_t ? &tmT8 : &tmX8;
            const int x = (of_t ? i - nk : kb0 + i) * BK;
            int r = 0;
            for (; r + 64 <= half; r += 64) tma_load_rows_cg2(dst + r * (BK * 2), m64, fb, x, a0 + r);
            for (; r < half; r += 8) tma_load_rows_cg2(dst + r * (BK * 2), m8, fb, x, a0 + r);
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
      while (!failed && ti.next(k)) {
        const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(k.w >> 3) << 17) |
                               ((uint32_t)(2 * W_ROWS >> 4) << 24);
        k_range(k, kb0, blocks);
        // the tile's K parts, each in the ring's next accumulator
        const int part_len = PARTS ? PART_BLOCKS : blocks;
        for (int i = 0; !failed && i < blocks;) {
          if (!mbar_wait_warp(&tmem_empty[acc], acc_phase ^ 1u, err)) { failed = true; break; }
          tc_fence_after();
          const uint32_t d_tmem = tmem_base + acc * acc_cols;
          const int start = i, end = blocks - i < part_len ? blocks : i + part_len;
          for (; i < end; ++i) {
            if (!mbar_wait_warp(&full[stage], phase, err)) { failed = true; break; }
            tc_fence_after();
            const uint32_t wlo = ring_lo + (uint32_t)(stage * (stage_bytes >> 4));
            const uint32_t alo = wlo + (W_BYTES >> 4);
            if (DOWN || i < nk) {
              if (elect_one()) {
#pragma unroll
                for (int j = 0; j < BK / 16; ++j)
                  tc_mma_cg2_lo(d_tmem, wlo + 2 * j, alo + 2 * j, DESC_HI, idesc,
                                (i > start || j > 0) ? 1u : 0u);
                tc_commit_mc(&empty[stage], 0x3);
                if (i + 1 == end) tc_commit_mc(&tmem_full[acc], 0x3);
              }
            } else if (elect_one()) {  // t: chunks of 16 columns against B_e's
              const int c0 = 4 * (i - nk);
#pragma unroll 1
              for (int j = 0; j < 4 && c0 + j < all_chunks; ++j)
                tc_mma_cg2_lo(d_tmem, wlo + 2 * ((c0 + j) % chunks), alo + 2 * j, DESC_HI, idesc,
                              (i > start || j > 0) ? 1u : 0u);
              tc_commit_mc(&empty[stage], 0x3);
              if (i + 1 == end) tc_commit_mc(&tmem_full[acc], 0x3);
            }
            if (++stage == stages) { stage = 0; phase ^= 1u; }
          }
          if (++acc == n_accs) { acc = 0; acc_phase ^= 1u; }
        }
      }
    }
  } else {
    // ---------------- epilogue (warps 2..9 of both CTAs) ----------------
    // warp: weight rows quarter * 32 .. + 31 of this CTA's 128 (its TMEM lanes), every other
    // CH-token chunk of the tile
    constexpr int CH = PARTS ? 16 : 32;
    const int quarter = warp & 3, we = warp - 2;
    int half = we >> 2;  // a tile's first chunk goes to either half by turns
    const uint32_t te_remote = mapa_shared(smem_u32(&tmem_empty[0]), 0);
    uint8_t* tiles = epi_smem + we * 2 * EPI_TILE;
    int acc = 0, buf = 0;
    uint32_t acc_phase = 0;
    bool waited = DOWN || !g.delta;
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
    bool more = ti.next(k);
    float bias = more ? bias_of(k) : 0.f;
    for (; !failed && more; k = after) {
      more = ti.next(after);
      const float bias_after = more ? bias_of(after) : 0.f;  // (it may come from memory)
      const int f0 = first_feature(k), feature = f0 + lane;
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16);
      if (!waited) {
        griddep_wait();
        waited = true;
      }
      k_range(k, kb0, blocks);
      // the low-rank part of CH tokens from t0 on
      auto add_delta = [&](float* v, int t0) {
        if (DOWN || !g.delta) return;
        const int n = k.nv - t0;
        const float* from = g.delta + (size_t)(k.r0 + t0) * g.n + feature;
        float d[CH];
#pragma unroll
        for (int j = 0; j < CH; ++j) d[j] = j < n && feature < g.n ? from[(size_t)j * g.n] : 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j) v[j] += d[j];
      };
      // sums in parts: added up here as they are done, a part's accumulator going back at once
      float sum[PARTS ? F32_T / 2 : 1];
      bool ok = true;
      const int parts = PARTS ? (blocks + PART_BLOCKS - 1) / PART_BLOCKS : 1;
      for (int p = 0; p < parts; ++p) {
        ok = __all_sync(0xffffffffu, mbar_wait(&tmem_full[acc], acc_phase, err));
        if (!ok) break;
        tc_fence_after();
        if constexpr (PARTS) {
#pragma unroll
          for (int c = 0; c < F32_T / (2 * CH); ++c) {
            const int t0 = (half + 2 * c) * CH;
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
      constexpr int UNROLL = PARTS ? F32_T / (2 * CH) : 1;  // (sum's indices are constants)
#pragma unroll UNROLL
      for (int c = 0; c < (PARTS ? F32_T : MAX_T) / (2 * CH); ++c) {
        const int t0 = (half + 2 * c) * CH;
        if (t0 >= k.nv || f0 >= limit) break;
        float v[CH];
        if constexpr (PARTS) {
#pragma unroll
          for (int j = 0; j < CH; ++j) v[j] = sum[c * CH + j];
        } else {
          uint32_t r[32];
          tmem_ld32(taddr + acc * acc_cols + t0, r);
          tmem_ld_wait();
          reg_fence32(r);
#pragma unroll
          for (int j = 0; j < CH; ++j) v[j] = __uint_as_float(r[j]);
        }
        const int n = k.nv - t0 < CH ? k.nv - t0 : CH;  // tokens of the chunk that exist
        if constexpr (DOWN) {
          const bool in = feature < g.n;  // (columns up to rp are zeros)
          if (feature < terms.rp) {
            const size_t row = k.r0 + t0;
            if (g.slices > 1) {
              float* at = g.part + ((size_t)k.f * g.rows + row) * terms.rp + feature;
#pragma unroll
              for (int j = 0; j < CH; ++j)
                if (j < n) at[(size_t)j * terms.rp] = in ? v[j] * bias : 0.f;
            } else {
              bf16* at = g.t + row * terms.cols;
#pragma unroll
              for (int j = 0; j < CH; ++j) {
                if (j >= n) continue;
                float x = in ? v[j] * bias : 0.f;
                for (int s = 0; s < terms.terms; ++s) {
                  const bf16 b = __float2bfloat16(x);
                  at[(size_t)j * terms.cols + terms.column(s, feature)] = b;
                  x -= __bfloat162float(b);
                }
              }
            }
          }
        } else if constexpr (PARTS) {
          // straight to memory, 32 features of a token
          add_delta(v, t0);
          const size_t row = k.r0 + t0;
          const bool in = feature < g.n;
          float rs[CH];
#pragma unroll
          for (int j = 0; j < CH; ++j)
            rs[j] = g.resid && in && j < n ? g.resid[(row + j) * g.ldr + feature] : 0.f;
          const float gate = g.gate && in ? __ldg(g.gate + feature) : 1.f;
#pragma unroll
          for (int j = 0; j < CH; ++j) {
            float x = v[j] + bias;
            if (g.act == FB_ACT_GELU) x = gelu_f<true>(x);
            if (!in || j >= n) continue;
            if (g.out_type == FB_F32)
              put(reinterpret_cast<float*>(g.out) + (row + j) * g.ldo + feature, fmaf(gate, x, rs[j]));
            else
              put(reinterpret_cast<bf16*>(g.out) + (row + j) * g.ldo + feature, x);
          }
        } else {
          add_delta(v, t0);
          uint8_t* tile = tiles + buf * EPI_TILE;
          buf ^= 1;
          if (elect_one()) bulk_wait_read<1>();  // the store from this tile two chunks ago
          __syncwarp();
          // two tokens' values of each lane's feature as one 4-byte store per lane: lanes
          // exchange with their neighbour, even lanes then hold two features of token j, odd
          // lanes of token j + 1
          uint32_t* tw = reinterpret_cast<uint32_t*>(tile) + (lane & 1) * 16 + (lane >> 1);
#pragma unroll
          for (int j = 0; j < CH; j += 2) {
            float y0 = v[j] + bias, y1 = v[j + 1] + bias;
            if (g.act == FB_ACT_GELU) gelu_f2(y0, y1);
            const float got = __shfl_xor_sync(0xffffffffu, (lane & 1) ? y0 : y1, 1);
            tw[j * 16] = (lane & 1) ? pack_bf16x2(got, y1) : pack_bf16x2(y0, got);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (elect_one()) {
#pragma unroll
            for (int b = 0; b < CH; b += 16)
              if (b + 16 <= n) tma_store_2d(&tmO, smem_u32(tile) + b * 64, f0, k.r0 + t0 + b);
            bulk_commit();
          }
          if (n % 16) {  // 16 bytes at a time: n is a multiple of 8 features
            const int b = n / 16 * 16;
            for (int i = lane; i < (n - b) * 4; i += 32) {
              const int tok = b + i / 4, q = i % 4;
              if (f0 + q * 8 < g.n)
                *reinterpret_cast<uint4*>(reinterpret_cast<bf16*>(g.out) +
                                          (size_t)(k.r0 + t0 + tok) * g.ldo + f0 + q * 8) =
                    *reinterpret_cast<const uint4*>(tile + tok * 64 + q * 16);
            }
            __syncwarp();
          }
        }
      }
      if constexpr (!PARTS) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_relaxed_cluster(te_remote + acc * (uint32_t)sizeof(uint64_t));
        if (++acc == n_accs) { acc = 0; acc_phase ^= 1u; }
      }
      bias = bias_after;
      half ^= 1;
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

// t's terms from the sums of K's slices, in slice order.
__global__ void __launch_bounds__(256) adapter_terms_kernel(const float* part, int slices, int rows,
                                                            Terms terms, bf16* t) {
  griddep_wait();
  griddep_launch();
  const size_t n = (size_t)rows * terms.rp;
  for (size_t i = blockIdx.x * 256ull + threadIdx.x; i < n; i += gridDim.x * 256ull) {
    float x = 0.f;
#pragma unroll 4
    for (int s = 0; s < slices; ++s) x += part[s * n + i];
    bf16* row = t + i / terms.rp * terms.cols;
    for (int s = 0; s < terms.terms; ++s) {
      const bf16 b = __float2bfloat16(x);
      row[terms.column(s, (int)(i % terms.rp))] = b;
      x -= __bfloat162float(b);
    }
  }
}

// ---- short segments ---------------------------------------------------------------------
// The low-rank part of up to 16 rows of a segment, scale (x A_e^T) B_e^T in fp32, by a cluster of
// eight CTAs: each forms its eighth of K's sums of t (mma.sync, A_e and x straight from memory into the
// operand registers, A_e the M side), all of them add the eighths up in CTA order through distributed
// shared memory, and each multiplies t with its eighth of B_e's rows (a feature per thread). What
// counts is to have all of A_e and B_e on their way at once. Rows without an adapter get zeros.
constexpr int D_CTAS = 8, D_WARPS = 8, D_THREADS = 32 * D_WARPS, D_ROWS = 16, D_RANKS = 64;
constexpr int D_SMEM = (D_WARPS * D_RANKS * D_ROWS + 2 * FB_ADAPTER_MAX_RANK * D_ROWS) * 4;

__device__ __forceinline__ float ld_cluster(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

__global__ void __cluster_dims__(D_CTAS, 1, 1) __launch_bounds__(D_THREADS, 2)
    adapter_delta_kernel(const AdapterArgs g, float* delta, int* err) {
  griddep_wait();
  griddep_launch();
  extern __shared__ __align__(16) float sm[];
  float* part = sm;                                     // [warp][64 of the rank][16 rows]
  float* own = part + D_WARPS * D_RANKS * D_ROWS;       // [rank][16]: this CTA's sums
  float* t = own + FB_ADAPTER_MAX_RANK * D_ROWS;        // [rank][16]: all of them
  __shared__ int found[4], scan[D_WARPS];
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  const uint32_t c = cluster_ctarank();
  const int want = blockIdx.x / D_CTAS;
  // ---- the want-th chunk of 16 rows: each thread up to four segments ----
  if (tid == 0) found[0] = -2;
  int chunks[4], sum = 0;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int s = 4 * tid + i;
    chunks[i] = 0;
    if (s < g.segments) {
      const int a = g.offsets[s], b = g.offsets[s + 1], e = g.adapter[s];
      bad = bad || a < 0 || b < a || b > g.rows || (s == 0 && a != 0) || e < -1 || e >= g.adapters;
      chunks[i] = (b - a + D_ROWS - 1) / D_ROWS;
      sum += chunks[i];
    }
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
    if (want >= at && want < at + chunks[i]) {
      const int s = 4 * tid + i;
      found[0] = g.adapter[s];
      found[1] = g.offsets[s] + (want - at) * D_ROWS;
      found[2] = g.offsets[s + 1];
    }
    at += chunks[i];
  }
  __syncthreads();
  const int e = found[0], r0 = found[1];
  if (e == -2) return;  // (the whole cluster)
  const int rows = found[2] - r0 < D_ROWS ? found[2] - r0 : D_ROWS;
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
    cluster_sync();
    const float scale = g.scale ? g.scale[e] : 1.f;
    for (int i = tid; i < g.rank * D_ROWS; i += D_THREADS) {
      float v = 0.f;
#pragma unroll
      for (uint32_t p = 0; p < D_CTAS; ++p) v += ld_cluster(mapa_shared(smem_u32(own + i), p));
      t[i] = v * scale;
    }
    cluster_sync();  // (no CTA leaves while its sums are read)
  }
  // ---- the product with this CTA's rows of B_e ----
  const int fa = (int)((int64_t)g.n * c / D_CTAS), fb = (int)((int64_t)g.n * (c + 1) / D_CTAS);
  for (int f = fa + tid; f < fb; f += D_THREADS) {
    float y[D_ROWS] = {};
    if (e >= 0) {
      const bf16* b = (const bf16*)g.b + ((size_t)e * g.n + f) * g.rank;
#pragma unroll 2
      for (int r = 0; r < g.rank; r += 8) {
        float w[8];
        load_bf16x8(b + r, w);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (4 * j >= rows) break;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float4 v = *reinterpret_cast<const float4*>(t + (r + i) * D_ROWS + 4 * j);
            y[4 * j] = fmaf(w[i], v.x, y[4 * j]);
            y[4 * j + 1] = fmaf(w[i], v.y, y[4 * j + 1]);
            y[4 * j + 2] = fmaf(w[i], v.z, y[4 * j + 2]);
            y[4 * j + 3] = fmaf(w[i], v.w, y[4 * j + 3]);
          }
        }
      }
    }
#pragma unroll
    for (int j = 0; j < D_ROWS; ++j)
      if (j < rows) delta[(size_t)(r0 + j) * g.n + f] = y[j];
  }
}

// ---- few rows ---------------------------------------------------------------------------
// Up to 32 rows read every weight once: a block takes 16 weight rows, its warps split K, and the
// weights go straight from memory into the operand registers of mma.sync (the weights are the M
// side, eight rows of x the N side), as in the products grouped by expert. The weights do not wait
// for the low-rank part; the epilogue does.
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
  for (int p0 = 0; p0 < rows; p0 += 8 * NT) {
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
    cfg.blockDim = dim3(THREADS, 1, 1);
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
// rows of x or t, in boxes of 64 and 8 rows
bool row_maps(CUtensorMap* m64, CUtensorMap* m8, const void* p, u64 cols, u64 rows, u64 ld) {
  return make_map<2>(m64, p, {cols, rows}, {ld}, {BK, 64}, true) &&
         make_map<2>(m8, p, {cols, rows}, {ld}, {BK, 8}, true);
}

template <bool DOWN, bool PARTS>
cudaError_t launch_tc(const AdapterArgs& g, TcArgs a, const bf16* t, int* err, int num_sms, cudaStream_t st) {
  auto kern = adapter_tc_kernel<DOWN, PARTS>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES);
  if (e != cudaSuccess) return e;
  const u64 K = g.k, N = g.n, R = g.rank, E = g.adapters, rows = g.rows;
  const Terms terms(g.rank, PARTS);
  CUtensorMap mw, mb{}, mx, mx8, mt{}, mt8{}, mo{};  // (zero: not used by this form)
  bool ok = row_maps(&mx, &mx8, g.x, K, rows, g.ldx);
  if (DOWN) {
    ok = ok && make_map<3>(&mw, g.a, {K, R, E}, {K, R * K}, {BK, W_ROWS, 1}, true);
  } else {
    ok = ok && make_map<3>(&mw, g.w, {K, N, 1}, {K, N * K}, {BK, W_ROWS, 1}, true);
    if (a.adapter)
      ok = ok && make_map<3>(&mb, g.b, {R, N, E}, {R, N * R}, {BK, W_ROWS, 1}, true) &&
           row_maps(&mt, &mt8, t, terms.cols, rows, terms.cols);
    if (!PARTS) ok = ok && make_map<2>(&mo, g.out, {N, rows}, {(u64)g.ldo}, {32, 16}, false);
  }
  if (!ok) return cudaErrorInvalidValue;
  const int occ = resident_clusters<DOWN, PARTS>(num_sms);
  const int mc = occ < num_sms / 2 ? occ : num_sms / 2;
  // no more clusters than there can be tiles: 16 rows at least each but a segment's last
  const int n_ft = DOWN ? a.slices : (g.n + 2 * W_ROWS - 1) / (2 * W_ROWS);
  const long long groups = a.groups < g.rows ? a.groups : g.rows;
  const long long tiles = (g.rows / T_STEP + groups) * n_ft;
  const int clusters = tiles < mc ? (int)tiles : mc;
  return launch_k(kern, dim3(2 * clusters), dim3(THREADS), SMEM_BYTES, st, mw, mb, mx, mx8, mt, mt8, mo, a, err);
}

// How a call is computed.
struct Plan {
  bool parts;   // sums in parts (fp32 results, very long K)
  bool by_row;  // the low-rank part formed by itself and added in the epilogue
  bool few;     // (then) the product by streamed weights
  int slices;   // of K, for t
  size_t t_bytes, part_bytes, delta_bytes;
};
size_t padded(size_t n) { return (n + 255) / 256 * 256; }
Plan plan_of(const AdapterArgs& g, int num_sms) {
  Plan p{};
  p.parts = in_parts(g);
  const int n_ft = (g.n + 2 * W_ROWS - 1) / (2 * W_ROWS);
  p.few = g.rows <= 32 && n_ft <= num_sms / 2 * (g.rows <= 8 ? 2 : 1);
  p.by_row = p.few || g.rows < 24 * g.segments;
  p.slices = 1;
  if (p.by_row) {
    p.delta_bytes = padded((size_t)g.rows * g.n * sizeof(float));
    return p;
  }
  const Terms terms(g.rank, p.parts);
  // t has a tile of weight rows alone: K is cut so that every cluster has about two tiles, of at
  // least eight K blocks
  const long long tiles = g.rows / (p.parts ? 128 : 256) + g.segments, nk = (g.k + BK - 1) / BK;
  long long s = (num_sms + tiles - 1) / tiles;
  if (s > nk / 8) s = nk / 8;
  p.slices = s < 1 ? 1 : s > 32 ? 32 : (int)s;
  p.t_bytes = padded((size_t)g.rows * terms.cols * sizeof(bf16));
  if (p.slices > 1) p.part_bytes = padded((size_t)p.slices * g.rows * terms.rp * sizeof(float));
  return p;
}

template <bool PARTS>
cudaError_t run(const AdapterArgs& g, const Plan& p, uint8_t* ws, int* err, int num_sms, cudaStream_t st) {
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
  cudaError_t e;
  if (p.by_row) {
    float* delta = (float*)ws;
    e = cudaFuncSetAttribute(adapter_delta_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, D_SMEM);
    if (e != cudaSuccess) return e;
    const long long chunks = g.rows / D_ROWS + (g.segments < g.rows ? g.segments : g.rows);
    e = launch_k(adapter_delta_kernel, dim3((unsigned)(chunks * D_CTAS)), dim3(D_THREADS), D_SMEM, st, g,
                 delta, err);
    if (e != cudaSuccess) return e;
    if (p.few) {
      auto kern = g.rows > 8        ? adapter_few_kernel<PARTS, 2, 4, 2>
                  : g.k > FEW_LONG_K ? adapter_few_kernel<PARTS, 1, 6, 2>
                                     : adapter_few_kernel<PARTS, 1, 4, 3>;
      return launch_k(kern, dim3((g.n + 15) / 16), dim3(FEW_THREADS), 0, st, g, (const float*)delta);
    }
    a.groups = 1;
    a.end = g.offsets + g.segments;
    a.delta = delta;
    return launch_tc<false, PARTS>(g, a, nullptr, err, num_sms, st);
  }
  a.groups = g.segments;
  a.offsets = g.offsets;
  a.adapter = g.adapter;
  a.slices = p.slices;
  a.t = (bf16*)ws;
  a.part = (float*)(ws + p.t_bytes);
  a.scale = g.scale;
  a.n = g.rank;
  e = launch_tc<true, PARTS>(g, a, nullptr, err, num_sms, st);
  if (e != cudaSuccess) return e;
  if (p.slices > 1) {
    const Terms terms(g.rank, PARTS);
    const long long need = ((long long)g.rows * terms.rp + 255) / 256, most = 8ll * num_sms;
    e = launch_k(adapter_terms_kernel, dim3((unsigned)(need < most ? need : most)), dim3(256), 0, st,
                 (const float*)a.part, p.slices, g.rows, terms, a.t);
    if (e != cudaSuccess) return e;
  }
  a.n = g.n;
  return launch_tc<false, PARTS>(g, a, a.t, err, num_sms, st);
}

}  // namespace

cudaError_t adapter_set_wait_limit(unsigned long long ns) { return fb_set_wait_limit_tu(ns); }

size_t adapter_ws_bytes(const AdapterArgs& g, int num_sms) {
  const Plan p = plan_of(g, num_sms);
  return p.t_bytes + p.part_bytes + p.delta_bytes;
}
int adapter_launches(const AdapterArgs& g, int num_sms) { return plan_of(g, num_sms).slices > 1 ? 3 : 2; }

cudaError_t adapter_gemm(const AdapterArgs& g, void* ws, int* err, int num_sms, cudaStream_t st) {
  if (num_sms < 2) return cudaErrorInvalidValue;
  const Plan p = plan_of(g, num_sms);
  return p.parts ? run<true>(g, p, (uint8_t*)ws, err, num_sms, st)
                 : run<false>(g, p, (uint8_t*)ws, err, num_sms, st);
}
