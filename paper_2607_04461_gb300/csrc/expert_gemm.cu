// Matrix products grouped by expert: rows offsets[e] .. offsets[e + 1] - 1 of the output are
//   out[r] = act(x W_e^T + b_e),  x = A[index[r]] (or row r of A)
// with act GELU (tanh form) or, over W_e's 2 n rows (gate rows, then up rows), SiLU or GELU of
// the first n results times the other n. The sizes of the groups are read on the device.
//
// tcgen05 kernel, a cluster of two CTAs per tile of 256 weight rows x w tokens of one expert
// (cta_group::2): the weight rows are the MMA's M side (128 per CTA, one per TMEM lane), the
// tokens its N side, any multiple of 16 up to 256, so that ragged groups cost at most 15 rows
// of padding each. Every CTA reads the offsets, picks the widest tile T that the launch uses
// (choose_width) and cuts each group into equal tiles no wider than that; clusters take the
// tiles in turn, weight rows fastest within a band of 16 MB of them (BAND_BYTES), then the
// expert's tokens, then its next band: so the weights are read from memory once.
//  * warp 0 loads weights, one TMA box of 128 rows x 64 k. Gated weights come as 16 gate rows
//    and 16 up rows by turns (a 5-dimensional map over the two halves), so that the two values
//    an output needs lie 16 lanes apart in one warp, and the weights stay as they are.
//  * warps 10 and up load token rows, a K block each by turns: boxes of 64 and 8 consecutive
//    rows, or with an index four rows of anywhere at a time (tile::gather4).
//  * warp 1 issues the MMAs, warps 2-9 of both CTAs run the epilogue: bias and activation on
//    TMEM columns, bf16 results through a shared-memory tile and TMA boxes of 16 tokens (the last,
//    partly filled box of a group leaves by plain stores, since the rows behind it are the next
//    expert's), fp32 results straight to memory (us, straight / through tiles, 8000 rows over 8
//    experts: fp32, 4096 x 512 gated 87 / 103, 4096 x 1536 107 / 110; bf16, 4096 x 512, with an epilogue by
//    the hardware tanh, 39 / 36).
// Sums are fp32 in TMEM. The tensor core's sums lose about 6e-8 of the result per K block of 64,
// which fp32 results would show: they take K in parts of 4 blocks, each into an accumulator of
// the ring, and the epilogue warps add the parts up; their tiles are no wider than 128. 2-norm of
// the error and us with parts of 3 / 4 / 7 / 14 blocks and one chain, 8192 rows over 8 experts,
// 4096 x 1536: 1.8e-7 113, 2.3e-7 110, 3.4e-7 107, 7.2e-7 106, 1.5e-6 104 (fp32 sums in order
// 3.2e-7).
// Every wait is bounded (mbar_wait): a role that gives up records it and the kernel ends.
#include <cudaTypedefs.h>

#include <atomic>

#include "kernels.h"

namespace {

constexpr int BK = 64;                  // 64 bf16 = 128 bytes: one swizzle row
constexpr int W_ROWS = 128;             // weight rows of a CTA
constexpr int W_BYTES = W_ROWS * BK * 2;
constexpr int TMEM_COLS = 512;
constexpr int MAX_STAGES = 8, MAX_ACCS = 8;
// Warps: weight loader, MMA, 8 epilogue warps, token loaders: two, or four that gather rows (in
// fp32, whose epilogue holds its sums in registers, two).
template <bool F32, bool GATHER>
struct Warps {
  static constexpr int LOADERS = GATHER && !F32 ? 4 : 2, THREADS = 32 * (10 + LOADERS);
};
constexpr int MAX_T = 256, T_STEP = 16, WIDTHS = MAX_T / T_STEP;
constexpr int MAX_E = FB_ROUTE_MAX_EXPERTS;
constexpr int SMEM_BYTES = 229888;      // (room for a normalisation block beside it, as the GEMM's)
constexpr int EPI_TILE = 2048;          // an epilogue warp's tile: 32 tokens x 32 rows, bf16
constexpr int EPI_BYTES = 8 * 2 * EPI_TILE;
constexpr int TABLE_BYTES = (2 * (MAX_E + 8) * 4 + 127) / 128 * 128;
constexpr int BAR_BYTES = 512;
__host__ __device__ constexpr int ring_bytes(bool f32) {  // (fp32 results use no tiles)
  return SMEM_BYTES - BAR_BYTES - TABLE_BYTES - (f32 ? 0 : EPI_BYTES);
}
static_assert(ring_bytes(false) % 128 == 0, "TMA tiles lie on 128-byte boundaries");
// The weights that the clusters take before an expert's next tokens: a band of its weight tiles
// that stays in L2 while all of the expert's tokens pass. us with bands of 16 / 32 / 64 MB / all
// of an expert: 2 experts of 120 MB, 380 rows each 70.7 / 71.3 / 74.3 / 87.4; 4 of 147 MB, 2000
// rows each 673 / 678 / 708 / 779; 8 of 73 MB, 3000 rows each 1037 / 1051 / 1120 / 1144; 8 of
// 28 MB, 390 rows each 71.6 / 72.0 / 71.4 / 71.8.
constexpr int64_t BAND_BYTES = 16ll << 20;
constexpr int PART_BLOCKS = 4;          // K blocks of one accumulator, for fp32 results
constexpr int F32_T = 128;              // widest tile then (its sums wait in registers)
// bf16 results of a longer K take the fp32 results' way (F32 in the templates: sums in parts, a
// thread's results straight to memory). One chain loses up to 6e-9 of the result per element of K
// where all terms have one sign, and keeps the epilogue waiting for all of it: 2-norm of the error
// of such bf16 results, one chain / parts (rounding alone 1.1e-3 to 1.8e-3), K = 65536 1.82e-3 /
// 1.78e-3, 2^18 2.4e-3 / 1.73e-3, 2^20 6.2e-3 / 1.29e-3, 2^23 4.9e-2 / 4e-4.
constexpr int LONG_K = 1 << 17;
bool in_parts(const ExpertArgs& g) { return g.out_type == FB_F32 || g.k > LONG_K; }

__host__ __device__ __forceinline__ int acc_cols_of(int T) { return (T + 31) / 32 * 32; }

// ---- activations ------------------------------------------------------------------------
// x sigmoid(z) as x / (1 + e^-z), z = x (SiLU) or 2 sqrt(2/pi) (x + 0.044715 x^3) (GELU): the
// same as x / 2 (1 + tanh(z / 2)), whose two terms cancel at negative x, so that the hardware
// tanh's error (up to 2^-11 of it) can be 10 % of SiLU at -6 and more than all of GELU at -4.
// EXACT, for fp32 results: expf and a quotient of 2 units. For bf16 results the hardware's ex2 and
// reciprocal (2^-22 each), which with the roundings of z stay below 2^-14 of the result; in both
// the result may be 0 where the divisor passes 2^126 (z < -87). Two instructions of the
// special-function unit for the tanh's one: 8000 rows over 8 experts, us with tanh / as here,
// 4096 x 512 GELU 36.6 / 38.1, SwiGLU 59.0 / 62.7; 4096 x 1536 and up the same within 1 %.
__device__ __forceinline__ float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float LOG2E = 1.4426950408889634f;
constexpr float GELU_K0 = -1.5957691216057308f, GELU_K1 = 0.044715f;  // -2 sqrt(2/pi)
constexpr float GELU_C0 = GELU_K0 * LOG2E, GELU_C1 = GELU_C0 * GELU_K1;
template <bool EXACT>
__device__ __forceinline__ float gelu_f(float x) {
  if (EXACT) return __fdividef(x, 1.f + expf(GELU_K0 * (x + GELU_K1 * x * x * x)));
  return x * rcp_approx(1.f + ex2_approx(x * fmaf(x * x, GELU_C1, GELU_C0)));
}
// gelu_f<false> on a pair, its fp32 arithmetic packed
__device__ __forceinline__ void gelu_f2(float& a, float& b) {
  const uint64_t x = f2_join(a, b);
  float z0, z1, d0, d1;
  f2_split(f2_mul(x, f2_fma(f2_mul(x, x), f2_join(GELU_C1, GELU_C1), f2_join(GELU_C0, GELU_C0))),
           z0, z1);
  f2_split(f2_add(f2_join(ex2_approx(z0), ex2_approx(z1)), f2_join(1.f, 1.f)), d0, d1);
  f2_split(f2_mul(x, f2_join(rcp_approx(d0), rcp_approx(d1))), a, b);
}
template <bool EXACT>
__device__ __forceinline__ float silu_of(float x) {
  if (EXACT) return __fdividef(x, 1.f + expf(-x));
  return x * rcp_approx(1.f + ex2_approx(-LOG2E * x));
}

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(bf16* p, float x) { *p = __float2bfloat16(x); }

// ---- TMA --------------------------------------------------------------------------------
__device__ __forceinline__ void tma_load_3d_cg2(uint32_t dst, const CUtensorMap* map, uint32_t bar,
                                                int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_load_5d_cg2(uint32_t dst, const CUtensorMap* map, uint32_t bar,
                                                int x, int d1, int d2, int d3, int d4) {
  asm volatile(
      "cp.async.bulk.tensor.5d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(d1), "r"(d2), "r"(d3), "r"(d4), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_load_rows_cg2(uint32_t dst, const CUtensorMap* map,
                                                  uint32_t bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
      : "memory");
}
// four rows of anywhere (the map's box is one row)
__device__ __forceinline__ void tma_gather4_cg2(uint32_t dst, const CUtensorMap* map, uint32_t bar,
                                                int x, int r0, int r1, int r2, int r3) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile::gather4.mbarrier::"
      "complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(r0), "r"(r1), "r"(r2), "r"(r3), "r"(bar)
      : "memory");
}

// An arrival that orders no memory: it says that TMEM has been read (tcgen05.wait::ld has returned),
// nothing else. A release at cluster scope waits for the warp's stores to be performed.
__device__ __forceinline__ void mbar_arrive_relaxed_cluster(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr)
               : "memory");
}

// ---- tiles ------------------------------------------------------------------------------
struct Tile {
  int e, f, r0, w, nv;  // expert, weight-row tile, first row, width, rows of it that exist
};
// The tiles of this cluster, one after the other. off: the group offsets; first: the token
// tiles before each group's. Most calls divide once or not at all.
struct TileIter {
  const int *off, *first;
  int t, step, n_ft, band, n_tiles, E;
  // the group of tile t: its tiles [start, end), rows [r0, r1), token tiles nt of `base` steps of
  // 16 rows, the first `more` of them of one more
  int e = 0, start = 0, end = 0, r0 = 0, r1 = 0, nt = 1, base = 0, more = 0;
  __device__ TileIter(const int* off_, const int* first_, int c, int G, int n_ft_, int band_, int E_)
      : off(off_), first(first_), t(c), step(G), n_ft(n_ft_), band(band_),
        n_tiles(first_[E_] * n_ft_), E(E_) {}
  // (the whole warp, converged)
  __device__ bool next(Tile& k) {
    if (t >= n_tiles) return false;
    if (t >= end) {  // the first group whose end lies behind t
      const int lane = threadIdx.x % 32;
      while (true) {
        const unsigned m =
            __ballot_sync(0xffffffffu, e + lane < E && first[e + lane + 1] * n_ft > t);
        if (m) {
          e += __ffs(m) - 1;
          break;
        }
        e += 32;
      }
      start = first[e] * n_ft;
      end = first[e + 1] * n_ft;
      r0 = off[e];
      r1 = off[e + 1];
      // its steps dealt out evenly: at most 15 rows of padding in all
      const int steps = (r1 - r0 + T_STEP - 1) / T_STEP;
      nt = first[e + 1] - first[e];
      base = nt > 1 ? steps / nt : steps;
      more = steps - base * nt;
    }
    const int u = t - start, f0 = n_ft > band ? u / (nt * band) * band : 0, v = u - f0 * nt;
    const int bw = n_ft - f0 < band ? n_ft - f0 : band;  // weight tiles of this band
    const int j = nt > 1 ? v / bw : 0;
    t += step;
    k.e = e;
    k.f = f0 + v - j * bw;
    k.w = (base + (j < more)) * T_STEP;
    k.r0 = r0 + (j * base + (j < more ? j : more)) * T_STEP;
    k.nv = r1 - k.r0 < k.w ? r1 - k.r0 : k.w;
    return true;
  }
};

template <bool GATED, bool F32, bool GATHER>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Warps<F32, GATHER>::THREADS, 1)
    expert_tc_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmA,
                     const __grid_constant__ CUtensorMap tmA8, const __grid_constant__ CUtensorMap tmO,
                     const ExpertArgs g, int* err) {
  constexpr int THREADS = Warps<F32, GATHER>::THREADS, LOADERS = Warps<F32, GATHER>::LOADERS;
  extern __shared__ __align__(1024) uint8_t smem[];  // (operand tiles need the alignment)
  if ((smem_u32(smem) & 1023u) != 0) {
    if (threadIdx.x == 0) fb_report(err, FB_DEVERR_BAD_ARG);
    return;
  }
  constexpr int RING_BYTES = ring_bytes(F32);
  uint8_t* epi_smem = smem + RING_BYTES;
  int* off = reinterpret_cast<int*>(smem + SMEM_BYTES - BAR_BYTES - TABLE_BYTES);
  int* first = off + MAX_E + 8;
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
  const int nw = GATED ? 2 * g.n : g.n, n_ft = (nw + 2 * W_ROWS - 1) / (2 * W_ROWS);
  const int nk = (g.k + BK - 1) / BK, E = g.experts;
  const int parts = F32 ? (nk + PART_BLOCKS - 1) / PART_BLOCKS : 1;
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
    tma_prefetch_desc(&tmA);
    if (!GATHER) tma_prefetch_desc(&tmA8);
    if (!F32) tma_prefetch_desc(&tmO);
  }
  if (threadIdx.x >= 64 && threadIdx.x < 64 + 2 * WIDTHS) cost[threadIdx.x - 64] = 0;
  if (warp == 1) tmem_alloc_cg2(tmem_holder, TMEM_COLS);
  // (copied rows: the offsets and all else but the rows were there before the copy began)
  if (!g.copied) griddep_wait();
  griddep_launch();
  // ---- the groups and the tile width ----
  __syncthreads();
  for (int i = threadIdx.x; i <= E; i += THREADS) {
    const int o = g.offsets[i], p = i ? g.offsets[i - 1] : 0;
    off[i] = o;
    if (o < p || o > g.max_rows || (i == 0 && o != 0)) *bad = 1;
  }
  __syncthreads();
  if (*bad) {  // (every CTA sees the same)
    if (threadIdx.x == 0) fb_report(err, FB_DEVERR_BAD_INDEX);
    for (int i = threadIdx.x; i <= E; i += THREADS) off[i] = 0;
    __syncthreads();
  }
  {
    // (nt tiles of widths that add up to r: 256 nt + r, see below)
    const int c = threadIdx.x % WIDTHS, T = T_STEP * (c + 1);
    unsigned tiles = 0, clocks = 0;
    for (int e = threadIdx.x / WIDTHS; e < E; e += THREADS / WIDTHS) {
      const int r = off[e + 1] - off[e], nt = (r + T - 1) / T;
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
    // choose_width: the width of the least estimated time in SM clocks (the rule and figures
    // of the dense GEMM's tiles: 256 + w clocks of operands, or 313 of issue, per K block; in
    // the fullest cluster each tile but the first takes its mainloop or its epilogue)
    const int T = T_STEP * (lane + 1);
    float est = 3e38f;
    if (lane < WIDTHS && (!F32 || T <= F32_T)) {
      const float n = (float)count[lane] * n_ft, rounds = ceilf(n / n_clusters);
      const float main = count[lane] ? (float)cost[lane] / count[lane] * nk : 0.f;
      const float epi = F32 ? 3300.f + 30.f * T : 2900.f + 12.f * T;
      est = main + (rounds - 1.f) * fmaxf(main, epi) + (F32 ? 28.f : 16.f) * T;
    }
    float best = est;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = fminf(best, __shfl_xor_sync(0xffffffffu, best, o));
    const int Tb = T_STEP * __ffs(__ballot_sync(0xffffffffu, est == best));
    int sum = 0;
    for (int e0 = 0; e0 <= E; e0 += 32) {
      const int e = e0 + lane;
      int n = e < E ? (off[e + 1] - off[e] + Tb - 1) / Tb : 0, s = n;
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
  const int fit = (int)(BAND_BYTES / ((int64_t)2 * W_ROWS * g.k * sizeof(bf16)));
  TileIter ti(off, first, cluster, n_clusters, n_ft, fit < 1 ? 1 : fit < n_ft ? fit : n_ft, E);
  Tile k;

  if (warp == 0) {
    // ---------------- weights (both CTAs) ----------------
    int stage = 0;
    uint32_t phase = 0;
    while (!failed && ti.next(k)) {
      const uint32_t bytes = 2 * (W_BYTES + k.w / 2 * BK * 2);
      for (int kb = 0; kb < nk; ++kb) {
        if (!mbar_wait_warp(&empty[stage], phase ^ 1u, err)) { failed = true; break; }
        if (elect_one()) {
          const uint32_t dst = smem_u32(smem) + stage * stage_bytes;
          const uint32_t fb = mapa_shared(smem_u32(&full[stage]), 0);
          if (rank == 0) mbar_expect_tx(&full[stage], bytes);
          if (GATED)
            tma_load_5d_cg2(dst, &tmW, fb, kb * BK, 0, 0, (2 * k.f + (int)rank) * 4, k.e);
          else
            tma_load_3d_cg2(dst, &tmW, fb, kb * BK, (2 * k.f + (int)rank) * W_ROWS, k.e);
        }
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp >= 10) {
    // ---------------- token rows (both CTAs) ----------------
    int stage = 0;
    uint32_t phase = 0;
    int turn = warp - 10;  // K blocks until this warp's next: they go round the loaders
    griddep_wait();
    while (!failed && ti.next(k)) {
      const int half = k.w / 2, a0 = k.r0 + half * (int)rank, end = k.r0 + k.nv;
      int src[4] = {0, 0, 0, 0};
      const int n4 = half / 4;
      if (GATHER && lane < n4) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int row = a0 + 4 * lane + j;
          src[j] = g.index[row < end ? row : end - 1];
          if (src[j] < 0 || src[j] >= g.a_rows) {
            fb_report(err, FB_DEVERR_BAD_INDEX);
            src[j] = 0;
          }
        }
      }
      for (int kb = 0; kb < nk; ++kb) {
        if (turn-- == 0) {
          turn = LOADERS - 1;
          if (!mbar_wait_warp(&empty[stage], phase ^ 1u, err)) { failed = true; break; }
          const uint32_t dst = smem_u32(smem) + stage * stage_bytes + W_BYTES;
          const uint32_t fb = mapa_shared(smem_u32(&full[stage]), 0);
          if (GATHER) {
#pragma unroll 4
            for (int i = 0; i < n4; ++i) {
              const int r0 = __shfl_sync(0xffffffffu, src[0], i), r1 = __shfl_sync(0xffffffffu, src[1], i);
              const int r2 = __shfl_sync(0xffffffffu, src[2], i), r3 = __shfl_sync(0xffffffffu, src[3], i);
              if (elect_one()) tma_gather4_cg2(dst + i * (4 * BK * 2), &tmA, fb, kb * BK, r0, r1, r2, r3);
            }
          } else if (elect_one()) {
            int i = 0;
            for (; i + 64 <= half; i += 64)
              tma_load_rows_cg2(dst + i * (BK * 2), &tmA, fb, kb * BK, a0 + i);
            for (; i < half; i += 8)
              tma_load_rows_cg2(dst + i * (BK * 2), &tmA8, fb, kb * BK, a0 + i);
          }
        }
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      // ---------------- MMA issuer (even CTA) ----------------
      const uint32_t ring_lo = desc_lo_k(smem_u32(smem));
      const int part_len = (nk + parts - 1) / parts;
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      while (!failed && ti.next(k)) {
        const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(k.w >> 3) << 17) |
                               ((uint32_t)(2 * W_ROWS >> 4) << 24);
        // the tile's K parts, each in the ring's next accumulator
        for (int p = 0, kb = 0; !failed && p < parts; ++p) {
          if (!mbar_wait_warp(&tmem_empty[acc], acc_phase ^ 1u, err)) { failed = true; break; }
          tc_fence_after();
          const uint32_t d_tmem = tmem_base + acc * acc_cols;
          const int start = kb, end = nk - kb < part_len ? nk : kb + part_len;
          for (; kb < end; ++kb) {
            if (!mbar_wait_warp(&full[stage], phase, err)) { failed = true; break; }
            tc_fence_after();
            const uint32_t wlo = ring_lo + (uint32_t)(stage * (stage_bytes >> 4));
            const uint32_t alo = wlo + (W_BYTES >> 4);
            if (elect_one()) {
#pragma unroll
              for (int j = 0; j < BK / 16; ++j)
                tc_mma_cg2_lo(d_tmem, wlo + 2 * j, alo + 2 * j, DESC_HI, idesc,
                              (kb > start || j > 0) ? 1u : 0u);
              tc_commit_mc(&empty[stage], 0x3);
              if (kb + 1 == end) tc_commit_mc(&tmem_full[acc], 0x3);
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
    // CH-token chunk of the tile; FW output features, a lane's own or (gated) a lane pair's
    constexpr int CH = F32 ? 16 : 32, FW = GATED ? 16 : 32;
    const int quarter = warp & 3, we = warp - 2;
    int half = we >> 2;  // a tile's first chunk goes to either half by turns
    const uint32_t te_remote = mapa_shared(smem_u32(&tmem_empty[0]), 0);
    uint8_t* tiles = epi_smem + we * 2 * EPI_TILE;
    int acc = 0, buf = 0;
    uint32_t acc_phase = 0;
    // first output feature of this warp, and the bias of this lane's weight row
    auto first_feature = [&](const Tile& q) {
      const int wrow = (2 * q.f + (int)rank) * W_ROWS + quarter * 32;  // of the interleaved rows
      return GATED ? wrow / 2 : wrow;
    };
    auto bias_of = [&](const Tile& q) {
      const int feature = first_feature(q) + (GATED ? lane & 15 : lane);
      return g.bias && feature < g.n
                 ? __ldg(g.bias + (size_t)q.e * nw + feature + (GATED && lane >= 16 ? g.n : 0))
                 : 0.f;
    };
    Tile after;
    bool more = ti.next(k);
    float bias = more ? bias_of(k) : 0.f;
    for (; !failed && more; k = after) {
      more = ti.next(after);
      const float bias_after = more ? bias_of(after) : 0.f;  // (it may come from memory)
      const int f0 = first_feature(k), feature = f0 + (GATED ? lane & 15 : lane);
      // tokens j and j + 1 of a gated chunk: lanes 0-15 form j's outputs, lanes 16-31 j + 1's
      auto gated = [&](float x0, float x1) {
        const float got = __shfl_xor_sync(0xffffffffu, lane < 16 ? x1 : x0, 16);
        const float gate = lane < 16 ? x0 : got, up = lane < 16 ? got : x1;
        return (g.act == FB_ACT_SWIGLU ? silu_of<F32>(gate) : gelu_f<F32>(gate)) * up;
      };
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16);
      // fp32 results: the parts' sums are added up here as they are done, a part's accumulator
      // going back to the ring at once
      float sum[F32 ? F32_T / 2 : 1];
      bool ok = true;
      for (int p = 0; p < parts; ++p) {
        ok = __all_sync(0xffffffffu, mbar_wait(&tmem_full[acc], acc_phase, err));
        if (!ok) break;
        tc_fence_after();
        if constexpr (F32) {
#pragma unroll
          for (int c = 0; c < F32_T / (2 * CH); ++c) {
            const int t0 = (half + 2 * c) * CH;
            if (t0 >= k.nv || f0 >= g.n) break;
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
      constexpr int UNROLL = F32 ? F32_T / (2 * CH) : 1;  // (sum's indices are constants)
#pragma unroll UNROLL
      for (int c = 0; c < (F32 ? F32_T : MAX_T) / (2 * CH); ++c) {
        const int t0 = (half + 2 * c) * CH;
        if (t0 >= k.nv || f0 >= g.n) break;
        float v[CH];
        if constexpr (F32) {
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
        if constexpr (F32) {
          // straight to memory, 32 or (gated, two tokens at once) 16 features of a token
          const int n = k.nv - t0;
          const size_t first_at = (size_t)(k.r0 + t0 + (GATED ? lane >> 4 : 0)) * g.ldo + feature;
          auto store = [&](auto* at) {
            if (GATED) {
#pragma unroll
              for (int j = 0; j < CH; j += 2, at += 2 * g.ldo) {
                const float y = gated(v[j] + bias, v[j + 1] + bias);
                if (j + (lane >> 4) < n && feature < g.n) put(at, y);
              }
            } else {
#pragma unroll
              for (int j = 0; j < CH; ++j, at += g.ldo) {
                const float x = v[j] + bias;
                if (j < n && feature < g.n) put(at, g.act == FB_ACT_GELU ? gelu_f<true>(x) : x);
              }
            }
          };
          if (g.out_type == FB_F32)
            store(reinterpret_cast<float*>(g.out) + first_at);
          else
            store(reinterpret_cast<bf16*>(g.out) + first_at);
          continue;
        }
        uint8_t* tile = tiles + buf * EPI_TILE;
        buf ^= 1;
        if (elect_one()) bulk_wait_read<1>();  // the store from this tile two chunks ago
        __syncwarp();
        if (GATED) {
#pragma unroll
          for (int j = 0; j < CH; j += 2)
            reinterpret_cast<bf16*>(tile)[j * 16 + lane] =
                __float2bfloat16(gated(v[j] + bias, v[j + 1] + bias));
        } else {
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
        }
        fence_proxy_async_smem();
        __syncwarp();
        const int n = k.nv - t0 < CH ? k.nv - t0 : CH;  // tokens of the chunk that exist
        if (elect_one()) {
#pragma unroll
          for (int b = 0; b < CH; b += 16)
            if (b + 16 <= n) tma_store_2d(&tmO, smem_u32(tile) + b * FW * 2, f0, k.r0 + t0 + b);
          bulk_commit();
        }
        if (n % 16) {  // 16 bytes at a time: n is a multiple of 8 features
          constexpr int PIECES = FW / 8;
          const int b = n / 16 * 16;
          for (int i = lane; i < (n - b) * PIECES; i += 32) {
            const int tok = b + i / PIECES, c = i % PIECES;
            if (f0 + c * 8 < g.n)
              *reinterpret_cast<uint4*>(reinterpret_cast<bf16*>(g.out) +
                                        (size_t)(k.r0 + t0 + tok) * g.ldo + f0 + c * 8) =
                  *reinterpret_cast<const uint4*>(tile + tok * FW * 2 + c * 16);
          }
          __syncwarp();
        }
      }
      if constexpr (!F32) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_relaxed_cluster(te_remote + acc * (uint32_t)sizeof(uint64_t));
        if (++acc == n_accs) { acc = 0; acc_phase ^= 1u; }
      }
      bias = bias_after;
      half ^= 1;
    }
    // own TMA stores complete (one lane issued them all)
    if (elect_one()) bulk_wait<0>();
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

// ---- few rows ---------------------------------------------------------------------------
// A handful of rows read every weight of their experts once: what counts is to have all SMs
// reading at full depth, also where 256-row tiles would be too few (one token's FFN down: 12
// tiles, 28.9 us; 11.3 here). A block takes 16 weight rows of one expert (gated: 8 gate rows and
// their up rows), its warps split k, and the weights go straight from memory into the operand
// registers of mma.sync (m16n8k16: the weights are the M side, eight token rows the N side): the
// tensor instruction is only there to keep the arithmetic out of the way of the loads. Its k
// index is a permuted one, the same for both operands: lane (g, t) of a step of 32 holds k
// 8 t .. 8 t + 7 of weight rows g and g + 8 and of token row g, 16 bytes each.
constexpr int FEW_WARPS = 8, FEW_THREADS = FEW_WARPS * 32, FEW_LONG_K = 2048;

__device__ __forceinline__ void mma_16816(float* c, uint32_t a0, uint32_t a1, uint32_t a2,
                                          uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// NT: eight token rows each; a group of more is taken in several passes. UN: steps of 32 k that a
// warp has on their way, BLOCKS per SM that leave it the registers for that. Inputs from memory,
// one token, us with 4 steps and 5 blocks an SM / 4 and 4 / 6 and 2: 4096 x 1536 gated 12.3 / 12.0
// / 14.0 (six steps a warp in all), 1536 x 4096 14.7 / 10.0 / 7.0, 1536 x 8960 29.4 / 21.1 / 12.1.
template <bool GATED, bool F32, int NT, int UN, int BLOCKS>
__global__ void __launch_bounds__(FEW_THREADS, BLOCKS) expert_few_kernel(const ExpertArgs g, int* err) {
  griddep_wait();
  griddep_launch();
  __shared__ float part[FEW_WARPS][16][8 * NT + 1];
  __shared__ int found[3];  // the block's expert, its rows
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, gr = lane / 4, t = lane % 4;
  const int blocks_n = GATED ? (g.n + 7) / 8 : (g.n + 15) / 16;
  // the blockIdx.x / blocks_n-th group that has rows
  const int want = blockIdx.x / blocks_n;
  if (warp == 0) {
    int seen = 0, at_e = -1, at_r0 = 0, at_r1 = 0;  // the group, in the lane that comes upon it
    bool bad = false;
    for (int e0 = 0; e0 < g.experts; e0 += 32) {
      const int e = e0 + lane;
      const int a = e >= g.experts ? 0 : g.offsets ? g.offsets[e] : 0;
      const int b = e >= g.experts ? 0 : g.offsets ? g.offsets[e + 1] : g.max_rows;
      const unsigned some = __ballot_sync(0xffffffffu, b > a);
      if (b > a && seen + __popc(some & ((1u << lane) - 1)) == want) {
        at_e = e;
        at_r0 = a;
        at_r1 = b;
      }
      seen += __popc(some);
      bad = bad || b < a || a < 0 || b > g.max_rows || (e == 0 && a != 0);
    }
    // one lane writes, once, and no group out of a table that holds anything bad
    const bool refused = __any_sync(0xffffffffu, bad);
    const unsigned has = __ballot_sync(0xffffffffu, at_e >= 0);
    if (lane == (has ? __ffs(has) - 1 : 0)) {
      found[0] = refused ? -1 : at_e;
      found[1] = at_r0;
      found[2] = at_r1;
      if (refused) fb_report(err, FB_DEVERR_BAD_INDEX);
    }
  }
  __syncthreads();
  const int e = found[0], r0 = found[1], r1 = found[2];
  if (e < 0) return;
  const int f0 = (blockIdx.x % blocks_n) * (GATED ? 8 : 16);
  const size_t nw = GATED ? 2 * (size_t)g.n : g.n;
  // this lane's two weight rows (past the last one: the last one again, not stored)
  const int fa = min(f0 + gr, g.n - 1), fb = GATED ? g.n + fa : min(f0 + 8 + gr, g.n - 1);
  const bf16* wa = g.W + ((size_t)e * nw + fa) * g.k + 8 * t;
  const bf16* wb = g.W + ((size_t)e * nw + fb) * g.k + 8 * t;
  const int steps = (g.k + 31) / 32;
  const int s0 = steps * warp / FEW_WARPS, s1 = steps * (warp + 1) / FEW_WARPS;
  for (int p0 = r0; p0 < r1; p0 += 8 * NT) {
    const bf16* x[NT];
    bool have[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int row = p0 + 8 * i + gr;
      have[i] = row < r1;
      int src = have[i] ? row : r0;
      if (g.index) src = g.index[src];
      if (src < 0 || src >= g.a_rows) {
        fb_report(err, FB_DEVERR_BAD_INDEX);
        src = 0;
      }
      x[i] = g.A + (size_t)src * g.lda + 8 * t;
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
      if constexpr (F32) {  // (the instruction's own sums cut a bit off per step)
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            sum[i][j] += c[i][j];
            c[i][j] = 0.f;
          }
      }
    }
    if constexpr (F32) {
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) c[i][j] = sum[i][j];
    }
    // c[i][0..1]: weight row gr, token rows 2 t and 2 t + 1 of part i; c[i][2..3]: row gr + 8
    __syncthreads();  // (the last pass's sums are read)
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        part[warp][gr][8 * i + 2 * t + j] = c[i][j];
        part[warp][gr + 8][8 * i + 2 * t + j] = c[i][2 + j];
      }
    __syncthreads();
    constexpr int F = GATED ? 8 : 16;
    for (int o = threadIdx.x; o < F * 8 * NT; o += FEW_THREADS) {
      const int f = o % F, row = o / F;
      if (f0 + f >= g.n || p0 + row >= r1) continue;
      float v = 0.f, up = 0.f;
#pragma unroll
      for (int w = 0; w < FEW_WARPS; ++w) {
        v += part[w][f][row];
        if (GATED) up += part[w][f + 8][row];
      }
      if (g.bias) {
        v += g.bias[e * nw + f0 + f];
        if (GATED) up += g.bias[e * nw + g.n + f0 + f];
      }
      if (GATED)
        v = (g.act == FB_ACT_SWIGLU ? silu_of<F32>(v) : gelu_f<F32>(v)) * up;
      else if (g.act == FB_ACT_GELU)
        v = gelu_f<F32>(v);
      const size_t at = (size_t)(p0 + row) * g.ldo + f0 + f;
      if (F32 && g.out_type == FB_F32)
        put(reinterpret_cast<float*>(g.out) + at, v);
      else
        put(reinterpret_cast<bf16*>(g.out) + at, v);
    }
  }
}

// Rows in expert order: dst[r] = A[index[r]], one warp per row.
__global__ void __launch_bounds__(256) gather_rows_kernel(const ExpertArgs g, bf16* dst, int* err) {
  griddep_wait();
  griddep_launch();
  const int lane = threadIdx.x % 32;
  const int total = min(g.offsets[g.experts], g.max_rows);  // (the product checks the offsets)
  for (int r = blockIdx.x * 8 + threadIdx.x / 32; r < total; r += gridDim.x * 8) {
    int s = g.index[r];
    if (s < 0 || s >= g.a_rows) {
      if (lane == 0) fb_report(err, FB_DEVERR_BAD_INDEX);
      s = 0;
    }
    const uint4* from = reinterpret_cast<const uint4*>(g.A + (size_t)s * g.lda);
    uint4* to = reinterpret_cast<uint4*>(dst + (size_t)r * g.k);
    const int n = g.k / 8;
#pragma unroll 8
    for (int i = lane; i < n; i += 32) to[i] = __ldg(from + i);
  }
}

// ---- host -------------------------------------------------------------------------------
PFN_cuTensorMapEncodeTiled_v12000 encoder() {
  static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    cudaDriverEntryPointQueryResult q;
    void* p = nullptr;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                         &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    cudaGetLastError();
    return static_cast<PFN_cuTensorMapEncodeTiled_v12000>(nullptr);
  }();
  return fn;
}

template <int R>
bool make_map(CUtensorMap* map, const void* ptr, const cuuint64_t (&dims)[R],
              const cuuint64_t (&stride_elems)[R - 1], const cuuint32_t (&box)[R], bool swizzle) {
  auto enc = encoder();
  if (!enc) return false;
  cuuint64_t strides[R - 1];
  cuuint32_t estr[R];
  for (int i = 0; i < R; ++i) {
    estr[i] = 1;
    if (i) strides[i - 1] = stride_elems[i - 1] * 2;
  }
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, R, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
             swizzle ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Clusters that the current device can hold at once, asked once per device.
template <bool GATED, bool F32, bool GATHER>
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
    cfg.blockDim = dim3(Warps<F32, GATHER>::THREADS, 1, 1);
    cfg.dynamicSmemBytes = SMEM_BYTES;
    if (cudaOccupancyMaxActiveClusters(&n, expert_tc_kernel<GATED, F32, GATHER>, &cfg) == cudaSuccess &&
        n > 0) {
      if (dev < DEVICES) known[dev].store(n, std::memory_order_relaxed);
      return n;
    }
  }
  cudaGetLastError();
  return num_sms / 2;
}

template <bool GATED, bool F32>
cudaError_t launch_few(const ExpertArgs& g, int* err, cudaStream_t st) {
  const int blocks_n = GATED ? (g.n + 7) / 8 : (g.n + 15) / 16;
  const long long groups = g.experts < g.max_rows ? g.experts : g.max_rows;  // with rows, at most
  auto kern = g.max_rows > 8        ? expert_few_kernel<GATED, F32, 2, 4, 2>
              : g.k > FEW_LONG_K ? expert_few_kernel<GATED, F32, 1, 6, 2>
                                    : expert_few_kernel<GATED, F32, 1, 4, GATED ? 4 : 3>;
  return launch_k(kern, dim3(groups * blocks_n), dim3(FEW_THREADS), 0, st, g, err);
}

template <bool GATED, bool F32, bool GATHER>
cudaError_t launch(const ExpertArgs& g, int* err, int num_sms, cudaStream_t st) {
  auto kern = expert_tc_kernel<GATED, F32, GATHER>;
  cudaError_t e =
      cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES);
  if (e != cudaSuccess) return e;
  typedef cuuint64_t u64;
  const u64 K = g.k, N = g.n, E = g.experts;
  CUtensorMap mw, ma, ma8{}, mo{};  // ma8: unused with an index, mo: with fp32 results
  const bool w_ok =
      GATED ? make_map<5>(&mw, g.W, {K, 16, 2, N / 16, E}, {K, N * K, 16 * K, 2 * N * K},
                          {BK, 16, 2, W_ROWS / 32, 1}, true)
            : make_map<3>(&mw, g.W, {K, N, E}, {K, N * K}, {BK, W_ROWS, 1}, true);
  const u64 rows = g.a_rows, lda = g.lda, orows = g.max_rows, ldo = g.ldo;
  if (!w_ok ||
      !make_map<2>(&ma, g.A, {K, rows}, {lda}, {BK, GATHER ? 1u : 64u}, true) ||
      (!GATHER && !make_map<2>(&ma8, g.A, {K, rows}, {lda}, {BK, 8}, true)) ||
      (!F32 && !make_map<2>(&mo, g.out, {N, orows}, {ldo}, {GATED ? 16u : 32u, 16}, false)))
    return cudaErrorInvalidValue;
  const int occ = resident_clusters<GATED, F32, GATHER>(num_sms);
  const int mc = occ < num_sms / 2 ? occ : num_sms / 2;
  // no more clusters than there can be tiles: 16 rows at least each but a group's last
  const int n_ft = ((GATED ? 2 * g.n : g.n) + 2 * W_ROWS - 1) / (2 * W_ROWS);
  const long long groups = g.experts < g.max_rows ? g.experts : g.max_rows;
  const long long tiles = (g.max_rows / T_STEP + groups) * n_ft;
  const int clusters = tiles < mc ? (int)tiles : mc;
  return launch_k(kern, dim3(2 * clusters), dim3(Warps<F32, GATHER>::THREADS), SMEM_BYTES, st, mw, ma, ma8, mo, g, err);
}

template <bool GATED, bool F32>
cudaError_t choose(const ExpertArgs& g, int* err, int num_sms, cudaStream_t st) {
  const int n_ft = ((GATED ? 2 * g.n : g.n) + 2 * W_ROWS - 1) / (2 * W_ROWS);
  const long long groups = g.experts < g.max_rows ? g.experts : g.max_rows;  // with rows, at most
  // Few rows whose tiles would leave SM pairs idle go to the streaming kernel; with tiles for all
  // pairs the TMA ring keeps memory busier than it does (us, streamed / tiles; 8 experts, rows x n
  // x k, gated): 2 x 4096 x 1536 gated 8.2 / 11.1, 2 x 1536 x 8960 11.3 / 28.9, 4 x 8960 x 1536
  // 13.5 / 15.4, 8 x 8960 x 1536 35.1 / 30.9, 8 x 1536 x 4096 11.4 / 16.4, 16 x 1536 x 4096
  // 19.3 / 21.2, 16 x 8960 x 1536 60.6 / 38.6; 2 experts, 32 x 2048 x 2048 5.6 / 11.2, 64 11.9 / 11.5.
  // (Without offsets it is always these.)
  if (!g.offsets ||
      (g.max_rows <= 32 && groups * n_ft <= num_sms / 2 * (g.max_rows <= 8 ? 2 : 1)))
    return launch_few<GATED, F32>(g, err, st);
  return g.index ? launch<GATED, F32, true>(g, err, num_sms, st)
                 : launch<GATED, F32, false>(g, err, num_sms, st);
}

}  // namespace

cudaError_t expert_gemm_set_wait_limit(unsigned long long ns) { return fb_set_wait_limit_tu(ns); }

// Large groups have their rows copied to expert order first; small ones are gathered by the
// product itself. A TMA gather costs its issuing warp 68 clocks per four rows whatever the form
// of the loop, which four loaders hide up to tiles of about 192 rows (two, with fp32 results, 96);
// the copy is one more launch, 2 to 3 us that the product's start does not hide, and 4 bytes per
// element. Measured (us, gathered / copied): 8 experts, 8960 x 1536, 64 rows a group 41.7 / 43.7,
// 128 45.6 / 46.5, 195 52.6 / 49.8, 256 68 / 61, 390 87 / 76, 6240 1084 / 899; 64 experts,
// 1024 x 1536 gated, 130 rows 73.0 / 79.9, 200 87 / 90, 300 129 / 124; fp32, 8 experts,
// 4096 x 1536, 64 rows 25.8 / 26.6, 96 28.6 / 30.2, 130 38.0 / 36.1. Weight rows that are few read
// each token few times and do not pay for the copy: 8 experts, 512 x 1536, 390 rows a group
// 11.8 / 15.2, 4000 47.8 / 74.6; 1536 x 8960 87 / 94, 654 / 726 (1536 x 1536 21.4 / 21.1,
// 124 / 129); 2048 x 1536 25.5 / 22.8, 170 / 162; fp32, 512 x 1536, 390 rows 15.5 / 16.0,
// 768 x 1536 23.8 / 21.2. (Six or eight loaders: 965 at 6240 rows, but every further warp slows
// all others; copies by cp.async into the ring 2278: the issuer then needs a proxy fence per K
// block, which waits for the SM's copies in flight.)
size_t expert_gemm_ws_bytes(const ExpertArgs& g) {
  const bool f32 = in_parts(g);
  const long long most = f32 ? 96 : 192;  // rows a group, on average
  const int nw = g.act >= FB_ACT_SWIGLU ? 2 * g.n : g.n;
  const bool copy = g.index && nw > (f32 ? 512 : 1536) && g.max_rows > most * g.experts;
  return copy ? (size_t)g.max_rows * g.k * sizeof(bf16) : 0;
}

cudaError_t expert_copy_rows(ExpertArgs* g, bf16* ws, int* err, int num_sms, cudaStream_t st) {
  // Four blocks an SM. The product's CTA (384 threads of 120 registers) fits beside one block of the
  // copy (256 of 40), not beside two: it starts on an SM as the copy drains there, and what overlaps
  // is the copy's tail. us of both, with 1 / 2 / 3 / 4 / 6 / 8 blocks: 390 rows a group over 8
  // experts, 8960 x 1536 75.0 / 72.7 / 70.8 / 71.6 / 71.8 / 71.8; 6240 896 / 886 / 834 / 840 / 863
  // / 810 (the clock varies by 3 %); 2000, 4096 x 1536 159 / 147 / 142 / 140 / 138 / 138.
  const int most = 4 * num_sms, need = (g->max_rows + 7) / 8;
  const cudaError_t e = launch_k(gather_rows_kernel, dim3(need < most ? need : most), dim3(256), 0,
                                 st, *g, ws, err);
  g->A = ws;
  g->lda = g->k;
  g->a_rows = g->max_rows;
  g->index = nullptr;
  g->copied = true;
  return e;
}

cudaError_t expert_gemm(const ExpertArgs& g, int* err, int num_sms, cudaStream_t st) {
  if (g.max_rows == 0) return cudaSuccess;
  if (num_sms < 2) return cudaErrorInvalidValue;
  const bool f32 = in_parts(g);
  if (g.act >= FB_ACT_SWIGLU)
    return f32 ? choose<true, true>(g, err, num_sms, st) : choose<true, false>(g, err, num_sms, st);
  return f32 ? choose<false, true>(g, err, num_sms, st) : choose<false, false>(g, err, num_sms, st);
}
