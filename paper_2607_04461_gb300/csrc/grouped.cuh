// What the products over groups of rows share (experts, adapters): tiles cut to each group's rows,
// TMA forms of an SM pair, activations, tensor maps.
#pragma once
#include <cudaTypedefs.h>

#include "common.cuh"

namespace {

constexpr int BK = 64;                  // 64 bf16 = 128 bytes: one swizzle row
constexpr int W_ROWS = 128;             // weight rows of a CTA
constexpr int W_BYTES = W_ROWS * BK * 2;
constexpr int MAX_T = 256, T_STEP = 16, WIDTHS = MAX_T / T_STEP;

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

// ---- mma.sync ---------------------------------------------------------------------------
__device__ __forceinline__ void mma_16816(float* c, uint32_t a0, uint32_t a1, uint32_t a2,
                                          uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// ---- tensor maps ------------------------------------------------------------------------
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

}  // namespace
