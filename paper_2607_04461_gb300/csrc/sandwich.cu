// The norms before and after a block, its gate and the scaled residual in one pass:
//   y  = sum_j weight[r][j] e[slot[r][j]]      (or row r of the block's output)
//   h' = resid_scale h + gate (Post(y) post_w + post_b)
//   a  = Pre(h') (mul_base + mul) + add
// with Post and Pre either RMSNorm, LayerNorm or nothing. The residual is not known before
// Post's statistics, and a not before those of h', so that the chain written as separate
// passes reads and writes h twice and y once more. Here a row lives in registers: h and y are
// read once, h' and a written once, which is all the traffic there is. Everything is held in
// fp32 and rounded once, as h' and a are stored; a is formed from h' before that rounding.
//
// THREADS threads hold a row in pieces of 4 values, VPT pieces each, at 16 bytes of fp32 and 8 of
// bf16 apart (a piece of 8 took twice the L1 cycles for every fp32 row, and L1 is what the
// parameter rows and the data go through: 199 us at 49920 rows of 1536, 141 with pieces of 4).
// VEC: rows begin on a boundary of 4 values; else one value at a time, neighbours on
// neighbouring lanes. Few rows, which are bound by the latency of one row's chain, get more
// threads and load the row's parameters (EARLY) together with the row. 3.9 TB/s of 6.8 at 1560
// rows of 1536 (y in bf16, h in fp32), 6.5 at 49920, one row 2.7 us. Rows of no alignment are
// bound by their instructions, 4 accesses for every one: 49920 rows of 1235 184 us, 4.0 TB/s
// (244 with a comparison per value and threads for 1536).
#include "kernels.h"

namespace {

// A piece of 4 values is two packed pairs: one instruction per pair and operation.
typedef uint64_t f2;
__device__ __forceinline__ f2 f2_both(float x) { return f2_join(x, x); }
__device__ __forceinline__ float f2_total(f2 v) {
  float a, b;
  f2_split(v, a, b);
  return a + b;
}

template <int THREADS, bool VEC>
struct Row {
  // value j of piece i of thread tid
  static __device__ __forceinline__ int col(int i, int j, int tid) {
    return VEC ? (i * THREADS + tid) * 4 + j : (i * 4 + j) * THREADS + tid;
  }
  // whether piece i holds anything (VEC: 4 values, else at least one)
  static __device__ __forceinline__ bool any(int i, int D, int tid) { return col(i, 0, tid) < D; }
  // A piece's bits: 4 words of fp32 (or scalar bf16), 2 words of bf16. Not converted, so that
  // nothing waits for the loads yet. Values past D are zeros.
  static __device__ __forceinline__ void load(const void* base, int type, size_t at, int i, int D,
                                              int tid, uint32_t* w) {
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = 0;
    if (VEC) {
      if (!any(i, D, tid)) return;
      const size_t o = at + col(i, 0, tid);
      if (type == FB_F32) {
        const uint4 a = *reinterpret_cast<const uint4*>(reinterpret_cast<const float*>(base) + o);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
      } else {
        const uint2 a = *reinterpret_cast<const uint2*>(reinterpret_cast<const bf16*>(base) + o);
        w[0] = a.x; w[1] = a.y;
      }
    } else if (type == FB_F32) {
      load_each(reinterpret_cast<const uint32_t*>(base) + at, i, D, tid, w);
    } else {
      load_each(reinterpret_cast<const uint16_t*>(base) + at, i, D, tid, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] <<= 16;
    }
  }
  // (a piece that lies wholly within the row needs one comparison)
  template <typename T>
  static __device__ __forceinline__ void load_each(const T* p, int i, int D, int tid, uint32_t* w) {
    p += col(i, 0, tid);
    if (col(i, 3, tid) < D) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = p[j * THREADS];
    } else {
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (col(i, j, tid) < D) w[j] = p[j * THREADS];
    }
  }
  static __device__ __forceinline__ void values(const uint32_t* w, int type, f2* v) {
    if (type == FB_F32 || !VEC) {
      v[0] = f2_join(__uint_as_float(w[0]), __uint_as_float(w[1]));
      v[1] = f2_join(__uint_as_float(w[2]), __uint_as_float(w[3]));
    } else {
      v[0] = f2_join(__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u));
      v[1] = f2_join(__uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xffff0000u));
    }
  }
  static __device__ __forceinline__ void store(void* base, int type, size_t at, int i, int D, int tid,
                                               const f2* x) {
    float v[4];
    f2_split(x[0], v[0], v[1]);
    f2_split(x[1], v[2], v[3]);
    if (VEC) {
      const size_t o = at + col(i, 0, tid);
      if (type == FB_F32) {
        *reinterpret_cast<float4*>(reinterpret_cast<float*>(base) + o) =
            make_float4(v[0], v[1], v[2], v[3]);
      } else {
        uint2 u;
        u.x = pack_bf16x2(v[0], v[1]);
        u.y = pack_bf16x2(v[2], v[3]);
        *reinterpret_cast<uint2*>(reinterpret_cast<bf16*>(base) + o) = u;
      }
    } else if (type == FB_F32) {
      float* p = reinterpret_cast<float*>(base) + at + col(i, 0, tid);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (col(i, 3, tid) < D || col(i, j, tid) < D) p[j * THREADS] = v[j];
    } else {
      bf16* p = reinterpret_cast<bf16*>(base) + at + col(i, 0, tid);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (col(i, 3, tid) < D || col(i, j, tid) < D) p[j * THREADS] = __float2bfloat16(v[j]);
    }
  }
  // A parameter row's piece, or `none` where there is no such row. Read-only loads: they need
  // not wait for stores. (As volatile statements they stay behind griddep_wait, which an
  // intrinsic for unchanging data would not have to.)
  static __device__ __forceinline__ void param(const float* p, float none, int i, int D, int tid,
                                               f2* x) {
    float v[4] = {none, none, none, none};
    if (p) {
      if constexpr (VEC) {
        asm volatile("ld.global.nc.v4.f32 {%0, %1, %2, %3}, [%4];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "l"(p + col(i, 0, tid)));
      } else {
        p += col(i, 0, tid);
        if (col(i, 3, tid) < D) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            asm volatile("ld.global.nc.f32 %0, [%1];" : "=f"(v[j]) : "l"(p + j * THREADS));
        } else {
#pragma unroll
          for (int j = 0; j < 3; ++j)
            if (col(i, j, tid) < D)
              asm volatile("ld.global.nc.f32 %0, [%1];" : "=f"(v[j]) : "l"(p + j * THREADS));
        }
      }
    }
    x[0] = f2_join(v[0], v[1]);
    x[1] = f2_join(v[2], v[3]);
  }
  // zeros in the place of values past D (in a piece that holds some; VEC: there are none)
  static __device__ __forceinline__ void clear_tail(f2* v, int i, int D, int tid) {
    if constexpr (!VEC) {
      if (col(i, 3, tid) < D) return;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float a, b;
        f2_split(v[j], a, b);
        v[j] = f2_join(col(i, 2 * j, tid) < D ? a : 0.f, col(i, 2 * j + 1, tid) < D ? b : 0.f);
      }
    }
  }
};

// Sums over the THREADS threads of a row. Two buffers by turns, one barrier per sum: a buffer is
// written again only behind the next sum's barrier, which no thread passes before it has read it.
template <int THREADS>
struct RowSum {
  float (*red)[THREADS / 32];
  int buf = 0;
  __device__ __forceinline__ float operator()(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (THREADS > 32) {
      if (threadIdx.x % 32 == 0) red[buf][threadIdx.x / 32] = v;
      __syncthreads();
      v = 0.f;
#pragma unroll
      for (int w = 0; w < THREADS / 32; ++w) v += red[buf][w];
      buf ^= 1;
    }
    return v;
  }
};

// mean (LayerNorm; else 0) and 1 / sqrt(variance + eps) of a row whose values past D are 0
template <class R, int VPT, class Sum>
__device__ __forceinline__ void row_stats(const f2 (*v)[2], int D, int tid, int kind, float eps,
                                          Sum& sum, float& mean, float& rstd) {
  mean = 0.f;
  rstd = 1.f;
  if (kind == FB_NORM_NONE) return;
  f2 q = 0;
  if (kind == FB_NORM_LAYER) {
    f2 t = 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) t = f2_add(t, v[i][j]);
    mean = sum(f2_total(t)) / D;
    const f2 m = f2_both(-mean);
#pragma unroll
    for (int i = 0; i < VPT; ++i)
      if (R::any(i, D, tid)) {
        f2 d[2] = {f2_add(v[i][0], m), f2_add(v[i][1], m)};
        R::clear_tail(d, i, D, tid);
        q = f2_fma(d[0], d[0], q);
        q = f2_fma(d[1], d[1], q);
      }
  } else {
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) q = f2_fma(v[i][j], v[i][j], q);
  }
  rstd = rsqrtf(sum(f2_total(q)) / D + eps);
}

constexpr unsigned SEGMENTS = 8;  // see run()

// row / group_rows (0 with group_rows 0); div: 2^64 / group_rows rounded up, exact for 32 bits
__device__ __forceinline__ unsigned group_of(unsigned row, int group_rows, unsigned long long div) {
  return group_rows == 0 ? 0 : group_rows == 1 ? row : (unsigned)__umul64hi(row, div);
}

template <int THREADS, int VPT, int ROWS, bool EARLY, bool VEC>
__global__ void __launch_bounds__(THREADS * ROWS)
    sandwich_kernel(const __grid_constant__ SandwichArgs s, unsigned segment, unsigned long long div,
                    int* err) {
  static_assert(ROWS == 1 || THREADS == 32, "several rows per block need one warp per row");
  using R = Row<THREADS, VEC>;
  constexpr int NE = EARLY ? VPT : 1;
  griddep_wait();
  griddep_launch();
  __shared__ float red[2][THREADS / 32];
  RowSum<THREADS> sum{red};
  const int D = s.dim, tid = threadIdx.x % THREADS, lane = threadIdx.x % 32;
  unsigned row = blockIdx.x * ROWS + threadIdx.x / THREADS;
  if (segment) {
    // rows of several segments by turns, each segment begun at another place: see run()
    const unsigned k = row % SEGMENTS, i = row / SEGMENTS + k * (segment / SEGMENTS);
    row = k * segment + (i < segment ? i : i - segment);
  }
  if (row >= (unsigned)s.rows) return;
  // this row's slots and weights, one per lane
  int slot = -1;
  float wt = 0.f;
  if (s.y && lane < s.parts) {
    slot = s.slot[(size_t)row * s.parts + lane];
    wt = s.weight[(size_t)row * s.parts + lane];
  }
  uint32_t hw[VPT][4], yw[VPT][4];
#pragma unroll
  for (int i = 0; i < VPT; ++i) R::load(s.h, s.h_type, row * s.ldh, i, D, tid, hw[i]);
  if (s.y && s.parts == 0) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) R::load(s.y, s.y_type, row * s.ldy, i, D, tid, yw[i]);
  }
  // The group's parameter rows. (Held as they are: formed again at every use, as the compiler
  // had it, they took the kernel from 146 us to 265 at 49920 rows of 1536 in groups of 1560.)
  const int64_t mod = (int64_t)group_of(row, s.group_rows, div) * s.ldm;
  const float* gate = s.gate ? s.gate + mod : nullptr;
  const float* mul = s.mul ? s.mul + mod : nullptr;
  const float* add = s.add ? s.add + mod : nullptr;
  asm volatile("" : "+l"(gate), "+l"(mul), "+l"(add));
  f2 pw[NE][2], pb[NE][2], gt[NE][2], mu[NE][2], ad[NE][2];
  auto before = [&](int i) {
    const int e = EARLY ? i : 0;
    R::param(s.post_w, 1.f, i, D, tid, pw[e]);
    R::param(s.post_b, 0.f, i, D, tid, pb[e]);
    R::param(gate, 1.f, i, D, tid, gt[e]);
  };
  auto behind = [&](int i) {
    const int e = EARLY ? i : 0;
    R::param(mul, 0.f, i, D, tid, mu[e]);
    R::param(add, 0.f, i, D, tid, ad[e]);
  };
  if (EARLY) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (!R::any(i, D, tid)) continue;
      if (s.y) before(i);
      if (s.a) behind(i);
    }
  }
  f2 h[VPT][2], y[VPT][2];
  float mean, rstd;
  if (s.y) {
    if (s.parts == 0) {
#pragma unroll
      for (int i = 0; i < VPT; ++i) R::values(yw[i], s.y_type, y[i]);
    } else {
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) y[i][j] = 0;
      if (slot >= s.y_rows) {
        fb_report(err, FB_DEVERR_BAD_INDEX);
        slot = -1;
      }
      // (a row's slots do not depend on the thread, so neither does the branch)
#pragma unroll 2
      for (int q = 0; q < s.parts; ++q) {
        const int sl = __shfl_sync(0xffffffffu, slot, q);
        const float w = __shfl_sync(0xffffffffu, wt, q);
        if (sl < 0) continue;
#pragma unroll
        for (int i = 0; i < VPT; ++i) R::load(s.y, s.y_type, sl * s.ldy, i, D, tid, yw[i]);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
          f2 v[2];
          R::values(yw[i], s.y_type, v);
#pragma unroll
          for (int j = 0; j < 2; ++j) y[i][j] = f2_fma(f2_both(w), v[j], y[i][j]);
        }
      }
    }
    row_stats<R, VPT>(y, D, tid, s.post, s.post_eps, sum, mean, rstd);
  }
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int e = EARLY ? i : 0;
    R::values(hw[i], s.h_type, h[i]);  // (zeros past D)
    if (!R::any(i, D, tid)) continue;
    if (s.y) {
      if (!EARLY) before(i);
      const f2 m = f2_both(-mean), r = f2_both(rstd), c = f2_both(s.resid_scale);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const f2 u = f2_fma(f2_mul(f2_add(y[i][j], m), r), pw[e][j], pb[e][j]);
        h[i][j] = f2_fma(c, h[i][j], f2_mul(gt[e][j], u));
      }
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j) h[i][j] = f2_mul(f2_both(s.resid_scale), h[i][j]);
    }
    if (s.h_out) R::store(s.h_out, s.h_type, row * s.ldho, i, D, tid, h[i]);
    R::clear_tail(h[i], i, D, tid);
  }
  if (!s.a) return;
  row_stats<R, VPT>(h, D, tid, s.pre, s.pre_eps, sum, mean, rstd);
  const f2 m = f2_both(-mean), r = f2_both(rstd), b = f2_both(s.mul_base);
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int e = EARLY ? i : 0;
    if (!R::any(i, D, tid)) continue;
    if (!EARLY) behind(i);
    f2 v[2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
      v[j] = f2_fma(f2_mul(f2_add(h[i][j], m), r), f2_add(b, mu[e][j]), ad[e][j]);
    R::store(s.a, s.a_type, row * s.lda, i, D, tid, v);
  }
}

// Many rows with parameters per group are taken from eight segments by turns, so that no more
// than an eighth of the running blocks change to the next group at a time: all at once they ask
// L2 for the same lines, about 3.6 us a group. 49920 rows of 1536, us in order / in segments:
// groups of 1560 269 / 166, 4096 184 / 158, 400 249 / 184, 100 244 / 218; one group 141.
template <int THREADS, int VPT, bool VEC, bool EARLY = false, int ROWS = 1>
cudaError_t run(const SandwichArgs& s, bool many, int* err, cudaStream_t st) {
  const bool spread = many && s.group_rows > 0 && s.group_rows < s.rows;
  const unsigned segment = spread ? (s.rows + SEGMENTS - 1) / SEGMENTS : 0;
  const unsigned rows = spread ? segment * SEGMENTS : s.rows;
  const unsigned long long div = s.group_rows > 1 ? ~0ull / s.group_rows + 1 : 0;
  return launch_k(sandwich_kernel<THREADS, VPT, ROWS, EARLY, VEC>, dim3((rows + ROWS - 1) / ROWS),
                  dim3(THREADS * ROWS), 0, st, s, segment, div, err);
}

// The forms by row width: few rows (EARLY), a middle number or rows of no alignment (two pieces a
// thread), many rows (four). us of the few / middle / many forms at 1536: 1 row 2.7 / 2.9 / 3.4,
// 608 3.6 / 4.1 / 4.3, 1560 10.0 / 7.5 / 9.3, 3040 - / 11.4 / 10.6, 49920 - / 167 / 141.
template <bool VEC>
cudaError_t few(const SandwichArgs& s, int* err, cudaStream_t st) {
  const int D = s.dim;
  if (D <= 256) return run<64, 1, VEC, true>(s, false, err, st);
  if (D <= 512) return run<128, 1, VEC, true>(s, false, err, st);
  if (D <= 1024) return run<256, 1, VEC, true>(s, false, err, st);
  if (D <= 1536) return run<192, 2, VEC, true>(s, false, err, st);
  if (D <= 2048) return run<256, 2, VEC, true>(s, false, err, st);
  if (D <= 4096) return run<512, 2, VEC, true>(s, false, err, st);
  return run<640, 2, VEC, true>(s, false, err, st);
}
template <bool VEC>
cudaError_t middle(const SandwichArgs& s, bool many, int* err, cudaStream_t st) {
  const int D = s.dim;
  if (D <= 256) return run<32, 2, VEC, false, 4>(s, many, err, st);
  if (D <= 512) return run<64, 2, VEC>(s, many, err, st);
  if (D <= 768) return run<96, 2, VEC>(s, many, err, st);
  if (D <= 1024) return run<128, 2, VEC>(s, many, err, st);
  if (D <= 1280) return run<160, 2, VEC>(s, many, err, st);
  if (D <= 1536) return run<192, 2, VEC>(s, many, err, st);
  if (D <= 2048) return run<256, 2, VEC>(s, many, err, st);
  if (D <= 2816) return run<352, 2, VEC>(s, many, err, st);
  if (D <= 4096) return run<512, 2, VEC>(s, many, err, st);
  if (D <= 5120) return run<320, 4, VEC>(s, many, err, st);
  if (D <= 8192) return run<512, 4, VEC>(s, many, err, st);
  return run<512, 8, VEC>(s, many, err, st);
}
cudaError_t many(const SandwichArgs& s, int* err, cudaStream_t st) {
  const int D = s.dim;
  if (D <= 256) return run<32, 2, true, false, 4>(s, true, err, st);
  if (D <= 512) return run<32, 4, true, false, 4>(s, true, err, st);
  if (D <= 1024) return run<64, 4, true>(s, true, err, st);
  if (D <= 1536) return run<96, 4, true>(s, true, err, st);
  if (D <= 2048) return run<128, 4, true>(s, true, err, st);
  if (D <= 4096) return run<256, 4, true>(s, true, err, st);
  if (D <= 5120) return run<320, 4, true>(s, true, err, st);
  if (D <= 8192) return run<512, 4, true>(s, true, err, st);
  return run<512, 8, true>(s, true, err, st);
}

// whether every row of the matrix (none: null) starts on a boundary of 4 values
bool aligned(const void* p, int type, int64_t ld) {
  return !p || (reinterpret_cast<uintptr_t>(p) % (type == FB_F32 ? 16 : 8) == 0 && ld % 4 == 0);
}

}  // namespace

cudaError_t sandwich_norm(const SandwichArgs& s, int* err, int num_sms, cudaStream_t st) {
  if (s.rows == 0) return cudaSuccess;
  const int D = s.dim;
  const int64_t ldm = s.group_rows ? s.ldm : 0;
  const bool vec = D % 4 == 0 && aligned(s.h, s.h_type, s.ldh) && aligned(s.y, s.y_type, s.ldy) &&
                   aligned(s.h_out, s.h_type, s.ldho) && aligned(s.a, s.a_type, s.lda) &&
                   aligned(s.post_w, FB_F32, 0) && aligned(s.post_b, FB_F32, 0) &&
                   aligned(s.gate, FB_F32, ldm) && aligned(s.mul, FB_F32, ldm) &&
                   aligned(s.add, FB_F32, ldm);
  if (s.rows <= 4 * num_sms && D <= 5120)
    return vec ? few<true>(s, err, st) : few<false>(s, err, st);
  const bool is_many = s.rows > 16 * num_sms;
  if (!vec) return middle<false>(s, is_many, err, st);
  return is_many ? many(s, err, st) : middle<true>(s, false, err, st);
}
