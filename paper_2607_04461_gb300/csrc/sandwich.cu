// The norms before and after a block, its gate and the scaled residual in one pass:
//   y  = sum_j weight[r][j] e[slot[r][j]]      (or row r of the block's output)
//   h' = resid_scale h + gate (Post(y) post_w + post_b)
//   a  = Pre(h') (mul_base + mul) + add
// with Post and Pre either RMSNorm, LayerNorm or nothing. The residual is not known before
// Post's statistics, and a not before those of h', so that the chain written as separate
// passes reads and writes h twice and y once more. Everything is held in fp32 and rounded
// once, as h' and a are stored; a is formed from h' before that rounding.
//
// One block per row, the row in shared memory.
#include "kernels.h"

namespace {

constexpr int THREADS = 256;

__device__ __forceinline__ float load_any(const void* p, int type, size_t i) {
  return type == FB_F32 ? reinterpret_cast<const float*>(p)[i]
                        : __bfloat162float(reinterpret_cast<const bf16*>(p)[i]);
}
__device__ __forceinline__ void store_any(void* p, int type, size_t i, float v) {
  if (type == FB_F32)
    reinterpret_cast<float*>(p)[i] = v;
  else
    reinterpret_cast<bf16*>(p)[i] = __float2bfloat16(v);
}

__device__ __forceinline__ float row_sum(float v, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
  __syncthreads();
  v = 0.f;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) v += red[w];
  return v;
}

// mean (LayerNorm; else 0) and 1 / sqrt(variance + eps) of the row x
__device__ __forceinline__ void row_stats(const float* x, int D, int kind, float eps, float* red,
                                          float& mean, float& rstd) {
  mean = 0.f;
  rstd = 1.f;
  if (kind == FB_NORM_NONE) return;
  if (kind == FB_NORM_LAYER) {
    float s = 0.f;
    for (int i = threadIdx.x; i < D; i += THREADS) s += x[i];
    mean = row_sum(s, red) / D;
  }
  float q = 0.f;
  for (int i = threadIdx.x; i < D; i += THREADS) q += (x[i] - mean) * (x[i] - mean);
  rstd = rsqrtf(row_sum(q, red) / D + eps);
}

__global__ void __launch_bounds__(THREADS) sandwich_kernel(const SandwichArgs s, int* err) {
  griddep_wait();
  griddep_launch();
  extern __shared__ float x[];
  __shared__ float red[THREADS / 32];
  const int D = s.dim;
  const size_t row = blockIdx.x;
  const size_t mod = s.group_rows ? row / s.group_rows * s.ldm : 0;
  float mean, rstd;
  if (s.y) {
    for (int i = threadIdx.x; i < D; i += THREADS) {
      float v = 0.f;
      if (s.parts == 0) v = load_any(s.y, s.y_type, row * s.ldy + i);
      for (int j = 0; j < s.parts; ++j) {
        const int slot = s.slot[row * s.parts + j];
        if (slot >= s.y_rows) fb_report(err, FB_DEVERR_BAD_INDEX);
        if (slot < 0 || slot >= s.y_rows) continue;
        v += s.weight[row * s.parts + j] * load_any(s.y, s.y_type, slot * s.ldy + i);
      }
      x[i] = v;
    }
    row_stats(x, D, s.post, s.post_eps, red, mean, rstd);
  }
  for (int i = threadIdx.x; i < D; i += THREADS) {
    float v = s.resid_scale * load_any(s.h, s.h_type, row * s.ldh + i);
    if (s.y) {
      const float u = (x[i] - mean) * rstd * (s.post_w ? s.post_w[i] : 1.f) +
                      (s.post_b ? s.post_b[i] : 0.f);
      v += (s.gate ? s.gate[mod + i] : 1.f) * u;
    }
    x[i] = v;
    if (s.h_out) store_any(s.h_out, s.h_type, row * s.ldho + i, v);
  }
  if (!s.a) return;
  row_stats(x, D, s.pre, s.pre_eps, red, mean, rstd);
  for (int i = threadIdx.x; i < D; i += THREADS)
    store_any(s.a, s.a_type, row * s.lda + i,
              (x[i] - mean) * rstd * (s.mul_base + (s.mul ? s.mul[mod + i] : 0.f)) +
                  (s.add ? s.add[mod + i] : 0.f));
}

}  // namespace

cudaError_t sandwich_norm(const SandwichArgs& s, int* err, int num_sms, cudaStream_t st) {
  if (s.rows == 0) return cudaSuccess;
  const size_t smem = (size_t)s.dim * sizeof(float);
  const cudaError_t e = cudaFuncSetAttribute(
      sandwich_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, FB_SANDWICH_MAX_DIM * 4);
  if (e != cudaSuccess) return e;
  return launch_k(sandwich_kernel, dim3(s.rows), dim3(THREADS), smem, st, s, err);
}
