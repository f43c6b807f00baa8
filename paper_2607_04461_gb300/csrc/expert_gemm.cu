// Matrix products grouped by expert: rows offsets[e] .. offsets[e + 1] - 1 of the output are
//   out[r] = act(x W_e^T + b_e),  x = A[index[r]] (or row r of A)
// with act GELU (tanh form) or, over W_e's 2 n rows (gate rows, then up rows), SiLU or GELU of
// the first n results times the other n. The sizes of the groups are read on the device.
//
// 64 x 64 tiles on the CUDA cores; a row tile belongs to one expert.
#include "kernels.h"

namespace {

constexpr int TR = 64, TC = 64, TK = 16, THREADS = 256;

__device__ __forceinline__ float act_value(int act, float x, float up) {
  switch (act) {
    case FB_ACT_GELU:
    case FB_ACT_GEGLU: {
      const float g = 0.5f * x * (1.f + tanhf(0.7978845608028654f * (x + 0.044715f * x * x * x)));
      return act == FB_ACT_GELU ? g : g * up;
    }
    case FB_ACT_SWIGLU: return x / (1.f + expf(-x)) * up;
  }
  return x;
}

__global__ void __launch_bounds__(THREADS) expert_gemm_kernel(const ExpertArgs g, int* err) {
  griddep_wait();
  griddep_launch();
  __shared__ float xs[TK][TR + 1], ws[TK][TC + 1], us[TK][TC + 1];
  __shared__ int s_e, s_r0, s_r1;
  __shared__ int src[TR];
  const bool gated = g.act >= FB_ACT_SWIGLU;
  if (threadIdx.x == 0) {
    s_e = -1;
    int tile = 0, prev = 0;
    for (int e = 0; e < g.experts; ++e) {
      const int r0 = g.offsets[e], r1 = g.offsets[e + 1];
      if (r0 != prev || r1 < r0 || r1 > g.max_rows) {
        fb_report(err, FB_DEVERR_BAD_INDEX);
        s_e = -1;
        break;
      }
      prev = r1;
      const int n = (r1 - r0 + TR - 1) / TR;
      if ((int)blockIdx.y >= tile && (int)blockIdx.y < tile + n) {
        s_e = e;
        s_r0 = r0 + ((int)blockIdx.y - tile) * TR;
        s_r1 = min(s_r0 + TR, r1);
      }
      tile += n;
    }
  }
  __syncthreads();
  if (s_e < 0) return;
  const int e = s_e, r0 = s_r0, nr = s_r1 - s_r0, c0 = blockIdx.x * TC;
  if (threadIdx.x < TR) {
    int s = r0 + min((int)threadIdx.x, nr - 1);
    if (g.index) s = g.index[s];
    if (s < 0 || s >= g.a_rows) {
      fb_report(err, FB_DEVERR_BAD_INDEX);
      s = 0;
    }
    src[threadIdx.x] = s;
  }
  __syncthreads();
  const size_t nw = gated ? 2 * (size_t)g.n : g.n;
  const bf16* W = g.W + (size_t)e * nw * g.k;
  const int tr = threadIdx.x / 16 * 4, tc = threadIdx.x % 16 * 4;
  float acc[4][4] = {}, acu[4][4] = {};
  for (int k0 = 0; k0 < g.k; k0 += TK) {
    for (int i = threadIdx.x; i < TR * TK; i += THREADS) {
      const int row = i / TK, k = i % TK;
      const bool in = k0 + k < g.k;
      xs[k][row] = in ? __bfloat162float(g.A[(size_t)src[row] * g.lda + k0 + k]) : 0.f;
      const bool win = in && c0 + row < g.n;
      ws[k][row] = win ? __bfloat162float(W[(size_t)(c0 + row) * g.k + k0 + k]) : 0.f;
      if (gated)
        us[k][row] = win ? __bfloat162float(W[((size_t)g.n + c0 + row) * g.k + k0 + k]) : 0.f;
    }
    __syncthreads();
    for (int k = 0; k < TK; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          acc[i][j] += xs[k][tr + i] * ws[k][tc + j];
          if (gated) acu[i][j] += xs[k][tr + i] * us[k][tc + j];
        }
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int c = c0 + tc + j;
      if (tr + i >= nr || c >= g.n) continue;
      float v = acc[i][j], u = acu[i][j];
      if (g.bias) {
        v += g.bias[e * nw + c];
        if (gated) u += g.bias[e * nw + g.n + c];
      }
      v = act_value(g.act, v, u);
      const size_t o = (size_t)(r0 + tr + i) * g.ldo + c;
      if (g.out_type == FB_F32)
        reinterpret_cast<float*>(g.out)[o] = v;
      else
        reinterpret_cast<bf16*>(g.out)[o] = __float2bfloat16(v);
    }
}

}  // namespace

cudaError_t expert_gemm(const ExpertArgs& g, int* err, int num_sms, cudaStream_t st) {
  if (g.max_rows == 0) return cudaSuccess;
  const dim3 grid((g.n + TC - 1) / TC, (g.max_rows + TR - 1) / TR + g.experts);
  return launch_k(expert_gemm_kernel, grid, dim3(THREADS), 0, st, g, err);
}
