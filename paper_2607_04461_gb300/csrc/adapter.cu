// A projection shared by all rows with a low-rank adapter for each segment of them:
//   y = x W^T + bias + scale_e (x A_e^T) B_e^T,  e the adapter of the row's segment
//
// The simple form: one kernel forms t = scale_e x A_e^T (fp32, a warp per element), one the
// product, 64 x 64 results a block through shared memory, and adds t B_e^T row by row.
#include "kernels.h"

namespace {

// Segment of row r (the last with offsets[i] <= r), -1 behind the last one.
__device__ int segment_of(const AdapterArgs& g, int r) {
  if (r >= g.offsets[g.segments]) return -1;
  int lo = 0, hi = g.segments;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (g.offsets[mid] <= r) lo = mid;
    else hi = mid;
  }
  return lo;
}
__device__ bool bad_segments(const AdapterArgs& g) {
  bool bad = g.offsets[0] != 0 || g.offsets[g.segments] > g.rows;
  for (int i = threadIdx.x; i < g.segments; i += blockDim.x)
    bad = bad || g.offsets[i + 1] < g.offsets[i] || g.adapter[i] < -1 || g.adapter[i] >= g.adapters;
  return __syncthreads_or(bad);
}

__global__ void __launch_bounds__(256) adapter_t_kernel(const AdapterArgs g, float* t, int* err) {
  griddep_wait();
  griddep_launch();
  if (bad_segments(g)) {
    if (threadIdx.x == 0) fb_report(err, FB_DEVERR_BAD_INDEX);
    return;
  }
  const int lane = threadIdx.x % 32;
  const long long n = (long long)g.rows * g.rank;
  for (long long i = blockIdx.x * 8ll + threadIdx.x / 32; i < n; i += gridDim.x * 8ll) {
    const int r = (int)(i / g.rank), j = (int)(i % g.rank);
    const int s = segment_of(g, r), e = s < 0 ? -1 : g.adapter[s];
    if (e < 0) continue;
    const bf16* x = (const bf16*)g.x + (size_t)r * g.ldx;
    const bf16* a = (const bf16*)g.a + ((size_t)e * g.rank + j) * g.k;
    float sum = 0.f;
    for (int k = lane; k < g.k; k += 32)
      sum = fmaf(__bfloat162float(x[k]), __bfloat162float(a[k]), sum);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (lane == 0) t[i] = sum * (g.scale ? g.scale[e] : 1.f);
  }
}

__global__ void __launch_bounds__(256) adapter_kernel(const AdapterArgs g, const float* t) {
  griddep_wait();
  griddep_launch();
  if (bad_segments(g)) return;
  __shared__ float xs[16][64 + 1], ws[16][64 + 1];
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  const int tiles_n = (g.n + 63) / 64;
  const int r0 = blockIdx.x / tiles_n * 64, f0 = blockIdx.x % tiles_n * 64;
  float c[4][4] = {};
  for (int k0 = 0; k0 < g.k; k0 += 16) {
    for (int i = threadIdx.x; i < 64 * 16; i += 256) {
      const int row = i / 16, k = k0 + i % 16;
      const bool in = k < g.k;
      xs[i % 16][row] = in && r0 + row < g.rows
                            ? __bfloat162float(((const bf16*)g.x)[(size_t)(r0 + row) * g.ldx + k]) : 0.f;
      ws[i % 16][row] = in && f0 + row < g.n
                            ? __bfloat162float(((const bf16*)g.w)[(size_t)(f0 + row) * g.k + k]) : 0.f;
    }
    __syncthreads();
    for (int k = 0; k < 16; ++k)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) c[i][j] = fmaf(xs[k][ty + 16 * i], ws[k][tx + 16 * j], c[i][j]);
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i) {
    const int r = r0 + ty + 16 * i;
    const int s = r < g.rows ? segment_of(g, r) : -1;
    if (s < 0) continue;
    const int e = g.adapter[s];
    for (int j = 0; j < 4; ++j) {
      const int f = f0 + tx + 16 * j;
      if (f >= g.n) continue;
      float y = c[i][j] + (g.bias ? g.bias[f] : 0.f);
      if (e >= 0) {
        const bf16* b = (const bf16*)g.b + ((size_t)e * g.n + f) * g.rank;
        float d = 0.f;
        for (int q = 0; q < g.rank; ++q) d = fmaf(t[(size_t)r * g.rank + q], __bfloat162float(b[q]), d);
        y += d;
      }
      if (g.act == FB_ACT_GELU)
        y = y / (1.f + expf(-1.5957691216057308f * (y + 0.044715f * y * y * y)));
      if (g.gate) y *= g.gate[f];
      if (g.resid) y += g.resid[(size_t)r * g.ldr + f];
      const size_t at = (size_t)r * g.ldo + f;
      if (g.out_type == FB_F32) ((float*)g.out)[at] = y;
      else ((bf16*)g.out)[at] = __float2bfloat16(y);
    }
  }
}

}  // namespace

size_t adapter_ws_bytes(const AdapterArgs& g) { return (size_t)g.rows * g.rank * sizeof(float); }
int adapter_launches(const AdapterArgs&) { return 2; }

cudaError_t adapter_gemm(const AdapterArgs& g, void* ws, int* err, int num_sms, cudaStream_t st) {
  const long long need = ((long long)g.rows * g.rank + 7) / 8, most = 8ll * num_sms;
  cudaError_t e = launch_k(adapter_t_kernel, dim3((unsigned)(need < most ? need : most)), dim3(256),
                           0, st, g, (float*)ws, err);
  if (e != cudaSuccess) return e;
  const long long blocks = (long long)((g.rows + 63) / 64) * ((g.n + 63) / 64);
  return launch_k(adapter_kernel, dim3((unsigned)blocks), dim3(256), 0, st, g, (const float*)ws);
}
