// Attention to encoder states of another length: the query rows of sequence s attend to the keys
// and values of states kv_of[s], whose number differs from one to the next.
//
// The simple form: a warp per (query row, head) goes over the keys 32 at a time, a lane a key for
// the scores and a lane head_dim / 32 columns for the values, with the running maximum and sum of
// an online softmax.
#include <cfloat>

#include "kernels.h"

namespace {

constexpr int WARPS = 8;

// Sequence of row r: the last s with off[s] <= r; -1 where r lies behind the last sequence. Checks
// the offsets that it comes upon.
__device__ int sequence_of(const CrossArgs& c, int r, bool* bad) {
  int lo = 0, hi = c.seqs;  // off[lo] <= r < off[hi]
  const int first = c.q_offsets[0], last = c.q_offsets[c.seqs];
  *bad = first != 0 || last < 0 || last > c.q_rows;
  if (*bad || r >= last) return -1;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (c.q_offsets[mid] <= r) lo = mid;
    else hi = mid;
  }
  return lo;
}

template <int D>
__global__ void __launch_bounds__(WARPS * 32) cross_kernel(const CrossArgs c, int* err) {
  griddep_wait();
  griddep_launch();
  constexpr int E = D / 32;
  const int lane = threadIdx.x % 32, group = c.heads / c.kv_heads;
  __shared__ float qs[WARPS][D];
  float* q = qs[threadIdx.x / 32];
  const bf16* K = (const bf16*)c.k;
  const bf16* V = (const bf16*)c.v;
  // every block checks the offsets
  bool broken = false;
  for (int s = threadIdx.x; s < c.seqs; s += WARPS * 32) {
    const int u = c.kv_of ? c.kv_of[s] : s;
    broken = broken || c.q_offsets[s + 1] < c.q_offsets[s] || u < 0 || u >= c.states;
  }
  for (int u = threadIdx.x; u < c.states; u += WARPS * 32)
    broken = broken || c.kv_offsets[u + 1] < c.kv_offsets[u];
  broken = broken || c.kv_offsets[0] != 0 || c.kv_offsets[c.states] > c.kv_rows;
  if (__syncthreads_or(broken)) {
    if (threadIdx.x == 0) fb_report(err, FB_DEVERR_BAD_INDEX);
    return;
  }
  const long long n = (long long)c.q_rows * c.heads;
  for (long long i = blockIdx.x * (long long)WARPS + threadIdx.x / 32; i < n;
       i += (long long)gridDim.x * WARPS) {
    const int r = (int)(i / c.heads), h = (int)(i % c.heads);
    bool bad;
    const int s = sequence_of(c, r, &bad);
    if (bad && lane == 0) fb_report(err, FB_DEVERR_BAD_INDEX);
    if (s < 0) continue;
    const int u = c.kv_of ? c.kv_of[s] : s;
    const int k0 = c.kv_offsets[u], k1 = c.kv_offsets[u + 1];
    __syncwarp();
    for (int e = lane; e < D; e += 32)
      q[e] = __bfloat162float(((const bf16*)c.q)[(size_t)r * c.ldq + (size_t)h * D + e]);
    __syncwarp();
    const size_t col = (size_t)(h / group) * D;
    float m = -FLT_MAX, l = 0.f, o[E] = {};
    for (int j0 = k0; j0 < k1; j0 += 32) {
      const int j = j0 + lane;
      float x = -INFINITY;
      if (j < k1 && (!c.valid || c.valid[j])) {
        const bf16* k = K + (size_t)j * c.ldk + col;
        x = 0.f;
        for (int e = 0; e < D; e += 8) {
          float kv[8];
          load_bf16x8(k + e, kv);
#pragma unroll
          for (int t = 0; t < 8; ++t) x = fmaf(q[e + t], kv[t], x);
        }
        x *= c.scale;
      }
      float top = x;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      const float m_new = fmaxf(m, top), alpha = expf(m - m_new), p = expf(x - m_new);
      m = m_new;
      float sum = p;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      l = l * alpha + sum;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] *= alpha;
      for (int t = 0; t < 32; ++t) {
        const float pt = __shfl_sync(0xffffffffu, p, t);
        if (pt == 0.f) continue;  // masked (and what is too small to count)
        const bf16* v = V + (size_t)(j0 + t) * c.ldv + col + lane * E;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(pt, __bfloat162float(v[e]), o[e]);
      }
    }
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
    bf16* out = (bf16*)c.out + (size_t)r * c.ldo + (size_t)h * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = __float2bfloat16(o[e] * inv);
  }
}

}  // namespace

cudaError_t cross_attention(const CrossArgs& c, int* err, int num_sms, cudaStream_t st) {
  const long long need = ((long long)c.q_rows * c.heads + WARPS - 1) / WARPS, most = 8ll * num_sms;
  const dim3 grid((unsigned)(need < most ? need : most));
  return c.head_dim == 128
             ? launch_k(cross_kernel<128>, grid, dim3(WARPS * 32), 0, st, c, err)
             : launch_k(cross_kernel<64>, grid, dim3(WARPS * 32), 0, st, c, err);
}
