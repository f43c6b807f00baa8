// The router of a mixture of experts: the top-k experts of each token, their weights, and the
// (token, expert) pairs sorted by expert, tokens in order within one (a stable counting sort).
//
// Logits compare as fp32 values and ties go to the lower expert, so the choice does not depend
// on how a sum was ordered. A NaN or -inf logit is never chosen, +inf counts as the largest
// finite value; a token without a logit left, or with valid = 0, goes nowhere.
//
// topk: one warp per token, its k largest (key, expert) pairs one after the other, each the
// largest below the last one. sort: one block per expert (and one for the pairs that go
// nowhere) counts the pairs of the experts before it and ranks its own.
#include <float.h>

#include "kernels.h"

namespace {

constexpr int WARPS = 4;
constexpr int SORT_THREADS = 1024;

// An fp32 value's bits in the order of the values; 0 for what is never chosen.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (!(x > -INFINITY)) return 0;  // NaN, -inf
  const uint32_t u = __float_as_uint(fminf(x, FLT_MAX) + 0.f);  // (-0 + 0 = +0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ float load_logit(const RouteArgs& r, size_t i) {
  return r.logits_type == FB_F32 ? reinterpret_cast<const float*>(r.logits)[i]
                                 : __bfloat162float(reinterpret_cast<const bf16*>(r.logits)[i]);
}

__global__ void __launch_bounds__(WARPS * 32) route_topk_kernel(const RouteArgs r) {
  griddep_wait();
  griddep_launch();
  const int lane = threadIdx.x % 32;
  const size_t t = (size_t)blockIdx.x * WARPS + threadIdx.x / 32;
  if (t >= (size_t)r.tokens) return;
  const bool live = !r.valid || r.valid[t];
  unsigned long long last = ~0ull;
  float first = 0.f, total = 0.f;
  float value[FB_ROUTE_MAX_TOP_K];
  int n = 0;
  for (int j = 0; j < r.top_k; ++j) {
    unsigned long long best = 0;
    for (int e = lane; live && e < r.experts; e += 32) {
      const unsigned long long c =
          (unsigned long long)order_key(load_logit(r, t * r.ldl + e)) << 32 | (uint32_t)~e;
      if (c < last && c > best) best = c;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long c = __shfl_xor_sync(0xffffffffu, best, o);
      if (c > best) best = c;
    }
    last = best;
    const uint32_t key = (uint32_t)(best >> 32);
    if (lane == 0) r.expert[t * r.top_k + j] = key ? (int)~(uint32_t)best : -1;
    if (key) {
      const float v = key_value(key);
      if (j == 0) first = v;
      value[n++] = expf(v - first);
      if (r.renorm) total += value[j];
    }
  }
  if (!r.renorm) {
    for (int e = lane; live && e < r.experts; e += 32) {
      const uint32_t key = order_key(load_logit(r, t * r.ldl + e));
      if (key) total += expf(key_value(key) - first);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  }
  if (lane == 0)
    for (int j = 0; j < r.top_k; ++j) r.weight[t * r.top_k + j] = j < n ? value[j] / total : 0.f;
}

__global__ void __launch_bounds__(SORT_THREADS) route_sort_kernel(const RouteArgs r) {
  griddep_wait();
  griddep_launch();
  __shared__ int warp_n[SORT_THREADS / 32];
  __shared__ int before;
  const int e = blockIdx.x, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const bool nowhere = e == r.experts;
  const int n = r.tokens * r.top_k;
  if (threadIdx.x == 0) before = 0;
  __syncthreads();
  int mine = 0;
  for (int i = threadIdx.x; i < n; i += SORT_THREADS) mine += r.expert[i] >= 0 && r.expert[i] < e;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  if (lane == 0) atomicAdd(&before, mine);
  __syncthreads();
  int base = before;
  if (threadIdx.x == 0) r.offsets[e] = base;
  for (int i0 = 0; i0 < n; i0 += SORT_THREADS) {
    const int i = i0 + threadIdx.x;
    const bool hit = i < n && r.expert[i] == (nowhere ? -1 : e);
    const unsigned m = __ballot_sync(0xffffffffu, hit);
    __syncthreads();
    if (lane == 0) warp_n[warp] = __popc(m);
    __syncthreads();
    int rank = base + __popc(m & ((1u << lane) - 1));
    for (int w = 0; w < SORT_THREADS / 32; ++w) {
      if (w < warp) rank += warp_n[w];
      base += warp_n[w];
    }
    if (hit) {
      r.slot[i] = nowhere ? -1 : rank;
      r.token[rank] = nowhere ? -1 : i / r.top_k;
    }
  }
}

}  // namespace

cudaError_t route(const RouteArgs& r, cudaStream_t st) {
  if (r.tokens > 0) {
    const cudaError_t e = launch_k(route_topk_kernel, dim3((r.tokens + WARPS - 1) / WARPS),
                                   dim3(WARPS * 32), 0, st, r);
    if (e != cudaSuccess) return e;
  }
  return launch_k(route_sort_kernel, dim3(r.experts + 1), dim3(SORT_THREADS), 0, st, r);
}
