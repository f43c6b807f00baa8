// The router of a mixture of experts: the top-k experts of each token, their weights, and the
// (token, expert) pairs sorted by expert, tokens in order within one (a stable counting sort).
//
// Logits compare as fp32 values and ties go to the lower expert, so the choice does not depend
// on how a sum was ordered. A NaN or -inf logit is never chosen, +inf counts as the largest
// finite value; a token without a logit left, or with valid = 0, goes nowhere.
//
// A worker, 8, 16 or 32 lanes (see route()), holds a token's logits as integers in the order of
// the values, the next token's on their way, and takes the largest k times.
// Pairs are ranked without atomics whose order could change them: a worker counts its own tokens
// in order, a block adds its workers' counts up, and
//  * few tokens (in_cluster) are one launch of a cluster of eight blocks, which read each other's
//    counts through distributed shared memory (one block up to 32 tokens);
//  * more tokens take three launches: choice and counts by blocks of up to 128 tokens, the
//    blocks' counts added up expert by expert, and the pairs put in their places.
// One token over 8 experts 2.7 us, 1560 5.9, 49920 over 64 (top 8) 26: bound by the latency of the
// chains and launches up to a few thousand tokens, then by the choice, 390 blocks in two rounds of
// 304 (46 registers: two an SM) at 46 % of the issue slots, and the two launches behind it; the
// 19 MB that the last one moves would take 2.8.
#include <float.h>

#include "kernels.h"

namespace {

constexpr int WARPS = 16, THREADS = WARPS * 32;
constexpr int MAX_E = FB_ROUTE_MAX_EXPERTS, MAX_K = FB_ROUTE_MAX_TOP_K;
constexpr int MAX_BLOCK_TOKENS = 128;  // of the three-launch form
constexpr int CLUSTER = 8;

// Whether one launch of a cluster takes all tokens. us, cluster / three launches, top 8 of 8
// experts, 512 tokens 5.8 / 7.2, 768 7.8 / 7.2 (top 2 5.1 / 6.3); of 64, 384 tokens 7.2 / 7.6,
// 512 8.7 / 7.9; of 256, 256 tokens 8.3 / 10.2, 384 11.0 / 10.3 (top 2 7.6 / 8.2); of 512, 256
// tokens 12.6 / 14.5, 384 17.1 / 14.5.
bool in_cluster(const RouteArgs& r) {
  return r.tokens <= (r.experts <= 8 ? 768 : r.experts <= 256 ? 384 : 256);
}

// An fp32 value's bits in the order of the values; 0 for what is never chosen.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (!(x > -INFINITY)) return 0;  // NaN, -inf
  const uint32_t u = __float_as_uint(fminf(x, FLT_MAX) + 0.f);  // (-0 + 0 = +0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// Workers of a block with L lanes each, and the experts that they take.
template <int L>
struct Work {
  static constexpr int WORKERS = THREADS / L, EXPERTS = 16 * L;  // (MAX_E for a warp)
};
struct Shared {
  uint16_t count[WARPS * MAX_E];  // [worker][expert]: its pairs, then those of the workers before
  int total[MAX_E];               // the block's pairs per expert
  int base[MAX_E];                // first place of the block's pairs of an expert
  int scan[WARPS];
};

// The logits of token t: R consecutive experts per lane; keys of 0 where there is none.
template <int R>
__device__ __forceinline__ void load_keys(const RouteArgs& r, int t, int sub, uint32_t* key) {
  const bool live = !r.valid || r.valid[t];
  const size_t at = (size_t)t * r.ldl + sub * R;
  const int n = live ? r.experts - sub * R : 0;
#pragma unroll
  for (int i = 0; i < R; ++i) key[i] = 0;
  if (r.logits_type == FB_F32) {
    const float* p = reinterpret_cast<const float*>(r.logits) + at;
    if (R % 4 == 0 && r.vec) {
#pragma unroll
      for (int i = 0; i < R; i += 4)
        if (i < n) {
          const float4 v = *reinterpret_cast<const float4*>(p + i);
          key[i] = order_key(v.x);
          key[i + 1] = order_key(v.y);
          key[i + 2] = order_key(v.z);
          key[i + 3] = order_key(v.w);
        }
      return;
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (i < n) key[i] = order_key(p[i]);
  } else {
    const bf16* p = reinterpret_cast<const bf16*>(r.logits) + at;
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (i < n) key[i] = order_key(__bfloat162float(p[i]));
  }
}

// Tokens first .. end - 1 of the block: experts and weights go out, pair (t, j) gets (expert,
// rank among the worker's pairs of it) in pairs[(t - first) top_k + j], or ~0 without an expert.
// Then the workers' counts are added up. Ends with a barrier.
template <int L, int R>
__device__ __forceinline__ void choose(const RouteArgs& r, int first, int end, Shared& sh,
                                       uint32_t* pairs) {
  constexpr int NJ = (MAX_K + L - 1) / L;  // choices that a lane keeps
  const int sub = threadIdx.x % L, worker = threadIdx.x / L, k = r.top_k;
  uint16_t* count = sh.count + worker * Work<L>::EXPERTS;
  for (int e = sub; e < r.experts; e += L) count[e] = 0;
  __syncwarp();
  const int per = (end - first + Work<L>::WORKERS - 1) / Work<L>::WORKERS;
  const int t0 = first + worker * per, t1 = min(end, t0 + per);
  uint32_t next[R];
#pragma unroll
  for (int i = 0; i < R; ++i) next[i] = 0;
  if (t0 < t1) load_keys<R>(r, t0, sub, next);
  for (int q = 0; q < per; ++q) {  // (all workers of a warp together; some have no token)
    const int t = t0 + q;
    const bool mine = t < t1;
    uint32_t key[R];
#pragma unroll
    for (int i = 0; i < R; ++i) key[i] = mine ? next[i] : 0;
    if (t + 1 < t1) load_keys<R>(r, t + 1, sub, next);
    uint32_t best, top_key = 0;  // the lane's largest key left, and its place
    int at;
    float total = 0.f, top = 0.f;
    int expert[NJ];
    uint32_t chosen[NJ];
#pragma unroll
    for (int i = 0; i < NJ; ++i) {
      expert[i] = -1;
      chosen[i] = 0;
    }
    auto find_best = [&] {
      best = key[0];
      at = 0;
#pragma unroll
      for (int i = 1; i < R; ++i)
        if (key[i] > best) {
          best = key[i];
          at = i;
        }
    };
    find_best();
    auto largest = [&](uint32_t& most, int& e) {
      if (L == 32) {
        // (lanes hold experts in order: the lowest lane with it has the lowest one)
        most = __reduce_max_sync(0xffffffffu, best);
        const int from = __ffs(__ballot_sync(0xffffffffu, best == most)) - 1;
        e = __shfl_sync(0xffffffffu, sub * R + at, from);
      } else {
        most = best;
        e = sub * R + at;
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) {
          const uint32_t m = __shfl_xor_sync(0xffffffffu, most, o);
          const int x = __shfl_xor_sync(0xffffffffu, e, o);
          if (m > most || (m == most && x < e)) {
            most = m;
            e = x;
          }
        }
      }
    };
    uint32_t most;
    int e;
    largest(most, e);
    top_key = most;
    top = key_value(most);
    if (!r.renorm && top_key) {
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (key[i]) total += expf(key_value(key[i]) - top);
    }
    // (no branch but the loop's: every lane removes what it holds of e and looks again)
#pragma unroll 1
    for (int j = 0;; ++j) {
#pragma unroll
      for (int i = 0; i < NJ; ++i) {
        const bool keep = j == i * L + sub && most;
        expert[i] = keep ? e : expert[i];
        chosen[i] = keep ? most : chosen[i];
      }
      if (j + 1 >= k) break;
      const int gone = e - sub * R;
#pragma unroll
      for (int i = 0; i < R; ++i) key[i] = i == gone ? 0 : key[i];
      find_best();
      largest(most, e);
    }
    float value[NJ];
#pragma unroll
    for (int i = 0; i < NJ; ++i) {
      value[i] = expert[i] < 0 ? 0.f : expf(key_value(chosen[i]) - top);
      if (r.renorm) total += value[i];
    }
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
#pragma unroll
    for (int i = 0; i < NJ; ++i) {
      const int j = i * L + sub;
      if (!mine || j >= k) continue;
      const size_t out = (size_t)t * k + j;
      r.expert[out] = expert[i];
      r.weight[out] = expert[i] < 0 ? 0.f : value[i] / total;
      // (a token's experts differ: no two lanes meet on a counter)
      const uint32_t rank = expert[i] < 0 ? 0 : count[expert[i]]++;
      pairs[(t - first) * k + j] = expert[i] < 0 ? ~0u : (uint32_t)expert[i] << 16 | rank;
    }
    __syncwarp();
  }
  __syncthreads();
  for (int e = threadIdx.x; e < r.experts; e += THREADS) {
    int sum = 0;
#pragma unroll 16
    for (int w = 0; w < Work<L>::WORKERS; ++w) {
      uint16_t& c = sh.count[w * Work<L>::EXPERTS + e];
      const int n = c;
      c = (uint16_t)sum;
      sum += n;
    }
    sh.total[e] = sum;
  }
  __syncthreads();
}

// Exclusive sums over all experts (one per thread, 0 behind the last); *all their total.
__device__ __forceinline__ int scan_experts(int n, Shared& sh, int* all) {
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  int s = n;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += v;
  }
  if (lane == 31) sh.scan[warp] = s;
  __syncthreads();
  int before = 0;
  *all = 0;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    if (w < warp) before += sh.scan[w];
    *all += sh.scan[w];
  }
  return before + s - n;
}

// The places of the block's pairs; token entries behind the last pair become -1.
template <int L>
__device__ __forceinline__ void place(const RouteArgs& r, int first, int end, const Shared& sh,
                                      const uint32_t* pairs, int all) {
  const int k = r.top_k, per = (end - first + Work<L>::WORKERS - 1) / Work<L>::WORKERS;
  for (int i = threadIdx.x; i < (end - first) * k; i += THREADS) {
    const int t = i / k, at = first * k + i;
    const uint32_t p = pairs[i];
    int slot = -1;
    if (p != ~0u) {
      const int e = p >> 16;
      slot = sh.base[e] + sh.count[t / per * Work<L>::EXPERTS + e] + (int)(p & 0xffffu);
      r.token[slot] = first + t;
    }
    r.slot[at] = slot;
    if (at >= all) r.token[at] = -1;
  }
}

// ---- one launch -------------------------------------------------------------------------
__device__ __forceinline__ int ld_cluster(uint32_t addr) {
  int v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

template <int L, int R, int C>
__device__ __forceinline__ void route_cluster(const RouteArgs& r) {
  __shared__ Shared sh;
  extern __shared__ uint32_t pairs[];
  const int rank = C > 1 ? (int)cluster_ctarank() : 0;
  const int share = (r.tokens + C - 1) / C;
  const int first = min(r.tokens, rank * share), end = min(r.tokens, first + share);
  choose<L, R>(r, first, end, sh, pairs);
  if (C > 1) cluster_sync();  // every block's totals are there
  int before = 0, n = 0;
  const int e = threadIdx.x;
  if (e < r.experts) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int v = C > 1 ? ld_cluster(mapa_shared(smem_u32(&sh.total[e]), c)) : sh.total[e];
      if (c < rank) before += v;
      n += v;
    }
  }
  int all;
  const int off = scan_experts(n, sh, &all);
  if (e < r.experts) sh.base[e] = off + before;
  if (rank == 0 && e < r.experts) r.offsets[e] = off;
  if (rank == 0 && e == 0) r.offsets[r.experts] = all;
  __syncthreads();
  place<L>(r, first, end, sh, pairs, all);
  if (C > 1) cluster_sync();  // (no block leaves while its totals are read)
}
template <int L, int R>
__global__ void __launch_bounds__(THREADS) route_block_kernel(const RouteArgs r) {
  griddep_wait();
  griddep_launch();
  route_cluster<L, R, 1>(r);
}
template <int L, int R>
__global__ void __cluster_dims__(CLUSTER, 1, 1) __launch_bounds__(THREADS)
    route_cluster_kernel(const RouteArgs r) {
  griddep_wait();
  griddep_launch();
  route_cluster<L, R, CLUSTER>(r);
}

// ---- three launches ---------------------------------------------------------------------
// counts: [blocks][experts], then [experts] totals. The ranks wait in slot.
template <int L, int R>
__global__ void __launch_bounds__(THREADS) route_choose_kernel(const RouteArgs r, int* counts, int block_tokens) {
  griddep_wait();
  griddep_launch();
  __shared__ Shared sh;
  __shared__ uint32_t pairs[MAX_BLOCK_TOKENS * MAX_K];
  const int first = blockIdx.x * block_tokens, end = min(r.tokens, first + block_tokens);
  choose<L, R>(r, first, end, sh, pairs);
  for (int e = threadIdx.x; e < r.experts; e += THREADS)
    counts[(size_t)blockIdx.x * r.experts + e] = sh.total[e];
  const int k = r.top_k, per = (end - first + Work<L>::WORKERS - 1) / Work<L>::WORKERS;
  for (int i = threadIdx.x; i < (end - first) * k; i += THREADS) {
    const uint32_t p = pairs[i];
    if (p != ~0u)
      r.slot[(size_t)first * k + i] =
          sh.count[i / k / per * Work<L>::EXPERTS + (p >> 16)] + (p & 0xffffu);
  }
}

// One warp per expert: the blocks' counts become those of the blocks before them.
__global__ void __launch_bounds__(128) route_sum_kernel(const RouteArgs r, int* counts, int blocks) {
  griddep_wait();
  griddep_launch();
  const int lane = threadIdx.x % 32, e = blockIdx.x * 4 + threadIdx.x / 32;
  if (e >= r.experts) return;
  constexpr int PER = 16;  // blocks a lane: one pass up to 512
  int sum = 0;
  for (int b0 = 0; b0 < blocks; b0 += 32 * PER) {
    int n[PER], s = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int b = b0 + PER * lane + j;
      n[j] = b < blocks ? counts[(size_t)b * r.experts + e] : 0;
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) s += n[j];
    int inc = s;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += v;
    }
    int at = sum + inc - s;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int b = b0 + PER * lane + j;
      if (b < blocks) counts[(size_t)b * r.experts + e] = at;
      at += n[j];
    }
    sum += __shfl_sync(0xffffffffu, inc, 31);
  }
  if (lane == 0) counts[(size_t)blocks * r.experts + e] = sum;
}

__global__ void __launch_bounds__(THREADS) route_place_kernel(const RouteArgs r, const int* counts,
                                                              int blocks, int block_tokens) {
  griddep_wait();
  griddep_launch();
  __shared__ Shared sh;
  const int e = threadIdx.x;
  int all;
  const int off = scan_experts(
      e < r.experts ? counts[(size_t)blocks * r.experts + e] : 0, sh, &all);
  if (e < r.experts) sh.base[e] = off + counts[(size_t)blockIdx.x * r.experts + e];
  if (blockIdx.x == 0 && e < r.experts) r.offsets[e] = off;
  if (blockIdx.x == 0 && e == 0) r.offsets[r.experts] = all;
  __syncthreads();
  const int k = r.top_k, first = blockIdx.x * block_tokens, end = min(r.tokens, first + block_tokens);
  for (int i = first * k + e; i < end * k; i += THREADS) {
    const int x = r.expert[i];
    int slot = -1;
    if (x >= 0) {
      slot = sh.base[x] + r.slot[i];
      r.token[slot] = i / k;
    }
    r.slot[i] = slot;
    if (i >= all) r.token[i] = -1;
  }
}

// Tokens of a block: few enough that every SM has a block or two.
int block_tokens(const RouteArgs& r) {
  return r.tokens <= 32 * 304 ? 32 : r.tokens <= 64 * 304 ? 64 : MAX_BLOCK_TOKENS;
}

template <int L, int R>
cudaError_t run(const RouteArgs& r, int* counts, cudaStream_t st) {
  if (in_cluster(r)) {
    const int share = (r.tokens + CLUSTER - 1) / CLUSTER;
    if (r.tokens <= 32)
      return launch_k(route_block_kernel<L, R>, dim3(1), dim3(THREADS),
                      (size_t)r.tokens * r.top_k * 4, st, r);
    return launch_k(route_cluster_kernel<L, R>, dim3(CLUSTER), dim3(THREADS),
                    (size_t)share * r.top_k * 4, st, r);
  }
  const int bt = block_tokens(r), blocks = (r.tokens + bt - 1) / bt;
  cudaError_t e = launch_k(route_choose_kernel<L, R>, dim3(blocks), dim3(THREADS), 0, st, r, counts, bt);
  if (e == cudaSuccess)
    e = launch_k(route_sum_kernel, dim3((r.experts + 3) / 4), dim3(128), 0, st, r, counts, blocks);
  if (e == cudaSuccess)
    e = launch_k(route_place_kernel, dim3(blocks), dim3(THREADS), 0, st, r, (const int*)counts,
                 blocks, bt);
  return e;
}

}  // namespace

size_t route_ws_bytes(const RouteArgs& r) {
  if (in_cluster(r)) return 0;
  const size_t bt = block_tokens(r);
  return ((r.tokens + bt - 1) / bt + 1) * r.experts * sizeof(int);
}

int route_launches(const RouteArgs& r) { return in_cluster(r) ? 1 : 3; }

cudaError_t route(const RouteArgs& r0, void* ws, cudaStream_t st) {
  RouteArgs r = r0;
  r.vec = reinterpret_cast<uintptr_t>(r.logits) % 16 == 0 && r.ldl % 4 == 0 && r.experts % 4 == 0;
  int* counts = static_cast<int*>(ws);
  // Eight or sixteen lanes a worker for many tokens, where a warp's instructions are shared by
  // several; a warp each for few, whose reductions take less time (us, 8 or 16 lanes / a warp): 16
  // experts top 4, 1 token 3.4 / 2.7, 8192 tokens 9.8 / 9.3, 16384 10.3 / 11.8, 49920 16.0 / 26.9;
  // 64 top 8, 1 token 4.8 / 3.2, 8192 12.4 / 11.2, 49920 27.9 / 41.8.
  if (r.experts <= 8) return run<8, 1>(r, counts, st);
  if (r.tokens > 12288) {
    if (r.experts <= 16) return run<8, 2>(r, counts, st);
    if (r.experts <= 32) return run<8, 4>(r, counts, st);
    if (r.experts <= 64) return run<8, 8>(r, counts, st);
    if (r.experts <= 128) return run<8, 16>(r, counts, st);
    if (r.experts <= 256) return run<16, 16>(r, counts, st);
  }
  if (r.experts <= 32) return run<32, 1>(r, counts, st);
  if (r.experts <= 64) return run<32, 2>(r, counts, st);
  if (r.experts <= 128) return run<32, 4>(r, counts, st);
  if (r.experts <= 256) return run<32, 8>(r, counts, st);
  return run<32, 16>(r, counts, st);
}
