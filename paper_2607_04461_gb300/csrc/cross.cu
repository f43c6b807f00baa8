// Attention to encoder states of another length: the query rows of sequence s attend to the keys
// and values of states kv_of[s], whose number differs from one sequence to the next:
//   o_r = sum_j w_j v_j,  w = softmax_j(scale q_r . k_j)  over the keys that are not masked
//
// One persistent kernel on tcgen05, one CTA per SM. A tile is 128 rows of (query, head): with
// G = heads / kv_heads, RQ = 128 / G consecutive queries (rounded down) by the G heads that share
// a kv head (one TMA box of three dimensions), so K and V are read once for all of them, for one
// token as for many. An item is a pair of query tiles of one sequence and kv head, which share each
// 128-key tile of K and V (the last one may be single), or, where a sequence has one query tile and
// there are more such than SMs, a pair of kv heads side by side (dual), which keeps twice as much of
// K and V on its way. Both lengths come from device memory: the CTAs draw whole items from a counter,
// or take an equal stretch each of all items' key tiles where whole ones would leave SMs idle (see
// Plan).
//  * warp 0: TMA. Lane 0 loads Q and a ring of K tiles, lane 1 a ring of V tiles.
//  * warp 1: MMA issuer. S_g = Q_g K^T (both K-major in shared memory), then O_g += P_g V (P from
//    TMEM, V MN-major); the order PV_A(j), S_A(j+1), PV_B(j), S_B(j+1) lets each group's softmax run
//    beside the other group's MMAs.
//  * warps 2-9: softmax, one row per thread, warps 2-5 tile A, 6-9 tile B: running maximum and
//    sum in fp32 registers, P = exp2(scale log2(e) s - m) as bf16 over S in TMEM, O rescaled in TMEM
//    only when the maximum grew by more than 2^8. P's rounding is 2^-8 of a term at most; the sum is of the
//    unrounded values, so that where few keys count it stays in the result (32 sequences of 1560 rows on 512
//    keys: 2.03e-3 off, rounding the result alone gives 1.66e-3). A sum of the rounded values would give
//    1.83e-3 and take 158 us for 153 (added half a tile later, beside the next load, 159). Its code is kept
//    short, since an item's end and the next one's start run as fast as their instructions arrive: masked
//    scores become -inf in TMEM by a loop over 32 at a time, and exponentials are taken 64 at a time from a
//    second read (both unrolled over the 128 registers of the first read: 128 us for those 110).
//  * warp 10: masks. A weight of zero does not stop a NaN in V, so the V rows of masked keys, and
//    of what follows the last key up to a multiple of 16, are overwritten by zeros in shared
//    memory once they have landed; with a mask it also lays out each key tile's 128 bits for the
//    softmax, which takes masked scores as -inf by selection.
//  * warp 11: fetches the CTA's segments (whole items, parts of cut ones), up to three ahead (with one
//    ahead 115 us where three take 110: 32 sequences of 1560 rows on 20 to 512 keys).
// The last key tile's MMAs cover ceil16 of its keys. Every wait is bounded (mbar_wait): a role
// that gives up records it and the kernel ends.
//
// Bounds: with many queries for each key the hand-over between softmax and issuer: a step of 2 x 128 x 128
// takes about 2600 clocks, of which the tensor pipe needs 2049 and the exponentials 1056 (31 a clock); it waits
// for the arithmetic around them (32 candidates of 1560 rows, 12 heads of 128: 153 us, 1.03 PFLOP/s, for 512
// shared keys, 388 us, 1.23 PFLOP/s, for 1560 own ones; 4096 rows on 8191 keys in cut items: 150 us, 1.37). With
// tokens on long states the bytes of K and V (64 requests, 4 kv heads of 128, 32 to 4096 keys, 92 MB:
// 28.3 us, half of it at the rate of a copy). What is left beside them: 4 to 5 us from launch to the first
// scores, some 3000 clocks at an item's end until the next one's scores are looked at (tried without gain:
// rows stored in 128-byte pieces, or through shared memory and TMA with a ring of two K tiles; slower, as
// longer code: rows that leave TMEM only before the next item's P), and the joining of cut items.
#include <cudaTypedefs.h>

#include <cfloat>

#include "kernels.h"

namespace {

constexpr int TB = 128;              // rows of a query tile, keys of a key tile
constexpr int SUB = TB * 64 * 2;     // 128 rows x 64 bf16: one swizzle width
constexpr int THREADS = 384;
constexpr uint32_t TMEM_COLS = 512;  // S|P of A [0,128), of B [128,256), O of A [256, ..), of B [384, ..)
constexpr uint32_t O_COL = 256;
constexpr int SEGS = 4;              // ring of segments: the current one and those ahead
constexpr int TAIL = 768;            // bytes of barriers and masks
constexpr int FOLD = 128;            // key tiles of one accumulator in long states (see fold)
constexpr int MASKS = 8;             // ring of key tiles' masks (> V slots + 2: see the mask warp)

template <int D>
struct Shape {
  static constexpr int SUBS = D / 64, TILE = SUBS * SUB;  // bytes of a Q, K or V tile
  static constexpr int KS = D == 128 ? 3 : 6, VS = D == 128 ? 2 : 5;  // ring slots (KS >= VS)
  static constexpr int RING = (2 + KS + VS) * TILE;
  static constexpr int SMEM = RING + TAIL;
  static_assert(KS >= VS && MASKS > VS + 2, "rings");
};

// floats of a warp's part: rows, (m, l)
__host__ __device__ constexpr int part_floats(int D) { return 32 * D + 64; }

struct Params {
  const int32_t *q_off, *kv_off, *kv_of;
  const uint8_t* valid;
  int seqs, states, q_rows, kv_rows, kv_heads, group, rq;
  bool dual;       // two kv heads side by side where a sequence has one query tile
  bf16* O;
  int64_t ldo;
  float scale_log2;
  float* ws;       // parts of cut items (null: whole items only): two slots a CTA
  float* sums;     // of long states (see fold): a slot a CTA
  int* counters;   // [gridDim.x][8], zero between launches
  int* err;
};

__device__ __forceinline__ float fmax3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
      "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
      "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
      "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, uint64_t* bar, int x,
                                            int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
      : "memory");
}

// mbar_wait for roles that are ahead of the others and in no hurry: they leave the issue slots alone
// between two looks.
__device__ __forceinline__ bool mbar_wait_idle(uint64_t* bar, uint32_t parity, int* err) {
  const uint32_t a = smem_u32(bar);
  if (mbar_try(a, parity)) return true;
  const uint64_t t0 = fb_globaltimer();
  for (uint32_t i = 1;; ++i) {
    __nanosleep(200);
    if (mbar_try(a, parity)) return true;
    if ((i & 7u) == 0) {
      if (*(volatile int*)err != 0) return false;
      if (fb_globaltimer() - t0 > fb_wait_limit()) {
        fb_report(err, FB_DEVERR_WAIT_TIMEOUT);
        return false;
      }
    }
  }
}

// ---- the work of a launch ---------------------------------------------------------------
typedef unsigned long long u64;
typedef uint32_t u32;

struct Seq {
  int q0, nq, k0, nk;
};
// Sequence s. Where the arrays hold something that they must not, that is reported and the sequence
// is taken to be empty.
__device__ __forceinline__ void load_seq(const Params& p, int s, Seq& q) {
  const int u = p.kv_of ? p.kv_of[s] : s;
  q.q0 = p.q_off[s];
  q.nq = p.q_off[s + 1] - q.q0;
  q.k0 = q.nk = 0;
  bool ok = q.q0 >= 0 && q.nq >= 0 && q.nq <= p.q_rows - q.q0 && (s || q.q0 == 0) && u >= 0 && u < p.states;
  if (ok) {
    q.k0 = p.kv_off[u];
    q.nk = p.kv_off[u + 1] - q.k0;
    ok = q.k0 >= 0 && q.nk >= 0 && q.nk <= p.kv_rows - q.k0 && (u || q.k0 == 0);
  }
  if (!ok) {
    fb_report(p.err, FB_DEVERR_BAD_INDEX);
    q = Seq{0, 0, 0, 0};
  }
}
// The items of a sequence: `heads` times `tiles` in pairs (the last one may be single). With several
// query tiles: its kv heads, and the query tiles, a pair of which shares each tile of K and V. With one
// (`dual`): once, and the kv heads, two of which run side by side on their own tiles of K and V.
// Costs are in quarters of what a key tile takes for two query tiles (1.2 us): 3 for one query tile, 5
// for two kv heads, 4 for an item's start and end. Items stand in a row, sequence by sequence; a
// position u in the row is a sum of costs.
struct Cost {
  int heads, tiles, n_kv;
  bool dual;
  u32 w, pair, single, head;  // a key tile of a pair; an item of a pair, of one, all of a head
  __device__ __forceinline__ Cost(const Params& p, const Seq& q) {
    tiles = (q.nq + p.rq - 1) / p.rq;
    dual = p.dual && tiles == 1 && p.kv_heads > 1;
    heads = dual ? 1 : p.kv_heads;
    if (dual) tiles = p.kv_heads;
    n_kv = (q.nk + TB - 1) / TB;
    w = dual ? 5 : 4;
    pair = w * n_kv + 4;
    single = 3u * n_kv + 4;
    head = (u32)(tiles / 2) * pair + (tiles & 1 ? single : 0);
  }
  __device__ __forceinline__ u32 all() const { return head * heads; }
  __device__ __forceinline__ u32 items() const { return (u32)((tiles + 1) / 2) * heads; }
  __device__ __forceinline__ bool two(int t) const { return 2 * t + 1 < tiles; }
  __device__ __forceinline__ u32 weight(int t) const { return two(t) ? w : 3; }
};
// Whole items are handed out as CTAs become free (a counter; what an item gives does not depend on
// who works on it), in the row's order, so that the CTAs work on neighbours, which share K and V
// in L2. Where that would leave CTAs idle, each takes an equal stretch of the row instead, whose
// ends may lie between an item's key tiles: each CTA of a cut item leaves its part in the scratch,
// and the one that comes last adds them up in CTA order.
struct Plan {
  bool cut;
  u32 units, ctas;  // all costs, the CTAs that work on cut items
  // cut: where this CTA's stretch begins (an item's sequence, head (behind the last: go on to the next
  // sequence), pair, position and the key tile in it) and ends
  int s, h, t, j;
  u32 u, end;
  Seq q;
};
// Where CTA c's stretch begins: floor(c units / ctas).
__device__ __forceinline__ u32 stretch_at(u32 c, u32 units, u32 ctas) {
  const u32 q = units / ctas;
  return q * c + (units - q * ctas) * c / ctas;
}
// The CTAs lo .. hi that hold parts of a cut item of n_kv key tiles at u0, each costing w: a CTA's
// beginning is moved to the item's where it lies before its third key tile, to its end where it
// lies in the last one (see begin_at).
__device__ __forceinline__ void holders(const Plan& pl, u32 u0, int n_kv, u32 w, int& lo, int& hi) {
  const u32 most = pl.units / pl.ctas + 1;
  auto from = [&](u32 y) {  // the first CTA that begins at y or behind
    u32 c = y / most;
    while (stretch_at(c, pl.units, pl.ctas) < y) ++c;
    return (int)c;
  };
  lo = from(u0 + 4 + 2 * w) - 1;
  hi = from(u0 + 4 + (u32)(n_kv - 1) * w) - 1;
}
// Position x within a sequence, which begins at u_s, moved to where a stretch may begin: key tile j
// of the item that x lies in, or the next item. Returns the position of that.
__device__ __forceinline__ u32 begin_at(const Cost& c, u32 u_s, u32 x, int& h, int& t, u32& u, int& j) {
  u32 v = x - u_s;
  h = (int)(v / c.head);
  v -= h * c.head;
  t = (int)(v / c.pair);
  if (t > c.tiles / 2) t = c.tiles / 2;
  v -= t * c.pair;  // within the item
  const u32 w = c.weight(t);
  u = x - v;
  j = v < 4 ? 0 : (int)((v - 4) / w);
  if (c.n_kv - j < 2 && v >= 4) {
    j = 0;
    u += c.two(t) ? c.pair : c.single;
    if (2 * ++t >= c.tiles) {
      t = 0;
      ++h;
    }
  }
  if (j < 2) j = 0;
  return j ? u + 4 + j * w : u;
}

// Adds up the sequences' costs and decides how the items are handed out; the thread whose sequence
// a stretch begins in writes where. TEAM: the threads that work on it, one warp (at most 32
// sequences, whose own each lane has at hand) or the whole block (which has to synchronise after it).
template <int TEAM>
__device__ __forceinline__ void make_plan(const Params& p, Seq q, Plan* plan, uint3* scan, int tid) {
  const int lane = tid % 32;
  const int per = (p.seqs + TEAM - 1) / TEAM, s0 = tid * per, s1 = s0 + per < p.seqs ? s0 + per : p.seqs;
  u32 sum = 0, big = 0, n = 0;
  for (int s = s0; s < s1; ++s) {
    if (TEAM > 32) load_seq(p, s, q);
    const Cost c(p, q);
    sum += c.all();
    n += c.items();
    const u32 most = c.tiles > 1 ? c.pair : c.tiles ? c.single : 0;
    big = most > big ? most : big;
  }
  u32 at = sum;  // of the lanes up to this one, then where this thread's first sequence begins
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u32 v = __shfl_up_sync(0xffffffffu, at, o);
    if (lane >= o) at += v;
  }
  u32 total = __shfl_sync(0xffffffffu, at, 31);
  at -= sum;
  big = __reduce_max_sync(0xffffffffu, big);
  n = __reduce_add_sync(0xffffffffu, n);
  if (TEAM > 32) {
    if (lane == 0) scan[tid / 32] = make_uint3(total, big, n);
    __syncthreads();
    total = big = n = 0;
#pragma unroll
    for (int w = 0; w < TEAM / 32; ++w) {
      const uint3 v = scan[w];
      if (w < tid / 32) at += v.x;
      total += v.x;
      big = v.y > big ? v.y : big;
      n += v.z;
    }
  }
  // Cut items: at least three key tiles a CTA, and storing and adding up the parts takes about as
  // long as three key tiles and another one a part.
  const u32 G = gridDim.x, mean = total / G, rounds = (n + G - 1) / G;
  const u32 t_whole = n <= G ? big : rounds <= (mean + big) / big ? rounds * big : mean + big;
  u32 ctas = total / 12 < G ? total / 12 : G;
  if (ctas < 1) ctas = 1;
  const u32 share = total / ctas;
  const u32 t_cut = share + share / 20 + 12 + 4 * (big / (share + 1) + 1);
  const bool cut = total > 0 && t_cut < t_whole - t_whole / 50;
  const u32 c = blockIdx.x;
  const bool work = total > 0 && c < ctas;
  if (tid == 0) {
    plan->cut = cut;
    plan->units = total;
    plan->ctas = ctas;
    if (cut && (!work || c + 1 == ctas)) plan->end = work ? total : 0;
    if (!work) plan->u = 0;
  }
  for (u32 e = 0; work && cut && e < 2; ++e) {  // this CTA's stretch, and the next one's
    const u32 x = stretch_at(c + e, total, ctas);
    if (x < at || x - at >= sum) continue;
    int s = s0, h, t, j;
    u32 u_s = at, u;
    if (per > 1) {
      for (;; ++s) {
        load_seq(p, s, q);
        const u32 all = Cost(p, q).all();
        if (x - u_s < all) break;
        u_s += all;
      }
    }
    const u32 y = begin_at(Cost(p, q), u_s, x, h, t, u, j);
    if (e) {
      plan->end = y;
    } else {
      plan->s = s;
      plan->h = h;
      plan->t = t;
      plan->j = j;
      plan->u = u;
      plan->q = q;
    }
  }
}

// A CTA's segments, one after the other: what the roles read of each, through a ring in shared
// memory.
struct __align__(16) Seg {
  int steps, ng;     // key tiles (-1: no further segment), query tiles
  int row, left;     // first query row, queries from there to the sequence's end
  int key, keys;     // first key, keys from there to the states' end
  int h, last;       // kv head; whether the states end with this segment
  int whole, lo, hi; // a whole item, or a part of one that CTAs lo .. hi share
  int dual;          // two kv heads, h and h + 1, of one query tile
};
// Key tiles j0 .. j1 - 1 of item (h, t) at u
__device__ __forceinline__ void fill(const Params& p, const Plan& pl, const Seq& q, const Cost& c, int h, int t,
                                     int j0, int j1, u32 u, Seg& g) {
  const int first = c.dual ? 0 : 2 * t * p.rq;  // query
  g.steps = j1 - j0;
  g.ng = c.two(t) ? 2 : 1;
  g.dual = c.dual && c.two(t);
  g.h = c.dual ? 2 * t : h;
  g.row = q.q0 + first;
  g.left = q.nq - first;
  g.key = q.k0 + j0 * TB;
  g.keys = q.nk - j0 * TB;
  g.last = j1 == c.n_kv;
  g.whole = j0 == 0 && g.last;
  g.lo = g.hi = 0;
  if (!g.whole) holders(pl, u, c.n_kv, c.weight(t), g.lo, g.hi);
}
// The segments of a CTA's stretch.
struct Stretch {
  int s, h, t, j;
  u32 u, end;
  Seq q;
  __device__ __forceinline__ explicit Stretch(const Plan& pl)
      : s(pl.s), h(pl.h), t(pl.t), j(pl.j), u(pl.u), end(pl.end), q(pl.q) {}
  __device__ __forceinline__ bool next(const Params& p, const Plan& pl, Seg& g) {
    if (u >= end) return false;
    Cost c(p, q);
    if (h >= c.heads) {  // the next sequence with queries (there is one: u < end)
      h = 0;
      do load_seq(p, ++s, q);
      while (q.nq == 0);
      c = Cost(p, q);
    }
    const u32 cost = c.two(t) ? c.pair : c.single;
    fill(p, pl, q, c, h, t, j, end - u < cost ? (int)((end - u - 4) / c.weight(t)) : c.n_kv, u, g);
    j = 0;
    u += cost;
    if (2 * ++t >= c.tiles) {
      t = 0;
      ++h;
    }
    return true;
  }
};
// Whole items by their number (a warp). Numbers only rise: 32 sequences at a time, one a lane.
struct Items {
  int s0 = -32;       // the sequences at hand
  u32 end = 0;        // first item behind them
  Seq q;              // this lane's sequence (at first, one of the first 32), and its first item
  u32 first = 0;
  __device__ __forceinline__ explicit Items(const Seq& q_) : q(q_) {}
  __device__ __forceinline__ bool find(const Params& p, const Plan& pl, u32 i, int lane, Seg& g) {
    while (i >= end) {
      if (s0 + 32 >= p.seqs) return false;
      s0 += 32;
      const int s = s0 + lane;
      u32 n = 0;
      if (s < p.seqs) {
        if (s0 > 0) load_seq(p, s, q);
        n = Cost(p, q).items();
      }
      u32 upto = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u32 v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
      }
      first = end + upto - n;
      end += __shfl_sync(0xffffffffu, upto, 31);
    }
    // the last sequence that begins at i or before (ones without items begin where the next does)
    const int of = 31 - __clz(__ballot_sync(0xffffffffu, first <= i && s0 + lane < p.seqs));
    Seq o;
    o.q0 = __shfl_sync(0xffffffffu, q.q0, of);
    o.nq = __shfl_sync(0xffffffffu, q.nq, of);
    o.k0 = __shfl_sync(0xffffffffu, q.k0, of);
    o.nk = __shfl_sync(0xffffffffu, q.nk, of);
    const Cost c(p, o);
    const u32 k = i - __shfl_sync(0xffffffffu, first, of), per = (u32)(c.tiles + 1) / 2;
    const int h = (int)(k / per), t = (int)(k - h * per);
    fill(p, pl, o, c, h, t, 0, c.n_kv, 0, g);
    return true;
  }
};

// ---- one row's results ------------------------------------------------------------------
// 32 columns of a row, scaled and rounded, in 32-byte stores where the rows allow it.
__device__ __forceinline__ void store32(bf16* to, bool st32, const uint32_t* u, float inv) {
  uint32_t w[16];
#pragma unroll
  for (int i = 0; i < 16; ++i)
    w[i] = pack_bf16x2(__uint_as_float(u[2 * i]) * inv, __uint_as_float(u[2 * i + 1]) * inv);
  if (st32) {
#pragma unroll
    for (int q = 0; q < 2; ++q) store_b32x8(to + q * 16, w + q * 8);
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      reinterpret_cast<uint4*>(to)[q] = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
  }
}

// Where CTA c leaves warp ww's part of an item that CTAs lo .. share: its O rows, [4-column group]
// [row][4], then (maximum, sum) of each row. A CTA holds two parts at most, and only of an item
// that begins with it one that is not its stretch's first.
template <int D>
__device__ __forceinline__ float* part_of(const Params& p, int lo, int c, int ww) {
  return p.ws + ((size_t)(c == lo ? 2 * c + 1 : 2 * c) * 8 + ww) * part_floats(D);
}
// Adds up the parts of CTAs lo .. hi for a warp's `live` rows, in CTA order, and stores them. out:
// this lane's row.
template <int D>
__device__ __forceinline__ void join(const Params& p, int lo, int hi, int ww, int lane, int live, bf16* out) {
  float m = -FLT_MAX, l = 0.f;  // of this lane's row, eight parts at a time
#pragma unroll 1
  for (int c0 = lo; c0 <= hi; c0 += 8) {
    float2 ml[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      ml[i] = c0 + i <= hi
                  ? __ldcg(reinterpret_cast<const float2*>(part_of<D>(p, lo, c0 + i, ww) + 32 * D) + lane)
                  : make_float2(-FLT_MAX, 0.f);
    float top = m;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, ml[i].x);
    l *= ex2(m - top);
    m = top;
#pragma unroll
    for (int i = 0; i < 8; ++i) l += ml[i].y * ex2(ml[i].x - m);
  }
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
  if (live > 8) {  // a lane its row, 32 columns at a time
    const bool st32 = ((reinterpret_cast<uintptr_t>(p.O) & 31) | (p.ldo & 15)) == 0;
#pragma unroll 1
    for (int k = 0; k < D / 32; ++k) {
      float acc[32] = {};
#pragma unroll 2
      for (int c = lo; c <= hi; ++c) {
        const float* from = part_of<D>(p, lo, c, ww);
        const float f = ex2(__ldcg(from + 32 * D + 2 * lane) - m);
        float4 v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __ldcg(reinterpret_cast<const float4*>(from) + (k * 8 + e) * 32 + lane);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          acc[4 * e] += f * v[e].x;
          acc[4 * e + 1] += f * v[e].y;
          acc[4 * e + 2] += f * v[e].z;
          acc[4 * e + 3] += f * v[e].w;
        }
      }
      uint32_t u[32];
#pragma unroll
      for (int e = 0; e < 32; ++e) u[e] = __float_as_uint(acc[e]);
      if (lane < live) store32(out + k * 32, st32, u, inv);
    }
    return;
  }
  // few rows: a lane four columns (D 64: of every other row); four parts of up to four (eight) rows
  // on their way
  constexpr int GROUPS = D / 4, AT = 32 / GROUPS;
  const int cg = lane % GROUPS, sub = lane / GROUPS;
#pragma unroll 1
  for (int r0 = 0; r0 < live; r0 += 4 * AT) {
    float4 acc[4] = {};
#pragma unroll 1
    for (int c0 = lo; c0 <= hi; c0 += 4) {
      float f[4];
      float4 v[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool in = c0 + i <= hi;
        const float* from = part_of<D>(p, lo, in ? c0 + i : hi, ww);
        f[i] = in ? __ldcg(from + 32 * D + 2 * lane) : -INFINITY;  // (of this lane's row)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          v[i][r] = __ldcg(reinterpret_cast<const float4*>(from) + cg * 32 + ((r0 + r * AT + sub) & 31));
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[i] = ex2(f[i] - m);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float fr = __shfl_sync(0xffffffffu, f[i], (r0 + r * AT + sub) & 31);
          if (fr != 0.f) {  // (rows behind the live ones may hold anything)
            acc[r].x += fr * v[i][r].x;
            acc[r].y += fr * v[i][r].y;
            acc[r].z += fr * v[i][r].z;
            acc[r].w += fr * v[i][r].w;
          }
        }
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = (r0 + r * AT + sub) & 31;
      const float ir = __shfl_sync(0xffffffffu, inv, row);
      bf16* to = reinterpret_cast<bf16*>(__shfl_sync(0xffffffffu, reinterpret_cast<u64>(out), row));
      if (r0 + r * AT + sub < live)
        *reinterpret_cast<uint2*>(to + cg * 4) = make_uint2(pack_bf16x2(acc[r].x * ir, acc[r].y * ir),
                                                            pack_bf16x2(acc[r].z * ir, acc[r].w * ir));
    }
  }
}

// The tensor core's sums cut bits off: where all terms have one sign, up to 8e-7 of the result per key tile
// (2^20 keys in one CTA lose 0.5 %, 2^23 5 %). Past FOLD_ROWS keys (4e-4) a warp therefore adds its O rows, with
// their maxima and sums (m, l), to what `sum` holds of the segment every FOLD key tiles, and begins again from
// zero (1e-4 at most, 2^23 keys too). END: what `sum` holds goes back into O and l. A lane's row each; sum lies
// as a part (see part_of). A kernel of its own (LONG), since this code beside the loop costs the others 2 to 3 %
// (32 sequences of 1560 rows on 20 to 512 keys 113.3 us for 110.1).
constexpr int FOLD_ROWS = 512 * TB;
template <int D, bool END>
__device__ __forceinline__ void fold(float* sum, bool first, uint32_t o_taddr, int lane, float m, float& l) {
  float2* ml = reinterpret_cast<float2*>(sum + 32 * D) + lane;
  const float2 was = first ? make_float2(m, 0.f) : *ml;
  const float f = ex2(was.x - m);
#pragma unroll 1
  for (int c = 0; c < D / 32; ++c) {
    uint32_t u[32];
    tmem_ld32(o_taddr + c * 32, u);
    tmem_ld_wait();
    reg_fence32(u);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float4* at = reinterpret_cast<float4*>(sum) + (c * 8 + e) * 32 + lane;
      float4 v = first ? make_float4(0.f, 0.f, 0.f, 0.f) : *at;
      v.x = fmaf(v.x, f, __uint_as_float(u[4 * e]));
      v.y = fmaf(v.y, f, __uint_as_float(u[4 * e + 1]));
      v.z = fmaf(v.z, f, __uint_as_float(u[4 * e + 2]));
      v.w = fmaf(v.w, f, __uint_as_float(u[4 * e + 3]));
      if (!END) *at = v;
      u[4 * e] = END ? __float_as_uint(v.x) : 0u;
      u[4 * e + 1] = END ? __float_as_uint(v.y) : 0u;
      u[4 * e + 2] = END ? __float_as_uint(v.z) : 0u;
      u[4 * e + 3] = END ? __float_as_uint(v.w) : 0u;
    }
    tmem_st32(o_taddr + c * 32, u);
  }
  tmem_st_wait();
  l = fmaf(was.y, f, l);
  if (!END) {
    *ml = make_float2(m, l);
    l = 0.f;
  }
}

// DUAL: p.dual, LONG: more than FOLD_ROWS keys
template <int D, bool MASKED, bool DUAL, bool LONG>
__global__ void __launch_bounds__(THREADS, 1)
    cross_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                 const __grid_constant__ CUtensorMap tmV, const Params p) {
  constexpr int SUBS = Shape<D>::SUBS, TILE = Shape<D>::TILE, KS = Shape<D>::KS, VS = Shape<D>::VS;
  extern __shared__ __align__(1024) uint8_t smem[];
  if ((smem_u32(smem) & 1023u) != 0) {
    if (threadIdx.x == 0) fb_report(p.err, FB_DEVERR_BAD_ARG);
    return;
  }
  uint8_t* Qs = smem;
  uint8_t* Ks = smem + 2 * TILE;
  uint8_t* Vs = Ks + KS * TILE;
  uint64_t* q_full = reinterpret_cast<uint64_t*>(smem + Shape<D>::RING);
  uint64_t* q_empty = q_full + 2;   // [2 query tiles], as q_full
  uint64_t* k_full = q_empty + 2;   // [KS]
  uint64_t* k_empty = k_full + KS;  // [KS]
  uint64_t* v_full = k_empty + KS;  // [VS]: the tile may be used
  uint64_t* v_land = v_full + VS;   // [VS]: a tile that the mask warp has to see first has landed
  uint64_t* m_full = v_land + VS;   // [MASKS]
  uint64_t* g_full = m_full + MASKS;  // [SEGS]
  uint64_t* g_empty = g_full + SEGS;  // [SEGS]
  uint64_t* s_full = g_empty + SEGS;  // [2 groups]
  uint64_t* p_full = s_full + 2;
  uint64_t* o_done = p_full + 2;
  uint64_t* begun = o_done + 2;  // the first K tile and its Q are on their way: one phase, never begun again
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(begun + 1);
  uint4* masks = reinterpret_cast<uint4*>(smem + Shape<D>::RING + TAIL - 16 * MASKS);  // [MASKS]
  static_assert(8 * (4 + 2 * KS + 2 * VS + MASKS + 2 * SEGS + 7) + 8 <= TAIL - 16 * MASKS, "barriers");
  __shared__ Plan plan;
  __shared__ uint3 scan[THREADS / 32];
  __shared__ Seg segs[SEGS], parts[8];

  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  int* err = p.err;
  bool failed = false;

  if (threadIdx.x == 0) {
    for (int s = 0; s < KS; ++s) {
      mbar_init(&k_full[s], 1);
      mbar_init(&k_empty[s], 1);
    }
    for (int s = 0; s < VS; ++s) {
      mbar_init(&v_full[s], 1);
      mbar_init(&v_land[s], 1);
    }
    for (int s = 0; s < MASKS; ++s) mbar_init(&m_full[s], 1);
    for (int s = 0; s < SEGS; ++s) {
      mbar_init(&g_full[s], 1);
      mbar_init(&g_empty[s], 12);  // two TMA lanes, the issuer, the mask warp, eight softmax warps
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&q_full[s], 1);
      mbar_init(&q_empty[s], 1);
      mbar_init(&s_full[s], 1);
      mbar_init(&p_full[s], 4);
      mbar_init(&o_done[s], 1);
    }
    mbar_init(begun, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_desc(&tmQ);
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  if (warp == 1) tmem_alloc(tmem_holder, TMEM_COLS);
  griddep_wait();
  griddep_launch();

  // Where no item can be cut there is nothing to plan; few sequences warp 11 adds up by itself, while
  // the others come to their roles.
  const bool few = p.seqs <= 32;
  Seq own{0, 0, 0, 0};  // of the first 32 sequences, a lane of warp 11 one each
  if (warp == 11 && lane < p.seqs) load_seq(p, lane, own);
  if (p.ws && !few) make_plan<THREADS>(p, Seq{}, &plan, scan, threadIdx.x);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_holder;

  // States that no sequence asks for are checked too (the others by load_seq): 32 a CTA by the mask warp
  // before its first segment, the others, where there are more, when the segments are done.
  auto bad_state = [&](int64_t u) {
    if (u >= p.states) return u == 0 && p.kv_off[0] != 0;
    const int a = p.kv_off[u], b = p.kv_off[u + 1];
    return b < a || b > p.kv_rows || (u == 0 && a != 0);
  };
  auto is_dual = [](const Seg& sg) { return DUAL && sg.dual; };
  uint32_t seg = 0;  // segments that this role has come to
  if (warp == 0) {
    // ---------------- TMA: lane 0 Q and K, lane 1 V ----------------
    if (lane < 2) {
      const uint32_t q_bytes = (uint32_t)(SUBS * 128 * p.group * p.rq);
      // key tiles; phases of the query tiles; which of the last key tiles were of two heads (bits)
      uint32_t t = 0, qph = 0, was_dual = 0;
      for (;; ++seg) {
        if (!mbar_wait(&g_full[seg % SEGS], (seg / SEGS) & 1, err)) { failed = true; break; }
        const Seg sg = segs[seg % SEGS];
        mbar_arrive(&g_empty[seg % SEGS]);
        if (sg.steps < 0) break;
        // (dual: tiles of the two kv heads by turns)
        const int tiles = is_dual(sg) ? 2 * sg.steps : sg.steps;
        if (lane == 0) {
          for (int i = 0; i < tiles; ++i, ++t) {
            const int s = t % KS, h = is_dual(sg) ? sg.h + (i & 1) : sg.h, j = is_dual(sg) ? i >> 1 : i;
            if (!mbar_wait(&k_empty[s], ((t / KS) & 1) ^ 1u, err)) { failed = true; break; }
            mbar_expect_tx(&k_full[s], TILE);
            for (int c = 0; c < SUBS; ++c)
              tma_load_2d(Ks + s * TILE + c * SUB, &tmK, &k_full[s], h * D + c * 64, sg.key + j * TB);
            if (i == 0) {
              for (int g = 0; g < sg.ng; ++g) {
                if (!mbar_wait(&q_empty[g], ((qph >> g) & 1) ^ 1u, err)) { failed = true; break; }
                qph ^= 1u << g;
                mbar_expect_tx(&q_full[g], q_bytes);
                for (int c = 0; c < SUBS; ++c)
                  tma_load_3d(Qs + g * TILE + c * SUB, &tmQ, &q_full[g], c * 64,
                              (is_dual(sg) ? sg.h + g : sg.h) * p.group,
                              is_dual(sg) ? sg.row : sg.row + g * p.rq);
              }
              if (failed) break;
              if (t == 0) mbar_arrive(begun);
            }
          }
        } else {
          for (int i = 0; i < tiles; ++i, ++t) {
            const int s = t % VS, h = is_dual(sg) ? sg.h + (i & 1) : sg.h, j = is_dual(sg) ? i >> 1 : i;
            // Slot s last held tile t - VS; its PV MMAs are done once S MMAs that the issuer issued
            // behind them are, which is when that tile's K slot is released (K and V tiles are counted
            // alike): those of the tile after it, or of the second one after it where either is one
            // head's of two.
            if (t >= VS) {
              const uint32_t a = t - VS + (DUAL && ((was_dual >> (VS - 2)) & 3) ? 2 : 1);
              if (!mbar_wait(&k_empty[a % KS], (a / KS) & 1, err)) { failed = true; break; }
            } else if (t == 0) {
              // The first K and Q come before everything else. (Not by their own barriers: S needs no V,
              // so that their slots may be on the next phase, and the one after it, before this lane looks.)
              if (!mbar_wait(begun, 0, err)) { failed = true; break; }
            }
            was_dual = was_dual << 1 | (uint32_t)is_dual(sg);
            uint64_t* bar = MASKED || (sg.keys - j * TB < TB && sg.keys % 16) ? &v_land[s] : &v_full[s];
            mbar_expect_tx(bar, TILE);
            for (int c = 0; c < SUBS; ++c)
              tma_load_2d(Vs + s * TILE + c * SUB, &tmV, bar, h * D + c * 64, sg.key + j * TB);
          }
        }
        if (failed) break;
      }
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer ----------------
    // Everything that the full tiles' operands depend on is counted under control flow that the
    // compiler sees to be uniform: the segment's bounds only enter votes (see elect_one).
    const uint32_t idesc_s = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(TB >> 4) << 24);  // + N
    const uint32_t idesc_pv = idesc_s | (1u << 16) | ((uint32_t)(D >> 3) << 17);
    const uint32_t q_lo[2] = {desc_lo_k(smem_u32(Qs)), desc_lo_k(smem_u32(Qs + TILE))};
    const uint32_t k_lo = desc_lo_k(smem_u32(Ks)), v_lo = desc_lo_mn(smem_u32(Vs), SUB);
    uint32_t ks = 0, kph = 0, vs = 0, vph = 0;  // the next K and V tiles: slots and phases
    auto next_k = [&] {
      kph ^= ks + 1 == KS;
      ks = ks + 1 == KS ? 0 : ks + 1;
    };
    auto next_v = [&] {
      vph ^= vs + 1 == VS;
      vs = vs + 1 == VS ? 0 : vs + 1;
    };
    uint32_t pph[2] = {0u, 0u}, qph[2] = {0u, 0u};
    bool ok = true;
    // short_: the states' last key tile, of n16 < 8 sixteens of keys
    auto issue_s = [&](int g, uint32_t slot, bool short_, uint32_t n16) {
      const uint32_t ka = k_lo + slot * (TILE >> 4);
      if (!short_) {
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t off = ((kk >> 2) * SUB + (kk & 3) * 32) >> 4;
          tc_mma_ss_lo(tmem + g * TB, q_lo[g] + off, ka + off, DESC_HI, idesc_s | (8u << 18), kk ? 1u : 0u);
        }
      } else {
        const uint32_t idesc = idesc_s | (n16 << 18);
#pragma unroll 1
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t off = ((kk >> 2) * SUB + (kk & 3) * 32) >> 4;
          tc_mma_ss_lo(tmem + g * TB, q_lo[g] + off, ka + off, DESC_HI, idesc, kk ? 1u : 0u);
        }
      }
      tc_commit(&s_full[g]);
    };
    auto issue_pv = [&](int g, uint32_t acc, bool short_, uint32_t n16) {
      const uint32_t va = v_lo + vs * (TILE >> 4);
      if (!short_) {
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
          tc_mma_ts_lo(tmem + O_COL + g * TB, tmem + g * TB + kk * 8, va + kk * (2048 >> 4),
                       DESC_HI, idesc_pv, kk ? 1u : acc);
      } else {
#pragma unroll 1
        for (uint32_t kk = 0; kk < n16; ++kk)
          tc_mma_ts_lo(tmem + O_COL + g * TB, tmem + g * TB + kk * 8, va + kk * (2048 >> 4),
                       DESC_HI, idesc_pv, kk ? 1u : acc);
      }
    };
    // the next segment's steps, sixteens of its last tile, tiles
    int steps = 0;
    uint32_t n16 = 8;
    bool some = false, two = false, dual = false, ends_short = false;
    auto fetch = [&] {
      if (!mbar_wait_warp(&g_full[seg % SEGS], (seg / SEGS) & 1, err)) return false;
      const Seg& sg = segs[seg % SEGS];
      steps = sg.steps;
      n16 = sg.last ? (uint32_t)(sg.keys - (steps - 1) * TB + 15) / 16 : 8u;
      two = __all_sync(0xffffffffu, sg.ng == 2);
      dual = DUAL && __all_sync(0xffffffffu, sg.dual != 0);
      some = __all_sync(0xffffffffu, steps > 0);
      ends_short = __all_sync(0xffffffffu, n16 < 8);
      __syncwarp();
      if (lane == 0) mbar_arrive(&g_empty[seg % SEGS]);
      ++seg;
      return true;
    };
    // S of group g in the next K slot; a group's first of a segment waits for its Q
    auto next_s = [&](int g, bool first, bool short_, uint32_t sixteens) {
      if (!mbar_wait_warp(&k_full[ks], kph, err)) return false;
      if (first) {
        if (!mbar_wait_warp(&q_full[g], qph[g], err)) return false;
        qph[g] ^= 1u;
      }
      tc_fence_after();
      if (elect_one()) issue_s(g, ks, short_, sixteens);
      return true;
    };
    ok = fetch();
    if (ok && some) {
      const bool s_short = __all_sync(0xffffffffu, steps == 1) && ends_short;
      ok = next_s(0, true, s_short, n16);
      if (ok && dual) next_k();
      if (ok && two) ok = next_s(1, true, s_short, n16);
      next_k();
    }
    // A key tile (dual: a tile of either head) at a time: its PV, and S of the one after it, which may
    // be the next segment's first (its Q has been on its way since this segment's last S).
    int left = steps;
    uint32_t x16 = n16;
    bool more = some, x_two = two, x_dual = dual, x_ends_short = ends_short, x_first = true;
    while (ok && more) {
      const bool end = __all_sync(0xffffffffu, left == 1);
      const bool x_short = end && x_ends_short;
      bool y_short = __all_sync(0xffffffffu, left == 2) && x_ends_short;
      if (end) {
        if (!(ok = fetch())) break;
        more = some;
        y_short = __all_sync(0xffffffffu, steps == 1) && ends_short;
      }
      const bool y_two = more && (end ? two : x_two), y_dual = DUAL && more && (end ? dual : x_dual);
      const uint32_t y16 = end ? n16 : x16;
      // this step's V and the next one's K first: they are normally there already, and these
      // waits overlap the tensor pipe's last instructions
      if (!(ok = mbar_wait_warp(&v_full[vs], vph, err))) break;
      if (more && !(ok = mbar_wait_warp(&k_full[ks], kph, err))) break;
      if (!(ok = mbar_wait_warp(&p_full[0], pph[0], err))) break;
      pph[0] ^= 1u;
      tc_fence_after();
      if (!end && !(DUAL && x_dual)) {
        if (elect_one()) {
          issue_pv(0, x_first ? 0u : 1u, false, 8u);
          issue_s(0, ks, y_short, y16);
        }
        if (x_two) {
          if (!(ok = mbar_wait_warp(&p_full[1], pph[1], err))) break;
          pph[1] ^= 1u;
          tc_fence_after();
          if (elect_one()) {
            issue_pv(1, x_first ? 0u : 1u, false, 8u);
            issue_s(1, ks, y_short, y16);
          }
        }
        --left;
        x_first = false;
      } else if (!end) {
        if (elect_one()) {
          issue_pv(0, x_first ? 0u : 1u, false, 8u);
          issue_s(0, ks, y_short, y16);
        }
        next_v();
        next_k();
        if (!(ok = mbar_wait_warp(&v_full[vs], vph, err))) break;
        if (!(ok = mbar_wait_warp(&k_full[ks], kph, err))) break;
        if (!(ok = mbar_wait_warp(&p_full[1], pph[1], err))) break;
        pph[1] ^= 1u;
        tc_fence_after();
        if (elect_one()) {
          issue_pv(1, x_first ? 0u : 1u, false, 8u);
          issue_s(1, ks, y_short, y16);
        }
        --left;
        x_first = false;
      } else {
        if (elect_one()) {
          issue_pv(0, x_first ? 0u : 1u, x_short, x16);
          tc_commit(&o_done[0]);
        }
        // S of a segment with one query tile goes behind both PVs of a pair: the K slot's release
        // stands for the V slots of the tiles before (see the V loads)
        const bool late = x_two && !y_two;
        if (more && !late && !(ok = next_s(0, true, y_short, y16))) break;
        if (x_two) {
          if (DUAL && x_dual) {
            next_v();
            if (!(ok = mbar_wait_warp(&v_full[vs], vph, err))) break;
          }
          if (!(ok = mbar_wait_warp(&p_full[1], pph[1], err))) break;
          pph[1] ^= 1u;
          tc_fence_after();
          if (elect_one()) {
            issue_pv(1, x_first ? 0u : 1u, x_short, x16);
            tc_commit(&o_done[1]);
          }
          if (more && late && !(ok = next_s(0, true, y_short, y16))) break;
        }
        if (y_dual) next_k();
        if (y_two && !(ok = next_s(1, true, y_short, y16))) break;
        left = steps;
        x16 = n16;
        x_two = two;
        x_dual = dual;
        x_ends_short = ends_short;
        x_first = true;
      }
      next_k();
      next_v();
    }
    failed = !ok;
  } else if (warp == 10) {
    // ---------------- masks ----------------
    // The mask of tile T goes into slot T % MASKS once tile T - 1 of V has landed. That tile was
    // loaded after the K slot of tile T - VS had been released, i.e. after the groups had announced
    // P of tile T - VS - 2: its mask, and those before it, have been read.
    uint32_t t = 0;                 // key tiles so far
    uint32_t land = 0;              // bit s: phase of v_land[s]
    if (bad_state(blockIdx.x * 32 + lane)) fb_report(err, FB_DEVERR_BAD_INDEX);
    for (; !failed; ++seg) {
      if (!__all_sync(0xffffffffu, mbar_wait_idle(&g_full[seg % SEGS], (seg / SEGS) & 1, err))) {
        failed = true;
        break;
      }
      const Seg sg = segs[seg % SEGS];
      __syncwarp();
      if (lane == 0) mbar_arrive(&g_empty[seg % SEGS]);
      if (sg.steps < 0) break;
      for (int e = 0; e < (is_dual(sg) ? 2 * sg.steps : sg.steps); ++e, ++t) {
        const int i = is_dual(sg) ? e >> 1 : e;
        const int n = sg.keys - i * TB < TB ? sg.keys - i * TB : TB, slot = t % VS;
        if (!MASKED && (n == TB || n % 16 == 0)) continue;
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int key = q * 32 + lane;
          bool on = key < n;
          if (MASKED) on = on && p.valid[(size_t)sg.key + i * TB + key] != 0;
          w[q] = __ballot_sync(0xffffffffu, on);
        }
        if (MASKED && lane == 0) {
          masks[t % MASKS] = make_uint4(w[0], w[1], w[2], w[3]);
          mbar_arrive(&m_full[t % MASKS]);
        }
        if (!mbar_wait_warp(&v_land[slot], (land >> slot) & 1, err)) { failed = true; break; }
        land ^= 1u << slot;
        const int rows = (n + 15) / 16 * 16;  // that the MMAs read
        constexpr int AT = 32 / (8 * SUBS);   // rows at a time: SUBS pieces of 128 bytes each
        bool wrote = false;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (w[q] == ~0u) continue;
          for (int r = lane / (8 * SUBS); r < 32 && q * 32 + r < rows; r += AT) {
            if ((w[q] >> r) & 1) continue;
            const int piece = lane % (8 * SUBS);
            *reinterpret_cast<uint4*>(Vs + slot * TILE + (piece / 8) * SUB + (q * 32 + r) * 128 +
                                      (piece % 8) * 16) = make_uint4(0, 0, 0, 0);
            wrote = true;
          }
        }
        if (wrote) fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&v_full[slot]);
      }
    }
  } else if (warp == 11) {
    // ---------------- segments ----------------
    if (p.ws && few) make_plan<32>(p, own, &plan, scan, lane);
    __syncwarp();
    Items items(own);
    const bool cut = p.ws && plan.cut;
    Stretch stretch(plan);
    u32 item = blockIdx.x;  // the CTA's first one; the others' numbers come from the counter
    for (bool first = true, more = true; more; first = false) {
      Seg g{};
      if (cut) {
        more = stretch.next(p, plan, g);
      } else {
        if (!first) {
          if (lane == 0) item = gridDim.x + atomicAdd(p.counters, 1);
          item = __shfl_sync(0xffffffffu, item, 0);
        }
        more = items.find(p, plan, item, lane, g);
      }
      if (!more) g.steps = -1;
      if (g.steps == 0) {  // no keys: zeros, written here, and the other roles never hear of it
        const int most = g.dual ? p.rq : g.ng * p.rq, n = g.left < most ? g.left : most;
        const int row = (g.dual ? 2 : 1) * p.group * D / 8;  // 16-byte pieces of a query
        for (int q = 0; q < n; ++q) {
          bf16* out = p.O + (size_t)(g.row + q) * p.ldo + (size_t)g.h * p.group * D;
          for (int i = lane; i < row; i += 32) reinterpret_cast<uint4*>(out)[i] = make_uint4(0, 0, 0, 0);
        }
        continue;
      }
      if (!__all_sync(0xffffffffu, mbar_wait_idle(&g_empty[seg % SEGS], ((seg / SEGS) & 1) ^ 1u, err))) {
        failed = true;
        break;
      }
      if (lane == 0) {
        segs[seg % SEGS] = g;
        mbar_arrive(&g_full[seg % SEGS]);
      }
      __syncwarp();
      ++seg;
    }
    // the last CTA to run out of items puts the counters back
    if (!cut && lane == 0 && atomicAdd(p.counters + 1, 1) == (int)gridDim.x - 1) {
      p.counters[0] = 0;
      p.counters[1] = 0;
    }
  } else {
    // ---------------- softmax: warps 2-5 tile A, 6-9 tile B ----------------
    const int g = (warp - 2) >> 2, quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
    const uint32_t s_col = g * TB, o_col = O_COL + g * TB;
    const bool lead = (warp & 3) == 2 && lane == 0;  // releases K slots and Q (one thread a group)
    const int qi = r / p.group, hi = r - qi * p.group;  // this row's query and head in the tile
    uint32_t cnt = 0, sc = 0, kt = 0;  // segments and S tiles of this group, K tiles of the CTA
    bool due = false;  // this warp has stored its part of `parts`, and not yet said so
    auto out_row = [&](const Seg& sg) {
      return p.O + (size_t)(sg.row + (is_dual(sg) ? 0 : g * p.rq) + qi) * p.ldo +
             (size_t)((is_dual(sg) ? sg.h + g : sg.h) * p.group + hi) * D;
    };
    // rows of this warp that exist in a segment: the tile's queries by the group's heads
    auto live_rows = [&](const Seg& sg) {
      const int left = is_dual(sg) ? sg.left : sg.left - g * p.rq, tile_q = left < p.rq ? left : p.rq;
      const int n = tile_q * p.group - quarter * 32;
      return n < 0 ? 0 : n > 32 ? 32 : n;
    };
    // A part's stores are waited for, and the counter goes up, behind the next segment's last key
    // tile (or at the end): they have long been performed then. The last of the item's CTAs to
    // come here adds the parts up, whoever it is, in CTA order.
    auto say_due = [&] {
      if (!due) return;
      due = false;
      const Seg& sg = parts[warp - 2];
      __threadfence();
      __syncwarp();
      int came = 0;
      int* counter = p.counters + sg.lo * 8 + warp - 2;
      if (lane == 0) came = atomicAdd(counter, 1);
      if (__shfl_sync(0xffffffffu, came, 0) != sg.hi - sg.lo) return;
      __threadfence();
      if (lane == 0) *counter = 0;
      join<D>(p, sg.lo, sg.hi, warp - 2, lane, live_rows(sg), out_row(sg));
    };
    if (!mbar_wait_warp(&g_full[0], 0, err)) failed = true;
    while (!failed) {
      const Seg& sg = segs[seg % SEGS];
      const int steps = sg.steps;
      if (steps < 0) break;
      // the next segment is waited for before this one's rows are stored (its entry is then read
      // without waiting for them), this one's entry given back after that
      auto next_is_there = [&] {
        const uint32_t a = seg + 1;
        return mbar_wait_warp(&g_full[a % SEGS], (a / SEGS) & 1, err);
      };
      auto done_with = [&] {
        __syncwarp();
        if (lane == 0) mbar_arrive(&g_empty[seg % SEGS]);
        ++seg;
      };
      if (g >= sg.ng) {
        kt += steps;
        failed = !next_is_there();
        done_with();
        continue;
      }
      const bool last_group = is_dual(sg) || g == sg.ng - 1;  // (this group's S comes last for a key tile)
      const int live = live_rows(sg), keys = sg.keys;
      const uint32_t kt_step = is_dual(sg) ? 2 : 1;
      if (is_dual(sg)) kt += g;
      // S of this group's next key tile is there; the tile's K slot (and at the last one its Q) is free
      auto scores_ready = [&](bool last) {
        const bool ok = __all_sync(0xffffffffu, mbar_wait(&s_full[g], sc & 1, err));
        if (ok && lead && last_group) mbar_arrive(&k_empty[kt % KS]);
        if (ok && lead && last) mbar_arrive(&q_empty[g]);
        return ok;
      };
      float m_used = -INFINITY, l = 0.f;
      if (live == 0) {  // nothing of this warp's exists: P of its rows may be anything
        for (int i = 0; i < steps; ++i, ++sc, kt += kt_step) {
          if (!scores_ready(i == steps - 1)) { failed = true; break; }
          if (lane == 0) mbar_arrive(&p_full[g]);
        }
      }
      for (int i = live > 0 ? 0 : steps; i < steps; ++i, ++sc, kt += kt_step) {
        if (!scores_ready(i == steps - 1)) { failed = true; break; }
        tc_fence_after();
        if (LONG && i % FOLD == 0 && i > 0)
          fold<D, false>(p.sums + ((size_t)blockIdx.x * 8 + warp - 2) * part_floats(D), i == FOLD, lane_base + o_col,
                         lane, m_used, l);
        const int valid = keys - i * TB;
        const int halves = valid > 64 ? 2 : 1;  // (without a key in the second half its P is not read)
        // the keys that there are, 32 to a word; the other scores become -inf where they are
        const uint32_t* mask = reinterpret_cast<const uint32_t*>(masks + kt % MASKS);
        bool all = valid >= TB;
        if (MASKED) {
          const bool seen = mbar_wait(&m_full[kt % MASKS], (kt / MASKS) & 1, err);
          if (!__all_sync(0xffffffffu, seen)) { failed = true; break; }
          all = (mask[0] & mask[1] & mask[2] & mask[3]) == ~0u;
        }
        if (!all) {
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            const int n = valid - c * 32;
            const uint32_t on = MASKED ? mask[c] : n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
            if (on == ~0u) continue;
            uint32_t u[32];
            tmem_ld32(lane_base + s_col + c * 32, u);
            tmem_ld_wait();
            reg_fence32(u);
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (!((on >> e) & 1)) u[e] = 0xff800000u;
            tmem_st32(lane_base + s_col + c * 32, u);
          }
          tmem_st_wait();
        }
        float top[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) top[k] = -INFINITY;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t u[64];
          tmem_ld32(lane_base + s_col + c * 64, u);
          tmem_ld32(lane_base + s_col + c * 64 + 32, u + 32);
          tmem_ld_wait();
          reg_fence32(u);
          reg_fence32(u + 32);
#pragma unroll
          for (int e = 0; e < 64; e += 16)
#pragma unroll
            for (int k = 0; k < 8; ++k)
              top[k] = fmax3(top[k], __uint_as_float(u[e + k]), __uint_as_float(u[e + 8 + k]));
        }
        // (at least the lowest finite value: a row without a key so far has exponentials of
        // exp2(-inf) = 0 and joins others with a factor of 0)
        const float mx = fmaxf(fmax3(fmax3(top[0], top[1], top[2]), fmax3(top[3], top[4], top[5]), fmaxf(top[6], top[7])) * p.scale_log2, -FLT_MAX);
        if (__all_sync(0xffffffffu, m_used == -INFINITY)) {  // the segment's first tile
          m_used = mx;
        } else if (__any_sync(0xffffffffu, mx > m_used + 8.f && lane < live)) {
          // (Rows that exist vote, and no others: what else lies in the tile, another sequence's queries or
          // what no load wrote, must not show in this one's bits. The warp's rows move together: each for
          // itself moves more often, 158 us for 151 of 4096 rows on 8191 keys.)
          const float m_new = fmaxf(m_used, mx);
          const float alpha = ex2(m_used - m_new);
          m_used = m_new;
          l *= alpha;
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            uint32_t u[32];
            tmem_ld32(lane_base + o_col + c * 32, u);
            tmem_ld_wait();
            reg_fence32(u);
#pragma unroll
            for (int e = 0; e < 32; ++e) u[e] = __float_as_uint(__uint_as_float(u[e]) * alpha);
            tmem_st32(lane_base + o_col + c * 32, u);
          }
        }
        const uint64_t sc2 = f2_join(p.scale_log2, p.scale_log2);
        const uint64_t nm2 = f2_join(-m_used, -m_used);
        uint64_t ls2[2] = {0ull, 0ull};
        // read again, half by half (P of keys 0-63 only overwrites columns 0-31): code for one half, and the
        // first read's registers need not be kept
#pragma unroll 1
        for (int c = 0; c < halves; ++c) {
          float h[64];
          {
            uint32_t u2[64];
            tmem_ld32(lane_base + s_col + c * 64, u2);
            tmem_ld32(lane_base + s_col + c * 64 + 32, u2 + 32);
            tmem_ld_wait();
            reg_fence32(u2);
            reg_fence32(u2 + 32);
#pragma unroll
            for (int e = 0; e < 64; ++e) h[e] = __uint_as_float(u2[e]);
          }
          uint32_t u[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            float t0, t1;
            f2_split(f2_fma(f2_join(h[2 * e], h[2 * e + 1]), sc2, nm2), t0, t1);
            const float e0 = ex2(t0), e1 = ex2(t1);
            ls2[e & 1] = f2_add(ls2[e & 1], f2_join(e0, e1));
            u[e] = pack_bf16x2(e0, e1);
          }
          tmem_st32(lane_base + s_col + c * 32, u);
        }
        {
          float a0, a1;
          f2_split(f2_add(ls2[0], ls2[1]), a0, a1);
          l += a0 + a1;
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[g]);
      }
      if (failed) break;
      if (is_dual(sg)) kt -= g;
      say_due();
      // the segment's rows: PV of its last key tile done
      if (!mbar_wait_warp(&o_done[g], cnt & 1, err)) { failed = true; break; }
      ++cnt;
      tc_fence_after();
      if (!next_is_there()) { failed = true; break; }
      if (live > 0) {
        if (LONG && steps > FOLD)
          fold<D, true>(p.sums + ((size_t)blockIdx.x * 8 + warp - 2) * part_floats(D), false, lane_base + o_col,
                        lane, m_used, l);
        bf16* out = out_row(sg);
        const bool in = lane < live;
        if (sg.whole) {  // (rows without a key, all masked: zeros)
          const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
          const bool st32 = ((reinterpret_cast<uintptr_t>(p.O) & 31) | (p.ldo & 15)) == 0;
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            uint32_t u[32];
            tmem_ld32(lane_base + o_col + c * 32, u);
            tmem_ld_wait();
            reg_fence32(u);
            if (in) store32(out + c * 32, st32, u, inv);
          }
        } else {
          float* part = part_of<D>(p, sg.lo, blockIdx.x, warp - 2);
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            uint32_t u[32];
            tmem_ld32(lane_base + o_col + c * 32, u);
            tmem_ld_wait();
            reg_fence32(u);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              reinterpret_cast<uint4*>(part)[(c * 8 + e) * 32 + lane] =
                  make_uint4(u[4 * e], u[4 * e + 1], u[4 * e + 2], u[4 * e + 3]);
          }
          reinterpret_cast<float2*>(part + 32 * D)[lane] = make_float2(m_used, l);
          if (lane == 0) parts[warp - 2] = sg;
          due = true;
        }
      }
      done_with();
    }
    if (!failed) say_due();
  }

  tc_fence_before();
  if (__syncthreads_or(failed)) {  // a role gave up: loads in flight land before the CTA exits
    const uint64_t t0 = fb_globaltimer();
    while (fb_globaltimer() - t0 < 100000ull) __nanosleep(1000);
  }
  bool bad = false;
#pragma unroll 4
  for (int64_t u = 32ll * gridDim.x + blockIdx.x * THREADS + threadIdx.x; u < p.states; u += (int64_t)gridDim.x * THREADS)
    bad = bad_state(u) || bad;
  if (bad) fb_report(err, FB_DEVERR_BAD_INDEX);
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, TMEM_COLS);
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

// rows of `heads` heads of D: boxes of 64 columns x `box_heads` heads x `box_rows` rows (K and V:
// the heads side by side, two dimensions)
bool map_q(CUtensorMap* m, const CrossArgs& c, int box_heads, int box_rows) {
  auto enc = encoder();
  if (!enc) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.heads, (cuuint64_t)c.q_rows};
  const cuuint64_t strides[2] = {(cuuint64_t)c.head_dim * 2, (cuuint64_t)c.ldq * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows}, es[3] = {1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(c.q), dims, strides, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool map_kv(CUtensorMap* m, const CrossArgs& c, const void* ptr, int64_t ld) {
  auto enc = encoder();
  if (!enc) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)c.kv_heads * c.head_dim, (cuuint64_t)c.kv_rows};
  const cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)TB}, es[2] = {1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(ptr), dims, strides, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int rows_of_tile(const CrossArgs& c) { return TB / (c.heads / c.kv_heads); }
// The most items that the rows can make: a sequence's last pair may be part-filled.
long long most_items(const CrossArgs& c) {
  const int two = 2 * rows_of_tile(c);
  const long long seqs = c.seqs < c.q_rows ? c.seqs : c.q_rows;
  return (c.q_rows / two + seqs) * c.kv_heads;
}
// Whether items may be worth cutting. With eight rounds of them for each CTA they are not, and
// neither are ones that all run side by side and have at most seven key tiles: the least that a cut
// costs is then more than the item (see make_plan). Without a key there is nothing to cut.
bool may_cut(const CrossArgs& c, int num_sms) {
  if (c.kv_rows == 0) return false;
  const long long fewest = (long long)c.q_rows / (2 * rows_of_tile(c)) * c.kv_heads;
  return fewest < 8ll * num_sms && (c.kv_rows > 7 * TB || most_items(c) > num_sms);
}

template <int D, bool MASKED, bool DUAL, bool LONG>
cudaError_t launch(const CrossArgs& c, const Params& p, int grid, cudaStream_t st) {
  CUtensorMap mq, mk, mv;
  const bool no_keys = c.kv_rows == 0;  // (any map: nothing is loaded then)
  if (!map_q(&mq, c, p.group, p.rq)) return cudaErrorInvalidValue;
  if (no_keys)
    mk = mv = mq;
  else if (!map_kv(&mk, c, c.k, c.ldk) || !map_kv(&mv, c, c.v, c.ldv))
    return cudaErrorInvalidValue;
  auto kern = cross_kernel<D, MASKED, DUAL, LONG>;
  const cudaError_t e =
      cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<D>::SMEM);
  if (e != cudaSuccess) return e;
  return launch_k(kern, dim3(grid), dim3(THREADS), Shape<D>::SMEM, st, mq, mk, mv, p);
}

template <int D, bool MASKED>
cudaError_t choose(const CrossArgs& c, const Params& p, int grid, cudaStream_t st) {
  if (c.kv_rows > FOLD_ROWS)
    return p.dual ? launch<D, MASKED, true, true>(c, p, grid, st) : launch<D, MASKED, false, true>(c, p, grid, st);
  return p.dual ? launch<D, MASKED, true, false>(c, p, grid, st) : launch<D, MASKED, false, false>(c, p, grid, st);
}

}  // namespace

cudaError_t cross_set_wait_limit(unsigned long long ns) { return fb_set_wait_limit_tu(ns); }

size_t cross_ws_bytes(const CrossArgs& c, int num_sms) {
  const size_t slot = (size_t)num_sms * 8 * part_floats(c.head_dim) * sizeof(float);
  return (may_cut(c, num_sms) ? 2 * slot : 0) + (c.kv_rows > FOLD_ROWS ? slot : 0);
}

cudaError_t cross_attention(const CrossArgs& c, void* ws, int* counters, int* err, int num_sms,
                            cudaStream_t st) {
  Params p;
  p.q_off = c.q_offsets;
  p.kv_off = c.kv_offsets;
  p.kv_of = c.kv_of;
  p.valid = c.valid;
  p.seqs = c.seqs;
  p.states = c.states;
  p.q_rows = c.q_rows;
  p.kv_rows = c.kv_rows;
  p.kv_heads = c.kv_heads;
  p.group = c.heads / c.kv_heads;
  p.rq = rows_of_tile(c);
  p.O = (bf16*)c.out;
  p.ldo = c.ldo;
  p.scale_log2 = c.scale * 1.4426950408889634f;
  // Two kv heads side by side keep twice as much of K and V on its way (64 tokens of 4 kv heads on 32 to
  // 4096 keys: 28.3 us for 30.9), but a step of both takes 3500 clocks for one's 2600: only where there are
  // more heads of sequences than SMs (as pairs they may be fewer). With longer sequences the items have two query tiles for the most part, and
  // the kernel without that took 149 us for 161 (32 of 1560 rows on 512 keys).
  const long long seqs = c.seqs < c.q_rows ? c.seqs : c.q_rows;
  p.dual = seqs * c.kv_heads > num_sms && c.q_rows <= seqs * p.rq;
  const long long tiles = (c.kv_rows + TB - 1) / TB;
  // (costs are counted in 32 bits)
  const bool room = may_cut(c, num_sms), cut = room && most_items(c) * (4.0 * tiles + 4) < 4e9;
  p.ws = cut ? (float*)ws : nullptr;
  p.sums = (float*)ws + (room ? (size_t)2 * num_sms * 8 * part_floats(c.head_dim) : 0);
  p.counters = counters;
  p.err = err;
  long long units = most_items(c);
  if (cut) units *= tiles;
  const int grid = (int)(units < num_sms ? units : num_sms);
  if (c.head_dim == 128)
    return c.valid ? choose<128, true>(c, p, grid, st) : choose<128, false>(c, p, grid, st);
  return c.valid ? choose<64, true>(c, p, grid, st) : choose<64, false>(c, p, grid, st);
}
