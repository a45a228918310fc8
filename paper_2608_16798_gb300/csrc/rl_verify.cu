// Verification of drafted tokens against the target's probabilities, from given random numbers.
//
// Sequence b has K_b drafted tokens x_0 .. and K_b + 1 target rows z_0 .., each with
// p = softmax(z / T); the drafts' own rows give q = softmax(zd / T), or q is 1 at x (no draft rows).
// Token j is accepted while u_j q(x_j) < p(x_j). At the first refusal the token drawn from
// max(p - q, 0) ends the sequence; with no refusal one more is drawn from the last row's p. A draw is
// the lowest v at which the running sum of its weights passes s_b times their total. T = 0: greedy,
// the row's first largest entry is both the test and the draw.
//
// Rows are worked on in the order of their place j in their sequences: by the time a late row starts
// its sequence has often been refused earlier, and it is skipped. Nothing waits for another row: the
// last of a sequence's rows to finish writes the sequence's result. Where there are rows for all SMs, a
// CTA takes a row (row_kernel, below); else one thread-block cluster does (verify_kernel):
//
// Every warp of the cluster owns one segment of the vocabulary. It brings the segment of both rows
// into its own shared memory by bulk copies (one barrier each, so a warp starts when its own data is
// there), folds them into (max, sum of exponentials) pairs, and writes these to a table in every CTA of
// the cluster. After one cluster barrier the first warp of each CTA merges the table: both rows'
// normalisers, the decision, and, for a draw from p alone, the segment that holds the token. A draw from
// max(p - q, 0) takes a second pass over the segments, still in shared memory, and a second exchange.
// The warp whose segment holds the token finds it by a scan. HBM is read once.
//
// Measured: one sequence of 4 drafts on bf16 rows of 304 KB (5 target and 4 draft rows, 80 CTAs) 11-13.4 us a call with
// host and launch, 8 sequences of 1 to 5 drafts on rows of 8 KB 12.7-16.8. What bounds it is the chain of a row (offsets,
// copy, folds, exchange, draw, result), each step a trip to L2 or to the other CTAs, and the fetch of its code from a
// cold L2; with 80 CTAs 7 of the 16.7 us that the profiler gives are the SMs' own.
#include <algorithm>
#include <cmath>
#include <map>
#include <mutex>
#include <utility>

#include "rl_device.cuh"
#include "rl_host.h"
#include "rl_segment.cuh"

namespace rl {
namespace verify {

using namespace seg;

constexpr int kWarps = 8;
constexpr int kMaxCluster = 16;
constexpr int kMaxSeg = kWarps * kMaxCluster;
// A refusal at place j is kept as kFirst - j, the earliest is the largest, with two bits below it: what was wrong
// with the row. They are reported with the sequence's result, and so not for rows behind its end, which may or may
// not have been looked at.
constexpr int kFirst = 1 << 28;
constexpr int kNoToken = 1, kNoNumbers = 2;
__device__ __forceinline__ int refusal(int j, int wrong) { return ((kFirst - j) << 2) | wrong; }
__device__ __forceinline__ int place_of(int f) { return kFirst - (f >> 2); }

struct Args {
  const void* target;
  const void* draft;       // or null
  int64_t ld_t, ld_d;
  int32_t V, n_seq, max_draft;
  int64_t n_draft;
  const int32_t* draft_ids;
  const int32_t* offsets;  // [n_seq + 1]
  const float* accept_u;
  const float* sample_u;
  float c;                 // log2(e) / T (greedy: log2(e))
  int32_t seg;             // elements of a segment
  int32_t seg_bytes;       // its shared memory per row
  int32_t held;            // rows held at once: 2 with draft rows
  int32_t check_from;      // first cluster that asks whether its sequence has been refused
  int32_t* out_ids;
  float* out_logp;
  int32_t* n_accepted;
  uint32_t* finished;      // [n_seq] rows that have finished
  int32_t* refused;        // [n_seq] the earliest refusal so far, 0: none
  int32_t* status;
};

// One entry per segment, the same table in every CTA of the cluster.
struct Table {
  Fold t[kMaxSeg];      // target
  Fold d[kMaxSeg];      // draft
  float r[kMaxSeg];     // weight of the segment in a draw from max(p - q, 0)
  int32_t arg[kMaxSeg]; // greedy: first largest entry
};

// What the first warp of a CTA finds for the others.
struct Decision {
  Fold t, d;     // both rows
  float left;    // of the draw: what is left to pass within the segment `at`
  int32_t at;    // -1: no segment has any weight
  int32_t over;  // nothing left to do: accepted, greedy, or no numbers
};

// Two rows' at once: their chains of reductions overlap.
__device__ __forceinline__ void merged2(const Fold* f, const Fold* g, int n, float c, int lane, Fold& rf, Fold& rg) {
  float mf = minus_inf(), mg = mf;
  for (int k = lane; k < n; k += 32) {
    mf = fmaxf(mf, f[k].m);
    mg = fmaxf(mg, g[k].m);
  }
  const float M = redux_max(mf), G = redux_max(mg);
  float sf = 0.f, sg = 0.f;
  for (int k = lane; k < n; k += 32) {
    sf += f[k].s == 0.f ? 0.f : f[k].s * power(f[k].m, M, c);
    sg += g[k].s == 0.f ? 0.f : g[k].s * power(g[k].m, G, c);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    sf += __shfl_xor_sync(0xffffffffu, sf, o);
    sg += __shfl_xor_sync(0xffffffffu, sg, o);
  }
  rf = Fold{M, sf};
  rg = Fold{G, sg};
}

// Whether the drafted token is accepted: u q < p with p and q from its entries in both rows (q = 1 without one).
__device__ __forceinline__ bool accepts(float u, float zt, const Fold& t, float zd, const Fold& d, bool two, float c) {
  const float px = ex2(exponent(zt, t.m, c)) / t.s;
  const float qx = two ? ex2(exponent(zd, d.m, c)) / d.s : 1.f;
  return u * qx < px;
}

__device__ __forceinline__ void report(const Args& p, int wrong) {
  if (wrong) flag_status(p.status, (wrong & kNoToken ? RL_DEV_BAD_TOKEN : 0) | (wrong & kNoNumbers ? RL_DEV_BAD_VALUE : 0));
}

// A row is finished (its result written, if it has one): the last of its sequence writes what the
// sequence comes to and leaves the sequence's words at zero. By one thread.
__device__ __forceinline__ void finish(const Args& p, int b, int o, int K) {
  if (p.max_draft == 0) {  // sequences of one row
    p.n_accepted[b] = 0;
    return;
  }
  __threadfence();
  if (atomicAdd(p.finished + b, 1u) != static_cast<uint32_t>(K)) return;
  __threadfence();
  const int f = atomicExch(p.refused + b, 0);
  p.finished[b] = 0;
  const int n = f ? place_of(f) : K;
  report(p, f & 3);
  p.n_accepted[b] = n;
  for (int j = n + 1; j <= K; ++j) {
    p.out_ids[o + b + j] = -1;
    p.out_logp[o + b + j] = 0.f;
  }
}

template <typename T, bool GREEDY>
__global__ void __launch_bounds__(kWarps * 32) verify_kernel(const Args p) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(8) uint64_t bars[kWarps][2];
  __shared__ __align__(16) Table tab;
  __shared__ int32_t skip;
  __shared__ Decision dec;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank(), C = cluster_nctarank();
  const int id = blockIdx.x / C, j = id / p.n_seq, b = id % p.n_seq;
  const int n_seg = static_cast<int>(C) * kWarps, g = static_cast<int>(rank) * kWarps + warp;

  const int o = p.offsets[b], o1 = p.offsets[b + 1];
  const int K = o1 - o;
  if (o < 0 || o1 < o || o1 > p.n_draft || K > p.max_draft) {
    if (j == 0 && rank == 0 && threadIdx.x == 0) {
      flag_status(p.status, RL_DEV_BAD_OFFSETS);
      p.n_accepted[b] = -1;
    }
    return;  // the whole cluster
  }
  if (j > K) return;
  // another CTA's shared memory may be written once that CTA has started
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  if (id >= p.check_from) {
    // one lane of one CTA asks and all are told what it saw, so that the cluster decides as one (loads of the
    // same word by several lanes could differ, and a CTA that stays would write to one that has left)
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (rank == 0 && warp == 0) {
      int f = 0;
      if (lane == 0) f = *reinterpret_cast<volatile int32_t*>(p.refused + b);
      f = __shfl_sync(0xffffffffu, f, 0);
      if (lane < C)
        asm volatile("st.shared::cluster.u32 [%0], %1;"
                     :: "r"(map_to_rank(smem_addr(&skip), lane)), "r"(f && place_of(f) < j ? 1 : 0) : "memory");
    }
    __syncwarp();
    cluster_sync_all();
    if (skip) {
      if (rank == 0 && threadIdx.x == 0) finish(p, b, o, K);
      return;
    }
  }
  const int64_t row = static_cast<int64_t>(o) + b + j, drow = static_cast<int64_t>(o) + j;
  const bool tested = j < K, two = tested && !GREEDY && p.draft != nullptr;
  const T* zt = static_cast<const T*>(p.target) + row * p.ld_t;
  const T* zd = two ? static_cast<const T*>(p.draft) + drow * p.ld_d : nullptr;
  const int e0 = min(g * p.seg, p.V), n = min(p.seg, p.V - e0);
  if (lane == 0) {
    mbar_init(&bars[warp][0], 1);
    mbar_init(&bars[warp][1], 1);
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  __syncwarp();
  uint8_t* mine = smem + static_cast<size_t>(warp) * p.held * p.seg_bytes;
  const T* t_end = static_cast<const T*>(p.target) + (p.n_draft + p.n_seq - 1) * p.ld_t + p.V;
  Segment<T> st = fetch(zt, e0, n, t_end, mine, &bars[warp][0], lane), sd{};
  if (two)
    sd = fetch(zd, e0, n, static_cast<const T*>(p.draft) + (p.n_draft - 1) * p.ld_d + p.V, mine + p.seg_bytes,
               &bars[warp][1], lane);
  // the drafted token's own entries, by every thread
  int x = -1;
  float zx = 0.f, zdx = 0.f, ua = 0.f;
  if (tested) {
    x = p.draft_ids[drow];
    ua = p.accept_u[drow];
    if (x < 0 || x >= p.V) {
      x = -1;
    } else {
      zx = Elem<T>::one(zt[x]);
      if (two) zdx = Elem<T>::one(zd[x]);
    }
  }
  const float us = p.sample_u[b];

  // ---- both rows' folds, to every CTA's table
  const float c = p.c;
  bool in_time = mbar_wait_bounded(&bars[warp][0], 0);
  st.blank_edges(lane);
  int arg = 0;
  const Fold ft = fold<T, GREEDY>(st, c, lane, arg);
  Fold fd{minus_inf(), 0.f};
  if (two) {
    in_time = mbar_wait_bounded(&bars[warp][1], 0) && in_time;
    sd.blank_edges(lane);
    int unused = 0;
    fd = fold<T, false>(sd, c, lane, unused);
  }
  if (!in_time && lane == 0) flag_status(p.status, RL_DEV_TIMEOUT);
  __syncwarp();
  if (id < p.check_from) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  if (lane < C) {
    put_f2(map_to_rank(smem_addr(&tab.t[g]), lane), ft.m, ft.s);
    if (two) put_f2(map_to_rank(smem_addr(&tab.d[g]), lane), fd.m, fd.s);
    if (GREEDY) put_f1(map_to_rank(smem_addr(&tab.arg[g]), lane), __int_as_float(arg));
  }
  __syncwarp();
  cluster_sync_all();

  // ---- the decision, by the first warp of every CTA alike
  const Fold* seg_t = tab.t;
  auto weight_p = [seg_t, c](const Fold& ht) {
    return [seg_t, ht, c](int k) { return seg_t[k].s == 0.f ? 0.f : seg_t[k].s * power(seg_t[k].m, ht.m, c); };
  };
  if (warp == 0) {
    Fold ht, hd{0.f, 1.f};
    if (two) merged2(tab.t, tab.d, n_seg, c, lane, ht, hd);
    else ht = merged(tab.t, n_seg, c, lane);
    const bool bad = is_bad(ht) || is_bad(hd);
    int token = -1;  // greedy
    if (GREEDY && !bad) {
      uint32_t best = 0xffffffffu;
      for (int k = lane; k < n_seg; k += 32)
        if (tab.t[k].m == ht.m) best = min(best, static_cast<uint32_t>(k * p.seg + tab.arg[k]));
      token = static_cast<int>(__reduce_min_sync(0xffffffffu, best));
    }
    bool accept = false;
    if (tested && !bad && x >= 0) accept = GREEDY ? x == token : accepts(ua, zx, ht, zdx, hd, two, c);
    const bool over = accept || bad || GREEDY;
    float left = 0.f;
    int at = -1;
    if (!over && !tested) at = pick(n_seg, us, lane, weight_p(ht), left);
    if (lane == 0) {
      dec = Decision{ht, hd, left, at, over};
      const int wrong = (tested && x < 0 ? kNoToken : 0) | (bad ? kNoNumbers : 0);
      if (rank == 0 && over) {
        if (p.max_draft == 0) report(p, wrong);
        else if (!accept) atomicMax(p.refused + b, refusal(j, wrong));
        p.out_ids[row] = accept ? x : token;
        p.out_logp[row] = bad ? __int_as_float(0x7fffffff)
                              : logp_of(accept ? zx : Elem<T>::one(zt[token]), ht, c);
        finish(p, b, o, K);
      }
      // ordered before the sequence's result by the cluster barrier that follows a refusal
      if (rank == 0 && !over && tested) atomicMax(p.refused + b, refusal(j, wrong));
    }
  }
  __syncthreads();
  if (dec.over) return;

  // ---- the draw: from max(p - q, 0) after a refusal, else from p
  const Fold ht = dec.t, hd = dec.d;
  const float it = 1.f / ht.s, id_ = 1.f / hd.s;
  int at = dec.at;
  float left = dec.left;
  bool plain = !tested;
  const int shift = sd.lo - st.lo;
  auto weights_p = [&](int k, float (&w)[Elem<T>::N]) {
    st.load(k, w);
    exps(w, ht.m, c);
  };
  auto weights_r = [&](int k, float (&w)[Elem<T>::N]) {
    constexpr int N = Elem<T>::N;
    weights_p(k, w);
    if (two) {
      float y[N];
      if (shift == 0) {
        sd.load(k, y);
      } else {
        // beyond the segment's ends, where p is zero, this may be any number
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = Elem<T>::one(sd.at[k * N + e + shift]);
      }
      exps(y, hd.m, c);
#pragma unroll
      for (int e = 0; e < N; ++e) w[e] = fmaxf(fmaf(-y[e], id_, w[e] * it), 0.f);
    } else {
      const int i = x - e0 + st.lo - k * N;
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e == i) w[e] = 0.f;
    }
  };
  if (!plain) {
    float2 r = make_float2(0.f, 0.f);
    const int nb = st.blocks();
#pragma unroll 2
    for (int k = lane; k < nb; k += 32) {
      float w[Elem<T>::N];
      weights_r(k, w);
#pragma unroll
      for (int e = 0; e < Elem<T>::N; e += 2) r = add2(r, make_float2(w[e], w[e + 1]));
    }
    const float sum = warp_sum(r.x + r.y);
    if (lane < C) put_f1(map_to_rank(smem_addr(&tab.r[g]), lane), sum);
    __syncwarp();
    cluster_sync_all();
    at = pick(n_seg, us, lane, [&](int k) { return tab.r[k]; }, left);
    plain = at < 0;  // p and q are equal up to rounding
    if (plain) at = pick(n_seg, us, lane, weight_p(ht), left);
  }
  if (at != g) return;
  const int nb = st.blocks();
  const int i = plain ? locate<T>(st.lo, nb, left, lane, weights_p) : locate<T>(st.lo, nb, left, lane, weights_r);
  if (lane == 0) {
    const int token = e0 + max(i, 0);
    p.out_ids[row] = token;
    p.out_logp[row] = logp_of(Elem<T>::one(zt[token]), ht, c);
    finish(p, b, o, K);
  }
}

// ---------------------------------------------------------------- many rows: a CTA takes a row
//
// Plain 16-byte loads, one tile of a warp ahead of the fold; several CTAs per SM hide each other's row
// ends. Nothing of a row is kept: a draw from p reads one tile of the row again (the fold leaves every
// tile's weight in a table), one from p without the drafted token that token's tile too, and a draw from
// max(p - q, 0) both rows (the first pass knows neither normaliser): at most one row of a sequence is read
// twice. What bounds it is HBM with the exponentials
// close behind (16 per clock and SM; at 6.8 TB/s 11.8 bf16 entries arrive in that time). Measured against a
// cluster per row with both rows in shared memory, whose exchanges leave the copies idle half of the time.
// 128 sequences of 4 drafts at V = 151,936 (bf16): 87.5 us, 369 MB read at 4.2 TB/s; 509 draws 36.9 us, 155 MB at
// 4.2 TB/s. The passes run at 5.8-6 TB/s; what is lost is the rows' ends, 7-10K cycles of the 43K of a draw
// (the sums' merge 2.5K, the tile 3.5K, the place in it 3.5K), and the second turn of CTAs.

constexpr int kMaxTiles = 1024;     // of a row

// A row in 16-byte blocks of memory, the first at the block that holds its first element.
template <typename T>
struct Blocks {
  const T* base;
  int lo, hi;  // the row is elements [lo, hi) from there
  __device__ __forceinline__ Blocks(const T* row, int V) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(row);
    base = reinterpret_cast<const T*>(a & ~uintptr_t(15));
    lo = static_cast<int>(row - base);
    hi = lo + V;
  }
  // Block k; what is not the row's is minus infinity.
  __device__ __forceinline__ uint4 load(int k) const {
    constexpr int N = Elem<T>::N;
    if (k * N >= lo && (k + 1) * N <= hi) return __ldg(reinterpret_cast<const uint4*>(base + static_cast<int64_t>(k) * N));
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int i = k * N + e;
      const T x = i >= lo && i < hi ? base[i] : Elem<T>::none();
      if (sizeof(T) == 2) w[e / 2] |= static_cast<uint32_t>(Elem<T>::bits(x)) << (16 * (e & 1));
      else w[e % 4] = Elem<T>::bits(x);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

template <typename T, bool GREEDY, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, 32 / WARPS) row_kernel(const Args p) {
  constexpr int N = Elem<T>::N;
  constexpr int kTile = kTileBlocks * 32 * N;  // elements of a tile
  __shared__ Fold tiles[kMaxTiles];            // a draw's weights by tile: sums, or (in s) max(p - q, 0)
  __shared__ Fold rows[2][WARPS];
  __shared__ int32_t args[WARPS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int j = blockIdx.x / p.n_seq, b = blockIdx.x % p.n_seq;
  const float c = p.c;
  const int o = p.offsets[b], o1 = p.offsets[b + 1];
  const int K = o1 - o;
  if (o < 0 || o1 < o || o1 > p.n_draft || K > p.max_draft) {
    if (j == 0 && threadIdx.x == 0) {
      flag_status(p.status, RL_DEV_BAD_OFFSETS);
      p.n_accepted[b] = -1;
    }
    return;
  }
  if (j > K) return;
  if (j > 0) {
    // one thread asks, so that the CTA decides as one
    int f = 0;
    if (threadIdx.x == 0) f = *reinterpret_cast<volatile int32_t*>(p.refused + b);
    if (__syncthreads_or(f && place_of(f) < j)) {
      if (threadIdx.x == 0) finish(p, b, o, K);
      return;
    }
  }
  const int64_t row = static_cast<int64_t>(o) + b + j, drow = static_cast<int64_t>(o) + j;
  const bool tested = j < K, two = tested && !GREEDY && p.draft != nullptr;
  const T* zt = static_cast<const T*>(p.target) + row * p.ld_t;
  const T* zd = two ? static_cast<const T*>(p.draft) + drow * p.ld_d : zt;
  const Blocks<T> bt(zt, p.V), bd(zd, p.V);
  int x = -1;
  float zx = 0.f, zdx = 0.f, ua = 0.f;
  const float us = p.sample_u[b];
  if (tested) {
    x = p.draft_ids[drow];
    ua = p.accept_u[drow];
    if (x < 0 || x >= p.V) {
      x = -1;
    } else {
      zx = Elem<T>::one(zt[x]);
      if (two) zdx = Elem<T>::one(zd[x]);
    }
  }

  // ---- one pass; the tiles go to the warps in turn
  const int nt = (bt.hi + kTile - 1) / kTile;
  const bool draws = !GREEDY && !two;  // the tiles' weights are of use
  auto pass = [&](const Blocks<T>& bl, int r) {
    const int n = (bl.hi + kTile - 1) / kTile;
    Running run{minus_inf(), {0.f, 0.f}, 0};
    uint4 w[2][kTileBlocks];
    auto load = [&](uint4 (&to)[kTileBlocks], int t) {
      const int k0 = t * kTileBlocks * 32 + lane;
#pragma unroll
      for (int i = 0; i < kTileBlocks; ++i) to[i] = bl.load(k0 + 32 * i);
    };
    auto take = [&](const uint4 (&from)[kTileBlocks], int t) {
      if (draws) run = Running{minus_inf(), {0.f, 0.f}, 0};
      add_tile<T, GREEDY>(run, from, t * kTileBlocks * 32 + lane, c);
      if (draws) {
        const Fold f = of_warp(run, c);
        if (lane == 0) tiles[t] = f;
      }
    };
    int t = warp;
    if (t < n) load(w[0], t);
    while (t < n) {
      load(w[1], t + WARPS);
      take(w[0], t);
      t += WARPS;
      if (t >= n) break;
      load(w[0], t + WARPS);
      take(w[1], t);
      t += WARPS;
    }
    if (draws) return;
    const Fold f = of_warp(run, c);
    if (lane == 0) rows[r][warp] = f;
    if (GREEDY) {
      const uint32_t best = __reduce_min_sync(0xffffffffu, run.m == f.m ? static_cast<uint32_t>(run.arg) : 0xffffffffu);
      if (lane == 0) args[warp] = static_cast<int32_t>(best);
    }
  };
  pass(bt, 0);
  if (two) pass(bd, 1);
  __syncthreads();

  // ---- the decision, by every warp that has work after it
  if (!two && warp != 0) return;
  Fold ht, hd{0.f, 1.f};
  if (two) {
    merged2(rows[0], rows[1], WARPS, c, lane, ht, hd);
  } else if (GREEDY) {
    ht = merged(rows[0], WARPS, c, lane);
  } else {
    // the tiles' weights become relative to the row's largest entry
    float m = minus_inf(), s = 0.f;
    for (int k = lane; k < nt; k += 32) m = fmaxf(m, tiles[k].m);
    const float M = redux_max(m);
    for (int k = lane; k < nt; k += 32) {
      const Fold f = tiles[k];
      const float mine = f.s == 0.f ? 0.f : f.s * power(f.m, M, c);
      tiles[k].s = mine;
      s += mine;
    }
    __syncwarp();  // other lanes read the table in pick, and write to it in weigh
    ht = Fold{M, warp_sum(s)};
  }
  const bool bad = is_bad(ht) || is_bad(hd);
  int token = -1;
  bool accept = false;
  if (GREEDY && !bad) {
    const uint32_t best = lane < WARPS && rows[0][lane].m == ht.m ? static_cast<uint32_t>(args[lane]) : 0xffffffffu;
    token = static_cast<int>(__reduce_min_sync(0xffffffffu, best)) - bt.lo;
  }
  if (tested && !bad && x >= 0) accept = GREEDY ? x == token : accepts(ua, zx, ht, zdx, hd, two, c);
  auto result = [&](int id, float lp, bool refused) {
    const int wrong = (tested && x < 0 ? kNoToken : 0) | (bad ? kNoNumbers : 0);
    if (p.max_draft == 0) report(p, wrong);
    else if (refused) atomicMax(p.refused + b, refusal(j, wrong));
    p.out_ids[row] = id;
    p.out_logp[row] = lp;
    finish(p, b, o, K);
  };
  if (accept || bad || GREEDY) {
    if (threadIdx.x == 0) {
      result(accept ? x : token, bad ? __int_as_float(0x7fffffff) : logp_of(accept ? zx : Elem<T>::one(zt[token]), ht, c),
             !accept);
    }
    return;
  }

  // ---- the draw: from max(p - q, 0) after a refusal, else from p
  const float it = 1.f / ht.s, id_ = 1.f / hd.s;
  const int shift = bd.lo - bt.lo;
  auto weights_p = [&](int k, float (&w)[N]) {
    Elem<T>::unpack(bt.load(k), w);
    exps(w, ht.m, c);
  };
  // max(p - q, 0) from the exponentials of p and the logits of q
  auto residual = [&](float (&w)[N], float (&y)[N]) {
    exps(y, hd.m, c);
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = fmaxf(fmaf(-y[e], id_, w[e] * it), 0.f);
  };
  // from the exponentials of p, of what a refusal draws from
  auto rest_of = [&](int k, float (&w)[N]) {
    if (two) {
      float y[N];
      if (shift == 0) {
        Elem<T>::unpack(bd.load(k), y);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const int i = k * N + e;
          y[e] = i >= bt.lo && i < bt.hi ? Elem<T>::one(bd.base[i + shift]) : minus_inf();
        }
      }
      residual(w, y);
    } else {
      const int i = x + bt.lo - k * N;
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e == i) w[e] = 0.f;
    }
  };
  auto weights_r = [&](int k, float (&w)[N]) {
    weights_p(k, w);
    rest_of(k, w);
  };
  // the weight of tile t, by a warp
  auto weigh = [&](int t, auto weights) {
    float2 r = make_float2(0.f, 0.f);
#pragma unroll 2
    for (int i = 0; i < kTileBlocks; ++i) {
      float w[N];
      weights(t * kTileBlocks * 32 + 32 * i + lane, w);
#pragma unroll
      for (int e = 0; e < N; e += 2) r = add2(r, make_float2(w[e], w[e + 1]));
    }
    const float sum = warp_sum(r.x + r.y);
    if (lane == 0) tiles[t].s = sum;
    __syncwarp();
  };
  if (two && shift == 0) {
    // as weigh, with a tile of both rows in flight
    for (int t = warp; t < nt; t += WARPS) {
      const int k0 = t * kTileBlocks * 32 + lane;
      uint4 w4[kTileBlocks], y4[kTileBlocks];
#pragma unroll
      for (int i = 0; i < kTileBlocks; ++i) w4[i] = bt.load(k0 + 32 * i);
#pragma unroll
      for (int i = 0; i < kTileBlocks; ++i) y4[i] = bd.load(k0 + 32 * i);
      float2 r = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kTileBlocks; ++i) {
        float w[N], y[N];
        Elem<T>::unpack(w4[i], w);
        Elem<T>::unpack(y4[i], y);
        exps(w, ht.m, c);
        residual(w, y);
#pragma unroll
        for (int e = 0; e < N; e += 2) r = add2(r, make_float2(w[e], w[e + 1]));
      }
      const float sum = warp_sum(r.x + r.y);
      if (lane == 0) tiles[t].s = sum;
    }
  } else if (two) {
    for (int t = warp; t < nt; t += WARPS) weigh(t, weights_r);
  }
  if (two) __syncthreads();
  if (warp != 0) return;
  if (tested && !two && x >= 0) weigh((x + bt.lo) / kTile, weights_r);  // p without the token
  bool plain = !tested;
  float left;
  auto weight = [&](int k) { return tiles[k].s; };
  int at = pick(nt, us, lane, weight, left);
  if (at < 0) {
    // p and q are equal up to rounding: a draw from p, whose tiles are weighed by this warp alone
    plain = true;
    __syncwarp();  // pick has read the table
    for (int t = 0; t < nt; ++t) weigh(t, weights_p);
    at = pick(nt, us, lane, weight, left);
  }
  const int first = at * kTileBlocks * 32;  // the tile's first block
  const int nb = min(kTileBlocks * 32, (bt.hi + N - 1) / N - first);
  // the tile's loads at once
  uint4 w4[kTileBlocks];
#pragma unroll
  for (int i = 0; i < kTileBlocks; ++i) w4[i] = bt.load(first + 32 * i + lane);
  const int i = locate<T>(0, nb, left, lane, [&](int k, float (&w)[N]) {
    uint4 mine = w4[0];
#pragma unroll
    for (int i = 1; i < kTileBlocks; ++i)
      if (k >= 32 * i) mine = w4[i];
    Elem<T>::unpack(mine, w);
    exps(w, ht.m, c);
    if (!plain) rest_of(first + k, w);
  });
  if (lane == 0) {
    const int drawn = min(max(first * N + i - bt.lo, 0), p.V - 1);
    result(drawn, logp_of(Elem<T>::one(zt[drawn]), ht, c), tested);
  }
}

// ---------------------------------------------------------------- host

constexpr int kSMs = 152;
// Shared memory per CTA for segments, beyond the table, barriers and decision (3.2 KB, static), and the block that may
// be read past the last segment.
constexpr int64_t kMostBytes = 220 * 1024;
constexpr int64_t kPastBytes = 16;
static_assert(sizeof(Table) == 3072 && kMostBytes + kPastBytes + sizeof(Table) + 512 <= 227 * 1024, "a CTA's shared memory");
constexpr int64_t kGoodBytes = 72 * 1024;  // three CTAs per SM: one's copies run under the others' arithmetic

inline int64_t segment(int64_t V, int64_t C) { return ((V + C * kWarps - 1) / (C * kWarps) + 7) / 8 * 8; }
inline int64_t segment_bytes(int64_t V, int64_t C, int es) { return segment(V, C) * es + 16; }

// CTAs per row: few enough that each holds a good piece of it, and as many as fill the GPU while a
// segment keeps at least 1 KB. 0: the row does not fit in 16 CTAs.
int cluster_of(int64_t V, int es, int rows_held, int64_t clusters) {
  auto bytes = [&](int C) { return segment_bytes(V, C, es) * kWarps * rows_held; };
  int C = 1;
  while (C < kMaxCluster && bytes(C) > kGoodBytes) C *= 2;
  if (bytes(C) > kMostBytes) return 0;
  while (C < kMaxCluster && clusters * C < kSMs && segment_bytes(V, 2 * C, es) >= 1024) C *= 2;
  return C;
}

// A row's tiles fit in the table.
inline bool fits_table(int64_t V, int es) { return V * es <= int64_t(kMaxTiles - 2) * kTileBlocks * 32 * 16; }

// Whether a CTA takes a row: where every SM has a row, rows are long, and a row's tiles fit in the table.
// Measured, a CTA per row against a cluster per row, us: 160 rows of 304 KB with drafts' rows 36.5 / 43.7,
// 152 without 15.4 / 22.0, 305 of 128 KB 23.0 / 27.2, 512 of 64 KB 24.0 / 27.9; 1,280 of 16 KB 30.1 / 22.0,
// 1,500 of 8 KB 30.4 / 20.7 (the ends of short rows are most of them).
inline bool by_rows(int64_t V, int es, int64_t rows) {
  return rows >= kSMs && V * es >= 48 * 1024 && fits_table(V, es);
}

// Half the warps in a CTA (twice the CTAs) where nothing is drafted and CTAs of 16 warps, two per SM, would take
// more than one turn. Measured, us with 8 / 16 warps: 305 rows of 304 KB 33.5 / 41.6, 509 43.7 / 49.8, 2,000
// 131.7 / 137.9, but 160 29.3 / 25.2; 509 rows of 80 KB 19.2 / 25.2. With drafted tokens more rows begin before
// their sequence's refusal is known: 256 sequences of up to 8 looked-up tokens 75.6 / 65.3.
inline bool small_ctas(const Args& a) { return a.max_draft == 0 && a.n_seq > 2 * kSMs; }

template <typename T, bool GREEDY>
rl_status run(Args& a, cudaStream_t s) {
  const int held = a.draft && !GREEDY ? 2 : 1, es = sizeof(T);
  const int64_t clusters = static_cast<int64_t>(a.n_seq) * (a.max_draft + 1);
  const int C = cluster_of(a.V, es, held, clusters);
  if (C == 0 && !fits_table(a.V, es))
    return set_error(RL_ERR_UNSUPPORTED, "rl_verify_drafts: V is too large (above 2.09 MB, and for 16 CTAs of 220 KB)");
  // a CTA per row also where 16 CTAs do not hold a row and its draft row, whatever the number of rows
  if (C == 0 || by_rows(a.V, es, a.n_draft + a.n_seq)) {
    if (small_ctas(a)) row_kernel<T, GREEDY, 8><<<static_cast<unsigned>(clusters), 8 * 32, 0, s>>>(a);
    else row_kernel<T, GREEDY, 16><<<static_cast<unsigned>(clusters), 16 * 32, 0, s>>>(a);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? RL_OK : cuda_error(e, "row_kernel launch");
  }
  a.seg = static_cast<int32_t>(segment(a.V, C));
  a.seg_bytes = static_cast<int32_t>(segment_bytes(a.V, C, es));
  a.held = held;
  const size_t smem = static_cast<size_t>(kWarps) * held * a.seg_bytes + kPastBytes;
  auto kern = verify_kernel<T, GREEDY>;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_error(e, "cudaGetDevice");
  // clusters resident at once, by device and shape
  static std::mutex mu;
  static std::map<std::pair<int, std::pair<int, size_t>>, int> resident;
  {
    std::lock_guard<std::mutex> lock(mu);
    const auto key = std::make_pair(dev, std::make_pair(C, smem));
    auto it = resident.find(key);
    if (it == resident.end()) {
      e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               static_cast<int>(kMostBytes + kPastBytes));
      if (e == cudaSuccess) e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
      if (e != cudaSuccess) return cuda_error(e, "cudaFuncSetAttribute(verify_kernel)");
      int n = 0;
      cfg.gridDim = dim3(C);
      e = cudaOccupancyMaxActiveClusters(&n, kern, &cfg);
      if (e != cudaSuccess) return cuda_error(e, "cudaOccupancyMaxActiveClusters(verify_kernel)");
      if (n <= 0) return set_error(RL_ERR_UNSUPPORTED, "verify_kernel: no cluster fits on the device");
      it = resident.emplace(key, n).first;
    }
    a.check_from = a.max_draft == 0 ? static_cast<int32_t>(clusters) : it->second;
  }
  cfg.gridDim = dim3(static_cast<unsigned>(clusters * C));
  e = cudaLaunchKernelEx(&cfg, kern, a);
  return e == cudaSuccess ? RL_OK : cuda_error(e, "verify_kernel launch");
}

}  // namespace verify
}  // namespace rl

extern "C" rl_status rl_verify_drafts(const void* target_logits, const void* draft_logits, rl_dtype dtype,
                                      int32_t n_seq, int64_t n_draft, int32_t max_draft, int64_t V, int64_t ld_target,
                                      int64_t ld_draft, const int32_t* draft_ids, const int32_t* draft_offsets,
                                      const float* accept_u, const float* sample_u, const rl_verify_params* params,
                                      int32_t* out_ids, int32_t* n_accepted, float* out_logp, void* ws,
                                      size_t ws_bytes, rl_stream_t stream) {
  using namespace rl;
  clear_error();
  const std::string f = "rl_verify_drafts: ";
  if (dtype != RL_BF16 && dtype != RL_F32) return set_error(RL_ERR_INVALID_ARG, f + "bad dtype");
  if (n_seq < 0 || n_draft < 0 || max_draft < 0 || V < 1) return set_error(RL_ERR_INVALID_ARG, f + "bad size");
  if (!params) return set_error(RL_ERR_INVALID_ARG, f + "params is NULL");
  if (!(params->temperature >= 0.f) || !std::isfinite(params->temperature) ||
      (params->temperature > 0.f && params->temperature < 1e-4f))
    return set_error(RL_ERR_INVALID_ARG, f + "temperature must be 0 (greedy) or at least 1e-4");
  if (ld_target < V || (draft_logits && ld_draft < V))
    return set_error(RL_ERR_INVALID_ARG, f + "a leading dimension is below V");
  if (n_seq == 0) return RL_OK;
  if (!target_logits || !draft_offsets || !sample_u || !out_ids || !n_accepted || !out_logp || !ws ||
      (n_draft > 0 && (!draft_ids || !accept_u)))
    return set_error(RL_ERR_INVALID_ARG, f + "a required pointer is NULL");
  if (!aligned16(target_logits) || !aligned16(draft_logits) || !aligned16(ws))
    return set_error(RL_ERR_ALIGNMENT, f + "logits and ws must be 16-byte aligned");
  if (V > (1 << 24) || n_draft + n_seq > (int64_t(1) << 30) || max_draft >= verify::kFirst ||
      static_cast<int64_t>(n_seq) * (static_cast<int64_t>(max_draft) + 1) > (int64_t(1) << 26))
    return set_error(RL_ERR_UNSUPPORTED, f + "at most 2^24 entries, 2^30 rows and 2^26 pairs of a sequence and a place");
  if (ws_bytes < rl_workspace_size(n_draft + n_seq, V, 0))
    return set_error(RL_ERR_WORKSPACE_TOO_SMALL, f + "ws_bytes below rl_workspace_size(n_draft + n_seq, V, 0)");
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  uint8_t* base = static_cast<uint8_t*>(ws);
  verify::Args a = {};
  a.target = target_logits;
  a.draft = draft_logits;
  a.ld_t = ld_target;
  a.ld_d = ld_draft;
  a.V = static_cast<int32_t>(V);
  a.n_seq = n_seq;
  a.max_draft = max_draft;
  a.n_draft = n_draft;
  a.draft_ids = draft_ids;
  a.offsets = draft_offsets;
  a.accept_u = accept_u;
  a.sample_u = sample_u;
  const bool greedy = params->temperature == 0.f;
  a.c = greedy ? kLog2e : kLog2e / params->temperature;
  a.out_ids = out_ids;
  a.out_logp = out_logp;
  a.n_accepted = n_accepted;
  a.status = reinterpret_cast<int32_t*>(base);
  if (n_seq <= kWsVerifySeqs) {
    // the header's words: zero before the call and after it
    a.finished = reinterpret_cast<uint32_t*>(base + kWsVerifyOffset);
    a.refused = reinterpret_cast<int32_t*>(a.finished + kWsVerifySeqs);
  } else {
    a.finished = reinterpret_cast<uint32_t*>(base + kWsHeader);
    a.refused = reinterpret_cast<int32_t*>(a.finished + n_seq);
    const cudaError_t e = max_draft == 0 ? cudaSuccess : cudaMemsetAsync(a.finished, 0, static_cast<size_t>(n_seq) * 8, s);
    if (e != cudaSuccess) return cuda_error(e, "rl_verify_drafts: cudaMemsetAsync");
  }
  if (dtype == RL_BF16) return greedy ? verify::run<uint16_t, true>(a, s) : verify::run<uint16_t, false>(a, s);
  return greedy ? verify::run<float, true>(a, s) : verify::run<float, false>(a, s);
}
