// The next token of every request from its logits row, by temperature, top-k, top-p and min-p, from given random numbers.
//
// With the entries in the order of their size (the lower index first among equals) and p = softmax(z / T), each filter
// keeps a beginning of that order: top-k its first k; top-p those before which less than top_p of the top-k ones' mass
// lies; min-p those with p >= min_p of the largest. What all of them keep is a threshold: the entries above a value, and
// of those equal to it the first few by index. The token is the lowest kept one, in vocabulary order, at which the
// running sum of the kept ones' weights passes u times their total.
//
// A thread-block cluster takes a row and holds it in shared memory, a segment per warp, so that HBM is read once:
//   1. every warp folds its segment into (max, sum of exponentials); one exchange gives every CTA the row's.
//   2. the threshold, only where a filter asks for one: counts of the entries by their distance from the largest in
//      steps of bf16 (the upper half of the ordered bit pattern), 1,024 bins, added up over the cluster. A bin of a bf16
//      row is one value, whose mass is its count times its weight; fp32 rows add up the weights too, as integers of 2^-40,
//      and go on into the bin that holds the border, 64 patterns a bin and then one. Borders farther below the largest
//      entry (8 powers of two) take coarser bins first. Integer sums: any order gives the same bits.
//   3. every warp sums the kept weights of its segment and counts the entries equal to the threshold; a second exchange;
//      the warp whose segment holds the token finds it by a scan.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <string>

#include "rl_device.cuh"
#include "rl_host.h"
#include "rl_segment.cuh"

namespace rl {
namespace sample {

using namespace seg;

constexpr int kMaxCluster = 16;
constexpr int kBinBits = 10, kBins = 1 << kBinBits;
constexpr int kBf16Shift = 16;  // patterns of a bf16 step
constexpr int kRestShift = 22;  // the bins cover all patterns

struct Args {
  const void* logits;
  int64_t ld, rows;
  int32_t V;
  const float* u;
  float temperature, top_p, min_p;
  int32_t top_k;
  const float* row_temperature;  // per row, or NULL
  const int32_t* row_top_k;
  const float* row_top_p;
  const float* row_min_p;
  int32_t seg, seg_bytes;
  int32_t* ids;
  float* logp;
  float* among;     // or NULL
  int32_t* n_kept;  // or NULL
  int32_t* status;
};

// A row's settings; whether they are ones that the library takes.
struct Settings {
  float T, top_p, min_p, u;
  int32_t top_k;
  __device__ __forceinline__ bool ok() const {
    return (T == 0.f || (T >= 1e-4f && T < 3e38f)) && top_k >= 0 && top_p > 0.f && top_p <= 1.f && min_p >= 0.f &&
           min_p <= 1.f && u >= 0.f && u < 1.f;
  }
};

// Larger numbers have larger keys; -0 has that of 0.
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t b = __float_as_uint(__fadd_rn(z, 0.f));
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu));
}
// The largest key of an entry of this type that is at most `key`.
template <typename T>
__device__ __forceinline__ uint32_t entry_key(uint32_t key) {
  if (sizeof(T) == 4) return key;
  if (key >> 31) return key & 0xffff0000u;
  return (key & 0xffffu) == 0xffffu ? key : (key & 0xffff0000u) - 1u;
}

constexpr float kMassUnit = 1099511627776.f;  // 2^40
__device__ __forceinline__ unsigned long long mass_of(float w) { return __float2ull_rn(w * kMassUnit); }

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ unsigned long long ld_cluster_u64(uint32_t addr) {
  unsigned long long v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void put_u1(uint32_t addr, uint32_t a) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" :: "r"(addr), "r"(a) : "memory");
}

// A border: entries above `key` and the first m of those equal to it; their number above it and their mass.
struct Border {
  uint32_t key, m, above;
  unsigned long long mass, unit;  // of the entries above; of one entry equal to it
};

template <int WARPS>
struct Shared {
  static constexpr int kSegs = WARPS * kMaxCluster;
  Fold fold[kSegs];      // every segment's, the same in every CTA of the cluster
  float sum[kSegs];      // of the kept weights above the threshold
  uint32_t above[kSegs]; // kept entries above it
  uint32_t equal[kSegs]; // entries equal to it
  alignas(16) uint32_t count[kBins];  // this CTA's
  alignas(16) unsigned long long mass[kBins];
  uint32_t warp_count[WARPS];
  unsigned long long warp_mass[WARPS];
  Border found;
  int32_t bin;  // that found is of (-1: none)
  uint64_t bar[WARPS];
};

// The bins of distances d0 .. d0 + (kBins << shift) from the largest entry's key.
struct Level {
  uint32_t d0;
  int shift;
};

template <typename T, int WARPS>
struct Row {
  Shared<WARPS>& sh;
  Segment<T> mine;
  Fold all;  // the row's
  float c;
  uint32_t top;  // the largest entry's key
  int C;
  bool masses;   // weights are wanted
  static constexpr int N = Elem<T>::N, kThreads = WARPS * 32, kOwn = kBins / kThreads;
  static constexpr int kSingle = sizeof(T) == 2 ? kBf16Shift : 0;  // bins of at most these patterns hold one value
  Level level{0u, -1};  // what the bins hold
  uint32_t above = 0;   // entries before the level's first bin
  unsigned long long mass = 0;
  uint32_t n[kOwn], run_n, all_n;            // this thread's bins over the cluster; entries before them; all bins'
  unsigned long long w[kOwn], run_w, all_w;  // the same for masses

  __device__ __forceinline__ float weight(float z) const { return ex2(exponent(z, all.m, c)); }

  // bf16 entries by their patterns, to bins of one step each below the largest entry's. The patterns of entries of its sign
  // fall (or, below zero, rise) by one a step; those of the other sign are out of range either way.
  __device__ __forceinline__ void count_near() {
    const int lane = threadIdx.x & 31, nb = mine.blocks();
    const uint32_t m = __float_as_uint(all.m) >> 16;
    const bool down = m < 0x8000u;
    for (int k = lane; k < nb; k += 32) {
      const uint4 q = *reinterpret_cast<const uint4*>(mine.at + k * N);
      const uint32_t v[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t lo = v[i] & 0xffffu, hi = v[i] >> 16;
        const uint32_t a = down ? m - lo : lo - m, b = down ? m - hi : hi - m;
        if (a < kBins) atomicAdd(&sh.count[a], 1u);
        if (b < kBins) atomicAdd(&sh.count[b], 1u);
      }
    }
  }

  // Counts the cluster's entries by the bins of `to`, and this thread's bins over the cluster with what lies before them.
  __device__ __forceinline__ void count(const Level& to) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const bool single = to.shift <= kSingle, weigh = masses && !single;
    if (level.shift >= 0) {
      cluster_sync_all();  // the other CTAs have read the last level's
      for (int i = threadIdx.x; i < kBins; i += kThreads) {
        sh.count[i] = 0;
        if (weigh) sh.mass[i] = 0;
      }
      __syncthreads();
    }
    const uint32_t m = __float_as_uint(all.m) >> 16;
    // (negative infinity is 0xff80: out of reach of a largest entry below zero only from steps that its bins do not have)
    if (sizeof(T) == 2 && to.d0 == 0 && to.shift == kBf16Shift && ((m >= kBins && m < 0x8000u) || (m > 0x8000u && m + kBins <= 0xff80u))) {
      count_near();
    } else {
      const int nb = mine.blocks();
      for (int k = lane; k < nb; k += 32) {
        float z[N];
        mine.load(k, z);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const uint32_t d = top - key_of(z[e]), bin = (d - to.d0) >> to.shift;
          if (z[e] > minus_inf() && d >= to.d0 && bin < kBins) {
            atomicAdd(&sh.count[bin], 1u);
            if (weigh) atomicAdd(&sh.mass[bin], mass_of(weight(z[e])));
          }
        }
      }
    }
    level = to;
    cluster_sync_all();
    // the cluster's sums: this thread's bins of every CTA
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      n[i] = 0;
      w[i] = 0;
    }
    const uint32_t at_n = smem_addr(&sh.count[threadIdx.x * kOwn]), at_w = smem_addr(&sh.mass[threadIdx.x * kOwn]);
#pragma unroll 4
    for (int r = 0; r < C; ++r) {
      const uint32_t from = map_to_rank(at_n, r);
#pragma unroll
      for (int i = 0; i < kOwn; i += 2) {
        const unsigned long long two = ld_cluster_u64(from + 4 * i);
        n[i] += static_cast<uint32_t>(two);
        n[i + 1] += static_cast<uint32_t>(two >> 32);
      }
    }
    if (weigh)
      for (int r = 0; r < C; ++r) {
        const uint32_t from = map_to_rank(at_w, r);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) w[i] += ld_cluster_u64(from + 8 * i);
      }
    uint32_t mine_n = 0;
    unsigned long long mine_w = 0;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      if (masses && single && n[i] != 0)
        w[i] = n[i] * mass_of(weight(value_of(entry_key<T>(top - (to.d0 + (static_cast<uint32_t>(threadIdx.x * kOwn + i) << to.shift))))));
      mine_n += n[i];
      mine_w += w[i];
    }
    // what lies before them
    run_n = mine_n;
    run_w = mine_w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t a = __shfl_up_sync(0xffffffffu, run_n, o);
      if (lane >= o) run_n += a;
    }
    if (masses)
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long a = __shfl_up_sync(0xffffffffu, run_w, o);
        if (lane >= o) run_w += a;
      }
    if (lane == 31) {
      sh.warp_count[warp] = run_n;
      sh.warp_mass[warp] = run_w;
    }
    __syncthreads();
    run_n += above - mine_n;
    run_w += mass - mine_w;
    all_n = 0;
    all_w = 0;
#pragma unroll
    for (int v = 0; v < WARPS; ++v) {
      const uint32_t a = sh.warp_count[v];
      run_n += v < warp ? a : 0;
      all_n += a;
      if (masses) {
        const unsigned long long b = sh.warp_mass[v];
        run_w += v < warp ? b : 0;
        all_w += b;
      }
    }
  }

  // The border of what top_k (0: off) and top_p (1: off) keep of the row; false: they keep everything.
  __device__ __forceinline__ bool search(int32_t top_k, float top_p, Border& found) {
    bool any = false, by_mass = top_k == 0;
    auto mass_goal = [&](double total) { return max(1ull, static_cast<unsigned long long>(ceil(static_cast<double>(top_p) * total))); };
    unsigned long long goal = by_mass ? mass_goal(static_cast<double>(all.s) * kMassUnit) : static_cast<unsigned long long>(top_k);
    Level to{0u, kBf16Shift};
    while (true) {
      if (to.d0 != level.d0 || to.shift != level.shift) count(to);
      if (threadIdx.x == 0) sh.bin = -1;
      __syncthreads();
      uint32_t a = run_n;
      unsigned long long m = run_w;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        if (by_mass ? m < goal && m + w[i] >= goal : a < goal && a + n[i] >= goal) {
          sh.bin = threadIdx.x * kOwn + i;
          sh.found.above = a;
          sh.found.mass = m;
          sh.found.m = n[i];
        }
        a += n[i];
        m += w[i];
      }
      __syncthreads();
      const int bin = sh.bin;
      Border b = sh.found;
      __syncthreads();  // and may be written again
      bool none = false;
      if (bin < 0) {
        none = to.d0 != 0 || to.shift != kBf16Shift;
        if (!none) {
          // not among the nearest: all that is farther away
          above += all_n;
          mass += all_w;
          to = Level{static_cast<uint32_t>(kBins) << kBf16Shift, kRestShift};
          continue;
        }
      } else {
        const uint32_t d0 = to.d0 + (static_cast<uint32_t>(bin) << to.shift);
        if (to.shift > kSingle) {
          above = b.above;
          mass = b.mass;
          to = Level{d0, max(0, to.shift - kBinBits)};
          continue;
        }
        b.key = entry_key<T>(top - d0);
        b.unit = masses ? mass_of(weight(value_of(b.key))) : 0;
        if (!by_mass) b.m = static_cast<uint32_t>(goal) - b.above;
        else if (b.unit) b.m = static_cast<uint32_t>(min(static_cast<unsigned long long>(b.m), (goal - b.mass + b.unit - 1) / b.unit));
        found = b;
        any = true;
      }
      if (by_mass || top_p >= 1.f) return any;
      // then top_p, of the mass of what top_k keeps
      by_mass = true;
      goal = mass_goal(none ? static_cast<double>(all.s) * kMassUnit : static_cast<double>(b.mass + b.m * b.unit));
      if (level.d0 != 0 || level.shift != kBf16Shift) {
        above = 0;
        mass = 0;
      }
      to = Level{0u, kBf16Shift};
    }
  }
};

template <typename T, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, 1024 / (WARPS * 32)) sample_kernel(const Args p) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(16) Shared<WARPS> sh;
  constexpr int N = Elem<T>::N;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank(), C = cluster_nctarank();
  const int64_t row = blockIdx.x / C;
  const int n_seg = static_cast<int>(C) * WARPS, g = static_cast<int>(rank) * WARPS + warp;
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // the other CTAs have started
  const T* z = static_cast<const T*>(p.logits) + row * p.ld;
  const int e0 = min(g * p.seg, p.V), n = min(p.seg, p.V - e0);
  if (lane == 0) {
    mbar_init(&sh.bar[warp], 1);
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  __syncwarp();
  const T* end = static_cast<const T*>(p.logits) + (p.rows - 1) * p.ld + p.V;
  const Segment<T> mine = fetch(z, e0, n, end, smem + static_cast<size_t>(warp) * p.seg_bytes, &sh.bar[warp], lane);
  for (int i = threadIdx.x; i < kBins; i += WARPS * 32) {  // while the row is on its way
    sh.count[i] = 0;
    sh.mass[i] = 0;
  }
  Settings set{p.temperature, p.top_p, p.min_p, p.u[row], p.top_k};
  if (p.row_temperature) set.T = p.row_temperature[row];
  if (p.row_top_k) set.top_k = p.row_top_k[row];
  if (p.row_top_p) set.top_p = p.row_top_p[row];
  if (p.row_min_p) set.min_p = p.row_min_p[row];
  const bool greedy = set.T == 0.f, known = set.ok();
  const float c = greedy || !known ? kLog2e : kLog2e / set.T;

  // ---- the row's largest entry and its normaliser
  const bool in_time = mbar_wait_bounded(&sh.bar[warp], 0);
  if (!in_time && lane == 0) flag_status(p.status, RL_DEV_TIMEOUT);
  mine.blank_edges(lane);
  int unused = 0;
  const Fold f = fold<T, false>(mine, c, lane, unused);
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  if (lane < C) put_f2(map_to_rank(smem_addr(&sh.fold[g]), lane), f.m, f.s);
  __syncwarp();
  cluster_sync_all();
  const Fold all = merged(sh.fold, n_seg, c, lane);
  if (is_bad(all) || !known) {  // the whole cluster
    if (rank == 0 && threadIdx.x == 0) {
      flag_status(p.status, RL_DEV_BAD_VALUE);
      p.ids[row] = -1;
      p.logp[row] = __int_as_float(0x7fc00000);
      if (p.among) p.among[row] = __int_as_float(0x7fc00000);
      if (p.n_kept) p.n_kept[row] = 0;
    }
    return;
  }

  // ---- the threshold: entries above zt are kept, and the first ties of those equal to it
  Row<T, WARPS> r{sh, mine, all, c, key_of(all.m), static_cast<int>(C), set.top_p < 1.f};
  float zt = minus_inf();
  uint32_t ties = 0;
  const bool by_k = !greedy && set.top_k > 0 && set.top_k < p.V, by_p = !greedy && set.top_p < 1.f;
  const bool by_m = !greedy && set.min_p > 0.f;
  if (greedy) {
    zt = all.m;
    ties = 1;
  }
  if (by_k || by_p) {
    Border b;
    if (r.search(by_k ? set.top_k : 0, set.top_p, b)) {
      zt = value_of(b.key);
      ties = b.m;
    }
  }
  const float rc = __fmul_rn(all.m, c);
  const bool apart = large(rc);
  auto exponent_of = [&](float v) { return apart ? (v - all.m) * c : fmaf(v, c, -rc); };
  // min_p, as an exponent from that of the largest entry, which the rounding of its product moves as all others
  const float least = by_m ? exponent_of(all.m) + log2f(set.min_p) : minus_inf();

  // ---- the kept weights of every segment
  const bool filtered = greedy || by_k || by_p || by_m;
  const bool pass = filtered || p.n_kept;
  const int nb = mine.blocks();
  if (pass) {
    float sum = 0.f;
    uint32_t above = 0, equal = 0;
    for (int k = lane; k - lane < nb; k += 32) {
      float v[N];
      bool any = false;
      if (k < nb) {
        mine.load(k, v);
        float most = v[0];
#pragma unroll
        for (int e = 1; e < N; ++e) most = fmaxf(most, v[e]);
        any = most >= zt;
      }
      if (!__ballot_sync(0xffffffffu, any)) continue;  // most blocks hold nothing that is kept
      if (!any) continue;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float x = exponent_of(v[e]);
        const bool in = x >= least, over = v[e] > zt && in;
        sum += over ? ex2(x) : 0.f;
        above += over;
        equal += v[e] == zt && in;
      }
    }
    sum = warp_sum(sum);
    above = __reduce_add_sync(0xffffffffu, above);
    equal = __reduce_add_sync(0xffffffffu, equal);
    if (lane < C) {
      put_f1(map_to_rank(smem_addr(&sh.sum[g]), lane), sum);
      put_u1(map_to_rank(smem_addr(&sh.above[g]), lane), above);
      put_u1(map_to_rank(smem_addr(&sh.equal[g]), lane), equal);
    }
    __syncwarp();
    cluster_sync_all();
  } else {
    __syncthreads();
  }

  // ---- the segment that holds the token, by every warp alike
  const float wt = ties ? ex2(exponent_of(zt)) : 0.f;
  const int M = (n_seg + 31) / 32, k0 = min(lane * M, n_seg), k1 = min(k0 + M, n_seg);
  uint32_t before = 0, kept = 0;  // entries equal to the threshold in the segments before; all kept
  if (pass) {
    uint32_t here = 0;
    for (int k = k0; k < k1; ++k) {
      here += sh.equal[k];
      kept += sh.above[k];
    }
    uint32_t run = here;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t a = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += a;
    }
    before = run - here;
    kept = __reduce_add_sync(0xffffffffu, kept) + min(ties, __shfl_sync(0xffffffffu, run, 31));
  }
  // a lane's segments are asked for in order: the ties of segment k come after those of the lane's segments before it
  auto ties_of = [&](int k) -> uint32_t {
    uint32_t b = before;
    for (int i = k0; i < k; ++i) b += sh.equal[i];
    return b >= ties ? 0u : min(ties - b, sh.equal[k]);
  };
  float total_kept = 0.f;
  auto weight = [&](int k) {
    if (!filtered) return sh.fold[k].s == 0.f ? 0.f : sh.fold[k].s * power(sh.fold[k].m, all.m, c);
    return fmaf(static_cast<float>(ties_of(k)), wt, sh.sum[k]);
  };
  for (int k = k0; k < k1; ++k) total_kept += weight(k);
  total_kept = warp_sum(total_kept);
  float left;
  const int at = pick(n_seg, set.u, lane, weight, left);
  // how many of the threshold's entries that segment keeps
  const uint32_t ties_there = filtered ? __shfl_sync(0xffffffffu, at >= k0 && at < k1 ? ties_of(at) : 0u, max(at, 0) / M) : 0u;
  if (at != g) return;
  uint32_t rest = ties_there;
  // the entries' weights in order, ties by their rank
  int token = -1;
  {
    int last = -1;
    float acc0 = 0.f;
    for (int b0 = 0; b0 < nb && token < 0; b0 += 32) {
      const int k = b0 + lane;
      float v[N], w[N], s = 0.f;
      uint32_t eq = 0, bits = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) w[e] = 0.f;
      if (k < nb) {
        mine.load(k, v);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          if (!(v[e] >= zt) || v[e] == minus_inf()) continue;
          const float x = exponent_of(v[e]);
          if (!(x >= least)) continue;
          if (v[e] > zt || !filtered) {
            w[e] = ex2(x);
          } else {
            ++eq;
            bits |= 1u << e;
          }
        }
      }
      uint32_t rank_eq = eq;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t a = __shfl_up_sync(0xffffffffu, rank_eq, o);
        if (lane >= o) rank_eq += a;
      }
      const uint32_t eq_all = __shfl_sync(0xffffffffu, rank_eq, 31);
      uint32_t used = rank_eq - eq;
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (bits >> e & 1) {
          if (used < rest) w[e] = wt;
          ++used;
        }
      rest -= min(rest, eq_all);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        s += w[e];
        if (w[e] > 0.f) last = k * N + e;
      }
      float run = s;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const float a = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += a;
      }
      const uint32_t over = __ballot_sync(0xffffffffu, s > 0.f && acc0 + run > left);
      if (over) {
        const int from = __ffs(over) - 1;
        float acc = acc0 + (run - s);
        int here = -1;
#pragma unroll
        for (int e = 0; e < N; ++e) {
          acc += w[e];
          if (here < 0 && w[e] > 0.f && acc > left) here = k * N + e;
        }
        token = __shfl_sync(0xffffffffu, here >= 0 ? here : last, from);
      }
      acc0 += __shfl_sync(0xffffffffu, run, 31);
    }
    // where rounding leaves the sum short of its goal: the last that has any weight
    if (token < 0) token = static_cast<int>(__reduce_max_sync(0xffffffffu, last));
  }
  if (lane != 0) return;
  token = min(max(e0 + token - mine.lo, 0), p.V - 1);
  const float zx = Elem<T>::one(z[token]);
  p.ids[row] = token;
  p.logp[row] = logp_of(zx, all, c);
  if (p.among) p.among[row] = (exponent_of(zx) - log2f(total_kept)) * kLn2;
  if (p.n_kept) p.n_kept[row] = static_cast<int32_t>(kept);
}

// ---------------------------------------------------------------- host

constexpr int kSMs = 152;
constexpr int64_t kPastBytes = 16;
constexpr int64_t kGoodBytes = 84 * 1024;   // two CTAs per SM: one's copies run under the other's arithmetic
constexpr int64_t kMostBytes = 200 * 1024;  // beside the tables
static_assert(sizeof(Shared<16>) <= 24 * 1024 && kMostBytes + kPastBytes + sizeof(Shared<16>) <= 227 * 1024, "a CTA's shared memory");

inline int64_t segment(int64_t V, int64_t parts) { return ((V + parts - 1) / parts + 7) / 8 * 8; }
inline int64_t segment_bytes(int64_t V, int64_t parts, int es) { return segment(V, parts) * es + 16; }

template <typename T, int WARPS>
rl_status launch(Args& a, int C, cudaStream_t s) {
  a.seg = static_cast<int32_t>(segment(a.V, C * WARPS));
  a.seg_bytes = static_cast<int32_t>(segment_bytes(a.V, C * WARPS, sizeof(T)));
  auto kern = sample_kernel<T, WARPS>;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_error(e, "cudaGetDevice");
  // once per device
  static std::atomic<uint64_t> ready{0};
  const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
  if (!(ready.load() & bit)) {
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kMostBytes + kPastBytes));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return cuda_error(e, "cudaFuncSetAttribute(sample_kernel)");
    ready |= bit;
  }
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cfg.blockDim = dim3(WARPS * 32);
  cfg.gridDim = dim3(static_cast<unsigned>(a.rows * C));
  cfg.dynamicSmemBytes = static_cast<size_t>(WARPS) * a.seg_bytes + kPastBytes;
  cfg.stream = s;
  e = cudaLaunchKernelEx(&cfg, kern, a);
  return e == cudaSuccess ? RL_OK : cuda_error(e, "sample_kernel launch");
}

template <typename T>
rl_status run(Args& a, cudaStream_t s) {
  const int es = sizeof(T);
  auto bytes = [&](int C) { return segment_bytes(a.V, C * 16, es) * 16; };
  int C = 1;
  while (C < kMaxCluster && bytes(C) > kGoodBytes) C *= 2;
  if (bytes(C) > kMostBytes)
    return set_error(RL_ERR_UNSUPPORTED, "rl_sample_tokens: V is too large (a row has to fit in 16 CTAs of 200 KB)");
  if (C == 1 && a.V * es <= 16 * 1024) return launch<T, 4>(a, 1, s);
  while (C < kMaxCluster && a.rows * C < kSMs && segment_bytes(a.V, 2 * C * 16, es) >= 1024) C *= 2;
  return launch<T, 16>(a, C, s);
}

}  // namespace sample
}  // namespace rl

extern "C" rl_status rl_sample_tokens(const void* logits, rl_dtype dtype, int64_t rows, int64_t V, int64_t ld,
                                      const float* sample_u, const rl_sample_params* params,
                                      const float* row_temperature, const int32_t* row_top_k, const float* row_top_p,
                                      const float* row_min_p, int32_t* out_ids, float* out_logp,
                                      float* out_filtered_logp, int32_t* n_kept, void* ws, size_t ws_bytes,
                                      rl_stream_t stream) {
  using namespace rl;
  clear_error();
  const std::string f = "rl_sample_tokens: ";
  if (dtype != RL_BF16 && dtype != RL_F32) return set_error(RL_ERR_INVALID_ARG, f + "bad dtype");
  if (rows < 0 || V < 1) return set_error(RL_ERR_INVALID_ARG, f + "bad size");
  if (!params) return set_error(RL_ERR_INVALID_ARG, f + "params is NULL");
  if (!(params->temperature >= 0.f) || !std::isfinite(params->temperature) ||
      (params->temperature > 0.f && params->temperature < 1e-4f))
    return set_error(RL_ERR_INVALID_ARG, f + "temperature must be 0 (greedy) or at least 1e-4");
  if (params->top_k < 0) return set_error(RL_ERR_INVALID_ARG, f + "top_k must not be negative");
  if (!(params->top_p > 0.f && params->top_p <= 1.f)) return set_error(RL_ERR_INVALID_ARG, f + "top_p must be in (0, 1]");
  if (!(params->min_p >= 0.f && params->min_p <= 1.f)) return set_error(RL_ERR_INVALID_ARG, f + "min_p must be in [0, 1]");
  if (ld < V) return set_error(RL_ERR_INVALID_ARG, f + "the leading dimension is below V");
  if (rows == 0) return RL_OK;
  if (!logits || !sample_u || !out_ids || !out_logp || !ws)
    return set_error(RL_ERR_INVALID_ARG, f + "a required pointer is NULL");
  if (!aligned16(logits) || !aligned16(ws)) return set_error(RL_ERR_ALIGNMENT, f + "logits and ws must be 16-byte aligned");
  if (V > (1 << 24) || rows > (1 << 26)) return set_error(RL_ERR_UNSUPPORTED, f + "at most 2^24 entries and 2^26 rows");
  if (ws_bytes < kWsHeader) return set_error(RL_ERR_WORKSPACE_TOO_SMALL, f + "workspace smaller than its header");
  sample::Args a = {};
  a.logits = logits;
  a.ld = ld;
  a.rows = rows;
  a.V = static_cast<int32_t>(V);
  a.u = sample_u;
  a.temperature = params->temperature;
  a.top_k = params->top_k;
  a.top_p = params->top_p;
  a.min_p = params->min_p;
  a.row_temperature = row_temperature;
  a.row_top_k = row_top_k;
  a.row_top_p = row_top_p;
  a.row_min_p = row_min_p;
  a.ids = out_ids;
  a.logp = out_logp;
  a.among = out_filtered_logp;
  a.n_kept = n_kept;
  a.status = static_cast<int32_t*>(ws);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  return dtype == RL_BF16 ? sample::run<uint16_t>(a, s) : sample::run<float>(a, s);
}
