// The next token of every request from its logits row, by temperature, top-k, top-p and min-p, from given random numbers.
//
// With the entries in the order of their size (the lower index first among equals) and p = softmax(z / T), each filter
// keeps a beginning of that order: top-k its first k; top-p those before which less than top_p of the top-k ones' mass
// lies; min-p those with p >= min_p of the largest. What all of them keep is a threshold: the entries above a value, and
// of those equal to it the first few by index. The token is the lowest kept one, in vocabulary order, at which the
// running sum of the kept ones' weights passes u times their total.
//
// A CTA takes a row, or with few rows a cluster of them; the row is cut into tiles of 2 KB, a warp each in turn.
//   1. every warp folds its tiles into (max, sum of exponentials); one exchange gives the row's.
//   2. the threshold, only where top-k or top-p ask for one: counts of the entries in 1,024 bins, added up over the cluster,
//      and a scan. A bf16 row's bins are single values, whose mass is their count times their weight; entries of 0.5 to 128
//      are counted in the first pass already, on the guess that the largest entry and the border are among them. Where
//      they are not, and for fp32 rows, more passes count by the distance of the ordered bit patterns from the largest
//      entry's, in steps of 2^16 patterns, then down to single ones within the bin that holds the border; masses are then
//      added up as integers of 2^-38. Integer sums: any order gives the same bits. min-p is a value, found by bisection.
//   3. a pass sums the kept weights of every tile and counts the entries equal to the threshold; a second exchange; the tile
//      that holds the token is found by a scan, and the token in it by another.
// HBM is read once: the rows at work at a time fit in L2, where the later passes find them, and tiles whose largest entry is
// below the threshold are not read again.
//
// What bounds it is the arithmetic beside the one exponential an entry (unpacking, the bins, the comparisons: 8 instructions
// an entry for the first pass, 6 for the bins, up to 8 for the pass over what is kept) and the chain of a row's steps. Measured:
// one row of 151,936 bf16 12 us without filters, 16 with top-k 50, 19 with top-p 0.4; 509 rows 40 without (57% of the copy's
// rate), 63 with top-k 50, 82 with top-p 0.4 (4 more before a tile's few kept entries were taken one by one), 60 with 0.7 / 20 /
// 0.8; 254 rows fp32 35 without, 44 with top-k 50, 102 with top-p 0.4, 226 with 0.95. Outside the window of step 2: 128 rows
// bf16 with top-p 0.95 53 us, inside 33. The first form held a row in the shared memory of a cluster (509 rows 155 with top-k 50,
// 207 with top-p 0.95): 76 rows at work at a time instead of all, each through four exchanges.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <string>

#include "rl_device.cuh"
#include "rl_host.h"
#include "rl_segment.cuh"

namespace rl {
namespace sample {

using namespace seg;

constexpr int kMostCluster = 8;
constexpr int kBinBits = 10, kBins = 1 << kBinBits;
constexpr int kBf16Shift = 16;  // patterns of a bf16 step
constexpr int kRestShift = 22;  // the bins cover all patterns
constexpr int kTileBlocks32 = kTileBlocks * 32;  // 16-byte blocks of a tile
// The window of the first pass: bf16 patterns of 0.5 up to 128, the largest first.
constexpr uint32_t kWindowLow = 0x3f00u, kWindowTop = kWindowLow + kBins - 1;

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
  int32_t tiles;  // of a CTA
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
    return (T == 0.f || (T >= 1e-4f && T < __int_as_float(0x7f800000))) && top_k >= 0 && top_p > 0.f && top_p <= 1.f && min_p >= 0.f &&
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

// Masses are integers of 2^-38 of the largest entry's weight: the sum of 2^24 of them stays below 2^63, and the roundings of V
// entries come to V 2^-39 of it at most, whichever way they go (2^-36 put the border of long flat tails elsewhere: 1.2e-4 at 2^24).
constexpr float kMassUnit = 274877906944.f;
// The logarithm of a token's share of the kept mass, x being its exponent and `others` the sum of the other kept weights, which has
// never been added to its own: a share close to 1 is then as exact as the small weights are. (From the total, whose half step is
// 2^-24 of it, the logarithm of a share of 1 - 2^-10 was relative 6e-5.) log(1 + r) = 2 artanh(r / (2 + r)), by its power series.
__device__ __forceinline__ float log_share(float x, float others, float total) {
  const float w = ex2(x);
  if (!(others < w)) return (x - log2f(total)) * kLn2;
  const float t = __fdividef(others, others + 2.f * w), y = t * t;  // up to 1/3: the first term left out is 2^-26 of the sum
  float s = 1.f / 13.f;
#pragma unroll
  for (int k = 11; k > 0; k -= 2) s = fmaf(s, y, 1.f / k);
  return 0.f - 2.f * t * s;
}
__device__ __forceinline__ unsigned long long mass_of(float w) { return __float2ull_rn(w * kMassUnit); }

__device__ __forceinline__ unsigned long long ld_cluster_u64(uint32_t addr) {
  unsigned long long v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void put_u2(uint32_t addr, uint32_t a, uint32_t b) {
  asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" :: "r"(addr), "r"(a), "r"(b) : "memory");
}

// Both halves of a pair of bf16 against a value: all ones where it holds.
__device__ __forceinline__ uint32_t above2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("set.gt.u32.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t least2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("set.ge.u32.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t equal2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("set.eq.u32.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// A row as the 16-byte blocks of memory that it covers.
template <typename T>
struct RowBlocks {
  static constexpr int N = Elem<T>::N;
  static constexpr uint32_t kNone = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
  const T* at;   // the first block
  int lo, hi;    // the row's elements are [lo, hi) from `at`
  int nb;        // blocks
  __device__ __forceinline__ RowBlocks(const T* row, int V) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(row), a0 = a & ~uintptr_t(15);
    at = reinterpret_cast<const T*>(a0);
    lo = static_cast<int>(a - a0) / static_cast<int>(sizeof(T));
    hi = lo + V;
    nb = (hi + N - 1) / N;
  }
  // Block k; elements of other rows, and blocks behind the last, are minus infinity.
  __device__ __forceinline__ uint4 block(int k) const {
    if (k > 0 && k < nb - 1) return __ldcg(reinterpret_cast<const uint4*>(at + static_cast<int64_t>(k) * N));
    uint4 q = make_uint4(kNone, kNone, kNone, kNone);
    if (k < 0 || k >= nb) return q;
    T e[N];
    memcpy(e, &q, sizeof(q));
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (k * N + i >= lo && k * N + i < hi) e[i] = at[k * N + i];
    memcpy(&q, e, sizeof(q));
    return q;
  }
  // A lane's blocks of tile t.
  __device__ __forceinline__ void tile(int t, int lane, uint4 (&w)[kTileBlocks]) const {
    const int k = t * kTileBlocks32 + lane;
    if (t > 0 && (t + 1) * kTileBlocks32 < nb) {
      const uint4* p = reinterpret_cast<const uint4*>(at) + k;
#pragma unroll
      for (int i = 0; i < kTileBlocks; ++i) w[i] = __ldcg(p + 32 * i);
    } else {
#pragma unroll
      for (int i = 0; i < kTileBlocks; ++i) w[i] = block(k + 32 * i);
    }
  }
};

// A barrier of all CTAs of a row, and two words of shared memory of one of them.
template <bool CLUSTER>
__device__ __forceinline__ void sync_all() {
  if (CLUSTER) cluster_sync_all();
  else __syncthreads();
}
template <bool CLUSTER>
__device__ __forceinline__ unsigned long long of_cta(const uint32_t* two, int r) {
  if (CLUSTER) return ld_cluster_u64(map_to_rank(smem_addr(two), r));
  return static_cast<unsigned long long>(two[1]) << 32 | two[0];
}

// A border: entries above `key` and the first m of those equal to it; their number above it and their mass.
struct Border {
  alignas(8) uint32_t key;
  uint32_t m;
  alignas(8) uint32_t above;
  unsigned long long mass, unit;  // of the entries above; of one entry equal to it
};

// A CTA's kept entries.
struct Part {
  float sum;  // weights of those above the threshold
  uint32_t equal, above;
};

template <int WARPS>
struct Shared {
  Fold fold[WARPS * kMostCluster];    // every warp's, the same in every CTA of the cluster
  alignas(16) uint32_t count[kBins + 32];  // this CTA's entries (and behind the bins those outside the window)
  static constexpr int kSort = WARPS == 4 ? 256 : 512;  // as many are sorted sooner than counted
  static constexpr int kList = WARPS == 4 ? 1024 : 4096;
  alignas(16) uint32_t low[kBins];  // and their mass
  alignas(16) uint32_t high[kBins];
  unsigned long long list[kList];  // the entries that may be kept, where they are few: by size, then by index
  alignas(8) uint32_t n_list;
  uint32_t n_equal;
  unsigned long long total;
  int32_t first, last;  // of the list's entries by index: the one at which the sum passes its goal, and the last of any weight
  uint32_t warp_count[WARPS];
  unsigned long long warp_mass[WARPS];
  Border found;
  int32_t bin;  // that found is of (-1: none)
  Fold all;     // the row's
  uint32_t least_key;  // min_p's value
  alignas(8) uint2 part_a[kMostCluster];  // every CTA's (sum, equal)
  uint32_t part_b[kMostCluster];          // above
  float warp_sum[WARPS];
  uint32_t warp_equal[WARPS], warp_above[WARPS];
};

// A tile's (max, sum) where nothing is filtered, else the kept weights above the threshold and the entries equal to it.
struct KeptOfTile {
  float sum;
  uint32_t equal;
};
union Tile {
  Fold fold;
  KeptOfTile kept;
};

// The bins of distances d0 .. d0 + (kBins << shift) from the largest entry's key; shift < 0: the window.
struct Level {
  uint32_t d0;
  int shift;
};

template <typename T, int WARPS, bool CLUSTER>
struct Row {
  Shared<WARPS>& sh;
  const RowBlocks<T>& row;
  int t0, t1;  // this CTA's tiles
  Fold all;    // the row's
  float c;
  uint32_t top;  // the largest entry's key
  int C;
  bool masses;   // weights are wanted
  static constexpr int N = Elem<T>::N, kThreads = WARPS * 32, kOwn = kBins / kThreads;
  static constexpr int kSingle = sizeof(T) == 2 ? kBf16Shift : 0;  // bins of at most these patterns hold one value
  bool listed = false;  // the CTA's entries that count are in its list
  uint32_t above = 0;  // entries before the level's first bin
  unsigned long long mass = 0;
  uint32_t n[kOwn], run_n, all_n;            // this thread's bins over the cluster; entries before them; all bins'
  unsigned long long w[kOwn], run_w, all_w;  // the same for masses

  __device__ __forceinline__ float weight(float z) const { return ex2(exponent(z, all.m, c)); }

  // Counts this CTA's entries by the bins of `to`.
  __device__ __forceinline__ void count(const Level& to) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const bool weigh = masses && to.shift > kSingle;
    sync_all<CLUSTER>();  // the other CTAs have read the last level's
    for (int i = threadIdx.x; i < kBins; i += kThreads) {
      sh.count[i] = 0;
      sh.low[i] = 0;
      sh.high[i] = 0;
    }
    __syncthreads();
    auto add = [&](float z) {
      const uint32_t d = top - key_of(z), bin = (d - to.d0) >> to.shift;
      if (!(z > minus_inf()) || d < to.d0 || bin >= kBins) return;
      atomicAdd(&sh.count[bin], 1u);
      if (!weigh) return;
      const unsigned long long m = mass_of(weight(z));
      const uint32_t lo = static_cast<uint32_t>(m), old = atomicAdd(&sh.low[bin], lo);
      const uint32_t hi = static_cast<uint32_t>(m >> 32) + (old + lo < old ? 1u : 0u);
      if (hi) atomicAdd(&sh.high[bin], hi);
    };
    if (sizeof(T) == 4 && listed) {
      for (int i = threadIdx.x; i < static_cast<int>(sh.n_list); i += kThreads) add(value_of(~static_cast<uint32_t>(sh.list[i] >> 32)));
    } else {
      for (int t = t0 + warp; t < t1; t += WARPS) {
        uint4 q[kTileBlocks];
        row.tile(t, lane, q);
#pragma unroll 1
        for (int i = 0; i < kTileBlocks; ++i) {
          float z[N];
          Elem<T>::unpack(q[0], z);
          q[0] = q[1], q[1] = q[2], q[2] = q[3];
#pragma unroll
          for (int e = 0; e < N; ++e) add(z[e]);
        }
      }
    }
    sync_all<CLUSTER>();
  }

  // The key of the first entry of a bin.
  __device__ __forceinline__ uint32_t key_at(const Level& l, int bin) const {
    if (l.shift < 0) return 0x8000ffffu | (kWindowTop - bin) << 16;
    return top - (l.d0 + (static_cast<uint32_t>(bin) << l.shift));
  }

  // The cluster's sums of the bins that the CTAs have counted: this thread's, and what lies before them.
  __device__ __forceinline__ void add_up(const Level& l) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    const bool single = l.shift < 0 ? sizeof(T) == 2 : l.shift <= kSingle;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      n[i] = 0;
      w[i] = 0;
    }
    const int own = threadIdx.x * kOwn;
#pragma unroll 4
    for (int r = 0; r < C; ++r) {
#pragma unroll
      for (int i = 0; i < kOwn; i += 2) {
        // the window's patterns rise where its bins fall
        const unsigned long long two = of_cta<CLUSTER>(&sh.count[l.shift < 0 ? kBins - 2 - own - i : own + i], r);
        const uint32_t a = static_cast<uint32_t>(two), b = static_cast<uint32_t>(two >> 32);
        n[i] += l.shift < 0 ? b : a;
        n[i + 1] += l.shift < 0 ? a : b;
      }
    }
    if (masses && !single && l.shift >= 0)
      for (int r = 0; r < C; ++r) {
#pragma unroll
        for (int i = 0; i < kOwn; i += 2) {
          const unsigned long long lo = of_cta<CLUSTER>(&sh.low[own + i], r), hi = of_cta<CLUSTER>(&sh.high[own + i], r);
          w[i] += (hi << 32) + (lo & 0xffffffffu);
          w[i + 1] += (hi & 0xffffffff00000000ull) + (lo >> 32);
        }
      }
    uint32_t mine_n = 0;
    unsigned long long mine_w = 0;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      // (of an fp32 row's window at least that: a bin's smallest value)
      if (masses && (single || l.shift < 0) && n[i] != 0)
        w[i] = n[i] * mass_of(weight(value_of(l.shift < 0 ? key_at(l, own + i) & 0xffff0000u : entry_key<T>(key_at(l, own + i)))));
      mine_n += n[i];
      mine_w += w[i];
    }
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
    // the warps' sums, by every warp: a lane each
    uint32_t of_n = lane < WARPS ? sh.warp_count[lane] : 0u;
    unsigned long long of_w = masses && lane < WARPS ? sh.warp_mass[lane] : 0ull;
#pragma unroll
    for (int o = 1; o < WARPS; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, of_n, o);
      if (lane >= o) of_n += x;
    }
    if (masses)
#pragma unroll
      for (int o = 1; o < WARPS; o <<= 1) {
        const unsigned long long x = __shfl_up_sync(0xffffffffu, of_w, o);
        if (lane >= o) of_w += x;
      }
    all_n = __shfl_sync(0xffffffffu, of_n, WARPS - 1);
    all_w = __shfl_sync(0xffffffffu, of_w, WARPS - 1);
    const uint32_t prev_n = __shfl_sync(0xffffffffu, of_n, max(warp - 1, 0));
    const unsigned long long prev_w = __shfl_sync(0xffffffffu, of_w, max(warp - 1, 0));
    run_n += above - mine_n + (warp ? prev_n : 0u);
    run_w += mass - mine_w + (warp ? prev_w : 0ull);
  }

  // Sorts the first `size` (a power of two) of the list, by all threads.
  __device__ __forceinline__ void sort_list(int size) {
    for (int k = 2; k <= size; k *= 2)
      for (int j = k / 2; j > 0; j /= 2) {
        for (int i = threadIdx.x; i < size / 2; i += kThreads) {
          const int x = 2 * i - (i & (j - 1)), y = x + j;  // the i-th pair at distance j
          const unsigned long long a = sh.list[x], b = sh.list[y];
          if ((a > b) == ((x & k) == 0)) {
            sh.list[x] = b;
            sh.list[y] = a;
          }
        }
        __syncthreads();
      }
  }
  // Fills the list up to a power of two behind its first `have`.
  __device__ __forceinline__ int fill_list(int have) {
    int size = 32;
    while (size < have) size *= 2;
    for (int i = have + threadIdx.x; i < size; i += kThreads) sh.list[i] = ~0ull;
    __syncthreads();
    return size;
  }

  // For an fp32 row whose window says that few entries can be kept: they are listed, so that the levels of a search count them
  // and not the row's; and the fewest are gathered in the first CTA and sorted by size, the border is read off the running
  // mass, what is kept is sorted by index, and the token is found by a scan: the row is done (true). `least`: min_p, as an
  // exponent. Measured, 254 rows of 151,936, listed / by levels over the row: the 50 largest 45 / 115 us, 0.4 of the mass 101 / 218.
  __device__ __forceinline__ bool finish_by_list(int32_t top_k, float top_p, float least, const Args& p, int64_t out, float u,
                                                 const T* z_row, const float* tile_max) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, rank = CLUSTER ? static_cast<int>(cluster_ctarank()) : 0;
    const Level level{0u, -1};
    add_up(level);
    if (threadIdx.x == 0) {
      sh.bin = -1;
      sh.n_list = 0;
      sh.n_equal = 0;
      sh.first = Shared<WARPS>::kSort;
      sh.last = 0;
    }
    __syncthreads();
    {
      // the bin by whose end top_k entries, or certainly top_p of the mass, have come
      const unsigned long long goal = static_cast<unsigned long long>(static_cast<double>(top_p) * static_cast<double>(all.s) * kMassUnit * (1.0 + 4e-6));
      uint32_t a = run_n;
      unsigned long long m = run_w;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        if (top_k ? a < top_k && a + n[i] >= top_k : m < goal && m + w[i] >= goal) {
          sh.bin = threadIdx.x * kOwn + i;
          sh.found.above = a + n[i];
        }
        a += n[i];
        m += w[i];
      }
    }
    __syncthreads();
    const int bin = sh.bin;
    const uint32_t most = sh.found.above;
    constexpr int kSort = Shared<WARPS>::kSort, kEach = kSort > kThreads ? kSort / kThreads : 1;
    if (bin < 0 || most > Shared<WARPS>::kList) return false;  // the same in every CTA
    const float edge = value_of(key_at(level, bin) & 0xffff0000u);
    for (int t = t0 + warp; t < t1; t += WARPS) {
      if (!(tile_max[t - t0] >= edge)) continue;
      uint4 q[kTileBlocks];
      row.tile(t, lane, q);
#pragma unroll
      for (int i = 0; i < kTileBlocks; ++i) {
        float z[N];
        Elem<T>::unpack(q[i], z);
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (z[e] >= edge)
            sh.list[atomicAdd(&sh.n_list, 1u)] =
                static_cast<unsigned long long>(~key_of(z[e])) << 32 | static_cast<uint32_t>((t * kTileBlocks32 + 32 * i + lane) * N + e);
      }
    }
    sync_all<CLUSTER>();
    if (most > kSort) {
      listed = true;
      return false;
    }
    int have = static_cast<int>(sh.n_list);
    if (rank == 0)
      for (int r = 1; r < C; ++r) {
        const int more = static_cast<int>(static_cast<uint32_t>(ld_cluster_u64(map_to_rank(smem_addr(&sh.n_list), r))));
        for (int i = threadIdx.x; i < more; i += kThreads) sh.list[have + i] = ld_cluster_u64(map_to_rank(smem_addr(&sh.list[i]), r));
        have += more;
      }
    if (CLUSTER) cluster_sync_all();
    if (rank != 0) return true;
    sort_list(fill_list(have));
    const int own = threadIdx.x * kEach;
    // the number kept: top_k's, then top_p's of the running mass, then min_p's
    if (threadIdx.x == 0) sh.bin = top_k ? top_k - 1 : have - 1;  // the last one
    if (masses) {
      unsigned long long v[kEach], mine = 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        v[i] = own + i < have ? mass_of(weight(value_of(~static_cast<uint32_t>(sh.list[own + i] >> 32)))) : 0;
        mine += v[i];
      }
      unsigned long long run = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long a = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += a;
      }
      if (lane == 31) sh.warp_mass[warp] = run;
      __syncthreads();
      run -= mine;
      for (int w = 0; w < warp; ++w) run += sh.warp_mass[w];
      unsigned long long upto = run;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        upto += v[i];
        if (top_k && own + i == top_k - 1) sh.total = upto;
      }
      __syncthreads();
      const double total = top_k ? static_cast<double>(sh.total) : static_cast<double>(all.s) * kMassUnit;
      const unsigned long long goal = max(1ull, static_cast<unsigned long long>(ceil(static_cast<double>(top_p) * total)));
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        if (run < goal && run + v[i] >= goal && own + i < have) atomicMin(&sh.bin, own + i);
        run += v[i];
      }
    }
    __syncthreads();
    int kept = sh.bin + 1;
    if (least > minus_inf()) {
      uint32_t over = 0;
      for (int i = threadIdx.x; i < kept; i += kThreads)
        over += exponent(value_of(~static_cast<uint32_t>(sh.list[i] >> 32)), all.m, c) >= least;
      if (over) atomicAdd(&sh.n_equal, over);
      __syncthreads();
      kept = max(1, static_cast<int>(sh.n_equal));
    }
    // the kept ones by index, with their weights
    for (int i = threadIdx.x; i < kept; i += kThreads) {
      const unsigned long long e = sh.list[i];
      sh.list[i] = e << 32 | __float_as_uint(weight(value_of(~static_cast<uint32_t>(e >> 32))));
    }
    sort_list(fill_list(kept));
    float v[kEach], mine = 0.f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      v[i] = own + i < kept ? __uint_as_float(static_cast<uint32_t>(sh.list[own + i])) : 0.f;
      mine += v[i];
    }
    float run = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const float a = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += a;
    }
    if (lane == 31) sh.warp_sum[warp] = run;
    __syncthreads();
    float before = 0.f, total = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float a = sh.warp_sum[w];
      before += w < warp ? a : 0.f;
      total += a;
    }
    run += before - mine;
    const float goal = u * total;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      run += v[i];
      if (v[i] > 0.f) {
        atomicMax(&sh.last, own + i);  // where rounding leaves the sum short of its goal
        if (run > goal) atomicMin(&sh.first, own + i);
      }
    }
    __syncthreads();
    if (warp == 0) {
      const int at = sh.first < kSort ? sh.first : sh.last;
      const int token = min(max(static_cast<int>(sh.list[at] >> 32) - row.lo, 0), p.V - 1);
      const float zx = Elem<T>::one(z_row[token]);
      float others = 0.f;  // while the token's entry is on its way
      if (p.among)
        for (int i = lane; i < kept; i += 32) others += i != at ? __uint_as_float(static_cast<uint32_t>(sh.list[i])) : 0.f;
      others = warp_sum(others);
      if (lane != 0) return true;
      p.ids[out] = token;
      p.logp[out] = logp_of(zx, all, c);
      if (p.among) p.among[out] = log_share(exponent(zx, all.m, c), others, total);
      if (p.n_kept) p.n_kept[out] = kept;
    }
    return true;
  }

  // The border of what top_k (0: off) and top_p (1: off) keep of the row; false: they keep everything. `first`: the level
  // to begin with, counted already if it is the window.
  __device__ __forceinline__ bool search(int32_t top_k, float top_p, const Level& first, Border& found) {
    bool any = false, by_mass = top_k == 0, fresh = true;
    auto mass_goal = [&](double total) { return max(1ull, static_cast<unsigned long long>(ceil(static_cast<double>(top_p) * total))); };
    unsigned long long goal = by_mass ? mass_goal(static_cast<double>(all.s) * kMassUnit) : static_cast<unsigned long long>(top_k);
    Level outer = first, to = first;
    while (true) {
      if (fresh) {
        if (to.shift >= 0) count(to);
        add_up(to);
      }
      fresh = true;
      if (threadIdx.x == 0) sh.bin = -1;
      __syncthreads();
      const int shift = to.shift < 0 ? kBf16Shift : to.shift;
      uint32_t a = run_n, a_hit = 0, n_hit = 0;
      unsigned long long m = run_w, m_hit = 0, w_hit = 0;
      int hit = -1;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        if (by_mass ? m < goal && m + w[i] >= goal : a < goal && a + n[i] >= goal) {
          hit = threadIdx.x * kOwn + i;
          a_hit = a, m_hit = m, n_hit = n[i], w_hit = w[i];
        }
        a += n[i];
        m += w[i];
      }
      if (hit >= 0) {  // one thread of all: the bin's border, if it is of one value
        Border f{entry_key<T>(key_at(to, hit)), n_hit, a_hit, m_hit, 0};
        if (shift <= kSingle) {
          f.unit = w_hit / n_hit;  // w is n times the value's mass
          if (!by_mass) f.m = static_cast<uint32_t>(goal) - a_hit;
          else f.m = static_cast<uint32_t>(min(static_cast<unsigned long long>(n_hit), (goal - m_hit + f.unit - 1) / f.unit));
        }
        sh.found = f;
        sh.bin = hit;
      }
      __syncthreads();
      const int bin = sh.bin;
      Border b = sh.found;
      __syncthreads();  // and may be written again
      bool none = false;
      const bool outermost = to.d0 == outer.d0 && to.shift == outer.shift;
      if (bin < 0) {
        none = !outermost;
        if (!none) {
          // not among the nearest: all that is farther away
          above += all_n;
          mass += all_w;
          to = Level{to.shift < 0 ? top - (0x8000ffffu | (kWindowLow - 1) << 16) : static_cast<uint32_t>(kBins) << kBf16Shift, kRestShift};
          continue;
        }
      } else {
        if (shift > kSingle) {
          const uint32_t k = key_at(to, bin);  // the window's first bin may reach above the largest
          above = b.above;
          mass = b.mass;
          to = Level{k > top ? 0u : top - k, max(0, shift - kBinBits)};
          continue;
        }
        found = b;
        any = true;
      }
      if (by_mass || top_p >= 1.f) return any;
      // then top_p, of the mass of what top_k keeps
      by_mass = true;
      goal = mass_goal(none ? static_cast<double>(all.s) * kMassUnit : static_cast<double>(b.mass + b.m * b.unit));
      fresh = !outermost;
      if (fresh) {
        above = 0;
        mass = 0;
        to = outer = Level{0u, kBf16Shift};  // the window's bins, if it had any, are gone
      }
    }
  }
};

// The smallest key of an entry of this type whose exponent is at least `least`.
template <typename T, typename X>
__device__ __forceinline__ uint32_t least_key(uint32_t top, float least, X exponent_of) {
  auto widen = [](uint32_t i) { return sizeof(T) == 4 ? i : i << 16 | (i & 0x8000u ? 0u : 0xffffu); };
  uint32_t lo = sizeof(T) == 4 ? 0x00800000u : 0x80u, hi = sizeof(T) == 4 ? top : top >> 16;  // the lowest finite; one that is
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (exponent_of(value_of(widen(mid))) >= least) hi = mid;
    else lo = mid + 1;
  }
  return widen(hi);
}

// As pick, but with the goal itself: the place among n weights w(k) at which their running sum passes `goal`; whether it does
// (rounding may leave it short); and the sum of the lane's other weights.
struct Picked {
  int at;
  float left, others;
  bool passed;
};
template <typename W>
__device__ __forceinline__ Picked pick_at(int n, float goal, int lane, W w) {
  const int M = (n + 31) / 32, k0 = min(lane * M, n), k1 = min(k0 + M, n);
  float sum = 0.f;
  for (int k = k0; k < k1; ++k) sum += w(k);
  float run = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const float up = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += up;
  }
  float before = run - sum, rest = 0.f, last_rest = 0.f, others = 0.f;
  int at = -1, last = -1;
  for (int k = k0; k < k1; ++k) {
    const float mine = w(k);
    bool here = false;
    if (mine > 0.f) {
      last = k;
      last_rest = goal - before;
      here = at < 0 && before + mine > goal;
      if (here) {
        at = k;
        rest = last_rest;
      }
    }
    others += here ? 0.f : mine;
    before += mine;
  }
  const uint32_t found = __ballot_sync(0xffffffffu, at >= 0), any = __ballot_sync(0xffffffffu, last >= 0);
  const int from = found ? __ffs(found) - 1 : any ? 31 - __clz(any) : 0;
  return {max(0, __shfl_sync(0xffffffffu, found ? at : last, from)), __shfl_sync(0xffffffffu, found ? rest : last_rest, from),
          lane == from ? others : sum, found != 0};
}

// What a pass over the row keeps: entries above (GE: and at) zt.
template <typename T, bool GE>
struct Keep {
  static constexpr int N = Elem<T>::N;
  float zt, ref, c;
  // Whether a block has an entry of at least zt.
  __device__ __forceinline__ bool reaches(const uint4& q) const {
    if constexpr (sizeof(T) == 2) {
      const uint32_t t = __float_as_uint(zt) >> 16, t2 = t | t << 16;
      return (least2(q.x, t2) | least2(q.y, t2) | least2(q.z, t2) | least2(q.w, t2)) != 0;
    } else {
      return fmaxf(fmaxf(__uint_as_float(q.x), __uint_as_float(q.y)), fmaxf(__uint_as_float(q.z), __uint_as_float(q.w))) >= zt;
    }
  }
  // Adds the number of a block's kept entries: pairs of counts of 16 bits.
  __device__ __forceinline__ void number(const uint4& q, uint32_t& n) const {
    if constexpr (sizeof(T) == 2) {
      const uint32_t t = __float_as_uint(zt) >> 16, t2 = t | t << 16;
      n += (above2(q.x, t2) & 0x00010001u) + (above2(q.y, t2) & 0x00010001u) + (above2(q.z, t2) & 0x00010001u) + (above2(q.w, t2) & 0x00010001u);
    } else {
      n += (__uint_as_float(q.x) > zt) + (__uint_as_float(q.y) > zt) + (__uint_as_float(q.z) > zt) + (__uint_as_float(q.w) > zt);
    }
  }
  // A block's kept entries, the others minus infinity. Adds the number of those equal to zt (not GE) to `equal`, and
  // with `count` that of the kept ones to `kept`, both pairs of counts of 16 bits.
  __device__ __forceinline__ void block(const uint4& q, float (&z)[N], uint32_t& equal, uint32_t& kept, bool count) const {
    if constexpr (sizeof(T) == 2) {
      const uint32_t t = __float_as_uint(zt) >> 16, t2 = t | t << 16;
      const uint32_t v[4] = {q.x, q.y, q.z, q.w};
      uint32_t m[4], r[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t ge = least2(v[i], t2);
        m[i] = GE ? ge : above2(v[i], t2);
        r[i] = (v[i] & m[i]) | (0xff80ff80u & ~m[i]);
        if (!GE) equal += (ge ^ m[i]) & 0x00010001u;
        if (count) kept += m[i] & 0x00010001u;
      }
      Elem<T>::unpack(make_uint4(r[0], r[1], r[2], r[3]), z);
    } else {
      Elem<T>::unpack(q, z);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const bool in = GE ? z[e] >= zt : z[e] > zt;
        if (!GE) equal += z[e] == zt;
        if (count) kept += in;
        z[e] = in ? z[e] : minus_inf();
      }
    }
  }
  // The kept weights of a lane's blocks of a tile.
  __device__ __forceinline__ float tile(const uint4 (&q)[kTileBlocks], uint32_t& equal, uint32_t& kept, bool count) const {
    const float rc = -__fmul_rn(ref, c);
    const float2 cc = make_float2(c, c), off = make_float2(rc, rc);
    float2 s = make_float2(0.f, 0.f);
    if (large(rc)) {  // of the row
#pragma unroll 1
      for (int i = 0; i < kTileBlocks; ++i) {
        float z[N];
        block(i < 2 ? (i == 0 ? q[0] : q[1]) : (i == 2 ? q[2] : q[3]), z, equal, kept, count);
#pragma unroll
        for (int e = 0; e < N; ++e) s.x += ex2((z[e] - ref) * c);
      }
      return s.x;
    }
#pragma unroll
    for (int i = 0; i < kTileBlocks; ++i) {
      if (!__any_sync(0xffffffffu, reaches(q[i]))) continue;  // most blocks of most rows
      float z[N];
      block(q[i], z, equal, kept, count);
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        const float2 x = __ffma2_rn(make_float2(z[e], z[e + 1]), cc, off);
        s = __fadd2_rn(s, make_float2(ex2(x.x), ex2(x.y)));
      }
    }
    return s.x + s.y;
  }
};
// The same for a bf16 row that keeps few entries: a lane takes the ones of at least zt of a block one after the other.
__device__ __forceinline__ float few_of_tile(const uint4 (&q)[kTileBlocks], float zt, float ref, float c, uint32_t& equal) {
  const uint32_t t = __float_as_uint(zt) >> 16, t2 = t | t << 16;
  const float rc = -__fmul_rn(ref, c);
  const bool apart = large(rc);  // of the row
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kTileBlocks; ++i) {
    // bit w: the low half of word w, bit 16 + w: the high one
    uint32_t b = (least2(q[i].x, t2) & 0x00010001u) | (least2(q[i].y, t2) & 0x00020002u) | (least2(q[i].z, t2) & 0x00040004u) |
                 (least2(q[i].w, t2) & 0x00080008u);
    while (b) {
      const int k = __ffs(b) - 1;
      b &= b - 1;
      const uint32_t w = k & 2 ? (k & 1 ? q[i].w : q[i].z) : (k & 1 ? q[i].y : q[i].x);
      const float z = k & 16 ? bf16_hi(w) : bf16_lo(w);
      if (z > zt) s += ex2(apart ? (z - ref) * c : fmaf(z, c, rc));
      else ++equal;
    }
  }
  return s;
}

// The sum of a warp's pairs of counts of 16 bits.
__device__ __forceinline__ uint32_t of_pairs(uint32_t n) { return __reduce_add_sync(0xffffffffu, (n & 0xffffu) + (n >> 16)); }

// One more of the bins of the window of a pair of patterns, both halves at a time: the smaller of a pattern's distance from
// the window's lowest, which wraps for lower ones, and of a word behind the bins, a lane's own (a condition on the
// addition costs more than the addition).
__device__ __forceinline__ void count_patterns(uint32_t bins, uint32_t pair, uint32_t behind, uint32_t one) {
  const uint32_t i = __viaddmin_u16x2(pair, ((0x10000u - kWindowLow) << 16) | (0x10000u - kWindowLow), behind);
  asm volatile("red.shared.add.u32 [%0], %1;" :: "r"(bins + (i & 0xffffu) * 4u), "r"(one) : "memory");
  asm volatile("red.shared.add.u32 [%0], %1;" :: "r"(bins + (i >> 16) * 4u), "r"(one) : "memory");
}
__device__ __forceinline__ void count_pattern(uint32_t bins, uint32_t pattern, uint32_t behind, uint32_t one) {
  const uint32_t i = min(pattern - kWindowLow, behind & 0xffffu);
  asm volatile("red.shared.add.u32 [%0], %1;" :: "r"(bins + i * 4u), "r"(one) : "memory");
}

// As add_tile, with the exponents' form decided once for the tile; the largest of the lane's entries.
template <typename T>
__device__ __forceinline__ float fold_tile(Running& r, const uint4 (&w)[kTileBlocks], float c) {
  constexpr int N = Elem<T>::N;
  const float top = largest<T>(w);
  if (top > r.m) {
    const float f = power(r.m, top, c);
    r.s.x *= f;
    r.s.y *= f;
    r.m = top;
  }
  const float ref = r.m == minus_inf() ? 0.f : r.m, rc = -__fmul_rn(ref, c);
  if (large(rc)) {
#pragma unroll 1
    for (int i = 0; i < kTileBlocks; ++i) {
      float z[N];
      Elem<T>::unpack(i < 2 ? (i == 0 ? w[0] : w[1]) : (i == 2 ? w[2] : w[3]), z);
#pragma unroll
      for (int e = 0; e < N; ++e) r.s.x += ex2((z[e] - ref) * c);
    }
    return top;
  }
  const float2 cc = make_float2(c, c), off = make_float2(rc, rc);
  float2 s0 = make_float2(0.f, 0.f), s1 = s0;  // two chains
#pragma unroll
  for (int i = 0; i < kTileBlocks; ++i) {
    float z[N];
    Elem<T>::unpack(w[i], z);
#pragma unroll
    for (int e = 0; e < N; e += 4) {
      const float2 a = __ffma2_rn(make_float2(z[e], z[e + 1]), cc, off), b = __ffma2_rn(make_float2(z[e + 2], z[e + 3]), cc, off);
      s0 = __fadd2_rn(s0, make_float2(ex2(a.x), ex2(a.y)));
      s1 = __fadd2_rn(s1, make_float2(ex2(b.x), ex2(b.y)));
    }
  }
  r.s = add2(r.s, add2(s0, s1));
  return top;
}

template <typename T, int WARPS, bool CLUSTER>
__global__ void __launch_bounds__(WARPS * 32, 1024 / (WARPS * 32)) sample_kernel(const Args p) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(16) Shared<WARPS> sh;
  Tile* tiles = reinterpret_cast<Tile*>(smem);
  float* tile_max = reinterpret_cast<float*>(tiles + p.tiles);
  constexpr int N = Elem<T>::N;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = CLUSTER ? static_cast<int>(cluster_ctarank()) : 0, C = CLUSTER ? static_cast<int>(cluster_nctarank()) : 1;
  const int64_t r = blockIdx.x / C;
  const T* z = static_cast<const T*>(p.logits) + r * p.ld;
  const RowBlocks<T> row(z, p.V);
  const int all_tiles = (row.nb + kTileBlocks32 - 1) / kTileBlocks32;
  const int t0 = min(rank * p.tiles, all_tiles), t1 = min(t0 + p.tiles, all_tiles);
  if (CLUSTER) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // the other CTAs have started
  uint4 q[kTileBlocks];
  if (t0 + warp < t1) row.tile(t0 + warp, lane, q);
  Settings set{p.temperature, p.top_p, p.min_p, p.u[r], p.top_k};
  if (p.row_temperature) set.T = p.row_temperature[r];
  if (p.row_top_k) set.top_k = p.row_top_k[r];
  if (p.row_top_p) set.top_p = p.row_top_p[r];
  if (p.row_min_p) set.min_p = p.row_min_p[r];
  for (int i = threadIdx.x; i < kBins; i += WARPS * 32) sh.count[i] = 0;
  __syncthreads();
  const bool greedy = set.T == 0.f, known = set.ok();
  const float c = greedy || !known ? kLog2e : kLog2e / set.T;
  const bool by_k = !greedy && set.top_k > 0 && set.top_k < p.V, by_p = !greedy && set.top_p < 1.f;
  const bool by_m = !greedy && set.min_p > 0.f, filtered = greedy || by_k || by_p || by_m;
  const bool window = by_k || by_p;

  // ---- the row's largest entry and its normaliser
  const uint32_t bins = smem_addr(sh.count), behind = (kBins + lane) * 0x10001u;
  uint32_t one;
  asm volatile("mov.u32 %0, 1;" : "=r"(one));
  Running run{minus_inf(), {0.f, 0.f}, 0};
  Fold f{minus_inf(), 0.f};
  const bool count_all = !filtered && p.n_kept;
  uint32_t live = 0;  // entries above minus infinity
  for (int t = t0 + warp; t < t1; t += WARPS) {
    uint4 now[kTileBlocks];
#pragma unroll
    for (int i = 0; i < kTileBlocks; ++i) now[i] = q[i];
    if (t + WARPS < t1) row.tile(t + WARPS, lane, q);
    const float most = redux_max(fold_tile<T>(run, now, c));
    if (filtered && lane == 0) tile_max[t - t0] = most;
    if (window) {
#pragma unroll
      for (int i = 0; i < kTileBlocks; ++i) {
        const uint32_t v[4] = {now[i].x, now[i].y, now[i].z, now[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (sizeof(T) == 2) count_patterns(bins, v[e], behind, one);
          else count_pattern(bins, v[e] >> 16, behind, one);
        }
      }
    } else if (!filtered) {
      if (count_all) {
#pragma unroll
        for (int i = 0; i < kTileBlocks; ++i) Keep<T, false>{minus_inf(), 0.f, 1.f}.number(now[i], live);
      }
      const Fold of = of_warp(run, c);
      if (lane == 0) tiles[t - t0].fold = of;
      const float m = fmaxf(f.m, of.m);
      f.s = (f.s == 0.f ? 0.f : f.s * power(f.m, m, c)) + (of.s == 0.f ? 0.f : of.s * power(of.m, m, c));
      f.m = m;
      run = Running{minus_inf(), {0.f, 0.f}, 0};
    }
  }
  if (filtered) f = of_warp(run, c);
  if (CLUSTER) {
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (lane < C) put_f2(map_to_rank(smem_addr(&sh.fold[rank * WARPS + warp]), lane), f.m, f.s);
    __syncwarp();
  } else if (lane == 0) {
    sh.fold[warp] = f;
  }
  sync_all<CLUSTER>();
  if (warp == 0) {
    const Fold all = merged(sh.fold, C * WARPS, c, lane);
    if (lane == 0) {
      sh.all = all;
      if (by_m && !is_bad(all) && known) {
        // min_p, as an exponent from that of the largest entry, which the rounding of its product moves as all others
        auto x = [&](float v) { return exponent(v, all.m, c); };
        sh.least_key = least_key<T>(key_of(all.m), x(all.m) + log2f(set.min_p), x);
      }
    }
  }
  __syncthreads();
  const Fold all = sh.all;
  if (is_bad(all) || !known) {  // the whole cluster
    if (rank == 0 && threadIdx.x == 0) {
      flag_status(p.status, RL_DEV_BAD_VALUE);
      p.ids[r] = -1;
      p.logp[r] = __int_as_float(0x7fc00000);
      if (p.among) p.among[r] = __int_as_float(0x7fc00000);
      if (p.n_kept) p.n_kept[r] = 0;
    }
    return;
  }

  // ---- the threshold: entries above zt are kept, and the first ties of those equal to it (GE: all of them)
  float zt = minus_inf();
  uint32_t ties = 0;
  uint32_t kept = 0;
  bool known_kept = false, ge = false;
  if (greedy) {
    zt = all.m;
    ties = 1;
    kept = 1;
    known_kept = true;
  } else if (by_k || by_p) {
    const uint32_t top = key_of(all.m);
    Row<T, WARPS, CLUSTER> s{sh, row, t0, t1, all, c, top, C, by_p};
    Border b;
    const bool in_window = top >= (0x80000000u | kWindowLow << 16) && top <= (0x8000ffffu | kWindowTop << 16);
    if (sizeof(T) == 4 && in_window) {
      const float least = by_m ? exponent(all.m, all.m, c) + log2f(set.min_p) : minus_inf();
      if (s.finish_by_list(by_k ? set.top_k : 0, set.top_p, least, p, r, set.u, z, tile_max)) return;
    }
    const bool is = s.search(by_k ? set.top_k : 0, set.top_p, in_window && (sizeof(T) == 2 || (!by_p && !s.listed)) ? Level{0u, -1} : Level{0u, kBf16Shift}, b);
    if (is) {
      zt = value_of(b.key);
      ties = b.m;
      kept = b.above + b.m;
      known_kept = true;
    }
  }
  if (by_m && value_of(sh.least_key) > zt) {
    zt = value_of(sh.least_key);
    ge = true;
    ties = 0;
    known_kept = false;
  }

  // ---- the kept weights of every tile
  const bool count = p.n_kept && !known_kept;
  if (filtered) {
    float sum = 0.f;
    uint32_t equal = 0, above = 0;
    const bool sparse = sizeof(T) == 2 && known_kept && kept <= static_cast<uint32_t>(p.V) / 16;
    auto over = [&](const auto& keep) {
      // this warp's tiles that have an entry to keep; the ones read last first: they are the likeliest to be in L2 still
      const int first = t0 + warp;
      auto before = [&](int t) {
        for (; t >= first; t -= WARPS) {
          if (tile_max[t - t0] >= zt) break;
          if (lane == 0) tiles[t - t0].kept = {0.f, 0u};
        }
        return t;
      };
      int t = first < t1 ? before(first + (t1 - 1 - first) / WARPS * WARPS) : first - WARPS;
      if (t >= first) row.tile(t, lane, q);
      while (t >= first) {
        uint4 now[kTileBlocks];
#pragma unroll
        for (int i = 0; i < kTileBlocks; ++i) now[i] = q[i];
        const int here = t;
        t = before(t - WARPS);
        if (t >= first) row.tile(t, lane, q);
        uint32_t eq = 0;
        const float s = warp_sum(sparse ? few_of_tile(now, zt, all.m, c, eq) : keep.tile(now, eq, above, count));
        eq = of_pairs(eq);
        if (lane == 0) tiles[here - t0].kept = {s, eq};
        sum += s;
        equal += eq;
      }
    };
    if (ge) over(Keep<T, true>{zt, all.m, c});
    else over(Keep<T, false>{zt, all.m, c});
    above = of_pairs(above);
    if (lane == 0) {
      sh.warp_sum[warp] = sum;
      sh.warp_equal[warp] = equal;
      sh.warp_above[warp] = above;
    }
  } else {
    live = of_pairs(live);
    if (lane == 0) {
      sh.warp_sum[warp] = f.s == 0.f ? 0.f : f.s * power(f.m, all.m, c);
      sh.warp_equal[warp] = 0;
      sh.warp_above[warp] = live;
    }
  }
  __syncthreads();
  if (warp == 0) {
    float sum = lane < WARPS ? sh.warp_sum[lane] : 0.f;
    sum = warp_sum(sum);
    const uint32_t equal = __reduce_add_sync(0xffffffffu, lane < WARPS ? sh.warp_equal[lane] : 0u);
    const uint32_t above = __reduce_add_sync(0xffffffffu, lane < WARPS ? sh.warp_above[lane] : 0u);
    if (!CLUSTER) {
      if (lane == 0) {
        sh.part_a[0] = make_uint2(__float_as_uint(sum), equal);
        sh.part_b[0] = above;
      }
    } else if (lane < C) {
      put_u2(map_to_rank(smem_addr(&sh.part_a[rank]), lane), __float_as_uint(sum), equal);
      asm volatile("st.shared::cluster.u32 [%0], %1;" :: "r"(map_to_rank(smem_addr(&sh.part_b[rank]), lane)), "r"(above) : "memory");
    }
    __syncwarp();
  }
  if (CLUSTER) cluster_sync_all();
  if (warp != 0) return;

  // ---- the CTA that holds the token, by the first warp of each alike
  const float wt = ties ? ex2(exponent(zt, all.m, c)) : 0.f;
  const Part part = lane < C ? Part{__uint_as_float(sh.part_a[lane].x), sh.part_a[lane].y, sh.part_b[lane]} : Part{0.f, 0u, 0u};
  uint32_t upto = part.equal;
#pragma unroll
  for (int o = 1; o < kMostCluster; o <<= 1) {
    const uint32_t a = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += a;
  }
  const uint32_t before = upto - part.equal, mine_ties = before >= ties ? 0u : min(ties - before, part.equal);
  const float mine = fmaf(static_cast<float>(mine_ties), wt, part.sum);
  const float total = warp_sum(mine);
  const Picked cta = pick_at(C, set.u * total, lane, [&](int) { return mine; });  // a lane has one
  if (cta.at != rank) return;
  // Not under the condition that the number is wanted. Built so (nvcc 13.0.88), a known number came out as the sum, 0, and under
  // a vote on the condition an unknown one as 0 too, though the condition is the same in all lanes: with a ballot of it
  // in the code, or with the sum taken by shuffles, the results are right. No kernel smaller than this one shows it.
  // (Intrinsic and redux.sync alike, so what follows the PTX.)
  const uint32_t counted = __reduce_add_sync(0xffffffffu, part.above);
  const uint32_t ties_before = __shfl_sync(0xffffffffu, before, rank);

  // ---- its tile
  const int nt = t1 - t0, M = (nt + 31) / 32, k0 = min(lane * M, nt), k1 = min(k0 + M, nt);
  uint32_t rank_eq = 0;
  if (ties)
    for (int k = k0; k < k1; ++k) rank_eq += tiles[k].kept.equal;
  uint32_t eq_run = rank_eq;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t a = __shfl_up_sync(0xffffffffu, eq_run, o);
    if (lane >= o) eq_run += a;
  }
  const uint32_t lane_before = ties_before + eq_run - rank_eq;
  auto ties_until = [&](int k) {  // entries equal to the threshold before tile k of this lane's
    uint32_t b = lane_before;
    for (int i = k0; i < k; ++i) b += tiles[i].kept.equal;
    return b;
  };
  const Picked tile = pick_at(nt, cta.left, lane, [&](int k) {
    if (!filtered) return tiles[k].fold.s == 0.f ? 0.f : tiles[k].fold.s * power(tiles[k].fold.m, all.m, c);
    if (!ties) return tiles[k].kept.sum;
    const uint32_t b = ties_until(k);
    return fmaf(b >= ties ? 0.f : static_cast<float>(min(ties - b, tiles[k].kept.equal)), wt, tiles[k].kept.sum);
  });
  const int at = tile.at;
  const float left = tile.left;
  uint32_t used = ties ? __shfl_sync(0xffffffffu, at >= k0 && at < k1 ? ties_until(at) : 0u, at / M) : 0u;

  // ---- and the token in it: the weights in order, ties by their rank
  row.tile(t0 + at, lane, q);
  int token = -1, last = -1;
  float acc0 = 0.f, others = cta.others + tile.others;  // the lane's part of what is kept beside the token
#pragma unroll
  for (int i = 0; i < kTileBlocks; ++i) {
    float v[N], w[N], s = 0.f;
    uint32_t eq = 0;
    Elem<T>::unpack(q[i], v);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      w[e] = (ge ? v[e] >= zt : v[e] > zt) ? v[e] : minus_inf();
      eq += ties && v[e] == zt;
    }
    exps(w, all.m, c);
    uint32_t eq_here = eq;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t a = __shfl_up_sync(0xffffffffu, eq_here, o);
      if (lane >= o) eq_here += a;
    }
    uint32_t nth = used + eq_here - eq;
    used += __shfl_sync(0xffffffffu, eq_here, 31);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if (ties && v[e] == zt) {
        if (nth < ties) w[e] = wt;
        ++nth;
      }
      s += w[e];
      if (w[e] > 0.f) last = ((t0 + at) * kTileBlocks32 + 32 * i + lane) * N + e;
    }
    float run_s = s;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const float a = __shfl_up_sync(0xffffffffu, run_s, o);
      if (lane >= o) run_s += a;
    }
    const uint32_t hit = __ballot_sync(0xffffffffu, token < 0 && s > 0.f && acc0 + run_s > left);
    if (hit) {
      const int from = __ffs(hit) - 1;
      float acc = acc0 + (run_s - s), beside = 0.f;
      int here = -1;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        acc += w[e];
        if (here < 0 && w[e] > 0.f && acc > left) here = ((t0 + at) * kTileBlocks32 + 32 * i + lane) * N + e;
      }
      if (here < 0) here = last;
#pragma unroll
      for (int e = 0; e < N; ++e) beside += here == ((t0 + at) * kTileBlocks32 + 32 * i + lane) * N + e ? 0.f : w[e];
      token = __shfl_sync(0xffffffffu, here, from);
      s = lane == from ? beside : s;
    }
    others += s;
    acc0 += __shfl_sync(0xffffffffu, run_s, 31);
  }
  // where rounding leaves the sum short of its goal: the last that has any weight
  const bool passed = cta.passed && tile.passed && token >= 0;
  if (token < 0) {  // (by shuffles: as above)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) last = max(last, __shfl_xor_sync(0xffffffffu, last, o));
    token = last;
  }
  token = min(max(token - row.lo, 0), p.V - 1);
  const float zx = Elem<T>::one(z[token]);
  others = warp_sum(others);
  if (lane != 0) return;
  p.ids[r] = token;
  p.logp[r] = logp_of(zx, all, c);
  if (p.among) {
    const float x = exponent(zx, all.m, c);
    p.among[r] = log_share(x, passed ? others : fmaxf(total - ex2(x), 0.f), total);
  }
  if (p.n_kept) p.n_kept[r] = static_cast<int32_t>(known_kept ? kept : counted);
}

// ---------------------------------------------------------------- host

constexpr int kSMs = 152;
constexpr int64_t kMostTiles = 2064;  // of a CTA: their tables take 24 KB beside the others
static_assert(sizeof(Shared<16>) + kMostTiles * 12 <= 100 * 1024 && sizeof(Shared<8>) <= 48 * 1024 && sizeof(Shared<16>) <= 48 * 1024,
              "two CTAs on an SM");

template <typename T, int WARPS, bool CLUSTER>
rl_status launch(Args& a, int C, int64_t all_tiles, cudaStream_t s) {
  a.tiles = static_cast<int32_t>((all_tiles + C - 1) / C);
  auto kern = sample_kernel<T, WARPS, CLUSTER>;
  // once per device
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_error(e, "cudaGetDevice");
  const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
  if (!(ready.load() & bit)) {
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(kMostTiles * (sizeof(Tile) + sizeof(float))));
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
  cfg.numAttrs = C > 1 ? 1 : 0;
  cfg.blockDim = dim3(WARPS * 32);
  cfg.gridDim = dim3(static_cast<unsigned>(a.rows * C));
  cfg.dynamicSmemBytes = static_cast<size_t>(a.tiles) * (sizeof(Tile) + sizeof(float));
  cfg.stream = s;
  e = cudaLaunchKernelEx(&cfg, kern, a);
  return e == cudaSuccess ? RL_OK : cuda_error(e, "sample_kernel launch");
}


template <typename T>
rl_status run(Args& a, cudaStream_t s) {
  const int64_t nb = (a.V + 7) * sizeof(T) / 16 + 1, tiles = (nb + kTileBlocks32 - 1) / kTileBlocks32;
  // many rows: small CTAs, which wait less for one another, and do what a row takes beside its entries with fewer warps
  // (their threads have eight bins each to sum up, and spill 96 bytes, fp32 148; the other forms 24 at most).
  // Measured, us by 8 / 4 warps, top-k 50: 2,000 rows of 32,000 bf16 80.5 / 70.2, 1,200 of 60,000 69.2 / 64.3, 1,000 of 32,000
  // fp32 50.9 / 41.8, but 600 of 32,000 bf16 25.4 / 27.0 and 509 of 151,936 62.0 / 64.4; by 16 / 8 warps 300 of 151,936 37.8 /
  // 41.7, 509 104 / 82
  if ((tiles <= 8 && a.rows > kSMs) || (tiles <= 64 && a.rows > 6 * kSMs)) return launch<T, 4, false>(a, 1, tiles, s);
  // else as many CTAs a row as fill the SMs twice over while each of their warps has a tile
  int C = 1;
  while (C < kMostCluster && ((a.rows * C * 2 <= 2 * kSMs && tiles >= 2 * C * 8) || tiles > kMostTiles * C)) C *= 2;
  if (tiles > kMostTiles * C) return set_error(RL_ERR_UNSUPPORTED, "rl_sample_tokens: V is too large");
  if (C > 1) return launch<T, 16, true>(a, C, tiles, s);
  return a.rows <= 2 * kSMs ? launch<T, 16, false>(a, 1, tiles, s) : launch<T, 8, false>(a, 1, tiles, s);
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
  if (V > (dtype == RL_BF16 ? 1 << 24 : 1 << 23) || rows > (1 << 26)) return set_error(RL_ERR_UNSUPPORTED, f + "at most 2^24 entries (fp32: 2^23) and 2^26 rows");
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
