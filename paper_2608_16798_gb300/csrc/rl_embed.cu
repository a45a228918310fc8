// The embedding of tokens, scaled, and its gradient.
//
//   out_t = scale W[id_t];      dW[v] += scale sum over the tokens t with id_t = v, in token order, of d_t
//
// The gradient's sums want the tokens of a row of W side by side: the tokens are sorted by id, stably (a radix sort in
// digits of up to 9 bits), the sorted list is cut into chunks of equal length whatever the ids, and a chunk's threads,
// a few columns each, go down its tokens. A run of equal ids is added up by the chunk in which it begins, up to a chunk's
// length into the next one; the parts of a longer run go to the workspace and are added up in order afterwards, so that a
// token that comes very often is shared by as many CTAs as it has chunks. Every element of dW gets one addition per call,
// and the order of all sums depends on the ids alone: repeated calls give the same bits. Up to 1,024 tokens are not sorted:
// every token's CTA looks for its like among all ids.
//
// Memory bounds both. Measured: 32,768 tokens of 4,096 columns, ids with frequencies that fall as 1 / rank over 151,936:
// forward 60 us (91% of the copy's rate over the rows that are named and written), backward 150 (the sort 17, the sums 118 at 80%
// of the copy's rate, the long runs 10). The digits' passes, chains of a few microseconds each, are what the sort costs.
// Rows that do not lie in 16-byte blocks, an element at a time: forward 72,544 x 1,792 bf16 in rows of 1,795 180 us.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <string>

#include "rl_device.cuh"
#include "rl_host.h"

namespace rl {
namespace embed {

// N elements as floats, from memory aligned for them.
template <typename T, int N>
struct Block;
template <>
struct Block<uint16_t, 8> {
  uint4 w;
  __device__ __forceinline__ void load(const uint16_t* p) { w = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void clear() { w = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = bf16_lo(w.x), v[1] = bf16_hi(w.x), v[2] = bf16_lo(w.y), v[3] = bf16_hi(w.y);
    v[4] = bf16_lo(w.z), v[5] = bf16_hi(w.z), v[6] = bf16_lo(w.w), v[7] = bf16_hi(w.w);
  }
  __device__ __forceinline__ void put(int e, uint16_t x) {  // into a cleared block
    uint32_t& word = e < 4 ? (e < 2 ? w.x : w.y) : (e < 6 ? w.z : w.w);
    word |= static_cast<uint32_t>(x) << (e & 1) * 16;
  }
};
template <>
struct Block<float, 4> {
  float4 w;
  __device__ __forceinline__ void load(const float* p) { w = __ldcs(reinterpret_cast<const float4*>(p)); }
  __device__ __forceinline__ void clear() { w = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(float (&v)[4]) const { v[0] = w.x, v[1] = w.y, v[2] = w.z, v[3] = w.w; }
  __device__ __forceinline__ void put(int e, float x) { (e < 2 ? (e == 0 ? w.x : w.y) : (e == 2 ? w.z : w.w)) = x; }
};
template <>
struct Block<uint16_t, 1> {
  uint16_t w;
  __device__ __forceinline__ void load(const uint16_t* p) { w = __ldcs(p); }
  __device__ __forceinline__ void clear() { w = 0; }
  __device__ __forceinline__ void put(int, uint16_t x) { w = x; }
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = bf16_to_f32(w); }
};
template <>
struct Block<float, 1> {
  float w;
  __device__ __forceinline__ void load(const float* p) { w = __ldcs(p); }
  __device__ __forceinline__ void clear() { w = 0.f; }
  __device__ __forceinline__ void put(int, float x) { w = x; }
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = w; }
};

// ---------------------------------------------------------------- forward

struct FwdArgs {
  const int32_t* ids;
  const void* w;
  void* out;
  int64_t T, D, ld_w, ld_out;
  int32_t V;
  float scale;
  int32_t* status;
};

constexpr int kFwdWarps = 8;
constexpr int kFwdElems = 32;  // elements per lane: a warp takes 1,024 columns of a token

__device__ __forceinline__ uint32_t pack(float a, float b) { return pack_bf16x2(a, b); }

// V8: rows of both matrices begin on 16-byte boundaries and D is a multiple of 8.
template <typename TW, typename TO, bool V8>
__global__ void __launch_bounds__(kFwdWarps * 32) lookup_kernel(const FwdArgs p) {
  const int lane = threadIdx.x & 31;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * kFwdWarps + threadIdx.x / 32;
  if (t >= p.T) return;
  const int32_t id = p.ids[t];
  const bool ok = id >= 0 && id < p.V;
  if (!ok && lane == 0 && blockIdx.y == 0) flag_status(p.status, RL_DEV_BAD_TOKEN);
  const TW* w = static_cast<const TW*>(p.w) + (ok ? id : 0) * p.ld_w;
  TO* out = static_cast<TO*>(p.out) + t * p.ld_out;
  const int64_t c0 = static_cast<int64_t>(blockIdx.y) * (32 * kFwdElems);
  if (V8) {
    constexpr int N = kFwdElems / 8;
    float v[N][8];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int64_t c = c0 + (j * 32 + lane) * 8;
      if (c < p.D && ok) {
        if (sizeof(TW) == 2) {
          const uint4 q = *reinterpret_cast<const uint4*>(w + c);
          v[j][0] = bf16_lo(q.x), v[j][1] = bf16_hi(q.x), v[j][2] = bf16_lo(q.y), v[j][3] = bf16_hi(q.y);
          v[j][4] = bf16_lo(q.z), v[j][5] = bf16_hi(q.z), v[j][6] = bf16_lo(q.w), v[j][7] = bf16_hi(q.w);
        } else {
          const float4 a = *reinterpret_cast<const float4*>(w + c), b = *reinterpret_cast<const float4*>(w + c + 4);
          v[j][0] = a.x, v[j][1] = a.y, v[j][2] = a.z, v[j][3] = a.w;
          v[j][4] = b.x, v[j][5] = b.y, v[j][6] = b.z, v[j][7] = b.w;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[j][e] = 0.f;
      }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int64_t c = c0 + (j * 32 + lane) * 8;
      if (c >= p.D) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[j][e] *= p.scale;
      if (sizeof(TO) == 2) {
        __stcs(reinterpret_cast<uint4*>(out + c), make_uint4(pack(v[j][0], v[j][1]), pack(v[j][2], v[j][3]),
                                                             pack(v[j][4], v[j][5]), pack(v[j][6], v[j][7])));
      } else {
        __stcs(reinterpret_cast<float4*>(out + c), make_float4(v[j][0], v[j][1], v[j][2], v[j][3]));
        __stcs(reinterpret_cast<float4*>(out + c + 4), make_float4(v[j][4], v[j][5], v[j][6], v[j][7]));
      }
    }
  } else {
#pragma unroll 8
    for (int j = 0; j < kFwdElems; ++j) {
      const int64_t c = c0 + j * 32 + lane;
      if (c >= p.D) break;
      float v = 0.f;
      if (ok) v = sizeof(TW) == 2 ? bf16_to_f32(reinterpret_cast<const uint16_t*>(w)[c]) : reinterpret_cast<const float*>(w)[c];
      v *= p.scale;
      if (sizeof(TO) == 2) reinterpret_cast<uint16_t*>(out)[c] = f32_to_bf16(v);
      else reinterpret_cast<float*>(out)[c] = v;
    }
  }
}

// ---------------------------------------------------------------- sorting the tokens by id

constexpr int kSortThreads = 256, kSortWarps = kSortThreads / 32;
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int64_t kMostTiles = 4096;

// What a sort is laid out for, from T and V alone.
struct Plan {
  int passes, bits;  // digits of `bits` bits
  int64_t rounds;    // a tile is kSortThreads * rounds tokens
  int64_t tiles;
  int64_t chunk, chunks;
  int64_t most_tiles, most_chunks;  // of any sort of up to T tokens: what the workspace has room for
};

struct SortArgs {
  const int32_t* keys;  // nullptr: the ids of the first pass
  const int32_t* ids;
  const int32_t* toks;  // nullptr in the first pass: the token's own index
  int32_t* keys_out;
  int32_t* toks_out;
  int64_t T, rounds, tiles;
  int32_t V, shift, mask;
  uint32_t* counts;  // [digits x tiles]
  uint32_t* totals;  // [digits]
  uint32_t* crossing;  // set to zero for the sums
  int32_t* status;
};

// The key of position i: ids outside [0, V) become V and sort behind all others.
__device__ __forceinline__ uint32_t key_at(const SortArgs& p, int64_t i) {
  if (p.keys) return static_cast<uint32_t>(p.keys[i]);
  const int32_t id = p.ids[i];
  return static_cast<uint32_t>(id >= 0 && id < p.V ? id : p.V);
}

// How often each warp's part of the tile has each digit, in the order of the positions.
__device__ __forceinline__ void count_tile(const SortArgs& p, uint32_t (&n)[kSortWarps][kDigits]) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < kSortWarps * kDigits; i += kSortThreads) (&n[0][0])[i] = 0;
  __syncthreads();
  const int64_t first = (static_cast<int64_t>(blockIdx.x) * kSortWarps + warp) * p.rounds * 32;
  for (int64_t k = 0; k < p.rounds; ++k) {
    const int64_t i = first + k * 32 + lane;
    const bool in = i < p.T;
    const uint32_t live = __ballot_sync(0xffffffffu, in);
    if (in) {
      const uint32_t d = (key_at(p, i) >> p.shift) & p.mask;
      const uint32_t peers = __match_any_sync(live, d);
      if (lane == __ffs(peers) - 1) n[warp][d] += __popc(peers);
    }
    __syncwarp();
  }
  __syncthreads();
}

__global__ void __launch_bounds__(kSortThreads) count_kernel(const SortArgs p) {
  __shared__ uint32_t n[kSortWarps][kDigits];
  count_tile(p, n);
  for (int d = threadIdx.x; d <= p.mask; d += kSortThreads) {
    uint32_t s = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) s += n[w][d];
    p.counts[d * p.tiles + blockIdx.x] = s;
  }
  if (p.keys) return;
  bool bad = false;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kSortThreads * p.rounds;
  for (int64_t i = first + threadIdx.x; i < min(p.T, first + kSortThreads * p.rounds); i += kSortThreads)
    bad |= p.ids[i] < 0 || p.ids[i] >= p.V;
  if (bad) flag_status(p.status, RL_DEV_BAD_TOKEN);
}

// Per digit (a warp each) the tiles' counts become the sums of the tiles before, and the total.
__global__ void __launch_bounds__(kSortThreads) prefix_kernel(const SortArgs p) {
  const int d = blockIdx.x * kSortWarps + threadIdx.x / 32, lane = threadIdx.x & 31;
  if (d > p.mask) return;
  uint32_t* c = p.counts + d * p.tiles;
  uint32_t run = 0;
  for (int64_t k = 0; k < p.tiles; k += 32) {
    const uint32_t mine = k + lane < p.tiles ? c[k + lane] : 0;
    uint32_t s = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += v;
    }
    if (k + lane < p.tiles) c[k + lane] = run + s - mine;
    run += __shfl_sync(0xffffffffu, s, 31);
  }
  if (lane == 0) p.totals[d] = run;
  if (d == 0 && lane == 0) *p.crossing = 0;
}

__global__ void __launch_bounds__(kSortThreads) scatter_kernel(const SortArgs p) {
  __shared__ uint32_t n[kSortWarps][kDigits];
  __shared__ uint32_t sums[kSortWarps];
  count_tile(p, n);
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  // where each digit begins: the totals of the lower ones, two digits a thread
  const int d0 = 2 * threadIdx.x;
  const uint32_t a = d0 <= p.mask ? p.totals[d0] : 0, b = d0 + 1 <= p.mask ? p.totals[d0 + 1] : 0;
  uint32_t s = a + b;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t v = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += v;
  }
  if (lane == 31) sums[warp] = s;
  __syncthreads();
  uint32_t before = s - a - b;
  for (int w = 0; w < warp; ++w) before += sums[w];
  // and within it this tile's, and within that each warp's
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int d = d0 + e;
    if (d > p.mask) break;
    uint32_t at = before + (e ? a : 0) + p.counts[d * p.tiles + blockIdx.x];
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      const uint32_t c = n[w][d];
      n[w][d] = at;
      at += c;
    }
  }
  __syncthreads();
  const int64_t first = (static_cast<int64_t>(blockIdx.x) * kSortWarps + warp) * p.rounds * 32;
  for (int64_t k = 0; k < p.rounds; ++k) {
    const int64_t i = first + k * 32 + lane;
    const bool in = i < p.T;
    const uint32_t live = __ballot_sync(0xffffffffu, in);
    if (in) {
      const uint32_t key = key_at(p, i), d = (key >> p.shift) & p.mask;
      const uint32_t peers = __match_any_sync(live, d);
      const uint32_t at = n[warp][d] + __popc(peers & ((1u << lane) - 1));
      __syncwarp(live);
      if (lane == __ffs(peers) - 1) n[warp][d] += __popc(peers);
      p.keys_out[at] = static_cast<int32_t>(key);
      p.toks_out[at] = p.toks ? p.toks[i] : static_cast<int32_t>(i);
    }
    __syncwarp();
  }
}

// ---------------------------------------------------------------- the same by one cluster, in shared memory

constexpr int kSortCtas = 16, kBlockThreads = 1024, kBlockWarps = kBlockThreads / 32;
constexpr int64_t kMostHeld = 11264;  // tokens a CTA holds
constexpr int64_t kMostSorted = kSortCtas * kMostHeld;
constexpr int kMostRounds = static_cast<int>(kMostHeld / kBlockThreads);
static_assert(kMostHeld % kBlockThreads == 0 && kMostHeld < 65536, "rounds of a warp, and its counters of 16 bits");

struct ClusterArgs {
  const int32_t* ids;
  int32_t* keys_out;
  int32_t* toks_out;
  uint32_t* crossing;  // set to zero for the sums
  int32_t* status;
  int32_t T, V, cap;  // cap: positions of a CTA, a multiple of 32
  uint32_t inverse;   // 2^32 / cap, rounded up
  int32_t passes, bits;
};

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void put_pair(uint32_t addr, uint32_t key, uint32_t tok) {
  asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" :: "r"(addr), "r"(key), "r"(tok) : "memory");
}

inline __host__ __device__ int64_t cluster_sort_bytes(int64_t cap) { return 2 * cap * 8 + int64_t(kBlockWarps) * kDigits * 2; }

// The stable radix sort of up to kMostSorted tokens: 16 CTAs hold the list, and a digit's pass writes every token to its
// place in the CTA that holds it. One launch where the passes through memory take three each. Measured (the kernel alone
// against the six): 32,768 tokens 17 / 39 us, 155,959 34 / 40.
__global__ void __launch_bounds__(kBlockThreads) cluster_sort_kernel(const ClusterArgs p) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ uint32_t total[kDigits];  // this CTA's tokens of each digit
  __shared__ uint32_t base[kDigits];   // where they go
  __shared__ uint32_t sums[kDigits / 32];
  uint2* buf[2] = {reinterpret_cast<uint2*>(smem), reinterpret_cast<uint2*>(smem) + p.cap};
  uint16_t(*n)[kDigits] = reinterpret_cast<uint16_t(*)[kDigits]>(smem + 2 * static_cast<size_t>(p.cap) * 8);
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const int rank = static_cast<int>(cluster_ctarank());
  const int first = rank * p.cap, mine = max(0, min(p.cap, p.T - first));  // positions first .. first + mine
  const int rounds = (p.cap / 32 + kBlockWarps - 1) / kBlockWarps, w0 = warp * rounds * 32;
  if (rank == 0 && threadIdx.x == 0) *p.crossing = 0;
  bool bad = false;
  for (int i = threadIdx.x; i < mine; i += kBlockThreads) {
    const int32_t id = p.ids[first + i];
    const bool ok = id >= 0 && id < p.V;
    bad |= !ok;
    buf[0][i] = make_uint2(static_cast<uint32_t>(ok ? id : p.V), static_cast<uint32_t>(first + i));
  }
  if (bad) flag_status(p.status, RL_DEV_BAD_TOKEN);
  const uint32_t mask = (1u << p.bits) - 1;
  for (int pass = 0; pass < p.passes; ++pass) {
    const int shift = pass * p.bits;
    const uint2* from = buf[pass & 1];
    for (int i = threadIdx.x; i < kBlockWarps * kDigits / 2; i += kBlockThreads) reinterpret_cast<uint32_t*>(&n[0][0])[i] = 0;
    __syncthreads();
    uint32_t peers[kMostRounds];  // the lanes with the same digit, round by round
#pragma unroll
    for (int k = 0; k < kMostRounds; ++k) {
      if (k >= rounds) break;
      const int i = w0 + k * 32 + lane;
      const bool in = i < mine;
      const uint32_t live = __ballot_sync(0xffffffffu, in);
      peers[k] = 0;
      if (in) {
        const uint32_t d = (from[i].x >> shift) & mask;
        peers[k] = __match_any_sync(live, d);
        if (lane == __ffs(peers[k]) - 1) n[warp][d] += static_cast<uint16_t>(__popc(peers[k]));
      }
      __syncwarp();
    }
    __syncthreads();
    for (uint32_t d = threadIdx.x; d <= mask; d += kBlockThreads) {  // each warp's start among the CTA's
      uint32_t run = 0;
#pragma unroll
      for (int w0 = 0; w0 < kBlockWarps; w0 += 16) {
        uint32_t c[16];
#pragma unroll
        for (int w = 0; w < 16; ++w) c[w] = n[w0 + w][d];
#pragma unroll
        for (int w = 0; w < 16; ++w) {
          n[w0 + w][d] = static_cast<uint16_t>(run);
          run += c[w];
        }
      }
      total[d] = run;
    }
    cluster_sync_all();
    uint32_t all = 0, before = 0;
    const uint32_t d = threadIdx.x;
    if (d <= mask) {
      uint32_t c[kSortCtas];
#pragma unroll
      for (int r = 0; r < kSortCtas; ++r) c[r] = ld_cluster_u32(map_to_rank(smem_addr(&total[d]), r));
#pragma unroll
      for (int r = 0; r < kSortCtas; ++r) {
        before += r < rank ? c[r] : 0;
        all += c[r];
      }
    }
    uint32_t run = all;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += v;
    }
    if (lane == 31 && warp < kDigits / 32) sums[warp] = run;
    __syncthreads();
    if (d <= mask) {
#pragma unroll
      for (int w = 0; w < kDigits / 32; ++w) run += w < warp ? sums[w] : 0;
      base[d] = run - all + before;
    }
    __syncthreads();
    const uint32_t to = smem_addr(buf[1 - (pass & 1)]);
#pragma unroll
    for (int k = 0; k < kMostRounds; ++k) {
      if (k >= rounds) break;
      const uint2 e = peers[k] != 0 ? from[w0 + k * 32 + lane] : make_uint2(0u, 0u);
      const uint32_t dg = (e.x >> shift) & mask;
      const uint32_t at = base[dg] + n[warp][dg] + __popc(peers[k] & ((1u << lane) - 1));
      __syncwarp();
      if (peers[k] != 0) {
        if (lane == __ffs(peers[k]) - 1) n[warp][dg] += static_cast<uint16_t>(__popc(peers[k]));
        const uint32_t cta = __umulhi(at, p.inverse);  // at / cap: exact, at is below 2^18 and cap below 2^14
        put_pair(map_to_rank(to + (at - cta * p.cap) * 8, cta), e.x, e.y);
      }
      __syncwarp();
    }
    cluster_sync_all();
  }
  next_may_start();  // not before: until here the SMs that this kernel leaves free are other streams'
  const uint2* sorted = buf[p.passes & 1];
  for (int i = threadIdx.x; i < mine; i += kBlockThreads) {
    p.keys_out[first + i] = static_cast<int32_t>(sorted[i].x);
    p.toks_out[first + i] = static_cast<int32_t>(sorted[i].y);
  }
}

// ---------------------------------------------------------------- the sums

struct SumArgs {
  const int32_t* keys;  // sorted
  const int32_t* toks;
  const void* d;
  float* dw;
  float* head;  // [chunks x stride]: the part of a long run that came in from the chunk before
  float* tail;  // [chunks x stride]: the part of a long run that begins in the chunk
  int32_t* list;       // the chunks in which a long run begins, in any order
  uint32_t* crossing;  // how many there are
  int64_t T, D, ld, chunk, stride;
  int32_t V;
  float scale;
};

constexpr int kSumThreads = 128;
constexpr int kMostChunk = 64;
constexpr int kAhead = 8;  // rows in flight

// A thread's N columns of a row, from column c.
template <typename T, int N>
__device__ __forceinline__ void load_columns(Block<T, N>& b, const T* row, int64_t c, int64_t D) {
  if (N == 1 || c + N <= D) {
    b.load(row + c);
  } else {
    b.clear();
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (c + e < D) b.put(e, row[c + e]);
  }
}

// dw += v for N columns from c. The additions are left to the L2 (red): nothing waits for the old values, which took 137 us
// where this takes 118 (32,768 tokens, 4,096 columns), and every element gets one of them. WHOLE: rows of dw in 16-byte blocks.
template <int N, bool WHOLE>
__device__ __forceinline__ void add_columns(float* row, const float (&v)[N], int64_t c, int64_t D) {
  if (WHOLE && N >= 4) {
#pragma unroll
    for (int e = 0; e < N; e += 4)
      if (c + e < D)
        asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};"
                     :: "l"(row + c + e), "f"(v[e]), "f"(v[e + 1]), "f"(v[e + 2]), "f"(v[e + 3]) : "memory");
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (c + e < D) asm volatile("red.relaxed.gpu.global.add.f32 [%0], %1;" :: "l"(row + c + e), "f"(v[e]) : "memory");
  }
}

// The first of the sorted positions [lo, hi) with a key above v (hi: none); at(i): the key at position i.
template <typename K>
__device__ __forceinline__ int end_of(int lo, int hi, int32_t v, K at) {
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (at(mid) > v) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// N columns a thread, CX threads along a row, kSumThreads / CX chunks a CTA. A run belongs to the chunk in which it begins,
// which goes on after its end for up to a chunk's length; a longer run is cut at the chunks' borders.
template <typename T, int N, bool WHOLE, int CX>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const SumArgs p) {
  constexpr int kChunks = kSumThreads / CX;
  __shared__ int32_t key[kChunks][2 * kMostChunk + 2];  // of positions a - 1 .. a + 2 chunk (-1: none)
  __shared__ int32_t tok[kChunks][2 * kMostChunk];
  const int y = threadIdx.x / CX, x = threadIdx.x % CX, L = static_cast<int>(p.chunk);
  const int64_t ch = static_cast<int64_t>(blockIdx.x) * kChunks + y;
  const int64_t a = ch * L;
  const int n = static_cast<int>(max(int64_t(0), min(p.chunk, p.T - a)));        // its positions
  const int m = static_cast<int>(max(int64_t(0), min(2 * p.chunk, p.T - a)));    // and the next chunk's
  after_previous();
  for (int i = x; i < m + 2; i += CX) {
    const int64_t at = a + i - 1;
    key[y][i] = n > 0 && at >= 0 && at < p.T ? p.keys[at] : -1;
  }
  for (int i = x; i < m; i += CX) tok[y][i] = p.toks[a + i];
  __syncthreads();
  const int64_t c = (static_cast<int64_t>(blockIdx.y) * CX + x) * N;
  if (c >= p.D || n <= 0) return;
  auto at = [&](int i) { return key[y][i + 1]; };
  // what comes in: a run of the chunk before that ends within this one is that chunk's
  int begin = 0;
  bool head = false;
  const int32_t v0 = at(0);
  if (at(-1) == v0) {
    const bool began_there = !(p.keys[a - L] == v0 && a > L && p.keys[a - L - 1] == v0);
    if (began_there && (n < L || n == m || at(n) != v0)) begin = end_of(0, n, v0, at);
    else head = true;
  }
  if (begin == n) return;
  // what goes on: to its end if that lies within the next chunk
  int end = n;
  bool tail = false;
  const int32_t v1 = at(n - 1);
  if (n < m && at(n) == v1) {
    const bool began_here = !(head && v1 == v0);
    if (began_here && at(m) != v1) end = end_of(n, m, v1, at);
    else tail = began_here && v1 < p.V;
  }
  if (tail && c == 0) p.list[atomicAdd(p.crossing, 1u)] = static_cast<int32_t>(ch);

  const T* d = static_cast<const T*>(p.d);
  float acc[N];
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] = 0.f;
  for (int i = begin; i < end; i += kAhead) {
    Block<T, N> rows[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      rows[k].clear();
      if (i + k < end && at(i + k) < p.V) load_columns<T, N>(rows[k], d + tok[y][i + k] * p.ld, c, p.D);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int j = i + k;
      if (j >= end) break;
      const int32_t v = at(j);
      if (v >= p.V) return;  // ids out of range: the last of the list
      float f[N];
      rows[k].get(f);
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] += f[e];
      if (j + 1 < end && at(j + 1) == v) continue;
      if (head || (tail && j + 1 == end)) {
        float* to = (head ? p.head : p.tail) + ch * p.stride + c;
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (c + e < p.D) to[e] = acc[e];
        head = false;
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] *= p.scale;
        add_columns<N, WHOLE>(p.dw + v * p.D, acc, c, p.D);
      }
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] = 0.f;
    }
  }
}

constexpr int kJoinWarps = 8;
constexpr int kJoinCtas = 8 * 152;

// The last chunk of a long run of v that begins in chunk `ch`, by a whole warp.
__device__ __forceinline__ int64_t last_chunk(const SumArgs& p, int64_t ch, int32_t v, int lane) {
  for (int64_t k = ch + 1;; k += 32) {
    const int64_t next = (k + lane + 1) * p.chunk;
    const uint32_t ends = __ballot_sync(0xffffffffu, next >= p.T || p.keys[next] != v);
    if (ends) return k + __ffs(ends) - 1;
  }
}

// The long runs: an item is one of them and 128 columns. Each warp takes a part of the run's chunks, four columns a lane, and
// the parts are added up in order.
template <bool WHOLE>
__global__ void __launch_bounds__(kJoinWarps * 32) join_kernel(const SumArgs p) {
  __shared__ __align__(16) float sum[kJoinWarps][128];
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  after_previous();
  const int64_t slices = (p.D + 127) / 128, items = *p.crossing * slices;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t ch = p.list[it / slices], c = it % slices * 128 + lane * 4;
    const int32_t v = p.keys[(ch + 1) * p.chunk];
    const int64_t last = last_chunk(p, ch, v, lane);
    const int64_t per = (last - ch + kJoinWarps - 1) / kJoinWarps;
    const int64_t from = ch + 1 + warp * per, to = min(from + per, last + 1);
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](const float* part) {
      const float4 f = __ldcs(reinterpret_cast<const float4*>(part + c));
      s.x += f.x, s.y += f.y, s.z += f.z, s.w += f.w;
    };
    if (c < p.D) {  // what lies behind D of a part is room for whole blocks
      if (warp == 0) add(p.tail + ch * p.stride);
#pragma unroll 8
      for (int64_t k = from; k < to; ++k) add(p.head + k * p.stride);
    }
    *reinterpret_cast<float4*>(&sum[warp][lane * 4]) = s;
    __syncthreads();
    if (warp == 0 && c < p.D) {
#pragma unroll
      for (int w = 1; w < kJoinWarps; ++w) {
        const float4 f = *reinterpret_cast<const float4*>(&sum[w][lane * 4]);
        s.x += f.x, s.y += f.y, s.z += f.z, s.w += f.w;
      }
      const float out[4] = {p.scale * s.x, p.scale * s.y, p.scale * s.z, p.scale * s.w};
      add_columns<4, WHOLE>(p.dw + v * p.D, out, c, p.D);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- few tokens

constexpr int kFewThreads = 256, kFewTokens = 1024;
constexpr int kFewX = 64, kFewY = kFewThreads / kFewX;  // threads along a row, parts of the tokens of an id

struct FewArgs {
  const int32_t* ids;
  const void* d;
  float* dw;
  int32_t T, V;
  int64_t D, ld;
  float scale;
  int32_t* status;
};

// A CTA for every token and kFewX * N columns: the first token of its id adds up those of all of them, in up to kFewY parts.
// No sort: every CTA looks at all ids. One launch. Measured, bf16: 512 x 1,024 of 32,000 7 us; 1,024 tokens of one id x 1,024 78.
template <typename T, int N, bool WHOLE>
__global__ void __launch_bounds__(kFewThreads) few_kernel(const FewArgs p) {
  constexpr int kRounds = kFewTokens / kFewThreads, kWarps = kFewThreads / 32;
  __shared__ uint16_t list[kFewTokens];
  __shared__ uint32_t count[kRounds * kWarps];
  __shared__ float part[kFewY][kFewX * N];
  const int t = blockIdx.x, tid = threadIdx.x, warp = tid / 32, lane = tid & 31;
  const int32_t v = p.ids[t];
  if (v < 0 || v >= p.V) {
    if (blockIdx.y == 0 && tid == 0) flag_status(p.status, RL_DEV_BAD_TOKEN);
    return;
  }
  uint32_t same[kRounds];
  bool earlier = false;
#pragma unroll
  for (int k = 0; k < kRounds; ++k) {
    const int i = k * kFewThreads + tid;
    const bool is = i < p.T && p.ids[i] == v;
    earlier |= is && i < t;
    same[k] = __ballot_sync(0xffffffffu, is);
    if (lane == 0) count[k * kWarps + warp] = __popc(same[k]);
  }
  if (__syncthreads_or(earlier)) return;
  static_assert(kRounds * kWarps == 32, "a warp's lane per count");
  uint32_t run = count[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t u = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += u;
  }
  const int n = static_cast<int>(__shfl_sync(0xffffffffu, run, 31));
  run -= count[lane];
#pragma unroll
  for (int k = 0; k < kRounds; ++k) {
    const uint32_t before = __shfl_sync(0xffffffffu, run, k * kWarps + warp);
    if (same[k] >> lane & 1) list[before + __popc(same[k] & ((1u << lane) - 1))] = static_cast<uint16_t>(k * kFewThreads + tid);
  }
  __syncthreads();
  const int x = tid % kFewX, y = tid / kFewX;
  const int64_t c = (static_cast<int64_t>(blockIdx.y) * kFewX + x) * N;
  const int per = (n + kFewY - 1) / kFewY, from = y * per, to = min(from + per, n);
  const T* d = static_cast<const T*>(p.d);
  float acc[N];
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] = 0.f;
  if (c < p.D) {
#pragma unroll 4
    for (int i = from; i < to; ++i) {
      Block<T, N> row;
      load_columns<T, N>(row, d + list[i] * p.ld, c, p.D);
      float f[N];
      row.get(f);
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] += f[e];
    }
  }
  if (n > 1) {
#pragma unroll
    for (int e = 0; e < N; ++e) part[y][x * N + e] = acc[e];
    __syncthreads();
    if (y == 0)
#pragma unroll
      for (int k = 1; k < kFewY; ++k)
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] += part[k][x * N + e];
  }
  if (y != 0 || c >= p.D) return;
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] *= p.scale;
  add_columns<N, WHOLE>(p.dw + v * p.D, acc, c, p.D);
}

// ---------------------------------------------------------------- host

constexpr int64_t kMostT = int64_t(1) << 30, kMostV = (int64_t(1) << 31) - 2, kMostD = 1 << 20;

Plan plan(int64_t T, int64_t V) {
  Plan q;
  int bits = 1;
  while ((V >> bits) != 0) ++bits;  // keys up to V itself
  q.passes = (bits + kDigitBits - 1) / kDigitBits;
  q.bits = (bits + q.passes - 1) / q.passes;
  q.rounds = std::max<int64_t>(4, (T + kSortThreads * kMostTiles - 1) / (kSortThreads * kMostTiles));
  const int64_t tile = kSortThreads * q.rounds;
  q.tiles = std::max<int64_t>(1, (T + tile - 1) / tile);
  q.chunk = T <= 8192 ? 16 : T <= 65536 ? 32 : kMostChunk;
  q.chunks = (T + q.chunk - 1) / q.chunk;
  q.most_tiles = std::min<int64_t>(kMostTiles, (T + kSortThreads * 4 - 1) / (kSortThreads * 4));
  q.most_chunks = std::max<int64_t>(
      {(std::min<int64_t>(T, 8192) + 15) / 16, (std::min<int64_t>(T, 65536) + 31) / 32, (T + kMostChunk - 1) / kMostChunk});
  return q;
}

inline size_t up(size_t n) { return (n + 255) / 256 * 256; }

struct Layout {
  int64_t stride;
  size_t keys[2], toks[2], counts, totals, list, crossing, head, tail, bytes;
};
Layout layout(const Plan& q, int64_t T, int64_t D) {
  Layout l;
  size_t at = kWsHeader;
  auto take = [&](size_t n) {
    const size_t o = at;
    at += up(n);
    return o;
  };
  for (int i = 0; i < 2; ++i) {
    l.keys[i] = take(size_t(T) * 4);
    l.toks[i] = take(size_t(T) * 4);
  }
  l.counts = take(size_t(q.most_tiles) * kDigits * 4);
  l.totals = take(kDigits * 4);
  l.crossing = take(4);
  l.list = take(size_t(q.most_chunks) * 4);
  l.stride = (D + 3) / 4 * 4;
  l.head = take(size_t(q.most_chunks) * l.stride * 4);
  l.tail = take(size_t(q.most_chunks) * l.stride * 4);
  l.bytes = at;
  return l;
}

rl_status check_sizes(const std::string& f, int64_t T, int64_t V, int64_t D) {
  if (T < 0 || V < 1 || D < 1) return set_error(RL_ERR_INVALID_ARG, f + "bad size");
  if (T > kMostT || V > kMostV || D > kMostD || V > (int64_t(1) << 40) / D || T > (int64_t(1) << 40) / D)
    return set_error(RL_ERR_UNSUPPORTED, f + "at most 2^30 tokens, 2^31 - 2 rows, 2^20 columns and 2^40 elements");
  return RL_OK;
}
inline bool element_aligned(const void* p, rl_dtype t) {
  return reinterpret_cast<uintptr_t>(p) % (t == RL_BF16 ? 2 : 4) == 0;
}
inline bool whole_blocks(const void* p, int64_t ld, size_t es) { return aligned16(p) && ld * es % 16 == 0; }

template <typename TW, typename TO>
rl_status forward(const FwdArgs& a, cudaStream_t s) {
  const dim3 grid(static_cast<unsigned>((a.T + kFwdWarps - 1) / kFwdWarps),
                  static_cast<unsigned>((a.D + 32 * kFwdElems - 1) / (32 * kFwdElems)));
  if (a.D % 8 == 0 && whole_blocks(a.w, a.ld_w, sizeof(TW)) && whole_blocks(a.out, a.ld_out, sizeof(TO)))
    lookup_kernel<TW, TO, true><<<grid, kFwdWarps * 32, 0, s>>>(a);
  else
    lookup_kernel<TW, TO, false><<<grid, kFwdWarps * 32, 0, s>>>(a);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? RL_OK : cuda_error(e, "lookup_kernel launch");
}

template <typename T, int N, bool WHOLE>
cudaError_t launch_sums(const SumArgs& a, int64_t chunks, cudaStream_t s) {
  const int64_t threads = (a.D + N - 1) / N;
  cudaError_t e = cudaSuccess;
  auto go = [&](auto kern, int cx) {
    const int64_t per = kSumThreads / cx;
    e = launch_after(kern, dim3(static_cast<unsigned>((chunks + per - 1) / per), static_cast<unsigned>((threads + cx - 1) / cx)),
                     dim3(kSumThreads), 0, s, a);
  };
  if (threads > 64) go(sum_kernel<T, N, WHOLE, 128>, 128);
  else if (threads > 32) go(sum_kernel<T, N, WHOLE, 64>, 64);
  else if (threads > 16) go(sum_kernel<T, N, WHOLE, 32>, 32);
  else go(sum_kernel<T, N, WHOLE, 16>, 16);
  return e;
}

// How the rows lie: those of d in 16-byte blocks, and those of dw too.
struct Rows {
  bool d, dw;
};
template <typename T>
Rows rows_of(const void* d, int64_t ld, const float* dw, int64_t D) {
  return {whole_blocks(d, ld, sizeof(T)), aligned16(dw) && D % 4 == 0};
}

template <typename T>
rl_status few(const FewArgs& a, cudaStream_t s) {
  constexpr int N = 16 / sizeof(T);
  const Rows r = rows_of<T>(a.d, a.ld, a.dw, a.D);
  auto go = [&](auto kern, int n) {
    kern<<<dim3(static_cast<unsigned>(a.T), static_cast<unsigned>((a.D + kFewX * n - 1) / (kFewX * n))), kFewThreads, 0, s>>>(a);
  };
  if (!r.d) go(few_kernel<T, 1, false>, 1);
  else if (r.dw) go(few_kernel<T, N, true>, N);
  else go(few_kernel<T, N, false>, N);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? RL_OK : cuda_error(e, "few_kernel launch");
}

template <typename T>
rl_status sums(const SumArgs& a, int64_t chunks, cudaStream_t s) {
  constexpr int N = 16 / sizeof(T);
  const Rows r = rows_of<T>(a.d, a.ld, a.dw, a.D);
  cudaError_t e = !r.d ? launch_sums<T, 1, false>(a, chunks, s)
                       : r.dw ? launch_sums<T, N, true>(a, chunks, s) : launch_sums<T, N, false>(a, chunks, s);
  if (e != cudaSuccess) return cuda_error(e, "sum_kernel launch");
  if (chunks > 2) {
    e = launch_after(r.dw ? join_kernel<true> : join_kernel<false>, dim3(kJoinCtas), dim3(kJoinWarps * 32), 0, s, a);
    if (e != cudaSuccess) return cuda_error(e, "join_kernel launch");
  }
  return RL_OK;
}

rl_status cluster_sort(ClusterArgs& a, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_error(e, "cudaGetDevice");
  const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
  if (!(ready.load() & bit)) {
    e = cudaFuncSetAttribute(cluster_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(cluster_sort_bytes(kMostHeld)));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(cluster_sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return cuda_error(e, "cudaFuncSetAttribute(cluster_sort_kernel)");
    ready |= bit;
  }
  a.cap = ((a.T + kSortCtas - 1) / kSortCtas + 31) / 32 * 32;
  a.inverse = static_cast<uint32_t>(((uint64_t(1) << 32) + a.cap - 1) / a.cap);
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kSortCtas;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3(kSortCtas);
  cfg.blockDim = dim3(kBlockThreads);
  cfg.dynamicSmemBytes = static_cast<size_t>(cluster_sort_bytes(a.cap));
  cfg.stream = s;
  e = cudaLaunchKernelEx(&cfg, cluster_sort_kernel, a);
  return e == cudaSuccess ? RL_OK : cuda_error(e, "cluster_sort_kernel launch");
}

}  // namespace embed
}  // namespace rl

extern "C" {

rl_status rl_embedding_fwd(const int32_t* token_ids, int64_t T, const void* weight, rl_dtype w_dtype, int64_t V, int64_t D,
                           int64_t ld_w, float scale, void* out, rl_dtype out_dtype, int64_t ld_out, void* ws,
                           size_t ws_bytes, rl_stream_t stream) {
  using namespace rl;
  clear_error();
  const std::string f = "rl_embedding_fwd: ";
  const rl_status st = embed::check_sizes(f, T, V, D);
  if (st != RL_OK) return st;
  if ((w_dtype != RL_BF16 && w_dtype != RL_F32) || (out_dtype != RL_BF16 && out_dtype != RL_F32))
    return set_error(RL_ERR_INVALID_ARG, f + "bad dtype");
  if (ld_w < D || ld_out < D) return set_error(RL_ERR_INVALID_ARG, f + "a leading dimension is below D");
  if (!std::isfinite(scale)) return set_error(RL_ERR_INVALID_ARG, f + "scale is not finite");
  if (T == 0) return RL_OK;
  if (!token_ids || !weight || !out || !ws) return set_error(RL_ERR_INVALID_ARG, f + "a required pointer is NULL");
  if (!embed::element_aligned(token_ids, RL_F32) || !embed::element_aligned(weight, w_dtype) ||
      !embed::element_aligned(out, out_dtype) || !aligned16(ws))
    return set_error(RL_ERR_ALIGNMENT, f + "ids and matrices must be aligned to their elements and ws to 16 bytes");
  if (ws_bytes < kWsHeader) return set_error(RL_ERR_WORKSPACE_TOO_SMALL, f + "workspace smaller than its header");
  embed::FwdArgs a = {};
  a.ids = token_ids;
  a.w = weight;
  a.out = out;
  a.T = T;
  a.D = D;
  a.ld_w = ld_w;
  a.ld_out = ld_out;
  a.V = static_cast<int32_t>(V);
  a.scale = scale;
  a.status = static_cast<int32_t*>(ws);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (w_dtype == RL_BF16)
    return out_dtype == RL_BF16 ? embed::forward<uint16_t, uint16_t>(a, s) : embed::forward<uint16_t, float>(a, s);
  return out_dtype == RL_BF16 ? embed::forward<float, uint16_t>(a, s) : embed::forward<float, float>(a, s);
}

size_t rl_embedding_workspace_size(int64_t T, int64_t V, int64_t D) {
  using namespace rl;
  clear_error();
  if (embed::check_sizes("rl_embedding_workspace_size: ", T, V, D) != RL_OK) return 0;
  return embed::layout(embed::plan(T, V), T, D).bytes;
}

rl_status rl_embedding_bwd(const int32_t* token_ids, int64_t T, const void* d_out, rl_dtype d_dtype, int64_t ld_d, int64_t V,
                           int64_t D, float scale, float* d_weight, void* ws, size_t ws_bytes, rl_stream_t stream) {
  using namespace rl;
  clear_error();
  const std::string f = "rl_embedding_bwd: ";
  const rl_status st = embed::check_sizes(f, T, V, D);
  if (st != RL_OK) return st;
  if (d_dtype != RL_BF16 && d_dtype != RL_F32) return set_error(RL_ERR_INVALID_ARG, f + "bad dtype");
  if (ld_d < D) return set_error(RL_ERR_INVALID_ARG, f + "the leading dimension is below D");
  if (!std::isfinite(scale)) return set_error(RL_ERR_INVALID_ARG, f + "scale is not finite");
  if (T == 0) return RL_OK;
  if (!token_ids || !d_out || !d_weight || !ws) return set_error(RL_ERR_INVALID_ARG, f + "a required pointer is NULL");
  if (!embed::element_aligned(token_ids, RL_F32) || !embed::element_aligned(d_out, d_dtype) ||
      !embed::element_aligned(d_weight, RL_F32) || !aligned16(ws))
    return set_error(RL_ERR_ALIGNMENT, f + "ids and matrices must be aligned to their elements and ws to 16 bytes");
  const embed::Plan q = embed::plan(T, V);
  const embed::Layout l = embed::layout(q, T, D);
  if (ws_bytes < l.bytes)
    return set_error(RL_ERR_WORKSPACE_TOO_SMALL, f + "ws_bytes below rl_embedding_workspace_size(T, V, D)");
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  uint8_t* base = static_cast<uint8_t*>(ws);
  if (T <= embed::kFewTokens) {
    embed::FewArgs a = {};
    a.ids = token_ids;
    a.d = d_out;
    a.dw = d_weight;
    a.T = static_cast<int32_t>(T);
    a.V = static_cast<int32_t>(V);
    a.D = D;
    a.ld = ld_d;
    a.scale = scale;
    a.status = reinterpret_cast<int32_t*>(base);
    return d_dtype == RL_BF16 ? embed::few<uint16_t>(a, s) : embed::few<float>(a, s);
  }
  auto ints = [&](size_t o) { return reinterpret_cast<int32_t*>(base + o); };
  embed::SumArgs a = {};
  a.crossing = reinterpret_cast<uint32_t*>(base + l.crossing);
  if (T <= embed::kMostSorted) {
    embed::ClusterArgs o = {};
    o.ids = token_ids;
    o.keys_out = ints(l.keys[0]);
    o.toks_out = ints(l.toks[0]);
    o.crossing = a.crossing;
    o.status = reinterpret_cast<int32_t*>(base);
    o.T = static_cast<int32_t>(T);
    o.V = static_cast<int32_t>(V);
    o.passes = q.passes;
    o.bits = q.bits;
    const rl_status r = embed::cluster_sort(o, s);
    if (r != RL_OK) return r;
    a.keys = o.keys_out;
    a.toks = o.toks_out;
  } else {
    embed::SortArgs o = {};
    o.ids = token_ids;
    o.T = T;
    o.rounds = q.rounds;
    o.tiles = q.tiles;
    o.V = static_cast<int32_t>(V);
    o.mask = (1 << q.bits) - 1;
    o.counts = reinterpret_cast<uint32_t*>(base + l.counts);
    o.totals = reinterpret_cast<uint32_t*>(base + l.totals);
    o.crossing = a.crossing;
    o.status = reinterpret_cast<int32_t*>(base);
    const unsigned tiles = static_cast<unsigned>(q.tiles);
    for (int i = 0; i < q.passes; ++i) {
      o.shift = i * q.bits;
      o.keys_out = ints(l.keys[i & 1]);
      o.toks_out = ints(l.toks[i & 1]);
      embed::count_kernel<<<tiles, embed::kSortThreads, 0, s>>>(o);
      embed::prefix_kernel<<<(o.mask + embed::kSortWarps) / embed::kSortWarps, embed::kSortThreads, 0, s>>>(o);
      embed::scatter_kernel<<<tiles, embed::kSortThreads, 0, s>>>(o);
      const cudaError_t e = cudaGetLastError();
      if (e != cudaSuccess) return cuda_error(e, "rl_embedding_bwd: sort launch");
      o.keys = o.keys_out;
      o.toks = o.toks_out;
    }
    a.keys = o.keys;
    a.toks = o.toks;
  }
  a.d = d_out;
  a.dw = d_weight;
  a.head = reinterpret_cast<float*>(base + l.head);
  a.tail = reinterpret_cast<float*>(base + l.tail);
  a.list = ints(l.list);
  a.T = T;
  a.D = D;
  a.ld = ld_d;
  a.chunk = q.chunk;
  a.stride = l.stride;
  a.V = static_cast<int32_t>(V);
  a.scale = scale;
  return d_dtype == RL_BF16 ? embed::sums<uint16_t>(a, q.chunks, s) : embed::sums<float>(a, q.chunks, s);
}

}  // extern "C"
