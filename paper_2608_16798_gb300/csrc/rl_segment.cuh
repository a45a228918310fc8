// Rows of logits in pieces that a warp holds in shared memory, and what is computed of them: (max, sum of exponentials)
// folds in a scale c = log2(e) / T, their merges, and draws of an element by a running sum of weights. Shared by the
// verification of drafted tokens and the sampling of tokens.
#pragma once

#include <cmath>

#include "rl_device.cuh"

namespace rl {
namespace seg {

template <typename T>
struct Elem;
template <>
struct Elem<uint16_t> {
  static constexpr int N = 8;  // per 16 bytes
  static __device__ __forceinline__ void unpack(uint4 w, float (&z)[8]) {
    z[0] = bf16_lo(w.x), z[1] = bf16_hi(w.x), z[2] = bf16_lo(w.y), z[3] = bf16_hi(w.y);
    z[4] = bf16_lo(w.z), z[5] = bf16_hi(w.z), z[6] = bf16_lo(w.w), z[7] = bf16_hi(w.w);
  }
  static __device__ __forceinline__ float one(uint16_t x) { return bf16_to_f32(x); }
  static __device__ __forceinline__ uint16_t none() { return 0xff80; }
  static __device__ __forceinline__ uint32_t bits(uint16_t x) { return x; }
};
template <>
struct Elem<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(uint4 w, float (&z)[4]) {
    z[0] = __uint_as_float(w.x), z[1] = __uint_as_float(w.y), z[2] = __uint_as_float(w.z), z[3] = __uint_as_float(w.w);
  }
  static __device__ __forceinline__ float one(float x) { return x; }
  static __device__ __forceinline__ float none() { return -__int_as_float(0x7f800000); }
  static __device__ __forceinline__ uint32_t bits(float x) { return __float_as_uint(x); }
};

__device__ __forceinline__ float minus_inf() { return -__int_as_float(0x7f800000); }

// A warp's segment of a row in shared memory: the 16-byte blocks of memory that it covers.
template <typename T>
struct Segment {
  T* at;       // the first block
  int lo, hi;  // its elements are [lo, hi) from there
  __device__ __forceinline__ int blocks() const { return (hi + Elem<T>::N - 1) / Elem<T>::N; }
  __device__ __forceinline__ void load(int k, float (&z)[Elem<T>::N]) const {
    Elem<T>::unpack(*reinterpret_cast<const uint4*>(at + k * Elem<T>::N), z);
  }
  // What the first and the last block hold of the neighbours becomes minus infinity.
  __device__ __forceinline__ void blank_edges(int lane) const {
    const T none = Elem<T>::none();
    if (lane < lo) at[lane] = none;
    if (hi + lane < blocks() * Elem<T>::N) at[hi + lane] = none;
    __syncwarp();
  }
};

// Starts the copy of elements [e0, e0 + n) of a row into `to` (seg_bytes) on `bar`, by a whole warp.
// What the last block of the whole array would read past its end comes by plain loads.
template <typename T>
__device__ __forceinline__ Segment<T> fetch(const T* row, int e0, int n, const T* end, uint8_t* to, uint64_t* bar,
                                            int lane) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(row + e0), b = reinterpret_cast<uintptr_t>(row + e0 + n);
  const uintptr_t a0 = a & ~uintptr_t(15);
  Segment<T> s;
  s.at = reinterpret_cast<T*>(to);
  s.lo = static_cast<int>(a - a0) / static_cast<int>(sizeof(T));
  s.hi = s.lo + n;
  if (n <= 0) {
    s.hi = s.lo = 0;
    if (lane == 0) mbar_arrive(bar);
    return s;
  }
  uintptr_t b0 = (b + 15) & ~uintptr_t(15);
  if (b0 > reinterpret_cast<uintptr_t>(end)) {
    b0 = b & ~uintptr_t(15);
    const int rest = static_cast<int>(b - b0) / static_cast<int>(sizeof(T));
    if (lane < rest && b0 + lane * sizeof(T) >= a)
      *reinterpret_cast<T*>(to + (b0 - a0) + lane * sizeof(T)) = reinterpret_cast<const T*>(b0)[lane];
    __syncwarp();
  }
  if (lane == 0) {
    const uint32_t bytes = b0 > a0 ? static_cast<uint32_t>(b0 - a0) : 0;
    if (bytes == 0) {
      mbar_arrive(bar);
    } else {
      mbar_arrive_expect_tx(bar, bytes);
      bulk_g2s(to, reinterpret_cast<const void*>(a0), bytes, bar);
    }
  }
  return s;
}

// (max, sum of 2^((z - max) c)) of what a lane or a warp has seen; (-inf, 0): nothing. NaNs and
// +infinity make the sum NaN.
struct Fold {
  float m, s;
};

// Two fp32 operations per instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<uint64_t&>(r))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
  return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<uint64_t&>(r)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return r;
}

// Exponents are taken relative to the rounded product ref c, in one fused operation with z c, and every
// change of reference uses the same rounded products, so that it adds no error of its own. The product's rounding
// error, at most half a unit below 2^24, would leave fp32's range as an exponent beyond about 2^31 (rows, or a lane's
// part of one, at finite masks of -1e10), so from 2^24 on they are relative to ref itself: the difference comes first,
// exact where it matters.
constexpr float kFused = 16777216.f;
__device__ __forceinline__ bool large(float ref_c) { return !(fabsf(ref_c) < kFused); }
__device__ __forceinline__ float exponent(float z, float ref, float c) {
  const float rc = __fmul_rn(ref, c);
  return large(rc) ? (z - ref) * c : fmaf(z, c, -rc);
}
// The factor from sums relative to m to sums relative to M >= m, whichever each of them is taken relative to.
__device__ __forceinline__ float power(float m, float M, float c) {
  const float mc = __fmul_rn(m, c), Mc = __fmul_rn(M, c);
  float x = __fsub_rn(mc, Mc);
  if (large(mc)) x = fmaf(m, c, -Mc);
  if (large(Mc)) x = large(mc) ? (m - M) * c : -fmaf(M, c, -mc);
  return ex2(x);
}
// 2^exponent of a block.
template <int N>
__device__ __forceinline__ void exps(float (&z)[N], float ref, float c) {
  const float rc = -__fmul_rn(ref, c);
  if (!large(rc)) {
    const float2 cc = make_float2(c, c), r = make_float2(rc, rc);
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      const float2 t = fma2(make_float2(z[e], z[e + 1]), cc, r);
      z[e] = ex2(t.x);
      z[e + 1] = ex2(t.y);
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = ex2((z[e] - ref) * c);
  }
}

constexpr int kTileBlocks = 4;  // 16-byte blocks per lane and tile

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// The largest entry of a lane's blocks (NaNs do not count unless there is nothing else).
template <typename T>
__device__ __forceinline__ float largest(const uint4 (&w)[kTileBlocks]) {
  if (sizeof(T) == 2) {
    uint32_t t = w[0].x;
#pragma unroll
    for (int i = 0; i < kTileBlocks; ++i)
      t = max_bf16x2(t, max_bf16x2(max_bf16x2(w[i].x, w[i].y), max_bf16x2(w[i].z, w[i].w)));
    return fmaxf(bf16_lo(t), bf16_hi(t));
  }
  float m = __uint_as_float(w[0].x);
#pragma unroll
  for (int i = 0; i < kTileBlocks; ++i)
    m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(w[i].x), __uint_as_float(w[i].y)),
                       fmaxf(__uint_as_float(w[i].z), __uint_as_float(w[i].w))));
  return m;
}

// A lane's sums over what it has seen.
struct Running {
  float m;
  float2 s;
  int32_t arg;  // greedy: first largest entry
};

template <typename T, bool GREEDY>
__device__ __forceinline__ void add_tile(Running& r, const uint4 (&w)[kTileBlocks], int k0, float c) {
  constexpr int N = Elem<T>::N;
  const float top = largest<T>(w);
  if (top > r.m) {
    const float f = power(r.m, top, c);
    r.s.x *= f;
    r.s.y *= f;
    r.m = top;
    if (GREEDY) {
#pragma unroll
      for (int i = kTileBlocks - 1; i >= 0; --i) {
        float z[N];
        Elem<T>::unpack(w[i], z);
#pragma unroll
        for (int e = N - 1; e >= 0; --e)
          if (z[e] == top) r.arg = (k0 + 32 * i) * N + e;
      }
    }
  }
  const float ref = r.m == minus_inf() ? 0.f : r.m;
#pragma unroll
  for (int i = 0; i < kTileBlocks; ++i) {
    float z[N];
    Elem<T>::unpack(w[i], z);
    exps(z, ref, c);
#pragma unroll
    for (int e = 0; e < N; e += 2) r.s = add2(r.s, make_float2(z[e], z[e + 1]));
  }
}

// The warp's sums of all its lanes.
__device__ __forceinline__ Fold of_warp(const Running& r, float c) {
  const float mine = r.s.x + r.s.y, M = redux_max(r.m);
  return Fold{M, warp_sum(mine == 0.f ? 0.f : mine * power(r.m, M, c))};
}

// A segment of a row: a tile of blocks at a time, one reference each.
template <typename T, bool GREEDY>
__device__ __forceinline__ Fold fold(const Segment<T>& seg, float c, int lane, int& arg) {
  constexpr uint32_t none = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
  const int nb = seg.blocks();
  Running r{minus_inf(), {0.f, 0.f}, 0};
  for (int k0 = lane; k0 - lane < nb; k0 += 32 * kTileBlocks) {
    uint4 w[kTileBlocks];
#pragma unroll
    for (int i = 0; i < kTileBlocks; ++i) {
      const int k = k0 + 32 * i;
      w[i] = k < nb ? *reinterpret_cast<const uint4*>(seg.at + k * Elem<T>::N) : make_uint4(none, none, none, none);
    }
    add_tile<T, GREEDY>(r, w, k0, c);
  }
  const Fold f = of_warp(r, c);
  if (GREEDY) {
    const uint32_t best = __reduce_min_sync(0xffffffffu, r.m == f.m ? static_cast<uint32_t>(r.arg) : 0xffffffffu);
    arg = static_cast<int>(best) - seg.lo;
  }
  return f;
}

__device__ __forceinline__ void put_f2(uint32_t addr, float a, float b) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" :: "r"(addr), "f"(a), "f"(b) : "memory");
}
__device__ __forceinline__ void put_f1(uint32_t addr, float a) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" :: "r"(addr), "f"(a) : "memory");
}

// The row's (max, sum) from its segments', the same bits in every lane of every CTA.
__device__ __forceinline__ Fold merged(const Fold* f, int n, float c, int lane) {
  float m = minus_inf();
  for (int k = lane; k < n; k += 32) m = fmaxf(m, f[k].m);
  const float M = redux_max(m);
  float s = 0.f;
  for (int k = lane; k < n; k += 32) s += f[k].s == 0.f ? 0.f : f[k].s * power(f[k].m, M, c);
  return Fold{M, warp_sum(s)};
}

// No numbers: a row without a finite largest entry, or with a NaN.
__device__ __forceinline__ bool is_bad(const Fold& f) { return !(f.s > 0.f && f.s < 3e38f); }

__device__ __forceinline__ float logp_of(float z, const Fold& row, float c) {
  return (exponent(z, row.m, c) - log2f(row.s)) * kLn2;
}

// The segment in which the running sum of the weights w(k) passes u times their total, and what is left
// to pass within it. The last segment with any weight where rounding leaves none; -1: no weight at all.
// In fp32: the running sum of some hundred weights (the FP64 form took half of the kernel's time).
template <typename W>
__device__ __forceinline__ int pick(int n, float u, int lane, W w, float& left) {
  const int M = (n + 31) / 32, k0 = min(lane * M, n), k1 = min(k0 + M, n);  // lane l holds M segments
  float sum = 0.f;
  for (int k = k0; k < k1; ++k) sum += w(k);
  float run = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const float up = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += up;
  }
  const float goal = u * __shfl_sync(0xffffffffu, run, 31);
  float before = run - sum;
  int at = -1, last = -1;
  float rest = 0.f, last_rest = 0.f;
  for (int k = k0; k < k1; ++k) {
    const float mine = w(k);
    if (mine > 0.f) {
      last = k;
      last_rest = goal - before;
      if (at < 0 && before + mine > goal) {
        at = k;
        rest = last_rest;
      }
    }
    before += mine;
  }
  const uint32_t found = __ballot_sync(0xffffffffu, at >= 0), any = __ballot_sync(0xffffffffu, last >= 0);
  if (any == 0) {
    left = 0.f;
    return -1;
  }
  const int from = found ? __ffs(found) - 1 : 31 - __clz(any);
  left = __shfl_sync(0xffffffffu, found ? rest : last_rest, from);
  return __shfl_sync(0xffffffffu, found ? at : last, from);
}

// The place within a segment at which the running sum of the weights of its elements passes `left`
// (the last with any weight where rounding leaves none; -1: none has any). The segment begins at element lo
// of its nb blocks; w(k, x): the weights of block k's elements.
template <typename T, typename W>
__device__ __forceinline__ int locate(int lo, int nb, float left, int lane, W w) {
  constexpr int N = Elem<T>::N;
  int last = -1;
  float before = 0.f;
#pragma unroll 1
  for (int k0 = 0; k0 < nb; k0 += 32) {
    const int k = k0 + lane;
    float x[N], sum = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = 0.f;
    if (k < nb) w(k, x);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      sum += x[e];
      if (x[e] > 0.f) last = k * N + e - lo;
    }
    float run = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const float up = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += up;
    }
    const uint32_t over = __ballot_sync(0xffffffffu, sum > 0.f && before + run > left);
    if (over) {
      const int from = __ffs(over) - 1;
      float acc = before + (run - sum);
      int at = -1;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        acc += x[e];
        if (at < 0 && x[e] > 0.f && acc > left) at = k * N + e - lo;
      }
      return __shfl_sync(0xffffffffu, at >= 0 ? at : last, from);
    }
    before += __shfl_sync(0xffffffffu, run, 31);
  }
  return static_cast<int>(__reduce_max_sync(0xffffffffu, last));
}

}  // namespace seg
}  // namespace rl
