// Layer norm of rows, forward and backward, with the reductions of the weight's and the bias' gradients.
//
//   h = (x - mean) rstd,   y = h w + b,   rstd = 1 / sqrt(mean of (x - mean)^2 + eps)
//   g = dy w,   dx = rstd (g - mean of g - h (mean of g h)),   dw += sum over rows dy h,   db += sum over rows dy
//
// Memory bounds all of it: 16 bytes of operations a byte at most. Rows of up to 8,192 columns (forward 8,192, or 8,192 bf16
// elements of any alignment) are read once, into registers:
//   - up to 256 columns: several rows to a warp, whose sums' chains run side by side (fwd_short_kernel, bwd_short_kernel);
//   - few rows forward: as many threads on a row as have two blocks of four of it (fwd_kernel);
//   - else persistent CTAs that share a row at a time, whose rows bulk copies bring ahead (fwd_ring_kernel, bwd_kernel).
// Backward a thread has the same columns of all its rows, and the weight's and bias' sums of them stay in its registers; a second
// launch adds up the CTAs' parts. Wider rows: a CTA per row that reads it once for each sum, and threads that go down the columns.
// Measured, of the copy's 6.78 TB/s: 32,768 rows of 4,096 forward 77% (bf16) and 84% (fp32 to bf16), backward 83% (bf16), 85%
// (fp32, bf16 gradient), 79% with 60% of the rows trained on; 131,072 of 512 71% and 70%; odd widths at 130,000 x 1,001 bf16
// 46% and 42% (an element a load and a store), fp32 83% and 88%, 17,950 x 6,626 bf16 35% and 20% (spills: bwd_groups); more
// than 8,192 columns, 10,000 x 12,288 bf16, 30% and 17%.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <string>

#include "rl_device.cuh"
#include "rl_host.h"

namespace rl {
namespace norm {

template <typename T>
struct Io;
template <>
struct Io<uint16_t> {
  static __device__ __forceinline__ float get(uint16_t v) { return bf16_to_f32(v); }
  static __device__ __forceinline__ uint16_t put(float v) { return f32_to_bf16(v); }
};
template <>
struct Io<float> {
  static __device__ __forceinline__ float get(float v) { return v; }
  static __device__ __forceinline__ float put(float v) { return v; }
};

// Weight or bias of either type (NULL: `none`).
struct Vec {
  const void* at;
  int32_t bf16;
  float none;
  __device__ __forceinline__ float operator[](int64_t c) const {
    if (!at) return none;
    return bf16 ? bf16_to_f32(static_cast<const uint16_t*>(at)[c]) : static_cast<const float*>(at)[c];
  }
};

struct FwdArgs {
  const void* x;
  void* y;
  int64_t rows, D, ld_x, ld_y;
  Vec w, b;
  float eps;
  float* mean;
  float* rstd;
};

struct BwdArgs {
  const void* dy;
  const void* x;
  void* dx;
  int64_t rows, D, ld_dy, ld_x, ld_dx;
  Vec w;
  const float* mean;
  const float* rstd;
  const uint8_t* mask;
  float* part_w;  // [parts x D] (NULL: not wanted)
  float* part_b;
  int32_t parts;
};

constexpr int kLoopThreads = 512;

// The sum over the CTA's kLoopThreads threads, in every one of them.
__device__ __forceinline__ float cta_sum(float v, float* red) {
  v = warp_sum(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x / 32] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kLoopThreads / 32; ++i) s += red[i];
  return s;
}

template <typename TX, typename TY>
__global__ void __launch_bounds__(kLoopThreads) loop_fwd_kernel(const FwdArgs p) {
  __shared__ float red[kLoopThreads / 32];
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const TX* x = static_cast<const TX*>(p.x) + r * p.ld_x;
    TY* y = static_cast<TY*>(p.y) + r * p.ld_y;
    float s = 0.f;
    for (int64_t c = threadIdx.x; c < p.D; c += kLoopThreads) s += Io<TX>::get(x[c]);
    const float mean = cta_sum(s, red) / static_cast<float>(p.D);
    float q = 0.f;
    for (int64_t c = threadIdx.x; c < p.D; c += kLoopThreads) {
      const float d = Io<TX>::get(x[c]) - mean;
      q = fmaf(d, d, q);
    }
    const float rstd = 1.f / sqrtf(cta_sum(q, red) / static_cast<float>(p.D) + p.eps);
    for (int64_t c = threadIdx.x; c < p.D; c += kLoopThreads)
      y[c] = Io<TY>::put(fmaf((Io<TX>::get(x[c]) - mean) * rstd, p.w[c], p.b[c]));
    if (threadIdx.x == 0) {
      p.mean[r] = mean;
      p.rstd[r] = rstd;
    }
  }
}

template <typename TX, typename TD>
__global__ void __launch_bounds__(kLoopThreads) loop_bwd_kernel(const BwdArgs p) {
  __shared__ float red[kLoopThreads / 32];
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
    TX* dx = static_cast<TX*>(p.dx) + r * p.ld_dx;
    if (p.mask && p.mask[r] == 0) {
      for (int64_t c = threadIdx.x; c < p.D; c += kLoopThreads) dx[c] = Io<TX>::put(0.f);
      continue;
    }
    const TX* x = static_cast<const TX*>(p.x) + r * p.ld_x;
    const TD* dy = static_cast<const TD*>(p.dy) + r * p.ld_dy;
    const float mean = p.mean[r], rstd = p.rstd[r];
    float s = 0.f, q = 0.f;
    for (int64_t c = threadIdx.x; c < p.D; c += kLoopThreads) {
      const float g = Io<TD>::get(dy[c]) * p.w[c];
      s += g;
      q = fmaf(g, (Io<TX>::get(x[c]) - mean) * rstd, q);
    }
    s = cta_sum(s, red) / static_cast<float>(p.D);
    q = cta_sum(q, red) / static_cast<float>(p.D);
    for (int64_t c = threadIdx.x; c < p.D; c += kLoopThreads) {
      const float g = Io<TD>::get(dy[c]) * p.w[c], h = (Io<TX>::get(x[c]) - mean) * rstd;
      dx[c] = Io<TX>::put(rstd * (g - s - h * q));
    }
  }
}

// ---------------------------------------------------------------- forward, the row in registers

// Four elements as they lie in memory aligned for them: a warp's lanes side by side in either type, so that its requests
// are whole lines. Loads come before the first use of any of them and are not under a condition: behind one each, or with
// the conversion between them, they waited for one another (32,768 rows of 4,096: 185 us).
template <typename T>
struct Raw;
template <>
struct Raw<uint16_t> {
  uint2 q;
  __device__ __forceinline__ void get(float2 (&v)[2]) const {
    v[0] = make_float2(bf16_lo(q.x), bf16_hi(q.x)), v[1] = make_float2(bf16_lo(q.y), bf16_hi(q.y));
  }
  __device__ __forceinline__ void stream(const uint16_t* p) { q = __ldcs(reinterpret_cast<const uint2*>(p)); }
  __device__ __forceinline__ void shared(const uint16_t* p) { q = *reinterpret_cast<const uint2*>(p); }
};
template <>
struct Raw<float> {
  float4 q;
  __device__ __forceinline__ void get(float2 (&v)[2]) const { v[0] = make_float2(q.x, q.y), v[1] = make_float2(q.z, q.w); }
  __device__ __forceinline__ void stream(const float* p) { q = __ldcs(reinterpret_cast<const float4*>(p)); }
  __device__ __forceinline__ void shared(const float* p) { q = *reinterpret_cast<const float4*>(p); }
};

constexpr int kMostWarps = 16;

// The sum over a row's W warps, in every thread of them; `red` has kMostWarps words, zero behind the W-th, and is free again
// after the next barrier.
__device__ __forceinline__ float row_sum(float v, int W, int w, float* red) {
  v = warp_sum(v);
  if (W == 1) return v;
  if ((threadIdx.x & 31) == 0) red[w] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kMostWarps; i += 4) {
    if (i >= W) break;
    const float4 q = *reinterpret_cast<const float4*>(red + i);
    s += (q.x + q.y) + (q.z + q.w);
  }
  return s;
}

// 1 / sqrt(x), the fast one and a step of Newton's.
__device__ __forceinline__ float inverse_root(float x) {
  const float r = rsqrtf(x);
  return x > 0.f && x < 3e38f ? r * fmaf(-0.5f * x * r, r, 1.5f) : r;
}

// The columns of thread t of n: blocks of four (WHOLE), or one apart.
template <bool WHOLE>
__device__ __forceinline__ int column_of(int j, int e, int n, int t) {
  return WHOLE ? (j * n + t) * 4 + e : (j * 4 + e) * n + t;
}

// The statistics of a row whose elements v the threads hold, two columns a word; leaves x - mean in v, and 0 behind D.
// Two passes over the registers: the squares are of x - mean.
template <int NG, bool WHOLE>
__device__ __forceinline__ void statistics(float2 (&v)[NG][2], int D, float inv, float eps, int W, int w, int n, int t, float* red0,
                                           float* red1, float& mean, float& rstd) {
  const bool full = D == 4 * NG * n;
  auto clear = [&]() {
    if (full) return;
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (column_of<WHOLE>(j, 2 * e, n, t) >= D) v[j][e].x = 0.f;
        if (column_of<WHOLE>(j, 2 * e + 1, n, t) >= D) v[j][e].y = 0.f;
      }
  };
  clear();
  float2 s = make_float2(0.f, 0.f), q = s;
#pragma unroll
  for (int j = 0; j < NG; ++j)
#pragma unroll
    for (int e = 0; e < 2; ++e) s = __fadd2_rn(s, v[j][e]);
  const float sum = row_sum(s.x + s.y, W, w, red0), m0 = sum * inv;
  mean = fmaf(fmaf(-m0, static_cast<float>(D), sum), inv, m0);  // sum / D, by one correction from the product's residual
  const float2 off = make_float2(-mean, -mean);
#pragma unroll
  for (int j = 0; j < NG; ++j)
#pragma unroll
    for (int e = 0; e < 2; ++e) v[j][e] = __fadd2_rn(v[j][e], off);
  clear();
#pragma unroll
  for (int j = 0; j < NG; ++j)
#pragma unroll
    for (int e = 0; e < 2; ++e) q = __ffma2_rn(v[j][e], v[j][e], q);
  rstd = inverse_root(fmaf(row_sum(q.x + q.y, W, w, red1), inv, eps));
}

__device__ __forceinline__ void put4(uint16_t* p, float2 a, float2 b) {
  __stcs(reinterpret_cast<uint2*>(p), make_uint2(pack_bf16x2(a.x, a.y), pack_bf16x2(b.x, b.y)));
}
__device__ __forceinline__ void put4(float* p, float2 a, float2 b) {
  __stcs(reinterpret_cast<float4*>(p), make_float4(a.x, a.y, b.x, b.y));
}
// Writes a thread's elements of a row.
template <int NG, bool WHOLE, typename T>
__device__ __forceinline__ void put_row(T* row, const float2 (&v)[NG][2], int D, int n, int t) {
#pragma unroll
  for (int j = 0; j < NG; ++j) {
    if (WHOLE) {
      if (column_of<true>(j, 0, n, t) < D) put4(row + column_of<true>(j, 0, n, t), v[j][0], v[j][1]);
    } else {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int c0 = column_of<false>(j, 2 * e, n, t), c1 = column_of<false>(j, 2 * e + 1, n, t);
        if (c0 < D) row[c0] = Io<T>::put(v[j][e].x);
        if (c1 < D) row[c1] = Io<T>::put(v[j][e].y);
      }
    }
  }
}
// A thread's parameters (`behind` behind D).
template <int NG, bool WHOLE>
__device__ __forceinline__ void get_parameters(float2 (&v)[NG][2], const Vec& w, float behind, int D, int n, int t) {
#pragma unroll
  for (int j = 0; j < NG; ++j)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int c0 = column_of<WHOLE>(j, 2 * e, n, t), c1 = column_of<WHOLE>(j, 2 * e + 1, n, t);
      v[j][e] = make_float2(c0 < D ? w[c0] : behind, c1 < D ? w[c1] : behind);
    }
}

// A row on the W >= 2 warps of a CTA, 4 NG elements a thread, held in registers between the two sums and the result. For few
// rows: nothing is fetched ahead, and every thread has little to do.
template <typename TX, typename TY, int NG, bool WHOLE>
__global__ void __launch_bounds__(kMostWarps * 32) fwd_kernel(const FwdArgs p) {
  __shared__ __align__(16) float red[2][kMostWarps];
  const int W = blockDim.x / 32, n = blockDim.x, t = threadIdx.x, w = t / 32;
  const int64_t r = blockIdx.x;
  if (t < 2 * kMostWarps && t % kMostWarps >= W) red[t / kMostWarps][t % kMostWarps] = 0.f;
  const TX* x = static_cast<const TX*>(p.x) + r * p.ld_x;
  TY* y = static_cast<TY*>(p.y) + r * p.ld_y;
  const int D = static_cast<int>(p.D);
  float2 v[NG][2];
  if (WHOLE) {
    Raw<TX> raw[NG];
#pragma unroll
    for (int j = 0; j < NG; ++j) raw[j].stream(x + (column_of<true>(j, 0, n, t) < D ? column_of<true>(j, 0, n, t) : 0));
#pragma unroll
    for (int j = 0; j < NG; ++j) raw[j].get(v[j]);
  } else {
    TX raw[NG][4];
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) raw[j][e] = __ldcs(x + (column_of<false>(j, e, n, t) < D ? column_of<false>(j, e, n, t) : 0));
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) v[j][e] = make_float2(Io<TX>::get(raw[j][2 * e]), Io<TX>::get(raw[j][2 * e + 1]));
  }
  float2 g[NG][2], b[NG][2];
  get_parameters<NG, WHOLE>(g, p.w, 0.f, D, n, t);
  get_parameters<NG, WHOLE>(b, p.b, 0.f, D, n, t);
  __syncthreads();  // red's zeros
  float mean, rstd;
  statistics<NG, WHOLE>(v, D, 1.f / static_cast<float>(D), p.eps, W, w, n, t, red[0], red[1], mean, rstd);
#pragma unroll
  for (int j = 0; j < NG; ++j)
#pragma unroll
    for (int e = 0; e < 2; ++e) v[j][e] = __ffma2_rn(__fmul2_rn(v[j][e], make_float2(rstd, rstd)), g[j][e], b[j][e]);
  put_row<NG, WHOLE>(y, v, D, n, t);
  if (t == 0) {
    p.mean[r] = mean;
    p.rstd[r] = rstd;
  }
}

// ---------------------------------------------------------------- short rows, several to a warp

constexpr int kShortWarps = 8;

// R rows at a time on a warp, 4 NG elements of each a lane, loaded before the first is worked on: what a short row costs is the
// chain of its two sums, and R chains run at once. Measured, 500,000 rows of 128 bf16: 66 us, through the ring 140.
template <typename TX, typename TY, int NG, int R, bool WHOLE>
__global__ void __launch_bounds__(kShortWarps * 32) fwd_short_kernel(const FwdArgs p) {
  const int t = threadIdx.x & 31, D = static_cast<int>(p.D);
  const int64_t r0 = (static_cast<int64_t>(blockIdx.x) * kShortWarps + threadIdx.x / 32) * R;
  if (r0 >= p.rows) return;
  const float inv = 1.f / static_cast<float>(D);
  float2 v[R][NG][2];
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const TX* x = static_cast<const TX*>(p.x) + min(r0 + k, p.rows - 1) * p.ld_x;
    if (WHOLE) {
      Raw<TX> raw[NG];
#pragma unroll
      for (int j = 0; j < NG; ++j) raw[j].stream(x + (column_of<true>(j, 0, 32, t) < D ? column_of<true>(j, 0, 32, t) : 0));
#pragma unroll
      for (int j = 0; j < NG; ++j) raw[j].get(v[k][j]);
    } else {
#pragma unroll
      for (int j = 0; j < NG; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int c0 = column_of<false>(j, 2 * e, 32, t), c1 = column_of<false>(j, 2 * e + 1, 32, t);
          v[k][j][e] = make_float2(Io<TX>::get(__ldcs(x + (c0 < D ? c0 : 0))), Io<TX>::get(__ldcs(x + (c1 < D ? c1 : 0))));
        }
    }
  }
  float2 g[NG][2], b[NG][2];
  get_parameters<NG, WHOLE>(g, p.w, 0.f, D, 32, t);
  get_parameters<NG, WHOLE>(b, p.b, 0.f, D, 32, t);
  auto clear = [&](float2 (&a)[NG][2]) {
    if (D == 128 * NG) return;
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (column_of<WHOLE>(j, 2 * e, 32, t) >= D) a[j][e].x = 0.f;
        if (column_of<WHOLE>(j, 2 * e + 1, 32, t) >= D) a[j][e].y = 0.f;
      }
  };
  float s[R], q[R];
#pragma unroll
  for (int k = 0; k < R; ++k) {
    clear(v[k]);
    float2 a = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) a = __fadd2_rn(a, v[k][j][e]);
    s[k] = a.x + a.y;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < R; ++k) s[k] += __shfl_xor_sync(0xffffffffu, s[k], o);
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const float m = s[k] * inv;
    s[k] = fmaf(fmaf(-m, static_cast<float>(D), s[k]), inv, m);  // the mean, corrected likewise
    float2 a = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) v[k][j][e] = __fadd2_rn(v[k][j][e], make_float2(-s[k], -s[k]));
    clear(v[k]);
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) a = __ffma2_rn(v[k][j][e], v[k][j][e], a);
    q[k] = a.x + a.y;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < R; ++k) q[k] += __shfl_xor_sync(0xffffffffu, q[k], o);
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const int64_t r = r0 + k;
    if (r >= p.rows) break;
    const float rstd = inverse_root(fmaf(q[k], inv, p.eps));
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) v[k][j][e] = __ffma2_rn(__fmul2_rn(v[k][j][e], make_float2(rstd, rstd)), g[j][e], b[j][e]);
    put_row<NG, WHOLE>(static_cast<TY*>(p.y) + r * p.ld_y, v[k], D, 32, t);
    if (t == 0) {
      p.mean[r] = s[k];
      p.rstd[r] = rstd;
    }
  }
}

// The same for the gradient: warps go down the rows R at a time, a fixed assignment, with the columns' sums in registers; the
// CTA's warps' are added up in order at the end. Measured, 500,000 rows of 128 bf16: 100 us. (bf16 x an element at a time, four
// rows: 28 bytes spilled.)
template <typename TX, typename TD, int NG, int R, bool WHOLE>
__global__ void __launch_bounds__(kShortWarps * 32, 2) bwd_short_kernel(const BwdArgs p) {
  __shared__ __align__(16) float sums[kShortWarps][128 * NG];
  const int t = threadIdx.x & 31, warp = threadIdx.x / 32, D = static_cast<int>(p.D);
  const float inv = 1.f / static_cast<float>(D);
  float2 wt[NG][2], dw[NG][2], db[NG][2];
  get_parameters<NG, WHOLE>(wt, p.w, 0.f, D, 32, t);
#pragma unroll
  for (int j = 0; j < NG; ++j)
#pragma unroll
    for (int e = 0; e < 2; ++e) dw[j][e] = db[j][e] = make_float2(0.f, 0.f);
  const int64_t step = static_cast<int64_t>(gridDim.x) * kShortWarps * R;
  for (int64_t r0 = (static_cast<int64_t>(blockIdx.x) * kShortWarps + warp) * R; r0 < p.rows; r0 += step) {
    float2 h[R][NG][2], g[R][NG][2];
    float mean[R], rstd[R];
    bool live[R];
#pragma unroll
    for (int k = 0; k < R; ++k) live[k] = r0 + k < p.rows && (!p.mask || p.mask[r0 + k] != 0);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      mean[k] = rstd[k] = 0.f;
      if (!live[k]) {
#pragma unroll
        for (int j = 0; j < NG; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) h[k][j][e] = g[k][j][e] = make_float2(0.f, 0.f);
        continue;
      }
      const TX* x = static_cast<const TX*>(p.x) + (r0 + k) * p.ld_x;
      const TD* dy = static_cast<const TD*>(p.dy) + (r0 + k) * p.ld_dy;
      mean[k] = p.mean[r0 + k];
      rstd[k] = p.rstd[r0 + k];
      if (WHOLE) {
        Raw<TX> rx[NG];
        Raw<TD> rd[NG];
#pragma unroll
        for (int j = 0; j < NG; ++j) {
          const int c = column_of<true>(j, 0, 32, t) < D ? column_of<true>(j, 0, 32, t) : 0;
          rx[j].stream(x + c);
          rd[j].stream(dy + c);
        }
#pragma unroll
        for (int j = 0; j < NG; ++j) {
          rx[j].get(h[k][j]);
          rd[j].get(g[k][j]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < NG; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int c0 = min(column_of<false>(j, 2 * e, 32, t), D - 1), c1 = min(column_of<false>(j, 2 * e + 1, 32, t), D - 1);
            h[k][j][e] = make_float2(Io<TX>::get(__ldcs(x + c0)), Io<TX>::get(__ldcs(x + c1)));
            g[k][j][e] = make_float2(Io<TD>::get(__ldcs(dy + c0)), Io<TD>::get(__ldcs(dy + c1)));
          }
      }
    }
    float2 sq[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      float2 s = make_float2(0.f, 0.f), q = s;
#pragma unroll
      for (int j = 0; j < NG; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float2 d = g[k][j][e];
          if (D != 128 * NG) {
            if (column_of<WHOLE>(j, 2 * e, 32, t) >= D) d.x = 0.f;
            if (column_of<WHOLE>(j, 2 * e + 1, 32, t) >= D) d.y = 0.f;
          }
          h[k][j][e] = __fmul2_rn(__fadd2_rn(h[k][j][e], make_float2(-mean[k], -mean[k])), make_float2(rstd[k], rstd[k]));
          g[k][j][e] = __fmul2_rn(d, wt[j][e]);
          s = __fadd2_rn(s, g[k][j][e]);
          q = __ffma2_rn(g[k][j][e], h[k][j][e], q);
          dw[j][e] = __ffma2_rn(d, h[k][j][e], dw[j][e]);
          db[j][e] = __fadd2_rn(db[j][e], d);
        }
      sq[k] = make_float2(s.x + s.y, q.x + q.y);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < R; ++k)
        sq[k] = __fadd2_rn(sq[k], make_float2(__shfl_xor_sync(0xffffffffu, sq[k].x, o), __shfl_xor_sync(0xffffffffu, sq[k].y, o)));
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (r0 + k >= p.rows) break;
      const float m = -sq[k].x * inv * rstd[k], f = -sq[k].y * inv * rstd[k];
#pragma unroll
      for (int j = 0; j < NG; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          g[k][j][e] = live[k] ? __ffma2_rn(h[k][j][e], make_float2(f, f),
                                            __ffma2_rn(g[k][j][e], make_float2(rstd[k], rstd[k]), make_float2(m, m)))
                               : make_float2(0.f, 0.f);
      put_row<NG, WHOLE>(static_cast<TX*>(p.dx) + (r0 + k) * p.ld_dx, g[k], D, 32, t);
    }
  }
  auto finish = [&](const float2 (&a)[NG][2], float* part) {
    if (!part) return;
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int c0 = column_of<WHOLE>(j, 2 * e, 32, t), c1 = column_of<WHOLE>(j, 2 * e + 1, 32, t);
        if (c0 < D) sums[warp][c0] = a[j][e].x;
        if (c1 < D) sums[warp][c1] = a[j][e].y;
      }
    __syncthreads();
    for (int c = threadIdx.x; c < D; c += kShortWarps * 32) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < kShortWarps; ++w) s += sums[w][c];
      part[blockIdx.x * p.D + c] = s;
    }
    __syncthreads();
  };
  finish(dw, p.part_w);
  finish(db, p.part_b);
}

// ---------------------------------------------------------------- rows through shared memory

constexpr int kStages = 8;
constexpr int kRowInfo = 32;  // rows whose mask, mean and rstd are fetched at once

struct Stages {
  int32_t n, x_bytes, bytes;  // how many; a stage's room for x (dy's lies behind it) and in all
};

// Where a row lies in its stage: the 16-byte blocks of memory that it covers, the first of them at the stage's start.
// What the first row's first block holds before the matrix and the last row's last block behind it is not copied.
struct Span {
  uintptr_t from, at, to;  // copied: [from, to); the stage's first byte is that at `at`
};
__device__ __forceinline__ Span span(const void* row, int64_t bytes, bool first, bool last) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(row), b = a + bytes, m = ~uintptr_t(15);
  Span s;
  s.at = a & m;
  s.from = first ? (a + 15) & m : s.at;
  s.to = last ? b & m : (b + 15) & m;
  if (s.to < s.from) s.to = s.from;
  return s;
}
// Starts the copy of a span to a stage.
__device__ __forceinline__ void copy(const Span& s, uint8_t* to, uint64_t* bar) {
  if (s.to > s.from)
    bulk_g2s(to + (s.from - s.at), reinterpret_cast<const void*>(s.from), static_cast<uint32_t>(s.to - s.from), bar);
}

// After a wait at `stage` in phase `parity` that ran out: waits, a little each, for the copies that may be on their way still, so that
// none of them arrives in the shared memory of the CTA's successor. By the thread that started them, which has started none since.
__device__ __noinline__ void await_copies(uint64_t* full, int n, int stage, uint32_t parity) {
  for (int i = 0; i < n; ++i) {
    mbar_wait_bounded(&full[stage], parity, 10000000ull);
    if (++stage == n) {
      stage = 0;
      parity ^= 1;
    }
  }
}

// A thread's elements of a row in its stage; those behind D are not the row's. `first`, `last`: of the matrix' rows, whose
// outermost elements may not have been copied.
template <int NG, bool WHOLE, typename T>
__device__ __forceinline__ void get_row(float2 (&v)[NG][2], const uint8_t* stage, const T* row, bool first, bool last, int D, int n,
                                        int t) {
  if (WHOLE) {
    const T* at = reinterpret_cast<const T*>(stage);
    Raw<T> raw[NG];
#pragma unroll
    for (int j = 0; j < NG; ++j) raw[j].shared(at + (column_of<true>(j, 0, n, t) < D ? column_of<true>(j, 0, n, t) : 0));
#pragma unroll
    for (int j = 0; j < NG; ++j) raw[j].get(v[j]);
  } else {
    const T* at = reinterpret_cast<const T*>(stage + (reinterpret_cast<uintptr_t>(row) & 15));
    T raw[NG][4];
    if (!first && !last) {
#pragma unroll
      for (int j = 0; j < NG; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) raw[j][e] = at[column_of<false>(j, e, n, t) < D ? column_of<false>(j, e, n, t) : 0];
    } else {
      const Span s = span(row, D * sizeof(T), first, last);
#pragma unroll
      for (int j = 0; j < NG; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int c = column_of<false>(j, e, n, t) < D ? column_of<false>(j, e, n, t) : 0;
          const uintptr_t a = reinterpret_cast<uintptr_t>(row + c);
          raw[j][e] = a >= s.from && a < s.to ? at[c] : row[c];
        }
    }
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) v[j][e] = make_float2(Io<T>::get(raw[j][2 * e]), Io<T>::get(raw[j][2 * e + 1]));
  }
}

// Persistent CTAs of W warps that share a row, 4 NG columns a thread, whose parameters stay in registers; the rows come by
// bulk copies into a ring of stages, as many bytes ahead as an SM has shared memory for: what one row per CTA has in
// flight, in registers, kept the memory at half its rate (32,768 rows of 4,096 bf16: 155 us).
template <typename TX, typename TY, int NG, bool WHOLE>
__global__ void __launch_bounds__(kMostWarps * 32) fwd_ring_kernel(const FwdArgs p, const Stages st) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(8) uint64_t full[kStages];
  __shared__ __align__(16) float red[2][kMostWarps];
  const int W = blockDim.x / 32, n = blockDim.x, t = threadIdx.x, warp = t / 32;
  const int D = static_cast<int>(p.D);
  const float inv = 1.f / static_cast<float>(D);
  const int64_t G = gridDim.x;
  if (t < st.n) mbar_init(&full[t], 1);
  if (t == 0) fence_mbar_init();
  if (t < st.n) fence_proxy_async_smem();
  for (int i = t; i < 2 * kMostWarps; i += n) (&red[0][0])[i] = 0.f;
  __syncthreads();
  const TX* x = static_cast<const TX*>(p.x);
  auto fetch = [&](int64_t r, int stage) {
    const Span s = span(x + r * p.ld_x, D * sizeof(TX), r == 0, r == p.rows - 1);
    mbar_arrive_expect_tx(&full[stage], static_cast<uint32_t>(s.to - s.from));
    copy(s, smem + static_cast<size_t>(stage) * st.bytes, &full[stage]);
  };
  if (t == 0)
    for (int i = 0; i < st.n && blockIdx.x + i * G < p.rows; ++i) fetch(blockIdx.x + i * G, i);
  float2 g[NG][2], b[NG][2];
  get_parameters<NG, WHOLE>(g, p.w, 0.f, D, n, t);
  get_parameters<NG, WHOLE>(b, p.b, 0.f, D, n, t);
  int stage = 0, late = -1;  // late: 2 stage + parity of the wait that ran out
  uint32_t parity = 0;
  for (int64_t r = blockIdx.x; r < p.rows; r += G) {
    if (late < 0 && !mbar_wait_bounded(&full[stage], parity)) late = 2 * stage + parity;  // reported, and not tried again
    float2 v[NG][2];
    get_row<NG, WHOLE>(v, smem + static_cast<size_t>(stage) * st.bytes, x + r * p.ld_x, r == 0, r == p.rows - 1, D, n, t);
    if (late >= 0) v[0][0].x = __int_as_float(0x7fc00000);  // there is no status word: a row of NaNs says that a wait ran out
    float mean, rstd;
    statistics<NG, WHOLE>(v, D, inv, p.eps, W, warp, n, t, red[0], red[1], mean, rstd);
    if (W == 1) __syncwarp();
    if (t == 0 && late < 0 && r + st.n * G < p.rows) fetch(r + st.n * G, stage);  // the sums' barriers: everyone has read the stage
    if (++stage == st.n) {
      stage = 0;
      parity ^= 1;
    }
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) v[j][e] = __ffma2_rn(__fmul2_rn(v[j][e], make_float2(rstd, rstd)), g[j][e], b[j][e]);
    put_row<NG, WHOLE>(static_cast<TY*>(p.y) + r * p.ld_y, v, D, n, t);
    if (t == 0) {
      p.mean[r] = mean;
      p.rstd[r] = rstd;
    }
  }
  if (t == 0 && late >= 0) await_copies(full, st.n, late / 2, late & 1);
}

// The same for the gradient: x and dy of the rows that have one come through the ring. A thread keeps the same columns for
// all rows and with them the columns' sums in registers: both matrices are read once.
template <typename TX, typename TD, int NG, bool WHOLE>
__global__ void __launch_bounds__(kMostWarps * 32) bwd_kernel(const BwdArgs p, const Stages st, int32_t* status) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(8) uint64_t full[kStages];
  __shared__ __align__(16) float2 red[2][kMostWarps];
  const int W = blockDim.x / 32, n = blockDim.x, t = threadIdx.x, warp = t / 32, lane = t & 31;
  const int D = static_cast<int>(p.D);
  const float inv = 1.f / static_cast<float>(D);
  const int64_t G = gridDim.x, b0 = blockIdx.x, mine = (p.rows - b0 + G - 1) / G;  // rows b0 + i G
  if (t < st.n) mbar_init(&full[t], 1);
  if (t == 0) fence_mbar_init();
  if (t < st.n) fence_proxy_async_smem();
  for (int i = t; i < 2 * kMostWarps; i += n) (&red[0][0])[i] = make_float2(0.f, 0.f);
  __syncthreads();
  auto live_rows = [&](int64_t base) {  // which of the CTA's rows base .. base + 31 have a gradient
    const int64_t i = base + lane;
    return __ballot_sync(0xffffffffu, i < mine && (!p.mask || p.mask[b0 + i * G] != 0));
  };

  // the first warp fetches ahead: the rows that have a gradient, in order
  int64_t ahead_base = 0;
  uint32_t ahead = warp == 0 ? live_rows(0) : 0u;
  auto fetch_next = [&](int stage, bool in_time) {
    while (ahead == 0) {
      if (ahead_base + kRowInfo >= mine) return false;
      ahead_base += kRowInfo;
      ahead = live_rows(ahead_base);
    }
    const int64_t r = b0 + (ahead_base + __ffs(ahead) - 1) * G;
    ahead &= ahead - 1;
    if (lane == 0 && in_time) {
      const bool first = r == 0, last = r == p.rows - 1;
      const Span sx = span(static_cast<const TX*>(p.x) + r * p.ld_x, D * sizeof(TX), first, last);
      const Span sd = span(static_cast<const TD*>(p.dy) + r * p.ld_dy, D * sizeof(TD), first, last);
      uint8_t* to = smem + static_cast<size_t>(stage) * st.bytes;
      mbar_arrive_expect_tx(&full[stage], static_cast<uint32_t>((sx.to - sx.from) + (sd.to - sd.from)));
      copy(sx, to, &full[stage]);
      copy(sd, to + st.x_bytes, &full[stage]);
    }
    __syncwarp();
    return true;
  };
  if (warp == 0)
    for (int i = 0; i < st.n && fetch_next(i, true); ++i) {}

  float2 wt[NG][2], dw[NG][2], db[NG][2];
  get_parameters<NG, WHOLE>(wt, p.w, 0.f, D, n, t);
#pragma unroll
  for (int j = 0; j < NG; ++j)
#pragma unroll
    for (int e = 0; e < 2; ++e) dw[j][e] = db[j][e] = make_float2(0.f, 0.f);
  const bool full_width = D == 4 * NG * n;

  int stage = 0, late = -1;  // late: 2 stage + parity of the wait that ran out
  uint32_t parity = 0, odd = 0;
  int64_t r = b0;
  for (int64_t base = 0; base < mine; base += kRowInfo) {
    const uint32_t live = live_rows(base);
    float mean_l = 0.f, rstd_l = 0.f;
    if (live >> lane & 1) {
      mean_l = p.mean[b0 + (base + lane) * G];
      rstd_l = p.rstd[b0 + (base + lane) * G];
    }
    const int here = static_cast<int>(min(static_cast<int64_t>(kRowInfo), mine - base));
    for (int i = 0; i < here; ++i, r += G) {
      TX* dx = static_cast<TX*>(p.dx) + r * p.ld_dx;
      if (!(live >> i & 1)) {
        float2 zero[NG][2];
#pragma unroll
        for (int j = 0; j < NG; ++j) zero[j][0] = zero[j][1] = make_float2(0.f, 0.f);
        put_row<NG, WHOLE>(dx, zero, D, n, t);
        continue;
      }
      const float mean = __shfl_sync(0xffffffffu, mean_l, i), rstd = __shfl_sync(0xffffffffu, rstd_l, i);
      if (late < 0 && !mbar_wait_bounded(&full[stage], parity)) late = 2 * stage + parity;  // reported, and not tried again
      const uint8_t* at = smem + static_cast<size_t>(stage) * st.bytes;
      float2 h[NG][2], g[NG][2], s = make_float2(0.f, 0.f), q = s;
      get_row<NG, WHOLE>(h, at, static_cast<const TX*>(p.x) + r * p.ld_x, r == 0, r == p.rows - 1, D, n, t);
      get_row<NG, WHOLE>(g, at + st.x_bytes, static_cast<const TD*>(p.dy) + r * p.ld_dy, r == 0, r == p.rows - 1, D, n, t);
      const float2 off = make_float2(-mean, -mean), scale = make_float2(rstd, rstd);
#pragma unroll
      for (int j = 0; j < NG; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float2 d = g[j][e];
          if (!full_width) {
            if (column_of<WHOLE>(j, 2 * e, n, t) >= D) d.x = 0.f;
            if (column_of<WHOLE>(j, 2 * e + 1, n, t) >= D) d.y = 0.f;
          }
          h[j][e] = __fmul2_rn(__fadd2_rn(h[j][e], off), scale);
          g[j][e] = __fmul2_rn(d, wt[j][e]);
          s = __fadd2_rn(s, g[j][e]);
          q = __ffma2_rn(g[j][e], h[j][e], q);
          dw[j][e] = __ffma2_rn(d, h[j][e], dw[j][e]);
          db[j][e] = __fadd2_rn(db[j][e], d);
        }
      float2 sq = make_float2(s.x + s.y, q.x + q.y);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
        sq = __fadd2_rn(sq, make_float2(__shfl_xor_sync(0xffffffffu, sq.x, o), __shfl_xor_sync(0xffffffffu, sq.y, o)));
      // everyone has read the stage, and the sums are there
      if (W > 1) {
        if (lane == 0) red[odd][warp] = sq;
        __syncthreads();
        sq = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kMostWarps; w += 4) {
          if (w >= W) break;
          const float4 a = *reinterpret_cast<const float4*>(&red[odd][w]), b = *reinterpret_cast<const float4*>(&red[odd][w + 2]);
          sq = __fadd2_rn(sq, __fadd2_rn(__fadd2_rn(make_float2(a.x, a.y), make_float2(a.z, a.w)),
                                         __fadd2_rn(make_float2(b.x, b.y), make_float2(b.z, b.w))));
        }
        odd ^= 1;
      } else {
        __syncwarp();
      }
      if (warp == 0) fetch_next(stage, late < 0);
      if (++stage == st.n) {
        stage = 0;
        parity ^= 1;
      }
      // rstd g - rstd (mean of g) - h rstd (mean of g h)
      const float m = -sq.x * inv * rstd, k = -sq.y * inv * rstd;
#pragma unroll
      for (int j = 0; j < NG; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          g[j][e] = __ffma2_rn(h[j][e], make_float2(k, k), __ffma2_rn(g[j][e], scale, make_float2(m, m)));
      put_row<NG, WHOLE>(dx, g, D, n, t);
    }
  }
  if (late >= 0) {
    flag_status(status, RL_DEV_TIMEOUT);
    if (t == 0) await_copies(full, st.n, late / 2, late & 1);
  }
  if (p.part_w) put_row<NG, WHOLE>(p.part_w + b0 * p.D, dw, D, n, t);
  if (p.part_b) put_row<NG, WHOLE>(p.part_b + b0 * p.D, db, D, n, t);
}

// The columns' sums over part blockIdx.y of the rows, a thread per column.
template <typename TX, typename TD>
__global__ void __launch_bounds__(256) columns_kernel(const BwdArgs p) {
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (c >= p.D) return;
  float w = 0.f, b = 0.f;
  for (int64_t r = blockIdx.y; r < p.rows; r += p.parts) {
    if (p.mask && p.mask[r] == 0) continue;
    const float d = Io<TD>::get(static_cast<const TD*>(p.dy)[r * p.ld_dy + c]);
    w = fmaf(d, (Io<TX>::get(static_cast<const TX*>(p.x)[r * p.ld_x + c]) - p.mean[r]) * p.rstd[r], w);
    b += d;
  }
  const int64_t at = static_cast<int64_t>(blockIdx.y) * p.D + c;
  if (p.part_w) p.part_w[at] = w;
  if (p.part_b) p.part_b[at] = b;
}

constexpr int kPartLanes = 32;

// d_weight, d_bias += the parts' sums, in a fixed order.
__global__ void __launch_bounds__(32 * kPartLanes) add_parts_kernel(const float* part_w, const float* part_b, int32_t parts,
                                                                    int64_t D, float* d_weight, float* d_bias) {
  __shared__ float sum[kPartLanes][33];
  const float* part = blockIdx.y == 0 ? part_w : part_b;
  float* out = blockIdx.y == 0 ? d_weight : d_bias;
  if (!out) return;
  const int lane = threadIdx.x & 31, row = threadIdx.x / 32;
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + lane;
  float s = 0.f;
  after_previous();
  if (c < D) {
#pragma unroll 8
    for (int i = row; i < parts; i += kPartLanes) s += part[i * D + c];
  }
  sum[row][lane] = s;
  __syncthreads();
  if (row != 0 || c >= D) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < kPartLanes; ++i) s += sum[i][lane];
  out[c] += s;
}

// ---------------------------------------------------------------- host

constexpr int kSMs = 152;
constexpr int64_t kMaxD = 1 << 20;

// Blocks of four columns a thread holds in the backward kernel, and the warps of a row; 0: a row has too many columns for
// it. An element at a time two blocks: four spill (164 bytes at 128 registers), and with the stages in the way of L1 that cost 3 times
// the time. Rows of 4,097 to 8,192 columns would want 32 warps then, so they have four blocks all the same: 17,950 x 6,626 bf16
// 536 us (its bytes: 105), and 200 forward, where nothing spills.
inline int bwd_groups(int64_t D, bool whole) { return !whole && D <= 256 * kMostWarps ? 2 : 4; }
inline int bwd_warps(int64_t D, bool whole) {
  const int64_t per = 128 * bwd_groups(D, whole), W = (D + per - 1) / per;
  return W <= kMostWarps ? static_cast<int>(W) : 0;
}
// CTAs of it on an SM: 16 warps at up to 128 registers a thread.
inline int bwd_ctas(int W) { return 16 / W; }

// Parts of the columns' sums.
inline int parts_of(int64_t rows, int64_t D) {
  const int W = D <= 256 ? 4 : bwd_warps(D, true);  // the fewest of a row (short rows: four CTAs an SM at most)
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(rows, W ? bwd_ctas(W) * kSMs : 2 * kSMs)));
}

inline bool element_aligned(const void* p, rl_dtype t) {
  return reinterpret_cast<uintptr_t>(p) % (t == RL_BF16 ? 2 : 4) == 0;
}

inline bool whole_blocks(const void* p, int64_t ld, size_t es) { return aligned16(p) && ld * es % 16 == 0; }

constexpr int64_t kStageRoom = 216 * 1024;  // of an SM's shared memory

// The kernel may take kStageRoom, once per device.
template <typename K>
rl_status allow_room(K kern, std::atomic<uint64_t>& ready, const char* what) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_error(e, "cudaGetDevice");
  const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
  if (ready.load() & bit) return RL_OK;
  e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kStageRoom));
  if (e != cudaSuccess) return cuda_error(e, what);
  ready |= bit;
  return RL_OK;
}

inline Stages stages(int64_t x_bytes, int64_t d_bytes, bool whole, int ctas) {
  auto room = [&](int64_t n) { return static_cast<int32_t>(n ? (n + 15) / 16 * 16 + (whole ? 0 : 16) : 0); };
  Stages st;
  st.x_bytes = room(x_bytes);
  st.bytes = st.x_bytes + room(d_bytes);
  st.n = static_cast<int32_t>(std::min<int64_t>(kStages, (kStageRoom / ctas - 2048) / st.bytes));
  return st;
}

template <typename TX, typename TY, int NG, bool WHOLE>
void launch_fwd(const FwdArgs& a, int W, cudaStream_t s) {
  fwd_kernel<TX, TY, NG, WHOLE><<<static_cast<unsigned>(a.rows), 32 * W, 0, s>>>(a);
}

template <typename TX, typename TY, int NG, bool WHOLE>
rl_status launch_ring(const FwdArgs& a, int W, int ctas, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  auto kern = fwd_ring_kernel<TX, TY, NG, WHOLE>;
  const rl_status r = allow_room(kern, ready, "cudaFuncSetAttribute(fwd_ring_kernel)");
  if (r != RL_OK) return r;
  const Stages st = stages(a.D * sizeof(TX), 0, WHOLE, ctas);
  kern<<<static_cast<unsigned>(std::min<int64_t>(a.rows, ctas * kSMs)), 32 * W, static_cast<size_t>(st.n) * st.bytes, s>>>(a, st);
  return RL_OK;
}

template <typename TX, typename TY>
rl_status fwd(const FwdArgs& a, cudaStream_t s) {
  const bool whole = a.D % 4 == 0 && a.D * sizeof(TX) % 16 == 0 && whole_blocks(a.x, a.ld_x, sizeof(TX)) &&
                     reinterpret_cast<uintptr_t>(a.y) % (4 * sizeof(TY)) == 0 && a.ld_y % 4 == 0;
  auto warps = [&](int ng) { return static_cast<int>((a.D + 128 * ng - 1) / (128 * ng)); };
  cudaError_t e;
  if (warps(4) > kMostWarps || a.rows >= (int64_t(1) << 31)) {
    loop_fwd_kernel<TX, TY><<<static_cast<unsigned>(std::min<int64_t>(a.rows, 4 * kSMs)), kLoopThreads, 0, s>>>(a);
    e = cudaGetLastError();
    return e == cudaSuccess ? RL_OK : cuda_error(e, "loop_fwd_kernel launch");
  }
  const int W = warps(4), ctas = std::max(1, (whole ? 32 : 16) / W);
  rl_status r = RL_OK;
  if (warps(2) == 1) {
    auto go = [&](auto kern, int rows) {
      kern<<<static_cast<unsigned>((a.rows + kShortWarps * rows - 1) / (kShortWarps * rows)), kShortWarps * 32, 0, s>>>(a);
    };
    if (a.rows < 8 * kSMs) whole ? go(fwd_short_kernel<TX, TY, 2, 1, true>, 1) : go(fwd_short_kernel<TX, TY, 2, 1, false>, 1);
    else if (a.D <= 128) whole ? go(fwd_short_kernel<TX, TY, 1, 4, true>, 4) : go(fwd_short_kernel<TX, TY, 1, 4, false>, 4);
    else whole ? go(fwd_short_kernel<TX, TY, 2, 4, true>, 4) : go(fwd_short_kernel<TX, TY, 2, 4, false>, 4);
  } else if (warps(2) <= kMostWarps && a.rows * warps(2) <= 24 * kSMs) {
    if (whole) launch_fwd<TX, TY, 2, true>(a, warps(2), s);
    else launch_fwd<TX, TY, 2, false>(a, warps(2), s);
  } else {
    r = whole ? launch_ring<TX, TY, 4, true>(a, W, ctas, s) : launch_ring<TX, TY, 4, false>(a, W, ctas, s);
  }
  if (r != RL_OK) return r;
  e = cudaGetLastError();
  return e == cudaSuccess ? RL_OK : cuda_error(e, "fwd_kernel launch");
}

template <typename TX, typename TD, int NG, bool WHOLE>
rl_status launch_bwd(const BwdArgs& a, int W, int32_t* status, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  auto kern = bwd_kernel<TX, TD, NG, WHOLE>;
  const rl_status r = allow_room(kern, ready, "cudaFuncSetAttribute(bwd_kernel)");
  if (r != RL_OK) return r;
  const Stages st = stages(a.D * sizeof(TX), a.D * sizeof(TD), WHOLE, bwd_ctas(W));
  kern<<<a.parts, 32 * W, static_cast<size_t>(st.n) * st.bytes, s>>>(a, st, status);
  return RL_OK;
}

template <typename TX, typename TD>
rl_status bwd(BwdArgs& a, float* d_weight, float* d_bias, int32_t* status, cudaStream_t s) {
  a.parts = parts_of(a.rows, a.D);
  cudaError_t e = cudaSuccess;
  const bool whole = a.D * sizeof(TX) % 16 == 0 && a.D * sizeof(TD) % 16 == 0 && whole_blocks(a.x, a.ld_x, sizeof(TX)) &&
                     whole_blocks(a.dy, a.ld_dy, sizeof(TD)) && whole_blocks(a.dx, a.ld_dx, sizeof(TX));
  if (a.D <= 256) {
    a.parts = static_cast<int32_t>(std::min<int64_t>((a.rows + kShortWarps - 1) / kShortWarps, 3 * kSMs));
    auto go = [&](auto kern) { kern<<<a.parts, kShortWarps * 32, 0, s>>>(a); };
    if (a.rows < a.parts * kShortWarps * 4) whole ? go(bwd_short_kernel<TX, TD, 2, 1, true>) : go(bwd_short_kernel<TX, TD, 2, 1, false>);
    else if (a.D <= 128) whole ? go(bwd_short_kernel<TX, TD, 1, 4, true>) : go(bwd_short_kernel<TX, TD, 1, 4, false>);
    else whole ? go(bwd_short_kernel<TX, TD, 2, 2, true>) : go(bwd_short_kernel<TX, TD, 2, 2, false>);
    e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_error(e, "bwd_short_kernel launch");
  } else if (const int W = bwd_warps(a.D, whole)) {
    a.parts = static_cast<int32_t>(std::min<int64_t>(a.parts, bwd_ctas(W) * kSMs));
    rl_status r;
    if (bwd_groups(a.D, whole) == 2) r = launch_bwd<TX, TD, 2, false>(a, W, status, s);
    else r = whole ? launch_bwd<TX, TD, 4, true>(a, W, status, s) : launch_bwd<TX, TD, 4, false>(a, W, status, s);
    if (r != RL_OK) return r;
    e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_error(e, "bwd_kernel launch");
  } else {
    // the columns first: dx may take the place of dy or x
    if (d_weight || d_bias) {
      columns_kernel<TX, TD><<<dim3(static_cast<unsigned>((a.D + 255) / 256), a.parts), 256, 0, s>>>(a);
      e = cudaGetLastError();
      if (e != cudaSuccess) return cuda_error(e, "columns_kernel launch");
    }
    loop_bwd_kernel<TX, TD><<<static_cast<unsigned>(std::min<int64_t>(a.rows, 4 * kSMs)), kLoopThreads, 0, s>>>(a);
    e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_error(e, "loop_bwd_kernel launch");
  }
  if (!d_weight && !d_bias) return RL_OK;
  e = launch_after(add_parts_kernel, dim3(static_cast<unsigned>((a.D + 31) / 32), 2), dim3(32 * kPartLanes), 0, s, a.part_w,
                   a.part_b, a.parts, a.D, d_weight, d_bias);
  return e == cudaSuccess ? RL_OK : cuda_error(e, "add_parts_kernel launch");
}

// What both directions check of a matrix.
rl_status check(const std::string& f, const char* name, const void* p, rl_dtype t, int64_t ld, int64_t D, bool required) {
  if (t != RL_BF16 && t != RL_F32) return set_error(RL_ERR_INVALID_ARG, f + name + ": bad dtype");
  if (required && !p) return set_error(RL_ERR_INVALID_ARG, f + name + " is NULL");
  if (ld < D) return set_error(RL_ERR_INVALID_ARG, f + name + ": a leading dimension is below D");
  if (!element_aligned(p, t)) return set_error(RL_ERR_ALIGNMENT, f + name + " is not aligned to its elements");
  return RL_OK;
}

rl_status check_sizes(const std::string& f, int64_t rows, int64_t D) {
  if (rows < 0 || D < 1) return set_error(RL_ERR_INVALID_ARG, f + "bad size");
  if (D > kMaxD || rows > (int64_t(1) << 40) / D) return set_error(RL_ERR_UNSUPPORTED, f + "at most 2^20 columns and 2^40 elements");
  return RL_OK;
}

}  // namespace norm
}  // namespace rl

extern "C" {

rl_status rl_layer_norm_fwd(const void* x, rl_dtype x_dtype, int64_t rows, int64_t D, int64_t ld_x, const void* weight,
                            const void* bias, rl_dtype w_dtype, float eps, void* y, rl_dtype y_dtype, int64_t ld_y,
                            float* mean, float* rstd, rl_stream_t stream) {
  using namespace rl;
  clear_error();
  const std::string f = "rl_layer_norm_fwd: ";
  rl_status st = norm::check_sizes(f, rows, D);
  if (st == RL_OK) st = norm::check(f, "x", x, x_dtype, ld_x, D, rows > 0);
  if (st == RL_OK) st = norm::check(f, "y", y, y_dtype, ld_y, D, rows > 0);
  if (st == RL_OK) st = norm::check(f, "weight", weight, w_dtype, D, D, false);
  if (st == RL_OK) st = norm::check(f, "bias", bias, w_dtype, D, D, false);
  if (st != RL_OK) return st;
  if (!(eps >= 0.f) || !std::isfinite(eps)) return set_error(RL_ERR_INVALID_ARG, f + "eps must be finite and not negative");
  if (rows == 0) return RL_OK;
  if (!mean || !rstd) return set_error(RL_ERR_INVALID_ARG, f + "mean or rstd is NULL");
  if (!norm::element_aligned(mean, RL_F32) || !norm::element_aligned(rstd, RL_F32))
    return set_error(RL_ERR_ALIGNMENT, f + "mean or rstd is not aligned to its elements");
  if (x == y && (x_dtype != y_dtype || ld_x != ld_y))
    return set_error(RL_ERR_INVALID_ARG, f + "y may be x only with its type and leading dimension");
  norm::FwdArgs a = {};
  a.x = x;
  a.y = y;
  a.rows = rows;
  a.D = D;
  a.ld_x = ld_x;
  a.ld_y = ld_y;
  a.w = {weight, w_dtype == RL_BF16, 1.f};
  a.b = {bias, w_dtype == RL_BF16, 0.f};
  a.eps = eps;
  a.mean = mean;
  a.rstd = rstd;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (x_dtype == RL_BF16) return y_dtype == RL_BF16 ? norm::fwd<uint16_t, uint16_t>(a, s) : norm::fwd<uint16_t, float>(a, s);
  return y_dtype == RL_BF16 ? norm::fwd<float, uint16_t>(a, s) : norm::fwd<float, float>(a, s);
}

size_t rl_layer_norm_workspace_size(int64_t rows, int64_t D) {
  rl::clear_error();
  if (rl::norm::check_sizes("rl_layer_norm_workspace_size: ", rows, D) != RL_OK) return 0;
  return rl::kWsHeader + size_t(2) * rl::norm::parts_of(rows, D) * D * sizeof(float);
}

rl_status rl_layer_norm_bwd(const void* d_y, rl_dtype dy_dtype, int64_t ld_dy, const void* x, rl_dtype x_dtype, int64_t ld_x,
                            int64_t rows, int64_t D, const void* weight, rl_dtype w_dtype, const float* mean,
                            const float* rstd, const uint8_t* mask, void* d_x, int64_t ld_dx, float* d_weight,
                            float* d_bias, void* ws, size_t ws_bytes, rl_stream_t stream) {
  using namespace rl;
  clear_error();
  const std::string f = "rl_layer_norm_bwd: ";
  rl_status st = norm::check_sizes(f, rows, D);
  if (st == RL_OK) st = norm::check(f, "d_y", d_y, dy_dtype, ld_dy, D, rows > 0);
  if (st == RL_OK) st = norm::check(f, "x", x, x_dtype, ld_x, D, rows > 0);
  if (st == RL_OK) st = norm::check(f, "d_x", d_x, x_dtype, ld_dx, D, rows > 0);
  if (st == RL_OK) st = norm::check(f, "weight", weight, w_dtype, D, D, false);
  if (st != RL_OK) return st;
  if (rows == 0) return RL_OK;
  if (!mean || !rstd || !ws) return set_error(RL_ERR_INVALID_ARG, f + "a required pointer is NULL");
  if ((d_x == d_y && (x_dtype != dy_dtype || ld_dx != ld_dy)) || (d_x == x && ld_dx != ld_x))
    return set_error(RL_ERR_INVALID_ARG, f + "d_x may be d_y or x only with its type and leading dimension");
  if (!aligned16(ws)) return set_error(RL_ERR_ALIGNMENT, f + "ws must be 16-byte aligned");
  for (const float* v : {mean, rstd, static_cast<const float*>(d_weight), static_cast<const float*>(d_bias)})
    if (!norm::element_aligned(v, RL_F32)) return set_error(RL_ERR_ALIGNMENT, f + "a vector is not aligned to its elements");
  if (ws_bytes < rl_layer_norm_workspace_size(rows, D))
    return set_error(RL_ERR_WORKSPACE_TOO_SMALL, f + "ws_bytes below rl_layer_norm_workspace_size(rows, D)");
  norm::BwdArgs a = {};
  a.dy = d_y;
  a.x = x;
  a.dx = d_x;
  a.rows = rows;
  a.D = D;
  a.ld_dy = ld_dy;
  a.ld_x = ld_x;
  a.ld_dx = ld_dx;
  a.w = {weight, w_dtype == RL_BF16, 1.f};
  a.mean = mean;
  a.rstd = rstd;
  a.mask = mask;
  float* parts = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + kWsHeader);
  a.part_w = d_weight ? parts : nullptr;
  a.part_b = d_bias ? parts + norm::parts_of(rows, D) * D : nullptr;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  int32_t* status = static_cast<int32_t*>(ws);
  if (x_dtype == RL_BF16)
    return dy_dtype == RL_BF16 ? norm::bwd<uint16_t, uint16_t>(a, d_weight, d_bias, status, s)
                               : norm::bwd<uint16_t, float>(a, d_weight, d_bias, status, s);
  return dy_dtype == RL_BF16 ? norm::bwd<float, uint16_t>(a, d_weight, d_bias, status, s)
                             : norm::bwd<float, float>(a, d_weight, d_bias, status, s);
}

}  // extern "C"
