// Layer norm of rows, forward and backward, with the reductions of the weight's and the bias' gradients.
//
//   h = (x - mean) rstd,   y = h w + b,   rstd = 1 / sqrt(mean of (x - mean)^2 + eps)
//   g = dy w,   dx = rstd (g - mean of g - h (mean of g h)),   dw += sum over rows dy h,   db += sum over rows dy
//
// The simple form: a CTA per row that reads it once for each of the sums, and for the columns' sums threads that go
// down a part of the rows.
#include <algorithm>
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

// Eight elements from or to memory aligned for them (two blocks of four floats).
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
  uint4 q;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(p));
  v[0] = bf16_lo(q.x), v[1] = bf16_hi(q.x), v[2] = bf16_lo(q.y), v[3] = bf16_hi(q.y);
  v[4] = bf16_lo(q.z), v[5] = bf16_hi(q.z), v[6] = bf16_lo(q.w), v[7] = bf16_hi(q.w);
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  asm volatile("ld.global.L1::no_allocate.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "l"(p));
  asm volatile("ld.global.L1::no_allocate.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "l"(p + 4));
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  __stcs(reinterpret_cast<uint4*>(p),
         make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])));
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
  __stcs(reinterpret_cast<float4*>(p + 4), make_float4(v[4], v[5], v[6], v[7]));
}
// Eight parameters (L1 keeps them for the next rows).
__device__ __forceinline__ void load8(const Vec& w, int64_t c, float (&v)[8]) {
  if (!w.at) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = w.none;
  } else if (w.bf16) {
    const uint4 q = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(w.at) + c));
    v[0] = bf16_lo(q.x), v[1] = bf16_hi(q.x), v[2] = bf16_lo(q.y), v[3] = bf16_hi(q.y);
    v[4] = bf16_lo(q.z), v[5] = bf16_hi(q.z), v[6] = bf16_lo(q.w), v[7] = bf16_hi(q.w);
  } else {
    const float4 a = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(w.at) + c));
    const float4 b = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(w.at) + c + 4));
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
}

constexpr int kMostWarps = 16;

// The sum over a row's W warps, in every thread of them; `red` has a word per warp and is free again after the next sum.
__device__ __forceinline__ float row_sum(float v, int W, int w, float* red) {
  v = warp_sum(v);
  if (W == 1) return v;
  if ((threadIdx.x & 31) == 0) red[w] = v;
  __syncthreads();
  float s = 0.f;
  for (int i = 0; i < W; ++i) s += red[i];
  return s;
}

// A row on W warps (blockDim = 32 W, rows per CTA), NV * 8 elements a thread, held in registers between the two sums and
// the result: x is read once. WHOLE: rows in 16-byte blocks, D a multiple of 8; else an element at a time.
template <typename TX, typename TY, int NV, bool WHOLE>
__global__ void __launch_bounds__(kMostWarps * 32) fwd_kernel(const FwdArgs p) {
  __shared__ float red[2][kMostWarps];
  const int W = blockDim.x / 32, n = blockDim.x, t = threadIdx.x, w = t / 32;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * blockDim.y + threadIdx.y;
  if (W == 1 && r >= p.rows) return;  // several rows a CTA: no barriers
  const TX* x = static_cast<const TX*>(p.x) + r * p.ld_x;
  TY* y = static_cast<TY*>(p.y) + r * p.ld_y;
  const int D = static_cast<int>(p.D);
  float v[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if (WHOLE) {
      const int c = (j * n + t) * 8;
      if (c < D) load8(x + c, v[j]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = (j * 8 + e) * n + t;
        if (c < D) v[j][e] = Io<TX>::get(__ldcs(x + c));
      }
    }
  }
  auto each = [&](auto f) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (WHOLE) {
        if ((j * n + t) * 8 < D) {
#pragma unroll
          for (int e = 0; e < 8; ++e) f(v[j][e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if ((j * 8 + e) * n + t < D) f(v[j][e]);
      }
    }
  };
  float s = 0.f;
  each([&](float a) { s += a; });
  const float mean = row_sum(s, W, w, red[0]) / static_cast<float>(D);
  float q = 0.f;
  each([&](float& a) {
    a -= mean;
    q = fmaf(a, a, q);
  });
  const float rstd = 1.f / sqrtf(row_sum(q, W, w, red[1]) / static_cast<float>(D) + p.eps);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if (WHOLE) {
      const int c = (j * n + t) * 8;
      if (c >= D) continue;
      float g[8], b[8];
      load8(p.w, c, g);
      load8(p.b, c, b);
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = fmaf(v[j][e] * rstd, g[e], b[e]);
      store8(y + c, g);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = (j * 8 + e) * n + t;
        if (c < D) y[c] = Io<TY>::put(fmaf(v[j][e] * rstd, p.w[c], p.b[c]));
      }
    }
  }
  if (t == 0) {
    p.mean[r] = mean;
    p.rstd[r] = rstd;
  }
}

// ---------------------------------------------------------------- backward, rows through shared memory

constexpr int kBwdStages = 8;
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

// Persistent CTAs of W warps that share a row, 4 NG columns a thread; the rows' x and dy come by bulk copies into a ring
// of stages. A thread keeps the same columns for all rows and with them the columns' sums in registers: both matrices are
// read once. WHOLE: rows in 16-byte blocks, D a multiple of 4, a thread's columns in groups of four; else one apart.
template <typename TX, typename TD, int NG, bool WHOLE>
__global__ void __launch_bounds__(kMostWarps * 32) bwd_kernel(const BwdArgs p, const Stages st, int32_t* status) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(8) uint64_t full[kBwdStages];
  __shared__ float2 red[2][kMostWarps];
  const int W = blockDim.x / 32, n = blockDim.x, t = threadIdx.x, warp = t / 32, lane = t & 31;
  const int D = static_cast<int>(p.D);
  const float inv = 1.f / static_cast<float>(D);
  const int64_t G = gridDim.x, b0 = blockIdx.x, mine = (p.rows - b0 + G - 1) / G;  // rows b0 + i G
  if (t < st.n) mbar_init(&full[t], 1);
  if (t == 0) fence_mbar_init();
  if (t < st.n) fence_proxy_async_smem();
  __syncthreads();
  auto column = [&](int j, int e) { return WHOLE ? (j * n + t) * 4 + e : (j * 4 + e) * n + t; };
  auto live_rows = [&](int64_t base) {  // the batch of rows base .. base + 31 of the CTA's that have a gradient
    const int64_t i = base + lane;
    return __ballot_sync(0xffffffffu, i < mine && (!p.mask || p.mask[b0 + i * G] != 0));
  };

  // the first warp fetches ahead: the rows that have a gradient, in order
  int64_t ahead_base = 0;
  uint32_t ahead = warp == 0 ? live_rows(0) : 0u;
  auto fetch_next = [&](int stage) {
    while (ahead == 0) {
      if (ahead_base + kRowInfo >= mine) return false;
      ahead_base += kRowInfo;
      ahead = live_rows(ahead_base);
    }
    const int64_t r = b0 + (ahead_base + __ffs(ahead) - 1) * G;
    ahead &= ahead - 1;
    if (lane == 0) {
      const bool first = r == 0, last = r == p.rows - 1;
      const Span sx = span(static_cast<const TX*>(p.x) + r * p.ld_x, D * sizeof(TX), first, last);
      const Span sd = span(static_cast<const TD*>(p.dy) + r * p.ld_dy, D * sizeof(TD), first, last);
      const uint32_t nx = static_cast<uint32_t>(sx.to - sx.from), nd = static_cast<uint32_t>(sd.to - sd.from);
      uint8_t* to = smem + static_cast<size_t>(stage) * st.bytes;
      mbar_arrive_expect_tx(&full[stage], nx + nd);
      if (nx) bulk_g2s(to + (sx.from - sx.at), reinterpret_cast<const void*>(sx.from), nx, &full[stage]);
      if (nd) bulk_g2s(to + st.x_bytes + (sd.from - sd.at), reinterpret_cast<const void*>(sd.from), nd, &full[stage]);
    }
    __syncwarp();
    return true;
  };
  if (warp == 0)
    for (int i = 0; i < st.n && fetch_next(i); ++i) {}

  float wt[NG][4], dw[NG][4], db[NG][4];
#pragma unroll
  for (int j = 0; j < NG; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = column(j, e);
      wt[j][e] = c < D ? p.w[c] : 0.f;
      dw[j][e] = db[j][e] = 0.f;
    }

  int stage = 0;
  uint32_t parity = 0, odd = 0;
  bool in_time = true;
  for (int64_t base = 0; base < mine; base += kRowInfo) {
    const uint32_t live = live_rows(base);
    float mean_l = 0.f, rstd_l = 0.f;
    if (live >> lane & 1) {
      mean_l = p.mean[b0 + (base + lane) * G];
      rstd_l = p.rstd[b0 + (base + lane) * G];
    }
    const int here = static_cast<int>(min(static_cast<int64_t>(kRowInfo), mine - base));
    for (int i = 0; i < here; ++i) {
      const int64_t r = b0 + (base + i) * G;
      TX* dx = static_cast<TX*>(p.dx) + r * p.ld_dx;
      float out[NG][4];
      if (live >> i & 1) {
        const float mean = __shfl_sync(0xffffffffu, mean_l, i), rstd = __shfl_sync(0xffffffffu, rstd_l, i);
        // a wait that ran out is reported and not tried again
        in_time = in_time && mbar_wait_bounded(&full[stage], parity);
        const uint8_t* at = smem + static_cast<size_t>(stage) * st.bytes;
        const TX* x = static_cast<const TX*>(p.x) + r * p.ld_x;
        const TD* dy = static_cast<const TD*>(p.dy) + r * p.ld_dy;
        float h[NG][4], g[NG][4], s = 0.f, q = 0.f;
        const bool edge = r == 0 || r == p.rows - 1;
        const Span sx = span(x, D * sizeof(TX), r == 0, r == p.rows - 1), sd = span(dy, D * sizeof(TD), r == 0, r == p.rows - 1);
        const TX* xs = reinterpret_cast<const TX*>(at + (reinterpret_cast<uintptr_t>(x) - sx.at));
        const TD* ds = reinterpret_cast<const TD*>(at + st.x_bytes + (reinterpret_cast<uintptr_t>(dy) - sd.at));
        auto in = [](const void* a, const Span& v) {
          return reinterpret_cast<uintptr_t>(a) >= v.from && reinterpret_cast<uintptr_t>(a) < v.to;
        };
#pragma unroll
        for (int j = 0; j < NG; ++j) {
          float xv[4], dv[4];
          if (WHOLE) {
            const int c = (j * n + t) * 4;
            if (c >= D) {
#pragma unroll
              for (int e = 0; e < 4; ++e) h[j][e] = g[j][e] = 0.f;
              continue;
            }
            if (sizeof(TX) == 2) {
              const uint2 v = *reinterpret_cast<const uint2*>(xs + c);
              xv[0] = bf16_lo(v.x), xv[1] = bf16_hi(v.x), xv[2] = bf16_lo(v.y), xv[3] = bf16_hi(v.y);
            } else {
              const float4 v = *reinterpret_cast<const float4*>(xs + c);
              xv[0] = v.x, xv[1] = v.y, xv[2] = v.z, xv[3] = v.w;
            }
            if (sizeof(TD) == 2) {
              const uint2 v = *reinterpret_cast<const uint2*>(ds + c);
              dv[0] = bf16_lo(v.x), dv[1] = bf16_hi(v.x), dv[2] = bf16_lo(v.y), dv[3] = bf16_hi(v.y);
            } else {
              const float4 v = *reinterpret_cast<const float4*>(ds + c);
              dv[0] = v.x, dv[1] = v.y, dv[2] = v.z, dv[3] = v.w;
            }
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int c = column(j, e);
              xv[e] = mean;
              dv[e] = 0.f;
              if (c >= D) continue;
              xv[e] = Io<TX>::get(!edge || in(x + c, sx) ? xs[c] : x[c]);
              dv[e] = Io<TD>::get(!edge || in(dy + c, sd) ? ds[c] : dy[c]);
            }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            h[j][e] = (xv[e] - mean) * rstd;
            g[j][e] = dv[e] * wt[j][e];
            s += g[j][e];
            q = fmaf(g[j][e], h[j][e], q);
            dw[j][e] = fmaf(dv[e], h[j][e], dw[j][e]);
            db[j][e] += dv[e];
          }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          s += __shfl_xor_sync(0xffffffffu, s, o);
          q += __shfl_xor_sync(0xffffffffu, q, o);
        }
        if (W > 1 && lane == 0) red[odd][warp] = make_float2(s, q);
        // everyone has read the stage, and the sums are there
        if (W > 1) __syncthreads();
        else __syncwarp();
        if (warp == 0) fetch_next(stage);
        if (W > 1) {
          s = q = 0.f;
          for (int w = 0; w < W; ++w) {
            const float2 v = red[odd][w];
            s += v.x;
            q += v.y;
          }
          odd ^= 1;
        }
        s *= inv;
        q *= inv;
        if (++stage == st.n) {
          stage = 0;
          parity ^= 1;
        }
#pragma unroll
        for (int j = 0; j < NG; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) out[j][e] = rstd * (g[j][e] - s - h[j][e] * q);
      } else {
#pragma unroll
        for (int j = 0; j < NG; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) out[j][e] = 0.f;
      }
#pragma unroll
      for (int j = 0; j < NG; ++j) {
        if (WHOLE) {
          const int c = (j * n + t) * 4;
          if (c >= D) continue;
          if (sizeof(TX) == 2)
            __stcs(reinterpret_cast<uint2*>(dx + c), make_uint2(pack_bf16x2(out[j][0], out[j][1]), pack_bf16x2(out[j][2], out[j][3])));
          else
            __stcs(reinterpret_cast<float4*>(dx + c), make_float4(out[j][0], out[j][1], out[j][2], out[j][3]));
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (column(j, e) < D) dx[column(j, e)] = Io<TX>::put(out[j][e]);
        }
      }
    }
  }
  if (!in_time && lane == 0) flag_status(status, RL_DEV_TIMEOUT);
  const int64_t part = b0 * p.D;
#pragma unroll
  for (int j = 0; j < NG; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = column(j, e);
      if (c >= D) continue;
      if (p.part_w) p.part_w[part + c] = dw[j][e];
      if (p.part_b) p.part_b[part + c] = db[j][e];
    }
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

// Columns of a warp, and warps of a row, in the backward kernel; 0: a row has too many columns for it.
inline int bwd_groups(int64_t D) { return D <= 256 ? 2 : 4; }
inline int bwd_warps(int64_t D) {
  const int64_t per = 128 * bwd_groups(D), W = (D + per - 1) / per;
  return W <= kMostWarps ? static_cast<int>(W) : 0;
}
// CTAs of it on an SM: 16 warps at up to 128 registers a thread.
inline int bwd_ctas(int W) { return 16 / W; }

// Parts of the columns' sums.
inline int parts_of(int64_t rows, int64_t D) {
  const int W = bwd_warps(D);
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(rows, W ? bwd_ctas(W) * kSMs : 2 * kSMs)));
}

inline bool element_aligned(const void* p, rl_dtype t) {
  return reinterpret_cast<uintptr_t>(p) % (t == RL_BF16 ? 2 : 4) == 0;
}

inline bool whole_blocks(const void* p, int64_t ld, size_t es) { return aligned16(p) && ld * es % 16 == 0; }

template <typename TX, typename TY, int NV>
void launch_fwd(const FwdArgs& a, int W, bool whole, cudaStream_t s) {
  const int per = W == 1 ? 4 : 1;  // rows a CTA
  const dim3 grid(static_cast<unsigned>((a.rows + per - 1) / per)), block(32 * W, per);
  if (whole) fwd_kernel<TX, TY, NV, true><<<grid, block, 0, s>>>(a);
  else fwd_kernel<TX, TY, NV < 4 ? NV : 2, false><<<grid, block, 0, s>>>(a);
}

template <typename TX, typename TY>
rl_status fwd(const FwdArgs& a, cudaStream_t s) {
  const bool whole = a.D % 8 == 0 && whole_blocks(a.x, a.ld_x, sizeof(TX)) && whole_blocks(a.y, a.ld_y, sizeof(TY)) &&
                     aligned16(a.w.at) && aligned16(a.b.at);
  auto warps = [&](int nv) { return static_cast<int>((a.D + 256 * nv - 1) / (256 * nv)); };
  const int most = whole ? 4 : 2;
  if (a.rows < (int64_t(1) << 31) && warps(most) <= kMostWarps) {
    // few rows: as many threads on each as have a block of it; else up to four blocks a thread
    if (warps(1) == 1 || (a.rows * warps(1) <= 16 * kSMs && warps(1) <= kMostWarps)) launch_fwd<TX, TY, 1>(a, warps(1), whole, s);
    else if (most == 2 || warps(2) == 1) launch_fwd<TX, TY, 2>(a, warps(2), whole, s);
    else launch_fwd<TX, TY, 4>(a, warps(4), whole, s);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? RL_OK : cuda_error(e, "fwd_kernel launch");
  }
  loop_fwd_kernel<TX, TY><<<static_cast<unsigned>(std::min<int64_t>(a.rows, 4 * kSMs)), kLoopThreads, 0, s>>>(a);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? RL_OK : cuda_error(e, "loop_fwd_kernel launch");
}

constexpr int64_t kStageRoom = 216 * 1024;  // of an SM's shared memory

template <typename TX, typename TD, int NG, bool WHOLE>
rl_status launch_bwd(const BwdArgs& a, int W, int32_t* status, cudaStream_t s) {
  Stages st;
  st.x_bytes = static_cast<int32_t>((a.D * sizeof(TX) + 15) / 16 * 16 + (WHOLE ? 0 : 16));
  st.bytes = st.x_bytes + static_cast<int32_t>((a.D * sizeof(TD) + 15) / 16 * 16 + (WHOLE ? 0 : 16));
  st.n = static_cast<int32_t>(std::min<int64_t>(kBwdStages, (kStageRoom / bwd_ctas(W) - 2048) / st.bytes));
  auto kern = bwd_kernel<TX, TD, NG, WHOLE>;
  // set on every call: the attribute is a device's, and cheap
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kStageRoom));
  if (e != cudaSuccess) return cuda_error(e, "cudaFuncSetAttribute(bwd_kernel)");
  kern<<<a.parts, 32 * W, static_cast<size_t>(st.n) * st.bytes, s>>>(a, st, status);
  return RL_OK;
}

template <typename TX, typename TD>
rl_status bwd(BwdArgs& a, float* d_weight, float* d_bias, int32_t* status, cudaStream_t s) {
  a.parts = parts_of(a.rows, a.D);
  cudaError_t e = cudaSuccess;
  if (const int W = bwd_warps(a.D)) {
    const bool whole = a.D * sizeof(TX) % 16 == 0 && a.D * sizeof(TD) % 16 == 0 && whole_blocks(a.x, a.ld_x, sizeof(TX)) &&
                       whole_blocks(a.dy, a.ld_dy, sizeof(TD)) && whole_blocks(a.dx, a.ld_dx, sizeof(TX));
    rl_status r;
    if (bwd_groups(a.D) == 2) r = whole ? launch_bwd<TX, TD, 2, true>(a, W, status, s) : launch_bwd<TX, TD, 2, false>(a, W, status, s);
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
  add_parts_kernel<<<dim3(static_cast<unsigned>((a.D + 31) / 32), 2), 32 * kPartLanes, 0, s>>>(a.part_w, a.part_b, a.parts, a.D,
                                                                                              d_weight, d_bias);
  e = cudaGetLastError();
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
