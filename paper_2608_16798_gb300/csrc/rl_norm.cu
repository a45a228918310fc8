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

// d_weight, d_bias += the parts' sums, in a fixed order.
__global__ void __launch_bounds__(512) add_parts_kernel(const float* part_w, const float* part_b, int32_t parts, int64_t D,
                                                        float* d_weight, float* d_bias) {
  __shared__ float sum[16][33];
  const float* part = blockIdx.y == 0 ? part_w : part_b;
  float* out = blockIdx.y == 0 ? d_weight : d_bias;
  if (!out) return;
  const int lane = threadIdx.x & 31, row = threadIdx.x / 32;
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + lane;
  float s = 0.f;
  if (c < D)
    for (int i = row; i < parts; i += 16) s += part[i * D + c];
  sum[row][lane] = s;
  __syncthreads();
  if (row != 0 || c >= D) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) s += sum[i][lane];
  out[c] += s;
}

// ---------------------------------------------------------------- host

constexpr int kSMs = 152;
constexpr int64_t kMaxD = 1 << 20;

inline int parts_of(int64_t rows, int64_t D) {
  (void)D;
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(rows, 2 * kSMs)));
}

inline bool element_aligned(const void* p, rl_dtype t) {
  return reinterpret_cast<uintptr_t>(p) % (t == RL_BF16 ? 2 : 4) == 0;
}

template <typename TX, typename TY>
rl_status fwd(const FwdArgs& a, cudaStream_t s) {
  loop_fwd_kernel<TX, TY><<<static_cast<unsigned>(std::min<int64_t>(a.rows, 4 * kSMs)), kLoopThreads, 0, s>>>(a);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? RL_OK : cuda_error(e, "loop_fwd_kernel launch");
}

template <typename TX, typename TD>
rl_status bwd(BwdArgs& a, float* d_weight, float* d_bias, cudaStream_t s) {
  a.parts = parts_of(a.rows, a.D);
  // the columns first: dx may take the place of dy or x
  cudaError_t e = cudaSuccess;
  if (d_weight || d_bias) {
    columns_kernel<TX, TD><<<dim3(static_cast<unsigned>((a.D + 255) / 256), a.parts), 256, 0, s>>>(a);
    e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_error(e, "columns_kernel launch");
  }
  loop_bwd_kernel<TX, TD><<<static_cast<unsigned>(std::min<int64_t>(a.rows, 4 * kSMs)), kLoopThreads, 0, s>>>(a);
  e = cudaGetLastError();
  if (e != cudaSuccess) return cuda_error(e, "loop_bwd_kernel launch");
  if (!d_weight && !d_bias) return RL_OK;
  add_parts_kernel<<<dim3(static_cast<unsigned>((a.D + 31) / 32), 2), 512, 0, s>>>(a.part_w, a.part_b, a.parts, a.D, d_weight,
                                                                                  d_bias);
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
  if (x_dtype == RL_BF16)
    return dy_dtype == RL_BF16 ? norm::bwd<uint16_t, uint16_t>(a, d_weight, d_bias, s)
                               : norm::bwd<uint16_t, float>(a, d_weight, d_bias, s);
  return dy_dtype == RL_BF16 ? norm::bwd<float, uint16_t>(a, d_weight, d_bias, s)
                             : norm::bwd<float, float>(a, d_weight, d_bias, s);
}

}  // extern "C"
