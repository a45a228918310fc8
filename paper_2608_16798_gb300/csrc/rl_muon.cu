// The orthogonalised update: momentum, Newton-Schulz products on the tensor cores (tcgen05), and
// the step on the weights.
//
//   buf = mu buf + g,  u = g + mu buf (Nesterov) or buf (or g without momentum)
//   X = u / (|u|_F + eps)          [s x l], the shorter side of the matrix first
//   per step:  A = X X^T,  B = b A + c A^2,  X <- a X + B X
//
// which sends every singular value x of X through a x + b x^3 + c x^5, towards 1.
//
// Precision. The products read fp16 operands (11 significant bits; all magnitudes are known:
// singular values stay below 1.25, so X, A and B are scaled by powers of two into fp16's range) and
// accumulate in fp32. What a rounding of these operands would put into the result is kept out of it
// in two ways. X itself is held in fp32 and enters a X unrounded: early steps only multiply small
// singular values by a, and an fp16 X there would drown them in the rounding of the large ones
// (simulated on a rank-16 signal over 1% noise: 2e-2 of the result against 3e-4). And the diagonals
// of A and B, an order larger than the rest once the singular values are near 1, are held in fp32
// and taken out of the products:
//   A = D + Ao:  (A^2)_ij = (Ao Ao)_ij + (d_i + d_j) Ao_ij, i != j;  (A^2)_ii = d_i^2 + (Ao Ao)_ii
//   B = E + Bo:  X <- (a + e_i) X_i + Bo X   in the last two steps
//                X <- a X_i + (e_i X'_i + Bo X')  before them, X' the operand's fp16 copy of X
// In the second form B as a whole multiplies one and the same X'. With X' = X + r it adds B r, which lies where B,
// and so the singular values that are already large, lie. The first form adds Bo r = B r - E r, half of it or less
// once the values are near 1, but E r lies in all directions, and what lies where X is small every further step
// multiplies by a: on a single direction 2e-2 of the result at 16 rows, 5e-1 after eight steps. Emulated over random,
// decaying, low-rank and rank-one matrices: at most 4e-3 of the result in 2-norm after up to eight steps (fewer
// than eight rows: 7e-3), 5e-5 to 1.5e-3 mostly; the result's rounding to bf16 costs 1.7e-3. Beyond eight steps the
// operands' other roundings show: directions that the matrix lacks grow by a per step from 1e-5. What the rounding of
// the old X costs: 0 to 0.4% of a call, 3% of small_kernel's.
#include <cuda.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <map>
#include <mutex>
#include <utility>

#include "rl_device.cuh"
#include "rl_host.h"
#include "rl_tc.cuh"
#include "rl_tmap.h"

namespace rl {
namespace muon {

constexpr int kSMs = 152;
constexpr float kXScale = 4096.f;  // X in fp16: elements below 1.25 * 2^12
constexpr float kAScale = 4096.f;  // A off its diagonal: below 1.6 * 2^12
constexpr float kBScale = 1024.f;  // B off its diagonal: below 31 * 2^10 for coefficients up to 8

__host__ __device__ inline int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// ---------------------------------------------------------------- layouts
//
// X (fp32) lies in blocks of 32 x 32: block (R, C) of a matrix at (R * l32 + C) * 1024, and in a
// block element (r, c) at (c / 4) * 128 + r * 4 + c % 4, so that a warp whose lanes hold one row each
// moves 512 contiguous bytes per instruction. It is held times 2^12, as its fp16 copy is.
//
// The fp16 operands are row-major, as TMA reads them. Of the symmetric matrices A and B only the 256 x
// 256 tiles on and above the diagonal are formed and stored: where a product wants a block from below
// it, the block's mirror image is loaded and the MMA told that the operand lies the other way round
// (MN-major). Of A there is a second copy, in blocks for the epilogue of B, where element (r, c) lies at
// (c / 8) * 256 + r * 8 + c % 8.

struct Shape {
  int32_t batch, m, n;   // the caller's matrices
  int32_t s, l;          // the shorter and the longer side
  int32_t sp, lp;        // padded with zeros: sp to 128, lp to 64
  int32_t tall;          // m > n: X is the transpose of the caller's matrix
};

__device__ __forceinline__ float* x_block(float* x, const Shape& sh, int b, int R, int C) {
  return x + ((static_cast<int64_t>(b) * (sh.sp >> 5) + R) * (sh.lp >> 5) + C) * 1024;
}

__device__ __forceinline__ void load_block_row(const float* blk, int lane, float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float4 t = *reinterpret_cast<const float4*>(blk + j * 128 + lane * 4);
    v[4 * j] = t.x;
    v[4 * j + 1] = t.y;
    v[4 * j + 2] = t.z;
    v[4 * j + 3] = t.w;
  }
}
__device__ __forceinline__ void store_block_row(float* blk, int lane, const float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    *reinterpret_cast<float4*>(blk + j * 128 + lane * 4) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
}

__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  uint32_t r;
  memcpy(&r, &h, 4);
  return r;
}
__device__ __forceinline__ float2 unpack_half2(uint32_t w) {
  __half2 h;
  memcpy(&h, &w, 4);
  return __half22float2(h);
}

// 32 values of one row as fp16.
__device__ __forceinline__ void pack_row(const float (&v)[32], uint4 (&w)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k)
    w[k] = make_uint4(pack_half2(v[8 * k], v[8 * k + 1]), pack_half2(v[8 * k + 2], v[8 * k + 3]),
                      pack_half2(v[8 * k + 4], v[8 * k + 5]), pack_half2(v[8 * k + 6], v[8 * k + 7]));
}

// Shared memory by its 32-bit address (a pointer made of an aligned integer is a generic one to the compiler,
// and generic loads are several times slower).
__device__ __forceinline__ uint4 lds_u4(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void sts_u4(uint32_t a, uint4 v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" :: "r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ float lds_f32(uint32_t a) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void sts_f32(uint32_t a, float v) {
  asm volatile("st.shared.f32 [%0], %1;" :: "r"(a), "f"(v) : "memory");
}

__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---------------------------------------------------------------- momentum and norm

struct PrepArgs {
  Shape sh;
  const void* grad;
  int64_t ld_grad, stride_grad;
  float* momentum;       // [batch x m x n] or null
  float mu;
  int32_t nesterov;
  float eps;
  float* x;              // u, then X
  uint16_t* x16;
  double* partial;       // [batch][parts]: sums of squares
  int32_t parts;         // CTAs of a matrix
  float* inv;            // [batch]: 1 / (|u| + eps)
  uint32_t* done;        // finished CTAs (zero at launch, set back by the last)
  int32_t* status;
};

template <bool BF16>
__device__ __forceinline__ float grad_at(const PrepArgs& p, int64_t i) {
  return BF16 ? bf16_to_f32(static_cast<const uint16_t*>(p.grad)[i]) : static_cast<const float*>(p.grad)[i];
}
template <bool BF16>
__device__ __forceinline__ float4 grad_at4(const PrepArgs& p, int64_t i) {
  if (!BF16) return *reinterpret_cast<const float4*>(static_cast<const float*>(p.grad) + i);
  const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p.grad) + i);
  return make_float4(bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y));
}
__device__ __forceinline__ float momentum_of(const PrepArgs& p, float g, float& buf) {
  buf = fmaf(p.mu, buf, g);
  return p.nesterov ? fmaf(p.mu, buf, g) : buf;
}

// The sum of the squares of 32 values as a double, without fp32 overflow or underflow: the values are
// scaled by the power of two that brings the largest to [1, 2).
__device__ __forceinline__ double sum_squares(const float (&v)[32]) {
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < 32; ++j) top = max_nan(top, fabsf(v[j]));
  const uint32_t e = __float_as_uint(top) >> 23;
  if (top == 0.f) return 0.0;
  if (e == 255u) return static_cast<double>(top) * static_cast<double>(top);  // infinite or NaN
  // 2^(127 - e) and what is left of it for subnormals, in two factors that are both normal
  const int k = 127 - static_cast<int>(e == 0 ? 1 : e);
  const float f1 = __uint_as_float(static_cast<uint32_t>(127 + k / 2) << 23);
  const float f2 = __uint_as_float(static_cast<uint32_t>(127 + (k - k / 2)) << 23);
  float ss = 0.f;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const float y = v[j] * f1 * f2;
    ss = fmaf(y, y, ss);
  }
  return static_cast<double>(ss) * __hiloint2double((1023 - 2 * k) << 20, 0);
}

constexpr int kPrepWarps = 8;

// u and its sum of squares. A warp forms one 32 x 32 block of X; a CTA's warps take eight blocks that
// lie side by side in the caller's rows, and such groups in turn, so that the CTAs' last steps (a fence and
// an atomic) are few. Bound by HBM: 6 or 8 bytes read and 8 written per element with a momentum. VEC: rows begin
// at multiples of four elements, and a lane takes 4 x 4 elements twice, as vectors of the caller's rows and,
// transposed in registers if the matrix is tall, of X.
template <bool BF16, bool VEC>
__global__ void __launch_bounds__(kPrepWarps * 32, VEC ? 3 : 2) momentum_kernel(const PrepArgs p) {
  __shared__ float tile[VEC ? 1 : kPrepWarps][32][33];
  __shared__ double sums[kPrepWarps];
  __shared__ bool last;
  const Shape& sh = p.sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int nR = sh.sp >> 5, nC = sh.lp >> 5;
  pdl_launch();
  pdl_wait();
  // which block: along the caller's rows first
  const int along = sh.tall ? nR : nC, across = sh.tall ? nC : nR;
  const int groups = (along + kPrepWarps - 1) / kPrepWarps;
  const int b = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
  double mine = 0.0;
  for (int64_t rest = part; rest < static_cast<int64_t>(groups) * across; rest += p.parts) {
    const int a_blk = static_cast<int>(rest % groups) * kPrepWarps + warp, x_blk = static_cast<int>(rest / groups);
    if (a_blk >= along) continue;
    float* blk = x_block(p.x, sh, b, sh.tall ? a_blk : x_blk, sh.tall ? x_blk : a_blk);
    const int64_t g0 = b * p.stride_grad, m0 = static_cast<int64_t>(b) * sh.m * sh.n;
    float v[32];
    if (VEC) {
      // micro-tile h: rows r0 + 16 h + [0, 4), columns c + [0, 4)
      const int q = lane & 7, c = a_blk * 32 + 4 * q, r0 = x_blk * 32 + 4 * (lane >> 3);
      const bool in = c < sh.n;
      float4 g[8], buf[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int r = r0 + 16 * (k >> 2) + (k & 3);
        g[k] = in && r < sh.m ? grad_at4<BF16>(p, g0 + r * p.ld_grad + c) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      if (p.momentum) {
        float* at = p.momentum + m0 + c;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int r = r0 + 16 * (k >> 2) + (k & 3);
          buf[k] = in && r < sh.m ? *reinterpret_cast<const float4*>(at + static_cast<int64_t>(r) * sh.n)
                                  : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int r = r0 + 16 * (k >> 2) + (k & 3);
          g[k].x = momentum_of(p, g[k].x, buf[k].x);
          g[k].y = momentum_of(p, g[k].y, buf[k].y);
          g[k].z = momentum_of(p, g[k].z, buf[k].z);
          g[k].w = momentum_of(p, g[k].w, buf[k].w);
          if (in && r < sh.m) *reinterpret_cast<float4*>(at + static_cast<int64_t>(r) * sh.n) = buf[k];
        }
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        v[4 * k] = g[k].x;
        v[4 * k + 1] = g[k].y;
        v[4 * k + 2] = g[k].z;
        v[4 * k + 3] = g[k].w;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float* t = v + 16 * h;  // row-major micro-tile
        const int rl = 16 * h + 4 * (lane >> 3);
        if (sh.tall) {  // X rows 4 q + e, columns rl ..
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<float4*>(blk + (rl >> 2) * 128 + (4 * q + e) * 4) =
                make_float4(t[e], t[4 + e], t[8 + e], t[12 + e]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<float4*>(blk + q * 128 + (rl + e) * 4) =
                make_float4(t[4 * e], t[4 * e + 1], t[4 * e + 2], t[4 * e + 3]);
        }
      }
    } else {
      // lane walks its row; all loads of the block before its first store
      const int c = a_blk * 32 + lane, r0 = x_blk * 32;
      const int rows = c < sh.n ? sh.m - r0 : 0;
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = j < rows ? grad_at<BF16>(p, g0 + (r0 + j) * p.ld_grad + c) : 0.f;
      if (p.momentum) {
        float* at = p.momentum + m0 + static_cast<int64_t>(r0) * sh.n + c;
        float buf[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) buf[j] = j < rows ? at[static_cast<int64_t>(j) * sh.n] : 0.f;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          v[j] = momentum_of(p, v[j], buf[j]);
          if (j < rows) at[static_cast<int64_t>(j) * sh.n] = buf[j];
        }
      }
      if (!sh.tall) {
        float(*own)[33] = tile[VEC ? 0 : warp];
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 32; ++j) own[j][lane] = v[j];
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = own[lane][j];
      }
      store_block_row(blk, lane, v);
    }
    mine += sum_squares(v);
  }
  mine = warp_sum(mine);
  if (lane == 0) sums[warp] = mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    double s = 0.0;
    for (int w = 0; w < kPrepWarps; ++w) s += sums[w];
    p.partial[blockIdx.x] = s;
    __threadfence();
    last = atomicAdd(p.done, 1u) == gridDim.x - 1;
    if (last) __threadfence();
  }
  __syncthreads();
  if (!last) return;
  // the last CTA: one warp per matrix adds its partial sums in a fixed order
  for (int k = warp; k < sh.batch; k += kPrepWarps) {
    double s = 0.0;
    for (int i = lane; i < p.parts; i += 32) s += __ldcg(p.partial + static_cast<int64_t>(k) * p.parts + i);
    s = warp_sum(s);
    if (lane == 0) {
      if (!(s <= 1.7e308)) flag_status(p.status, RL_DEV_BAD_VALUE);
      // finite also for a zero matrix without eps, whose X is 0
      p.inv[k] = static_cast<float>(fmin(1.0 / (sqrt(s) + static_cast<double>(p.eps)), 3e38));
    }
  }
  if (threadIdx.x == 0) *p.done = 0;
}

// X in fp16 for the first product.
__global__ void __launch_bounds__(kPrepWarps * 32) normalise_kernel(const PrepArgs p) {
  const Shape& sh = p.sh;
  const int lane = threadIdx.x & 31;
  const int nR = sh.sp >> 5, nC = sh.lp >> 5;
  pdl_launch();
  pdl_wait();
  const int64_t blk = static_cast<int64_t>(blockIdx.x) * kPrepWarps + (threadIdx.x >> 5);
  const int64_t per = static_cast<int64_t>(nR) * nC;
  if (blk >= per * sh.batch) return;
  const int b = static_cast<int>(blk / per);
  const int R = static_cast<int>(blk % per) / nC, C = static_cast<int>(blk % per) % nC;
  float v[32];
  load_block_row(x_block(p.x, sh, b, R, C), lane, v);
  const float f = p.inv[b];
#pragma unroll
  for (int j = 0; j < 32; ++j) v[j] = v[j] * f * kXScale;
  uint4 w[4];
  pack_row(v, w);
  uint16_t* to = p.x16 + (static_cast<int64_t>(b) * sh.sp + R * 32 + lane) * sh.lp + C * 32;
#pragma unroll
  for (int k = 0; k < 4; ++k) *reinterpret_cast<uint4*>(to + 8 * k) = w[k];
}

// ---------------------------------------------------------------- the products

enum Mode { GRAM = 0, POLY = 1, APPLY = 2, FINAL = 3 };  // FINAL: the last step's APPLY

struct MmArgs {
  Shape sh;
  int32_t nt_m;          // tiles of the product's rows
  int32_t per;           // items of one matrix (GRAM, POLY: see symmetric_tile)
  int32_t nkb;           // 64-element blocks of the contraction
  int32_t splits;        // GRAM: parts of the contraction, each an item
  float ca, cb, cc;      // the step's coefficients
  uint16_t* a16;         // A off its diagonal, row-major
  uint16_t* a_blk;       // the same in blocks
  float* d;              // [batch x sp] the diagonal of A
  float* e;              // [batch x sp] a + the diagonal of B
  float* x;
  const float* inv;      // first step: X is still u, to be multiplied by this
  int32_t early;         // not one of the last two steps
  float* parts;          // GRAM with splits > 1: [split][tile][TILE x TILE] sums
  // the last step's outputs
  float scale;           // of the update, 2^-12 taken in
  uint16_t* update;      // bf16 [batch x m x n] or null
  float* weights;
  uint16_t* weights_bf16;
  int64_t ld_w, stride_w;
  int32_t vec;           // the caller's rows begin at multiples of four elements
  float decay, step;     // w <- decay w - step (2^12 X)
  int32_t* status;
};

constexpr int BK = 64;
constexpr uint32_t A_BYTES = 128 * BK * 2;
constexpr uint32_t STAGE_BYTES = 2 * A_BYTES;
constexpr uint32_t HALF_BYTES = 64 * BK * 2;
constexpr int NS = 5;
constexpr int kEpiWarps = 8;
constexpr int kThreads = 64 + 32 * kEpiWarps;  // warp 0 TMA, warp 1 MMA, then the epilogue
constexpr uint32_t SLAB_BYTES = 4096;          // 32 x 64 fp16 values on their way out
constexpr uint32_t EPI_BYTES = 2 * SLAB_BYTES; // per epilogue warp
constexpr size_t kSmem = NS * STAGE_BYTES + kEpiWarps * EPI_BYTES + 1024;
static_assert(kSmem <= 232448 - 1024, "shared memory of the product kernels");

// fp16 operands, fp32 accumulator, M x N; A and/or B MN-major.
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, bool a_mn, bool b_mn) {
  return (1u << 4) | (a_mn ? (1u << 15) : 0u) | (b_mn ? (1u << 16) : 0u) | (static_cast<uint32_t>(N >> 3) << 17) |
         (static_cast<uint32_t>(M >> 4) << 24);
}

// Item t of a symmetric product: the 256 x 256 tiles on and above the diagonal column by column, and
// with 128 x 128 tiles the four parts of each of them. False where the matrix has no such part.
template <int CG>
__device__ __forceinline__ bool symmetric_tile(int t, int nt, int& i, int& j) {
  const int big = CG == 2 ? t : t >> 2;
  j = static_cast<int>((sqrtf(8.f * big + 1.f) - 1.f) * 0.5f);
  while (j * (j + 1) / 2 > big) --j;
  while ((j + 1) * (j + 2) / 2 <= big) ++j;
  i = big - j * (j + 1) / 2;
  if (CG == 2) return true;
  i = 2 * i + (t & 1);
  j = 2 * j + (t >> 1 & 1);
  return i < nt && j < nt;
}

// Two-dimensional bulk store of a slab (bulk-group completion).
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, int c0, int c1, const void* src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];"
               :: "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(smem_addr(src)) : "memory");
}

// 32 values of a lane's row as fp16 into half `h` of a slab: 32 rows of 128 bytes with the 128-byte
// swizzle (16-byte chunk k of row r at chunk k ^ r % 8).
__device__ __forceinline__ void fill_slab(uint32_t slab, int h, int lane, const uint4 (&w)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) sts_u4(slab + lane * 128 + (((4 * h + k) ^ (lane & 7)) << 4), w[k]);
}

__device__ __forceinline__ uint16_t* a_block(const MmArgs& p, int b, int r0, int c0) {
  const int nb = p.sh.sp >> 5;
  return p.a_blk + ((static_cast<int64_t>(b) * nb + (r0 >> 5)) * nb + (c0 >> 5)) * 1024;
}

// The value on the diagonal of a 32 x 32 block on the diagonal (lane: row), which becomes `to`. By selects:
// as branches the 32 cases took 3,000 cycles.
__device__ __forceinline__ float take_diagonal(float (&v)[32], int lane, float to) {
  float own = 0.f;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    own = j == lane ? v[j] : own;
    v[j] = j == lane ? to : v[j];
  }
  return own;
}

// The new X (scaled) of 32 elements of a row from the old x and v = 2^10 Bo X', with e = a + the diagonal of B: see
// the precision of the early steps above.
__device__ __forceinline__ void new_x(float (&v)[32], const float (&x)[32], float e, float a, bool early) {
  if (early) {
    const float eb = e - a;
#pragma unroll
    for (int j = 0; j < 32; j += 2) {
      const float2 r = unpack_half2(pack_half2(x[j], x[j + 1]));
      v[j] = fmaf(a, x[j], fmaf(eb, r.x, v[j] * (1.f / kBScale)));
      v[j + 1] = fmaf(a, x[j + 1], fmaf(eb, r.y, v[j + 1] * (1.f / kBScale)));
    }
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = fmaf(e, x[j], v[j] * (1.f / kBScale));
  }
}

// What becomes of a 32 x 32 block (lane: row) of X X^T, scaled by 2^24: A off its diagonal, scaled, in w
// and in its block.
__device__ __forceinline__ void gram_of(const MmArgs& p, int b, int r0, int c0, int lane, float (&v)[32],
                                        uint4 (&w)[4]) {
#pragma unroll
  for (int j = 0; j < 32; ++j) v[j] *= kAScale / (kXScale * kXScale);
  if (r0 == c0)
    p.d[static_cast<int64_t>(b) * p.sh.sp + r0 + lane] = take_diagonal(v, lane, 0.f) * (1.f / kAScale);
  pack_row(v, w);
  uint16_t* blk = a_block(p, b, r0, c0) + lane * 8;
#pragma unroll
  for (int k = 0; k < 4; ++k) *reinterpret_cast<uint4*>(blk + k * 256) = w[k];
}

// B = b A + c A^2 from Ao Ao, scaled by 2^24, and the diagonal of A, di at this lane's row.
struct Poly {
  float ca, cb, cc, di, k1, k2, k3;
  __device__ __forceinline__ Poly(const MmArgs& p, float di)
      : ca(p.ca), cb(p.cb), cc(p.cc), di(di), k2(p.cc * (kBScale / kAScale)), k3(p.cc * (kBScale / (kAScale * kAScale))) {
    k1 = fmaf(k2, di, p.cb * (kBScale / kAScale));
  }
  // a + the element on the diagonal, from that of Ao Ao
  __device__ __forceinline__ float diagonal(float v) const {
    return ca + fmaf(cb, di, cc * fmaf(di, di, v * (1.f / (kAScale * kAScale))));
  }
  // Eight elements off it, scaled: B_ij = h_ij (k1 + k2 d_j) + k3 v_ij with h the fp16 values of A_ij
  __device__ __forceinline__ void off_diagonal(float* o, uint4 h, const float4* d) const {
    const uint32_t w[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const float4 dj = d[m];
      const float2 a0 = unpack_half2(w[2 * m]), a1 = unpack_half2(w[2 * m + 1]);
      o[4 * m] = fmaf(a0.x, fmaf(k2, dj.x, k1), k3 * o[4 * m]);
      o[4 * m + 1] = fmaf(a0.y, fmaf(k2, dj.y, k1), k3 * o[4 * m + 1]);
      o[4 * m + 2] = fmaf(a1.x, fmaf(k2, dj.z, k1), k3 * o[4 * m + 2]);
      o[4 * m + 3] = fmaf(a1.y, fmaf(k2, dj.w, k1), k3 * o[4 * m + 3]);
    }
  }
};

// The same of Ao Ao, scaled by 2^24: B off its diagonal, scaled. a: this lane's row of the block of A;
// di: the diagonal of A at its row.
__device__ __forceinline__ void poly_of(const MmArgs& p, int b, int r0, int c0, int lane, float (&v)[32],
                                        const uint4 (&a)[4], float di) {
  const int64_t row = static_cast<int64_t>(b) * p.sh.sp;
  const Poly poly(p, di);
  // (Ao Ao)_ii goes into e; what it leaves in its place comes to k3 0 + 0 (..) = 0, as Ao_ii is 0
  if (r0 == c0) p.e[row + r0 + lane] = poly.diagonal(take_diagonal(v, lane, 0.f));
  const float4* d = reinterpret_cast<const float4*>(p.d + row + c0);
#pragma unroll
  for (int k = 0; k < 4; ++k) poly.off_diagonal(v + 8 * k, a[k], d + 2 * k);
}

// The last step's X (lane: row) to the caller's outputs, through 32 x 33 floats of shared memory so that
// lanes walk the caller's rows: four elements each where rows begin at multiples of four (p.vec; w holds the
// block's weights then, loaded ahead), else one, eight rows at a time. The code stays short on purpose:
// unrolled over all 32 rows it outgrew, with the products', the instruction cache.
__device__ __forceinline__ void final_out(const MmArgs& p, int b, int r0, int c0, int lane, const float (&v)[32],
                                          uint32_t tile, float4 (&w)[8]) {
  const Shape& sh = p.sh;
  const int col0 = sh.tall ? r0 : c0, row0 = sh.tall ? c0 : r0;
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 32; ++j) sts_f32(tile + (lane * 33 + j) * 4, v[j]);
  __syncwarp();
  // element (row0 + j, col0 + k) is at (j, k) of the tile, of the transpose at (k, j)
  const uint32_t sr = sh.tall ? 4 : 132, sc = sh.tall ? 132 : 4;
  if (p.vec) {
    const int k = 4 * (lane & 7), col = col0 + k;
    if (col < sh.n) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int j = 4 * i + (lane >> 3), row = row0 + j;
        const uint32_t x = tile + j * sr + k * sc;
        const float4 o = make_float4(lds_f32(x), lds_f32(x + sc), lds_f32(x + 2 * sc), lds_f32(x + 3 * sc));
        if (row < sh.m) {
          if (p.update)
            *reinterpret_cast<uint2*>(p.update + (static_cast<int64_t>(b) * sh.m + row) * sh.n + col) =
                make_uint2(pack_bf16x2(o.x * p.scale, o.y * p.scale), pack_bf16x2(o.z * p.scale, o.w * p.scale));
          if (p.weights) {
            const int64_t at = b * p.stride_w + row * p.ld_w + col;
            const float4 y = make_float4(fmaf(-p.step, o.x, p.decay * w[i].x), fmaf(-p.step, o.y, p.decay * w[i].y),
                                         fmaf(-p.step, o.z, p.decay * w[i].z), fmaf(-p.step, o.w, p.decay * w[i].w));
            *reinterpret_cast<float4*>(p.weights + at) = y;
            if (p.weights_bf16)
              *reinterpret_cast<uint2*>(p.weights_bf16 + at) = make_uint2(pack_bf16x2(y.x, y.y), pack_bf16x2(y.z, y.w));
          }
        }
      }
    }
    __syncwarp();
    return;
  }
  const int col = col0 + lane, rows = col < sh.n ? sh.m - row0 : 0;
  uint16_t* up = p.update ? p.update + (static_cast<int64_t>(b) * sh.m + row0) * sh.n + col : nullptr;
  const int64_t w0 = b * p.stride_w + row0 * p.ld_w + col;
  const uint32_t from = tile + lane * sc;
#pragma unroll 1
  for (int j0 = 0; j0 < 32; j0 += 8) {
    float x[8], y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = lds_f32(from + (j0 + j) * sr);
    if (p.weights) {
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = j0 + j < rows ? p.weights[w0 + (j0 + j) * p.ld_w] : 0.f;
    }
    if (up) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j0 + j < rows) up[static_cast<int64_t>(j0 + j) * sh.n] = f32_to_bf16(x[j] * p.scale);
    }
    if (p.weights) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        y[j] = fmaf(-p.step, x[j], p.decay * y[j]);
        if (j0 + j < rows) {
          p.weights[w0 + (j0 + j) * p.ld_w] = y[j];
          if (p.weights_bf16) p.weights_bf16[w0 + (j0 + j) * p.ld_w] = f32_to_bf16(y[j]);
        }
      }
    }
  }
  __syncwarp();
}

// The weights of a block, ahead of final_out.
__device__ __forceinline__ void load_weights(const MmArgs& p, int b, int r0, int c0, int lane, float4 (&w)[8]) {
  const Shape& sh = p.sh;
  const int col = (sh.tall ? r0 : c0) + 4 * (lane & 7), row0 = (sh.tall ? c0 : r0) + (lane >> 3);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (col < sh.n && row0 + 4 * i < sh.m)
      w[i] = *reinterpret_cast<const float4*>(p.weights + b * p.stride_w + (row0 + 4 * i) * p.ld_w + col);
}

// One product, persistent: CTAs (CG = 1) or CTA pairs (CG = 2) take square tiles of 128 CG in turn.
// Per stage of 64 along the contraction a CTA holds 128 rows of the left operand and 128 of the right
// one's (of a pair's 256). Two accumulators in TMEM, so that the epilogue of one tile runs under the
// products of the next.
//
// Measured on 4,096 x 4,096 (pairs), us: A 51 (one triangle of tiles, 73 GFLOP: 1.4 PFLOP/s), B 57, the
// new X 107 (1.28 PFLOP/s; a library's fp16 product of this size, which writes fp16 and nothing else, 81: 1.70). The
// products issue at 150-157 cycles per 256 x 256 x 16; the tensor pipe is active 66-71% of the active cycles. The rest is the last turn of tiles (136
// symmetric or 256 tiles on 76 pairs) and, for X, the epilogue's 128 MB of fp32 state (11K cycles a tile; twice the
// epilogue warps gave 1,203 us against 1,185 for the whole update). Smaller matrices take 3 to 5 us more than their
// products per launch: prologue, first loads, epilogue.
template <int MODE, int CG>
__global__ void __launch_bounds__(kThreads, 1) product_kernel(const __grid_constant__ CUtensorMap tmA,
                                                              const __grid_constant__ CUtensorMap tmAt,
                                                              const __grid_constant__ CUtensorMap tmB,
                                                              const __grid_constant__ CUtensorMap tmOut,
                                                              const MmArgs p) {
  constexpr int TILE = 128 * CG;
  constexpr bool APPLIES = MODE == APPLY || MODE == FINAL;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t full[NS], empty[NS], accf[2], acce[2];
  __shared__ uint32_t tbase;
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? cluster_ctarank() : 0;
  const int unit = blockIdx.x / CG, units = gridDim.x / CG;
  const int n_tiles = p.sh.batch * p.per;
  const int n_items = n_tiles * (MODE == GRAM ? p.splits : 1);

  if (threadIdx.x == 0) {
    for (int s = 0; s < NS; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int k = 0; k < 2; ++k) {
      mbar_init(&accf[k], 1);
      mbar_init(&acce[k], kEpiWarps * CG);
    }
    fence_mbar_init();
  }
  if (warp == 1) {
    if (CG == 2) tc::tmem_alloc_pair(&tbase, 2 * TILE);
    else tc::tmem_alloc(&tbase, 2 * TILE);
  }
  tc::fence_before_sync();
  if (CG == 2) cluster_sync_all();
  else __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = tbase;
  if (warp == 0 && lane == 0) {
    const CUtensorMap* used[4] = {&tmA, &tmAt, &tmB, &tmOut};
    for (const CUtensorMap* m : used)
      asm volatile("prefetch.tensormap [%0];" :: "l"(reinterpret_cast<uint64_t>(m)) : "memory");
  }
  pdl_launch();
  pdl_wait();

  // item -> matrix, tile row and column, K blocks; false if there is no such tile
  auto decode = [&](int item, int& b, int& ti, int& tj, int& kb0, int& nkb) -> bool {
    int part = 0;
    if (MODE == GRAM && p.splits > 1) {
      part = item / n_tiles;
      item -= part * n_tiles;
    }
    b = item / p.per;
    const int t = item - b * p.per;
    kb0 = MODE == GRAM ? static_cast<int>(static_cast<int64_t>(part) * p.nkb / p.splits) : 0;
    nkb = (MODE == GRAM ? static_cast<int>(static_cast<int64_t>(part + 1) * p.nkb / p.splits) : p.nkb) - kb0;
    if (!APPLIES) return symmetric_tile<CG>(t, p.nt_m, ti, tj);
    ti = t % p.nt_m;
    tj = t / p.nt_m;
    return true;
  };
  // whether K block k0 of an operand's rows m0 .. of a symmetric matrix is stored the other way round
  auto below = [](int m0, int k0) { return (k0 >> 8) < (m0 >> 8); };

  if (warp == 0) {
    if (lane == 0) {
      // the launch before wrote the operands through the generic proxy; TMA reads them
      asm volatile("fence.proxy.async.global;" ::: "memory");
      uint32_t g = 0;
      bool ok = true;
      for (int item = unit; item < n_items && ok; item += units) {
        int b, ti, tj, kb0, nkb;
        if (!decode(item, b, ti, tj, kb0, nkb)) continue;
        const int y0 = b * p.sh.sp;  // the matrix's first row in the maps
        const int m0 = ti * TILE + static_cast<int>(rank) * 128, n0 = tj * TILE + static_cast<int>(rank) * 128;
        for (int kb = 0; kb < nkb; ++kb, ++g) {
          const int s = g % NS;
          const int k0 = (kb0 + kb) * BK;
          const uint32_t use = g / NS;
          if (use > 0 && !mbar_wait_bounded(&empty[s], (use - 1) & 1)) {
            flag_status(p.status, RL_DEV_TIMEOUT);
            ok = false;
            break;
          }
          uint8_t* st = sm + s * STAGE_BYTES;
          if (rank == 0) mbar_arrive_expect_tx(&full[s], CG * STAGE_BYTES);
          const uint32_t bar = CG == 2 ? map_to_rank(smem_addr(&full[s]), 0) : 0;
          auto load = [&](uint8_t* dst, const CUtensorMap* map, int c0, int c1) {
            if (CG == 2) tc::tma_load_2d_pair(dst, map, c0, c1, bar);
            else tc::tma_load_2d(dst, map, c0, c1, &full[s]);
          };
          if (MODE != GRAM && below(m0, k0)) {
            load(st, &tmAt, m0, y0 + k0);
            load(st + HALF_BYTES, &tmAt, m0 + 64, y0 + k0);
          } else {
            load(st, &tmA, k0, y0 + m0);
          }
          if (APPLIES || (MODE == POLY && below(n0, k0))) {
            const CUtensorMap* map = APPLIES ? &tmB : &tmAt;
            load(st + A_BYTES, map, n0, y0 + k0);
            load(st + A_BYTES + HALF_BYTES, map, n0 + 64, y0 + k0);
          } else {
            load(st + A_BYTES, &tmA, k0, y0 + n0);
          }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      const uint64_t k_major = tc::desc_kmajor_sw128(0), mn_major = tc::desc_mnmajor_sw128(0, HALF_BYTES, 1024);
      const uint32_t stage0 = smem_addr(sm) >> 4;
      uint32_t g = 0;
      bool ok = true;
      uint32_t t = 0;
      for (int item = unit; item < n_items && ok; item += units, ++t) {
        int b, ti, tj, kb0, nkb;
        if (!decode(item, b, ti, tj, kb0, nkb)) {
          --t;  // not a use of an accumulator
          continue;
        }
        const uint32_t buf = t & 1;
        if (t >= 2) {
          const bool got = CG == 2 ? mbar_wait_cluster_bounded(&acce[buf], ((t >> 1) - 1) & 1)
                                   : mbar_wait_bounded(&acce[buf], ((t >> 1) - 1) & 1);
          if (!got) {
            flag_status(p.status, RL_DEV_TIMEOUT);
            break;
          }
        }
        tc::fence_after_sync();
        const uint32_t acc = tmem + buf * TILE;
        for (int kb = 0; kb < nkb; ++kb, ++g) {
          const int s = g % NS;
          if (!mbar_wait_bounded(&full[s], (g / NS) & 1)) {
            flag_status(p.status, RL_DEV_TIMEOUT);
            ok = false;
            break;
          }
          tc::fence_after_sync();
          const int k0 = (kb0 + kb) * BK;
          const bool a_mn = MODE != GRAM && below(ti * TILE, k0);
          const bool b_mn = APPLIES || (MODE == POLY && below(tj * TILE, k0));
          const uint32_t idesc = idesc_f16(TILE, TILE, a_mn, b_mn);
          // descriptors differ in their start address only, in units of 16 bytes
          const uint64_t at = stage0 + s * (STAGE_BYTES >> 4);
          const uint64_t ad = (a_mn ? mn_major : k_major) + at, bd = (b_mn ? mn_major : k_major) + at + (A_BYTES >> 4);
          const uint32_t da = a_mn ? 128 : 2, db = b_mn ? 128 : 2;
#pragma unroll
          for (int k = 0; k < BK / 16; ++k) {
            if (CG == 2) tc::mma_bf16_pair(acc, ad + k * da, bd + k * db, idesc, (kb | k) != 0 ? 1u : 0u);
            else tc::mma_bf16(acc, ad + k * da, bd + k * db, idesc, (kb | k) != 0 ? 1u : 0u);
          }
          if (CG == 2) tc::mma_commit_pair(&empty[s], 0x3);
          else tc::mma_commit(&empty[s]);
        }
        if (!ok) break;
        if (CG == 2) tc::mma_commit_pair(&accf[buf], 0x3);
        else tc::mma_commit(&accf[buf]);
      }
    }
  } else {
    // Two warps per TMEM lane quarter, each with half of the tile's 32-column blocks. What a block needs
    // from memory is loaded one block ahead, the first before the products are done.
    constexpr int NBLK = TILE / 64;
    const int q = warp & 3, first = ((warp - 2) >> 2) * NBLK;
    uint8_t* slabs = sm + NS * STAGE_BYTES + (warp - 2) * EPI_BYTES;
    const uint32_t tile = smem_addr(slabs);
    uint32_t slab = 0;
    uint32_t t = 0;
    for (int item = unit; item < n_items; item += units) {
      int b, ti, tj, kb0, nkb;
      if (!decode(item, b, ti, tj, kb0, nkb)) continue;
      const uint32_t buf = t & 1, phase = (t >> 1) & 1;
      ++t;
      const int r0 = ti * TILE + static_cast<int>(rank) * 128 + 32 * q;
      const int cols = APPLIES ? p.sh.lp : p.sh.sp;
      // the 64-column halves past the matrix are another one's or nothing
      const int blocks = r0 < p.sh.sp ? min(NBLK, (cols - tj * TILE) / 32 - first) : 0;
      const int cb = tj * TILE + first * 32;  // the warp's first column
      const bool in_parts = MODE == GRAM && p.splits > 1;
      float x[32], f = 0.f;
      uint4 a[4];
      auto prefetch = [&](int i) {
        if (i >= blocks) return;
        if (APPLIES) load_block_row(x_block(p.x, p.sh, b, r0 >> 5, (cb >> 5) + i), lane, x);
        if (MODE == POLY) {
          const uint16_t* blk = a_block(p, b, r0, cb + 32 * i) + lane * 8;
#pragma unroll
          for (int k = 0; k < 4; ++k) a[k] = *reinterpret_cast<const uint4*>(blk + k * 256);
        }
      };
      if (r0 < p.sh.sp) {
        const int64_t row = static_cast<int64_t>(b) * p.sh.sp + r0 + lane;
        if (APPLIES) f = p.e[row];
        if (MODE == POLY) f = p.d[row];
      }
      prefetch(0);
      if (!mbar_wait_sleep_bounded(&accf[buf], phase)) {
        if (lane == 0) flag_status(p.status, RL_DEV_TIMEOUT);
        break;
      }
      tc::fence_after_sync();
      const uint32_t tq = tmem + buf * TILE + (static_cast<uint32_t>(32 * q) << 16) + first * 32;
#pragma unroll 1  // unrolled it was slower: see final_out
      for (int i = 0; i < NBLK; ++i) {
        float v[32];
        tc::tmem_ld32(tq + i * 32, v);
        if (i == NBLK - 1) {
          tc::fence_before_sync();
          __syncwarp();
          if (lane == 0) {
            if (rank != 0) mbar_arrive_remote(map_to_rank(smem_addr(&acce[buf]), 0));
            else mbar_arrive(&acce[buf]);
          }
        }
        if (i >= blocks) continue;
        const int c0 = cb + 32 * i;
        float4 wts[8];
        if (MODE == FINAL && p.vec && p.weights) load_weights(p, b, r0, c0, lane, wts);
        if (in_parts) {
          store_block_row(p.parts + static_cast<int64_t>(item) * TILE * TILE +
                              (static_cast<int64_t>((rank * 4 + q) * (TILE / 32) + first + i)) * 1024, lane, v);
          continue;
        }
        uint4 w[4];
        if (MODE == GRAM) gram_of(p, b, r0, c0, lane, v, w);
        if (MODE == POLY) poly_of(p, b, r0, c0, lane, v, a, f);
        if (APPLIES) {
          if (p.inv) {
            const float inv = p.inv[b];
#pragma unroll
            for (int j = 0; j < 32; ++j) x[j] = x[j] * inv * kXScale;
          }
          new_x(v, x, f, p.ca, MODE == APPLY && p.early);
        }
        prefetch(i + 1);
        if (MODE == FINAL) {
          final_out(p, b, r0, c0, lane, v, tile, wts);
          continue;
        }
        if (MODE == APPLY) store_block_row(x_block(p.x, p.sh, b, r0 >> 5, c0 >> 5), lane, v);
        if (MODE != GRAM) pack_row(v, w);
        uint8_t* sb = slabs + slab * SLAB_BYTES;
        if ((i & 1) == 0) {
          if (lane == 0) tc::bulk_wait_read_1();  // the slab's previous store has read it
          __syncwarp();
        }
        fill_slab(smem_addr(sb), i & 1, lane, w);
        if (i & 1) {
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            tma_store_2d(&tmOut, c0 - 32, b * p.sh.sp + r0, sb);
            bulk_commit();
          }
          slab ^= 1;
        }
      }
    }
    if (lane == 0) tc::bulk_wait_all();
  }
  tc::fence_before_sync();
  if (CG == 2) cluster_sync_all();
  else __syncthreads();
  if (warp == 1) {
    tc::fence_after_sync();
    if (CG == 2) tc::tmem_dealloc_pair(tmem, 2 * TILE);
    else tc::tmem_dealloc(tmem, 2 * TILE);
  }
}

// A from the parts of its contraction, added in order: one warp per 32 x 32 block.
template <int CG>
__global__ void __launch_bounds__(256) gram_sum_kernel(const MmArgs p) {
  constexpr int TILE = 128 * CG, NB = TILE / 32;
  const int lane = threadIdx.x & 31;
  pdl_launch();
  pdl_wait();
  const int n_tiles = p.sh.batch * p.per;
  const int64_t blk = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  if (blk >= static_cast<int64_t>(n_tiles) * NB * NB) return;
  const int tile = static_cast<int>(blk / (NB * NB)), in = static_cast<int>(blk % (NB * NB));
  const int b = tile / p.per;
  int ti, tj;
  if (!symmetric_tile<CG>(tile - b * p.per, p.nt_m, ti, tj)) return;
  const int r0 = ti * TILE + in / NB * 32, c0 = tj * TILE + in % NB * 32;
  if (r0 >= p.sh.sp || c0 >= p.sh.sp) return;
  // two parts' loads in flight
  float v[32], t[2][32];
  const float* src = p.parts + static_cast<int64_t>(tile) * TILE * TILE + static_cast<int64_t>(in) * 1024;
  auto load = [&](int k, float (&to)[32]) {
    if (k < p.splits) load_block_row(src + static_cast<int64_t>(k) * n_tiles * TILE * TILE, lane, to);
  };
  load(0, v);
  load(1, t[0]);
  for (int k = 1; k < p.splits; k += 2) {
    load(k + 1, t[1]);
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] += t[0][j];
    if (k + 1 == p.splits) break;
    load(k + 2, t[0]);
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] += t[1][j];
  }
  uint4 w[4];
  gram_of(p, b, r0, c0, lane, v, w);
  uint16_t* to = p.a16 + (static_cast<int64_t>(b) * p.sh.sp + r0 + lane) * p.sh.sp + c0;
#pragma unroll
  for (int k = 0; k < 4; ++k) *reinterpret_cast<uint4*>(to + 8 * k) = w[k];
}

// ---------------------------------------------------------------- matrices of at most 256 x 256
//
// All steps of one matrix in one CTA pair, the operands in shared memory and X (fp32) in TMEM: fifteen
// launches that wait for each other (6 us each) become fifteen rounds of products, an epilogue in registers
// and a cluster barrier. CTA r owns rows [128 r, 128 r + 128). It holds, in the layout of the 128-byte
// swizzle (64 columns a block),
//   xk  its rows of X: left and right operand of X X^T (K-major), half of the right one's rows each
//   xn  all rows of X, its half of the columns: right operand of Bo X (MN-major)
//   sy  its rows of Ao, then, in their place, of Bo: operands of Ao Ao (K-major) and Bo X
// so that the pair's MMAs find their halves; of the new X the 64-column blocks in xk are, as they lie, halves of blocks
// of xn, and go there by bulk copies to both CTAs under the next step's first product.
//
// 256 x 256, five steps: 55.6 us a call (104 by launches), nearly all of it this kernel. What bounds it is the chain of
// a step, in cycles: three products of 2,500 each, their epilogues 1,250 (A), 2,280 (B) and about 2,500 (X; before the
// last two steps about 1,000 more for the rounding of the old X, by the call's time with and without it), and 800 for the fence and the cluster barrier before each product. Stores of the new X straight to the other CTA made the
// last epilogue 4,000 and its fence 1,200 (59 us); 16 warps gave 60.

constexpr int kSmallSide = 256;
constexpr int kSmallWarps = 8;
constexpr int kSmallThreads = 32 * kSmallWarps;
constexpr int kSmallParts = kSmallWarps / 4;  // warps that share the rows of a TMEM lane quarter
constexpr uint32_t kBlk = 128 * 128;  // bytes of 128 rows of a 64-column block

struct SmallSmem {
  uint32_t xk, xn, sy, bytes;
};
__host__ __device__ constexpr SmallSmem small_smem(int lp) {
  return SmallSmem{0, static_cast<uint32_t>(lp) / 64 * kBlk, static_cast<uint32_t>(lp) / 64 * kBlk * 2,
                   static_cast<uint32_t>(lp) / 64 * kBlk * 2 +
                       (4 * kBlk > kSmallWarps * 4352 ? 4 * kBlk : kSmallWarps * 4352)};
}

// 32 fp32 columns of this warp's 32 TMEM lanes.
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const float (&v)[32]) {
  uint32_t r[32];
#pragma unroll
  for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(v[j]);
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
      :: "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
         "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
         "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
         "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
      : "memory");
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// Bulk copy of shared memory to a CTA of the cluster (addresses and barrier from map_to_rank).
__device__ __forceinline__ void bulk_s2s(uint32_t to, uint32_t from, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               :: "r"(to), "r"(from), "r"(bytes), "r"(bar) : "memory");
}

__global__ void __launch_bounds__(kSmallThreads, 1) small_kernel(const MmArgs p, int steps) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t accf, spread;
  __shared__ uint32_t tbase;
  __shared__ __align__(16) float d[kSmallSide];
  __shared__ float e[128];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int b = blockIdx.x / 2, lp = p.sh.lp, q = warp & 3, part = warp >> 2;
  const SmallSmem at = small_smem(lp);
  const int row = 32 * q + lane, grow = static_cast<int>(rank) * 128 + row;  // this lane's row: here, of the matrix
  if (threadIdx.x < kSmallSide) d[threadIdx.x] = 0.f;  // rows and columns past the matrix's last block of 64 stay so
  if (threadIdx.x < 128) e[threadIdx.x] = 0.f;
  if (threadIdx.x == 0) {
    mbar_init(&accf, 1);
    mbar_init(&spread, 1);
    fence_mbar_init();
  }
  if (warp == 0) tc::tmem_alloc_pair(&tbase, 512);
  tc::fence_before_sync();
  cluster_sync_all();
  tc::fence_after_sync();
  const uint32_t acc = tbase + (static_cast<uint32_t>(32 * q) << 16), xt = acc + 256;
  pdl_launch();
  pdl_wait();
  bool dead = false;  // a wait ran out: the rest runs through without waiting
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (!mbar_wait_bounded(bar, parity, dead ? 1000 : kWaitLimitNs)) {
      if (!dead && lane == 0) flag_status(p.status, RL_DEV_TIMEOUT);
      dead = true;
    }
  };
  // this lane's row of the 64-column block of 128 rows at `blk`, 16-byte chunk k
  auto chunk = [&](uint32_t blk, int k) -> uint32_t { return blk + row * 128 + ((k ^ (row & 7)) << 4); };
  const uint32_t own = smem_addr(sm), base = own >> 4;
  // columns [32 cb, 32 cb + 32) of this lane's row, as fp16 into a CTA's 128 rows of X, Ao or Bo
  auto put = [&](uint32_t region, int cb, const float (&v)[32]) {
    uint4 w[4];
    pack_row(v, w);
#pragma unroll
    for (int k = 0; k < 4; ++k) sts_u4(chunk(own + region + (cb >> 1) * kBlk, 4 * (cb & 1) + k), w[k]);
  };
  // this CTA's rows of X, blocks of 64 columns, to xn of the CTA that has the columns
  auto spread_x = [&] {
    mbar_arrive_expect_tx(&spread, at.sy - at.xn);
    for (int c = 0; c < lp / 64; ++c) {
      const int owner = c / (lp / 128), cn = c % (lp / 128);
      bulk_s2s(map_to_rank(own + at.xn + cn * 2 * kBlk + rank * kBlk, owner), own + at.xk + c * kBlk, kBlk,
               map_to_rank(smem_addr(&spread), owner));
    }
  };
  // X, normalised and scaled, into TMEM and the operands
  const float inv = p.inv[b];
  // 64-column blocks of Ao and Bo, and of X, that hold anything; a warp's 32-column blocks are every other one
  const int ks = (p.sh.s + 63) / 64, kx = (p.sh.l + 63) / 64;
#pragma unroll 1
  for (int cb = part; cb < lp / 32; cb += kSmallParts) {
    float v[32];
    load_block_row(x_block(p.x, p.sh, b, grow >> 5, cb), lane, v);
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = v[j] * inv * kXScale;
    tmem_st32(xt + cb * 32, v);
    put(at.xk, cb, v);
  }

  const uint64_t k_major = tc::desc_kmajor_sw128(0), mn_major = tc::desc_mnmajor_sw128(0, 2 * kBlk, 1024);
  // The products whose operands both CTAs have written by now; everyone returns when they are done.
  uint32_t rounds = 0;
  auto multiply = [&](uint32_t left, uint32_t right, int n, int k_blocks, bool right_mn, auto then) {
    asm volatile("fence.proxy.async;" ::: "memory");  // what was written for the MMAs, here and in the peer
    __syncwarp();
    tc::fence_before_sync();
    cluster_sync_all();
    tc::fence_after_sync();
    if (rank == 0 && threadIdx.x == 0) {
      const uint32_t idesc = idesc_f16(2 * 128, n, false, right_mn);
      for (int c = 0; c < k_blocks; ++c) {
        // 64 along the contraction: a block of a K-major operand, 64 rows of an MN-major one
        const uint64_t l = k_major + base + ((left + c * kBlk) >> 4);
        const uint64_t r = right_mn ? mn_major + base + ((right + c * (kBlk / 2)) >> 4)
                                    : k_major + base + ((right + c * kBlk) >> 4);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          tc::mma_bf16_pair(tbase, l + k * 2, r + k * (right_mn ? 128 : 2), idesc, (c | k) != 0 ? 1u : 0u);
      }
      tc::mma_commit_pair(&accf, 0x3);
    }
    then();
    wait(&accf, rounds++ & 1);
    tc::fence_after_sync();
  };
#pragma unroll 1
  for (int step = 0; step < steps; ++step) {
    // ---- A = X X^T: its diagonal to both CTAs' d, the rest to sy
    multiply(at.xk, at.xk, kSmallSide, kx, false, [&] {
      if (threadIdx.x == 0) spread_x();
    });
#pragma unroll 1
    for (int cb = part; cb < 2 * ks; cb += kSmallParts) {
      const int c0 = 32 * cb;
      float v[32];
      tc::tmem_ld32(acc + c0, v);
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] *= kAScale / (kXScale * kXScale);
      if (c0 == (grow & ~31)) {
        const float di = take_diagonal(v, lane, 0.f) * (1.f / kAScale);
        d[grow] = di;
        asm volatile("st.shared::cluster.f32 [%0], %1;" :: "r"(map_to_rank(smem_addr(&d[grow]), rank ^ 1)), "f"(di) : "memory");
      }
      put(at.sy, cb, v);
    }
    // ---- B = b A + c A^2: a + its diagonal to e, the rest in Ao's place
    multiply(at.sy, at.sy, kSmallSide, ks, false, [] {});
    const Poly poly(p, d[grow]);
#pragma unroll 1
    for (int cb = part; cb < 2 * ks; cb += kSmallParts) {
      const int c0 = 32 * cb;
      float v[32];
      tc::tmem_ld32(acc + c0, v);
      if (c0 == (grow & ~31)) e[row] = poly.diagonal(take_diagonal(v, lane, 0.f));
      uint32_t blk[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        blk[k] = chunk(own + at.sy + (cb >> 1) * kBlk, 4 * (cb & 1) + k);
        poly.off_diagonal(v + 8 * k, lds_u4(blk[k]), reinterpret_cast<const float4*>(d + c0 + 8 * k));
      }
      uint4 w[4];
      pack_row(v, w);
#pragma unroll
      for (int k = 0; k < 4; ++k) sts_u4(blk[k], w[k]);
    }
    // ---- X <- e X + Bo X, kept in TMEM and as operands of the next step
    wait(&spread, step & 1);  // and the peer's, behind the barrier
    multiply(at.sy, at.xn, lp, ks, true, [] {});
    const float f = e[row];
    const bool last = step == steps - 1;
#pragma unroll 1
    for (int cb = part; cb < 2 * kx; cb += kSmallParts) {
      const int c0 = 32 * cb;
      float v[32], x[32];
      tc::tmem_ld32(acc + c0, v);
      tc::tmem_ld32(xt + c0, x);
      new_x(v, x, f, p.ca, step < steps - 2);
      if (last) {
        float4 wts[8];
        const int r0 = grow & ~31;
        if (p.vec && p.weights) load_weights(p, b, r0, c0, lane, wts);
        final_out(p, b, r0, c0, lane, v, own + at.sy + warp * 4352, wts);
        continue;
      }
      tmem_st32(xt + c0, v);
      put(at.xk, cb, v);
    }
  }
  tc::fence_before_sync();
  cluster_sync_all();
  if (warp == 0) {
    tc::fence_after_sync();
    tc::tmem_dealloc_pair(tbase, 512);
  }
}

// ---------------------------------------------------------------- host

// How the products are cut: the tile (128 or, by CTA pairs, 256) of each, and the parts of the first
// one's contraction.
struct Plan {
  int cg_gram, cg_poly, cg_apply, splits;
};

// Matrices of at most 256 x 256 go to small_kernel, padded to 256 x 128 or 256 x 256.
inline bool is_small(const Shape& s) { return s.l <= kSmallSide; }

// Items of a symmetric product of one matrix (symmetric_tile).
inline int64_t symmetric_items(int64_t sp, int cg) {
  const int64_t n = round_up(sp, 256) / 256;
  return n * (n + 1) / 2 * (cg == 2 ? 1 : 4);
}

// The cheapest by what the kernels take, measured from 256 x 256 to 4,096 x 4,096, us: per wave of tiles
// 3 + 0.3 per K block with single CTAs and 4.6 + 0.45 with pairs (both are bound by what L2 delivers, a
// pair's block does four times the work), and 4 for a sum of parts. E.g. X X^T of 2,048 x 2,048: singles 16.5, pairs in
// two parts 13.7 and their sum; B X of 1,000 x 2,777: singles 18.6 (176 tiles, two waves), pairs 16.0. A charge of 5.5
// for the sum, as it was with one part's loads in flight, cuts A differently for one shape in 15; of 18 such ones 17 take
// less with 4 (whole updates: 2 x 467 x 1,217 136 for 146, 1,969 x 5,674 499 for 527, 12 x 363 x 5,303 522 for 542), one
// more (4 x 723 x 2,793 292 for 284).
Plan plan_of(int64_t batch, int64_t sp, int64_t lp) {
  Plan p = {};
  auto cost = [](int cg, int64_t items, double nkb) {
    const int64_t units = kSMs / cg, waves = (items + units - 1) / units;
    return static_cast<double>(waves) * (cg == 2 ? 4.6 + 0.45 * nkb : 3.0 + 0.3 * nkb);
  };
  double poly = 1e300, apply = 1e300, gram = 1e300;
  for (int cg = 1; cg <= 2; ++cg) {
    const int64_t T = 128 * cg, sym = batch * symmetric_items(sp, cg);
    const int64_t all = batch * ((sp + T - 1) / T) * ((lp + T - 1) / T);
    if (cost(cg, sym, sp / BK) < poly) poly = cost(cg, sym, sp / BK), p.cg_poly = cg;
    if (cost(cg, all, sp / BK) < apply) apply = cost(cg, all, sp / BK), p.cg_apply = cg;
    // parts of at least four K blocks that all run at once
    for (int64_t k = 1; k == 1 || (k * sym <= kSMs / cg && lp / BK >= 4 * k); ++k) {
      const double t = cost(cg, k * sym, static_cast<double>(lp / BK) / k) + (k > 1 ? 4.0 : 0.0);
      if (t < gram) gram = t, p.cg_gram = cg, p.splits = static_cast<int>(k);
    }
  }
  return p;
}

struct Layout {
  size_t x, x16a, x16b, a16, a_blk, b16, d, e, inv, partial, parts, bytes;
  int32_t n_parts;  // partial sums of squares per matrix: CTAs of its momentum pass
};

Shape shape_of(int32_t batch, int64_t m, int64_t n) {
  Shape s;
  s.batch = batch;
  s.m = static_cast<int32_t>(m);
  s.n = static_cast<int32_t>(n);
  s.s = std::min(s.m, s.n);
  s.l = std::max(s.m, s.n);
  s.sp = static_cast<int32_t>(round_up(s.s, 128));
  s.lp = static_cast<int32_t>(round_up(s.l, 64));
  s.tall = m > n;
  if (is_small(s)) {
    s.sp = kSmallSide;
    s.lp = static_cast<int32_t>(round_up(s.l, 128));
  }
  return s;
}

Layout layout_of(const Shape& s) {
  Layout w = {};
  size_t at = kWsHeader;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) & ~size_t(255);
    return here;
  };
  const size_t B = s.batch, sp = s.sp, lp = s.lp;
  const int64_t along = (s.tall ? s.sp : s.lp) / 32, across = (s.tall ? s.lp : s.sp) / 32;
  w.n_parts = static_cast<int32_t>(std::min<int64_t>((along + kPrepWarps - 1) / kPrepWarps * across,
                                                     std::max<int64_t>(1, 6 * kSMs / s.batch)));
  w.x = take(B * sp * lp * 4);
  w.inv = take(B * 4);
  w.partial = take(B * w.n_parts * 8);
  if (is_small(s)) {
    w.bytes = at;
    return w;
  }
  w.x16a = take(B * sp * lp * 2);
  w.x16b = take(B * sp * lp * 2);
  w.a16 = take(B * sp * sp * 2);
  w.a_blk = take(B * sp * sp * 2);
  w.b16 = take(B * sp * sp * 2);
  w.d = take(B * sp * 4);
  w.e = take(B * sp * 4);
  const Plan p = plan_of(s.batch, s.sp, s.lp);
  const size_t T = 128 * p.cg_gram;
  w.parts = take(p.splits > 1 ? p.splits * B * symmetric_items(s.sp, p.cg_gram) * T * T * 4 : 0);
  w.bytes = at;
  return w;
}

// Launch with programmatic dependence on the launch before it (its prologue may start early) and, for
// pairs, a cluster of two.
template <typename... KArgs, typename... Args>
rl_status launch(const char* what, void (*kern)(KArgs...), int64_t grid, int threads, size_t smem, int cluster,
                 cudaStream_t s, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.numAttrs = 1;
  if (cluster > 1) {
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.numAttrs = 2;
  }
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, args...);
  return e == cudaSuccess ? RL_OK : cuda_error(e, what);
}

// Shared memory beyond the default, once per device and kernel.
template <int MODE, int CG>
rl_status allow_smem() {
  static std::mutex mu;
  static std::map<int, bool> done;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_error(e, "cudaGetDevice");
  std::lock_guard<std::mutex> lock(mu);
  if (!done[dev]) {
    e = cudaFuncSetAttribute(product_kernel<MODE, CG>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(kSmem));
    if (e != cudaSuccess) return cuda_error(e, "cudaFuncSetAttribute(product_kernel)");
    done[dev] = true;
  }
  return RL_OK;
}

template <int MODE, int CG>
rl_status product(const CUtensorMap& a, const CUtensorMap& at, const CUtensorMap& b, const CUtensorMap& out,
                  const MmArgs& p, cudaStream_t s) {
  rl_status st = allow_smem<MODE, CG>();
  if (st != RL_OK) return st;
  const int64_t items = static_cast<int64_t>(p.sh.batch) * p.per * (MODE == GRAM ? p.splits : 1);
  const int64_t units = std::min<int64_t>(items, kSMs / CG);
  return launch("product_kernel launch", product_kernel<MODE, CG>, units * CG, kThreads, kSmem, CG, s, a, at, b,
                out, p);
}

rl_status small(const MmArgs& p, int steps, cudaStream_t s) {
  const size_t smem = small_smem(p.sh.lp).bytes + 1024;
  static std::mutex mu;
  static std::map<int, bool> done;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_error(e, "cudaGetDevice");
  {
    std::lock_guard<std::mutex> lock(mu);
    if (!done[dev]) {
      e = cudaFuncSetAttribute(small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               static_cast<int>(small_smem(kSmallSide).bytes + 1024));
      if (e != cudaSuccess) return cuda_error(e, "cudaFuncSetAttribute(small_kernel)");
      done[dev] = true;
    }
  }
  return launch("small_kernel launch", small_kernel, 2 * static_cast<int64_t>(p.sh.batch), kSmallThreads, smem, 2, s, p,
                steps);
}

}  // namespace muon
}  // namespace rl

using namespace rl;
using namespace rl::muon;

static rl_status muon_check(const char* fn, int32_t batch, int64_t m, int64_t n) {
  const std::string f = std::string(fn) + ": ";
  if (batch < 0 || m < 0 || n < 0) return set_error(RL_ERR_INVALID_ARG, f + "negative size");
  if (std::min(m, n) > 32768 || std::max(m, n) > (int64_t(1) << 24) ||
      round_up(std::min(m, n), 128) * batch > (int64_t(1) << 24))
    return set_error(RL_ERR_UNSUPPORTED, f + "the shorter side is at most 32,768, the longer one 2^24, and batch times "
                                             "the shorter side (rounded up to 128) 2^24");
  return RL_OK;
}

extern "C" {

size_t rl_muon_workspace_size(int32_t batch, int64_t m, int64_t n) {
  clear_error();
  if (muon_check("rl_muon_workspace_size", batch, m, n) != RL_OK) return 0;
  if (batch == 0 || m == 0 || n == 0) return kWsHeader;
  return layout_of(shape_of(batch, m, n)).bytes;
}

rl_status rl_muon_update(int32_t batch, int64_t m, int64_t n, const void* grad, rl_dtype grad_dtype, int64_t ld_grad,
                         int64_t stride_grad, float* momentum, float* weights, uint16_t* weights_bf16, int64_t ld_w,
                         int64_t stride_w, uint16_t* update, const rl_muon_params* params, void* ws, size_t ws_bytes,
                         rl_stream_t stream) {
  clear_error();
  const std::string f = "rl_muon_update: ";
  rl_status st = muon_check("rl_muon_update", batch, m, n);
  if (st != RL_OK) return st;
  if (!params) return set_error(RL_ERR_INVALID_ARG, f + "params is NULL");
  if (grad_dtype != RL_BF16 && grad_dtype != RL_F32) return set_error(RL_ERR_INVALID_ARG, f + "bad grad_dtype");
  const rl_muon_params& P = *params;
  for (int k = 0; k < 3; ++k)
    if (!(std::fabs(P.ns_coef[k]) <= 8.f))
      return set_error(RL_ERR_INVALID_ARG, f + "ns_coef must be finite and at most 8 in magnitude");
  if (P.ns_steps < 1 || P.ns_steps > 16) return set_error(RL_ERR_INVALID_ARG, f + "ns_steps outside [1, 16]");
  if (!(P.eps >= 0.f) || !std::isfinite(P.eps) || !std::isfinite(P.lr) || !std::isfinite(P.weight_decay) ||
      !std::isfinite(P.update_scale) || !(P.momentum >= 0.f && P.momentum < 1.f))
    return set_error(RL_ERR_INVALID_ARG, f + "eps >= 0, momentum in [0, 1) and finite lr, weight_decay, update_scale "
                                             "are needed");
  if (batch == 0 || m == 0 || n == 0) return RL_OK;
  if (!grad || !ws) return set_error(RL_ERR_INVALID_ARG, f + "grad or ws is NULL");
  if (!weights && !update) return set_error(RL_ERR_INVALID_ARG, f + "neither weights nor update is given");
  if (weights_bf16 && !weights) return set_error(RL_ERR_INVALID_ARG, f + "weights_bf16 without weights");
  if (P.momentum > 0.f && !momentum) return set_error(RL_ERR_INVALID_ARG, f + "momentum > 0 without a momentum buffer");
  if (ld_grad < n || stride_grad < 0) return set_error(RL_ERR_INVALID_ARG, f + "ld_grad < n or stride_grad < 0");
  if (weights) {
    const int64_t last = (m - 1) * ld_w + n;  // elements that one matrix spans
    const bool apart = stride_w >= last || (stride_w >= n && ld_w >= (batch - 1) * stride_w + n);
    if (ld_w < n || (batch > 1 && !apart))
      return set_error(RL_ERR_INVALID_ARG, f + "ld_w < n, or the batch's weights overlap");
  }
  if (reinterpret_cast<uintptr_t>(ws) % 16 != 0) return set_error(RL_ERR_ALIGNMENT, f + "ws not 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(grad) % (grad_dtype == RL_F32 ? 4 : 2)) != 0 ||
      reinterpret_cast<uintptr_t>(momentum) % 4 != 0 || reinterpret_cast<uintptr_t>(weights) % 4 != 0 ||
      reinterpret_cast<uintptr_t>(weights_bf16) % 2 != 0 || reinterpret_cast<uintptr_t>(update) % 2 != 0)
    return set_error(RL_ERR_ALIGNMENT, f + "a pointer is not aligned to its element");
  const Shape sh = shape_of(batch, m, n);
  const Layout w = layout_of(sh);
  if (ws_bytes < w.bytes) return set_error(RL_ERR_WORKSPACE_TOO_SMALL, f + "ws_bytes below rl_muon_workspace_size");

  uint8_t* base = static_cast<uint8_t*>(ws);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  int32_t* status = reinterpret_cast<int32_t*>(base);

  PrepArgs pa = {};
  pa.sh = sh;
  pa.grad = grad;
  pa.ld_grad = ld_grad;
  pa.stride_grad = stride_grad;
  pa.momentum = P.momentum > 0.f ? momentum : nullptr;
  pa.mu = P.momentum;
  pa.nesterov = P.nesterov;
  pa.eps = P.eps;
  pa.x = reinterpret_cast<float*>(base + w.x);
  pa.x16 = reinterpret_cast<uint16_t*>(base + w.x16a);
  pa.partial = reinterpret_cast<double*>(base + w.partial);
  pa.parts = w.n_parts;
  pa.inv = reinterpret_cast<float*>(base + w.inv);
  pa.done = reinterpret_cast<uint32_t*>(base + kWsMuonDoneOffset);
  pa.status = status;
  // rows of the gradient and of the momentum that begin at multiples of four elements
  const size_t ge = grad_dtype == RL_F32 ? 16 : 8;
  const bool vec = n % 4 == 0 && ld_grad % 4 == 0 && stride_grad % 4 == 0 && reinterpret_cast<uintptr_t>(grad) % ge == 0 &&
                   aligned16(pa.momentum);
  auto momentum_pass = grad_dtype == RL_BF16 ? (vec ? momentum_kernel<true, true> : momentum_kernel<true, false>)
                                             : (vec ? momentum_kernel<false, true> : momentum_kernel<false, false>);
  st = launch("momentum_kernel launch", momentum_pass, static_cast<int64_t>(batch) * w.n_parts, kPrepWarps * 32, 0, 1, s,
              pa);
  if (st != RL_OK) return st;
  if (!is_small(sh)) {
    const int64_t blocks = static_cast<int64_t>(batch) * (sh.sp / 32) * (sh.lp / 32);
    st = launch("normalise_kernel launch", normalise_kernel, (blocks + kPrepWarps - 1) / kPrepWarps, kPrepWarps * 32, 0,
                1, s, pa);
    if (st != RL_OK) return st;
  }

  MmArgs a = {};
  a.sh = sh;
  a.ca = P.ns_coef[0];
  a.cb = P.ns_coef[1];
  a.cc = P.ns_coef[2];
  a.a16 = reinterpret_cast<uint16_t*>(base + w.a16);
  a.a_blk = reinterpret_cast<uint16_t*>(base + w.a_blk);
  a.d = reinterpret_cast<float*>(base + w.d);
  a.e = reinterpret_cast<float*>(base + w.e);
  a.x = pa.x;
  a.parts = reinterpret_cast<float*>(base + w.parts);
  a.scale = P.update_scale / kXScale;
  a.update = update;
  a.weights = weights;
  a.weights_bf16 = weights_bf16;
  a.ld_w = ld_w;
  a.stride_w = stride_w;
  a.vec = n % 4 == 0 && reinterpret_cast<uintptr_t>(update) % 8 == 0 &&
          (!weights || (ld_w % 4 == 0 && stride_w % 4 == 0 && aligned16(weights) &&
                        reinterpret_cast<uintptr_t>(weights_bf16) % 8 == 0));
  a.decay = static_cast<float>(1.0 - static_cast<double>(P.lr) * P.weight_decay);
  a.step = static_cast<float>(static_cast<double>(P.lr) * P.update_scale / kXScale);
  a.status = status;
  a.inv = pa.inv;
  if (is_small(sh)) return small(a, P.ns_steps, s);

  // boxes of 64 columns: 128 rows of a K-major operand, 64 of an MN-major one, 32 of an output
  uint16_t* x16[2] = {reinterpret_cast<uint16_t*>(base + w.x16a), reinterpret_cast<uint16_t*>(base + w.x16b)};
  CUtensorMap xk[2], xn[2], ak, at, bk, bt;
  const int64_t rows = static_cast<int64_t>(batch) * sh.sp;
  const auto F16 = CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  auto map = [&](CUtensorMap* m, const void* at, int64_t cols, int box_rows) {
    if (st == RL_OK) st = tmap_2d(m, F16, at, cols, rows, cols * 2, 64, box_rows, CU_TENSOR_MAP_SWIZZLE_128B);
  };
  CUtensorMap xout[2], aout, bout;
  for (int k = 0; k < 2; ++k) {
    map(&xk[k], x16[k], sh.lp, 128);
    map(&xn[k], x16[k], sh.lp, 64);
    map(&xout[k], x16[k], sh.lp, 32);
  }
  map(&ak, base + w.a16, sh.sp, 128);
  map(&at, base + w.a16, sh.sp, 64);
  map(&aout, base + w.a16, sh.sp, 32);
  map(&bk, base + w.b16, sh.sp, 128);
  map(&bt, base + w.b16, sh.sp, 64);
  map(&bout, base + w.b16, sh.sp, 32);
  if (st != RL_OK) return st;

  const Plan plan = plan_of(batch, sh.sp, sh.lp);
  for (int k = 0; k < P.ns_steps; ++k) {
    const int T = 128 * plan.cg_gram;
    a.nt_m = static_cast<int32_t>(round_up(sh.sp, T) / T);
    a.per = static_cast<int32_t>(symmetric_items(sh.sp, plan.cg_gram));
    a.splits = plan.splits;
    a.nkb = sh.lp / BK;
    const CUtensorMap& x = xk[k & 1];
    st = plan.cg_gram == 2 ? product<GRAM, 2>(x, x, x, aout, a, s) : product<GRAM, 1>(x, x, x, aout, a, s);
    if (st != RL_OK) return st;
    if (plan.splits > 1) {
      const int64_t warps = static_cast<int64_t>(batch) * a.per * (T / 32) * (T / 32);
      auto kern = plan.cg_gram == 2 ? gram_sum_kernel<2> : gram_sum_kernel<1>;
      st = launch("gram_sum_kernel launch", kern, (warps + 7) / 8, 256, 0, 1, s, a);
      if (st != RL_OK) return st;
    }
    const int TP = 128 * plan.cg_poly;
    a.nt_m = static_cast<int32_t>(round_up(sh.sp, TP) / TP);
    a.per = static_cast<int32_t>(symmetric_items(sh.sp, plan.cg_poly));
    a.splits = 1;
    a.nkb = sh.sp / BK;
    st = plan.cg_poly == 2 ? product<POLY, 2>(ak, at, ak, bout, a, s) : product<POLY, 1>(ak, at, ak, bout, a, s);
    if (st != RL_OK) return st;
    const int TA = 128 * plan.cg_apply;
    a.nt_m = static_cast<int32_t>(round_up(sh.sp, TA) / TA);
    a.per = a.nt_m * static_cast<int32_t>(round_up(sh.lp, TA) / TA);
    a.inv = k == 0 ? pa.inv : nullptr;
    a.early = k < P.ns_steps - 2;
    const CUtensorMap &xr = xn[k & 1], &xo = xout[(k + 1) & 1];
    if (k == P.ns_steps - 1)
      st = plan.cg_apply == 2 ? product<FINAL, 2>(bk, bt, xr, xo, a, s) : product<FINAL, 1>(bk, bt, xr, xo, a, s);
    else
      st = plan.cg_apply == 2 ? product<APPLY, 2>(bk, bt, xr, xo, a, s) : product<APPLY, 1>(bk, bt, xr, xo, a, s);
    if (st != RL_OK) return st;
  }
  return RL_OK;
}

}  // extern "C"
