// Orthogonalised updates: the quintic Newton-Schulz iteration on matrices, and the optimizer step around it.
//
//     X = U / ||U||_F  (n x m, n the shorter side: a tall matrix is transposed),   then `steps` times
//     A = X X^T,   Q = a I + b A + c A A,   X <- Q X          (a, b, c) = (3.4445, -4.7750, 2.0315)
// which applies a s + b s^3 + c s^5 to the singular values and leaves the singular vectors.  It maps [0, 1.2025] into itself, so every
// |entry| of X is at most 1.21, of A 1.45, of Q 3.45.
//
// The iteration multiplies what is off by its slope, up to 3.4 per step where singular values are small, so operands of 8 or 11 significant
// bits are off by 1e-2 or 1e-3 afterwards (a fifth or 3e-2 where a few directions dominate).  Operands are therefore kept as two IEEE halves, v = hi + lo
// (22 bits, scaled by 2^12 so that neither is subnormal where it matters), and a product is hi hi + hi lo + lo hi on the
// tensor cores: three times the work of one 16-bit product, and errors like those of an fp32 product.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "pe_sm100.cuh"

namespace pe {

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float NS_SCALE = 4096.f;                     // planes hold 2^12 v
constexpr float NS_UNSCALE = 1.f / 4096.f;

// hi + lo of an already scaled value
__device__ __forceinline__ void ns_split(float v, __half& hi, __half& lo) {
  hi = __float2half_rn(v);
  lo = __float2half_rn(v - __half2float(hi));
}
__device__ __forceinline__ uint32_t ns_pack(__half a, __half b) {
  const __half2 h = __halves2half2(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// ---------------------------------------------------------------- momentum, norms, the first operand
// What the iteration starts from: a matrix as given (bf16 or fp32), or the momentum after this step.
struct NsSource {
  const void* given;          // given matrices, or NULL: momentum
  int bf16;
  float* m;                   // momentum, updated by ns_norms_kernel
  const float* sum_g;
  float grad_scale, beta;     // grad_scale = s / B
  int nesterov;
};
__device__ __forceinline__ float ns_source_value(const NsSource& s, long long i) {      // after ns_norms_kernel
  if (s.given) return s.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(s.given)[i]) : static_cast<const float*>(s.given)[i];
  const float m = s.m[i];
  return s.nesterov ? fmaf(s.beta, m, (1.f - s.beta) * (s.sum_g[i] * s.grad_scale)) : m;
}
// Squared Frobenius norms, as gridDim.x partial sums per matrix (gridDim.y matrices), in 64 bits: no scale of the gradients overflows or vanishes.
// Updates the momentum by the way, and zeroes the counters of split products and the word behind them, which says whether a product gave up.
constexpr int NS_NORM_THREADS = 256;
// WIDE: fp32, four elements to an access.
template <bool WIDE>
__global__ void __launch_bounds__(NS_NORM_THREADS)
ns_norms_kernel(NsSource s, long long elems, double* __restrict__ partial, unsigned int* __restrict__ counters, int n_counters) {
  sm100::griddep_launch_dependents();
  sm100::griddep_wait();
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int k = threadIdx.x; k < n_counters; k += blockDim.x) counters[k] = 0u;
  __shared__ double warp_sum[NS_NORM_THREADS / 32];
  const long long base = (long long)blockIdx.y * elems, stride = (long long)gridDim.x * blockDim.x;
  double sum = 0.0;
  if constexpr (WIDE) {
    const long long quads = elems / 4;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < quads; i += 2 * stride) {
      float4 g[2], m[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const long long at = i + k * stride;
        g[k] = m[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (at < quads) {
          g[k] = reinterpret_cast<const float4*>((s.given ? static_cast<const float*>(s.given) : s.sum_g) + base)[at];
          if (!s.given) m[k] = reinterpret_cast<const float4*>(s.m + base)[at];
        }
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float v[4] = {g[k].x, g[k].y, g[k].z, g[k].w};
        if (!s.given) {
          float mom[4] = {m[k].x, m[k].y, m[k].z, m[k].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float one = v[e] * s.grad_scale;
            mom[e] = fmaf(s.beta, mom[e], (1.f - s.beta) * one);
            v[e] = s.nesterov ? fmaf(s.beta, mom[e], (1.f - s.beta) * one) : mom[e];
          }
          if (i + k * stride < quads) reinterpret_cast<float4*>(s.m + base)[i + k * stride] = make_float4(mom[0], mom[1], mom[2], mom[3]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += (double)v[e] * (double)v[e];
      }
    }
  } else {
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < elems; i += 4 * stride) {
      float v[4];
  #pragma unroll
      for (int k = 0; k < 4; ++k) {
        const long long at = base + i + k * stride;
        v[k] = 0.f;
        if (i + k * stride < elems) {
          if (s.given) {
            v[k] = ns_source_value(s, at);
          } else {
            const float g = s.sum_g[at] * s.grad_scale, m = fmaf(s.beta, s.m[at], (1.f - s.beta) * g);
            s.m[at] = m;
            v[k] = s.nesterov ? fmaf(s.beta, m, (1.f - s.beta) * g) : m;
          }
        }
      }
  #pragma unroll
      for (int k = 0; k < 4; ++k) sum += (double)v[k] * (double)v[k];
    }
  }
#pragma unroll
  for (int k = 16; k > 0; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
  if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int w = 0; w < NS_NORM_THREADS / 32; ++w) t += warp_sum[w];
    partial[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = t;
  }
}
// X = U / ||U||_F as planes [2][count][n][ld]; a block takes 64 x 64 of it.  tall: U is [m, n] and goes through shared memory transposed.
// ||U|| = 0 gives X = 0.
constexpr int NS_INIT_TILE = 64;
__global__ void __launch_bounds__(256)
ns_init_kernel(NsSource s, int n, int m, int ld, int tall, int tiles_m, const double* __restrict__ partial, int partials, __half* __restrict__ planes,
               int count) {
  sm100::griddep_launch_dependents();
  sm100::griddep_wait();
  __shared__ float tile[NS_INIT_TILE][NS_INIT_TILE + 1];      // [row of X][column of X]
  __shared__ double inverse;
  const int mat = blockIdx.y, r0 = (int)(blockIdx.x / tiles_m) * NS_INIT_TILE, c0 = (int)(blockIdx.x % tiles_m) * NS_INIT_TILE;
  if (threadIdx.x < 32) {
    double t = 0.0;
    for (int k = threadIdx.x; k < partials; k += 32) t += partial[(size_t)mat * partials + k];
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) t += __shfl_xor_sync(0xffffffffu, t, k);
    if (threadIdx.x == 0) inverse = t == 0.0 ? 0.0 : (double)NS_SCALE / sqrt(t);
  }
  __syncthreads();
  const double inv = inverse;
  const long long base = (long long)mat * n * m;
  const int fast = threadIdx.x & 63, slow = threadIdx.x >> 6;
#pragma unroll 4
  for (int k = slow; k < NS_INIT_TILE; k += 4) {
    const int r = tall ? fast : k, c = tall ? k : fast;
    float v = 0.f;
    if (r0 + r < n && c0 + c < m)
      v = (float)(inv * (double)ns_source_value(s, base + (tall ? (long long)(c0 + c) * n + r0 + r : (long long)(r0 + r) * m + c0 + c)));
    tile[r][c] = v;
  }
  __syncthreads();
  const size_t plane = (size_t)count * n * ld;
  for (int k = threadIdx.x; k < NS_INIT_TILE * NS_INIT_TILE / 8; k += 256) {
    const int r = k >> 3, c = (k & 7) * 8;
    if (r0 + r >= n || c0 + c >= ld) continue;      // (ld is a multiple of 8: columns from m on are written with zeros)
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      __half h0, l0, h1, l1;
      ns_split(tile[r][c + 2 * e], h0, l0);
      ns_split(tile[r][c + 2 * e + 1], h1, l1);
      hi[e] = ns_pack(h0, h1);
      lo[e] = ns_pack(l0, l1);
    }
    __half* at = planes + ((size_t)mat * n + r0 + r) * ld + c0 + c;
    *reinterpret_cast<uint4*>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    *reinterpret_cast<uint4*>(at + plane) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  }
}

// ---------------------------------------------------------------- small matrices
// n <= 64 and m <= 128: one block takes a matrix through all of it, in fp32 in shared memory.  The tensor-core path is 17 launches of 4.4 us there, whatever the
// size; this takes one (64 x 64: 75 us by the products, 38 us here; 64 x 128: 79 and 58; 64 x 256: 83 and 101).
constexpr int NS_SMALL_N = 64, NS_SMALL_M = 128;
constexpr int NS_SMALL_THREADS = 256;
constexpr int NS_SMALL_LD = NS_SMALL_N + 4;               // rows of A and Q
struct NsResult {
  void* result;                 // bf16 or fp32, or NULL and
  int out_bf16;
  float* theta;                 // theta <- theta - step X - wd theta
  __nv_bfloat16* theta_lp;
  float step, wd;
};
__host__ __device__ constexpr int ns_small_ld(int m) { return (m + 31) / 32 * 32 + 4; }      // 4 words past a multiple of 32: rows start 4 banks apart
// out[i][j] = rows ty + 16 i of a times rows tx + 16 j of b, over k (a multiple of 4); sums of even and odd terms side by side
__device__ __forceinline__ void ns_small_rows(const float* a, const float* b, int ld, int k, int ty, int tx, float (&out)[4][4]) {
  uint64_t acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0ull;
#pragma unroll 4
  for (int q = 0; q < k; q += 4) {
    ulonglong2 x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = *reinterpret_cast<const ulonglong2*>(a + (ty + 16 * i) * ld + q);
      y[i] = *reinterpret_cast<const ulonglong2*>(b + (tx + 16 * i) * ld + q);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        acc[i][j] = sm100::f32x2_fma(x[i].x, y[j].x, acc[i][j]);
        acc[i][j] = sm100::f32x2_fma(x[i].y, y[j].y, acc[i][j]);
      }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float lo, hi;
      sm100::f32x2_unpack(acc[i][j], lo, hi);
      out[i][j] = lo + hi;
    }
}
__global__ void __launch_bounds__(NS_SMALL_THREADS)
ns_small_kernel(NsSource s, NsResult o, int n, int m, int tall, int steps) {
  sm100::griddep_launch_dependents();
  sm100::griddep_wait();
  extern __shared__ __align__(16) float ns_small[];
  __shared__ double warp_sum[NS_SMALL_THREADS / 32];
  const int ld = ns_small_ld(m), width = ld - 4, ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  float *X = ns_small, *A = X + NS_SMALL_N * ld, *Q = A + NS_SMALL_N * NS_SMALL_LD;
  const long long base = (long long)blockIdx.x * n * m;
  for (int i = threadIdx.x; i < NS_SMALL_N * ld; i += NS_SMALL_THREADS) X[i] = 0.f;
  __syncthreads();
  double sum = 0.0;
  for (int i = threadIdx.x; i < n * m; i += NS_SMALL_THREADS) {
    float v;
    if (s.given) {
      v = ns_source_value(s, base + i);
    } else {
      const float g = s.sum_g[base + i] * s.grad_scale, mom = fmaf(s.beta, s.m[base + i], (1.f - s.beta) * g);
      s.m[base + i] = mom;
      v = s.nesterov ? fmaf(s.beta, mom, (1.f - s.beta) * g) : mom;
    }
    sum += (double)v * (double)v;
    X[tall ? (i % n) * ld + i / n : (i / m) * ld + i % m] = v;
  }
#pragma unroll
  for (int k = 16; k > 0; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
  if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = sum;
  __syncthreads();
  sum = 0.0;
  for (int w = 0; w < NS_SMALL_THREADS / 32; ++w) sum += warp_sum[w];
  const double inv = sum == 0.0 ? 0.0 : 1.0 / sqrt(sum);
  for (int i = threadIdx.x; i < NS_SMALL_N * width; i += NS_SMALL_THREADS) {
    float* x = X + i / width * ld + i % width;
    *x = (float)((double)*x * inv);
  }
  __syncthreads();
  for (int k = 0; k < steps; ++k) {
    float c[4][4];
    ns_small_rows(X, X, ld, width, ty, tx, c);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) A[(ty + 16 * i) * NS_SMALL_LD + tx + 16 * j] = c[i][j];
    __syncthreads();
    ns_small_rows(A, A, NS_SMALL_LD, NS_SMALL_N, ty, tx, c);      // (A is symmetric: its rows are its columns)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = (ty + 16 * i) * NS_SMALL_LD + tx + 16 * j;
        Q[at] = fmaf(NS_C, c[i][j], fmaf(NS_B, A[at], ty + 16 * i == tx + 16 * j ? NS_A : 0.f));
      }
    __syncthreads();
    for (int c0 = 0; c0 < width; c0 += 64) {      // 64 columns of Q X at a time: rows ty + 16 i, columns c0 + 4 tx ..
      uint64_t acc[4][2];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i][0] = acc[i][1] = 0ull;
      const bool in = c0 + 4 * tx < width;
      if (in) {
#pragma unroll 4
        for (int q = 0; q < NS_SMALL_N; q += 4) {
          float4 w[4];
          ulonglong2 x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[i] = *reinterpret_cast<const float4*>(Q + (ty + 16 * i) * NS_SMALL_LD + q);
            x[i] = *reinterpret_cast<const ulonglong2*>(X + (q + i) * ld + c0 + 4 * tx);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float f[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint64_t ff = sm100::f32x2_pack(f[e], f[e]);
              acc[i][0] = sm100::f32x2_fma(ff, x[e].x, acc[i][0]);
              acc[i][1] = sm100::f32x2_fma(ff, x[e].y, acc[i][1]);
            }
          }
        }
      }
      __syncthreads();      // these columns have been read
      if (in) {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<ulonglong2*>(X + (ty + 16 * i) * ld + c0 + 4 * tx) = make_ulonglong2(acc[i][0], acc[i][1]);
      }
    }
    __syncthreads();
  }
  for (int i = threadIdx.x; i < n * m; i += NS_SMALL_THREADS) {
    const float v = X[tall ? (i % n) * ld + i / n : (i / m) * ld + i % m];
    if (o.result) {
      if (o.out_bf16) static_cast<__nv_bfloat16*>(o.result)[base + i] = __float2bfloat16_rn(v);
      else static_cast<float*>(o.result)[base + i] = v;
    } else {
      const float th = o.theta[base + i], next = th - o.step * v - o.wd * th;
      o.theta[base + i] = next;
      if (o.theta_lp) o.theta_lp[base + i] = __float2bfloat16_rn(next);
    }
  }
}

// ---------------------------------------------------------------- products
// A pair of thread blocks contracts one 256 x NT tile of one matrix.  Warp 0 of each block feeds its share of the operands by TMA (both
// planes of 64 values of the contraction index per stage), warp 1 of the leader issues the MMAs, eight warps per block add up what is in
// tensor memory and write the tile out.
//
// The tensor cores add to their fp32 accumulator by truncation, which pulls long sums of one sign (the diagonal of A) towards zero, a
// little per instruction.  So an accumulator takes one stage, the small cross terms before hi hi, and the stages are added
// up in registers, rounded to nearest: two accumulators in turn, drained while the other one fills.  (8192 x 2048: 1.4e-6 off the exact polynomial and
// 1526 us; two stages to an accumulator 3.1e-6 and 1470, all of them 5.7e-5 and 1410.  fp32 products in the same steps are 1.3e-6 off.)
enum : int { NS_SYMMETRIC = 0, NS_PLANES = 1, NS_FINAL = 2 };
struct NsProduct {
  int rows, cols, k;             // of the product: [rows, cols], contracted over k
  int tiles_n;                   // column tiles; NS_SYMMETRIC: those that touch the upper triangle are worked on
  int units;                     // tiles per matrix
  int count;
  int splits;                    // slices of the contraction index, each a pair's; the last one done adds the partial tiles up in their order
  float* partial;                // [splits][units * count][2][8 warps][NT / 2][32], where there are several
  unsigned int* counters;        // [units * count][2], zero before and after a product
  unsigned int* gave_up;         // set where a wait of this call's products ran out: the last one then writes nothing
  int add;                       // NS_SYMMETRIC: 0, or 1: the result is a I + b A + c (product), A by map_add
  // NS_FINAL: the result itself, [rows, cols] per matrix, or transposed: [cols, rows]
  int transposed;
  NsResult to;
  unsigned int* dev_status;
};
constexpr int NS_THREADS = 320;
constexpr int NS_BK = 64;
constexpr int NS_TMEM_COLS = 512;
// Write-out of planes.  A warp stages 32 x 32 pieces in the operand buffers (which nothing reads any more) as 32 rows of 64 bytes with the 64-byte swizzle,
// and TMA stores them; what lies outside the matrix is dropped there.  (Stored from registers, a row of 64 bytes to a lane touches 32 lines per instruction:
// 6 us for a 256 x 128 tile and its mirror image.)
constexpr int NS_PIECE = 32 * 64;
__device__ __forceinline__ uint32_t ns_piece_offset(int row, int col) {      // bytes; col: of halves
  return (uint32_t)(row * 64 + (((col >> 3) ^ (row >> 1)) & 3) * 16 + (col & 7) * 2);
}
template <int NT>
struct NsTile {
  static constexpr int A_PLANE = 128 * 128;                  // 128 rows of 64 halves
  static constexpr int B_PLANE = (NT / 2) * 128;
  static constexpr int STAGE_BYTES = 2 * A_PLANE + 2 * B_PLANE;
  static constexpr int STAGES = NT == 256 ? 3 : 4;
  static constexpr int ADD_BYTES = 8 * 2 * NS_PIECE;         // the first piece of A of each warp, fetched during the product
  static constexpr int BAR_BYTES = 512;
  static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + ADD_BYTES + BAR_BYTES + 1024;
  static_assert(SMEM_BYTES <= 227 * 1024, "shared memory of a block");
  // once the operands have been read: two pieces, their mirror images and two planes for each of eight warps, and (NT > 64) two pieces of A each
  static_assert(8 * 8 * NS_PIECE + (NT > 64 ? 8 * 4 * NS_PIECE : 0) <= STAGES * STAGE_BYTES, "pieces in the operands' place");
  // B with the contraction index slow: rows of 64 columns (128 bytes), or of the 32 that a block has of a 64-column tile (64 bytes)
  static constexpr int B_ROW = NT == 64 ? 64 : 128;
};
enum : int { NS_WAIT_EMPTY = 101, NS_WAIT_FULL = 102, NS_WAIT_ACC_EMPTY = 103, NS_WAIT_ACC_FULL = 104, NS_WAIT_ADD = 105 };

// Instruction descriptor: IEEE half operands, A row by row (K-major), B row by row or (b_mn) with the contraction index slow.
__host__ __device__ constexpr uint32_t ns_idesc(int N, bool b_mn) {
  return (1u << 4) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(256 >> 4) << 24);
}

// A lane's row of a piece, hi then lo NS_PIECE bytes on; with mirror also as a column of the piece 2 NS_PIECE on.  Of a piece on the diagonal each value from
// the diagonal on goes to both places of the piece itself.
template <bool MIRROR>
__device__ __forceinline__ void ns_stage(uint8_t* piece, int lane, const float (&v)[32], bool diagonal) {
#pragma unroll
  for (int j = 0; j < 32; j += 8) {
    __half h[8], l[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) ns_split(v[j + e], h[e], l[e]);
    if (!MIRROR || !diagonal) {
      uint8_t* at = piece + ns_piece_offset(lane, j);
      *reinterpret_cast<uint4*>(at) = make_uint4(ns_pack(h[0], h[1]), ns_pack(h[2], h[3]), ns_pack(h[4], h[5]), ns_pack(h[6], h[7]));
      *reinterpret_cast<uint4*>(at + NS_PIECE) = make_uint4(ns_pack(l[0], l[1]), ns_pack(l[2], l[3]), ns_pack(l[4], l[5]), ns_pack(l[6], l[7]));
    }
    if constexpr (MIRROR) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        uint8_t* at = piece + ns_piece_offset(j + e, lane);
        if (!diagonal) {
          *reinterpret_cast<__half*>(at + 2 * NS_PIECE) = h[e];
          *reinterpret_cast<__half*>(at + 3 * NS_PIECE) = l[e];
        } else if (j + e >= lane) {
          uint8_t* own = piece + ns_piece_offset(lane, j + e);
          *reinterpret_cast<__half*>(at) = *reinterpret_cast<__half*>(own) = h[e];
          *reinterpret_cast<__half*>(at + NS_PIECE) = *reinterpret_cast<__half*>(own + NS_PIECE) = l[e];
        }
      }
    }
  }
}
__device__ __forceinline__ void ns_load_piece(uint32_t dst, const CUtensorMap* map, uint32_t bar, int col, int row, int plane) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(col), "r"(row), "r"(plane) : "memory");
}
__device__ __forceinline__ void ns_store_piece(const CUtensorMap* map, uint32_t src, int col, int row, int plane) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(src), "r"(col),
               "r"(row), "r"(plane) : "memory");
}

template <int NT, bool B_MN, int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(NS_THREADS, 1)
ns_product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_out,
                  const __grid_constant__ CUtensorMap map_add, const __grid_constant__ NsProduct p) {
  using namespace sm100;
  using Tile = NsTile<NT>;
  constexpr int STAGES = Tile::STAGES, ACC = 2, COLS = NT / 2;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t add_base = smem_base + STAGES * Tile::STAGE_BYTES, bar_base = add_base + Tile::ADD_BYTES;
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (STAGES + s); };
  auto acc_full_bar = [&](int a) { return bar_base + 8u * (2 * STAGES + a); };
  auto acc_empty_bar = [&](int a) { return bar_base + 8u * (2 * STAGES + ACC + a); };
  auto add_bar = [&](int w, int c) { return bar_base + 8u * (2 * STAGES + 2 * ACC + w * (COLS / 32) + c); };      // warp w's piece c of A
  uint8_t* tail = smem_gen + STAGES * Tile::STAGE_BYTES + Tile::ADD_BYTES + 8 * (2 * STAGES + 2 * ACC + 8 * (COLS / 32));
  static_assert(8 * (2 * STAGES + 2 * ACC + 8 * (COLS / 32)) + 16 <= Tile::BAR_BYTES, "barrier area too small");
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(tail);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tail + 8);
  volatile int* split_flag = reinterpret_cast<volatile int*>(tail + 12);

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int slice = (int)(blockIdx.x >> 1) % p.splits;
  const long long unit = (blockIdx.x >> 1) / p.splits;
  const int mat = (int)(unit / p.units);
  int tile_m = 0, tile_n = (int)(unit - (long long)mat * p.units);
  if constexpr (EPI == NS_SYMMETRIC) {      // row by row, the tiles from the diagonal on
    constexpr int PER = 256 / NT;
    while (tile_n >= p.tiles_n - tile_m * PER) { tile_n -= p.tiles_n - tile_m * PER; ++tile_m; }
    tile_n += tile_m * PER;
  } else {
    tile_m = tile_n / p.tiles_n;
    tile_n -= tile_m * p.tiles_n;
  }
  const int all_stages = (p.k + NS_BK - 1) / NS_BK, stage0 = (int)((long long)all_stages * slice / p.splits);
  const int stages = (int)((long long)all_stages * (slice + 1) / p.splits) - stage0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int a = 0; a < ACC; ++a) { mbar_init(acc_full_bar(a), 1); mbar_init(acc_empty_bar(a), 16); }
    if (EPI == NS_SYMMETRIC)
      for (int w = 0; w < 8 * (COLS / 32); ++w) mbar_init(add_bar(0, w), 1);
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 2 && elect_one()) {      // (parameters of the launch: not what the kernel before writes)
    prefetch_tensormap(&map_a);
    prefetch_tensormap(&map_b);
    if (EPI != NS_FINAL) prefetch_tensormap(&map_out);
    if (EPI == NS_SYMMETRIC) prefetch_tensormap(&map_add);
  }
  if (warp == 1) { tmem_alloc_pair(smem_u32(const_cast<uint32_t*>(tmem_slot)), NS_TMEM_COLS); tmem_relinquish_pair(); }
  tc_fence_before();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  griddep_launch_dependents();
  griddep_wait();

  if (warp == 0) {
    // ---------------------------------------------------------- TMA producer (both blocks)
    const bool strict = wait_cycle_limit() < WAIT_CYCLE_LIMIT_STRICT;
    int s = 0;
    uint32_t ph = 1;
    for (int ks = 0; ks < stages; ++ks) {
      if (!mbar_wait_warp(empty_bar(s), ph, abort_flag, p.dev_status, NS_WAIT_EMPTY, strict)) break;
      if (elect_one()) {
        if (rank == 0) mbar_arrive_expect_tx(full_bar(s), 2 * Tile::STAGE_BYTES);
        const uint32_t leader_full = map_to_cta(full_bar(s), 0), dst = smem_base + s * Tile::STAGE_BYTES;
        const int k0 = (stage0 + ks) * NS_BK, row = tile_m * 256 + (int)rank * 128, col = tile_n * NT + (int)rank * (NT / 2);
#pragma unroll
        for (int plane = 0; plane < 2; ++plane) {
          const int z = plane * p.count + mat;
          tma_load_3d_pair(dst + plane * Tile::A_PLANE, &map_a, leader_full, k0, row, z);
          const uint32_t b = dst + 2 * Tile::A_PLANE + plane * Tile::B_PLANE;
          if constexpr (B_MN) {
#pragma unroll
            for (int j = 0; j < (NT == 256 ? 2 : 1); ++j) tma_load_3d_pair(b + j * (NS_BK * 128), &map_b, leader_full, col + 64 * j, k0, z);
          } else {
            tma_load_3d_pair(b, &map_b, leader_full, k0, col, z);
          }
        }
      }
      __syncwarp();
      if (++s == STAGES) { s = 0; ph ^= 1u; }
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------- MMA issuer (leader block)
    if (rank == 0) {
      const bool strict = wait_cycle_limit() < WAIT_CYCLE_LIMIT_STRICT;
      const uint32_t idesc = ns_idesc(NT, B_MN);
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int ks = 0; ks < stages && ok; ++ks) {
        const int buf = ks % ACC;
        if (!mbar_wait_warp(acc_empty_bar(buf), ((uint32_t)(ks / ACC) & 1u) ^ 1u, abort_flag, p.dev_status, NS_WAIT_ACC_EMPTY, strict)) { ok = false; break; }
        tc_fence_after();
        if (!mbar_wait_warp(full_bar(s), ph, abort_flag, p.dev_status, NS_WAIT_FULL, strict)) { ok = false; break; }
        tc_fence_after();
        if (elect_one()) {
          const uint32_t d_tmem = tmem_base + (uint32_t)(buf * NT);
          const uint32_t a_src = smem_base + s * Tile::STAGE_BYTES, b_src = a_src + 2 * Tile::A_PLANE;
          uint32_t accumulate = 0;
          const int k_left = p.k - (stage0 + ks) * NS_BK;
#pragma unroll
          for (int term = 0; term < 3; ++term) {        // hi lo, lo hi, hi hi
            const uint32_t ap = a_src + (term == 1 ? Tile::A_PLANE : 0), bp = b_src + (term == 0 ? Tile::B_PLANE : 0);
#pragma unroll
            for (int k = 0; k < NS_BK / 16; ++k) {
              if (k * 16 < k_left) {
                const uint64_t ad = make_smem_desc(ap + k * 32, 16u, 1024u, 2u);
                const uint64_t bd = B_MN ? make_smem_desc(bp + k * 16 * Tile::B_ROW, NS_BK * Tile::B_ROW, 8 * Tile::B_ROW, NT == 64 ? 4u : 2u) : make_smem_desc(bp + k * 32, 16u, 1024u, 2u);
                umma_ss_pair<0>(d_tmem, ad, bd, idesc, accumulate);
                accumulate = 1;
              }
            }
          }
          umma_commit_pair(empty_bar(s));
          umma_commit_pair(acc_full_bar(buf));
        }
        __syncwarp();
        if (++s == STAGES) { s = 0; ph ^= 1u; }
      }
    }
  } else {
    // ---------------------------------------------------------- epilogue (both blocks)
    const int q = warp & 3, h = (warp - 2) >> 2;      // lanes of tensor memory that this warp may read, half of the columns
    const uint32_t lane_base = tmem_base + ((uint32_t)(q * 32) << 16);
    const int c0 = tile_n * NT + h * COLS;
    float acc[COLS];
#pragma unroll
    for (int j = 0; j < COLS; ++j) acc[j] = 0.f;
    bool ok = true;
    // A's pieces that this warp adds: the first one into a place of its own at once, the others into the operands' place later.
    const int row0 = tile_m * 256 + (int)rank * 128 + q * 32;
    auto piece_counts = [&](int c) {      // (the warp as one) is this piece inside, and not below the diagonal, where it is the mirror image of another
      const int col = c0 + c * 32;
      return col < p.cols && row0 < p.rows && (EPI != NS_SYMMETRIC || col + 31 >= row0);
    };
    constexpr int ADD_PLACE = 8 * 8 * NS_PIECE;      // behind the staging areas
    auto add_at = [&](int c) {      // byte offset from smem_base
      return c == 0 ? (uint32_t)(STAGES * Tile::STAGE_BYTES + (warp - 2) * (2 * NS_PIECE)) : (uint32_t)(ADD_PLACE + ((warp - 2) * 2 + (c & 1)) * (2 * NS_PIECE));
    };
    auto fetch_add = [&](int c) {
      if (piece_counts(c) && elect_one()) {
        const uint32_t bar = add_bar(warp - 2, c);
        mbar_arrive_expect_tx(bar, 2 * NS_PIECE);
        ns_load_piece(smem_base + add_at(c), &map_add, bar, c0 + c * 32, row0, mat);
        ns_load_piece(smem_base + add_at(c) + NS_PIECE, &map_add, bar, c0 + c * 32, row0, p.count + mat);
      }
      __syncwarp();
    };
    if (EPI == NS_SYMMETRIC && p.add) fetch_add(0);
    for (int a = 0; a < stages; ++a) {
      const int buf = a % ACC;
      if (!mbar_wait_warp(acc_full_bar(buf), (uint32_t)(a / ACC) & 1u, abort_flag, p.dev_status, NS_WAIT_ACC_FULL)) { ok = false; break; }
      tc_fence_after();
#pragma unroll
      for (int c = 0; c < COLS / 32; ++c) {
        uint32_t v[32];
        tmem_ld_32x32b_x32_wait(lane_base + (uint32_t)(buf * NT + h * COLS + c * 32), v);
        if (c == COLS / 32 - 1) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(map_to_cta(acc_empty_bar(buf), 0));
        }
#pragma unroll
        for (int j = 0; j < 32; ++j) acc[c * 32 + j] += __uint_as_float(v[j]);
      }
    }
    if (EPI == NS_SYMMETRIC && p.add && piece_counts(0))      // (landed before anybody leaves, written out or not)
      ok = mbar_wait_warp(add_bar(warp - 2, 0), 0, abort_flag, p.dev_status, NS_WAIT_ADD) && ok;
    bool write = true;
    if (p.splits > 1) {      // (all eight warps of the block, whatever their waits said)
      const size_t tiles = (size_t)p.units * p.count, mine = ((size_t)unit * 2 + rank) * 8 + (warp - 2);
      float* at = p.partial + (slice * tiles * 16 + mine) * (COLS * 32) + lane;
#pragma unroll
      for (int j = 0; j < COLS; ++j) __stcg(at + j * 32, acc[j]);
      if (!ok && lane == 0) *reinterpret_cast<volatile unsigned int*>(p.gave_up) = 1u;      // (before this slice counts as done)
      __threadfence();
      named_bar_sync(1, 256);
      if (threadIdx.x == 64) {
        const unsigned int before = atomicAdd(p.counters + unit * 2 + rank, 1u);
        if (before == (unsigned int)p.splits - 1) p.counters[unit * 2 + rank] = 0u;
        *split_flag = before == (unsigned int)p.splits - 1;
      }
      named_bar_sync(1, 256);
      write = *split_flag != 0;
      if (write) {
        __threadfence();
        at = p.partial + mine * (COLS * 32) + lane;
#pragma unroll
        for (int j = 0; j < COLS; ++j) acc[j] = __ldcg(at + j * 32);
        for (int k = 1; k < p.splits; ++k) {
          at += tiles * 16 * (COLS * 32);
#pragma unroll
          for (int j = 0; j < COLS; ++j) acc[j] += __ldcg(at + j * 32);
        }
      }
    }
    if (EPI == NS_FINAL && *reinterpret_cast<volatile unsigned int*>(p.gave_up) != 0u) write = false;      // (an earlier product, or a slice of this tile)
    if (ok && write) {
      // A warp's 32 x 32 pieces; lanes hold rows.
      if constexpr (EPI == NS_SYMMETRIC && COLS > 32) {
        if (p.add) {
          fetch_add(1);
          if constexpr (COLS > 64) fetch_add(2);
        }
      }
      uint8_t* const staging = smem_gen + (warp - 2) * (8 * NS_PIECE);
      const uint32_t staging_s = smem_base + (uint32_t)(warp - 2) * (8 * NS_PIECE);
      int used = 0;      // pieces staged
#pragma unroll
      for (int c = 0; c < COLS / 32; ++c) {
        const int col = c0 + c * 32;
        if (EPI == NS_SYMMETRIC && c == 2 && p.add) {      // piece 1 has been read, or does not count: its place is free
          __syncwarp();
          fetch_add(3);
        }
        if (!piece_counts(c)) continue;
        float v[32];
        if constexpr (EPI == NS_FINAL) {
          // along the lanes in memory: rows of the result by way of shared memory, columns (a transposed result) as they are
          float* turn = reinterpret_cast<float*>(staging);      // [32][33]
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = acc[c * 32 + j] * (NS_UNSCALE * NS_UNSCALE);
          if (!p.transposed) {
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 32; ++j) turn[lane * 33 + j] = v[j];
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = turn[j * 33 + lane];
          }
          const int slow0 = p.transposed ? col : row0, fast = (p.transposed ? row0 : col) + lane;
          const int n_slow = (p.transposed ? p.cols : p.rows) - slow0, n_fast = p.transposed ? p.rows : p.cols;
          const size_t base = (size_t)mat * p.rows * p.cols + (size_t)slow0 * n_fast + fast;
          if (fast < n_fast) {
            if (!p.to.result) {
              float* th = p.to.theta + base;
#pragma unroll
              for (int j0 = 0; j0 < 32; j0 += 8) {      // eight loads in flight
                float old[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) old[j] = j0 + j < n_slow ? th[(size_t)(j0 + j) * n_fast] : 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                  if (j0 + j < n_slow) {
                    const float next = old[j] - p.to.step * v[j0 + j] - p.to.wd * old[j];
                    th[(size_t)(j0 + j) * n_fast] = next;
                    if (p.to.theta_lp) p.to.theta_lp[base + (size_t)(j0 + j) * n_fast] = __float2bfloat16_rn(next);
                  }
              }
            } else if (p.to.out_bf16) {
              __nv_bfloat16* to = static_cast<__nv_bfloat16*>(p.to.result) + base;
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (j < n_slow) to[(size_t)j * n_fast] = __float2bfloat16_rn(v[j]);
            } else {
              float* to = static_cast<float*>(p.to.result) + base;
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (j < n_slow) to[(size_t)j * n_fast] = v[j];
            }
          }
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = acc[c * 32 + j] * NS_UNSCALE;      // 2^12 of the value
          const bool diagonal = EPI == NS_SYMMETRIC && col == row0;
          if constexpr (EPI == NS_SYMMETRIC) {
            if (p.add) {
              if (!mbar_wait_warp(add_bar(warp - 2, c), 0, abort_flag, p.dev_status, NS_WAIT_ADD)) break;
              const uint8_t* from = smem_gen + add_at(c);
#pragma unroll
              for (int j = 0; j < 32; j += 8) {      // (zeros outside the matrix)
                const uint4 h4 = *reinterpret_cast<const uint4*>(from + ns_piece_offset(lane, j)), l4 = *reinterpret_cast<const uint4*>(from + NS_PIECE + ns_piece_offset(lane, j));
                const uint32_t hw[4] = {h4.x, h4.y, h4.z, h4.w}, lw[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&hw[e])), l = __half22float2(*reinterpret_cast<const __half2*>(&lw[e]));
                  v[j + 2 * e] = fmaf(NS_C, v[j + 2 * e], NS_B * (h.x + l.x));
                  v[j + 2 * e + 1] = fmaf(NS_C, v[j + 2 * e + 1], NS_B * (h.y + l.y));
                }
              }
              if (diagonal) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                  if (j == lane) v[j] += NS_A * NS_SCALE;
              }
            }
          }
          uint8_t* piece = staging + (used & 1) * (4 * NS_PIECE);
          const uint32_t piece_s = staging_s + (uint32_t)(used & 1) * (4 * NS_PIECE);
          if (used >= 2) {      // the stores of the piece before last have read this place
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
            __syncwarp();
          }
          ns_stage<EPI == NS_SYMMETRIC>(piece, lane, v, diagonal);
          fence_async_smem();
          __syncwarp();
          if (lane == 0) {
            ns_store_piece(&map_out, piece_s, col, row0, mat);
            ns_store_piece(&map_out, piece_s + NS_PIECE, col, row0, p.count + mat);
            if (EPI == NS_SYMMETRIC && !diagonal) {
              ns_store_piece(&map_out, piece_s + 2 * NS_PIECE, row0, col, mat);
              ns_store_piece(&map_out, piece_s + 3 * NS_PIECE, row0, col, p.count + mat);
            }
            bulk_commit_group();
          }
          ++used;
        }
      }
      if (EPI != NS_FINAL && lane == 0) bulk_wait_all();
    }
  }

  // ---------------------------------------------------------------- teardown
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {      // a wait gave up: loads in flight may still land here, so the block stays a while
    if (threadIdx.x == 0) *reinterpret_cast<volatile unsigned int*>(p.gave_up) = 1u;
    const long long t0 = clock64();
    while (clock64() - t0 < (1ll << 22)) __nanosleep(1000);
  }
  __syncwarp();
  cluster_sync_all();
  if (warp == 1) { tc_fence_after(); tmem_dealloc_pair(tmem_base, NS_TMEM_COLS); }
}

}  // namespace pe
