// Normalisation layers: forward pass, and the backward pass with the per-example gradients of gain and bias summed through phi.
//
// For a row x of d features: mu = mean(x) (0 for the root-mean-square form), r = 1 / sqrt(mean((x - mu)^2) + eps),
// xh = (x - mu) r, y = xh * gain + bias.  Backward, with w = dy * gain:
//     dx = r (w - xh mean(w xh) - mean(w))            (without the last term in the root-mean-square form)
//     G_b = sum_{t in b} dy xh,  H_b = sum_{t in b} dy,   outputs sum_b G_b, sum_b phi(G_b), sum_b H_b, sum_b phi(H_b).
// Both are bound by HBM: the forward pass reads x and writes y, the backward pass reads x and dy and writes dx; sums are fp32.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "pe_sm100.cuh"

namespace pe {

// ---------------------------------------------------------------- loads and stores of E consecutive elements
template <typename T, int E>
struct NormVec;
template <int E>
struct NormVec<float, E> {      // E = 4: one 16-byte access; E = 1
  float v[E];
  __device__ __forceinline__ void load(const float* p) {
    if constexpr (E == 4) {
      const float4 q = __ldcs(reinterpret_cast<const float4*>(p));
      v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    } else {
      v[0] = __ldcs(p);
    }
  }
  __device__ __forceinline__ void get(float (&f)[E]) const {
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = v[e];
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = 0.f;
  }
  static __device__ __forceinline__ void store(float* p, const float (&f)[E]) {
    if constexpr (E == 4) __stcs(reinterpret_cast<float4*>(p), make_float4(f[0], f[1], f[2], f[3]));
    else __stcs(p, f[0]);
  }
};
template <int E>
struct NormVec<__nv_bfloat16, E> {      // E = 8: one 16-byte access; E = 1
  uint32_t v[E == 8 ? 4 : 1];
  __device__ __forceinline__ void load(const __nv_bfloat16* p) {
    if constexpr (E == 8) {
      const uint4 q = __ldcs(reinterpret_cast<const uint4*>(p));
      v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    } else {
      v[0] = __ldcs(reinterpret_cast<const unsigned short*>(p));
    }
  }
  __device__ __forceinline__ void get(float (&f)[E]) const {      // bf16 is the upper half of an fp32
    if constexpr (E == 8) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        f[2 * k] = __uint_as_float(v[k] << 16);
        f[2 * k + 1] = __uint_as_float(v[k] & 0xffff0000u);
      }
    } else {
      f[0] = __uint_as_float(v[0] << 16);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int k = 0; k < (E == 8 ? 4 : 1); ++k) v[k] = 0u;
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&f)[E]) {      // rounded once, to nearest even
    if constexpr (E == 8) {
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * k], f[2 * k + 1]);
        w[k] = *reinterpret_cast<const uint32_t*>(&h);
      }
      __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
    } else {
      const __nv_bfloat16 h = __float2bfloat16_rn(f[0]);
      __stcs(reinterpret_cast<unsigned short*>(p), *reinterpret_cast<const unsigned short*>(&h));
    }
  }
};
// E elements of a gain or bias, which every row's group reads, from L1.  wide: 16-byte aligned (4 bytes suffice for the caller); one float at a time
// costs as many sectors per load as the whole vector.
template <int E>
__device__ __forceinline__ void norm_load_param(const float* p, int col, bool wide, float (&f)[E]) {
  if constexpr (E % 4 == 0) {
    if (wide) {
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        const float4 q = __ldg(reinterpret_cast<const float4*>(p + col + e));
        f[e] = q.x; f[e + 1] = q.y; f[e + 2] = q.z; f[e + 3] = q.w;
      }
      return;
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) f[e] = __ldg(p + col + e);
}

// ---------------------------------------------------------------- a row's group of threads
// A block is `groups` groups of G threads, a row at a time per group.  G is a power of two up to 32, or a multiple of 32.  Sums over a
// group: over the lanes by exchanges, over several warps by way of shared memory; `turn` alternates between two slots so that one
// barrier per sum is enough.  Every thread of the block calls these (groups without a row too), so barriers always meet.
constexpr int NORM_MAX_WARPS = 32;
constexpr int NORM_WIDE_GROUPS = 8;              // groups of at least 64 threads in a block of at most 512
template <int N>
__device__ __forceinline__ void norm_group_sum(float (&v)[N], int G, int group, int thread_in_group, float* slots, int& turn) {
#pragma unroll
  for (int s = 16; s > 0; s >>= 1)
    if (s < G) {
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], s);
    }
  if (G > 32) {
    const int warps = G >> 5, first = group * warps;
    float* slot = slots + turn * (NORM_MAX_WARPS * N);
    if ((thread_in_group & 31) == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) slot[(first + (thread_in_group >> 5)) * N + k] = v[k];
    }
    sm100::named_bar_sync(1 + group, G);      // (at most NORM_WIDE_GROUPS groups of more than a warp)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = 0.f;
    for (int w = 0; w < warps; ++w) {
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] += slot[(first + w) * N + k];
    }
    turn ^= 1;
  }
}

// The group sum of norm_group_sum for N = 8, 4 or 2 values, by halving exchanges: 9 instead of 40 exchanges for 8 values.  Needs G >= 32.
// `then` is applied to every sum before it goes to all lanes.
template <int N, typename Then>
__device__ __forceinline__ void norm_rows_sum(float (&v)[N], int G, int group, int thread_in_group, float* slots, int& turn, Then then) {
  const int lane = threadIdx.x & 31;
  float a[N];
#pragma unroll
  for (int k = 0; k < N; ++k) a[k] = v[k];
  int held = N, s = 16;
#pragma unroll
  for (int step = 0; step < 5; ++step) {
    if (held > 1) {      // (compile-time after unrolling) the lane keeps the half of its values that its bit picks
      const int half = held / 2;
      const bool high = lane & s;
#pragma unroll
      for (int k = 0; k < N / 2; ++k)
        if (k < half) {
          const float give = high ? a[k] : a[k + half], keep = high ? a[k + half] : a[k];
          a[k] = keep + __shfl_xor_sync(0xffffffffu, give, s);
        }
      held = half;
    } else {
      a[0] += __shfl_xor_sync(0xffffffffu, a[0], s);
    }
    s >>= 1;
  }
  // lane bits 4, 3, .. pick value bits log2(N) - 1, ..
  constexpr int SHIFT = N == 8 ? 2 : N == 4 ? 3 : 4;
  if (G > 32) {
    const int warps = G >> 5, first = group * warps;
    float* slot = slots + turn * ((int)(blockDim.x >> 5) * N);
    if ((lane & ((1 << SHIFT) - 1)) == 0) slot[(first + (thread_in_group >> 5)) * N + (lane >> SHIFT)] = a[0];
    sm100::named_bar_sync(1 + group, G);      // (at most NORM_WIDE_GROUPS groups of more than a warp)
    // a lane sums the warps' values (l mod N / 2) 2 and the one after it, of every 64 / N-th warp
    float2 q = make_float2(0.f, 0.f);
    for (int w = lane / (N / 2); w < warps; w += 64 / N) {
      const float2 one = *reinterpret_cast<const float2*>(slot + (first + w) * N + (lane % (N / 2)) * 2);
      q.x += one.x;
      q.y += one.y;
    }
#pragma unroll
    for (int s2 = 16; s2 >= N / 2; s2 >>= 1) {
      q.x += __shfl_xor_sync(0xffffffffu, q.x, s2);
      q.y += __shfl_xor_sync(0xffffffffu, q.y, s2);
    }
    q.x = then(q.x);
    q.y = then(q.y);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = __shfl_sync(0xffffffffu, k & 1 ? q.y : q.x, k / 2);
    turn ^= 1;
  } else {
    a[0] = then(a[0]);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = __shfl_sync(0xffffffffu, a[0], k << SHIFT);
  }
}

struct NormAsIs {
  __device__ __forceinline__ float operator()(float s) const { return s; }
};

// Either way of summing, with `then`.
template <int N, typename Then>
__device__ __forceinline__ void norm_sums(float (&v)[N], int G, int group, int thread_in_group, float* slots, int& turn, Then then) {
  if (G >= 32) {
    norm_rows_sum<N>(v, G, group, thread_in_group, slots, turn, then);
  } else {
    norm_group_sum<N>(v, G, group, thread_in_group, slots, turn);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = then(v[k]);
  }
}

// ---------------------------------------------------------------- rows by way of shared memory
constexpr int NORM_COLS = 8;                     // features per thread
constexpr int NORM_MAX_THREADS = 512;
static_assert(NORM_MAX_THREADS / 64 <= NORM_WIDE_GROUPS && 1 + NORM_WIDE_GROUPS <= 16, "a named barrier for every group");
constexpr int NORM_STAGES = 3;
template <typename T> __host__ __device__ constexpr int norm_rows() { return sizeof(T) == 2 ? 4 : 2; }      // R: a slot of 256 threads is 32 KB
enum : int { NORM_WAIT_ROWS = 201, NORM_WAIT_SUMS = 202 };

// Bytes of a slot: R rows of one tensor and what alignment to 16 bytes adds at both ends (slab: of every row).
__host__ __device__ constexpr size_t norm_slot_bytes(int R, int cols, int elem, bool whole) {
  return whole ? (((size_t)R * cols * elem + 15) / 16 * 16 + 32) : (size_t)R * (((size_t)cols * elem + 15) / 16 * 16 + 32);
}

// Copies n bytes from global memory at `src` to shared memory at dst + (src & 15), dst 16-byte aligned: the 16-byte aligned part by a bulk copy
// counted on `bar`, whose bytes are returned; begin, end: the tensor.  Only where an aligned word reaches out of the tensor its bytes are copied one element at a time.
template <typename T>
__device__ __forceinline__ uint32_t norm_fetch(uint32_t dst, uint8_t* dst_gen, const T* src, size_t n, const T* begin, const T* end, uint32_t bar, bool issue) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(src), lo0 = a & ~(uintptr_t)15, hi0 = (a + n + 15) & ~(uintptr_t)15;
  uintptr_t lo = lo0, hi = hi0;
  if (lo < reinterpret_cast<uintptr_t>(begin)) lo += 16;
  if (hi > reinterpret_cast<uintptr_t>(end)) hi -= 16;
  if (hi < lo) hi = lo;
  if (!issue) {      // first call: the odd ends, and the number of bytes to expect
    for (uintptr_t q = a; q < a + n && q < lo; q += sizeof(T)) *reinterpret_cast<T*>(dst_gen + (q - lo0)) = *reinterpret_cast<const T*>(q);
    for (uintptr_t q = hi > a ? hi : a; q < a + n; q += sizeof(T)) *reinterpret_cast<T*>(dst_gen + (q - lo0)) = *reinterpret_cast<const T*>(q);
    return (uint32_t)(hi - lo);
  }
  if (hi > lo)
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst + (uint32_t)(lo - lo0)), "l"(lo),
                 "r"((uint32_t)(hi - lo)), "r"(bar) : "memory");
  return 0;
}

// The same where both ends are 16-byte aligned.
__device__ __forceinline__ void norm_fetch_aligned(uint32_t dst, const void* src, uint32_t n, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(n), "r"(bar) : "memory");
}

// A thread's 8 features of a row in shared memory, as pairs: vector i is `offset[i]` bytes past byte `at`.  Vectors that are out of range have offset 0
// (norm_offsets), which only the first one has otherwise.  ZERO: they are zeros; else they hold the first one again, and the caller writes none of them.  (Weighting
// what they hold with zero does not do in sums: an infinity there is NaN.)  Threads whose first vector is out of range are left out.
template <typename T, int E, bool ZERO>
__device__ __forceinline__ void norm_row_pairs(const uint8_t* shared, uint32_t at, const uint32_t (&offset)[NORM_COLS / E], uint64_t (&o)[NORM_COLS / 2]) {
  constexpr int NV = NORM_COLS / E;
  float f[NV][E];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const uint8_t* q = shared + (at + offset[i]);
    if (ZERO && i > 0 && offset[i] == 0u) {
#pragma unroll
      for (int e = 0; e < E; ++e) f[i][e] = 0.f;
      continue;
    }
    if constexpr (E == 8) {
      const uint4 v = *reinterpret_cast<const uint4*>(q);
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int h = 0; h < 4; ++h) { f[i][2 * h] = __uint_as_float(w[h] << 16); f[i][2 * h + 1] = __uint_as_float(w[h] & 0xffff0000u); }
    } else if constexpr (E == 4) {
      const float4 v = *reinterpret_cast<const float4*>(q);
      f[i][0] = v.x; f[i][1] = v.y; f[i][2] = v.z; f[i][3] = v.w;
    } else {
      f[i][0] = (float)*reinterpret_cast<const T*>(q);
    }
  }
#pragma unroll
  for (int j = 0; j < NORM_COLS / 2; ++j) o[j] = sm100::f32x2_pack(f[2 * j / E][2 * j % E], f[(2 * j + 1) / E][(2 * j + 1) % E]);
}
template <typename T, int E>
__device__ __forceinline__ void norm_offsets(int G, int t, int cols, uint32_t (&offset)[NORM_COLS / E]) {
#pragma unroll
  for (int i = 0; i < NORM_COLS / E; ++i) offset[i] = (i * G + t) * E < cols ? (uint32_t)(i * G) * (uint32_t)(E * sizeof(T)) : 0u;
}

// s / d, with a reciprocal and a correction by the remainder: the quotient itself where it is a float, so that the mean of equal values is that value.
__device__ __forceinline__ float norm_mean(float s, float d, float inv_d) {
  const float m = s * inv_d, rest = fmaf(-m, d, s), better = fmaf(rest, inv_d, m);
  return better == better ? better : m;      // (an infinite sum has no remainder)
}
// 1 / sqrt(v) by the hardware's estimate and one Newton step for y^-2 - v = 0.
__device__ __forceinline__ float norm_rstd(float v) {
  const float y = rsqrtf(v), rest = fmaf(-v * y, y, 1.f), better = fmaf(0.5f * y, rest, y);
  return better == better ? better : y;      // (v = 0 or infinite)
}

struct NormMean {
  float d, inv_d;
  __device__ __forceinline__ float operator()(float s) const { return norm_mean(s, d, inv_d); }
};
struct NormRstd {
  float inv_d, eps;
  __device__ __forceinline__ float operator()(float s) const { return norm_rstd(fmaf(s, inv_d, eps)); }
};

// ---------------------------------------------------------------- forward
// NV vectors of E features per thread: vector i of a thread is features (i G + thread) E ..
// The row stays in registers between its sums (mean first, then the squared deviations: no cancellation) and the output.  Arithmetic is on pairs of
// features where a vector has them, one instruction for both.  WARP: a row to at most 32 lanes; three blocks to an SM keep 96 KB of loads in flight.
template <typename T, int E, int NV, bool RMS, bool WARP>
__global__ void __launch_bounds__(WARP ? 256 : 512, WARP ? 3 : 1)
norm_forward_kernel(const T* __restrict__ x, const float* __restrict__ gain, const float* __restrict__ bias, long long rows, int d, float eps,
                    T* __restrict__ y, float* __restrict__ mean, float* __restrict__ rstd, int G, int wide) {
  using namespace sm100;
  constexpr int W = E > 1 ? E / 2 : 1;      // pairs of a vector; a vector of one feature is a pair with a zero
  __shared__ float slots[2 * NORM_MAX_WARPS];
  griddep_launch_dependents();
  griddep_wait();
  const int group = threadIdx.x / G, t = threadIdx.x - group * G, groups = blockDim.x / G;
  int turn = 0;
  const long long row = (long long)blockIdx.x * groups + group;
  const bool live = row < rows;
  NormVec<T, E> in[NV];
  {
    const T* at = x + row * d;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * G + t) * E;
      if (live && col < d) in[i].load(at + col);
      else in[i].zero();
    }
  }
  auto pairs = [&](int i, uint64_t (&o)[W]) {
    float f[E];
    in[i].get(f);
#pragma unroll
    for (int j = 0; j < W; ++j) o[j] = f32x2_pack(f[E > 1 ? 2 * j : 0], E > 1 ? f[2 * j + 1] : 0.f);
  };
  float mu = 0.f, lo, hi;
  if constexpr (!RMS) {
    uint64_t s2 = 0ull;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      uint64_t f[W];
      pairs(i, f);
#pragma unroll
      for (int j = 0; j < W; ++j) s2 = f32x2_add(s2, f[j]);
    }
    f32x2_unpack(s2, lo, hi);
    float s[1] = {lo + hi};
    norm_group_sum<1>(s, G, group, t, slots, turn);
    mu = norm_mean(s[0], (float)d, 1.f / (float)d);
  }
  const uint64_t mu2 = f32x2_pack(mu, mu);
  uint64_t q2 = 0ull;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if ((i * G + t) * E < d) {
      uint64_t f[W];
      pairs(i, f);
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const uint64_t c = RMS ? f[j] : f32x2_sub(f[j], mu2);
        q2 = f32x2_fma(c, c, q2);
      }
    }
  f32x2_unpack(q2, lo, hi);
  float q[1] = {E > 1 ? lo + hi : lo};
  norm_group_sum<1>(q, G, group, t, slots, turn);
  const float r = norm_rstd(fmaf(q[0], 1.f / (float)d, eps));
  if (!live) return;
  if (t == 0) {
    if (!RMS && mean) mean[row] = mu;
    if (rstd) rstd[row] = r;
  }
  const uint64_t r2 = f32x2_pack(r, r);
  T* at = y + row * d;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = (i * G + t) * E;
    if (col < d) {
      float g[E], b[E], o[E];
      if (gain) norm_load_param<E>(gain, col, wide, g);
      if (bias) norm_load_param<E>(bias, col, wide, b);
      uint64_t f[W];
      pairs(i, f);
#pragma unroll
      for (int j = 0; j < W; ++j) {
        uint64_t h = f32x2_mul(RMS ? f[j] : f32x2_sub(f[j], mu2), r2);
        const uint64_t g2 = f32x2_pack(g[E > 1 ? 2 * j : 0], E > 1 ? g[2 * j + 1] : 0.f), b2 = f32x2_pack(b[E > 1 ? 2 * j : 0], E > 1 ? b[2 * j + 1] : 0.f);
        h = gain ? (bias ? f32x2_fma(h, g2, b2) : f32x2_mul(h, g2)) : (bias ? f32x2_add(h, b2) : h);
        if constexpr (E > 1) f32x2_unpack(h, o[2 * j], o[2 * j + 1]);
        else f32x2_unpack(h, o[0], hi);
      }
      NormVec<T, E>::store(at + col, o);
    }
  }
}

// The same for many rows: as in the backward pass below, blocks stay, a thread keeps gain and bias of its 8 features in registers, and rows come through a
// ring of bulk copies.  (Read again for every row, gain and bias are 8 bytes per feature from L1 beside 4 from HBM: 58 % of the copy rate with bf16
// rows, 87 % with fp32 ones.)
template <typename T, int E, bool RMS>
__global__ void __launch_bounds__(NORM_MAX_THREADS, E == 1 ? 1 : 2)      // (one feature at a time takes more registers)
norm_forward_ring_kernel(const T* __restrict__ x, const float* __restrict__ gain, const float* __restrict__ bias, long long rows, int d, float eps,
                         T* __restrict__ y, float* __restrict__ mean, float* __restrict__ rstd, int G, int wide, unsigned int* dev_status) {
  using namespace sm100;
  constexpr int NV = NORM_COLS / E, R = norm_rows<T>(), P = NORM_COLS / 2, S = NORM_STAGES;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(16) float slots[2 * (NORM_MAX_THREADS / 32) * R];
  __shared__ int abort_flag;
  const int group = threadIdx.x / G, t = threadIdx.x - group * G, groups = blockDim.x / G;
  const size_t slot = norm_slot_bytes(R, d, sizeof(T), true);
  uint8_t* ring = smem + (size_t)group * S * slot;
  const uint32_t ring_s = smem_u32(ring), bars = smem_u32(smem) + (uint32_t)((size_t)groups * S * slot) + group * S * 8;
  if (threadIdx.x == 0) abort_flag = 0;
  if (t == 0) {
    for (int s = 0; s < S; ++s) mbar_init(bars + 8 * s, 1);
    fence_barrier_init();
  }
  griddep_launch_dependents();
  griddep_wait();
  const long long workers = (long long)gridDim.x * groups, me = (long long)blockIdx.x * groups + group;
  const long long r0 = rows * me / workers, r1 = rows * (me + 1) / workers;
  const int turns = (int)((rows + workers * R - 1) / (workers * R));
  int n_rows = (int)(r1 - r0);
  __syncthreads();
  auto issue = [&](int b) {
    const int row = b * R;
    if (row >= n_rows) return;
    const int n = min(R, n_rows - row), s = b % S;
    const T* src = x + (r0 + row) * d;
    const uint32_t bar = bars + 8 * s, dst = ring_s + (uint32_t)(s * slot);
    if constexpr (E > 1) {
      mbar_arrive_expect_tx(bar, (uint32_t)(n * d * (int)sizeof(T)));
      norm_fetch_aligned(dst, src, (uint32_t)(n * d * (int)sizeof(T)), bar);
    } else {
      const uint32_t bytes = norm_fetch(dst, ring + s * slot, src, (size_t)n * d * sizeof(T), x, x + rows * d, bar, false);
      mbar_arrive_expect_tx(bar, bytes);
      norm_fetch(dst, ring + s * slot, src, (size_t)n * d * sizeof(T), x, x + rows * d, bar, true);
    }
  };
  if (t == 0)
    for (int b = 0; b < S - 1; ++b) issue(b);
  uint64_t g2[P], b2[P];
  {
    float f[NV][E], h[NV][E];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * G + t) * E;
#pragma unroll
      for (int e = 0; e < E; ++e) { f[i][e] = 1.f; h[i][e] = 0.f; }
      if (gain && col < d) norm_load_param<E>(gain, col, wide, f[i]);
      if (bias && col < d) norm_load_param<E>(bias, col, wide, h[i]);
    }
#pragma unroll
    for (int j = 0; j < P; ++j) {
      g2[j] = f32x2_pack(f[2 * j / E][2 * j % E], f[(2 * j + 1) / E][(2 * j + 1) % E]);
      b2[j] = f32x2_pack(h[2 * j / E][2 * j % E], h[(2 * j + 1) / E][(2 * j + 1) % E]);
    }
  }
  const bool active = t * E < d;
  uint32_t offset[NV];
  norm_offsets<T, E>(G, t, d, offset);
  uint64_t inside[P];      // 1 or 0: features out of range do not deviate from the mean
#pragma unroll
  for (int j = 0; j < P; ++j) inside[j] = f32x2_pack(2 * j < E || offset[2 * j / E] != 0u ? 1.f : 0.f, 2 * j + 1 < E || offset[(2 * j + 1) / E] != 0u ? 1.f : 0.f);
  const float fd = (float)d, inv_d = 1.f / fd;
  int turn = 0, sl = 0;
  uint32_t phase = 0;
  bool waits = true;
  const bool strict = wait_cycle_limit() < WAIT_CYCLE_LIMIT_STRICT;
  const uint32_t ring0 = (uint32_t)((size_t)group * S * slot) + (uint32_t)(t * E * sizeof(T)), row_bytes = (uint32_t)(d * sizeof(T));
  uint32_t at = ring0;
  char* out = reinterpret_cast<char*>(y + r0 * d + t * E);
  for (int b = 0; b < turns; ++b) {
    const int row0 = b * R;
    if (waits && row0 < n_rows) waits = mbar_wait_bounded(bars + 8 * sl, phase, &abort_flag, dev_status, NORM_WAIT_ROWS, strict);
    __syncwarp();
    const uint32_t first = at + (E > 1 ? 0u : (uint32_t)(reinterpret_cast<uintptr_t>(x + (r0 + row0) * d) & 15));
    // rows behind the last one hold what was there before: their results are not written
    auto pairs = [&](int k, uint64_t (&o)[P]) { norm_row_pairs<T, E, true>(smem, first + k * row_bytes, offset, o); };
    auto pairs_written = [&](int k, uint64_t (&o)[P]) { norm_row_pairs<T, E, false>(smem, first + k * row_bytes, offset, o); };
    float mu[R], q[R];
#pragma unroll
    for (int k = 0; k < R; ++k) mu[k] = q[k] = 0.f;
    if constexpr (!RMS) {
      if (active) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
          uint64_t f[P], s2 = 0ull;
          pairs(k, f);
#pragma unroll
          for (int j = 0; j < P; ++j) s2 = f32x2_add(s2, f[j]);
          float lo, hi;
          f32x2_unpack(s2, lo, hi);
          mu[k] = lo + hi;
        }
      }
      norm_sums<R>(mu, G, group, t, slots, turn, NormMean{fd, inv_d});
    }
    if (active) {
#pragma unroll
      for (int k = 0; k < R; ++k) {
        uint64_t f[P], s2 = 0ull;
        pairs(k, f);
        const uint64_t m2 = f32x2_pack(-mu[k], -mu[k]);
#pragma unroll
        for (int j = 0; j < P; ++j) {
          const uint64_t c = RMS ? f[j] : f32x2_add(f[j], m2);
          s2 = f32x2_fma(E == 8 || RMS ? c : f32x2_mul(c, inside[j]), c, s2);
        }
        float lo, hi;
        f32x2_unpack(s2, lo, hi);
        q[k] = lo + hi;
      }
    }
    norm_sums<R>(q, G, group, t, slots, turn, NormRstd{inv_d, eps});
    __syncwarp();
    // a thread of the group (or block) has given up: these sums, or later ones, are of rows that are not there, and no more rows count
    if (*(volatile int*)&abort_flag) n_rows = min(n_rows, row0);
    if (t == 0) {
      if (waits) issue(b + S - 1);      // every thread of the group has left the slot before this one
#pragma unroll
      for (int k = 0; k < R; ++k)
        if (row0 + k < n_rows) {
          if (!RMS && mean) mean[r0 + row0 + k] = mu[k];
          if (rstd) rstd[r0 + row0 + k] = q[k];
        }
    }
    auto write_row = [&](int k) {
      uint64_t f[P];
      pairs_written(k, f);
      const uint64_t m2 = f32x2_pack(-mu[k], -mu[k]), r2 = f32x2_pack(q[k], q[k]);
      float o[NV][E];
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const uint64_t h = f32x2_mul(RMS ? f[j] : f32x2_add(f[j], m2), r2);
        f32x2_unpack(f32x2_fma(h, g2[j], b2[j]), o[2 * j / E][2 * j % E], o[(2 * j + 1) / E][(2 * j + 1) % E]);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (E == 8 || (i * G + t) * E < d) NormVec<T, E>::store(reinterpret_cast<T*>(out + (k * row_bytes + (uint32_t)(i * G) * (uint32_t)(E * sizeof(T)))), o[i]);
    };
    if (active) {
      if (row0 + R <= n_rows) {
#pragma unroll
        for (int k = 0; k < R; ++k) write_row(k);
      } else {
#pragma unroll
        for (int k = 0; k < R; ++k)
          if (row0 + k < n_rows) write_row(k);
      }
    }
    out += (size_t)R * row_bytes;
    at += (uint32_t)slot;
    if (++sl == S) { sl = 0; at = ring0; phase ^= 1u; }
  }
  __syncthreads();
  if (abort_flag) {      // a wait gave up: copies in flight may still land here
    const long long t0 = clock64();
    while (clock64() - t0 < (1ll << 22)) __nanosleep(1000);
  }
}

// Rows too wide for a block's registers: three passes over the row, the later ones from L2.  (A feature's number is an int, NORM_MAX_FORWARD_D keeps it below 2^31 a
// step behind the row's end too; with unsigned ones 64 x 64 x 40000 bf16 took 529 us and 352.)
constexpr int NORM_WIDE_THREADS = 1024, NORM_MAX_FORWARD_D = INT32_MAX - NORM_WIDE_THREADS;
template <typename T, bool RMS>
__global__ void __launch_bounds__(NORM_WIDE_THREADS)
norm_forward_wide_kernel(const T* __restrict__ x, const float* __restrict__ gain, const float* __restrict__ bias, long long rows, int d, float eps,
                         T* __restrict__ y, float* __restrict__ mean, float* __restrict__ rstd) {
  __shared__ float slots[2 * NORM_MAX_WARPS];
  sm100::griddep_launch_dependents();
  sm100::griddep_wait();
  const int G = blockDim.x;
  const float inv_d = 1.f / (float)d;
  int turn = 0;
  for (long long row = blockIdx.x; row < rows; row += gridDim.x) {
    const T* xr = x + row * d;
    float mu = 0.f;
    if constexpr (!RMS) {
      float s[1] = {0.f};
      for (int c = threadIdx.x; c < d; c += G) s[0] += (float)xr[c];
      norm_group_sum<1>(s, G, 0, threadIdx.x, slots, turn);
      mu = s[0] / (float)d;      // rounded once: a row of one value keeps it
    }
    float q[1] = {0.f};
    for (int c = threadIdx.x; c < d; c += G) {
      const float f = (float)xr[c] - mu;
      q[0] = fmaf(f, f, q[0]);
    }
    norm_group_sum<1>(q, G, 0, threadIdx.x, slots, turn);
    const float r = 1.f / sqrtf(q[0] * inv_d + eps);
    if (threadIdx.x == 0) {
      if (!RMS && mean) mean[row] = mu;
      if (rstd) rstd[row] = r;
    }
    for (int c = threadIdx.x; c < d; c += G) {
      const float h = ((float)xr[c] - mu) * r;
      const float g = gain ? __ldg(gain + c) : 1.f, b = bias ? __ldg(bias + c) : 0.f;
      y[row * d + c] = (T)fmaf(h, g, b);
    }
  }
}

// ---------------------------------------------------------------- backward
// Rows are dealt out evenly and in order over workers (groups of threads); a thread keeps the sums of its own 8 features in registers.  Examples
// end anywhere in a worker's rows, so what a worker has found is an element of a monoid, joined in the workers' order:
//     an element without an end of an example: `head`, the sum over its rows
//     otherwise: `head`, the sum up to the first end (of an example that may have begun in an earlier worker), `tot`, sums of G and of phi(G) over
//     the examples that lie wholly inside, `tail`, the sum after the last end.
// (L without an end, R): head = L.head + R.head, the rest R's.  (L with an end, R without): tail = L.tail + R.head.  Both with:
// the example L.tail + R.head is complete and goes into tot.  No atomics: the sums' order is fixed by the launch's shape.
enum : int { NORM_HEAD = 0, NORM_TOT = 1, NORM_STAT = 2, NORM_TAIL = 3, NORM_PARTS = 4 };
enum : int { NORM_END = 1, NORM_LOST = 2 };
__device__ __forceinline__ float norm_phi(int phi, float g) {
  return phi == 1 ? g * g : phi == 2 ? (float)((g > 0.f) - (g < 0.f)) : g;
}
// Joins element R (has_end r_end) to L (l_end), for one feature and one of (gain, bias).
__device__ __forceinline__ void norm_join(int phi, bool l_end, float (&L)[NORM_PARTS], bool r_end, const float (&R)[NORM_PARTS]) {
  if (!l_end) {
    L[NORM_HEAD] += R[NORM_HEAD];
    if (r_end) { L[NORM_TOT] = R[NORM_TOT]; L[NORM_STAT] = R[NORM_STAT]; L[NORM_TAIL] = R[NORM_TAIL]; }
  } else {
    const float g = L[NORM_TAIL] + R[NORM_HEAD];
    if (r_end) {
      L[NORM_TOT] += g + R[NORM_TOT];
      L[NORM_STAT] += norm_phi(phi, g) + R[NORM_STAT];
      L[NORM_TAIL] = R[NORM_TAIL];
    } else {
      L[NORM_TAIL] = g;
    }
  }
}

struct NormBackward {
  const float *gain, *mean, *rstd;      // mean NULL: root-mean-square form
  const int* offsets;                   // packed batch: B + 1 row offsets; NULL: examples of T rows
  long long rows;                       // rows of the tensors
  int B, T, d, phi, G;                  // G threads per row
  int wide;                             // gain is 16-byte aligned
  uint32_t bars_at;                     // bytes of shared memory before the ring's barriers
  float* sums[4];                       // gain_sum, gain_stat, bias_sum, bias_stat, or NULL
  int accumulate;
  int cluster;                          // NORM_CLUSTER: blocks of a cluster
  float* parts;                         // [blocks][NORM_PARTS][kinds][d]; a block's element
  int* ends;                            // [blocks][blocks of a cluster]: NORM_END where an example ends in the block's rows, NORM_LOST where a wait gave up
  float* heads;                         // what the blocks' threads keep here until their rows are done (see there)
  unsigned int* dev_status;
  const float2* row_means;              // of each row: (mean(w xh), mean(w)), where a kernel before this one found them
};

// The sums over all examples from the element of all rows: what came before the first end is an example of its own, and behind the last one nothing is left.
__device__ __forceinline__ void norm_write_sums(const NormBackward& p, int kind, int col, const float (&L)[NORM_PARTS]) {
  const float sum = L[NORM_HEAD] + L[NORM_TOT], stat = norm_phi(p.phi, L[NORM_HEAD]) + L[NORM_STAT];
  float *const out_sum = p.sums[2 * kind], *const out_stat = p.sums[2 * kind + 1];
  if (out_sum) out_sum[col] = p.accumulate ? out_sum[col] + sum : sum;
  if (out_stat) out_stat[col] = p.accumulate ? out_stat[col] + stat : stat;
}

// The rows that belong to examples.  Offsets that break the rules are cut to the tensor.
__device__ __forceinline__ void norm_span(const NormBackward& p, long long& first, long long& last) {
  first = 0;
  last = p.rows;
  if (p.offsets) {
    first = p.offsets[0];
    last = p.offsets[p.B];
    first = first < 0 ? 0 : first > p.rows ? p.rows : first;
    last = last < first ? first : last > p.rows ? p.rows : last;
  }
}
// Example ends, one after the other: next() is the first end after row `r`.
struct NormEnds {
  const int* offsets;
  int B, T, b;
  long long last;
  __device__ __forceinline__ NormEnds(const NormBackward& p, long long last_) : offsets(p.offsets), B(p.B), T(p.T), b(0), last(last_) {}
  // end of the example that row r belongs to (binary search the first time)
  __device__ __forceinline__ long long find(long long r) {
    if (!offsets) return (r / T + 1) * T;
    int lo = 0, hi = B;      // the smallest k in [1, B] with offsets[k] > r
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (offsets[mid] > r) hi = mid;
      else lo = mid;
    }
    b = hi;
    const long long e = offsets[b];
    return e > r ? e : last;      // never stuck, whatever the offsets hold
  }
  __device__ __forceinline__ long long after(long long end) {      // end of the example that begins at row `end`
    if (!offsets) return end + T;
    while (b < B) {
      const long long e = offsets[++b];
      if (e > end) return e;
    }
    return last > end ? last : end + 1;
  }
};

// KINDS: 1 for the gain alone, 2 with the bias.
// NORM_WHOLE: a group has the whole row and finds the row's two means itself.  NORM_CLUSTER: wider rows are cut into slices for the blocks of a cluster,
// which exchange their sums by way of each other's shared memory.  NORM_SLAB: wider still; blockIdx.x picks the features (a grid's y has 65535 at most) and row_means has the means.
//
// A worker's rows come through a ring in shared memory, NORM_STAGES slots of R rows, filled by bulk copies that the group's first thread issues two slots
// ahead: 128 KB in flight on an SM without a register spent on them, whatever the rows' alignment.  (With the next row's loads in registers,
// a tensor of 1074 MB, bf16 rows of 2048 features, took 1467 us, a third of the copy rate: too little in flight.)  One barrier serves the sums of R rows, and tells that the slot
// before has been read.  Arithmetic is on pairs of features, one instruction for both; with c = x - mu,
//     mean(w xh) = r mean(w c),   dx = w r + c (-r^3 mean(w c)) - r mean(w),   G += (dy r) c.
// SHORT: many examples end, and the sums over them stay in registers; otherwise they are kept beside the heads in the workspace (L2), which costs
// nothing where an example has 32 rows or more and leaves registers for rows that overlap.
enum : int { NORM_WHOLE = 0, NORM_CLUSTER = 1, NORM_SLAB = 2 };
constexpr int NORM_MAX_CLUSTER = 8;
template <typename T, int E, bool RMS, int KINDS, int MODE, bool SHORT>
__global__ void __launch_bounds__(NORM_MAX_THREADS, 1)
norm_backward_kernel(const T* __restrict__ x, const T* __restrict__ dy, T* __restrict__ dx, const NormBackward p) {
  using namespace sm100;
  constexpr int NV = NORM_COLS / E, R = norm_rows<T>(), P = NORM_COLS / 2, SUMS = RMS ? R : 2 * R, S = NORM_STAGES;
  constexpr bool WHOLE = MODE == NORM_WHOLE;      // (rows come in one piece)
  constexpr bool SUMMED = MODE != NORM_SLAB;      // the means are found here
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(16) float slots[2 * (NORM_MAX_THREADS / 32) * SUMS];
  __shared__ int group_end[256];
  __shared__ int abort_flag;
  __shared__ __align__(16) float exchanged[MODE == NORM_CLUSTER ? 2 : 1][MODE == NORM_CLUSTER ? NORM_MAX_CLUSTER : 1][SUMS];      // the blocks' sums, of two turns
  __shared__ uint64_t exchange_bar[2];
  const int G = p.G, d = p.d, group = threadIdx.x / G, t = threadIdx.x - group * G, groups = blockDim.x / G, threads = blockDim.x;
  const int rank = MODE == NORM_CLUSTER ? (int)cluster_ctarank() : MODE == NORM_SLAB ? (int)blockIdx.x : 0;      // the slice of a row
  const int block = MODE == NORM_CLUSTER ? (int)blockIdx.x / p.cluster : MODE == NORM_SLAB ? (int)blockIdx.y : (int)blockIdx.x;
  const int blocks = MODE == NORM_CLUSTER ? (int)gridDim.x / p.cluster : MODE == NORM_SLAB ? (int)gridDim.y : (int)gridDim.x;
  const int col0 = rank * G * NORM_COLS, cols = WHOLE ? d : max(0, min(d - col0, G * NORM_COLS));
  const size_t slot = norm_slot_bytes(R, WHOLE ? d : G * NORM_COLS, sizeof(T), WHOLE);
  // [group][stage][x, dy], later the workers' elements in the same place; behind both (p.bars_at) a barrier per group and stage.  (Memory of a barrier is nobody
  // else's, even after its last phase: elements that were written over barriers were lost now and then.)
  uint8_t* ring = smem + (size_t)group * S * 2 * slot;
  const uint32_t ring_s = smem_u32(ring), bars = smem_u32(smem) + p.bars_at + group * S * 8;
  if (threadIdx.x == 0) {
    abort_flag = 0;
    if (MODE == NORM_CLUSTER)
      for (int k = 0; k < 2; ++k) mbar_init(smem_u32(&exchange_bar[k]), 1);
  }
  if (t == 0) {
    for (int s = 0; s < S; ++s) mbar_init(bars + 8 * s, 1);
    fence_barrier_init();
  }
  griddep_launch_dependents();
  griddep_wait();
  long long first, last;
  norm_span(p, first, last);
  const long long workers = (long long)blocks * groups, me = (long long)block * groups + group, span = last - first;
  // (span < 2^40 and workers < 2^20: the products fit)
  const long long r0 = first + span * me / workers, r1 = first + span * (me + 1) / workers;
  const int turns = (int)((span + workers * R - 1) / (workers * R));      // every group of the block takes as many
  const int n_rows = (int)(r1 - r0);
  if constexpr (MODE == NORM_CLUSTER) cluster_sync_all();      // every block of the cluster runs before one writes to it
  else __syncthreads();
  // Rows r0 + b R .. into slot b % S: by the group's first thread, or (slices of rows) by its first warp, a lane to a row.
  auto issue = [&](int b) {
    const long long row = r0 + (long long)b * R;
    if (row >= r1) return;
    const int n = (int)min((long long)R, r1 - row), s = b % S;
    const uint32_t bar = bars + 8 * s, at = (uint32_t)(s * 2 * slot);
    if constexpr (WHOLE) {
      if constexpr (E > 1) {
        const uint32_t bytes = (uint32_t)(n * d * (int)sizeof(T));
        mbar_arrive_expect_tx(bar, 2 * bytes);
        norm_fetch_aligned(ring_s + at, x + row * d, bytes, bar);
        norm_fetch_aligned(ring_s + at + (uint32_t)slot, dy + row * d, bytes, bar);
      } else {
        const T *const x_end = x + p.rows * d, *const y_end = dy + p.rows * d;
        uint32_t bytes = 0;
#pragma unroll
        for (int pass = 0; pass < 2; ++pass) {
          bytes += norm_fetch(ring_s + at, ring + at, x + row * d, (size_t)n * d * sizeof(T), x, x_end, bar, pass == 1);
          bytes += norm_fetch(ring_s + at + (uint32_t)slot, ring + at + slot, dy + row * d, (size_t)n * d * sizeof(T), dy, y_end, bar, pass == 1);
          if (pass == 0) mbar_arrive_expect_tx(bar, bytes);
        }
      }
    } else {      // (one thread doing this for all rows kept the others waiting: 32 x 512 x 8192, 278 us and 206)
      const uint32_t mine = at + t * (uint32_t)(slot / R);
      const T *const xs = x + (row + t) * d + col0, *const ys = dy + (row + t) * d + col0;
      if constexpr (E > 1) {
        const uint32_t bytes = (uint32_t)(cols * (int)sizeof(T));
        if (t == 0) mbar_arrive_expect_tx(bar, 2 * n * bytes);
        __syncwarp();
        if (t < n) {
          norm_fetch_aligned(ring_s + mine, xs, bytes, bar);
          norm_fetch_aligned(ring_s + mine + (uint32_t)slot, ys, bytes, bar);
        }
      } else {
        const T *const x_end = x + p.rows * d, *const y_end = dy + p.rows * d;
        const size_t size = (size_t)cols * sizeof(T);
        uint32_t bytes = 0;
        if (t < n) bytes = norm_fetch(ring_s + mine, ring + mine, xs, size, x, x_end, bar, false) +
                           norm_fetch(ring_s + mine + (uint32_t)slot, ring + mine + slot, ys, size, dy, y_end, bar, false);
#pragma unroll
        for (int q = 1; q < R; q *= 2) bytes += __shfl_xor_sync(0xffffffffu, bytes, q);
        __syncwarp();      // what lanes have copied themselves is there before the arrival
        if (t == 0) mbar_arrive_expect_tx(bar, bytes);
        __syncwarp();
        if (t < n) {
          norm_fetch(ring_s + mine, ring + mine, xs, size, x, x_end, bar, true);
          norm_fetch(ring_s + mine + (uint32_t)slot, ring + mine + slot, ys, size, dy, y_end, bar, true);
        }
      }
    }
  };
  const bool issues = WHOLE ? t == 0 : t < 32;
  if (issues)
    for (int b = 0; b < S - 1; ++b) issue(b);
  uint64_t gain[P], run[KINDS][P], tot[SHORT ? KINDS : 1][SHORT ? P : 1], stat[SHORT ? KINDS : 1][SHORT ? P : 1];
  {
    float f[NV][E];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = col0 + (i * G + t) * E;
#pragma unroll
      for (int e = 0; e < E; ++e) f[i][e] = 1.f;
      if (p.gain && col < d) norm_load_param<E>(p.gain, col, p.wide, f[i]);
    }
#pragma unroll
    for (int j = 0; j < P; ++j) gain[j] = f32x2_pack(f[2 * j / E][2 * j % E], f[(2 * j + 1) / E][(2 * j + 1) % E]);
  }
#pragma unroll
  for (int k = 0; k < KINDS; ++k)
#pragma unroll
    for (int j = 0; j < P; ++j) {
      run[k][j] = 0ull;
      if constexpr (SHORT) tot[k][j] = stat[k][j] = 0ull;
    }
  // [head, then tot, stat unless SHORT][kind][feature of a thread][thread]; written by the thread that reads it
  constexpr int KEPT = KINDS * NORM_COLS;
  float* const heads = p.heads + (((size_t)rank * blocks + block) * (SHORT ? 1 : 3) * KEPT) * threads + threadIdx.x;
  if constexpr (!SHORT) {
#pragma unroll 4
    for (int k = KEPT; k < 3 * KEPT; ++k) heads[(size_t)k * threads] = 0.f;
  }
  bool any_end = false;
  NormEnds ends(p, last);
  long long end = r0 < r1 ? ends.find(r0) : last;
  int end_row = (int)min(end - r0, (long long)INT32_MAX) - 1;      // the example's last row, counted from r0
  const float inv_d = 1.f / (float)d;
  int turn = 0, sl = 0;
  uint32_t phase = 0;
  const uint32_t ring0 = (uint32_t)((size_t)group * S * 2 * slot) + (uint32_t)(t * E * sizeof(T));      // this thread's first vector of slot 0
  const uint32_t row_bytes = WHOLE ? (uint32_t)(d * sizeof(T)) : (uint32_t)(slot / R), out_bytes = (uint32_t)(d * sizeof(T));
  uint32_t at = ring0;
  bool waits = true, exchange_waits = true;
  const float *mean_at = RMS ? nullptr : p.mean + r0, *rstd_at = p.rstd + r0;
  char* out = reinterpret_cast<char*>(dx + r0 * d + col0 + t * E);
  const bool strict = wait_cycle_limit() < WAIT_CYCLE_LIMIT_STRICT;
  // A row's mean and rstd (and means): a lane holds those of one row of `chunk`, and of the chunk after it, so that no turn waits for them.
  const int chunk = G < 32 ? G : 32, in_chunk = t & (chunk - 1);
  float mu_held, rs_held, mu_next, rs_next;
  float2 w_held = make_float2(0.f, 0.f), w_next = w_held;
  auto row_values = [&](int row, float& m, float& r, float2& w) {
    row += in_chunk;
    const bool live = row < n_rows;
    m = (!RMS && live) ? __ldg(mean_at + row) : 0.f;
    r = live ? __ldg(rstd_at + row) : 0.f;
    if constexpr (!SUMMED) w = live ? p.row_means[r0 + row] : make_float2(0.f, 0.f);
  };
  row_values(0, mu_held, rs_held, w_held);
  row_values(chunk, mu_next, rs_next, w_next);
  int held_end = chunk;      // rows up to here are held
  float mu[R], rs[R];
  float2 means[SUMMED ? 1 : R];
  const bool active = t * E < cols;      // a thread with features
  uint32_t offset[NV];
  norm_offsets<T, E>(G, t, cols, offset);
  // this thread's features of row k of the slot, as pairs; summed: those out of range are zeros, so that they have no part in the row's means
  auto pairs = [&](auto summed, uint32_t tensor_at, const T* tensor, long long row, int k, uint64_t (&o)[P]) {
    if constexpr (E == 1 && !WHOLE) tensor_at += (uint32_t)(reinterpret_cast<uintptr_t>(tensor + (row + k) * d + col0) & 15);
    norm_row_pairs<T, E, decltype(summed)::value>(smem, tensor_at + k * row_bytes, offset, o);
  };
  for (int b = 0; b < turns; ++b) {
    const int row0 = b * R;
    uint32_t at_x = at, at_y = at + (uint32_t)slot;
    if constexpr (E == 1 && WHOLE) {      // where in a 16-byte word the rows begin
      const uint32_t skip = (uint32_t)((r0 + row0) * d) * (uint32_t)sizeof(T);
      at_x += (skip + (uint32_t)reinterpret_cast<uintptr_t>(x)) & 15;
      at_y += (skip + (uint32_t)reinterpret_cast<uintptr_t>(dy)) & 15;
    }
    if (waits && row0 < n_rows) waits = mbar_wait_bounded(bars + 8 * sl, phase, &abort_flag, p.dev_status, NORM_WAIT_ROWS, strict);
    __syncwarp();
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if ((k == 0 || G < R) && row0 + k >= held_end) {      // (block-uniform; chunks of at least R rows end with a turn)
        mu_held = mu_next; rs_held = rs_next; w_held = w_next;
        held_end += chunk;
        row_values(held_end, mu_next, rs_next, w_next);
      }
      const int from = (row0 + k) & (chunk - 1);
      mu[k] = RMS ? 0.f : __shfl_sync(0xffffffffu, mu_held, from, chunk);
      rs[k] = __shfl_sync(0xffffffffu, rs_held, from, chunk);
      if constexpr (!SUMMED) means[k] = make_float2(__shfl_sync(0xffffffffu, w_held.x, from, chunk), __shfl_sync(0xffffffffu, w_held.y, from, chunk));
    }
    float s[SUMS];
#pragma unroll
    for (int k = 0; k < SUMS; ++k) s[k] = 0.f;
    auto sums_of = [&](int k, float mean_k, float rstd_k, float& wc, float& ws) {
      uint64_t fx[P], fy[P], s0 = 0ull, s1 = 0ull;
      pairs(std::integral_constant<bool, SUMMED>{}, at_x, x, r0 + row0, k, fx);
      pairs(std::integral_constant<bool, SUMMED>{}, at_y, dy, r0 + row0, k, fy);
      const uint64_t m2 = f32x2_pack(-mean_k, -mean_k), r2 = f32x2_pack(rstd_k, rstd_k);
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const uint64_t c = RMS ? fx[j] : f32x2_add(fx[j], m2);
        if constexpr (SUMMED) {
          const uint64_t w = f32x2_mul(fy[j], gain[j]);
          s0 = f32x2_fma(w, c, s0);
          if constexpr (!RMS) s1 = f32x2_add(s1, w);
        }
        run[0][j] = f32x2_fma(f32x2_mul(fy[j], r2), c, run[0][j]);
        if constexpr (KINDS > 1) run[1][j] = f32x2_add(run[1][j], fy[j]);
      }
      float lo, hi;
      f32x2_unpack(s0, lo, hi);
      wc = lo + hi;
      f32x2_unpack(s1, lo, hi);
      ws = lo + hi;
    };
    auto example_ends = [&] {
      // (opaque to the compiler, which would else compute the words' addresses before the loop and keep all of them)
      float* at = heads;
      int step = threads;
      asm volatile("" : "+l"(at), "+r"(step));
      // (each test once, not once per feature)
      auto all = [&](auto what) {
#pragma unroll
        for (int q = 0; q < KINDS; ++q)
#pragma unroll
          for (int j = 0; j < P; ++j) {
            what(q, j);
            run[q][j] = 0ull;
          }
      };
      if (!any_end) {
        all([&](int q, int j) {
          float g[2];
          f32x2_unpack(run[q][j], g[0], g[1]);
          at[(q * NORM_COLS + 2 * j) * step] = g[0];
          at[(q * NORM_COLS + 2 * j + 1) * step] = g[1];
        });
      } else if constexpr (SHORT) {
        if (p.phi == 1) {
          all([&](int q, int j) {
            tot[q][j] = f32x2_add(tot[q][j], run[q][j]);
            stat[q][j] = f32x2_fma(run[q][j], run[q][j], stat[q][j]);
          });
        } else if (p.phi == 0) {
          all([&](int q, int j) { tot[q][j] = f32x2_add(tot[q][j], run[q][j]); });      // (and stat is the same)
        } else {
          all([&](int q, int j) {
            float g[2];
            f32x2_unpack(run[q][j], g[0], g[1]);
            tot[q][j] = f32x2_add(tot[q][j], run[q][j]);
            stat[q][j] = f32x2_add(stat[q][j], f32x2_pack(norm_phi(2, g[0]), norm_phi(2, g[1])));
          });
        }
      } else {
        all([&](int q, int j) {
          float g[2];
          f32x2_unpack(run[q][j], g[0], g[1]);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            at[(KEPT + q * NORM_COLS + 2 * j + e) * step] += g[e];
            at[(2 * KEPT + q * NORM_COLS + 2 * j + e) * step] += norm_phi(p.phi, g[e]);
          }
        });
      }
      any_end = true;
      end = ends.after(end);
      end_row = (int)min(end - r0, (long long)INT32_MAX) - 1;
    };
    // R whole rows of one example, without a branch between them; otherwise row by row, in a loop that stays one: an example's end is much code
    const bool full = row0 + R <= n_rows;
    if (full && end_row >= row0 + R - 1) {
      if (active) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
          float ws;
          sums_of(k, mu[k], rs[k], s[k], ws);
          if constexpr (!RMS) s[R + k] = ws;
        }
      }
      if (end_row == row0 + R - 1) example_ends();
    } else {
      const int rows_left = min(R, n_rows - row0);
#pragma unroll 1
      for (int k = 0; k < rows_left; ++k) {
        if (active) {
          float mean_k = mu[0], rstd_k = rs[0], wc, ws;
#pragma unroll
          for (int q = 1; q < R; ++q) {
            mean_k = k == q ? mu[q] : mean_k;
            rstd_k = k == q ? rs[q] : rstd_k;
          }
          sums_of(k, mean_k, rstd_k, wc, ws);
#pragma unroll
          for (int q = 0; q < R; ++q) {
            s[q] = k == q ? wc : s[q];
            if constexpr (!RMS) s[R + q] = k == q ? ws : s[R + q];
          }
        }
        if (row0 + k == end_row) example_ends();
      }
    }
    bool lost;      // a thread of the group (or block) has given up: these sums, or later ones, are of rows that are not there
    if constexpr (SUMMED) {
      norm_sums<SUMS>(s, G, group, t, slots, turn, NormAsIs{});
      __syncwarp();
      lost = *(volatile int*)&abort_flag != 0;
      if constexpr (MODE == NORM_CLUSTER) {
        // Every block sends its sums to all of them; a barrier of each counts what has arrived.  A block's words of a turn are written again two turns later, when it has
        // read them: its own sums of the turn in between are only sent then, and everybody waits for those.  (A barrier of the cluster per turn instead:
        // 32 x 512 x 8192, 299 us and 278.)
        const uint32_t bar = smem_u32(&exchange_bar[b & 1]);
        if (exchange_waits && threadIdx.x == 0) mbar_arrive_expect_tx(bar, (uint32_t)(p.cluster * SUMS * sizeof(float)));
        if (exchange_waits && !lost && (int)threadIdx.x < p.cluster) {      // (sums of rows that are not there are not sent: the others' waits for them run out)
          const uint32_t to = map_to_cta(smem_u32(&exchanged[b & 1][rank][0]), threadIdx.x), to_bar = map_to_cta(bar, threadIdx.x);
#pragma unroll
          for (int k = 0; k < SUMS; k += 2)
            asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(to + 4 * k), "f"(s[k]), "f"(s[k + 1]), "r"(to_bar) : "memory");
        }
        if (exchange_waits) exchange_waits = mbar_wait_bounded(bar, (uint32_t)(b >> 1) & 1u, &abort_flag, p.dev_status, NORM_WAIT_SUMS, strict);
        __syncwarp();
#pragma unroll
        for (int k = 0; k < SUMS; ++k) s[k] = 0.f;
        for (int q = 0; q < p.cluster; ++q)
#pragma unroll
          for (int k = 0; k < SUMS; ++k) s[k] += exchanged[b & 1][q][k];
      }
    } else {
      __syncthreads();
      lost = *(volatile int*)&abort_flag != 0;
    }
    __syncwarp();
    // every thread of the group has left the slot before this one
    if (issues && (WHOLE ? waits : __all_sync(0xffffffffu, waits))) issue(b + S - 1);      // (a slot whose wait gave up is not filled again: its barrier's phase is open, and must not be arrived at)
    auto write_row = [&](int k) {
      float k0 = 0.f, k1;
      if constexpr (SUMMED) {
        k1 = -rs[k] * (rs[k] * (rs[k] * (s[k] * inv_d)));      // (s: sums of w c)
        if constexpr (!RMS) k0 = -rs[k] * (s[R + k] * inv_d);
      } else {
        k1 = -rs[k] * (rs[k] * means[k].x);
        if constexpr (!RMS) k0 = -rs[k] * means[k].y;
      }
      uint64_t fx[P], fy[P];
      pairs(std::false_type{}, at_x, x, r0 + row0, k, fx);
      pairs(std::false_type{}, at_y, dy, r0 + row0, k, fy);
      const uint64_t m2 = f32x2_pack(-mu[k], -mu[k]), r2 = f32x2_pack(rs[k], rs[k]), k02 = f32x2_pack(k0, k0), k12 = f32x2_pack(k1, k1);
      float o[NV][E];
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const uint64_t c = RMS ? fx[j] : f32x2_add(fx[j], m2), w = f32x2_mul(fy[j], gain[j]);
        const uint64_t v = f32x2_fma(c, k12, RMS ? f32x2_mul(w, r2) : f32x2_fma(w, r2, k02));
        f32x2_unpack(v, o[2 * j / E][2 * j % E], o[(2 * j + 1) / E][(2 * j + 1) % E]);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (E == 8 || (i * G + t) * E < cols) NormVec<T, E>::store(reinterpret_cast<T*>(out + (k * out_bytes + (uint32_t)(i * G) * (uint32_t)(E * sizeof(T)))), o[i]);
    };
    if (dx && active && !lost && exchange_waits) {
      if (full) {
#pragma unroll
        for (int k = 0; k < R; ++k) write_row(k);
      } else {
#pragma unroll
        for (int k = 0; k < R; ++k)
          if (row0 + k < n_rows) write_row(k);
      }
    }
    out += (size_t)R * out_bytes;
    at += 2 * (uint32_t)slot;
    if (++sl == S) { sl = 0; at = ring0; phase ^= 1u; }
  }
  // The ring has been read for the last time: it holds the workers' elements now, part q, kind k, feature c of every thread.
  __syncthreads();
  if (abort_flag) {      // a wait gave up: copies in flight may still land here
    const long long t0 = clock64();
    while (clock64() - t0 < (1ll << 22)) __nanosleep(1000);
  }
  float* words = reinterpret_cast<float*>(smem);
  auto word = [&](int q, int k, int c, int thread) -> float& { return words[((q * KINDS + k) * NORM_COLS + c) * threads + thread]; };
#pragma unroll
  for (int k = 0; k < KINDS; ++k)
#pragma unroll
    for (int j = 0; j < P; ++j) {
      float g[2], a[2], v[2];
      f32x2_unpack(run[k][j], g[0], g[1]);
      if constexpr (SHORT) {
        f32x2_unpack(tot[k][j], a[0], a[1]);
        f32x2_unpack(p.phi == 0 ? tot[k][j] : stat[k][j], v[0], v[1]);
      } else {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          a[e] = heads[(KEPT + k * NORM_COLS + 2 * j + e) * threads];
          v[e] = heads[(2 * KEPT + k * NORM_COLS + 2 * j + e) * threads];
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int c = 2 * j + e;
        word(NORM_HEAD, k, c, threadIdx.x) = any_end ? heads[(k * NORM_COLS + c) * threads] : g[e];      // without an end all is `head`
        word(NORM_TOT, k, c, threadIdx.x) = a[e];
        word(NORM_STAT, k, c, threadIdx.x) = v[e];
        word(NORM_TAIL, k, c, threadIdx.x) = any_end ? g[e] : 0.f;
      }
    }
  if (t == 0) group_end[group] = any_end;
  __syncthreads();
  // The block's groups are joined, a (kind, feature of a thread, thread of a group) at a time.
  for (int item = threadIdx.x; item < KINDS * NORM_COLS * G; item += threads) {
    const int kc = item / G, tt = item - kc * G, k = kc / NORM_COLS, c = kc - k * NORM_COLS;
    const int col = col0 + (c / E * G + tt) * E + c % E;
    if (col >= d) continue;
    float L[NORM_PARTS] = {word(0, k, c, tt), word(1, k, c, tt), word(2, k, c, tt), word(3, k, c, tt)};
    bool le = group_end[0] != 0;
    for (int g = 1; g < groups; ++g) {
      const bool re = group_end[g] != 0;
      const int th = g * G + tt;
      const float Rr[NORM_PARTS] = {word(0, k, c, th), word(1, k, c, th), word(2, k, c, th), word(3, k, c, th)};
      norm_join(p.phi, le, L, re, Rr);
      le |= re;
    }
    if (MODE == NORM_WHOLE && blocks == 1) {      // nothing to join with
      if (!abort_flag) norm_write_sums(p, k, col, L);
      continue;
    }
    float* out = p.parts + ((size_t)block * NORM_PARTS * KINDS + k) * d + col;
#pragma unroll
    for (int q = 0; q < NORM_PARTS; ++q) out[(size_t)q * KINDS * d] = L[q];
  }
  if (threadIdx.x == 0) {
    int found = abort_flag ? NORM_LOST : 0;
    for (int g = 0; g < groups; ++g) found |= group_end[g] ? NORM_END : 0;
    if (MODE == NORM_SLAB) atomicOr(p.ends + block, found);      // (zeroed by norm_row_means_kernel)
    else p.ends[MODE == NORM_CLUSTER ? block * p.cluster + rank : block] = found;
  }
  if constexpr (MODE == NORM_CLUSTER) cluster_sync_all();      // nobody leaves while its shared memory may be written
}

// The two means of every row, for rows wider than a block of norm_backward_kernel: a block per row.
template <typename T, bool RMS>
__global__ void __launch_bounds__(1024)
norm_row_means_kernel(const T* __restrict__ x, const T* __restrict__ dy, const NormBackward p, float2* __restrict__ row_means, int blocks) {
  __shared__ float slots[2 * NORM_MAX_WARPS * 2];
  sm100::griddep_launch_dependents();
  sm100::griddep_wait();
  if (blockIdx.x == 0)
    for (int b = threadIdx.x; b < blocks; b += blockDim.x) p.ends[b] = 0;
  long long first, last;
  norm_span(p, first, last);
  const float inv_d = 1.f / (float)p.d;
  int turn = 0;
  for (long long row = first + blockIdx.x; row < last; row += gridDim.x) {
    const float mu = RMS ? 0.f : __ldg(p.mean + row), r = __ldg(p.rstd + row);
    float s[2] = {0.f, 0.f};
    for (int c = threadIdx.x; c < p.d; c += blockDim.x) {
      const float h = ((float)x[row * p.d + c] - mu) * r, w = (float)dy[row * p.d + c] * (p.gain ? __ldg(p.gain + c) : 1.f);
      s[0] = fmaf(w, h, s[0]);
      s[1] += w;
    }
    norm_group_sum<2>(s, blockDim.x, 0, threadIdx.x, slots, turn);
    if (threadIdx.x == 0) row_means[row] = make_float2(s[0] * inv_d, s[1] * inv_d);
  }
}

// Joins the blocks' elements, in their order: a block per 32 features, its warps take consecutive elements and are joined in turn.  Where a wait gave up in any of
// them all sums are left as they were.
constexpr int NORM_JOIN_WARPS = 32, NORM_JOIN_BATCH = 4;      // elements whose words a warp has in flight
template <int KINDS>
__global__ void __launch_bounds__(32 * NORM_JOIN_WARPS)
norm_join_kernel(const NormBackward p, int blocks) {
  __shared__ float joined[NORM_JOIN_WARPS][NORM_PARTS][32];
  __shared__ int warp_end[NORM_JOIN_WARPS];
  sm100::griddep_launch_dependents();
  sm100::griddep_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int d = p.d, phi = p.phi, units = (d + 31) / 32, kind = blockIdx.x / units, col = (blockIdx.x - kind * units) * 32 + lane;
  const int b0 = (int)((long long)blocks * warp / NORM_JOIN_WARPS), b1 = (int)((long long)blocks * (warp + 1) / NORM_JOIN_WARPS);
  float L[NORM_PARTS] = {0.f, 0.f, 0.f, 0.f};      // no rows: an element without an end
  bool le = false;
  const int ranks = p.cluster > 0 ? p.cluster : 1;
  int lost = 0;
  for (int i = threadIdx.x; i < blocks * ranks; i += blockDim.x) lost |= p.ends[i] & NORM_LOST;
  for (int b = b0; b < b1; b += NORM_JOIN_BATCH) {
    float R[NORM_JOIN_BATCH][NORM_PARTS];
    int re[NORM_JOIN_BATCH];
#pragma unroll
    for (int k = 0; k < NORM_JOIN_BATCH; ++k) {
      const bool live = b + k < b1;
      const float* at = p.parts + ((size_t)(b + k) * NORM_PARTS * KINDS + kind) * d + col;
      re[k] = live ? p.ends[(b + k) * ranks] & NORM_END : 0;
#pragma unroll
      for (int q = 0; q < NORM_PARTS; ++q) R[k][q] = live && col < d ? at[(size_t)q * KINDS * d] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < NORM_JOIN_BATCH; ++k) {      // (behind the last: nothing is added)
      norm_join(phi, le, L, re[k] != 0, R[k]);
      le |= re[k] != 0;
    }
  }
#pragma unroll
  for (int q = 0; q < NORM_PARTS; ++q) joined[warp][q][lane] = L[q];
  if (lane == 0) warp_end[warp] = le;
  if (__syncthreads_or(lost) || warp != 0 || col >= d) return;
  for (int w = 1; w < NORM_JOIN_WARPS; ++w) {
    const bool re = warp_end[w] != 0;
    const float R[NORM_PARTS] = {joined[w][0][lane], joined[w][1][lane], joined[w][2][lane], joined[w][3][lane]};
    norm_join(phi, le, L, re, R);
    le |= re;
  }
  norm_write_sums(p, kind, col, L);
}

}  // namespace pe
