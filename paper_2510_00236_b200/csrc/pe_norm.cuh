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
template <int E>
__device__ __forceinline__ void norm_load_param(const float* p, int col, float (&f)[E]) {
  // parameters: 4-byte aligned only (E elements of a gain or bias are read by every row's group, from L1)
#pragma unroll
  for (int e = 0; e < E; ++e) f[e] = __ldg(p + col + e);
}

// ---------------------------------------------------------------- a row's group of threads
// A block is `groups` groups of G threads, a row at a time per group.  G is a power of two up to 32, or a multiple of 32.  Sums over a
// group: over the lanes by exchanges, over several warps by way of shared memory; `turn` alternates between two slots so that one
// barrier per sum is enough.  Every thread of the block calls these (groups without a row too), so barriers always meet.
constexpr int NORM_MAX_WARPS = 32;
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
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = 0.f;
    for (int w = 0; w < warps; ++w) {
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] += slot[(first + w) * N + k];
    }
    turn ^= 1;
  }
}

// ---------------------------------------------------------------- forward
// NV vectors of E features per thread: vector i of a thread is features (i G + thread) E ..
// The row stays in registers between its sums (mean first, then the squared deviations: no cancellation) and the output.
template <typename T, int E, int NV, bool RMS>
__global__ void __launch_bounds__(1024)
norm_forward_kernel(const T* __restrict__ x, const float* __restrict__ gain, const float* __restrict__ bias, long long rows, int d, float eps,
                    T* __restrict__ y, float* __restrict__ mean, float* __restrict__ rstd, int G) {
  __shared__ float slots[2 * NORM_MAX_WARPS];
  sm100::griddep_launch_dependents();
  sm100::griddep_wait();
  const int group = threadIdx.x / G, t = threadIdx.x - group * G, groups = blockDim.x / G;
  const float inv_d = 1.f / (float)d;
  int turn = 0;
  for (long long base = (long long)blockIdx.x * groups; base < rows; base += (long long)gridDim.x * groups) {
    const long long row = base + group;
    const bool live = row < rows;
    const T* xr = x + row * d;
    NormVec<T, E> in[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * G + t) * E;
      if (live && col < d) in[i].load(xr + col);
      else in[i].zero();
    }
    float mu = 0.f;
    if constexpr (!RMS) {
      float s[1] = {0.f};
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float f[E];
        in[i].get(f);
#pragma unroll
        for (int e = 0; e < E; ++e) s[0] += f[e];
      }
      norm_group_sum<1>(s, G, group, t, slots, turn);
      mu = s[0] / (float)d;      // rounded once: a row of one value keeps it
    }
    float q[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if ((i * G + t) * E < d) {
        float f[E];
        in[i].get(f);
#pragma unroll
        for (int e = 0; e < E; ++e) q[0] = fmaf(f[e] - mu, f[e] - mu, q[0]);
      }
    }
    norm_group_sum<1>(q, G, group, t, slots, turn);
    const float r = 1.f / sqrtf(q[0] * inv_d + eps);
    if (live) {
      if (t == 0) {
        if (!RMS && mean) mean[row] = mu;
        if (rstd) rstd[row] = r;
      }
      T* yr = y + row * d;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int col = (i * G + t) * E;
        if (col < d) {
          float f[E], g[E], b[E], o[E];
          in[i].get(f);
          if (gain) norm_load_param<E>(gain, col, g);
          if (bias) norm_load_param<E>(bias, col, b);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float h = (f[e] - mu) * r;
            o[e] = gain ? (bias ? fmaf(h, g[e], b[e]) : h * g[e]) : (bias ? h + b[e] : h);
          }
          NormVec<T, E>::store(yr + col, o);
        }
      }
    }
  }
}

// Rows too wide for a block's registers: three passes over the row, the later ones from L2.
template <typename T, bool RMS>
__global__ void __launch_bounds__(1024)
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
constexpr int NORM_COLS = 8;                     // features per thread
enum : int { NORM_HEAD = 0, NORM_TOT = 1, NORM_STAT = 2, NORM_TAIL = 3, NORM_PARTS = 4 };
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
  float* parts;                         // [blocks][NORM_PARTS][kinds][d]; a block's element
  int* ends;                            // [blocks]: whether an example ends in the block's rows
  const float2* row_means;              // of each row: (mean(w xh), mean(w)), where a kernel before this one found them
};

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

// KINDS: 1 for the gain alone, 2 with the bias.  WHOLE: a group has the whole row and finds the row's two means itself.  Otherwise blockIdx.y picks the features and row_means has them.
template <typename T, int E, bool RMS, int KINDS, bool WHOLE, int MAX_THREADS>
__global__ void __launch_bounds__(MAX_THREADS)
norm_backward_kernel(const T* __restrict__ x, const T* __restrict__ dy, T* __restrict__ dx, const NormBackward p) {
  constexpr int NV = NORM_COLS / E;
  extern __shared__ float smem[];
  __shared__ float slots[2 * NORM_MAX_WARPS * 2];
  sm100::griddep_launch_dependents();
  sm100::griddep_wait();
  const int G = p.G, d = p.d, group = threadIdx.x / G, t = threadIdx.x - group * G, groups = blockDim.x / G;
  const int col0 = WHOLE ? 0 : blockIdx.y * G * NORM_COLS;
  long long first, last;
  norm_span(p, first, last);
  const long long workers = (long long)gridDim.x * groups, me = (long long)blockIdx.x * groups + group, span = last - first;
  // (span < 2^40 and workers < 2^20: the products fit)
  const long long r0 = first + span * me / workers, r1 = first + span * (me + 1) / workers;
  const long long longest = (span + workers - 1) / workers;      // every group of the block takes as many turns
  float gain[NV][E];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int col = col0 + (i * G + t) * E;
#pragma unroll
    for (int e = 0; e < E; ++e) gain[i][e] = 1.f;
    if (p.gain && col < d) norm_load_param<E>(p.gain, col, gain[i]);
  }
  float run[KINDS][NV][E], head[KINDS][NV][E], tot[KINDS][NV][E], stat[KINDS][NV][E];
#pragma unroll
  for (int k = 0; k < KINDS; ++k)
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) run[k][i][e] = head[k][i][e] = tot[k][i][e] = stat[k][i][e] = 0.f;
  bool any_end = false;
  NormEnds ends(p, last);
  long long end = r0 < r1 ? ends.find(r0) : last;
  const float inv_d = 1.f / (float)d;
  int turn = 0;
  for (long long k = 0; k < longest; ++k) {
    const long long row = r0 + k;
    const bool live = row < r1;
    NormVec<T, E> vx[NV], vy[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = col0 + (i * G + t) * E;
      if (live && col < d) {
        vx[i].load(x + row * d + col);
        vy[i].load(dy + row * d + col);
      } else {
        vx[i].zero();
        vy[i].zero();
      }
    }
    const float mu = (!RMS && live) ? __ldg(p.mean + row) : 0.f;
    const float r = live ? __ldg(p.rstd + row) : 0.f;
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float fx[E], fy[E];
      vx[i].get(fx);
      vy[i].get(fy);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float h = (fx[e] - mu) * r, w = fy[e] * gain[i][e];
        s[0] = fmaf(w, h, s[0]);
        s[1] += w;
        run[0][i][e] = fmaf(fy[e], h, run[0][i][e]);
        if constexpr (KINDS > 1) run[1][i][e] += fy[e];
      }
    }
    if constexpr (WHOLE) {
      norm_group_sum<2>(s, G, group, t, slots, turn);
      s[0] *= inv_d;
      s[1] *= inv_d;
    } else if (live) {
      const float2 m = p.row_means[row];
      s[0] = m.x;
      s[1] = m.y;
    }
    if (live) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int col = col0 + (i * G + t) * E;
        if (col < d) {
          float fx[E], fy[E], o[E];
          vx[i].get(fx);
          vy[i].get(fy);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float h = (fx[e] - mu) * r, w = fy[e] * gain[i][e];
            const float a = fmaf(-h, s[0], w);
            o[e] = r * (RMS ? a : a - s[1]);
          }
          if (dx) NormVec<T, E>::store(dx + row * d + col, o);
        }
      }
      if (row + 1 == end) {      // the example ends with this row
#pragma unroll
        for (int k2 = 0; k2 < KINDS; ++k2)
#pragma unroll
          for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const float g = run[k2][i][e];
              if (!any_end) {
                head[k2][i][e] = g;
              } else {
                tot[k2][i][e] += g;
                stat[k2][i][e] += norm_phi(p.phi, g);
              }
              run[k2][i][e] = 0.f;
            }
        any_end = true;
        end = ends.after(end);
      }
    }
  }
  // this worker's element: without an end all of its sum is `head`
#pragma unroll
  for (int k = 0; k < KINDS; ++k)
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (!any_end) { head[k][i][e] = run[k][i][e]; run[k][i][e] = 0.f; }
  // The block's groups are joined by way of shared memory, one (kind) at a time: [groups][NORM_PARTS][G * 8].
  int* group_end = reinterpret_cast<int*>(smem + (size_t)groups * NORM_PARTS * G * NORM_COLS);
  if (t == 0) group_end[group] = any_end;
  const int width = G * NORM_COLS;
#pragma unroll
  for (int k = 0; k < KINDS; ++k) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float* at = smem + (size_t)group * NORM_PARTS * width + (i * G + t) * E + e;
        at[NORM_HEAD * width] = head[k][i][e];
        at[NORM_TOT * width] = tot[k][i][e];
        at[NORM_STAT * width] = stat[k][i][e];
        at[NORM_TAIL * width] = run[k][i][e];
      }
    __syncthreads();
    bool l_end = false;
    for (int g = 0; g < groups; ++g) l_end |= group_end[g] != 0;
    for (int c = threadIdx.x; c < width && col0 + c < d; c += blockDim.x) {
      float L[NORM_PARTS] = {smem[c], smem[NORM_TOT * width + c], smem[NORM_STAT * width + c], smem[NORM_TAIL * width + c]};
      bool le = group_end[0] != 0;
      for (int g = 1; g < groups; ++g) {
        const float* at = smem + (size_t)g * NORM_PARTS * width + c;
        const bool re = group_end[g] != 0;
        const float R[NORM_PARTS] = {at[0], at[NORM_TOT * width], at[NORM_STAT * width], at[NORM_TAIL * width]};
        norm_join(p.phi, le, L, re, R);
        le |= re;
      }
      float* out = p.parts + ((size_t)blockIdx.x * NORM_PARTS * KINDS + k) * d + col0 + c;
#pragma unroll
      for (int q = 0; q < NORM_PARTS; ++q) out[(size_t)q * KINDS * d] = L[q];
    }
    if (k == 0 && threadIdx.x == 0 && (WHOLE || blockIdx.y == 0)) p.ends[blockIdx.x] = l_end;
  }
}

// The two means of every row, for rows wider than a block of norm_backward_kernel: a block per row.
template <typename T, bool RMS>
__global__ void __launch_bounds__(1024)
norm_row_means_kernel(const T* __restrict__ x, const T* __restrict__ dy, const NormBackward p, float2* __restrict__ row_means) {
  __shared__ float slots[2 * NORM_MAX_WARPS * 2];
  sm100::griddep_launch_dependents();
  sm100::griddep_wait();
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

// Joins the blocks' elements, in their order: a block per 32 features, its warps take consecutive elements and are joined in turn.
constexpr int NORM_JOIN_WARPS = 16;
template <int KINDS>
__global__ void __launch_bounds__(32 * NORM_JOIN_WARPS)
norm_join_kernel(const float* __restrict__ parts, const int* __restrict__ ends, int blocks, int d, int phi, int accumulate,
                 float* __restrict__ gain_sum, float* __restrict__ gain_stat, float* __restrict__ bias_sum, float* __restrict__ bias_stat) {
  __shared__ float joined[NORM_JOIN_WARPS][NORM_PARTS][32];
  __shared__ int warp_end[NORM_JOIN_WARPS];
  sm100::griddep_launch_dependents();
  sm100::griddep_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int units = (d + 31) / 32, kind = blockIdx.x / units, col = (blockIdx.x - kind * units) * 32 + lane;
  const int b0 = (int)((long long)blocks * warp / NORM_JOIN_WARPS), b1 = (int)((long long)blocks * (warp + 1) / NORM_JOIN_WARPS);
  float L[NORM_PARTS] = {0.f, 0.f, 0.f, 0.f};      // no rows: an element without an end
  bool le = false;
  for (int b = b0; b < b1; ++b) {
    const bool re = ends[b] != 0;
    float R[NORM_PARTS];
    const float* at = parts + ((size_t)b * NORM_PARTS * KINDS + kind) * d + col;
#pragma unroll
    for (int q = 0; q < NORM_PARTS; ++q) R[q] = col < d ? at[(size_t)q * KINDS * d] : 0.f;
    norm_join(phi, le, L, re, R);
    le |= re;
  }
#pragma unroll
  for (int q = 0; q < NORM_PARTS; ++q) joined[warp][q][lane] = L[q];
  if (lane == 0) warp_end[warp] = le;
  __syncthreads();
  if (warp != 0 || col >= d) return;
  for (int w = 1; w < NORM_JOIN_WARPS; ++w) {
    const bool re = warp_end[w] != 0;
    const float R[NORM_PARTS] = {joined[w][0][lane], joined[w][1][lane], joined[w][2][lane], joined[w][3][lane]};
    norm_join(phi, le, L, re, R);
    le |= re;
  }
  // what came before the first end is an example of its own; behind the last end nothing is left
  float sum = L[NORM_HEAD] + L[NORM_TOT], stat = norm_phi(phi, L[NORM_HEAD]) + L[NORM_STAT];
  float *const out_sum = kind ? bias_sum : gain_sum, *const out_stat = kind ? bias_stat : gain_stat;
  if (out_sum) out_sum[col] = accumulate ? out_sum[col] + sum : sum;
  if (out_stat) out_stat[col] = accumulate ? out_stat[col] + stat : stat;
}

}  // namespace pe
