// Entry points of the normalisation layers: argument checks, the choice of the launch, and the launches.
#include <algorithm>
#include <type_traits>

#include "pe_host.cuh"
#include "pe_norm.cuh"

namespace pe {

// Lets `kernel` use `smem` bytes of shared memory on the current device; asked of the driver once per kernel, device and largest size so far.  (What a kernel may use
// without asking is 48 KB together with its static shared memory, which is below 4 KB in all of them.)
template <typename Kernel>
static pe_status_t allow_smem(Kernel kernel, std::atomic<int> (&allowed)[MAX_DEVICES], int smem) {
  if (smem <= 44 * 1024) return PE_OK;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return PE_ERR_CUDA; }
  if (allowed[dev].load(std::memory_order_acquire) >= smem) return PE_OK;
  std::lock_guard<std::mutex> lock(g_dev_mutex);      // (the attribute is the last one set: it only grows)
  if (allowed[dev].load(std::memory_order_relaxed) >= smem) return PE_OK;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) { cudaGetLastError(); return PE_ERR_CUDA; }
  allowed[dev].store(smem, std::memory_order_release);
  return PE_OK;
}

// ---------------------------------------------------------------- forward
struct ForwardPlan {
  int G, nv, threads;      // threads per row, vectors per thread, threads per block; G = 0: the kernel for rows of any width
};
// A power of two of lanes per row while one vector each covers it, then a warp with up to 8 vectors each, then several warps.
static ForwardPlan plan_forward(int d, int E) {
  const int vectors = (d - 1) / E + 1;
  ForwardPlan p = {32, 1, 256};
  if (vectors <= 32) {
    p.G = 1;
    while (p.G < vectors) p.G *= 2;
  } else if (vectors <= 256) {
    while (p.nv * 32 < vectors) p.nv *= 2;
  } else if (vectors <= 4096) {
    p.nv = vectors <= 1024 ? 4 : 8;
    p.G = (vectors + 32 * p.nv - 1) / (32 * p.nv) * 32;
  } else {
    p.G = 0;
    p.threads = NORM_WIDE_THREADS;
    return p;
  }
  p.threads = p.G * std::max(1, 256 / p.G);
  return p;
}

// Threads to a row where each has 8 of its features: a power of two up to a warp, whole warps above.
static int row_threads(int d) {
  const int threads = (d - 1) / NORM_COLS + 1;
  if (threads > 32) return (threads + 31) / 32 * 32;
  int G = 1;
  while (G < threads) G *= 2;
  return G;
}

template <typename T, int E, bool RMS>
static pe_status_t launch_forward(DeviceInfo* di, const T* x, const float* gain, const float* bias, long long rows, int d, float eps, T* y,
                                  float* mean, float* rstd, cudaStream_t st) {
  const int wide = aligned(gain, 16) && aligned(bias, 16), ring_G = row_threads(d);
  // The ring where gain and bias out of L1 would hold rows up (16-bit rows of 1024 features or more: 256 x 1024 x 2048, 400 us against 563; 64 x 256 x 512, 11.4 and
  // 11.2) or single features would (256 x 256 x 333, 52 and 128); fp32 rows go faster without (64 x 256 x 1024, 26.7 and 23.6), and so do few rows
  // (8 x 256 x 1024, 7.0 and 5.8).
  if constexpr (E == 1 || sizeof(T) == 2) {
    if (ring_G <= NORM_MAX_THREADS && rows * d >= (1ll << 22) && (E == 1 || d >= 1024)) {
      const int groups = std::max(1, 256 / ring_G), threads = ring_G * groups, smem = (int)(groups * NORM_STAGES * (norm_slot_bytes(norm_rows<T>(), d, sizeof(T), true) + 8));
      const long long most = (long long)di->sm_count * std::max(1, std::min((E == 1 ? 512 : 1024) / threads, 220 * 1024 / (smem + 4096)));
      const long long blocks = std::max(1ll, std::min(most, rows / (2ll * norm_rows<T>() * groups)));      // two turns at least
      auto kernel = norm_forward_ring_kernel<T, E, RMS>;
      static std::atomic<int> allowed[MAX_DEVICES];
      const pe_status_t rc = allow_smem(kernel, allowed, smem);
      if (rc != PE_OK) return rc;
      return launch_dependent(kernel, dim3((unsigned)blocks), threads, smem, st, x, gain, bias, rows, d, eps, y, mean, rstd, ring_G, wide, di->status_ptr);
    }
  }
  const ForwardPlan p = plan_forward(d, E);
  if (p.G == 0)
    return launch_dependent(norm_forward_wide_kernel<T, RMS>, dim3((unsigned)std::min<long long>(rows, 2ll * di->sm_count)), p.threads, 0, st, x, gain,
                            bias, rows, d, eps, y, mean, rstd);
  const int groups = p.threads / p.G;
  const long long blocks = (rows + groups - 1) / groups;
  if (blocks >= (1ll << 31)) return PE_ERR_DIM;
  const dim3 grid((unsigned)blocks);
  auto run = [&](auto nv) {
    constexpr int NV = decltype(nv)::value;
    if (p.G <= 32) return launch_dependent(norm_forward_kernel<T, E, NV, RMS, true>, grid, p.threads, 0, st, x, gain, bias, rows, d, eps, y, mean, rstd, p.G, wide);
    return launch_dependent(norm_forward_kernel<T, E, NV, RMS, false>, grid, p.threads, 0, st, x, gain, bias, rows, d, eps, y, mean, rstd, p.G, wide);
  };
  switch (p.nv) {
    case 1: return run(std::integral_constant<int, 1>{});
    case 2: return run(std::integral_constant<int, 2>{});
    case 4: return run(std::integral_constant<int, 4>{});
    default: return run(std::integral_constant<int, 8>{});
  }
}

static bool norm_size_ok(long long rows, int d) { return rows >= 0 && d >= 1 && rows < (1ll << 40) && (rows == 0 || rows <= ((1ll << 40) - 1) / d); }
// (byte offsets of a turn's rows are 32 bits in the backward pass: three bf16 rows or one of fp32 before the last one)
constexpr int NORM_MAX_BACKWARD_D = 1 << 28;
static bool kind_ok(pe_norm_t kind) { return kind == PE_NORM_LAYER || kind == PE_NORM_RMS; }

template <typename T>
static pe_status_t forward_impl(const T* x, const float* gain, const float* bias, long long rows, int d, pe_norm_t kind, float eps, T* y, float* mean,
                                float* rstd, cudaStream_t st) {
  if (!norm_size_ok(rows, d) || d > NORM_MAX_FORWARD_D || !(eps >= 0.f)) return PE_ERR_DIM;
  if (!kind_ok(kind)) return PE_ERR_PHI;
  if (rows > 0 && (!x || !y)) return PE_ERR_NULL;
  const size_t al = sizeof(T) == 2 ? 16 : 4;
  if (!aligned(x, al) || !aligned(y, al) || !aligned(gain, 4) || !aligned(bias, 4) || !aligned(mean, 4) || !aligned(rstd, 4)) return PE_ERR_ALIGN;
  DeviceInfo* di = nullptr;
  const pe_status_t rc = device_info(&di);
  if (rc != PE_OK) return rc;
  if (rows == 0) return PE_OK;
  constexpr int E = 16 / (int)sizeof(T);
  const bool rms = kind == PE_NORM_RMS;
  if (d % E == 0 && aligned(x, 16) && aligned(y, 16))
    return rms ? launch_forward<T, E, true>(di, x, gain, bias, rows, d, eps, y, mean, rstd, st)
               : launch_forward<T, E, false>(di, x, gain, bias, rows, d, eps, y, mean, rstd, st);
  return rms ? launch_forward<T, 1, true>(di, x, gain, bias, rows, d, eps, y, mean, rstd, st)
             : launch_forward<T, 1, false>(di, x, gain, bias, rows, d, eps, y, mean, rstd, st);
}

// ---------------------------------------------------------------- backward
constexpr int NORM_SLAB_THREADS = 256;       // a block of the two-pass kernel: 2048 features
constexpr int NORM_SM_COUNT = 148;           // the workspace is sized for launches of at most this many SMs
struct BackwardPlan {
  int mode;                                  // NORM_WHOLE up to 4096 features, NORM_CLUSTER up to 32768, NORM_SLAB
  int G, groups, blocks, slabs;              // threads per row (of a slice), rows at a time, blocks along the rows, slices
  bool kept;                                 // room for sums over long examples beside the heads: not for narrow rows, whose workers are many
  size_t ends_at, heads_at, means_at, bytes; // workspace: elements, their flags, heads, the rows' means
};
static BackwardPlan plan_backward(long long rows, int d, int kinds, int sm_count) {
  BackwardPlan p = {};
  sm_count = std::min(sm_count, NORM_SM_COUNT);
  p.G = row_threads(d);
  p.slabs = 1;
  if (p.G > NORM_MAX_THREADS) {
    p.slabs = (p.G + NORM_MAX_THREADS - 1) / NORM_MAX_THREADS;
    p.mode = NORM_CLUSTER;
    p.G = row_threads((d + p.slabs - 1) / p.slabs);
    if (p.slabs > NORM_MAX_CLUSTER) {
      p.mode = NORM_SLAB;
      p.G = NORM_SLAB_THREADS;
      p.slabs = (d + NORM_COLS * p.G - 1) / (NORM_COLS * p.G);
    }
  }
  // A block of 512 threads to an SM leaves half as many elements to join as two of 256 (512 x 16 x 1536, 45 us and 36; 2048 features, 537 M values, 571 and 557); rows of
  // fewer than 64 threads would need more shared memory than there is.
  p.groups = std::max(1, (p.mode == NORM_WHOLE && p.G >= 64 ? NORM_MAX_THREADS : 256) / p.G);
  p.kept = p.mode == NORM_CLUSTER || (p.mode == NORM_WHOLE && p.G >= 64);
  const long long want = std::max(1ll, rows / (8ll * p.groups));      // at least eight rows to a worker
  const long long most = p.mode == NORM_WHOLE ? sm_count * std::max(1, 512 / (p.G * p.groups)) : std::max(1, (p.mode == NORM_SLAB ? 2 : 1) * sm_count / p.slabs);
  p.blocks = (int)std::min(want, most);
  p.ends_at = align_up((size_t)p.blocks * NORM_PARTS * kinds * d * sizeof(float), 256);
  p.heads_at = p.ends_at + align_up((size_t)p.blocks * (p.mode == NORM_CLUSTER ? p.slabs : 1) * sizeof(int), 256);
  p.means_at = p.heads_at + align_up((size_t)p.blocks * p.slabs * (p.kept ? 3 : 1) * kinds * NORM_COLS * p.G * p.groups * sizeof(float), 256);
  p.bytes = p.means_at + (p.mode == NORM_SLAB ? align_up((size_t)rows * sizeof(float2), 256) : 0);
  return p;
}

template <typename T, int E, bool RMS, int KINDS, int MODE, bool SHORT>
static pe_status_t launch_rows(const T* x, const T* dy, T* dx, const NormBackward& a, const BackwardPlan& p, int smem, cudaStream_t st) {
  auto kernel = norm_backward_kernel<T, E, RMS, KINDS, MODE, SHORT>;
  static std::atomic<int> allowed[MAX_DEVICES];
  const pe_status_t rc = allow_smem(kernel, allowed, smem);
  return rc != PE_OK ? rc : launch_dependent(kernel, MODE == NORM_SLAB ? dim3(p.slabs, p.blocks) : dim3(p.blocks), p.G * p.groups, smem, st, x, dy, dx, a);
}
template <typename T, int E, bool RMS, int KINDS, bool SHORT>
static pe_status_t launch_cluster(const T* x, const T* dy, T* dx, NormBackward& a, BackwardPlan& p, int smem, cudaStream_t st) {
  auto kernel = norm_backward_kernel<T, E, RMS, KINDS, NORM_CLUSTER, SHORT>;
  static std::atomic<int> allowed[MAX_DEVICES];
  const pe_status_t rc = allow_smem(kernel, allowed, smem);
  if (rc != PE_OK) return rc;
  a.cluster = p.slabs;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(p.G); cfg.dynamicSmemBytes = (size_t)smem; cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.slabs; attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return PE_ERR_CUDA; }
  // clusters of this size that the device runs at a time (0: not asked yet); more would wait for a second round
  static std::atomic<int> clusters[MAX_DEVICES][NORM_MAX_CLUSTER + 1];
  int most = clusters[dev][p.slabs].load();
  if (most == 0) {
    cfg.numAttrs = 1;
    cfg.gridDim = dim3((unsigned)(p.slabs * p.blocks));
    if (cudaOccupancyMaxActiveClusters(&most, kernel, &cfg) != cudaSuccess || most < 1) { cudaGetLastError(); return PE_ERR_CUDA; }
    clusters[dev][p.slabs].store(most);
  }
  p.blocks = std::min(p.blocks, most);
  cfg.numAttrs = 2;
  cfg.gridDim = dim3((unsigned)(p.slabs * p.blocks));
  if (cudaLaunchKernelEx(&cfg, kernel, x, dy, dx, a) != cudaSuccess) { cudaGetLastError(); return PE_ERR_CUDA; }
  return check_launch();
}
template <typename T, int E, bool RMS, int KINDS>
static pe_status_t launch_backward(DeviceInfo* di, const T* x, const T* dy, T* dx, NormBackward& a, BackwardPlan& p, char* ws, cudaStream_t st) {
  const int threads = p.G * p.groups;
  // the ring, in the same place later the workers' elements, and the barriers
  const size_t slot = norm_slot_bytes(norm_rows<T>(), p.mode == NORM_WHOLE ? a.d : p.G * NORM_COLS, sizeof(T), p.mode == NORM_WHOLE);
  a.bars_at = (uint32_t)std::max((size_t)p.groups * NORM_STAGES * 2 * slot, (size_t)threads * NORM_PARTS * KINDS * NORM_COLS * sizeof(float));
  const int smem = (int)a.bars_at + p.groups * NORM_STAGES * 8;
  a.G = p.G;
  a.parts = reinterpret_cast<float*>(ws);
  a.ends = reinterpret_cast<int*>(ws + p.ends_at);
  a.heads = reinterpret_cast<float*>(ws + p.heads_at);
  a.dev_status = di->status_ptr;
  a.row_means = reinterpret_cast<const float2*>(ws + p.means_at);
  if (p.mode == NORM_WHOLE)
    return a.rows < 32ll * a.B || !p.kept ? launch_rows<T, E, RMS, KINDS, NORM_WHOLE, true>(x, dy, dx, a, p, smem, st)
                                          : launch_rows<T, E, RMS, KINDS, NORM_WHOLE, false>(x, dy, dx, a, p, smem, st);
  if (p.mode == NORM_CLUSTER)
    return a.rows < 32ll * a.B ? launch_cluster<T, E, RMS, KINDS, true>(x, dy, dx, a, p, smem, st) : launch_cluster<T, E, RMS, KINDS, false>(x, dy, dx, a, p, smem, st);
  const pe_status_t rc = launch_dependent(norm_row_means_kernel<T, RMS>, dim3((unsigned)std::min<long long>(a.rows, 2ll * di->sm_count)), 1024, 0, st, x, dy,
                                          a, reinterpret_cast<float2*>(ws + p.means_at), p.blocks);
  if (rc != PE_OK) return rc;
  return launch_rows<T, E, RMS, KINDS, NORM_SLAB, true>(x, dy, dx, a, p, smem, st);
}

template <typename T>
static pe_status_t backward_impl(const T* x, const T* dy, const float* gain, const float* mean, const float* rstd, const int* offsets, bool packed, int B,
                                 int T_, long long rows, int d, pe_norm_t kind, pe_phi_t phi, int accumulate, T* dx, float* gain_sum, float* gain_stat,
                                 float* bias_sum, float* bias_stat, void* workspace, size_t workspace_bytes, cudaStream_t st) {
  if (B < 0 || T_ < 0 || !norm_size_ok(rows, d) || d > NORM_MAX_BACKWARD_D || (packed && rows >= (1ll << 31))) return PE_ERR_DIM;
  if (!kind_ok(kind) || (phi != PE_PHI_IDENTITY && phi != PE_PHI_SQUARE && phi != PE_PHI_SIGN)) return PE_ERR_PHI;
  const bool empty = B == 0 || rows == 0;
  if (!empty && (!x || !dy || !rstd || (kind == PE_NORM_LAYER && !mean) || (packed && !offsets))) return PE_ERR_NULL;
  if (!dx && !gain_sum && !gain_stat && !bias_sum && !bias_stat) return PE_ERR_NULL;
  const size_t al = sizeof(T) == 2 ? 16 : 4;
  if (!aligned(x, al) || !aligned(dy, al) || !aligned(dx, al)) return PE_ERR_ALIGN;
  for (const void* q : {(const void*)gain, (const void*)mean, (const void*)rstd, (const void*)offsets, (const void*)gain_sum, (const void*)gain_stat,
                        (const void*)bias_sum, (const void*)bias_stat})
    if (!aligned(q, 4)) return PE_ERR_ALIGN;
  DeviceInfo* di = nullptr;
  pe_status_t rc = device_info(&di);
  if (rc != PE_OK) return rc;
  if (empty) {
    if (!accumulate)
      for (float* q : {gain_sum, gain_stat, bias_sum, bias_stat})
        if (q && cudaMemsetAsync(q, 0, (size_t)d * sizeof(float), st) != cudaSuccess) { cudaGetLastError(); return PE_ERR_CUDA; }
    return PE_OK;
  }
  const bool bias = bias_sum || bias_stat, rms = kind == PE_NORM_RMS;
  const int kinds = bias ? 2 : 1;
  BackwardPlan p = plan_backward(rows, d, kinds, di->sm_count);
  if (!workspace || workspace_bytes < p.bytes) return PE_ERR_WORKSPACE;
  if (!aligned(workspace, 256)) return PE_ERR_ALIGN;
  NormBackward a = {};
  a.gain = gain; a.mean = mean; a.rstd = rstd; a.offsets = packed ? offsets : nullptr;
  a.wide = aligned(gain, 16); a.rows = rows; a.B = B; a.T = T_; a.d = d; a.phi = (int)phi; a.accumulate = accumulate;
  a.sums[0] = gain_sum; a.sums[1] = gain_stat; a.sums[2] = bias_sum; a.sums[3] = bias_stat;
  constexpr int E = 16 / (int)sizeof(T);
  char* ws = static_cast<char*>(workspace);
  const bool vec = d % E == 0 && aligned(x, 16) && aligned(dy, 16) && aligned(dx, 16);
  auto with = [&](auto e) {
    constexpr int EE = decltype(e)::value;
    if (rms) return bias ? launch_backward<T, EE, true, 2>(di, x, dy, dx, a, p, ws, st) : launch_backward<T, EE, true, 1>(di, x, dy, dx, a, p, ws, st);
    return bias ? launch_backward<T, EE, false, 2>(di, x, dy, dx, a, p, ws, st) : launch_backward<T, EE, false, 1>(di, x, dy, dx, a, p, ws, st);
  };
  rc = vec ? with(std::integral_constant<int, E>{}) : with(std::integral_constant<int, 1>{});
  if (rc != PE_OK || (!bias && !gain_sum && !gain_stat)) return rc;
  if (p.mode == NORM_WHOLE && p.blocks == 1) return PE_OK;      // (the one block has written them)
  const dim3 grid((unsigned)(kinds * ((d + 31) / 32)));
  return bias ? launch_dependent(norm_join_kernel<2>, grid, 32 * NORM_JOIN_WARPS, 0, st, a, p.blocks)
              : launch_dependent(norm_join_kernel<1>, grid, 32 * NORM_JOIN_WARPS, 0, st, a, p.blocks);
}

pe_status_t norm_set_wait_limit(long long cycles) {
  if (cudaMemcpyToSymbol(sm100::g_wait_cycle_limit, &cycles, sizeof cycles) != cudaSuccess) { cudaGetLastError(); return PE_ERR_CUDA; }
  return PE_OK;
}

}  // namespace pe

using namespace pe;

extern "C" {

pe_status_t pe_norm_forward(const void* x, const float* gain, const float* bias, long long rows, int d, pe_norm_t kind, float eps, void* y, float* mean,
                            float* rstd, pe_stream_t stream) {
  return forward_impl(static_cast<const __nv_bfloat16*>(x), gain, bias, rows, d, kind, eps, static_cast<__nv_bfloat16*>(y), mean, rstd,
                      reinterpret_cast<cudaStream_t>(stream));
}
pe_status_t pe_norm_forward_f32(const float* x, const float* gain, const float* bias, long long rows, int d, pe_norm_t kind, float eps, float* y, float* mean,
                                float* rstd, pe_stream_t stream) {
  return forward_impl(x, gain, bias, rows, d, kind, eps, y, mean, rstd, reinterpret_cast<cudaStream_t>(stream));
}

size_t pe_norm_backward_workspace_bytes(long long rows, int d) {
  if (!norm_size_ok(rows, d) || d > NORM_MAX_BACKWARD_D || rows == 0) return 0;
  return plan_backward(rows, d, 2, NORM_SM_COUNT).bytes;
}

pe_status_t pe_norm_backward(const void* x, const void* dy, const float* gain, const float* mean, const float* rstd, int B, int T, int d, pe_norm_t kind,
                             pe_phi_t phi, int accumulate, void* dx, float* gain_sum, float* gain_stat, float* bias_sum, float* bias_stat, void* workspace,
                             size_t workspace_bytes, pe_stream_t stream) {
  return backward_impl(static_cast<const __nv_bfloat16*>(x), static_cast<const __nv_bfloat16*>(dy), gain, mean, rstd, nullptr, false, B, T,
                       (long long)B * T, d, kind, phi, accumulate, static_cast<__nv_bfloat16*>(dx), gain_sum, gain_stat, bias_sum, bias_stat, workspace,
                       workspace_bytes, reinterpret_cast<cudaStream_t>(stream));
}
pe_status_t pe_norm_backward_f32(const float* x, const float* dy, const float* gain, const float* mean, const float* rstd, int B, int T, int d,
                                 pe_norm_t kind, pe_phi_t phi, int accumulate, float* dx, float* gain_sum, float* gain_stat, float* bias_sum,
                                 float* bias_stat, void* workspace, size_t workspace_bytes, pe_stream_t stream) {
  return backward_impl(x, dy, gain, mean, rstd, nullptr, false, B, T, (long long)B * T, d, kind, phi, accumulate, dx, gain_sum, gain_stat, bias_sum,
                       bias_stat, workspace, workspace_bytes, reinterpret_cast<cudaStream_t>(stream));
}
pe_status_t pe_norm_backward_ragged(const void* x, const void* dy, const float* gain, const float* mean, const float* rstd, const int* seq_offsets, int B,
                                    long long total_rows, int d, pe_norm_t kind, pe_phi_t phi, int accumulate, void* dx, float* gain_sum,
                                    float* gain_stat, float* bias_sum, float* bias_stat, void* workspace, size_t workspace_bytes, pe_stream_t stream) {
  return backward_impl(static_cast<const __nv_bfloat16*>(x), static_cast<const __nv_bfloat16*>(dy), gain, mean, rstd, seq_offsets, true, B, 1, total_rows, d,
                       kind, phi, accumulate, static_cast<__nv_bfloat16*>(dx), gain_sum, gain_stat, bias_sum, bias_stat, workspace, workspace_bytes,
                       reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
