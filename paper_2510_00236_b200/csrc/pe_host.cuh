// Host-side state and helpers shared by the translation units behind the C ABI.
#pragma once
#include <atomic>
#include <cstddef>
#include <cstdint>
#include <mutex>

#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/pestats.h"

namespace pe {

extern std::atomic<long long> g_launches;     // kernels launched since load

constexpr int MAX_DEVICES = 64;
struct DeviceInfo {
  std::atomic<int> state{0};     // 0 unknown, 1 ready, -1 failed
  int cc_major = 0, sm_count = 0;
  unsigned int* status_ptr = nullptr;
  bool tc_attr_set[64] = {};
  bool tok_attr_set = false;
};
extern std::mutex g_dev_mutex;      // guards the lazily filled per-device state (first calls from several host threads)

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                   const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                   CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

pe_status_t device_info(DeviceInfo** out);    // of the current device
EncodeTiledFn encode_fn();
// pe_set_wait_limit_cycles for the kernels of the other translation units (each has its own copy of the limit)
pe_status_t ns_set_wait_limit(long long cycles);
pe_status_t norm_set_wait_limit(long long cycles);
pe_status_t ns_plan_query(int product, int count, int rows, int cols, long long* plan);      // PE_PLAN_ORTHOGONALIZE

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

inline pe_status_t check_launch() {
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return PE_ERR_CUDA;
  g_launches.fetch_add(1);
  return PE_OK;
}

// Launches `kernel` as a programmatic dependent of the kernel before it in the stream (every kernel launched this way waits for
// that one to complete before it touches what others may have written: griddep_wait).
template <typename Kernel, typename... Args>
pe_status_t launch_dependent(Kernel kernel, dim3 grid, int threads, int smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid; cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = (size_t)smem; cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr; cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) { cudaGetLastError(); return PE_ERR_CUDA; }
  return check_launch();
}

}  // namespace pe
