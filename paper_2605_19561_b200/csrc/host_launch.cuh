// What the library's translation units share on the host: the launch of a kernel with its count, alignment checks, the current device.
#pragma once
#include <cuda_runtime.h>
#include <atomic>
#include "../../include/torq.h"

namespace torq {

extern std::atomic<int64_t> g_launches;

// SMs and error word of the current device; TORQ_ERR_LAUNCH or TORQ_ERR_ARCH where there is none that the library runs on.
torq_status current_device(int* sm_count, int** err_word);

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline torq_status launch_status() {
  g_launches.fetch_add(1, std::memory_order_relaxed);
  return cudaGetLastError() == cudaSuccess ? TORQ_OK : TORQ_ERR_LAUNCH;
}

// Launch of a kernel: `cluster` CTAs per cluster along x (1 or 2; the grid
// is a multiple of it) and programmatic stream serialization, so that the launch processing of
// this kernel overlaps the tail of the kernel before it (the kernel itself waits for that kernel
// to complete before it touches global memory).
template <typename... KArgs, typename... Args>
void launch_tc(void (*kernel)(KArgs...), int cluster, dim3 grid, dim3 threads, int smem, cudaStream_t s, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = threads;
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

}  // namespace torq
