// Launches of thread-block clusters: their configuration, and how many fit on the device.
#pragma once
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

namespace wbi {

inline cudaLaunchConfig_t config_of(uint32_t n_clusters, uint32_t threads, uint32_t size, cudaLaunchAttribute* at, cudaStream_t stream, size_t smem = 0) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n_clusters * size);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  at->id = cudaLaunchAttributeClusterDimension;
  at->val.clusterDim.x = size;
  at->val.clusterDim.y = at->val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cfg;
}

// How many clusters of `size` blocks fit on the device at once: fewer than its places for blocks divided by size, because a
// cluster lies within one group of SMs.  Asked for once per kernel, which `known` belongs to.
struct ClusterCounts {
  std::atomic<int32_t> plus_one[64][17];
};
template <typename K> uint32_t resident_clusters(K kernel, uint32_t threads, int dev, uint32_t size, ClusterCounts& known, size_t smem = 0) {
  const bool keep = (uint32_t)dev < 64;
  if (const int32_t n = keep ? known.plus_one[dev][size].load(std::memory_order_acquire) : 0) return (uint32_t)(n - 1);
  cudaLaunchAttribute at[1];
  const cudaLaunchConfig_t cfg = config_of(1, threads, size, at, nullptr, smem);
  int n = 0;
  if ((size > 8 && cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) ||
      cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
    (void)cudaGetLastError();
    n = 0;
  }
  if (keep) known.plus_one[dev][size].store(n + 1, std::memory_order_release);
  return (uint32_t)n;
}

}  // namespace wbi
