// What the verification kernels share: probabilities as they are read, and the race for the next token.
#pragma once
#include <atomic>

#include "wb_kv.cuh"

namespace wbi {

__device__ __forceinline__ float prob(const float* p, uint64_t i) { return __ldg(p + i); }
__device__ __forceinline__ float prob(const uint16_t* p, uint64_t i) { return __uint_as_float((uint32_t)__ldg(p + i) << 16); }
__device__ __forceinline__ uint64_t key_max(uint64_t a, uint64_t b) { return a > b ? a : b; }


// The best of a thread so far: its key (score bits above the complemented index; scores are not negative, so their bits order as
// they do, and a larger complement is a lower index), and the score itself.  A candidate whose weight is below the rounded product
// of that and its race variate is spared the division (all but about ln n of n are): the weight is then below the exact product
// too, because it is a number that the product could have been rounded to, so its quotient is at most the score, and an equal one
// of a later index does not win.  (A NaN product, of zero and infinity, spares nothing.)
struct Best {
  uint64_t key = 0;                     // below every key: no weight is positive
  float bar = 0.f;
  __device__ __forceinline__ void offer(float w, float e, uint32_t v) {
    if (!(w > 0.f) || w < bar * e) return;
    const float score = __fdiv_rn(w, e);
    if (!(score >= 0.f)) return;        // a NaN or negative race variate takes no part
    key = key_max(key, (uint64_t)__float_as_uint(score) << 32 | (uint32_t)~v);
    bar = fmaxf(bar, score);
  }
};

// Eight probabilities from a 16-byte boundary.
__device__ __forceinline__ void load8(const float* p, float* x) {
  const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load8(const uint16_t* p, float* x) {
  const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p));
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
}

inline cudaLaunchConfig_t config_of(uint32_t n_seqs, uint32_t threads, uint32_t size, cudaLaunchAttribute* at, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n_seqs * size);
  cfg.blockDim = dim3(threads);
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
template <typename K> uint32_t resident_clusters(K kernel, uint32_t threads, int dev, uint32_t size, ClusterCounts& known) {
  const bool keep = (uint32_t)dev < 64;
  if (const int32_t n = keep ? known.plus_one[dev][size].load(std::memory_order_acquire) : 0) return (uint32_t)(n - 1);
  cudaLaunchAttribute at[1];
  const cudaLaunchConfig_t cfg = config_of(1, threads, size, at, nullptr);
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
