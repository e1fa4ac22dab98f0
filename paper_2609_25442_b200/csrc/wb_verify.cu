// Verification of drafted tokens (speculative sampling with an exponential race).
//
// Per sequence: find the first rejected draft (a gather of one probability of each kind per drafted
// token), then one pass over that position's rows, keeping the largest w(v) / race(v) and its index.
// The bound is memory: one target row, one drafter row and one race row per sequence.
//
// A thread-block cluster serves a sequence: every block finds the first rejection for itself (the gather
// is a few loads, an exchange would cost as much), takes its share of the vocabulary, and the cluster's
// first block joins the shares over distributed shared memory.  The winner is the maximum of a 64-bit
// key (score bits above the complemented index), so it does not depend on the order of the joining.
#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>

#include "wb_kv.cuh"

namespace cg = cooperative_groups;
using namespace wbi;

namespace {

constexpr uint32_t kVerifyThreads = 512;

__device__ __forceinline__ float prob(const float* p, uint64_t i) { return __ldg(p + i); }
__device__ __forceinline__ float prob(const uint16_t* p, uint64_t i) { return __uint_as_float((uint32_t)__ldg(p + i) << 16); }

__device__ __forceinline__ uint64_t key_max(uint64_t a, uint64_t b) { return a > b ? a : b; }

// Scores are positive, so their bits order as they do; a larger complement is a lower index.
__device__ __forceinline__ uint64_t race_key(float w, float e, uint32_t v, uint64_t best) {
  if (!(w > 0.f)) return best;
  const float score = __fdiv_rn(w, e);
  if (!(score >= 0.f)) return best;     // a NaN or negative race variate takes no part
  return key_max(best, (uint64_t)__float_as_uint(score) << 32 | (uint32_t)~v);
}

// mode 0: w = p; 1: w = max(p - q, 0); 2: w = p except for index `skip`
template <typename T>
__device__ __forceinline__ uint64_t race_range(const T* p, const T* q, const float* e, uint32_t v0, uint32_t v1, uint32_t skip, int mode) {
  uint64_t best = 0;                    // below every key: no weight is positive
  for (uint32_t v = v0 + threadIdx.x; v < v1; v += kVerifyThreads) {
    float w = prob(p, v);
    if (mode == 1) w -= prob(q, v);
    if (mode == 2 && v == skip) w = 0.f;
    best = race_key(w, __ldg(e + v), v, best);
  }
  return best;
}

template <typename T>
__global__ void __launch_bounds__(kVerifyThreads) wb_verify_kernel(wb_verify_args a) {
  cg::cluster_group cluster = cg::this_cluster();
  const uint32_t rank = cluster.block_rank(), size = cluster.num_blocks(), s = blockIdx.x / size;
  __shared__ uint64_t warp_best[kVerifyThreads / 32];
  __shared__ uint64_t block_best;
  __shared__ int s_accepted;
  const int32_t start = min(max(__ldg(a.draft_start + s), 0), (int32_t)a.n_drafts);
  const int32_t count = min(min(max(__ldg(a.draft_start + s + 1), start), (int32_t)a.n_drafts) - start, (int32_t)a.max_drafts);
  const T* target = reinterpret_cast<const T*>(a.target) + (uint64_t)(start + (int32_t)s) * a.target_stride;
  const T* draft = a.draft ? reinterpret_cast<const T*>(a.draft) + (uint64_t)start * a.draft_stride : nullptr;
  if (threadIdx.x < 32) {
    int accepted = 0;
    for (int i0 = 0; i0 < count; i0 += 32) {
      const int i = i0 + (int)threadIdx.x;
      bool ok = false;
      if (i < count) {
        const uint32_t x = (uint32_t)__ldg(a.draft_tokens + start + i);
        if (x < a.vocab) {
          const float p = prob(target, (uint64_t)i * a.target_stride + x);
          const float q = draft ? prob(draft, (uint64_t)i * a.draft_stride + x) : 1.f;
          ok = __fmul_rn(__ldg(a.uniform + start + i), q) < p;
        }
      }
      const uint32_t fail = ~__ballot_sync(0xFFFFFFFFu, ok);
      if (fail) { accepted = i0 + __ffs(fail) - 1; break; }
      accepted = i0 + 32;
    }
    if (threadIdx.x == 0) s_accepted = accepted;
  }
  __syncthreads();
  const int accepted = s_accepted;
  const bool rejected = accepted < count;
  const T* p = target + (uint64_t)accepted * a.target_stride;
  const T* q = rejected && draft ? draft + (uint64_t)accepted * a.draft_stride : nullptr;
  const uint32_t skip = rejected && !draft ? (uint32_t)__ldg(a.draft_tokens + start + accepted) : 0xFFFFFFFFu;
  const float* e = a.race + (uint64_t)s * a.race_stride;
  const uint32_t share = (a.vocab + size - 1) / size, v0 = min(rank * share, a.vocab), v1 = min(v0 + share, a.vocab);
  int mode = !rejected ? 0 : q ? 1 : 2;
  uint64_t best;
  for (;;) {
    best = race_range<T>(p, q, e, v0, v1, skip, mode);
#pragma unroll
    for (int d = 16; d; d >>= 1) best = key_max(best, __shfl_xor_sync(0xFFFFFFFFu, best, d));
    if ((threadIdx.x & 31) == 0) warp_best[threadIdx.x >> 5] = best;
    __syncthreads();
    if (threadIdx.x < 32) {
      best = threadIdx.x < kVerifyThreads / 32 ? warp_best[threadIdx.x] : 0;
#pragma unroll
      for (int d = 16; d; d >>= 1) best = key_max(best, __shfl_xor_sync(0xFFFFFFFFu, best, d));
      if (threadIdx.x == 0) block_best = best;
    }
    cluster.sync();
    // every block reads all shares: all of them have to know whether any weight was positive
    best = 0;
    for (uint32_t r = 0; r < size; ++r) best = key_max(best, *cluster.map_shared_rank(&block_best, r));
    cluster.sync();                      // block_best may be overwritten or its block may end
    if (best || mode == 0) break;
    mode = 0;                            // nothing positive was left: draw from the target's row itself
  }
  if (rank == 0) {
    if (threadIdx.x == 0) a.accepted[s] = accepted;
    int32_t* tokens = a.tokens + (uint64_t)s * (a.max_drafts + 1);
    for (int i = (int)threadIdx.x; i <= (int)a.max_drafts; i += kVerifyThreads)
      tokens[i] = i < accepted ? __ldg(a.draft_tokens + start + i) : i == accepted ? (best ? (int32_t)~(uint32_t)best : 0) : -1;
  }
}

template <typename T>
wb_status launch_verify(const wb_verify_args& a, cudaStream_t stream) {
  const uint32_t size = 8;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.n_seqs * size);
  cfg.blockDim = dim3(kVerifyThreads);
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = size;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, wb_verify_kernel<T>, a) != cudaSuccess) { (void)cudaGetLastError(); return WB_ERR_CUDA; }
  return WB_OK;
}

}  // namespace

extern "C" wb_status wb_verify_drafts(const wb_verify_args* args, void* stream) {
  if (!args) return WB_ERR_INVALID_ARG;
  const wb_verify_args& a = *args;
  if (a.dtype != WB_F32 && a.dtype != WB_BF16) return WB_ERR_DTYPE;
  if (!a.vocab || a.vocab > 0x7FFFFFFFu || a.max_drafts > (1u << 20) || a.n_seqs > (1u << 24) || a.n_drafts > (1u << 30) ||
      a.reserved)
    return WB_ERR_INVALID_ARG;
  if (a.target_stride < a.vocab || a.race_stride < a.vocab || (a.draft && a.draft_stride < a.vocab)) return WB_ERR_INVALID_ARG;
  if (!a.n_seqs) return WB_OK;
  if (!a.target || !a.draft_start || !a.race || !a.accepted || !a.tokens) return WB_ERR_INVALID_ARG;
  if (a.n_drafts && (!a.draft_tokens || !a.uniform)) return WB_ERR_INVALID_ARG;
  const uint32_t e = a.dtype == WB_F32 ? 4 : 2;
  if (((uintptr_t)a.target | (uintptr_t)a.draft) % e || ((uintptr_t)a.race | (uintptr_t)a.uniform | (uintptr_t)a.draft_tokens |
      (uintptr_t)a.draft_start | (uintptr_t)a.accepted | (uintptr_t)a.tokens) % 4)
    return WB_ERR_INVALID_ARG;
  return a.dtype == WB_F32 ? launch_verify<float>(a, (cudaStream_t)stream) : launch_verify<uint16_t>(a, (cudaStream_t)stream);
}
