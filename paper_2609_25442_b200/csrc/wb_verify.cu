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

#include <cmath>

#include "wb_verify.cuh"

namespace cg = cooperative_groups;
using namespace wbi;

namespace {

// w = p, or max(p - q, 0) where there is a q; index `skip` has none.  Rows that start on 16-byte boundaries are read eight
// elements at a time; others element by element, six in flight (192 rows of 128255: 59 us,
// with four or eight 67 and 64; of 128256: 44).
template <typename T, bool SUB, uint32_t kVerifyThreads>
__device__ __forceinline__ Best race_range(const T* p, const T* q, const float* e, uint32_t v0, uint32_t v1, uint32_t skip) {
  Best best;
  uint32_t v = v0;
  if ((((uintptr_t)(p + v0) | (uintptr_t)(e + v0) | (SUB ? (uintptr_t)(q + v0) : 0)) & 15u) == 0) {
    const uint32_t whole = v0 + (v1 - v0) / 8 * 8;
    for (v = v0 + threadIdx.x * 8; v < whole; v += kVerifyThreads * 8) {
      float x[8], y[8], z[8];
      load8(p + v, x);
      load8(e + v, z);
      if (SUB) load8(q + v, y);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float w = SUB ? x[i] - y[i] : x[i];
        if (v + i == skip) w = 0.f;
        best.offer(w, z[i], v + i);
      }
    }
    v = whole;
  }
  for (v += threadIdx.x; v < v1; v += 6 * kVerifyThreads) {
    float x[6], y[6], z[6];
#pragma unroll
    for (int i = 0; i < 6; ++i) {
      const uint32_t at = min(v + i * kVerifyThreads, v1 - 1);
      x[i] = prob(p, at);
      z[i] = __ldg(e + at);
      if (SUB) y[i] = prob(q, at);
    }
#pragma unroll
    for (int i = 0; i < 6; ++i) {
      const uint32_t at = v + i * kVerifyThreads;
      float w = SUB ? x[i] - y[i] : x[i];
      if (at >= v1 || at == skip) w = 0.f;
      best.offer(w, z[i], at);
    }
  }
  return best;
}

template <typename T, uint32_t kVerifyThreads>
__global__ void __launch_bounds__(kVerifyThreads, 1024 / kVerifyThreads) wb_verify_kernel(wb_verify_args a) {
  cg::cluster_group cluster = cg::this_cluster();
  const uint32_t rank = cluster.block_rank(), size = cluster.num_blocks(), s = blockIdx.x / size;
  __shared__ uint64_t warp_best[kVerifyThreads / 32];
  __shared__ uint64_t block_best;
  __shared__ int s_accepted;
  const int32_t start = min(max(__ldg(a.draft_start + s), 0), (int32_t)a.n_drafts);
  const int32_t count = min(min(max(__ldg(a.draft_start + s + 1), start), (int32_t)a.n_drafts) - start, (int32_t)a.max_drafts);
  const T* target = reinterpret_cast<const T*>(a.target) + (uint64_t)(start + (int32_t)s) * a.target_stride;
  const T* draft = a.draft ? reinterpret_cast<const T*>(a.draft) + (uint64_t)start * a.draft_stride : nullptr;
  const float* e = a.race + (uint64_t)s * a.race_stride;
  const uint32_t share = ((a.vocab + size - 1) / size + 7) / 8 * 8, v0 = min(rank * share, a.vocab), v1 = min(v0 + share, a.vocab);
  // the race is needed whatever is accepted: it comes into the second-level cache while that is found out
  for (uint32_t v = v0 + threadIdx.x * 32; v < v1; v += kVerifyThreads * 32) asm volatile("prefetch.global.L2 [%0];" ::"l"(e + v));
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
  int mode = !rejected ? 0 : q ? 1 : 2;      // w = p; max(p - q, 0); p except for index `skip`
  uint64_t best;
  for (;;) {
    best = mode == 1 ? race_range<T, true, kVerifyThreads>(p, q, e, v0, v1, 0xFFFFFFFFu).key : race_range<T, false, kVerifyThreads>(p, nullptr, e, v0, v1, mode == 2 ? skip : 0xFFFFFFFFu).key;
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

template <typename T, uint32_t kVerifyThreads>
wb_status launch_verify(const wb_verify_args& a, uint32_t size, cudaStream_t stream) {
  cudaLaunchAttribute at[1];
  const cudaLaunchConfig_t cfg = config_of(a.n_seqs, kVerifyThreads, size, at, stream);
  if (cudaLaunchKernelEx(&cfg, wb_verify_kernel<T, kVerifyThreads>, a) != cudaSuccess) { (void)cudaGetLastError(); return WB_ERR_CUDA; }
  return WB_OK;
}

// A sequence gets as many blocks as let all sequences run at once: 16 of 512 threads (not a portable cluster size, but every
// B200's), 8 of 512, then 8 to 1 of 256.  One size too large and a second wave of clusters waits for the first; both sides, bf16
// rows of 128256: 14 | 15 sequences with 16 x 512 take 16.4 | 20.5 us, the latter with 8 x 512 16.4; 32 | 36 with 8 x 512 18.5 | 26.6, the latter
// with 8 x 256 22.5; 68 | 72 with 8 25.5 | 34.8, with 7 26.6 | 26.6; 75 | 84 with 7 28.7 | 38.9, with 6 28.7 | 30.7; 90 | 98 with 6 30.7 | 44.0, with 5
// 32.8 | 32.8; 110 | 118 with 5 33.1 | 49.2, with 4 35.8 | 36.9; 130 | 148 with 4 37.8 | 54.2, with 3 41.0 | 42.0; 180 | 192 with 3 45.1 | 65.5, with 2
// 53.2 | 53.2.  (Each with the drafts' and the race's rows out of the caches.)
template <typename T> wb_status launch_verify_of(const wb_verify_args& a, cudaStream_t stream) {
  static ClusterCounts known[2];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { (void)cudaGetLastError(); return WB_ERR_CUDA; }
  for (uint32_t size : {16u, 8u})
    if (a.n_seqs <= resident_clusters(wb_verify_kernel<T, 512>, 512, dev, size, known[0])) return launch_verify<T, 512>(a, size, stream);
  for (uint32_t size = 8; size > 1; --size)
    if (a.n_seqs <= resident_clusters(wb_verify_kernel<T, 256>, 256, dev, size, known[1])) return launch_verify<T, 256>(a, size, stream);
  return launch_verify<T, 256>(a, 1, stream);
}

}  // namespace

extern "C" wb_status wb_verify_drafts(const wb_verify_args* args, void* stream) {
  if (!args) return WB_ERR_INVALID_ARG;
  const wb_verify_args& a = *args;
  if (a.dtype != WB_F32 && a.dtype != WB_BF16) return WB_ERR_DTYPE;
  if (!a.vocab || a.vocab > 0x7FFFFFFFu || a.max_drafts > (1u << 20) || a.n_seqs > (1u << 24) || a.n_drafts > (1u << 30) ||
      a.reserved)
    return WB_ERR_INVALID_ARG;
  auto bad_pitch = [&](uint64_t pitch) { return pitch && pitch < a.vocab; };       // 0: one row for all
  if (bad_pitch(a.target_stride) || bad_pitch(a.race_stride) || (a.draft && bad_pitch(a.draft_stride))) return WB_ERR_INVALID_ARG;
  if (!a.n_seqs) return WB_OK;
  if (!a.target || !a.draft_start || !a.race || !a.accepted || !a.tokens) return WB_ERR_INVALID_ARG;
  if (a.n_drafts && (!a.draft_tokens || !a.uniform)) return WB_ERR_INVALID_ARG;
  const uint32_t e = a.dtype == WB_F32 ? 4 : 2;
  if (((uintptr_t)a.target | (uintptr_t)a.draft) % e || ((uintptr_t)a.race | (uintptr_t)a.uniform | (uintptr_t)a.draft_tokens |
      (uintptr_t)a.draft_start | (uintptr_t)a.accepted | (uintptr_t)a.tokens) % 4)
    return WB_ERR_INVALID_ARG;
  return a.dtype == WB_F32 ? launch_verify_of<float>(a, (cudaStream_t)stream) : launch_verify_of<uint16_t>(a, (cudaStream_t)stream);
}
