// Verification of a tree of drafted tokens: a path from the root is accepted child by child, and one more token is drawn by an
// exponential race from what the rejected children have left of the target's distribution.
//
// Per sequence a gather of one probability of each kind per row, then one pass over the rows of the vocabulary where the path
// ends.  If the drafter sampled, a rejected child that has a sibling behind it costs a pass more: the sibling's chance is relative to
// the sum of what is left.  The bound is memory: one target row, one drafter row and one race row per sequence.
//
// A thread-block cluster serves a sequence.  Every block walks the tree by itself, one warp over the gathered values in shared memory
// (an exchange per step would cost more), so all of them come to the same passes, of which each takes its share; sums
// are joined in the blocks' order in 64 bits, the race by the maximum of a 64-bit key.
//
// One tree of 60 rows, certain drafter, 151936 fp32: 14.4 to 16.4 us on the device.  48 sampled trees of up to 24 rows, 128256 bf16: 34 to 35 us, of which the
// rows of the last pass are 7.5; the trees with the most rejected siblings make the most passes, 3 us each, and the others wait for
// them.  (62 us with what is left formed element by element over the siblings, a loop of ten instructions each.)
#include <cooperative_groups.h>

#include <cmath>

#include "wb_verify.cuh"

namespace cg = cooperative_groups;
using namespace wbi;

namespace {

constexpr uint32_t kRows = 512;        // rows of a tree whose values are gathered before the walk
constexpr uint32_t kKids = 256;        // children of a row that are looked at

// What the rejected children have left of an element: each took away the drafter's distribution times the sum before it.
__device__ __forceinline__ float left_of(float p, float q, const float* mass, uint32_t n) {
  for (uint32_t j = 0; j < n; ++j) p = fmaxf(__fsub_rn(p, __fmul_rn(mass[j], q)), 0.f);
  return p;
}

// A share [v0, v1) of the rows: the race over what is left (RACE), or its sum.  Without drafter rows the `n` tokens of `gone` are
// left out; they are looked up only for candidates that would win, which are few.
template <typename T, bool SUB, bool RACE, uint32_t THREADS>
__device__ __forceinline__ void tree_range(const T* p, const T* q, const float* e, uint32_t v0, uint32_t v1, const float* mass, const int32_t* gone,
                                           uint32_t n, Best& best, double& sum) {
  // N elements: what is left of them, and then their part in the race or in the sum (two sums, whose additions do not wait for each other)
  double sums[2] = {0., 0.};
  auto take = [&](auto& x, const auto& y, const auto& z, auto at, uint32_t end) {
    constexpr int N = sizeof(x) / sizeof(float);
    if (SUB)
      for (uint32_t j = 0; j < n; ++j) {
        const float m = mass[j];
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = fmaxf(__fsub_rn(x[i], __fmul_rn(m, y[i])), 0.f);
      }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t v = at(i);
      if (v >= end) continue;
      if (!RACE) {
        sums[i & 1] += x[i];
        continue;
      }
      if (!(x[i] > 0.f) || x[i] < best.bar * z[i]) continue;
      bool out = false;
      if (!SUB)
        for (uint32_t k = 0; k < n; ++k) out |= gone[k] == (int32_t)v;
      if (!out) best.offer(x[i], z[i], v);
    }
  };
  uint32_t v = v0;
  if ((((uintptr_t)(p + v0) | (RACE ? (uintptr_t)(e + v0) : 0) | (SUB ? (uintptr_t)(q + v0) : 0)) & 15u) == 0) {
    const uint32_t whole = v0 + (v1 - v0) / 8 * 8;
    constexpr int U = RACE && SUB ? 1 : 2;        // groups of eight in flight: as many as 64 registers hold
    for (v = v0 + threadIdx.x * 8; v < whole; v += U * THREADS * 8) {
      float x[U][8], y[U][8], z[U][8];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t at = min(v + u * THREADS * 8, whole - 8);      // (the last group may be read again, not used)
        load8(p + at, x[u]);
        if (RACE) load8(e + at, z[u]);
        if (SUB) load8(q + at, y[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) take(x[u], y[u], z[u], [&](int i) { return v + u * THREADS * 8 + i; }, whole);
    }
    v = whole;
  }
  for (v += threadIdx.x; v < v1; v += 6 * THREADS) {
    float x[6], y[6], z[6];
#pragma unroll
    for (int i = 0; i < 6; ++i) {
      const uint32_t at = min(v + i * THREADS, v1 - 1);
      x[i] = prob(p, at);
      if (RACE) z[i] = __ldg(e + at);
      if (SUB) y[i] = prob(q, at);
    }
    take(x, y, z, [&](int i) { return v + i * THREADS; }, v1);
  }
  sum += sums[0] + sums[1];
}

template <typename T, bool SUB, uint32_t THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) wb_verify_tree_kernel(const __grid_constant__ wb_verify_tree_args a) {
  cg::cluster_group cluster = cg::this_cluster();
  const uint32_t rank = cluster.block_rank(), size = cluster.num_blocks(), s = blockIdx.x / size, tid = threadIdx.x, lane = tid & 31;
  __shared__ int32_t up[kRows], token[kRows];
  __shared__ float chance_p[kRows], chance_q[kRows], coin[kRows];
  __shared__ float mass_of[kKids];
  __shared__ int32_t gone[kKids];
  __shared__ double warp_sum[THREADS / 32], block_sum[2];
  __shared__ uint64_t warp_best[THREADS / 32], block_best;
  __shared__ int32_t s_here, s_kids, s_more;
  const int32_t start = min(max(__ldg(a.new_start + s), 0), (int32_t)a.n_tokens);
  const int32_t n = min(max(__ldg(a.new_start + s + 1), start), (int32_t)a.n_tokens) - start;
  int32_t* const path = a.path + (uint64_t)s * a.max_depth;
  int32_t* const emitted = a.emitted + (uint64_t)s * (a.max_depth + 1);
  if (n == 0) {                          // no row, nothing to draw from
    if (rank == 0) {
      if (tid == 0) a.accepted[s] = 0;
      for (uint32_t i = tid; i <= a.max_depth; i += THREADS) {
        if (i < a.max_depth) path[i] = -1;
        emitted[i] = -1;
      }
    }
    return;
  }
  const T* const target = reinterpret_cast<const T*>(a.target) + (uint64_t)start * a.target_stride;
  const T* const draft = SUB ? reinterpret_cast<const T*>(a.draft) + (uint64_t)start * a.draft_stride : nullptr;
  const float* e = a.race + (uint64_t)s * a.race_stride;
  const uint32_t share = ((a.vocab + size - 1) / size + 7) / 8 * 8, v0 = min(rank * share, a.vocab), v1 = min(v0 + share, a.vocab);
  // the race is needed whatever is accepted: it comes into the second-level cache while that is found out
  for (uint32_t v = v0 + tid * 32; v < v1; v += THREADS * 32) asm volatile("prefetch.global.L2 [%0];" ::"l"(e + v));
  // a row's parent (-1 if it is no child), its token, and its parent's probabilities of that
  auto parent_of = [&](int32_t i) {
    const int32_t p = __ldg(a.parent + start + i);
    return p >= 0 && p < i && (uint32_t)__ldg(a.tokens + start + i) < a.vocab ? p : -1;
  };
  auto p_of = [&](int32_t i, int32_t parent) { return prob(target, (uint64_t)parent * a.target_stride + (uint32_t)__ldg(a.tokens + start + i)); };
  auto q_of = [&](int32_t i, int32_t parent) { return SUB ? prob(draft, (uint64_t)parent * a.draft_stride + (uint32_t)__ldg(a.tokens + start + i)) : 1.f; };
  for (int32_t i = (int32_t)tid; i < min(n, (int32_t)kRows); i += THREADS) {
    const int32_t p = parent_of(i);
    up[i] = p;
    if (p < 0) continue;
    token[i] = __ldg(a.tokens + start + i);
    chance_p[i] = p_of(i, p);
    chance_q[i] = q_of(i, p);
    coin[i] = __ldg(a.uniform + start + i);
  }
  __syncthreads();

  // ---- the walk: the first warp's lanes hold the same state ----------------------------------------------
  int32_t here = 0, next = 1, depth = 0;         // the row that was accepted last, and where its children are looked for from
  uint32_t kids = 0, summed = 0;                 // its rejected children, and of how many of them the sum is known
  float mass = 1.f;                              // the sum of what they left
  auto walk = [&]() {                            // true if it needs a sum to go on
    while ((uint32_t)depth < a.max_depth) {
      bool took = false;
      for (int32_t i0 = next & ~31; i0 < n && !took; i0 += 32) {
        const int32_t i = i0 + (int32_t)lane;
        const bool child = i < n && i >= next && (i < (int32_t)kRows ? up[i] : parent_of(i)) == here;
        uint32_t todo = __ballot_sync(0xFFFFFFFFu, child);
        if (!todo) continue;
        float p = 0.f, q = 1.f, u = 1.f;
        int32_t x = -1;
        if (child) {
          const bool near = i < (int32_t)kRows;
          x = near ? token[i] : __ldg(a.tokens + start + i);
          p = near ? chance_p[i] : p_of(i, here);
          q = near ? chance_q[i] : q_of(i, here);
          u = near ? coin[i] : __ldg(a.uniform + start + i);
        }
        for (; todo; todo &= todo - 1) {
          const int l = __ffs(todo) - 1;
          if (kids == kKids) return false;
          if (SUB && kids > summed) {
            next = i0 + l;
            return true;
          }
          const float pl = __shfl_sync(0xFFFFFFFFu, p, l), ql = __shfl_sync(0xFFFFFFFFu, q, l), ul = __shfl_sync(0xFFFFFFFFu, u, l);
          const int32_t xl = __shfl_sync(0xFFFFFFFFu, x, l);
          float w = pl;
          if (SUB) {
            w = left_of(pl, ql, mass_of, kids);
          } else {
            bool again = false;                  // a sibling of the same token was rejected before
            for (uint32_t j = lane; j < kids; j += 32) again |= gone[j] == xl;
            if (__any_sync(0xFFFFFFFFu, again)) w = 0.f;
          }
          if (__fmul_rn(ul, __fmul_rn(mass, ql)) < w) {
            here = i0 + l;
            next = here + 1;
            if (rank == 0 && lane == 0) {
              path[depth] = here;
              emitted[depth] = xl;
            }
            ++depth;
            kids = summed = 0;
            mass = 1.f;
            took = true;
            break;
          }
          if (lane == 0) {
            if (SUB) mass_of[kids] = mass; else gone[kids] = xl;
          }
          __syncwarp();
          ++kids;
          if (!SUB) mass = fmaxf(__fsub_rn(mass, w), 0.f);
        }
      }
      if (!took) return false;
    }
    return false;
  };
  uint32_t turn = 0;
  for (;;) {
    if (tid < 32) {
      const bool more = walk();
      if (lane == 0) {
        s_here = here;
        s_kids = (int32_t)kids;
        s_more = more;
      }
    }
    __syncthreads();
    if (!SUB || !s_more) break;
    double sum = 0.;
    Best none;
    tree_range<T, SUB, false, THREADS>(target + (uint64_t)s_here * a.target_stride, draft + (uint64_t)s_here * a.draft_stride, e, v0, v1, mass_of, gone,
                                       (uint32_t)s_kids, none, sum);
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    if (lane == 0) warp_sum[tid >> 5] = sum;
    __syncthreads();
    if (tid == 0) {
      for (uint32_t w = 1; w < THREADS / 32; ++w) sum += warp_sum[w];
      block_sum[turn] = sum;
    }
    cluster.sync();
    // a lane fetches a block's sum; they are added in the blocks' order
    const double part = lane < size ? *cluster.map_shared_rank(&block_sum[turn], lane) : 0.;
    sum = 0.;
    for (uint32_t r = 0; r < size; ++r) sum += __shfl_sync(0xFFFFFFFFu, part, r);
    turn ^= 1;                           // the other place is free: everybody has read it before the next time all meet
    mass = (float)sum;
    summed = kids;
  }

  // ---- the race where the path ends -------------------------------------------------------------------------
  const uint32_t rejected = (uint32_t)s_kids;
  const T* p = target + (uint64_t)s_here * a.target_stride;
  bool all = rejected == 0;              // nothing was taken away
  uint64_t winner;
  for (;;) {
    Best best;
    double none = 0.;
    if (SUB && !all) tree_range<T, true, true, THREADS>(p, draft + (uint64_t)s_here * a.draft_stride, e, v0, v1, mass_of, gone, rejected, best, none);
    else tree_range<T, false, true, THREADS>(p, nullptr, e, v0, v1, mass_of, gone, all ? 0 : rejected, best, none);
    winner = best.key;
#pragma unroll
    for (int d = 16; d; d >>= 1) winner = key_max(winner, __shfl_xor_sync(0xFFFFFFFFu, winner, d));
    if (lane == 0) warp_best[tid >> 5] = winner;
    __syncthreads();
    if (tid < 32) {
      winner = lane < THREADS / 32 ? warp_best[lane] : 0;
#pragma unroll
      for (int d = 16; d; d >>= 1) winner = key_max(winner, __shfl_xor_sync(0xFFFFFFFFu, winner, d));
      if (tid == 0) block_best = winner;
    }
    cluster.sync();
    // every block reads all shares: all of them have to know whether any weight was positive
    winner = lane < size ? *cluster.map_shared_rank(&block_best, lane) : 0;
#pragma unroll
    for (int d = 16; d; d >>= 1) winner = key_max(winner, __shfl_xor_sync(0xFFFFFFFFu, winner, d));
    cluster.sync();                      // block_best may be overwritten or its block may end
    if (winner || all) break;
    all = true;                          // nothing positive was left: draw from the target's row itself
  }
  if (rank == 0 && tid < 32) {
    if (lane == 0) a.accepted[s] = depth;
    for (uint32_t i = (uint32_t)depth + lane; i <= a.max_depth; i += 32) {
      if (i < a.max_depth) path[i] = -1;
      emitted[i] = i == (uint32_t)depth ? (winner ? (int32_t)~(uint32_t)winner : 0) : -1;
    }
  }
}

template <typename T, bool SUB, uint32_t THREADS>
wb_status launch_verify(const wb_verify_tree_args& a, uint32_t size, cudaStream_t stream) {
  cudaLaunchAttribute at[1];
  const cudaLaunchConfig_t cfg = config_of(a.n_seqs, THREADS, size, at, stream);
  if (cudaLaunchKernelEx(&cfg, wb_verify_tree_kernel<T, SUB, THREADS>, a) != cudaSuccess) { (void)cudaGetLastError(); return WB_ERR_CUDA; }
  return WB_OK;
}

// A sequence gets as many blocks as let all sequences run at once, as in wb_verify_drafts.
template <typename T, bool SUB> wb_status launch_verify_of(const wb_verify_tree_args& a, cudaStream_t stream) {
  static ClusterCounts known[2];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { (void)cudaGetLastError(); return WB_ERR_CUDA; }
  for (uint32_t size : {16u, 8u})
    if (a.n_seqs <= resident_clusters(wb_verify_tree_kernel<T, SUB, 512>, 512, dev, size, known[0])) return launch_verify<T, SUB, 512>(a, size, stream);
  for (uint32_t size = 16; size > 1; --size)
    if (a.n_seqs <= resident_clusters(wb_verify_tree_kernel<T, SUB, 256>, 256, dev, size, known[1])) return launch_verify<T, SUB, 256>(a, size, stream);
  return launch_verify<T, SUB, 256>(a, 1, stream);
}

}  // namespace

extern "C" wb_status wb_verify_tree(const wb_verify_tree_args* args, void* stream) {
  if (!args) return WB_ERR_INVALID_ARG;
  const wb_verify_tree_args& a = *args;
  if (a.dtype != WB_F32 && a.dtype != WB_BF16) return WB_ERR_DTYPE;
  if (!a.vocab || a.vocab > 0x7FFFFFFFu || a.max_depth > (1u << 20) || a.n_seqs > (1u << 24) || a.n_tokens > (1u << 30) || a.reserved)
    return WB_ERR_INVALID_ARG;
  auto bad_pitch = [&](uint64_t pitch) { return pitch && pitch < a.vocab; };       // 0: one row for all
  if (bad_pitch(a.target_stride) || bad_pitch(a.race_stride) || (a.draft && bad_pitch(a.draft_stride))) return WB_ERR_INVALID_ARG;
  if (!a.n_seqs) return WB_OK;
  if (!a.new_start || !a.race || !a.accepted || !a.emitted || (a.max_depth && !a.path)) return WB_ERR_INVALID_ARG;
  if (a.n_tokens && (!a.target || !a.parent || !a.tokens || !a.uniform)) return WB_ERR_INVALID_ARG;
  const uint32_t e = a.dtype == WB_F32 ? 4 : 2;
  if (((uintptr_t)a.target | (uintptr_t)a.draft) % e || ((uintptr_t)a.race | (uintptr_t)a.uniform | (uintptr_t)a.tokens | (uintptr_t)a.parent |
      (uintptr_t)a.new_start | (uintptr_t)a.accepted | (uintptr_t)a.path | (uintptr_t)a.emitted) % 4)
    return WB_ERR_INVALID_ARG;
  const cudaStream_t st = (cudaStream_t)stream;
  if (a.dtype == WB_F32) return a.draft ? launch_verify_of<float, true>(a, st) : launch_verify_of<float, false>(a, st);
  return a.draft ? launch_verify_of<uint16_t, true>(a, st) : launch_verify_of<uint16_t, false>(a, st);
}
