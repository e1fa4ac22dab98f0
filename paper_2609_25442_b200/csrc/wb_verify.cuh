// What the verification kernels share: probabilities as they are read, and the race for the next token.
#pragma once
#include "wb_cluster.cuh"
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

}  // namespace wbi
