// What the attention kernels share: their parameters, barriers and copies with bounded waits, the
// workspace, and small numeric helpers.
#pragma once
#include "wb_kv.cuh"

namespace wbi {

struct AttendArgs {
  KvView c;
  KvBatch b;
  const char* q;
  char* out;
  uint64_t q_token, q_head, o_token, o_head;   // bytes
  float* lse;
  float scale_log2;                             // softmax scale times log2(e)
  uint32_t n_heads, group, window;
  uint32_t box_rows;
  uint32_t words;                               // of a row of mask
  uint32_t row_blocks;                          // clusters only: of a sequence's rows, at most
  const uint32_t* mask;                         // trees only: what a row sees of its sequence's new tokens
  uint32_t* error;                              // workspace: first word, bits of AttendError
  char* cuts;                                   // CutItem of every block
  float* partials;
};

// What a joining kernel reads of the item that is cut first in a block.
struct CutItem {
  uint32_t parts;          // 0: none
  uint32_t s, h, rb;       // sequence, kv head, row block; for the row kernel: first row of the step's tensors, kv head, rows
};

enum AttendError : uint32_t {
  kGaveUp = 1,             // a wait lasted too long
  kMisplaced = 2,          // shared memory not where tiles need it
  kTooLong = 4,            // a sequence was longer than max_len
};

constexpr float kLn2 = 0.69314718055994531f;
constexpr uint64_t kAttendWaitNs = 2000000000ull;   // a wait that lasts this long records an error and gives up

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_arrive_n(uint32_t bar, uint32_t n) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(n) : "memory");
}
__device__ __forceinline__ void bar_arrive_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// False if the phase did not complete within kAttendWaitNs.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
  if (bar_try(bar, parity)) return true;
  uint64_t t0, t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
  for (uint32_t it = 1;; ++it) {
    if (bar_try(bar, parity)) return true;
    if ((it & 255u) == 0) {
      asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
      if (t - t0 > kAttendWaitNs) return false;
    }
  }
}

// After a wait that gave up, the caller goes on without waiting (and with wrong numbers): the kernel ends, and the
// error word tells.
__device__ __forceinline__ bool wait_or_give_up(uint32_t bar, uint32_t parity, bool ok, uint32_t* error) {
  if (ok && !bar_wait(bar, parity)) {
    atomicOr(error, kGaveUp);
    return false;
  }
  return ok;
}

// A value that all lanes of a converged warp share, such that the compiler knows it.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __shfl_sync(0xFFFFFFFFu, x, 0); }
__device__ __forceinline__ int32_t uniform(int32_t x) { return __shfl_sync(0xFFFFFFFFu, x, 0); }

// One box of a cache map: elements [x, ..) of the box's slots from `slot` on of (head, page).
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t slot, int32_t head, int32_t page, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               ::"r"(dst), "l"(map), "r"(x), "r"(slot), "r"(head), "r"(page), "r"(bar) : "memory");
}
__device__ __forceinline__ void load_bulk(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two E4M3 codes, in the high bytes of the halves of x, as two bf16 values: sign, exponent and mantissa
// bits are moved to their places, which reads as the value times 2^-120 (the difference of the biases, subnormal
// codes included), and one exact product puts that right.  (A NaN code reads as 480: rows that
// wb_kv_write makes have such codes only where their scale is not finite either.)
__device__ __forceinline__ uint32_t e4m3_to_bf16x2(uint32_t x) {
  uint32_t r = (x & 0x80008000u) | ((x >> 4) & 0x07F007F0u);
  asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(r) : "r"(0x7B807B80u));
  return r;
}

// A sequence that is longer than the call was checked for has nothing to attend over: with its length cut its new tokens would
// stand at other positions than they were written to, and its results would look right.
__device__ __forceinline__ KvSeq attend_seq(const KvBatch& b, uint32_t s) {
  KvSeq q = kv_seq(b, s);
  if (q.len > b.max_len) q.len = 0;
  return q;
}
__device__ __forceinline__ void report_too_long(const AttendArgs& a, uint32_t s) {
  if (blockIdx.x != 0) return;
  const KvSeq q = kv_seq(a.b, s);
  if (q.n_new > 0 && q.len > a.b.max_len) atomicOr(a.error, kTooLong);
}

// First position that any of the sequence's new tokens attends over.  (A tree's row that sees none of the tree, itself included, stands
// before it.)
template <bool TREE> __device__ __forceinline__ int32_t first_position(const KvSeq& q, uint32_t window) {
  return window ? max(0, q.len - q.n_new - (int32_t)window + (TREE ? 0 : 1)) : 0;
}

// Word w of the row of mask of row t of the step's tensors; before the tree everything is seen, beyond the mask nothing.
__device__ __forceinline__ uint32_t tree_word(const AttendArgs& a, uint32_t t, int32_t w) {
  return w < 0 ? 0xFFFFFFFFu : (uint32_t)w < a.words ? __ldg(a.mask + (uint64_t)t * a.words + w) : 0u;
}
// The lowest position that row i of a tree, row t of the step's tensors, sees: its own is the first new token's place plus the rows
// that it sees, less one.
__device__ __forceinline__ int32_t tree_low(const AttendArgs& a, const KvSeq& q, uint32_t t, int32_t i) {
  if (!a.window) return 0;
  int32_t sees = 0;
  for (int32_t w = 0; w <= i >> 5; ++w) sees += __popc(tree_word(a, t, w) & (w == i >> 5 ? 0xFFFFFFFFu >> (31 - (i & 31)) : 0xFFFFFFFFu));
  return q.len - q.n_new + sees - (int32_t)a.window;
}

}  // namespace wbi
