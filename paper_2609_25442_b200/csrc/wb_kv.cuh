// What the paged-cache kernels share: the cache and the batch as kernel parameters, the place of a
// position, and the host checks of both.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "wb_internal.h"

// The opaque handle: a validated description and the tensor maps of keys and values.
struct wb_kv {
  wb_kv_desc d;
  // 4-D maps (element, slot, head, page) with a box of 128 bytes (or a row, if shorter) x box_rows slots,
  // swizzled for conflict-free matrix loads; box_rows = gcd(page_size, kKvTile), so a box never crosses
  // a page, and coordinates outside the cache read as zeros
  CUtensorMap map_k, map_v;
  uint32_t box_rows;
  int device;                // the one that was current at wb_kv_open: calls launch there and nowhere else
};

namespace wbi {

constexpr uint32_t kKvTile = 64;   // cache rows of a tile of the row kernel, and at most in a box

struct KvView {
  char* k;
  char* v;
  float* k_scale;
  float* v_scale;
  uint64_t page_stride, head_stride;   // elements
  uint32_t n_pages, n_kv_heads, page_size, head_dim;
};

inline KvView kv_view(const wb_kv* kv) {
  const wb_kv_desc& d = kv->d;
  return KvView{(char*)d.k, (char*)d.v, d.k_scale, d.v_scale, d.page_stride, d.head_stride, (uint32_t)d.n_pages,
                d.n_kv_heads, d.page_size, d.head_dim};
}

struct KvBatch {
  const int32_t* table;
  const int32_t* new_start;
  const int32_t* kv_len;
  uint32_t n_seqs, n_tokens, table_stride, table_pitch;
  int32_t max_len;
};

inline KvBatch kv_batch(const wb_kv_batch* b) {
  return KvBatch{b->page_table, b->new_start, b->kv_len, b->n_seqs, b->n_tokens, b->table_stride,
                 b->table_pitch ? b->table_pitch : b->table_stride, (int32_t)b->max_len};
}

inline bool on_kv_device(const wb_kv* kv) {
  int dev = -1;
  return cudaGetDevice(&dev) == cudaSuccess && dev == kv->device;
}

inline wb_status check_batch_arrays(const wb_kv_batch* b) {
  if (!b || b->n_seqs > WB_KV_MAX_SEQS || (b->table_pitch && b->table_pitch < b->table_stride)) return WB_ERR_INVALID_ARG;
  if (b->n_tokens > 0x7FFFFFFFu || b->max_len > 0x7FFFFFFFu || b->max_new > b->n_tokens) return WB_ERR_INVALID_ARG;
  if (b->n_seqs && (!b->new_start || !b->kv_len || (b->table_stride && !b->page_table))) return WB_ERR_INVALID_ARG;
  if (((uintptr_t)b->page_table | (uintptr_t)b->new_start | (uintptr_t)b->kv_len) & 3u) return WB_ERR_INVALID_ARG;
  return WB_OK;
}

inline wb_status check_batch(const wb_kv* kv, const wb_kv_batch* b) {
  if (!kv) return WB_ERR_INVALID_ARG;
  if (wb_status s = check_batch_arrays(b)) return s;
  // positions are 32-bit: a row of the table covers fewer than 2^31 of them
  if ((uint64_t)b->table_stride * kv->d.page_size > 0x7FFFFFFFull) return WB_ERR_INVALID_ARG;
  return on_kv_device(kv) ? WB_OK : WB_ERR_INVALID_ARG;
}

inline wb_status check_heads(const wb_heads* h, uint32_t n_tokens, bool allow_f32) {
  if (!h || h->reserved) return WB_ERR_INVALID_ARG;
  if (h->dtype != WB_BF16 && !(allow_f32 && h->dtype == WB_F32)) return WB_ERR_DTYPE;
  if (!n_tokens) return WB_OK;
  const uint64_t per = h->dtype == WB_F32 ? 4 : 8;
  if (!h->data || ((uintptr_t)h->data & 15u) || h->token_stride % per || h->head_stride % per) return WB_ERR_INVALID_ARG;
  return WB_OK;
}

// One sequence of the batch, with every value that came from device memory brought into range.
struct KvSeq {
  int32_t row0, n_new;   // its rows of the step's tensors
  int32_t len;           // tokens in the cache; the position of new token i is len - n_new + i
};

__device__ __forceinline__ KvSeq kv_seq(const KvBatch& b, uint32_t s) {
  KvSeq q;
  q.row0 = min(max(__ldg(b.new_start + s), 0), (int32_t)b.n_tokens);
  const int32_t end = min(max(__ldg(b.new_start + s + 1), q.row0), (int32_t)b.n_tokens);
  q.n_new = end - q.row0;
  q.len = max(__ldg(b.kv_len + s), 0);
  return q;
}

// The last sequence whose rows start at or before `row` (sequences without new tokens share a start).
__device__ __forceinline__ uint32_t kv_seq_of_row(const KvBatch& b, int32_t row) {
  uint32_t lo = 0, hi = b.n_seqs;   // new_start[lo] <= row < new_start[hi]
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) >> 1;
    if (__ldg(b.new_start + mid) <= row) lo = mid; else hi = mid;
  }
  return lo;
}

// Page of position `pos` of sequence s, or -1 if the table does not cover it or names no page.
__device__ __forceinline__ int32_t kv_page(const KvBatch& b, uint32_t n_pages, uint32_t page_size, uint32_t s, int32_t pos) {
  if (pos < 0) return -1;
  const uint32_t i = (uint32_t)pos / page_size;
  if (i >= b.table_stride) return -1;
  const int32_t p = __ldg(b.table + (uint64_t)s * b.table_pitch + i);
  return (uint32_t)p < n_pages ? p : -1;
}

constexpr uint32_t kTokensPerBlock = 32;   // of the kernels that move rows, at most; fewer where that leaves SMs without a block

// Where the block's tokens live: page and slot of each, page -1 for one that has no place.  One warp: it finds the first token's
// sequence by a 32-way search (a load per factor of 32, where a search per token would be five), and the others' by counting
// the starts that follow.  `position`: their positions too, INT32_MIN of one that no sequence holds.
__device__ __forceinline__ void place_by_warp(const KvView& c, const KvBatch& b, uint32_t t0, uint32_t n, int2* place, int32_t* position, uint32_t lane) {
  const int32_t first = (int32_t)t0, row = (int32_t)(t0 + lane);
  uint32_t lo = 0, hi = b.n_seqs;                     // new_start[lo] <= first < new_start[hi]
  while (hi - lo > 1) {
    const uint32_t step = (hi - lo + 31) / 32, at = lo + lane * step;
    const bool before = at < hi && (lane == 0 || __ldg(b.new_start + at) <= first);
    const uint32_t k = 31 - __clz(__ballot_sync(0xFFFFFFFFu, before));
    lo += k * step;
    hi = min(hi, lo + step);
  }
  // sequences after the first that start within the block's tokens
  uint32_t s = lo;
  if (n > 1 && b.n_seqs > 1) {
    const uint32_t next = lo + 1 + lane;
    const int32_t start = next < b.n_seqs ? __ldg(b.new_start + next) : 0x7FFFFFFF;
#pragma unroll
    for (int j = 0; j < 32; ++j) s += __shfl_sync(0xFFFFFFFFu, start, j) <= row;
    if (s == lo + 32) s = kv_seq_of_row(b, row);      // more than 32 of them (most without tokens)
  }
  if (lane < n) {
    const KvSeq q = kv_seq(b, s);
    const int32_t at = row - q.row0, pos = q.len - q.n_new + at;
    const int32_t page = at >= 0 && at < q.n_new ? kv_page(b, c.n_pages, c.page_size, s, pos) : -1;
    place[lane] = make_int2(page, page < 0 ? 0 : pos % (int32_t)c.page_size);
    if (position) position[lane] = at >= 0 && at < q.n_new ? pos : INT32_MIN;
  }
}
__device__ __forceinline__ void place_tokens(const KvView& c, const KvBatch& b, uint32_t t0, uint32_t n, int2* place) {
  if (threadIdx.x < 32) place_by_warp(c, b, t0, n, place, nullptr, threadIdx.x);
  __syncthreads();
}

// A step's tensor as a kernel parameter.
struct Rows {
  char* data;
  uint64_t token_stride, head_stride;   // bytes
};

inline Rows rows_of(const wb_heads* h) {
  const uint64_t e = h->dtype == WB_F32 ? 4 : 2;
  return Rows{(char*)h->data, h->token_stride * e, h->head_stride * e};
}

// ---- conversions -----------------------------------------------------------------------------
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint16_t pack_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 unpack_e4m3x2(uint16_t codes) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(codes));
  float lo, hi;
  asm("{ .reg .b16 l, h; mov.b32 {l, h}, %2; cvt.f32.f16 %0, l; cvt.f32.f16 %1, h; }" : "=f"(lo), "=f"(hi) : "r"(h));
  return make_float2(lo, hi);
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

}  // namespace wbi
