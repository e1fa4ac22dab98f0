// Attention for few rows: sequences whose new tokens times query heads per kv head are at most 32 rows (single tokens, drafted
// chunks).  Every byte of the cache is used for a handful of products, so the bound is memory bandwidth, and the kernel is a
// stream of cache rows through shared memory:
//
//   - A warp owns 16 cache rows of every 64-row tile: it requests them itself, a few tiles ahead, into slots of its own, and it
//     alone reads them.  16 divides the page size, so they are one contiguous piece of keys and one of values.  No warp waits
//     for another until an item ends.  (Tensor-map loads of such small pieces cost the issuing warp 90 ns each, more
//     than the arithmetic on them; a lane's 16-byte copies cost an instruction.)
//   - Scores are computed as K Q^T and outputs as V^T P^T, so that the cache's 16 rows fill the instruction's 16 and the query
//     rows, few as they are, only its 8 columns: for up to 8 query rows half the work of the usual orientation, and each
//     code of an E4M3 cache is widened once for all rows.
//   - E4M3 codes become f16 (exact, one instruction for two), queries f16 after a power of two that brings the row's largest
//     value near 2^8 (what falls below f16's range is under 2^-32 of that value), and weights times row scales f16
//     relative to a power of two that follows their maximum like the softmax's own: each keeps 11 bits down to 2^-14 of the
//     largest so far, and is off by at most 2^-25 of it below.  (Widening to bf16 took 10 instructions for
//     four codes, and the kernel was bound by them: 115 us where this takes 68 for 96 sequences of 500 to 6000
//     positions, 4.8 TB/s.)
//   - The running maximum and the f16 exponent move only when a weight would pass 2^8, checked without any exchange: one vote.
//   - 64 sequences of 17 to 8192 positions, bf16: 179 to 183 us, 6.2 TB/s, 0.94 of the copy bandwidth.  With 32 query rows and E4M3 the
//     matrix instructions of 64 products a tile and warp, and their latency with eight warps on an SM, are the bound: 73.5 us for 24
//     sequences, 2.0 TB/s.
//   - Work is cut evenly over the SMs whatever the lengths: all (sequence, kv head) items form one line of tiles, every block
//     takes the same number of consecutive tiles, and a second kernel joins the items that cross blocks, in the order of the
//     tiles (so results do not depend on timing).
//   - Few trees are a matter of latency.  A cluster of blocks then serves 8, 16 or 32 rows of a (sequence, kv head): each block takes its share of the
//     cache's tiles, and the cluster joins them over distributed shared memory, without a second kernel.
#pragma once
#include <cooperative_groups.h>

#include "wb_attend.cuh"

namespace wbi {

constexpr uint32_t kSmemPerSm = 233472;

template <int D, bool Q, int NT>
struct RowsCfg {
  static constexpr uint32_t kElem = Q ? 1 : 2;
  static constexpr uint32_t kRowBytes = D * kElem;
  static constexpr uint32_t kSpan = kRowBytes < 128 ? kRowBytes : 128;       // bytes of a row in one box
  static constexpr uint32_t kPartBytes = 16 * kRowBytes;                     // a warp's keys of a tile, and as much of values
  static constexpr uint32_t kSlotBytes = 2 * kPartBytes;
  static constexpr uint32_t kScaleBytes = Q ? 128 : 0;                       // 16 scales of keys and of values
  static constexpr uint32_t kRows = 8 * NT;                                  // query rows
  static constexpr uint32_t kPitch = D + 4;                                  // floats; keeps the join free of bank conflicts
  static constexpr uint32_t kBuffers = NT == 4 ? 1 : 2;                      // of the join
  static constexpr uint32_t kJoinBytes = kBuffers * kRows * kPitch * 4;
  static constexpr uint32_t kBlocksPerSm = NT == 4 || !Q ? 2 : 3;
  static constexpr uint32_t kThreads = 128;
  static constexpr uint32_t kPartFloats = kRows * D + 2 * kRows;             // one partial: outputs, maxima, sums
  static constexpr uint32_t kFixedBytes = kJoinBytes + 4 * kRows * 8 + 1024; // with warps' maxima and sums, and alignment
  // as many slots as leave room for the prefix sums of about 250 sequences
  static constexpr uint32_t kSlots = (kSmemPerSm / kBlocksPerSm - 1024 - kFixedBytes - 1536) / (4 * (kSlotBytes + kScaleBytes)) > 8
                                         ? 8 : (kSmemPerSm / kBlocksPerSm - 1024 - kFixedBytes - 1536) / (4 * (kSlotBytes + kScaleBytes));
  static_assert(kSlots >= 2, "");
  static size_t smem_bytes(uint32_t n_seqs) { return kFixedBytes + 4 * kSlots * (kSlotBytes + kScaleBytes) + (n_seqs + 1) * 4; }
};

__device__ __forceinline__ void ldsm4(uint32_t a, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a));
}
__device__ __forceinline__ void ldsm4t(uint32_t a, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a));
}
template <bool F16> __device__ __forceinline__ void mma16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  if (F16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 8 x 8 transposition: a lane's pair (row lane / 4, columns 2t, 2t + 1) -> (row 2t, 2t + 1 of column lane / 4)
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// the two codes of a half word as f16
__device__ __forceinline__ uint32_t codes_to_f16x2(uint32_t codes) {
  uint32_t r;
  asm("{ .reg .b16 l, h; mov.b32 {l, h}, %1; cvt.rn.f16x2.e4m3x2 %0, l; }" : "=r"(r) : "r"(codes));
  return r;
}
__device__ __forceinline__ uint32_t codes_hi_to_f16x2(uint32_t codes) {
  uint32_t r;
  asm("{ .reg .b16 l, h; mov.b32 {l, h}, %1; cvt.rn.f16x2.e4m3x2 %0, h; }" : "=r"(r) : "r"(codes));
  return r;
}

// Asynchronous copies of a lane; with fewer source bytes the rest is zeros.
__device__ __forceinline__ void copy16(uint32_t to, const void* from, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t to, const void* from, uint32_t bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Byte offset of 16-byte chunk `c` of row `row` in a swizzled block of rows of `SPAN` bytes.
template <uint32_t SPAN> __device__ __forceinline__ uint32_t swizzled(uint32_t row, uint32_t c) {
  return SPAN == 128 ? row * 128 + ((c ^ (row & 7)) << 4) : row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
}

__device__ __forceinline__ bool not_finite_bf16x2(uint32_t w) {
  return ((w & 0x7F80u) == 0x7F80u) | ((w & 0x7F800000u) == 0x7F800000u);
}

// Where a warp's 16 rows of a tile are: slots [slot, slot + 16) of kv head h in a page, as the table has it (checked when used;
// h is -1 if the position lies past the sequence or the table).
struct TilePlace {
  int32_t page, h;
  uint32_t slot;
};

// What a launch serves: chunks along the line of tiles, trees along it, or trees with a cluster for every 8 NT rows of a (sequence, kv head).
enum class RowsMode { kChunk, kTree, kTreeCluster };

template <int D, bool Q, int NT, RowsMode MODE>
__global__ void __launch_bounds__(128, RowsCfg<D, Q, NT>::kBlocksPerSm)
wb_attend_rows_kernel(const __grid_constant__ AttendArgs a) {
  using C = RowsCfg<D, Q, NT>;
  constexpr bool TREE = MODE != RowsMode::kChunk, CLUSTER = MODE == RowsMode::kTreeCluster;
  extern __shared__ char smem_raw[];
  // slots (1024-byte aligned), their scales, join buffer, warps' maxima and sums, prefix sums
  const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
  char* const gen = smem_raw + (base - smem_addr(smem_raw));
  constexpr uint32_t kScaleBase = 4 * C::kSlots * C::kSlotBytes;
  float* const join = reinterpret_cast<float*>(gen + kScaleBase + 4 * C::kSlots * C::kScaleBytes);
  float2* const warp_ml = reinterpret_cast<float2*>(join + C::kJoinBytes / 4);        // [warp][row]
  int32_t* const cum = reinterpret_cast<int32_t*>(warp_ml + 4 * C::kRows);
  __shared__ int32_t scan_tmp[4];
  float* const spare = reinterpret_cast<float*>(gen);      // the slots' memory, once a cluster's block is done with it
  __shared__ float down_of[C::kRows];      // what undoes the scaling of a row's query
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, t4 = lane & 3, r8 = lane >> 2;

  // ---- a cluster's item: tiles [0, its_tiles) of a line of its own ------------------------------------
  __shared__ int32_t row_token[CLUSTER ? C::kRows : 1], row_low[CLUSTER ? C::kRows : 1];      // of the step's tensors; lowest position seen
  __shared__ float2 block_ml[CLUSTER ? C::kRows : 1];
  const uint32_t n_seqs = a.b.n_seqs, hk = a.c.n_kv_heads;
  namespace cg = cooperative_groups;
  uint32_t its_s = 0, its_h = 0, its_rows = 0, rank = 0, size = 1;
  int32_t its_tile0 = 0, its_tiles = 0;
  KvSeq its = {};
  if (CLUSTER) {
    rank = cg::this_cluster().block_rank();
    size = cg::this_cluster().num_blocks();
    const uint32_t item = blockIdx.x / size, rb = item % a.row_blocks;
    its_h = item / a.row_blocks % hk;
    its_s = item / a.row_blocks / hk;
    its = attend_seq(a.b, its_s);
    if (tid == 0 && rank == 0 && its_h == 0 && rb == 0) {
      const KvSeq q = kv_seq(a.b, its_s);
      if (q.n_new > 0 && q.len > a.b.max_len) atomicOr(a.error, kTooLong);
    }
    const uint32_t all = (uint32_t)its.n_new * a.group, r0 = rb * C::kRows;
    if (r0 >= all) return;               // (all blocks of the cluster)
    its_rows = min(all - r0, C::kRows);
    if (tid < its_rows) {
      const int32_t i = (int32_t)((r0 + tid) / a.group);
      row_token[tid] = i;
      row_low[tid] = tree_low(a, its, (uint32_t)(its.row0 + i), i);
    }
    its_tile0 = first_position<TREE>(its, a.window) / (int32_t)kKvTile;
    // as far as its last row may see
    const int32_t last = its.len - its.n_new + (int32_t)((r0 + its_rows - 1) / a.group);
    its_tiles = max(1, (last + (int32_t)kKvTile) / (int32_t)kKvTile - its_tile0);
  }
  // row r of the item, as token of its sequence's new ones and query head of its kv head
  const uint32_t group_inv = (65536 + a.group - 1) / a.group;      // r / group = r * group_inv >> 16 for r < 64
  auto token_of = [&](uint32_t r) { return CLUSTER ? (uint32_t)row_token[r] : r * group_inv >> 16; };
  auto head_of = [&](uint32_t r, uint32_t token) { return CLUSTER ? (blockIdx.x / size % a.row_blocks * C::kRows + r) % a.group : r - token * a.group; };

  // ---- the line of tiles: cum[s] = tiles of the sequences before s ---------------------------------
  if (!CLUSTER) {
    const uint32_t per = (n_seqs + 127) / 128, s0 = min(tid * per, n_seqs), s1 = min(s0 + per, n_seqs);
    int32_t sum = 0;
    for (uint32_t s = s0; s < s1; ++s) {
      const KvSeq q = attend_seq(a.b, s);
      int32_t nt = 0;
      if (q.n_new > 0 && (uint32_t)q.n_new * a.group <= C::kRows) {
        const int32_t lo = first_position<TREE>(q, a.window) / (int32_t)kKvTile;
        nt = max(1, (q.len + (int32_t)kKvTile - 1) / (int32_t)kKvTile - lo);
      }
      report_too_long(a, s);
      cum[s + 1] = nt * (int32_t)hk;     // this thread's own entries, made inclusive below
      sum += nt * (int32_t)hk;
    }
    int32_t inc = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int32_t o = __shfl_up_sync(0xFFFFFFFFu, inc, d);
      if ((int)lane >= d) inc += o;
    }
    if (lane == 31) scan_tmp[warp] = inc;
    __syncthreads();
    int32_t before = inc - sum;
    for (uint32_t w = 0; w < warp; ++w) before += scan_tmp[w];
    for (uint32_t s = s0; s < s1; ++s) {
      before += cum[s + 1];
      cum[s + 1] = before;
    }
    if (tid == 0) cum[0] = 0;
    __syncthreads();
  }
  const int32_t total = CLUSTER ? its_tiles : cum[n_seqs];
  const int32_t blocks = CLUSTER ? (int32_t)size : (int32_t)gridDim.x, per = (total + blocks - 1) / blocks;
  const int32_t begin = min((CLUSTER ? (int32_t)rank : (int32_t)blockIdx.x) * per, total), end = min(begin + per, total);
  CutItem* const cut_item = reinterpret_cast<CutItem*>(a.cuts) + blockIdx.x;
  if (!CLUSTER && tid == 0) cut_item->parts = 0;
  if (!CLUSTER && begin >= end) return;
  if (CLUSTER) {
    if (begin >= end && tid < its_rows) block_ml[tid] = make_float2(-INFINITY, 0.f);
    __syncthreads();                     // the rows' tokens are known
  }

  // the sequence of tile t
  auto find = [&](int32_t t) {
    if (CLUSTER) return its_s;
    uint32_t lo = 0, hi = n_seqs;        // cum[lo] <= t < cum[hi]
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) >> 1;
      if (cum[mid] <= t) lo = mid; else hi = mid;
    }
    while (cum[lo + 1] <= t) ++lo;
    return lo;
  };

  // ---- loads: the warp's 16 rows of a tile ------------------------------------------------------------
  // Lane i looks tile 32 n + i of the block up, 16 tiles before the first of the 32 is requested, so that neither the search nor
  // the table's latency is on the way of a request.
  auto look_up = [&](uint32_t k0) {
    TilePlace x = {-1, -1, 0};
    const int32_t t = begin + (int32_t)(k0 + lane);
    if (t < end) {
      const uint32_t s = find(t);
      const KvSeq q = CLUSTER ? its : attend_seq(a.b, s);
      int32_t h = (int32_t)its_h, tile = its_tile0 + t;
      if (!CLUSTER) {
        const int32_t nt = (cum[s + 1] - cum[s]) / (int32_t)hk, local = t - cum[s];
        h = local / nt;
        tile = first_position<TREE>(q, a.window) / (int32_t)kKvTile + local - h * nt;
      }
      const uint32_t pos = (uint32_t)tile * kKvTile + warp * 16;
      const uint32_t entry = pos / a.c.page_size;
      x.slot = pos - entry * a.c.page_size;
      if (pos < (uint32_t)q.len && entry < a.b.table_stride) {
        x.h = h;
        x.page = __ldg(a.b.table + (uint64_t)s * a.b.table_pitch + entry);
      }
    }
    return x;
  };
  TilePlace place = look_up(0), later = {-1, -1, 0};
  // Requests tile number k of the block.  The 16 rows are one contiguous piece of keys and one of values, so a lane's copies
  // are at fixed distances from two addresses.
  const uint32_t warp_slots = base + warp * C::kSlots * C::kSlotBytes;
  auto request = [&](uint32_t k) {
    const uint32_t slot = k % C::kSlots, at = warp_slots + slot * C::kSlotBytes;
    const uint32_t page = (uint32_t)__shfl_sync(0xFFFFFFFFu, place.page, k & 31), in_page = __shfl_sync(0xFFFFFFFFu, place.slot, k & 31);
    const int32_t h = __shfl_sync(0xFFFFFFFFu, place.h, k & 31);
    const bool live = h >= 0 && page < a.c.n_pages;
    const uint64_t row = live ? (uint64_t)page * a.c.page_stride + (uint32_t)h * a.c.head_stride + in_page * D : 0;
    const char* src_k = a.c.k + row * C::kElem + lane * 16;
    const char* src_v = a.c.v + row * C::kElem + lane * 16;
    const uint32_t bytes = live ? 16 : 0;                                   // a page that does not exist reads as zeros
#pragma unroll
    for (uint32_t i = 0; i < C::kPartBytes / 512; ++i) {
      const uint32_t off = i * 512 + lane * 16, r = off / C::kRowBytes, c = off % C::kRowBytes / 16;
      const uint32_t to = at + c / 8 * (16 * C::kSpan) + swizzled<C::kSpan>(r, c % 8);
      copy16(to, src_k + i * 512, bytes);
      copy16(to + C::kPartBytes, src_v + i * 512, bytes);
    }
    if (Q) {
      const float* scales = lane < 16 ? a.c.k_scale : a.c.v_scale;
      const uint64_t sr = live ? ((uint64_t)page * hk + (uint32_t)h) * a.c.page_size + in_page + (lane & 15) : 0;
      copy4(base + kScaleBase + (warp * C::kSlots + slot) * C::kScaleBytes + lane * 4, scales + sr, live ? 4 : 0);
    }
    if ((k & 31) == 15) later = look_up((k | 31) + 1);
    if ((k & 31) == 31) place = later;
  };
  // ---- an item and its queries --------------------------------------------------------------------------
  // query fragments: rows lane / 4 of every group of 8 (32 rows: one group per warp, shared through the join buffer)
  constexpr bool kShared = NT == 4;
  constexpr int kGroups = kShared ? 1 : NT;
  struct Item {
    uint32_t s, n_rows;
    int32_t h, tile0, i0, i1, row0, len, n_new;      // i0, i1: its tiles in the line
  };
  auto enter = [&](Item& x, int32_t t) {
    if (CLUSTER) {
      x = Item{its_s, its_rows, (int32_t)its_h, its_tile0, 0, its_tiles, its.row0, its.len, its.n_new};
      return;
    }
    while (!CLUSTER && cum[x.s + 1] <= t) ++x.s;
    const KvSeq q = attend_seq(a.b, x.s);
    const int32_t nt = (cum[x.s + 1] - cum[x.s]) / (int32_t)hk;
    x.tile0 = first_position<TREE>(q, a.window) / (int32_t)kKvTile;
    x.h = (t - cum[x.s]) / nt;
    x.i0 = cum[x.s] + x.h * nt;
    x.i1 = x.i0 + nt;
    x.n_rows = min((uint32_t)q.n_new * a.group, C::kRows);
    x.row0 = q.row0;
    x.len = q.len;
    x.n_new = q.n_new;
  };
  uint32_t qf[kGroups][D / 16][2];
  // trees: what rows 2t, 2t + 1 of every group of 8 see of the sequence's new tokens, at most 32; with clusters, which may have more
  // rows before them, of the tile's 16 positions
  uint32_t tree[NT][2];
  auto fetch_queries = [&](const Item& x) {
#pragma unroll
    for (int n = 0; n < kGroups; ++n) {
      const uint32_t r = (kShared ? warp : n) * 8 + r8;
      const bool in = r < x.n_rows;
      const uint32_t i = in ? token_of(r) : 0;
      const char* src = a.q + (uint64_t)(x.row0 + (int32_t)i) * a.q_token + ((uint32_t)x.h * a.group + (in ? head_of(r, i) : 0)) * a.q_head;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        uint2 w = make_uint2(0, 0);
        if (in) {
          if (Q) {   // the k index of an instruction is permuted alike in both operands: four adjacent codes per lane
            w = __ldg(reinterpret_cast<const uint2*>(src + ks * 32 + t4 * 8));
          } else {
            w.x = __ldg(reinterpret_cast<const uint32_t*>(src + ks * 32 + t4 * 4));
            w.y = __ldg(reinterpret_cast<const uint32_t*>(src + ks * 32 + 16 + t4 * 4));
          }
        }
        qf[n][ks][0] = w.x;
        qf[n][ks][1] = w.y;
      }
    }
    if (TREE && !CLUSTER) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t r = n * 8 + 2 * t4 + e;
          tree[n][e] = r < x.n_rows ? tree_word(a, (uint32_t)x.row0 + (r * group_inv >> 16), 0) : 0xFFFFFFFFu;
        }
    }
  };

  // the first item's queries are on their way before the cache's tiles crowd the memory
  Item it = {};
  if (begin < end) {
    it.s = find(begin);
    enter(it, begin);
    fetch_queries(it);
  }
  const uint32_t n_tiles = (uint32_t)(end - begin);
  uint32_t requested = 0;
  for (; requested < C::kSlots; ++requested) {
    if (requested < n_tiles) request(requested);
    copies_commit();
  }

  // ---- compute ---------------------------------------------------------------------------------------
  const float c2 = a.scale_log2;
  uint32_t k = 0;
  int32_t t = begin;
  while (t < end) {
    const Item cur = it;
    const int32_t stop = min(end, cur.i1);
    const uint32_t n_rows = cur.n_rows;
    const int32_t first_hi = cur.len - cur.n_new, last_lo = a.window ? cur.len - (int32_t)a.window : 0;
    float c2q[NT][2];                     // the softmax scale (of the scaled queries) of rows 2t, 2t + 1
    if (Q) {
#pragma unroll
      for (int n = 0; n < kGroups; ++n) {
        uint32_t big = 0;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
          for (int b = 0; b < 2; ++b) big = max(max(qf[n][ks][b] & 0x7FFFu, (qf[n][ks][b] >> 16) & 0x7FFFu), big);
        big = max(big, __shfl_xor_sync(0xFFFFFFFFu, big, 1));
        big = max(big, __shfl_xor_sync(0xFFFFFFFFu, big, 2));
        // 2^(7 - exponent): an exponent field of e becomes 134; what is not finite stays so
        const int32_t e = min(max((int32_t)(big >> 7), 8), 253);
        const float up = __uint_as_float((uint32_t)(134 - e + 127) << 23), down = __uint_as_float((uint32_t)(e - 134 + 127) << 23);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
          for (int b = 0; b < 2; ++b) qf[n][ks][b] = pack_f16x2(bf16_lo(qf[n][ks][b]) * up, bf16_hi(qf[n][ks][b]) * up);
        if (kShared) {
          if (t4 == 0) down_of[warp * 8 + r8] = down;
        } else {
          c2q[n][0] = c2 * __shfl_sync(0xFFFFFFFFu, down, t4 * 8);
          c2q[n][1] = c2 * __shfl_sync(0xFFFFFFFFu, down, t4 * 8 + 4);
        }
      }
    }
    const uint2* const shared_q = reinterpret_cast<const uint2*>(join) + lane;      // [group][k step][lane]
    if (kShared) {
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) reinterpret_cast<uint2*>(join)[(warp * (D / 16) + ks) * 32 + lane] = make_uint2(qf[0][ks][0], qf[0][ks][1]);
      __syncthreads();
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (!Q) c2q[n][0] = c2q[n][1] = c2;
      if (Q && kShared) {
        c2q[n][0] = c2 * down_of[n * 8 + 2 * t4];
        c2q[n][1] = c2 * down_of[n * 8 + 2 * t4 + 1];
      }
    }
    auto query = [&](int n, int ks, uint32_t& b0, uint32_t& b1) {
      if (kShared) {
        const uint2 x = shared_q[(n * (D / 16) + ks) * 32];
        b0 = x.x;
        b1 = x.y;
      } else {
        b0 = qf[kShared ? 0 : n][ks][0];
        b1 = qf[kShared ? 0 : n][ks][1];
      }
    };
    // how far row r sees; a row that is none sees everything
    auto sees_to = [&](uint32_t r) { return r < n_rows ? first_hi + (int32_t)token_of(r) : 0x7FFFFFFF; };
    // whether row 2t + e of group n does not see a position that it reaches: it lies before its window, or is not in its mask
    auto hidden = [&](int n, int e, int32_t up, int32_t pos) {
      if (CLUSTER) return !(tree[n][e] >> (pos & 15) & 1) || (a.window && up != 0x7FFFFFFF && pos < first_hi && pos < row_low[n * 8 + 2 * t4 + e]);
      if (!TREE) return a.window && up != 0x7FFFFFFF && pos <= up - (int32_t)a.window;
      if (pos >= first_hi) return !(tree[n][e] >> ((pos - first_hi) & 31) & 1);
      // (its own position is first_hi plus the rows that it sees, less one)
      return a.window && up != 0x7FFFFFFF && pos < first_hi + __popc(tree[n][e] & 0xFFFFFFFFu >> (31 - ((up - first_hi) & 31))) - (int32_t)a.window;
    };

    float acc[NT][D / 16][4];
    // the score that the weights are relative to, the score above which it moves, sums; 2^-(f16 exponent), the weight
    // above which it moves.  (Differences are formed before they are scaled: scores of any finite size give weights of 1 and less.)
    float ref[NT][2], thr[NT][2], sum[NT][2], ei[NT][2], lim[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i) acc[n][i][0] = acc[n][i][1] = acc[n][i][2] = acc[n][i][3] = 0.f;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        ref[n][e] = 0.f;
        thr[n][e] = -INFINITY;
        sum[n][e] = ei[n][e] = lim[n][e] = 0.f;
      }
    }

    for (; t < stop; ++t, ++k) {
      const uint32_t slot = k % C::kSlots;
      copies_wait<C::kSlots - 1>();
      __syncwarp();
      const uint32_t sk = base + (warp * C::kSlots + slot) * C::kSlotBytes, sv = sk + C::kPartBytes;
      const int32_t pos0 = (cur.tile0 + t - cur.i0) * (int32_t)kKvTile + (int32_t)(warp * 16);
      // scores: keys lane / 4, + 8 (registers 0 1, 2 3) x rows 2t, 2t + 1
      float sc[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) sc[n][0] = sc[n][1] = sc[n][2] = sc[n][3] = 0.f;
      if (Q) {
#pragma unroll
        for (int ks = 0; ks < D / 16; ks += 2) {
          uint32_t w[4];
          ldsm4(sk + swizzled<C::kSpan>(lane & 15, ks + (lane >> 4)), w);
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint32_t f[4] = {codes_to_f16x2(w[2 * u]), codes_to_f16x2(w[2 * u + 1]), codes_hi_to_f16x2(w[2 * u]), codes_hi_to_f16x2(w[2 * u + 1])};
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              uint32_t b0, b1;
              query(n, ks + u, b0, b1);
              mma16816<true>(sc[n], f, b0, b1);
            }
          }
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          uint32_t w[4];
          ldsm4(sk + (ks >> 2) * 2048 + swizzled<128>(lane & 15, (ks & 3) * 2 + (lane >> 4)), w);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            uint32_t b0, b1;
            query(n, ks, b0, b1);
            mma16816<false>(sc[n], w, b0, b1);
          }
        }
      }
      float vs[2] = {1.f, 1.f};
      if (Q) {
        const float* scales = reinterpret_cast<const float*>(gen + kScaleBase + (warp * C::kSlots + slot) * C::kScaleBytes) + r8;
        const float k0 = scales[0], k1 = scales[8];
        vs[0] = scales[16];
        vs[1] = scales[24];
#pragma unroll
        for (int n = 0; n < NT; ++n) { sc[n][0] *= k0; sc[n][1] *= k0; sc[n][2] *= k1; sc[n][3] *= k1; }
      }
      // rows that some query row does not see, or that lie past the end of the cache
      const bool partial = (TREE ? pos0 + 15 >= first_hi : pos0 + 15 > first_hi) || pos0 < last_lo;
      if (CLUSTER && partial) {
        const int32_t j = pos0 - first_hi;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t r = n * 8 + 2 * t4 + e;
            tree[n][e] = 0xFFFFFFFFu;
            if (r < n_rows && j > -16) {
              const uint32_t t = (uint32_t)cur.row0 + token_of(r);
              tree[n][e] = __funnelshift_r(tree_word(a, t, j >> 5), tree_word(a, t, (j >> 5) + 1), j & 31);
            }
          }
      }
      if (partial) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int32_t up = sees_to(n * 8 + 2 * t4 + e), pos = pos0 + (int32_t)r8;
            if (pos > up || hidden(n, e, up, pos)) sc[n][e] = -INFINITY;
            if (pos + 8 > up || hidden(n, e, up, pos + 8)) sc[n][2 + e] = -INFINITY;
          }
      }
      // a new reference where a weight would pass 2^8
      bool grow = false;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) grow |= fmaxf(sc[n][e], sc[n][2 + e]) > thr[n][e];
      if (__any_sync(0xFFFFFFFFu, grow)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float m = fmaxf(sc[n][e], sc[n][2 + e]);
            m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
            m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
            m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
            if (m > thr[n][e]) {
              const float corr = thr[n][e] == -INFINITY ? 0.f : fast_exp2((ref[n][e] - m) * c2q[n][e]);
              ref[n][e] = m;
              thr[n][e] = fmaxf(m + __fdividef(8.f, c2q[n][e]), -3.0e38f);       // finite: -inf means that nothing was seen yet
              sum[n][e] *= corr;
#pragma unroll
              for (int i = 0; i < D / 16; ++i) { acc[n][i][e] *= corr; acc[n][i][2 + e] *= corr; }
            }
          }
      }
      uint32_t pf[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sc[n][e] = fast_exp2((sc[n][e] - ref[n][e & 1]) * c2q[n][e & 1]);
          sum[n][e & 1] += sc[n][e];
        }
        if (Q) {
          float p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) p[e] = sc[n][e] * vs[e >> 1];
          if (partial) {
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = sc[n][e] == 0.f ? 0.f : p[e];      // a scale of a position that is not seen may be anything
          }
          const float m0 = fmaxf(p[0], p[2]), m1 = fmaxf(p[1], p[3]);
          if (__any_sync(0xFFFFFFFFu, m0 > lim[n][0] || m1 > lim[n][1])) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float m = e ? m1 : m0;
              m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
              m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
              m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
              const uint32_t b = min(max(__float_as_uint(m) >> 23, 1u), 246u), old = __float_as_uint(lim[n][e]) >> 23;
              if (m > lim[n][e] && b + 8 > old) {
                // 2^(old - new); from nothing (old = 0) there is nothing to scale
                const float corr = old == 0 ? 0.f : __uint_as_float((uint32_t)max(127 + (int32_t)old - (int32_t)(b + 8), 0) << 23);
                ei[n][e] = __uint_as_float((254u - b) << 23);
                lim[n][e] = __uint_as_float((b + 8) << 23);
#pragma unroll
                for (int i = 0; i < D / 16; ++i) { acc[n][i][e] *= corr; acc[n][i][2 + e] *= corr; }
              }
            }
          }
          pf[n][0] = transpose8(pack_f16x2(p[0] * ei[n][0], p[1] * ei[n][1]));
          pf[n][1] = transpose8(pack_f16x2(p[2] * ei[n][0], p[3] * ei[n][1]));
        } else {
          pf[n][0] = transpose8(pack_bf16x2(sc[n][0], sc[n][1]));
          pf[n][1] = transpose8(pack_bf16x2(sc[n][2], sc[n][3]));
        }
      }
      // outputs: columns lane / 4, + 8 of 16 (codes: 2 (lane / 4), + 1) x rows 2t, 2t + 1
      if (Q) {
#pragma unroll
        for (int c = 0; c < D / 16; c += 2) {
          uint32_t w[4];
          ldsm4t(sv + swizzled<C::kSpan>(lane & 15, c + (lane >> 4)), w);
          if (partial) {      // a weight of zero must not meet a NaN code: 0x7F becomes 0x7E (its row's scale makes it NaN again)
#pragma unroll
            for (int u = 0; u < 4; ++u) w[u] -= (((w[u] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7;
          }
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint32_t x = __byte_perm(w[2 * u], 0, 0x3120), y = __byte_perm(w[2 * u + 1], 0, 0x3120);
            const uint32_t f[4] = {codes_to_f16x2(x), codes_hi_to_f16x2(x), codes_to_f16x2(y), codes_hi_to_f16x2(y)};
#pragma unroll
            for (int n = 0; n < NT; ++n) mma16816<true>(acc[n][c + u], f, pf[n][0], pf[n][1]);
          }
        }
      } else {
        const uint32_t row = (lane & 7) + ((lane >> 4) << 3);
        // bf16 values of positions that a row does not see are multiplied by a weight of zero, which only finite
        // ones survive: those past the end are cleared, and where the chunk itself or a window cuts the tile, values
        // that are not finite are taken out and added by hand to the rows that do see them
        uint32_t keep[2];
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int32_t pos = pos0 + e * 8 + (int32_t)t4 * 2;
          keep[e] = (pos < cur.len ? 0xFFFFu : 0u) | (pos + 1 < cur.len ? 0xFFFF0000u : 0u);
        }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          uint32_t w[4];
          ldsm4t(sv + (i >> 2) * 2048 + swizzled<128>(row, (i & 3) * 2 + ((lane >> 3) & 1)), w);
          if (partial) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              w[e] &= keep[e >> 1];
              if (not_finite_bf16x2(w[e])) {
                odd = true;
                if ((w[e] & 0x7F80u) == 0x7F80u) w[e] &= 0xFFFF0000u;
                if ((w[e] & 0x7F800000u) == 0x7F800000u) w[e] &= 0xFFFFu;
              }
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n) mma16816<false>(acc[n][i], w, pf[n][0], pf[n][1]);
        }
        if (partial && __any_sync(0xFFFFFFFFu, odd)) {
          const char* vals = gen + (warp * C::kSlots + slot) * C::kSlotBytes + C::kPartBytes;
#pragma unroll 1
          for (int key = 0; key < 16; ++key) {
            const int32_t pos = pos0 + key;
            const int from = (key & 7) * 4 + (int)t4;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float p[2];
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float x = __shfl_sync(0xFFFFFFFFu, sc[n][e], from), y = __shfl_sync(0xFFFFFFFFu, sc[n][2 + e], from);
                p[e] = key < 8 ? x : y;
              }
#pragma unroll
              for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                  const uint32_t d = i * 16 + half * 8 + r8;
                  const uint32_t v = *reinterpret_cast<const uint16_t*>(vals + (d >> 6) * 2048 + swizzled<128>(key, (d >> 3) & 7) + (d & 7) * 2);
                  if ((v & 0x7F80u) != 0x7F80u) continue;
#pragma unroll
                  for (int e = 0; e < 2; ++e) {
                    const int32_t up = sees_to(n * 8 + 2 * t4 + e);
                    if (pos < cur.len && pos <= up && !hidden(n, e, up, pos)) acc[n][i][2 * half + e] += p[e] * __uint_as_float(v << 16);
                  }
                }
            }
          }
        }
      }
      // the slot is read: the tile kSlots on may come
      __syncwarp();
      if (requested < n_tiles) request(requested++);
      copies_commit();
    }

    if (!CLUSTER && t < end) {         // the next item's queries arrive during the join
      enter(it, t);
      fetch_queries(it);
    }

    // ---- join the four warps of the block, in order -------------------------------------------------
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        sum[n][e] += __shfl_xor_sync(0xFFFFFFFFu, sum[n][e], 4);
        sum[n][e] += __shfl_xor_sync(0xFFFFFFFFu, sum[n][e], 8);
        sum[n][e] += __shfl_xor_sync(0xFFFFFFFFu, sum[n][e], 16);
        if (r8 == 0) warp_ml[warp * C::kRows + n * 8 + 2 * t4 + e] = make_float2(thr[n][e] == -INFINITY ? -INFINITY : __fmul_rn(ref[n][e], c2q[n][e]), sum[n][e]);
      }
    __syncthreads();
    float mine[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) m = fmaxf(m, warp_ml[w * C::kRows + n * 8 + 2 * t4 + e].x);
        mine[n][e] = thr[n][e] == -INFINITY ? 1.f : fast_exp2(__fmul_rn(ref[n][e], c2q[n][e]) - m);      // (nothing seen: zeros, or NaN; the product is rounded, as m was)
        if (Q && ei[n][e] != 0.f) mine[n][e] *= lim[n][e] * (1.f / 256.f);
      }
    if (CLUSTER) {
      // a cluster's block is done with its slots, which then have room for the other warps' buffers: one round instead of four, which
      // took 3 us, and four times the code, 48 KiB at 32 rows, which a block that runs it once has to wait for
      static_assert((4 - C::kBuffers) * C::kRows * C::kPitch * 4 <= 4 * C::kSlots * C::kSlotBytes, "");
      float* const buf = warp < C::kBuffers ? join + warp * (C::kRows * C::kPitch) : spare + (warp - C::kBuffers) * (C::kRows * C::kPitch);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t d = Q ? i * 16 + 2 * r8 + (e >> 1) : i * 16 + r8 + 8 * (e >> 1);
            buf[(n * 8 + 2 * t4 + (e & 1)) * C::kPitch + d] = acc[n][i][e] * mine[n][e & 1];
          }
      __syncthreads();
    }
#pragma unroll
    for (uint32_t round = 0; round < (CLUSTER ? 0 : 4 / C::kBuffers); ++round) {
      if (round == warp / C::kBuffers) {
        float* const buf = join + warp % C::kBuffers * (C::kRows * C::kPitch);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t d = Q ? i * 16 + 2 * r8 + (e >> 1) : i * 16 + r8 + 8 * (e >> 1);
              float* at = buf + (n * 8 + 2 * t4 + (e & 1)) * C::kPitch + d;
              const float x = acc[n][i][e] * mine[n][e & 1];
              *at = round == 0 ? x : *at + x;
            }
      }
      __syncthreads();
    }

    // ---- result: whole items directly, cut ones through the workspace ------------------------------
    // a thread owns four columns of every (512 / D)-th row
    constexpr uint32_t kStep = 512 / D;
    const uint32_t d4 = (tid % (D / 4)) * 4, row_first = tid / (D / 4);
    const bool whole = cur.i0 >= begin && cur.i1 <= end;
    auto total_of = [&](uint32_t r, float& m, float& l) {
      m = -INFINITY;
      l = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) m = fmaxf(m, warp_ml[w * C::kRows + r].x);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float2 ml = warp_ml[w * C::kRows + r];
        l += ml.x == -INFINITY ? ml.y : ml.y * fast_exp2(ml.x - m);
      }
    };
    auto joined = [&](uint32_t r) {
      float4 x = *reinterpret_cast<const float4*>(join + r * C::kPitch + d4);
      if (C::kBuffers == 2) {
        const float4 y = *reinterpret_cast<const float4*>(join + (C::kRows + r) * C::kPitch + d4);
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
      }
      return x;
    };
    auto write_row = [&](uint32_t r, float4 o, float m, float l) {
      const uint32_t i = token_of(r), head = (uint32_t)cur.h * a.group + head_of(r, i);
      const uint64_t token = (uint64_t)(cur.row0 + (int32_t)i);
      const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN;
      *reinterpret_cast<uint2*>(a.out + token * a.o_token + head * a.o_head + d4 * 2) =
          make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
      if (a.lse && d4 == 0) a.lse[token * a.n_heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
    };
    if (CLUSTER) {
      if (tid < n_rows) {
        float m, l;
        total_of(tid, m, l);
        block_ml[tid] = make_float2(m, l);
      }
      for (uint32_t r = row_first; r < n_rows; r += kStep) {      // (a thread's own elements; the warps in their order)
        float4 x = *reinterpret_cast<const float4*>(join + r * C::kPitch + d4);
#pragma unroll
        for (uint32_t w = 1; w < 4; ++w) {
          const float4 y = *reinterpret_cast<const float4*>((w < C::kBuffers ? join + w * (C::kRows * C::kPitch) : spare + (w - C::kBuffers) * (C::kRows * C::kPitch)) +
                                                            r * C::kPitch + d4);
          x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
        }
        *reinterpret_cast<float4*>(join + r * C::kPitch + d4) = x;
      }
    } else if (whole) {
      for (uint32_t r = row_first; r < n_rows; r += kStep) {
        float m, l;
        total_of(r, m, l);
        write_row(r, joined(r), m, l);
      }
    } else {
      float* part = a.partials + (size_t)(2 * blockIdx.x + (cur.i0 >= begin ? 1 : 0)) * C::kPartFloats;
      for (uint32_t r = row_first; r < n_rows; r += kStep) {
        float m, l;
        total_of(r, m, l);
        __stcg(reinterpret_cast<float4*>(part + r * D + d4), joined(r));
        if (d4 == 0) {
          __stcg(part + C::kRows * D + r, l == 0.f ? -INFINITY : m);
          __stcg(part + C::kRows * D + C::kRows + r, l);
        }
      }
      if (tid == 0 && cur.i0 >= begin) *cut_item = CutItem{(uint32_t)((cur.i1 - 1) / per - cur.i0 / per) + 1, (uint32_t)cur.row0, (uint32_t)cur.h, n_rows};
    }
    __syncthreads();       // the join buffer is free again
  }

  // ---- the cluster's result: a thread joins four columns of a row over the blocks, in their order -------
  if (CLUSTER) {
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    // (whole warps go through this loop together: its_rows rows of D / 4 threads, in steps of 128)
    for (uint32_t x = rank * 128 + tid; x - lane < its_rows * (D / 4); x += size * 128) {
      const uint32_t r = min(x / (D / 4), its_rows - 1), c = x % (D / 4) * 4, first = lane & ~(D / 4 - 1);      // the row's first lane
      // a lane fetches a block's maximum and sum
      float2 mine = make_float2(-INFINITY, 0.f);
      if (lane - first < size) mine = cluster.map_shared_rank(block_ml, lane - first)[r];
      float top = mine.x;
#pragma unroll
      for (uint32_t d = 8; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
      top = __shfl_sync(0xFFFFFFFFu, top, first);
      const float f_mine = mine.x == -INFINITY ? 1.f : fast_exp2(mine.x - top);        // (nothing seen: NaN, or nothing to add)
      float l = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      float4 y[16];
#pragma unroll
      for (uint32_t k = 0; k < 16; ++k)
        if (k < size) y[k] = *reinterpret_cast<const float4*>(cluster.map_shared_rank(join, k) + r * C::kPitch + c);
#pragma unroll
      for (uint32_t k = 0; k < 16; ++k) {
        const float lk = __shfl_sync(0xFFFFFFFFu, mine.y, first + k), f = __shfl_sync(0xFFFFFFFFu, f_mine, first + k);
        if (k >= size || lk == 0.f) continue;
        l += lk * f;
        o.x += y[k].x * f; o.y += y[k].y * f; o.z += y[k].z * f; o.w += y[k].w * f;
      }
      if (x >= its_rows * (D / 4)) continue;
      const uint32_t i = token_of(r), head = its_h * a.group + head_of(r, i);
      const uint64_t token = (uint64_t)(its.row0 + (int32_t)i);
      const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN;
      *reinterpret_cast<uint2*>(a.out + token * a.o_token + head * a.o_head + c * 2) = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
      if (a.lse && c == 0) a.lse[token * a.n_heads + head] = l == 0.f ? -INFINITY : (top + log2f(l)) * kLn2;
    }
    cluster.sync();        // nobody's memory goes before all have read it
  }
}

// Joins the items that blocks' shares cut: block (x, y) takes four rows of the item that is cut first in block x.  A kernel of its
// own: the last block to finish an item would have to find that out (a fence and an atomic) and read all parts alone, a
// single token over 4097 positions took 15.9 us, with this 13.3.  A warp joins every eighth part, and the warps' results are joined in order.
template <int D, int NT>
__global__ void __launch_bounds__(256) wb_attend_join_rows_kernel(const __grid_constant__ AttendArgs a) {
  constexpr uint32_t kRows = 8 * NT, kPart = kRows * D + 2 * kRows;
  constexpr uint32_t kLanes = D / 4, kAtOnce = 32 / kLanes, kG = 4 / kAtOnce;      // a lane owns four columns of kG rows
  __shared__ float4 sums[8][4][kLanes];
  __shared__ float2 ml[8][4];
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, c = lane % kLanes, r0 = blockIdx.y * 4;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const CutItem it = reinterpret_cast<const CutItem*>(a.cuts)[blockIdx.x];       // (parts, first row, kv head, rows)
  if (r0 >= it.rb || !it.parts) return;
  const float* const parts = a.partials + (size_t)2 * blockIdx.x * kPart;
  float4 o[kG];
  float m[kG], l[kG];
#pragma unroll
  for (uint32_t g = 0; g < kG; ++g) {
    o[g] = make_float4(0.f, 0.f, 0.f, 0.f);
    m[g] = -INFINITY;
    l[g] = 0.f;
  }
#pragma unroll 4
  for (uint32_t p = warp; p < it.parts; p += 8) {
    const float* src = parts + (size_t)(2 * p + (p == 0 ? 1 : 0)) * kPart;
#pragma unroll
    for (uint32_t g = 0; g < kG; ++g) {
      const uint32_t r = min(r0 + g * kAtOnce + lane / kLanes, it.rb - 1);
      const float mp = src[kRows * D + r], lp = src[kRows * D + kRows + r], next = fmaxf(m[g], mp);
      const float4 x = *reinterpret_cast<const float4*>(src + r * D + c * 4);
      const float f = m[g] == -INFINITY ? 1.f : fast_exp2(m[g] - next), h = mp == -INFINITY ? 1.f : fast_exp2(mp - next);   // (nothing seen: zeros, or NaN)
      o[g].x = o[g].x * f + x.x * h; o[g].y = o[g].y * f + x.y * h; o[g].z = o[g].z * f + x.z * h; o[g].w = o[g].w * f + x.w * h;
      l[g] = l[g] * f + lp * h;
      m[g] = next;
    }
  }
#pragma unroll
  for (uint32_t g = 0; g < kG; ++g) {
    sums[warp][g * kAtOnce + lane / kLanes][c] = o[g];
    if (c == 0) ml[warp][g * kAtOnce + lane / kLanes] = make_float2(m[g], l[g]);
  }
  __syncthreads();
  const uint32_t i = tid / kLanes, r = r0 + i;      // now a thread owns four columns of one row
  if (i >= 4 || r >= it.rb) return;
  float top = -INFINITY, all = 0.f;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int w = 0; w < 8; ++w) top = fmaxf(top, ml[w][i].x);
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    const float2 part = ml[w][i];
    const float f = part.x == -INFINITY ? 1.f : fast_exp2(part.x - top);
    const float4 y = sums[w][i][c % kLanes];
    all += part.y * f;
    x.x += y.x * f; x.y += y.y * f; x.z += y.z * f; x.w += y.w * f;
  }
  const float inv = all > 0.f ? 1.f / all : all == 0.f ? 0.f : NAN;
  const uint32_t token = r / a.group, head = it.h * a.group + r - token * a.group;
  const uint64_t row = (uint64_t)it.s + token;
  *reinterpret_cast<uint2*>(a.out + row * a.o_token + head * a.o_head + c * 8) = make_uint2(pack_bf16x2(x.x * inv, x.y * inv), pack_bf16x2(x.z * inv, x.w * inv));
  if (a.lse && c == 0) a.lse[row * a.n_heads + head] = all == 0.f ? -INFINITY : (top + log2f(all)) * kLn2;
}

}  // namespace wbi
