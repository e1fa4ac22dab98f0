// Attention for many rows: a block holds 256 rows (new token x query head of one kv head, as two tiles of 128) of a
// sequence against 128 cache rows at a time.  Scores and the weighted sum of values are tcgen05 products with fp32
// accumulators in tensor memory; the bound is the tensor core, with the exponentials close behind.
//
//   - Tensor memory (512 columns): scores of tile 0 and 1 (128 each), outputs of tile 0 and 1 (D each).  A tile's weights
//     replace its scores as bf16, and enter the second product from there.
//   - Warps 0-3 and 4-7 are the softmax of tile 0 and tile 1, one thread per row: no exchange between threads.  While
//     one tile's weights are computed, the tensor core works for the other.
//   - A row's outputs are rescaled only when its maximum has grown by more than 2^8: weights stay below 256, where
//     bf16's relative precision is the same, and sums are fp32 in either case.
//   - One warp issues all products in the order  QK0 QK1 | PV0 QK0' PV1 QK1' | ..., one requests cache tiles into a
//     ring of slots (keys, values, keys, ...) by tensor-map loads, a box per page piece.
//   - E4M3 caches: tiles arrive as codes, four more warps widen them to bf16 slots; the row scales multiply scores and
//     weights in the softmax, where each is a value of its own.
//   - Work is cut as in the kernel for few rows: one line of 128-row tiles over all (sequence, kv head, row block)
//     items, an equal share for every SM, cut items joined in order by the block that ends last.
#pragma once
#include "wb_attend.cuh"

namespace wbi {

constexpr uint32_t kQRows = 256;       // rows of a block
constexpr uint32_t kKeys = 128;        // cache rows of a step

template <int D, bool Q>
struct TilesCfg {
  static constexpr uint32_t kSpans = D / 64;                       // 128-byte spans of a bf16 row
  static constexpr uint32_t kSpanBytes = kKeys * 128;              // one span of 128 rows
  static constexpr uint32_t kSlotBytes = kSpans * kSpanBytes;      // a bf16 tile of keys or values
  static constexpr uint32_t kQBytes = 2 * kSlotBytes;
  static constexpr uint32_t kSlots = Q ? (D == 128 ? 4 : 6) : (D == 128 ? 5 : 10);
  static constexpr uint32_t kRawBytes = Q ? kKeys * D : 0;         // a tile of codes
  static constexpr uint32_t kRaws = Q && D == 64 ? 4 : 2;
  static constexpr uint32_t kScaleSlots = 4;                       // 128 scales each; keys and values in turn
  static constexpr uint32_t kRowSpan = D * (Q ? 1 : 2) < 128 ? D * (Q ? 1 : 2) : 128;   // bytes of a row in a box
  static constexpr uint32_t kRowSpans = D * (Q ? 1 : 2) / kRowSpan;
  static constexpr uint32_t kThreads = Q ? 512 : 384;
  // registers: the compiler gives every thread kLaunchRegs; the softmax warps take over what the others leave
  // (256 * kSoftmaxRegs + (kThreads - 256) * kOtherRegs = kThreads * kLaunchRegs)
  static constexpr int kLaunchRegs = Q ? 128 : 168, kSoftmaxRegs = Q ? 192 : 208, kOtherRegs = Q ? 64 : 88;
  static_assert(256 * kSoftmaxRegs + ((int)kThreads - 256) * kOtherRegs <= (int)kThreads * kLaunchRegs, "");
  static constexpr uint32_t kMaxSeqs = Q ? 128 : 512;              // sequences of a launch (prefix sums in shared memory)
  static constexpr uint32_t kPartFloats = 2 * (D * 128 + 256);
  static constexpr uint32_t kOffSlots = kQBytes;
  static constexpr uint32_t kOffRaw = kOffSlots + kSlots * kSlotBytes;
  static constexpr uint32_t kOffScale = kOffRaw + kRaws * kRawBytes;
  static constexpr uint32_t kOffBars = kOffScale + (Q ? kScaleSlots * kKeys * 4 : 0);
  static constexpr uint32_t kBars = 1 + 6 + 2 * kSlots + (Q ? 2 * kRaws + 2 * kScaleSlots : 0);
  static constexpr uint32_t kOffMisc = kOffBars + kBars * 8;       // tensor memory address, last flag, odd flags
  static constexpr uint32_t kOffCum = kOffMisc + 32;
  static constexpr uint32_t kSmemBytes = kOffCum + (kMaxSeqs + 1) * 4;
  static_assert(kSmemBytes <= 232448, "");
};

// ---- tcgen05 ------------------------------------------------------------------------------------
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }"
               ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
#define WB_R32(r) "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), \
    "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), \
    "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
#define WB_W32(r) "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), \
    "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), \
    "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
// 32 columns of the warp's 32 lanes
__device__ __forceinline__ void tm_load32(uint32_t addr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
               "%24,%25,%26,%27,%28,%29,%30,%31}, [%32];" : WB_W32(r) : "r"(addr));
}
__device__ __forceinline__ void tm_store32(uint32_t addr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
               "%24,%25,%26,%27,%28,%29,%30,%31};" ::WB_R32(r), "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Shared-memory matrix descriptor, 128-byte swizzle: groups of eight 128-byte rows, 1024 bytes apart; `lead` is the distance
// of the next 128 bytes of a row (used where rows run along the operand's M or N).
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t r, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// ---- geometry -----------------------------------------------------------------------------------
struct RowBlock {
  int32_t kt0, n;          // first tile of 128 cache rows, number of tiles (at least one)
};
__device__ __forceinline__ RowBlock row_block(const KvSeq& q, uint32_t group, uint32_t window, uint32_t rb) {
  const uint32_t rows = (uint32_t)q.n_new * group, r0 = rb * kQRows, r1 = min(r0 + kQRows, rows);
  const int32_t base = q.len - q.n_new;
  const int32_t hi = base + (int32_t)((r1 - 1) / group);
  const int32_t lo = window ? max(0, base + (int32_t)(r0 / group) - (int32_t)window + 1) : 0;
  RowBlock b;
  b.kt0 = lo / (int32_t)kKeys;
  b.n = max(1, (hi + (int32_t)kKeys) / (int32_t)kKeys - b.kt0);
  return b;
}
__device__ __forceinline__ uint32_t row_blocks(const KvSeq& q, uint32_t group, uint32_t skip_rows) {
  const uint64_t rows = (uint64_t)q.n_new * group;
  return rows > skip_rows ? (uint32_t)((rows + kQRows - 1) / kQRows) : 0;
}

// Where a block is in the line of tiles; every warp walks it alike.
struct Walk {
  uint32_t s, h, rb, n_rb;
  KvSeq seq;
  RowBlock blk;
  int32_t item0;           // the item's first tile in the line
};

__device__ __forceinline__ int32_t warp_inclusive(int32_t x) {
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int32_t o = __shfl_up_sync(0xFFFFFFFFu, x, d);
    if ((int)(threadIdx.x & 31) >= d) x += o;
  }
  return x;
}

// The item that holds tile t; by a whole warp.
__device__ __forceinline__ Walk walk_to(const AttendArgs& a, const int32_t* cum, uint32_t skip_rows, int32_t t) {
  Walk w;
  uint32_t lo = 0, hi = a.b.n_seqs;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) >> 1;
    if (cum[mid] <= t) lo = mid; else hi = mid;
  }
  while (cum[lo + 1] <= t) ++lo;
  w.s = lo;
  w.seq = attend_seq(a.b, lo);
  w.n_rb = row_blocks(w.seq, a.group, skip_rows);
  const int32_t per_head = (cum[lo + 1] - cum[lo]) / (int32_t)a.c.n_kv_heads;
  const int32_t local = t - cum[lo];
  w.h = (uint32_t)(local / per_head);
  int32_t rem = local - (int32_t)w.h * per_head;
  const uint32_t lane = threadIdx.x & 31;
  for (uint32_t rb0 = 0;; rb0 += 32) {
    const uint32_t rb = rb0 + lane;
    const int32_t n = rb < w.n_rb ? row_block(w.seq, a.group, a.window, rb).n : 0;
    const int32_t inc = warp_inclusive(n);
    const uint32_t over = __ballot_sync(0xFFFFFFFFu, inc > rem);
    if (over || rb0 + 32 >= w.n_rb) {
      const int l = over ? __ffs(over) - 1 : 31;
      w.rb = min(rb0 + (uint32_t)l, w.n_rb - 1);
      rem -= __shfl_sync(0xFFFFFFFFu, inc - n, l);
      break;
    }
    rem -= __shfl_sync(0xFFFFFFFFu, inc, 31);
  }
  w.blk = row_block(w.seq, a.group, a.window, w.rb);
  w.item0 = t - rem;
  return w;
}
__device__ __forceinline__ void walk_on(Walk& w, const AttendArgs& a, const int32_t* cum, uint32_t skip_rows) {
  w.item0 += w.blk.n;
  if (++w.rb == w.n_rb) {
    w.rb = 0;
    if (++w.h == a.c.n_kv_heads) {
      w.h = 0;
      do ++w.s; while (cum[w.s + 1] == cum[w.s]);
      w.seq = attend_seq(a.b, w.s);
      w.n_rb = row_blocks(w.seq, a.group, skip_rows);
    }
  }
  w.blk = row_block(w.seq, a.group, a.window, w.rb);
}

// Values that are not finite were taken out of a tile some rows of which do not see them: a row that does see one has it
// added here (its weight is positive, whatever it is).  Rare, so straight from the cache.
__device__ __noinline__ void add_odd_values(const AttendArgs& a, const Walk& w, int32_t kt_begin, int32_t kt_end, int32_t lo, int32_t hi,
                                            int32_t cut_hi, int32_t cut_lo, uint32_t d0, float* o) {
  for (int32_t kt = kt_begin; kt < kt_end; ++kt) {
    if (!(kt * (int32_t)kKeys + (int32_t)kKeys - 1 > cut_hi || kt * (int32_t)kKeys < cut_lo)) continue;
    for (int32_t pos = max(lo, kt * (int32_t)kKeys); pos <= min(hi, kt * (int32_t)kKeys + (int32_t)kKeys - 1); ++pos) {
      const int32_t page = kv_page(a.b, a.c.n_pages, a.c.page_size, w.s, pos);
      if (page < 0) continue;
      const uint16_t* v = reinterpret_cast<const uint16_t*>(a.c.v) + (uint64_t)page * a.c.page_stride + w.h * a.c.head_stride +
                          ((uint32_t)pos % a.c.page_size) * a.c.head_dim + d0;
      for (int d = 0; d < 32; ++d)
        if ((v[d] & 0x7F80u) == 0x7F80u) o[d] += __uint_as_float((uint32_t)v[d] << 16);
    }
  }
}

template <int D, bool Q>
__global__ void __launch_bounds__(TilesCfg<D, Q>::kThreads, 1)
wb_attend_tiles_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                       uint32_t skip_rows) {
  using C = TilesCfg<D, Q>;
  extern __shared__ __align__(1024) char smem[];
  const uint32_t base = smem_addr(smem);
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t bars = base + C::kOffBars;
  const uint32_t q_full = bars, s_full = bars + 8, p_full = bars + 24, o_full = bars + 40, full = bars + 56, empty = full + 8 * C::kSlots,
                 raw_full = empty + 8 * C::kSlots, raw_empty = raw_full + 8 * C::kRaws, scale_full = raw_empty + 8 * C::kRaws,
                 scale_empty = scale_full + 8 * C::kScaleSlots;
  volatile uint32_t* const misc = reinterpret_cast<volatile uint32_t*>(smem + C::kOffMisc);   // [0] tensor memory, [1] last, [2..4] odd
  int32_t* const cum = reinterpret_cast<int32_t*>(smem + C::kOffCum);
  if (base & 1023u) {      // swizzled tiles need it; never the case without static shared memory
    if (tid == 0) atomicMax(a.error, 2u);
    return;
  }

  // ---- the line of tiles -----------------------------------------------------------------------------
  const uint32_t n_seqs = a.b.n_seqs, hk = a.c.n_kv_heads;
  if (tid == 0) {
    cum[0] = 0;
    bar_init(q_full, 256);
    for (uint32_t i = 0; i < 2; ++i) {
      bar_init(s_full + 8 * i, 1);
      bar_init(p_full + 8 * i, 128);
      bar_init(o_full + 8 * i, 1);
    }
    for (uint32_t i = 0; i < C::kSlots; ++i) {
      bar_init(full + 8 * i, Q ? 128 : 32);
      bar_init(empty + 8 * i, 1);
    }
    if (Q) {
      for (uint32_t i = 0; i < C::kRaws; ++i) {
        bar_init(raw_full + 8 * i, 32);
        bar_init(raw_empty + 8 * i, 128);
      }
      for (uint32_t i = 0; i < C::kScaleSlots; ++i) {
        bar_init(scale_full + 8 * i, 32);
        bar_init(scale_empty + 8 * i, 256);
      }
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    misc[2] = misc[3] = misc[4] = 0;
  }
  for (uint32_t s = warp; s < n_seqs; s += C::kThreads / 32) {
    const KvSeq q = attend_seq(a.b, s);
    const uint32_t nb = row_blocks(q, a.group, skip_rows);
    int32_t sum = 0;
    for (uint32_t rb = lane; rb < nb; rb += 32) sum += row_block(q, a.group, a.window, rb).n;
    sum = __reduce_add_sync(0xFFFFFFFFu, sum);
    if (lane == 0) cum[s + 1] = sum * (int32_t)hk;
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(base + C::kOffMisc) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  __syncthreads();
  if (warp == 0) {
    int32_t before = 0;
    for (uint32_t s0 = 0; s0 < n_seqs; s0 += 32) {
      const uint32_t s = s0 + lane;
      const int32_t inc = warp_inclusive(s < n_seqs ? cum[s + 1] : 0);
      if (s < n_seqs) cum[s + 1] = before + inc;
      before += __shfl_sync(0xFFFFFFFFu, inc, 31);
    }
  }
  tc_before();
  __syncthreads();
  tc_after();
  const uint32_t tmem = misc[0];
  const int32_t total = cum[n_seqs];
  const int32_t per = (total + (int32_t)gridDim.x - 1) / (int32_t)gridDim.x;
  const int32_t begin = min((int32_t)blockIdx.x * per, total), end = min(begin + per, total);

  if (begin < end) {
    if (warp < 8) {
      // ---- softmax: one thread per row ---------------------------------------------------------------
      asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kSoftmaxRegs));
      const uint32_t i = warp >> 2, row = tid & 127;
      const uint32_t tm_lane = tmem + ((warp & 3) << 21);
      const uint32_t tm_s = tm_lane + i * 128, tm_o = tm_lane + 256 + i * 128;
      const float c2 = a.scale_log2;
      uint32_t jg = 0, item = 0;                    // steps and items so far
      bool ok = true;
      Walk w = walk_to(a, cum, skip_rows, begin);
      for (int32_t t = begin; t < end; ++item) {
        const int32_t item1 = w.item0 + w.blk.n, stop = min(end, item1);
        const uint32_t n_rows = (uint32_t)w.seq.n_new * a.group, r = w.rb * kQRows + i * 128 + row;
        const bool in = r < n_rows;
        const uint32_t tok = (in ? r : n_rows - 1) / a.group;
        const uint32_t head = w.h * a.group + (in ? r - tok * a.group : 0);
        const int32_t base_pos = w.seq.len - w.seq.n_new;
        const int32_t hi = base_pos + (int32_t)tok, lo = a.window ? hi - (int32_t)a.window + 1 : 0;
        const int32_t cut_hi = base_pos + (int32_t)(w.rb * kQRows / a.group);
        const int32_t cut_lo = a.window ? base_pos + (int32_t)((min(n_rows, (w.rb + 1) * kQRows) - 1) / a.group) - (int32_t)a.window + 1 : 0;
        if (tid == 0) misc[2 + (item + 1) % 3] = 0;
        // the row's query, swizzled as the products read it
        {
          const uint4* src = reinterpret_cast<const uint4*>(a.q + (uint64_t)(w.seq.row0 + (int32_t)tok) * a.q_token + head * a.q_head);
          char* dst = smem + i * C::kSlotBytes;
#pragma unroll
          for (uint32_t c = 0; c < D / 8; ++c) {
            const uint4 x = in ? __ldg(src + c) : make_uint4(0, 0, 0, 0);
            *reinterpret_cast<uint4*>(dst + (c >> 3) * C::kSpanBytes + row * 128 + (((c & 7) ^ (row & 7)) << 4)) = x;
          }
          fence_async();
          tc_before();
          bar_arrive(q_full);
        }
        float mref = -INFINITY;                     // the maximum that the weights are relative to, times c2
        uint64_t sum2 = 0;
        for (bool first = true; t < stop; ++t, ++jg, first = false) {
          const int32_t kt = w.blk.kt0 + t - w.item0;
          const int32_t pos0 = kt * (int32_t)kKeys;
          const bool cut = pos0 + (int32_t)kKeys - 1 > cut_hi || pos0 < cut_lo;
          uint32_t x[128];
          ok = wait_or_give_up(s_full + 8 * i, jg & 1, ok, a.error);
          tc_after();
          tm_load32(tm_s, x);
          tm_load32(tm_s + 32, x + 32);
          tm_load32(tm_s + 64, x + 64);
          tm_load32(tm_s + 96, x + 96);
          tm_wait_load();
          const float4* kscale = nullptr;
          const float4* vscale = nullptr;
          if (Q) {
            const uint32_t sk = (2 * jg) % C::kScaleSlots;
            ok = wait_or_give_up(scale_full + 8 * sk, (2 * jg / C::kScaleSlots) & 1, ok, a.error);
            kscale = reinterpret_cast<const float4*>(smem + C::kOffScale + sk * (kKeys * 4));
            vscale = reinterpret_cast<const float4*>(smem + C::kOffScale + (sk + 1) * (kKeys * 4));
#pragma unroll
            for (int c = 0; c < 32; ++c) {
              const float4 f = kscale[c];
              x[4 * c] = __float_as_uint(__uint_as_float(x[4 * c]) * f.x);
              x[4 * c + 1] = __float_as_uint(__uint_as_float(x[4 * c + 1]) * f.y);
              x[4 * c + 2] = __float_as_uint(__uint_as_float(x[4 * c + 2]) * f.z);
              x[4 * c + 3] = __float_as_uint(__uint_as_float(x[4 * c + 3]) * f.w);
            }
          }
          if (cut) {
            const int32_t h1 = hi - pos0, l1 = lo - pos0;
#pragma unroll
            for (int c = 0; c < 128; ++c)
              if (c > h1 || c < l1) x[c] = 0xFF800000u;
          }
          float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int c = 0; c < 128; c += 4)
#pragma unroll
            for (int e = 0; e < 4; ++e) m4[e] = fmaxf(m4[e], __uint_as_float(x[c + e]));
          const float m = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * c2;
          const bool grow = m > mref + 8.f;
          float corr = 1.f;
          if (grow) {
            corr = mref == -INFINITY ? 0.f : fast_exp2(mref - m);
            mref = m;
          }
          // the step's commit covered the previous product, so nothing writes the outputs now
          if (!first && __any_sync(0xFFFFFFFFu, grow)) {
#pragma unroll
            for (int c = 0; c < D; c += 32) {
              uint32_t o[32];
              tm_load32(tm_o + c, o);
              tm_wait_load();
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * corr);
              tm_store32(tm_o + c, o);
            }
          }
          if (Q) ok = wait_or_give_up(scale_full + 8 * ((2 * jg + 1) % C::kScaleSlots), ((2 * jg + 1) / C::kScaleSlots) & 1, ok, a.error);
          sum2 = mul2(sum2, pack2(corr, corr));
          const float ref = mref == -INFINITY ? 0.f : mref;
          const uint64_t c22 = pack2(c2, c2), ref2 = pack2(-ref, -ref);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            uint32_t p[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const int c = half * 64 + 2 * e;
              float u, v;
              unpack2(fma2(pack2(__uint_as_float(x[c]), __uint_as_float(x[c + 1])), c22, ref2), u, v);
              u = fast_exp2(u);
              v = fast_exp2(v);
              sum2 = add2(sum2, pack2(u, v));
              if (Q) {
                const float2 f = reinterpret_cast<const float2*>(vscale)[half * 32 + e];
                // a scale of a position that is not seen may be anything
                u = cut && u == 0.f ? 0.f : u * f.x;
                v = cut && v == 0.f ? 0.f : v * f.y;
              }
              p[e] = pack_bf16x2(u, v);
            }
            tm_store32(tm_s + half * 32, p);
          }
          if (!Q && cut) {
            // values past the end, and values that are not finite, must not meet weights of zero
            const uint32_t vq = 2 * jg + 1, slot = vq % C::kSlots;
            ok = wait_or_give_up(full + 8 * slot, (vq / C::kSlots) & 1, ok, a.error);
            char* v = smem + C::kOffSlots + slot * C::kSlotBytes + row * 128;
            const bool past = pos0 + (int32_t)row >= w.seq.len;
#pragma unroll 1
            for (uint32_t c = 0; c < D / 8; ++c) {
              uint4* at = reinterpret_cast<uint4*>(v + (c >> 3) * C::kSpanBytes + (((c & 7) ^ (row & 7)) << 4));
              uint4 y = *at;
              uint32_t* yw = reinterpret_cast<uint32_t*>(&y);
              bool odd = false;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if ((yw[e] & 0x7F80u) == 0x7F80u) { odd = true; yw[e] &= 0xFFFF0000u; }
                if ((yw[e] & 0x7F800000u) == 0x7F800000u) { odd = true; yw[e] &= 0xFFFFu; }
              }
              if (past) {
                *at = make_uint4(0, 0, 0, 0);
              } else if (odd) {
                misc[2 + item % 3] = 1;      // before the value goes: whoever finds it gone finds the flag
                __threadfence_block();
                *at = y;
              }
            }
            fence_async();
          }
          tm_wait_store();
          tc_before();
          bar_arrive(p_full + 8 * i);
          if (Q) {
            bar_arrive(scale_empty + 8 * ((2 * jg) % C::kScaleSlots));
            bar_arrive(scale_empty + 8 * ((2 * jg + 1) % C::kScaleSlots));
          }
        }
        // ---- outputs ---------------------------------------------------------------------------------
        float l, l1;
        unpack2(sum2, l, l1);
        l += l1;
        ok = wait_or_give_up(o_full + 8 * i, item & 1, ok, a.error);
        tc_after();
        const int32_t from = max(w.item0, begin);
        const bool odd = !Q && misc[2 + item % 3] != 0;
        const bool whole = w.item0 >= begin && item1 <= end;
        char* dst = a.out + (uint64_t)(w.seq.row0 + (int32_t)tok) * a.o_token + head * a.o_head;
        float* lse = a.lse ? a.lse + (uint64_t)(w.seq.row0 + (int32_t)tok) * a.n_heads + head : nullptr;
        float* part = a.partials + (size_t)(2 * blockIdx.x + (w.item0 >= begin ? 1 : 0)) * C::kPartFloats + i * (D * 128 + 256) + row;
        const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t o[32];
          tm_load32(tm_o + c, o);
          tm_wait_load();
          if (odd && in) {
            float y[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) y[e] = __uint_as_float(o[e]);
            add_odd_values(a, w, w.blk.kt0 + from - w.item0, w.blk.kt0 + stop - w.item0, lo, hi, cut_hi, cut_lo, c, y);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(y[e]);
          }
          if (whole) {
            if (in)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                uint32_t y[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  y[k] = pack_bf16x2(__uint_as_float(o[8 * e + 2 * k]) * inv, __uint_as_float(o[8 * e + 2 * k + 1]) * inv);
                *reinterpret_cast<uint4*>(dst + (c + 8 * e) * 2) = make_uint4(y[0], y[1], y[2], y[3]);
              }
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) __stcg(part + (c + e) * 128, __uint_as_float(o[e]));
          }
        }
        tc_before();       // the outputs' columns may be written again once every thread has arrived for the next item
        if (whole) {
          if (in && lse) *lse = l == 0.f ? -INFINITY : (mref + log2f(l)) * kLn2;
        } else {
          __stcg(part + D * 128, l == 0.f ? -INFINITY : mref);
          __stcg(part + D * 128 + 128, l);
          __threadfence();
          asm volatile("bar.sync 1, 256;" ::: "memory");
          const uint32_t first = (uint32_t)(w.item0 / per), count = (uint32_t)((item1 - 1) / per) - first + 1;
          if (tid == 0) {
            __threadfence();
            const bool last = atomicAdd(a.counters + first, 1u) == count - 1;
            if (last) a.counters[first] = 0;
            misc[1] = last;
          }
          asm volatile("bar.sync 1, 256;" ::: "memory");
          if (misc[1]) {
            __threadfence();
            const float* parts = a.partials + i * (D * 128 + 256) + row;
            auto part_of = [&](uint32_t p) { return parts + (size_t)(2 * (first + p) + (p == 0 ? 1 : 0)) * C::kPartFloats; };
            float top = -INFINITY, all = 0.f;
            for (uint32_t p = 0; p < count; ++p) top = fmaxf(top, __ldcg(part_of(p) + D * 128));
            for (uint32_t p = 0; p < count; ++p) {
              const float mp = __ldcg(part_of(p) + D * 128);
              all += __ldcg(part_of(p) + D * 128 + 128) * (mp == -INFINITY ? 0.f : fast_exp2(mp - top));
            }
            const float scale = all > 0.f ? 1.f / all : all == 0.f ? 0.f : NAN;
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              float o[32] = {};
#pragma unroll 1
              for (uint32_t p = 0; p < count; ++p) {
                const float* src = part_of(p);
                const float mp = __ldcg(src + D * 128), f = mp == -INFINITY ? 0.f : fast_exp2(mp - top);
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] += f * __ldcg(src + (c + e) * 128);
              }
              if (in)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  uint32_t y[4];
#pragma unroll
                  for (int k = 0; k < 4; ++k) y[k] = pack_bf16x2(o[8 * e + 2 * k] * scale, o[8 * e + 2 * k + 1] * scale);
                  *reinterpret_cast<uint4*>(dst + (c + 8 * e) * 2) = make_uint4(y[0], y[1], y[2], y[3]);
                }
            }
            if (in && lse) *lse = all == 0.f ? -INFINITY : (top + log2f(all)) * kLn2;
          }
        }
        if (t < end) walk_on(w, a, cum, skip_rows);
      }
    } else if (warp < 12) {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kOtherRegs));
      if (warp == 8) {
        // ---- products: one lane issues them all --------------------------------------------------------
        Walk w = walk_to(a, cum, skip_rows, begin);
        if (lane == 0) {
          constexpr uint32_t kF32Bf16 = 1u << 4 | 1u << 7 | 1u << 10 | 8u << 24;
          constexpr uint32_t kQk = kF32Bf16 | (kKeys / 8) << 17, kPv = kF32Bf16 | 1u << 16 | (uint32_t)(D / 8) << 17;
          uint32_t jg = 0, item = 0;
          bool ok = true;
          auto slot_wait = [&](uint32_t q) {
            const uint32_t slot = q % C::kSlots;
            ok = wait_or_give_up(full + 8 * slot, (q / C::kSlots) & 1, ok, a.error);
            return base + C::kOffSlots + slot * C::kSlotBytes;
          };
          auto scores = [&](uint32_t i, uint32_t k_addr) {
#pragma unroll
            for (uint32_t ks = 0; ks < D / 16; ++ks) {
              const uint32_t off = (ks >> 2) * C::kSpanBytes + (ks & 3) * 32;
              tc_mma_ss(tmem + i * 128, smem_desc(base + i * C::kSlotBytes + off, 16), smem_desc(k_addr + off, 16), kQk, ks > 0);
            }
          };
          auto values = [&](uint32_t i, uint32_t v_addr, bool add) {
#pragma unroll
            for (uint32_t ks = 0; ks < kKeys / 16; ++ks)
              tc_mma_ts(tmem + 256 + i * 128, tmem + i * 128 + ks * 8, smem_desc(v_addr + ks * 2048, C::kSpanBytes), kPv, add || ks > 0);
          };
          for (int32_t t = begin; t < end; ++item) {
            const int32_t stop = min(end, w.item0 + w.blk.n);
            ok = wait_or_give_up(q_full, item & 1, ok, a.error);
            tc_after();
            uint32_t k_addr = slot_wait(2 * jg);
            tc_after();
            scores(0, k_addr);
            tc_commit(s_full);
            scores(1, k_addr);
            tc_commit(s_full + 8);
            tc_commit(empty + 8 * ((2 * jg) % C::kSlots));
            for (bool first = true; t < stop; ++t, ++jg, first = false) {
              const uint32_t v_addr = slot_wait(2 * jg + 1);
              const bool more = t + 1 < stop;
              ok = wait_or_give_up(p_full, jg & 1, ok, a.error);
              tc_after();
              values(0, v_addr, !first);
              if (more) {
                k_addr = slot_wait(2 * jg + 2);
                scores(0, k_addr);
                tc_commit(s_full);
              } else {
                tc_commit(o_full);
              }
              ok = wait_or_give_up(p_full + 8, jg & 1, ok, a.error);
              tc_after();
              values(1, v_addr, !first);
              tc_commit(empty + 8 * ((2 * jg + 1) % C::kSlots));
              if (more) {
                scores(1, k_addr);
                tc_commit(s_full + 8);
                tc_commit(empty + 8 * ((2 * jg + 2) % C::kSlots));
              } else {
                tc_commit(o_full + 8);
              }
            }
            if (t < end) walk_on(w, a, cum, skip_rows);
          }
        }
        __syncwarp();
      } else if (warp == 9) {
        // ---- cache tiles: one lane per page piece ------------------------------------------------------
        const uint32_t pieces = kKeys / a.box_rows;
        uint32_t jg = 0;
        bool ok = true;
        Walk w = walk_to(a, cum, skip_rows, begin);
        for (int32_t t = begin; t < end;) {
          const int32_t stop = min(end, w.item0 + w.blk.n);
          for (; t < stop; ++t, ++jg) {
            const int32_t pos = (w.blk.kt0 + t - w.item0) * (int32_t)kKeys + (int32_t)(lane * a.box_rows);
            int32_t page = -1;
            if (lane < pieces && pos < w.seq.len) page = kv_page(a.b, a.c.n_pages, a.c.page_size, w.s, pos);
            const uint32_t in_page = (uint32_t)pos % a.c.page_size, r0 = lane * a.box_rows;
            const int32_t where = page < 0 ? (int32_t)a.c.n_pages : page;      // outside the cache: zeros
#pragma unroll
            for (uint32_t kv = 0; kv < 2; ++kv) {
              const uint32_t q = 2 * jg + kv, ring = Q ? C::kRaws : C::kSlots, slot = q % ring;
              const uint32_t bar = (Q ? raw_full : full) + 8 * slot;
              if (q >= ring) ok = wait_or_give_up((Q ? raw_empty : empty) + 8 * slot, (q / ring + 1) & 1, ok, a.error);
              const uint32_t sc = q % C::kScaleSlots;
              if (Q && q >= C::kScaleSlots) ok = wait_or_give_up(scale_empty + 8 * sc, (q / C::kScaleSlots + 1) & 1, ok, a.error);
              const uint32_t dst = base + (Q ? C::kOffRaw + slot * C::kRawBytes : C::kOffSlots + slot * C::kSlotBytes);
              if (lane < pieces) {
                bar_arrive_tx(bar, a.box_rows * D * (Q ? 1 : 2));
#pragma unroll
                for (uint32_t e = 0; e < C::kRowSpans; ++e)
                  load_box(dst + e * (kKeys * C::kRowSpan) + r0 * C::kRowSpan, kv ? &map_v : &map_k, (int32_t)(e * 64), (int32_t)in_page, (int32_t)w.h, where, bar);
                if (Q && page >= 0) {
                  bar_arrive_tx(scale_full + 8 * sc, a.box_rows * 4);
                  load_bulk(base + C::kOffScale + (sc * kKeys + r0) * 4, (kv ? a.c.v_scale : a.c.k_scale) + ((uint64_t)page * hk + w.h) * a.c.page_size + in_page,
                            a.box_rows * 4, scale_full + 8 * sc);
                } else if (Q) {
                  for (uint32_t e = 0; e < a.box_rows; ++e) reinterpret_cast<float*>(smem + C::kOffScale)[sc * kKeys + r0 + e] = 0.f;
                  bar_arrive(scale_full + 8 * sc);
                }
              } else {
                bar_arrive(bar);
                if (Q) bar_arrive(scale_full + 8 * sc);
              }
            }
          }
          if (t < end) walk_on(w, a, cum, skip_rows);
        }
      }
    } else if (Q) {
      // ---- codes -> bf16: one thread per cache row -------------------------------------------------------
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kOtherRegs));
      const uint32_t row = tid & 127;
      const uint32_t n = 2 * (uint32_t)(end - begin);
      bool ok = true;
      for (uint32_t q = 0; q < n; ++q) {
        const uint32_t raw = q % C::kRaws, slot = q % C::kSlots;
        ok = wait_or_give_up(raw_full + 8 * raw, (q / C::kRaws) & 1, ok, a.error);
        if (q >= C::kSlots) ok = wait_or_give_up(empty + 8 * slot, (q / C::kSlots + 1) & 1, ok, a.error);
        const char* src = smem + C::kOffRaw + raw * C::kRawBytes + row * D;
        char* dst = smem + C::kOffSlots + slot * C::kSlotBytes + row * 128;
#pragma unroll
        for (uint32_t c = 0; c < D / 16; ++c) {
          const uint4 x = *reinterpret_cast<const uint4*>(src + (D == 128 ? ((c ^ (row & 7)) << 4) : ((c ^ ((row >> 1) & 3)) << 4)));
          const uint32_t xs[4] = {x.x, x.y, x.z, x.w};
          uint32_t y[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            y[2 * e] = e4m3_to_bf16x2(__byte_perm(xs[e], 0, 0x1404));
            y[2 * e + 1] = e4m3_to_bf16x2(__byte_perm(xs[e], 0, 0x3424));
          }
          char* to = dst + (c >> 2) * C::kSpanBytes;
          *reinterpret_cast<uint4*>(to + ((((2 * c) & 7) ^ (row & 7)) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
          *reinterpret_cast<uint4*>(to + ((((2 * c + 1) & 7) ^ (row & 7)) << 4)) = make_uint4(y[4], y[5], y[6], y[7]);
        }
        fence_async();
        bar_arrive(full + 8 * slot);
        bar_arrive(raw_empty + 8 * raw);
      }
    }
  }
  tc_before();
  __syncthreads();
  if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

}  // namespace wbi
