// Attention for many rows: a block holds 256 rows (new token x query head of one kv head, as two tiles of 128) of a
// sequence against 128 cache rows at a time.  Scores and the weighted sum of values are tcgen05 products with fp32
// accumulators in tensor memory.  2048 tokens over 16384 positions, 32 heads of 128 over 8, bf16: 430 us, 1200
// TFLOP/s, over 200 passes from a cool GPU; 479 us, 1075 TFLOP/s, where the passes go on and the power limit sets the
// clock (a plain bf16 matrix product: 1635 and 1405).
//
//   - Tensor memory (512 columns): scores of tile 0 and 1 (128 each), outputs of tile 0 and 1 (D each).  A tile's weights
//     replace its scores as bf16, and enter the second product from there.
//   - Warps 0-3 and 4-7 are the softmax of tile 0 and tile 1, one thread per row: no exchange between threads.  While
//     one tile's weights are computed, the tensor core works for the other.  What bounds a step is this chain of one tile: scores,
//     1.0 us of softmax, the two products, and the hand-overs between; both tiles' products take 1.1 us of its 1.95.
//     (Steps of 64 cache rows with two score buffers per tile take the products out of the chain, but the scores' product then
//     reads the queries from shared memory twice as often: 527 us.  Part of the exponentials as polynomials: 436 us and more, the
//     arithmetic pipes are as busy as the exponential unit.)
//   - A row's outputs are rescaled only when its maximum has grown by more than 2^8: weights stay below 256, where
//     bf16's relative precision is the same, and sums are fp32 in either case.
//   - One warp issues all products in the order  QK0 QK1 | PV0 QK0' PV1 QK1' | ..., one requests cache tiles into a
//     ring of slots (keys, values, keys, ...) by tensor-map loads, a box per page piece and lane.
//   - E4M3 caches: tiles arrive as codes, four more warps widen them to bf16 slots; the row scales multiply scores and
//     weights in the softmax, where each is a value of its own.  This takes 682 us where bf16 takes 430 (tensor core 36 % busy,
//     issue slots 45 %, ALU 32 %): the step's chain is a microsecond longer, by the scales' loads, products and barriers, and by the
//     widening warps' share of the schedulers; 616 us with nothing widened, 530 without scales as well.
//   - Work is cut as in the kernel for few rows: one line of 128-row tiles over all (sequence, kv head, row block)
//     items, an equal share for every SM; a second kernel joins the cut items.
#pragma once
#include "wb_attend.cuh"

namespace wbi {

constexpr uint32_t kQRows = 256;       // rows of a block
constexpr uint32_t kKeys = 128;        // cache rows of a step
// An item counts for kItemCost tiles more than it has: its queries, first scores and outputs take that long.  They come first in its
// stretch of the line, where it is never cut.  (Seven ragged prompts of 100 to 1000 tokens, bf16, heads of 64: 94 us without, 81, 79, 75 and
// 76 with 1, 2, 3 and 4.)
constexpr int32_t kItemCost = 3;

template <int D, bool Q>
struct TilesCfg {
  static constexpr uint32_t kSpans = D / 64;                       // 128-byte spans of a bf16 row
  static constexpr uint32_t kSpanBytes = kKeys * 128;              // one span of 128 rows
  static constexpr uint32_t kSlotBytes = kSpans * kSpanBytes;      // a bf16 tile of keys or values
  static constexpr uint32_t kQBytes = 2 * kSlotBytes;
  static constexpr uint32_t kSlots = Q ? (D == 128 ? 3 : 6) : (D == 128 ? 5 : 10);
  static constexpr uint32_t kRawBytes = Q ? kKeys * D : 0;         // a tile of codes
  static constexpr uint32_t kRaws = Q && D == 64 ? 8 : 4;
  // 128 scales each; keys and values in turn.  No fewer than the tiles of codes: a load of scales into a slot then comes after the
  // widening threads have given back the codes of the slot's last user, which they do behind a proxy fence.
  static constexpr uint32_t kScaleSlots = D == 64 ? 8 : 4;
  static_assert(!Q || kScaleSlots >= kRaws, "");
  static constexpr uint32_t kRowSpan = D * (Q ? 1 : 2) < 128 ? D * (Q ? 1 : 2) : 128;   // bytes of a row in a box
  static constexpr uint32_t kRowSpans = D * (Q ? 1 : 2) / kRowSpan;
  // the quarter of a row's weights after which their product may start (3: all; measured best of 0, 1, 3)
  static constexpr int kHalfAt = Q ? 3 : 1;
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
  static constexpr uint32_t kBars = 1 + 8 + 2 * kSlots + (Q ? 2 * kRaws + 3 * kScaleSlots : 0);
  static constexpr uint32_t kOffMisc = kOffBars + kBars * 8;  // tensor memory address, flags, share
  static constexpr uint32_t kOffCum = kOffMisc + 64;
  static constexpr uint32_t kSmemBytes = kOffCum + (kMaxSeqs + 1) * 4;
  static_assert(kSmemBytes <= 232448, "");
};

// ---- tcgen05 ------------------------------------------------------------------------------------
// The warp that issues products stays converged: every lane computes the same descriptors (so that they live in uniform
// registers) and only the leader's instruction is let through.  Issued from a branch that one lane takes, each product costs
// about 80 clocks of moves into uniform registers, more than the product itself.
__device__ __forceinline__ void tc_commit(uint32_t bar, uint32_t leader) {
  asm volatile("{ .reg .pred e; setp.ne.u32 e, %1, 0; @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0]; }"
               ::"r"(bar), "r"(leader) : "memory");
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add, uint32_t leader) {
  asm volatile("{ .reg .pred p, e; setp.ne.u32 p, %4, 0; setp.ne.u32 e, %5, 0; @e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add), "r"(leader) : "memory");
}
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add, uint32_t leader) {
  asm volatile("{ .reg .pred p, e; setp.ne.u32 p, %4, 0; setp.ne.u32 e, %5, 0; @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }"
               ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(add), "r"(leader) : "memory");
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
__device__ __forceinline__ void tm_store16(uint32_t addr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
               "r"(r[14]), "r"(r[15]), "r"(addr) : "memory");
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

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Four scales; volatile, so that they are not all fetched ahead (128 registers hold the scores already).
__device__ __forceinline__ ulonglong2 load_scales(uint32_t addr) {
  ulonglong2 f;
  asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(f.x), "=l"(f.y) : "r"(addr));
  return f;
}

// ---- geometry -----------------------------------------------------------------------------------
struct RowBlock {
  int32_t kt0, n;          // first tile of 128 cache rows; its length in the line: kItemCost and its tiles (at least one)
};
__device__ __forceinline__ RowBlock row_block(const KvSeq& q, uint32_t group, uint32_t window, uint32_t rb) {
  const uint32_t rows = (uint32_t)q.n_new * group, r0 = rb * kQRows, r1 = min(r0 + kQRows, rows);
  const int32_t base = q.len - q.n_new;
  const int32_t hi = base + (int32_t)((r1 - 1) / group);
  const int32_t lo = window ? max(0, base + (int32_t)(r0 / group) - (int32_t)window + 1) : 0;
  RowBlock b;
  b.kt0 = lo / (int32_t)kKeys;
  b.n = kItemCost + max(1, (hi + (int32_t)kKeys) / (int32_t)kKeys - b.kt0);
  return b;
}
__device__ __forceinline__ uint32_t row_blocks(const KvSeq& q, uint32_t group, uint32_t skip_rows) {
  const uint64_t rows = (uint64_t)q.n_new * group;
  return rows > skip_rows ? (uint32_t)((rows + kQRows - 1) / kQRows) : 0;
}

// A block's share of the line begins at the multiple of `per` that is its number, moved to the next end of an item where that is
// not more than kSnap tiles away: joining a cut item costs more than so many tiles.  So an item [i0, i1) is cut at the multiples
// of `per` that lie more than kSnap tiles inside.
constexpr int32_t kSnap = 2;
__device__ __forceinline__ int32_t cuts_of(int32_t i0, int32_t i1, int32_t per) {
  const int32_t lo = (i0 + kItemCost + kSnap + per) / per, hi = (i1 - kSnap - 1) / per;    // multiples in (i0 + kItemCost + kSnap, i1 - kSnap)
  return max(0, hi - lo + 1);
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

// The beginning of block x's share.
__device__ __forceinline__ int32_t share_begin(const AttendArgs& a, const int32_t* cum, uint32_t skip_rows, int32_t x, int32_t per, int32_t total) {
  const int32_t t = x * per;
  if (t <= 0 || t >= total) return t <= 0 ? 0 : total;
  const Walk w = walk_to(a, cum, skip_rows, t);
  if (t - w.item0 <= kItemCost + kSnap) return w.item0;
  if (w.item0 + w.blk.n - t <= kSnap) return w.item0 + w.blk.n;
  return t;
}

// Values that are not finite were taken out of a tile that not every row sees (of any tile, where a scale was not finite): a row that
// does see one has it added here (its weight is positive, whatever it is).  Rare, so straight from the cache.
template <bool Q>
__device__ __noinline__ void add_odd_values(const AttendArgs& a, const Walk& w, int32_t kt_begin, int32_t kt_end, int32_t lo, int32_t hi, uint32_t d0,
                                            float* o) {
  for (int32_t pos = max(lo, kt_begin * (int32_t)kKeys); pos <= min(hi, kt_end * (int32_t)kKeys - 1); ++pos) {
    const int32_t page = kv_page(a.b, a.c.n_pages, a.c.page_size, w.s, pos);
    if (page < 0) continue;
    const uint32_t slot = (uint32_t)pos % a.c.page_size;
    const uint64_t at = (uint64_t)page * a.c.page_stride + w.h * a.c.head_stride + slot * a.c.head_dim + d0;
    if (Q) {
      const float s = a.c.v_scale[((uint64_t)page * a.c.n_kv_heads + w.h) * a.c.page_size + slot];
      if (isfinite(s)) continue;
      for (int d = 0; d < 32; ++d) o[d] += unpack_e4m3x2((uint8_t)a.c.v[at + d]).x * s;
    } else {
      const uint16_t* v = reinterpret_cast<const uint16_t*>(a.c.v) + at;
      for (int d = 0; d < 32; ++d)
        if ((v[d] & 0x7F80u) == 0x7F80u) o[d] += __uint_as_float((uint32_t)v[d] << 16);
    }
  }
}

// A thread's row of the block.
struct RowOf {
  bool in;
  uint32_t tok, head;      // row and head of the step's tensors
  int32_t hi, lo;          // positions that it sees
};
__device__ __forceinline__ RowOf row_of(const AttendArgs& a, const Walk& w, uint32_t r0) {
  RowOf x;
  const uint32_t n_rows = (uint32_t)w.seq.n_new * a.group, r = w.rb * kQRows + r0;
  x.in = r < n_rows;
  x.tok = (x.in ? r : n_rows - 1) / a.group;
  x.head = w.h * a.group + (x.in ? r - x.tok * a.group : 0);
  x.hi = w.seq.len - w.seq.n_new + (int32_t)x.tok;
  x.lo = a.window ? x.hi - (int32_t)a.window + 1 : 0;
  x.tok += (uint32_t)w.seq.row0;
  return x;
}

// The queries of a warp's 32 rows into shared memory, swizzled as the products read them; lane i knows row i.  Eight lanes copy 128
// bytes of a row together (a thread copying its own row would touch a line per thread and load).
template <int D>
__device__ __forceinline__ void copy_queries(const AttendArgs& a, uint32_t tile, uint32_t row0, const RowOf& x) {
  const uint32_t lane = threadIdx.x & 31, c = lane & 7;
  const uint64_t mine = (uint64_t)(a.q + (uint64_t)x.tok * a.q_token + x.head * a.q_head);
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) {
    const uint32_t from = i * 4 + (lane >> 3), row = row0 + from;
    const uint64_t src = __shfl_sync(0xFFFFFFFFu, mine, from);
    const uint32_t bytes = __shfl_sync(0xFFFFFFFFu, (uint32_t)x.in, from) ? 16 : 0;      // a row that is none: zeros
#pragma unroll
    for (uint32_t sp = 0; sp < D / 64; ++sp)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tile + sp * (kKeys * 128) + row * 128 + ((c ^ (row & 7)) << 4)),
                   "l"(src + sp * 128 + c * 16), "r"(bytes) : "memory");
  }
}
__device__ __forceinline__ void queries_arrived() {
  asm volatile("cp.async.wait_all;" ::: "memory");
  fence_async();
}

// One cache row of a value tile: cleared if it lies past the end; else its values that are not finite are taken out and the
// flag is raised, which both tiles read after their last product.  True if anything was written.
template <int D>
__device__ __forceinline__ bool clear_values(char* tile, uint32_t row, bool past, volatile uint32_t* flag) {
  char* v = tile + row * 128;
  if (past) {
#pragma unroll
    for (uint32_t c = 0; c < D / 8; ++c) *reinterpret_cast<uint4*>(v + (c >> 3) * (kKeys * 128) + ((c & 7) << 4)) = make_uint4(0, 0, 0, 0);
    return true;
  }
  bool odd = false;
#pragma unroll
  for (uint32_t c = 0; c < D / 8; ++c) {
    const uint4 y = *reinterpret_cast<const uint4*>(v + (c >> 3) * (kKeys * 128) + ((c & 7) << 4));
    // an exponent of all ones, in either half: adding the lowest bit of the exponent carries into the sign's place
    const uint32_t any = (((y.x & 0x7FFF7FFFu) + 0x00800080u) | ((y.y & 0x7FFF7FFFu) + 0x00800080u) | ((y.z & 0x7FFF7FFFu) + 0x00800080u) |
                          ((y.w & 0x7FFF7FFFu) + 0x00800080u)) & 0x80008000u;
    odd |= any != 0;
  }
  if (!odd) return false;
  *flag = 1;
  for (uint32_t c = 0; c < D / 2; ++c) {
    uint32_t* at = reinterpret_cast<uint32_t*>(v + (c >> 5) * (kKeys * 128)) + (c & 31);
    uint32_t y = *at;
    if ((y & 0x7F80u) == 0x7F80u) y &= 0xFFFF0000u;
    if ((y & 0x7F800000u) == 0x7F800000u) y &= 0xFFFFu;
    *at = y;
  }
  return true;
}


template <int D, bool Q>
__global__ void __launch_bounds__(TilesCfg<D, Q>::kThreads, 1)
wb_attend_tiles_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                       uint32_t skip_rows) {
  using C = TilesCfg<D, Q>;
  extern __shared__ __align__(1024) char smem[];
  const uint32_t base = smem_addr(smem);
  const uint32_t tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  const uint32_t bars = base + C::kOffBars;
  const uint32_t q_full = bars, s_full = bars + 8, p_half = bars + 24, p_full = bars + 40, o_full = bars + 56, full = bars + 72, empty = full + 8 * C::kSlots,
                 raw_full = empty + 8 * C::kSlots, raw_empty = raw_full + 8 * C::kRaws, scale_full = raw_empty + 8 * C::kRaws,
                 scale_ready = scale_full + 8 * C::kScaleSlots, scale_empty = scale_ready + 8 * C::kScaleSlots;
  volatile uint32_t* const misc = reinterpret_cast<volatile uint32_t*>(smem + C::kOffMisc);   // [0] tensor memory, [5, 6] share, [8..15] items' flags
  int32_t* const cum = reinterpret_cast<int32_t*>(smem + C::kOffCum);
  if (base & 1023u) {      // swizzled tiles need it; never the case without static shared memory
    if (tid == 0) atomicOr(a.error, kMisplaced);
    return;
  }

  // ---- the line of tiles -----------------------------------------------------------------------------
  const uint32_t n_seqs = a.b.n_seqs, hk = a.c.n_kv_heads;
  if (tid == 0) {
    cum[0] = 0;
    bar_init(q_full, 256);
    for (uint32_t i = 0; i < 2; ++i) {
      bar_init(s_full + 8 * i, 1);
      bar_init(p_half + 8 * i, 128);
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
        bar_init(scale_ready + 8 * i, 128);
        bar_init(scale_empty + 8 * i, 256);
      }
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    for (int i = 8; i < 16; ++i) misc[i] = 0;
  }
  for (uint32_t s = warp; s < n_seqs; s += C::kThreads / 32) {
    const KvSeq q = attend_seq(a.b, s);
    const uint32_t nb = row_blocks(q, a.group, skip_rows);
    int32_t sum = 0;
    for (uint32_t rb = lane; rb < nb; rb += 32) sum += row_block(q, a.group, a.window, rb).n;
    sum = __reduce_add_sync(0xFFFFFFFFu, sum);
    if (lane == 0) {
      cum[s + 1] = sum * (int32_t)hk;
      report_too_long(a, s);
    }
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
  if (warp < 2) {
    const int32_t t = share_begin(a, cum, skip_rows, (int32_t)(blockIdx.x + warp), per, total);
    if (lane == 0) misc[5 + warp] = (uint32_t)t;
  }
  __syncthreads();
  const int32_t begin = (int32_t)misc[5], end = (int32_t)misc[6];
  CutItem* const cut_item = reinterpret_cast<CutItem*>(a.cuts) + blockIdx.x;
  if (tid == 0) cut_item->parts = 0;

  if (begin < end) {
    if (warp < 8) {
      // ---- softmax: one thread per row ---------------------------------------------------------------
      asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kSoftmaxRegs));
      const uint32_t i = warp >> 2, row = tid & 127;
      const uint32_t tm_lane = tmem + ((warp & 3) << 21);
      const uint32_t tm_s = tm_lane + i * 128, tm_o = tm_lane + 256 + i * 128;
      const float c2 = a.scale_log2;
      uint32_t jg = 0, item = 0;                    // steps and items of the block so far
      uint32_t js = 0, is = 0;                      // those that this tile took part in
      bool ok = true;
      Walk w = walk_to(a, cum, skip_rows, begin);
      RowOf x0 = row_of(a, w, i * 128 + row);
      const uint32_t q_tile = base + i * C::kSlotBytes, warp_row = (warp & 3) * 32;
      copy_queries<D>(a, q_tile, warp_row, x0);
      queries_arrived();
      bar_arrive(q_full);
      for (int32_t t = begin; t < end; ++item) {
        const int32_t item1 = w.item0 + w.blk.n, stop = min(end, item1), tile0 = w.item0 + kItemCost;      // the item's first tile in the line
        t = max(t, tile0);
        const int32_t from = t;
        const uint32_t n_rows = (uint32_t)w.seq.n_new * a.group;
        const int32_t base_pos = w.seq.len - w.seq.n_new;
        // tiles that not every row of the block sees whole
        const int32_t cut_hi = base_pos + (int32_t)(w.rb * kQRows / a.group);
        const int32_t cut_lo = a.window ? base_pos + (int32_t)((min(n_rows, (w.rb + 1) * kQRows) - 1) / a.group) - (int32_t)a.window + 1 : 0;
        // rows of a warp are in the order of their tokens: its first row sees the least far, its last row's window begins last
        const int32_t warp_hi = __shfl_sync(0xFFFFFFFFu, x0.hi, 0), warp_lo = a.window ? __shfl_sync(0xFFFFFFFFu, x0.lo, 31) : 0;
        const bool takes_part = i == 0 || n_rows > w.rb * kQRows + 128;
        if (tid == 0) misc[8 + (item + 5) % 8] = 0;     // that of three items ago: the other tile is at most one behind, nobody five ahead
        Walk w2 = w;                                // the next item, once this one's last scores are there
        RowOf x2 = x0;
        // the scores of this item are done with: the next one's queries take their place while its last weights are computed
        auto prepare_next = [&]() {
          walk_on(w2, a, cum, skip_rows);
          x2 = row_of(a, w2, i * 128 + row);
          copy_queries<D>(a, q_tile, warp_row, x2);
        };
        // the score that the weights are relative to (differences are formed before they are scaled: scores of any finite size
        // give weights of 2^8 and less), and that above which it moves
        float ref = 0.f, limit = -INFINITY;
        uint64_t sum2[2] = {0, 0};
        for (bool first = true; t < stop; ++t, ++jg, first = false) {
          const uint32_t sk = (2 * jg) % C::kScaleSlots, sv = sk + 1;
          if (!takes_part) {                        // keeps the pace of the scales' ring
            if (Q) {
              ok = wait_or_give_up(scale_ready + 8 * sk, (2 * jg / C::kScaleSlots) & 1, ok, a.error);
              ok = wait_or_give_up(scale_ready + 8 * sv, (2 * jg / C::kScaleSlots) & 1, ok, a.error);
              bar_arrive(scale_empty + 8 * sk);
              bar_arrive(scale_empty + 8 * sv);
            }
            continue;
          }
          const int32_t pos0 = (w.blk.kt0 + t - tile0) * (int32_t)kKeys;
          const bool cut = pos0 + (int32_t)kKeys - 1 > cut_hi || pos0 < cut_lo;
          if (!Q && cut && i == 0) {
            // Values past the end, and values that are not finite, must not meet weights of zero.  Only the first tile's threads
            // write, one to a row: each then orders its own writes before the products, which wait for this tile's
            // weights first, and the other tile's products follow this one's.
            const uint32_t vq = 2 * jg + 1, slot = vq % C::kSlots;
            ok = wait_or_give_up(full + 8 * slot, (vq / C::kSlots) & 1, ok, a.error);
            if (clear_values<D>(smem + C::kOffSlots + slot * C::kSlotBytes, row, pos0 + (int32_t)row >= w.seq.len, misc + 8 + item % 8)) fence_async();
          }
          float x[128];
          ok = wait_or_give_up(s_full + 8 * i, js & 1, ok, a.error);
          ++js;
          tc_after();
#pragma unroll
          for (int c = 0; c < 128; c += 32) tm_load32(tm_s + c, reinterpret_cast<uint32_t*>(x) + c);
          if (t + 1 == stop && stop < end) prepare_next();
          tm_wait_load();
          if (Q) {
            ok = wait_or_give_up(scale_ready + 8 * sk, (2 * jg / C::kScaleSlots) & 1, ok, a.error);
            const uint32_t scales = base + C::kOffScale + sk * (kKeys * 4);
#pragma unroll
            for (int c = 0; c < 128; c += 4) {
              const ulonglong2 f = load_scales(scales + 4 * c);
              unpack2(mul2(pack2(x[c], x[c + 1]), f.x), x[c], x[c + 1]);
              unpack2(mul2(pack2(x[c + 2], x[c + 3]), f.y), x[c + 2], x[c + 3]);
            }
          }
          // masks: a bit per column for both ends at once, in groups of columns that some row of the warp does not see whole
          // (a comparison and a selection per column and end took 1.1 us of the step)
          if (pos0 + (int32_t)kKeys - 1 > warp_hi || pos0 < warp_lo) {
            const int32_t h1 = x0.hi - pos0 + 1, l1 = x0.lo - pos0;
#pragma unroll
            for (int c = 0; c < 128; c += 32) {
              if (pos0 + c + 31 <= warp_hi && pos0 + c >= warp_lo) continue;
              const int32_t up = min(max(h1 - c, 0), 32), low = min(max(l1 - c, 0), 32);
              const uint32_t bits = (uint32_t)((1ull << up) - 1) & ~(uint32_t)((1ull << low) - 1);
#pragma unroll
              for (int e = 0; e < 32; ++e) x[c + e] = bits & 1u << e ? x[c + e] : -INFINITY;
            }
          }
          float m4[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
          for (int c = 4; c < 124; c += 8)
#pragma unroll
            for (int e = 0; e < 4; ++e) m4[e] = max3(m4[e], x[c + 2 * e], x[c + 2 * e + 1]);
          m4[0] = max3(m4[0], x[124], x[125]);
          m4[1] = max3(m4[1], x[126], x[127]);
          const float m = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
          const bool grow = m > limit;
          // the step's commit covered the previous product, so nothing writes the outputs now
          if (__any_sync(0xFFFFFFFFu, grow)) {
            float corr = 1.f;
            if (grow) {
              corr = limit == -INFINITY ? 0.f : fast_exp2((ref - m) * c2);
              ref = m;
              limit = fmaxf(m + __fdividef(8.f, c2), -3.0e38f);      // finite: -inf means that nothing was seen yet
            }
            const uint64_t corr2 = pack2(corr, corr);
            sum2[0] = mul2(sum2[0], corr2);
            sum2[1] = mul2(sum2[1], corr2);
            if (!first) {
#pragma unroll 1
              for (int c = 0; c < D; c += 32) {
                uint32_t o[32];
                tm_load32(tm_o + c, o);
                tm_wait_load();
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * corr);
                tm_store32(tm_o + c, o);
              }
            }
          }
          if (Q) ok = wait_or_give_up(scale_ready + 8 * sv, (2 * jg / C::kScaleSlots) & 1, ok, a.error);
          const uint64_t c22 = pack2(c2, c2), ref2 = pack2(-ref, -ref);
          const uint32_t vscales = base + C::kOffScale + sv * (kKeys * 4);
#pragma unroll
          for (int quarter = 0; quarter < 4; ++quarter) {
            uint32_t p[16];
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
              const int c = quarter * 32 + 2 * e;
              ulonglong2 f;
              if (Q) f = load_scales(vscales + 4 * c);
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                float u, v;
                unpack2(mul2(add2(pack2(x[c + 2 * k], x[c + 2 * k + 1]), ref2), c22), u, v);
                const uint64_t y = pack2(fast_exp2(u), fast_exp2(v));
                sum2[k] = add2(sum2[k], y);
                unpack2(Q ? mul2(y, k ? f.y : f.x) : y, u, v);
                p[e + k] = pack_bf16x2(u, v);
              }
            }
            tm_store16(tm_s + quarter * 16, p);
            if (quarter == C::kHalfAt) {      // the product of these weights starts while the rest is computed
              tm_wait_store();
              tc_before();
              bar_arrive(p_half + 8 * i);
            }
          }
          if (C::kHalfAt < 3) {
            tm_wait_store();
            tc_before();
            bar_arrive(p_full + 8 * i);
          }
          if (Q) {
            bar_arrive(scale_empty + 8 * sk);
            bar_arrive(scale_empty + 8 * sv);
          }
        }
        if (t < end) {
          if (!takes_part) prepare_next();
          queries_arrived();
          // Neither tile's warps get an item ahead of the other's: a tile that takes no part in an item has nothing to wait for, and
          // its arrivals for the items after would stand in for the other's.
          asm volatile("bar.sync 1, 256;" ::: "memory");
          bar_arrive(q_full);
        }
        // ---- outputs ---------------------------------------------------------------------------------
        if (takes_part) {
          float l, l1;
          unpack2(add2(sum2[0], sum2[1]), l, l1);
          l += l1;
          ok = wait_or_give_up(o_full + 8 * i, is & 1, ok, a.error);
          ++is;
          tc_after();
          const bool odd = misc[8 + item % 8] != 0;
          const int32_t cuts = cuts_of(w.item0, item1, per);
          char* dst = a.out + (uint64_t)x0.tok * a.o_token + x0.head * a.o_head;
          float* part = a.partials + (size_t)(2 * blockIdx.x + (w.item0 >= begin ? 1 : 0)) * C::kPartFloats + i * (D * 128 + 256) + row;
          const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN;
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            uint32_t o[32];
            tm_load32(tm_o + c, o);
            tm_wait_load();
            if (odd && x0.in) {
              float y[32];
#pragma unroll
              for (int e = 0; e < 32; ++e) y[e] = __uint_as_float(o[e]);
              add_odd_values<Q>(a, w, w.blk.kt0 + from - tile0, w.blk.kt0 + stop - tile0, x0.lo, x0.hi, c, y);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(y[e]);
            }
            if (cuts == 0) {
              if (x0.in)
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
              for (int e = 0; e < 32; ++e) part[(c + e) * 128] = __uint_as_float(o[e]);
            }
          }
          if (cuts == 0) {
            if (x0.in && a.lse)
              a.lse[(uint64_t)x0.tok * a.n_heads + x0.head] = l == 0.f ? -INFINITY : (ref * c2 + log2f(l)) * kLn2;
          } else {
            part[D * 128] = l == 0.f ? -INFINITY : ref * c2;
            part[D * 128 + 128] = l;
            if (tid == 0 && w.item0 >= begin) *cut_item = CutItem{(uint32_t)cuts + 1, w.s, w.h, w.rb};
          }
        }
        w = w2;
        x0 = x2;
      }
    } else if (warp < 12) {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kOtherRegs));
      if (warp == 8) {
        // ---- products ------------------------------------------------------------------------------------
        constexpr uint32_t kF32Bf16 = 1u << 4 | 1u << 7 | 1u << 10 | 8u << 24;
        constexpr uint32_t kQk = kF32Bf16 | (kKeys / 8) << 17, kPv = kF32Bf16 | 1u << 16 | (uint32_t)(D / 8) << 17;
        const uint32_t leader = lane == 0, tm = uniform(tmem);
        const int32_t t_end = uniform(end);
        uint32_t jg = 0, item = 0, js = 0;          // steps, items, steps of the second tile
        bool ok = true;
        auto wait_all = [&](uint32_t bar, uint32_t parity) {
          ok = wait_or_give_up(bar, parity, ok, a.error);
          __syncwarp();
          tc_after();
        };
        auto slot_wait = [&](uint32_t q) {
          const uint32_t slot = q % C::kSlots;
          wait_all(full + 8 * slot, (q / C::kSlots) & 1);
          return base + C::kOffSlots + slot * C::kSlotBytes;
        };
        auto scores = [&](uint32_t i, uint32_t k_addr) {
          const uint64_t qd = smem_desc(base + i * C::kSlotBytes, 16), kd = smem_desc(k_addr, 16);
#pragma unroll
          for (uint32_t ks = 0; ks < D / 16; ++ks) {
            const uint32_t off = ((ks >> 2) * C::kSpanBytes + (ks & 3) * 32) >> 4;
            tc_mma_ss(tm + i * 128, qd + off, kd + off, kQk, ks > 0, leader);
          }
          tc_commit(s_full + 8 * i, leader);
        };
        auto values = [&](uint32_t i, uint32_t v_addr, uint32_t add, uint32_t step) {
          const uint64_t vd = smem_desc(v_addr, C::kSpanBytes);
          wait_all(p_half + 8 * i, step & 1);
#pragma unroll
          for (uint32_t ks = 0; ks < kKeys / 16; ++ks) {
            if (ks == 2 * (C::kHalfAt + 1)) wait_all(p_full + 8 * i, step & 1);
            tc_mma_ts(tm + 256 + i * 128, tm + i * 128 + ks * 8, vd + (ks * 2048 >> 4), kPv, ks > 0 ? 1u : add, leader);
          }
        };
        Walk w = walk_to(a, cum, skip_rows, begin);
        for (int32_t t = uniform(begin); t < t_end; ++item) {
          const int32_t stop = uniform(min(end, w.item0 + w.blk.n));
          t = uniform(max(t, w.item0 + kItemCost));
          const uint32_t two = uniform((uint32_t)((uint32_t)w.seq.n_new * a.group > w.rb * kQRows + 128));
          wait_all(q_full, item & 1);
          uint32_t k_addr = slot_wait(2 * jg);
          scores(0, k_addr);
          if (two) scores(1, k_addr);
          tc_commit(empty + 8 * ((2 * jg) % C::kSlots), leader);
          for (uint32_t add = 0; t < stop; ++t, ++jg, add = 1) {
            const uint32_t v_addr = slot_wait(2 * jg + 1);
            const bool more = t + 1 < stop;
            if (more) k_addr = slot_wait(2 * jg + 2);
            values(0, v_addr, add, jg);
            if (more) scores(0, k_addr); else tc_commit(o_full, leader);
            if (two) {
              values(1, v_addr, add, js);
              ++js;
              if (more) scores(1, k_addr); else tc_commit(o_full + 8, leader);
            }
            tc_commit(empty + 8 * ((2 * jg + 1) % C::kSlots), leader);
            if (more) tc_commit(empty + 8 * ((2 * jg + 2) % C::kSlots), leader);
          }
          if (t < t_end) walk_on(w, a, cum, skip_rows);
        }
        // the last commit arrives before the block ends (waited for even after a wait that gave up)
        (void)wait_or_give_up(empty + 8 * ((2 * jg - 1) % C::kSlots), ((2 * jg - 1) / C::kSlots) & 1, true, a.error);
        __syncwarp();
      } else if (warp == 9) {
        // ---- cache tiles: one lane per page piece ------------------------------------------------------
        const uint32_t pieces = kKeys / a.box_rows;
        uint32_t jg = 0;
        bool ok = true;
        Walk w = walk_to(a, cum, skip_rows, begin);
        for (int32_t t = begin; t < end;) {
          const int32_t stop = min(end, w.item0 + w.blk.n), tile0 = w.item0 + kItemCost;
          for (t = max(t, tile0); t < stop; ++t, ++jg) {
            const int32_t pos = (w.blk.kt0 + t - tile0) * (int32_t)kKeys + (int32_t)(lane * a.box_rows);
            int32_t page = -1;
            if (lane < pieces && pos < w.seq.len) page = kv_page(a.b, a.c.n_pages, a.c.page_size, w.s, pos);
            const uint32_t in_page = (uint32_t)pos % a.c.page_size, r0 = lane * a.box_rows;
            const int32_t where = page < 0 ? (int32_t)a.c.n_pages : page;      // outside the cache: zeros
#pragma unroll
            for (uint32_t kv = 0; kv < 2; ++kv) {
              const uint32_t q = 2 * jg + kv, ring = Q ? C::kRaws : C::kSlots, slot = q % ring, sc = q % C::kScaleSlots;
              const uint32_t bar = (Q ? raw_full : full) + 8 * slot, sbar = scale_full + 8 * sc;
              if (q >= ring) ok = wait_or_give_up((Q ? raw_empty : empty) + 8 * slot, (q / ring + 1) & 1, ok, a.error);
              if (Q && q >= C::kScaleSlots) ok = wait_or_give_up(scale_empty + 8 * sc, (q / C::kScaleSlots + 1) & 1, ok, a.error);
              const uint32_t dst = base + (Q ? C::kOffRaw + slot * C::kRawBytes : C::kOffSlots + slot * C::kSlotBytes);
              if (lane < pieces) {
                bar_arrive_tx(bar, a.box_rows * D * (Q ? 1 : 2));
#pragma unroll
                for (uint32_t e = 0; e < C::kRowSpans; ++e)
                  load_box(dst + e * (kKeys * C::kRowSpan) + r0 * C::kRowSpan, kv ? &map_v : &map_k, (int32_t)(e * 64), (int32_t)in_page, (int32_t)w.h, where, bar);
                if (Q && page >= 0) {
                  bar_arrive_tx(sbar, a.box_rows * 4);
                  load_bulk(base + C::kOffScale + (sc * kKeys + r0) * 4, (kv ? a.c.v_scale : a.c.k_scale) + ((uint64_t)page * hk + w.h) * a.c.page_size + in_page,
                            a.box_rows * 4, sbar);
                } else if (Q) {
                  for (uint32_t e = 0; e < a.box_rows; ++e) reinterpret_cast<float*>(smem + C::kOffScale)[sc * kKeys + r0 + e] = 0.f;
                  fence_async();      // before this lane's next load into the same place
                  bar_arrive(sbar);
                }
              } else {
                bar_arrive(bar);
                if (Q) bar_arrive(sbar);
              }
            }
          }
          if (t < end) walk_on(w, a, cum, skip_rows);
        }
        // every load lands before the block ends, also where the others gave up waiting and left some unread
        const uint32_t n = 2 * jg, ring = Q ? C::kRaws : C::kSlots;
        for (uint32_t q = n > ring ? n - ring : 0; q < n; ++q) (void)wait_or_give_up((Q ? raw_full : full) + 8 * (q % ring), (q / ring) & 1, true, a.error);
        if (Q)
          for (uint32_t q = n > C::kScaleSlots ? n - C::kScaleSlots : 0; q < n; ++q)
            (void)wait_or_give_up(scale_full + 8 * (q % C::kScaleSlots), (q / C::kScaleSlots) & 1, true, a.error);
      }
    } else if (Q) {
      // ---- codes -> bf16: one thread per cache row -------------------------------------------------------
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kOtherRegs));
      const uint32_t row = tid & 127;
      bool ok = true;
      Walk w = walk_to(a, cum, skip_rows, begin);
      int32_t t = begin;
      uint32_t item = 0;
      for (uint32_t q = 0; t < end; ++q) {
        if ((q & 1) == 0) t = max(t, w.item0 + kItemCost);
        const uint32_t raw = q % C::kRaws, slot = q % C::kSlots, sc = q % C::kScaleSlots;
        ok = wait_or_give_up(scale_full + 8 * sc, (q / C::kScaleSlots) & 1, ok, a.error);
        if (q & 1) {
          // a weight of zero must not meet a scale that is none: one past the end may be anything, and one that is not
          // finite is taken out here and added to the rows that see it at the end
          float* at = reinterpret_cast<float*>(smem + C::kOffScale) + sc * kKeys + row;
          const bool past = (w.blk.kt0 + t - w.item0 - kItemCost) * (int32_t)kKeys + (int32_t)row >= w.seq.len;
          if (past || !isfinite(*at)) {
            if (!past) misc[8 + item % 8] = 1;
            *at = 0.f;                // (ordered before the next load into the same place by the fence below: see kScaleSlots)
          }
          if (++t == min(end, w.item0 + w.blk.n) && t < end) {
            walk_on(w, a, cum, skip_rows);
            ++item;
          }
        }
        bar_arrive(scale_ready + 8 * sc);
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

// Joins the items that blocks' shares cut: block (x, y) takes 32 rows of the item that is cut first in block x, its parts in order;
// a lane owns a row, a warp an eighth of the columns.  A kernel of its own, because the last of many blocks to finish an
// item would read all of its parts alone (256 rows x D fp32 each: 18 parts took it 20 us, this takes 3).
template <int D>
__global__ void __launch_bounds__(256) wb_attend_join_kernel(const __grid_constant__ AttendArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  constexpr uint32_t kPart = 2 * (D * 128 + 256), N = D / 8;
  const uint32_t x = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const CutItem it = reinterpret_cast<const CutItem*>(a.cuts)[x];
  if (!it.parts) return;
  Walk w;
  w.seq = attend_seq(a.b, it.s);
  w.h = it.h;
  w.rb = it.rb;
  const uint32_t r = blockIdx.y * 32 + lane;
  const RowOf row = row_of(a, w, r);
  if (!__any_sync(0xFFFFFFFFu, row.in)) return;
  const float* parts = a.partials + (r >> 7) * (D * 128 + 256) + (r & 127);
  auto part_of = [&](uint32_t p) { return parts + (size_t)(2 * (x + p) + (p == 0 ? 1 : 0)) * kPart; };
  float top = -INFINITY, sum = 0.f, o[N] = {};
#pragma unroll 4
  for (uint32_t p = 0; p < it.parts; ++p) top = fmaxf(top, part_of(p)[D * 128]);
#pragma unroll 2
  for (uint32_t p = 0; p < it.parts; ++p) {
    const float* src = part_of(p);
    const float m = src[D * 128], f = m == -INFINITY ? 0.f : fast_exp2(m - top);
    sum += f * src[D * 128 + 128];
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) o[e] += f * src[(warp * N + e) * 128];
  }
  if (!row.in) return;
  const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : NAN;
  uint4* dst = reinterpret_cast<uint4*>(a.out + (uint64_t)row.tok * a.o_token + row.head * a.o_head + warp * N * 2);
#pragma unroll
  for (uint32_t e = 0; e < N; e += 8)
    dst[e / 8] = make_uint4(pack_bf16x2(o[e] * inv, o[e + 1] * inv), pack_bf16x2(o[e + 2] * inv, o[e + 3] * inv),
                            pack_bf16x2(o[e + 4] * inv, o[e + 5] * inv), pack_bf16x2(o[e + 6] * inv, o[e + 7] * inv));
  if (warp == 0 && a.lse) a.lse[(uint64_t)row.tok * a.n_heads + row.head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

}  // namespace wbi
