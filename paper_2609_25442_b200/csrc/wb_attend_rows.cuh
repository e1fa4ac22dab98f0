// Attention for few rows: sequences whose new tokens times query heads per kv head are at most 64 rows
// (single tokens, drafted chunks).  Every byte of the cache is used for a handful of products, so the bound
// is memory bandwidth, and the kernel is a stream of cache tiles through shared memory:
//
//   - A tile is 64 cache rows of one kv head, keys and values.  One warp requests it by tensor-map loads (a box
//     per page piece; pages that do not exist read as zeros), several tiles ahead.
//   - A compute warp owns 16 of a tile's rows and 16 query rows, with its own running maximum and sum: scores
//     and products on m16n8k16 matrix instructions, P straight from the score registers.  No two warps talk
//     until an item ends.  The legacy matrix path is enough here: a tile takes 32 instructions per warp,
//     far less time than its 16-32 KB take to arrive.
//   - E4M3 tiles are widened to bf16 in registers between the shared load and the matrix instruction; the row
//     scales multiply scores and weights.
//   - Work is cut evenly over the SMs whatever the lengths: all (sequence, kv head) items form one line of
//     tiles, every block takes the same number of consecutive tiles, and an item that crosses blocks is joined by
//     the block that finishes it last, in the order of the tiles (so results do not depend on timing).
#pragma once
#include "wb_attend.cuh"

namespace wbi {

template <int D, bool Q, int MT>
struct RowsCfg {
  static constexpr uint32_t kElem = Q ? 1 : 2;
  static constexpr uint32_t kRowBytes = D * kElem;
  static constexpr uint32_t kSpan = kRowBytes < 128 ? kRowBytes : 128;       // bytes of a row in one box
  static constexpr uint32_t kSpans = kRowBytes / kSpan;
  static constexpr uint32_t kTileBytes = kKvTile * kRowBytes;                // keys, and as much of values
  static constexpr uint32_t kScaleBytes = Q ? kKvTile * 4 : 0;
  static constexpr uint32_t kStageBytes = 2 * kTileBytes;                    // the scales lie behind all stages
  static constexpr uint32_t kStages = (MT == 1 ? 98304u : 163840u) / (2 * kTileBytes) > 8 ? 8 : (MT == 1 ? 98304u : 163840u) / (2 * kTileBytes);
  static constexpr uint32_t kWarps = 4 * MT;                                 // compute warps
  static constexpr uint32_t kThreads = 32 * (kWarps + 1);
  static constexpr uint32_t kRegs = D / 2;                                   // accumulator registers of a lane: 16 x D
  static constexpr uint32_t kJoinBytes = MT * kRegs * 32 * 4;
  static constexpr uint32_t kPartFloats = MT * (kRegs * 32 + 32);            // one partial: accumulators, maxima, sums
  static size_t smem_bytes(uint32_t n_seqs) {
    return 1024 + kStages * (kStageBytes + 2 * kScaleBytes) + kJoinBytes + (n_seqs + 1) * 4 + MT * 4 * 16 * 8;
  }
};

__device__ __forceinline__ void ldsm4(uint32_t a, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a));
}
__device__ __forceinline__ void ldsm4t(uint32_t a, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a));
}
__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Byte offset of 16-byte chunk `c` of row `row` in a swizzled block of rows of `SPAN` bytes.
template <uint32_t SPAN> __device__ __forceinline__ uint32_t swizzled(uint32_t row, uint32_t c) {
  return SPAN == 128 ? row * 128 + ((c ^ (row & 7)) << 4) : row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
}

__device__ __forceinline__ bool not_finite_bf16x2(uint32_t w) {
  return ((w & 0x7F80u) == 0x7F80u) | ((w & 0x7F800000u) == 0x7F800000u);
}

template <int D, bool Q, int MT>
__global__ void __launch_bounds__(RowsCfg<D, Q, MT>::kThreads, MT == 1 ? 2 : 1)
wb_attend_rows_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using C = RowsCfg<D, Q, MT>;
  extern __shared__ char smem_raw[];
  // stages (1024-byte aligned), their scales, join buffer, warps' maxima and sums, prefix sums
  const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
  char* const gen = smem_raw + (base - smem_addr(smem_raw));
  const uint32_t scale_base = C::kStages * C::kStageBytes;
  float* const join = reinterpret_cast<float*>(gen + scale_base + C::kStages * 2 * C::kScaleBytes);
  float2* const warp_ml = reinterpret_cast<float2*>(join + C::kJoinBytes / 4);        // [mt][kw][16]
  int32_t* const cum = reinterpret_cast<int32_t*>(warp_ml + MT * 4 * 16);
  __shared__ __align__(8) uint64_t bars[2 * C::kStages];
  __shared__ int32_t scan_tmp[32];
  __shared__ uint32_t s_last;
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t full = smem_addr(bars), empty = full + 8 * C::kStages;

  if (tid == 0) {
    for (uint32_t i = 0; i < C::kStages; ++i) {
      bar_init(full + 8 * i, 32);
      bar_init(empty + 8 * i, C::kWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }

  // ---- the line of tiles: cum[s] = tiles of the sequences before s ---------------------------------
  const uint32_t n_seqs = a.b.n_seqs, hk = a.c.n_kv_heads, rows_max = 16 * MT;
  {
    const uint32_t per = (n_seqs + C::kThreads - 1) / C::kThreads, s0 = min(tid * per, n_seqs), s1 = min(s0 + per, n_seqs);
    int32_t sum = 0;
    for (uint32_t s = s0; s < s1; ++s) {
      const KvSeq q = attend_seq(a.b, s);
      int32_t nt = 0;
      if (q.n_new > 0 && (uint32_t)q.n_new * a.group <= rows_max) {
        const int32_t lo = first_position(q, a.window) / (int32_t)kKvTile;
        nt = max(1, (q.len + (int32_t)kKvTile - 1) / (int32_t)kKvTile - lo);
      }
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
  const int32_t total = cum[n_seqs];
  const int32_t per = (total + (int32_t)gridDim.x - 1) / (int32_t)gridDim.x;
  const int32_t begin = min((int32_t)blockIdx.x * per, total), end = min(begin + per, total);
  if (begin >= end) return;

  // the sequence that tile `t` of the line belongs to
  auto find = [&](int32_t t) {
    uint32_t lo = 0, hi = n_seqs;        // cum[lo] <= t < cum[hi]
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) >> 1;
      if (cum[mid] <= t) lo = mid; else hi = mid;
    }
    return lo;
  };

  if (warp == C::kWarps) {
    // ---- producer: one lane per page piece of a tile ---------------------------------------------
    const uint32_t pieces = kKvTile / a.box_rows;
    uint32_t s = find(begin);
    int32_t t = begin;
    uint32_t k = 0;
    bool ok = true;
    while (t < end) {
      while (cum[s + 1] <= t) ++s;
      const KvSeq q = attend_seq(a.b, s);
      const int32_t tile0 = first_position(q, a.window) / (int32_t)kKvTile;
      const int32_t nt = (cum[s + 1] - cum[s]) / (int32_t)hk;
      const int32_t stop = min(end, cum[s + 1]);
      for (; t < stop; ++t, ++k) {
        const int32_t local = t - cum[s], h = local / nt, tile = tile0 + local - h * nt;
        const uint32_t stage = k % C::kStages;
        int32_t page = -1;
        const int32_t pos = tile * (int32_t)kKvTile + (int32_t)(lane * a.box_rows);
        if (lane < pieces && pos < q.len) page = kv_page(a.b, a.c.n_pages, a.c.page_size, s, pos);
        if (k >= C::kStages) ok = wait_or_give_up(empty + 8 * stage, (k / C::kStages + 1) & 1, ok, a.error);
        const uint32_t st = base + stage * C::kStageBytes, bar = full + 8 * stage;
        if (lane < pieces) {
          const uint32_t slot = (uint32_t)pos % a.c.page_size, row = lane * a.box_rows;
          const int32_t where = page < 0 ? (int32_t)a.c.n_pages : page;      // outside: zeros
          uint32_t bytes = 2 * a.box_rows * C::kRowBytes;
          if (Q && page >= 0) bytes += 2 * a.box_rows * 4;
          if (Q && page < 0)
            for (uint32_t i = 0; i < a.box_rows; ++i) {
              float* sc = reinterpret_cast<float*>(gen + scale_base + stage * (2 * C::kScaleBytes)) + row + i;
              sc[0] = 0.f;
              sc[kKvTile] = 0.f;
            }
          bar_arrive_tx(bar, bytes);
#pragma unroll
          for (uint32_t i = 0; i < C::kSpans; ++i) {
            const uint32_t off = i * (kKvTile * C::kSpan) + row * C::kSpan;
            load_box(st + off, &map_k, (int32_t)(i * C::kSpan / C::kElem), (int32_t)slot, h, where, bar);
            load_box(st + C::kTileBytes + off, &map_v, (int32_t)(i * C::kSpan / C::kElem), (int32_t)slot, h, where, bar);
          }
          if (Q && page >= 0) {
            const uint64_t at = ((uint64_t)page * hk + h) * a.c.page_size + slot;
            const uint32_t to = base + scale_base + stage * (2 * C::kScaleBytes) + row * 4;
            load_bulk(to, a.c.k_scale + at, a.box_rows * 4, bar);
            load_bulk(to + C::kScaleBytes, a.c.v_scale + at, a.box_rows * 4, bar);
          }
        } else {
          bar_arrive(bar);
        }
      }
    }
    return;      // the compute warps wait for every load
  }

  // ---- compute warps ---------------------------------------------------------------------------------
  const uint32_t mt = warp >> 2, kw = warp & 3, t4 = lane & 3, r8 = lane >> 2;
  const float c2 = a.scale_log2;
  uint32_t s = find(begin), k = 0;
  int32_t t = begin;
  bool ok = true;
  while (t < end) {
    while (cum[s + 1] <= t) ++s;
    const KvSeq seq = attend_seq(a.b, s);
    const int32_t tile0 = first_position(seq, a.window) / (int32_t)kKvTile;
    const int32_t nt = (cum[s + 1] - cum[s]) / (int32_t)hk;
    const int32_t h = (t - cum[s]) / nt, item0 = cum[s] + h * nt, item1 = item0 + nt, stop = min(end, item1);
    const uint32_t n_rows = (uint32_t)seq.n_new * a.group;

    // this lane's two query rows: their range of positions and their fragments
    int32_t hi[2], lo[2];
    uint32_t qf[D / 16][4];
    int32_t token[2];
    uint32_t head[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t r = mt * 16 + r8 + 8 * j;
      const bool in = r < n_rows;
      const uint32_t i = in ? r / a.group : 0;
      token[j] = in ? seq.row0 + (int32_t)i : -1;
      head[j] = (uint32_t)h * a.group + (in ? r - i * a.group : 0);
      hi[j] = in ? seq.len - seq.n_new + (int32_t)i : 0x7FFFFFFF;      // a row that is none sees everything
      lo[j] = in && a.window ? hi[j] - (int32_t)a.window + 1 : 0;
      const char* src = a.q + (uint64_t)max(token[j], 0) * a.q_token + head[j] * a.q_head;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        uint32_t x = 0, y = 0;
        if (in) {
          if (Q) {   // the k index of an instruction is permuted alike in both operands: four adjacent codes per lane
            const uint2 w = __ldg(reinterpret_cast<const uint2*>(src + ks * 32 + t4 * 8));
            x = w.x; y = w.y;
          } else {
            x = __ldg(reinterpret_cast<const uint32_t*>(src + ks * 32 + t4 * 4));
            y = __ldg(reinterpret_cast<const uint32_t*>(src + ks * 32 + 16 + t4 * 4));
          }
        }
        qf[ks][j] = x;
        qf[ks][2 + j] = y;
      }
    }
    const int32_t first_hi = seq.len - seq.n_new, last_lo = a.window ? seq.len - (int32_t)a.window : 0;

    float acc[D / 8][4];
#pragma unroll
    for (int i = 0; i < D / 8; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
    float top[2] = {-INFINITY, -INFINITY}, mc[2] = {0.f, 0.f}, sum[2] = {0.f, 0.f};   // raw maximum; maximum * c2, rounded once

    for (; t < stop; ++t, ++k) {
      const uint32_t stage = k % C::kStages;
      ok = wait_or_give_up(full + 8 * stage, (k / C::kStages) & 1, ok, a.error);
      const uint32_t st = base + stage * C::kStageBytes;
      const int32_t pos0 = (tile0 + t - item0) * (int32_t)kKvTile + (int32_t)(kw * 16);
      float sc[2][4] = {};
      // scores of 16 rows x 16 keys
      if (Q) {
        const uint32_t row = kw * 16 + (lane & 15);
#pragma unroll
        for (int ks = 0; ks < D / 16; ks += 2) {
          uint32_t w[4];
          ldsm4(st + swizzled<C::kSpan>(row, ks + (lane >> 4)), w);
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
              const uint32_t x = w[2 * u + n];
              mma16816(sc[n], qf[ks + u], e4m3_to_bf16x2(__byte_perm(x, 0, 0x1404)), e4m3_to_bf16x2(__byte_perm(x, 0, 0x3424)));
            }
        }
      } else {
        const uint32_t row = kw * 16 + (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          uint32_t w[4];
          ldsm4(st + (ks >> 2) * (kKvTile * 128) + swizzled<128>(row, (ks & 3) * 2 + ((lane >> 3) & 1)), w);
          mma16816(sc[0], qf[ks], w[0], w[1]);
          mma16816(sc[1], qf[ks], w[2], w[3]);
        }
      }
      float vs[2][2] = {{1.f, 1.f}, {1.f, 1.f}};
      if (Q) {
        const float2* scales = reinterpret_cast<const float2*>(gen + scale_base + stage * (2 * C::kScaleBytes)) + kw * 8;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const float2 ksc = scales[n * 4 + t4], vsc = scales[kKvTile / 2 + n * 4 + t4];
          sc[n][0] *= ksc.x; sc[n][1] *= ksc.y; sc[n][2] *= ksc.x; sc[n][3] *= ksc.y;
          vs[n][0] = vsc.x; vs[n][1] = vsc.y;
        }
      }
      // a tile that some row sees only in part, or that passes the end of the cache
      const bool partial = pos0 + 15 > first_hi || pos0 < last_lo;
      if (partial) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int32_t pos = pos0 + n * 8 + (int32_t)t4 * 2 + (e & 1);
            if (pos > hi[e >> 1] || pos < lo[e >> 1]) sc[n][e] = -INFINITY;
          }
      }
      // running maximum; the accumulators are rescaled only when some row's maximum moved
      float corr[2];
      bool moved = false;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float m = fmaxf(fmaxf(sc[0][2 * j], sc[0][2 * j + 1]), fmaxf(sc[1][2 * j], sc[1][2 * j + 1]));
        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
        corr[j] = 1.f;
        if (m > top[j]) {
          moved = true;
          const float next = m * c2;
          corr[j] = top[j] == -INFINITY ? 0.f : fast_exp2(mc[j] - next);
          top[j] = m;
          mc[j] = next;
        }
      }
      if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          acc[i][0] *= corr[0]; acc[i][1] *= corr[0];
          acc[i][2] *= corr[1]; acc[i][3] *= corr[1];
        }
        sum[0] *= corr[0];
        sum[1] *= corr[1];
      }
      uint32_t pf[4];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[e] = fast_exp2(fmaf(sc[n][e], c2, -mc[e >> 1]));
          sum[e >> 1] += p[e];
          // a scale of a position that is not seen may be anything
          if (Q) p[e] = partial && p[e] == 0.f ? 0.f : p[e] * vs[n][e & 1];
          sc[n][e] = p[e];
        }
        pf[2 * n] = pack_bf16x2(p[0], p[1]);
        pf[2 * n + 1] = pack_bf16x2(p[2], p[3]);
      }
      // values
      const uint32_t sv = st + C::kTileBytes;
      if (Q) {
        const uint32_t row = kw * 16 + (lane & 15);
#pragma unroll
        for (int c = 0; c < D / 16; c += 2) {
          uint32_t w[4];
          ldsm4t(sv + swizzled<C::kSpan>(row, c + (lane >> 4)), w);
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint32_t x = w[2 * u], y = w[2 * u + 1];
            mma16816(acc[2 * (c + u)], pf, e4m3_to_bf16x2(__byte_perm(x, 0, 0x2404)), e4m3_to_bf16x2(__byte_perm(y, 0, 0x2404)));
            mma16816(acc[2 * (c + u) + 1], pf, e4m3_to_bf16x2(__byte_perm(x, 0, 0x3414)), e4m3_to_bf16x2(__byte_perm(y, 0, 0x3414)));
          }
        }
      } else {
        const uint32_t row = kw * 16 + (lane & 15);
        // bf16 values of positions that a row does not see are multiplied by a weight of zero, which only finite
        // ones survive: those past the end are cleared, and where the tile's own chunk or a window cuts it, values
        // that are not finite are taken out and added by hand to the rows that do see them
        uint32_t keep[2] = {0xFFFFFFFFu, 0xFFFFFFFFu};
        bool odd = false;
        if (partial) {
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const int32_t pos = pos0 + n * 8 + (int32_t)t4 * 2;
            keep[n] = (pos < seq.len ? 0xFFFFu : 0u) | (pos + 1 < seq.len ? 0xFFFF0000u : 0u);
          }
        }
#pragma unroll
        for (int c = 0; c < D / 8; c += 2) {
          uint32_t w[4];
          ldsm4t(sv + (c >> 3) * (kKvTile * 128) + swizzled<128>(row, (c & 7) + (lane >> 4)), w);
          if (partial) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              w[i] &= keep[i & 1];
              if (not_finite_bf16x2(w[i])) {
                odd = true;
                if ((w[i] & 0x7F80u) == 0x7F80u) w[i] &= 0xFFFF0000u;
                if ((w[i] & 0x7F800000u) == 0x7F800000u) w[i] &= 0xFFFFu;
              }
            }
          }
          mma16816(acc[c], pf, w[0], w[1]);
          mma16816(acc[c + 1], pf, w[2], w[3]);
        }
        if (partial && __any_sync(0xFFFFFFFFu, odd)) {
          const char* vals = gen + stage * C::kStageBytes + C::kTileBytes;
#pragma unroll
          for (int key = 0; key < 16; ++key) {
            const int from = (int)(lane & ~3u) + ((key & 7) >> 1);
            const float p0 = __shfl_sync(0xFFFFFFFFu, sc[key >> 3][key & 1], from);
            const float p1 = __shfl_sync(0xFFFFFFFFu, sc[key >> 3][2 + (key & 1)], from);
            const int32_t pos = pos0 + key;
            if (pos >= seq.len) continue;
            const uint32_t vr = kw * 16 + key;
#pragma unroll 1
            for (int c = 0; c < D / 8; ++c) {
              const uint32_t v = *reinterpret_cast<const uint32_t*>(vals + (c >> 3) * (kKvTile * 128) + swizzled<128>(vr, c & 7) + t4 * 4);
              if (!not_finite_bf16x2(v)) continue;
              const float x = bf16_lo(v), y = bf16_hi(v);
              const bool ox = (v & 0x7F80u) == 0x7F80u, oy = (v & 0x7F800000u) == 0x7F800000u;
#pragma unroll
              for (int cc = 0; cc < D / 8; ++cc)
                if (cc == c) {
                  if (pos <= hi[0] && pos >= lo[0]) { if (ox) acc[cc][0] += p0 * x; if (oy) acc[cc][1] += p0 * y; }
                  if (pos <= hi[1] && pos >= lo[1]) { if (ox) acc[cc][2] += p1 * x; if (oy) acc[cc][3] += p1 * y; }
                }
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) bar_arrive(empty + 8 * stage);
    }

    // ---- join the four warps of these query rows, in order ----------------------------------------
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      sum[j] += __shfl_xor_sync(0xFFFFFFFFu, sum[j], 1);
      sum[j] += __shfl_xor_sync(0xFFFFFFFFu, sum[j], 2);
      if (t4 == 0) warp_ml[(mt * 4 + kw) * 16 + r8 + 8 * j] = make_float2(top[j] == -INFINITY ? -INFINITY : mc[j], sum[j]);
    }
    asm volatile("bar.sync 1, %0;" ::"n"(32 * C::kWarps) : "memory");
    float all_m[2], all_l[2], mine[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float2 ml[4];
      all_m[j] = -INFINITY;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        ml[w] = warp_ml[(mt * 4 + w) * 16 + r8 + 8 * j];
        all_m[j] = fmaxf(all_m[j], ml[w].x);
      }
      all_l[j] = 0.f;
      mine[j] = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = ml[w].x == -INFINITY ? 0.f : fast_exp2(ml[w].x - all_m[j]);
        all_l[j] += ml[w].y * f;
        if (w == (int)kw) mine[j] = f;
      }
    }
    float* buf = join + mt * (C::kRegs * 32) + lane;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (w == (int)kw) {
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = acc[i][e] * mine[e >> 1];
            if (w > 0) x += buf[(i * 4 + e) * 32];
            if (w < 3) buf[(i * 4 + e) * 32] = x;
            acc[i][e] = x;
          }
      }
      asm volatile("bar.sync 1, %0;" ::"n"(32 * C::kWarps) : "memory");
    }

    // ---- result: whole items directly, cut ones through the workspace ------------------------------
    const bool whole = item0 >= begin && item1 <= end;
    if (!whole && kw == 3) {
      float* part = a.partials + (size_t)(2 * blockIdx.x + (item0 >= begin ? 1 : 0)) * C::kPartFloats + mt * (C::kRegs * 32 + 32);
#pragma unroll
      for (int i = 0; i < D / 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) __stcg(part + (i * 4 + e) * 32 + lane, acc[i][e]);
      if (t4 == 0) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          __stcg(part + C::kRegs * 32 + r8 + 8 * j, all_m[j]);
          __stcg(part + C::kRegs * 32 + 16 + r8 + 8 * j, all_l[j]);
        }
      }
      __threadfence();
    }
    bool mine_to_write = whole && kw == 3;
    uint32_t i0 = 0, i1 = D / 8;
    if (!whole) {
      asm volatile("bar.sync 1, %0;" ::"n"(32 * C::kWarps) : "memory");
      const uint32_t first = (uint32_t)(item0 / per), count = (uint32_t)((item1 - 1) / per) - first + 1;
      if (tid == 0) {
        __threadfence();
        s_last = atomicAdd(a.counters + first, 1u) == count - 1;
        if (s_last) a.counters[first] = 0;
      }
      asm volatile("bar.sync 1, %0;" ::"n"(32 * C::kWarps) : "memory");
      if (s_last) {
        // every block's part is there: each warp joins a quarter of its rows' columns
        __threadfence();
        mine_to_write = true;
        i0 = kw * (D / 32);
        i1 = i0 + D / 32;
        auto part_of = [&](uint32_t p) {
          return a.partials + (size_t)(2 * (first + p) + (p == 0 ? 1 : 0)) * C::kPartFloats + mt * (C::kRegs * 32 + 32);
        };
        all_m[0] = all_m[1] = -INFINITY;
        for (uint32_t p = 0; p < count; ++p)
#pragma unroll
          for (int j = 0; j < 2; ++j) all_m[j] = fmaxf(all_m[j], __ldcg(part_of(p) + C::kRegs * 32 + r8 + 8 * j));
        float o[D / 32][4] = {};
        all_l[0] = all_l[1] = 0.f;
#pragma unroll 2
        for (uint32_t p = 0; p < count; ++p) {
          const float* part = part_of(p);
          float f[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float m = __ldcg(part + C::kRegs * 32 + r8 + 8 * j);
            f[j] = m == -INFINITY ? 0.f : fast_exp2(m - all_m[j]);
            all_l[j] += f[j] * __ldcg(part + C::kRegs * 32 + 16 + r8 + 8 * j);
          }
#pragma unroll
          for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][e] += f[e >> 1] * __ldcg(part + ((i0 + i) * 4 + e) * 32 + lane);
        }
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if ((uint32_t)i / (D / 32) == kw) acc[i][e] = o[i % (D / 32)][e];
      }
    }
    if (mine_to_write) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (token[j] < 0) continue;
        const float inv = all_l[j] > 0.f ? 1.f / all_l[j] : all_l[j] == 0.f ? 0.f : NAN;
        char* dst = a.out + (uint64_t)token[j] * a.o_token + head[j] * a.o_head;
#pragma unroll
        for (uint32_t i = 0; i < D / 8; i += 2) {
          if (i < i0 || i >= i1) continue;
          if (Q) {
            *reinterpret_cast<uint2*>(dst + (i * 8 + 4 * t4) * 2) =
                make_uint2(pack_bf16x2(acc[i][2 * j] * inv, acc[i + 1][2 * j] * inv), pack_bf16x2(acc[i][2 * j + 1] * inv, acc[i + 1][2 * j + 1] * inv));
          } else {
            *reinterpret_cast<uint32_t*>(dst + (i * 8 + 2 * t4) * 2) = pack_bf16x2(acc[i][2 * j] * inv, acc[i][2 * j + 1] * inv);
            *reinterpret_cast<uint32_t*>(dst + (i * 8 + 8 + 2 * t4) * 2) = pack_bf16x2(acc[i + 1][2 * j] * inv, acc[i + 1][2 * j + 1] * inv);
          }
        }
        if (a.lse && i0 == 0 && t4 == 0)
          a.lse[(uint64_t)token[j] * a.n_heads + head[j]] = all_l[j] == 0.f ? -INFINITY : (all_m[j] + log2f(all_l[j])) * kLn2;
      }
    }
  }
}

}  // namespace wbi
