// New tokens' keys turned by their positions and appended, with their values, to the paged cache; their queries turned on the
// way.  A pair (a, b) of a row's elements becomes (a cos - b sin, b cos + a sin), the angle of its index at the token's position
// being a row of a table: each product and each sum is rounded to fp32 by itself, then the result to bf16, or to a code
// of the row's own scale.
//
// Each element is read once and written once, so the bound is memory bandwidth: 13.7 thousand tokens of 32 query and 8 key heads of 128, bf16 to
// E4M3, take 59 to 61 us, 5.1 to 5.2 TB/s, into a bf16 cache 62.6, 5.4 TB/s.  (With the next row in registers 72 us, with blocks that look 8 tokens up and end 82: latency, not
// bytes, was what they waited for.)  A thread has 32 elements of a row, as four
// pieces of 8 that lie so that both elements of a pair are in one thread (or in two of one row, where a quarter of the row turns), and
// their 16 angles at most stay in registers while it goes through the rows of one token: the table is read once per token and
// slot instead of once per row.
#include <algorithm>
#include <atomic>

#include "wb_kv.cuh"

using namespace wbi;

namespace {

constexpr uint32_t kThreads = 256;

struct RotateArgs {
  KvView c;
  KvBatch b;
  Rows q, q_out, k, v;
  const float2* table;
  const int32_t* positions;
  uint32_t n_positions, n_heads;
  uint32_t per_block;        // tokens
  uint32_t slots;            // rows of a token that are worked on at once: a power of two, at most kThreads / (D / 32)
};

// Rows in flight per thread: 64 KiB a block, or of fp32 rows 96 KiB, and two blocks an SM (their registers allow no third).
template <bool F32> constexpr uint32_t kDepth = F32 ? 3 : 4;
template <bool F32> constexpr uint32_t kRingBytes = kDepth<F32> * (F32 ? 8 : 4) * kThreads * 16;

// PART: the turning elements are the first D / PART of a row.
template <int D, int PART, bool PAIRS, bool F32, bool Q>
__global__ void __launch_bounds__(kThreads, 2)
wb_kv_write_rotated_kernel(const __grid_constant__ RotateArgs a) {
  constexpr uint32_t LANES = D / 32, ROWS = kThreads / LANES, N = F32 ? 2 : 1, HALF = D / PART / 2;
  constexpr uint32_t DEPTH = kDepth<F32>;
  constexpr int kAngles = PART == 1 ? 16 : 8;      // of a thread: of pieces 0, 1 (2, 3), or of piece 0 or two
  __shared__ int2 places[2][kTokensPerBlock];
  __shared__ int32_t positions[2][kTokensPerBlock];
  const uint32_t t0 = blockIdx.x * a.per_block, n = min(a.per_block, a.b.n_tokens - t0), warp = threadIdx.x / 32;
  const uint32_t lane = threadIdx.x % LANES, row_slot = threadIdx.x / LANES, slot = row_slot % a.slots;
  const uint32_t hk = a.c.n_kv_heads, hq = a.n_heads, rows = hq + 2 * hk, at_once = ROWS / a.slots;
  // A thread's pieces of the rows that come next, asked for DEPTH rows ahead; only the thread itself reads them.
  extern __shared__ uint4 ring[];                  // [DEPTH][4 N][kThreads]
  const uint32_t per_token = (rows + a.slots - 1) / a.slots, steps = (n + at_once - 1) / at_once * per_token;
  uint32_t asked = 0, ask_tok = row_slot / a.slots, ask_r = slot;
  auto ask = [&]() {
    if (asked < steps && ask_tok < n && ask_r < rows) {
      const bool is_q = ask_r < hq, is_v = ask_r >= hq + hk;
      const uint32_t h = is_q ? ask_r : is_v ? ask_r - hq - hk : ask_r - hq;
      const Rows& src = is_q ? a.q : is_v ? a.v : a.k;
      const char* from = src.data + (uint64_t)(t0 + ask_tok) * src.token_stride + h * src.head_stride + lane * (16 * N);
      uint4* to = ring + asked % DEPTH * (4 * N * kThreads) + threadIdx.x;
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j)
#pragma unroll
        for (uint32_t i = 0; i < N; ++i)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to + (j * N + i) * kThreads)),
                       "l"(from + j * (LANES * 16 * N) + i * 16) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    ++asked;
    ask_r += a.slots;
    if (asked % per_token == 0) {
      ask_r = slot;
      ask_tok += at_once;
    }
  };
#pragma unroll
  for (uint32_t i = 0; i < DEPTH; ++i) ask();
  uint32_t step = 0;
  // 32 tokens at a time; one warp finds where the next ones go, and has their angles brought near, while these are worked on
  auto place_ahead = [&](uint32_t c0) {
    const uint32_t m = min(kTokensPerBlock, n - c0), l = threadIdx.x % 32, buf = c0 / kTokensPerBlock & 1;
    place_by_warp(a.c, a.b, t0 + c0, m, places[buf], positions[buf], l);
    if (l < m) {
      const int32_t pos = a.positions ? __ldg(a.positions + t0 + c0 + l) : positions[buf][l];
      if ((uint32_t)pos < a.n_positions)
        for (uint32_t i = 0; i < HALF; i += 16) asm volatile("prefetch.global.L1 [%0];" ::"l"(a.table + (uint64_t)(uint32_t)pos * HALF + i) : "memory");
    }
  };
  if (warp == 0) place_ahead(0);
  for (uint32_t tok0 = 0; tok0 < n; tok0 += at_once) {
    if (tok0 % kTokensPerBlock == 0) {
      __syncthreads();
      if (tok0 + kTokensPerBlock < n && warp == tok0 / kTokensPerBlock % (kThreads / 32)) place_ahead(tok0 + kTokensPerBlock);
    }
    const uint32_t tok = min(tok0 + row_slot / a.slots, n - 1), buf = tok / kTokensPerBlock & 1, in_chunk = tok % kTokensPerBlock;
    const int32_t place_pos = positions[buf][in_chunk];
    const bool mine = tok0 + row_slot / a.slots < n && place_pos != INT32_MIN;
    const uint64_t t = t0 + tok;
    const int32_t pos = a.positions ? __ldg(a.positions + t) : place_pos;
    // a position that the table does not have turns everything into NaN
    const bool known = (uint32_t)pos < a.n_positions;
    float2 cs[kAngles];
    auto fetch = [&](int i, uint32_t index) {        // two angles
      const float4 x = known ? __ldg(reinterpret_cast<const float4*>(a.table + (uint64_t)(uint32_t)pos * HALF + index)) : make_float4(NAN, NAN, NAN, NAN);
      cs[i] = make_float2(x.x, x.y);
      cs[i + 1] = make_float2(x.z, x.w);
    };
    if (PAIRS) {
#pragma unroll
      for (int j = 0; j < (PART == 1 ? 4 : PART == 2 ? 2 : 1); ++j)
#pragma unroll
        for (int i = 0; i < 4; i += 2) fetch(j * 4 + i, (lane * 8 + j * (LANES * 8)) / 2 + i);
    } else {
#pragma unroll
      for (int j = 0; j < (PART == 1 ? 2 : 1); ++j)
#pragma unroll
        for (int i = 0; i < 8; i += 2) fetch(j * 8 + i, (PART == 4 ? lane % (LANES / 2) : lane) * 8 + j * (LANES * 8) + i);
    }
    const int2 at = places[buf][in_chunk];
    for (uint32_t r = slot; r < per_token * a.slots; r += a.slots, ++step) {
      const bool is_q = r < hq, is_v = r >= hq + hk, in = mine && r < rows;
      const uint32_t h = is_q ? r : is_v ? r - hq - hk : r - hq;
      asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
      const uint4* mine_now = ring + step % DEPTH * (4 * N * kThreads) + threadIdx.x;
      float x[4][8];
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) {
        uint4 raw[N];
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) raw[i] = mine_now[(j * N + i) * kThreads];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint4 y = raw[F32 ? e / 4 : 0];
          const uint32_t i = F32 ? e % 4 : e / 2, w = i == 0 ? y.x : i == 1 ? y.y : i == 2 ? y.z : y.w;
          x[j][e] = F32 ? __uint_as_float(w) : e & 1 ? bf16_hi(w) : bf16_lo(w);
        }
      }
      ask();
      auto turn = [&](float& u, float& w, float2 z) {
        const float uc = __fmul_rn(u, z.x), ws = __fmul_rn(w, z.y), wc = __fmul_rn(w, z.x), us = __fmul_rn(u, z.y);
        u = __fsub_rn(uc, ws);
        w = __fadd_rn(wc, us);
      };
      if (PART == 4 && !PAIRS) {      // the partner is in another lane of the row, or, of all but piece 0, nowhere
        const bool second = lane >= LANES / 2;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float other = __shfl_xor_sync(0xFFFFFFFFu, x[0][e], LANES / 2);
          if (!is_v) {
            const float c = __fmul_rn(x[0][e], cs[e].x), s = __fmul_rn(other, cs[e].y);
            x[0][e] = second ? __fadd_rn(c, s) : __fsub_rn(c, s);
          }
        }
      } else if (!is_v) {
        if (PAIRS) {
          // (a quarter of the row in pairs: piece 0 of all lanes)
#pragma unroll
          for (int j = 0; j < (PART == 1 ? 4 : PART == 2 ? 2 : 1); ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) turn(x[j][2 * i], x[j][2 * i + 1], cs[j * 4 + i]);
        } else if (PART == 1) {
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) turn(x[j][e], x[j + 2][e], cs[(j * 8 + e) % kAngles]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) turn(x[0][e], x[1][e], cs[e]);
        }
      }
      const bool live = in && (is_q || at.x >= 0);
      if (is_q || !Q) {
        char* to = is_q ? a.q_out.data + t * a.q_out.token_stride + h * a.q_out.head_stride + lane * 16
                        : (is_v ? a.c.v : a.c.k) + ((uint64_t)(uint32_t)at.x * a.c.page_stride + h * a.c.head_stride + (uint32_t)at.y * D + lane * 8) * 2;
        if (live)
#pragma unroll
          for (uint32_t j = 0; j < 4; ++j)
            __stcs(reinterpret_cast<uint4*>(to + j * (LANES * 16)), make_uint4(pack_bf16x2(x[j][0], x[j][1]), pack_bf16x2(x[j][2], x[j][3]),
                                                                               pack_bf16x2(x[j][4], x[j][5]), pack_bf16x2(x[j][6], x[j][7])));
      }
      if (Q) {
        // magnitudes are compared as unsigned patterns, so that a NaN wins and makes the whole row NaN
        uint32_t m = 0;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(x[j][e]) & 0x7FFFFFFFu);
#pragma unroll
        for (uint32_t d = LANES / 2; d; d >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
        if (!live || is_q) continue;
        const float amax = __uint_as_float(m);
        float scale = 1.f, inv = 1.f;
        if (m) {
          scale = __fdiv_rn(amax, 448.f);
          if (scale == 0.f) scale = __uint_as_float(1u);
          inv = __fdiv_rn(448.f, amax);
        }
        const bool divide = !isfinite(inv);       // 448 / amax overflows (or is NaN): divide by the scale instead
        char* to = (is_v ? a.c.v : a.c.k) + (uint64_t)(uint32_t)at.x * a.c.page_stride + h * a.c.head_stride + (uint32_t)at.y * D + lane * 8;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
          uint32_t code[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            code[e] = divide ? pack_e4m3x2(__fdiv_rn(x[j][2 * e], scale), __fdiv_rn(x[j][2 * e + 1], scale))
                             : pack_e4m3x2(__fmul_rn(x[j][2 * e], inv), __fmul_rn(x[j][2 * e + 1], inv));
          *reinterpret_cast<uint2*>(to + j * (LANES * 8)) = make_uint2(code[0] | code[1] << 16, code[2] | code[3] << 16);
        }
        if (lane == 0) (is_v ? a.c.v_scale : a.c.k_scale)[((uint64_t)(uint32_t)at.x * hk + h) * a.c.page_size + at.y] = scale;
      }
    }
  }
}

template <int D, int PART, bool PAIRS, bool F32, bool Q>
cudaError_t launch_of(const RotateArgs& a, int dev, uint32_t grid, cudaStream_t stream) {
  auto kernel = wb_kv_write_rotated_kernel<D, PART, PAIRS, F32, Q>;
  static std::atomic<uint64_t> done{0};      // devices on which the kernel may have that much shared memory
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (!(done.load(std::memory_order_acquire) & bit)) {
    if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes<F32>)) return e;
    done.fetch_or(bit, std::memory_order_release);
  }
  kernel<<<grid, kThreads, kRingBytes<F32>, stream>>>(a);
  return cudaPeekAtLastError();
}
template <int D, int PART, bool PAIRS>
cudaError_t launch_type(const RotateArgs& a, bool f32, bool q, int dev, uint32_t grid, cudaStream_t stream) {
  if (f32) return q ? launch_of<D, PART, PAIRS, true, true>(a, dev, grid, stream) : launch_of<D, PART, PAIRS, true, false>(a, dev, grid, stream);
  return q ? launch_of<D, PART, PAIRS, false, true>(a, dev, grid, stream) : launch_of<D, PART, PAIRS, false, false>(a, dev, grid, stream);
}
template <int D>
cudaError_t launch_dim(const RotateArgs& a, uint32_t part, bool pairs, bool f32, bool q, int dev, uint32_t grid, cudaStream_t stream) {
  if (part == 1) return pairs ? launch_type<D, 1, true>(a, f32, q, dev, grid, stream) : launch_type<D, 1, false>(a, f32, q, dev, grid, stream);
  if (part == 2) return pairs ? launch_type<D, 2, true>(a, f32, q, dev, grid, stream) : launch_type<D, 2, false>(a, f32, q, dev, grid, stream);
  return pairs ? launch_type<D, 4, true>(a, f32, q, dev, grid, stream) : launch_type<D, 4, false>(a, f32, q, dev, grid, stream);
}

}  // namespace

extern "C" wb_status wb_kv_write_rotated(const wb_kv* kv, const wb_kv_batch* batch, const wb_rotation* rot, const wb_heads* q, uint32_t n_heads,
                                         const wb_heads* q_out, const wb_heads* k, const wb_heads* v, void* stream) {
  if (wb_status s = check_batch(kv, batch)) return s;
  if (wb_status s = check_heads(k, batch->n_tokens, true)) return s;
  if (wb_status s = check_heads(v, batch->n_tokens, true)) return s;
  if (k->dtype != v->dtype) return WB_ERR_DTYPE;
  if ((q != nullptr) != (n_heads != 0) || (q_out != nullptr) != (n_heads != 0) || n_heads > 65535) return WB_ERR_INVALID_ARG;
  if (q) {
    if (wb_status s = check_heads(q, batch->n_tokens, true)) return s;
    if (wb_status s = check_heads(q_out, batch->n_tokens, false)) return s;
    if (q->dtype != k->dtype) return WB_ERR_DTYPE;
    // in place, or into other memory
    if (batch->n_tokens && q->data == q_out->data &&
        (q->dtype != WB_BF16 || q->token_stride != q_out->token_stride || q->head_stride != q_out->head_stride))
      return WB_ERR_INVALID_ARG;
  }
  const uint32_t d = kv->d.head_dim;
  if (!rot || rot->reserved || rot->interleaved > 1 || rot->n_positions > 0x7FFFFFFFu) return WB_ERR_INVALID_ARG;
  if (rot->rotary_dim != d && rot->rotary_dim != d / 2 && rot->rotary_dim != d / 4) return WB_ERR_INVALID_ARG;
  if ((rot->n_positions && !rot->table) || ((uintptr_t)rot->table & 15u) || ((uintptr_t)rot->positions & 3u)) return WB_ERR_INVALID_ARG;
  // the tokens' own places have to be in the table
  if (!rot->positions && batch->max_len > rot->n_positions) return WB_ERR_INVALID_ARG;
  if (!batch->n_tokens || !batch->n_seqs) return WB_OK;
  RotateArgs a = {};
  a.c = kv_view(kv);
  a.b = kv_batch(batch);
  if (q) {
    a.q = rows_of(q);
    a.q_out = rows_of(q_out);
  }
  a.k = rows_of(k);
  a.v = rows_of(v);
  a.table = (const float2*)rot->table;
  a.positions = rot->positions;
  a.n_positions = rot->n_positions;
  a.n_heads = n_heads;
  // Eight slots for a token leave six rows to each of its threads at 32 query and 8 key heads.  With so few tokens that not every SM would
  // get a block, a token gets more of them, up to a slot per row.  The grid is what fits at once.
  const uint32_t most = kThreads / (d / 32);
  a.slots = 8;
  while (a.slots > most / kTokensPerBlock && a.slots / 2 >= n_heads + 2 * a.c.n_kv_heads) a.slots /= 2;
  while (a.slots < most && (uint64_t)batch->n_tokens * a.slots < (uint64_t)most * kNumSMs) a.slots *= 2;
  const uint32_t at_once = most / a.slots, groups = (batch->n_tokens + at_once - 1) / at_once;
  a.per_block = (groups + 2 * kNumSMs - 1) / (2 * kNumSMs) * at_once;
  const uint32_t grid = (batch->n_tokens + a.per_block - 1) / a.per_block, part = d / rot->rotary_dim;
  const bool f32 = k->dtype == WB_F32, e = kv->d.dtype == WB_E4M3, pairs = rot->interleaved != 0;
  const cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t err = d == 128 ? launch_dim<128>(a, part, pairs, f32, e, kv->device, grid, st) : launch_dim<64>(a, part, pairs, f32, e, kv->device, grid, st);
  if (err != cudaSuccess) (void)cudaGetLastError();
  return err == cudaSuccess ? WB_OK : WB_ERR_CUDA;
}
