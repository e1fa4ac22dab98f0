// Paged key/value cache: opening a cache, appending new tokens' keys and values to it (quantised to
// E4M3 with one scale per row, or rounded to bf16), and reading rows back.
//
// Both directions move rows of head_dim elements between a step's tensor [token][head][D] and the
// slots of the batch's positions; each element is read once and written once, so the bound is memory
// bandwidth (and, for one token per sequence, the chain of dependent loads batch -> table -> row).
#include <algorithm>
#include <cstdlib>
#include <cstring>
#include <new>
#include <numeric>

#include "wb_kv.cuh"

using namespace wbi;

namespace {

constexpr uint32_t kRowThreads = 256;
constexpr uint32_t kTokensPerBlock = 32;   // at most; fewer where that leaves SMs without a block

struct Rows {
  char* data;
  uint64_t token_stride, head_stride;   // bytes
};

Rows rows_of(const wb_heads* h) {
  const uint64_t e = h->dtype == WB_F32 ? 4 : 2;
  return Rows{(char*)h->data, h->token_stride * e, h->head_stride * e};
}

// Eight elements of a row, the unit of a lane: 16 bytes of bf16, 32 of fp32.
template <bool F32>
__device__ __forceinline__ void store8(char* p, const float* x) {
  if (F32) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(x[0], x[1], x[2], x[3]));
    __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(x[4], x[5], x[6], x[7]));
  } else {
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                                   pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])));
  }
}

// Where the block's tokens live: page and slot of each, page -1 for one that has no place.  One warp: it finds the first token's
// sequence by a 32-way search (a load per factor of 32, where a search per token would be five), and the others' by counting
// the starts that follow.
__device__ __forceinline__ void place_tokens(const KvView& c, const KvBatch& b, uint32_t t0, uint32_t n, int2* place) {
  if (threadIdx.x < 32) {
    const uint32_t lane = threadIdx.x;
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
    }
  }
  __syncthreads();
}

// step tensor -> cache.  A thread has 32 elements of a row, as four pieces of 8 (D / 32 pieces apart, so that the threads of a row
// read and write whole sectors): with so few threads to a row its maximum takes two exchanges at most, and the two exact divisions
// of its scale are shared by 32 elements (16 threads to a row, 8 elements each: 42 us for 13.4 thousand tokens of 8 heads of 128
// where this takes 18.4 to 20.5, 4.5 to 4.1 TB/s; what it writes, 28 MB, stays in the second-level cache).
template <int D, bool F32, bool Q>
__global__ void __launch_bounds__(kRowThreads, F32 ? 4 : 6)
wb_kv_write_kernel(KvView c, KvBatch b, Rows k, Rows v, uint32_t per_block) {
  constexpr uint32_t LANES = D / 32, ROWS = kRowThreads / LANES, N = F32 ? 2 : 1;      // N 16-byte loads for 8 elements
  __shared__ int2 place[kTokensPerBlock];
  const uint32_t t0 = blockIdx.x * per_block, n = min(per_block, b.n_tokens - t0);
  const uint32_t lane = threadIdx.x % LANES, per_token = 2 * c.n_kv_heads, total = n * per_token;
  bool placed = false;
  for (uint32_t r = threadIdx.x / LANES; r < (total + ROWS - 1) / ROWS * ROWS; r += ROWS) {
    const bool in = r < total;
    const uint32_t tok = in ? r / per_token : 0, w = in ? r - tok * per_token : 0;
    const bool is_v = w >= c.n_kv_heads;
    const uint32_t h = w - (is_v ? c.n_kv_heads : 0);
    const Rows& src = is_v ? v : k;
    const char* from = src.data + (uint64_t)(t0 + tok) * src.token_stride + h * src.head_stride + lane * (16 * N);
    uint4 raw[4][N];               // as loaded: the rows wait in half the registers that their values would take
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j)
#pragma unroll
      for (uint32_t i = 0; i < N; ++i)
        raw[j][i] = in ? __ldcs(reinterpret_cast<const uint4*>(from + j * (LANES * 16 * N)) + i) : make_uint4(0, 0, 0, 0);
    if (!placed) {                 // the rows are on their way meanwhile
      place_tokens(c, b, t0, n, place);
      placed = true;
    }
    const int2 at = place[tok];
    const bool live = in && at.x >= 0;
    char* base = is_v ? c.v : c.k;
    const uint64_t off = (uint64_t)(uint32_t)at.x * c.page_stride + h * c.head_stride + (uint32_t)at.y * D + lane * 8;
    if (!Q) {
      if (live)
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
          uint4 y = raw[j][0];
          if (F32)
            y = make_uint4(pack_bf16x2(__uint_as_float(raw[j][0].x), __uint_as_float(raw[j][0].y)), pack_bf16x2(__uint_as_float(raw[j][0].z), __uint_as_float(raw[j][0].w)),
                           pack_bf16x2(__uint_as_float(raw[j][N - 1].x), __uint_as_float(raw[j][N - 1].y)), pack_bf16x2(__uint_as_float(raw[j][N - 1].z), __uint_as_float(raw[j][N - 1].w)));
          __stcs(reinterpret_cast<uint4*>(base + (off + j * (LANES * 8)) * 2), y);
        }
      continue;
    }
    auto value = [&](uint32_t j, int e) {
      if (F32) {
        const uint4 q = raw[j][e / 4 % N];
        return __uint_as_float(e % 4 == 0 ? q.x : e % 4 == 1 ? q.y : e % 4 == 2 ? q.z : q.w);
      }
      const uint4 q = raw[j][0];
      const uint32_t word = e / 2 == 0 ? q.x : e / 2 == 1 ? q.y : e / 2 == 2 ? q.z : q.w;
      return e & 1 ? bf16_hi(word) : bf16_lo(word);
    };
    // magnitudes are compared as unsigned patterns, so that a NaN wins and makes the whole row NaN
    uint32_t m = 0;
    if (F32) {
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(value(j, e)) & 0x7FFFFFFFu);
    } else {
      uint32_t m2 = 0;             // two at a time
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) {
        m2 = __vmaxu2(m2, __vmaxu2(raw[j][0].x & 0x7FFF7FFFu, raw[j][0].y & 0x7FFF7FFFu));
        m2 = __vmaxu2(m2, __vmaxu2(raw[j][0].z & 0x7FFF7FFFu, raw[j][0].w & 0x7FFF7FFFu));
      }
      m = max(m2 << 16, m2 & 0xFFFF0000u);
    }
#pragma unroll
    for (uint32_t d = LANES / 2; d; d >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
    const float amax = __uint_as_float(m);
    float scale = 1.f, inv = 1.f;
    if (m) {
      scale = __fdiv_rn(amax, 448.f);
      if (scale == 0.f) scale = __uint_as_float(1u);
      inv = __fdiv_rn(448.f, amax);
    }
    if (!live) continue;
    const bool divide = !isfinite(inv);       // 448 / amax overflows (or is NaN): divide by the scale instead
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
      uint32_t code[4];
      if (divide) {
#pragma unroll
        for (int e = 0; e < 4; ++e) code[e] = pack_e4m3x2(__fdiv_rn(value(j, 2 * e), scale), __fdiv_rn(value(j, 2 * e + 1), scale));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) code[e] = pack_e4m3x2(value(j, 2 * e) * inv, value(j, 2 * e + 1) * inv);
      }
      *reinterpret_cast<uint2*>(base + off + j * (LANES * 8)) = make_uint2(code[0] | code[1] << 16, code[2] | code[3] << 16);
    }
    if (lane == 0) (is_v ? c.v_scale : c.k_scale)[((uint64_t)(uint32_t)at.x * c.n_kv_heads + h) * c.page_size + at.y] = scale;
  }
}

constexpr uint32_t kAhead = 4;      // rows whose loads a thread has in flight

// cache -> step tensor.  56 thousand tokens of 8 heads of 128 from codes to bf16: 67.5 to 69 us, 5.1 TB/s.
template <int D, bool F32, bool Q>
__global__ void __launch_bounds__(kRowThreads)
wb_kv_read_kernel(KvView c, KvBatch b, Rows k, Rows v, uint32_t per_block) {
  constexpr uint32_t LANES = D / 8, ROWS = kRowThreads / LANES;
  __shared__ int2 place[kTokensPerBlock];
  const uint32_t t0 = blockIdx.x * per_block, n = min(per_block, b.n_tokens - t0);
  place_tokens(c, b, t0, n, place);
  const uint32_t lane = threadIdx.x % LANES, per_token = 2 * c.n_kv_heads, total = n * per_token;
  for (uint32_t r0 = threadIdx.x / LANES; r0 < total; r0 += kAhead * ROWS) {
    uint4 raw[kAhead];
    float scale[kAhead];
    uint32_t tok[kAhead], which[kAhead];
#pragma unroll
    for (uint32_t u = 0; u < kAhead; ++u) {
      const uint32_t r = min(r0 + u * ROWS, total - 1);      // (the last rows may be read again, not written)
      tok[u] = r / per_token;
      which[u] = r - tok[u] * per_token;
      const bool is_v = which[u] >= c.n_kv_heads;
      const uint32_t h = which[u] - (is_v ? c.n_kv_heads : 0);
      const int2 at = place[tok[u]];
      raw[u] = make_uint4(0, 0, 0, 0);
      scale[u] = 0.f;
      if (at.x >= 0) {
        const char* src = (is_v ? c.v : c.k) + ((uint64_t)(uint32_t)at.x * c.page_stride + h * c.head_stride + (uint32_t)at.y * D + lane * 8) * (Q ? 1 : 2);
        if (Q) {
          const uint2 x = __ldcs(reinterpret_cast<const uint2*>(src));
          raw[u].x = x.x;
          raw[u].y = x.y;
          scale[u] = __ldg((is_v ? c.v_scale : c.k_scale) + ((uint64_t)(uint32_t)at.x * c.n_kv_heads + h) * c.page_size + at.y);
        } else {
          raw[u] = __ldcs(reinterpret_cast<const uint4*>(src));
        }
      }
    }
#pragma unroll
    for (uint32_t u = 0; u < kAhead; ++u) {
      if (r0 + u * ROWS >= total) continue;
      const bool is_v = which[u] >= c.n_kv_heads;
      const Rows& dst = is_v ? v : k;
      char* to = dst.data + (uint64_t)(t0 + tok[u]) * dst.token_stride + (which[u] - (is_v ? c.n_kv_heads : 0)) * dst.head_stride + lane * (F32 ? 32 : 16);
      if (!Q && !F32) {
        __stcs(reinterpret_cast<uint4*>(to), raw[u]);
        continue;
      }
      float x[8];
      const uint32_t w[4] = {raw[u].x, raw[u].y, raw[u].z, raw[u].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (Q) {
          const float2 f = unpack_e4m3x2((uint16_t)(w[e >> 1] >> (16 * (e & 1))));
          x[2 * e] = f.x * scale[u];
          x[2 * e + 1] = f.y * scale[u];
        } else {
          x[2 * e] = bf16_lo(w[e]);
          x[2 * e + 1] = bf16_hi(w[e]);
        }
      }
      store8<F32>(to, x);
    }
  }
}

template <bool WRITE, int D, bool F32, bool Q>
void launch_rows(const KvView& c, const KvBatch& b, const Rows& k, const Rows& v, cudaStream_t stream) {
  // as many tokens per block as leave eight blocks for every SM (four where they are read: measured best of 4, 8, 16)
  const uint32_t per = std::min(kTokensPerBlock, std::max(1u, b.n_tokens / (kNumSMs * (WRITE ? 8 : 4))));
  const uint32_t grid = (b.n_tokens + per - 1) / per;
  if (WRITE) wb_kv_write_kernel<D, F32, Q><<<grid, kRowThreads, 0, stream>>>(c, b, k, v, per);
  else wb_kv_read_kernel<D, F32, Q><<<grid, kRowThreads, 0, stream>>>(c, b, k, v, per);
}

template <bool WRITE>
wb_status move_rows(const wb_kv* kv, const wb_kv_batch* batch, const wb_heads* k, const wb_heads* v, void* stream) {
  if (wb_status s = check_batch(kv, batch)) return s;
  if (wb_status s = check_heads(k, batch->n_tokens, true)) return s;
  if (wb_status s = check_heads(v, batch->n_tokens, true)) return s;
  if (k->dtype != v->dtype) return WB_ERR_DTYPE;
  if (!batch->n_tokens || !batch->n_seqs) return WB_OK;
  const KvView c = kv_view(kv);
  const KvBatch b = kv_batch(batch);
  const Rows rk = rows_of(k), rv = rows_of(v);
  const cudaStream_t st = (cudaStream_t)stream;
  const bool f32 = k->dtype == WB_F32, q = kv->d.dtype == WB_E4M3;
  if (c.head_dim == 128) {
    if (f32) q ? launch_rows<WRITE, 128, true, true>(c, b, rk, rv, st) : launch_rows<WRITE, 128, true, false>(c, b, rk, rv, st);
    else q ? launch_rows<WRITE, 128, false, true>(c, b, rk, rv, st) : launch_rows<WRITE, 128, false, false>(c, b, rk, rv, st);
  } else {
    if (f32) q ? launch_rows<WRITE, 64, true, true>(c, b, rk, rv, st) : launch_rows<WRITE, 64, true, false>(c, b, rk, rv, st);
    else q ? launch_rows<WRITE, 64, false, true>(c, b, rk, rv, st) : launch_rows<WRITE, 64, false, false>(c, b, rk, rv, st);
  }
  return cudaPeekAtLastError() == cudaSuccess ? WB_OK : (cudaGetLastError(), WB_ERR_CUDA);
}

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                   const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                   CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

bool encode_map(const wb_kv_desc& d, void* base, uint32_t box_rows, CUtensorMap* out) {
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult res = cudaDriverEntryPointSymbolNotFound;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &res) != cudaSuccess ||
      res != cudaDriverEntryPointSuccess || !fn) {
    (void)cudaGetLastError();
    return false;
  }
  const bool q = d.dtype == WB_E4M3;
  const uint64_t e = q ? 1 : 2;
  const uint32_t width = std::min<uint32_t>(d.head_dim, 128 / (uint32_t)e);
  const cuuint64_t dims[4] = {d.head_dim, d.page_size, d.n_kv_heads, d.n_pages};
  // a stride of an extent of one is never used, but has to be a legal one
  const uint64_t row = d.head_dim * e, head = d.n_kv_heads > 1 ? d.head_stride * e : row * d.page_size;
  const uint64_t page = d.n_pages > 1 ? d.page_stride * e : head * d.n_kv_heads;
  const cuuint64_t strides[3] = {row, head, page};
  const cuuint32_t box[4] = {width, box_rows, 1, 1}, unit[4] = {1, 1, 1, 1};
  return reinterpret_cast<EncodeTiledFn>(fn)(
             out, q ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, base, dims, strides, box, unit,
             CU_TENSOR_MAP_INTERLEAVE_NONE, width * e == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

extern "C" wb_status wb_kv_open(const wb_kv_desc* d, wb_kv** out) {
  if (!d || !out) return WB_ERR_INVALID_ARG;
  if (d->dtype != WB_BF16 && d->dtype != WB_E4M3) return WB_ERR_DTYPE;
  const uint64_t e = d->dtype == WB_BF16 ? 2 : 1;
  if ((d->head_dim != 64 && d->head_dim != 128) || !d->n_kv_heads || !d->n_pages || !d->page_size || d->page_size % 16 ||
      d->page_size > 65536)
    return WB_ERR_INVALID_ARG;
  if (d->n_pages > 0x7FFFFFFFull || d->n_kv_heads > 65535 ||
      d->n_pages * d->n_kv_heads > 0x7FFFFFFFull / d->page_size)
    return WB_ERR_INVALID_ARG;
  if (!d->k || !d->v || ((uintptr_t)d->k & 15u) || ((uintptr_t)d->v & 15u)) return WB_ERR_INVALID_ARG;
  if (d->page_stride % 16 || d->head_stride % 16 || d->page_stride >= (1ull << 39) / e || d->head_stride >= (1ull << 39) / e)
    return WB_ERR_INVALID_ARG;
  if ((d->n_kv_heads > 1 && d->head_stride < (uint64_t)d->page_size * d->head_dim) ||
      (d->n_pages > 1 && d->page_stride < (uint64_t)(d->n_kv_heads - 1) * d->head_stride + (uint64_t)d->page_size * d->head_dim))
    return WB_ERR_INVALID_ARG;
  if ((d->dtype == WB_E4M3) != (d->k_scale != nullptr) || (d->dtype == WB_E4M3) != (d->v_scale != nullptr)) return WB_ERR_INVALID_ARG;
  if (((uintptr_t)d->k_scale & 15u) || ((uintptr_t)d->v_scale & 15u)) return WB_ERR_INVALID_ARG;
  wb_kv* kv = new (std::nothrow) wb_kv();
  if (!kv) return WB_ERR_OOM;
  kv->d = *d;
  kv->box_rows = std::gcd(d->page_size, kKvTile);
  if (cudaGetDevice(&kv->device) != cudaSuccess) {
    (void)cudaGetLastError();
    delete kv;
    return WB_ERR_CUDA;
  }
  if (!encode_map(kv->d, d->k, kv->box_rows, &kv->map_k) || !encode_map(kv->d, d->v, kv->box_rows, &kv->map_v)) {
    delete kv;
    return WB_ERR_CUDA;
  }
  *out = kv;
  return WB_OK;
}

extern "C" void wb_kv_free(wb_kv* kv) { delete kv; }

extern "C" wb_status wb_kv_write(const wb_kv* kv, const wb_kv_batch* batch, const wb_heads* k, const wb_heads* v, void* stream) {
  return move_rows<true>(kv, batch, k, v, stream);
}

extern "C" wb_status wb_kv_read(const wb_kv* kv, const wb_kv_batch* batch, const wb_heads* k, const wb_heads* v, void* stream) {
  return move_rows<false>(kv, batch, k, v, stream);
}
