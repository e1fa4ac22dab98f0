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

// Eight elements of a row, the unit of a lane: 16 bytes of bf16, 32 of fp32, 8 codes.
template <bool F32>
__device__ __forceinline__ void load8(const char* p, float* x) {
  if (F32) {
    const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  } else {
    const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
  }
}
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

// Where the block's tokens live: page and slot of each, page -1 for one that has no place.
__device__ __forceinline__ void place_tokens(const KvView& c, const KvBatch& b, uint32_t t0, uint32_t n, int2* place) {
  for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) {
    const int32_t row = (int32_t)(t0 + i);
    const uint32_t s = kv_seq_of_row(b, row);
    const KvSeq q = kv_seq(b, s);
    const int32_t at = row - q.row0;
    const int32_t pos = q.len - q.n_new + at;
    const bool in = at >= 0 && at < q.n_new;
    const int32_t page = in ? kv_page(b, c.n_pages, c.page_size, s, pos) : -1;
    place[i] = make_int2(page, page < 0 ? 0 : pos % (int32_t)c.page_size);
  }
  __syncthreads();
}

// step tensor -> cache.  A row is D / 8 lanes wide; its maximum is found across them.
template <int D, bool F32, bool Q>
__global__ void __launch_bounds__(kRowThreads)
wb_kv_write_kernel(KvView c, KvBatch b, Rows k, Rows v, uint32_t per_block) {
  constexpr uint32_t LANES = D / 8, ROWS = kRowThreads / LANES;
  __shared__ int2 place[kTokensPerBlock];
  const uint32_t t0 = blockIdx.x * per_block, n = min(per_block, b.n_tokens - t0);
  place_tokens(c, b, t0, n, place);
  const uint32_t lane = threadIdx.x % LANES, per_token = 2 * c.n_kv_heads;
  const uint32_t total = n * per_token, padded = (total + ROWS - 1) / ROWS * ROWS;
#pragma unroll 4
  for (uint32_t r = threadIdx.x / LANES; r < padded; r += ROWS) {
    const bool in = r < total;
    const uint32_t i = in ? r / per_token : 0, w = in ? r - i * per_token : 0;
    const bool is_v = w >= c.n_kv_heads;
    const uint32_t h = is_v ? w - c.n_kv_heads : w;
    const int2 at = place[i];
    const bool live = in && at.x >= 0;
    const Rows& src = is_v ? v : k;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
    if (live) load8<F32>(src.data + (t0 + i) * src.token_stride + h * src.head_stride + lane * (F32 ? 32 : 16), x);
    char* base = is_v ? c.v : c.k;
    const uint64_t off = (uint64_t)at.x * c.page_stride + h * c.head_stride + (uint32_t)at.y * D + lane * 8;
    if (!Q) {
      if (live) store8<false>(base + off * 2, x);
      continue;
    }
    // magnitudes are compared as unsigned patterns, so that a NaN wins and makes the whole row NaN
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(x[e]) & 0x7FFFFFFFu);
#pragma unroll
    for (uint32_t d = LANES / 2; d; d >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
    const float amax = __uint_as_float(m);
    float scale = 1.f, inv = 1.f;
    if (m) {
      scale = __fdiv_rn(amax, 448.f);
      if (scale == 0.f) scale = __uint_as_float(1u);
      inv = __fdiv_rn(448.f, amax);
    }
    if (!isfinite(inv)) {   // 448 / amax overflows (or is NaN): divide instead
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = __fdiv_rn(x[e], scale);
      inv = 1.f;
    }
    if (live) {
      uint2 codes;
      codes.x = pack_e4m3x2(x[0] * inv, x[1] * inv) | (uint32_t)pack_e4m3x2(x[2] * inv, x[3] * inv) << 16;
      codes.y = pack_e4m3x2(x[4] * inv, x[5] * inv) | (uint32_t)pack_e4m3x2(x[6] * inv, x[7] * inv) << 16;
      __stcs(reinterpret_cast<uint2*>(base + off), codes);
      if (lane == 0) (is_v ? c.v_scale : c.k_scale)[((uint64_t)at.x * c.n_kv_heads + h) * c.page_size + at.y] = scale;
    }
  }
}

// cache -> step tensor
template <int D, bool F32, bool Q>
__global__ void __launch_bounds__(kRowThreads)
wb_kv_read_kernel(KvView c, KvBatch b, Rows k, Rows v, uint32_t per_block) {
  constexpr uint32_t LANES = D / 8, ROWS = kRowThreads / LANES;
  __shared__ int2 place[kTokensPerBlock];
  const uint32_t t0 = blockIdx.x * per_block, n = min(per_block, b.n_tokens - t0);
  place_tokens(c, b, t0, n, place);
  const uint32_t lane = threadIdx.x % LANES, per_token = 2 * c.n_kv_heads, total = n * per_token;
#pragma unroll 4
  for (uint32_t r = threadIdx.x / LANES; r < total; r += ROWS) {
    const uint32_t i = r / per_token, w = r - i * per_token;
    const bool is_v = w >= c.n_kv_heads;
    const uint32_t h = is_v ? w - c.n_kv_heads : w;
    const int2 at = place[i];
    const char* base = is_v ? c.v : c.k;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
    if (at.x >= 0) {
      const uint64_t off = (uint64_t)at.x * c.page_stride + h * c.head_stride + (uint32_t)at.y * D + lane * 8;
      if (Q) {
        const uint2 codes = __ldcs(reinterpret_cast<const uint2*>(base + off));
        const float s = __ldg((is_v ? c.v_scale : c.k_scale) + ((uint64_t)at.x * c.n_kv_heads + h) * c.page_size + at.y);
        const uint32_t q[2] = {codes.x, codes.y};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = unpack_e4m3x2((uint16_t)(q[e >> 1] >> (16 * (e & 1))));
          x[2 * e] = f.x * s;
          x[2 * e + 1] = f.y * s;
        }
      } else {
        load8<false>(base + off * 2, x);
      }
    }
    const Rows& dst = is_v ? v : k;
    store8<F32>(dst.data + (t0 + i) * dst.token_stride + h * dst.head_stride + lane * (F32 ? 32 : 16), x);
  }
}

template <bool WRITE, int D, bool F32, bool Q>
void launch_rows(const KvView& c, const KvBatch& b, const Rows& k, const Rows& v, cudaStream_t stream) {
  // as many tokens per block as leave eight blocks for every SM
  const uint32_t per = std::min(kTokensPerBlock, std::max(1u, b.n_tokens / (kNumSMs * 8)));
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
