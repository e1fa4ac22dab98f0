// Attention of a chunk of new tokens over the paged cache.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "wb_attend.cuh"
#include "wb_attend_rows.cuh"

using namespace wbi;

namespace {

constexpr uint32_t kHeaderBytes = 256;
constexpr uint32_t kMaxRowTiles = 3;                    // wb_attend_rows_kernel: up to 16 * 3 rows
constexpr uint32_t kMaxRowBlocks = 2 * kNumSMs;

// One warp per (token, head): lanes own D / 32 elements, keys one after the other, the softmax's maximum
// and sum carried along.
template <int D, bool Q>
__global__ void __launch_bounds__(128) wb_attend_plain_kernel(AttendArgs a, uint32_t skip_rows) {
  constexpr int N = D / 32;
  const uint32_t lane = threadIdx.x & 31;
  const uint64_t id = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (id >= (uint64_t)a.b.n_tokens * a.n_heads) return;
  const int32_t row = (int32_t)(id / a.n_heads);
  const uint32_t h = (uint32_t)(id - (uint64_t)row * a.n_heads), g = h / a.group;
  const uint32_t s = kv_seq_of_row(a.b, row);
  const KvSeq q = attend_seq(a.b, s);
  if (row - q.row0 >= q.n_new || (uint32_t)q.n_new * a.group <= skip_rows) return;
  const int32_t pos = q.len - q.n_new + row - q.row0;
  const int32_t first = a.window && pos >= (int32_t)a.window ? pos - (int32_t)a.window + 1 : 0;
  float x[N], acc[N], top = -INFINITY, sum = 0.f;
  for (int e = 0; e < N; ++e) {
    x[e] = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(a.q + row * a.q_token + h * a.q_head)[lane * N + e] << 16) * a.scale_log2 * kLn2;
    acc[e] = 0.f;
  }
  for (int32_t j = first; j <= pos; ++j) {
    const int32_t page = kv_page(a.b, a.c.n_pages, a.c.page_size, s, j);
    float kk[N], vv[N];
    for (int e = 0; e < N; ++e) kk[e] = vv[e] = 0.f;
    if (page >= 0) {
      const uint32_t slot = (uint32_t)j % a.c.page_size;
      const uint64_t off = (uint64_t)page * a.c.page_stride + g * a.c.head_stride + slot * D + lane * N;
      const uint64_t sc = ((uint64_t)page * a.c.n_kv_heads + g) * a.c.page_size + slot;
      for (int e = 0; e < N; ++e) {
        if (Q) {
          kk[e] = unpack_e4m3x2((uint8_t)a.c.k[off + e]).x * a.c.k_scale[sc];
          vv[e] = unpack_e4m3x2((uint8_t)a.c.v[off + e]).x * a.c.v_scale[sc];
        } else {
          kk[e] = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(a.c.k)[off + e] << 16);
          vv[e] = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(a.c.v)[off + e] << 16);
        }
      }
    }
    float d = 0.f;
    for (int e = 0; e < N; ++e) d += x[e] * kk[e];
    for (int o = 16; o; o >>= 1) d += __shfl_xor_sync(0xFFFFFFFFu, d, o);
    const float m = fmaxf(top, d);
    if (m == -INFINITY) continue;
    const float old = __expf(top - m), w = __expf(d - m);
    sum = sum * old + w;
    for (int e = 0; e < N; ++e) acc[e] = acc[e] * old + w * vv[e];
    top = m;
  }
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
  for (int e = 0; e < N; ++e)
    reinterpret_cast<uint16_t*>(a.out + row * a.o_token + h * a.o_head)[lane * N + e] = (uint16_t)pack_bf16x2(acc[e] * inv, 0.f);
  if (a.lse && lane == 0) a.lse[(uint64_t)row * a.n_heads + h] = sum > 0.f ? top + logf(sum) : -INFINITY;
}

template <int D, bool Q, int MT>
cudaError_t launch_rows(const AttendArgs& a, const wb_kv* kv, cudaStream_t stream) {
  using C = RowsCfg<D, Q, MT>;
  const size_t smem = C::smem_bytes(a.b.n_seqs);
  auto kernel = wb_attend_rows_kernel<D, Q, MT>;
  // every block gets the same share of the tiles, so the grid is exactly what fits at once: two blocks per SM for
  // up to 16 rows (unless thousands of sequences make the table of prefix sums too large), else one
  const uint32_t per_sm = MT == 1 && smem <= 113 * 1024 ? 2 : 1;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  kernel<<<kNumSMs * per_sm, C::kThreads, smem, stream>>>(a, kv->map_k, kv->map_v);
  return cudaPeekAtLastError();
}

template <int D, bool Q>
cudaError_t launch_rows_of(uint32_t rows, const AttendArgs& a, const wb_kv* kv, cudaStream_t stream) {
  if (rows <= 16) return launch_rows<D, Q, 1>(a, kv, stream);
  if (rows <= 32) return launch_rows<D, Q, 2>(a, kv, stream);
  return launch_rows<D, Q, 3>(a, kv, stream);
}

size_t counter_bytes(const wb_kv* kv, uint32_t n_seqs) { return ((size_t)n_seqs * kv->d.n_kv_heads * 4 + 255) / 256 * 256; }
template <int D> constexpr size_t partial_bytes() {
  return (size_t)2 * 4 * std::max(kMaxRowBlocks * RowsCfg<D, false, 1>::kPartFloats, kNumSMs * RowsCfg<D, false, 3>::kPartFloats);
}

}  // namespace

extern "C" size_t wb_kv_attend_workspace_bytes(const wb_kv* kv, uint32_t n_heads, uint32_t n_seqs) {
  if (!kv || !n_heads || n_seqs > WB_KV_MAX_SEQS) return 0;
  return kHeaderBytes + counter_bytes(kv, n_seqs) + (kv->d.head_dim == 128 ? partial_bytes<128>() : partial_bytes<64>());
}

extern "C" wb_status wb_kv_attend(const wb_kv* kv, const wb_kv_batch* batch, const wb_heads* q, uint32_t n_heads,
                                  const wb_heads* out, float* lse, float scale, uint32_t window, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  if (wb_status s = check_batch(kv, batch)) return s;
  if (wb_status s = check_heads(q, batch->n_tokens, false)) return s;
  if (wb_status s = check_heads(out, batch->n_tokens, false)) return s;
  if (!n_heads || n_heads % kv->d.n_kv_heads || n_heads / kv->d.n_kv_heads > 64) return WB_ERR_INVALID_ARG;
  if (!(scale > 0.f) || !std::isfinite(scale) || window > 0x7FFFFFFFu) return WB_ERR_INVALID_ARG;
  if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < wb_kv_attend_workspace_bytes(kv, n_heads, batch->n_seqs))
    return WB_ERR_INVALID_ARG;
  if (!batch->n_tokens || !batch->n_seqs) return WB_OK;
  AttendArgs a;
  a.c = kv_view(kv);
  a.b = kv_batch(batch);
  a.q = (const char*)q->data;
  a.out = (char*)out->data;
  a.q_token = q->token_stride * 2; a.q_head = q->head_stride * 2;
  a.o_token = out->token_stride * 2; a.o_head = out->head_stride * 2;
  a.lse = lse;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.n_heads = n_heads;
  a.group = n_heads / kv->d.n_kv_heads;
  a.window = window;
  a.box_rows = kv->box_rows;
  a.error = (uint32_t*)workspace;
  a.counters = (uint32_t*)((char*)workspace + kHeaderBytes);
  a.partials = (float*)((char*)workspace + kHeaderBytes + counter_bytes(kv, batch->n_seqs));
  const bool e = kv->d.dtype == WB_E4M3;
  const cudaStream_t st = (cudaStream_t)stream;
  const uint64_t rows = (uint64_t)batch->max_new * a.group;
  cudaError_t err = cudaSuccess;
  if (rows <= 16 * kMaxRowTiles || batch->n_seqs > 1) {
    const uint32_t r = (uint32_t)std::min<uint64_t>(rows, 16 * kMaxRowTiles);
    if (kv->d.head_dim == 128) err = e ? launch_rows_of<128, true>(r, a, kv, st) : launch_rows_of<128, false>(r, a, kv, st);
    else err = e ? launch_rows_of<64, true>(r, a, kv, st) : launch_rows_of<64, false>(r, a, kv, st);
  }
  if (err == cudaSuccess && rows > 16 * kMaxRowTiles) {
    const uint32_t skip = batch->n_seqs > 1 ? 16 * kMaxRowTiles : 0;
    const uint32_t grid = (uint32_t)(((uint64_t)batch->n_tokens * n_heads + 3) / 4);
    if (kv->d.head_dim == 128) e ? wb_attend_plain_kernel<128, true><<<grid, 128, 0, st>>>(a, skip) : wb_attend_plain_kernel<128, false><<<grid, 128, 0, st>>>(a, skip);
    else e ? wb_attend_plain_kernel<64, true><<<grid, 128, 0, st>>>(a, skip) : wb_attend_plain_kernel<64, false><<<grid, 128, 0, st>>>(a, skip);
    err = cudaPeekAtLastError();
  }
  if (err != cudaSuccess) (void)cudaGetLastError();
  return err == cudaSuccess ? WB_OK : WB_ERR_CUDA;
}
