// Attention of a chunk of new tokens over the paged cache.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "wb_kv.cuh"

using namespace wbi;

namespace {

struct AttendArgs {
  KvView c;
  KvBatch b;
  const char* q;
  char* out;
  uint64_t q_token, q_head, o_token, o_head;   // bytes
  float* lse;
  float scale;
  uint32_t n_heads, group, window;
};

// One warp per (token, head): lanes own D / 32 elements, keys one after the other, the softmax's maximum
// and sum carried along.
template <int D, bool Q>
__global__ void __launch_bounds__(128) wb_attend_rows_kernel(AttendArgs a) {
  constexpr int N = D / 32;
  const uint32_t lane = threadIdx.x & 31;
  const uint64_t id = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (id >= (uint64_t)a.b.n_tokens * a.n_heads) return;
  const int32_t row = (int32_t)(id / a.n_heads);
  const uint32_t h = (uint32_t)(id - (uint64_t)row * a.n_heads), g = h / a.group;
  const uint32_t s = kv_seq_of_row(a.b, row);
  const KvSeq q = kv_seq(a.b, s);
  if (row - q.row0 >= q.n_new) return;
  const int32_t pos = q.len - q.n_new + row - q.row0;
  const int32_t first = a.window && pos >= (int32_t)a.window ? pos - (int32_t)a.window + 1 : 0;
  float x[N], acc[N], top = -INFINITY, sum = 0.f;
  for (int e = 0; e < N; ++e) {
    x[e] = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(a.q + row * a.q_token + h * a.q_head)[lane * N + e] << 16) * a.scale;
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

}  // namespace

extern "C" size_t wb_kv_attend_workspace_bytes(const wb_kv* kv, uint32_t n_heads, uint32_t n_seqs) {
  if (!kv || !n_heads || n_seqs > WB_KV_MAX_SEQS) return 0;
  return 256;
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
  a.scale = scale;
  a.n_heads = n_heads;
  a.group = n_heads / kv->d.n_kv_heads;
  a.window = window;
  const uint32_t grid = (uint32_t)(((uint64_t)batch->n_tokens * n_heads + 3) / 4);
  const bool e = kv->d.dtype == WB_E4M3;
  const cudaStream_t st = (cudaStream_t)stream;
  if (kv->d.head_dim == 128) e ? wb_attend_rows_kernel<128, true><<<grid, 128, 0, st>>>(a) : wb_attend_rows_kernel<128, false><<<grid, 128, 0, st>>>(a);
  else e ? wb_attend_rows_kernel<64, true><<<grid, 128, 0, st>>>(a) : wb_attend_rows_kernel<64, false><<<grid, 128, 0, st>>>(a);
  return cudaPeekAtLastError() == cudaSuccess ? WB_OK : (cudaGetLastError(), WB_ERR_CUDA);
}
