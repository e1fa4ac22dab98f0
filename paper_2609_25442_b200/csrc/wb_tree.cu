// Trees of drafted tokens over the paged cache: which rows of its tree a row sees and at which position it stands, and the
// accepted path's rows brought together in the cache.  Both are latency: masks of 37 trees 4 us, the paths of 8 sequences 4.2, of 256 from E4M3
// caches 8.3 (13 MB moved).
#include <algorithm>

#include "wb_kv.cuh"

using namespace wbi;

namespace {

constexpr uint32_t kMaskThreads = 128;
constexpr uint32_t kParents = 2048;        // of a tree, that are kept in shared memory

// A block per sequence, a thread per row, which walks to the root: its ancestors come in falling order, so a word of
// the mask is complete when the next one's turn comes.  A few microseconds of dependent steps, as many as the tree is deep.
__global__ void __launch_bounds__(kMaskThreads) wb_kv_tree_kernel(KvBatch b, const int32_t* parent, uint32_t* mask, uint32_t words, int32_t* positions) {
  __shared__ int32_t known[kParents];
  const KvSeq q = kv_seq(b, blockIdx.x);
  const int32_t* up = parent + q.row0;
  for (int32_t i = (int32_t)threadIdx.x; i < min(q.n_new, (int32_t)kParents); i += kMaskThreads) known[i] = __ldg(up + i);
  __syncthreads();
  for (int32_t i = (int32_t)threadIdx.x; i < q.n_new; i += kMaskThreads) {
    uint32_t* row = mask + (uint64_t)(q.row0 + i) * words;
    int32_t at = i, depth = 0;
    uint32_t w = words;                     // words from here on are written
    while (w > (uint32_t)at / 32 + 1) row[--w] = 0;
    uint32_t bits = 0;
    for (;;) {
      if ((uint32_t)at / 32 < w) bits |= 1u << (at & 31);      // (a row behind the words' reach is in none)
      const int32_t p = at < (int32_t)kParents ? known[at] : __ldg(up + at);
      const bool root = p < 0 || p >= at;
      const uint32_t next = root ? 0 : (uint32_t)p / 32 + 1;   // words that are still to come
      if (next < w) {
        if ((uint32_t)at / 32 < w) row[--w] = bits;
        while (w > next) row[--w] = 0;
        bits = 0;
      }
      if (root) break;
      at = p;
      ++depth;
    }
    if (positions) positions[q.row0 + i] = q.len - q.n_new + depth;
  }
}

constexpr uint32_t kKeepThreads = 256;
constexpr uint32_t kKeepRows = 8;          // rows that a thread has in flight

// A thread owns 16 bytes of every row of one head (of keys or of values): it reads them of up to eight rows of the path, then writes
// them to the rows' new places.  Places rise with the path and lie at or before the rows that go there, so a place is written after
// the row that stood there has been read, and no thread touches another's bytes.
template <int LANES, bool Q>
__global__ void __launch_bounds__(kKeepThreads) wb_kv_keep_kernel(KvView c, KvBatch b, const int32_t* path, const int32_t* accepted, uint32_t depth) {
  __shared__ int2 from[32], to[32];
  __shared__ int32_t s_n;
  const uint32_t s = blockIdx.x, group = (blockIdx.y * kKeepThreads + threadIdx.x) / LANES, lane = threadIdx.x % LANES;
  const uint32_t hk = c.n_kv_heads;
  const bool is_v = group >= hk, in = group < 2 * hk;
  const uint32_t h = group - (is_v ? hk : 0);
  const KvSeq q = kv_seq(b, s);
  const int32_t first = q.len - q.n_new, most = min(min(max(__ldg(accepted + s), 0), (int32_t)depth), q.n_new - 1);
  path += (uint64_t)s * depth;
  constexpr uint32_t kRow = LANES * 16;
  char* const rows = (is_v ? c.v : c.k) + (uint64_t)h * c.head_stride * (Q ? 1 : 2) + lane * 16;
  float* const scales = is_v ? c.v_scale : c.k_scale;
  for (int32_t j0 = 0; j0 < most; j0 += 32) {
    if (threadIdx.x < 32) {
      const int32_t j = j0 + (int32_t)threadIdx.x;
      const int32_t at = j < most ? __ldg(path + j) : -1, before = j < most && j > 0 ? __ldg(path + j - 1) : 0;
      // a path rises; it ends where it does not
      const uint32_t bad = ~__ballot_sync(0xFFFFFFFFu, j < most && at > before && at < q.n_new);
      const int32_t n = bad ? __ffs(bad) - 1 : 32;
      int2 x = make_int2(-1, 0), y = make_int2(-1, 0);
      if ((int32_t)threadIdx.x < n && at != j + 1) {
        const int32_t src = first + at, dst = first + 1 + j;
        x = make_int2(kv_page(b, c.n_pages, c.page_size, s, src), src % (int32_t)c.page_size);
        y = make_int2(kv_page(b, c.n_pages, c.page_size, s, dst), dst % (int32_t)c.page_size);
        if (y.x < 0) x.x = -1;
      }
      from[threadIdx.x] = x;
      to[threadIdx.x] = y;
      if (threadIdx.x == 0) s_n = n;
    }
    __syncthreads();
    const int32_t n = s_n;
    if (in)
      for (int32_t k0 = 0; k0 < n; k0 += kKeepRows) {
        uint4 x[kKeepRows];
        float f[kKeepRows];
#pragma unroll
        for (int32_t k = 0; k < (int32_t)kKeepRows; ++k) {
          const int2 at = from[min(k0 + k, 31)];
          if (k0 + k < n && at.x >= 0) {
            x[k] = *reinterpret_cast<const uint4*>(rows + (uint64_t)(uint32_t)at.x * c.page_stride * (Q ? 1 : 2) + (uint32_t)at.y * kRow);
            if (Q && lane == 0) f[k] = scales[((uint64_t)(uint32_t)at.x * hk + h) * c.page_size + (uint32_t)at.y];
          }
        }
#pragma unroll
        for (int32_t k = 0; k < (int32_t)kKeepRows; ++k) {
          if (k0 + k < n && from[min(k0 + k, 31)].x >= 0) {
            const int2 at = to[min(k0 + k, 31)];
            *reinterpret_cast<uint4*>(rows + (uint64_t)(uint32_t)at.x * c.page_stride * (Q ? 1 : 2) + (uint32_t)at.y * kRow) = x[k];
            if (Q && lane == 0) scales[((uint64_t)(uint32_t)at.x * hk + h) * c.page_size + (uint32_t)at.y] = f[k];
          }
        }
      }
    if (n < 32) return;
    __syncthreads();
  }
}

template <int LANES, bool Q>
void launch_keep(const KvView& c, const KvBatch& b, const int32_t* path, const int32_t* accepted, uint32_t depth, cudaStream_t stream) {
  const dim3 grid(b.n_seqs, (2 * c.n_kv_heads * LANES + kKeepThreads - 1) / kKeepThreads);
  wb_kv_keep_kernel<LANES, Q><<<grid, kKeepThreads, 0, stream>>>(c, b, path, accepted, depth);
}

}  // namespace

extern "C" wb_status wb_kv_tree_masks(const wb_kv_batch* batch, const int32_t* parent, uint32_t* mask, uint32_t words, int32_t* positions,
                                      void* stream) {
  if (wb_status s = check_batch_arrays(batch)) return s;
  if ((((uintptr_t)parent | (uintptr_t)mask | (uintptr_t)positions) & 3u) || (uint64_t)words * 32 < batch->max_new || words > 0x7FFFFFu)
    return WB_ERR_INVALID_ARG;
  if (!batch->n_tokens || !batch->n_seqs) return WB_OK;
  if (!parent || !mask || !words) return WB_ERR_INVALID_ARG;
  wb_kv_tree_kernel<<<batch->n_seqs, kMaskThreads, 0, (cudaStream_t)stream>>>(kv_batch(batch), parent, mask, words, positions);
  return cudaPeekAtLastError() == cudaSuccess ? WB_OK : (cudaGetLastError(), WB_ERR_CUDA);
}

extern "C" wb_status wb_kv_keep(const wb_kv* kv, const wb_kv_batch* batch, const int32_t* path, const int32_t* accepted, uint32_t depth,
                                void* stream) {
  if (wb_status s = check_batch(kv, batch)) return s;
  if ((((uintptr_t)path | (uintptr_t)accepted) & 3u) || depth > 0x7FFFFFu) return WB_ERR_INVALID_ARG;
  if (!batch->n_seqs || !depth) return WB_OK;
  if (!path || !accepted) return WB_ERR_INVALID_ARG;
  const KvView c = kv_view(kv);
  const KvBatch b = kv_batch(batch);
  const bool q = kv->d.dtype == WB_E4M3;
  const cudaStream_t st = (cudaStream_t)stream;
  if (c.head_dim == 128) q ? launch_keep<8, true>(c, b, path, accepted, depth, st) : launch_keep<16, false>(c, b, path, accepted, depth, st);
  else q ? launch_keep<4, true>(c, b, path, accepted, depth, st) : launch_keep<8, false>(c, b, path, accepted, depth, st);
  return cudaPeekAtLastError() == cudaSuccess ? WB_OK : (cudaGetLastError(), WB_ERR_CUDA);
}
