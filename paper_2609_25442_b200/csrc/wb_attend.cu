// Attention of a chunk of new tokens over the paged cache: which kernel takes a sequence, and the launches.
//
// Two kernels share a batch by the sequences' rows (new tokens x query heads per kv head).  Up to 32 rows the cache's bytes are the
// bound, and a kernel that streams them through the legacy matrix instructions is the faster; beyond, the products are, and they
// need tensor memory, in a kernel that fills tiles of 128 rows whatever there are.  24 sequences of 300 to 5000 positions with 8 to 32
// rows: 73 us (E4M3) and 75 us (bf16) with the border at 32, 103 and 91 with it at 16, 129 and 95 at 8.  Both are launched where a
// batch may hold both kinds; each leaves the other's alone.  The row kernel comes with 8, 16 and 32 rows, chosen for the whole batch by
// max_new: 64 sequences that decode one token with 4 rows each take 194 us with 8, 234 with 32, and 257 where max_new says that there
// may be long chunks too; 96 over E4M3, 8 rows each, 85, 159 and 159 (caches cold).
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>

#include "wb_attend.cuh"
#include "wb_attend_rows.cuh"
#include "wb_attend_tiles.cuh"

using namespace wbi;

namespace {

constexpr uint32_t kHeaderBytes = 256;
constexpr uint32_t kMaxRows = 32;                       // of wb_attend_rows_kernel
constexpr uint32_t kMaxRowBlocks = 3 * kNumSMs;

// A kernel's dynamic shared memory is raised once per device to the most that it may ask for; with `regs`, the kernel has to have been
// compiled to that many registers and no static shared memory.  Returns an error only where it cannot run at all.
template <typename K> cudaError_t prepare_kernel(K kernel, uint32_t most, int regs, int dev, std::atomic<uint64_t>& done) {
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  cudaFuncAttributes f;
  cudaError_t e;
  if ((e = cudaFuncGetAttributes(&f, kernel)) != cudaSuccess) return e;
  if (regs && (f.numRegs != regs || f.sharedSizeBytes != 0)) return cudaErrorInvalidConfiguration;
  most = std::min<uint32_t>(most, 232448 - (uint32_t)f.sharedSizeBytes);
  if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most)) != cudaSuccess) return e;
  done.fetch_or(bit, std::memory_order_release);
  return cudaSuccess;
}

// A joining kernel is set up while the kernel before it still runs, and waits for that one's end itself.
cudaError_t launch_join(void (*kernel)(AttendArgs), dim3 grid, uint32_t threads, const AttendArgs& a, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <int D, bool Q, int NT>
cudaError_t launch_rows(const AttendArgs& a, int dev, cudaStream_t stream) {
  using C = RowsCfg<D, Q, NT>;
  const size_t smem = C::smem_bytes(a.b.n_seqs);
  auto kernel = wb_attend_rows_kernel<D, Q, NT>;
  // every block gets the same share of the tiles, so the grid is what fits at once (with thousands of sequences the table of
  // prefix sums takes the place of a block)
  const uint32_t per_sm = std::min<uint32_t>(C::kBlocksPerSm, (uint32_t)(kSmemPerSm / (smem + 2048)));
  static std::atomic<uint64_t> done{0};
  cudaError_t e = prepare_kernel(kernel, 232448, 0, dev, done);
  if (e != cudaSuccess) return e;
  const uint32_t grid = kNumSMs * std::max(1u, per_sm);
  kernel<<<grid, C::kThreads, smem, stream>>>(a);
  if ((e = cudaPeekAtLastError()) != cudaSuccess) return e;
  return launch_join(wb_attend_join_rows_kernel<D, NT>, dim3(grid, 2 * NT), 256, a, stream);
}

template <int D, bool Q>
cudaError_t launch_rows_of(uint32_t rows, const AttendArgs& a, int dev, cudaStream_t stream) {
  if (rows <= 8) return launch_rows<D, Q, 1>(a, dev, stream);
  if (rows <= 16) return launch_rows<D, Q, 2>(a, dev, stream);
  return launch_rows<D, Q, 4>(a, dev, stream);
}

template <int D, bool Q>
cudaError_t launch_tiles(const AttendArgs& all, const wb_kv* kv, uint32_t skip_rows, cudaStream_t stream) {
  using C = TilesCfg<D, Q>;
  auto kernel = wb_attend_tiles_kernel<D, Q>;
  // the softmax warps wait for registers that the others give back: the launch has to have them
  static std::atomic<uint64_t> done{0};
  cudaError_t e = prepare_kernel(kernel, C::kSmemBytes, C::kLaunchRegs, kv->device, done);
  if (e != cudaSuccess) return e;
  for (uint32_t s0 = 0; s0 < all.b.n_seqs; s0 += C::kMaxSeqs) {
    AttendArgs a = all;
    a.b.n_seqs = std::min(C::kMaxSeqs, all.b.n_seqs - s0);
    a.b.table += (uint64_t)s0 * a.b.table_pitch;
    a.b.new_start += s0;
    a.b.kv_len += s0;
    kernel<<<kNumSMs, C::kThreads, C::kSmemBytes, stream>>>(a, kv->map_k, kv->map_v, skip_rows);
    if ((e = cudaPeekAtLastError()) != cudaSuccess) return e;
    if ((e = launch_join(wb_attend_join_kernel<D>, dim3(kNumSMs, kQRows / 32), 256, a, stream)) != cudaSuccess) return e;
  }
  return cudaSuccess;
}


constexpr uint32_t kCutBytes = (kMaxRowBlocks * sizeof(CutItem) + 255) / 256 * 256;
template <int D> constexpr size_t partial_bytes() {
  return (size_t)2 * 4 * std::max({kMaxRowBlocks * RowsCfg<D, true, 2>::kPartFloats, 2 * kNumSMs * RowsCfg<D, true, 4>::kPartFloats,
                                   kNumSMs * TilesCfg<D, false>::kPartFloats});
}

}  // namespace

extern "C" size_t wb_kv_attend_workspace_bytes(const wb_kv* kv, uint32_t n_heads, uint32_t n_seqs) {
  if (!kv || !n_heads || n_seqs > WB_KV_MAX_SEQS) return 0;
  return kHeaderBytes + kCutBytes + (kv->d.head_dim == 128 ? partial_bytes<128>() : partial_bytes<64>());
}

extern "C" wb_status wb_kv_attend(const wb_kv* kv, const wb_kv_batch* batch, const wb_heads* q, uint32_t n_heads,
                                  const wb_heads* out, float* lse, float scale, uint32_t window, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  if (wb_status s = check_batch(kv, batch)) return s;
  if (wb_status s = check_heads(q, batch->n_tokens, false)) return s;
  if (wb_status s = check_heads(out, batch->n_tokens, false)) return s;
  if (!n_heads || n_heads % kv->d.n_kv_heads || n_heads / kv->d.n_kv_heads > 64) return WB_ERR_INVALID_ARG;
  if (!(scale > 0.f) || !std::isfinite(scale) || window > 0x7FFFFFFFu) return WB_ERR_INVALID_ARG;
  if ((uintptr_t)lse & 3u) return WB_ERR_INVALID_ARG;
  if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < wb_kv_attend_workspace_bytes(kv, n_heads, batch->n_seqs))
    return WB_ERR_INVALID_ARG;
  if (!batch->n_tokens || !batch->n_seqs) return WB_OK;
  // positions from -n_tokens to max_len, and what windows and tiles add to them, are counted in 31 bits, and so are tiles
  if ((uint64_t)batch->max_len + batch->n_tokens > 0x7FFFFF00ull) return WB_ERR_INVALID_ARG;
  const uint64_t group = n_heads / kv->d.n_kv_heads, row_blocks = (uint64_t)batch->n_tokens * group / kQRows + batch->n_seqs;
  if (row_blocks * (batch->max_len / kKvTile + 2) * kv->d.n_kv_heads > 0x7FFFFFFFull) return WB_ERR_INVALID_ARG;
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
  a.window = window < batch->max_len ? window : 0;      // (the kernels' first positions are differences with it)
  a.box_rows = kv->box_rows;
  a.error = (uint32_t*)workspace;
  a.cuts = (char*)workspace + kHeaderBytes;
  a.partials = (float*)((char*)workspace + kHeaderBytes + kCutBytes);
  const bool e = kv->d.dtype == WB_E4M3;
  const cudaStream_t st = (cudaStream_t)stream;
  const uint64_t rows = (uint64_t)batch->max_new * a.group;
  cudaError_t err = cudaSuccess;
  if (rows <= kMaxRows || batch->n_seqs > 1) {
    const uint32_t r = (uint32_t)std::min<uint64_t>(rows, kMaxRows);
    if (kv->d.head_dim == 128) err = e ? launch_rows_of<128, true>(r, a, kv->device, st) : launch_rows_of<128, false>(r, a, kv->device, st);
    else err = e ? launch_rows_of<64, true>(r, a, kv->device, st) : launch_rows_of<64, false>(r, a, kv->device, st);
  }
  if (err == cudaSuccess && rows > kMaxRows) {
    const uint32_t skip = batch->n_seqs > 1 ? kMaxRows : 0;
    if (kv->d.head_dim == 128) err = e ? launch_tiles<128, true>(a, kv, skip, st) : launch_tiles<128, false>(a, kv, skip, st);
    else err = e ? launch_tiles<64, true>(a, kv, skip, st) : launch_tiles<64, false>(a, kv, skip, st);
  }
  if (err != cudaSuccess) (void)cudaGetLastError();
  return err == cudaSuccess ? WB_OK : WB_ERR_CUDA;
}

extern "C" wb_status wb_kv_attend_check(void* workspace, void* stream) {
  if (!workspace || ((uintptr_t)workspace & 255u)) return WB_ERR_INVALID_ARG;
  uint32_t error = 0;
  const cudaStream_t st = (cudaStream_t)stream;
  if (cudaMemcpyAsync(&error, workspace, 4, cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess ||
      (error && cudaMemsetAsync(workspace, 0, 4, st) != cudaSuccess)) {
    (void)cudaGetLastError();
    return WB_ERR_CUDA;
  }
  return error & (kGaveUp | kMisplaced) ? WB_ERR_CUDA : error & kTooLong ? WB_ERR_INVALID_ARG : WB_OK;
}
