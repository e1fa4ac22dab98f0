// Attention of a chunk of new tokens over the paged cache: which kernel takes a sequence, and the launches.
//
// Two kernels share a batch of chunks by the sequences' rows (new tokens x query heads per kv head).  Up to 32 rows the cache's bytes are the
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
#include "wb_cluster.cuh"

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

template <int D, bool Q, int NT, bool TREE>
cudaError_t launch_rows(const AttendArgs& a, int dev, cudaStream_t stream) {
  using C = RowsCfg<D, Q, NT>;
  const size_t smem = C::smem_bytes(a.b.n_seqs);
  auto kernel = wb_attend_rows_kernel<D, Q, NT, TREE ? RowsMode::kTree : RowsMode::kChunk>;
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

template <int D, bool Q, bool TREE>
cudaError_t launch_rows_of(uint32_t rows, const AttendArgs& a, int dev, cudaStream_t stream) {
  if (rows <= 8) return launch_rows<D, Q, 1, TREE>(a, dev, stream);
  if (rows <= 16) return launch_rows<D, Q, 2, TREE>(a, dev, stream);
  if constexpr (!TREE || Q) return launch_rows<D, Q, 4, TREE>(a, dev, stream);
  return cudaErrorInvalidValue;        // (bf16 trees of more rows go to the other kernel)
}

template <int D, bool Q, Rows256 MODE>
cudaError_t launch_tiles(const AttendArgs& all, const wb_kv* kv, uint32_t skip_rows, cudaStream_t stream) {
  using C = TilesCfg<D, Q>;
  auto kernel = wb_attend_tiles_kernel<D, Q, MODE>;
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
    if ((e = launch_join(wb_attend_join_kernel<D>, dim3(kNumSMs, (MODE == Rows256::kTreeShared ? kQRows / 2 : kQRows) / 32), 256, a, stream)) != cudaSuccess) return e;
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

namespace {

// The checks and parameters that both forms share; `todo` is false if there is nothing to do.
wb_status attend_args(const wb_kv* kv, const wb_kv_batch* batch, const wb_heads* q, uint32_t n_heads, const wb_heads* out, float* lse,
                      float scale, uint32_t window, void* workspace, size_t workspace_bytes, AttendArgs& a, bool& todo) {
  todo = false;
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
  a.mask = nullptr;
  a.words = a.row_blocks = 0;
  todo = true;
  return WB_OK;
}

// Trees by clusters, a cluster for every 8 NT rows of a (sequence, kv head), if all of them fit at once and a block's share is
// small: `taken` tells.  `whole`: only with as many blocks in a cluster as there may be.
//
// What the kernels along the line cost more is a second launch and its reads, 4 to 10 us; what clusters cost more are uneven
// shares and, beyond 32 rows, cache tiles read once per 32 of them.  Both sides, bf16, heads of 128, cluster | line, us: one sequence, 8 kv
// heads, 4 rows 1000 positions 8.2 | 9.5, 8000 14.0 | 16.1, 16 thousand 21.1 | 19.0, 30 thousand 33.4 | 31.4; 32 rows 13.3 | 18.5, 23.1 |
// 34.1, 35.3 | 42.8, 56.0 | 53.0; 128 rows 15.4 | 19.2, 35.1 | 35.9, 59.5 | 42.9; with 4 kv heads, which leaves clusters of 16, 26.0 | 46.1
// and 41.2 | 47.7 of the latter two.  64 items of 32 rows, 256 and 2000 positions: 14.2 | 13.2 and 25.6 | 23.8.
// Hence the bounds on items beyond 32 rows.  128 rows, bf16 and E4M3, heads of 128, 300 positions: 40 items 13.6 | 14.9 and 12.1 | 15.9, 48 13.8 | 14.8 and
// 15.5 | 15.8, 96 17.0 | 14.9 and 18.6 | 15.9; a window of 1000: 40 18.5 | 20.8 and 21.1 | 21.6, 48 19.8 | 20.9 and 22.5 | 21.6, 64 21.4 | 20.0 and
// 24.0 | 22.1, 72 23.4 | 20.2 and 26.4 | 22.4.  Beyond 128 rows, where the other kernel's tiles are not shared out, 256 rows: 300 positions 48 items 13.9 | 19.4
// and 16.0 | 20.8, 64 15.8 | 19.6 and 17.3 | 21.0, 96 19.1 | 19.7 and 20.8 | 21.2; 1000 positions 64 20.8 | 22.9 and 22.6 | 25.8, 72 21.5 | 23.2 and 23.5 | 25.9,
// 96 28.3 | 23.2 and 30.3 | 26.0; the window 64 22.2 | 25.6 and 25.4 | 27.1, 72 23.5 | 25.7 and 26.9 | 27.2.
constexpr uint32_t kClusterTiles = 16, kClusterTilesWide = 8, kClusterItems = 48, kClusterItemsWide = 64;
template <int D, bool Q, int NT>
cudaError_t launch_clusters(AttendArgs a, uint64_t rows, uint32_t max_tiles, bool whole, int dev, cudaStream_t stream, bool& taken) {
  using C = RowsCfg<D, Q, NT>;
  const size_t smem = C::smem_bytes(0);
  auto kernel = wb_attend_rows_kernel<D, Q, NT, RowsMode::kTreeCluster>;
  static std::atomic<uint64_t> done{0};
  static ClusterCounts known;
  a.row_blocks = (uint32_t)((rows + C::kRows - 1) / C::kRows);
  const uint64_t items = (uint64_t)a.b.n_seqs * a.c.n_kv_heads * a.row_blocks;
  if (items > (rows > kQRows / 2 ? kClusterItemsWide : rows > kMaxRows ? kClusterItems : C::kBlocksPerSm * kNumSMs)) return cudaSuccess;
  if (cudaError_t e = prepare_kernel(kernel, 232448, 0, dev, done)) return e;
  const uint32_t most = std::min(16u, max_tiles);
  for (uint32_t size = most; size * (rows <= kMaxRows || size == 16 ? kClusterTiles : kClusterTilesWide) >= max_tiles && (!whole || size == most); --size) {
    if (items > resident_clusters(kernel, C::kThreads, dev, size, known, smem)) continue;
    cudaLaunchAttribute at[1];
    const cudaLaunchConfig_t cfg = config_of((uint32_t)items, C::kThreads, size, at, stream, smem);
    taken = true;
    return cudaLaunchKernelEx(&cfg, kernel, a);
  }
  return cudaSuccess;
}
// Few rows to a block make its work shorter, as long as every cluster still has all the blocks that it can use.
template <int D, bool Q>
cudaError_t launch_clusters_of(const AttendArgs& a, uint64_t rows, uint32_t max_tiles, int dev, cudaStream_t stream, bool& taken) {
  taken = false;
  if (max_tiles > 16 * kClusterTiles) return cudaSuccess;
  cudaError_t e = launch_clusters<D, Q, 1>(a, rows, max_tiles, rows > 8, dev, stream, taken);
  if (!taken && e == cudaSuccess && rows > 8) e = launch_clusters<D, Q, 2>(a, rows, max_tiles, rows > 16, dev, stream, taken);
  if (!taken && e == cudaSuccess && rows > 16) e = launch_clusters<D, Q, 4>(a, rows, max_tiles, false, dev, stream, taken);
  return e;
}

template <Rows256 MODE> cudaError_t launch_tiles_of(const AttendArgs& a, const wb_kv* kv, uint32_t skip_rows, cudaStream_t stream) {
  const bool q = kv->d.dtype == WB_E4M3;
  if (kv->d.head_dim == 128) return q ? launch_tiles<128, true, MODE>(a, kv, skip_rows, stream) : launch_tiles<128, false, MODE>(a, kv, skip_rows, stream);
  return q ? launch_tiles<64, true, MODE>(a, kv, skip_rows, stream) : launch_tiles<64, false, MODE>(a, kv, skip_rows, stream);
}

template <bool TREE> wb_status launch_attend(const AttendArgs& a, const wb_kv* kv, const wb_kv_batch* batch, cudaStream_t st) {
  const bool e = kv->d.dtype == WB_E4M3;
  const uint64_t rows = (uint64_t)batch->max_new * a.group;
  cudaError_t err = cudaSuccess;
  if constexpr (TREE) {
    bool taken = false;
    // tiles that a row may see: up to max_len, or of a window and the tree (which may begin within a tile)
    const uint64_t reach = a.window ? std::min<uint64_t>(batch->max_len, (uint64_t)a.window + batch->max_new) : batch->max_len;
    const uint32_t tiles = (uint32_t)std::max<uint64_t>(1, (reach + kKvTile - 1) / kKvTile + (a.window ? 1 : 0));
    if (kv->d.head_dim == 128) err = e ? launch_clusters_of<128, true>(a, rows, tiles, kv->device, st, taken) : launch_clusters_of<128, false>(a, rows, tiles, kv->device, st, taken);
    else err = e ? launch_clusters_of<64, true>(a, rows, tiles, kv->device, st, taken) : launch_clusters_of<64, false>(a, rows, tiles, kv->device, st, taken);
    if (taken || err != cudaSuccess) {
      if (err != cudaSuccess) (void)cudaGetLastError();
      return err == cudaSuccess ? WB_OK : WB_ERR_CUDA;
    }
  }
  // (a batch of trees is of a kind: sequences with few rows go with the others instead of costing two launches of their own)
  const bool mixed = !TREE && batch->n_seqs > 1;
  // (trees of 17 to 32 rows over a bf16 cache: the second kernel shares their tiles out, 4 sequences of 8000 positions 39.7 us instead of 52.
  // Over codes it widens, which takes longer than the row kernel's products: 96 sequences of 1500 positions, 8 kv heads of 128, 20 rows 210 us
  // instead of 147, heads of 64 141 instead of 94; only of 300 positions 61 instead of 69, heads of 64 53 instead of 45)
  const bool few = rows <= (TREE && !e ? kMaxRows / 2 : kMaxRows);
  if (few || mixed) {
    const uint32_t r = (uint32_t)std::min<uint64_t>(rows, kMaxRows);
    if (kv->d.head_dim == 128) err = e ? launch_rows_of<128, true, TREE>(r, a, kv->device, st) : launch_rows_of<128, false, TREE>(r, a, kv->device, st);
    else err = e ? launch_rows_of<64, true, TREE>(r, a, kv->device, st) : launch_rows_of<64, false, TREE>(r, a, kv->device, st);
  }
  if (err == cudaSuccess && (!few || (mixed && rows > kMaxRows))) {
    const uint32_t skip = mixed ? kMaxRows : 0;
    constexpr Rows256 kMode = TREE ? Rows256::kTree : Rows256::kChunk;
    err = TREE && rows <= kQRows / 2 ? launch_tiles_of<Rows256::kTreeShared>(a, kv, skip, st) : launch_tiles_of<kMode>(a, kv, skip, st);
  }
  if (err != cudaSuccess) (void)cudaGetLastError();
  return err == cudaSuccess ? WB_OK : WB_ERR_CUDA;
}

}  // namespace

extern "C" wb_status wb_kv_attend(const wb_kv* kv, const wb_kv_batch* batch, const wb_heads* q, uint32_t n_heads,
                                  const wb_heads* out, float* lse, float scale, uint32_t window, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  AttendArgs a;
  bool todo;
  if (wb_status s = attend_args(kv, batch, q, n_heads, out, lse, scale, window, workspace, workspace_bytes, a, todo)) return s;
  if (!todo) return WB_OK;
  return launch_attend<false>(a, kv, batch, (cudaStream_t)stream);
}

extern "C" wb_status wb_kv_attend_tree(const wb_kv* kv, const wb_kv_batch* batch, const uint32_t* mask, uint32_t words, const wb_heads* q,
                                       uint32_t n_heads, const wb_heads* out, float* lse, float scale, uint32_t window, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  AttendArgs a;
  bool todo;
  if (wb_status s = attend_args(kv, batch, q, n_heads, out, lse, scale, window, workspace, workspace_bytes, a, todo)) return s;
  if (((uintptr_t)mask & 3u) || (uint64_t)words * 32 < batch->max_new || words > 0x7FFFFFu) return WB_ERR_INVALID_ARG;
  // a window that reaches back over a whole tree never ends inside one
  if (window && window < batch->max_new) return WB_ERR_INVALID_ARG;
  if (!todo || !batch->max_new) return WB_OK;      // (without new tokens there are rows that no sequence holds, and no trees)
  if (!mask || !words) return WB_ERR_INVALID_ARG;
  a.mask = mask;
  a.words = words;
  return launch_attend<true>(a, kv, batch, (cudaStream_t)stream);
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
