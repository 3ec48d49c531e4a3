// amoeba_copy_blocks: blocks of the cache copied to other blocks of the same pools.
//
// A work item is a piece of one block's contiguous bytes in one layer of one worker's pool (header-centric blocks are one run,
// token-first ones a run of keys and one of values), moved by the bulk-copy rings of copy_engine.cuh; layer slowest, so that CTAs that
// run together touch neighbouring memory.  Bound by the bytes, read once and written once: 64 blocks of 64 KiB in 32 layers, four workers,
// 46.8 us (5.7 TB/s; a large transformation's copies reach 6.7, the start and end of these take about 5 us).
#include "cache_view.cuh"

namespace amoeba {

struct BlockCopyParams {
    CacheView cache;            // of layer_begin
    int64_t layer_stride, run;  // bytes of a contiguous run
    const int2* pairs;
    const int32_t* num_pairs;
    int32_t* status;
    int32_t pairs_cap, n_layers, workers, runs;  // runs: of a block in a layer of a pool
#ifdef AMOEBA_CHECK_ITEMS
    int64_t span;               // bytes from the first layer's begin to the last one's end
#endif
};

constexpr int kCopyPiece = 8192, kCopyLeast = 2048;  // bytes of an item

struct BlockCopyItems {
    const BlockCopyParams& p;
    int32_t n_pairs, piece, pieces;
    __device__ __forceinline__ int64_t units() const { return (int64_t)n_pairs * p.n_layers * p.workers * p.runs; }
    __device__ __forceinline__ BlockCopyItems(const BlockCopyParams& p_, int rings) : p(p_), piece(kCopyPiece) {
        n_pairs = min(max(__ldcg(p.num_pairs), 0), p.pairs_cap);
        // few blocks: smaller pieces, as long as there are rings without one
        auto count = [&] { return pieces = (int32_t)((p.run + piece - 1) / piece); };
        while (units() * count() < rings && piece > kCopyLeast) piece /= 2;
    }
    __device__ __forceinline__ int64_t count() const { return units() * pieces; }
    __device__ __forceinline__ Item operator()(int64_t w) const {
        const int64_t unit = w / pieces;
        const int64_t off = (w - unit * pieces) * piece;
        const int32_t per_pair = p.workers * p.runs;
        const int64_t lp = unit / per_pair;
        const int32_t wr = (int32_t)(unit - lp * per_pair), worker = wr / p.runs, run = wr - worker * p.runs;
        const int64_t layer = lp / n_pairs;
        const int2 ids = __ldcg(p.pairs + (lp - layer * n_pairs));  // (written while this kernel was waiting)
        Item it;
        it.src_map = it.dst_map = nullptr;
        it.src = it.dst = nullptr;
        it.src_pitch = it.dst_pitch = 0;
        it.n_rows = 0;
        it.row_bytes = (int32_t)min((int64_t)piece, p.run - off);
        if (ids.x < 0 || ids.y < 0 || ids.x == ids.y) return it;
        if (ids.x >= p.cache.num_blocks || ids.y >= p.cache.num_blocks) {
            report(p.status, AMOEBA_ERR_BAD_BLOCK_ID);
            return it;
        }
        const int64_t at = layer * p.layer_stride + run * p.cache.kv_stride + off;
        const int64_t from = at + ids.x * p.cache.block_stride, to = at + ids.y * p.cache.block_stride;
#ifdef AMOEBA_CHECK_ITEMS
        if (!rows_inside(from, 0, 1, it.row_bytes, p.span) || !rows_inside(to, 0, 1, it.row_bytes, p.span)) {
            report(p.status, AMOEBA_ERR_INTERNAL);
            return it;
        }
#endif
        it.n_rows = 1;
        it.src = p.cache.pools[worker] + from;
        it.dst = p.cache.pools[worker] + to;
        return it;
    }
};

__global__ void __launch_bounds__(1024) copy_blocks(const __grid_constant__ BlockCopyParams p, const RingShape rs) {
    extern __shared__ __align__(128) char smem[];
    const PairRing r = pair_ring_setup(smem, rs);
    grid_dependency_launch();
    grid_dependency_wait();  // the pairs and blocks are there
    const BlockCopyItems items(p, (int)gridDim.x * r.nrings);
    const bool ok = pair_bulk_ring(r.role, items, items.count(), (int64_t)r.ring * gridDim.x + blockIdx.x,
                                   (int64_t)gridDim.x * r.nrings, r.stages, r.full, r.empty, r.abort, rs);
    if (!ok && threadIdx.x % 32 == 0) report(p.status, AMOEBA_ERR_TIMEOUT);
}

}  // namespace amoeba

using namespace amoeba;

extern "C" amoeba_status amoeba_copy_blocks(const amoeba_layout* layout, void* const* pools, const int32_t* d_pairs,
                                            const int32_t* d_num_pairs, int32_t pairs_cap, int32_t layer_begin, int32_t layer_end,
                                            int32_t* d_status, void* cuda_stream) {
    if (!layout || !pools || !d_status || pairs_cap < 0 || layer_begin < 0 || layer_end < layer_begin) return AMOEBA_ERR_INVALID_ARG;
    if (pairs_cap && (!d_pairs || !d_num_pairs)) return AMOEBA_ERR_INVALID_ARG;
    if ((uintptr_t)d_pairs % 8) return AMOEBA_ERR_ALIGNMENT;
    BlockCopyParams p{};
    int64_t bytes = 0;
    amoeba_status st = amoeba_layout_kv_pool_bytes(layout, &bytes);
    if (st != AMOEBA_OK) return st;
    if (layer_end > layout->model.num_layers) return AMOEBA_ERR_INVALID_ARG;
    if (layer_begin == layer_end || pairs_cap == 0) return AMOEBA_OK;
    if ((st = make_cache_view(layout, layer_begin, pools, &p.cache)) != AMOEBA_OK) return st;
    const bool head_major = layout->kv_order == AMOEBA_KV_HEAD_MAJOR;
    p.layer_stride = bytes / layout->model.num_layers;
    p.run = p.cache.block_stride;  // (a token-first block's keys, or its values)
    p.runs = head_major ? 1 : 2;
    p.pairs = reinterpret_cast<const int2*>(d_pairs), p.num_pairs = d_num_pairs, p.status = d_status;
    p.pairs_cap = pairs_cap, p.n_layers = layer_end - layer_begin, p.workers = layout->tp;
#ifdef AMOEBA_CHECK_ITEMS
    p.span = p.n_layers * p.layer_stride;
#endif
    const DeviceInfo dev = cached_device_info();
    if (!dev.sms) return AMOEBA_ERR_CUDA;
    KernelOpts opt{};
#ifdef AMOEBA_CHECK_ITEMS
    opt.wait_tries = operator_wait_polls();
#endif
    const BulkShape bs = bulk_shape(dev, opt, kKvDefaults, 3, kCopyPiece);
    const int64_t most = (int64_t)pairs_cap * p.n_layers * p.workers * p.runs * ((p.run + kCopyLeast - 1) / kCopyLeast);
    const int grid = (int)std::min<int64_t>(most, dev.sms);
    if (ensure_dynamic_smem((const void*)copy_blocks, (int)bs.smem) != cudaSuccess) return AMOEBA_ERR_CUDA;
    return launch_kernel(copy_blocks, grid, bs.threads, bs.smem, static_cast<cudaStream_t>(cuda_stream), true, p, bs.ring);
}
