// amoeba_evict_kv: long sequences cut to a budget by their tokens' scores.
//
// Two launches: which tokens stay (one CTA per layer, sequence and key head: a radix selection of the budget-th largest
// score and an ordered list of the kept indices), and the move of their keys, values and scores.  Memory-bound: the
// scores are read once, what stays is read and written once.
#include "cache_view.cuh"

namespace amoeba {

struct EvictParams {
    CacheView cache;  // of layer_begin
    float* scores[AMOEBA_MAX_TP];
    int64_t layer_stride;   // bytes between layers of a pool
    int64_t layer_scores;   // floats between layers of a score pool
    const int32_t *src_bt, *seq_lens, *dst_bt;
    int32_t *new_lens, *status;
    int32_t* kept;          // [layers][num_seqs][kv_heads][budget]
    int32_t num_seqs, max_blocks, dst_max_blocks, budget, recent, kv_heads, layers, has_scores, in_place;
    int32_t vec;            // bytes of one token's key
};

// The sequence's length, or -1 if it is refused; the whole block asks together.
__device__ __forceinline__ int checked_len(const EvictParams& p, int s, bool reports) {
    const int len = p.seq_lens[s], T = p.cache.block_tokens;
    int code = 0;
    if (len < 0 || len > (int64_t)p.max_blocks * T) return reports && threadIdx.x == 0 ? (report(p.status, AMOEBA_ERR_INVALID_ARG), -1) : -1;
    const int keep = min(len, p.budget), n_src = (len + T - 1) / T, n_dst = (keep + T - 1) / T;
    if (n_dst > p.dst_max_blocks) return reports && threadIdx.x == 0 ? (report(p.status, AMOEBA_ERR_INVALID_ARG), -1) : -1;
    for (int i = threadIdx.x; i < n_src; i += blockDim.x) {
        const int b = p.src_bt[(int64_t)s * p.max_blocks + i];
        if (b < 0 || b >= p.cache.num_blocks) code = 1;
    }
    for (int i = threadIdx.x; i < n_dst; i += blockDim.x) {
        const int b = p.dst_bt[(int64_t)s * p.dst_max_blocks + i];
        if (b < 0 || b >= p.cache.num_blocks) code = 1;
    }
    if (!__syncthreads_or(code)) return len;
    if (reports && threadIdx.x == 0) report(p.status, AMOEBA_ERR_BAD_BLOCK_ID);
    return -1;
}

// Scores as whole numbers of the same order: a NaN is 0, below -infinity; -0 is 0.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0;
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kSelectThreads = 512;

__global__ void __launch_bounds__(kSelectThreads) evict_select(const __grid_constant__ EvictParams p) {
    __shared__ int32_t s_hist[256];
    __shared__ int64_t s_warp[kSelectThreads / 32];
    __shared__ uint32_t s_key;
    __shared__ int32_t s_need;
    const int tid = threadIdx.x;
    const int h = blockIdx.x % p.kv_heads, s = blockIdx.x / p.kv_heads % p.num_seqs;
    const int l = blockIdx.x / p.kv_heads / p.num_seqs;
    const bool first = l == 0 && h == 0;
    const int len = checked_len(p, s, first);
    if (first && tid == 0) p.new_lens[s] = min(len, p.budget);
    if (len <= p.budget) return;
    const int free = len - p.recent, need = p.budget - p.recent;
    const int w = h / p.cache.heads, hw = h - w * p.cache.heads, T = p.cache.block_tokens;
    int32_t* kept = p.kept + ((int64_t)(l * p.num_seqs + s) * p.kv_heads + h) * p.budget;
    for (int i = tid; i < p.recent; i += kSelectThreads) kept[need + i] = free + i;
    if (need == 0) return;
    const float* scores = p.scores[w] + l * p.layer_scores;
    const int32_t* table = p.src_bt + (int64_t)s * p.max_blocks;
    auto key_of = [&](int i) {
        return order_of(scores[((int64_t)table[i / T] * p.cache.heads + hw) * T + i % T]);
    };
    // The need-th largest key, eight bits at a time; s_need of the tokens that have exactly that key stay.
    uint32_t prefix = 0;
    int left = need;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kSelectThreads) s_hist[i] = 0;
        __syncthreads();
        const uint32_t above = shift == 24 ? 0 : ~0u << (shift + 8);
        for (int i = tid; i < free; i += kSelectThreads) {
            const uint32_t k = key_of(i);
            if ((k & above) == prefix) atomicAdd(&s_hist[k >> shift & 255], 1);
        }
        __syncthreads();
        if (tid < 32) {  // from the largest digit down
            int mine[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) mine[i] = s_hist[255 - tid * 8 - i], sum += mine[i];
            int before = sum;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int up = __shfl_up_sync(~0u, before, o);
                if (tid >= o) before += up;
            }
            before -= sum;
            if (before < left && left <= before + sum) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (before < left && left <= before + mine[i]) {
                        s_key = prefix | (uint32_t)(255 - tid * 8 - i) << shift;
                        s_need = left - before;
                    }
                    before += mine[i];
                }
            }
        }
        __syncthreads();
        prefix = s_key;
        left = s_need;
    }
    // In order: thread t lists the kept ones of its run of consecutive tokens.
    const int per = (free + kSelectThreads - 1) / kSelectThreads, begin = min(free, tid * per), end = min(free, begin + per);
    int32_t more = 0, equal = 0;
    for (int i = begin; i < end; ++i) {
        const uint32_t k = key_of(i);
        more += k > prefix;
        equal += k == prefix;
    }
    int64_t incl = (int64_t)more << 32 | (uint32_t)equal;
    const int64_t mine = incl;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int64_t up = __shfl_up_sync(~0u, incl, o);
        if (tid % 32 >= o) incl += up;
    }
    if (tid % 32 == 31) s_warp[tid / 32] = incl;
    __syncthreads();
    for (int i = 0; i < tid / 32; ++i) incl += s_warp[i];
    incl -= mine;
    int rank_eq = (int)(uint32_t)incl, at = (int)(incl >> 32) + min(rank_eq, left);
    for (int i = begin; i < end; ++i) {
        const uint32_t k = key_of(i);
        if (k > prefix || (k == prefix && rank_eq++ < left)) kept[at++] = i;
    }
}

constexpr int kMoveThreads = 256;

// Out of place: CTA (chunk of destination rows, layer, sequence, head); a row is a token's key and value.
__global__ void __launch_bounds__(kMoveThreads) evict_move(const __grid_constant__ EvictParams p, int rows, int chunks) {
    int u = blockIdx.x;
    const int chunk = u % chunks;
    u /= chunks;
    const int h = u % p.kv_heads, s = u / p.kv_heads % p.num_seqs, l = u / p.kv_heads / p.num_seqs;
    const int n = p.new_lens[s], begin = chunk * rows, T = p.cache.block_tokens;
    if (begin >= n) return;
    const bool cut = p.seq_lens[s] > n;
    const int w = h / p.cache.heads, hw = h - w * p.cache.heads;
    const int32_t *src_bt = p.src_bt + (int64_t)s * p.max_blocks, *dst_bt = p.dst_bt + (int64_t)s * p.dst_max_blocks;
    const int32_t* kept = p.kept + ((int64_t)(l * p.num_seqs + s) * p.kv_heads + h) * p.budget;
    char* pool = p.cache.pools[w] + l * p.layer_stride + hw * p.cache.head_stride;
    const int count = min(rows, n - begin), vecs = p.vec / 16;
    for (int i = threadIdx.x; i < count * vecs; i += kMoveThreads) {
        const int j = begin + i / vecs, c = i % vecs * 16, from = cut ? kept[j] : j;
        const char* a = pool + src_bt[from / T] * p.cache.block_stride + from % T * p.cache.tok_stride + c;
        char* b = pool + dst_bt[j / T] * p.cache.block_stride + j % T * p.cache.tok_stride + c;
        const uint4 key = *reinterpret_cast<const uint4*>(a), value = *reinterpret_cast<const uint4*>(a + p.cache.kv_stride);
        *reinterpret_cast<uint4*>(b) = key;
        *reinterpret_cast<uint4*>(b + p.cache.kv_stride) = value;
    }
    if (p.has_scores) {
        float* scores = p.scores[w] + l * p.layer_scores;
        for (int i = threadIdx.x; i < count; i += kMoveThreads) {
            const int j = begin + i, from = cut ? kept[j] : j;
            scores[((int64_t)dst_bt[j / T] * p.cache.heads + hw) * T + j % T] =
                scores[((int64_t)src_bt[from / T] * p.cache.heads + hw) * T + from % T];
        }
    }
}

// In place: one CTA per (layer, sequence, head) takes the kept tokens in order, a chunk at a time.  Token j of the new
// order comes from index kept[j] >= j, so what a chunk overwrites has been read by it or by an earlier one.
__global__ void __launch_bounds__(kMoveThreads) evict_close_up(const __grid_constant__ EvictParams p, int rows) {
    extern __shared__ __align__(16) char smem[];
    const int u = blockIdx.x;
    const int h = u % p.kv_heads, s = u / p.kv_heads % p.num_seqs, l = u / p.kv_heads / p.num_seqs;
    const int n = p.new_lens[s], T = p.cache.block_tokens;
    if (n < 0 || p.seq_lens[s] <= n) return;
    const int w = h / p.cache.heads, hw = h - w * p.cache.heads;
    const int32_t* bt = p.src_bt + (int64_t)s * p.max_blocks;
    const int32_t* kept = p.kept + ((int64_t)(l * p.num_seqs + s) * p.kv_heads + h) * p.budget;
    char* pool = p.cache.pools[w] + l * p.layer_stride + hw * p.cache.head_stride;
    float* scores = p.has_scores ? p.scores[w] + l * p.layer_scores : nullptr;
    const int vecs = p.vec / 16;
    uint4* buf = reinterpret_cast<uint4*>(smem);
    float* sbuf = reinterpret_cast<float*>(smem + (int64_t)rows * 2 * p.vec);
    for (int begin = 0; begin < n; begin += rows) {
        const int count = min(rows, n - begin);
        for (int i = threadIdx.x; i < count * vecs; i += kMoveThreads) {
            const int from = kept[begin + i / vecs];
            const char* a = pool + bt[from / T] * p.cache.block_stride + from % T * p.cache.tok_stride + i % vecs * 16;
            buf[2 * i] = *reinterpret_cast<const uint4*>(a);
            buf[2 * i + 1] = *reinterpret_cast<const uint4*>(a + p.cache.kv_stride);
        }
        if (scores)
            for (int i = threadIdx.x; i < count; i += kMoveThreads) {
                const int from = kept[begin + i];
                sbuf[i] = scores[((int64_t)bt[from / T] * p.cache.heads + hw) * T + from % T];
            }
        __syncthreads();
        for (int i = threadIdx.x; i < count * vecs; i += kMoveThreads) {
            const int j = begin + i / vecs;
            char* b = pool + bt[j / T] * p.cache.block_stride + j % T * p.cache.tok_stride + i % vecs * 16;
            *reinterpret_cast<uint4*>(b) = buf[2 * i];
            *reinterpret_cast<uint4*>(b + p.cache.kv_stride) = buf[2 * i + 1];
        }
        if (scores)
            for (int i = threadIdx.x; i < count; i += kMoveThreads) {
                const int j = begin + i;
                scores[((int64_t)bt[j / T] * p.cache.heads + hw) * T + j % T] = sbuf[i];
            }
        __syncthreads();
    }
}

}  // namespace amoeba

using namespace amoeba;

extern "C" amoeba_status amoeba_evict_workspace_bytes(const amoeba_layout* layout, int32_t num_layers, int32_t num_seqs,
                                                      int32_t budget, int64_t* bytes) {
    int64_t pool = 0;
    if (!layout || !bytes || num_layers < 0 || num_seqs < 0 || budget < 1) return AMOEBA_ERR_INVALID_ARG;
    const amoeba_status st = amoeba_layout_kv_pool_bytes(layout, &pool);
    if (st != AMOEBA_OK) return st;
    *bytes = ((int64_t)num_layers * num_seqs * layout->model.num_kv_heads * budget * 4 + 15) / 16 * 16;
    return AMOEBA_OK;
}

extern "C" amoeba_status amoeba_evict_kv(const amoeba_layout* layout, int32_t layer_begin, int32_t layer_end,
                                         void* const* pools, float* const* score_pools, const int32_t* d_src_bt,
                                         const int32_t* d_seq_lens, int32_t num_seqs, int32_t max_blocks_per_seq,
                                         const int32_t* d_dst_bt, int32_t dst_max_blocks_per_seq, int32_t budget,
                                         int32_t recent, int32_t* d_new_lens, int32_t* d_status, void* d_workspace,
                                         int64_t workspace_bytes, void* cuda_stream) {
    EvictParams p{};
    if (!layout || num_seqs < 0 || max_blocks_per_seq < 0 || dst_max_blocks_per_seq < 0 || budget < 1 || recent < 0 ||
        recent > budget || !d_status || layer_begin < 0 || layer_end < layer_begin)
        return AMOEBA_ERR_INVALID_ARG;
    amoeba_status st;
    if (layer_end == layer_begin || num_seqs == 0) return AMOEBA_OK;
    if ((st = make_cache_view(layout, layer_begin, pools, &p.cache)) != AMOEBA_OK) return st;
    if (layer_end > layout->model.num_layers) return AMOEBA_ERR_INVALID_ARG;
    if (!d_seq_lens || !d_new_lens || d_new_lens == d_seq_lens || !d_src_bt || !d_dst_bt) return AMOEBA_ERR_INVALID_ARG;
    p.in_place = d_src_bt == d_dst_bt;
    if (p.in_place && dst_max_blocks_per_seq != max_blocks_per_seq) return AMOEBA_ERR_INVALID_ARG;
    if (!score_pools && recent != budget) return AMOEBA_ERR_INVALID_ARG;
    int64_t pool_bytes = 0, need = 0;
    if ((st = amoeba_layout_kv_pool_bytes(layout, &pool_bytes)) != AMOEBA_OK) return st;
    p.layers = layer_end - layer_begin;
    if ((st = amoeba_evict_workspace_bytes(layout, p.layers, num_seqs, budget, &need)) != AMOEBA_OK) return st;
    if (!d_workspace || workspace_bytes < need) return AMOEBA_ERR_INVALID_ARG;
    if ((uintptr_t)d_workspace % 16) return AMOEBA_ERR_ALIGNMENT;
    p.layer_stride = pool_bytes / layout->model.num_layers;
    p.layer_scores = (int64_t)layout->num_blocks * p.cache.heads * layout->block_tokens;
    p.has_scores = score_pools != nullptr;
    for (int r = 0; score_pools && r < layout->tp; ++r) {
        if (!score_pools[r]) return AMOEBA_ERR_INVALID_ARG;
        if ((uintptr_t)score_pools[r] % 16) return AMOEBA_ERR_ALIGNMENT;
        p.scores[r] = score_pools[r] + layer_begin * p.layer_scores;
    }
    p.src_bt = d_src_bt, p.seq_lens = d_seq_lens, p.dst_bt = d_dst_bt;
    p.new_lens = d_new_lens, p.status = d_status;
    p.kept = static_cast<int32_t*>(d_workspace);
    p.num_seqs = num_seqs, p.max_blocks = max_blocks_per_seq, p.dst_max_blocks = dst_max_blocks_per_seq;
    p.budget = budget, p.recent = recent, p.kv_heads = layout->model.num_kv_heads;
    p.vec = layout->model.head_dim * layout->model.elem_bytes;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const int64_t units = (int64_t)p.layers * num_seqs * p.kv_heads;
    // rows of a chunk: 64 KiB of keys and values
    const int rows = 65536 / (2 * p.vec);
    const int64_t most = std::min<int64_t>(budget, (int64_t)max_blocks_per_seq * layout->block_tokens);
    const int64_t chunks = rows ? (most + rows - 1) / rows : 0;
    if (rows < 1 || units > INT32_MAX || units * std::max<int64_t>(chunks, 1) > INT32_MAX) return AMOEBA_ERR_UNSUPPORTED;
    evict_select<<<(int)units, kSelectThreads, 0, stream>>>(p);
    if ((st = launch_result()) != AMOEBA_OK || chunks == 0) return st;
    if (p.in_place) {
        const int smem = rows * (2 * p.vec + 4);
        if (ensure_dynamic_smem((const void*)evict_close_up, smem) != cudaSuccess) return AMOEBA_ERR_CUDA;
        evict_close_up<<<(int)units, kMoveThreads, smem, stream>>>(p, rows);
    } else {
        evict_move<<<(int)(units * chunks), kMoveThreads, 0, stream>>>(p, rows, (int)chunks);
    }
    return launch_result();
}
