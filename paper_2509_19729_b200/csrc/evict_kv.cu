// amoeba_evict_kv: long sequences cut to a budget by their tokens' scores.
//
// Two launches: which tokens stay (for each layer, sequence and key head, by the budget-th largest score: an ordered list of
// the kept indices), and the move of their keys, values and scores.  Memory-bound: the scores are read once, what stays is
// read and written once.  Measured: 32 sequences of 700 to 8192 tokens cut to 1024, two layers, 8 key heads of 128: 118 us, of
// which the selection is 25 (latency: one unit takes a CTA 10 to 20 us) and the move 84 (5.6 TB/s of rows of 256 bytes); one of
// 131072 cut to 16384: 51 us, 25 and 22.  (Both in one kernel took 117 and 67 us.)
#include "cache_view.cuh"
#include "cluster.cuh"
#include "copy_engine.cuh"

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

// The sequence's length, or -1 if it is refused.  The whole cluster asks together, each CTA looking at its part of the tables;
// bad: [kMaxCluster] in shared memory.  Another CTA's shared memory may be written once that CTA runs: every CTA arrives at the
// cluster's barrier before it looks at the tables and waits there after, in front of its first remote store.
__device__ __forceinline__ int checked_len(const EvictParams& p, int s, bool reports, uint32_t rank, uint32_t size, int32_t* bad) {
    if (size > 1) cluster_arrive();
    const int len = p.seq_lens[s], T = p.cache.block_tokens;
    int code = 0;
    bool fits = len >= 0 && len <= min((int64_t)p.max_blocks * T, (int64_t)kMaxTokens);
    if (fits) {
        const int keep = min(len, p.budget), n_src = (len + T - 1) / T, n_dst = (keep + T - 1) / T;
        fits = n_dst <= p.dst_max_blocks;
        if (fits) {
#pragma unroll 4
            for (int i = rank * blockDim.x + threadIdx.x; i < n_src; i += blockDim.x * size) {
                const int b = p.src_bt[(int64_t)s * p.max_blocks + i];
                if (b < 0 || b >= p.cache.num_blocks) code = 1;
            }
#pragma unroll 4
            for (int i = rank * blockDim.x + threadIdx.x; i < n_dst; i += blockDim.x * size) {
                const int b = p.dst_bt[(int64_t)s * p.dst_max_blocks + i];
                if (b < 0 || b >= p.cache.num_blocks) code = 1;
            }
        }
    }
    if (size > 1) cluster_wait();
    if (!fits) {  // all threads of the cluster alike
        if (reports && threadIdx.x == 0) report(p.status, AMOEBA_ERR_INVALID_ARG);
        return -1;
    }
    code = __syncthreads_or(code);
    if (size > 1) {
        if (threadIdx.x < size) store_remote(&bad[rank], threadIdx.x, code);
        cluster_sync();
        for (uint32_t r = 0; r < size; ++r) code |= bad[r];
    }
    if (!code) return len;
    if (reports && threadIdx.x == 0) report(p.status, AMOEBA_ERR_BAD_BLOCK_ID);
    return -1;
}

// Scores as whole numbers of the same order: a NaN is 0, below -infinity; -0 is 0.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0;
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// ------------------------------------------------------------------------------------------------ which tokens stay
// A cluster of CTAs for each (layer, sequence, key head): each takes a run of the tokens, its scores as ordered whole numbers
// in shared memory.  The smallest score that stays is found from the top, 11, 11 and 10 bits at a time, from counts of the
// digits that all CTAs of the cluster add up; then every warp lists the kept ones of its own run of tokens in order.
constexpr int kSelectKeys = 12288;  // keys that a CTA holds, unless eight CTAs need to hold more
constexpr int kDigits = 2048;

struct SelectShared {
    alignas(16) int32_t count[kDigits];  // of this CTA's tokens, by digit
    alignas(16) int32_t total[kDigits];  // of the cluster's
    int32_t warp[32];
    int32_t more, equal;      // this CTA's tokens above the limit, and at it
    int32_t found[2];         // digit, and how many at it stay
    int32_t before[32][2];
    int32_t bad[kMaxCluster];
};

template <int kSelectThreads>
__global__ void __launch_bounds__(kSelectThreads) evict_select(const __grid_constant__ EvictParams p, int room) {
    constexpr int kSelectWarps = kSelectThreads / 32;
    constexpr int kOwn = kSelectThreads < 512 ? kDigits / kSelectThreads : 4, kDigitThreads = kDigits / kOwn;  // digits of a thread
    extern __shared__ __align__(16) uint32_t s_keys[];
    __shared__ SelectShared sh;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    grid_dependency_launch();
    const uint32_t rank = cluster_rank(), size = cluster_size();
    const int unit = blockIdx.x / size;
    const int h = unit % p.kv_heads, s = unit / p.kv_heads % p.num_seqs, l = unit / p.kv_heads / p.num_seqs;
    const bool first = l == 0 && h == 0 && rank == 0;
    const int len = checked_len(p, s, first, rank, size, sh.bad);
    if (first && tid == 0) p.new_lens[s] = min(len, p.budget);
    if (len <= p.budget) return;  // the whole cluster
    const int free = len - p.recent, need = p.budget - p.recent;
    const int w = h / p.cache.heads, hw = h - w * p.cache.heads, T = p.cache.block_tokens;
    int32_t* kept = p.kept + ((int64_t)(l * p.num_seqs + s) * p.kv_heads + h) * p.budget;
    for (int i = rank * kSelectThreads + tid; i < p.recent; i += size * kSelectThreads) kept[need + i] = free + i;
    if (need == 0) return;

    const int run = (free + size * 32 - 1) / (size * 32) * 32;  // tokens of a CTA
    const int begin = min(free, (int)rank * run), n = min(free - begin, run);
    const float* scores = p.scores[w] + l * p.layer_scores;
    const int32_t* table = p.src_bt + (int64_t)s * p.max_blocks;
    auto score_at = [&](int i) { return ((int64_t)table[i / T] * p.cache.heads + hw) * T + i % T; };
    const bool held = n <= room;
    if (held) {
        if (T % 4 == 0) {  // (run is a multiple of 32: four tokens from a multiple of four on are in one block)
            constexpr int kAtOnce = 4;
            for (int base = tid * 4; base < n; base += kSelectThreads * 4 * kAtOnce) {
                int64_t at[kAtOnce];
                float4 x[kAtOnce];
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int i = base + u * kSelectThreads * 4;
                    if (i < n) at[u] = score_at(begin + i);
                }
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u)
                    if (base + u * kSelectThreads * 4 < n) x[u] = *reinterpret_cast<const float4*>(scores + at[u]);
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u)
                    if (base + u * kSelectThreads * 4 < n)
                        *reinterpret_cast<uint4*>(s_keys + base + u * kSelectThreads * 4) =
                            make_uint4(order_of(x[u].x), order_of(x[u].y), order_of(x[u].z), order_of(x[u].w));
            }
        } else {
            for (int i = tid; i < n; i += kSelectThreads) s_keys[i] = order_of(scores[score_at(begin + i)]);
        }
    }
    auto key_of = [&](int i) { return held ? s_keys[i] : order_of(scores[score_at(begin + i)]); };

    uint32_t limit = 0;  // found so far, from the top
    int left = need;     // how many of the tokens that agree with it stay
    for (int round = 0; round < 3; ++round) {
        const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, bits = round == 2 ? 10 : 11;
        const uint32_t above = round == 0 ? 0u : ~0u << (shift + bits);
        for (int i = tid; i < kDigits; i += kSelectThreads) sh.count[i] = 0;
        __syncthreads();
        // (plain additions: gathering a warp's equal digits first takes longer than adding them one by one)
        const uint32_t ones = (1u << bits) - 1;
        if (held) {
#pragma unroll 2
            for (int i = tid * 4; i < n; i += kSelectThreads * 4) {
                const uint4 k = *reinterpret_cast<const uint4*>(s_keys + i);
                if ((k.x & above) == limit) atomicAdd(&sh.count[k.x >> shift & ones], 1);
                if ((k.y & above) == limit && i + 1 < n) atomicAdd(&sh.count[k.y >> shift & ones], 1);
                if ((k.z & above) == limit && i + 2 < n) atomicAdd(&sh.count[k.z >> shift & ones], 1);
                if ((k.w & above) == limit && i + 3 < n) atomicAdd(&sh.count[k.w >> shift & ones], 1);
            }
        } else {
            for (int i = tid; i < n; i += kSelectThreads) {
                const uint32_t k = order_of(scores[score_at(begin + i)]);
                if ((k & above) == limit) atomicAdd(&sh.count[k >> shift & ones], 1);
            }
        }
        __syncthreads();
        const int32_t* total = sh.count;
        if (size > 1) {  // every CTA adds up its part of the digits and hands the sums to all
            cluster_sync();
            const int part = kDigits / size;
            for (int d = rank * part + tid; d < (int)(rank + 1) * part; d += kSelectThreads) {
                int v[kMaxCluster], sum = 0;
#pragma unroll
                for (uint32_t r = 0; r < kMaxCluster; ++r) v[r] = r < size ? load_remote(&sh.count[d], r) : 0;
#pragma unroll
                for (uint32_t r = 0; r < kMaxCluster; ++r) sum += v[r];
                for (uint32_t r = 0; r < size; ++r) store_remote(&sh.total[d], r, sum);
            }
            cluster_sync();
            total = sh.total;
        }
        // from the largest digit down: thread t has kOwn of them, from 2047 - kOwn * t on
        int mine[kOwn] = {}, before = 0, sum = 0;
        if (tid < kDigitThreads) {
#pragma unroll
            for (int j = 0; j < kOwn; j += 4) {
                const int4 four = *reinterpret_cast<const int4*>(&total[kDigits - 4 - tid * kOwn - j]);
                mine[j] = four.w, mine[j + 1] = four.z, mine[j + 2] = four.y, mine[j + 3] = four.x;
                sum += four.x + four.y + four.z + four.w;
            }
            before = sum;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int up = __shfl_up_sync(~0u, before, o);
                if (lane >= o) before += up;
            }
            if (lane == 31) sh.warp[warp] = before;
        }
        __syncthreads();
        if (tid < kDigitThreads) {
            before -= sum;
            for (int i = 0; i < warp; ++i) before += sh.warp[i];
            if (before < left && left <= before + sum) {
#pragma unroll
                for (int j = 0; j < kOwn; ++j) {
                    if (before < left && left <= before + mine[j])
                        sh.found[0] = kDigits - 1 - tid * kOwn - j, sh.found[1] = left - before;
                    before += mine[j];
                }
            }
        }
        __syncthreads();
        limit |= (uint32_t)sh.found[0] << shift;
        left = sh.found[1];
    }

    // Every warp's run of tokens, counted, and then listed behind those of the warps and CTAs before; four tokens a lane.
    const int per = (n + kSelectThreads * 4 - 1) / (kSelectThreads * 4) * 128;
    const int from = min(n, warp * per), to = min(n, from + per);
    auto four = [&](int i, uint32_t (&k)[4]) {  // keys from i on; behind the end 0, which is below any limit but a NaN's
        if (held && i + 3 < to) {
            const uint4 x = *reinterpret_cast<const uint4*>(s_keys + i);
            k[0] = x.x, k[1] = x.y, k[2] = x.z, k[3] = x.w;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) k[j] = i + j < to ? key_of(i + j) : 0;
        }
    };
    int more = 0, equal = 0;
#pragma unroll 2
    for (int base = from; base < to; base += 128) {
        const int i = base + lane * 4;
        uint32_t k[4];
        four(i, k);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            more += k[j] > limit;
            equal += k[j] == limit && i + j < to;
        }
    }
    more = __reduce_add_sync(~0u, more), equal = __reduce_add_sync(~0u, equal);
    if (lane == 0) sh.before[warp][0] = more, sh.before[warp][1] = equal;
    __syncthreads();
    if (tid == 0) {
        int a = 0, b = 0;
        for (int i = 0; i < kSelectWarps; ++i) a += sh.before[i][0], b += sh.before[i][1];
        sh.more = a, sh.equal = b;
    }
    if (size > 1) cluster_sync();
    else __syncthreads();
    more = equal = 0;
    for (uint32_t r = 0; r < rank; ++r) more += load_remote(&sh.more, r), equal += load_remote(&sh.equal, r);
    for (int i = 0; i < warp; ++i) more += sh.before[i][0], equal += sh.before[i][1];
    for (int base = from; base < to; base += 128) {
        const int i = base + lane * 4;
        uint32_t k[4];
        four(i, k);
        int mine = 0;  // above the limit in the low half, at it in the high one
#pragma unroll
        for (int j = 0; j < 4; ++j) mine += (k[j] > limit) + (k[j] == limit && i + j < to ? 0x10000 : 0);
        int incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int up = __shfl_up_sync(~0u, incl, o);
            if (lane >= o) incl += up;
        }
        int m = more + ((incl - mine) & 0xffff), e = equal + ((incl - mine) >> 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool is_more = k[j] > limit, is_equal = k[j] == limit && i + j < to;
            if (is_more || (is_equal && e < left)) kept[m + min(e, left)] = begin + i + j;
            m += is_more, e += is_equal;
        }
        const int all = __shfl_sync(~0u, incl, 31);
        more += all & 0xffff, equal += all >> 16;
    }
    if (size > 1) cluster_sync();  // no CTA ends while another reads its counts
}

// ------------------------------------------------------------------------------------------------ the move
// Rows are tokens: a key and a value of `vec` bytes each.  The offsets of a chunk of rows are worked out once, a thread a row,
// and the rows then copied 16 bytes a lane with as many loads in flight as a lane has stores.
constexpr int kMoveThreads = 256, kMoveRows = 256;  // rows: at most, a thread each

struct MoveUnit {
    int s, h, l, n, w, hw;
    bool cut;
    const int32_t *src_bt, *dst_bt, *kept;
    char* pool;
    float* scores;
};
__device__ __forceinline__ MoveUnit move_unit(const EvictParams& p, int u) {
    MoveUnit m;
    m.h = u % p.kv_heads, m.s = u / p.kv_heads % p.num_seqs, m.l = u / p.kv_heads / p.num_seqs;
    m.n = p.new_lens[m.s];
    m.cut = p.seq_lens[m.s] > m.n;
    m.w = m.h / p.cache.heads, m.hw = m.h - m.w * p.cache.heads;
    m.src_bt = p.src_bt + (int64_t)m.s * p.max_blocks, m.dst_bt = p.dst_bt + (int64_t)m.s * p.dst_max_blocks;
    m.kept = p.kept + ((int64_t)(m.l * p.num_seqs + m.s) * p.kv_heads + m.h) * p.budget;
    m.pool = p.cache.pools[m.w] + m.l * p.layer_stride + m.hw * p.cache.head_stride;
    m.scores = p.has_scores ? p.scores[m.w] + m.l * p.layer_scores : nullptr;
    return m;
}
struct RowPlace {
    int64_t bytes;   // of the token's key in the head's part of the pool
    int64_t score;
};
__device__ __forceinline__ RowPlace place(const EvictParams& p, const MoveUnit& m, const int32_t* bt, int i) {
    const int T = p.cache.block_tokens, b = i / T, t = i - b * T;
    const int64_t block = bt[b];
    return RowPlace{block * p.cache.block_stride + t * p.cache.tok_stride, (block * p.cache.heads + m.hw) * T + t};
}

// Out of place: a CTA takes chunks of destination rows of one unit.
template <int kVecs>  // 16-byte pieces of a key, or 0: any number
__global__ void __launch_bounds__(kMoveThreads, 4) evict_move(const __grid_constant__ EvictParams p, int chunks, int rows) {
    __shared__ int64_t s_from[kMoveRows], s_to[kMoveRows];
    grid_dependency_wait();
    const MoveUnit m = move_unit(p, blockIdx.x / chunks);
    const int begin = blockIdx.x % chunks * rows;
    if (begin >= m.n) return;
    const int count = min(rows, m.n - begin), tid = threadIdx.x;
    if (tid < count) {
        const int j = begin + tid;
        const RowPlace to = place(p, m, m.dst_bt, j), from = place(p, m, m.src_bt, m.cut ? m.kept[j] : j);
        s_from[tid] = from.bytes, s_to[tid] = to.bytes;
        if (m.scores) m.scores[to.score] = m.scores[from.score];
    }
    __syncthreads();
    const int vecs = kVecs ? kVecs : p.vec / 16;
    const int all = count * vecs * 2;  // piece i: row i / (2 vecs), key or value, 16 bytes of it
    constexpr int kUnroll = 8;
    for (int base = tid; base < all; base += kMoveThreads * kUnroll) {
        uint4 x[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int i = base + u * kMoveThreads, row = i / (2 * vecs), c = i - row * 2 * vecs, kv = c >= vecs;
            if (i < all)
                x[u] = ld_stream(reinterpret_cast<const uint4*>(m.pool + s_from[row] + kv * p.cache.kv_stride + (c - kv * vecs) * 16));
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int i = base + u * kMoveThreads, row = i / (2 * vecs), c = i - row * 2 * vecs, kv = c >= vecs;
            if (i < all) st_stream(reinterpret_cast<uint4*>(m.pool + s_to[row] + kv * p.cache.kv_stride + (c - kv * vecs) * 16), x[u]);
        }
    }
}

// In place: a cluster of CTAs takes the kept tokens of one unit in order, a chunk at a time.  Token j of the new order
// comes from index kept[j] >= j, so what a chunk overwrites has been read with it or with an earlier one: all of the chunk
// is read into registers before any of it is written.
constexpr int kCloseThreads = 512, kCloseHeld = 8;  // 16-byte pieces that a thread holds
template <int kVecs>
__global__ void __launch_bounds__(kCloseThreads) evict_close_up(const __grid_constant__ EvictParams p, int rows) {
    extern __shared__ __align__(16) char smem[];  // [rows] from, [rows] to
    int64_t *s_from = reinterpret_cast<int64_t*>(smem), *s_to = s_from + rows;
    grid_dependency_wait();
    const uint32_t rank = cluster_rank(), size = cluster_size();
    const MoveUnit m = move_unit(p, blockIdx.x / size);
    if (m.n < 0 || !m.cut) return;  // the whole cluster
    const int vecs = kVecs ? kVecs : p.vec / 16, tid = threadIdx.x;
    for (int base = 0; base < m.n; base += rows * size) {
        const int begin = base + rank * rows, count = max(0, min(rows, m.n - begin)), all = count * vecs * 2;
        // rows <= kCloseThreads: a thread holds one row's score
        float score = 0.f;
        int64_t score_to = -1;
        if (tid < count) {
            const RowPlace to = place(p, m, m.src_bt, begin + tid), from = place(p, m, m.src_bt, m.kept[begin + tid]);
            s_from[tid] = from.bytes, s_to[tid] = to.bytes;
            if (m.scores) score = m.scores[from.score], score_to = to.score;
        }
        __syncthreads();
        uint4 x[kCloseHeld];
#pragma unroll
        for (int u = 0; u < kCloseHeld; ++u) {
            const int i = tid + u * kCloseThreads, row = i / (2 * vecs), c = i - row * 2 * vecs, kv = c >= vecs;
            if (i < all)
                x[u] = *reinterpret_cast<const uint4*>(m.pool + s_from[row] + kv * p.cache.kv_stride + (c - kv * vecs) * 16);
        }
        if (size > 1) cluster_sync();
        else __syncthreads();
#pragma unroll
        for (int u = 0; u < kCloseHeld; ++u) {
            const int i = tid + u * kCloseThreads, row = i / (2 * vecs), c = i - row * 2 * vecs, kv = c >= vecs;
            if (i < all) *reinterpret_cast<uint4*>(m.pool + s_to[row] + kv * p.cache.kv_stride + (c - kv * vecs) * 16) = x[u];
        }
        if (score_to >= 0) m.scores[score_to] = score;
        __syncthreads();  // the offsets are used up
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
    const int64_t tokens = (int64_t)max_blocks_per_seq * layout->block_tokens, most = std::min<int64_t>(budget, tokens);
    const int pieces = p.vec / 16 * 2;
    // in place: a row's pieces have to fit into what a CTA's threads hold
    const int rows = std::min(kCloseThreads, kCloseThreads * kCloseHeld / pieces);
    if (rows < 1 || units * std::max<int64_t>((most + 31) / 32, kMaxCluster) > INT32_MAX) return AMOEBA_ERR_UNSUPPORTED;
    const DeviceInfo dev = cached_device_info();
    if (!dev.sms) return AMOEBA_ERR_CUDA;
    // CTAs to a unit: as many as hold its scores; a CTA of a full cluster may hold more, and reads them anew past that.
    int cluster = 1;
    while (cluster < kMaxCluster && tokens > (int64_t)cluster * kSelectKeys) cluster *= 2;
    const int64_t slice = (tokens + cluster * 32 - 1) / (cluster * 32) * 32;
    const int room = (int)std::min<int64_t>(slice, (dev.smem_optin - (int)sizeof(SelectShared) - 1024) / 4 / 32 * 32);
    // (few and long units: as many threads as a CTA may have)
    st = cluster == kMaxCluster ? launch_clusters(evict_select<1024>, units * cluster, 1024, (size_t)room * 4, cluster, false, stream, p, room)
         : units > 2 * dev.sms ? launch_clusters(evict_select<256>, units * cluster, 256, (size_t)room * 4, cluster, false, stream, p, room)
                               : launch_clusters(evict_select<512>, units * cluster, 512, (size_t)room * 4, cluster, false, stream, p, room);
    if (st != AMOEBA_OK || tokens == 0) return st;
    if (p.in_place) {
        // One CTA moves about 100 GB/s; with few units, several CTAs to each.
        int group = 1;
        while (group < kMaxCluster && units * group * 2 <= 2 * dev.sms && (int64_t)group * rows < most) group *= 2;
        auto* kernel = p.vec == 256 ? evict_close_up<16> : p.vec == 128 ? evict_close_up<8> : evict_close_up<0>;
        return launch_clusters(kernel, units * group, kCloseThreads, (size_t)rows * 16, group, true, stream, p, rows);
    }
    auto* kernel = p.vec == 256 ? evict_move<16> : p.vec == 128 ? evict_move<8> : evict_move<0>;
    // Out of place: long chunks, in which looking up the rows counts for little, if that leaves four CTAs to an SM.
    int chunk = kMoveRows;
    while (chunk > 32 && units * ((most + chunk - 1) / chunk) < 4 * dev.sms) chunk /= 2;
    const int64_t chunks = std::max<int64_t>((most + chunk - 1) / chunk, 1);
    return launch_clusters(kernel, units * chunks, kMoveThreads, 0, 1, true, stream, p, (int)chunks, chunk);
}
