// How the operators that read the cache share the work out.
//
// A unit is one (sequence, key head, tile of query rows); its work is a run of tiles of consecutive tokens.  All units'
// tiles are laid end to end in the order (sequence, head, row tile), and every CTA takes an equal run of them, wherever
// it begins and ends: one very long sequence is spread over as many CTAs as its share of the work, and a batch of any
// mix finishes together.  The lengths are known only on the device, so every CTA adds them up for itself; there is no
// planning launch and nothing for the host to know.
#pragma once
#include "cache_view.cuh"

namespace amoeba {

struct Shape {  // what the split depends on, besides the batch
    int32_t group;      // query heads per key head
    int32_t kv_heads;   // of all workers
    int32_t window;     // 0 = none
    int32_t rows;       // query rows per row tile
    int32_t tile;       // tokens per tile, a power of two
    int32_t min_rows, max_rows;  // sequences with more or fewer rows (new tokens * group) are not this launch's
    int32_t rowless;    // 1: sequences without rows have one row tile all the same
    int32_t start;      // what a unit's start and end cost, in tiles (take_weighted_share)
};

struct Range {
    int32_t lo, hi;  // tokens that some row of the tile sees
    int32_t base;    // lo rounded down to a tile
    int32_t tiles;   // at least 1, so that rows that see nothing are answered too
};

__device__ __forceinline__ Range row_tile_range(const Shape& p, const Seq& q, int m) {
    Range r;
    const int n = q.qn * p.group;
    int p0 = q.len - q.qn, p1 = q.len - 1;  // cache indices of the tile's first and last rows
    if (n > p.rows && !q.level) {
        const int last = (int)min((int64_t)n, (int64_t)(m + 1) * p.rows) - 1;
        p1 = p0 + last / p.group;
        p0 += m * p.rows / p.group;
    }
    r.hi = min(max(p1 + 1, 0), q.len);
    r.lo = p.window > 0 ? min(max(p0 - p.window + 1, 0), r.hi) : min(q.first, r.hi);
    r.base = r.lo & -p.tile;  // (a power of two)
    r.tiles = max(1, (r.hi - r.base + p.tile - 1) >> __ffs(p.tile) - 1);
    return r;
}

__device__ __forceinline__ int row_tiles(const Shape& p, const Seq& q) {
    const int n = q.qn * p.group;
    if (n == 0) return p.rowless && q.ok ? 1 : 0;
    return n < p.min_rows || n > p.max_rows ? 0 : (n - 1) / p.rows + 1;
}

// Tiles of one head of a sequence.
__device__ __forceinline__ int64_t head_tiles(const Shape& p, const Seq& q) {
    const int nm = row_tiles(p, q);
    if (q.level) return (int64_t)nm * row_tile_range(p, q, 0).tiles;
    int64_t n = 0;
    for (int m = 0; m < nm; ++m) n += row_tile_range(p, q, m).tiles;
    return n;
}

// First tile of CTA c's share.
__device__ __forceinline__ int64_t share_begin(int64_t total, int ctas, int c) {
    return total < (1 << 20) ? (uint32_t)total * (uint32_t)c / (uint32_t)ctas : total * c / ctas;  // (ctas < 4096)
}
struct Walk {
    int32_t s, h, m, t;  // sequence, key head, row tile, tile of it
    int32_t nm;
    Seq seq;
    Range range;

    template <class B>
    __device__ __forceinline__ void open(const Shape& p, const B& b, int block_tokens, int seq_index) {
        s = seq_index;
        seq = sequence(b, s, block_tokens);
        nm = row_tiles(p, seq);
        h = m = t = 0;
        if (nm) range = row_tile_range(p, seq, 0);
    }
    // To the tile `off` tiles into the (non-empty) sequence that is open.
    __device__ __forceinline__ void seek(const Shape& p, int64_t off) {
        if (seq.level) {  // all units have as many
            const int64_t unit = off >> 31 == 0 ? (uint32_t)off / (uint32_t)range.tiles : off / range.tiles;
            t = (int)(off - unit * range.tiles);
            h = (int)(unit / nm), m = (int)(unit - (int64_t)h * nm);
            return;
        }
        const int64_t per_head = head_tiles(p, seq);
        h = (off | per_head) >> 31 == 0 ? (int)((uint32_t)off / (uint32_t)per_head) : (int)(off / per_head);
        off -= h * per_head;
        for (m = 0;; ++m) {
            range = row_tile_range(p, seq, m);
            if (off < range.tiles) break;
            off -= range.tiles;
        }
        t = (int)off;
    }
    // To the first tile of the `unit`-th unit of the open sequence.
    __device__ __forceinline__ void to_unit(const Shape& p, int unit) {
        h = unit / nm;
        m = unit - h * nm;
        t = 0;
        range = row_tile_range(p, seq, m);
    }
    // To the next tile; the caller knows that there is one.
    template <class B>
    __device__ __forceinline__ void next(const Shape& p, const B& b, int block_tokens) {
        if (++t < range.tiles) return;
        t = 0;
        if (++m < nm) {
            range = row_tile_range(p, seq, m);
            return;
        }
        m = 0;
        if (++h < p.kv_heads) {
            if (nm > 1) range = row_tile_range(p, seq, 0);
            return;
        }
        do open(p, b, block_tokens, s + 1);
        while (nm == 0 && s + 1 < b.num_seqs);
    }
};

// Sum over the block of one value per thread; `shared` holds one value per warp.
template <int kThreads>
__device__ __forceinline__ int64_t block_sum(int64_t v, int64_t* shared) {
#pragma unroll
    for (int o = 16; o; o /= 2) v += __shfl_xor_sync(~0u, v, o);
    __syncthreads();
    if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) v += shared[w];
    return v;
}

// The run of tiles that is a CTA's share, and the unit that it begins in: what the join of cut units goes by.
struct Cut {
    int64_t begin, end;  // empty shares: begin = end
    int32_t s, h, m;     // the first tile's unit,
    int32_t t, tiles;    // its place in it, and the unit's tiles
    int32_t rows;        // of the unit
};
__device__ __forceinline__ void write_cut(const Shape& p, Cut* cuts, const Walk& w, int64_t begin, int64_t end) {
    if (threadIdx.x == 0)
        cuts[blockIdx.x] = Cut{begin, end, w.s, w.h, w.m, w.t, w.range.tiles, min(p.rows, w.seq.qn * p.group - w.m * p.rows)};
}

// This CTA's share: [*begin, *end) of all tiles, with `walk` at the first of them.  CTA 0 reports bad sequences.
template <int kThreads, class B>
__device__ void take_share(const Shape& p, const B& b, int block_tokens, Walk* walk, int64_t* begin_out, int64_t* end_out,
                           int32_t* status) {
    __shared__ int64_t s_warp[kThreads / 32];
    __shared__ int64_t s_off;
    __shared__ int32_t s_seq;
    const int tid = threadIdx.x;
    int64_t mine = 0, sum = 0;
    for (int s = tid; s < b.num_seqs; s += kThreads) {
        const Seq q = sequence(b, s, block_tokens);
        if (!q.ok && blockIdx.x == 0) report(status, AMOEBA_ERR_INVALID_ARG);
        mine = p.kv_heads * head_tiles(p, q);
        sum += mine;
    }
    const int64_t all = block_sum<kThreads>(sum, s_warp);
    const int ctas = (int)max((int64_t)1, min((int64_t)gridDim.x, all));
    const int64_t begin = (int)blockIdx.x < ctas ? share_begin(all, ctas, blockIdx.x) : all;
    const int64_t end = (int)blockIdx.x < ctas ? share_begin(all, ctas, blockIdx.x + 1) : all;
    *begin_out = begin, *end_out = end;
    int64_t run = 0;
    for (int base = 0; base < b.num_seqs; base += kThreads) {
        const int s = base + tid;
        if (b.num_seqs > kThreads)
            mine = s < b.num_seqs ? p.kv_heads * head_tiles(p, sequence(b, s, block_tokens)) : 0;
        int64_t incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int64_t up = __shfl_up_sync(~0u, incl, o);
            if (tid % 32 >= o) incl += up;
        }
        __syncthreads();
        if (tid % 32 == 31) s_warp[tid / 32] = incl;
        __syncthreads();
        int64_t before = run;
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < tid / 32) before += s_warp[w];
            run += s_warp[w];
        }
        const int64_t first = before + incl - mine;
        if (begin >= first && begin < first + mine) s_seq = s, s_off = begin - first;
        if (run > begin) break;  // block-uniform
    }
    __syncthreads();
    if (end > begin) {
        walk->open(p, b, block_tokens, s_seq);
        walk->seek(p, s_off);
    }
}

// The same where units are short and what starting and ending one costs counts: every unit weighs p.start tiles more, and the CTAs' shares
// are even by weight.  A border that falls into a unit's extra weight moves to its first tile.  [*begin, *end) are tiles as above.
// scratch: shared memory that nothing else uses yet.
struct ShareBorder {
    int64_t off, before;  // weight in front of it in its sequence, tiles in front of the sequence
    int64_t at;           // its tile
    int32_t s;
    Walk walk;
};
template <int kThreads, class B>
__device__ void take_weighted_share(const Shape& p, const B& b, int block_tokens, Walk* walk, int64_t* begin_out, int64_t* end_out,
                                    int32_t* status, char* scratch, int most_ctas) {
    constexpr int kWarps = kThreads / 32;
    int64_t* const s_warp = reinterpret_cast<int64_t*>(scratch);  // [2][kWarps]
    ShareBorder* const border = reinterpret_cast<ShareBorder*>(s_warp + 2 * kWarps);
    const int tid = threadIdx.x, lane = tid % 32;
    int64_t tiles = 0, weight = 0, sums[2] = {0, 0};
    auto look = [&](int s) {
        const Seq q = sequence(b, s, block_tokens);
        tiles = p.kv_heads * head_tiles(p, q), weight = tiles + (int64_t)p.kv_heads * row_tiles(p, q) * p.start;
        return q.ok;
    };
    for (int s = tid; s < b.num_seqs; s += kThreads) {
        if (!look(s) && blockIdx.x == 0) report(status, AMOEBA_ERR_INVALID_ARG);
        sums[0] += tiles, sums[1] += weight;
    }
    const int64_t all_tiles = block_sum<kThreads>(sums[0], s_warp), all = block_sum<kThreads>(sums[1], s_warp + kWarps);
    const int ctas = (int)max((int64_t)1, min((int64_t)most_ctas, all_tiles));
    const int c = min((int)blockIdx.x, ctas);
    const int64_t at[2] = {share_begin(all, ctas, c), share_begin(all, ctas, min(c + 1, ctas))};
    int64_t run_tiles = 0, run = 0;
    for (int base = 0; base < b.num_seqs; base += kThreads) {
        const int s = base + tid;
        if (b.num_seqs > kThreads) {
            tiles = weight = 0;
            if (s < b.num_seqs) look(s);
        }
        int64_t incl[2] = {tiles, weight};
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int64_t up0 = __shfl_up_sync(~0u, incl[0], o), up1 = __shfl_up_sync(~0u, incl[1], o);
            if (lane >= o) incl[0] += up0, incl[1] += up1;
        }
        __syncthreads();
        if (lane == 31) s_warp[tid / 32] = incl[0], s_warp[kWarps + tid / 32] = incl[1];
        __syncthreads();
        int64_t before_tiles = run_tiles, before = run;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < tid / 32) before_tiles += s_warp[w], before += s_warp[kWarps + w];
            run_tiles += s_warp[w], run += s_warp[kWarps + w];
        }
        const int64_t first = before + incl[1] - weight;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (at[i] >= first && at[i] < first + weight)
                border[i].s = s, border[i].off = at[i] - first, border[i].before = before_tiles + incl[0] - tiles;
        if (run > at[1]) break;  // block-uniform
    }
    __syncthreads();
    if (tid < 64 && at[tid / 32] < all) {  // a warp to each border
        ShareBorder& x = border[tid / 32];
        Walk w{};
        w.open(p, b, block_tokens, x.s);
        const int64_t head = head_tiles(p, w.seq), heavy = head + (int64_t)w.nm * p.start;
        int64_t off = x.off;
        w.h = (off | heavy) >> 31 == 0 ? (int)((uint32_t)off / (uint32_t)heavy) : (int)(off / heavy);
        off -= w.h * heavy;
        int64_t tile = x.before + w.h * head;
        for (w.m = 0;; ++w.m) {
            w.range = row_tile_range(p, w.seq, w.m);
            if (off < w.range.tiles + p.start) break;
            off -= w.range.tiles + p.start, tile += w.range.tiles;
        }
        w.t = max((int)off - p.start, 0);
        __syncwarp();
        if (lane == 0) x.walk = w, x.at = tile + w.t;
    }
    __syncthreads();
    *begin_out = at[0] < all ? border[0].at : all_tiles;
    *end_out = at[1] < all ? border[1].at : all_tiles;
    if (*end_out > *begin_out) *walk = border[0].walk;
    __syncthreads();  // the scratch is free
}

}  // namespace amoeba
