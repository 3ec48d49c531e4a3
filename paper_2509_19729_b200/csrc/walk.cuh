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

}  // namespace amoeba
