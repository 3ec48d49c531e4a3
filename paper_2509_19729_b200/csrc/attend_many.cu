// amoeba_attend for many rows: the matrix products run on the fifth-generation tensor cores.
//
// A unit has 256 query rows, two tiles of 128, and takes 128 tokens at a time.  One thread issues the products: S = Q K^T
// from shared memory into tensor memory (a row per lane, a token per column), and O += P V with P, the weights in 16
// bits, read from tensor memory where the softmax threads have written it over S.  Two warpgroups do the softmax, one
// for each tile, a thread for each row, so that maxima and sums need no exchange between threads; while one works on its
// S the tensor core has the other's products to do.  Three warps load keys and values through the block table into the
// 128-byte-swizzled layout that the products read: boxes of a tensor map, or 16 bytes at a time where a tile is not wanted whole or
// the blocks have no box's shape (umma.cuh).
//
// The first half of a tile's weights is handed on while the second is formed.  A row's logits are read from tensor memory twice,
// for the maximum and for the weights: kept in between they would fill 128 registers.
//
// Measured: four sequences, about 1830 new tokens each, 9 to 12 thousand cached, 32 query heads on 8 key heads of 128: 965 us
// (1.10 PFLOP/s) in short runs, 1.12 ms (0.95) when it runs on and the power limit takes the clock from 1965 to 1700 MHz.  Of a
// tile's 3.4 thousand clocks the tensor core is busy about 2.5; the rest is a row's softmax, 310 clocks for the maximum and 1500
// for the weights, whose 128 exponentials take 1024 on the special-function unit that two rows of the other tile use as well.  (A
// polynomial on the multiply-add units in place of every eighth exponential made it slower, 1010 us.)
//
// The running maximum of a row is only raised, and O scaled down, when a tile exceeds it by more than 2^8: the weights
// stay below 2^8 until then and the result is the same, as numerator and sum have the same factor.  That makes the
// scaling of O, a pass through tensor memory, rare.
//
// Tensor memory: columns 0-127 and 128-255 S and P of the two tiles, 256 and 256 + D their O.
#include "attend.cuh"
#include "umma.cuh"

namespace amoeba {

constexpr int kManyThreads = 384, kLoadWarps = 3, kLoadThreads = 32 * kLoadWarps;
constexpr float kRaise = 8.f;

template <int D>
struct ManyShape {
    static constexpr int kTileBytes = 128 * D * 2;  // 128 rows of queries, keys or values
    static constexpr int kStages = D == 128 ? 5 : 8;
    static constexpr int kSmem = (2 + kStages) * kTileBytes + 1024;  // up to 1 KiB goes to the alignment
};

struct ManyBarriers {
    uint64_t full[8], empty[8];  // ring of tiles: K, V, K, V, ...
    uint64_t q_full, q_empty;
    uint64_t s_full[2], p_half[2], p_full[2], o_full[2], o_free[2];
    uint64_t drain;
    uint32_t tmem;
    int32_t abort;
};

// ---- shares
// CTAs that work on the same keys at the same time find them in L2 (a batch's cache does not fit there, and every unit reads
// all of its sequence's).  So the units are dealt out whole and in order as long as there are plenty, and neighbours run through
// the same keys side by side; the last one or two units per CTA are cut so that all CTAs finish together, whatever the
// units before have cost each.  With more sequences than the table below holds, all units are cut as in walk.cuh.
constexpr int kDealtSeqs = 256;
struct Share {
    int32_t first_unit[kDealtSeqs + 1];  // of every sequence, and the end
    int32_t rounds;                      // units dealt to each
    int64_t begin, end;                  // of this CTA's run of tiles of the cut units
    int32_t begin_seq;
    int64_t begin_off;
};

// All threads of the block.  False: this CTA has nothing to do.  done: [kMaxSms] for the tiles of the units dealt to every CTA.
__device__ bool make_share(const AttendParams& p, Share& sh, int32_t* done) {
    __shared__ int64_t s_warp[kManyThreads / 32];
    const Shape& shape = p.shape;
    const Batch& b = p.batch;
    const int tid = threadIdx.x, ctas = gridDim.x, T = p.cache.block_tokens, S = b.num_seqs;
    sh.rounds = 0;
    if (S > kDealtSeqs) {
        Walk w{};
        int64_t begin, end;
        take_share<kManyThreads>(shape, b, T, &w, &begin, &end, p.status);
        if (tid == 0) {
            sh.begin = begin, sh.end = end;
            if (end > begin) {
                sh.begin_seq = w.s;
                int64_t off = w.t + w.h * head_tiles(shape, w.seq);
                for (int m = 0; m < w.m; ++m) off += row_tile_range(shape, w.seq, m).tiles;
                sh.begin_off = off;
            }
        }
        write_cut(shape, p.cuts, w, begin, end);
        __syncthreads();
        return end > begin;
    }
    // units and tiles before every sequence
    int32_t units = 0;
    int64_t tiles = 0;
    for (int base = 0; base < S; base += kManyThreads) {
        const int s = base + tid;
        int64_t n_units = 0, n_tiles = 0;
        if (s < S) {
            const Seq q = sequence(b, s, T);
            if (!q.ok && blockIdx.x == 0) report(p.status, AMOEBA_ERR_INVALID_ARG);
            n_units = (int64_t)shape.kv_heads * row_tiles(shape, q);
            n_tiles = shape.kv_heads * head_tiles(shape, q);
        }
        int64_t u = n_units, t = n_tiles;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int64_t uu = __shfl_up_sync(~0u, u, o), tt = __shfl_up_sync(~0u, t, o);
            if (tid % 32 >= o) u += uu, t += tt;
        }
        __syncthreads();
        if (tid % 32 == 31) s_warp[tid / 32] = u;
        __syncthreads();
        int64_t before = units;
        for (int w = 0; w < kManyThreads / 32; ++w) {
            if (w < tid / 32) before += s_warp[w];
            units += (int32_t)s_warp[w];
        }
        if (s < S) sh.first_unit[s] = (int32_t)(before + u - n_units);
        __syncthreads();
        if (tid % 32 == 31) s_warp[tid / 32] = t;
        __syncthreads();
        for (int w = 0; w < kManyThreads / 32; ++w) tiles += s_warp[w];
    }
    for (int c = tid; c < kMaxSms; c += kManyThreads) done[c] = 0;
    if (tid == 0) sh.first_unit[S] = units, sh.begin = sh.end = 0;
    __syncthreads();
    const int rounds = max(units / ctas - 1, 0), dealt = rounds * ctas;
    if (tid == 0) sh.rounds = rounds;
    // tiles of the dealt units, by CTA and in all (row tiles of a sequence cost the same for every head)
    int64_t mine = 0;
    int s = 0;
    for (int u = tid; u < dealt; u += kManyThreads) {
        while (sh.first_unit[s + 1] <= u) ++s;
        const Seq q = sequence(b, s, T);
        const int n = row_tile_range(shape, q, (u - sh.first_unit[s]) % row_tiles(shape, q)).tiles;
        atomicAdd(&done[u % ctas], n);
        mine += n;
    }
    const int64_t first_cut = block_sum<kManyThreads>(mine, s_warp);  // and the barrier behind the sums by CTA
    // every CTA gets what it lacks to an even share, in order, until all is given out
    const int64_t even = (tiles + ctas - 1) / ctas;
    if (tid < 32) {
        int64_t run = first_cut;
        for (int base = 0; base < ctas; base += 32) {
            const int c = base + tid;
            const int64_t want = c < ctas ? max(even - done[c], (int64_t)0) : 0;
            int64_t incl = want;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int64_t up = __shfl_up_sync(~0u, incl, o);
                if (tid >= o) incl += up;
            }
            const int64_t begin = min(run + incl - want, tiles), end = min(run + incl, tiles);
            if (c == (int)blockIdx.x) sh.begin = begin, sh.end = end;
            run += __shfl_sync(~0u, incl, 31);
        }
    }
    __syncthreads();
    // the sequence of this CTA's first tile
    const int64_t at = sh.begin;
    if (sh.end > at) {
        int64_t run = 0;
        for (int base = 0; base < S; base += kManyThreads) {
            const int i = base + tid;
            const int64_t n = i < S ? shape.kv_heads * head_tiles(shape, sequence(b, i, T)) : 0;
            int64_t incl = n;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int64_t up = __shfl_up_sync(~0u, incl, o);
                if (tid % 32 >= o) incl += up;
            }
            __syncthreads();
            if (tid % 32 == 31) s_warp[tid / 32] = incl;
            __syncthreads();
            int64_t before = run;
            for (int w = 0; w < kManyThreads / 32; ++w) {
                if (w < tid / 32) before += s_warp[w];
                run += s_warp[w];
            }
            const int64_t first = before + incl - n;
            if (at >= first && at < first + n) sh.begin_seq = i, sh.begin_off = at - first;
        }
        __syncthreads();
    }
    if (tid == 0) {
        Walk w{};
        if (sh.end > at) {
            w.open(shape, b, T, sh.begin_seq);
            w.seek(shape, sh.begin_off);
        }
        write_cut(shape, p.cuts, w, at, sh.end);
    }
    return rounds > 0 || sh.end > at;
}

// The parts of units in a CTA's share, one after the other: tiles [w.t, w.t + tiles) of w's unit.
struct Parts {
    Walk w;
    int32_t round = 0, tiles = 0, q_tiles, rows;  // rows of the unit, 1 .. 256
    bool from_start, to_end, opened = false;
    int64_t left;

    __device__ __forceinline__ Parts(const Share& sh) : left(sh.end - sh.begin) {}
    __device__ __forceinline__ bool next(const AttendParams& p, const Share& sh) {
        const Shape& shape = p.shape;
        if (round < sh.rounds) {
            const int u = blockIdx.x + round++ * gridDim.x;
            int lo = 0, hi = p.batch.num_seqs;  // first_unit[lo] <= u < first_unit[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (sh.first_unit[mid] <= u) lo = mid;
                else hi = mid;
            }
            w.open(shape, p.batch, p.cache.block_tokens, lo);
            w.to_unit(shape, u - sh.first_unit[lo]);
            tiles = w.range.tiles;
        } else {
            if (left == 0) return false;
            if (!opened) {
                opened = true;
                w.open(shape, p.batch, p.cache.block_tokens, sh.begin_seq);
                w.seek(shape, sh.begin_off);
            } else {
                w.t += tiles - 1;
                w.next(shape, p.batch, p.cache.block_tokens);
            }
            tiles = (int)min(left, (int64_t)(w.range.tiles - w.t));
            left -= tiles;
        }
        rows = min(kManyRows, w.seq.qn * shape.group - w.m * kManyRows);
        q_tiles = rows > 128 ? 2 : 1;
        from_start = w.t == 0;
        to_end = w.t + tiles == w.range.tiles;
        return true;
    }
};

// ---- loading
template <int D>
struct Loader : TileLoader<D, kLoadWarps> {
    using Base = TileLoader<D, kLoadWarps>;
    const AttendParams& p;
    const uint32_t smem;  // two query tiles, then the ring
    ManyBarriers& b;
    RingPlace at;
    static constexpr int kTile = ManyShape<D>::kTileBytes;

    __device__ __forceinline__ Loader(const AttendParams& p_, const CacheMaps& maps, int box_rows, uint32_t smem_, ManyBarriers& b_, int warp,
                                      int lane)
        : Base(p_.cache, maps, box_rows, warp, lane), p(p_), smem(smem_), b(b_) {}
    // Starts the loads of the tile's keys (kv = 0) or values (1).
    __device__ __forceinline__ bool tile(const Range& range, int key0, const typename Base::Group& group, int kv) {
        if (!__all_sync(~0u, mbar_wait_bounded(&b.empty[at.slot], at.phase, polls(p), &b.abort))) return false;
        Base::tokens(range.lo, range.hi, key0, group, kv, smem + (2 + at.slot) * kTile, &b.full[at.slot]);
        if (++at.slot == ManyShape<D>::kStages) at.slot = 0, at.phase ^= 1;
        return true;
    }
    __device__ __forceinline__ bool queries(const Parts& part, uint32_t q_phase) {
        if (!__all_sync(~0u, mbar_wait_bounded(&b.q_empty, q_phase, polls(p), &b.abort))) return false;
        for (int t = 0; t < part.q_tiles; ++t)
            Base::queries(p.q, part.w, p.shape.group, part.w.m * kManyRows + t * 128, min(128, part.rows - t * 128), smem + t * kTile);
        arrive_when_loaded(&b.q_full);
        return true;
    }
};

template <int D>
__device__ RingPlace load_loop(const AttendParams& p, const CacheMaps& maps, int box_rows, const Share& share, char* smem, ManyBarriers& b) {
    Loader<D> load(p, maps, box_rows, smem_u32(smem), b, (int)(threadIdx.x - kManyThreads + kLoadThreads) / 32, (int)threadIdx.x % 32);
    uint32_t q_phase = 1;
    bool ok = true;
    Parts part(share);
    while (ok && part.next(p, share)) {
        const Walk& w = part.w;
        load.open(w, p.batch);
        int key0 = w.range.base + w.t * kManyTile;
        auto at = load.groups(w.range.lo, w.range.hi, key0), next = load.groups(w.range.lo, w.range.hi, key0 + kManyTile);
        ok = load.queries(part, q_phase);
        q_phase ^= 1;
        for (int i = 0; ok && i < part.tiles; ++i, key0 += kManyTile) {
            ok = load.tile(w.range, key0, at, 0);
            if (ok) ok = load.tile(w.range, key0, at, 1);
            at = next;
            if (i + 2 < part.tiles) next = load.groups(w.range.lo, w.range.hi, key0 + 2 * kManyTile);
        }
    }
    cp_async_commit();
    cp_async_wait<0>();
    if (!ok) b.abort = 1, report(p.status, AMOEBA_ERR_TIMEOUT);
    return load.at;
}

// ---- products: one warp, one of its lanes issues
template <class T, int D>
__device__ bool multiply(const AttendParams& p, const Share& share, uint32_t smem, ManyBarriers& b) {
    constexpr int kTile = ManyShape<D>::kTileBytes, kStages = ManyShape<D>::kStages;
    constexpr uint32_t kS = product<T>(128, false), kO = product<T>(D, true);
    const uint32_t tmem = __shfl_sync(~0u, b.tmem, 0), leader = elect_one();
    int slot = 0;  // of the next K; V is the one behind
    uint32_t phase = 0, q_phase = 0, p_phase[2] = {0, 0}, o_phase[2] = {1, 1};
    auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(~0u, mbar_wait_bounded(bar, parity, polls(p), &b.abort)); };
    const uint64_t q_op = operand(smem, 16);
    auto logits = [&](int t, int k_slot) {
        const uint64_t k_op = operand(smem + (2 + __shfl_sync(~0u, k_slot, 0)) * kTile, 16);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            const uint32_t step = (k / 4 * (128 * 128) + k % 4 * 32) >> 4;
            umma_smem(leader, tmem + t * 128, q_op + (t * kTile >> 4) + step, k_op + step, kS, k > 0);
        }
    };
    auto weigh = [&](int t, int v_slot, int half, bool accumulate) {
        const uint64_t v_op = operand(smem + (2 + __shfl_sync(~0u, v_slot, 0)) * kTile, 128 * 128);
#pragma unroll
        for (int k = half * 4; k < half * 4 + 4; ++k)
            umma_tmem(leader, tmem + 256 + t * D, tmem + t * 128 + k * 8, v_op + (k * 2048 >> 4), kO, accumulate || k > 0);
    };
    Parts part(share);
    while (part.next(p, share)) {
        if (!wait(&b.q_full, q_phase)) return false;
        q_phase ^= 1;
        if (!wait(&b.full[slot], phase)) return false;
        fence_async_smem();
        tmem_fence_after();
        #pragma unroll
        for (int t = 0; t < 2; ++t) {
            if (t >= part.q_tiles) break;
            logits(t, slot);
            umma_commit(leader, &b.s_full[t]);
        }
        umma_commit(leader, &b.empty[slot]);
        if (part.tiles == 1) umma_commit(leader, &b.q_empty);
        for (int i = 0; i < part.tiles; ++i) {
            int v_slot = slot + 1, k_slot = slot + 2;
            uint32_t v_phase = phase, k_phase = phase;
            if (v_slot >= kStages) v_slot -= kStages, v_phase ^= 1;
            if (k_slot >= kStages) k_slot -= kStages, k_phase ^= 1;
            if (!wait(&b.full[v_slot], v_phase)) return false;
            fence_async_smem();
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                if (t >= part.q_tiles) break;
                if (i == 0) {
                    if (!wait(&b.o_free[t], o_phase[t])) return false;
                    o_phase[t] ^= 1;
                }
                // the first half of the weights is multiplied while the second is formed
                if (!wait(&b.p_half[t], p_phase[t])) return false;
                tmem_fence_after();
                weigh(t, v_slot, 0, i > 0);
                if (!wait(&b.p_full[t], p_phase[t])) return false;
                p_phase[t] ^= 1;
                tmem_fence_after();
                weigh(t, v_slot, 1, true);
                umma_commit(leader, &b.o_full[t]);
                if (i + 1 < part.tiles) {
                    if (t == 0) {
                        if (!wait(&b.full[k_slot], k_phase)) return false;
                        fence_async_smem();
                    }
                    logits(t, k_slot);
                    umma_commit(leader, &b.s_full[t]);
                }
            }
            umma_commit(leader, &b.empty[v_slot]);
            if (i + 1 < part.tiles) umma_commit(leader, &b.empty[k_slot]);
            if (i + 2 == part.tiles) umma_commit(leader, &b.q_empty);
            slot = k_slot, phase = k_phase;
        }
    }
    return true;
}
// Waits for what `multiply` has issued, also after it gave up.
__device__ __forceinline__ void drain_products(ManyBarriers& b) {
    umma_commit(elect_one(), &b.drain);
    mbar_drain(&b.drain, 0);
    __syncwarp();
}

// ---- softmax: a thread per row
// Hides the logits of tokens outside [lo, hi), and of bad blocks (table: null, or the unit has some), from the row: -infinity.
__device__ __noinline__ void hide(uint32_t s_tmem, int key0, int lo, int hi, const int32_t* table, int unit_hi, const CacheView& v) {
#pragma unroll 1
    for (int j = 0; j < 4; ++j) {
        const int first = key0 + j * 32, a = min(max(lo - first, 0), 32), b = min(max(hi - first, a), 32);
        uint32_t see = (uint32_t)((1ull << b) - (1ull << a));
        for (int k = 0; table && k < 32 && first + k < unit_hi; ++k) {
            const int block = table[(first + k) / v.block_tokens];
            if (block < 0 || block >= v.num_blocks) see &= ~(1u << k);
        }
        __syncwarp();
        uint32_t s[32];
        tmem_load32(s, s_tmem + j * 32);
        tmem_load_wait();
#pragma unroll
        for (int k = 0; k < 32; ++k)
            if (!(see & 1u << k)) s[k] = 0xff800000u;
        __syncwarp();
        tmem_store32(s_tmem + j * 32, s);
    }
    tmem_store_wait();
}
// The largest of the row's logits.  The row is read once more for the weights: kept, it would fill 128 registers.
__device__ __forceinline__ float row_max(uint32_t s_tmem) {
    uint32_t s[4][32];
    float top[4];
    tmem_load32(s[0], s_tmem);
    tmem_load32(s[1], s_tmem + 32);
    tmem_load_wait();
    tmem_load32(s[2], s_tmem + 64);
    tmem_load32(s[3], s_tmem + 96);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (j == 2) tmem_load_wait();
        top[j] = __uint_as_float(s[j][0]);
#pragma unroll
        for (int k = 1; k < 31; k += 2) top[j] = max3(top[j], __uint_as_float(s[j][k]), __uint_as_float(s[j][k + 1]));
        top[j] = fmaxf(top[j], __uint_as_float(s[j][31]));
    }
    return fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
}
// Writes the weights 2^(c * logit - ref) over the logits, in 16 bits, and returns their sum in 32; `half` gets
// this thread's arrival when the first 64 are there.
template <class T>
__device__ __forceinline__ float row_weights(uint32_t s_tmem, float c, float ref, uint64_t* half) {
    const uint64_t c2 = pair2(c, c), ref2 = pair2(-ref, -ref);
    uint64_t sum[2] = {0, 0};
    uint32_t s[2][32], w16[32];
    tmem_load32(s[0], s_tmem);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        tmem_load_wait();
        if (j < 3) tmem_load32(s[(j + 1) % 2], s_tmem + (j + 1) * 32);
#pragma unroll
        for (int k = 0; k < 32; k += 2) {
            float x, y;
            split2(fma2(pair2(__uint_as_float(s[j % 2][k]), __uint_as_float(s[j % 2][k + 1])), c2, ref2), x, y);
            x = fast_exp2(x), y = fast_exp2(y);
            sum[k / 2 % 2] = add2(sum[k / 2 % 2], pair2(x, y));
            w16[j % 2 * 16 + k / 2] = Elem<T>::pack(x, y);
        }
        if (j % 2) tmem_store32(s_tmem + j / 2 * 32, w16);  // over logits that have been read
        if (j == 1) {
            tmem_store_wait();
            tmem_fence_before();
            mbar_arrive(half);
        }
    }
    float a, b;
    split2(add2(sum[0], sum[1]), a, b);
    return a + b;
}

template <class T, int D>
__device__ bool softmax(const AttendParams& p, const Share& share, ManyBarriers& b) {
    const Shape& sh = p.shape;
    const int t = threadIdx.x / 128, r = threadIdx.x;  // row of the unit
    const uint32_t lanes = (uint32_t)(threadIdx.x % 128 / 32 * 32) << 16;
    const uint32_t s_tmem = b.tmem + lanes + t * 128, o_tmem = b.tmem + lanes + 256 + t * D;
    const float c = p.scale_log2;
    uint32_t s_phase = 0, o_phase = 0;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
        return __all_sync(~0u, mbar_wait_bounded(bar, parity, polls(p), &b.abort));  // and the warp is together again
    };
    bool ok = true;  // a warp that gives up goes on to the barriers below, where the others of its warpgroup wait for it
    Parts part(share);
    while (part.next(p, share)) {
        const Walk& w = part.w;
        // a bad block anywhere in the unit: its tokens are looked up one by one below
        const int32_t* table = p.batch.table + (int64_t)w.s * p.batch.max_blocks;
        int bad = 0;
        for (int i = w.range.lo / p.cache.block_tokens + (int)threadIdx.x % 128; i * (int64_t)p.cache.block_tokens < w.range.hi; i += 128)
            bad |= table[i] < 0 || table[i] >= p.cache.num_blocks;
        asm volatile(
            "{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %0, 0;\n\t"
            "barrier.cta.red.or.pred q, %1, 128, p;\n\tselp.s32 %0, 1, 0, q;\n\t}"
            : "+r"(bad) : "r"(1 + t) : "memory");
        if (bad && threadIdx.x % 128 == 0) report(p.status, AMOEBA_ERR_BAD_BLOCK_ID);
        if (ok && t < part.q_tiles) ok = [&] {
            const int row = w.m * kManyRows + r;
            const bool there = r < part.rows;
            const int pos = w.seq.len - w.seq.qn + row / sh.group;
            // (rows that are not there see zeros or anything: nothing is written for them)
            const int see_hi = there ? pos + 1 : INT32_MAX, see_lo = there && sh.window > 0 ? max(pos - sh.window + 1, 0) : 0;
            float m_ref = -INFINITY, l = 0.f;
            for (int i = 0; i < part.tiles; ++i) {
                const int key0 = w.range.base + (w.t + i) * kManyTile;
                if (!wait(&b.s_full[t], s_phase)) return false;
                s_phase ^= 1;
                tmem_fence_after();
                if (__any_sync(~0u, key0 + kManyTile > see_hi || key0 < see_lo) || bad)
                    hide(s_tmem, key0, see_lo, see_hi, bad ? table : nullptr, w.range.hi, p.cache);
                const float m = row_max(s_tmem) * c;
                const bool raise = m > m_ref + kRaise || (m_ref == -INFINITY && m > -INFINITY);
                if (__any_sync(~0u, raise)) {
                    const float m_new = raise ? m : m_ref;
                    const float f = raise ? fast_exp2(m_ref - m_new) : 1.f;
                    // (a row that has seen nothing yet has O = 0)
                    const bool scales = __any_sync(~0u, raise && m_ref > -INFINITY);
                    l *= f;
                    m_ref = m_new;
                    if (i > 0 && scales) {
                        if (!wait(&b.o_full[t], o_phase ^ 1)) return false;  // of the tile before
                        tmem_fence_after();
#pragma unroll
                        for (int j = 0; j < D / 32; ++j) {
                            uint32_t o[32];
                            tmem_load32(o, o_tmem + j * 32);
                            tmem_load_wait();
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                            tmem_store32(o_tmem + j * 32, o);
                        }
                    }
                }
                const float ref = m_ref == -INFINITY ? 0.f : m_ref;
                l += row_weights<T>(s_tmem, c, ref, &b.p_half[t]);
                tmem_store_wait();
                tmem_fence_before();
                mbar_arrive(&b.p_full[t]);
                o_phase ^= 1;
            }
            if (!wait(&b.o_full[t], o_phase ^ 1)) return false;
            tmem_fence_after();
            const bool direct = part.from_start && part.to_end;
            const float inv = l == 0.f ? 0.f : 1.f / l;
            const int64_t at = (int64_t)(2 * blockIdx.x + (part.from_start ? 1 : 0)) * kManyRows + r;
            char* out = there ? row_of<D>(p.out, p, w.seq, w.h, row) : nullptr;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                uint32_t o[32];
                __syncwarp();  // (rows that are not there have parted from the others)
                tmem_load32(o, o_tmem + j * 32);
                tmem_load_wait();
                if (!there) continue;
                if (direct) {
#pragma unroll
                    for (int k = 0; k < 32; k += 8) {
                        uint32_t x[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            x[i] = Elem<T>::pack(__uint_as_float(o[k + 2 * i]) * inv, __uint_as_float(o[k + 2 * i + 1]) * inv);
                        *reinterpret_cast<uint4*>(out + (j * 32 + k) * 2) = make_uint4(x[0], x[1], x[2], x[3]);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 32; k += 4)
                        *reinterpret_cast<uint4*>(p.part_o + at * D + j * 32 + k) = make_uint4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                }
            }
            tmem_fence_before();
            mbar_arrive(&b.o_free[t]);
            if (there && !direct) p.part_m[at] = m_ref, p.part_l[at] = l;
            if (there && direct && p.lse)
                *lse_of(p, w.seq, w.h, row) = l == 0.f ? -INFINITY : (m_ref + log2f(l)) * kLn2;
            return true;
        }();
        if (!ok) b.abort = 1;
    }
    return ok;
}

template <class T, int D>
__global__ void __launch_bounds__(kManyThreads, 1) attend_many(const __grid_constant__ AttendParams p, const __grid_constant__ CacheMaps maps,
                                                            int box_rows) {
    extern __shared__ char smem_raw[];
    __shared__ ManyBarriers b;
    char* smem = smem_raw + (1024 - smem_u32(smem_raw) % 1024) % 1024;
    const int warp = threadIdx.x / 32;
    __shared__ Share share;
    const bool busy = make_share(p, share, reinterpret_cast<int32_t*>(smem));
    grid_dependency_launch();
    if (!busy) {
        grid_dependency_wait();
        return;
    }
    __syncthreads();
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&b.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < ManyShape<D>::kStages; ++i) mbar_init(&b.full[i], kLoadThreads), mbar_init(&b.empty[i], 1);
        mbar_init(&b.q_full, kLoadThreads), mbar_init(&b.q_empty, 1), mbar_init(&b.drain, 1);
        for (int t = 0; t < 2; ++t)
            mbar_init(&b.s_full[t], 1), mbar_init(&b.p_half[t], 128), mbar_init(&b.p_full[t], 128), mbar_init(&b.o_full[t], 1), mbar_init(&b.o_free[t], 128);
        b.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    RingPlace loaded;
    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        if (warp == 8) {
            if (!multiply<T, D>(p, share, smem_u32(smem), b)) b.abort = 1, report(p.status, AMOEBA_ERR_TIMEOUT);
            __syncwarp();
            drain_products(b);
        } else {
            loaded = load_loop<D>(p, maps, box_rows, share, smem, b);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        if (!softmax<T, D>(p, share, b)) b.abort = 1, report(p.status, AMOEBA_ERR_TIMEOUT);
    }
    grid_dependency_wait();  // attend_few in front is done when this kernel is
    tmem_fence_before();
    __syncthreads();
    if (warp == 8) {
        tmem_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(b.tmem));
    }
    if (warp > 8 && b.abort) drain_ring<ManyShape<D>::kStages>(b.full, loaded);
}

template <class T, int D>
static amoeba_status launch(const AttendParams& p, const CacheMaps& maps, int box_rows, int ctas, cudaStream_t stream) {
    if (ensure_dynamic_smem((const void*)attend_many<T, D>, ManyShape<D>::kSmem) != cudaSuccess) return AMOEBA_ERR_CUDA;
    return launch_kernel(attend_many<T, D>, ctas, kManyThreads, ManyShape<D>::kSmem, stream, true, p, maps, box_rows);
}

amoeba_status launch_attend_many(const AttendParams& p, int tp, int32_t dtype, int head_dim, int ctas, cudaStream_t stream) {
    CacheMaps maps;
    const int rows = make_cache_maps(&maps, p.cache, tp, head_dim, dtype);
    if (dtype == AMOEBA_FP16)
        return head_dim == 64 ? launch<__half, 64>(p, maps, rows, ctas, stream) : launch<__half, 128>(p, maps, rows, ctas, stream);
    return head_dim == 64 ? launch<__nv_bfloat16, 64>(p, maps, rows, ctas, stream) : launch<__nv_bfloat16, 128>(p, maps, rows, ctas, stream);
}

}  // namespace amoeba
