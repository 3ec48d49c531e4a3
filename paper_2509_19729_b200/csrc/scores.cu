// amoeba_accumulate_scores: the attention weight that every cached token received, summed over the rows.
//
// exp(scale * q . k - lse) needs no running statistics, so a token's sum is finished by the warp that has read its key:
// every key is read once, the rows are walked in order for it, and no two warps add to the same score.  The exponent is formed as
// (scale * q . k - lse) * log2(e): logit and lse may be large and near each other, so only their difference is rounded.
#include "umma.cuh"

namespace amoeba {

struct ScoreParams {
    CacheView cache;
    Batch batch;
    Rows q;
    Shape shape;
    float* scores[AMOEBA_MAX_TP];  // worker pools, advanced to the layer: [block][header][token]
    const float* lse;
    const int32_t* scored;
    int32_t* status;
    float scale;
    int32_t q_heads, window;
#ifdef AMOEBA_CHECK_ITEMS
    int32_t polls;  // of every wait in score_many
#endif
};

// ------------------------------------------------------------------------------------------------ few rows
// Up to 8*NT rows a sequence.  Bound by the bytes of the keys.  A warp takes 16 tokens of every tile of 64; S^T = K Q^T as in
// attend.cu, so that a token's sum runs along the columns.  The loads of 16 tokens are half of attend_few's and the arithmetic
// on them nearly as long, so it takes many warps rather than deep rings: 5 CTAs an SM with two stages 93 us, 4 with three 98, 2
// with six 172 (64 sequences of 512 to 8192 tokens, 8 key heads of 128; now 98 us, 5.7 TB/s, 86 % of a copy's rate).
constexpr int kScoreThreads = 128, kScoreWarps = 4, kScoreTile = 16 * kScoreWarps;
template <int D, int NT>
struct ScoreShape {
    static constexpr int kStage = 16 * D * 2, kStages = NT == 4 ? 4 : 2, kCtas = NT == 1 ? 5 : NT == 2 ? 3 : 2;  // CTAs per SM
    static constexpr int kSmem = kScoreWarps * kStages * kStage;
    // Partial sums of a logit: the matrix instructions cut what they add to a sum instead of rounding it, and a weight is off by as
    // much as its logit.  With one sum the scores of a step are 1.0e-6 off (relative, against 64 bits), with two 0.63e-6, with four
    // 0.45e-6, for which registers are left with up to eight rows.
    static constexpr int kSums = NT == 1 ? 4 : 2;
};

template <class T, int D, int NT>
__global__ void __launch_bounds__(kScoreThreads, ScoreShape<D, NT>::kCtas) score_few(const __grid_constant__ ScoreParams p) {
    using F = ScoreShape<D, NT>;
    constexpr int kSteps = D / 16;
    extern __shared__ __align__(128) char smem[];
    __shared__ uint32_t s_mask[kScoreWarps][F::kStages];
    __shared__ int64_t s_slot[kScoreWarps][F::kStages];  // of the 16 tokens' first score, where they lie in one block
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, quad = lane / 4, pair = lane % 4;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * F::kStages * F::kStage;
    const Shape& sh = p.shape;
    const int bt = p.cache.block_tokens;
    const bool one_block = bt % 16 == 0;
    Walk walk;
    int64_t begin, end;
    take_share<kScoreThreads>(sh, p.batch, bt, &walk, &begin, &end, p.status);
    int64_t n = end - begin;
    grid_dependency_launch();
    if (n == 0) return;

    Ahead<D, false, kScoreTile> ahead(p.cache, p.batch, sh, p.status, walk, n, warp * 16);
    int slot_in = 0, slot = 0;
    auto load = [&] {
        if (ahead.left > 0) {
            int64_t first;
            const uint32_t mask = ahead.load(ring + slot_in * F::kStage, &first);
            if (lane == 0) s_mask[warp][slot_in] = mask, s_slot[warp][slot_in] = first;
        }
        cp_async_commit();
        slot_in = slot_in + 1 == F::kStages ? 0 : slot_in + 1;
    };
#pragma unroll
    for (int i = 0; i < F::kStages - 1; ++i) load();

    uint32_t qf[NT][kSteps][2];
    int see_lo[NT][2], see_hi[NT][2];
    float lse[NT][2];
    int scored = 0, rows = 0;
    float* scores = nullptr;
    bool fresh = true;
    for (; n > 0; --n) {
        if (fresh) {
            fresh = false;
            const Seq& q = walk.seq;
            const int g = sh.group, w = walk.h / p.cache.heads, h = walk.h - w * p.cache.heads;
            rows = q.qn * g;
            scores = p.scores[w];
            scored = p.scored ? p.scored[walk.s] : 0;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int r = t * 8 + quad, tok = r / g;
                const char* src = p.q.base[w] + (int64_t)(q.q0 + tok) * p.q.stride + (h * g + r - tok * g) * (D * 2);
#pragma unroll
                for (int j = 0; j < kSteps; ++j)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        qf[t][j][i] = r < rows ? *reinterpret_cast<const uint32_t*>(src + (j * 16 + i * 8 + pair * 2) * 2) : 0u;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int rr = t * 8 + pair * 2 + b, token = rr / g, pos = q.len - q.qn + token;
                    const float x = rr < rows ? p.lse[(int64_t)(q.q0 + token) * p.q_heads + walk.h * g + rr - token * g] : -INFINITY;
                    lse[t][b] = x;
                    see_hi[t][b] = x == -INFINITY ? 0 : pos + 1;  // a row that saw nothing adds nothing
                    see_lo[t][b] = p.window > 0 ? pos - p.window + 1 : 0;
                }
            }
        }
        cp_async_wait<F::kStages - 2>();
        __syncwarp();
        const uint32_t k_smem = ring + slot * F::kStage, mask = s_mask[warp][slot];
        const int64_t first = s_slot[warp][slot];
        load();  // into the slot that the last round has read
        __syncwarp();  // the matrix instructions want the warp together
        slot = slot + 1 == F::kStages ? 0 : slot + 1;
        const int key0 = walk.t * kScoreTile + warp * 16 + quad;
        float sum[2] = {0.f, 0.f};
        if (mask) {
            float st[F::kSums][NT][4];
#pragma unroll
            for (int t = 0; t < F::kSums * NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) st[t / NT][t % NT][i] = 0.f;
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
                uint32_t a[4];
                ldmatrix4(a, k_smem + swizzled<D>(lane % 16, 2 * j + lane / 16));
#pragma unroll
                for (int t = 0; t < NT; ++t) mma16816<T>(st[j % F::kSums][t], a, qf[t][j][0], qf[t][j][1]);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = key0 + i / 2 * 8;
                    float logit = st[0][t][i] + st[1][t][i];
                    if (F::kSums == 4) logit += st[2 % F::kSums][t][i] + st[3 % F::kSums][t][i];
                    if (key < see_hi[t][i % 2] && key >= see_lo[t][i % 2])
                        sum[i / 2] += fast_exp2(fmaf(logit, p.scale, -lse[t][i % 2]) * kLog2e);
                }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            sum[i] += __shfl_xor_sync(~0u, sum[i], 1);
            sum[i] += __shfl_xor_sync(~0u, sum[i], 2);
            if (pair == i && (mask >> (quad + i * 8) & 1u)) {
                const int key = key0 + i * 8;
                int64_t at = first + quad + i * 8;
                if (!one_block) {
                    const int block = p.batch.table[(int64_t)walk.s * p.batch.max_blocks + key / bt];
                    at = ((int64_t)block * p.cache.heads + walk.h % p.cache.heads) * bt + key % bt;
                }
                float* to = scores + at;
                *to = (key < scored ? *to : 0.f) + sum[i];
            }
        }
        if (n > 1) {
            const int h = walk.h, s = walk.s;
            walk.next(sh, p.batch, bt);
            fresh = walk.h != h || walk.s != s;
        }
    }
}

// ------------------------------------------------------------------------------------------------ many rows
// The products on the fifth-generation tensor cores, 128 tokens by 128 query rows: S^T = K Q^T, so that a thread has a token
// and sums along its own columns.  A CTA keeps 128 rows in shared memory and runs through its tokens, 128 at a time, then the
// next 128 rows of the same sequence and head, then its next head; the tokens of a head are dealt out to CTAs in tiles, all
// rows with them, so a score has one thread.  Four warpgroups take the tiles in turn, each with its own logits in tensor
// memory, so that the products run ahead.  Six prompts of 4 to 32 thousand tokens, 32 queries of each, 32 query heads on 8 key
// heads of 128: 81 us; without the loads it would take about 60 (a tile's 16384 exponentials are 1024 of the 2 thousand clocks that
// it takes), without the sums as much (the keys at a copy's rate, and about 12 us to start, to share the work out and to end).
// A logit is one sum of D / 16 instructions, each of which cuts it (ScoreShape::kSums): the scores are 7.6e-7 off, against 3.5e-7
// in plain torch.  All 512 columns of tensor memory hold logits, so there is no room for second sums.
constexpr int kScoreGroups = 4, kScoreManyThreads = 128 * (kScoreGroups + 1), kScoreLoadWarps = 3;
template <int D>
struct ScoreManyShape {
    static constexpr int kTileBytes = 128 * D * 2, kStages = D == 128 ? 4 : 8;
    static constexpr int kSmem = (2 + kStages) * kTileBytes + 1024;
};
struct ScoreBarriers {
    uint64_t k_full[8], k_empty[8], q_full[2], q_empty[2], s_full[kScoreGroups], s_empty[kScoreGroups], drain;
    uint32_t tmem;
    int32_t abort;
};

__device__ __forceinline__ int score_passes(const Shape& sh, const Seq& q) {  // of 128 rows
    const int n = q.qn * sh.group;
    return n < sh.min_rows ? 0 : (n + 127) / 128;
}
// Tiles times passes of one head: what it costs.
__device__ __forceinline__ int64_t score_cost(const Shape& sh, const Seq& q) {
    return (int64_t)((q.len + 127) / 128) * score_passes(sh, q);
}

// The runs of tiles [t0, t1) of heads that a CTA has: its share of the cost, each end moved up to a whole tile.
struct Runs {
    Walk w;
    int32_t t0, t1, passes, rows;
    int64_t off, left;  // cost in front of this CTA in its sequence, and what is left of its share
    bool opened = false;

    __device__ __forceinline__ bool next(const ScoreParams& p) {
        const Shape& sh = p.shape;
        while (left > 0) {
            if (opened) {
                ++w.h, off = 0;
                if (w.h == sh.kv_heads) {
                    do w.open(sh, p.batch, p.cache.block_tokens, w.s + 1);
                    while (score_cost(sh, w.seq) == 0);
                }
            }
            const int64_t cost = score_cost(sh, w.seq);
            if (!opened) w.h = (int)(off / cost), off %= cost;
            opened = true;
            passes = score_passes(sh, w.seq);
            rows = w.seq.qn * sh.group;
            const int64_t stop = min(cost, off + left);
            t0 = (int)((off + passes - 1) / passes), t1 = (int)((stop + passes - 1) / passes);
            left -= stop - off;
            if (t0 < t1) return true;
        }
        return false;
    }
};

__device__ void take_runs(const ScoreParams& p, Runs* r, int32_t* status) {
    __shared__ int64_t s_warp[kScoreManyThreads / 32], s_off;
    __shared__ int32_t s_seq;
    const Shape& sh = p.shape;
    const int tid = threadIdx.x, S = p.batch.num_seqs, T = p.cache.block_tokens;
    int64_t sum = 0;
    for (int s = tid; s < S; s += kScoreManyThreads) sum += sh.kv_heads * score_cost(sh, sequence(p.batch, s, T));
    const int64_t all = block_sum<kScoreManyThreads>(sum, s_warp);
    const int64_t begin = share_begin(all, gridDim.x, blockIdx.x), end = share_begin(all, gridDim.x, blockIdx.x + 1);
    int64_t run = 0;
    for (int base = 0; base < S && run <= begin; base += kScoreManyThreads) {
        const int s = base + tid;
        const int64_t mine = s < S ? sh.kv_heads * score_cost(sh, sequence(p.batch, s, T)) : 0;
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
        for (int w = 0; w < kScoreManyThreads / 32; ++w) {
            if (w < tid / 32) before += s_warp[w];
            run += s_warp[w];
        }
        const int64_t first = before + incl - mine;
        if (begin >= first && begin < first + mine) s_seq = s, s_off = begin - first;
    }
    __syncthreads();
    r->left = end - begin;
    if (r->left > 0) {
        r->w.open(sh, p.batch, T, s_seq);
        r->off = s_off;
    }
}

template <int D>
__device__ bool score_load(const ScoreParams& p, const CacheMaps& maps, int box_rows, uint32_t smem, ScoreBarriers& b, Runs run,
                           RingPlace* loaded) {
    using S = ScoreManyShape<D>;
    TileLoader<D, kScoreLoadWarps> load(p.cache, maps, box_rows, (int)(threadIdx.x - (kScoreManyThreads - 32 * kScoreLoadWarps)) / 32,
                                         threadIdx.x % 32);
    auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(~0u, mbar_wait_bounded(bar, parity, polls(p), &b.abort)); };
    RingPlace ring;
    int qb = 0;
    uint32_t q_phase = 1;
    bool ok = true;
    while (ok && run.next(p)) {
        load.open(run.w, p.batch);
        const int len = run.w.seq.len;
        for (int j = 0; ok && j < run.passes; ++j) {
            if (!(ok = wait(&b.q_empty[qb], q_phase))) break;
            load.template queries<true>(p.q, run.w, p.shape.group, j * 128, min(128, run.rows - j * 128), smem + qb * S::kTileBytes);
            arrive_when_loaded(&b.q_full[qb]);
            if (qb ^= 1, qb == 0) q_phase ^= 1;
            auto at = load.groups(0, len, run.t0 * 128), next = load.groups(0, len, run.t0 * 128 + 128);
            for (int t = run.t0; t < run.t1; ++t) {
                if (!(ok = wait(&b.k_empty[ring.slot], ring.phase))) break;
                load.tokens(0, len, t * 128, at, 0, smem + (2 + ring.slot) * S::kTileBytes, &b.k_full[ring.slot]);
                if (++ring.slot == S::kStages) ring.slot = 0, ring.phase ^= 1;
                at = next;
                if (t + 2 < run.t1) next = load.groups(0, len, (t + 2) * 128);
            }
        }
    }
    cp_async_commit();
    cp_async_wait<0>();
    *loaded = ring;
    return ok;
}

template <class T, int D>
__device__ bool score_multiply(const ScoreParams& p, uint32_t smem, ScoreBarriers& b, Runs run) {
    using S = ScoreManyShape<D>;
    constexpr uint32_t kIdesc = product<T>(128, false);
    const uint32_t tmem = __shfl_sync(~0u, b.tmem, 0), leader = elect_one();
    auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(~0u, mbar_wait_bounded(bar, parity, polls(p), &b.abort)); };
    int slot = 0, qb = 0;
    uint32_t phase = 0, q_phase = 0, free = (1u << kScoreGroups) - 1;  // bit g: parity to wait for at s_empty[g]
    while (run.next(p)) {
        for (int j = 0; j < run.passes; ++j) {
            if (!wait(&b.q_full[qb], q_phase)) return false;
            for (int i = 0; i < run.t1 - run.t0; ++i) {
                const int g = i % kScoreGroups;
                if (!wait(&b.k_full[slot], phase)) return false;
                if (!wait(&b.s_empty[g], free >> g & 1)) return false;
                free ^= 1u << g;
                fence_async_smem();
                tmem_fence_after();
                const uint64_t k_op = operand(smem + (2 + __shfl_sync(~0u, slot, 0)) * S::kTileBytes, 16);
                const uint64_t q_op = operand(smem + __shfl_sync(~0u, qb, 0) * S::kTileBytes, 16);
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint32_t step = (k / 4 * (128 * 128) + k % 4 * 32) >> 4;
                    umma_smem(leader, tmem + __shfl_sync(~0u, g, 0) * 128, k_op + step, q_op + step, kIdesc, k > 0);
                }
                umma_commit(leader, &b.s_full[g]);
                umma_commit(leader, &b.k_empty[slot]);
                if (++slot == S::kStages) slot = 0, phase ^= 1;
            }
            umma_commit(leader, &b.q_empty[qb]);
            if (qb ^= 1, qb == 0) q_phase ^= 1;
        }
    }
    return true;
}

// Sum over the 128 rows of e^(c * logit + row) for one token; kCut: of those rows that see it.  `empty` gets this thread's
// arrival when the logits are read.
template <bool kCut>
__device__ __forceinline__ float column_sum(uint32_t from, const float (&row)[128], const int32_t (&pos)[128], int key, int window, float c,
                                            uint64_t* empty) {
    const uint64_t c2 = pair2(c, c), e2 = pair2(kLog2e, kLog2e);
    uint64_t sum[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t s[32];
        if (kCut) __syncwarp();
        tmem_load32(s, from + i * 32);
        tmem_load_wait();
        if (i == 3) {
            tmem_fence_before();
            mbar_arrive(empty);
        }
#pragma unroll
        for (int k = 0; k < 32; k += 4) {
            const float4 r = *reinterpret_cast<const float4*>(&row[i * 32 + k]);
            float x[4];
            split2(mul2(fma2(pair2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), c2, pair2(r.x, r.y)), e2), x[0], x[1]);
            split2(mul2(fma2(pair2(__uint_as_float(s[k + 2]), __uint_as_float(s[k + 3])), c2, pair2(r.z, r.w)), e2), x[2], x[3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = fast_exp2(x[e]);
            if (kCut) {
                const int4 at = *reinterpret_cast<const int4*>(&pos[i * 32 + k]);
                const int seen[4] = {at.x, at.y, at.z, at.w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (key > seen[e] || (window > 0 && key <= seen[e] - window)) x[e] = 0.f;
            }
            sum[0] = add2(sum[0], pair2(x[0], x[1]));
            sum[1] = add2(sum[1], pair2(x[2], x[3]));
        }
    }
    float lo, hi;
    split2(add2(sum[0], sum[1]), lo, hi);
    return lo + hi;
}

// s_row: [2][128] of this warpgroup, -lse of the pass's rows; s_pos: their cache indices.  A pass has rows that add nothing:
// those behind its last row, which repeat that one (their logits are infinite or NaN only where its own are), and those with
// lse -infinity, whose queries may be anything, so that with one of them all tiles are summed with a look at who sees them.
__device__ bool score_sum(const ScoreParams& p, ScoreBarriers& b, Runs run, float (*s_row)[128], int32_t (*s_pos)[128]) {
    const int g = threadIdx.x / 128, tid = threadIdx.x % 128, G = p.shape.group, T = p.cache.block_tokens;
    const uint32_t lanes = (uint32_t)(tid / 32 * 32) << 16;
    auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(~0u, mbar_wait_bounded(bar, parity, polls(p), &b.abort)); };
    const float c = p.scale;
    int pass = 0;
    uint32_t full = 0;  // parity to wait for at s_full[g]
    bool ok = true;     // a warp that gives up goes on to the barriers below, where the others of its warpgroup wait for it
    while (run.next(p)) {
        const Seq& q = run.w.seq;
        const int w = run.w.h / p.cache.heads, hw = run.w.h - w * p.cache.heads;
        const int32_t* table = p.batch.table + (int64_t)run.w.s * p.batch.max_blocks;
        const int scored = p.scored ? p.scored[run.w.s] : 0;
        float* scores = p.scores[w];
        for (int j = 0; j < run.passes; ++j, pass ^= 1) {
            const int row = j * 128 + tid, tok = row / G;
            float lse = -INFINITY;
            int pos = -1;
            if (row < run.rows) {
                lse = p.lse[(int64_t)(q.q0 + tok) * p.q_heads + run.w.h * G + row - tok * G];
                pos = q.len - q.qn + tok;
            }
            int mute = row < run.rows && lse == -INFINITY;
            s_row[pass][tid] = lse == -INFINITY ? -INFINITY : -lse;
            s_pos[pass][tid] = mute ? -1 : pos;
            asm volatile(
                "{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %0, 0;\n\t"
                "barrier.cta.red.or.pred q, %1, 128, p;\n\tselp.s32 %0, 1, 0, q;\n\t}"
                : "+r"(mute) : "r"(1 + g) : "memory");
            // what the pass's first row and its last one see, if they are there
            const int first_pos = q.len - q.qn + j * 128 / G;
            const int last_pos = q.len - q.qn + (min(run.rows, j * 128 + 128) - 1) / G;
            // the block of the next tile's token is asked for a tile early
            int at = (run.t0 + g) * 128 + tid, i_block = at / T, in_block = at - i_block * T, block = -1;
            if (run.t0 + g < run.t1 && at < q.len) block = table[i_block];
            for (int t = run.t0 + g; ok && t < run.t1; t += kScoreGroups, full ^= 1) {
                const int key0 = t * 128, key = key0 + tid;
                float* to = nullptr;
                float old = 0.f;
                if (key < q.len) {
                    if (block >= 0 && block < p.cache.num_blocks) {
                        to = scores + ((int64_t)block * p.cache.heads + hw) * T + in_block;
                        if (j > 0 || key < scored) old = *to;
                    } else {
                        report(p.status, AMOEBA_ERR_BAD_BLOCK_ID);
                    }
                }
                at = key + 128 * kScoreGroups;
                if (t + kScoreGroups < run.t1 && at < q.len) {
                    i_block = at / T, in_block = at - i_block * T;
                    block = table[i_block];
                }
                const bool cut = mute || key0 + 127 > first_pos || (p.window > 0 && key0 <= last_pos - p.window);
                if (!wait(&b.s_full[g], full)) {
                    ok = false, b.abort = 1;
                    break;
                }
                tmem_fence_after();
                const uint32_t from = b.tmem + lanes + g * 128;
                const float sum = cut ? column_sum<true>(from, s_row[pass], s_pos[pass], key, p.window, c, &b.s_empty[g])
                                      : column_sum<false>(from, s_row[pass], s_pos[pass], key, p.window, c, &b.s_empty[g]);
                if (to) *to = old + sum;
            }
        }
    }
    return ok;
}

template <class T, int D>
__global__ void __launch_bounds__(kScoreManyThreads, 1) score_many(const __grid_constant__ ScoreParams p, const __grid_constant__ CacheMaps maps,
                                                                int box_rows) {
    extern __shared__ char smem_raw[];
    __shared__ ScoreBarriers b;
    __shared__ __align__(16) float s_row[kScoreGroups][2][128];
    __shared__ __align__(16) int32_t s_pos[kScoreGroups][2][128];
    using S = ScoreManyShape<D>;
    char* smem = smem_raw + (1024 - smem_u32(smem_raw) % 1024) % 1024;
    const int warp = threadIdx.x / 32;
    Runs run;
    take_runs(p, &run, p.status);
    if (run.left == 0) {
        grid_dependency_wait();
        return;
    }
    if (warp == 4 * kScoreGroups) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&b.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) mbar_init(&b.k_full[i], 32 * kScoreLoadWarps), mbar_init(&b.k_empty[i], 1);
        for (int i = 0; i < 2; ++i) mbar_init(&b.q_full[i], 32 * kScoreLoadWarps), mbar_init(&b.q_empty[i], 1);
        for (int i = 0; i < kScoreGroups; ++i) mbar_init(&b.s_full[i], 1), mbar_init(&b.s_empty[i], 128);
        mbar_init(&b.drain, 1);
        b.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    bool ok;
    RingPlace loaded;
    if (warp < 4 * kScoreGroups) {
        ok = score_sum(p, b, run, s_row[warp / 4], s_pos[warp / 4]);
    } else if (warp == 4 * kScoreGroups) {
        ok = score_multiply<T, D>(p, smem_u32(smem), b, run);
        __syncwarp();
        umma_commit(elect_one(), &b.drain);
        mbar_drain(&b.drain, 0);
    } else {
        ok = score_load<D>(p, maps, box_rows, smem_u32(smem), b, run, &loaded);
    }
    if (!ok) b.abort = 1, report(p.status, AMOEBA_ERR_TIMEOUT);
    grid_dependency_wait();  // score_few in front is done when this kernel is
    tmem_fence_before();
    __syncthreads();
    if (warp == 4 * kScoreGroups) {
        tmem_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(b.tmem));
    }
    if (warp > 4 * kScoreGroups && b.abort) drain_ring<S::kStages>(b.k_full, loaded);
}

template <class T, int D, int NT>
static amoeba_status run_score_few(const ScoreParams& p, int sms, cudaStream_t stream) {
    using F = ScoreShape<D, NT>;
    if (ensure_dynamic_smem((const void*)score_few<T, D, NT>, F::kSmem) != cudaSuccess) return AMOEBA_ERR_CUDA;
    return launch_kernel(score_few<T, D, NT>, F::kCtas * sms, kScoreThreads, F::kSmem, stream, false, p);
}

// As in attend.cu: few rows, or none, by the kernel that only reads; more by the tensor cores'.
template <class T, int D>
static amoeba_status run_scores(ScoreParams& p, const amoeba_layout* layout, int32_t dtype, int sms, cudaStream_t stream) {
    const int64_t rows = (int64_t)p.batch.max_q_len * p.shape.group, few_rows = rows <= 32 ? rows : p.shape.group;
    const int most = few_rows <= 8 ? 8 : few_rows <= 16 ? 16 : 32;
    p.shape.max_rows = most;
    const amoeba_status st = most == 8    ? run_score_few<T, D, 1>(p, sms, stream)
                             : most == 16 ? run_score_few<T, D, 2>(p, sms, stream)
                                          : run_score_few<T, D, 4>(p, sms, stream);
    if (st != AMOEBA_OK || rows <= 32) return st;
    p.shape.min_rows = most + 1;
    if (ensure_dynamic_smem((const void*)score_many<T, D>, ScoreManyShape<D>::kSmem) != cudaSuccess) return AMOEBA_ERR_CUDA;
    CacheMaps maps;
    const int box_rows = make_cache_maps(&maps, p.cache, layout->tp, D, dtype);
    return launch_kernel(score_many<T, D>, sms, kScoreManyThreads, ScoreManyShape<D>::kSmem, stream, true, p, maps, box_rows);
}

}  // namespace amoeba

using namespace amoeba;

extern "C" amoeba_status amoeba_accumulate_scores(const amoeba_layout* layout, int32_t dtype, int32_t layer,
                                                  const void* const* pools, const amoeba_batch* batch,
                                                  const void* const* q, int64_t q_stride, float scale, int32_t window,
                                                  const float* d_lse, const int32_t* d_scored_lens,
                                                  float* const* score_pools, int32_t* d_status, void* cuda_stream) {
    ScoreParams p{};
    amoeba_status st;
    if ((st = check_elements(layout, dtype)) != AMOEBA_OK) return st;
    if ((st = make_cache_view(layout, layer, pools, &p.cache)) != AMOEBA_OK) return st;
    if ((st = make_batch(batch, &p.batch)) != AMOEBA_OK) return st;
    if (!d_status || (!d_lse && p.batch.num_rows) || !score_pools || window < 0 || !positive(scale)) return AMOEBA_ERR_INVALID_ARG;
    const amoeba_model& m = layout->model;
    if ((st = make_rows(layout, p.batch, q, q_stride, (int64_t)m.num_q_heads / layout->tp * m.head_dim, &p.q)) != AMOEBA_OK)
        return st;
    const int64_t layer_scores = (int64_t)layout->num_blocks * p.cache.heads * layout->block_tokens;
    for (int r = 0; r < layout->tp; ++r) {
        if (!score_pools[r]) return AMOEBA_ERR_INVALID_ARG;
        if ((uintptr_t)score_pools[r] % 16) return AMOEBA_ERR_ALIGNMENT;
        p.scores[r] = score_pools[r] + layer * layer_scores;
    }
    if (p.batch.num_seqs == 0) return AMOEBA_OK;
    p.lse = d_lse;
    p.scored = d_scored_lens;
    p.status = d_status;
#ifdef AMOEBA_CHECK_ITEMS
    p.polls = operator_wait_polls();
#endif
    p.scale = scale;
    p.q_heads = m.num_q_heads;
    p.shape.group = m.num_q_heads / m.num_kv_heads;
    p.shape.kv_heads = m.num_kv_heads;
    p.shape.rows = INT32_MAX;  // all rows of a sequence in one unit, whose tiles run over the whole sequence
    p.shape.tile = kScoreTile;
    p.shape.rowless = 1;
    if (((int64_t)p.batch.max_q_len + 128) * p.shape.group > INT32_MAX) return AMOEBA_ERR_UNSUPPORTED;
    const DeviceInfo dev = cached_device_info();
    if (!dev.sms) return AMOEBA_ERR_CUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    p.window = std::min(window, 1 << 30);  // not the shape's: every token gets a value, zero if no row sees it
    if (dtype == AMOEBA_FP16)
        return m.head_dim == 64 ? run_scores<__half, 64>(p, layout, dtype, dev.sms, stream) : run_scores<__half, 128>(p, layout, dtype, dev.sms, stream);
    return m.head_dim == 64 ? run_scores<__nv_bfloat16, 64>(p, layout, dtype, dev.sms, stream)
                            : run_scores<__nv_bfloat16, 128>(p, layout, dtype, dev.sms, stream);
}
