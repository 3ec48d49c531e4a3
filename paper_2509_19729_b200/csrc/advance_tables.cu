// amoeba_advance_tables: block tables, block counts, rows, positions and slots of a step, from the sequences' lengths.
//
// One launch of one cluster.  With n = ceil(length / block_tokens) blocks before and after,
//   blocks(s) = what a growing or forked sequence lacks,  rows(s) = its new tokens,  copies(s) = 1 if its first new block is a copy,
// and their sums over the sequences in front of s, the r-th free id overall (ascending) goes to the sequence with
// blocks[s] <= r < blocks[s + 1], as its entry r - blocks[s] of the new ones, and who hands it out knows the rows and slots of the tokens
// that it holds.  So nothing has to be read back from the table.  The sums every CTA makes for itself; the pool's counts are dealt
// to the CTAs in tiles of 1024, whose free blocks are exchanged once.
//
// What bounds it is latency: a launch, the dependent loads of a look at a sequence's last block, one or two barriers of the
// cluster, a search for every block.  The counts (4 bytes a block) are read once.  Measured, a step and the way back: 8 sequences 9.3 us,
// 128 in 36 500 blocks 15, 256 with prompts of 50 000 tokens and 60 forks 27, 1024 in 750 000 blocks 36.  (A warp to a sequence's
// entries and the blocks dealt by warps took 20, 85, 188 and 651.)
#include "cache_view.cuh"
#include "cluster.cuh"

namespace amoeba {

struct StepParams {
    int32_t *table, *refs;
    const int32_t *lens, *new_lens, *parents, *shared, *first_pos;
    int32_t *lens_out, *starts, *positions, *num_pairs, *free_count, *status;
    int64_t* slots;
    int2* pairs;
    int32_t num_seqs, max_blocks, num_rows, pairs_cap, num_blocks, block_tokens;
    int32_t shift;          // block_tokens = 2^shift, or -1
    int32_t max_len;        // tokens that a row of the table has room for
    int32_t tiles;          // in the pool (large launches)
    int32_t words;          // of 32 blocks, of a CTA (others)

    __device__ __forceinline__ int whole(int tokens) const { return shift >= 0 ? tokens >> shift : tokens / block_tokens; }
    __device__ __forceinline__ int blocks_of(int tokens) const { return whole(tokens + block_tokens - 1); }
    __device__ __forceinline__ bool inside(int b) const { return b >= 0 && b < num_blocks; }
};

constexpr int kStepMost = 1024;    // threads
constexpr int kStepCluster = 16;   // CTAs
constexpr uint32_t kBadArg = 1, kBadBlock = 2;

// In dynamic shared memory: sums over the sequences in front of every one, and at [num_seqs] over all; then what the CTA knows of
// its part of the pool.  In large launches that is every size-th tile, which has a word of 32 blocks for each warp, so that all CTAs have
// blocks to hand out; in others a run of words, no more than there are threads.
struct StepShared {
    int32_t* sums[4];   // blocks, rows, copies; entries of the table that are shared with a parent's or given back
    int32_t* first;     // cache index of the first new token; -1: refused
    uint32_t* free;     // the free blocks' bits, by words
    int32_t* before;    // free blocks in front of a word, of its tile or of the CTA
    int32_t* count;     // of a tile: free blocks in it,
    int32_t* start;     // and in all tiles of the pool in front of it

    __device__ __forceinline__ StepShared(char* smem, const StepParams& p, int words, int tiles) {
        const int n = p.num_seqs + 1;
        sums[0] = reinterpret_cast<int32_t*>(smem);
        sums[1] = sums[0] + n, sums[2] = sums[1] + n, sums[3] = sums[2] + n, first = sums[3] + n;
        free = reinterpret_cast<uint32_t*>(first + n);
        before = reinterpret_cast<int32_t*>(free + words);
        count = before + words, start = count + tiles;
    }
};
static int64_t step_smem(int64_t num_seqs, int64_t words, int64_t tiles) { return (5 * (num_seqs + 1) + 2 * words + 2 * tiles) * 4; }
constexpr int kStepStatic = 26 * 1024;  // bytes of shared memory beside those

// What a sequence asks for.  The loads come in three steps, so that others can be started in between.
struct Need {
    int32_t blocks = 0, rows = 0, copies = 0, entries = 0, first = -1;
};
struct Ask {
    int32_t old = 0, now = 0, parent = -1, share = 0, from = 0, last = -1, count = 0;
    bool ok = false;

    __device__ __forceinline__ void lengths(const StepParams& p, int s) {
        old = p.lens[s], now = p.new_lens[s];
        if (p.parents) parent = p.parents[s];
        ok = old >= 0 && old <= p.max_len && now >= 0 && now <= p.max_len && parent < p.num_seqs;
    }
    __device__ __forceinline__ void more(const StepParams& p, int s) {
        if (!ok) return;
        if (parent >= 0) share = p.shared[s], from = p.lens[parent];
        else if (now > old && p.whole(old) * p.block_tokens != old) last = p.table[(int64_t)s * p.max_blocks + p.whole(old)];
    }
    __device__ __forceinline__ void counts(const StepParams& p) {
        if (p.inside(last)) count = p.refs[last];
    }
    __device__ __forceinline__ Need need(const StepParams& p, uint32_t* bad) const {
        Need n;
        if (!ok || (parent >= 0 && (old != 0 || from > p.max_len || share < 0 || share > from || share > now))) {
            *bad |= kBadArg;
            return n;
        }
        n.first = parent >= 0 ? share : old;
        if (now < old) {
            n.entries = p.blocks_of(old) - p.blocks_of(now);
            return n;
        }
        int have = p.whole(n.first);
        if (parent >= 0) n.entries = have;
        if (have * p.block_tokens != n.first) {
            // The last block is not full: a fork gets a copy of its parent's, and a sequence one of a block that others name too.
            n.copies = parent >= 0;
            if (parent < 0 && now > old) {
                if (count < 1) *bad |= kBadBlock;
                n.copies = count > 1;
            }
            if (!n.copies) ++have;
        }
        n.blocks = max(p.blocks_of(now) - have, 0);
        n.rows = p.starts ? now - n.first : 0;
        return n;
    }
};

// The last s in [0, n) with before[s] <= at; before[0] = 0.
__device__ __forceinline__ int last_at_most(const int32_t* before, int n, int at) {
    int lo = 0;
    while (n > 1) {
        const int half = n / 2;
        if (before[lo + half] <= at) lo += half, n -= half;
        else n = half;
    }
    return lo;
}

// Sums do not pass 2^31 - 1.
__device__ __forceinline__ uint32_t add_up(uint32_t a, uint32_t b) { return min(a + b, 0x7fffffffu); }

__device__ __forceinline__ void step_sync(uint32_t size) {
    if (size > 1) cluster_sync();
    else __syncthreads();
}

// Sums over the block in front of every thread of N values a thread, none above 2^31 - 1; total: of all.  Only the first `busy` warps
// have any.  shared: [N][32], not in use since the last barrier.
template <int N, int kWarps>
__device__ __forceinline__ void sum_before(uint32_t* v, uint32_t* total, uint32_t (*shared)[32], int busy) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (warp < busy) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            uint32_t incl = v[k];
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const uint32_t up = __shfl_up_sync(~0u, incl, o);
                if (lane >= o) incl = add_up(incl, up);
            }
            if (lane == 31) shared[k][warp] = incl;
            v[k] = __shfl_up_sync(~0u, incl, 1);
            if (lane == 0) v[k] = 0;
        }
    }
    __syncthreads();
    if (busy > 1) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (warp != k % kWarps) continue;
            uint32_t incl = lane < busy ? shared[k][lane] : 0;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const uint32_t up = __shfl_up_sync(~0u, incl, o);
                if (lane >= o) incl = add_up(incl, up);
            }
            shared[k][lane] = incl;
        }
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if (warp > 0 && warp < busy) v[k] = add_up(v[k], shared[k][warp - 1]);
        total[k] = shared[k][busy - 1];
    }
}

// A block that gets new tokens, with what the rows of its tokens need.
struct Handed {
    int64_t slot;       // of the sequence's cache index 0, were all its blocks in a row with this one
    int32_t lo, hi;     // cache indices of the new tokens in the block
    int32_t row, pos;   // row and position of cache index 0
};
constexpr int64_t kNoSlot = INT64_MIN;

template <int kThreads>
__global__ void __launch_bounds__(kThreads, 1) advance_tables(const __grid_constant__ StepParams p) {
    constexpr int kWarps = kThreads / 32;
    extern __shared__ __align__(16) char smem[];
    constexpr bool kLarge = kThreads == kStepMost;
    __shared__ uint32_t s_sum[5][32];
    __shared__ Handed s_block[kWarps][32];
    __shared__ int32_t s_freed, s_count;
    __shared__ uint32_t s_bad;
    __shared__ int32_t s_all_bad[kStepCluster], s_all_freed[kStepCluster];  // in the first CTA
    const uint32_t rank = cluster_rank(), size = cluster_size();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, S = p.num_seqs, T = p.block_tokens;
    const int tiles = kLarge ? (p.tiles + (int)size - 1) / (int)size : 0;  // of this CTA; the last may lie behind the pool
    const int words = kLarge ? tiles * kWarps : p.words;
    const StepShared sh(smem, p, words, tiles);
    const int32_t *const blocks = sh.sums[0], *const rows = sh.sums[1], *const copied = sh.sums[2], *const entries = sh.sums[3];
    if (tid == 0) s_freed = 0, s_bad = 0;
    grid_dependency_launch();
    grid_dependency_wait();

    // ---- the free blocks, and what the first sequences ask for
    Ask ask;
    if (tid < S) ask.lengths(p, tid);
    // First block of this warp's i-th word, the (warp + i * kWarps)-th of the CTA.
    const uint32_t step = (kLarge ? size : 1) * kThreads, own_block = kLarge ? rank * kThreads + warp * 32 : (rank * p.words + warp) * 32;
    auto first_block = [&](int i) { return own_block + (uint32_t)i * step; };
    const int own_words = kLarge ? tiles : (words - warp + kWarps - 1) / kWarps;
    constexpr int kAtOnce = 16;
    for (int i0 = 0; i0 < own_words || i0 == 0; i0 += kAtOnce) {
        int count[kAtOnce];  // loaded without a question, so that the loads overlap
        const uint32_t b0 = first_block(i0) + lane, last = (uint32_t)p.num_blocks - 1;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) count[i] = p.refs[min(b0 + i * step, last)];
        if (i0 == 0 && tid < S) ask.more(p, tid), ask.counts(p);
        uint32_t mine = 0;  // lane i keeps word i
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const uint32_t word = __ballot_sync(~0u, count[i] == 0 && b0 + i * step <= last);
            if (lane == i) mine = word;
        }
        if (lane < min(kAtOnce, own_words - i0)) sh.free[(i0 + lane) * kWarps + warp] = mine;
    }
    if (!kLarge) __syncthreads();

    // ---- the sums in front of every sequence (and, in launches that are not large, of every word)
    uint32_t bad = 0, run[4] = {0, 0, 0, 0};
    for (int base = 0; base < S || base == 0; base += kThreads) {
        const int s = base + tid;
        Need n;
        if (s < S) {
            Ask a = ask;
            if (base > 0) {
                a = Ask();
                a.lengths(p, s), a.more(p, s), a.counts(p);
            }
            n = a.need(p, &bad);
            sh.first[s] = n.first;
        }
        uint32_t v[5] = {(uint32_t)n.blocks, (uint32_t)n.rows, (uint32_t)n.copies, (uint32_t)n.entries, 0}, total[5];
        const bool counts = !kLarge && base == 0;
        if (counts && tid < words) v[4] = __popc(sh.free[tid]);
        if (base > 0) __syncthreads();
        sum_before<kLarge ? 4 : 5, kWarps>(v, total, s_sum, min(kWarps, (max(S - base, counts ? words : 1) + 31) / 32));
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (s < S) sh.sums[k][s] = (int32_t)add_up(run[k], v[k]);
            run[k] = add_up(run[k], total[k]);
        }
        if (counts && tid < words) sh.before[tid] = (int32_t)v[4];
        if (counts && tid == 0) s_count = (int32_t)total[4];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (tid == 0) sh.sums[k][S] = (int32_t)run[k];
    if (bad) atomicOr(&s_bad, bad);
    if (kLarge) {
        __syncthreads();
        for (int t = warp; t < tiles; t += kWarps) {  // words of a tile
            const int own = __popc(sh.free[t * kWarps + lane]);
            int sum = own;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int up = __shfl_up_sync(~0u, sum, o);
                if (lane >= o) sum += up;
            }
            sh.before[t * kWarps + lane] = sum - own;
            if (lane == 31) sh.count[t] = sum;
        }
    }
    step_sync(size);

    // ---- the free blocks of all CTAs, and who gets what: the sequences in front of the first that does not fit
    uint32_t n_free = 0;
    int in_front = 0;  // free blocks in front of this CTA's run of words
    if (kLarge) {
        for (int base = 0; base < p.tiles; base += kThreads) {
            const int t = base + tid;
            uint32_t v[1] = {t >= p.tiles ? 0u : (uint32_t)load_remote(&sh.count[(uint32_t)t / size], (uint32_t)t % size)}, total[1];
            if (base > 0) __syncthreads();
            sum_before<1, kWarps>(v, total, s_sum, min(kWarps, (p.tiles - base + 31) / 32));
            if (t < p.tiles && (uint32_t)t % size == rank) sh.start[(uint32_t)t / size] = (int32_t)(n_free + v[0]);
            n_free += total[0];
        }
        for (int t = tid; t < tiles; t += kThreads)
            if ((int64_t)t * size + rank >= p.tiles) sh.start[t] = INT32_MAX;
    } else {
        const int own = lane >= (int)size ? 0 : size > 1 ? load_remote(&s_count, lane) : s_count;
        n_free = __reduce_add_sync(~0u, (uint32_t)own);
        in_front = (int)__reduce_add_sync(~0u, lane < (int)rank ? (uint32_t)own : 0u);
    }
    // No CTA ends while another reads its counts: the barrier that all arrive at here, or, where there is something to share, to copy or
    // to give back, behind that: free blocks are handed out when it is done.
    const bool in_turn = entries[S] > 0 || copied[S] > 0;  // (the same in all CTAs)
    if (size > 1 && !in_turn) cluster_arrive();
    int fits = S;
    if (blocks[S] > (int)n_free || rows[S] > p.num_rows || copied[S] > p.pairs_cap) {
        fits = 0;
        for (int hi = S; hi - fits > 1;) {
            const int mid = (fits + hi) / 2;
            if (blocks[mid] <= (int)n_free && rows[mid] <= p.num_rows && copied[mid] <= p.pairs_cap) fits = mid;
            else hi = mid;
        }
    }
    const int n_taken = blocks[fits], n_rows = rows[fits], n_copies = copied[fits], n_entries = entries[S];
    const int all = size * kThreads, me = (warp * size + rank) * 32 + lane;
    auto copies = [&](int s) { return copied[s + 1] > copied[s]; };
    auto parent_of = [&](int s) { return p.parents ? p.parents[s] : -1; };
    int freed = 0;
    auto give_back = [&](int b) {
        const int count = p.inside(b) ? atomicAdd(&p.refs[b], -1) : 0;
        if (count > 0) {
            freed += count == 1;
            return;
        }
        bad |= kBadBlock;  // no count left: it was not this table's to give back
        if (p.inside(b)) atomicAdd(&p.refs[b], 1);
    };
    auto can_share = [&](int b) {  // in the pool, and counted in front of the call
        if (p.inside(b)) {
            const uint32_t word = (uint32_t)b / 32, tile = word / kWarps, of = kLarge ? tile % size : word / p.words;
            const int32_t* const at = reinterpret_cast<const int32_t*>(sh.free) + (kLarge ? tile / size * kWarps + word % kWarps : word - of * p.words);
            if (!((uint32_t)(size > 1 ? load_remote(at, of) : *at) >> (b % 32) & 1u)) return true;
        }
        bad |= kBadBlock;
        return false;
    };

    // ---- shared and given back blocks, sources of copies: everything that reads other sequences' rows of the table
    for (int e = me; e < n_entries; e += all) {
        const int s = last_at_most(entries, S, e), j = e - entries[s], parent = parent_of(s);
        int32_t* const row = p.table + (int64_t)s * p.max_blocks;
        if (parent < 0) {
            give_back(row[p.blocks_of(p.new_lens[s]) + j]);
        } else if (s < fits) {
            const int b = p.table[(int64_t)parent * p.max_blocks + j];
            row[j] = b;
            if (can_share(b)) freed -= atomicAdd(&p.refs[b], 1) == 0;  // (its last other user has just given it back)
        }
    }
    for (int s = me; n_copies > 0 && s < fits; s += all) {
        if (!copies(s)) continue;
        const int parent = parent_of(s), b = p.table[(int64_t)(parent >= 0 ? parent : s) * p.max_blocks + p.whole(sh.first[s])];
        p.pairs[copied[s]].x = parent < 0 || can_share(b) ? b : -1;
        if (parent < 0) give_back(b);
    }
    if (size > 1 && in_turn) cluster_sync();
    else __syncthreads();

    // ---- the free blocks to their sequences, a warp's word of every tile; rows, positions and slots of the tokens in them
    const bool writes_rows = p.positions || p.slots;
    auto write_row = [&](int row, int position, int64_t slot) {
        if (p.positions) p.positions[row] = position;
        if (p.slots) p.slots[row] = slot;
    };
    auto end_of = [&](int s) { return sh.first[s] + rows[s + 1] - rows[s]; };
    for (int i = 0; i < own_words; ++i) {
        const int w = i * kWarps + warp, front = kLarge ? sh.start[i] : in_front;
        if (front >= n_taken) break;
        const uint32_t word = sh.free[w];
        const int r0 = front + sh.before[w], n = min(__popc(word), n_taken - r0);
        const int k = __popc(word & ((1u << lane) - 1)), r = r0 + k;
        if (n <= 0) continue;
        if (word >> lane & 1u && k < n) {
            const int b = (int)(first_block(i) + lane), s = last_at_most(blocks, fits, r), j = r - blocks[s], first = sh.first[s];
            const bool copy = copies(s);
            const int column = (copy ? p.whole(first) : p.blocks_of(first)) + j;
            p.table[(int64_t)s * p.max_blocks + column] = b;
            p.refs[b] = 1;
            if (j == 0 && copy) p.pairs[copied[s]].y = b;
            const int64_t begin = (int64_t)column * T;
            s_block[warp][k] = Handed{(int64_t)b * T - begin, (int)max(begin, (int64_t)first), (int)min(begin + T, (int64_t)end_of(s)),
                                      rows[s] - first, p.first_pos ? p.first_pos[s] - first : 0};
        }
        __syncwarp();
        if (writes_rows) {
            if (T >= 32) {
                for (int i = 0; i < n; ++i) {
                    const Handed x = s_block[warp][i];
                    for (int index = x.lo + lane; index < x.hi; index += 32) write_row(x.row + index, x.pos + index, x.slot + index);
                }
            } else {
                const int at_once = 32 / T, part = lane / T;  // blocks at a time
                for (int i = part; i < n && part < at_once; i += at_once) {
                    const Handed x = s_block[warp][i];
                    const int index = x.lo + lane - part * T;
                    if (index < x.hi) write_row(x.row + index, x.pos + index, x.slot + index);
                }
            }
        }
        __syncwarp();
    }
    for (int e = me; e < n_entries; e += all) {
        const int s = last_at_most(entries, S, e);
        if (parent_of(s) < 0) p.table[(int64_t)s * p.max_blocks + p.blocks_of(p.new_lens[s]) + e - entries[s]] = -1;
    }

    // ---- lengths, row starts, and the rows in blocks that were there: what is left of a last block
    for (int base = warp * 32; base <= S; base += kThreads) {
        const int s = base + lane;
        if (base / 32 % (int)size != (int)rank) continue;
        Handed x{0, 0, 0, 0, 0};
        if (s < S) {
            Ask a = ask;  // (of the first sequences)
            if (base >= kThreads) a.lengths(p, s);
            const int old = a.old, now = a.now, first = sh.first[s];
            const bool grows = now > old || a.parent >= 0, stays = first < 0 || (grows && s >= fits);
            p.lens_out[s] = stays ? old : now;
            const int n = stays ? 0 : p.whole(first);
            if (writes_rows && !stays && n * T != first && !copies(s) && rows[s + 1] > rows[s]) {
                const int b = base >= kThreads ? p.table[(int64_t)s * p.max_blocks + n] : a.last;
                x = Handed{p.inside(b) ? ((int64_t)b - n) * T : kNoSlot, first, (int)min((int64_t)end_of(s), ((int64_t)n + 1) * T), rows[s] - first,
                           p.first_pos ? p.first_pos[s] - first : 0};
                if (T < 128)
                    for (int index = x.lo; index < x.hi; ++index) write_row(x.row + index, x.pos + index, x.slot == kNoSlot ? -1 : x.slot + index);
            }
        }
        if (p.starts && s <= S) p.starts[s] = rows[min(s, fits)];
        for (unsigned more = T < 128 ? 0 : __ballot_sync(~0u, x.hi > x.lo); more; more &= more - 1) {
            const int of = __ffs(more) - 1, lo = __shfl_sync(~0u, x.lo, of), hi = __shfl_sync(~0u, x.hi, of);
            const int row = __shfl_sync(~0u, x.row, of), pos = __shfl_sync(~0u, x.pos, of);
            const int64_t slot = __shfl_sync(~0u, x.slot, of);
            for (int index = lo + lane; index < hi; index += 32) write_row(row + index, pos + index, slot == kNoSlot ? -1 : slot + index);
        }
    }
    if (writes_rows)
        for (int r = n_rows + me; r < p.num_rows; r += all) {
            if (p.positions) p.positions[r] = 0;
            if (p.slots) p.slots[r] = -1;
        }

    // ---- one code, always the same for the same call, and the counts
    if (bad) atomicOr(&s_bad, bad);
    if (freed) atomicAdd(&s_freed, freed);
    __syncthreads();
    if (size > 1 && !in_turn) cluster_wait();
    if (tid == 0) {
        if (size > 1) store_remote(&s_all_bad[rank], 0, (int32_t)s_bad), store_remote(&s_all_freed[rank], 0, s_freed);
        else s_all_bad[0] = (int32_t)s_bad, s_all_freed[0] = s_freed;
    }
    if (size > 1) {
        cluster_arrive();
        if (rank > 0) return;
        cluster_wait();
    }
    if (tid == 0) {
        uint32_t all_bad = 0;
        int all_freed = 0;
        for (uint32_t r = 0; r < size; ++r) all_bad |= (uint32_t)s_all_bad[r], all_freed += s_all_freed[r];
        if (p.num_pairs) *p.num_pairs = n_copies;
        if (p.free_count) *p.free_count = (int)n_free - n_taken + all_freed;
        if ((all_bad & kBadArg) || (fits < S && blocks[fits + 1] <= (int)n_free)) report(p.status, AMOEBA_ERR_INVALID_ARG);
        else if (fits < S) report(p.status, AMOEBA_ERR_NO_FREE_BLOCKS);
        else if (all_bad & kBadBlock) report(p.status, AMOEBA_ERR_BAD_BLOCK_ID);
    }
}

}  // namespace amoeba

using namespace amoeba;

extern "C" amoeba_status amoeba_advance_tables(const amoeba_layout* layout, const amoeba_table_step* step, int32_t* d_status,
                                               void* cuda_stream) {
    int64_t pool = 0;
    if (!layout || !step || !d_status) return AMOEBA_ERR_INVALID_ARG;
    const amoeba_status st = amoeba_layout_kv_pool_bytes(layout, &pool);
    if (st != AMOEBA_OK) return st;
    if (layout->block_tokens > kMaxTokens) return AMOEBA_ERR_UNSUPPORTED;
    const amoeba_table_step& a = *step;
    if (a.num_seqs < 0 || a.max_blocks_per_seq < 0 || a.num_rows < 0 || a.pairs_cap < 0) return AMOEBA_ERR_INVALID_ARG;
    if (!a.d_block_refs && layout->num_blocks) return AMOEBA_ERR_INVALID_ARG;
    if (a.num_seqs && (!a.d_seq_lens || !a.d_new_lens || !a.d_lens_out || (a.max_blocks_per_seq && !a.d_block_table))) return AMOEBA_ERR_INVALID_ARG;
    if (!a.d_parents != !a.d_shared_lens) return AMOEBA_ERR_INVALID_ARG;
    if (!a.d_q_starts && (a.d_positions || a.d_slots || a.num_rows)) return AMOEBA_ERR_INVALID_ARG;
    if (a.d_first_positions && !a.d_positions) return AMOEBA_ERR_INVALID_ARG;
    if (a.pairs_cap && (!a.d_pairs || !a.d_num_pairs)) return AMOEBA_ERR_INVALID_ARG;
    if ((uintptr_t)a.d_pairs % 8 || (uintptr_t)a.d_slots % 8) return AMOEBA_ERR_ALIGNMENT;
    // (entries and rows are numbered in 32 bits, and counted on past the last one)
    if ((int64_t)a.num_seqs * a.max_blocks_per_seq > (1 << 30) || a.num_rows > (1 << 30)) return AMOEBA_ERR_UNSUPPORTED;
    StepParams p{};
    p.table = a.d_block_table, p.refs = a.d_block_refs;
    p.lens = a.d_seq_lens, p.new_lens = a.d_new_lens, p.parents = a.d_parents, p.shared = a.d_shared_lens;
    p.lens_out = a.d_lens_out, p.starts = a.d_q_starts, p.first_pos = a.d_first_positions, p.positions = a.d_positions;
    p.slots = a.d_slots, p.pairs = reinterpret_cast<int2*>(a.d_pairs), p.num_pairs = a.d_num_pairs, p.free_count = a.d_free_count;
    p.status = d_status;
    p.num_seqs = a.num_seqs, p.max_blocks = a.max_blocks_per_seq, p.num_rows = a.num_rows, p.pairs_cap = a.pairs_cap;
    p.num_blocks = layout->num_blocks, p.block_tokens = layout->block_tokens;
    p.shift = (p.block_tokens & (p.block_tokens - 1)) == 0 ? __builtin_ctz((unsigned)p.block_tokens) : -1;
    p.max_len = (int32_t)std::min<int64_t>((int64_t)a.max_blocks_per_seq * layout->block_tokens, kMaxTokens);
    const DeviceInfo dev = cached_device_info();
    if (!dev.sms) return AMOEBA_ERR_CUDA;
    // A few sequences and blocks are soonest done by one small CTA (8 sequences, 136 blocks: 4.6 us a call, 8 by one of 1024 threads); then a
    // cluster's loads and stores count, then its bytes (750 000 blocks, both calls: 35 us by 16 CTAs, 51 by 8).
    const bool large = p.num_blocks > 65536 || p.num_seqs > 512 || p.num_rows > 8192;
    const bool small = p.num_blocks <= 8192 && p.num_seqs <= 256 && p.num_rows <= 1024;
    const int cluster = small ? 1 : large ? kStepCluster : kMaxCluster, threads = large ? kStepMost : 256;
    p.tiles = large ? (int32_t)(((int64_t)p.num_blocks + threads - 1) / threads) : 0;
    p.words = large ? 0 : (p.num_blocks + 32 * cluster - 1) / (32 * cluster);
    const int64_t tiles = (p.tiles + cluster - 1) / cluster, smem = step_smem(p.num_seqs, large ? tiles * (threads / 32) : p.words, tiles);
    if (smem > dev.smem_optin - kStepStatic) return AMOEBA_ERR_TOO_LARGE;
    if (large && allow_large_clusters((const void*)advance_tables<kStepMost>) != cudaSuccess) return AMOEBA_ERR_CUDA;
    return launch_clusters(large ? advance_tables<kStepMost> : advance_tables<256>, cluster, threads, (size_t)smem, cluster, true,
                           static_cast<cudaStream_t>(cuda_stream), p);
}
