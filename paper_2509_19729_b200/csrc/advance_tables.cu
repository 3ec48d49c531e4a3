// amoeba_advance_tables: block tables, block counts, rows, positions and slots of a step, from the sequences' lengths.
//
// One launch of one cluster.  With n = ceil(length / block_tokens) blocks before and after,
//   blocks(s) = what a growing or forked sequence lacks,  rows(s) = its new tokens,  copies(s) = 1 if its first new block is a copy,
// and their prefix sums over the sequences, the r-th free id overall (ascending) goes to the sequence with
// blocks[s] <= r < blocks[s + 1], and row r to the one with rows[s] <= r < rows[s + 1].  The free ids are counted warp by warp in
// contiguous runs, so that an id's rank needs one exchange of counts between the CTAs; the prefix sums every CTA makes for itself.
//
// What bounds it is latency: a launch, the dependent loads of a look at a sequence's last block, two or three barriers of the
// cluster and a search for every block and row.  The counts (4 bytes a block) are read once.
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
    int32_t warp_words;     // words of 32 blocks that a warp looks at

    __device__ __forceinline__ int whole(int tokens) const { return shift >= 0 ? tokens >> shift : tokens / block_tokens; }
    __device__ __forceinline__ int blocks_of(int tokens) const { return whole(tokens + block_tokens - 1); }
    __device__ __forceinline__ bool inside(int b) const { return b >= 0 && b < num_blocks; }
};

constexpr int kStepThreads = 1024, kStepWarps = kStepThreads / 32;
constexpr int kStepIds = 4096;  // free ids that a CTA lists at a time
constexpr uint32_t kBadArg = 1, kBadBlock = 2;

// In dynamic shared memory: sums over the sequences in front of every one, and at [num_seqs] over all; then the bits of the free
// blocks that the CTA looks at.
struct StepShared {
    int32_t *blocks, *rows, *copies;
    int32_t* entries;  // entries of the table that are shared with a parent's or given back
    int32_t* first;    // cache index of the first new token; -1: refused
    int32_t* ids;      // [kStepIds] free blocks, counted from the CTA's first
    uint32_t* free;    // [kStepWarps * warp_words]

    __device__ __forceinline__ StepShared(char* smem, const StepParams& p) {
        const int n = p.num_seqs + 1;
        blocks = reinterpret_cast<int32_t*>(smem);
        rows = blocks + n, copies = rows + n, entries = copies + n, first = entries + n, ids = first + n;
        free = reinterpret_cast<uint32_t*>(ids + kStepIds);
    }
};
static int64_t step_smem(int64_t num_seqs, int64_t warp_words) { return (5 * (num_seqs + 1) + kStepIds + kStepWarps * warp_words) * 4; }

// What a sequence asks for.  The loads come in two steps, so that others can be started in between.
struct Need {
    int32_t blocks = 0, rows = 0, copies = 0, entries = 0, first = -1;
};
struct Ask {
    int32_t old = 0, now = 0, parent = -1, share = 0, from = 0, last = -1;
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
                const int count = p.inside(last) ? p.refs[last] : 0;
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

__global__ void __launch_bounds__(kStepThreads, 1) advance_tables(const __grid_constant__ StepParams p) {
    extern __shared__ __align__(16) char smem[];
    __shared__ uint32_t s_sum[4][kStepWarps];
    __shared__ int32_t s_free[kStepWarps];   // of every warp, then before it
    __shared__ int32_t s_count;              // free blocks that this CTA looks at
    __shared__ int32_t s_freed;
    __shared__ uint32_t s_bad;
    __shared__ int32_t s_all_bad[kMaxCluster], s_all_freed[kMaxCluster];  // in the first CTA
    const uint32_t rank = cluster_rank(), size = cluster_size();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, S = p.num_seqs;
    const StepShared sh(smem, p);
    if (tid == 0) s_freed = 0, s_bad = 0;
    grid_dependency_launch();
    grid_dependency_wait();

    // ---- the free blocks, and what the first sequences ask for
    Ask ask;
    if (tid < S) ask.lengths(p, tid);
    const int64_t cta_block = (int64_t)rank * kStepWarps * p.warp_words * 32;
    uint32_t* const words = sh.free + warp * p.warp_words;
    int found = 0;
    constexpr int kAtOnce = 8;
    for (int w0 = 0; w0 < p.warp_words; w0 += kAtOnce) {
        bool is[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int64_t b = cta_block + ((int64_t)warp * p.warp_words + w0 + i) * 32 + lane;
            is[i] = w0 + i < p.warp_words && b < p.num_blocks && p.refs[b] == 0;
        }
        if (w0 == 0 && tid < S) ask.more(p, tid);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const uint32_t word = __ballot_sync(~0u, is[i]);
            if (w0 + i < p.warp_words) {
                if (lane == 0) words[w0 + i] = word;
                found += __popc(word);
            }
        }
    }
    if (lane == 0) s_free[warp] = found;

    // ---- the sums in front of every sequence
    uint32_t bad = 0, run[4] = {0, 0, 0, 0};
    for (int base = 0; base < S || base == 0; base += kStepThreads) {
        const int s = base + tid;
        Need n;
        if (s < S) {
            if (base > 0) {
                ask = Ask();
                ask.lengths(p, s);
                ask.more(p, s);
            }
            n = ask.need(p, &bad);
            sh.first[s] = n.first;
        }
        uint32_t incl[4] = {(uint32_t)n.blocks, (uint32_t)n.rows, (uint32_t)n.copies, (uint32_t)n.entries}, before[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const uint32_t up = __shfl_up_sync(~0u, incl[k], o);
                if (lane >= o) incl[k] = add_up(incl[k], up);
            }
            before[k] = __shfl_up_sync(~0u, incl[k], 1);
            if (lane == 0) before[k] = 0;
            if (lane == 31) s_sum[k][warp] = incl[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t all = s_sum[k][lane];  // (as many warps as lanes)
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const uint32_t up = __shfl_up_sync(~0u, all, o);
                if (lane >= o) all = add_up(all, up);
            }
            const uint32_t total = __shfl_sync(~0u, all, 31), warps = __shfl_sync(~0u, all, max(warp - 1, 0));
            if (s < S) (sh.blocks + k * (S + 1))[s] = (int32_t)add_up(run[k], add_up(warp ? warps : 0, before[k]));
            run[k] = add_up(run[k], total);
        }
        if (base == 0 && warp == 0) {
            const int own = s_free[lane];
            int sum = own;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int up = __shfl_up_sync(~0u, sum, o);
                if (lane >= o) sum += up;
            }
            s_free[lane] = sum - own;
            if (lane == 31) s_count = sum;
        }
        if (base + kStepThreads < S) __syncthreads();
    }
    if (tid < 4) (sh.blocks + tid * (S + 1))[S] = (int32_t)(tid == 0 ? run[0] : tid == 1 ? run[1] : tid == 2 ? run[2] : run[3]);
    if (bad) atomicOr(&s_bad, bad);
    step_sync(size);

    // ---- who gets it: the sequences in front of the first that does not fit
    int n_free = 0, rank_before = 0;
    for (uint32_t r = 0; r < size; ++r) {
        const int n = size > 1 ? load_remote(&s_count, r) : s_count;
        if (r < rank) rank_before += n;
        n_free += n;
    }
    int fits = S;
    if (sh.blocks[S] > n_free || sh.rows[S] > p.num_rows || sh.copies[S] > p.pairs_cap) {
        fits = 0;
        for (int hi = S; hi - fits > 1;) {
            const int mid = (fits + hi) / 2;
            if (sh.blocks[mid] <= n_free && sh.rows[mid] <= p.num_rows && sh.copies[mid] <= p.pairs_cap) fits = mid;
            else hi = mid;
        }
    }
    const int n_taken = sh.blocks[fits], n_rows = sh.rows[fits], n_copies = sh.copies[fits], n_entries = sh.entries[S];
    const int all = size * kStepThreads, me = rank * kStepThreads + tid;
    auto copies = [&](int s) { return sh.copies[s + 1] > sh.copies[s]; };
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

    // ---- shared and given back blocks, sources of copies: everything that reads other sequences' rows of the table
    for (int e = me; e < n_entries; e += all) {
        const int s = last_at_most(sh.entries, S, e), j = e - sh.entries[s], parent = parent_of(s);
        int32_t* const row = p.table + (int64_t)s * p.max_blocks;
        if (parent < 0) {
            give_back(row[p.blocks_of(p.new_lens[s]) + j]);
        } else if (s < fits) {
            const int b = p.table[(int64_t)parent * p.max_blocks + j];
            row[j] = b;
            if (!p.inside(b)) bad |= kBadBlock;
            else freed -= atomicAdd(&p.refs[b], 1) == 0;  // (its last other user has just given it back)
        }
    }
    for (int s = me; n_copies > 0 && s < fits; s += all) {
        if (!copies(s)) continue;
        const int parent = parent_of(s), b = p.table[(int64_t)(parent >= 0 ? parent : s) * p.max_blocks + p.whole(sh.first[s])];
        p.pairs[sh.copies[s]].x = p.inside(b) ? b : -1;
        if (parent < 0) give_back(b);
        else if (!p.inside(b)) bad |= kBadBlock;
    }
    if (p.parents || p.pairs_cap > 0) step_sync(size);  // (without these no row is read that is not the reader's own)

    // ---- the free blocks to their sequences
    for (int e = me; e < n_entries; e += all) {
        const int s = last_at_most(sh.entries, S, e);
        if (parent_of(s) < 0) p.table[(int64_t)s * p.max_blocks + p.blocks_of(p.new_lens[s]) + e - sh.entries[s]] = -1;
    }
    const int mine = min(s_count, n_taken - rank_before);  // of the free blocks that this CTA looks at
    for (int base = 0; base < mine; base += kStepIds) {
        const int end = min(mine, base + kStepIds);
        int r0 = s_free[warp];
        for (int w = 0; w < p.warp_words && r0 < end; ++w) {
            const uint32_t word = words[w];
            const int r = r0 + __popc(word & ((1u << lane) - 1));
            if (word >> lane & 1u && r >= base && r < end) sh.ids[r - base] = (warp * p.warp_words + w) * 32 + lane;
            r0 += __popc(word);
        }
        __syncthreads();
        for (int i = tid; i < end - base; i += kStepThreads) {
            const int b = (int)cta_block + sh.ids[i], r = rank_before + base + i, s = last_at_most(sh.blocks, fits, r), j = r - sh.blocks[s];
            const int have = copies(s) ? p.whole(sh.first[s]) : p.blocks_of(sh.first[s]);
            p.table[(int64_t)s * p.max_blocks + have + j] = b;
            p.refs[b] = 1;
            if (j == 0 && copies(s)) p.pairs[sh.copies[s]].y = b;
        }
        if (end < mine) __syncthreads();
    }
    if (bad) atomicOr(&s_bad, bad);
    if (freed) atomicAdd(&s_freed, freed);
    __syncthreads();
    if (tid == 0) {
        if (size > 1) store_remote(&s_all_bad[rank], 0, (int32_t)s_bad), store_remote(&s_all_freed[rank], 0, s_freed);
        else s_all_bad[0] = (int32_t)s_bad, s_all_freed[0] = s_freed;
    }
    step_sync(size);

    // ---- rows, lengths, counts
    if (p.starts)
        for (int s = me; s <= S; s += all) p.starts[s] = sh.rows[min(s, fits)];
    for (int s = me; s < S; s += all) {
        const int old = p.lens[s], now = p.new_lens[s];
        const bool grows = now > old || parent_of(s) >= 0;
        p.lens_out[s] = sh.first[s] < 0 || (grows && s >= fits) ? old : now;
    }
    if (p.positions || p.slots)
        for (int r = me; r < p.num_rows; r += all) {
            int position = 0;
            int64_t slot = -1;
            if (r < n_rows) {
                const int s = last_at_most(sh.rows, fits, r), j = r - sh.rows[s], index = sh.first[s] + j;
                position = p.first_pos ? p.first_pos[s] + j : index;
                if (p.slots) {
                    const int n = p.whole(index), b = __ldcg(&p.table[(int64_t)s * p.max_blocks + n]);
                    if (p.inside(b)) slot = ((int64_t)b - n) * p.block_tokens + index;
                }
            }
            if (p.positions) p.positions[r] = position;
            if (p.slots) p.slots[r] = slot;
        }
    if (rank == 0 && tid == 0) {
        uint32_t all_bad = 0;
        int all_freed = 0;
        for (uint32_t r = 0; r < size; ++r) all_bad |= (uint32_t)s_all_bad[r], all_freed += s_all_freed[r];
        if (p.num_pairs) *p.num_pairs = n_copies;
        if (p.free_count) *p.free_count = n_free - n_taken + all_freed;
        // One code, always the same for the same call.
        if ((all_bad & kBadArg) || (fits < S && sh.blocks[fits + 1] <= n_free)) report(p.status, AMOEBA_ERR_INVALID_ARG);
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
    const int cluster = p.num_blocks <= 8192 && p.num_seqs <= kStepThreads && p.num_rows <= 4 * kStepThreads ? 1 : kMaxCluster;
    p.warp_words = (int32_t)(((int64_t)p.num_blocks + cluster * kStepThreads - 1) / (cluster * kStepThreads));
    const int64_t smem = step_smem(p.num_seqs, p.warp_words);
    if (smem > dev.smem_optin - 2048) return AMOEBA_ERR_TOO_LARGE;
    return launch_clusters(advance_tables, cluster, kStepThreads, (size_t)smem, cluster, true, static_cast<cudaStream_t>(cuda_stream), p);
}
