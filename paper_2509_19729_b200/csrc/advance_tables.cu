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
    int32_t max_len;        // tokens that a row of the table has room for
    int32_t warp_words;     // words of 32 blocks that a warp looks at
};

constexpr int kStepThreads = 1024, kStepWarps = kStepThreads / 32;
constexpr int kEntryRun = 128;  // table entries that a warp takes at a time
constexpr uint32_t kBadArg = 1, kBadBlock = 2;

// Per sequence, in dynamic shared memory; then the bits of the free blocks that the CTA looks at.
struct StepShared {
    int32_t *blocks, *rows, *copies;  // [num_seqs + 1] before every sequence
    int32_t* first;                   // [num_seqs] cache index of the first new token; -1: refused
    int32_t* touched;                 // [num_seqs] the forked and the shortened ones, in any order
    uint32_t* free;                   // [kStepWarps * warp_words]
};
__device__ __forceinline__ StepShared step_shared(char* smem, const StepParams& p) {
    StepShared sh;
    sh.blocks = reinterpret_cast<int32_t*>(smem);
    sh.rows = sh.blocks + p.num_seqs + 1;
    sh.copies = sh.rows + p.num_seqs + 1;
    sh.first = sh.copies + p.num_seqs + 1;
    sh.touched = sh.first + p.num_seqs;
    sh.free = reinterpret_cast<uint32_t*>(sh.touched + p.num_seqs);
    return sh;
}
static int64_t step_smem(int64_t num_seqs, int64_t warp_words) { return (5 * num_seqs + 3 + kStepWarps * warp_words) * 4; }

// What a sequence asks for.
struct Need {
    int32_t blocks, rows, copy, first;
    bool touched;
};
__device__ __forceinline__ Need need_of(const StepParams& p, int s, uint32_t* bad) {
    const int T = p.block_tokens, old = p.lens[s], now = p.new_lens[s], parent = p.parents ? p.parents[s] : -1;
    Need n{0, 0, 0, -1, false};
    bool ok = old >= 0 && old <= p.max_len && now >= 0 && now <= p.max_len && parent < p.num_seqs;
    int share = 0;
    if (ok && parent >= 0) {
        const int from = p.lens[parent];
        share = p.shared[s];
        ok = old == 0 && from <= p.max_len && share >= 0 && share <= from && share <= now;
    }
    if (!ok) {
        *bad |= kBadArg;
        return n;
    }
    n.first = parent >= 0 ? share : old;
    n.touched = parent >= 0 || now < old;
    if (now < old) return n;
    int have = n.first / T;
    if (have * T != n.first) {
        // The last block is not full: a fork gets a copy of its parent's, and a sequence one of a block that others name too.
        n.copy = parent >= 0;
        if (parent < 0 && now > old) {
            const int b = p.table[(int64_t)s * p.max_blocks + have];
            const int count = b >= 0 && b < p.num_blocks ? p.refs[b] : 0;
            if (count < 1) *bad |= kBadBlock;
            n.copy = count > 1;
        }
        if (!n.copy) ++have;
    }
    n.blocks = max((now + T - 1) / T - have, 0);
    n.rows = p.starts ? now - n.first : 0;
    return n;
}

// The last s in [0, n) with before[s] <= at; before[0] = 0.
__device__ __forceinline__ int last_at_most(const int32_t* before, int n, int at) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (before[mid] <= at) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ void step_sync(uint32_t size) {
    if (size > 1) cluster_sync();
    else __syncthreads();
}

// Calls entry(s, place in the table, column) for the columns [begin(s), end(s)) of the touched sequences, whose warps all share them.
// A lane looks at one sequence each first, so that their loads overlap.
template <class Range, class Entry>
__device__ __forceinline__ void for_entries(const StepParams& p, const StepShared& sh, int n_touched, uint32_t rank, uint32_t size,
                                            Range range, Entry entry) {
    const int lane = threadIdx.x % 32, warps = size * kStepWarps, mine = rank * kStepWarps + threadIdx.x / 32;
    for (int base = 0; base < n_touched; base += 32) {
        const int s_own = base + lane < n_touched ? sh.touched[base + lane] : -1;
        int2 r_own = make_int2(0, 0);
        if (s_own >= 0) r_own = range(s_own);
        for (int i = 0; i < min(32, n_touched - base); ++i) {
            const int s = __shfl_sync(~0u, s_own, i), lo = __shfl_sync(~0u, r_own.x, i), hi = __shfl_sync(~0u, r_own.y, i);
            const int turn = (int)((uint32_t)s * 37u % (uint32_t)warps), at = mine >= turn ? mine - turn : mine - turn + warps;
            for (int64_t j = lo + (int64_t)at * kEntryRun + lane; j - lane < hi; j += (int64_t)warps * kEntryRun)
#pragma unroll
                for (int k = 0; k < kEntryRun; k += 32)
                    if (j + k < hi) entry(s, (int64_t)s * p.max_blocks + j + k, (int)j + k);
        }
    }
}

__global__ void __launch_bounds__(kStepThreads, 1) advance_tables(const __grid_constant__ StepParams p) {
    extern __shared__ __align__(16) char smem[];
    __shared__ int64_t s_sum[3][kStepWarps];
    __shared__ int32_t s_free[kStepWarps];   // of every warp, then before it
    __shared__ int32_t s_count;              // free blocks that this CTA looks at
    __shared__ int32_t s_touched, s_freed;
    __shared__ uint32_t s_bad;
    __shared__ int32_t s_all_bad[kMaxCluster], s_all_freed[kMaxCluster];  // in the first CTA
    const uint32_t rank = cluster_rank(), size = cluster_size();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, S = p.num_seqs, T = p.block_tokens;
    const StepShared sh = step_shared(smem, p);
    if (tid == 0) s_touched = s_freed = 0, s_bad = 0;

    // ---- the free blocks
    const int64_t first_block = ((int64_t)rank * kStepWarps + warp) * p.warp_words * 32;
    uint32_t* const words = sh.free + warp * p.warp_words;
    int found = 0;
#pragma unroll 8
    for (int w = 0; w < p.warp_words; ++w) {
        const int64_t b = first_block + w * 32 + lane;
        const uint32_t word = __ballot_sync(~0u, b < p.num_blocks && p.refs[b] == 0);
        if (lane == 0) words[w] = word;
        found += __popc(word);
    }
    if (lane == 0) s_free[warp] = found;
    __syncthreads();

    // ---- what the sequences ask for, and the sums before each
    uint32_t bad = 0;
    int64_t run[3] = {0, 0, 0};
    for (int base = 0; base < S; base += kStepThreads) {
        const int s = base + tid;
        Need n{0, 0, 0, 0, false};
        if (s < S) {
            n = need_of(p, s, &bad);
            sh.first[s] = n.first;
            if (n.touched) sh.touched[atomicAdd(&s_touched, 1)] = s;
        }
        const int64_t own[3] = {n.blocks, n.rows, n.copy};
        int64_t incl[3] = {own[0], own[1], own[2]};
#pragma unroll
        for (int k = 0; k < 3; ++k) {
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int64_t up = __shfl_up_sync(~0u, incl[k], o);
                if (lane >= o) incl[k] += up;
            }
            if (lane == 31) s_sum[k][warp] = incl[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            int64_t warps = s_sum[k][lane];  // (as many warps as lanes)
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int64_t up = __shfl_up_sync(~0u, warps, o);
                if (lane >= o) warps += up;
            }
            const int64_t total = __shfl_sync(~0u, warps, 31), before = __shfl_sync(~0u, warps, max(warp - 1, 0));
            if (s < S) (k == 0 ? sh.blocks : k == 1 ? sh.rows : sh.copies)[s] =
                (int32_t)min(run[k] + (warp ? before : 0) + incl[k] - own[k], (int64_t)INT32_MAX);
            run[k] += total;
        }
        __syncthreads();
    }
    if (tid == 0) {
        sh.blocks[S] = (int32_t)min(run[0], (int64_t)INT32_MAX);
        sh.rows[S] = (int32_t)min(run[1], (int64_t)INT32_MAX);
        sh.copies[S] = (int32_t)min(run[2], (int64_t)INT32_MAX);
    }
    if (warp == 0) {
        const int own = s_free[lane];
        int incl = own;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int up = __shfl_up_sync(~0u, incl, o);
            if (lane >= o) incl += up;
        }
        s_free[lane] = incl - own;
        if (lane == 31) s_count = incl;
    }
    if (bad) atomicOr(&s_bad, bad);
    step_sync(size);

    // ---- who gets it: the sequences before the first that does not fit
    int n_free = 0, rank_before = 0;
    for (uint32_t r = 0; r < size; ++r) {
        const int n = size > 1 ? load_remote(&s_count, r) : s_count;
        if (r < rank) rank_before += n;
        n_free += n;
    }
    int fits = 0;
    for (int hi = S + 1; hi - fits > 1;) {  // the largest number of sequences that fits
        const int mid = (fits + hi) / 2;
        if (sh.blocks[mid] <= n_free && sh.rows[mid] <= p.num_rows && sh.copies[mid] <= p.pairs_cap) fits = mid;
        else hi = mid;
    }
    const int n_taken = sh.blocks[fits], n_rows = sh.rows[fits], n_copies = sh.copies[fits], n_touched = s_touched;
    const int all = size * kStepThreads, me = rank * kStepThreads + tid;
    auto have = [&](int s) {  // blocks that a growing sequence keeps or shares
        const bool copy = sh.copies[s + 1] > sh.copies[s];
        return copy ? sh.first[s] / T : (sh.first[s] + T - 1) / T;
    };
    // Counts down: a block with no count left was not this table's to give back.
    int freed = 0;
    auto give_back = [&](int b) {
        if (b < 0 || b >= p.num_blocks) {
            bad |= kBadBlock;
            return;
        }
        const int count = atomicAdd(&p.refs[b], -1);
        if (count <= 0) {
            atomicAdd(&p.refs[b], 1);
            bad |= kBadBlock;
        }
        freed += count == 1;
    };

    // ---- shared and given back blocks, sources of copies: everything that reads other sequences' rows of the table
    for_entries(
        p, sh, n_touched, rank, size,
        [&](int s) {
            if (p.parents && p.parents[s] >= 0) return make_int2(0, s < fits ? sh.first[s] / T : 0);
            return make_int2((p.new_lens[s] + T - 1) / T, (p.lens[s] + T - 1) / T);
        },
        [&](int s, int64_t place, int col) {
            const int parent = p.parents ? p.parents[s] : -1;
            if (parent < 0) {
                give_back(p.table[place]);
                return;
            }
            const int b = p.table[(int64_t)parent * p.max_blocks + col];
            p.table[place] = b;
            if (b < 0 || b >= p.num_blocks) bad |= kBadBlock;
            else freed -= atomicAdd(&p.refs[b], 1) == 0;  // (its last other user has just given it back)
        });
    if (n_copies > 0)
        for (int s = me; s < fits; s += all) {
            if (sh.copies[s + 1] == sh.copies[s]) continue;
            const int parent = p.parents ? p.parents[s] : -1;
            const int b = p.table[(int64_t)(parent >= 0 ? parent : s) * p.max_blocks + sh.first[s] / T];
            const bool there = b >= 0 && b < p.num_blocks;
            p.pairs[sh.copies[s]].x = there ? b : -1;
            if (!there) bad |= kBadBlock;
            if (parent < 0) give_back(b);
        }
    if (p.parents || p.pairs_cap > 0) step_sync(size);  // (without these no row is read that is not the reader's own)

    // ---- the free blocks to their sequences
    for_entries(
        p, sh, n_touched, rank, size,
        [&](int s) {
            if (p.parents && p.parents[s] >= 0) return make_int2(0, 0);
            return make_int2((p.new_lens[s] + T - 1) / T, (p.lens[s] + T - 1) / T);
        },
        [&](int, int64_t place, int) { p.table[place] = -1; });
    int r0 = rank_before + s_free[warp];
    for (int w = 0; w < p.warp_words && r0 < n_taken; ++w) {
        const uint32_t word = words[w];
        const int r = r0 + __popc(word & ((1u << lane) - 1));
        if (word >> lane & 1u && r < n_taken) {
            const int b = (int)(first_block + w * 32 + lane), s = last_at_most(sh.blocks, fits, r), j = r - sh.blocks[s];
            p.table[(int64_t)s * p.max_blocks + have(s) + j] = b;
            p.refs[b] = 1;
            if (j == 0 && sh.copies[s + 1] > sh.copies[s]) p.pairs[sh.copies[s]].y = b;
        }
        r0 += __popc(word);
    }
    if (bad) atomicOr(&s_bad, bad);
    if (freed) atomicAdd(&s_freed, freed);
    __syncthreads();
    if (size > 1) {
        if (tid == 0) store_remote(&s_all_bad[rank], 0, (int32_t)s_bad), store_remote(&s_all_freed[rank], 0, s_freed);
    } else if (tid == 0) {
        s_all_bad[0] = (int32_t)s_bad, s_all_freed[0] = s_freed;
    }
    step_sync(size);

    // ---- rows, lengths, counts
    if (p.starts)
        for (int s = me; s <= S; s += all) p.starts[s] = sh.rows[min(s, fits)];
    for (int s = me; s < S; s += all) {
        const int old = p.lens[s], now = p.new_lens[s];
        const bool grows = now > old || (p.parents && p.parents[s] >= 0);
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
                    const int b = __ldcg(&p.table[(int64_t)s * p.max_blocks + index / T]);
                    if (b >= 0 && b < p.num_blocks) slot = (int64_t)b * T + index % T;
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
    p.max_len = (int32_t)std::min<int64_t>((int64_t)a.max_blocks_per_seq * layout->block_tokens, kMaxTokens);
    const DeviceInfo dev = cached_device_info();
    if (!dev.sms) return AMOEBA_ERR_CUDA;
    const int cluster = p.num_blocks <= 4096 && p.num_seqs <= kStepThreads && p.num_rows <= 4 * kStepThreads ? 1 : kMaxCluster;
    p.warp_words = (int32_t)(((int64_t)p.num_blocks + cluster * kStepThreads - 1) / (cluster * kStepThreads));
    const int64_t smem = step_smem(p.num_seqs, p.warp_words);
    if (smem > dev.smem_optin - 2048) return AMOEBA_ERR_TOO_LARGE;
    return launch_clusters(advance_tables, cluster, kStepThreads, (size_t)smem, cluster, false, static_cast<cudaStream_t>(cuda_stream), p);
}
