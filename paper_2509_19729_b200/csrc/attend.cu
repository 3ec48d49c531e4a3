// amoeba_attend: attention of a ragged chunk of new tokens over the paged cache.
//
// One unit of work is a (sequence, key head, tile of query rows), the rows of a unit being the new tokens times the
// query heads that share the key head, so that grouped heads read their keys once.  The softmax runs along the tokens
// with a running maximum and sum per row; units are cut where the shares of the CTAs end (walk.cuh), and the cut ones
// are joined by their maxima and sums in a second small launch.
#include "attend.cuh"
#include "warp_mma.cuh"

namespace amoeba {

constexpr int kMaxFewRows = 32;   // rows of a unit of attend_few
constexpr int kMaxGroupRows = 8;  // of a group by attend_few
constexpr int kUnitStart = 3;     // tiles of 64 tokens that a unit's start and end cost: 5000 clocks, 1660 a tile that is in flight already

// ------------------------------------------------------------------------------------------------ groups' numbers
// What the sequences of a group come to; the warp together.
struct GroupSums {
    int32_t first, end;        // sequences; none if the numbers are bad
    int32_t q0, q1, row;       // rows, and the first sequence that has any
    int32_t with_rows, least;  // sequences with rows, and the fewest tokens in front of the new ones
    int32_t alone, taking;     // what a tile of the prefix costs all sequences by themselves, and what joining their sums with the group's does
    bool ok;
};
// What a tile of 128 tokens costs so many rows of attend_many, in tiles of 128 rows: the last, of up to 128, is half as large.
__device__ __forceinline__ int rows_cost(int rows) { return rows / kManyRows * 2 + (rows % kManyRows > 128 ? 2 : rows % kManyRows > 0); }
__device__ __forceinline__ GroupSums sum_group(const Batch& b, const int32_t* group_starts, int g, int block_tokens, int heads, int few_cost) {
    GroupSums x{group_starts[g], group_starts[g + 1], INT32_MAX, 0, INT32_MAX, 0, INT32_MAX, 0, 0, true};
#pragma unroll 4
    for (int s = x.first + (int)threadIdx.x % 32; s < x.end; s += 32) {
        const Seq q = sequence(b, s, block_tokens);
        x.ok &= q.ok;
        if (q.qn == 0) continue;
        const bool few = q.qn * heads <= kMaxFewRows;
        x.least = min(x.least, q.len - q.qn);
        x.row = min(x.row, s);
        x.q0 = min(x.q0, q.q0);
        x.q1 = max(x.q1, q.q0 + q.qn);
        x.alone += few ? few_cost : rows_cost(q.qn * heads);
        x.taking += few ? 1 : 5 * rows_cost(q.qn * heads);
        ++x.with_rows;
    }
    x.ok = __all_sync(~0u, x.ok);
    x.least = __reduce_min_sync(~0u, x.least);
    x.row = __reduce_min_sync(~0u, x.row);
    x.with_rows = __reduce_add_sync(~0u, x.with_rows);
    x.q0 = __reduce_min_sync(~0u, x.q0);
    x.q1 = __reduce_max_sync(~0u, x.q1);
    x.alone = __reduce_add_sync(~0u, x.alone);
    x.taking = __reduce_add_sync(~0u, x.taking);
    return x;
}
// Whether a group's numbers are refused.
__device__ __forceinline__ bool refused(const GroupSums& x, int prefix, int max_group_rows) {
    return x.end > x.first && (prefix < 0 || (x.with_rows > 0 && x.q1 - x.q0 > max_group_rows));
}
// Whether the groups' sequences are in order; the block together.
__device__ __forceinline__ bool groups_in_order(const int32_t* starts, int groups, int num_seqs) {
    bool bad = false;
    for (int g = threadIdx.x; g < groups; g += blockDim.x) bad |= starts[g] < 0 || starts[g + 1] < starts[g] || starts[g + 1] > num_seqs;
    return !__syncthreads_or(bad);
}
// All that is reported of groups, where nothing is shared.
template <class B>
__device__ void check_groups(const AttendParams<B>& p) {
    const SharedBatch& b = p.batch;
    bool bad = !groups_in_order(b.group_starts, b.num_groups, b.num_seqs);
    for (int g = threadIdx.x / 32; !bad && g < b.num_groups; g += blockDim.x / 32)
        bad = refused(sum_group(b, b.group_starts, g, p.cache.block_tokens, p.shape.group, 0), b.prefix_lens[g], b.max_group_rows);
    if (bad) report(p.status, AMOEBA_ERR_INVALID_ARG);
}

// ------------------------------------------------------------------------------------------------ few rows
// Up to 8*NT rows a unit.  Bound by the bytes of the cache: 2 * 2 * D a token and key head against at most 32 rows of
// arithmetic, which warp-level matrix instructions do in a fraction of the time.  Every warp works alone on every
// fourth run of 16 tokens, with its own ring of asynchronous loads and its own running maximum, sum and output, so
// that nothing but the end of a unit makes warps wait for one another.  The product is formed the other way round,
// S^T = K Q^T and O^T = V^T P^T: then 8 rows fill a matrix instruction, where 16 would be needed the usual way.  The weights are
// rounded to the element type for the second product, half a step of it, which is what the output is rounded by too.
// Measured: 128 sequences of 512 to 8192 tokens, 8 key heads of 128, one row each: 340 us, 6.28 TB/s (96 % of a copy's
// rate); about 5 us of it before the loads run at full rate, and as much for the last units and the join.
constexpr int kFewThreads = 128, kFewWarps = 4, kFewTile = 16 * kFewWarps;
template <int D, int NT>
struct FewShape {
    static constexpr int kStage = 2 * 16 * D * 2;  // 16 tokens' keys and values
    static constexpr int kMerge = kFewWarps * 8 * NT * (D + 4) * 4;
    static constexpr int kCtas = NT * D > 128 ? 1 : 2;  // per SM
    static constexpr int kStages = D == 64 ? 4 : NT == 1 ? 3 : NT == 2 ? 6 : 4;
    static constexpr int kSmem = kFewWarps * kStages * kStage + kMerge;
};

template <class T, int D, int NT, class B>
__global__ void __launch_bounds__(kFewThreads, FewShape<D, NT>::kCtas)
attend_few(const __grid_constant__ AttendParams<B> p) {
    using F = FewShape<D, NT>;
    constexpr int R = 8 * NT, kSteps = D / 16, kPitch = D + 4;
    extern __shared__ __align__(128) char smem[];
    __shared__ uint32_t s_mask[kFewWarps][F::kStages];
    __shared__ float s_m[kFewWarps][R], s_l[kFewWarps][R];
    float* s_o = reinterpret_cast<float*>(smem + kFewWarps * F::kStages * F::kStage);
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int quad = lane / 4, pair = lane % 4;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * F::kStages * F::kStage;
    const Shape& sh = p.shape;

    Walk walk{};
    int64_t n;
    if constexpr (B::kShared) {
        if (p.batch.waits) grid_dependency_wait();
        if (p.batch.check_blocks() && blockIdx.x == gridDim.x - 1) return check_groups(p);
    }
    if (p.whole) {
        walk.open(sh, p.batch, p.cache.block_tokens, blockIdx.x / sh.kv_heads);
        if (!walk.seq.ok && tid == 0) report(p.status, AMOEBA_ERR_INVALID_ARG);
        walk.h = blockIdx.x % sh.kv_heads;
        n = walk.nm ? walk.range.tiles : 0;
    } else {
        int64_t begin, end;
        if constexpr (B::kShared)
            take_weighted_share<kFewThreads>(sh, p.batch, p.cache.block_tokens, &walk, &begin, &end, p.status, smem,
                                             p.batch.split && !p.batch.by_groups() ? __ldcg(p.batch.split + 1) : (int)gridDim.x - p.batch.check_blocks());
        else
            take_share<kFewThreads>(sh, p.batch, p.cache.block_tokens, &walk, &begin, &end, p.status);
        write_cut(sh, p.cuts, walk, begin, end);
        n = end - begin;
    }
    grid_dependency_launch();
    if (n == 0) {
        if (B::kShared) grid_dependency_wait();  // (what ends behind this kernel ends behind those in front of it too)
        return;
    }

    Ahead<D, true, kFewTile, B> ahead(p.cache, p.batch, sh, p.status, walk, n, warp * 16);
    int slot_in = 0, slot = 0;
    auto load = [&] {
        if (ahead.left > 0) {
            int64_t first;
            const uint32_t mask = ahead.load(ring + slot_in * F::kStage, &first);
            if (lane == 0) s_mask[warp][slot_in] = mask;
        }
        cp_async_commit();
        slot_in = slot_in + 1 == F::kStages ? 0 : slot_in + 1;
    };
#pragma unroll
    for (int i = 0; i < F::kStages - 1; ++i) load();

    uint32_t qf[NT][kSteps][2];     // Q^T, the right operand of S^T = K Q^T
    int see_lo[NT][2], see_hi[NT][2];  // tokens that this lane's rows see: [lo, hi)
    float m_run[NT][2], l_run[NT][2], o[NT][kSteps][4];
    bool fresh = true;
    bool from_start = false;  // of the unit, in this CTA

    for (; n > 0; --n) {
        if (fresh) {
            fresh = false;
            from_start = walk.t == 0;
            const int rows = walk.seq.qn * sh.group, first = walk.m * R;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int r = first + t * 8 + quad;
                const bool there = r < rows;
                const char* src = there ? row_of<D>(p.q, p, walk.seq, walk.h, r) : nullptr;
#pragma unroll
                for (int j = 0; j < kSteps; ++j)
#pragma unroll
                    for (int b = 0; b < 2; ++b)
                        qf[t][j][b] = there ? *reinterpret_cast<const uint32_t*>(src + (j * 16 + b * 8 + pair * 2) * 2) : 0u;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int rr = first + t * 8 + pair * 2 + b;
                    const int pos = last_seen(walk.seq, rr / sh.group);
                    see_hi[t][b] = rr < rows ? pos + 1 : 0;
                    see_lo[t][b] = sh.window > 0 ? pos - sh.window + 1 : 0;
                    m_run[t][b] = -INFINITY;
                    l_run[t][b] = 0.f;
                }
#pragma unroll
                for (int j = 0; j < kSteps; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[t][j][i] = 0.f;
            }
        }
        cp_async_wait<F::kStages - 2>();
        __syncwarp();
        load();  // into the slot that the last round has read
        __syncwarp();  // the matrix instructions want the warp together
        const uint32_t k_smem = ring + slot * F::kStage, v_smem = k_smem + 16 * D * 2;
        const uint32_t mask = s_mask[warp][slot];
        slot = slot + 1 == F::kStages ? 0 : slot + 1;

        float st[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t) st[t][0] = st[t][1] = st[t][2] = st[t][3] = 0.f;
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            uint32_t a[4];
            ldmatrix4(a, k_smem + swizzled<D>(lane % 16, 2 * j + lane / 16));
#pragma unroll
            for (int t = 0; t < NT; ++t) mma16816<T>(st[t], a, qf[t][j][0], qf[t][j][1]);
        }
        // st[t]: tokens quad and quad + 8, rows 2*pair and 2*pair + 1
        const int key0 = walk.range.base + walk.t * kFewTile + warp * 16 + quad;
        uint32_t pf[NT][2];
        bool grew = false;
        float alpha[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = key0 + (i / 2) * 8;
                const bool sees = (mask >> (quad + (i / 2) * 8) & 1u) && key < see_hi[t][i % 2] && key >= see_lo[t][i % 2];
                st[t][i] = sees ? st[t][i] * p.scale_log2 : -INFINITY;
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                float top = fmaxf(st[t][b], st[t][b + 2]);
                top = fmaxf(top, __shfl_xor_sync(~0u, top, 4));
                top = fmaxf(top, __shfl_xor_sync(~0u, top, 8));
                top = fmaxf(top, __shfl_xor_sync(~0u, top, 16));
                const float m_new = fmaxf(m_run[t][b], top);
                grew |= m_new > m_run[t][b];
                const float ref = m_new == -INFINITY ? 0.f : m_new;
                alpha[t][b] = fast_exp2(m_run[t][b] - ref);
                m_run[t][b] = m_new;
                st[t][b] = fast_exp2(st[t][b] - ref);
                st[t][b + 2] = fast_exp2(st[t][b + 2] - ref);
                l_run[t][b] = l_run[t][b] * alpha[t][b] + st[t][b] + st[t][b + 2];
            }
            pf[t][0] = transpose8x8(Elem<T>::pack(st[t][0], st[t][1]));
            pf[t][1] = transpose8x8(Elem<T>::pack(st[t][2], st[t][3]));
        }
        if (__any_sync(~0u, grew)) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int j = 0; j < kSteps; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[t][j][i] *= alpha[t][i % 2];
        }
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            uint32_t a[4];
            ldmatrix4_trans(a, v_smem + swizzled<D>(lane % 8 + lane / 16 * 8, 2 * j + lane / 8 % 2));
#pragma unroll
            for (int t = 0; t < NT; ++t) mma16816<T>(o[t][j], a, pf[t][0], pf[t][1]);
        }

        const bool unit_ends = walk.t + 1 == walk.range.tiles;
        if (!unit_ends && n > 1) {
            ++walk.t;
            continue;
        }
        // The unit, or this CTA's part of it, ends: join the four warps.
        fresh = true;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                float l = l_run[t][b];
                l += __shfl_xor_sync(~0u, l, 4);
                l += __shfl_xor_sync(~0u, l, 8);
                l += __shfl_xor_sync(~0u, l, 16);
                const int r = t * 8 + pair * 2 + b;
                if (quad == 0) s_m[warp][r] = m_run[t][b], s_l[warp][r] = l;
#pragma unroll
                for (int j = 0; j < kSteps; ++j) {
                    float* to = s_o + (warp * R + r) * kPitch + j * 16 + quad;
                    to[0] = o[t][j][b];
                    to[8] = o[t][j][b + 2];
                }
            }
        __syncthreads();
        const int rows = min(R, walk.seq.qn * sh.group - walk.m * R);
        const bool direct = from_start && unit_ends;
        const int64_t part = (int64_t)(2 * blockIdx.x + (from_start ? 1 : 0)) * R;
        for (int i = tid; i < rows * (D / 4); i += kFewThreads) {
            const int r = i / (D / 4), d = i % (D / 4) * 4;
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < kFewWarps; ++w) top = fmaxf(top, s_m[w][r]);
            const float ref = top == -INFINITY ? 0.f : top;
            Joined j;
            j.top = top;
#pragma unroll
            for (int w = 0; w < kFewWarps; ++w) {
                const float f = fast_exp2(s_m[w][r] - ref);
                const float4 x = *reinterpret_cast<const float4*>(s_o + (w * R + r) * kPitch + d);
                j.l += f * s_l[w][r];
                j.acc.x += f * x.x, j.acc.y += f * x.y, j.acc.z += f * x.z, j.acc.w += f * x.w;
            }
            if (goes_on(p, walk.seq) && d == 0 && from_start && !direct) p.sums.l[head_of(p, walk.seq, walk.h, walk.m * R + r)] = kCutRow;
            if (direct && goes_on(p, walk.seq)) {
                write_sums<D>(p, walk.seq, walk.h, walk.m * R + r, d, j);
            } else if (direct) {
                write_row<T, D>(p, walk.seq, walk.h, walk.m * R + r, d, j);
            } else {
                *reinterpret_cast<float4*>(p.part_o + (part + r) * D + d) = j.acc;
                if (d == 0) p.part_m[part + r] = top, p.part_l[part + r] = j.l;
            }
        }
        __syncthreads();
        if (n > 1) walk.next(sh, p.batch, p.cache.block_tokens);
    }
    if (B::kShared) grid_dependency_wait();
}

// ------------------------------------------------------------------------------------------------ joining
// Joins the parts of the units that were cut, by their maxima and sums; in order, so the same call gives the same bits.  kWarps
// warps to a row: with few rows a unit may be in as many parts as there are CTAs, so eight warps take every eighth part each;
// with many rows a warp does four rows, and walks all parts of each: two or three, as long as there are units enough, but up to
// one for each CTA where a few units of many rows run over a long cache.  Bound by its few dependent loads: 9 us by itself for 296
// shares of 8 rows, of which the launch in front hides a part.
constexpr int kJoinWarps = 8, kJoinThreads = 32 * kJoinWarps;
template <int kWarps>
constexpr int kJoinRows = kWarps == 1 ? 4 * kJoinWarps : 1;  // of a block

// `groups` blocks to every share: the unit that it begins in is joined there, if that began in the share before; with what `prefix` adds
// to a row.
template <class T, int D, int kWarps, class B, class Prefix>
__device__ __forceinline__ void join_rows(const AttendParams<B>& p, int ctas, int block, int groups, Prefix prefix) {
    constexpr int kRows = kJoinRows<kWarps>, kLanes = D / 4, kAtOnce = 32 / kLanes;  // lanes to a part's row, parts at once
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int mine = block / groups, first_row = block % groups * kRows, R = p.shape.rows;
    const Cut cut = p.cuts[mine];
    if (cut.begin == cut.end || cut.t == 0 || first_row >= cut.rows) return;
    const int64_t first = cut.begin - cut.t, last = first + cut.tiles;
    const Seq q = sequence(p.batch, cut.s, p.cache.block_tokens);
    int c0 = mine - 1;
    while (p.cuts[c0].begin == p.cuts[c0].end) --c0;  // (empty shares)
    if (p.cuts[c0].begin > first) return;
    int c1 = mine;  // behind the last part
    for (bool more = true; more; c1 += 32) {
        const unsigned in = __ballot_sync(~0u, c1 + lane < ctas && p.cuts[c1 + lane].begin < last);
        more = in == ~0u;
        if (!more) c1 += __popc(in) - 32;
    }
#pragma unroll
    for (int i = 0; i < kRows; i += kJoinWarps) {
        const int r = first_row + (kWarps == 1 ? i + warp : 0);
        Joined j;
        if (r < cut.rows) {
#pragma unroll (kWarps == 1 ? 2 : 8)
            for (int c = c0 + (kWarps == 1 ? 0 : warp) * kAtOnce + lane / kLanes; c < c1; c += kWarps * kAtOnce) {
                if (p.cuts[c].begin == p.cuts[c].end) continue;
                const int64_t part = (int64_t)(2 * c + (c == c0)) * R + r;
                j.add(p.part_m[part], p.part_l[part], *reinterpret_cast<const float4*>(p.part_o + part * D + lane % kLanes * 4));
            }
            prefix(q, cut.h, cut.m * R + r, (kWarps == 1 ? 0 : warp) * kAtOnce + lane / kLanes, kWarps * kAtOnce, j);
        }
        if (kAtOnce == 2) j.add_lower_half();  // the second half of the warp has every other part
        if (kWarps > 1) {
            __shared__ float4 s_acc[kWarps][kLanes];
            __shared__ float s_top[kWarps], s_l[kWarps];
            if (lane < kLanes) s_acc[warp][lane] = j.acc;
            if (lane == 0) s_top[warp] = j.top, s_l[warp] = j.l;
            __syncthreads();
            if (warp) return;
            for (int w = 1; w < kWarps; ++w) j.add(s_top[w], s_l[w], s_acc[w][lane % kLanes]);
        }
        if (r >= cut.rows || lane >= kLanes) continue;
        if (q.level) write_sums<D>(p, q, cut.h, cut.m * R + r, lane * 4, j);
        else write_row<T, D>(p, q, cut.h, cut.m * R + r, lane * 4, j);
    }
}
// Blocks [0, few_ctas * few_rows) join what attend_few has cut, the others what attend_many has.
template <class T, int D, class B>
__global__ void __launch_bounds__(kJoinThreads) attend_join(const __grid_constant__ AttendParams<B> few, int few_ctas, int few_rows,
                                                            const __grid_constant__ AttendParams<B> many, int many_ctas) {
    grid_dependency_wait();
    const int block = (int)blockIdx.x - few_ctas * few_rows;
    auto none = [](const Seq&, int, int, int, int, Joined&) {};
    if (block < 0) join_rows<T, D, kJoinWarps>(few, few_ctas, blockIdx.x, few_rows, none);
    else join_rows<T, D, 1>(many, many_ctas, block, kManyRows / kJoinRows<1>, none);
}

// What the groups' pass has left: sums of whole rows, and where it was attend_many's the parts of its cut units.
struct PrefixSums {
    Sums rows, parts;
    const Group* groups;
    const int64_t* tile0;
    const int32_t* row_group;  // [num_rows] -1: none
    const int32_t* split;      // where the groups' pass was attend_many's: its CTAs
    int32_t num_groups, num_rows;
    int32_t row_warps;         // warps of attend_finish to a row
};
// What is to be known of a group to find its parts; the loads in two steps.
struct PrefixPlace {
    int32_t ctas = 0;
    int64_t total = 0, tile0 = 0;
    int4 group = {0, 0, 0, 0};

    __device__ __forceinline__ void all(const PrefixSums& x) {
        if (x.split) ctas = __ldcg(x.split), total = __ldcg(x.tile0 + x.num_groups);
    }
    __device__ __forceinline__ void of(const PrefixSums& x, int g) {
        if (x.split) group = __ldcg(reinterpret_cast<const int4*>(x.groups + g)), tile0 = __ldcg(x.tile0 + g);
    }
};
// Adds the prefix's sums of a row (of a kv head's, from the first of the sequence) to j: every step-th part from `first` on.
template <int D, class B>
__device__ __forceinline__ void add_prefix(const AttendParams<B>& p, const PrefixSums& x, const PrefixPlace& at_group, const Seq& q, int kv_head, int row,
                                           int first, int step, Joined& j) {
    const int d = (int)threadIdx.x % 32 % (D / 4) * 4, tok = row / p.shape.group;
    if (x.split) {
        const int4 group = at_group.group;
        const int64_t even = divide(at_group.total + at_group.ctas - 1, at_group.ctas);
        const int tiles = (group.z - 1) / kManyTile + 1, row_tiles = (int)(((int64_t)group.y * p.shape.group - 1) / kManyRows) + 1;
        const int in_group = (q.q0 - group.x) * p.shape.group + row, m = in_group / kManyRows, r = in_group % kManyRows;
        const int64_t begin = at_group.tile0 + ((int64_t)kv_head * row_tiles + m) * tiles;
        const int c0 = (int)divide(begin, even), c1 = (int)divide(begin + tiles - 1, even);
        if (c0 < c1) {
#pragma unroll 4
            for (int c = c0 + first; c <= c1; c += step) {
                const int64_t part = (int64_t)(2 * c + (c == c0)) * kManyRows + r;
                j.add(x.parts.m[part], x.parts.l[part], *reinterpret_cast<const float4*>(x.parts.o + part * D + d));
            }
            return;
        }
    }
    const int64_t at = (int64_t)(q.q0 + tok) * p.q_heads + kv_head * p.shape.group + row - tok * p.shape.group;
    if (first == 0) j.add(x.rows.m[at], x.rows.l[at], *reinterpret_cast<const float4*>(x.rows.o + at * D + d));
}
// The cut units of attend_few, a block to a share as in join_rows: a warp to a row if it is in few parts, else all of them.
template <class T, int D, class Prefix>
__device__ __forceinline__ void finish_cut(const AttendParams<SharedBatch>& p, int ctas, int mine, Prefix prefix) {
    constexpr int kLanes = D / 4, kAtOnce = 32 / kLanes, kMost = 32;  // parts of a row for one warp
    __shared__ float4 s_acc[kJoinWarps][kLanes];
    __shared__ float s_top[kJoinWarps], s_l[kJoinWarps];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, R = p.shape.rows;
    const Cut cut = p.cuts[mine];
    if (cut.begin == cut.end || cut.t == 0) return;
    const int64_t first = cut.begin - cut.t, last = first + cut.tiles;
    const Seq q = sequence(p.batch, cut.s, p.cache.block_tokens);
    int c0 = mine - 1;
    while (p.cuts[c0].begin == p.cuts[c0].end) --c0;  // (empty shares)
    if (p.cuts[c0].begin > first) return;
    int c1 = mine;  // behind the last part
    for (bool more = true; more; c1 += 32) {
        const unsigned in = __ballot_sync(~0u, c1 + lane < ctas && p.cuts[c1 + lane].begin < last);
        more = in == ~0u;
        if (!more) c1 += __popc(in) - 32;
    }
    const bool alone = c1 - c0 <= kMost;
    const int begin = (alone ? 0 : warp) * kAtOnce + lane / kLanes, step = (alone ? 1 : kJoinWarps) * kAtOnce;
    for (int r = alone ? warp : 0; r < cut.rows; r += alone ? kJoinWarps : 1) {
        Joined j;
#pragma unroll 4
        for (int c = c0 + begin; c < c1; c += step) {
            if (p.cuts[c].begin == p.cuts[c].end) continue;
            const int64_t part = (int64_t)(2 * c + (c == c0)) * R + r;
            j.add(p.part_m[part], p.part_l[part], *reinterpret_cast<const float4*>(p.part_o + part * D + lane % kLanes * 4));
        }
        prefix(q, cut.h, cut.m * R + r, begin, step, j);
        if (kAtOnce == 2) j.add_lower_half();
        if (!alone) {
            if (lane < kLanes) s_acc[warp][lane] = j.acc;
            if (lane == 0) s_top[warp] = j.top, s_l[warp] = j.l;
            __syncthreads();
            for (int w = 1; warp == 0 && w < kJoinWarps; ++w) j.add(s_top[w], s_l[w], s_acc[w][lane % kLanes]);
            __syncthreads();
        }
        if ((alone || warp == 0) && lane < kLanes) write_row<T, D>(p, q, cut.h, cut.m * R + r, lane * 4, j);
    }
}
// The end of both passes: what was cut of the sequences', with the prefixes' sums where there are any; then x.row_warps warps to a row
// for the rows with a prefix whose own tokens were not cut, kHeads query heads at a time, whose loads of their own sums overlap.  Bound by four or five loads one after the other: 12 us
// by itself for 128 rows of 32 heads, whose prefixes are in 5 to 10 parts, of which the launch in front hides some.
// Four blocks to an SM, 64 registers (the whole call 115.4 us; three 116.5, five and six, which spill, 116.3 and 117.2).
template <class T, int D, int kHeads>
__global__ void __launch_bounds__(kJoinThreads, kHeads == 1 ? 4 : 3) attend_finish(const __grid_constant__ AttendParams<SharedBatch> few, int few_ctas,
                                                              const __grid_constant__ AttendParams<SharedBatch> many, int many_ctas,
                                                              const __grid_constant__ PrefixSums x) {
    constexpr int kLanes = D / 4, kAtOnce = 32 / kLanes;
    grid_dependency_wait();
    auto prefix = [&](const Seq& q, int kv_head, int row, int first, int step, Joined& j) {
        if (q.first <= 0) return;
        PrefixPlace at;
        at.all(x), at.of(x, q.group);
        add_prefix<D>(few, x, at, q, kv_head, row, first, step, j);
    };
    const int many_groups = kManyRows / kJoinRows<1>;
    int block = blockIdx.x;
    if (block < few_ctas) return finish_cut<T, D>(few, few_ctas, block, prefix);
    block -= few_ctas;
    if (block < many_ctas * many_groups) return join_rows<T, D, 1>(many, many_ctas, block, many_groups, prefix);
    block -= many_ctas * many_groups;
    const int64_t warp = (int64_t)block * kJoinWarps + threadIdx.x / 32;
    const int row = (int)(warp / x.row_warps), first = (int)(warp - (int64_t)row * x.row_warps), stride = x.row_warps;
    const int lane = threadIdx.x % 32, half = lane / kLanes, d = lane % kLanes * 4;
    PrefixPlace place;
    place.all(x);
    const int g = row < x.num_rows ? x.row_group[row] : -1;
    if (g < 0) return;
    place.of(x, g);
    for (int head0 = first; head0 < few.q_heads; head0 += kHeads * stride) {
        float l[kHeads], m[kHeads];
        float4 o[kHeads];
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
            const int64_t at = (int64_t)row * few.q_heads + min(head0 + i * stride, few.q_heads - 1);
            l[i] = few.sums.l[at], m[i] = few.sums.m[at], o[i] = *reinterpret_cast<const float4*>(few.sums.o + at * D + d);
        }
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
            const int head = head0 + i * stride;
            if (head >= few.q_heads || l[i] == kCutRow) continue;  // (of a cut row only l is there)
            const int kv_head = head / few.shape.group, r = head - kv_head * few.shape.group;
            Seq q{};
            q.q0 = row;
            Joined j;
            if (half == 0) j.add(m[i], l[i], o[i]);
            add_prefix<D>(few, x, place, q, kv_head, r, half, kAtOnce, j);
            if (kAtOnce == 2) j.add_lower_half();
            if (half == 0) write_row<T, D>(few, q, kv_head, r, d, j);
        }
    }
}

// The workspace holds the parts of cut units, two for each CTA; these bound the grids without asking the device.
constexpr int kMaxFewCtas = 2 * kMaxSms;

// One kernel's part of the workspace: where the shares begin, then the parts.
template <class B>
static int64_t workspace_part(AttendParams<B>* p, char* ws, int64_t parts, int64_t rows, int head_dim) {
    const int64_t o = kMaxFewCtas * (int64_t)sizeof(Cut), m = o + parts * rows * head_dim * 4, l = m + parts * rows * 4;
    if (p) {
        p->cuts = reinterpret_cast<Cut*>(ws);
        p->part_o = reinterpret_cast<float*>(ws + o);
        p->part_m = reinterpret_cast<float*>(ws + m);
        p->part_l = reinterpret_cast<float*>(ws + l);
    }
    return l + parts * rows * 4;
}
template <class B>
static int64_t few_workspace(AttendParams<B>* p, char* ws, int head_dim) {
    return workspace_part(p, ws, 2 * kMaxFewCtas, kMaxFewRows, head_dim);
}
template <class B>
static int64_t many_workspace(AttendParams<B>* p, char* ws, int head_dim) {
    return workspace_part(p, ws, 2 * kMaxSms, kManyRows, head_dim);
}
static int64_t rows_of(const amoeba_layout* l, int32_t max_q_len) {
    return (int64_t)max_q_len * (l->model.num_q_heads / l->model.num_kv_heads);
}

template <class T, int D, int NT, class B>
static amoeba_status run_few(AttendParams<B>& p, int sms, int* ctas, cudaStream_t stream) {
    using F = FewShape<D, NT>;
    p.shape.rows = 8 * NT;
    p.shape.tile = kFewTile;
    p.shape.start = kUnitStart;
    if (ensure_dynamic_smem((const void*)attend_few<T, D, NT, B>, F::kSmem) != cudaSuccess) return AMOEBA_ERR_CUDA;
    *ctas = std::min(F::kCtas * sms, kMaxFewCtas);
    return launch_kernel(attend_few<T, D, NT, B>, (p.whole ? p.batch.num_seqs * p.shape.kv_heads : *ctas) + p.batch.check_blocks(),
                         kFewThreads, F::kSmem, stream, B::kShared, p);
}

// The launches of a pass, and what is left for the join behind them.
template <class B>
struct Pass {
    AttendParams<B> few, many;
    int few_ctas = 0, few_rows = 0, many_ctas = 0;
    bool cuts = false;  // something may be cut
    int many_blocks() const { return many_ctas * (kManyRows / kJoinRows<1>); }
};

// Sequences with few rows (new tokens times query heads per key head) are read by attend_few, whose time is that of reading
// the cache; the others by attend_many.  Which there are is known only on the device: a batch that may hold longer
// ones gets both, and each skips the other's.  The launches follow one another closely: a kernel's blocks may be in place
// before the kernel in front of it ends, and wait there for its results if they read them (attend_join) or end only after
// it (attend_many).
template <class T, int D, class B>
static amoeba_status run_pass(AttendParams<B>& p, int tp, int32_t dtype, char* ws, int sms, cudaStream_t stream, Pass<B>* pass) {
    const int64_t rows = (int64_t)p.batch.max_q_len * p.shape.group;
    const int64_t few_bytes = few_workspace(&p, ws, D);
    // In a batch with longer pieces attend_few gets the single tokens (and what has as few rows): its rows cost registers.  Groups
    // all go to one kernel: small ones beside large ones are not worth a launch.
    const bool groups = p.batch.by_groups(), few = !groups || rows <= kMaxGroupRows;
    const int64_t few_rows = rows <= kMaxFewRows ? rows : p.shape.group;
    const int most = !few ? 0 : few_rows <= 8 ? 8 : few_rows <= 16 ? 16 : kMaxFewRows;
    p.shape.min_rows = 0;
    p.shape.max_rows = most;
    amoeba_status st = !few         ? AMOEBA_OK
                       : most == 8  ? run_few<T, D, 1>(p, sms, &pass->few_ctas, stream)
                       : most == 16 ? run_few<T, D, 2>(p, sms, &pass->few_ctas, stream)
                                    : run_few<T, D, 4>(p, sms, &pass->few_ctas, stream);
    if (st != AMOEBA_OK) return st;
    if (p.whole) pass->few_ctas = 0;  // nothing is cut
    pass->few_rows = (int)std::min<int64_t>(rows, most);
    pass->cuts = !p.whole || rows > kMaxFewRows;
    pass->few = pass->many = p;
    if (few && rows <= kMaxFewRows) return AMOEBA_OK;
    AttendParams<B>& many = pass->many;
    many_workspace(&many, ws + few_bytes, D);
    many.shape.min_rows = most + 1;
    many.shape.max_rows = INT32_MAX;
    many.shape.rows = kManyRows;
    many.shape.tile = kManyTile;
    pass->many_ctas = std::min(sms, kMaxSms);
    return launch_attend_many(many, tp, dtype, D, pass->many_ctas, stream);
}
template <class T, int D, class B>
static amoeba_status run_join(const Pass<B>& x, cudaStream_t stream) {
    if (!x.cuts) return AMOEBA_OK;
    return launch_kernel(attend_join<T, D, B>, x.few_ctas * x.few_rows + x.many_blocks(), kJoinThreads, 0, stream, true, x.few, x.few_ctas,
                         x.few_rows, x.many, x.many_ctas);
}
// Short sequences are not worth cutting: what the shares and the join take, about 5 us, is what a CTA needs for 512
// tokens, or for 1024 when there are units enough to fill the GPU (one sequence of 256 tokens, 8 key heads: 7.9 us whole,
// 9.5 cut; of 1024: 20.5 and 11.3; 32 sequences of 1024: 24 and 29; of 2048: 41 and 47, but there one long one would
// hold up all).  With max_q_len 0 sequences are only looked at.
template <class B>
static bool not_cut(const AttendParams<B>& p, int sms) {
    const int64_t tokens = (int64_t)p.batch.max_blocks * p.cache.block_tokens;
    return p.batch.max_q_len == 0 || tokens <= 512 || (tokens <= 1024 && (int64_t)p.batch.num_seqs * p.shape.kv_heads >= sms);
}
template <class T, int D>
static amoeba_status run_attend(AttendParams<Batch>& p, int tp, int32_t dtype, char* ws, int sms, cudaStream_t stream) {
    Pass<Batch> x;
    p.whole = not_cut(p, sms);
    const amoeba_status st = run_pass<T, D>(p, tp, dtype, ws, sms, stream, &x);
    return st != AMOEBA_OK ? st : run_join<T, D>(x, stream);
}

}  // namespace amoeba

using namespace amoeba;

extern "C" amoeba_status amoeba_attend_workspace_bytes(const amoeba_layout* layout, const amoeba_batch* batch,
                                                       int64_t* bytes) {
    int64_t pool = 0;
    if (!layout || !batch || !bytes || batch->num_seqs < 0 || batch->max_q_len < 0) return AMOEBA_ERR_INVALID_ARG;
    const amoeba_status st = amoeba_layout_kv_pool_bytes(layout, &pool);
    if (st != AMOEBA_OK) return st;
    *bytes = few_workspace<Batch>(nullptr, nullptr, layout->model.head_dim);
    if (rows_of(layout, batch->max_q_len) > kMaxFewRows)
        *bytes += many_workspace<Batch>(nullptr, nullptr, layout->model.head_dim);
    return AMOEBA_OK;
}

// Checks the arguments that both calls have and fills in all but the workspace.
template <class B>
static amoeba_status make_params(const amoeba_layout* layout, int32_t dtype, int32_t layer, const void* const* pools,
                                 const amoeba_batch* batch, const void* const* q, int64_t q_stride, float scale, int32_t window,
                                 void* const* out, int64_t out_stride, float* d_lse, int32_t* d_status, AttendParams<B>* p) {
    amoeba_status st;
    if ((st = check_elements(layout, dtype)) != AMOEBA_OK) return st;
    if ((st = make_cache_view(layout, layer, pools, &p->cache)) != AMOEBA_OK) return st;
    if ((st = make_batch(batch, &p->batch)) != AMOEBA_OK) return st;
    if (!d_status || window < 0 || !positive(scale)) return AMOEBA_ERR_INVALID_ARG;
    const amoeba_model& m = layout->model;
    const int64_t row = (int64_t)m.num_q_heads / layout->tp * m.head_dim;
    if ((st = make_rows(layout, p->batch, q, q_stride, row, &p->q)) != AMOEBA_OK) return st;
    if ((st = make_rows(layout, p->batch, out, out_stride, row, &p->out)) != AMOEBA_OK) return st;
    for (int r = 0; r < layout->tp; ++r)  // other CTAs may still read the rows that one has answered
        for (int o = 0; o < layout->tp; ++o)
            if (q[r] && q[r] == out[o]) return AMOEBA_ERR_INVALID_ARG;
    p->lse = d_lse;
    p->status = d_status;
#ifdef AMOEBA_CHECK_ITEMS
    p->polls = operator_wait_polls();
#endif
    p->scale_log2 = scale * kLog2e;
    p->q_heads = m.num_q_heads;
    p->shape.group = m.num_q_heads / m.num_kv_heads;
    p->shape.kv_heads = m.num_kv_heads;
    p->shape.window = std::min(window, 1 << 30);
    return AMOEBA_OK;
}

// (units are numbered in 32 bits)
static bool units_fit(const amoeba_layout* l, int64_t num_seqs, int64_t rows) {
    return rows <= INT32_MAX && num_seqs * l->model.num_kv_heads <= INT32_MAX / (rows / kManyRows + 1);
}

// Calls run with the element type and head size as its template arguments.
#define AMOEBA_BY_ELEMENT(run, ...)                                                                                   \
    (dtype == AMOEBA_FP16 ? (layout->model.head_dim == 64 ? run<__half, 64>(__VA_ARGS__) : run<__half, 128>(__VA_ARGS__)) \
                          : (layout->model.head_dim == 64 ? run<__nv_bfloat16, 64>(__VA_ARGS__) : run<__nv_bfloat16, 128>(__VA_ARGS__)))

extern "C" amoeba_status amoeba_attend(const amoeba_layout* layout, int32_t dtype, int32_t layer,
                                       const void* const* pools, const amoeba_batch* batch, const void* const* q,
                                       int64_t q_stride, float scale, int32_t window, void* const* out,
                                       int64_t out_stride, float* d_lse, int32_t* d_status, void* d_workspace,
                                       int64_t workspace_bytes, void* cuda_stream) {
    AttendParams<Batch> p{};
    amoeba_status st = make_params(layout, dtype, layer, pools, batch, q, q_stride, scale, window, out, out_stride, d_lse, d_status, &p);
    if (st != AMOEBA_OK) return st;
    int64_t need = 0;
    if ((st = amoeba_attend_workspace_bytes(layout, batch, &need)) != AMOEBA_OK) return st;
    if (!d_workspace || workspace_bytes < need) return AMOEBA_ERR_INVALID_ARG;
    if ((uintptr_t)d_workspace % 16) return AMOEBA_ERR_ALIGNMENT;
    if (p.batch.num_seqs == 0 || p.batch.num_rows == 0) return AMOEBA_OK;
    if (!units_fit(layout, p.batch.num_seqs, rows_of(layout, p.batch.max_q_len))) return AMOEBA_ERR_UNSUPPORTED;
    const DeviceInfo dev = cached_device_info();
    if (!dev.sms) return AMOEBA_ERR_CUDA;
    return AMOEBA_BY_ELEMENT(run_attend, p, layout->tp, dtype, static_cast<char*>(d_workspace), dev.sms, static_cast<cudaStream_t>(cuda_stream));
}

// ------------------------------------------------------------------------------------------------ shared prefixes
// amoeba_attend_shared is two passes of the above.  The softmax's sums over disjoint sets of tokens join by their maxima:
//   m = max(m1, m2),   l = l1 2^(m1 - m) + l2 2^(m2 - m),   o = o1 2^(m1 - m) + o2 2^(m2 - m),   out = o / l.
// The groups attend as if each were one sequence with all rows of its sequences, every row seeing the whole prefix: that reads the
// prefix once, and has rows enough for the tensor cores where a sequence by itself has a few.  The sequences attend over their own tokens.
// Both leave the sums of rows with a prefix in the workspace, in 32 bits and not yet divided, and attend_finish joins them.
//
// Measured (one B200): 128 sequences of 64 to 2048 tokens of their own behind 8192, 32 query heads on 8 key heads of 128, a token each: 115 us
// (569 MB once each: 88), 477 if every sequence reads its prefix; 16 behind 131 072, 64 query heads: 126 us (98), 918 by themselves.

struct PrefixParams {
    Batch batch;
    const int32_t *group_starts, *prefix_lens;
    Group* groups;
    int64_t* tile0;
    int2* own;
    int32_t *row_group, *split, *status;
    int32_t num_groups, max_group_rows, block_tokens;
    int32_t kv_heads, group;  // query heads per key head
    int32_t sms, few_cost;    // few_cost: of a tile of attend_few
    int32_t always;
    int32_t tile_bytes;       // keys and values of 64 tokens and a key head
    int32_t few_ctas;         // to an SM, of the sequences' pass; 0: the passes do not run side by side
};

// What a group shares: no more than its shortest sequence has in front of its new tokens, and nothing where fewer than two have
// rows, one is bad, or it does not pay; then its sequences attend by themselves.  One block, a warp to a group.
//
// Whether it pays is counted in what 128 rows of attend_many cost over 128 tokens, 1650 clocks: every tile of the prefix costs 1 for up to
// 128 rows of a sequence, 2 for up to 256, and 2 where the rows are few and it is the reading that counts, 4 where attend_few has 32.
// A tile of the group's rows costs 5 to start and end, joining its sums with a sequence's 1 for few rows and 5 for 128; and the launches
// for all groups together as much as 28 on every SM, 25 us.  (2 groups of up to 5 sequences, 74 new tokens each behind up to 946: 89 us
// shared, 74 not; two of 7, 230 new tokens behind 9000: 610 and 605.)
//
// The two passes run side by side where the sequences' is attend_few's, whose time is that of reading: the groups' CTAs, one to an SM, take
// long to start and are bound by their products, and would leave the memory idle in front of it and behind.  The SMs are shared out
// by the clocks that each is known to take: a tile of 128 tokens and 256 rows 3300, of up to 128 rows 2600, a unit's begin and end 20 000
// beside the other pass, the kernel's 35 000; a tile of 64 tokens of attend_few 1000 (two CTAs to an SM), but all together no less than
// 6.3 TB/s.  (128 sequences behind 8192 tokens: 142 us one after the other, 120 with 32 SMs for the group, 129 with 24 or 48; chosen: 28.)
constexpr int kTileClocks = 3300, kTurnClocks = 2600, kSwitchClocks = 20000, kFewClocks = 1000;
constexpr float kStartClocks = 35000.f, kBytesPerClock = 3300.f;
constexpr int kPrefixThreads = 1024, kPrefixWarps = kPrefixThreads / 32;
__global__ void __launch_bounds__(kPrefixThreads, 1) prefix_groups(const __grid_constant__ PrefixParams p) {
    struct Plan {
        Group group;
        int32_t first, end;  // sequences
    };
    __shared__ Plan s_plan[kPrefixThreads];
    __shared__ int64_t s_tiles[kPrefixThreads], s_warp[kPrefixWarps];
    __shared__ unsigned long long s_gain, s_groups, s_rest, s_tiles64;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, S = p.batch.num_seqs, G = p.num_groups;
    grid_dependency_launch();
    grid_dependency_wait();
    for (int s = tid; s < S; s += kPrefixThreads) p.own[s] = make_int2(0, -1);
    for (int r = tid; r < p.batch.num_rows; r += kPrefixThreads) p.row_group[r] = -1;
    if (tid == 0) s_groups = s_rest = s_tiles64 = 0;
    const bool in_order = groups_in_order(p.group_starts, G, S);
    if (!in_order && tid == 0) report(p.status, AMOEBA_ERR_INVALID_ARG);
    int64_t run = 0;
    for (int base = 0; base < G; base += kPrefixThreads) {
        const int end = min(G, base + kPrefixThreads);
        if (tid == 0) s_gain = 0;
        __syncthreads();
        for (int g = base + warp; g < end; g += kPrefixWarps) {
            Plan out{{0, 0, 0, 0}, 0, 0};
            if (in_order) {
                const GroupSums x = sum_group(p.batch, p.group_starts, g, p.block_tokens, p.group, p.few_cost);
                const int given = p.prefix_lens[g], len = min(given, x.least), key_tiles = (len - 1) / kManyTile + 1;
                const bool wrong = refused(x, given, p.max_group_rows);
                if (wrong && lane == 0) report(p.status, AMOEBA_ERR_INVALID_ARG);
                if (!wrong && x.ok && x.with_rows > 1 && len > 0) {
                    const int rows = (x.q1 - x.q0) * p.group, row_tiles = (rows - 1) / kManyRows + 1;
                    const int64_t gain = (int64_t)(x.alone - rows_cost(rows)) * key_tiles - 5 * row_tiles - x.taking;
                    if (gain > 0 || p.always) {
                        out = Plan{{x.q0, x.q1 - x.q0, len, x.row}, x.first, x.end};
                        if (lane == 0 && gain > 0) atomicAdd(&s_gain, (unsigned long long)(gain * p.kv_heads));
                    }
                }
            }
            if (lane == 0) s_plan[g - base] = out;
        }
        __syncthreads();
        const bool pays = p.always || s_gain > 28ull * p.sms;
        for (int g = base + warp; g < end; g += kPrefixWarps) {
            Plan x = s_plan[g - base];
            if (!pays) x.group.qn = x.group.len = 0;
            int64_t tiles = 0;
            if (x.group.len > 0) {
                for (int s = x.first + lane; s < x.end; s += 32) p.own[s] = make_int2(x.group.len, g);
                for (int r = lane; r < x.group.qn; r += 32) p.row_group[x.group.q0 + r] = g;
                const int rows = x.group.qn * p.group, units = p.kv_heads * ((rows - 1) / kManyRows + 1);
                tiles = (int64_t)units * ((x.group.len - 1) / kManyTile + 1);
                if (lane == 0) atomicAdd(&s_groups, (unsigned long long)(tiles * (rows > 128 ? kTileClocks : kTurnClocks) + units * (int64_t)kSwitchClocks));
            }
            if (lane == 0) p.groups[g] = x.group, s_tiles[g - base] = tiles;
        }
        __syncthreads();
        // the first tile of every group
        const int64_t own = base + tid < G ? s_tiles[tid] : 0;
        int64_t incl = own;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int64_t up = __shfl_up_sync(~0u, incl, o);
            if (lane >= o) incl += up;
        }
        if (lane == 31) s_warp[warp] = incl;
        __syncthreads();
        int64_t warps = s_warp[lane];
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int64_t up = __shfl_up_sync(~0u, warps, o);
            if (lane >= o) warps += up;
        }
        const int64_t total = __shfl_sync(~0u, warps, 31), before = __shfl_sync(~0u, warps, max(warp - 1, 0));
        if (base + tid < G) p.tile0[base + tid] = run + (warp ? before : 0) + incl - own;
        run += total;
        __syncthreads();
    }
    if (tid == 0) p.tile0[G] = run;
    if (!p.few_ctas) {
        if (tid == 0) p.split[0] = p.sms, p.split[1] = 0;
        return;
    }
    // How many SMs the groups' pass gets, so that both end together.
    unsigned long long clocks = 0, tiles64 = 0;
    for (int s = tid; s < S; s += kPrefixThreads) {
        const Seq q = sequence(p.batch, s, p.block_tokens);
        if (q.qn == 0) continue;
        const int64_t n = (int64_t)p.kv_heads * ((q.len - p.own[s].x + 63) / 64);
        clocks += (n + kUnitStart * p.kv_heads) * kFewClocks, tiles64 += n;
    }
    if (warp * 32 < S) {
#pragma unroll
        for (int o = 16; o; o /= 2) clocks += __shfl_xor_sync(~0u, clocks, o), tiles64 += __shfl_xor_sync(~0u, tiles64, o);
        if (lane == 0) atomicAdd(&s_rest, clocks), atomicAdd(&s_tiles64, tiles64);
    }
    __syncthreads();
    if (warp) return;
    const float groups = (float)s_groups, rest = (float)s_rest, reading = (float)s_tiles64 * p.tile_bytes / kBytesPerClock;
    float best = INFINITY;
    int sms = 0;
    for (int m = 1 + lane; groups > 0.f && m < p.sms; m += 32) {
        const float t = fmaxf(kStartClocks + groups / m, fmaxf(rest / (p.sms - m), reading));
        if (t < best) best = t, sms = m;
    }
#pragma unroll
    for (int o = 16; o; o /= 2) {
        const float t = __shfl_xor_sync(~0u, best, o);
        const int m = __shfl_xor_sync(~0u, sms, o);
        if (t < best || (t == best && m < sms)) best = t, sms = m;
    }
    if (lane == 0) p.split[0] = sms, p.split[1] = (p.sms - sms) * p.few_ctas;
}

// Where the parts of the workspace begin: both passes' own, the sums that each leaves, the plan.
struct SharedSpace {
    int64_t groups_pass, rest_pass, group_sums, rest_sums, groups, tile0, own, row_group, split, end;
};
// Sums of all rows and query heads.
static int64_t sums_space(const amoeba_layout* l, int64_t rows, char* ws, Sums* out) {
    const int64_t heads = (rows * l->model.num_q_heads + 3) / 4 * 4, o = heads * l->model.head_dim * 4;
    if (out) *out = Sums{reinterpret_cast<float*>(ws), reinterpret_cast<float*>(ws + o), reinterpret_cast<float*>(ws + o + heads * 4)};
    return o + heads * 8;
}
static SharedSpace shared_space(const amoeba_layout* l, const amoeba_batch* b, const amoeba_prefixes* x) {
    const int D = l->model.head_dim;
    const int64_t few = few_workspace<Batch>(nullptr, nullptr, D), many = many_workspace<Batch>(nullptr, nullptr, D);
    auto ints = [](int64_t n) { return (n * 4 + 15) / 16 * 16; };
    SharedSpace s;
    s.groups_pass = 0;
    s.rest_pass = few + (rows_of(l, x->max_group_rows) > kMaxGroupRows ? many : 0);
    s.group_sums = s.rest_pass + few + (rows_of(l, b->max_q_len) > kMaxFewRows ? many : 0);
    s.rest_sums = s.group_sums + sums_space(l, b->num_rows, nullptr, nullptr);
    s.groups = s.rest_sums + sums_space(l, b->num_rows, nullptr, nullptr);
    s.tile0 = s.groups + (int64_t)x->num_groups * sizeof(Group);
    s.own = s.tile0 + ((int64_t)x->num_groups / 2 + 1) * 16;
    s.row_group = s.own + ints(2 * (int64_t)b->num_seqs);
    s.split = s.row_group + ints(b->num_rows);
    s.end = s.split + 16;
    return s;
}

template <class T, int D>
static amoeba_status run_shared(AttendParams<SharedBatch>& p, const amoeba_layout* layout, int32_t dtype, const amoeba_batch* batch,
                                const amoeba_prefixes* prefixes, char* ws, int sms, cudaStream_t stream) {
    const SharedSpace at = shared_space(layout, batch, prefixes);
    const int32_t group_rows = std::min(prefixes->max_group_rows, p.batch.num_rows);
    amoeba_status st;
    Pass<SharedBatch> rest;
    p.whole = not_cut(p, sms);
    p.batch.group_starts = prefixes->d_group_starts, p.batch.prefix_lens = prefixes->d_prefix_lens;
    p.batch.num_groups = prefixes->num_groups, p.batch.max_group_rows = group_rows;
    p.batch.waits = 1;
    // Where all sequences by themselves take less than the launches for the groups would, they attend by themselves, and the groups' numbers
    // are only checked.  A tile of 128 tokens takes an SM about 1.5 us, twice that with 17 to 32 rows, 1.7 us for 256 (8 sequences of 160
    // tokens: 13.6 us with the launches, 5.5 without; 8 of up to 950 tokens, 32 key heads: 24.5 and 17).
    const int64_t rows = rows_of(layout, p.batch.max_q_len);
    const int few_cost = rows > 16 && rows <= kMaxFewRows ? 4 : 2;
    const int64_t tiles = ((int64_t)p.batch.max_blocks * p.cache.block_tokens + kManyTile - 1) / kManyTile;
    if (!prefixes->always && (int64_t)p.batch.num_seqs * p.shape.kv_heads * std::max<int64_t>(few_cost, (rows + 127) / 128) * tiles <= 32 * sms) {
        if ((st = run_pass<T, D>(p, layout->tp, dtype, ws + at.rest_pass, sms, stream, &rest)) != AMOEBA_OK) return st;
        return run_join<T, D>(rest, stream);
    }
    PrefixParams x{};
    x.batch = p.batch;
    x.group_starts = prefixes->d_group_starts, x.prefix_lens = prefixes->d_prefix_lens;
    x.groups = reinterpret_cast<Group*>(ws + at.groups), x.tile0 = reinterpret_cast<int64_t*>(ws + at.tile0);
    x.own = reinterpret_cast<int2*>(ws + at.own), x.row_group = reinterpret_cast<int32_t*>(ws + at.row_group);
    x.status = p.status;
    x.num_groups = prefixes->num_groups, x.max_group_rows = group_rows, x.block_tokens = layout->block_tokens;
    x.kv_heads = p.shape.kv_heads, x.group = p.shape.group, x.sms = std::min(sms, kMaxSms), x.few_cost = few_cost, x.always = prefixes->always;
    x.split = reinterpret_cast<int32_t*>(ws + at.split);
    // Side by side: groups of attend_many, sequences of attend_few alone.
    const bool many_groups = prefixes->num_groups && rows_of(layout, group_rows) > kMaxGroupRows, side_by_side = many_groups && rows <= kMaxFewRows;
    const int few_ctas = rows <= 8 ? FewShape<D, 1>::kCtas : rows <= 16 ? FewShape<D, 2>::kCtas : FewShape<D, 4>::kCtas;
    x.tile_bytes = 64 * 2 * D * 2, x.few_ctas = side_by_side ? few_ctas : 0;
    if ((st = launch_kernel(prefix_groups, 1, kPrefixThreads, 0, stream, true, x)) != AMOEBA_OK) return st;
    p.batch.own = x.own;
    sums_space(layout, p.batch.num_rows, ws + at.rest_sums, &p.sums);
    Pass<SharedBatch> groups;
    AttendParams<SharedBatch> g = p;
    g.batch.groups = x.groups, g.batch.tile0 = x.tile0, g.batch.split = x.split;
    g.batch.num_seqs = prefixes->num_groups;
    g.batch.max_q_len = group_rows;
    g.whole = not_cut(g, sms);
    sums_space(layout, p.batch.num_rows, ws + at.group_sums, &g.sums);
    if (many_groups) {
        if ((st = run_pass<T, D>(g, layout->tp, dtype, ws + at.groups_pass, sms, stream, &groups)) != AMOEBA_OK) return st;
        p.batch.waits = 0;
        if (side_by_side) p.batch.split = x.split;
    }
    if ((st = run_pass<T, D>(p, layout->tp, dtype, ws + at.rest_pass, sms, stream, &rest)) != AMOEBA_OK) return st;
    if (prefixes->num_groups == 0 || group_rows == 0) return run_join<T, D>(rest, stream);
    PrefixSums sums{};
    sums.rows = g.sums;
    if (many_groups) {
        sums.parts = Sums{groups.many.part_o, groups.many.part_m, groups.many.part_l};
        sums.split = x.split;
    } else {
        g.batch.waits = 0;
        if ((st = run_pass<T, D>(g, layout->tp, dtype, ws + at.groups_pass, sms, stream, &groups)) != AMOEBA_OK) return st;
        if ((st = run_join<T, D>(groups, stream)) != AMOEBA_OK) return st;
    }
    sums.groups = x.groups, sums.tile0 = x.tile0, sums.row_group = x.row_group;
    sums.num_groups = prefixes->num_groups, sums.num_rows = p.batch.num_rows;
    // A warp to a head, unless there are rows enough to fill the GPU as it is.
    sums.row_warps = p.batch.num_rows >= 1024 ? 1 : p.q_heads;
    const int64_t grid = rest.few_ctas + rest.many_blocks() + ((int64_t)sums.num_rows * sums.row_warps + kJoinWarps - 1) / kJoinWarps;
    if (grid > INT32_MAX) return AMOEBA_ERR_UNSUPPORTED;
    return launch_kernel(sums.row_warps > 1 ? attend_finish<T, D, 1> : attend_finish<T, D, 4>, (int)grid, kJoinThreads, 0, stream, true, rest.few,
                         rest.few_ctas, rest.many, rest.many_ctas, sums);
}

extern "C" amoeba_status amoeba_attend_shared_workspace_bytes(const amoeba_layout* layout, const amoeba_batch* batch,
                                                              const amoeba_prefixes* prefixes, int64_t* bytes) {
    int64_t pool = 0;
    if (!layout || !batch || !prefixes || !bytes || batch->num_seqs < 0 || batch->max_q_len < 0 || batch->num_rows < 0 ||
        prefixes->num_groups < 0 || prefixes->max_group_rows < 0)
        return AMOEBA_ERR_INVALID_ARG;
    const amoeba_status st = amoeba_layout_kv_pool_bytes(layout, &pool);
    if (st != AMOEBA_OK) return st;
    *bytes = shared_space(layout, batch, prefixes).end;
    return AMOEBA_OK;
}

extern "C" amoeba_status amoeba_attend_shared(const amoeba_layout* layout, int32_t dtype, int32_t layer, const void* const* pools,
                                              const amoeba_batch* batch, const amoeba_prefixes* prefixes, const void* const* q,
                                              int64_t q_stride, float scale, void* const* out, int64_t out_stride, float* d_lse,
                                              int32_t* d_status, void* d_workspace, int64_t workspace_bytes, void* cuda_stream) {
    AttendParams<SharedBatch> p{};
    amoeba_status st = make_params(layout, dtype, layer, pools, batch, q, q_stride, scale, 0, out, out_stride, d_lse, d_status, &p);
    if (st != AMOEBA_OK) return st;
    int64_t need = 0;
    if ((st = amoeba_attend_shared_workspace_bytes(layout, batch, prefixes, &need)) != AMOEBA_OK) return st;
    if (prefixes->num_groups && (!prefixes->d_group_starts || !prefixes->d_prefix_lens)) return AMOEBA_ERR_INVALID_ARG;
    if (prefixes->always != 0 && prefixes->always != 1) return AMOEBA_ERR_INVALID_ARG;
    if (!d_workspace || workspace_bytes < need) return AMOEBA_ERR_INVALID_ARG;
    if ((uintptr_t)d_workspace % 16) return AMOEBA_ERR_ALIGNMENT;
    if (p.batch.num_seqs == 0 || p.batch.num_rows == 0) return AMOEBA_OK;
    const int32_t group_rows = std::min(prefixes->max_group_rows, p.batch.num_rows);
    if (!units_fit(layout, p.batch.num_seqs, rows_of(layout, p.batch.max_q_len)) ||
        !units_fit(layout, prefixes->num_groups, rows_of(layout, group_rows)))
        return AMOEBA_ERR_UNSUPPORTED;
    const DeviceInfo dev = cached_device_info();
    if (!dev.sms) return AMOEBA_ERR_CUDA;
    return AMOEBA_BY_ELEMENT(run_shared, p, layout, dtype, batch, prefixes, static_cast<char*>(d_workspace), dev.sms,
                             static_cast<cudaStream_t>(cuda_stream));
}
