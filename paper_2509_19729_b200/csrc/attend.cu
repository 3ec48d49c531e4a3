// amoeba_attend: attention of a ragged chunk of new tokens over the paged cache.
//
// One unit of work is a (sequence, key head, tile of query rows), the rows of a unit being the new tokens times the
// query heads that share the key head, so that grouped heads read their keys once.  The softmax runs along the tokens
// with a running maximum and sum per row; units are cut where the shares of the CTAs end (walk.cuh), and the cut ones
// are joined by their maxima and sums in a second small launch.
#include "attend.cuh"
#include "warp_mma.cuh"

namespace amoeba {

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

template <class T, int D, int NT>
__global__ void __launch_bounds__(kFewThreads, FewShape<D, NT>::kCtas)
attend_few(const __grid_constant__ AttendParams p) {
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
    if (p.whole) {
        walk.open(sh, p.batch, p.cache.block_tokens, blockIdx.x / sh.kv_heads);
        if (!walk.seq.ok && tid == 0) report(p.status, AMOEBA_ERR_INVALID_ARG);
        walk.h = blockIdx.x % sh.kv_heads;
        n = walk.nm ? walk.range.tiles : 0;
    } else {
        int64_t begin, end;
        take_share<kFewThreads>(sh, p.batch, p.cache.block_tokens, &walk, &begin, &end, p.status);
        write_cut(sh, p.cuts, walk, begin, end);
        n = end - begin;
    }
    grid_dependency_launch();
    if (n == 0) return;

    Ahead<D, true, kFewTile> ahead(p.cache, p.batch, sh, p.status, walk, n, warp * 16);
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
                    const int pos = walk.seq.len - walk.seq.qn + rr / sh.group;
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
            float l = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kFewWarps; ++w) {
                const float f = fast_exp2(s_m[w][r] - ref);
                const float4 x = *reinterpret_cast<const float4*>(s_o + (w * R + r) * kPitch + d);
                l += f * s_l[w][r];
                acc.x += f * x.x, acc.y += f * x.y, acc.z += f * x.z, acc.w += f * x.w;
            }
            if (direct) {
                const float inv = l == 0.f ? 0.f : 1.f / l;
                const int row = walk.m * R + r;
                *reinterpret_cast<uint2*>(row_of<D>(p.out, p, walk.seq, walk.h, row) + d * 2) =
                    make_uint2(Elem<T>::pack(acc.x * inv, acc.y * inv), Elem<T>::pack(acc.z * inv, acc.w * inv));
                if (d == 0 && p.lse) *lse_of(p, walk.seq, walk.h, row) = l == 0.f ? -INFINITY : (top + log2f(l)) * kLn2;
            } else {
                *reinterpret_cast<float4*>(p.part_o + (part + r) * D + d) = acc;
                if (d == 0) p.part_m[part + r] = top, p.part_l[part + r] = l;
            }
        }
        __syncthreads();
        if (n > 1) walk.next(sh, p.batch, p.cache.block_tokens);
    }
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

struct Joined {
    float top = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    __device__ __forceinline__ void add(float top2, float l2, const float4& x) {
        const float up = fmaxf(top, top2), ref = up == -INFINITY ? 0.f : up, f = fast_exp2(top - ref), g = fast_exp2(top2 - ref);
        l = l * f + l2 * g;
        acc.x = acc.x * f + x.x * g, acc.y = acc.y * f + x.y * g, acc.z = acc.z * f + x.z * g, acc.w = acc.w * f + x.w * g;
        top = up;
    }
};

// `groups` blocks to every share: the unit that it begins in is joined there, if that began in the share before.
template <class T, int D, int kWarps>
__device__ __forceinline__ void join_rows(const AttendParams& p, int ctas, int block, int groups) {
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
        }
        if (kAtOnce == 2) {  // the second half of the warp has every other part
            const float4 x = make_float4(__shfl_down_sync(~0u, j.acc.x, 16), __shfl_down_sync(~0u, j.acc.y, 16),
                                         __shfl_down_sync(~0u, j.acc.z, 16), __shfl_down_sync(~0u, j.acc.w, 16));
            const float top = __shfl_down_sync(~0u, j.top, 16), l = __shfl_down_sync(~0u, j.l, 16);
            j.add(top, l, x);
        }
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
        const float inv = j.l == 0.f ? 0.f : 1.f / j.l;
        const int row = cut.m * R + r;
        *reinterpret_cast<uint2*>(row_of<D>(p.out, p, q, cut.h, row) + lane * 8) =
            make_uint2(Elem<T>::pack(j.acc.x * inv, j.acc.y * inv), Elem<T>::pack(j.acc.z * inv, j.acc.w * inv));
        if (lane == 0 && p.lse) *lse_of(p, q, cut.h, row) = j.l == 0.f ? -INFINITY : (j.top + log2f(j.l)) * kLn2;
    }
}
// Blocks [0, few_ctas * few_rows) join what attend_few has cut, the others what attend_many has.
template <class T, int D>
__global__ void __launch_bounds__(kJoinThreads) attend_join(const __grid_constant__ AttendParams few, int few_ctas, int few_rows,
                                                            const __grid_constant__ AttendParams many, int many_ctas) {
    grid_dependency_wait();
    const int block = (int)blockIdx.x - few_ctas * few_rows;
    if (block < 0) join_rows<T, D, kJoinWarps>(few, few_ctas, blockIdx.x, few_rows);
    else join_rows<T, D, 1>(many, many_ctas, block, kManyRows / kJoinRows<1>);
}

// The workspace holds the parts of cut units, two for each CTA; these bound the grids without asking the device.
constexpr int kMaxFewCtas = 2 * kMaxSms;
constexpr int kMaxFewRows = 32;

// One kernel's part of the workspace: where the shares begin, then the parts.
static int64_t workspace_part(AttendParams* p, char* ws, int64_t parts, int64_t rows, int head_dim) {
    const int64_t o = kMaxFewCtas * (int64_t)sizeof(Cut), m = o + parts * rows * head_dim * 4, l = m + parts * rows * 4;
    if (p) {
        p->cuts = reinterpret_cast<Cut*>(ws);
        p->part_o = reinterpret_cast<float*>(ws + o);
        p->part_m = reinterpret_cast<float*>(ws + m);
        p->part_l = reinterpret_cast<float*>(ws + l);
    }
    return l + parts * rows * 4;
}
static int64_t few_workspace(AttendParams* p, char* ws, int head_dim) {
    return workspace_part(p, ws, 2 * kMaxFewCtas, kMaxFewRows, head_dim);
}
static int64_t many_workspace(AttendParams* p, char* ws, int head_dim) {
    return workspace_part(p, ws, 2 * kMaxSms, kManyRows, head_dim);
}
static int64_t rows_of(const amoeba_layout* l, int32_t max_q_len) {
    return (int64_t)max_q_len * (l->model.num_q_heads / l->model.num_kv_heads);
}

template <class T, int D, int NT>
static amoeba_status run_few(AttendParams& p, int sms, int* ctas, cudaStream_t stream) {
    using F = FewShape<D, NT>;
    p.shape.rows = 8 * NT;
    p.shape.tile = kFewTile;
    if (ensure_dynamic_smem((const void*)attend_few<T, D, NT>, F::kSmem) != cudaSuccess) return AMOEBA_ERR_CUDA;
    *ctas = std::min(F::kCtas * sms, kMaxFewCtas);
    return launch_kernel(attend_few<T, D, NT>, p.whole ? p.batch.num_seqs * p.shape.kv_heads : *ctas, kFewThreads, F::kSmem, stream,
                         false, p);
}

// Sequences with few rows (new tokens times query heads per key head) are read by attend_few, whose time is that of reading
// the cache; the others by attend_many.  Which there are is known only on the device: a batch that may hold longer
// ones gets both, and each skips the other's.  The launches follow one another closely: a kernel's blocks may be in place
// before the kernel in front of it ends, and wait there for its results if they read them (attend_join) or end only after
// it (attend_many).
template <class T, int D>
static amoeba_status run_attend(AttendParams& p, int tp, int32_t dtype, char* ws, int sms, cudaStream_t stream) {
    const int64_t rows = (int64_t)p.batch.max_q_len * p.shape.group;
    const int64_t few_bytes = few_workspace(&p, ws, D);
    // In a batch with longer pieces attend_few gets the single tokens (and what has as few rows): its rows cost registers.
    const int64_t few_rows = rows <= kMaxFewRows ? rows : p.shape.group;
    const int most = few_rows <= 8 ? 8 : few_rows <= 16 ? 16 : kMaxFewRows;
    p.shape.min_rows = 0;
    p.shape.max_rows = most;
    int few_ctas = 0;
    amoeba_status st = most == 8    ? run_few<T, D, 1>(p, sms, &few_ctas, stream)
                       : most == 16 ? run_few<T, D, 2>(p, sms, &few_ctas, stream)
                                    : run_few<T, D, 4>(p, sms, &few_ctas, stream);
    if (st != AMOEBA_OK || (p.whole && rows <= kMaxFewRows)) return st;
    if (p.whole) few_ctas = 0;  // nothing is cut
    const int few_most = (int)std::min<int64_t>(rows, most);
    AttendParams many = p;
    int many_ctas = 0, many_blocks = 0;
    if (rows > kMaxFewRows) {
        many_workspace(&many, ws + few_bytes, D);
        many.shape.min_rows = most + 1;
        many.shape.max_rows = INT32_MAX;
        many.shape.rows = kManyRows;
        many.shape.tile = kManyTile;
        many_ctas = std::min(sms, kMaxSms);
        many_blocks = many_ctas * (kManyRows / kJoinRows<1>);
        if ((st = launch_attend_many(many, tp, dtype, D, many_ctas, stream)) != AMOEBA_OK) return st;
    }
    return launch_kernel(attend_join<T, D>, few_ctas * few_most + many_blocks, kJoinThreads, 0, stream, true, p, few_ctas, few_most, many,
                         many_ctas);
}

}  // namespace amoeba

using namespace amoeba;

extern "C" amoeba_status amoeba_attend_workspace_bytes(const amoeba_layout* layout, const amoeba_batch* batch,
                                                       int64_t* bytes) {
    int64_t pool = 0;
    if (!layout || !batch || !bytes || batch->num_seqs < 0 || batch->max_q_len < 0) return AMOEBA_ERR_INVALID_ARG;
    const amoeba_status st = amoeba_layout_kv_pool_bytes(layout, &pool);
    if (st != AMOEBA_OK) return st;
    *bytes = few_workspace(nullptr, nullptr, layout->model.head_dim);
    if (rows_of(layout, batch->max_q_len) > kMaxFewRows)
        *bytes += many_workspace(nullptr, nullptr, layout->model.head_dim);
    return AMOEBA_OK;
}

extern "C" amoeba_status amoeba_attend(const amoeba_layout* layout, int32_t dtype, int32_t layer,
                                       const void* const* pools, const amoeba_batch* batch, const void* const* q,
                                       int64_t q_stride, float scale, int32_t window, void* const* out,
                                       int64_t out_stride, float* d_lse, int32_t* d_status, void* d_workspace,
                                       int64_t workspace_bytes, void* cuda_stream) {
    AttendParams p{};
    amoeba_status st;
    if ((st = check_elements(layout, dtype)) != AMOEBA_OK) return st;
    if ((st = make_cache_view(layout, layer, pools, &p.cache)) != AMOEBA_OK) return st;
    if ((st = make_batch(batch, &p.batch)) != AMOEBA_OK) return st;
    if (!d_status || window < 0 || !positive(scale)) return AMOEBA_ERR_INVALID_ARG;
    const amoeba_model& m = layout->model;
    const int64_t row = (int64_t)m.num_q_heads / layout->tp * m.head_dim;
    if ((st = make_rows(layout, p.batch, q, q_stride, row, &p.q)) != AMOEBA_OK) return st;
    if ((st = make_rows(layout, p.batch, out, out_stride, row, &p.out)) != AMOEBA_OK) return st;
    for (int r = 0; r < layout->tp; ++r)  // other CTAs may still read the rows that one has answered
        for (int o = 0; o < layout->tp; ++o)
            if (q[r] && q[r] == out[o]) return AMOEBA_ERR_INVALID_ARG;
    int64_t need = 0;
    if ((st = amoeba_attend_workspace_bytes(layout, batch, &need)) != AMOEBA_OK) return st;
    if (!d_workspace || workspace_bytes < need) return AMOEBA_ERR_INVALID_ARG;
    if ((uintptr_t)d_workspace % 16) return AMOEBA_ERR_ALIGNMENT;
    if (p.batch.num_seqs == 0 || p.batch.num_rows == 0) return AMOEBA_OK;
    p.lse = d_lse;
    p.status = d_status;
#ifdef AMOEBA_CHECK_ITEMS
    p.polls = operator_wait_polls();
#endif
    p.scale_log2 = scale * kLog2e;
    p.q_heads = m.num_q_heads;
    p.shape.group = m.num_q_heads / m.num_kv_heads;
    p.shape.kv_heads = m.num_kv_heads;
    p.shape.window = std::min(window, 1 << 30);
    // (units are numbered in 32 bits)
    const int64_t rows = rows_of(layout, p.batch.max_q_len);
    if (rows > INT32_MAX || (int64_t)p.batch.num_seqs * m.num_kv_heads > INT32_MAX / (rows / kManyRows + 1)) return AMOEBA_ERR_UNSUPPORTED;
    const DeviceInfo dev = cached_device_info();
    if (!dev.sms) return AMOEBA_ERR_CUDA;
    // Short sequences are not worth cutting: what the shares and the join take, about 5 us, is what a CTA needs for 512
    // tokens, or for 1024 when there are units enough to fill the GPU (one sequence of 256 tokens, 8 key heads: 7.9 us whole,
    // 9.5 cut; of 1024: 20.5 and 11.3; 32 sequences of 1024: 24 and 29; of 2048: 41 and 47, but there one long one would
    // hold up all).  With max_q_len 0 sequences are only looked at.
    const int64_t tokens = (int64_t)p.batch.max_blocks * layout->block_tokens;
    p.whole = rows == 0 || tokens <= 512 || (tokens <= 1024 && p.batch.num_seqs * m.num_kv_heads >= dev.sms);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    char* ws = static_cast<char*>(d_workspace);
    if (dtype == AMOEBA_FP16)
        return m.head_dim == 64 ? run_attend<__half, 64>(p, layout->tp, dtype, ws, dev.sms, stream)
                                : run_attend<__half, 128>(p, layout->tp, dtype, ws, dev.sms, stream);
    return m.head_dim == 64 ? run_attend<__nv_bfloat16, 64>(p, layout->tp, dtype, ws, dev.sms, stream)
                            : run_attend<__nv_bfloat16, 128>(p, layout->tp, dtype, ws, dev.sms, stream);
}
