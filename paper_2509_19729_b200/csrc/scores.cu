// amoeba_accumulate_scores: the attention weight that every cached token received, summed over the rows.
//
// exp(scale * q . k - lse) needs no running statistics, so a token's sum is finished by the warp that has read its key:
// every key is read once, the rows are walked in order for it, and no two warps add to the same score.
#include "walk.cuh"
#include "warp_mma.cuh"

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
    float scale_log2;
    int32_t q_heads, window;
};

// A warp takes 16 tokens of every tile of 64; S^T = K Q^T as in attend.cu, so that a token's sum runs along the columns.
constexpr int kScoreThreads = 128, kScoreWarps = 4, kScoreTile = 16 * kScoreWarps, kScoreStages = 6, kScoreCtas = 2;

template <class T, int D>
__global__ void __launch_bounds__(kScoreThreads, kScoreCtas) accumulate_scores(const __grid_constant__ ScoreParams p) {
    constexpr int kSteps = D / 16, kStage = 16 * D * 2;
    extern __shared__ __align__(128) char smem[];
    __shared__ uint32_t s_mask[kScoreWarps][kScoreStages];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, quad = lane / 4, pair = lane % 4;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * kScoreStages * kStage;
    const Shape& sh = p.shape;
    Walk walk;
    int64_t begin, end;
    take_share<kScoreThreads>(sh, p.batch, p.cache.block_tokens, &walk, &begin, &end, p.status);
    int64_t n = end - begin;
    if (n == 0) return;

    Walk ahead = walk;
    int64_t to_load = n;
    int slot_in = 0, slot = 0;
    auto load = [&] {
        if (to_load > 0) {
            const int key0 = ahead.t * kScoreTile + warp * 16;
            const uint32_t mask = load16<D, false>(p.cache, p.batch.table + (int64_t)ahead.s * p.batch.max_blocks,
                                                   p.cache.head_base(ahead.h), key0, 0, ahead.range.hi,
                                                   ring + slot_in * kStage, p.status);
            if (lane == 0) s_mask[warp][slot_in] = mask;
            if (--to_load > 0) ahead.next(sh, p.batch, p.cache.block_tokens);
        }
        cp_async_commit();
        slot_in = slot_in + 1 == kScoreStages ? 0 : slot_in + 1;
    };
#pragma unroll
    for (int i = 0; i < kScoreStages - 1; ++i) load();

    for (; n > 0; --n) {
        cp_async_wait<kScoreStages - 2>();
        __syncwarp();
        load();
        const uint32_t k_smem = ring + slot * kStage;
        const uint32_t mask = s_mask[warp][slot];
        slot = slot + 1 == kScoreStages ? 0 : slot + 1;
        uint32_t a[kSteps][4];
#pragma unroll
        for (int j = 0; j < kSteps; ++j) ldmatrix4(a[j], k_smem + swizzled<D>(lane % 16, 2 * j + lane / 16));

        const Seq& q = walk.seq;
        const int g = sh.group, rows = q.qn * g, w = walk.h / p.cache.heads, h = walk.h - w * p.cache.heads;
        const int key0 = walk.t * kScoreTile + warp * 16 + quad;
        float sum[2] = {0.f, 0.f};
        if (mask)
            for (int first = 0; first < rows; first += 8) {
                const int r = first + quad;
                const bool there = r < rows;
                const int tok = r / g;
                const char* src = p.q.base[w] + (int64_t)(q.q0 + tok) * p.q.stride + (h * g + r - tok * g) * (D * 2);
                float st[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < kSteps; ++j) {
                    uint32_t b[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        b[i] = there ? *reinterpret_cast<const uint32_t*>(src + (j * 16 + i * 8 + pair * 2) * 2) : 0u;
                    mma16816<T>(st, a[j], b[0], b[1]);
                }
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int rr = first + pair * 2 + b;
                    if (rr >= rows) continue;
                    const int t = rr / g, pos = q.len - q.qn + t;
                    const float lse = p.lse[(int64_t)(q.q0 + t) * p.q_heads + walk.h * g + rr - t * g];
                    if (lse == -INFINITY) continue;
                    const int lo = p.window > 0 ? pos - p.window + 1 : 0;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int key = key0 + i * 8;
                        if (key <= pos && key >= lo) sum[i] += fast_exp2(st[2 * i + b] * p.scale_log2 - lse * kLog2e);
                    }
                }
            }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            sum[i] += __shfl_xor_sync(~0u, sum[i], 1);
            sum[i] += __shfl_xor_sync(~0u, sum[i], 2);
            if (pair == 0 && (mask >> (quad + i * 8) & 1u)) {
                const int key = key0 + i * 8, bt = p.cache.block_tokens;
                const int block = p.batch.table[(int64_t)walk.s * p.batch.max_blocks + key / bt];
                float* to = p.scores[w] + ((int64_t)block * p.cache.heads + h) * bt + key % bt;
                *to = (p.scored && key < p.scored[walk.s] ? *to : 0.f) + sum[i];
            }
        }
        if (n > 1) walk.next(sh, p.batch, p.cache.block_tokens);
    }
}

template <class T, int D>
static amoeba_status run_scores(const ScoreParams& p, int sms, cudaStream_t stream) {
    constexpr int smem = kScoreWarps * kScoreStages * 16 * D * 2;
    if (ensure_dynamic_smem((const void*)accumulate_scores<T, D>, smem) != cudaSuccess) return AMOEBA_ERR_CUDA;
    accumulate_scores<T, D><<<kScoreCtas * sms, kScoreThreads, smem, stream>>>(p);
    return launch_result();
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
    if (!d_status || !d_lse || !score_pools || window < 0 || !positive(scale)) return AMOEBA_ERR_INVALID_ARG;
    const amoeba_model& m = layout->model;
    if ((st = make_rows(layout, q, q_stride, (int64_t)m.num_q_heads / layout->tp * m.head_dim, &p.q)) != AMOEBA_OK)
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
    p.scale_log2 = scale * kLog2e;
    p.q_heads = m.num_q_heads;
    p.shape.group = m.num_q_heads / m.num_kv_heads;
    p.shape.kv_heads = m.num_kv_heads;
    p.shape.rows = INT32_MAX;  // all rows of a sequence in one unit; its tiles run over the whole sequence
    p.shape.tile = kScoreTile;
    p.shape.max_rows = INT32_MAX;
    p.shape.rowless = 1;
    const DeviceInfo dev = cached_device_info();
    if (!dev.sms) return AMOEBA_ERR_CUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    p.window = std::min(window, 1 << 30);  // not the shape's: every token gets a value, zero if no row sees it
    if (dtype == AMOEBA_FP16)
        return m.head_dim == 64 ? run_scores<__half, 64>(p, dev.sms, stream) : run_scores<__half, 128>(p, dev.sms, stream);
    return m.head_dim == 64 ? run_scores<__nv_bfloat16, 64>(p, dev.sms, stream)
                            : run_scores<__nv_bfloat16, 128>(p, dev.sms, stream);
}
