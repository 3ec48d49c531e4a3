// What the kernels of amoeba_attend share: their parameters and where a unit's rows lie.
#pragma once
#include "walk.cuh"

namespace amoeba {

struct AttendParams {
    CacheView cache;
    Batch batch;
    Rows q, out;
    Shape shape;
    float* lse;
    int32_t* status;
    Cut* cuts;               // [CTAs]
    float *part_o, *part_m, *part_l;  // of the cut units: [2 * CTAs][rows][D], [2 * CTAs][rows]
    float scale_log2;        // scale * log2(e): the softmax runs in powers of two
    int32_t q_heads;         // of all workers
    int32_t whole;           // 1: one CTA per unit, nothing is cut
#ifdef AMOEBA_CHECK_ITEMS
    int32_t polls;           // of every wait in attend_many
#endif
};

// Where row r of a unit lies in a row buffer.
template <int D>
__device__ __forceinline__ char* row_of(const Rows& rows, const AttendParams& p, const Seq& q, int kv_head, int r) {
    const int w = kv_head / p.cache.heads, h = kv_head - w * p.cache.heads, g = p.shape.group;
    const int tok = r / g;
    return rows.base[w] + (int64_t)(q.q0 + tok) * rows.stride + (h * g + r - tok * g) * (D * 2);
}
__device__ __forceinline__ float* lse_of(const AttendParams& p, const Seq& q, int kv_head, int r) {
    const int g = p.shape.group, tok = r / g;
    return p.lse + (int64_t)(q.q0 + tok) * p.q_heads + kv_head * g + r - tok * g;
}

// The kernel for many rows (attend_many.cu): 256 rows a unit, 128 tokens a tile.
constexpr int kManyRows = 256, kManyTile = 128;
constexpr int kMaxSms = 192;  // bounds the grids, and so the workspace, without asking the device
amoeba_status launch_attend_many(const AttendParams& p, int tp, int32_t dtype, int head_dim, int ctas, cudaStream_t stream);

}  // namespace amoeba
