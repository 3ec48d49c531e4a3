// What the kernels of amoeba_attend share: their parameters and where a unit's rows lie.
#pragma once
#include "walk.cuh"

namespace amoeba {

// The kernel for many rows (attend_many.cu): 256 rows a unit, 128 tokens a tile.
constexpr int kManyRows = 256, kManyTile = 128;
constexpr int kMaxSms = 192;  // bounds the grids, and so the workspace, without asking the device
// Sums of rows and query heads that are not yet divided: weights times values, the largest logit in powers of two, the weights.
struct Sums {
    float *o, *m, *l;  // [rows][query heads][D], [rows][query heads]; or parts as below
};

// B: Batch, or SharedBatch: then rows with a prefix go to `sums`, by both passes, and are joined behind them.
template <class B>
struct AttendParams {
    CacheView cache;
    B batch;
    Rows q, out;
    Shape shape;
    float* lse;
    int32_t* status;
    Cut* cuts;               // [CTAs]
    float *part_o, *part_m, *part_l;  // of the cut units: [2 * CTAs][rows][D], [2 * CTAs][rows]
    float scale_log2;        // scale * log2(e): the softmax runs in powers of two
    int32_t q_heads;         // of all workers
    int32_t whole;           // 1: one CTA per unit, nothing is cut
    Sums sums;               // of a SharedBatch
#ifdef AMOEBA_CHECK_ITEMS
    int32_t polls;           // of every wait in attend_many
#endif
};

// Where row r of a unit lies in a row buffer.
template <int D, class B>
__device__ __forceinline__ char* row_of(const Rows& rows, const AttendParams<B>& p, const Seq& q, int kv_head, int r) {
    const int w = kv_head / p.cache.heads, h = kv_head - w * p.cache.heads, g = p.shape.group;
    const int tok = r / g;
    return rows.base[w] + (int64_t)(q.q0 + tok) * rows.stride + (h * g + r - tok * g) * (D * 2);
}
// Its place among the rows and query heads of all workers.
template <class B>
__device__ __forceinline__ int64_t head_of(const AttendParams<B>& p, const Seq& q, int kv_head, int r) {
    const int g = p.shape.group, tok = r / g;
    return (int64_t)(q.q0 + tok) * p.q_heads + kv_head * g + r - tok * g;
}
template <class B>
__device__ __forceinline__ float* lse_of(const AttendParams<B>& p, const Seq& q, int kv_head, int r) {
    return p.lse + head_of(p, q, kv_head, r);
}

// Sums of one or more parts of a row, four of its values.
struct Joined {
    float top = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    __device__ __forceinline__ void add(float top2, float l2, const float4& x) {
        const float up = fmaxf(top, top2), ref = up == -INFINITY ? 0.f : up, f = fast_exp2(top - ref), g = fast_exp2(top2 - ref);
        l = l * f + l2 * g;
        acc.x = acc.x * f + x.x * g, acc.y = acc.y * f + x.y * g, acc.z = acc.z * f + x.z * g, acc.w = acc.w * f + x.w * g;
        top = up;
    }
    // For the first half of the warp: what the second has.
    __device__ __forceinline__ void add_lower_half() {
        const float4 x = make_float4(__shfl_down_sync(~0u, acc.x, 16), __shfl_down_sync(~0u, acc.y, 16), __shfl_down_sync(~0u, acc.z, 16),
                                     __shfl_down_sync(~0u, acc.w, 16));
        const float top2 = __shfl_down_sync(~0u, top, 16), l2 = __shfl_down_sync(~0u, l, 16);
        add(top2, l2, x);
    }
};
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
    return (uint64_t)(a | b) >> 32 == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}
// Whether a unit's rows are to be joined with sums over other tokens.
template <class B>
__device__ __forceinline__ bool goes_on(const AttendParams<B>&, const Seq& q) { return B::kShared && (q.level || q.first > 0); }
constexpr float kCutRow = -1.f;  // in place of a row's sum of weights: the unit was cut, its parts are elsewhere
// What a row comes to, its values d .. d + 3, to the output.
template <class T, int D, class B>
__device__ __forceinline__ void write_row(const AttendParams<B>& p, const Seq& q, int kv_head, int row, int d, const Joined& j) {
    const float inv = j.l == 0.f ? 0.f : 1.f / j.l;
    *reinterpret_cast<uint2*>(row_of<D>(p.out, p, q, kv_head, row) + d * 2) =
        make_uint2(Elem<T>::pack(j.acc.x * inv, j.acc.y * inv), Elem<T>::pack(j.acc.z * inv, j.acc.w * inv));
    if (d == 0 && p.lse) *lse_of(p, q, kv_head, row) = j.l == 0.f ? -INFINITY : (j.top + log2f(j.l)) * kLn2;
}
template <int D, class B>
__device__ __forceinline__ void write_sums(const AttendParams<B>& p, const Seq& q, int kv_head, int row, int d, const Joined& j) {
    const int64_t at = head_of(p, q, kv_head, row);
    *reinterpret_cast<float4*>(p.sums.o + at * D + d) = j.acc;
    if (d == 0) p.sums.m[at] = j.top, p.sums.l[at] = j.l;
}

template <class B>
amoeba_status launch_attend_many(const AttendParams<B>& p, int tp, int32_t dtype, int head_dim, int ctas, cudaStream_t stream);

}  // namespace amoeba
