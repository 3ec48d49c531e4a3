// One layer of an instance's paged cache as the serving operators address it, and the batch of new tokens.
#pragma once
#include <cmath>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "launch.hpp"
#include "plan.hpp"

namespace amoeba {

// Strides in bytes; both storage orders are the same four numbers.
struct CacheView {
    char* pools[AMOEBA_MAX_TP];  // worker pools, advanced to the layer
    int64_t block_stride, head_stride, kv_stride, tok_stride;
    int32_t num_blocks, block_tokens, heads;  // heads: key heads per worker
};

struct Rows {
    char* base[AMOEBA_MAX_TP];
    int64_t stride;  // bytes between rows
};

struct Batch {
    static constexpr bool kShared = false;
    const int32_t *table, *lens, *starts;
    int32_t num_seqs, max_blocks, num_rows, max_q_len;
    __host__ __device__ bool by_groups() const { return false; }
    __host__ __device__ int check_blocks() const { return 0; }
};

// The rows of all sequences of a group, over the tokens [0, len) that these have in common; row: of the block table.
struct Group {
    int32_t q0, qn, len, row;
};
// A batch whose sequences share prefixes, in one of two readings: the groups over their prefixes, every row of a group seeing all of
// it (`groups` not null, num_seqs of them), or the sequences over the tokens behind those.
struct SharedBatch : Batch {
    static constexpr bool kShared = true;
    const Group* groups;
    const int64_t* tile0;  // [groups + 1] first tile of every group in the end-to-end order of all groups' tiles
    const int2* own;       // [num_seqs] tokens in front of x are those of group y; null: nothing is shared
    const int32_t* split;  // CTAs of the groups' pass and of the sequences', which run side by side; null: all of a launch's
    int32_t waits;         // 1: what is read here is written by the kernel in front; 0: that one has waited for it
    // What there is to be checked where nothing is shared, because it would not pay.
    const int32_t *group_starts, *prefix_lens;
    int32_t num_groups, max_group_rows;
    __host__ __device__ bool by_groups() const { return groups != nullptr; }
    __host__ __device__ int check_blocks() const { return !own && !groups; }  // blocks beside a launch's own that check the groups' numbers
};

// Cached tokens of a sequence at most: their indices, rounded up to tiles and blocks or moved by a window, stay below 2^31.
constexpr int32_t kMaxTokens = 1 << 30;

// One sequence of the batch: its rows q0 .. q0+qn-1 are the tokens at cache indices len-qn .. len-1.
struct Seq {
    int32_t q0, qn, len;
    bool ok;
    int32_t row;    // of the block table
    int32_t first;  // tokens in front of it are another pass's
    bool level;     // every row sees all len tokens
    int32_t group;  // whose pass that is
};
// Cache index up to which the sequence's new token `tok` sees, itself included.
__device__ __forceinline__ int last_seen(const Seq& q, int tok) { return q.level ? q.len - 1 : q.len - q.qn + tok; }

__device__ __forceinline__ Seq sequence(const Batch& b, int s, int block_tokens) {
    Seq q;
    int q1;
    if (b.starts) {
        q.q0 = b.starts[s];
        q1 = b.starts[s + 1];
    } else {
        q.q0 = s;
        q1 = s + 1;
    }
    q.len = b.lens[s];
    q.ok = q.q0 >= 0 && q1 >= q.q0 && q1 <= b.num_rows && q1 - q.q0 <= b.max_q_len && q.len >= 0 &&
           q.len <= min((int64_t)b.max_blocks * block_tokens, (int64_t)kMaxTokens);
    q.qn = q.ok ? q1 - q.q0 : 0;
    q.row = s, q.first = 0, q.level = false, q.group = -1;
    return q;
}
__device__ __forceinline__ Seq sequence(const SharedBatch& b, int s, int block_tokens) {
    if (!b.groups) {
        Seq q = sequence(static_cast<const Batch&>(b), s, block_tokens);
        if (b.own) {
            const int2 own = __ldcg(b.own + s);
            q.first = own.x, q.group = own.y;
        }
        return q;
    }
    const int4 g = __ldcg(reinterpret_cast<const int4*>(b.groups) + s);
    Seq q;
    q.q0 = g.x, q.qn = g.y, q.len = g.z, q.row = g.w, q.first = 0, q.group = s;
    q.ok = q.level = true;
    return q;
}

__device__ __forceinline__ void report(int32_t* status, amoeba_status code) { atomicCAS(status, 0, (int)code); }

template <class T>
struct Elem;
template <>
struct Elem<__half> {
    static __device__ __forceinline__ float2 unpack(uint32_t v) {
        return __half22float2(*reinterpret_cast<const __half2*>(&v));
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};
template <>
struct Elem<__nv_bfloat16> {
    static __device__ __forceinline__ float2 unpack(uint32_t v) {
        return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};

__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ void grid_dependency_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// ---------------------------------------------------------------------------------------------- host side
// Fills the view of layer `layer`; checks layout, element type, layer and pool pointers.
inline amoeba_status make_cache_view(const amoeba_layout* l, int32_t layer, const void* const* pools, CacheView* v) {
    if (!l || !pools) return AMOEBA_ERR_INVALID_ARG;
    int64_t bytes = 0;
    const amoeba_status st = amoeba_layout_kv_pool_bytes(l, &bytes);
    if (st != AMOEBA_OK) return st;
    const amoeba_model& m = l->model;
    if (layer < 0 || layer >= m.num_layers) return AMOEBA_ERR_INVALID_ARG;
    if (l->block_tokens > kMaxTokens) return AMOEBA_ERR_UNSUPPORTED;
    const int64_t vec = (int64_t)m.head_dim * m.elem_bytes;
    const int64_t layer_stride = bytes / m.num_layers;
    if (vec % 16 || layer_stride % 16) return AMOEBA_ERR_ALIGNMENT;
    v->heads = m.num_kv_heads / l->tp;
    v->num_blocks = l->num_blocks;
    v->block_tokens = l->block_tokens;
    const int64_t T = l->block_tokens;
    if (l->kv_order == AMOEBA_KV_HEAD_MAJOR) {
        v->tok_stride = vec;
        v->kv_stride = T * vec;
        v->head_stride = 2 * T * vec;
        v->block_stride = v->heads * v->head_stride;
    } else {
        v->head_stride = vec;
        v->tok_stride = v->heads * vec;
        v->block_stride = T * v->tok_stride;
        v->kv_stride = (int64_t)l->num_blocks * v->block_stride;
    }
    for (int r = 0; r < l->tp; ++r) {
        if (!pools[r]) return AMOEBA_ERR_INVALID_ARG;
        if ((uintptr_t)pools[r] % 16) return AMOEBA_ERR_ALIGNMENT;
        v->pools[r] = static_cast<char*>(const_cast<void*>(pools[r])) + layer * layer_stride;
    }
    return AMOEBA_OK;
}

// The operators that interpret elements: 16-bit types, heads of 64 or 128.
inline amoeba_status check_elements(const amoeba_layout* l, int32_t dtype) {
    if (!l) return AMOEBA_ERR_INVALID_ARG;
    if (dtype != AMOEBA_FP16 && dtype != AMOEBA_BF16) return AMOEBA_ERR_UNSUPPORTED;
    if (l->model.elem_bytes != 2 || (l->model.head_dim != 64 && l->model.head_dim != 128)) return AMOEBA_ERR_UNSUPPORTED;
    return AMOEBA_OK;
}

inline amoeba_status make_batch(const amoeba_batch* b, Batch* out) {
    if (!b || b->num_seqs < 0 || b->max_blocks_per_seq < 0 || b->num_rows < 0 || b->max_q_len < 0)
        return AMOEBA_ERR_INVALID_ARG;
    if (b->num_seqs && (!b->d_seq_lens || (b->max_blocks_per_seq && !b->d_block_table))) return AMOEBA_ERR_INVALID_ARG;
    if (!b->d_q_starts && (b->num_rows < b->num_seqs || (b->num_seqs && b->max_q_len < 1))) return AMOEBA_ERR_INVALID_ARG;
    *out = Batch{b->d_block_table, b->d_seq_lens, b->d_q_starts, b->num_seqs, b->max_blocks_per_seq, b->num_rows,
                 b->max_q_len};
    return AMOEBA_OK;
}

// The workers' row buffers; without rows their addresses do not matter.
inline amoeba_status make_rows(const amoeba_layout* l, const Batch& b, const void* const* ptrs, int64_t stride, int64_t row_elems,
                               Rows* out) {
    if (!ptrs) return AMOEBA_ERR_INVALID_ARG;
    if (stride == 0) stride = row_elems;
    if (stride < row_elems) return AMOEBA_ERR_INVALID_ARG;
    out->stride = stride * l->model.elem_bytes;
    if (out->stride % 16) return AMOEBA_ERR_ALIGNMENT;
    for (int r = 0; r < l->tp; ++r) {
        if (!ptrs[r] && b.num_rows) return AMOEBA_ERR_INVALID_ARG;
        if ((uintptr_t)ptrs[r] % 16) return AMOEBA_ERR_ALIGNMENT;
        out->base[r] = static_cast<char*>(const_cast<void*>(ptrs[r]));
    }
    return AMOEBA_OK;
}

// Launches a kernel; early: its blocks may start before the kernel in front of it in the stream has ended (that one has
// called grid_dependency_launch in all its blocks, or they have ended), and call grid_dependency_wait before they use its
// results.
template <class... P, class... A>
inline amoeba_status launch_kernel(void (*kernel)(P...), int grid, int threads, size_t smem, cudaStream_t stream, bool early,
                                   const A&... args) {
    cudaLaunchConfig_t c{};
    c.gridDim = dim3((unsigned)grid);
    c.blockDim = dim3((unsigned)threads);
    c.dynamicSmemBytes = smem;
    c.stream = stream;
    cudaLaunchAttribute a{};
    a.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    a.val.programmaticStreamSerializationAllowed = 1;
    c.attrs = &a;
    c.numAttrs = early ? 1 : 0;
    if (cudaLaunchKernelEx(&c, kernel, static_cast<P>(args)...) != cudaSuccess) {
        (void)cudaGetLastError();
        return AMOEBA_ERR_CUDA;
    }
    count_launch();
    return AMOEBA_OK;
}

#ifdef AMOEBA_CHECK_ITEMS
int32_t operator_wait_polls();  // what a test has set (cache_maps.cu)
#endif

inline bool positive(float x) { return x > 0.f && x < INFINITY; }

}  // namespace amoeba
