// Warp-level pieces shared by the operators that read the cache with few query rows: asynchronous 16-byte loads into
// swizzled shared memory, 8x8 matrix loads and the 16x8x16 matrix instruction.
#pragma once
#include "copy_engine.cuh"
#include "walk.cuh"

namespace amoeba {

// 16 bytes global -> shared; src_bytes 0 writes zeros and reads nothing.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int src_bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
// The same, for what is not read again soon: it is the first to leave L2.
__device__ __forceinline__ void cp_async16_once(uint32_t dst, const void* src, int src_bytes, uint64_t policy) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst), "l"(src), "r"(src_bytes), "l"(policy) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// Transposes an 8x8 matrix of 16-bit elements spread over the warp.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

template <class T>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16816<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Byte offset of 16-byte chunk c of row r in a tile of D-element rows: the chunks of a row are permuted by its number,
// so that the eight rows of a matrix load fall into different banks.
template <int D>
__device__ __forceinline__ int swizzled(int r, int c) {
    return r * (D * 2) + ((c & 8) | ((c ^ r) & 7)) * 16;
}

// One warp's loads of 16 consecutive tokens' keys (and, kValues, values) of one head at a time, [K][V][16][D] swizzled, ahead
// of the warp's own walk over the tiles (kTile tokens each, the warp's 16 at `offset` in every tile).  The block that the
// next tokens lie in is looked up one step early.
template <int D, bool kValues, int kTile, class B = Batch>
struct Ahead {
    const CacheView& v;
    const B& b;
    const Shape& shape;
    int32_t* status;
    const int lane, offset;
    const bool one_block;  // 16 tokens lie in one block
    uint64_t policy = 0;   // of a SharedBatch's loads
    Walk w;
    int64_t left;          // tiles to go
    const int32_t* table;
    const char* head;
    int32_t hw, block = -1, in_block = 0;

    __device__ __forceinline__ Ahead(const CacheView& v_, const B& b_, const Shape& s_, int32_t* status_, const Walk& w_, int64_t n,
                                     int offset_)
        : v(v_), b(b_), shape(s_), status(status_), lane(threadIdx.x & 31), offset(offset_), one_block(v_.block_tokens % 16 == 0), w(w_),
          left(n) {
        if (B::kShared) policy = policy_evict_first();
        if (left > 0) {
            open();
            look_up();
        }
    }
    __device__ __forceinline__ void open() {
        table = b.table + (int64_t)w.seq.row * b.max_blocks;
        const int r = w.h / v.heads;
        hw = w.h - r * v.heads;
        head = v.pools[r] + hw * v.head_stride;
    }
    __device__ __forceinline__ void start(uint32_t dst, const void* src, int src_bytes) const {
        if (B::kShared) cp_async16_once(dst, src, src_bytes, policy);
        else cp_async16(dst, src, src_bytes);
    }
    __device__ __forceinline__ int key0() const { return w.range.base + w.t * kTile + offset; }
    __device__ __forceinline__ void look_up() {
        const int k = key0();
        block = -1;
        if (one_block && k < w.range.hi && k + 16 > w.range.lo) {
            const int i = k / v.block_tokens;
            in_block = k - i * v.block_tokens;
            block = table[i];
        }
    }
    // Starts the loads into `dst`; tokens outside [lo, hi) of the unit and of bad blocks become zeros.  Returns the mask of
    // the others; *slot: of the 16 tokens' first score in the worker's score pool, where they lie in one block.
    __device__ __forceinline__ uint32_t load(uint32_t dst, int64_t* slot) {
        constexpr int kChunks = D / 8, kStep = 32 / kChunks, kRows = 16 / kStep;
        const int c = lane % kChunks, r0 = lane / kChunks, lo = w.range.lo, hi = w.range.hi, k0 = key0();
        uint32_t mask = 0;
        bool bad = false;
        if (one_block) {
            const bool ok = block >= 0 && block < v.num_blocks;
            bad = !ok && k0 < hi && k0 + 16 > lo;
            if (ok) {
                const int a = max(lo - k0, 0), z = min(hi - k0, 16);
                mask = ((1u << z) - 1) & ~((1u << a) - 1);
            }
            *slot = ((int64_t)block * v.heads + hw) * v.block_tokens + in_block;
            const char* src = head + (ok ? block * v.block_stride + in_block * v.tok_stride : 0) + r0 * v.tok_stride + c * 16;
            if (mask == 0xffffu) {
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    const char* s = src + i * kStep * v.tok_stride;
                    start(dst + swizzled<D>(r0 + i * kStep, c), s, 16);
                    if (kValues) start(dst + 16 * D * 2 + swizzled<D>(r0 + i * kStep, c), s + v.kv_stride, 16);
                }
            } else {
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    const int r = r0 + i * kStep;
                    const bool in = mask >> r & 1u;
                    const char* s = in ? src + i * kStep * v.tok_stride : head;
                    start(dst + swizzled<D>(r, c), s, in ? 16 : 0);
                    if (kValues) start(dst + 16 * D * 2 + swizzled<D>(r, c), in ? s + v.kv_stride : s, in ? 16 : 0);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int r = r0 + i * kStep, key = k0 + r;
                bool in = key >= lo && key < hi;
                const char* s = head;
                if (in) {
                    const int own = table[key / v.block_tokens];
                    in = own >= 0 && own < v.num_blocks;
                    bad |= !in;
                    if (in) s = head + own * v.block_stride + (key % v.block_tokens) * v.tok_stride + c * 16;
                }
                start(dst + swizzled<D>(r, c), s, in ? 16 : 0);
                if (kValues) start(dst + 16 * D * 2 + swizzled<D>(r, c), in ? s + v.kv_stride : s, in ? 16 : 0);
                const uint32_t there = __ballot_sync(~0u, in);
#pragma unroll
                for (int j = 0; j < kStep; ++j) mask |= (there >> (j * kChunks) & 1u) << (i * kStep + j);
            }
        }
        if (bad) report(status, AMOEBA_ERR_BAD_BLOCK_ID);
        if (--left > 0) {
            const int h = w.h, s = w.s;
            w.next(shape, b, v.block_tokens);
            if (w.h != h || w.s != s) open();
            look_up();
        }
        return mask;
    }
};

}  // namespace amoeba
