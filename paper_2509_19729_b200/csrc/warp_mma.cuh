// Warp-level pieces shared by the operators that read the cache with few query rows: asynchronous 16-byte loads into
// swizzled shared memory, 8x8 matrix loads and the 16x8x16 matrix instruction.
#pragma once
#include "cache_view.cuh"

namespace amoeba {

// 16 bytes global -> shared; src_bytes 0 writes zeros and reads nothing.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int src_bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
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

// Starts the loads of 16 consecutive tokens' keys (and, with_values, values) of one head into `dst`, [K][V][16][D]
// swizzled, by one warp; tokens outside [lo, hi) and of bad blocks become zeros.  Returns the mask of the others.
// table: the sequence's row of the block table; head: the head's base address in its pool.
template <int D, bool kValues>
__device__ __forceinline__ uint32_t load16(const CacheView& v, const int32_t* table, const char* head, int key0, int lo,
                                           int hi, uint32_t dst, int32_t* status) {
    constexpr int kChunks = D / 8, kStep = 32 / kChunks, kRows = 16 / kStep;
    const int lane = threadIdx.x & 31, c = lane % kChunks, r0 = lane / kChunks;
    uint32_t mask = 0;
    bool bad = false;
    if (v.block_tokens % 16 == 0) {  // key0 is a multiple of 16: all in one block
        int block = -1;
        if (key0 < hi && key0 + 16 > lo) {
            block = table[key0 / v.block_tokens];
            bad = block < 0 || block >= v.num_blocks;
        }
        const bool ok = block >= 0 && !bad;
        const char* src = head + (ok ? block * v.block_stride + (key0 % v.block_tokens) * v.tok_stride : 0) + c * 16;
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int r = r0 + i * kStep;
            const bool in = ok && key0 + r >= lo && key0 + r < hi;
            const char* s = in ? src + r * v.tok_stride : head;
            cp_async16(dst + swizzled<D>(r, c), s, in ? 16 : 0);
            if (kValues) cp_async16(dst + 16 * D * 2 + swizzled<D>(r, c), in ? s + v.kv_stride : s, in ? 16 : 0);
        }
        if (ok) {
            const int a = max(lo - key0, 0), b = min(hi - key0, 16);
            mask = ((1u << b) - 1) & ~((1u << a) - 1);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int r = r0 + i * kStep, key = key0 + r;
            bool in = key >= lo && key < hi;
            const char* s = head;
            if (in) {
                const int block = table[key / v.block_tokens];
                in = block >= 0 && block < v.num_blocks;
                bad |= !in;
                if (in) s = head + block * v.block_stride + (key % v.block_tokens) * v.tok_stride + c * 16;
            }
            cp_async16(dst + swizzled<D>(r, c), s, in ? 16 : 0);
            if (kValues) cp_async16(dst + 16 * D * 2 + swizzled<D>(r, c), in ? s + v.kv_stride : s, in ? 16 : 0);
            const uint32_t there = __ballot_sync(~0u, in);
#pragma unroll
            for (int j = 0; j < kStep; ++j) mask |= (there >> (j * kChunks) & 1u) << (i * kStep + j);
        }
    }
    if (bad) report(status, AMOEBA_ERR_BAD_BLOCK_ID);
    return mask;
}

}  // namespace amoeba
