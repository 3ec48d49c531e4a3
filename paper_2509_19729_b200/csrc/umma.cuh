// Fifth-generation tensor core pieces (tcgen05) shared by the operators with many query rows: products of 128-row tiles in the
// 128-byte-swizzled layout, tensor memory, and the warps that load such tiles through the block table.
#pragma once
#include "cache_maps.hpp"
#include "copy_engine.cuh"
#include "walk.cuh"
#include "warp_mma.cuh"

namespace amoeba {

// Polls of a wait before it gives up, for mbar_wait_bounded: 0, its own budget.  The checked build lets a test set fewer, so that the
// give-up paths run.
template <class P>
__device__ __forceinline__ uint32_t polls(const P& p) {
#ifdef AMOEBA_CHECK_ITEMS
    return p.polls;
#else
    return 0;
#endif
}

// ---- tensor memory and products
__device__ __forceinline__ void tmem_load32(uint32_t (&r)[32], uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
        "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_store32(uint32_t addr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,"
        "%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
        "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Issued by the lane whose `leader` is 1; the whole warp comes here together, so that the operands stay in uniform registers.
__device__ __forceinline__ void umma_smem(uint32_t leader, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate),
        "r"(leader)
        : "memory");
}
__device__ __forceinline__ void umma_tmem(uint32_t leader, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate),
        "r"(leader)
        : "memory");
}
// The barrier gets one arrival when all products issued so far are done.
__device__ __forceinline__ void umma_commit(uint32_t leader, uint64_t* bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar)), "r"(leader)
        : "memory");
}
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t is;
    asm volatile(
        "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
    return is;
}

// Shared-memory operand in the 128-byte swizzle: groups of eight 128-byte rows 1 KiB apart; `leading` bytes from one
// 64-element half of a row to the next where the rows run along the product's sum (values).
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t leading) {
    return (uint64_t)((addr >> 4) & 0x3fff) | (uint64_t)(leading >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// Product of 16-bit operands into 32 bits, 128 rows, n columns; b_rows: the second operand's rows run along the sum.
template <class T>
__device__ constexpr uint32_t product(int n, bool b_rows) {
    const uint32_t f = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
    return 1u << 4 | f << 7 | f << 10 | (b_rows ? 1u << 16 : 0u) | (uint32_t)(n / 8) << 17 | 8u << 24;
}

// Byte offset of 16-byte chunk c of row r in a tile: 64-element halves of all rows one behind the other.
__device__ __forceinline__ int tile_offset(int r, int c) { return c / 8 * (128 * 128) + r * 128 + ((c ^ r) & 7) * 16; }

// ---- two 32-bit values at a time
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ uint64_t pair2(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void split2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// ---- loading
// One arrival of this thread, when all the asynchronous loads that it has started are done.  The products' warp makes them
// visible to the tensor core (fence_async_smem after its wait): a fence here would wait for the loads still in flight.
__device__ __forceinline__ void arrive_when_loaded(uint64_t* bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// A box of a worker's pool (cache_maps.hpp) into shared memory, by the TMA unit.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int dim, int token, int kv, int head, int block,
                                         uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::
            "r"(dst), "l"(map), "r"(dim), "r"(token), "r"(kv), "r"(head), "r"(block), "r"(smem_u32(bar))
        : "memory");
}
// Where a loading thread is in its ring of tiles: the next one, and the parity that it waits for at its `empty` (the first round
// waits for nothing).
struct RingPlace {
    int slot = 0;
    uint32_t phase = 1;
};
// After some warp has given up: waits until the boxes that this thread has started are there, as the block may not end before.
// Bounded: a tile that not all warps got to never fills.
template <int kStages>
__device__ __forceinline__ void drain_ring(uint64_t* full, RingPlace at) {
    for (int i = 0; i < kStages; ++i)  // (a tile that was never loaded counts as filled in the round before)
        for (uint32_t n = 0; n < kDrainWaitTries && !mbar_test_wait(&full[i], i < at.slot ? at.phase ^ 1 : at.phase); ++n) __nanosleep(64);
}
// The tiles that kWarps warps load together: by boxes where all 128 tokens are wanted and the blocks have a box's shape, else
// each lane 16 bytes at a time.
template <int D, int kWarps>
struct TileLoader {
    const CacheView& v;
    const CacheMaps& maps;
    const int box_rows, warp, lane;    // box_rows 0: no maps
    const char* head = nullptr;        // the key head's part of its pool,
    const int32_t* table = nullptr;    // the sequence's blocks
    const CUtensorMap* map = nullptr;
    int hw = 0;                        // head of the worker
    static constexpr int kChunks = D / 8, kStep = 32 / kChunks;  // a warp loads kStep rows at a time

    __device__ __forceinline__ TileLoader(const CacheView& v_, const CacheMaps& maps_, int box_rows_, int warp_, int lane_)
        : v(v_), maps(maps_), box_rows(box_rows_), warp(warp_), lane(lane_) {}
    __device__ __forceinline__ void open(const Walk& w, const Batch& b) {
        const int r = w.h / v.heads;
        hw = w.h - r * v.heads;
        head = v.pools[r] + hw * v.head_stride;
        map = &maps.worker[r];
        table = b.table + (int64_t)w.s * b.max_blocks;
    }
    // The blocks that the 16 groups of eight tokens of the tile at key0 lie in, one per lane; -1: no token in [lo, hi).  Asked
    // for well ahead: nothing here waits for the answer.
    struct Group {
        int32_t block, in_block;
    };
    __device__ __forceinline__ Group groups(int lo, int hi, int key0) const {
        const int key = key0 + lane * 8;
        Group g{-1, 0};
        if (v.block_tokens % 8 == 0 && lane < 16 && key < hi && key + 8 > lo) {
            const int i = key / v.block_tokens;
            g.in_block = key - i * v.block_tokens;
            g.block = table[i];
        }
        return g;
    }
    // Starts the loads of the keys (kv = 0) or values (1) of 128 tokens, which arrive at `bar` with one arrival of each thread;
    // zeros outside [lo, hi) and for bad blocks.
    __device__ __forceinline__ void tokens(int lo, int hi, int key0, const Group& group, int kv, uint32_t dst, uint64_t* bar) const {
        const bool good = group.block >= 0 && group.block < v.num_blocks;
        if (box_rows && key0 >= lo && key0 + 128 <= hi && __all_sync(~0u, lane >= 16 || good)) {
            constexpr int kHalves = D / 64;
            const int i = warp + lane * kWarps, row = i / kHalves * box_rows, half = i % kHalves;
            const int block = __shfl_sync(~0u, group.block, row / 8 & 15), token = __shfl_sync(~0u, group.in_block, row / 8 & 15);
            if (row < 128) {
                mbar_arrive_expect_tx(bar, box_rows * 128);
                load_box(dst + half * (128 * 128) + row * 128, map, half * 64, token, kv, hw, block, bar);
            } else {
                mbar_arrive(bar);
            }
            return;
        }
        const int c = lane % kChunks, sub = lane / kChunks;
        const char* from = head + kv * v.kv_stride + c * 16;
        if (v.block_tokens % 8 == 0) {
            const int64_t at = good ? group.block * v.block_stride + group.in_block * v.tok_stride : -1;
            const int64_t step = kStep * v.tok_stride;
#pragma unroll
            for (int j = 0; j < (16 + kWarps - 1) / kWarps; ++j) {
                const int g = warp + j * kWarps, r0 = g * 8 + sub;
                const int64_t own = __shfl_sync(~0u, at, g & 15);
                const char* src = from + (own >= 0 ? own : 0) + sub * v.tok_stride;
                const int l = own >= 0 ? lo - key0 - r0 : 128, h = hi - key0 - r0;  // rows [l, h) of r0, r0 + kStep, ... are wanted
                if (g < 16) {
#pragma unroll
                    for (int i = 0; i < 8 / kStep; ++i)
                        cp_async16(dst + g * 1024 + tile_offset(i * kStep + sub, c), src + i * step, i * kStep >= l && i * kStep < h ? 16 : 0);
                }
            }
        } else {
#pragma unroll 1
            for (int g = warp; g < 16; g += kWarps) {
#pragma unroll 1
                for (int i = 0; i < 8 / kStep; ++i) {
                    const int r = g * 8 + i * kStep + sub, key = key0 + r;
                    bool in = key >= lo && key < hi;
                    const char* src = head;
                    if (in) {
                        const int block = table[key / v.block_tokens];
                        in = block >= 0 && block < v.num_blocks;
                        if (in) src = from + block * v.block_stride + key % v.block_tokens * v.tok_stride;
                    }
                    cp_async16(dst + tile_offset(r, c), src, in ? 16 : 0);
                }
            }
        }
        arrive_when_loaded(bar);
    }
    // Starts the loads of `count` (at most 128) query rows of w's sequence and key head, from row `row` on; behind them zeros, or
    // (kRepeat) the last of them over and over.
    template <bool kRepeat = false>
    __device__ __forceinline__ void queries(const Rows& q, const Walk& w, int group, int row, int count, uint32_t dst) const {
        const int c = lane % kChunks, sub = lane / kChunks, worker = w.h / v.heads;
        const char* base = q.base[worker] + (int64_t)w.seq.q0 * q.stride + (w.h - worker * v.heads) * group * (D * 2) + c * 16;
        for (int first = warp * 32; first < 128; first += kWarps * 32) {
            const int r = row + (kRepeat ? min(first + lane, count - 1) : first + lane), tok = r / group;
            const int64_t mine = kRepeat || first + lane < count ? tok * q.stride + (r - tok * group) * (D * 2) : -1;
#pragma unroll
            for (int i = 0; i < 32; i += kStep) {
                const int64_t off = __shfl_sync(~0u, mine, i + sub);
                cp_async16(dst + tile_offset(first + i + sub, c), off >= 0 ? base + off : v.pools[0], off >= 0 ? 16 : 0);
            }
        }
    }
};

}  // namespace amoeba
