// Tensor maps (tiled TMA) of one layer of a worker's pool, for the operators that load tiles of 128 tokens.
#pragma once
#include <cuda.h>

#include "cache_view.cuh"

namespace amoeba {

// Rows of a box: tokens of one block that a copy moves, a power of two from 8 to 128 that divides block_tokens; 0: there is
// none, and the tiles are loaded 16 bytes at a time.
inline int map_box_rows(int block_tokens) {
    for (int b = 128; b >= 8; b /= 2)
        if (block_tokens % b == 0) return b;
    return 0;
}
// Map of {dim, token of the block, K/V, head, block} with boxes of 64 elements of `box_rows` tokens, 128-byte swizzled.
// False: the driver refused, or has no such call.
bool encode_cache_map(CUtensorMap* out, const CacheView& v, int worker, int head_dim, int box_rows, int32_t dtype);

// The maps of all workers, as kernel parameters.
struct CacheMaps {
    CUtensorMap worker[AMOEBA_MAX_TP];
};
// Fills the maps; returns the box rows, 0 if they cannot be used.
inline int make_cache_maps(CacheMaps* maps, const CacheView& v, int tp, int head_dim, int32_t dtype) {
    const int rows = map_box_rows(v.block_tokens);
    for (int r = 0; rows && r < tp; ++r)
        if (!encode_cache_map(&maps->worker[r], v, r, head_dim, rows, dtype)) return 0;
    return rows;
}

}  // namespace amoeba
