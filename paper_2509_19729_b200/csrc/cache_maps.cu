// Encoding of the cache's tensor maps: cuTensorMapEncodeTiled, looked up through the runtime so that the library does not
// link against the driver.
#include "cache_maps.hpp"

#include <atomic>
#include <mutex>

#ifdef AMOEBA_CHECK_ITEMS
static std::atomic<int32_t> g_wait_polls{0};
namespace amoeba {
int32_t operator_wait_polls() { return g_wait_polls; }
}  // namespace amoeba
extern "C" AMOEBA_API void amoeba_checked_set_wait_polls(int32_t polls) { g_wait_polls = polls < 0 ? 0 : polls; }
#endif

namespace amoeba {

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiled encoder() {
    static std::once_flag once;
    static EncodeTiled fn = nullptr;
    std::call_once(once, [] {
        void* sym = nullptr;
        cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiled>(sym);
        else
            (void)cudaGetLastError();
    });
    return fn;
}

bool encode_cache_map(CUtensorMap* out, const CacheView& v, int worker, int head_dim, int box_rows, int32_t dtype) {
    const EncodeTiled encode = encoder();
    if (!encode) return false;
    const cuuint64_t dims[5] = {(cuuint64_t)head_dim, (cuuint64_t)v.block_tokens, 2, (cuuint64_t)v.heads, (cuuint64_t)v.num_blocks};
    const cuuint64_t strides[4] = {(cuuint64_t)v.tok_stride, (cuuint64_t)v.kv_stride, (cuuint64_t)v.head_stride,
                                   (cuuint64_t)v.block_stride};
    const cuuint32_t box[5] = {64, (cuuint32_t)box_rows, 1, 1, 1}, steps[5] = {1, 1, 1, 1, 1};
    return encode(out, dtype == AMOEBA_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, v.pools[worker],
                  dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace amoeba
