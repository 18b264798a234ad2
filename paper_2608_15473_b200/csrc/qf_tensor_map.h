// Host side: the driver's descriptor encoder, and descriptors of scaled pools.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdio>
#include <mutex>

#include "qf_common.cuh"

namespace qf {

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_tiled(char *msg, size_t msg_len)
{
    static std::mutex mu;
    static EncodeTiledFn encode = nullptr;
    std::lock_guard<std::mutex> lock(mu);
    if (!encode) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult qres;
        cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres);
        if (e != cudaSuccess || qres != cudaDriverEntryPointSuccess || !fn) {
            snprintf(msg, msg_len, "cuTensorMapEncodeTiled entry point not available");
            return nullptr;
        }
        encode = (EncodeTiledFn)fn;
    }
    return encode;
}

// A pool of codes in boxes of one (page, KV head) block of 16 rows: [block, row, 128 B] (head-major), or [token row, head, 128 B],
// 16 rows of one head (token-major).  Either way the outermost coordinate says which page.  swizzled: 128B swizzle, else rows as they are.  Encoded for every call (under a
// microsecond), so nothing is remembered about a pointer.
inline int make_scaled_map(CUtensorMap *out, const void *pool, long long num_pages, int num_kv_heads, bool nhd, bool swizzled,
                           char *msg, size_t msg_len)
{
    EncodeTiledFn encode = encode_tiled(msg, msg_len);
    if (!encode) return -1;
    const cuuint64_t hkv = (cuuint64_t)num_kv_heads, rows = (cuuint64_t)num_pages * kPageSize;
    const cuuint64_t dims[3] = {(cuuint64_t)kHeadDim, nhd ? hkv : (cuuint64_t)kPageSize, nhd ? rows : (cuuint64_t)num_pages * hkv};
    const cuuint64_t strides[2] = {(cuuint64_t)kHeadDim, (nhd ? hkv : (cuuint64_t)kPageSize) * kHeadDim};
    const cuuint32_t box[3] = {(cuuint32_t)kHeadDim, nhd ? 1u : (cuuint32_t)kPageSize, nhd ? (cuuint32_t)kPageSize : 1u}, ones[3] = {1, 1, 1};
    const CUresult r = encode(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void *>(pool), dims, strides, box, ones,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, swizzled ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
                              nhd ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r == CUDA_SUCCESS) return 0;
    snprintf(msg, msg_len, "cuTensorMapEncodeTiled failed with CUresult %d", (int)r);
    return -1;
}

}  // namespace qf
