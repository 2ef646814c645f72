// Tensor maps of the 8-bit products' operands (host side).
#pragma once

#include <cuda.h>

#include "internal.cuh"

namespace svdc {

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

inline EncodeTiledFn tensor_map_encoder() {
    static EncodeTiledFn fn = [] {
        void *ptr = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            return reinterpret_cast<EncodeTiledFn>(ptr);
        return (EncodeTiledFn) nullptr;
    }();
    return fn;
}

// bytes [rows x cols], rows `ld` bytes apart, or `count` such matrices `stride` bytes apart (count 0: one, as a map of two dimensions), in
// boxes of 128 bytes x box_rows (x 1) with the 128-byte swizzle; bytes beyond a matrix read as zero, which is e4m3's zero.  Where rows begin
// at multiples of 256 bytes, L2 fetches so many at a time, two groups of K that are read one after the other (1 x 18432 x 9216 31.7 -> 29.5
// us); elsewhere half of such a fetch may belong to another row (256 x 6912 x 9000 27.1 -> 29.3 us, 40 x 18432 x 400 4.8 -> 5.2).
inline int byte_map(CUtensorMap *m, const void *base, int64_t rows, int cols, int64_t ld, int box_rows, int64_t count = 0, int64_t stride = 0) {
    EncodeTiledFn fn = tensor_map_encoder();
    if (!fn) return SVDCACHE_ERR_CUDA;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)count};
    const cuuint64_t strides[2] = {(cuuint64_t)ld, (cuuint64_t)stride};
    const cuuint32_t box[3] = {128, (cuuint32_t)box_rows, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, count > 0 ? 3 : 2, const_cast<void *>(base), dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                          ld % 256 == 0 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? SVDCACHE_OK : SVDCACHE_ERR_CUDA;
}

}  // namespace svdc
