// Host side of the tensor-map loads: the driver's encode function and maps of row-major tensors, 128-byte swizzle.
#pragma once

#include <atomic>

#include <cuda.h>

#include "common.cuh"

namespace cobalt {

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline int encode_function(EncodeTiled* out)
{
    static std::atomic<EncodeTiled> cached{nullptr};         // the same for every device
    EncodeTiled known = cached.load(std::memory_order_relaxed);
    if (!known) {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        COBALT_CUDA_TRY(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found));
        if (found != cudaDriverEntryPointSuccess || !f) return COBALT_ERR_UNSUPPORTED;
        known = reinterpret_cast<EncodeTiled>(f);
        cached.store(known, std::memory_order_relaxed);
    }
    *out = known;
    return COBALT_OK;
}

// A tensor of bf16 (elem_bytes 2) or one-byte values of up to five dimensions, the first one contiguous; strides of the others in
// elements.
inline int make_map(CUtensorMap* map, const void* ptr, int rank, const uint64_t (&dim)[5], const uint64_t (&stride)[5], const uint32_t (&box)[5],
                    int elem_bytes = 2)
{
    EncodeTiled encode;
    const int rc = encode_function(&encode);
    if (rc != COBALT_OK) return rc;
    cuuint64_t dims[5], bytes[4];
    cuuint32_t boxes[5], ones[5] = {1, 1, 1, 1, 1};
    for (int i = 0; i < rank; ++i) {
        dims[i] = dim[i];
        boxes[i] = box[i];
        if (i > 0) bytes[i - 1] = stride[i] * elem_bytes;
    }
    const CUresult r = encode(map, elem_bytes == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, rank, const_cast<void*>(ptr),
                              dims, bytes, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? COBALT_OK : record_cuda_error(cudaErrorInvalidValue);
}

// [rows, columns], columns contiguous; boxes of box_columns (128 bytes) by box_rows.
inline int matrix_map(CUtensorMap* map, const void* ptr, int64_t rows, int64_t columns, uint32_t box_columns, uint32_t box_rows, int elem_bytes = 2)
{
    const uint64_t dim[5] = {static_cast<uint64_t>(columns), static_cast<uint64_t>(rows)}, stride[5] = {1, static_cast<uint64_t>(columns)};
    const uint32_t box[5] = {box_columns, box_rows};
    return make_map(map, ptr, 2, dim, stride, box, elem_bytes);
}

}  // namespace cobalt
