// Tensor maps for TMA loads of 16-bit tiles whose rows are 16, 32 or 64 values, in the swizzle of their width.
#pragma once
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>

#include <initializer_list>

#include "serve_internal.h"

namespace bcast_serve {

// cuTensorMapEncodeTiled from the driver that is loaded, or nullptr.
inline PFN_cuTensorMapEncodeTiled_v12000 encode_tiled()
{
    static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess ||
            r != cudaDriverEntryPointSuccess)
            p = nullptr;
        return (PFN_cuTensorMapEncodeTiled_v12000)p;
    }();
    return fn;
}

// An array of `size` (innermost first, contiguous), the outer dimensions' strides in elements, read in boxes of
// `box`.  What a box covers outside the array reads as zero.
inline int tensor_map(CUtensorMap *map, CUtensorMapDataType type, const void *base, std::initializer_list<int64_t> size,
                      std::initializer_list<int64_t> stride, std::initializer_list<int64_t> box)
{
    const auto encode = encode_tiled();
    if (!encode) return bcast_internal_cuda_failed((int)cudaErrorSymbolNotFound);
    cuuint64_t s[5], st[4];
    cuuint32_t b[5], one[5] = {1, 1, 1, 1, 1};
    cuuint32_t n = 0;
    for (int64_t v : size) s[n++] = (cuuint64_t)v;
    n = 0;
    for (int64_t v : stride) st[n++] = (cuuint64_t)v * 2;
    n = 0;
    for (int64_t v : box) b[n++] = (cuuint32_t)v;
    const int64_t row = *box.begin() * 2;
    const auto swizzle = row == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : row == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B;
    const CUresult r = encode(map, type, n, const_cast<void *>(base), s, st, b, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? BCAST_OK : bcast_internal_cuda_failed((int)cudaErrorInvalidValue);
}

}  // namespace bcast_serve
