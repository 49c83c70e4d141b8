// Tensor maps (host side): the driver's encoder, and a map over rows of bf16 elements with three outer dimensions.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <mutex>

#include "wkv_internal.cuh"

namespace wkv {

typedef CUresult (*TensorMapEncoder)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                     const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                     CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline TensorMapEncoder tensor_map_encoder()
{
    static TensorMapEncoder fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &qres) == cudaSuccess &&
            qres == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<TensorMapEncoder>(p);
        else
            (void)cudaGetLastError();
    });
    return fn;
}

struct RowDim {
    unsigned long long size;      // elements along it
    unsigned long long stride;    // bytes
    unsigned box;                 // of a loaded tile
};
// Rows of d bf16 elements, boxes of 64 of them (128 bytes, 128-byte swizzle, zeros beyond the tensor) times dims[].box; or, with
// `codes`, rows of d bytes, boxes of `codes` of them, not swizzled.  slot[i] is
// the coordinate (1 .. 3) that dims[i] became: dimensions follow in order of increasing stride, those of size one last with a
// stride of their own making.
inline bool make_row_tensor_map(const void *base, int d, const RowDim (&dims)[3], CUtensorMap *tmap, int (&slot)[3], int codes = 0)
{
    TensorMapEncoder enc = tensor_map_encoder();
    if (!enc) {
        set_error_detail("cuTensorMapEncodeTiled is not available from the driver");
        return false;
    }
    int order[3] = {0, 1, 2};
    std::stable_sort(order, order + 3, [&](int x, int y) {
        const bool x1 = dims[x].size == 1, y1 = dims[y].size == 1;
        if (x1 != y1) return y1;
        return !x1 && dims[x].stride < dims[y].stride;
    });
    unsigned long long running = (unsigned long long)d * (codes ? 1ull : 2ull);
    cuuint64_t gdim[4] = {(cuuint64_t)d, 0, 0, 0}, gstride[3];
    cuuint32_t box[4] = {codes ? (cuuint32_t)codes : 64, 1, 1, 1}, estr[4] = {1, 1, 1, 1};
    for (int i = 0; i < 3; ++i) {
        const RowDim &x = dims[order[i]];
        const unsigned long long stride = x.size == 1 ? running : x.stride;
        if (stride == 0 || stride % 16 || stride >= (1ull << 40) || x.size > 0xffffffffull || x.box > 256) {
            set_error_detail("layout cannot be described by a tensor map (dimension %d: size %llu, stride %llu bytes)", order[i], x.size, stride);
            return false;
        }
        gdim[i + 1] = x.size;
        gstride[i] = stride;
        box[i + 1] = x.box;
        slot[order[i]] = i + 1;
        if (stride * x.size > running) running = stride * x.size;
    }
    const CUresult r = enc(tmap, codes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(base), gdim, gstride, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, codes ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        set_error_detail("cuTensorMapEncodeTiled failed with code %d", (int)r);
        return false;
    }
    return true;
}

}  // namespace wkv
