// Tensor maps of the tiled copies, through the driver's encoder (looked up at run time: the library does not link libcuda).
#include "tensorcore.cuh"

namespace aweq {

using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                            const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static aweq_status encode_map(CUtensorMap *map, CUtensorMapDataType type, int rank, const void *base, const cuuint64_t *dims,
                              const cuuint64_t *strides, const cuuint32_t *box)
{
    static const Encode encode = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<Encode>(f);
    }();
    if (!encode) return AWEQ_ERR_UNSUPPORTED;
    const cuuint32_t step[4] = {1, 1, 1, 1};
    const CUresult r = encode(map, type, (cuuint32_t)rank, const_cast<void *>(base), dims, strides, box, step,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? AWEQ_OK : cuda_failed(cudaErrorInvalidValue);
}

aweq_status tma_bytes_map(CUtensorMap *map, const void *base, long long rows, long long cols, long long ld, int box_rows)
{
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, pitch[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {128, (cuuint32_t)box_rows};
    return encode_map(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, dims, pitch, box);
}

aweq_status tma_pool_map(CUtensorMap *map, const void *base, long long pages, int tokens, int heads, int dim, long long page_stride,
                         long long token_stride, long long head_stride, int box_tokens)
{
    const cuuint64_t dims[4] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)tokens, (cuuint64_t)pages};
    const cuuint64_t strides[3] = {(cuuint64_t)head_stride * 2, (cuuint64_t)token_stride * 2, (cuuint64_t)page_stride * 2};
    const cuuint32_t box[4] = {64, 1, (cuuint32_t)box_tokens, 1};
    return encode_map(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 4, base, dims, strides, box);
}

}  // namespace aweq
