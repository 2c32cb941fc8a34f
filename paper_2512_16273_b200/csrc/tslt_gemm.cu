// Tensor maps for the matrix-product engine.
#include "tslt_gemm.cuh"

namespace tslt {
namespace gemm {

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeFn encoder() {
    static EncodeFn fn = nullptr;  // every thread that races here stores the same pointer
    if (!fn) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult res;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &res) != cudaSuccess) return nullptr;
        fn = reinterpret_cast<EncodeFn>(p);
    }
    return fn;
}

static bool encode(CUtensorMap* map, Element e, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
    const EncodeFn fn = encoder();
    const cuuint32_t step[3] = {1, 1, 1};
    const CUtensorMapDataType type = e == kElemInt8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : e == kElemBf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
    const auto once = [&] {
        return fn(map, type, rank, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    };
    if (!fn) return false;
    CUresult r = once();
    if (r == CUDA_ERROR_INVALID_CONTEXT || r == CUDA_ERROR_NOT_INITIALIZED) {
        // a thread that has used the device through nothing that binds its context yet: the driver's calls do not bind it themselves
        int dev = -1;
        if (cudaGetDevice(&dev) != cudaSuccess || cudaSetDevice(dev) != cudaSuccess) return false;
        r = once();
    }
    return r == CUDA_SUCCESS;
}

bool encode_map(CUtensorMap* map, Element e, const void* base, long long inner, long long outer, long long row_bytes, int box_outer) {
    const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer}, strides[1] = {(cuuint64_t)row_bytes};
    const cuuint32_t box[2] = {e == kElemInt8 ? 128u : e == kElemBf16 ? 64u : 32u, (cuuint32_t)box_outer};
    return encode(map, e, base, 2, dims, strides, box);
}

bool encode_blocks(CUtensorMap* map, const void* base, long long rows, long long row_bytes, long long blocks, long long block_bytes, int box_blocks) {
    const cuuint64_t dims[3] = {64, (cuuint64_t)rows, (cuuint64_t)blocks}, strides[2] = {(cuuint64_t)row_bytes, (cuuint64_t)block_bytes};
    const cuuint32_t box[3] = {64, 64, (cuuint32_t)box_blocks};
    return encode(map, kElemBf16, base, 3, dims, strides, box);
}

}  // namespace gemm
}  // namespace tslt
