// tensor_map.cu -- tensor maps of the first-order operators' TMA copies
// (tc_tiles.cuh).
#include "soma_api.h"
#include "tc_tiles.cuh"

namespace soma {

namespace {

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                            const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                            const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's encoder, found through the runtime: the library does not link
// the driver.
Encode encoder() {
  static const Encode f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                         &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<Encode>(p);
  }();
  return f;
}

CUtensorMapDataType type_of(int dtype) {
  return dtype == SOMA_FP32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
         : dtype == SOMA_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                              : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
}

}  // namespace

bool make_tile_map(CUtensorMap* map, const void* base, int dtype, int64_t rows, int64_t cols,
                   int64_t stride, int box_rows) {
  const Encode encode = encoder();
  if (!encode) return false;
  const int width = dtype == SOMA_FP32 ? 4 : 2;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)stride * width};
  const cuuint32_t box[2] = {128u / width, (cuuint32_t)box_rows};
  const cuuint32_t step[2] = {1, 1};
  return encode(map, type_of(dtype), 2, const_cast<void*>(base), dims, strides, box, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool make_box_map(CUtensorMap* map, const void* base, int dtype, const int64_t (&size)[3],
                  const int64_t (&stride)[2], const int (&box_size)[3]) {
  const Encode encode = encoder();
  if (!encode) return false;
  const int width = dtype == SOMA_FP32 ? 4 : 2;
  const cuuint64_t dims[3] = {(cuuint64_t)size[0], (cuuint64_t)size[1], (cuuint64_t)size[2]};
  const cuuint64_t strides[2] = {(cuuint64_t)stride[0] * width, (cuuint64_t)stride[1] * width};
  const cuuint32_t box[3] = {(cuuint32_t)box_size[0], (cuuint32_t)box_size[1],
                             (cuuint32_t)box_size[2]};
  const cuuint32_t step[3] = {1, 1, 1};
  return encode(map, type_of(dtype), 3, const_cast<void*>(base), dims, strides, box, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace soma
