// rf_ops.cpp -- tensor maps for the operators around the attention.
#include "rf_ops.h"

#include <cudaTypedefs.h>

#include <cstdio>

namespace rf {

namespace {
PFN_cuTensorMapEncodeTiled_v12000 find_encode() {
  void* ptr = nullptr;
  cudaDriverEntryPointQueryResult q;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault,
                                       &q) != cudaSuccess ||
      q != cudaDriverEntryPointSuccess)
    return nullptr;
  return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(ptr);
}
}  // namespace

rf_status make_tensor_map(CUtensorMap* m, int dtype, const void* base, int rank,
                          const uint64_t* dims, const uint64_t* strides, const uint32_t* box) {
  static const PFN_cuTensorMapEncodeTiled_v12000 encode = find_encode();
  if (!encode) return fail(RF_ERR_CUDA, "cuTensorMapEncodeTiled entry point not found");
  cuuint64_t d[3], s[2];
  cuuint32_t b[3], e[3] = {1, 1, 1};
  for (int i = 0; i < rank; ++i) {
    d[i] = dims[i];
    b[i] = box[i];
    if (i > 0) s[i - 1] = strides[i - 1];
  }
  const CUresult r =
      encode(m, dtype == RF_FP32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                : dtype == RF_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                   : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
             static_cast<cuuint32_t>(rank), const_cast<void*>(base), d, s, b, e,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    char buf[96];
    std::snprintf(buf, sizeof(buf), "cuTensorMapEncodeTiled failed (CUresult %d)",
                  static_cast<int>(r));
    return fail(RF_ERR_CUDA, buf);
  }
  return RF_OK;
}

}  // namespace rf
