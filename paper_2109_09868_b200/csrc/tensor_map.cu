// Tensor maps, encoded by the driver's function of that name (looked up once; the library links no driver library).
#include "async.cuh"

namespace approxifer {

cudaError_t make_tensor_map(CUtensorMap* map, const void* base, int rank, const uint64_t* extent, const uint64_t* stride, const uint32_t* box) {
  using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                              CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static std::atomic<void*> found{nullptr};
  void* fn = found.load(std::memory_order_acquire);
  if (fn == nullptr) {
    cudaDriverEntryPointQueryResult state;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &state);
    if (e != cudaSuccess) return e;
    if (state != cudaDriverEntryPointSuccess || fn == nullptr) return cudaErrorNotSupported;
    found.store(fn, std::memory_order_release);
  }
  cuuint64_t ext[5], bytes[5];
  cuuint32_t bx[5], ones[5];
  for (int i = 0; i < rank; ++i) ext[i] = extent[i], bx[i] = box[i], ones[i] = 1;
  for (int i = 1; i < rank; ++i) bytes[i - 1] = stride[i] * 2;
  const CUresult r = reinterpret_cast<Encode>(fn)(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(base), ext, bytes, bx, ones,
                                                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace approxifer
