// Tensor maps, encoded by the driver's function of that name (looked up once; the library links no driver library).
#include "async.cuh"

namespace approxifer {
namespace {

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                            CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
cudaError_t find_encode(Encode* encode) {
  static std::atomic<void*> found{nullptr};
  void* fn = found.load(std::memory_order_acquire);
  if (fn == nullptr) {
    cudaDriverEntryPointQueryResult state;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &state);
    if (e != cudaSuccess) return e;
    if (state != cudaDriverEntryPointSuccess || fn == nullptr) return cudaErrorNotSupported;
    found.store(fn, std::memory_order_release);
  }
  *encode = reinterpret_cast<Encode>(fn);
  return cudaSuccess;
}

}  // namespace

cudaError_t make_tensor_map(CUtensorMap* map, const void* base, int rank, const uint64_t* extent, const uint64_t* stride, const uint32_t* box) {
  Encode encode;
  const cudaError_t e = find_encode(&encode);
  if (e != cudaSuccess) return e;
  cuuint64_t ext[5], bytes[5];
  cuuint32_t bx[5], ones[5];
  for (int i = 0; i < rank; ++i) ext[i] = extent[i], bx[i] = box[i], ones[i] = 1;
  for (int i = 1; i < rank; ++i) bytes[i - 1] = stride[i] * 2;
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(base), ext, bytes, bx, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

cudaError_t make_scales_map(CUtensorMap* map, const void* base, int64_t row_blocks, int64_t col_blocks, int rows) {
  Encode encode;
  const cudaError_t e = find_encode(&encode);
  if (e != cudaSuccess) return e;
  const cuuint64_t ext[3] = {128, (cuuint64_t)col_blocks, (cuuint64_t)row_blocks}, bytes[2] = {512, 512 * (cuuint64_t)col_blocks};  // (in words of four bytes)
  const cuuint32_t box[3] = {128, 2, (cuuint32_t)rows}, ones[3] = {1, 1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<void*>(base), ext, bytes, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

cudaError_t make_store_map(CUtensorMap* map, void* base, bool f32, int64_t rows, int64_t cols, int64_t rstride) {
  Encode encode;
  const cudaError_t e = find_encode(&encode);
  if (e != cudaSuccess) return e;
  const cuuint64_t ext[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, bytes[1] = {(cuuint64_t)rstride * (f32 ? 4 : 2)};
  const cuuint32_t box[2] = {f32 ? 16u : 32u, 32}, ones[2] = {1, 1};
  const CUresult r = encode(map, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, ext, bytes, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace approxifer
