// Tensor maps for TMA.  The driver's encoder is looked up through the runtime, so the library has no link-time dependency on libcuda (it has to load on
// machines without a driver).
#include <mutex>

#include "tc5.cuh"

namespace cdq {

cudaError_t encode_map_3d(CUtensorMap* map, const void* base, long long x, long long y, long long z, long long ldx, long long ldz, int bx, int by) {
  typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                               const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static EncodeFn encode = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess)
      encode = (EncodeFn)fn;
  });
  if (!encode) return cudaErrorNotSupported;
  const cuuint64_t dim[3] = {(cuuint64_t)x, (cuuint64_t)y, (cuuint64_t)z};
  const cuuint64_t stride[2] = {(cuuint64_t)ldx * 2, (cuuint64_t)(z > 1 ? ldz : ldx * y) * 2};
  const cuuint32_t box[3] = {(cuuint32_t)bx, (cuuint32_t)by, 1}, step[3] = {1, 1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dim, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace cdq
