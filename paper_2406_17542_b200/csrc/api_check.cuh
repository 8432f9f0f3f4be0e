// How the entry points report a CUDA call that failed.
#pragma once

#include "common.cuh"

namespace cdq {

void note_cuda_error(cudaError_t e, const char* what, const char* file, int line);   // text of cdq_last_error_detail()
bool debug_sync();

}  // namespace cdq

#define CDQ_CUDA(expr)                                  \
  do {                                                  \
    cudaError_t _e = (expr);                            \
    if (_e == cudaSuccess && cdq::debug_sync()) _e = cudaDeviceSynchronize(); \
    if (_e != cudaSuccess) {                            \
      cdq::note_cuda_error(_e, #expr, strrchr("/" __FILE__, '/') + 1, __LINE__);             \
      return CDQ_ERR_CUDA;                              \
    }                                                   \
  } while (0)
