// Status of a failed CUDA call at a C entry, its message kept for archead_last_error().
#pragma once

#include <cuda_runtime.h>

#include "archead.h"

namespace archead {

void set_last_error_message(const char *msg);

inline archead_status status_of(cudaError_t e) {
  if (e == cudaSuccess) return ARCHEAD_OK;
  set_last_error_message(cudaGetErrorString(e));
  cudaGetLastError();  // (a later call's launch would be taken to have failed)
  return e == cudaErrorMemoryAllocation ? ARCHEAD_ERR_OOM : ARCHEAD_ERR_CUDA;
}

#define AH_TRY(call)                                                     \
  do {                                                                   \
    cudaError_t e_ = (call);                                             \
    if (e_ != cudaSuccess) return ::archead::status_of(e_);              \
  } while (0)

inline bool is_aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline bool is_dtype(int d) { return d == ARCHEAD_DTYPE_BF16 || d == ARCHEAD_DTYPE_FP32 || d == ARCHEAD_DTYPE_FP16; }
inline int dtype_bytes(int d) { return d == ARCHEAD_DTYPE_FP32 ? 4 : 2; }

// A stream being captured into a graph (or one that must not be asked).
inline bool is_capturing(cudaStream_t s) {
  cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(s, &st) == cudaSuccess) return st != cudaStreamCaptureStatusNone;
  cudaGetLastError();
  return true;
}

}  // namespace archead
