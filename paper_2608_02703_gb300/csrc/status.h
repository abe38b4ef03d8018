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

// Waits for the stream, then reads and clears a handle's error word.  The clearing has been done when it returns:
// the next call may be on another stream, and what its kernels latch is not to be lost.
inline cudaError_t take_error_word(int *err, cudaStream_t s, int *word) {
  cudaError_t e = cudaMemcpyAsync(word, err, sizeof(int), cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaMemsetAsync(err, 0, sizeof(int), s);
  const cudaError_t end = cudaStreamSynchronize(s);  // (`word` is the caller's own: no copy stays under way)
  return e == cudaSuccess ? end : e;
}

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
