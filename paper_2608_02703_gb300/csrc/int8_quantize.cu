// Symmetric quantisation of activations to 8 bits, one scale per token:
// scale = max|x| / 127, code = clamp(rint(x / scale), -127, 127), divisions in
// fp32, ties to even; code 0 where the scale is 0 or not finite.
#include <cuda_fp16.h>

#include "device.cuh"
#include "int8.h"

namespace archead {

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

__device__ __forceinline__ int8_t token_code(float v, float s) {
  if (!(s > 0.f) || isinf(s)) return 0;
  return (int8_t)fminf(fmaxf(rintf(__fdiv_rn(v, s)), -127.f), 127.f);
}

// One block a row, which it reads twice (the second time from cache).
template <typename T>
__global__ void __launch_bounds__(256) int8_quantize_kernel(const T *__restrict__ x, int64_t K, int64_t ldx,
                                                            int8_t *__restrict__ codes, int64_t ldc, int64_t k_fill,
                                                            float *__restrict__ scales) {
  __shared__ uint32_t wmax[8];
  const int64_t m = blockIdx.x;
  const T *row = x + m * ldx;
  uint32_t mx = 0;  // bits of |x|: ordered as the values are, infinities and NaNs above all others
  for (int64_t k = threadIdx.x; k < K; k += 256) mx = max(mx, __float_as_uint(to_f32(row[k])) & 0x7FFFFFFFu);
  mx = __reduce_max_sync(0xffffffffu, mx);
  if ((threadIdx.x & 31) == 0) wmax[threadIdx.x >> 5] = mx;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) mx = max(mx, wmax[w]);
  const float s = __fdiv_rn(__uint_as_float(mx), 127.f);
  if (threadIdx.x == 0) scales[m] = s;
  int8_t *out = codes + m * ldc;
  for (int64_t k = threadIdx.x; k < K; k += 256) out[k] = token_code(to_f32(row[k]), s);
  for (int64_t k = K + threadIdx.x; k < k_fill; k += 256) out[k] = 0;
}

cudaError_t launch_int8_quantize(const void *x, int dtype, int64_t M, int64_t K, int64_t ldx, int8_t *codes,
                                 int64_t ldc, int64_t k_fill, float *scales, cudaStream_t s) {
  const auto run = [&](auto t) {
    using T = decltype(t);
    int8_quantize_kernel<T><<<(unsigned)M, 256, 0, s>>>(static_cast<const T *>(x), K, ldx, codes, ldc, k_fill, scales);
    return cudaGetLastError();
  };
  return dtype == ARCHEAD_DTYPE_FP32 ? run(float{}) : dtype == ARCHEAD_DTYPE_FP16 ? run(__half{}) : run(__nv_bfloat16{});
}

__global__ void int8_pad_kernel(const int8_t *__restrict__ codes, int64_t n, int K, int K_pad, int8_t *__restrict__ out) {
  for (int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
    const int64_t m = i / K_pad;
    const int k = (int)(i % K_pad);
    out[i] = k < K ? codes[m * K + k] : 0;
  }
}

cudaError_t launch_int8_pad(const int8_t *codes, int64_t M, int K, int K_pad, int8_t *out, cudaStream_t s) {
  const int64_t n = M * K_pad;
  int8_pad_kernel<<<(unsigned)(n < 256 * 4096 ? (n + 255) / 256 : 4096), 256, 0, s>>>(codes, n, K, K_pad, out);
  return cudaGetLastError();
}

}  // namespace archead
