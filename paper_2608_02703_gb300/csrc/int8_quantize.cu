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

__device__ __forceinline__ int token_code(float v, float s) {
  if (!(s > 0.f) || isinf(s)) return 0;
  return (int)fminf(fmaxf(rintf(__fdiv_rn(v, s)), -127.f), 127.f);
}

// Eight codes c[0..7] of columns 8 g .. 8 g + 7, to their places.
template <bool kWide>
__device__ __forceinline__ void store_codes8(void *row, int64_t g, const int (&c)[8], int64_t limit) {
  if constexpr (kWide) {
    uint32_t *w = static_cast<uint32_t *>(row) + (g >> 2) * 16 + (g & 3);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __halves2half2(__int2half_rn(c[2 * i]), __int2half_rn(c[2 * i + 1]));
      w[4 * i] = *reinterpret_cast<const uint32_t *>(&h);
    }
  } else {
    int8_t *o = static_cast<int8_t *>(row) + 8 * g;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (8 * g + i < limit) o[i] = (int8_t)c[i];
  }
}

// One block a row, which it reads twice (the second time from cache).
template <typename T, bool kWide>
__global__ void __launch_bounds__(256) int8_quantize_kernel(const T *__restrict__ x, int64_t K, int64_t ldx,
                                                            void *__restrict__ codes, int64_t ldc, int64_t k_fill,
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
  char *out = static_cast<char *>(codes) + m * ldc * (kWide ? 2 : 1);
  for (int64_t g = threadIdx.x; 8 * g < k_fill; g += 256) {
    int c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = 8 * g + i < K ? token_code(to_f32(row[8 * g + i]), s) : 0;
    store_codes8<kWide>(out, g, c, k_fill);
  }
}

cudaError_t launch_int8_quantize(const void *x, int dtype, int64_t M, int64_t K, int64_t ldx, void *codes, bool wide,
                                 int64_t ldc, int64_t k_fill, float *scales, cudaStream_t s) {
  const auto run = [&](auto t) {
    using T = decltype(t);
    if (wide)
      int8_quantize_kernel<T, true><<<(unsigned)M, 256, 0, s>>>(static_cast<const T *>(x), K, ldx, codes, ldc, k_fill, scales);
    else
      int8_quantize_kernel<T, false><<<(unsigned)M, 256, 0, s>>>(static_cast<const T *>(x), K, ldx, codes, ldc, k_fill, scales);
    return cudaGetLastError();
  };
  return dtype == ARCHEAD_DTYPE_FP32 ? run(float{}) : dtype == ARCHEAD_DTYPE_FP16 ? run(__half{}) : run(__nv_bfloat16{});
}

template <bool kWide>
__global__ void int8_pad_kernel(const int8_t *__restrict__ codes, int64_t n, int K, int K_pad, char *__restrict__ out) {
  const int per = K_pad / 8;
  for (int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
    const int64_t m = i / per, g = i % per;
    int c[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) c[j] = 8 * g + j < K ? codes[m * K + 8 * g + j] : 0;
    store_codes8<kWide>(out + m * K_pad * (kWide ? 2 : 1), g, c, K_pad);
  }
}

cudaError_t launch_int8_pad(const int8_t *codes, int64_t M, int K, int K_pad, void *out, bool wide, cudaStream_t s) {
  const int64_t n = M * (K_pad / 8);
  const unsigned blocks = (unsigned)(n < 256 * 4096 ? (n + 255) / 256 : 4096);
  if (wide)
    int8_pad_kernel<true><<<blocks, 256, 0, s>>>(codes, n, K, K_pad, static_cast<char *>(out));
  else
    int8_pad_kernel<false><<<blocks, 256, 0, s>>>(codes, n, K, K_pad, static_cast<char *>(out));
  return cudaGetLastError();
}

}  // namespace archead
