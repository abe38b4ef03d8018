// Product of 8-bit token and weight codes: exact 32-bit sums, then the token's
// and the channel's scale.
#include <cuda_fp16.h>

#include "device.cuh"
#include "int8.h"

namespace archead {

// ------------------------------------------------------------------------
// Weight layout (int8.h): one word a thread.
// ------------------------------------------------------------------------
__global__ void int8_layout_kernel(const int8_t *__restrict__ src, int64_t N, int K, int KC, int64_t words,
                                   uint32_t *__restrict__ dst) {
  for (int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; i < words; i += (int64_t)gridDim.x * blockDim.x) {
    const int j = (int)(i & 3), lane = (int)(i >> 2) & 31;
    const int block = (int)(i >> 7) & 3, strip = (int)(i >> 9) & 7;
    const int64_t st = i >> 12;
    const int64_t n = st / KC * kI8PadN + strip * kI8Strip + (lane >> 2) + 8 * (j & 1);
    const int k = (int)(st % KC) * kI8PadK + block * kI8Block + 8 * (lane & 3) + 4 * (j >> 1);
    uint32_t w = 0;
    if (n < N) {
#pragma unroll
      for (int b = 0; b < 4; ++b)
        if (k + b < K) w |= (uint32_t)(uint8_t)src[n * K + k + b] << (8 * b);
    }
    dst[i] = w;
  }
}

cudaError_t launch_int8_layout(const archead_int8_weight *w, const int8_t *codes, cudaStream_t s) {
  const int64_t words = w->N_pad * w->K_pad / 4;
  const int64_t blocks = (words + 255) / 256;
  int8_layout_kernel<<<(unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(
      codes, w->N, w->K, w->K_pad / kI8PadK, words, reinterpret_cast<uint32_t *>(w->codes));
  return cudaGetLastError();
}

// ------------------------------------------------------------------------
// Simple product: a warp takes 16 channels x 8 tokens over the whole of K.
// ------------------------------------------------------------------------
__device__ __forceinline__ void store_out(const I8Out &o, int64_t m, int64_t n, float v) {
  const int64_t i = m * o.ld + n;
  if (o.dtype == ARCHEAD_DTYPE_FP32)
    static_cast<float *>(o.y)[i] = v;
  else if (o.dtype == ARCHEAD_DTYPE_FP16)
    static_cast<__half *>(o.y)[i] = __float2half_rn(v);
  else
    static_cast<__nv_bfloat16 *>(o.y)[i] = __float2bfloat16_rn(v);
}

__global__ void __launch_bounds__(128) int8_product_kernel(const uint4 *__restrict__ codes,
                                                           const float *__restrict__ scales,
                                                           const int8_t *__restrict__ x,
                                                           const float *__restrict__ x_scales, int64_t M, int64_t N,
                                                           int K_pad, I8Out out) {
  const int lane = lane_id(), gq = lane >> 2, cq = lane & 3;
  const int64_t strip = blockIdx.x * 4 + (threadIdx.x >> 5);
  if (strip * kI8Strip >= N) return;
  const int64_t m0 = (int64_t)blockIdx.y * 8;
  const int KB = K_pad / kI8Block;
  const uint4 *a = codes + ((strip >> 3) * KB * 8 + (strip & 7) * 4) * 32 + lane;
  const int64_t mb = m0 + gq < M ? m0 + gq : M - 1;  // (columns past M are computed and not stored)
  const int8_t *b = x + mb * K_pad + 8 * cq;
  int d[4] = {0, 0, 0, 0};
  for (int kb = 0; kb < KB; ++kb) {
    const uint4 w = a[((kb >> 2) * 32 + (kb & 3)) * 32];
    const uint2 v = *reinterpret_cast<const uint2 *>(b + kb * kI8Block);
    asm volatile(
        "mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
        : "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w), "r"(v.x), "r"(v.y));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t n = strip * kI8Strip + gq + 8 * (i >> 1), m = m0 + 2 * cq + (i & 1);
    if (n < N && m < M) store_out(out, m, n, (float)d[i] * x_scales[m] * scales[n]);
  }
}

cudaError_t launch_int8_product(const archead_int8_weight *w, const int8_t *x, const float *x_scales, int64_t M,
                                I8Out out, cudaStream_t s) {
  const int64_t strips = (w->N + kI8Strip - 1) / kI8Strip;
  for (int64_t m = 0; m < M; m += 8 * 65535) {  // grid.y
    const int64_t part = M - m < 8 * 65535 ? M - m : 8 * 65535;
    I8Out o = out;
    const int e = out.dtype == ARCHEAD_DTYPE_FP32 ? 4 : 2;
    o.y = static_cast<char *>(out.y) + m * out.ld * e;
    int8_product_kernel<<<dim3((unsigned)((strips + 3) / 4), (unsigned)((part + 7) / 8)), 128, 0, s>>>(
        reinterpret_cast<const uint4 *>(w->codes), w->scales, x + m * w->K_pad, x_scales + m, part, w->N, w->K_pad, o);
  }
  return cudaGetLastError();
}

}  // namespace archead
