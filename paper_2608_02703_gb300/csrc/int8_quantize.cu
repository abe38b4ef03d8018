// Quantisation of activations to 8 bits, one scale per token (definition and
// arithmetic: int8_quant.cuh), and the widening of given codes.
//
// Memory bound: x is read once and its codes are written.  1, 2, 4 or 8 warps
// take a row, so that each lane keeps its part, up to 32 values, in registers
// between the maximum and the codes; longer rows are read a second time (from
// cache).  Rows that do not start on 16 bytes (odd sizes, rows apart) go by
// neighbouring values in neighbouring lanes.
#include "int8_quant.cuh"

namespace archead {

namespace {

constexpr int kThreads = 256;

// Place of column k among a row's widened codes (int8.h), in fp16 elements.
__device__ __forceinline__ int64_t wide_place(int64_t k) {
  const int c = (int)(k & 31);
  return (k & ~(int64_t)31) + 2 * (4 * ((c & 7) >> 1) + (c >> 3)) + (c & 1);
}

__device__ __forceinline__ __half widened(int c) { return __int2half_rn((int8_t)c); }

// Codes of columns 8 g .. 8 g + 7 (the low bytes of c).
template <bool kWide>
__device__ __forceinline__ void store_codes8(char *row, int64_t g, const int (&c)[8]) {
  if constexpr (kWide) {
    uint32_t *w = reinterpret_cast<uint32_t *>(row) + (g >> 2) * 16 + (g & 3);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __halves2half2(widened(c[2 * i]), widened(c[2 * i + 1]));
      w[4 * i] = *reinterpret_cast<const uint32_t *>(&h);
    }
  } else {
    *reinterpret_cast<uint2 *>(row + 8 * g) =
        make_uint2(pack_bytes(c[0], c[1], c[2], c[3]), pack_bytes(c[4], c[5], c[6], c[7]));
  }
}

template <bool kWide>
__device__ __forceinline__ void store_code(char *row, int64_t k, int c) {
  if constexpr (kWide)
    reinterpret_cast<__half *>(row)[wide_place(k)] = widened(c);
  else
    row[k] = (char)c;
}

// kVec: rows of x on 16 bytes, rows of codes on 8, K a multiple of 8.
template <typename T, bool kWide, bool kVec>
__global__ void __launch_bounds__(kThreads) int8_quantize_kernel(const T *__restrict__ x, int64_t M, int64_t K,
                                                                 int64_t ldx, char *__restrict__ codes, int64_t pitch,
                                                                 int64_t k_fill, int per, float *__restrict__ scales) {
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  __shared__ uint32_t s_max[kThreads / 32];
  constexpr int kU = kVec ? 4 : 32;  // a lane's loads: of eight values, or of one
  constexpr int kStep = kVec ? 8 : 1;
  const int warp = threadIdx.x >> 5, lane = lane_id(), part = warp % per;
  const int64_t m = (int64_t)blockIdx.x * (kThreads / 32 / per) + warp / per;
  const bool there = m < M;
  const T *row = x + m * ldx;
  const int64_t k0 = kStep * (part * 32 + lane), stride = (int64_t)kStep * 32 * per;
  const bool held = k_fill <= kU * stride;  // (the same for all)
  float v[kU][kStep];
  uint32_t mx = 0;
  if (there) {
    if (held) {
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int64_t k = k0 + u * stride;
        if constexpr (kVec) {
          load8(row + k, true, K - k, v[u]);  // (K - k is 8 or more, or not above 0)
          mx = abs_max8(v[u], mx);
        } else {
          v[u][0] = k < K ? to_f32(row[k]) : 0.f;
          mx = max(mx, __float_as_uint(v[u][0]) & 0x7FFFFFFFu);
        }
      }
    } else {
      for (int64_t k = k0; k < K; k += stride) {
        if constexpr (kVec) {
          float t[8];
          load8(row + k, true, K - k, t);
          mx = abs_max8(t, mx);
        } else {
          mx = max(mx, __float_as_uint(to_f32(row[k])) & 0x7FFFFFFFu);
        }
      }
    }
  }
  mx = __reduce_max_sync(0xffffffffu, mx);
  if (per > 1) {
    if (lane == 0) s_max[warp] = mx;
    __syncthreads();
    for (int i = 0; i < per; ++i) mx = max(mx, s_max[warp - part + i]);
  }
  if (!there) return;
  const float s = token_scale(mx);
  if (part == 0 && lane == 0) scales[m] = s;
  const TokenQuantizer q(s);
  char *out = codes + m * pitch;
  const auto put = [&](int64_t k, const float(&t)[kStep]) {
    if constexpr (kVec) {
      int c[8];
      q.codes8(t, c);
      store_codes8<kWide>(out, k >> 3, c);
    } else {
      store_code<kWide>(out, k, q.code(t[0]));
    }
  };
  if (held) {
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (k0 + u * stride < k_fill) put(k0 + u * stride, v[u]);
  } else {
    for (int64_t k = k0; k < k_fill; k += stride) {
      float t[kStep];
      if constexpr (kVec) load8(row + k, true, K - k, t);
      else t[0] = k < K ? to_f32(row[k]) : 0.f;
      put(k, t);
    }
  }
}

// Codes [M][K] into padded rows.  kVec: K a multiple of 8.
template <bool kWide, bool kVec>
__global__ void __launch_bounds__(kThreads) int8_pad_kernel(const int8_t *__restrict__ codes, int64_t n, int K,
                                                            int K_pad, char *__restrict__ out) {
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  constexpr int kStep = kVec ? 8 : 1;
  const uint32_t per = K_pad / kStep;
  for (int64_t i = blockIdx.x * (int64_t)kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) {
    const int64_t m = i / per;
    const int k = (int)(i - m * per) * kStep;
    char *row = out + m * K_pad * (kWide ? 2 : 1);
    if constexpr (kVec) {
      const uint2 w = k < K ? *reinterpret_cast<const uint2 *>(codes + m * K + k) : make_uint2(0, 0);
      const int c[8] = {(int)w.x, (int)(w.x >> 8), (int)(w.x >> 16), (int)(w.x >> 24),
                        (int)w.y, (int)(w.y >> 8), (int)(w.y >> 16), (int)(w.y >> 24)};
      store_codes8<kWide>(row, k >> 3, c);
    } else {
      store_code<kWide>(row, k, k < K ? codes[m * K + k] : 0);
    }
  }
}

}  // namespace

cudaError_t launch_int8_quantize(const void *x, int dtype, int64_t M, int64_t K, int64_t ldx, void *codes, bool wide,
                                 int64_t ldc, int64_t k_fill, float *scales, cudaStream_t s) {
  // Warps of a row: as many as keep it in registers, up to a block's.
  int per = 1;
  while (per < kThreads / 32 && k_fill > 1024 * per) per *= 2;
  const int64_t pitch = ldc * (wide ? 2 : 1);
  const unsigned blocks = (unsigned)((M + kThreads / 32 / per - 1) / (kThreads / 32 / per));
  const auto run = [&](auto t) {
    using T = decltype(t);
    const auto launch = [&](auto kern) {
      kern<<<blocks, kThreads, 0, s>>>(static_cast<const T *>(x), M, K, ldx, static_cast<char *>(codes), pitch, k_fill,
                                       per, scales);
      return cudaGetLastError();
    };
    const bool vec = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && ldx * (int64_t)sizeof(T) % 16 == 0 && K % 8 == 0 &&
                     pitch % 8 == 0;
    if (wide) return vec ? launch(int8_quantize_kernel<T, true, true>) : launch(int8_quantize_kernel<T, true, false>);
    return vec ? launch(int8_quantize_kernel<T, false, true>) : launch(int8_quantize_kernel<T, false, false>);
  };
  return dtype == ARCHEAD_DTYPE_FP32 ? run(float{}) : dtype == ARCHEAD_DTYPE_FP16 ? run(__half{}) : run(__nv_bfloat16{});
}

cudaError_t launch_int8_pad(const int8_t *codes, int64_t M, int K, int K_pad, void *out, bool wide, cudaStream_t s) {
  const bool vec = K % 8 == 0;  // (codes start on 16 bytes)
  const int64_t n = M * (K_pad / (vec ? 8 : 1));
  const auto launch = [&](auto kern) {
    const int64_t blocks = (n + kThreads - 1) / kThreads;
    kern<<<(unsigned)(blocks < 65536 ? blocks : 65536), kThreads, 0, s>>>(codes, n, K, K_pad, static_cast<char *>(out));
    return cudaGetLastError();
  };
  if (wide) return vec ? launch(int8_pad_kernel<true, true>) : launch(int8_pad_kernel<true, false>);
  return vec ? launch(int8_pad_kernel<false, true>) : launch(int8_pad_kernel<false, false>);
}

}  // namespace archead
