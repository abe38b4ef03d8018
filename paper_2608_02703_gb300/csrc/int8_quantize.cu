// Quantisation of activations to 8 bits, one scale per token (definition and
// arithmetic: int8_quant.cuh), and the widening of given codes.
//
// Memory bound: x is read once and its codes are written.  1, 2, 4 or 8 warps
// take a row, so that each lane keeps its part, 16 or 32 values, in registers
// between the maximum and the codes; longer rows are read a second time (from
// cache).  Rows that do not start on 16 bytes (odd sizes, rows apart) go by
// neighbouring values in neighbouring lanes.  4096 rows of 2560 in fp32 take 10.6 us
// (5 TB/s, of which 2 us are the launch), of 4096 in bf16 10.6, of 2501, by values,
// 17.0 and 16.7.  (Aligned chunks joined by shuffles took 14.3 and 12.7 there, but
// lost at short rows: 5555 x 196 4.6 and 5.0 us against 3.6 and 4.0.)
#include "int8_quant.cuh"

namespace archead {

namespace {

constexpr int kThreads = 256;

// Place of column k among a row's widened codes (int8.h), in fp16 elements.
__device__ __forceinline__ int wide_place(int k) {
  const int c = k & 31;
  return (k & ~31) + 2 * (4 * ((c & 7) >> 1) + (c >> 3)) + (c & 1);
}

__device__ __forceinline__ __half widened(int c) { return __int2half_rn((int8_t)c); }

// Codes of columns 8 g .. 8 g + 7 (the low bytes of c).
template <bool kWide>
__device__ __forceinline__ void store_codes8(char *row, int g, const int (&c)[8]) {
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
__device__ __forceinline__ void store_code(char *row, int k, int c) {
  if constexpr (kWide)
    reinterpret_cast<__half *>(row)[wide_place(k)] = widened(c);
  else
    row[k] = (char)c;
}

// A lane's loads of a row: of eight values (kVec: rows of x on 16 bytes, rows of
// codes on 8, K a multiple of 8), or of two neighbours a stride of lanes apart.
template <typename T, bool kVec>
struct Part;
template <typename T>
struct Part<T, true> {
  static constexpr int kValues = 8, kLoads = 4;
  Raw8<T> raw;
  __device__ __forceinline__ void load(const T *row, int k, int K) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i)
      raw.r[i] = k < K ? __ldcs(reinterpret_cast<const uint4 *>(row + k) + i) : make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ uint32_t most() const { return abs_max8(raw); }
  template <bool kWide>
  __device__ __forceinline__ void store(const TokenQuantizer &q, char *out, int k, int) const {
    float v[8];
    int c[8];
    raw.values(v);
    q.codes8(v, c);
    store_codes8<kWide>(out, k >> 3, c);
  }
};
template <typename T>
struct Part<T, false> {
  static constexpr int kValues = 2, kLoads = 8;  // (values k and k + 32)
  T a, b;
  __device__ __forceinline__ void load(const T *row, int k, int K) {
    a = k < K ? row[k] : T(0.f);
    b = k + 32 < K ? row[k + 32] : T(0.f);
  }
  __device__ __forceinline__ uint32_t most() const { return abs_bits(abs_max(to_f32(a), to_f32(b))); }
  template <bool kWide>
  __device__ __forceinline__ void store(const TokenQuantizer &q, char *out, int k, int k_fill) const {
    int c0, c1;
    if (q.fast) q.codes2(to_f32(a), to_f32(b), c0, c1);
    else c0 = q.slow(to_f32(a)), c1 = q.slow(to_f32(b));
    store_code<kWide>(out, k, c0);
    if (k + 32 < k_fill) store_code<kWide>(out, k + 32, c1);
  }
};

// 2^per_log2 warps a row.  (K < 2^30, k_fill too.)
template <typename T, bool kWide, bool kVec>
__global__ void __launch_bounds__(kThreads, kVec && sizeof(T) == 4 ? 4 : 5)
    int8_quantize_kernel(const T *__restrict__ x, int64_t M, int K, int64_t ldx, char *__restrict__ codes,
                         int64_t pitch, int k_fill, int per_log2, float *__restrict__ scales) {
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  __shared__ uint32_t s_max[kThreads / 32];
  using P = Part<T, kVec>;
  constexpr int kU = P::kLoads;
  const int warp = threadIdx.x >> 5, lane = lane_id(), part = warp & ((1 << per_log2) - 1);
  const int64_t m = ((int64_t)blockIdx.x << (3 - per_log2)) + (warp >> per_log2);
  const bool there = m < M;
  const T *row = x + m * ldx;
  const int stride = (P::kValues * 32) << per_log2, k0 = part * P::kValues * 32 + (kVec ? P::kValues : 1) * lane;
  const bool held = k_fill <= kU * stride;  // (the same for all)
  P v[kU];
  uint32_t mx = 0;
  if (there) {
    for (int base = k0; base - k0 < K; base += kU * stride) {
#pragma unroll
      for (int u = 0; u < kU; ++u) v[u].load(row, base + u * stride, K);
#pragma unroll
      for (int u = 0; u < kU; ++u) mx = max(mx, v[u].most());
    }
  }
  mx = __reduce_max_sync(0xffffffffu, mx);
  if (per_log2 > 0) {
    if (lane == 0) s_max[warp] = mx;
    __syncthreads();
    for (int i = 0; i < 1 << per_log2; ++i) mx = max(mx, s_max[warp - part + i]);
  }
  if (!there) return;
  const float s = token_scale(mx);
  if (part == 0 && lane == 0) scales[m] = s;
  const TokenQuantizer q(s);
  char *out = codes + m * pitch;
  for (int base = k0; base - k0 < k_fill; base += kU * stride) {
    if (!held) {
#pragma unroll
      for (int u = 0; u < kU; ++u) v[u].load(row, base + u * stride, K);
    }
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (base + u * stride < k_fill) v[u].template store<kWide>(q, out, base + u * stride, k_fill);
  }
}

// Codes [M][K] into padded rows, eight a thread; 2^log2 threads a row.  A row may
// start on any byte: its codes come out of the aligned words they lie in.
template <bool kWide>
__global__ void __launch_bounds__(kThreads) int8_pad_kernel(const int8_t *__restrict__ codes, int64_t M, int K,
                                                            int K_pad, int log2, char *__restrict__ out) {
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  const int64_t m = ((int64_t)blockIdx.x << (8 - log2)) + (threadIdx.x >> log2);
  if (m >= M) return;
  const int8_t *row = codes + m * K, *end = codes + M * K;
  const int shift = 8 * (int)(reinterpret_cast<uintptr_t>(row) & 3);
  char *to = out + m * K_pad * (kWide ? 2 : 1);
  for (int k = 8 * (threadIdx.x & ((1 << log2) - 1)); k < K_pad; k += 8 << log2) {
    uint32_t lo = 0, hi = 0;
    const uint32_t *w = reinterpret_cast<const uint32_t *>(row + k - shift / 8);
    if (k + 8 <= K && reinterpret_cast<const int8_t *>(w + 2 + (shift > 0)) <= end) {
      const uint32_t w0 = w[0], w1 = w[1], w2 = shift > 0 ? w[2] : 0;
      lo = __funnelshift_r(w0, w1, shift);
      hi = __funnelshift_r(w1, w2, shift);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (k + j < K) lo |= (uint32_t)(uint8_t)row[k + j] << (8 * j);
        if (k + 4 + j < K) hi |= (uint32_t)(uint8_t)row[k + 4 + j] << (8 * j);
      }
    }
    const int c[8] = {(int)lo, (int)(lo >> 8), (int)(lo >> 16), (int)(lo >> 24),
                      (int)hi, (int)(hi >> 8), (int)(hi >> 16), (int)(hi >> 24)};
    store_codes8<kWide>(to, k >> 3, c);
  }
}

}  // namespace

cudaError_t launch_int8_quantize(const void *x, int dtype, int64_t M, int64_t K, int64_t ldx, void *codes, bool wide,
                                 int64_t ldc, int64_t k_fill, float *scales, cudaStream_t s) {
  const bool vec = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && ldx * (dtype == ARCHEAD_DTYPE_FP32 ? 4 : 2) % 16 == 0 &&
                   K % 8 == 0 && ldc * (wide ? 2 : 1) % 8 == 0;
  // Warps of a row: as many as keep it in registers, up to a block's.
  const int held = vec ? 1024 : 512;  // values of a warp
  int per_log2 = 0;
  while (per_log2 < 3 && k_fill > held << per_log2) ++per_log2;
  const int64_t pitch = ldc * (wide ? 2 : 1);
  const unsigned blocks = (unsigned)((M + (8 >> per_log2) - 1) >> (3 - per_log2));
  const auto run = [&](auto t) {
    using T = decltype(t);
    const auto launch = [&](auto kern) {
      kern<<<blocks, kThreads, 0, s>>>(static_cast<const T *>(x), M, (int)K, ldx, static_cast<char *>(codes), pitch,
                                       (int)k_fill, per_log2, scales);
      return cudaGetLastError();
    };
    if (wide) return vec ? launch(int8_quantize_kernel<T, true, true>) : launch(int8_quantize_kernel<T, true, false>);
    return vec ? launch(int8_quantize_kernel<T, false, true>) : launch(int8_quantize_kernel<T, false, false>);
  };
  return dtype == ARCHEAD_DTYPE_FP32 ? run(float{}) : dtype == ARCHEAD_DTYPE_FP16 ? run(__half{}) : run(__nv_bfloat16{});
}

cudaError_t launch_int8_pad(const int8_t *codes, int64_t M, int K, int K_pad, void *out, bool wide, cudaStream_t s) {
  int log2 = 4;  // (K_pad / 8 is 16 or more)
  while (log2 < 8 && K_pad > 8 << log2) ++log2;
  const unsigned blocks = (unsigned)((M + (kThreads >> log2) - 1) >> (8 - log2));
  if (wide)
    int8_pad_kernel<true><<<blocks, kThreads, 0, s>>>(codes, M, K, K_pad, log2, static_cast<char *>(out));
  else
    int8_pad_kernel<false><<<blocks, kThreads, 0, s>>>(codes, M, K, K_pad, log2, static_cast<char *>(out));
  return cudaGetLastError();
}

}  // namespace archead
