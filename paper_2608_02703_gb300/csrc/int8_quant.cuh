// Per-token quantisation to 8 bits on the device, shared by the quantiser and
// the product's kernels: scale = max|x| / 127, code = clamp(rint(x / scale),
// -127, 127), divisions in fp32, ties to even; code 0 where the scale is 0 or
// not finite.
#pragma once

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

// Eight neighbouring values as they are stored: loads under way.
template <typename T>
struct Raw8 {
  uint4 r[sizeof(T) / 2];
  // vec: 16-byte loads.  Values from `left` on are 0.
  __device__ __forceinline__ void load(const T *p, bool vec, int64_t left) {
    if (vec && left >= 8) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) r[i] = reinterpret_cast<const uint4 *>(p)[i];
    } else {
      alignas(16) T t[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = i < left ? p[i] : T(0.f);
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) r[i] = reinterpret_cast<const uint4 *>(t)[i];
    }
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        v[4 * i] = __uint_as_float(r[i].x), v[4 * i + 1] = __uint_as_float(r[i].y);
        v[4 * i + 2] = __uint_as_float(r[i].z), v[4 * i + 3] = __uint_as_float(r[i].w);
      }
    } else {
      const uint32_t u[4] = {r[0].x, r[0].y, r[0].z, r[0].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2 && __is_same(T, __nv_bfloat16)) {
          v[2 * i] = bf16_lo(u[i]), v[2 * i + 1] = bf16_hi(u[i]);
        } else {
          const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&u[i]));
          v[2 * i] = f.x, v[2 * i + 1] = f.y;
        }
      }
    }
  }
};

// A running maximum of |v| whose NaNs stay; its bits order as the values do, a
// NaN above infinity.
__device__ __forceinline__ float abs_max(float a, float b) {
  asm("max.NaN.xorsign.abs.f32 %0, %0, %1;\n" : "+f"(a) : "f"(b));  // (the sign is of no account)
  return a;
}
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// The largest |value| of eight as abs_bits; 16-bit types compare as integers, two at once.
template <typename T>
__device__ __forceinline__ uint32_t abs_max8(const Raw8<T> &raw) {
  if constexpr (sizeof(T) == 4) {
    float v[8];
    raw.values(v);
    float m = abs_max(abs_max(abs_max(v[0], v[1]), abs_max(v[2], v[3])), abs_max(abs_max(v[4], v[5]), abs_max(v[6], v[7])));
    return abs_bits(m);
  } else {
    constexpr uint32_t kAbs = 0x7FFF7FFFu;
    const uint32_t m = __vmaxu2(__vmaxu2(raw.r[0].x & kAbs, raw.r[0].y & kAbs), __vmaxu2(raw.r[0].z & kAbs, raw.r[0].w & kAbs));
    const uint16_t h = max((uint16_t)m, (uint16_t)(m >> 16));
    return abs_bits(to_f32(*reinterpret_cast<const T *>(&h)));
  }
}

__device__ __forceinline__ float token_scale(uint32_t max_bits) { return __fdiv_rn(__uint_as_float(max_bits), 127.f); }

// A row's quantiser: bit for bit the definition, without a division for each
// value.  With inv the correctly rounded reciprocal of the scale s, q0 = v inv
// is within one and a half units in the last place of v / s, r = v - q0 s is exact
// in an FMA, and q0 + r inv, rounded once, is v / s correctly rounded (P. Markstein,
// "Computation of elementary functions on the IBM RISC System/6000 processor", 1990;
// tried with every mantissa of s for the values at each half code up to 127.5 and
// three floats to either side: 7.5e9 quotients, all equal).  Adding 1.5 *
// 2^23 rounds it to an integer, ties to even, in the sum's low bits.  Rows whose scale
// is outside [2^-80, 2^100] (residuals may underflow, quotients may pass 127)
// are divided.
struct TokenQuantizer {
  float s, inv;
  bool fast, zero;
  __device__ __forceinline__ explicit TokenQuantizer(float scale) : s(scale) {
    zero = !(s > 0.f) || isinf(s);
    fast = s >= 8.27180613e-25f && s <= 1.26765060e30f;
    inv = fast ? __frcp_rn(s) : 0.f;
  }
  __device__ __forceinline__ int slow(float v) const {
    return zero ? 0 : (int)fminf(fmaxf(rintf(__fdiv_rn(v, s)), -127.f), 127.f);
  }
  // Two codes as the low bytes of c0 and c1.
  __device__ __forceinline__ void codes2(float v0, float v1, int &c0, int &c1) const {
    const float2 v = make_float2(v0, v1), i = make_float2(inv, inv);
    const float2 q0 = __fmul2_rn(v, i);
    const float2 r = __ffma2_rn(make_float2(-q0.x, -q0.y), make_float2(s, s), v);
    const float2 n = __fadd2_rn(__ffma2_rn(r, i, q0), make_float2(12582912.f, 12582912.f));
    c0 = __float_as_int(n.x);
    c1 = __float_as_int(n.y);
  }
  __device__ __forceinline__ void codes8(const float (&v)[8], int (&c)[8]) const {
    if (fast) {  // (the same for a whole row)
#pragma unroll
      for (int i = 0; i < 8; i += 2) codes2(v[i], v[i + 1], c[i], c[i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = slow(v[i]);
    }
  }
};

// The low bytes of four words as one.
__device__ __forceinline__ uint32_t pack_bytes(int a, int b, int c, int d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

// Codes of M rows of x into shared memory (rows `pitch` apart, zero up to
// K_pad) and their scales, by a block of kWarps warps: several warps a row
// where there are few rows.  sync: a barrier of those warps; the caller adds
// the one that the codes need.
template <typename T, int kWarps, typename Sync>
__device__ __forceinline__ void quantize_to_shared(const T *x, int64_t ldx, int M, int K, int K_pad, bool vec, int8_t *xs,
                                                   int pitch, float *s_scale, uint32_t *s_max, Sync sync) {
  constexpr int kU = sizeof(T) == 4 ? 2 : 4;  // loads a lane has under way, kept where they are the whole of its part
  const int warp = threadIdx.x >> 5, lane = lane_id();
  int per = kWarps;  // warps a row
  while (per > 1 && per * M > kWarps) per /= 2;
  const int at_once = kWarps / per, part = warp % per, k0 = 8 * (part * 32 + lane), stride = 256 * per;
  for (int m0 = 0; m0 < M; m0 += at_once) {
    const int m = m0 + warp / per;
    const T *row = x + (int64_t)m * ldx;
    Raw8<T> raw[kU];
    float v[8];
    uint32_t mx = 0;
    if (m < M) {
      for (int base = k0; base - k0 < K; base += kU * stride) {
#pragma unroll
        for (int u = 0; u < kU; ++u) raw[u].load(row + base + u * stride, vec, K - (base + u * stride));
#pragma unroll
        for (int u = 0; u < kU; ++u) mx = max(mx, abs_max8(raw[u]));
      }
      mx = __reduce_max_sync(0xffffffffu, mx);
    }
    if (per > 1) {
      if (lane == 0) s_max[warp] = mx;
      sync();
      for (int i = 0; i < per; ++i) mx = max(mx, s_max[warp - part + i]);
      sync();
    }
    if (m < M) {
      const float s = token_scale(mx);
      if (part == 0 && lane == 0) s_scale[m] = s;
      const TokenQuantizer q(s);
      const bool held = K <= kU * stride;
      for (int base = k0; base - k0 < K_pad; base += kU * stride) {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const int k = base + u * stride;
          if (!held) raw[u].load(row + k, vec, K - k);
          if (k < K_pad) {
            int c[8];
            raw[u].values(v);
            q.codes8(v, c);
            *reinterpret_cast<uint2 *>(xs + m * pitch + k) =
                make_uint2(pack_bytes(c[0], c[1], c[2], c[3]), pack_bytes(c[4], c[5], c[6], c[7]));
          }
        }
        if (held) {
          // (K_pad may pass what was held: zeros)
          for (int k = base + kU * stride; k < K_pad; k += stride) *reinterpret_cast<uint2 *>(xs + m * pitch + k) = make_uint2(0, 0);
          break;
        }
      }
    }
  }
}

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ void store_i8_out(const I8Out &o, int64_t m, int64_t n, float v) {
  const int64_t i = m * o.ld + n;
  if (o.dtype == ARCHEAD_DTYPE_FP32)
    static_cast<float *>(o.y)[i] = v;
  else if (o.dtype == ARCHEAD_DTYPE_FP16)
    static_cast<__half *>(o.y)[i] = from_f32<__half>(v);
  else
    static_cast<__nv_bfloat16 *>(o.y)[i] = from_f32<__nv_bfloat16>(v);
}

}  // namespace archead
