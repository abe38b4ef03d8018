// Root-mean-square norm with the residual's addition and an output in 8 bits.
//
//   h = round(x + r),  rstd = 1 / sqrt(mean(h^2) + eps),  y = (h rstd) w
//
// An 8-bit code is whole: one unit in the last place of rstd, which the order of a
// sum can change, would turn a code that stands next to a border.  So rstd
// is the correctly rounded value (but for one in some 2^19): the sum of squares is
// carried as two floats, and a step of Newton's method on two floats gives the root.
// (64-bit arithmetic runs at two operations a cycle here; rows whose sum leaves fp32's
// range take it.)  y and its quotients are then roundings of fp32 products.
//
// Memory bound, with a residual and fp32 (4096 x 2560, rows and codes: 26 us, 88% of the copy rate); in 16 bits,
// with twice the values a byte, as much by latency: a row's warps load, sum, store and end, and of the next row nothing is
// under way (4096 x 4096, sum, rows and codes, 28 us, 79%).  1 to 16 warps take a row and
// keep their part of it in registers, so that x and r are read once.  Rows that do not start on 16 bytes, or whose
// width is no multiple of 8, go by single values in neighbouring lanes (4096 x 4093 45 us).  Above 8192 columns the loads
// of a row, all under way at once, do not fit into the registers of 512 threads: 56 to 216 bytes a thread are spilled,
// by single values up to 528 (1024 x 16384 38 us, 1024 x 16383 104).
#include <type_traits>

#include "norm_rows.cuh"

namespace archead {

namespace {

// A sum as two floats: hi, and lo that takes what rounding hi lost (D. Knuth, The Art
// of Computer Programming 2, 4.2.2: the error of a sum is a float, and found by
// six additions).  The intrinsics are never joined to fused operations.  The two low parts are added first: so two lanes that
// add each other's sums get the same (hi's error is exact in either order), and all lanes of a row one factor.
struct Sum2 {
  float hi = 0.f, lo = 0.f;
  __device__ __forceinline__ void add(float v, float rest) {
    const float s = __fadd_rn(hi, v), b = __fsub_rn(s, hi);
    const float e = __fadd_rn(__fsub_rn(hi, __fsub_rn(s, b)), __fsub_rn(v, b));
    hi = s;
    lo = __fadd_rn(e, __fadd_rn(lo, rest));
  }
};

// Two such sums side by side: the packed operations take half as many instructions, of
// which a value has four (4096 x 4096 in bf16 37 us with single ones, 33 with these).
struct Sum2x2 {
  float2 hi = {0.f, 0.f}, lo = {0.f, 0.f};
  static __device__ __forceinline__ float2 minus(float2 a, float2 b) {  // (one rounding, as a - b)
    return __ffma2_rn(b, make_float2(-1.f, -1.f), a);
  }
  __device__ __forceinline__ void add_square(float2 v, bool exact) {
    const float2 sq = __fmul2_rn(v, v), s = __fadd2_rn(hi, sq), b = minus(s, hi);
    float2 e = __fadd2_rn(minus(hi, minus(s, b)), minus(sq, b));
    if (!exact) e = __fadd2_rn(e, __ffma2_rn(v, v, make_float2(-sq.x, -sq.y)));
    hi = s;
    lo = __fadd2_rn(lo, e);
  }
  __device__ __forceinline__ Sum2 total() const {
    Sum2 t;
    t.add(hi.x, lo.x);
    t.add(hi.y, lo.y);
    return t;
  }
};

// 1 / sqrt(total / d + eps), rounded to fp32, of a total in two floats that is at
// most 2^80 and, unless eps covers what is lost below, at least 2^-80.
constexpr float kMostSquares = 1.20892582e24f, kLeastSquares = 8.27180613e-25f;
__device__ __forceinline__ float inverse_root(Sum2 t, const NormParams &p) {
  const float q = __fmul_rn(t.hi, p.per_d_hi);
  const float rest = __fmaf_rn(t.lo, p.per_d_hi, __fmaf_rn(t.hi, p.per_d_lo, __fmaf_rn(t.hi, p.per_d_hi, -q)));
  Sum2 a;
  a.add(q, rest);
  a.add(p.eps_hi, p.eps_lo);
  const float ah = __fadd_rn(a.hi, a.lo), al = __fsub_rn(a.lo, __fsub_rn(ah, a.hi));
  const float r = rsqrtf(ah);
  if (!(r < INFINITY)) return r;  // (a of 0, or NaN)
  // e = 1 - a r^2 with r^2 and a r^2 in two floats; the root is r (1 + e / 2) to some 2^-42.
  const float rr = __fmul_rn(r, r), rre = __fmaf_rn(r, r, -rr);
  const float u = __fmul_rn(ah, rr), ue = __fmaf_rn(ah, rr, -u);
  const float e = __fsub_rn(__fsub_rn(1.f, u), __fadd_rn(ue, __fmaf_rn(ah, rre, __fmul_rn(al, rr))));
  return __fmaf_rn(r, 0.5f * e, r);
}

__device__ __forceinline__ Sum2 warp_sum(Sum2 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float hi = __shfl_xor_sync(0xffffffffu, v.hi, o), lo = __shfl_xor_sync(0xffffffffu, v.lo, o);
    v.add(hi, lo);
  }
  return v;
}

// kU chunks of 256 columns a warp: 256 kU 2^per_log2 >= d.
template <typename T, bool kVec, int kU>
__global__ void __launch_bounds__(kU == 8 ? 512 : 256, kU == 8 ? 1 : kU > 2 ? (kVec ? 3 : 2) : 3) rms_norm_kernel(const __grid_constant__ NormParams p) {
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  __shared__ float2 s_pair[kMaxWarps];
  __shared__ double s_sum[kMaxWarps];
  __shared__ uint32_t s_max[kMaxWarps];
  const int warp = threadIdx.x >> 5, lane = lane_id(), per = 1 << p.per_log2, part = warp & (per - 1);
  const int group = warp >> p.per_log2;
  const int64_t m = (int64_t)blockIdx.x * ((blockDim.x >> 5) >> p.per_log2) + group;
  if (m >= p.M) return;
  const int d = p.d;
  const auto first = [&](int u) { return (u * per + part) * 256; };
  // All loads are under way before the first value is looked at.  (With x unpacked before the residual was
  // asked for, a block of 4096 x 4096 waited twice for memory: 31 us, in this way 26.)
  float v[kU][8];
  constexpr bool kEarly = sizeof(T) == 2;  // (fp32 weights would take too many registers)
  Chunk<T, kVec> cx[kU], cr[kU], cw[kEarly ? kU : 1];
  const T *x = static_cast<const T *>(p.x) + m * p.ldx;
#pragma unroll
  for (int u = 0; u < kU; ++u) cx[u].load(x, first(u), d);
  if (p.residual) {
    const T *res = static_cast<const T *>(p.residual) + m * p.ldr;
#pragma unroll
    for (int u = 0; u < kU; ++u) cr[u].load(res, first(u), d);
  }
  if constexpr (kEarly) {
    if (!p.weight_fp32) {
#pragma unroll
      for (int u = 0; u < kU; ++u) cw[u].load(static_cast<const T *>(p.weight), first(u), d);
    }
  }
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    cx[u].values(v[u]);
    if (p.residual) {
      float r[8];
      cr[u].values(r);
#pragma unroll
      for (int j = 0; j < 8; j += 2) add_rounded<T>(v[u][j], v[u][j + 1], r[j], r[j + 1]);
    }
  }
  if (p.sum) {
    T *out = static_cast<T *>(p.sum) + m * p.lds;
#pragma unroll
    for (int u = 0; u < kU; ++u) store8<T, kVec>(out, first(u), d, v[u]);
  }
  Sum2x2 squares;
#pragma unroll
  for (int u = 0; u < kU; ++u)
#pragma unroll
    for (int j = 0; j < 8; j += 2)  // (a 16-bit value's square is exact in fp32)
      squares.add_square(make_float2(v[u][j], v[u][j + 1]), sizeof(T) == 2);
  Sum2 sum = squares.total();
  sum = warp_sum(sum);
  if (per > 1) {
    if (lane == 0) s_pair[warp] = make_float2(sum.hi, sum.lo);
    row_sync(group, per);
    sum = Sum2{};
    for (int i = 0; i < per; ++i) sum.add(s_pair[warp - part + i].x, s_pair[warp - part + i].y);
  }
  float rstd;
  if (sum.hi <= kMostSquares && (sum.hi >= kLeastSquares || p.eps_covers)) {  // (the same for a row's warps)
    rstd = inverse_root(sum, p);
  } else {  // squares that leave fp32's range, or NaN
    double t = 0.;
#pragma unroll
    for (int u = 0; u < kU; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) t += (double)v[u][j] * (double)v[u][j];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    if (per > 1) {
      if (lane == 0) s_sum[warp] = t;
      row_sync(group, per);
      t = 0.;
      for (int i = 0; i < per; ++i) t += s_sum[warp - part + i];
    }
    rstd = (float)(1. / sqrt(t / d + p.eps));
  }
  if (p.rstd && part == 0 && lane == 0) p.rstd[m] = rstd;
  uint32_t mx = 0;
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    float w[8];
    if (kEarly && !p.weight_fp32)
      cw[kEarly ? u : 0].values(w);
    else
      load8<float, kVec>(static_cast<const float *>(p.weight), first(u), d, w);
    float most = 0.f;
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const float2 y = __fmul2_rn(__fmul2_rn(make_float2(v[u][j], v[u][j + 1]), make_float2(rstd, rstd)),
                                  make_float2(w[j], w[j + 1]));
      v[u][j] = y.x;
      v[u][j + 1] = y.y;
      // (columns past the end are zeros, but not times an infinite rstd)
      if (kVec || first(u) + column<kVec>(lane, j) < d) most = abs_max(most, y.x);
      if (kVec || first(u) + column<kVec>(lane, j + 1) < d) most = abs_max(most, y.y);
    }
    if (!kVec || first(u) + 8 * lane < d) mx = max(mx, abs_bits(most));
  }
  if (p.y) {
    const auto store_rows = [&](auto t) {
      using Y = decltype(t);
      Y *out = static_cast<Y *>(p.y) + m * p.ldy;
#pragma unroll
      for (int u = 0; u < kU; ++u) store8<Y, kVec>(out, first(u), d, v[u]);
    };
    if (p.y_dtype == ARCHEAD_DTYPE_FP32) store_rows(float{});
    else if (p.y_dtype == ARCHEAD_DTYPE_FP16) store_rows(__half{});
    else store_rows(__nv_bfloat16{});
  }
  if (!p.codes) return;
  mx = __reduce_max_sync(0xffffffffu, mx);
  if (per > 1) {
    if (lane == 0) s_max[warp] = mx;
    row_sync(group, per);
    for (int i = 0; i < per; ++i) mx = max(mx, s_max[warp - part + i]);
  }
  const float s = token_scale(mx);
  if (part == 0 && lane == 0) p.scales[m] = s;
  const TokenQuantizer q(s);
  int8_t *out = p.codes + m * d;
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    int c[8];
    q.codes8(v[u], c);
    if constexpr (kVec) {
      const int k = first(u) + 8 * lane;
      if (k < d)
        *reinterpret_cast<uint2 *>(out + k) =
            make_uint2(pack_bytes(c[0], c[1], c[2], c[3]), pack_bytes(c[4], c[5], c[6], c[7]));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int k = first(u) + column<false>(lane, j);
        if (k < d) out[k] = (int8_t)c[j];
      }
    }
  }
}

}  // namespace

cudaError_t launch_rms_norm(NormParams p, int dtype, int sm_count, cudaStream_t s) {
  const int size = dtype == ARCHEAD_DTYPE_FP32 ? 4 : 2, y_size = p.y_dtype == ARCHEAD_DTYPE_FP32 ? 4 : 2;
  const bool vec = p.d % 8 == 0 && on16(p.x) && p.ldx * size % 16 == 0 && on16(p.residual) && p.ldr * size % 16 == 0 &&
                   on16(p.sum) && p.lds * size % 16 == 0 && on16(p.weight) && on16(p.y) && p.ldy * y_size % 16 == 0;
  // Much of a warp's work does not depend on how much of the row it has (sums, root, scale), so it takes up to four
  // chunks where rows are many (4096 x 4096 in bf16 26 us, with two 28), and two where they are few and a row's time
  // is what counts (1000 rows 11.3, with four 12.6), or where it loads single values.
  const Split f = split(p.d, vec && p.M > 8 * (int64_t)sm_count ? 4 : 2);
  p.per_log2 = f.per_log2;
  p.eps_hi = (float)p.eps;
  p.eps_lo = (float)(p.eps - (double)p.eps_hi);
  p.per_d_hi = (float)(1. / p.d);
  p.per_d_lo = (float)(1. / p.d - (double)p.per_d_hi);
  p.eps_covers = p.eps * p.d >= 8.67361738e-19;  // 2^-60
  const int rows = f.warps >> f.per_log2;
  const unsigned blocks = (unsigned)((p.M + rows - 1) / rows);
  const auto run = [&](auto t, auto v) {
    using T = decltype(t);
    constexpr bool kVec = decltype(v)::value;
    const auto launch = [&](auto kern) {
      kern<<<blocks, 32 * f.warps, 0, s>>>(p);
      return cudaGetLastError();
    };
    return f.chunks == 1   ? launch(rms_norm_kernel<T, kVec, 1>)
           : f.chunks == 2 ? launch(rms_norm_kernel<T, kVec, 2>)
           : f.chunks == 3 ? launch(rms_norm_kernel<T, kVec, 3>)
           : f.chunks == 4 ? launch(rms_norm_kernel<T, kVec, 4>)
                           : launch(rms_norm_kernel<T, kVec, 8>);
  };
  const auto both = [&](auto t) { return vec ? run(t, std::true_type{}) : run(t, std::false_type{}); };
  return dtype == ARCHEAD_DTYPE_FP32 ? both(float{}) : dtype == ARCHEAD_DTYPE_FP16 ? both(__half{}) : both(__nv_bfloat16{});
}

}  // namespace archead
