// What surrounds the products of the dense head's cross entropy: tokens that count
// are gathered, their partial sums joined, and dx goes back to its rows.  All three
// are bound by memory, and small beside the products but for the fewest tokens.
#include <string.h>

#include <algorithm>

#include "int8_quant.cuh"
#include "loss.h"

namespace archead {

namespace {

constexpr int kThreads = 256;

// A block's sums of two counts (all threads get them).
__device__ __forceinline__ int2 block_sum(int2 v, int2 *s) {
  v.x = __reduce_add_sync(0xffffffffu, v.x);
  v.y = __reduce_add_sync(0xffffffffu, v.y);
  if (lane_id() == 0) s[threadIdx.x >> 5] = v;
  __syncthreads();
  int2 t = make_int2(0, 0);
  for (int i = 0; i < kThreads / 32; ++i) t.x += s[i].x, t.y += s[i].y;
  __syncthreads();
  return t;
}

// Block b takes rows [b per, (b + 1) per), in turns of eight: a warp copies a row.  Every block counts all
// tokens, so that one launch does for the places, the number and the copies; the first loads of
// a row are under way meanwhile.  The rows of x behind the last token that counts are zeros up to a whole
// stage: G's rows are there, and 0 times what scratch holds may be NaN.
constexpr int kCopyLoads = 8;  // of 16 bytes, of a lane, at once

__global__ void __launch_bounds__(kThreads) ce_gather_kernel(const __grid_constant__ CeRowsParams p) {
  __shared__ int2 s_sum[kThreads / 32];
  __shared__ float s_max[kThreads / 32];
  // In this order: what is launched behind this may read the weights before it waits for it.
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = lane_id();
  const bool gradient = p.grad != nullptr;
  const auto counts = [&](int64_t m) { return p.targets[m] != p.ignore && (!gradient || p.grad[m] != 0.f); };
  const int64_t m0 = (int64_t)blockIdx.x * p.rows_per_block, m1 = min(p.M, m0 + p.rows_per_block);
  const uint16_t *x = static_cast<const uint16_t *>(p.x);
  const bool vec = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && p.ldx % 8 == 0 && p.d % 8 == 0;
  uint4 held[kCopyLoads];  // (rows on 16 bytes)
  const auto load = [&](int64_t m, int k0) {
    if (vec && m < m1) {
      const uint16_t *from = x + m * p.ldx;
#pragma unroll
      for (int i = 0; i < kCopyLoads; ++i) {
        const int k = k0 + 8 * (lane + 32 * i);
        if (k < p.d) held[i] = *reinterpret_cast<const uint4 *>(from + k);
      }
    }
  };
  // Column k of a row: panel k / 64.
  const auto place_of = [&](int64_t row, int k) { return p.at.x + ((int64_t)(k >> 6) * p.rows + row) * 64 + (k & 63); };
  const bool twice = p.half == kCeStep / 2;  // (G's two parts are one stage, and x stands behind itself)
  const auto put8 = [&](int64_t row, int k, uint4 v) {
    *reinterpret_cast<uint4 *>(place_of(row, k)) = v;
    if (twice) *reinterpret_cast<uint4 *>(place_of(row + p.half, k)) = v;
  };
  const auto clear = [&](int64_t row, int k) { put8(row, k, make_uint4(0, 0, 0, 0)); };
  if (!p.direct || gradient) load(m0 + warp, 0);
  int2 n = make_int2(0, 0);  // before m0, in all
  float most = 0.f;
#pragma unroll 4
  for (int64_t m = threadIdx.x; m < p.M; m += kThreads)
    if (counts(m)) {
      n.x += m < m0;
      ++n.y;
      if (gradient) most = fmaxf(most, fabsf(p.grad[m]));
    }
  n = block_sum(n, s_sum);
  float scale = 1.f;
  if (gradient) {
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    if (lane == 0) s_max[warp] = most;
    __syncthreads();
    for (int i = 0; i < kThreads / 32; ++i) most = fmaxf(most, s_max[i]);
    // The largest factor goes to [2^14, 2^15): G's elements, at most a factor each, fit fp16, and those of a
    // likelihood of 2^-28 are in its normal range still.  (bf16 has the range of fp32: no rounding changes.)
    if (most > 0.f && most < INFINITY) scale = exp2f((float)min(max(14 - ilogbf(most), -100), 100));
  }
  const int rows = p.direct ? (int)p.M : n.y;
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.at.header = {rows, scale, 1.f / scale};
  int at = n.x;  // tokens that count before this turn's rows
  for (int64_t base = m0; base < m1; base += kThreads / 32) {
    const int64_t m = base + warp;
    // Each warp sees which of the eight rows count.
    const int64_t other = base + lane;
    const unsigned votes = __ballot_sync(0xffffffffu, lane < kThreads / 32 && other < m1 && counts(other));
    const bool in = votes >> warp & 1;
    const int place = p.direct ? (int)m : at + __popc(votes & ((1u << warp) - 1));
    at += __popc(votes);
    if (lane == 0 && m < m1) {
      p.at.place[m] = in ? place : -1;
      if (in || p.direct) {
        const int64_t t = in ? p.targets[m] : -1;
        p.at.target[place] = t >= 0 && t < p.V ? (int)t : -1;
        if (gradient) p.at.lse[place] = in ? p.lse[m] : 0.f, p.at.factor[place] = in ? p.grad[m] * scale : 0.f;
      }
    }
    if (p.direct && !gradient) continue;  // (nobody reads a copy)
    if (p.direct && m < m1 && !in) {
      for (int k = 8 * lane; k < p.x_pitch; k += 256) clear(m, k);
    } else if (m < m1 && in) {
      const auto put = [&](int k, uint16_t v) {
        *place_of(place, k) = v;
        if (twice) *place_of(place + p.half, k) = v;
      };
      if (vec) {
        for (int k0 = 0; k0 < p.d; k0 += 256 * kCopyLoads) {
          if (k0 > 0) load(m, k0);
#pragma unroll
          for (int i = 0; i < kCopyLoads; ++i) {
            const int k = k0 + 8 * (lane + 32 * i);
            if (k < p.d) put8(place, k, held[i]);
          }
        }
      } else {
        const uint16_t *from = x + m * p.ldx;
        for (int k = lane; k < p.d; k += 8 * 32) {
          uint16_t v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (k + 32 * i < p.d) v[i] = from[k + 32 * i];
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (k + 32 * i < p.d) put(k + 32 * i, v[i]);
        }
      }
      for (int k = p.d + lane; k < p.x_pitch; k += 32) put(k, 0);
    }
    load(m + kThreads / 32, 0);
  }
  if (blockIdx.x == gridDim.x - 1) {
    const int end = twice ? p.half : (rows + kCeStep - 1) / kCeStep * kCeStep;
    for (int r = rows + warp; r < end; r += kThreads / 32)
      for (int k = 8 * lane; k < p.x_pitch; k += 256) clear(r, k);
  }
}

// A block takes eight tokens, 64 of its threads one of them: every 64th partial sum each, joined in
// that order.
constexpr int kFinishTokens = 8, kFinishLanes = 64;

// Sums s e^m of two sets.
__device__ __forceinline__ LsePair joined(LsePair a, LsePair b) {
  if (a.m == -INFINITY) return {b.m, a.s + b.s};  // (s is 0, or NaN)
  if (b.m == -INFINITY) return {a.m, a.s + b.s};
  const float m = fmaxf(a.m, b.m);
  if (m == INFINITY) return {m, a.s + b.s};  // (s is infinite there)
  return {m, a.s * expf(a.m - m) + b.s * expf(b.m - m)};
}

__global__ void __launch_bounds__(kFinishTokens *kFinishLanes) ce_finish_kernel(const CeFinishParams p) {
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  __shared__ float2 s_part[kFinishLanes / 4][kFinishTokens];
  const int token = threadIdx.x % kFinishTokens, part = threadIdx.x / kFinishTokens;
  const int64_t m = (int64_t)blockIdx.x * kFinishTokens + token;
  const int place = m < p.M ? p.at.place[m] : -1;
  const int parts = p.at.header->count <= kCeTile ? p.parts.by_pair : p.parts.by_tile;
  const int target = place >= 0 ? p.at.target[place] : -1;
  const float tlogit = target >= 0 ? p.at.tlogit[place] : 0.f;
  LsePair t{-INFINITY, 0.f};
  if (place >= 0)
    for (int i = part; i < parts; i += 4 * kFinishLanes) {
      float2 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = i + j * kFinishLanes;
        v[j] = at < parts ? p.at.part[at * p.rows + place] : make_float2(-INFINITY, 0.f);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) t = joined(t, {v[j].x, v[j].y});
    }
  // A warp's four threads of a token, then its warps.
#pragma unroll
  for (int o = kFinishTokens; o < 32; o *= 2) {
    const float m2 = __shfl_xor_sync(0xffffffffu, t.m, o), s2 = __shfl_xor_sync(0xffffffffu, t.s, o);
    t = joined(t, {m2, s2});
  }
  if (lane_id() < kFinishTokens) s_part[threadIdx.x >> 5][token] = make_float2(t.m, t.s);
  __syncthreads();
  if (part > 0 || m >= p.M) return;
  float ce = 0.f, lse = 0.f;
  if (place >= 0) {
    for (int i = 1; i < kFinishLanes / 4; ++i) t = joined(t, {s_part[i][token].x, s_part[i][token].y});
    if (target < 0) {
      atomicOr(p.err, kErrTargetRange);
      ce = lse = NAN;
    } else {
      const float log_s = logf(t.s);
      lse = t.m + log_s;
      ce = (t.m - tlogit) + log_s;
    }
  }
  p.ce[m] = ce;
  if (p.lse) p.lse[m] = lse;
}

// dx's rows: the sum of the splits, in order (and of G's second part, in rows of its own), without the
// factors' scale, and, of a G in one part, what its rounding took at the target; zeros for tokens that do not
// count.  A thread takes four columns.
template <typename T>
__global__ void __launch_bounds__(kThreads) ce_dx_kernel(const CeDxParams p) {
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  const int64_t m = blockIdx.x;
  const int place = p.at.place[m], k = 4 * (blockIdx.y * kThreads + threadIdx.x);
  if (k >= p.d) return;
  const float unscale = p.at.header->unscale;
  float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
  if (place >= 0) {
    const float *from = p.at.dx + (int64_t)place * p.pitch + k;  // (columns past d are there, to a whole tile)
    const int64_t step = p.rows * p.pitch, half = (int64_t)p.half * p.pitch;
    const int parts = p.half > 0 ? 2 * p.splits : p.splits;
    for (int i = 0; i < parts; i += 8) {
      float4 v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int at = i + j;
        v[j] = at < parts ? *reinterpret_cast<const float4 *>(from + (p.half > 0 ? (at >> 1) * step + (at & 1) * half : at * step))
                          : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) t.x += v[j].x, t.y += v[j].y, t.z += v[j].z, t.w += v[j].w;
    }
  }
  const int target = place >= 0 && p.half == 0 ? p.at.target[place] : -1;
  if (target >= 0) {
    const float rest = p.at.rest[place];
    const T *w = static_cast<const T *>(p.w) + target * p.ldw + k;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    if (k + 4 <= p.d) {  // (w's rows start on 16 bytes)
      const uint2 raw = *reinterpret_cast<const uint2 *>(w);
      T h[4];
      memcpy(h, &raw, 8);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = to_f32(h[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (k + i < p.d) x[i] = to_f32(w[i]);
    }
    t.x += rest * x[0], t.y += rest * x[1], t.z += rest * x[2], t.w += rest * x[3];
  }
  T *out = static_cast<T *>(p.dx) + m * p.ld + k;
  const float x[4] = {t.x * unscale, t.y * unscale, t.z * unscale, t.w * unscale};
  if (p.vec && k + 4 <= p.d) {
    const T h[4] = {from_f32<T>(x[0]), from_f32<T>(x[1]), from_f32<T>(x[2]), from_f32<T>(x[3])};
    uint2 w;
    memcpy(&w, h, 8);
    *reinterpret_cast<uint2 *>(out) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (k + i < p.d) out[i] = from_f32<T>(x[i]);
  }
}

template <typename P>
cudaError_t launch(void (*kern)(const P), const P &p, dim3 grid, int threads, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, p);
}

}  // namespace

cudaError_t launch_ce_gather(const CeRowsParams &p0, cudaStream_t s) {
  CeRowsParams p = p0;
  p.rows_per_block = (int)std::max<int64_t>(8, (p.M + 1023) / 1024);
  return launch(ce_gather_kernel, p, dim3((unsigned)((p.M + p.rows_per_block - 1) / p.rows_per_block)), kThreads, s);
}

cudaError_t launch_ce_finish(const CeFinishParams &p, cudaStream_t s) {
  return launch(ce_finish_kernel, p, dim3((unsigned)((p.M + kFinishTokens - 1) / kFinishTokens)),
                kFinishTokens * kFinishLanes, s);
}

cudaError_t launch_ce_dx(const CeDxParams &p0, cudaStream_t s) {
  CeDxParams p = p0;
  p.vec = (reinterpret_cast<uintptr_t>(p.dx) & 7) == 0 && p.ld % 4 == 0;
  const dim3 grid((unsigned)p.M, (unsigned)((p.d + 4 * kThreads - 1) / (4 * kThreads)));
  return p.fp16 ? launch(ce_dx_kernel<__half>, p, grid, kThreads, s)
                : launch(ce_dx_kernel<__nv_bfloat16>, p, grid, kThreads, s);
}

}  // namespace archead
