// Gradient of the root-mean-square norm, n = h rstd, g = dy w:
//
//   dx = rstd (g - n mean(g n)) + dsum,   dw[k] = sum over the rows of dy n
//
// A block takes rows in turn; its threads keep their columns' sums of dy n, the
// weight's gradient, which leave as one part a block and are joined by a second launch.  A thread copies what it will
// need of the next rows into shared memory (cp.async), each of the `stages` - 1 rows ahead
// in a group of its own: no thread reads another's, so that nothing but the sum over
// the row is waited for.  (Without rows ahead a block waited twice a row for memory:
// 4096 x 4096 in bf16 took 51 us, now 28 and 4 for the weight's.)  Rows that do not start on 16 bytes are loaded
// together, by single values, into registers; of the widest, of which two do not fit into shared memory,
// everything is loaded where it is used, the second time from cache.
//
// Bound by what a multiprocessor does beside memory (unpacking, twice, and sums over the row: 62% of the copy rate, in
// fp32 55%: 4096 x 4096 71 us); a third block of eight warps gained 10%, more rows ahead nothing.  By single values a
// row of more than 4096 columns does not fit into the registers (160 to 480 bytes a thread are spilled): 2048 x 8191 in
// bf16 takes 73 us, where 4096 x 4093 takes 45.
#include <algorithm>
#include <type_traits>

#include "internal.h"
#include "norm_rows.cuh"

namespace archead {

namespace {

// Blocks of a multiprocessor that the gradient's registers allow.
constexpr int grad_blocks(int chunks, bool vec) { return chunks == 8 ? 1 : chunks > 2 || !vec ? 2 : 3; }

template <typename T>
struct GradRing {
  static constexpr int kPieces = (int)sizeof(T) / 2;  // of 16 bytes, of eight values
  uint32_t at;  // this thread's first piece
  int threads, chunks, row;  // row: bytes of a stage
  __device__ __forceinline__ uint32_t place(int stage, int tensor, int u) const {
    return at + stage * row + ((tensor * chunks + u) * kPieces * threads) * 16;
  }
  __device__ __forceinline__ void copy(int stage, int tensor, int u, const T *from, int k0, int d) const {
    const int k = k0 + 8 * lane_id();
    const uint32_t to = place(stage, tensor, u);
    const int bytes = k < d ? 16 : 0;  // (the rest is filled with zeros)
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(to + i * threads * 16),
                   "l"(from + (k < d ? k + 8 / kPieces * i : 0)), "r"(bytes)
                   : "memory");
  }
  __device__ __forceinline__ void values(int stage, int tensor, int u, float (&v)[8]) const {
    Raw8<T> raw;
    const uint32_t from = place(stage, tensor, u);
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n"
                   : "=r"(raw.r[i].x), "=r"(raw.r[i].y), "=r"(raw.r[i].z), "=r"(raw.r[i].w)
                   : "r"(from + i * threads * 16)
                   : "memory");
    raw.values(v);
  }
};

template <typename T, bool kVec, int kU>
__global__ void __launch_bounds__(kU == 8 ? 512 : 256, grad_blocks(kU, kVec)) rms_norm_grad_kernel(const __grid_constant__ NormGradParams p) {
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  __shared__ float s_sum[2][kMaxWarps];
  extern __shared__ uint4 s_dyn[];  // the ring, then [groups][d] parts where several groups of warps take rows
  const int warp = threadIdx.x >> 5, lane = lane_id(), per = 1 << p.per_log2, part = warp & (per - 1);
  const int groups = (blockDim.x >> 5) >> p.per_log2, group = warp >> p.per_log2;
  const int d = p.d, stages = kVec ? p.stages : 0;
  const auto first = [&](int u) { return (u * per + part) * 256; };
  float acc[kU][8];
#pragma unroll
  for (int u = 0; u < kU; ++u)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[u][j] = 0.f;
  const int64_t step = (int64_t)gridDim.x * groups;
  const int64_t m0 = (int64_t)blockIdx.x * groups + group;
  const int tensors = p.dsum ? 3 : 2;
  GradRing<T> ring;
  ring.threads = blockDim.x;
  ring.chunks = kU;
  ring.row = tensors * kU * GradRing<T>::kPieces * (int)blockDim.x * 16;
  ring.at = smem_u32(s_dyn) + threadIdx.x * 16;
  // (A group of copies for every row, empty past the last one.)
  const auto fetch_row = [&](int64_t m, int stage) {
    if (m < p.M) {
      const T *g = static_cast<const T *>(p.dy) + m * p.ldg, *h = static_cast<const T *>(p.h) + m * p.ldh;
#pragma unroll
      for (int u = 0; u < kU; ++u) ring.copy(stage, 0, u, g, first(u), d);
#pragma unroll
      for (int u = 0; u < kU; ++u) ring.copy(stage, 1, u, h, first(u), d);
      if (p.dsum) {
        const T *r = static_cast<const T *>(p.dsum) + m * p.lds;
#pragma unroll
        for (int u = 0; u < kU; ++u) ring.copy(stage, 2, u, r, first(u), d);
      }
    }
    asm volatile("cp.async.commit_group;\n" ::: "memory");
  };
  for (int i = 0; i + 1 < stages; ++i) fetch_row(m0 + i * step, i);
  float4 *weights = reinterpret_cast<float4 *>(reinterpret_cast<char *>(s_dyn) + stages * ring.row) + lane;
  if (kVec && p.weights) {  // (of a lane's eight the first four, of all lanes, then the others)
    if (group == 0)
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        float w[8];
        load_weight8<T, kVec>(p.weight, p.weight_fp32, first(u), d, w);
        weights[first(u) / 4] = make_float4(w[0], w[1], w[2], w[3]);
        weights[first(u) / 4 + 32] = make_float4(w[4], w[5], w[6], w[7]);
      }
    if (groups > 1) __syncthreads();  // (otherwise each thread has written what it reads)
  }
  const auto weight = [&](int u, float (&w)[8]) {
    if (kVec && p.weights) {
      const float4 a = weights[first(u) / 4], b = weights[first(u) / 4 + 32];
      w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
    } else {
      load_weight8<T, kVec>(p.weight, p.weight_fp32, first(u), d, w);
    }
  };
  float rstd_next = m0 < p.M ? p.rstd[m0] : 0.f;
  int stage = 0, turn = 0;
  for (int64_t m = m0; m < p.M; m += step, turn ^= 1) {  // (the same for a row's warps)
    const float rstd = rstd_next;
    if (m + step < p.M) rstd_next = p.rstd[m + step];
    if (stages > 0) {
      fetch_row(m + (stages - 1) * step, stage == 0 ? stages - 1 : stage - 1);
      switch (stages) {  // the oldest of the groups under way
        case 2: asm volatile("cp.async.wait_group 1;\n" ::: "memory"); break;
        case 3: asm volatile("cp.async.wait_group 2;\n" ::: "memory"); break;
        case 4: asm volatile("cp.async.wait_group 3;\n" ::: "memory"); break;
        default: asm volatile("cp.async.wait_group 5;\n" ::: "memory"); break;  // (6)
      }
    }
    const T *dy = static_cast<const T *>(p.dy) + m * p.ldg, *h = static_cast<const T *>(p.h) + m * p.ldh;
    // (Single values: a row's loads are under way together, and stay in registers.)
    constexpr bool kHeld = !kVec && kU <= 4;
    Chunk<T, kVec> held[3][kHeld ? kU : 1];
    if constexpr (kHeld) {
#pragma unroll
      for (int u = 0; u < kU; ++u) held[0][u].load(dy, first(u), d);
#pragma unroll
      for (int u = 0; u < kU; ++u) held[1][u].load(h, first(u), d);
      if (p.dsum) {
        const T *r = static_cast<const T *>(p.dsum) + m * p.lds;
#pragma unroll
        for (int u = 0; u < kU; ++u) held[2][u].load(r, first(u), d);
      }
    }
    const auto values = [&](int u, float (&g)[8], float (&n)[8]) {  // dy and h
      if constexpr (kHeld) {
        held[0][u].values(g);
        held[1][u].values(n);
      } else if (stages > 0) {
        ring.values(stage, 0, u, g);
        ring.values(stage, 1, u, n);
      } else {
        load8<T, kVec>(dy, first(u), d, g);
        load8<T, kVec>(h, first(u), d, n);
      }
    };
    float2 dots = {0.f, 0.f};
    const float2 r2 = make_float2(rstd, rstd);
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      float g[8], n[8], w[8];
      weight(u, w);
      values(u, g, n);
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        const float2 dy2 = make_float2(g[j], g[j + 1]), n2 = __fmul2_rn(make_float2(n[j], n[j + 1]), r2);
        const float2 a = __ffma2_rn(dy2, n2, make_float2(acc[u][j], acc[u][j + 1]));
        acc[u][j] = a.x;
        acc[u][j + 1] = a.y;
        dots = __ffma2_rn(__fmul2_rn(dy2, make_float2(w[j], w[j + 1])), n2, dots);
      }
    }
    float dot = dots.x + dots.y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
    if (per > 1) {
      if (lane == 0) s_sum[turn][warp] = dot;
      row_sync(group, per);
      dot = 0.f;
      for (int i = 0; i < per; ++i) dot += s_sum[turn][warp - part + i];
    }
    const float minus = -dot / (float)d;
    T *dx = static_cast<T *>(p.dx) + m * p.ldx;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      float g[8], n[8], w[8], add[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, out[8];
      weight(u, w);
      values(u, g, n);
      if (p.dsum) {
        if constexpr (kHeld)
          held[2][u].values(add);
        else if (stages > 0)
          ring.values(stage, 2, u, add);
        else
          load8<T, kVec>(static_cast<const T *>(p.dsum) + m * p.lds, first(u), d, add);
      }
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        const float2 n2 = __fmul2_rn(make_float2(n[j], n[j + 1]), r2);
        const float2 g2 = __fmul2_rn(make_float2(g[j], g[j + 1]), make_float2(w[j], w[j + 1]));
        const float2 t = __ffma2_rn(r2, __ffma2_rn(n2, make_float2(minus, minus), g2), make_float2(add[j], add[j + 1]));
        out[j] = t.x;
        out[j + 1] = t.y;
      }
      store8<T, kVec>(dx, first(u), d, out);
    }
    if (stages > 0 && ++stage == stages) stage = 0;
  }
  if (!p.dweight) return;
  float *to = p.parts + (int64_t)blockIdx.x * d;
  if (groups > 1) {
    __syncthreads();  // (the parts take the ring's place; its copies have landed or were empty)
    float *s_part = reinterpret_cast<float *>(s_dyn);
#pragma unroll
    for (int u = 0; u < kU; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int k = first(u) + column<kVec>(lane, j);
        if (k < d) s_part[group * d + k] = acc[u][j];
      }
    __syncthreads();
    for (int k = threadIdx.x; k < d; k += blockDim.x) {
      float t = s_part[k];
      for (int i = 1; i < groups; ++i) t += s_part[i * d + k];
      to[k] = t;
    }
  } else {
#pragma unroll
    for (int u = 0; u < kU; ++u) store8<float, kVec>(to, first(u), d, acc[u]);
  }
}

// dweight[k] = sum of the parts (+ dweight[k]): a block takes 32 columns, each of its warps every
// 16th part.
constexpr int kPartWarps = 16;

__global__ void __launch_bounds__(32 * kPartWarps)
    norm_weight_kernel(const float *__restrict__ parts, int count, int d, int accumulate, float *__restrict__ dweight) {
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  __shared__ float s[kPartWarps][32];
  const int k = blockIdx.x * 32 + lane_id(), warp = threadIdx.x >> 5;
  float t = 0.f;
  if (k < d)
    for (int i = warp; i < count; i += 8 * kPartWarps) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int at = i + j * kPartWarps;
        v[j] = at < count ? parts[(int64_t)at * d + k] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) t += v[j];
    }
  s[warp][lane_id()] = t;
  __syncthreads();
  if (warp > 0 || k >= d) return;
#pragma unroll
  for (int i = 1; i < kPartWarps; ++i) t += s[i][lane_id()];
  dweight[k] = accumulate ? dweight[k] + t : t;
}

// Shared memory of a multiprocessor, and what of it a block takes beside its ring and weights.
constexpr int kSmemOfSm = 228 * 1024, kSmemOfBlock = 1024 + 256;

}  // namespace

cudaError_t launch_rms_norm_backward(NormGradParams p, int dtype, int sm_count, cudaStream_t s) {
  const int size = dtype == ARCHEAD_DTYPE_FP32 ? 4 : 2;
  const bool vec = p.d % 8 == 0 && on16(p.dy) && p.ldg * size % 16 == 0 && on16(p.h) && p.ldh * size % 16 == 0 &&
                   on16(p.dsum) && p.lds * size % 16 == 0 && on16(p.dx) && p.ldx * size % 16 == 0 && on16(p.weight);
  const Split f = split(p.d, 2);  // (4096 x 4096 in bf16 31.4 us; four chunks a warp in two blocks of a multiprocessor 32.9, one block of them 39)
  p.per_log2 = f.per_log2;
  const int groups = f.warps >> f.per_log2;
  // As many blocks of a multiprocessor as its registers and rings of two rows allow, with the weights
  // beside them or, for one block that has no room for them, without.
  const int row = (p.dsum ? 3 : 2) * f.chunks * 32 * f.warps * 8 * size, weights = (f.chunks << f.per_log2) * 1024;
  int per_sm = grad_blocks(f.chunks, vec) + 1;
  p.stages = 0;
  p.weights = vec;
  while (vec && per_sm > 1 && p.stages < 2) p.stages = (kSmemOfSm / --per_sm - kSmemOfBlock - weights) / row;
  if (p.stages < 2) p.weights = 0, p.stages = vec ? (kSmemOfSm - kSmemOfBlock) / row : 0;
  if (p.stages < 2) p.stages = 0, per_sm = grad_blocks(f.chunks, vec);
  p.stages = p.stages < 4 ? p.stages : p.stages < 6 ? 4 : 6;
  p.blocks = (int)std::min<int64_t>((p.M + groups - 1) / groups, std::min(per_sm * sm_count, kNormParts));
  const int parts = groups > 1 ? groups * p.d * (int)sizeof(float) : 0;  // (32 KB at most: see split)
  const size_t smem = std::max(p.stages * row + (p.weights ? weights : 0), parts);
  const auto run = [&](auto t, auto v) {
    using T = decltype(t);
    constexpr bool kVec = decltype(v)::value;
    const auto launch = [&](auto kern) {
      cudaError_t e = smem > 40000 ? opt_in_smem(reinterpret_cast<const void *>(kern), kSmemOfSm - kSmemOfBlock) : cudaSuccess;
      if (e != cudaSuccess) return e;
      kern<<<(unsigned)p.blocks, 32 * f.warps, smem, s>>>(p);
      return cudaGetLastError();
    };
    return f.chunks == 1   ? launch(rms_norm_grad_kernel<T, kVec, 1>)
           : f.chunks == 2 ? launch(rms_norm_grad_kernel<T, kVec, 2>)
           : f.chunks == 3 ? launch(rms_norm_grad_kernel<T, kVec, 3>)
           : f.chunks == 4 ? launch(rms_norm_grad_kernel<T, kVec, 4>)
                           : launch(rms_norm_grad_kernel<T, kVec, 8>);
  };
  const auto both = [&](auto t) { return vec ? run(t, std::true_type{}) : run(t, std::false_type{}); };
  const cudaError_t e = dtype == ARCHEAD_DTYPE_FP32   ? both(float{})
                        : dtype == ARCHEAD_DTYPE_FP16 ? both(__half{})
                                                      : both(__nv_bfloat16{});
  if (e != cudaSuccess || !p.dweight) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((p.d + 31) / 32));
  cfg.blockDim = dim3(32 * kPartWarps);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, norm_weight_kernel, (const float *)p.parts, p.blocks, p.d, p.accumulate, p.dweight);
}

}  // namespace archead
