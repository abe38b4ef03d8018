// Selection of the next beams: of each batch entry's beams x vocabulary
// candidates, value = (score - lse) + logit, the n largest (include/archead.h).
//
// Two launches.  The first reads the logits once: a block takes a slice of a
// row and leaves the slice's (max, sum of exp) and its n best logits.  The
// second, a block for each batch entry, joins the slices' sums into the
// log-sum-exp of each beam and merges the slices' lists.
#include <cuda_fp16.h>

#include "beam.h"
#include "device.cuh"

namespace archead {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float load_logit(const float *p) { return *p; }
__device__ __forceinline__ float load_logit(const __half *p) { return __half2float(*p); }
__device__ __forceinline__ float load_logit(const __nv_bfloat16 *p) { return __bfloat162float(*p); }

// Key of (logit, token): a larger logit, or the lower token of equal ones, has
// the larger key.  (Adding 0 makes the two zeros one.)  0 is no candidate.
__device__ __forceinline__ uint64_t make_key(float l, uint32_t token) {
  const uint32_t b = __float_as_uint(l + 0.f);
  return (uint64_t)(b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) << 32 | (uint32_t)~token;
}
__device__ __forceinline__ float key_logit(uint64_t key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ uint32_t key_token(uint64_t key) { return ~(uint32_t)key; }

__device__ __forceinline__ uint64_t warp_max_key(uint64_t k) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const uint64_t other = __shfl_xor_sync(0xffffffffu, k, o);
    k = other > k ? other : k;
  }
  return k;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) beam_slice_kernel(SelectParams p) {
  __shared__ float red[kThreads / 32];
  __shared__ uint64_t kred[kThreads / 32];
  const int r = blockIdx.x / p.slices, sl = blockIdx.x % p.slices, t = threadIdx.x;
  if (p.ended && p.ended[r]) return;
  const int v0 = sl * p.slice_len, v1 = min(p.vocab, v0 + p.slice_len);
  const T *row = static_cast<const T *>(p.logits) + (int64_t)r * p.ld;
  float m = -INFINITY;
  for (int v = v0 + t; v < v1; v += kThreads) m = fmaxf(m, load_logit(row + v));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if ((t & 31) == 0) red[t >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) m = fmaxf(m, red[w]);
  __syncthreads();
  const float ref = m == -INFINITY ? 0.f : m;
  float s = 0.f;
  for (int v = v0 + t; v < v1; v += kThreads) s += expf(load_logit(row + v) - ref);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((t & 31) == 0) red[t >> 5] = s;
  __syncthreads();
  const int64_t part = (int64_t)r * p.slices + sl;
  if (t == 0) {
    s = 0.f;
    for (int w = 0; w < kThreads / 32; ++w) s += red[w];
    p.part[part] = make_float2(m, s);
  }
  // The n best, one after the other.
  uint64_t last = ~0ull;
  for (int i = 0; i < p.n; ++i) {
    uint64_t best = 0;
    for (int v = v0 + t; v < v1; v += kThreads) {
      const float l = load_logit(row + v);
      const uint64_t k = l > -INFINITY ? make_key(l, v) : 0;
      if (k < last && k > best) best = k;
    }
    best = warp_max_key(best);
    __syncthreads();
    if ((t & 31) == 0) kred[t >> 5] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) best = kred[w] > best ? kred[w] : best;
    if (t == 0) p.keys[part * p.n + i] = best;
    last = best;
  }
}

// A candidate in the order of the result: value, then beam, then its key.
struct Cand {
  float v;
  int beam;
  uint64_t key;
};
__device__ __forceinline__ bool before(const Cand &a, const Cand &b) {
  if (a.v != b.v) return a.v > b.v;
  if (a.beam != b.beam) return a.beam < b.beam;
  return a.key > b.key;
}

__global__ void __launch_bounds__(kThreads) beam_merge_kernel(SelectParams p) {
  extern __shared__ int smem[];
  int *head = smem;                                          // [beams * slices]
  float *base = reinterpret_cast<float *>(head + p.beams * p.slices);  // [beams]
  __shared__ Cand red[kThreads / 32];
  const int b = blockIdx.x, t = threadIdx.x;
  const int lists = p.beams * p.slices;
  for (int i = t; i < lists; i += kThreads) head[i] = 0;
  for (int k = t; k < p.beams; k += kThreads) {
    const int r = b * p.beams + k;
    const float score = p.scores[r];
    if (p.ended && p.ended[r]) {
      base[k] = score;
      continue;
    }
    const float2 *part = p.part + (int64_t)r * p.slices;
    float m = -INFINITY, s = 0.f;
    for (int i = 0; i < p.slices; ++i) m = fmaxf(m, part[i].x);
    const float ref = m == -INFINITY ? 0.f : m;
    for (int i = 0; i < p.slices; ++i) s += part[i].y * expf(part[i].x - ref);
    base[k] = score - (m + logf(s));
  }
  __syncthreads();
  for (int i = 0; i < p.n; ++i) {
    Cand best = {-INFINITY, p.beams, 0};
    int from = -1;
    for (int j = t; j < lists; j += kThreads) {
      const int k = j / p.slices, r = b * p.beams + k;
      Cand c = {-INFINITY, k, 0};
      if (p.ended && p.ended[r]) {
        if (j % p.slices == 0 && head[j] == 0) c.v = base[k], c.key = ~(uint64_t)(uint32_t)p.end_token;
      } else if (head[j] < p.n) {
        c.key = p.keys[((int64_t)r * p.slices + j % p.slices) * p.n + head[j]];
        if (c.key) c.v = base[k] + key_logit(c.key);
      }
      if (!isfinite(c.v)) continue;
      if (from < 0 || before(c, best)) best = c, from = j;
    }
    Cand mine = best;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      Cand other;
      other.v = __shfl_xor_sync(0xffffffffu, best.v, o);
      other.beam = __shfl_xor_sync(0xffffffffu, best.beam, o);
      other.key = __shfl_xor_sync(0xffffffffu, best.key, o);
      if (before(other, best)) best = other;
    }
    if ((t & 31) == 0) red[t >> 5] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w)
      if (before(red[w], best)) best = red[w];
    if (from >= 0 && mine.beam == best.beam && mine.key == best.key) ++head[from];
    if (t == 0) {
      const bool none = best.v == -INFINITY;
      const int64_t o = (int64_t)b * p.n + i;
      p.out_scores[o] = best.v;
      p.out_parents[o] = none ? -1 : best.beam;
      p.out_tokens[o] = none ? -1 : (int32_t)key_token(best.key);
    }
    __syncthreads();
  }
}

}  // namespace

int beam_slices(int64_t rows, int64_t vocab, int sm_count) {
  const int64_t want = (4 * sm_count + rows - 1) / rows, most = (vocab + 1023) / 1024;
  return (int)(want < most ? want : most);
}

size_t beam_scratch_bytes(int64_t max_rows, int max_out, int sm_count) {
  return (size_t)(max_rows + 4 * sm_count) * (sizeof(float2) + max_out * sizeof(uint64_t)) + 512;
}

cudaError_t launch_beam_select(SelectParams p, int dtype, int64_t batch, void *ws, int sm_count, cudaStream_t s) {
  p.slices = beam_slices(p.rows, p.vocab, sm_count);
  p.slice_len = (p.vocab + p.slices - 1) / p.slices;
  p.part = static_cast<float2 *>(ws);
  p.keys = reinterpret_cast<uint64_t *>(static_cast<char *>(ws) + ((size_t)p.rows * p.slices * sizeof(float2) + 255) / 256 * 256);
  const unsigned grid = (unsigned)p.rows * p.slices;
  if (dtype == ARCHEAD_DTYPE_FP32)
    beam_slice_kernel<float><<<grid, kThreads, 0, s>>>(p);
  else if (dtype == ARCHEAD_DTYPE_FP16)
    beam_slice_kernel<__half><<<grid, kThreads, 0, s>>>(p);
  else
    beam_slice_kernel<__nv_bfloat16><<<grid, kThreads, 0, s>>>(p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  beam_merge_kernel<<<(unsigned)batch, kThreads, (p.beams * p.slices + p.beams) * 4, s>>>(p);
  return cudaGetLastError();
}

}  // namespace archead
