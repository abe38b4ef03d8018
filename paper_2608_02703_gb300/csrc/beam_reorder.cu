// Reordering of the decoder's states: row b * beams + k of each state takes
// what row b * beams + parents[b][k] held before (include/archead.h).
//
// Memory bound.  A thread takes one vector (up to 16 bytes) of a row's place for
// all beams of a batch entry: it reads the vectors of the parents and then writes
// those of the rows that change, so that the exchange needs no second buffer and
// no order among blocks.  Its place costs two divisions by constants.  In place,
// rows that keep their contents are neither read (unless another beam takes them)
// nor written; a parent that several beams take comes from the first-level cache
// the second time.
//
// Moving two of each four beams of 8 batch entries' 16 states of 8 x 3001 x 128
// bf16 in place (3.1 GB) takes 449 us, the copy rate; with blocks of 256 threads 468,
// with two vectors a thread 509, with a branch around what lies past the end 490,
// with 64-bit divisions 549.
#include <algorithm>

#include "beam.h"

namespace archead {

namespace {

constexpr int kThreads = 128;

__device__ __forceinline__ uint32_t divided(uint32_t n, const Divisor &d) {
  return d.m ? __umulhi(n, d.m) >> d.shift : n;
}

template <int kMax, typename T>
__device__ __forceinline__ void move_rows(const ReorderState &st, const int *parent, int beams, bool place, int64_t row0,
                                          uint32_t n, T zero) {
  const uint32_t o = divided(n, st.per), in = n - o * st.per.d, i = divided(in, st.chunk);
  const bool there = n < st.total;
  const int64_t offset =
      row0 * st.row_stride + o * st.outer_stride + i * st.inner_stride + (int64_t)(in - i * st.chunk.d) * sizeof(T);
  const char *src = st.src + offset;
  char *dst = st.dst + offset;
  T v[kMax];
#pragma unroll
  for (int k = 0; k < kMax; ++k) {
    v[k] = zero;
    if (k < beams && there) {
      const int q = parent[k];
      if (q >= 0 && !(place && q == k)) v[k] = *reinterpret_cast<const T *>(src + q * st.row_stride);
    }
  }
#pragma unroll
  for (int k = 0; k < kMax; ++k)
    if (k < beams && there && !(place && parent[k] == k)) *reinterpret_cast<T *>(dst + k * st.row_stride) = v[k];
}

template <int kMax>
__global__ void __launch_bounds__(kThreads) beam_reorder_kernel(const __grid_constant__ ReorderParams p) {
  __shared__ int parent[kMax];
  const int tile = blockIdx.x;
  int lo = 0, hi = p.count - 1;  // the last state whose first tile is not after this one
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (p.st[mid].first_tile <= tile) lo = mid;
    else hi = mid - 1;
  }
  const ReorderState &st = p.st[lo];
  const uint32_t n = (uint32_t)(tile - st.first_tile) * kThreads + threadIdx.x;
  for (int64_t b = blockIdx.y; b < p.batch; b += gridDim.y) {
    __syncthreads();
    int q = -1;
    if (threadIdx.x < p.beams) {
      q = p.parents[b * p.beams + threadIdx.x];
      if (q < 0 || q >= p.beams) q = -1;
      parent[threadIdx.x] = q;
    }
    if (!__syncthreads_or(threadIdx.x < p.beams && !(p.place && q == (int)threadIdx.x))) continue;
    const int64_t row0 = b * p.beams;
    if (kMax <= 16 && st.width == 16)
      move_rows<kMax>(st, parent, p.beams, p.place, row0, n, make_uint4(0, 0, 0, 0));
    else if (kMax <= 32 && st.width == 8)
      move_rows<kMax>(st, parent, p.beams, p.place, row0, n, make_uint2(0, 0));
    else if (st.width == 4)
      move_rows<kMax>(st, parent, p.beams, p.place, row0, n, 0u);
    else if (st.width == 2)
      move_rows<kMax>(st, parent, p.beams, p.place, row0, n, (uint16_t)0);
    else
      move_rows<kMax>(st, parent, p.beams, p.place, row0, n, (uint8_t)0);
  }
}

}  // namespace

int reorder_vector_bytes(int beams) { return beams <= 16 ? 16 : beams <= 32 ? 8 : 4; }
int reorder_tile() { return kThreads; }

cudaError_t launch_beam_reorder(const ReorderParams &p, cudaStream_t s) {
  const dim3 grid(p.tiles, (unsigned)std::min<int64_t>(p.batch, 65535));
  const auto run = [&](auto kern) {
    kern<<<grid, kThreads, 0, s>>>(p);
    return cudaGetLastError();
  };
  return p.beams <= 4    ? run(beam_reorder_kernel<4>)
         : p.beams <= 8  ? run(beam_reorder_kernel<8>)
         : p.beams <= 16 ? run(beam_reorder_kernel<16>)
         : p.beams <= 32 ? run(beam_reorder_kernel<32>)
                         : run(beam_reorder_kernel<64>);
}

}  // namespace archead
