// Warp-level kernel of the INT8 product (few tokens), and the weight's layout.
//
// Memory bound: N K bytes of codes are streamed once.  A producer warp keeps a
// ring of 16 KB slots filled by bulk copies; 16 consumer warps read them as the
// A fragments of mma.sync m16n8k32 (s8, exact 32-bit sums; this chip's rate of
// it, 75 T multiply-adds a second, is 1.4 times what 8 tokens need at the rate
// of the memory).  The tokens' codes lie in shared memory; where they are few
// every block quantises them itself, which saves a launch.
//
// A slot holds eight segments of 2 KB (a strip of 16 channels x 128 of K), one
// a warp; even and odd slots go to the two halves of the warps.  The segments
// are kw neighbouring K stages of 8 / kw strips: with too few strips for all
// multiprocessors a block takes fewer of them and runs along K faster.  The
// warps of a strip join their sums through shared memory.
//
// 8 tokens of 151936 x 4096 take 95 us, 97% of the copy rate (1 token 92).
//
// (Loading fragments from global memory straight into registers, four to eight
// 512-byte loads ahead in 16 or 32 warps, stalled on them: 140 us.)
#include "int8_quant.cuh"

#include <algorithm>

#include "internal.h"
#include "status.h"

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
// The product
// ------------------------------------------------------------------------
namespace {

constexpr int kWarps = 16;                     // consumers
constexpr int kThreads = 32 * (kWarps + 1);
constexpr int kSegment = kI8Strip * kI8PadK;   // bytes
constexpr int kSlot = 8 * kSegment;
constexpr int kMostSlots = 12;

struct I8DecodeParams {
  const uint8_t *codes;
  const float *scales;
  const void *x;  // activations [M] rows ldx apart (quantised here), or codes int8
  int64_t ldx;
  const float *x_scales;  // of codes
  I8Out out;
  int64_t N;
  int M, K, K_pad, KC;
  int tiles;       // of 128 channels
  // Rounds: the first ones and the last ones (see launch_int8_decode), each with
  // its K stages a slot, slots a round and first strip.
  int first_rounds, rounds;
  int kw[2], steps[2];
  int64_t last_strip;
  int slots;       // of the ring: even, so that a slot always goes to the same warps
  bool vec;        // x: 16-byte loads
  int *err;
  int64_t wait_budget;
  int64_t drain_budget;  // of the waits for what is in flight when a block ends: no less than the default
};

// This block's round r.
struct Round {
  int kw, steps, strips;
  int64_t strip;  // its first
  __device__ __forceinline__ Round(const I8DecodeParams &p, int r) {
    const bool last = r >= p.first_rounds;
    kw = last ? p.kw[1] : p.kw[0];
    steps = last ? p.steps[1] : p.steps[0];
    strips = 8 / kw;
    strip = (last ? p.last_strip : 0) + ((int64_t)(last ? r - p.first_rounds : r) * gridDim.x + blockIdx.x) * strips;
  }
};

// Where the tokens' codes come from.
enum I8Source {
  kFromActivations,  // quantised into shared memory by every block
  kFromCodes,        // copied into shared memory
  kFromGlobal        // read in place (padded rows): more of them than shared memory holds
};

__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, 512;\n" ::: "memory"); }

// Lets the bulk copies issued so far land before the producer ends: a consumer whose
// wait gives up may let the block end before they have.
__device__ __forceinline__ void drain_ring(uint64_t *full, int slots, int issued, int64_t budget, int *err) {
  for (int k = issued > slots ? issued - slots : 0; k < issued; ++k)
    mbar_wait_warp(&full[k % slots], (uint32_t)(k / slots) & 1, budget, nullptr, err);
}

template <int kTiles, I8Source kSource, typename T>
__global__ void __launch_bounds__(kThreads, 1) int8_decode_kernel(const I8DecodeParams p) {
  extern __shared__ uint4 smem16[];
  __shared__ float s_scale[8 * kTiles];
  __shared__ uint32_t s_max[kWarps];
  __shared__ uint64_t full[kMostSlots], empty[kMostSlots];
  __shared__ int abort_flag;
  uint8_t *ring = reinterpret_cast<uint8_t *>(smem16);
  int *sums = reinterpret_cast<int *>(ring + p.slots * kSlot);  // [2][kWarps][128 kTiles]
  int8_t *xs = reinterpret_cast<int8_t *>(sums + 2 * kWarps * 128 * kTiles);
  const int warp = threadIdx.x >> 5, lane = lane_id();
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.slots; ++i) mbar_init(&full[i], 1), mbar_init(&empty[i], 8);
    abort_flag = 0;
    fence_mbar_init();
  }
  __syncthreads();

  if (warp == kWarps) {
    // ------------------------------ producer ------------------------------
    const bool leader = elect_one();
    int slot = 0, issued = 0;
    uint32_t ph = 0;
    for (int r = 0; r < p.rounds; ++r) {
      const Round now(p, r);
      const int strips = now.strips, kw = now.kw;
      const int64_t s = now.strip, tile = s >> 3;
      const uint8_t *src = p.codes + tile * p.KC * kSlot + (s & 7) * kSegment;
      for (int e = 0; e < now.steps; ++e) {
        if (!mbar_wait_warp(&empty[slot], ph ^ 1, p.wait_budget, &abort_flag, p.err)) goto issued_all;
        if (leader) {
          const int n = tile < p.tiles ? min(kw, p.KC - e * kw) : 0;  // stages there are
          mbar_arrive_expect_tx(&full[slot], (uint32_t)(n * strips * kSegment));
          for (int q = 0; q < n; ++q)
            bulk_g2s(ring + slot * kSlot + q * strips * kSegment, src + (int64_t)(e * kw + q) * kSlot,
                     strips * kSegment, &full[slot]);
        }
        __syncwarp();
        ++issued;
        if (++slot == p.slots) slot = 0, ph ^= 1;
      }
    }
  issued_all:
    drain_ring(full, p.slots, issued, p.drain_budget, p.err);
    return;
  }

  // ------------------------------ consumers ------------------------------
  const int pitch = kSource == kFromGlobal ? p.K_pad : p.K_pad + 32;  // (+32: the eight tokens' loads meet all banks)
  const int gq = lane >> 2, cq = lane & 3;
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  if constexpr (kSource == kFromActivations) {
    quantize_to_shared<T, kWarps>(static_cast<const T *>(p.x), p.ldx, p.M, p.K, p.K_pad, p.vec, xs, pitch, s_scale,
                                  s_max, consumers_sync);
  } else {
    if (threadIdx.x < 8 * kTiles) s_scale[threadIdx.x] = threadIdx.x < p.M ? p.x_scales[threadIdx.x] : 0.f;
    if constexpr (kSource == kFromCodes) {
      // Several warps a row where there are few rows.
      int per = kWarps;
      while (per > 1 && per * p.M > kWarps) per /= 2;
      for (int m = warp / per; m < p.M; m += kWarps / per) {
        const int8_t *row = static_cast<const int8_t *>(p.x) + m * p.ldx;
        int8_t *to = xs + m * pitch;
        if (p.vec) {  // (whole rows of 16 bytes)
#pragma unroll 4
          for (int k = 16 * (warp % per * 32 + lane); k < p.K_pad; k += 512 * per)
            *reinterpret_cast<uint4 *>(to + k) =
                k < p.K ? *reinterpret_cast<const uint4 *>(row + k) : make_uint4(0, 0, 0, 0);
        } else {
          // A row may start on any byte: its codes come out of the aligned words they lie in.
          const int shift = 8 * (int)(reinterpret_cast<uintptr_t>(row) & 3), second = shift > 0;
          const uint32_t *words = reinterpret_cast<const uint32_t *>(row - shift / 8);
          const int k0 = 4 * (warp % per * 32 + lane);
#pragma unroll 4
          for (int k = k0; k + 8 <= p.K; k += 128 * per)
            *reinterpret_cast<uint32_t *>(to + k) = __funnelshift_r(words[k / 4], words[k / 4 + second], shift);
          // The last ones, whose second word may lie past the row, by bytes; then zeros.
          for (int k = k0 + (p.K - k0 < 8 ? 0 : (p.K - k0 - 8) / (128 * per) + 1) * (128 * per); k < p.K_pad; k += 128 * per) {
            uint32_t v = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (k + j < p.K) v |= (uint32_t)(uint8_t)row[k + j] << (8 * j);
            *reinterpret_cast<uint32_t *>(to + k) = v;
          }
        }
      }
    }
  }
  consumers_sync();
  const int8_t *xb[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    // (Columns of tokens past M are computed from what is there and not stored.)
    if constexpr (kSource == kFromGlobal)
      xb[t] = static_cast<const int8_t *>(p.x) + (int64_t)min(8 * t + gq, p.M - 1) * pitch + 8 * cq;
    else
      xb[t] = xs + (8 * t + gq) * pitch + 8 * cq;
  }

  const int half = warp >> 3, pos = warp & 7;
  int slot = half;
  uint32_t ph = 0;
  int turn = 0;  // slots so far, modulo 2
  bool ok = true;
  for (int r = 0; r < p.rounds; ++r) {
    // The channel whose outputs this thread will write (the same for all its tokens).
    const Round now(p, r);
    const int strips = now.strips, kw = now.kw, q = pos / strips;
    const int row = threadIdx.x & 15, strip = (threadIdx.x >> 4) & (strips - 1);
    const int64_t n = (now.strip + strip) * kI8Strip + row;
    const float sw = n < p.N ? p.scales[n] : 0.f;
    int d[kTiles][4] = {};
    for (int e = 0; e < now.steps; ++e, turn ^= 1) {
      if (turn != half) continue;
      // After a wait that gave up the loops go on for the barriers below, without
      // work and without releasing a slot that this warp has not seen full: the
      // producer would copy into one whose copy is under way.
      ok = ok && mbar_wait_warp(&full[slot], ph, p.wait_budget, &abort_flag, p.err);
      const int kc = e * kw + q;
      if (ok && kc < p.KC) {
        const uint4 *a = reinterpret_cast<const uint4 *>(ring + slot * kSlot + pos * kSegment) + lane;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 w = a[32 * i];
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            const uint2 b = *reinterpret_cast<const uint2 *>(xb[t] + kc * kI8PadK + i * kI8Block);
            asm volatile(
                "mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                : "+r"(d[t][0]), "+r"(d[t][1]), "+r"(d[t][2]), "+r"(d[t][3])
                : "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w), "r"(b.x), "r"(b.y));
          }
        }
      }
      __syncwarp();
      if (ok && lane == 0) mbar_arrive(&empty[slot]);
      slot += 2;
      if (slot >= p.slots) slot = half, ph ^= 1;
    }
    // Element (row, token) of tile t: d[t][i], row gq + 8 (i >> 1), token 8 t + 2 cq + (i & 1).
    int *buf = sums + (r & 1) * kWarps * 128 * kTiles;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
      *reinterpret_cast<int4 *>(buf + (warp * kTiles + t) * 128 + 4 * lane) =
          make_int4(d[t][0], d[t][1], d[t][2], d[t][3]);
    consumers_sync();  // (the other buffer is read before the next one)
    if (n >= p.N || !ok) continue;
    for (int m = (threadIdx.x >> 4) / strips; m < p.M; m += 2 * kWarps / strips) {
      const int at = (m >> 3) * 128 + 4 * (4 * (row & 7) + ((m & 7) >> 1)) + 2 * (row >> 3) + (m & 1);
      int v = 0;
      for (int w = strip; w < kWarps; w += strips) v += buf[w * kTiles * 128 + at];
      store_i8_out(p.out, m, n, (float)v * s_scale[m] * sw);
    }
  }
}

size_t decode_smem(int tiles, int x_pitch, int slots) {
  return (size_t)slots * kSlot + (size_t)2 * kWarps * 128 * tiles * 4 + (size_t)8 * tiles * x_pitch;
}
constexpr size_t kMostSmem = 226 * 1024;  // (static shared memory beside it)

template <int kTiles, I8Source kSource, typename T>
cudaError_t launch_decode_t(const I8DecodeParams &p, int grid, size_t smem, cudaStream_t s) {
  auto kern = int8_decode_kernel<kTiles, kSource, T>;
  cudaError_t e = opt_in_smem(reinterpret_cast<const void *>(kern), (int)kMostSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;  // (what comes before is waited for before anything but the weight is read)
  return cudaLaunchKernelEx(&cfg, kern, p);
}

template <I8Source kSource, typename T>
cudaError_t launch_decode_n(int tiles, const I8DecodeParams &p, int grid, size_t smem, cudaStream_t s) {
  return tiles == 1 ? launch_decode_t<1, kSource, T>(p, grid, smem, s) : launch_decode_t<2, kSource, T>(p, grid, smem, s);
}

// Tokens (in eights: 1 or 2) that one launch takes of M, with a ring of at
// least four slots; 0: not even eight fit into shared memory.
int decode_tiles(int64_t M, int K_pad) {
  int tiles = M <= 8 ? 1 : 2;
  while (tiles > 0 && decode_smem(tiles, K_pad + 32, 4) > kMostSmem) tiles /= 2;
  return tiles;
}

}  // namespace

bool int8_decode_fits(int64_t M, int K_pad) { return decode_tiles(M, K_pad) * 8 >= M; }

bool int8_decode_quantizes(int64_t M, int K, int K_pad) {
  return M * K <= kI8FusedQuantize && int8_decode_fits(M, K_pad);
}

cudaError_t launch_int8_decode(const archead_int8_weight *w, const void *x, int dtype, int64_t ldx,
                               const float *x_scales, int64_t M, I8Out out, cudaStream_t s) {
  I8DecodeParams p{};
  p.codes = w->codes;
  p.scales = w->scales;
  p.N = w->N;
  p.K = w->K;
  p.K_pad = w->K_pad;
  p.KC = w->K_pad / kI8PadK;
  p.tiles = (int)(w->N_pad / kI8PadN);
  p.ldx = ldx;
  p.err = w->err;
  p.wait_budget = w->wait_budget;
  p.drain_budget = std::max(w->wait_budget, kDefaultWaitBudget);
  // Rounds of kw[0] K stages a slot while every block has one, then rounds of kw[1]
  // >= kw[0] for the strips that are left: the fewest slots for the busiest block,
  // where a round's end costs about as much as two.  (8 tokens of 20000 x 1024 8.0
  // us, with one kw for all 9.6; 1 token of 10007 x 2501 8.9 and 10.0.)
  const int64_t all = (w->N + kI8Strip - 1) / kI8Strip;
  int64_t least = INT64_MAX;
  for (int kw0 = 1; kw0 <= 8; kw0 *= 2) {
    const int64_t full = all / ((int64_t)w->sm_count * (8 / kw0)), left = all - full * w->sm_count * (8 / kw0);
    for (int kw1 = kw0; kw1 <= 8; kw1 *= 2) {
      const int64_t per_round = (int64_t)w->sm_count * (8 / kw1), rounds = (left + per_round - 1) / per_round;
      const int steps0 = (p.KC + kw0 - 1) / kw0, steps1 = (p.KC + kw1 - 1) / kw1;
      const int64_t cost = full * (steps0 + 2) + rounds * (steps1 + 2);
      if (cost < least) {
        least = cost;
        p.kw[0] = kw0;
        p.kw[1] = kw1;
        p.steps[0] = steps0;
        p.steps[1] = steps1;
        p.first_rounds = (int)full;
        p.rounds = (int)(full + rounds);
        p.last_strip = all - left;
      }
    }
  }
  const int64_t last_blocks = (all - p.last_strip + 8 / p.kw[1] - 1) / (8 / p.kw[1]);
  const int grid = p.first_rounds > 0 ? w->sm_count : (int)std::min<int64_t>(w->sm_count, last_blocks);
  const int tiles = decode_tiles(M, w->K_pad), step = 8 * std::max(1, tiles);
  const int pitch = tiles == 0 ? 0 : w->K_pad + 32;
  const int most = (int)((kMostSmem - decode_smem(std::max(1, tiles), pitch, 0)) / kSlot);
  const int64_t slots = (int64_t)p.first_rounds * p.steps[0] + (int64_t)(p.rounds - p.first_rounds) * p.steps[1];
  const int64_t needed = (slots + 1) / 2 * 2;
  p.slots = (int)std::min<int64_t>({(int64_t)kMostSlots, (int64_t)most / 2 * 2, needed});
  const size_t smem = decode_smem(std::max(1, tiles), pitch, p.slots);
  const int e = x_scales ? 1 : dtype_bytes(dtype), ye = dtype_bytes(out.dtype);
  for (int64_t m = 0; m < M; m += step) {
    p.M = (int)std::min<int64_t>(step, M - m);
    p.x = static_cast<const char *>(x) + m * ldx * e;
    p.x_scales = x_scales ? x_scales + m : nullptr;
    p.out = out;
    p.out.y = static_cast<char *>(out.y) + m * out.ld * ye;
    p.vec = (reinterpret_cast<uintptr_t>(p.x) & 15) == 0 && ldx * e % 16 == 0;
    cudaError_t err;
    if (!x_scales)
      err = dtype == ARCHEAD_DTYPE_FP32   ? launch_decode_n<kFromActivations, float>(tiles, p, grid, smem, s)
            : dtype == ARCHEAD_DTYPE_FP16 ? launch_decode_n<kFromActivations, __half>(tiles, p, grid, smem, s)
                                          : launch_decode_n<kFromActivations, __nv_bfloat16>(tiles, p, grid, smem, s);
    else if (tiles == 0)
      err = launch_decode_t<1, kFromGlobal, int8_t>(p, grid, smem, s);
    else
      err = launch_decode_n<kFromCodes, int8_t>(tiles, p, grid, smem, s);
    if (err != cudaSuccess) return err;
  }
  return cudaSuccess;
}

}  // namespace archead
