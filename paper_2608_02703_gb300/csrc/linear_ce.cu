// Products of the dense head's cross entropy and its gradient: x [M][d], W [V][d].
//
//   loss      l = x W^T, of each token the sum of exp(l - max) and its target's l
//   gradient  by pieces of the vocabulary:  G = g (exp(l - lse) - [target]), l again,
//             then  dx += G W  and  dW = G^T x
//
// Pairs of blocks (a cluster of two) work on units of 256 x 256 outputs with
// tcgen05.mma over both multiprocessors: each block loads half of A's rows and half
// of B's, 16 KB of each for 64 of the summed dimension, and holds half of the unit's
// rows in its tensor memory.  (One block alone would need 24 KB a stage for half
// of the outputs, which is more than shared memory moves beside the MMAs.)  Per block:
//   warp 0      loads stages by TMA; all bytes of a pair's stage complete on the
//               leader's (rank 0's) barrier
//   warp 1      of the leader issues the MMAs of both blocks; their commits free the
//               stage, and announce the accumulator, in both
//   warps 4-11  read the accumulator (one of two, so that the next unit's MMAs run
//               meanwhile): a thread has a row and half of its columns
// Operands are read as they lie: x, W and G with the summed dimension innermost
// (l; G in dx), or with it outermost (W in dx, G and x in dW).  The copy of x and G are in
// panels of 64 columns, so that each box is one run of memory.
//
// Tokens are the rows of l and of dx, so that a thread sums a token's exponentials
// without its neighbours.  Partial sums leave by tile and are joined in a fixed
// order; nothing is added by atomics.
//
// Bound by the tensor cores with many tokens: their pipe is active 97 to 99% of the time in
// the logits' kernels and 94% in the gradient's (4096 tokens x 32000 x 4096).  2048 tokens x 151936
// x 4096 take 1.33 to 1.47 ms (the library's bf16 rate in a burst is 1.31, at the power limit 1.48); loss and gradients
// of 4096 tokens 11.6 to 11.8 ms, 89 to 90% of the burst.  Of some hundred tokens a part of the MMAs' rows is empty (300
// tokens x 32000 x 2048 take what 512 do, 184 us, of which 81 would be needed).  Few tokens are
// bound by memory, which reads W three times and writes dW: the loss of 16 tokens x 151936 x 4096 196 to 200 us (92% of
// the copy rate), loss and gradients of 64 x 262144 x 2560 925 to 960 us (82 to 85%).
#include <algorithm>

#include "int8_quant.cuh"
#include "internal.h"
#include "loss.h"
#include "prefill_kernel.cuh"  // tcgen05 wrappers, ring positions

namespace archead {

namespace {

enum Mode { kLoss, kSoftmax, kGrad };

constexpr int kOperandBytes = 128 * kCeStep * 2;     // a block's part of A or B: 16 KB
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kAcc = 2;                              // accumulators of 256 columns
constexpr int kEpiWarps = 8;
constexpr int kThreads = 128 + 32 * kEpiWarps;
// Steps of a sum in tensor memory where it is taken in parts, which epilogue warps add in registers: of a logit, and of
// an element of dx or dW.  Tensor cores round their additions toward zero, by up to 2^-23 of the sum so far each, and
// always so.  For a logit see the epilogue; of a gradient's terms of one sign 16384 lose some 2^-14 in this way (in one
// sum 2^18 lost 1.2e-3, more than fp16's rounding).
constexpr int kSegment = 16, kGradSegment = 256;
constexpr int kBoxBytes = 32 * 64 * 2;               // outputs that a warp stages: 32 rows of 64 columns
// The gradient's outputs of few tokens are bound by what leaves: there a warp fills a box while its last one is read.
// The loss has no boxes, and epilogue warps that hold a unit's sums in registers.
template <Mode kMode>
struct Geom {
  static constexpr int kBoxes = kMode == kGrad ? 2 : kMode == kSoftmax ? 1 : 0;
  static constexpr int kStages = kMode == kGrad ? 5 : kMode == kSoftmax ? 6 : 7;
  static constexpr int kOutOff = kStages * kStageBytes;
  static constexpr int kBarOff = kOutOff + kEpiWarps * kBoxes * kBoxBytes;
  static constexpr int kBars = 2 * kStages + 2 * kAcc + 1;
  static constexpr int kSmem = kBarOff + kBars * 8 + 32 + 16;
  // Sums in parts: registers of the loading warpgroup and of the others, whose sum is at most that of the launch.
  // (The gradient's loads and MMAs want more: 4096 tokens x 32000 x 4096, gradients alone, 1920 us, with 56 1960.)
  static constexpr int kRegs0 = kMode == kGrad ? 88 : 72, kRegsE = kMode == kGrad ? 200 : 208;
  static constexpr int kRegsInAll = 128 * kRegs0 + 32 * kEpiWarps * kRegsE;
  static_assert(kRegsInAll <= 65536 / kThreads / 8 * 8 * kThreads, "registers");
  static_assert(kSmem <= 227 * 1024, "shared memory");
  static_assert(kStages <= 16, "kinds of the stages");
};
static_assert(kAcc * kCeTile <= kPfTmemCols, "TMEM columns");

struct Params {
  CUtensorMap a[2], b[2];  // (kGrad: of dx, of dW)
  CUtensorMap out;         // G (kSoftmax) or dW (kGrad): boxes of 64 columns x 32 rows
  CUtensorMap out_dx;      // sums of dx (kGrad): boxes of 32 columns x 32 rows
  CeScratch at;
  int64_t V, d, rows;
  int64_t first_tile;      // vocabulary tile that the piece starts with
  int tiles;               // vocabulary tiles of the piece
  int64_t piece;           // G's columns
  int nt;                  // vocabulary columns of a unit (kLoss, kSoftmax), a multiple of 32 or 64
  int a_rows;              // token rows of a block's part of A that are loaded: 32, 64 or 128
  int a_both;              // the second block has tokens, too
  int direct, M;           // x is read where it lies, and all M tokens have rows (kLoss, kSoftmax)
  int half;                // rows of G's first part, where it has a second one behind it (kSoftmax: kTwo), else 0
  int splits, dx_pitch, add_dx, want_dx, want_dw, box_out;
  void *dw;
  int64_t lddw;
  int accumulate, fp16;
  int *err;
  int64_t wait_budget, drain_budget;
};

// Instruction descriptor: kind::f16, fp32 sums, 256 x n outputs of two blocks; majors: 1 where the
// summed dimension is outermost.
__host__ __device__ constexpr uint32_t idesc_pair(bool fp16, int n, int a_major, int b_major) {
  return (1u << 4) | (fp16 ? 0u : (1u << 7) | (1u << 10)) | (uint32_t)a_major << 15 | (uint32_t)b_major << 16 |
         (uint32_t)(n >> 3) << 17 | (256u >> 4) << 24;
}

// Descriptor of an operand with the summed dimension outermost, 128-byte swizzle: boxes of 64 (rows of
// A or B) x 64 (summed), 8 KB each; eight of the summed dimension are 1 KB.
__device__ __forceinline__ uint64_t smem_desc_outer(uint32_t saddr) {
  uint64_t desc = (uint64_t)((saddr >> 4) & 0x3FFF);
  desc |= (uint64_t)(8192 >> 4) << 16;  // from 64 rows to the next
  desc |= (uint64_t)(1024 >> 4) << 32;  // from eight of the sum to the next
  desc |= (uint64_t)1 << 46;
  desc |= (uint64_t)2 << 61;
  return desc;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t of_rank(uint32_t saddr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(r) : "r"(saddr), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
// A box into this block's shared memory, its bytes counted on the barrier at `bar` of either block.
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap *map, int c0, int c1, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], "
      "[%4];\n" ::"r"(dst),
      "l"(map), "r"(c0), "r"(c1), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d_tmem),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Arrives, when the MMAs issued so far are done, on the barrier at this place in both blocks.
__device__ __forceinline__ void commit_pair(uint64_t *bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n" ::"r"(
          smem_u32(bar)),
      "h"((uint16_t)3)
      : "memory");
}
// (Relaxed: what it tells is that tensor memory has been read, which tcgen05's own wait and fences
// order.  With release semantics it waited for all the thread's stores, 3000 cycles a unit.)
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];\n" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void store_cluster(uint32_t addr, int v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;\n" ::"r"(addr), "r"(v) : "memory");
}

// A unit: outputs of tile (row, col), sums over the steps [k0, k1) of 64.
struct Unit {
  int row, col, k0, k1, split;
  bool dw;
};

// The units of this pair, in the same order for every role.  kGrad: those of the longer kind (of dx or
// of dW), one pair after the other; then the others, which the pairs that had one of the long less
// begin with (as many as make up for it), so that all end together.
template <Mode kMode>
struct Units {
  int pairs, me, nm, nd, ks, kt, n1, n2, head, ahead, i;
  bool dw_first;
  __device__ Units(const Params &p, int count) {
    pairs = gridDim.x >> 1;
    me = blockIdx.x >> 1;
    nm = kMode != kGrad && p.rows == kCeTile ? 1 : (count + kCeTile - 1) / kCeTile;  // (see the loads)
    i = me;
    const int64_t cols = min((int64_t)p.tiles * kCeTile, p.V - p.first_tile * kCeTile);
    if (kMode != kGrad) {
      ks = (int)((p.d + kCeStep - 1) / kCeStep);
      n1 = nm * (int)((cols + p.nt - 1) / p.nt);
      return;
    }
    ks = (int)((cols + kCeStep - 1) / kCeStep);
    kt = p.half == 0 ? (count + kCeStep - 1) / kCeStep : count == 0 ? 0 : 2 * p.half / kCeStep;
    nd = (int)((p.d + kCeTile - 1) / kCeTile);
    const int n_dx = p.want_dx ? nm * nd * p.splits : 0, n_dw = p.want_dw ? p.tiles * nd : 0;
    // (A unit of dW takes its epilogue's time, some six steps, at least.)
    const int dx_steps = max(1, ks / p.splits), dw_steps = max(6, kt);
    dw_first = dw_steps > dx_steps;
    n1 = dw_first ? n_dw : n_dx;
    n2 = dw_first ? n_dx : n_dw;
    const int longer = max(dx_steps, dw_steps), shorter = min(dx_steps, dw_steps);
    head = n1 % pairs;  // pairs with one of the longer units more
    ahead = head > 0 ? (longer + shorter / 2) / shorter : 0;
  }
  __device__ __forceinline__ void unit_of_dx(const Params &p, uint32_t at, Unit &u) const {
    const uint32_t t = at / (uint32_t)p.splits, split = at % (uint32_t)p.splits;
    u = {(int)(t % (uint32_t)nm), (int)(t / (uint32_t)nm), 0, 0, (int)split, false};
    u.k0 = (int)((uint32_t)ks * split / (uint32_t)p.splits);  // (2^18 steps, 32 splits)
    u.k1 = (int)((uint32_t)ks * (split + 1) / (uint32_t)p.splits);
  }
  __device__ __forceinline__ void unit_of_dw(const Params &p, uint32_t at, Unit &u) const {
    // (Neighbours take a vocabulary tile's columns: G is read once by all of them, and whole rows of dW are written.)
    u = {(int)(at / (uint32_t)nd), (int)(at % (uint32_t)nd), 0, kt, 0, true};
  }
  __device__ bool next(const Params &p, Unit &u) {
    if (kMode != kGrad) {
      if (i >= n1) return false;
      u = {i % nm, i / nm, 0, ks, 0, false};
      i += pairs;
      return true;
    }
    // (32 bits: divisions of 64 took longer than the rest of a short unit's epilogue)
    uint32_t at = i;
    const bool first = i < n1;
    if (first) {
      i += pairs;
    } else {
      // Round r of the shorter kind.  In the first `ahead` rounds only the pairs from `head` on take part.
      if (i < (1 << 30)) i = (1 << 30) + (me < head ? ahead : 0);  // (rounds from here on)
      const int r = i - (1 << 30), few = pairs - head;
      at = r < ahead ? r * few + (me - head) : ahead * few + (r - ahead) * pairs + me;
      if (at >= (uint32_t)n2) return false;
      ++i;
    }
    if (first == dw_first)
      unit_of_dw(p, at, u);
    else
      unit_of_dx(p, at, u);
    return true;
  }
};

template <typename T>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
  if constexpr (sizeof(T) == 2 && __is_same(T, __nv_bfloat16)) return pack_bf16x2(a, b);
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint32_t pack_out(float a, float b, bool fp16) {
  return fp16 ? pack16<__half>(a, b) : pack16<__nv_bfloat16>(a, b);
}

// N columns of an accumulator's row.
template <int N>
__device__ __forceinline__ void read_columns(uint32_t taddr, float (&v)[N]) {
  uint32_t r[N / 16][16];
#pragma unroll
  for (int c = 0; c < N / 16; ++c) tmem_ld16<false>(taddr + 16 * c, r[c]);
#pragma unroll
  for (int c = 0; c < N / 16; ++c) tmem_wait_ld(r[c]);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = __uint_as_float(r[i / 16][i % 16]);
}

// 32 columns of an accumulator's row, read while the 32 before them are worked on.
struct Columns32 {
  uint32_t a[16], b[16];
  __device__ __forceinline__ explicit Columns32(uint32_t taddr) { load(taddr); }
  __device__ __forceinline__ void load(uint32_t taddr) {
    tmem_ld16<false>(taddr, a);
    tmem_ld16<false>(taddr + 16, b);
  }
  // What has been read, and the next at `taddr` where there is more.
  __device__ __forceinline__ void take(float (&v)[32], uint32_t taddr, bool more) {
    tmem_wait_ld(a);
    tmem_wait_ld(b);
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(a[i]), v[16 + i] = __uint_as_float(b[i]);
    if (more) load(taddr);
  }
};

// A warp's box of outputs on its way to memory: rows of 128 bytes, swizzled as TMA has them.
template <int kBoxes>
struct OutBox {
  uint32_t base;  // shared memory, 1024-byte aligned
  int lane;
  uint32_t at = 0;
  int turn = 0;
  // Before the first value: the next box's last content has been read.
  __device__ __forceinline__ void begin() {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;\n" ::"n"(kBoxes - 1) : "memory");
    __syncwarp();
    at = base + turn * kBoxBytes;
    if (kBoxes > 1) turn ^= 1;
  }
  // Columns 8 j .. 8 j + 7 of this lane's row.
  __device__ __forceinline__ void put(int j, uint32_t a, uint32_t b, uint32_t c, uint32_t d, int off = 0) const {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(at + off + lane * 128 + ((j ^ (lane & 7)) << 4)), "r"(a),
                 "r"(b), "r"(c), "r"(d)
                 : "memory");
  }
  __device__ __forceinline__ void store(const CUtensorMap *map, int col, int row, int off = 0) const {
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];\n" ::"l"(map), "r"(col),
                   "r"(row), "r"(at + off)
                   : "memory");
      asm volatile("cp.async.bulk.commit_group;\n" ::: "memory");
    }
  }
  __device__ __forceinline__ void end() const {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;\n" ::: "memory");
    __syncwarp();
  }
};

// One more 32 columns, from `base` on, of a token's sum: sum e^m, m the largest logit.
__device__ __forceinline__ void sum_columns(float (&v)[32], int64_t base, int64_t V, int target, float *tlogit, float &m,
                                            float &sum) {
  const int lim = (int)min((int64_t)32, V - base);  // columns that are there
  if (lim < 32) {
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (j >= lim) v[j] = -INFINITY;
  }
  const int64_t at = (int64_t)target - base;
  if (target >= 0 && at >= 0 && at < 32) {
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      int which = (int)at;
      asm volatile("" : "+r"(which));  // (otherwise the values go through local memory, all of them)
      if (j == which) *tlogit = v[j];
    }
  }
  __syncwarp();
  float tops[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
  for (int j = 4; j < 32; ++j) tops[j & 3] = fmaxf(tops[j & 3], v[j]);
  const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  if (top > m) {
    sum *= ex2_approx((m - top) * kLog2e);
    m = top;
  }
  // (Differences first: of large logits a product with log2 e would be rounded by more than the difference is.)
  const float minus = fabsf(m) == INFINITY ? 0.f : -m;  // (nothing but -inf so far, or a sum that is infinite)
  float2 part[2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
  for (int j = 0; j < 32; j += 2) {
    const float2 e = __fmul2_rn(__fadd2_rn(make_float2(v[j], v[j + 1]), make_float2(minus, minus)), make_float2(kLog2e, kLog2e));
    part[j >> 1 & 1] = __fadd2_rn(part[j >> 1 & 1], make_float2(ex2_approx(e.x), ex2_approx(e.y)));
  }
  sum += (part[0].x + part[0].y) + (part[1].x + part[1].y);
}

// The i-th 32 columns of a half: every other 32 of the unit (kLoss), every other 64 (kSoftmax: a box's), or 128 (kGrad).
template <Mode kMode>
__device__ __forceinline__ int chunk_of(int half, int i) {
  return kMode == kLoss ? half + 2 * i : kMode == kSoftmax ? 2 * half + (i & 1) + 4 * (i >> 1) : 4 * half + i;
}

// 32 columns of an accumulator's row added to what is held.
__device__ __forceinline__ void add_columns(uint32_t taddr, float (&held)[32]) {
  float v[32];
  read_columns<32>(taddr, v);
#pragma unroll
  for (int j = 0; j < 32; ++j) held[j] += v[j];
}

// What rounding to w, 16 bits each, took from a and b, as 16 bits.
template <typename T>
__device__ __forceinline__ uint32_t rest16(float a, float b, uint32_t w) {
  float2 r;
  if constexpr (__is_same(T, __nv_bfloat16))
    r = make_float2(bf16_lo(w), bf16_hi(w));
  else
    r = __half22float2(*reinterpret_cast<const __half2 *>(&w));
  return pack16<T>(a - r.x, b - r.y);
}

// kParts: sums over more than a segment are taken in parts.  kTwo: G has two parts (kSoftmax).
template <Mode kMode, bool kParts, bool kTwo = false>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    linear_ce_kernel(const __grid_constant__ Params p) {
  using G = Geom<kMode>;
  constexpr int kStages = G::kStages, kPart = kMode == kGrad ? kGradSegment : kSegment;
  extern __shared__ uint8_t smem[];  // 1024-byte aligned (the swizzle's period)
  uint64_t *full = reinterpret_cast<uint64_t *>(smem + G::kBarOff), *empty = full + kStages;
  uint64_t *acc_full = empty + kStages, *acc_empty = acc_full + kAcc, *drain = acc_empty + kAcc;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(drain + 1);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
  volatile int *issued = abort_flag + 1, *peer_abort = abort_flag + 2, *peer_issued = abort_flag + 3;
  volatile uint8_t *kinds = reinterpret_cast<volatile uint8_t *>(abort_flag + 4);  // of the stages: dW's or not
  const int warp = threadIdx.x >> 5, lane = lane_id();
  const uint32_t rank = cluster_rank();
  const bool leader = rank == 0;
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");

  if (smem_u32(smem) & 1023) {  // the same for every block: nothing has been started
    if (threadIdx.x == 0) atomicOr(p.err, kErrLayout);
    return;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(&full[i], 1), mbar_init(&empty[i], 1);
    for (int i = 0; i < kAcc; ++i) mbar_init(&acc_full[i], 1), mbar_init(&acc_empty[i], 2 * kEpiWarps);
    mbar_init(drain, 1);
    *abort_flag = *issued = *peer_abort = *peer_issued = 0;
    fence_mbar_init();
  }
  if (warp == 0 && elect_one()) {
    const auto fetch = [](const CUtensorMap *m) { asm volatile("prefetch.tensormap [%0];\n" ::"l"(m) : "memory"); };
    fetch(&p.a[0]);
    fetch(&p.b[0]);
    if (kMode == kGrad) fetch(&p.a[1]), fetch(&p.b[1]);
    if (kMode != kLoss) fetch(&p.out);
    if (kMode == kGrad) fetch(&p.out_dx);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(tmem_slot)),
                 "r"(kPfTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // (barriers of both blocks are there before either signals the other's)
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  Unit u;

  // Bytes of a stage of both blocks.
  const auto stage_bytes = [&](bool dw) {
    if (kMode == kGrad && dw) return 2u * kStageBytes;
    const uint32_t b = kMode == kGrad ? 2u * kOperandBytes : (uint32_t)p.nt * kCeStep * 2;
    return b + (uint32_t)p.a_rows * (kCeStep * 2) * (p.a_both ? 2 : 1);
  };
  // A stage's boxes of this block: rows of A from a_row on, of B from b_row on, summed dimension from k on.
  const auto load_a = [&](int s, bool dw, int a_row, int k) {
    const uint32_t a = smem_u32(smem) + s * kStageBytes, bar = of_rank(smem_u32(&full[s]), 0);
    const int rows = (int)p.rows;
    if (kMode == kGrad && dw) {
      tma_load_pair(a, &p.a[1], 0, a_row / 64 * rows + k, bar);
      tma_load_pair(a + 8192, &p.a[1], 0, (a_row / 64 + 1) * rows + k, bar);
    } else if (leader || p.a_both) {  // (rows that are not loaded give outputs that are not used)
      if (kMode != kGrad && p.direct)
        tma_load_pair(a, &p.a[0], k, a_row, bar);
      else
        tma_load_pair(a, &p.a[0], 0, k / 64 * rows + a_row, bar);
    }
  };
  const auto load_b = [&](int s, bool dw, int b_row, int k) {
    const uint32_t b = smem_u32(smem) + s * kStageBytes + kOperandBytes, bar = of_rank(smem_u32(&full[s]), 0);
    const int rows = (int)p.rows;
    if (kMode == kGrad && dw) {
      tma_load_pair(b, &p.b[1], 0, b_row / 64 * rows + k, bar);
      tma_load_pair(b + 8192, &p.b[1], 0, (b_row / 64 + 1) * rows + k, bar);
    } else if (kMode == kGrad) {
      const int kb = k + (int)p.first_tile * kCeTile;
      tma_load_pair(b, &p.b[0], b_row, kb, bar);
      tma_load_pair(b + 8192, &p.b[0], b_row + 64, kb, bar);
    } else {
      tma_load_pair(b, &p.b[0], k, b_row, bar);
    }
  };
  const auto first_b_row = [&](const Unit &u) {
    return kMode == kGrad ? u.col * kCeTile + 128 * (int)rank
                          : (int)p.first_tile * kCeTile + u.col * p.nt + p.nt / 2 * (int)rank;
  };
  // Where there is one tile of tokens the units do not depend on how many of them count, and what no launch of
  // this call writes may be read while the launch before ends (that one has waited for what came before
  // the call): all that the MMAs take where x is read directly, else the first stages' weights.
  int early = 0;
  if (kMode != kGrad && !p.direct && p.rows == kCeTile && warp == 0) {
    Units<kMode> mine(p, 1);
    if (mine.next(p, u)) {
      early = min(kStages, u.k1);
      if (elect_one())
        for (int k = 0; k < early; ++k) {
          if (leader) mbar_arrive_expect_tx(&full[k], stage_bytes(false));
          load_b(k, false, first_b_row(u), k * kCeStep);
        }
      __syncwarp();
    }
  }
  if (kMode == kGrad || !p.direct || warp >= 4) asm volatile("griddepcontrol.wait;\n" ::: "memory");
  const int count = kMode != kGrad && p.direct ? p.M : p.at.header->count;
  Units<kMode> units(p, count);

  if (warp < 4) {
    if (kParts) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(G::kRegs0) : "memory");
    if (warp == 0) {
      // ------------------------------ loads ------------------------------
      const bool one = elect_one();
      RingPos<kStages> r;
      int n = 0;
      while (units.next(p, u)) {
        const int a_row = u.row * kCeTile + 128 * (int)rank;
        const int b_row = first_b_row(u);
        for (int k = u.k0; k < u.k1; ++k) {
          if (!mbar_wait_warp(&empty[r.s], r.ph ^ 1, p.wait_budget, abort_flag, p.err)) goto loads_end;
          if (one) {
            kinds[r.s] = u.dw;
            if (n >= early) {
              if (leader) mbar_arrive_expect_tx(&full[r.s], stage_bytes(u.dw));
              load_b(r.s, u.dw, b_row, kMode == kGrad && u.dw && p.half > 0 ? 0 : k * kCeStep);  // (x is the same for both parts)
            }
            load_a(r.s, u.dw, a_row, k * kCeStep);
          }
          ++n;
          r.next();
          __syncwarp();
        }
      }
      // The commits that free the last stages arrive in both blocks before either ends.
      for (int i = 0; i < kStages; ++i, r.next())
        if (!mbar_wait_warp(&empty[r.s], r.ph ^ 1, p.wait_budget, abort_flag, p.err)) break;
    loads_end:
      if (lane == 0) *issued = n;
    } else if (warp == 1 && leader) {
      // ------------------------------ MMAs ------------------------------
      const bool one = elect_one();
      const uint32_t base = smem_u32(smem);
      RingPos<kStages> r;
      RingPos<kAcc> acc;
      bool stop = false;
      while (!stop && units.next(p, u)) {
        const bool a_outer = kMode == kGrad && u.dw, b_outer = kMode == kGrad;
        const uint32_t idesc = idesc_pair(p.fp16, kMode == kGrad ? kCeTile : p.nt, a_outer, b_outer);
        const uint64_t a0 = a_outer ? smem_desc_outer(base) : smem_desc_sw128(base);
        const uint64_t b0 = b_outer ? smem_desc_outer(base + kOperandBytes) : smem_desc_sw128(base + kOperandBytes);
        const uint32_t a_step = a_outer ? 2048 >> 4 : 32 >> 4, b_step = b_outer ? 2048 >> 4 : 32 >> 4;  // 16 of the sum
        int k = u.k0;
        do {
          const int end = kParts ? min(u.k1, k + kPart) : u.k1;
          if (!mbar_wait_warp(&acc_empty[acc.s], acc.ph ^ 1, p.wait_budget, abort_flag, p.err)) {
            stop = true;
            break;
          }
          tc_fence_after();
          const uint32_t d = tmem_base + acc.s * kCeTile;
          const int start = k;
          for (; k < end; ++k) {
            if (!mbar_wait_warp(&full[r.s], r.ph, p.wait_budget, abort_flag, p.err)) {
              stop = true;
              break;
            }
            tc_fence_after();
            if (one) {
              const uint64_t a = a0 + (uint32_t)(r.s * (kStageBytes >> 4)), b = b0 + (uint32_t)(r.s * (kStageBytes >> 4));
#pragma unroll
              for (int q = 0; q < 4; ++q) mma_pair(d, a + q * a_step, b + q * b_step, idesc, k > start || q > 0);
              commit_pair(&empty[r.s]);
            }
            __syncwarp();
            r.next();
          }
          if (stop) break;
          if (one) commit_pair(&acc_full[acc.s]);
          __syncwarp();
          acc.next();
        } while (k < u.k1);
      }
      if (one) commit_pair(drain);
      __syncwarp();
    }
  } else {
    // ------------------------------ epilogue ------------------------------
    if (kParts) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(G::kRegsE) : "memory");
    const int quad = warp & 3, half = (warp - 4) >> 2;
    OutBox<G::kBoxes> box{smem_u32(smem) + G::kOutOff + (warp - 4) * G::kBoxes * kBoxBytes, lane};
    const uint32_t taddr0 = tmem_base + ((uint32_t)(quad * 32) << 16);
    // With one row of tiles a token's sum goes on over all of this pair's units.
    const bool through = kMode == kLoss && count <= kCeTile;
    float m = -INFINITY, sum = 0.f;
    int64_t last_row = -1;
    RingPos<kAcc> acc;
    const float unscale = kMode == kGrad ? p.at.header->unscale : 1.f;
    while (units.next(p, u)) {
      const int64_t row = (int64_t)u.row * kCeTile + 128 * (int)rank + 32 * quad + lane;
      // (Of a G in two parts the second's products with W have rows of their own, which are added with the splits of dx.)
      const auto counts = [&](int64_t at) {
        return kMode == kGrad && p.half > 0 ? at < 2 * p.half && (at & (p.half - 1)) < count : at < count;
      };
      bool live = counts(row);
      // (under way while the MMAs are waited for)
      const int t = kMode != kGrad && live ? p.at.target[row] : -1;
      const float lse = kMode == kSoftmax && live ? p.at.lse[row] : 0.f;
      const float f = kMode == kSoftmax && live ? p.at.factor[row] : 0.f;
      if (kMode == kSoftmax) live = live && f != 0.f;  // (read directly, rows that do not count are among them)
      const int64_t row0 = row - lane;
      // The sum of l over a segment: tensor cores round its additions toward zero, by up to 2^-23 of the
      // sum so far each, and always so.  Sums of up to 1024 products are added to one another here (2048 tokens x
      // 151936 x 4096: the loss in error by 4e-7 of itself, in one sum 1.6e-6).  G takes l in the same parts as the loss
      // that its lse comes from: of a target that the model is sure of, 1 - p is as small as what l would differ by (1e-4
      // for l = 20 of 4096 products in one sum).
      // (G's rows up to a whole stage are read as dW's summed dimension; rows past the tokens that count are zeros
      // there, and of no account in dx.)
      const int stage_rows = kTwo ? p.half : (count + kCeStep - 1) / kCeStep * kCeStep;
      const bool wanted = kMode == kSoftmax ? row0 < stage_rows
                          : kMode == kGrad && u.dw ? p.first_tile * kCeTile + row0 < p.V : counts(row0);
      const int chunks = kMode == kGrad ? kCeTile / 32 : p.nt / 32;
      // The sum of all parts but the last.
      const auto add_parts = [&](float (&held)[4][32]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 32; ++j) held[i][j] = 0.f;
        for (int k = u.k0; k + kPart < u.k1; k += kPart) {
          if (!mbar_wait_warp(&acc_full[acc.s], acc.ph, p.wait_budget, abort_flag, p.err)) return false;
          tc_fence_after();
          if (wanted) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int c = chunk_of<kMode>(half, i);
              if (c < chunks) add_columns(taddr0 + acc.s * kCeTile + 32 * c, held[i]);
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_cluster(of_rank(smem_u32(&acc_empty[acc.s]), 0));
          acc.next();
        }
        return true;
      };
      float held[kParts && kMode != kGrad ? 4 : 1][32];
      bool stop = false;
      if constexpr (kParts && kMode != kGrad) {
        stop = !add_parts(held);
      } else if constexpr (kParts) {
        if (u.k1 - u.k0 > kPart) {  // the whole sums take the last part's place, and go on as those of one part do
          float sums[4][32];
          stop = !add_parts(sums) || !mbar_wait_warp(&acc_full[acc.s], acc.ph, p.wait_budget, abort_flag, p.err);
          if (!stop && wanted) {
            tc_fence_after();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t at = taddr0 + acc.s * kCeTile + 32 * chunk_of<kMode>(half, i);
              add_columns(at, sums[i]);
              tmem_st32(at, sums[i]);
            }
            asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory");
          }
        }
      }
      if (stop || !mbar_wait_warp(&acc_full[acc.s], acc.ph, p.wait_budget, abort_flag, p.err)) break;
      tc_fence_after();
      const uint32_t taddr = taddr0 + acc.s * kCeTile;
      if constexpr (kMode == kLoss) {
        const int64_t col0 = (int64_t)u.col * p.nt;
        if (!through) m = -INFINITY, sum = 0.f;
        if (wanted) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int c = chunk_of<kMode>(half, i);
            if (c < chunks) {
              add_columns(taddr + 32 * c, held[i]);
              sum_columns(held[i], col0 + 32 * c, p.V, t, &p.at.tlogit[row], m, sum);
            }
          }
          if (live && !through) p.at.part[((int64_t)u.col * kCeParts + half) * p.rows + row] = make_float2(m, sum);
          if (live) last_row = row;
        }
      } else if constexpr (kMode == kSoftmax) {
        const int64_t col0 = p.first_tile * kCeTile + u.col * p.nt;
        if (wanted) {
          const float minus = -lse;
          const float2 f2 = make_float2(f, f);
          const bool all_live = __all_sync(0xffffffffu, live);
          const auto softmax = [&](float (&v)[32], int c) {
            const int64_t base = col0 + 32 * c;
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              const float2 e = __fmul2_rn(__fadd2_rn(make_float2(v[j], v[j + 1]), make_float2(minus, minus)),
                                          make_float2(kLog2e, kLog2e));
              const float2 g = __fmul2_rn(make_float2(ex2_approx(e.x), ex2_approx(e.y)), f2);
              v[j] = g.x;
              v[j + 1] = g.y;
            }
            const int64_t at = (int64_t)t - base;
            const int hit = t >= 0 && at >= 0 && at < 32 ? (int)at : -1;
            if (__any_sync(0xffffffffu, hit >= 0)) {
              float at_target = 0.f;
#pragma unroll
              for (int j = 0; j < 32; ++j) {
                v[j] -= j == hit ? f : 0.f;
                at_target = j == hit ? v[j] : at_target;
              }
              if (!kTwo && hit >= 0)
                p.at.rest[row] = at_target - (p.fp16 ? __half2float(__float2half_rn(at_target))
                                                     : __bfloat162float(__float2bfloat16_rn(at_target)));
            }
            if (!all_live || p.V - base < 32) {
              const int lim = live ? (int)max((int64_t)0, min((int64_t)32, p.V - base)) : 0;
#pragma unroll
              for (int j = 0; j < 32; ++j) v[j] = j < lim ? v[j] : 0.f;
            }
            if ((c & 1) == 0) box.begin();
            // (The second part goes through the box of a warp that has no tokens: those of two quarters on.)
            constexpr int kSecondBox = 2 * kBoxBytes;
            const auto put = [&](auto type) {
              using T = decltype(type);
#pragma unroll
              for (int j = 0; j < 32; j += 8) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = pack16<T>(v[j + 2 * i], v[j + 2 * i + 1]);
                box.put((c & 1) * 4 + j / 8, w[0], w[1], w[2], w[3]);
                if constexpr (kTwo) {
#pragma unroll
                  for (int i = 0; i < 4; ++i) w[i] = rest16<T>(v[j + 2 * i], v[j + 2 * i + 1], w[i]);
                  box.put((c & 1) * 4 + j / 8, w[0], w[1], w[2], w[3], kSecondBox);
                }
              }
            };
            if (p.fp16) put(__half{});
            else put(__nv_bfloat16{});
            if (c & 1) {
              const int to = (u.col * p.nt + 32 * c) / 64 * (int)p.rows + (int)row0;
              box.store(&p.out, 0, to);
              if constexpr (kTwo) box.store(&p.out, 0, to + p.half, kSecondBox);
            }
          };
          if constexpr (kParts) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int c = chunk_of<kMode>(half, i);
              if (c < chunks) {
                add_columns(taddr + 32 * c, held[i]);
                softmax(held[i], c);
              }
            }
          } else {
            Columns32 next(taddr + 64 * half);
#pragma unroll 1
            for (int c = 2 * half; c < chunks; c += c & 1 ? 3 : 1) {  // (as chunk_of)
              float v[32];
              const int after = c + (c & 1 ? 3 : 1);
              next.take(v, taddr + 32 * after, after < chunks);
              softmax(v, c);
            }
          }
        }
      } else {
        const int64_t col0 = (int64_t)u.col * kCeTile + 128 * half;
        const int64_t n0 = p.first_tile * kCeTile + row0;
        const uint32_t mine = taddr + 128 * half;
        if (u.dw && p.box_out) {
#pragma unroll 1
          for (int c = 0; c < 2; ++c) {
            if (!wanted || col0 + 64 * c >= p.d) break;  // (the same for the warp)
            float v[64];
            if (u.k1 > u.k0) {
              read_columns<64>(mine + 64 * c, v);
            } else {
#pragma unroll
              for (int j = 0; j < 64; ++j) v[j] = 0.f;
            }
            box.begin();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              uint32_t w[4];
#pragma unroll
              for (int i = 0; i < 4; ++i)
                w[i] = pack_out(v[8 * j + 2 * i] * unscale, v[8 * j + 2 * i + 1] * unscale, p.fp16);
              box.put(j, w[0], w[1], w[2], w[3]);
            }
            box.store(&p.out, (int)(col0 + 64 * c), (int)n0);
          }
        } else if (!u.dw && !p.add_dx) {
          if (wanted) {  // (rows past the tokens that count are never read)
#pragma unroll 1
            for (int c = 0; c < 4 && col0 + 32 * c < p.d; ++c) {
              float v[32];
              read_columns<32>(mine + 32 * c, v);
              box.begin();
#pragma unroll
              for (int j = 0; j < 8; ++j)
                box.put(j, __float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]), __float_as_uint(v[4 * j + 2]),
                        __float_as_uint(v[4 * j + 3]));
              box.store(&p.out_dx, (int)(col0 + 32 * c), u.split * (int)p.rows + (int)row0);
            }
          }
        } else
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          float v[32];
          const int64_t base = col0 + 32 * c;
          __syncwarp();
          if (u.k1 > u.k0) {
            read_columns<32>(mine + 32 * c, v);
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = 0.f;
          }
          if (!u.dw) {
            if (!live || base >= p.d) continue;
            // (the pitch is a multiple of 256: what is past d is never read)
            float4 *out = reinterpret_cast<float4 *>(p.at.dx + ((int64_t)u.split * p.rows + row) * p.dx_pitch + base);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              float4 o = out[j];
              o.x += v[4 * j], o.y += v[4 * j + 1], o.z += v[4 * j + 2], o.w += v[4 * j + 3];
              out[j] = o;
            }
          } else {
            const int64_t n = p.first_tile * kCeTile + row;
            if (n >= p.V || base >= p.d) continue;
            uint16_t *out = static_cast<uint16_t *>(p.dw) + n * p.lddw + base;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int left = (int)min((int64_t)8, p.d - (base + 8 * j));
              if (left <= 0) break;
              float x[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) x[i] = v[8 * j + i] * unscale;
              if (left == 8) {
                uint4 *to = reinterpret_cast<uint4 *>(out + 8 * j);
                if (p.accumulate) {
                  float o[8];
                  if (p.fp16) {
                    Raw8<__half> raw;
                    raw.r[0] = *to;
                    raw.values(o);
                  } else {
                    Raw8<__nv_bfloat16> raw;
                    raw.r[0] = *to;
                    raw.values(o);
                  }
#pragma unroll
                  for (int i = 0; i < 8; ++i) x[i] += o[i];
                }
                *to = make_uint4(pack_out(x[0], x[1], p.fp16), pack_out(x[2], x[3], p.fp16),
                                 pack_out(x[4], x[5], p.fp16), pack_out(x[6], x[7], p.fp16));
              } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                  if (i >= left) break;
                  uint16_t *to = out + 8 * j + i;
                  if (p.fp16) {
                    __half *h = reinterpret_cast<__half *>(to);
                    *h = __float2half_rn(x[i] + (p.accumulate ? __half2float(*h) : 0.f));
                  } else {
                    __nv_bfloat16 *h = reinterpret_cast<__nv_bfloat16 *>(to);
                    *h = __float2bfloat16_rn(x[i] + (p.accumulate ? __bfloat162float(*h) : 0.f));
                  }
                }
              }
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_cluster(of_rank(smem_u32(&acc_empty[acc.s]), 0));
      acc.next();
    }
    if (through && last_row >= 0)
      p.at.part[(int64_t)((blockIdx.x >> 1) * kCeParts + half) * p.rows + last_row] = make_float2(m, sum);
    if (kMode != kLoss) box.end();
  }

  // ------------------------------ end ------------------------------
  __syncthreads();
  // MMAs under way read and write both blocks' memories: they end before either block does.
  if (warp == 1) mbar_wait_warp(drain, 0, p.drain_budget, nullptr, p.err);
  if (threadIdx.x == 0) {
    const uint32_t peer = rank ^ 1;
    store_cluster(of_rank(smem_u32((void *)peer_abort), peer), *abort_flag);
    store_cluster(of_rank(smem_u32((void *)peer_issued), peer), *issued);
  }
  __syncwarp();
  cluster_sync();  // (all MMAs have ended; neither block touches the other's memory after this, but for the below)
  if (*abort_flag | *peer_abort) {
    // A wait gave up somewhere: the blocks may have loaded unlike numbers of stages.  A stage completes
    // when both have, so the one that is behind loads what it owes (from the matrices' first
    // places; its slots are free, as the other's are), and the leader waits for the last of them.
    const int mine = *issued, theirs = *peer_issued;
    if (warp == 0) {
      if (elect_one())
        for (int n = mine; n < theirs; ++n) {
          const int s = n % kStages;
          uint32_t dw;
          asm volatile("ld.shared::cluster.u8 %0, [%1];\n" : "=r"(dw) : "r"(of_rank(smem_u32((void *)&kinds[s]), rank ^ 1)));
          if (leader) mbar_arrive_expect_tx(&full[s], stage_bytes(dw));
          load_a(s, dw, 0, 0);
          load_b(s, dw, 0, 0);
        }
      __syncwarp();
      if (leader) drain_copies(full, kStages, max(mine, theirs), p.drain_budget, p.err);
    }
    __syncthreads();
    cluster_sync();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(tmem_base), "r"(kPfTmemCols) : "memory");
  }
}

template <Mode kMode, bool kParts, bool kTwo = false>
cudaError_t launch(const Params &p, int64_t units, int clusters, cudaStream_t s) {
  auto kern = linear_ce_kernel<kMode, kParts, kTwo>;
  constexpr int kSmem = Geom<kMode>::kSmem;
  cudaError_t e = opt_in_smem(reinterpret_cast<const void *>(kern), kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * std::max<int64_t>(1, std::min<int64_t>(units, clusters))));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, p);
}

Params common(const CeCall &c) {
  Params p{};
  p.at = c.loss->at;
  p.V = c.V;
  p.d = c.d;
  p.rows = c.rows;
  p.fp16 = c.fp16;
  p.a_rows = c.M <= 32 ? 32 : c.M <= 64 ? 64 : 128;
  p.a_both = c.M > 128;
  p.err = c.loss->err;
  p.wait_budget = c.loss->wait_budget;
  p.drain_budget = std::max(c.loss->wait_budget, kDefaultWaitBudget);
  return p;
}

int64_t tiles_of(int64_t n) { return (n + kCeTile - 1) / kCeTile; }

// x and G lie in panels of 64 columns, the width of a box: [columns / 64][rows][64].
bool panel_map(CUtensorMap *map, const void *base, int64_t rows, int64_t cols, int box_rows) {
  return make_tma_map_16(map, base, (cols + 63) / 64 * rows, 64, 64, box_rows);
}

// Columns of a unit of logits, a multiple of `grain`: 256, or fewer where few rounds of the pairs are
// the shorter ones for it.  A step of 64 takes its MMAs' time, two cycles a column, or its
// loads', some 45 bytes a cycle of a multiprocessor; the last unit's epilogue 16 a column.  (700
// tokens, 400 of which count, x 10007 x 1000: 80 units for 76 pairs with 256 columns.)
int unit_columns(const CeCall &c, int64_t cols, int grain, int a_rows) {
  const int64_t nm = c.rows / kCeTile, steps = (c.d + kCeStep - 1) / kCeStep, pairs = c.loss->clusters;
  if (nm * tiles_of(cols) > 4 * pairs) return kCeTile;
  int best = kCeTile;
  int64_t least = INT64_MAX;
  for (int nt = kCeTile; nt >= 2 * grain; nt -= grain) {
    const int64_t rounds = (nm * ((cols + nt - 1) / nt) + pairs - 1) / pairs;
    const int64_t cost = rounds * steps * std::max(2 * nt, (a_rows * 128 + 64 * nt) / 45) + 16 * nt;
    if (cost < least) least = cost, best = nt;
  }
  return best;
}

bool logits_maps(const CeCall &c, Params &p, int64_t cols, int grain) {
  p.nt = unit_columns(c, cols, grain, p.a_rows);
  p.direct = c.direct;
  p.M = (int)c.M;
  return (c.direct ? make_tma_map_16(&p.a[0], c.x, c.M, c.d, c.ldx, p.a_rows)
                   : panel_map(&p.a[0], c.loss->at.x, c.rows, c.d, p.a_rows)) &&
         make_tma_map_16(&p.b[0], c.w, c.V, c.d, c.ldw, p.nt / 2);
}

// Units of a launch if all tokens count.
int64_t logits_units(const CeCall &c, const Params &p) {
  const int64_t cols = std::min<int64_t>((int64_t)p.tiles * kCeTile, c.V - p.first_tile * kCeTile);
  return c.rows / kCeTile * ((cols + p.nt - 1) / p.nt);
}

}  // namespace

// (A block that was launched with fewer registers than it hands on would wait for them.)
template <Mode kMode, bool kTwo = false>
static cudaError_t registers_do() {
  cudaFuncAttributes a;
  const cudaError_t e = cudaFuncGetAttributes(&a, linear_ce_kernel<kMode, true, kTwo>);
  return e != cudaSuccess ? e : a.numRegs * kThreads < Geom<kMode>::kRegsInAll ? cudaErrorInvalidConfiguration : cudaSuccess;
}

cudaError_t ce_clusters(int *clusters) {
  auto kern = linear_ce_kernel<kLoss, true>;
  constexpr int kSmem = Geom<kLoss>::kSmem;
  cudaError_t e = opt_in_smem(reinterpret_cast<const void *>(kern), kSmem);
  if (e != cudaSuccess) return e;
  if ((e = registers_do<kLoss>()) != cudaSuccess || (e = registers_do<kSoftmax>()) != cudaSuccess ||
      (e = registers_do<kSoftmax, true>()) != cudaSuccess || (e = registers_do<kGrad>()) != cudaSuccess)
    return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaOccupancyMaxActiveClusters(clusters, kern, &cfg);
  if (e == cudaSuccess && *clusters < 1) e = cudaErrorInvalidConfiguration;
  return e;
}

cudaError_t launch_ce_logits(const CeCall &c, CeParts *parts, cudaStream_t s) {
  Params p = common(c);
  p.first_tile = 0;
  p.tiles = (int)tiles_of(c.V);
  if (!logits_maps(c, p, c.V, 32)) return cudaErrorInvalidValue;
  const int64_t units = logits_units(c, p), columns = (c.V + p.nt - 1) / p.nt;
  parts->by_tile = (int)columns * kCeParts;
  parts->by_pair = (int)std::min<int64_t>({units, columns, c.loss->clusters}) * kCeParts;
  return launch<kLoss, true>(p, units, c.loss->clusters, s);
}

int64_t ce_piece_tiles(const archead_loss *l, const CeCall &c) {
  // (Pieces of 64 MB, which would stay in L2 until they have been read, took up to 26% more, most with few columns:
  // more launches, and sums of dx that are read and written more often.)
  const int64_t tiles = tiles_of(c.V), most = std::max<int64_t>(1, l->g_bytes / (c.rows * kCeTile * 2));
  const int64_t pieces = (tiles + most - 1) / most;
  return (tiles + pieces - 1) / pieces;
}

// dx is cut along the vocabulary where its tiles are fewer than the pairs (without dW, whose units even
// the pairs' times out: than half).
int ce_dx_splits(const archead_loss *l, int64_t M, int64_t V, int64_t d, bool want_dw) {
  const int64_t units = tiles_of(M) * tiles_of(d), steps = (V + kCeStep - 1) / kCeStep;
  return (int)std::max<int64_t>(1, std::min<int64_t>({(want_dw ? 1 : 2) * l->clusters / units, 32, steps / 8}));
}

cudaError_t launch_ce_gradient(const CeCall &c, cudaStream_t s) {
  Params p = common(c);
  const int64_t tiles = tiles_of(c.V), per = ce_piece_tiles(c.loss, c);
  p.piece = per * kCeTile;
  p.splits = c.splits;
  p.dx_pitch = c.dx_pitch;
  p.want_dx = c.want_dx;
  p.want_dw = c.dw != nullptr;
  p.dw = c.dw;
  p.lddw = c.lddw;
  p.accumulate = c.accumulate;
  Params g = p;  // of the products with G
  p.half = g.half = c.half;
  if (c.half > 0) g.a_rows = 2 * c.half;
  if (g.want_dx && !make_tma_map_f32(&g.out_dx, c.loss->at.dx, c.rows * c.splits, c.dx_pitch, 32)) return cudaErrorInvalidValue;
  // (A box is cut off at whole 16 bytes past the matrix's edge: what lies between rows would be written.)
  g.box_out = g.want_dw && !c.accumulate && c.d % 8 == 0;
  if (g.box_out && !make_tma_map_16(&g.out, c.dw, c.V, c.d, c.lddw, 32)) return cudaErrorInvalidValue;
  if (!logits_maps(c, p, std::min(c.V, p.piece), 64) || !panel_map(&p.out, c.loss->at.G, c.rows, p.piece, 32) ||
      !panel_map(&g.a[0], c.loss->at.G, c.rows, p.piece, g.a_rows) ||
      !make_tma_map_16(&g.b[0], c.w, c.V, c.d, c.ldw, 64) ||
      !panel_map(&g.a[1], c.loss->at.G, c.rows, p.piece, 64) || !panel_map(&g.b[1], c.loss->at.x, c.rows, c.d, 64))
    return cudaErrorInvalidValue;
  const int64_t nm = c.rows / kCeTile, nd = tiles_of(c.d);
  // Whether any sum is longer than a segment: of tokens, or of a split of a piece.
  const int64_t steps = std::max(g.want_dw ? c.rows : 0, g.want_dx ? (p.piece + c.splits - 1) / c.splits : 0) / kCeStep;
  const bool parts = steps >= kGradSegment;
  const bool cut = c.d > kSegment * kCeStep;  // (the logits' sums)
  const auto of_g = c.half > 0 ? cut ? launch<kSoftmax, true, true> : launch<kSoftmax, false, true>
                          : cut ? launch<kSoftmax, true> : launch<kSoftmax, false>;
  for (int64_t first = 0; first < tiles; first += per) {
    p.first_tile = g.first_tile = first;
    p.tiles = g.tiles = (int)std::min(per, tiles - first);
    cudaError_t e = of_g(p, logits_units(c, p), c.loss->clusters, s);
    if (e != cudaSuccess) return e;
    g.add_dx = first > 0;
    const int64_t units = (g.want_dx ? nm * nd * g.splits : 0) + (g.want_dw ? g.tiles * nd : 0);
    e = parts ? launch<kGrad, true>(g, units, c.loss->clusters, s) : launch<kGrad, false>(g, units, c.loss->clusters, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace archead
