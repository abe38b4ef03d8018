// Tensor-memory kernel of the INT8 product: more tokens than the warp-level
// kernel takes.
//
// 8-bit codes are exact in fp16, and this chip's tensor cores do fp16 products
// far faster than 8-bit integer ones (warp-level: 299 against 75 T
// multiply-adds a second), so the kernel runs kind::f16 MMAs on widened codes.
// Products are integers up to 2^14 and their fp32 sums exact up to 2^24.
//
// The weight's 128 channels of a tile are the MMA's M side (one TMEM lane
// each), the tokens its N side.  Per stage of 128 of K:
//   - one warp loads the tokens' widened codes (fp16, in the K order of the
//     weight's words, 128-byte swizzle) by TMA, another the tile's 16 KB of
//     codes with one bulk copy;
//   - a converter warpgroup (several take stages in turn) widens the codes and
//     stores them as the A operand in tensor memory, whose tcgen05.st.16x128b
//     registers are the fragment registers that the words hold;
//   - one thread issues eight MMAs into a TMEM accumulator that holds the whole
//     K of the unit; up to 128 tokens a unit two threads take stages in turn, each
//     with an accumulator of its own (a thread needs some 700 cycles for a stage's
//     eight MMAs, which run 312 for 64 tokens and 536 for 128);
//   - epilogue warps read the accumulators, scale, round and store.
//
// Bound: by the tensor cores from some 200 tokens on (512 tokens of 151936 x 4096
// 338 us, 2048 1.32 ms: all of the rate that the library's bf16 product reaches in a
// burst; at the power limit 375 us and 1.40 to 1.44 ms), by memory for fewer of a
// large weight (64 tokens 99 us, 128 106: 95 and 92%), and by its
// start, its stages' pace and its join for a small weight (64 tokens of 4096 x 512
// 5.7 us, the quantiser's launch included).
#include <cuda_fp16.h>

#include <limits.h>

#include <algorithm>

#include "int8_quant.cuh"
#include "prefill_kernel.cuh"  // tcgen05 wrappers, ring positions

namespace archead {

// Instance for units of up to NT tokens; kSplit: the blocks of a cluster share
// the K of one unit and join their sums.  TMEM: kAcc accumulators of NT columns,
// then kA stages of the A operand (64 columns: 128 of K).
//
// Up to 128 tokens a unit, the x ring and the A ring are one: a stage's barrier
// completes with its x and its A operand, and the MMAs' commit frees both.  A
// satisfied barrier probe takes some 90 cycles, and with one for each the issuing
// thread needed longer for a stage than its MMAs.
template <int NT, bool kSplit>
struct I8Geom {
  static constexpr bool kOne = NT <= 128;
  static constexpr int kConv = NT == 256 ? 2 : NT == 128 && kSplit ? 3 : 4;  // converter warpgroups
  static constexpr int kXS = NT == 64 ? (kSplit ? 4 : 6) : NT == 128 ? (kSplit ? 3 : 4) : 2;
  static constexpr int kA = kOne ? kXS : 4;        // A stages
  static constexpr int kIssue = kOne && kXS % 2 == 0 ? 2 : 1;  // issuing threads (see there)
  static constexpr int kAcc = (kPfTmemCols - kA * 64) / (NT * kIssue);  // units whose accumulators there are
  static constexpr int kEpi = NT == 64 ? 1 : 2;    // epilogue warpgroups
  static constexpr int kCols = NT / kEpi;          // accumulator columns a thread takes
  static constexpr int kThreads = 128 * (1 + kConv + kEpi);
  static constexpr int kBoxBytes = NT * 64 * 2;
  static constexpr int kXBytes = 2 * kBoxBytes;
  static constexpr int kCodeSlot = kI8PadN * kI8PadK;  // 16 KB
  static constexpr int kCS = NT == 64 ? 8 : NT == 128 ? (kSplit ? 4 : 6) : 5;
  static constexpr int kCodeOff = kXS * kXBytes;
  static constexpr int kJoinOff = kCodeOff + kCS * kCodeSlot;  // sums of this block's tokens, from every block of the cluster
  static constexpr int kJoinBytes = kSplit ? NT * kI8PadN * 4 : 0;
  static constexpr int kBarOff = kJoinOff + kJoinBytes;
  static constexpr int kBars = 2 * kXS + 2 * kCS + 2 * kA + 2 * kAcc + 1;
  static constexpr int kSmem = kBarOff + kBars * 8 + 16;
  static constexpr int kRegs0 = NT == 256 ? 48 : 56;
  static constexpr int kRegsC = NT == 64 || kConv == 3 ? 72 : 56;
  static constexpr int kRegsP = NT == 64 ? 128 : NT == 128 ? (kSplit ? 104 : 112) : 160;
  static_assert(128 * (kRegs0 + kConv * kRegsC + kEpi * kRegsP) <= 65536 / kThreads / 8 * 8 * kThreads, "registers");
  static_assert(kAcc * kIssue * NT + kA * 64 <= kPfTmemCols, "TMEM columns");
  static_assert(kSmem <= 227 * 1024, "shared memory");
  static_assert(kA >= kConv && kCS >= kA, "stages and slots (see the converters)");
  static_assert(kIssue == 1 || (kA % 2 == 0 && kConv % 2 == 0 && kCS % 2 == 0), "stages of two issuers (see the converters)");
};

struct I8GemmParams {
  CUtensorMap tmap_x;  // fp16 [M][K_pad], box 64 x nt
  const uint8_t *codes;
  const float *scales, *x_scales;
  I8Out out;
  int64_t N;
  int M, nt, num_mt, units;
  int KC;        // stages of K
  int ks_log2;   // log2 of the blocks that share a unit's K
  int *err;
  int64_t wait_budget;
  int64_t drain_budget;  // of the waits for what is in flight when a block ends: no less than the default
};

__host__ __device__ constexpr uint32_t idesc_f16(int m, int n) {
  return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// One probe of a barrier's phase, without suspending.
__device__ __forceinline__ bool mbar_test_a(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
               : "=r"(ok)
               : "r"(bar), "r"(parity)
               : "memory");
  return ok != 0;
}

// Four signed codes as two fp16 pairs, exact: the offset-binary byte u in the
// mantissa of fp16 1024 is 1024 + u = 1152 + code.
__device__ __forceinline__ void widen_int8x4(uint32_t w, uint32_t &lo, uint32_t &hi) {
  const uint32_t u = w ^ 0x80808080u;
  const __half2 bias = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));  // 1152
  const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
  const __half2 ra = __hsub2(*reinterpret_cast<const __half2 *>(&a), bias);
  const __half2 rb = __hsub2(*reinterpret_cast<const __half2 *>(&b), bias);
  lo = *reinterpret_cast<const uint32_t *>(&ra);
  hi = *reinterpret_cast<const uint32_t *>(&rb);
}

// One channel's sums of kCols tokens, of which `cols` are there.  xs: the
// tokens' scales, token 32 c + lane in xs[c].  (Loaded by every thread where
// they were used, a load waited for the store before it, which may have been
// to the same place: 256 tokens of 4096 x 512 took 13.1 us, with this 8.9.)
template <typename T, int kCols>
__device__ __forceinline__ void store_channel(const I8Out &o, int64_t m0, int64_t n, bool there, const float (&acc)[kCols],
                                              int cols, const float (&xs)[(kCols + 31) / 32], float sw) {
  T *y = static_cast<T *>(o.y) + m0 * o.ld + n;
#pragma unroll
  for (int i = 0; i < kCols; ++i, y += o.ld) {
    const float s = __shfl_sync(0xffffffffu, xs[i / 32], i % 32);
    if (there && i < cols) *y = from_f32<T>(acc[i] * s * sw);
  }
}

template <int kCols>
__device__ __forceinline__ void store_channel(const I8Out &o, int64_t m0, int64_t n, bool there, const float (&acc)[kCols],
                                              int cols, const float (&xs)[(kCols + 31) / 32], float sw) {
  if (o.dtype == ARCHEAD_DTYPE_FP32)
    store_channel<float>(o, m0, n, there, acc, cols, xs, sw);
  else if (o.dtype == ARCHEAD_DTYPE_FP16)
    store_channel<__half>(o, m0, n, there, acc, cols, xs, sw);
  else
    store_channel<__nv_bfloat16>(o, m0, n, there, acc, cols, xs, sw);
}

__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory"); }

template <int NT, bool kSplit>
__global__ void __launch_bounds__(I8Geom<NT, kSplit>::kThreads, 1)
    int8_gemm_kernel(const __grid_constant__ I8GemmParams p) {
  using G = I8Geom<NT, kSplit>;
  constexpr int kXS = G::kXS, kCS = G::kCS, kA = G::kA, kAcc = G::kAcc;
  extern __shared__ uint8_t smem[];  // 1024-byte aligned (the swizzle's period)
  uint64_t *bars = reinterpret_cast<uint64_t *>(smem + G::kBarOff);
  uint64_t *x_full = bars, *x_empty = x_full + kXS, *c_full = x_empty + kXS, *c_empty = c_full + kCS;
  uint64_t *a_full = c_empty + kCS, *a_empty = a_full + kA, *acc_full = a_empty + kA, *acc_empty = acc_full + kAcc;
  uint64_t *drain = acc_empty + kAcc;
  if (G::kOne) x_full = a_full, x_empty = a_empty;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(drain + 1);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1), *x_issued = abort_flag + 1;
  const int warp = threadIdx.x >> 5, lane = lane_id();

  if (smem_u32(smem) & 1023) {  // the same for every block: nothing has been started
    if (threadIdx.x == 0) atomicOr(p.err, kErrLayout);
    return;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < kXS && !G::kOne; ++i) mbar_init(&x_full[i], 1), mbar_init(&x_empty[i], 1);
    for (int i = 0; i < kCS; ++i) mbar_init(&c_full[i], 1), mbar_init(&c_empty[i], 4);
    for (int i = 0; i < kA; ++i) mbar_init(&a_full[i], G::kOne ? 5 : 4), mbar_init(&a_empty[i], 1);
    for (int i = 0; i < kAcc; ++i) mbar_init(&acc_full[i], G::kIssue), mbar_init(&acc_empty[i], 4 * G::kEpi);
    mbar_init(drain, G::kIssue);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc(tmem_slot, kPfTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // A block's shared memory may be written by its peers from when it is known to
  // run: the cluster meets twice, here (waited for by the epilogue before its
  // first remote store, by the others at the end) and at the join.
  if constexpr (kSplit) cluster_arrive_relaxed();
  const uint32_t tmem_base = *tmem_slot;
  const uint32_t a_base = tmem_base + kAcc * G::kIssue * NT;
  bool mma_leader = false;

  // Unit u: tokens u % num_mt of tile u / num_mt.  With kSplit a cluster has one
  // unit and this block one slice of its K.
  const int ks = kSplit ? 1 << p.ks_log2 : 1, slice = kSplit ? (int)blockIdx.x & (ks - 1) : 0;
  const int u0 = kSplit ? (int)blockIdx.x >> p.ks_log2 : (int)blockIdx.x, step = kSplit ? p.units : (int)gridDim.x;
  const int begin = kSplit ? p.KC * slice / ks : 0, end = kSplit ? p.KC * (slice + 1) / ks : p.KC;
  // Over several rounds half of the tiles at work start in the middle of K: all read
  // the same tokens, and did so at the same time from the same places of L2 (128
  // tokens of 151936 x 4096 115 us, with this 105; 256 210 and 179, 512 383 and 338; with
  // four starts or eight 345 and 350).  In one round there is nothing to gain (512
  // tokens of 4096 x 4096 16.6 us and 16.8).
  const int at_once = p.units <= (int)gridDim.x ? 0 : max(2, (int)gridDim.x / p.num_mt);
  const auto first_of = [&](int u) {
    if constexpr (kSplit) return begin;
    return at_once > 0 && 2 * (u / p.num_mt % at_once) >= at_once ? (begin + end) / 2 : begin;
  };
  int met = 0;  // times this thread has met its cluster
  int issued = 0;  // stages whose copies this warp has issued
  int stopped = INT_MAX;  // stage at which this converter's wait gave up, counted over all units

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(G::kRegs0) : "memory");
    if (warp == 0) {
      // ------------------------------ tokens ------------------------------
      const bool leader = elect_one();
      RingPos<kXS> r;
      asm volatile("griddepcontrol.wait;\n" ::: "memory");  // the widened codes come from the grid before
      for (int u = u0; u < p.units; u += step) {
        const int m0 = u % p.num_mt * p.nt;
        for (int e = begin, k = first_of(u); e < end; ++e, k = k + 1 < end ? k + 1 : begin) {
          if (!mbar_wait_warp(&x_empty[r.s], r.ph ^ 1, p.wait_budget, abort_flag, p.err)) goto done;
          if (leader) {
            uint8_t *dst = smem + r.s * G::kXBytes;
            mbar_arrive_expect_tx(&x_full[r.s], (uint32_t)p.nt * 256);
            tma_load_2d(dst, &p.tmap_x, k * 128, m0, &x_full[r.s]);
            tma_load_2d(dst + G::kBoxBytes, &p.tmap_x, k * 128 + 64, m0, &x_full[r.s]);
          }
          ++issued;
          r.next();
          __syncwarp();
        }
      }
    } else if (warp == 2) {
      // ------------------------------ weight codes ------------------------------
      const bool leader = elect_one();
      RingPos<kCS> r;
      for (int u = u0; u < p.units; u += step) {
        const uint8_t *src = p.codes + (int64_t)(u / p.num_mt) * p.KC * G::kCodeSlot;
        for (int e = begin, k = first_of(u); e < end; ++e, k = k + 1 < end ? k + 1 : begin) {
          if (!mbar_wait_warp(&c_empty[r.s], r.ph ^ 1, p.wait_budget, abort_flag, p.err)) goto done;
          if (leader) {
            mbar_arrive_expect_tx(&c_full[r.s], G::kCodeSlot);
            bulk_g2s(smem + G::kCodeOff + r.s * G::kCodeSlot, src + (int64_t)k * G::kCodeSlot, G::kCodeSlot,
                     &c_full[r.s]);
          }
          ++issued;
          r.next();
          __syncwarp();
        }
      }
    } else if (warp == 1 || (warp == 3 && G::kIssue == 2)) {
      // ------------------------------ MMAs ------------------------------
      const bool leader = elect_one();
      mma_leader = leader;
      const uint32_t idesc = idesc_f16(128, p.nt);
      const uint64_t xdesc = smem_desc_sw128(smem_u32(smem));
      constexpr uint32_t kBox = G::kBoxBytes >> 4;
      RingPos<kXS> xr;
      RingPos<kA> ar;
      RingPos<kAcc> accr;
      // Of two issuing threads each takes every other stage, counted over all
      // units: with an even number of stages in the ring a stage's place is then
      // always the same thread's, and it has seen that place's last phase.
      const int me = warp >> 1;
      int turn = 0;
      bool polled = false;  // the next stage's barrier was seen complete
      for (int u = u0; u < p.units; u += step) {
        if (!mbar_wait_warp(&acc_empty[accr.s], accr.ph ^ 1, p.wait_budget, abort_flag, p.err)) goto done;
        const uint32_t d = tmem_base + (accr.s * G::kIssue + (G::kIssue == 2 ? me : 0)) * NT;
        bool first = true;
        for (int e = begin; e < end; ++e) {
          const bool mine = G::kIssue == 1 || turn == me;
          turn ^= 1;
          if (!mine) {
            xr.next();
            ar.next();
            continue;
          }
          if (!G::kOne && !mbar_wait_warp(&x_full[xr.s], xr.ph, p.wait_budget, abort_flag, p.err)) goto done;
          if (!__all_sync(0xffffffffu, polled) &&
              !mbar_wait_warp(&a_full[ar.s], ar.ph, p.wait_budget, abort_flag, p.err))
            goto done;
          tc_fence_after();
          const uint32_t a = a_base + ar.s * 64;
          const uint64_t b = xdesc + (uint32_t)((G::kOne ? ar.s : xr.s) * (G::kXBytes >> 4));
          const RingPos<kA> now = ar, ahead = ar.ahead(G::kIssue);
          ar.next();
          if (leader) {
#pragma unroll
            for (int q = 0; q < 4; ++q)  // (+2 in the descriptor: 32 bytes)
              tc_mma_ts(d, a + 8 * q, b + 2 * q, idesc, q > 0 || !first);
          }
          first = false;
          __syncwarp();
          polled = mbar_test_a(smem_u32(&a_full[ahead.s]), ahead.ph);  // (under way while the others are issued)
          if (leader) {
#pragma unroll
            for (int q = 0; q < 4; ++q) tc_mma_ts(d, a + 8 * (q + 4), b + kBox + 2 * q, idesc, 1);
            if (!G::kOne) tc_commit(&x_empty[xr.s]);
            tc_commit(&a_empty[now.s]);
          }
          __syncwarp();
          xr.next();
        }
        if (leader) tc_commit(&acc_full[accr.s]);  // (of all this thread's MMAs, if it had any)
        __syncwarp();
        accr.next();
      }
    }
  } else if (warp < 4 + 4 * G::kConv) {
    // ------------------------------ converters ------------------------------
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(G::kRegsC) : "memory");
    const int cg = (warp - 4) >> 2, cw = warp & 3;
    RingPos<kCS> cr;
    RingPos<kA> ar;
    cr.next(cg);
    ar.next(cg);  // (cg < kConv <= kA)
    int n = cg;  // this warpgroup's next stage, of the stages of unit u
    for (int u = u0; u < p.units; u += step) {
      const int len = end - begin;
      for (; n < len; n += G::kConv) {
        // A parity shows only one phase from the next, so a barrier may be at most
        // one behind what is waited for.  The A stage's: this warpgroup's last
        // stage n - kConv waited for the MMAs of n - kConv - kA, which with kA >=
        // kConv are behind those that used this place before the last.  Then the
        // code slot's: that the A stage is free says that the MMAs of n - kA are
        // done, so with kCS >= kA those of n - kCS are, and its codes had come.
        // Both hold for the MMAs of one thread, which end in order.  Of two
        // threads those of stages an even number apart do: kConv, kA and kCS are
        // even then.  (With five code slots a converter could pass a barrier whose
        // copy, from DRAM out of order, had not come.)
        if (!mbar_wait_warp(&a_empty[ar.s], ar.ph ^ 1, p.wait_budget, abort_flag, p.err) ||
            !mbar_wait_warp(&c_full[cr.s], cr.ph, p.wait_budget, abort_flag, p.err)) {
          stopped = (u - u0) / step * len + n;
          goto done;
        }
        tc_fence_after();
        const uint4 *codes = reinterpret_cast<const uint4 *>(smem + G::kCodeOff + cr.s * G::kCodeSlot) + cw * 256 + lane;
        const uint32_t acol = a_base + ((uint32_t)(cw * 32) << 16) + ar.s * 64;
        uint4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = codes[32 * i];
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // the warp's strips of 16 channels
#pragma unroll
          for (int half = 0; half < 2; ++half) {  // 64 of K: four steps of 16
            uint32_t a[16];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint4 v = w[2 * half + i];
              widen_int8x4(v.x, a[8 * i], a[8 * i + 2]);
              widen_int8x4(v.y, a[8 * i + 1], a[8 * i + 3]);
              widen_int8x4(v.z, a[8 * i + 4], a[8 * i + 6]);
              widen_int8x4(v.w, a[8 * i + 5], a[8 * i + 7]);
              if (h == 0) w[2 * half + i] = codes[128 + 32 * (2 * half + i)];
            }
            tmem_st_frag4(acol + ((uint32_t)(16 * h) << 16) + 32 * half, a);
          }
        }
        asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory");
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&c_empty[cr.s]), mbar_arrive(&a_full[ar.s]);
        cr.next(G::kConv);
        ar.next(G::kConv);
      }
      n -= len;
    }
  } else {
    // ------------------------------ epilogue ------------------------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(G::kRegsP) : "memory");
    constexpr int kCols = G::kCols;
    const int pw = (warp - 4 - 4 * G::kConv) >> 2, lg = warp & 3;
    const int col0 = kCols * pw;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(lg * 32) << 16) + col0;
    RingPos<kAcc> accr;
    int stages = 0;  // of the units before, modulo 2
    if constexpr (kSplit) {
      cluster_wait();
      met = 1;
    }
    asm volatile("griddepcontrol.wait;\n" ::: "memory");  // (the tokens' scales)
    for (int u = u0; u < p.units; u += step) {
      const int64_t n = (int64_t)(u / p.num_mt) * kI8PadN + lg * 32 + lane;
      const int mu = u % p.num_mt * p.nt;
      const int m0 = mu + col0, cols = min(kCols, min(p.M, mu + p.nt) - m0);  // (may be negative: none)
      const float sw = p.scales[n];
      float xs[kCols / 32];
#pragma unroll
      for (int c = 0; c < kCols / 32; ++c)
        xs[c] = 32 * c + lane < cols ? p.x_scales[m0 + 32 * c + lane] : 0.f;
      if (!mbar_wait_warp(&acc_full[accr.s], accr.ph, p.wait_budget, abort_flag, p.err)) goto done;
      tc_fence_after();
      float acc[kCols];
      // The first accumulator: of two that of the thread that had the unit's first stage.
      const uint32_t acc0 = lane_addr + (accr.s * G::kIssue + (G::kIssue == 2 ? stages : 0)) * NT;
#pragma unroll
      for (int c = 0; c < kCols; c += 16) {
        uint32_t v[16];
        tmem_ld16<false>(acc0 + c, v);
        tmem_wait_ld(v);
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[c + i] = __uint_as_float(v[i]);
      }
      if (G::kIssue == 2 && end - begin > 1) {
        const uint32_t acc1 = lane_addr + (accr.s * 2 + (stages ^ 1)) * NT;
#pragma unroll
        for (int c = 0; c < kCols; c += 16) {
          uint32_t v[16];
          tmem_ld16<false>(acc1 + c, v);
          tmem_wait_ld(v);
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[c + i] += __uint_as_float(v[i]);
        }
      }
      stages ^= (end - begin) & 1;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&acc_empty[accr.s]);
      accr.next();
      if constexpr (kSplit) {
        // Block q of the cluster takes the tokens from q NT / ks on: the sums go
        // into its shared memory, by slice, and after the cluster's barrier it
        // adds them up in the order of the slices.  (The number of slices is a
        // constant in each copy of this: with shifts and branches for every
        // token a join took 3 to 7 us.)
        const auto join = [&](auto log2) {
          constexpr int kS = 1 << decltype(log2)::value, kPer = NT / kS, kMine = kPer / G::kEpi;
          const uint32_t place = smem_u32(smem) + G::kJoinOff + (slice * kPer * kI8PadN + lg * 32 + lane) * 4;
#pragma unroll
          for (int q = 0; q < kCols / kPer; ++q) {
            if (q * kPer >= cols) break;
            uint32_t to;
            asm("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(to) : "r"(place), "r"(pw * (kCols / kPer) + q));
#pragma unroll
            for (int i = 0; i < kPer; ++i)
              asm volatile("st.shared::cluster.f32 [%0], %1;\n" ::"r"(to + i * (kI8PadN * 4)), "f"(acc[q * kPer + i])
                           : "memory");
          }
          const int64_t mb = mu + slice * kPer + pw * kMine;
          const int lim = min(p.M, mu + p.nt) - (int)mb;  // tokens of this thread (none or less: none)
          float xq[(kMine + 31) / 32], v[kMine];
#pragma unroll
          for (int c = 0; c < (kMine + 31) / 32; ++c)
            xq[c] = 32 * c + lane < min(lim, kMine) ? p.x_scales[mb + 32 * c + lane] : 0.f;
          cluster_arrive();
          cluster_wait();
          met = 2;
          const float *sums = reinterpret_cast<const float *>(smem + G::kJoinOff) + pw * kMine * kI8PadN + lg * 32 + lane;
#pragma unroll
          for (int i = 0; i < kMine; ++i) v[i] = sums[i * kI8PadN];
#pragma unroll
          for (int s = 1; s < kS; ++s)
#pragma unroll
            for (int i = 0; i < kMine; ++i) v[i] += sums[(s * kPer + i) * kI8PadN];
          store_channel<kMine>(p.out, mb, n, n < p.N, v, lim, xq, sw);
        };
        if (p.ks_log2 == 1) join(Int<1>{});
        else if (p.ks_log2 == 2) join(Int<2>{});
        else join(Int<3>{});
        break;
      }
      store_channel<kCols>(p.out, m0, n, n < p.N, acc, cols, xs, sw);
    }
  }
done:
  if (mma_leader) {
    tc_commit(drain);  // (each issuing thread's)
    mbar_wait(drain, 0, p.drain_budget, nullptr, p.err);
  }
  if (threadIdx.x == 0) *x_issued = issued;
  if (kSplit && met < 2) {  // every thread meets its cluster twice, whatever became of its work
    __syncwarp();
    if (met == 0) cluster_wait();
    cluster_arrive();
    cluster_wait();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, kPfTmemCols);
  }
  // Without a wait that gave up every copy has been used.  Otherwise what is under
  // way lands before the block ends.  A barrier that a stage's tokens share with its
  // converters takes first what these owe: nobody else arrives any more, and a stage
  // is issued only when the one before in its place has been multiplied.
  if (*abort_flag) {
    if (warp == 0) drain_copies(x_full, kXS, issued, p.drain_budget, p.err);
    if (warp == 2) drain_copies(c_full, kCS, issued, p.drain_budget, p.err);
    if (G::kOne && lane == 0)
      for (int k = stopped; k < *x_issued; k += G::kConv) mbar_arrive(&a_full[k % kA]);
  }
}

namespace {

template <int NT, bool kSplit>
cudaError_t launch_gemm_t(const I8GemmParams &p, int grid, cudaStream_t s) {
  auto kern = int8_gemm_kernel<NT, kSplit>;
  using G = I8Geom<NT, kSplit>;
  cudaError_t e = opt_in_smem(reinterpret_cast<const void *>(kern), G::kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(G::kThreads);
  cfg.dynamicSmemBytes = G::kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 1 << p.ks_log2;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = kSplit ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, p);
}

}  // namespace

template <int NT>
static cudaError_t clusters_of(int (&room)[4]) {
  using G = I8Geom<NT, true>;
  auto kern = int8_gemm_kernel<NT, true>;
  cudaError_t e = opt_in_smem(reinterpret_cast<const void *>(kern), G::kSmem);
  for (int log2 = 1; log2 <= 3 && e == cudaSuccess; ++log2) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(1 << log2);
    cfg.blockDim = dim3(G::kThreads);
    cfg.dynamicSmemBytes = G::kSmem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 1 << log2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&room[log2], kern, &cfg);
  }
  return e;
}

cudaError_t int8_gemm_room(archead_int8_weight *w) {
  cudaError_t e = clusters_of<64>(w->clusters[0]);
  if (e == cudaSuccess) e = clusters_of<128>(w->clusters[1]);
  return e;
}

// How a product is cut: the least estimated time over the instances (units of up
// to 64, 128 or 256 tokens, spread evenly) and over clusters of 1, 2, 4 or 8
// blocks along K.  The estimate, in ns, goes by measured times of 4 to 32 stages
// (128 of K): a stage of up to 64 tokens takes some 267, of 128 358 where many
// blocks run (317 where few do), of 256 683; the start and the last epilogue 3 a
// token and more for the larger instances; a join 1300.
I8GemmPlan int8_gemm_plan(const archead_int8_weight *w, int64_t M) {
  I8GemmPlan best;
  double least = 1e300;
  const int64_t tiles = w->N_pad / kI8PadN;
  const int KC = w->K_pad / kI8PadK;
  for (int NT = 64; NT <= 256; NT *= 2) {
    const int64_t fewest = (M + NT - 1) / NT;
    for (int64_t num_mt = fewest; num_mt < fewest + 3; ++num_mt) {
      const int nt = (int)(((M + num_mt - 1) / num_mt + 15) / 16 * 16);
      const int64_t units = tiles * num_mt;
      const double stage = NT == 64 ? 250 + 0.3 * nt : NT == 128 ? std::max(300.0, 217 + 1.1 * nt) : std::max(420.0, 120 + 2.2 * nt);
      const double start = 3 * nt + (NT == 64 ? 0 : NT == 128 ? 300 : 1000);
      for (int log2 = 0; log2 <= (NT == 256 ? 0 : 3) && 1 << log2 <= KC; ++log2) {
        const int64_t at_once = log2 == 0 ? w->sm_count : w->clusters[NT == 128][log2];
        if (at_once < 1) continue;
        const double rounds = (double)((units + at_once - 1) / at_once);
        const double cost = rounds * ((KC + (1 << log2) - 1) >> log2) * stage + start + (log2 > 0 ? 1300 * rounds : 0);
        if (cost < least) {
          least = cost;
          best.NT = NT;
          best.nt = nt;
          best.ks_log2 = log2;
          best.num_mt = num_mt;
          best.units = units;
        }
      }
      if (nt <= 16) break;
    }
  }
  return best;
}

cudaError_t launch_int8_gemm(const archead_int8_weight *w, const I8GemmPlan &f, const uint16_t *x,
                             const float *x_scales, int64_t M, I8Out out, cudaStream_t s) {
  I8GemmParams p{};
  if (!make_tma_map_bf16(&p.tmap_x, x, M, w->K_pad, f.nt)) return cudaErrorInvalidValue;
  if (f.units << f.ks_log2 > 0x7fffffff - w->sm_count) return cudaErrorInvalidValue;
  p.codes = w->codes;
  p.scales = w->scales;
  p.x_scales = x_scales;
  p.out = out;
  p.N = w->N;
  p.M = (int)M;
  p.nt = f.nt;
  p.num_mt = (int)f.num_mt;
  p.units = (int)f.units;
  p.KC = w->K_pad / kI8PadK;
  p.ks_log2 = f.ks_log2;
  p.err = w->err;
  p.wait_budget = w->wait_budget;
  p.drain_budget = std::max(w->wait_budget, kDefaultWaitBudget);
  if (f.ks_log2 > 0) {
    const int grid = (int)f.units << f.ks_log2;
    return f.NT == 64 ? launch_gemm_t<64, true>(p, grid, s) : launch_gemm_t<128, true>(p, grid, s);
  }
  const int grid = (int)std::min<int64_t>(f.units, w->sm_count);
  return f.NT == 64    ? launch_gemm_t<64, false>(p, grid, s)
         : f.NT == 128 ? launch_gemm_t<128, false>(p, grid, s)
                       : launch_gemm_t<256, false>(p, grid, s);
}

}  // namespace archead
