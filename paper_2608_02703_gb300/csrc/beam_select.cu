// Selection of the next beams: of each batch entry's beams x vocabulary
// candidates, value = (score - lse) + logit, the n largest (include/archead.h).
//
// One launch that reads the logits once and a few of them again; bound by
// memory, at few rows by latency (512 rows of 151936 in fp32 57 us, 81% of the copy
// rate, 128 rows 21 us, 54%; 4 rows 8.2 us, of which some 3 are the reading and the
// launch, the rest the merge's steps, each of which waits for the one before).
//
// A warp takes segments of 512 logits (16 a lane, copied some segments ahead into
// shared memory by asynchronous copies that each thread waits for itself) and
// keeps, without meeting any other, its lanes' sums of exp(l - m) for a reference
// m near the maximum; each segment leaves its largest logit.  The block that
// finishes last of a batch entry
//   - joins the blocks' sums, in their order, into each beam's log-sum-exp;
//   - finds the n best segments by their largest values: no other holds one of
//     the n best candidates;
//   - reads those again and takes the n best candidates of them.
// Both searches go by a threshold first, which n entries reach for certain and
// few more: for the segments one from the threads' largest values, for the
// candidates the n-th best segment's.  Entries compare by value, beam, logit and
// token (segments by their number), so there are no ties.  Where more pass than
// the list takes (equal values, a segment that holds most of the best) the
// search is made again with a threshold that bounds what passes: of the maxima
// of G groups of threads the n-th largest is no more than the n-th of all, and
// no more than n groups hold what reaches it.
//
// (Keeping a list of the n best in every block cost more than the reading: lists
// with a threshold that all warps share met at a barrier for every tile, lists
// of a warp's own let too much pass; 512 rows of 151936 in bf16 took 69 us, now 39.
// The merge's steps as functions and short loops, for fewer instructions to fetch,
// took 24.8 us for 128 rows in fp32 against 22.)
//
// Sums are fp32: each thread's over its logits of the segments in turn, then a
// fixed tree; a row's depends on its logits alone, so that equal beams tie.
#include <cuda_fp16.h>

#include <algorithm>

#include "beam.h"
#include "device.cuh"
#include "internal.h"

namespace archead {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kE = 16;                     // logits of a lane and segment
constexpr int kSegment = 32 * kE;
constexpr int kList = 64 + 1024;           // entries: the best so far, and what passes a threshold of groups
constexpr float kLog2e = 1.4426950408889634f;

// Key of (logit, token): a larger logit, or the lower token of equal ones, has
// the larger key.  (Adding 0 makes the two zeros one.)  0 is no candidate.
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ uint64_t make_key(float l, uint32_t token) {
  return (uint64_t)ordered(l) << 32 | (uint32_t)~token;
}
__device__ __forceinline__ uint32_t key_token(uint64_t key) { return ~(uint32_t)key; }

__device__ __forceinline__ float exp_of(float d) {  // e^d, d <= 0: relative error of a few 2^-23
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(d * kLog2e));
  return y;
}

__device__ __forceinline__ float exp2_of(float d) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(d));
  return y;
}

// The largest of three; of the warp's.  NaNs are left out unless all are.
__device__ __forceinline__ float max3(float a, float b, float c) {
  asm("max.f32 %0, %0, %1, %2;\n" : "+f"(a) : "f"(b), "f"(c));
  return a;
}
__device__ __forceinline__ float warp_max(float v) {
  asm("redux.sync.max.f32 %0, %0, 0xffffffff;\n" : "+f"(v));
  return v;
}

// A thread's sum of exp(l - m) for a reference m: a maximum seen before, replaced
// when a logit passes it by 16 (terms stay below e^16, whose sums fp32 holds as
// exactly as any).  It is kept as sum of 2^(l log2e - c) with c = m log2e
// rounded: an FMA rounds only that difference, and what c misses of m log2e is
// put right where m changes and at the end.  A reference whose c would overflow
// (rows masked with the type's lowest value), or none yet, takes exp(l - m) as
// it stands.
struct RunningSum {
  float m = -INFINITY, c = 0.f, s = 0.f;
  __device__ __forceinline__ static bool scaled(float m) { return fabsf(m) < 1e38f; }
  template <int kN>
  __device__ __forceinline__ void add(const float (&x)[kN], float top) {
    if (top > m + 16.f) {
      s = value();
      if (m > -INFINITY) s *= exp_of(m - top);
      m = top;
      c = m * kLog2e;
      if (scaled(m)) s *= exp2_of(fmaf(m, kLog2e, -c));
    }
    if (scaled(m)) {
      float2 sum = make_float2(0.f, 0.f);
      const float2 scale = make_float2(kLog2e, kLog2e), shift = make_float2(-c, -c);
#pragma unroll
      for (int i = 0; i < kN; i += 2) {
        const float2 d = __ffma2_rn(make_float2(x[i], x[i + 1]), scale, shift);
        sum = __fadd2_rn(sum, make_float2(exp2_of(d.x), exp2_of(d.y)));
      }
      s += sum.x + sum.y;
    } else {
      const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int i = 0; i < kN; ++i) s += exp_of(x[i] - ref);
    }
  }
  // The sum of exp(l - m).
  __device__ __forceinline__ float value() const { return scaled(m) ? s * exp2_of(-fmaf(m, kLog2e, -c)) : s; }
};

// A lane's sixteen logits of a segment, as they are stored.
template <typename T>
struct Raw {
  static constexpr int kPer = 16 / sizeof(T);  // of a 16-byte load
  static constexpr int kLoads = kE / kPer;
  uint4 r[kLoads];
  // Place of value i within the segment.
  static __device__ __forceinline__ int place(int i) { return (i / kPer) * 32 * kPer + lane_id() * kPer + i % kPer; }
  // The values of load c; tokens from `end` on read as -inf.
  static __device__ __forceinline__ uint4 some(const T *row, int v, int end) {
    alignas(16) T t[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) t[j] = v + j < end ? row[v + j] : T(-INFINITY);
    return *reinterpret_cast<const uint4 *>(t);
  }
  __device__ __forceinline__ void load(const T *row, int v0, int end, bool vec) {
#pragma unroll
    for (int c = 0; c < kLoads; ++c) {
      const int v = v0 + place(c * kPer);
      r[c] = vec && v + kPer <= end ? __ldg(reinterpret_cast<const uint4 *>(row + v)) : some(row, v, end);
    }
  }
  // The same of a row that starts on 16 bytes, through this thread's places (16 bytes of each
  // 256 threads') of a ring slot.
  static __device__ __forceinline__ void start(uint32_t slot, const T *row, int v0, int end) {
    if (v0 + kSegment <= end) {
      const T *src = row + v0 + place(0);
#pragma unroll
      for (int c = 0; c < kLoads; ++c)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(slot + c * kThreads * 16),
                     "l"(src + c * 32 * kPer)
                     : "memory");
    } else {
#pragma unroll
      for (int c = 0; c < kLoads; ++c) {
        const int v = v0 + place(c * kPer);
        if (v + kPer <= end) {
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(slot + c * kThreads * 16), "l"(row + v)
                       : "memory");
        } else {
          const uint4 q = some(row, v, end);
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(slot + c * kThreads * 16), "r"(q.x), "r"(q.y),
                       "r"(q.z), "r"(q.w)
                       : "memory");
        }
      }
    }
  }
  __device__ __forceinline__ void take(uint32_t slot) {
#pragma unroll
    for (int c = 0; c < kLoads; ++c)
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n"
                   : "=r"(r[c].x), "=r"(r[c].y), "=r"(r[c].z), "=r"(r[c].w)
                   : "r"(slot + c * kThreads * 16)
                   : "memory");
  }
  // The largest value (NaNs left out, unless all are).
  __device__ __forceinline__ float top(const float (&x)[kE]) const {
    if constexpr (__is_same(T, __nv_bfloat16)) {
      __nv_bfloat162 m = *reinterpret_cast<const __nv_bfloat162 *>(&r[0].x);
#pragma unroll
      for (int i = 1; i < kE / 2; ++i)
        m = __hmax2(m, reinterpret_cast<const __nv_bfloat162 *>(&r[i / 4])[i % 4]);
      return fmaxf(__low2float(m), __high2float(m));
    } else {
      float m = fmaxf(x[0], x[1]);
#pragma unroll
      for (int i = 2; i < kE; i += 2) m = max3(m, x[i], x[i + 1]);
      return m;
    }
  }
  __device__ __forceinline__ void values(float (&x)[kE]) const {
#pragma unroll
    for (int c = 0; c < kLoads; ++c) {
      const uint32_t u[4] = {r[c].x, r[c].y, r[c].z, r[c].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
          x[4 * c + i] = __uint_as_float(u[i]);
        } else if constexpr (__is_same(T, __nv_bfloat16)) {
          x[8 * c + 2 * i] = bf16_lo(u[i]), x[8 * c + 2 * i + 1] = bf16_hi(u[i]);
        } else {
          const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&u[i]));
          x[8 * c + 2 * i] = f.x, x[8 * c + 2 * i + 1] = f.y;
        }
      }
    }
  }
};

// Groups of threads whose maxima give a threshold.
__device__ __forceinline__ int groups_log2(int n) { return n <= 16 ? 6 : n <= 32 ? 7 : 8; }

// A candidate, or a segment: value and beam in v; logit and token, or largest
// logit and number, in k.  The zero is none.
struct Entry {
  uint64_t v, k;
};
__device__ __forceinline__ bool above(const Entry &a, const Entry &b) {  // (as one number: no branches)
  return ((unsigned __int128)a.v << 64 | a.k) > ((unsigned __int128)b.v << 64 | b.k);
}
__device__ __forceinline__ Entry shfl_xor(const Entry &e, int o) {
  return {__shfl_xor_sync(0xffffffffu, e.v, o), __shfl_xor_sync(0xffffffffu, e.k, o)};
}
__device__ __forceinline__ Entry make_entry(float base, int beam, float logit, uint32_t number) {
  const float v = base + logit;
  if (!isfinite(v)) return {0, 0};
  return {(uint64_t)ordered(v) << 32 | (uint32_t)~beam, make_key(logit, number)};
}

// The best entries seen, in shared memory.
struct List {
  Entry *item;    // [kList]
  Entry *groups;  // [256]
  Entry *mark;    // the n-th of the groups
  int *count;
  int n;

  __device__ __forceinline__ int push(Entry key) {
    const int at = atomicAdd(count, 1);
    if (at < kList) item[at] = key;
    return at;
  }

  // The n-th largest of the groups' maxima, from each thread's maximum; none if
  // fewer groups have one.  A group's threads share the work of its rank.
  __device__ Entry nth_of_groups(Entry mine) {
    const int t = threadIdx.x, log2 = 8 - groups_log2(n), per = 1 << log2, G = kThreads >> log2;
    for (int o = 1; o < per; o *= 2) {
      const Entry other = shfl_xor(mine, o);
      if (above(other, mine)) mine = other;
    }
    const int g = t >> log2;
    if (mine.v == 0) mine.k = g;  // (groups without a candidate differ too: ranks are 0 .. G - 1)
    if ((t & (per - 1)) == 0) groups[g] = mine;
    __syncthreads();
    int rank = 0;
#pragma unroll 16
    for (int i = t & (per - 1); i < G; i += per) rank += above(groups[i], mine);
    for (int o = 1; o < per; o *= 2) rank += __shfl_xor_sync(0xffffffffu, rank, o);
    if (rank == n - 1 && (t & (per - 1)) == 0) *mark = mine.v ? mine : Entry{0, 0};
    __syncthreads();
    return *mark;
  }

  // Orders the list's n best at its start; what is left of it is dropped.
  // Returns the n-th (or none: the zero) as the threshold.
  __device__ Entry tighten() {
    const int t = threadIdx.x;
    __syncthreads();
    int len = min(*count, kList);
    while (len > max(64, 2 * n)) {
      // First drop what a threshold from its own groups of threads excludes.
      constexpr int kMost = (kList + kThreads - 1) / kThreads;
      Entry mine[kMost], best = {0, 0};
#pragma unroll
      for (int j = 0; j < kMost; ++j) {
        mine[j] = t + j * kThreads < len ? item[t + j * kThreads] : Entry{0, 0};
        if (above(mine[j], best)) best = mine[j];
      }
      const Entry least = nth_of_groups(best);
      if (t == 0) *count = 0;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kMost; ++j)
        if (t + j * kThreads < len && !above(least, mine[j])) push(mine[j]);
      __syncthreads();
      const int now = *count;
      if (now == len) break;  // (nothing to drop)
      __syncthreads();
      len = now;
    }
    if (len <= kThreads) {
      // 256, 128 or 64 entries: 1, 2 or 4 threads an entry.
      const int log2 = len <= 64 ? 2 : len <= 128 ? 1 : 0, per = 1 << log2, e = t >> log2;
      Entry mine{};
      int rank = 0;
      if (e < len) {
        mine = item[e];
#pragma unroll 8
        for (int i = t & (per - 1); i < len; i += per) rank += above(item[i], mine);
      }
      for (int o = 1; o < per; o *= 2) rank += __shfl_xor_sync(0xffffffffu, rank, o);
      __syncthreads();
      if (e < len && (t & (per - 1)) == 0 && rank < n) item[rank] = mine;
    } else {
      // (as many as no threshold of groups could drop)
      constexpr int kMost = (kList + kThreads - 1) / kThreads;
      Entry mine[kMost];
      int rank[kMost];
#pragma unroll
      for (int j = 0; j < kMost; ++j) {
        rank[j] = 0;
        mine[j] = t + j * kThreads < len ? item[t + j * kThreads] : Entry{0, 0};
        if (t + j * kThreads < len)
          for (int i = 0; i < len; ++i) rank[j] += above(item[i], mine[j]);
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kMost; ++j)
        if (t + j * kThreads < len && rank[j] < n) item[rank[j]] = mine[j];
    }
    if (t == 0) *count = min(len, n);
    __syncthreads();
    return len >= n ? item[n - 1] : Entry{0, 0};
  }
};

// A value that n of the threads' values (ordered, 0: none) reach, at most twice as
// many as that or so: the least of the warps' k-th largest, with 8 k >= n, the
// values dealt out evenly.  0: fewer have one.
__device__ __forceinline__ uint32_t reached_by(int n, uint32_t mine, uint32_t *shared) {
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  shared[t] = mine;
  __syncthreads();
  mine = shared[lane * kWarps + warp];
  uint32_t kth = 0;
  for (int k = 0; k < n; k += kWarps) {
    kth = __reduce_max_sync(0xffffffffu, mine);
    if (__ffs(__ballot_sync(0xffffffffu, mine == kth)) - 1 == lane) mine = 0;
  }
  __syncthreads();
  if (lane == 0) shared[warp] = kth;
  __syncthreads();
  uint32_t least = shared[0];
#pragma unroll
  for (int w = 1; w < kWarps; ++w) least = min(least, shared[w]);
  return least;
}

__device__ __forceinline__ float warp_max_f(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float warp_sum_f(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Segments under way ahead of the one at work.
template <typename T>
constexpr int kAhead = sizeof(T) == 4 ? 2 : 3;
template <typename T>
constexpr int kRing = (kAhead<T> + 1) * kThreads * kE * (int)sizeof(T);

// A block's share of a row: the segments' largest logits, and (m, sum).
template <typename T>
__device__ void reduce_slice(const SelectParams &p, int r, int sl, uint4 *ring, float *red) {
  constexpr uint32_t kSlot = kThreads * Raw<T>::kLoads * 16;
  const uint32_t ring0 = smem_u32(ring) + 16 * threadIdx.x, ring1 = ring0 + kRing<T>;
  const int warp = threadIdx.x >> 5, lane = lane_id();
  const int s1 = min(p.segments, (sl + 1) * p.slice_segments);
  const T *row = static_cast<const T *>(p.logits) + (int64_t)r * p.ld;
  float *tops = p.tops + (int64_t)r * p.segments;
  RunningSum sum;
  int next = sl * p.slice_segments + warp;
  uint32_t in = ring0, out = ring0;
  const auto start = [&] {
    if (p.vec && next < s1) Raw<T>::start(in, row, next * kSegment, p.vocab);
    next += kWarps;
    in = in + kSlot == ring1 ? ring0 : in + kSlot;
    asm volatile("cp.async.commit_group;\n" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < kAhead<T>; ++i) start();
  for (int s = sl * p.slice_segments + warp; s < s1; s += kWarps) {
    start();
    Raw<T> raw;
    if (p.vec) {
      asm volatile("cp.async.wait_group %0;\n" ::"n"(kAhead<T>) : "memory");
      raw.take(out);
    } else {
      raw.load(row, s * kSegment, p.vocab, false);
    }
    out = out + kSlot == ring1 ? ring0 : out + kSlot;
    float x[kE];
    raw.values(x);
    const float top = raw.top(x);
    const float most = warp_max(top);
    if (lane == 0) tops[s] = fmaxf(most, -INFINITY);
    sum.add(x, top);
  }
  asm volatile("cp.async.wait_all;\n" ::: "memory");
  // The threads' sums, to the block's reference.
  const float m = sum.m, wm = warp_max_f(m);
  if (lane == 0) red[warp] = wm;
  __syncthreads();
  float all = red[0];
#pragma unroll
  for (int w = 1; w < kWarps; ++w) all = fmaxf(all, red[w]);
  const float ws = warp_sum_f(sum.value() * exp_of(m - (all == -INFINITY ? 0.f : all)));
  if (lane == 0) red[kWarps + warp] = ws;
  __syncthreads();
  if (threadIdx.x == 0) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) s += red[kWarps + w];
    p.part[(int64_t)r * p.slices + sl] = make_float2(all, s);
  }
}

static_assert(kRing<__half> >= kList * (int)sizeof(Entry), "the merge's list takes the ring's place");

// The n best candidates of a batch entry.
template <typename T>
__device__ void merge(const SelectParams &p, int b, List &list, Entry *best_segments, float *base, bool *ended) {
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31, r0 = b * p.beams;
  const float *tops = p.tops + (int64_t)r0 * p.segments;
  // A warp looks at 128 segments of a beam at a time (a job), four a lane, the
  // next job's loads under way.
  constexpr int kU = 4;
  const int per_beam = (p.segments + 32 * kU - 1) / (32 * kU), jobs = p.beams * per_beam;
  float next[kU], top[kU];
  int k = 0, s0 = 0;  // of the job at work: beam, this lane's first segment
  const auto load_job = [&](int job) {
    const int beam = job / per_beam, s = (job - beam * per_beam) * 32 * kU + lane;
#pragma unroll
    for (int j = 0; j < kU; ++j)
      next[j] = job < jobs && s + 32 * j < p.segments ? __ldcg(tops + (int64_t)beam * p.segments + s + 32 * j) : -INFINITY;
  };
  const auto take_job = [&](int job) {
#pragma unroll
    for (int j = 0; j < kU; ++j) top[j] = next[j];
    k = job / per_beam;
    s0 = (job - k * per_beam) * 32 * kU + lane;
    load_job(job + kWarps);
    if (ended[k]) {  // one segment, whose logit is 0
#pragma unroll
      for (int j = 0; j < kU; ++j) top[j] = s0 + 32 * j == 0 ? 0.f : -INFINITY;
    }
  };
  load_job(warp);
  {
    float2 q = make_float2(-INFINITY, 0.f);
    float score = 0.f;
    bool over = false;
    const auto load_beam = [&](int beam) {
      if (beam >= p.beams) return;
      score = p.scores[r0 + beam];
      over = p.ended && p.ended[r0 + beam];
      q = lane < p.slices ? __ldcg(p.part + (int64_t)(r0 + beam) * p.slices + lane) : make_float2(-INFINITY, 0.f);
    };
    load_beam(warp);
    for (int beam = warp; beam < p.beams; beam += kWarps) {  // a warp a beam
      const float plus = score;
      const bool done = over;
      float m = q.x, s = q.y;  // a lane's blocks, in turn
      load_beam(beam + kWarps);
      for (int i = lane + 32; i < p.slices && !done; i += 32) {
        const float2 more = __ldcg(p.part + (int64_t)(r0 + beam) * p.slices + i);
        const float now = fmaxf(m, more.x), ref = now == -INFINITY ? 0.f : now;
        s = s * exp_of(m - ref) + more.y * exp_of(more.x - ref);
        m = now;
      }
      const float most = warp_max_f(m);
      s = warp_sum_f(s * exp_of(m - (most == -INFINITY ? 0.f : most)));
      if (lane == 0) base[beam] = done ? plus : plus - (most + logf(s)), ended[beam] = done;
    }
  }
  if (t == 0) *list.count = 0;
  __syncthreads();

  // The n best segments, of those whose value reaches a first threshold.
  constexpr int kHeld = 3;  // jobs whose values stay in registers
  const bool held = jobs <= kHeld * kWarps;
  float keep[kHeld][kU], best_v = -INFINITY;
  const auto look = [&](float plus) {
#pragma unroll
    for (int j = 0; j < kU; ++j) {
      const float v = plus + top[j];
      if (v < INFINITY) best_v = fmaxf(best_v, v);
    }
  };
  Entry least;
  const auto find = [&](float bar) {
#pragma unroll
    for (int j = 0; j < kU; ++j)
      if (base[k] + top[j] >= bar) {
        const Entry e = make_entry(base[k], k, top[j], s0 + 32 * j);
        if (e.v && !above(least, e)) list.push(e);
      }
  };
  if (held) {
#pragma unroll
    for (int h = 0; h < kHeld; ++h) {
      if (warp + h * kWarps >= jobs) break;
      take_job(warp + h * kWarps);
#pragma unroll
      for (int j = 0; j < kU; ++j) keep[h][j] = top[j];
      look(base[k]);
    }
  } else {
    for (int job = warp; job < jobs; job += kWarps) {
      take_job(job);
      look(base[k]);
    }
  }
  least = {(uint64_t)reached_by(p.n, best_v > -INFINITY ? ordered(best_v) : 0, reinterpret_cast<uint32_t *>(list.groups))
               << 32,
           0};
  while (true) {
    const float bar = least.v ? unordered((uint32_t)(least.v >> 32)) : -INFINITY;
    if (held) {
#pragma unroll
      for (int h = 0; h < kHeld; ++h) {
        if (warp + h * kWarps >= jobs) break;
        k = (warp + h * kWarps) / per_beam;
        s0 = (warp + h * kWarps - k * per_beam) * 32 * kU + lane;
#pragma unroll
        for (int j = 0; j < kU; ++j) top[j] = keep[h][j];
        find(bar);
      }
    } else {
      load_job(warp);
      for (int job = warp; job < jobs; job += kWarps) {
        take_job(job);
        find(bar);
      }
    }
    __syncthreads();
    const bool over = *list.count > kList;
    const Entry nth = list.tighten();
    if (above(nth, least)) least = nth;
    if (!over) break;
    // More than the list takes: the n-th of those it took is a higher threshold.
    if (t == 0) *list.count = 0;
    __syncthreads();
  }

  // The candidates of those segments.
  const int chosen = *list.count;
  if (t < chosen) best_segments[t] = list.item[t];
  __syncthreads();
  if (t == 0) *list.count = 0;  // (each thread has read it)
  __syncthreads();
  // (As a candidate's, the threshold's token is the last of its segment.)
  least.k = (least.k & ~0xFFFFFFFFull) | (uint32_t)~((key_token(least.k) + 1) * kSegment - 1);
  // This lane's logits of the c-th segment, of a beam and from token v (an ended
  // beam: a logit of 0 in place 0).
  const auto load_segment = [&](int c, Raw<T> &raw, int &beam, int &v) {
    beam = v = 0;
    if (c >= chosen) return;
    const Entry seg = best_segments[c];
    beam = (int)~(uint32_t)seg.v;
    v = (int)key_token(seg.k) * kSegment;
    if (!ended[beam]) raw.load(static_cast<const T *>(p.logits) + (int64_t)(r0 + beam) * p.ld, v, p.vocab, p.vec);
  };
  const auto values_of = [&](int c, const Raw<T> &raw, int beam, float(&x)[kE]) {
    if (c < chosen && !ended[beam]) {
      raw.values(x);
    } else {
#pragma unroll
      for (int i = 0; i < kE; ++i) x[i] = -INFINITY;
      if (c < chosen && lane == 0) x[0] = 0.f;
    }
  };
  Raw<T> ahead;
  int next_k, next_v;
  if (p.beams * p.segments <= 2 * p.n) {
    // (Few segments, small vocabularies: most of a segment may pass.)  A threshold
    // from the threads' best candidates: 4 beams of 1000 tokens, n = 8, 7.6 us, without
    // this 10.6; 16 of 250, n = 32, 11.9 and 24.4; but 8 of 4000, n = 16, 9.4 and 8.5.
    float best = -INFINITY;
    for (int c = warp; c < chosen; c += kWarps) {
      float x[kE];
      load_segment(c, ahead, next_k, next_v);
      values_of(c, ahead, next_k, x);
#pragma unroll
      for (int i = 0; i < kE; ++i) {
        const float v = base[next_k] + x[i];
        if (v < INFINITY) best = fmaxf(best, v);
      }
    }
    const uint32_t reached = reached_by(p.n, best > -INFINITY ? ordered(best) : 0, reinterpret_cast<uint32_t *>(list.groups));
    const Entry nth = {(uint64_t)reached << 32, 0};
    if (above(nth, least)) least = nth;
  }
  // The candidates that reach the threshold, straight away: about as many as
  // there are segments.  The next segment's loads are under way.
  const float bar = least.v ? unordered((uint32_t)(least.v >> 32)) : -INFINITY;
  load_segment(warp, ahead, next_k, next_v);
  for (int c = warp; c < chosen; c += kWarps) {
    float x[kE];
    k = next_k;
    const int v = next_v;
    values_of(c, ahead, k, x);
    load_segment(c + kWarps, ahead, next_k, next_v);
    const float plus = base[k];
    uint32_t pass = 0;
#pragma unroll
    for (int i = 0; i < kE; ++i) pass |= (uint32_t)(plus + x[i] >= bar) << i;
    while (__any_sync(0xffffffffu, pass)) {  // (few: a value is found again by its number)
      const int i = __ffs(pass) - 1;
      float l = 0.f;
#pragma unroll
      for (int j = 0; j < kE; ++j) l = i == j ? x[j] : l;
      if (pass) {
        pass &= pass - 1;
        const Entry e = make_entry(plus, k, l, v + Raw<T>::place(i));
        if (e.v && !above(least, e)) list.push(e);
      }
    }
  }
  __syncthreads();
  if (*list.count > kList) {
    // More than the list takes (a segment that holds many of the best): again,
    // eight segments, one a warp, at a time, with a threshold that rises.
    __syncthreads();
    if (t == 0) *list.count = 0;
    for (int c = 0; c < chosen; c += kWarps) {
      float x[kE];
      int v;
      load_segment(c + warp, ahead, k, v);
      values_of(c + warp, ahead, k, x);
      const float plus = base[k];
      Entry top_entry = {0, 0};
#pragma unroll
      for (int i = 0; i < kE; ++i) {
        const Entry e = make_entry(plus, k, x[i], v + Raw<T>::place(i));
        if (above(e, top_entry)) top_entry = e;
      }
      // (At most n groups' 16 * 256 / G candidates reach it: 1024.)
      const Entry mark = list.nth_of_groups(top_entry);
      if (above(mark, least)) least = mark;
#pragma unroll
      for (int i = 0; i < kE; ++i) {
        const Entry e = make_entry(plus, k, x[i], v + Raw<T>::place(i));
        if (e.v && !above(least, e)) list.push(e);
      }
      const Entry nth = list.tighten();
      if (above(nth, least)) least = nth;
    }
  } else {
    list.tighten();
  }
  const int len = *list.count;
  for (int i = t; i < p.n; i += kThreads) {
    const int64_t o = (int64_t)b * p.n + i;
    const bool there = i < len;
    const Entry e = there ? list.item[i] : Entry{0, 0};
    p.out_scores[o] = there ? unordered((uint32_t)(e.v >> 32)) : -INFINITY;
    k = there ? (int)~(uint32_t)e.v : -1;
    p.out_parents[o] = k;
    p.out_tokens[o] = !there ? -1 : ended[k] ? p.end_token : (int32_t)key_token(e.k);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 ? 3 : 4) beam_select_kernel(const SelectParams p) {
  extern __shared__ uint4 smem16[];
  __shared__ Entry groups[256], mark, best_segments[ARCHEAD_BEAM_MAX_OUT];
  __shared__ float red[ARCHEAD_BEAM_MAX_BEAMS];
  __shared__ bool ended[ARCHEAD_BEAM_MAX_BEAMS];
  __shared__ int count, before;
  const int r = blockIdx.x / p.slices, sl = blockIdx.x - r * p.slices, b = r / p.beams;
  if (!(p.ended && p.ended[r])) reduce_slice<T>(p, r, sl, smem16, red);
  // (One thread's release and acquire order the whole block's stores and loads: what
  // the barriers put before the one and behind the other comes with it.  Full fences
  // around a relaxed addition took 0.3 us more.)
  __syncthreads();
  if (threadIdx.x == 0) {
    asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;\n" : "=r"(before) : "l"(p.counters + b) : "memory");
  }
  __syncthreads();
  if (before != p.beams * p.slices - 1) return;
  if (threadIdx.x == 0) p.counters[b] = 0;
  List list = {reinterpret_cast<Entry *>(smem16), groups, &mark, &count, p.n};
  merge<T>(p, b, list, best_segments, red, ended);
}

}  // namespace

// Blocks of a row.  Up to one row a multiprocessor: about two blocks a
// multiprocessor in all, whose starts and ends then overlap, and no fewer than one
// and a half (128 rows of 151936 in fp32: two a row 22.0 us, three 23.7, one 23.9;
// 32 rows in bf16: nine 10.2 us, four 10.9, sixteen 11.3).  More rows: blocks of
// some 49000 logits, many enough that rows that have ended leave no multiprocessor
// idle (160 rows of 262144 in bf16, 64 of them ended: five a row 21.4 us, two 26.0,
// one 32.9, and with none ended 28.6, 27.2, 33.0; 512 rows of 151936, 128 of them
// ended: three 33.1 us, two 35.8, six 36.2; 300 rows of 20000 in fp32, 60 of them
// ended: one 13.2 us, two 15.0).
constexpr int kSliceSegments = 96;
static int beam_slices(int64_t rows, int64_t segments, int sm_count) {
  const int64_t most = (segments + kWarps - 1) / kWarps;
  int64_t n = 2 * sm_count / rows;
  if (2 * rows * n < 3 * sm_count) ++n;
  if (rows > sm_count) n = std::max<int64_t>(1, (segments + kSliceSegments / 2) / kSliceSegments);
  return (int)std::min(most, n);
}

// Scratch: counters of the batch entries (at most one a row), the blocks' sums, the segments' largest logits.
static size_t up(size_t bytes) { return (bytes + 255) / 256 * 256; }
size_t beam_counter_bytes(int64_t max_rows) { return up((size_t)max_rows * sizeof(int)); }
size_t beam_scratch_bytes(int64_t max_rows, int64_t max_vocab, int sm_count) {
  const size_t segments = (size_t)((max_vocab + kSegment - 1) / kSegment);
  const size_t blocks = (size_t)max_rows * (segments / kSliceSegments + 1) + 4 * sm_count;
  return beam_counter_bytes(max_rows) + up(blocks * sizeof(float2)) +
         (size_t)max_rows * segments * sizeof(float);
}

cudaError_t launch_beam_select(SelectParams p, int dtype, void *ws, int64_t max_rows, int sm_count, cudaStream_t s) {
  p.segments = (p.vocab + kSegment - 1) / kSegment;
  p.slices = beam_slices(p.rows, p.segments, sm_count);
  p.slice_segments = (p.segments + p.slices - 1) / p.slices;
  char *at = static_cast<char *>(ws);
  p.counters = reinterpret_cast<int *>(at);
  at += beam_counter_bytes(max_rows);
  p.part = reinterpret_cast<float2 *>(at);
  p.tops = reinterpret_cast<float *>(at + up((size_t)p.rows * p.slices * sizeof(float2)));
  const int size = dtype == ARCHEAD_DTYPE_FP32 ? 4 : 2;
  p.vec = (reinterpret_cast<uintptr_t>(p.logits) & 15) == 0 && p.ld * size % 16 == 0;
  const unsigned grid = (unsigned)p.rows * p.slices;
  const auto run = [&](auto kern, int smem) {
    cudaError_t e = opt_in_smem(reinterpret_cast<const void *>(kern), smem);
    if (e != cudaSuccess) return e;
    kern<<<grid, kThreads, smem, s>>>(p);
    return cudaGetLastError();
  };
  return dtype == ARCHEAD_DTYPE_FP32   ? run(beam_select_kernel<float>, kRing<float>)
         : dtype == ARCHEAD_DTYPE_FP16 ? run(beam_select_kernel<__half>, kRing<__half>)
                                       : run(beam_select_kernel<__nv_bfloat16>, kRing<__nv_bfloat16>);
}

}  // namespace archead
