// Internal definitions of the INT8 product (int8_*.cu): the weight handle,
// its device layout and the kernel launchers.
//
//  Codes, "fragment-native".  The channels (N padded with zero rows to N_PAD,
//  a multiple of 128) are cut into tiles of 128 and these into strips of 16, K
//  (padded with zero codes to K_PAD, a multiple of 128) into stages of 128 and
//  these into blocks of 32.  A (tile, stage) is 16 KB, one bulk copy: [strip
//  0..7][block 0..3][lane 0..31][word j 0..3] of 32-bit words.  Word j of lane
//  (gq = lane/4, cq = lane%4) holds row 16 strip + gq + 8 (j & 1) of the tile,
//  columns 8 cq + 4 (j >> 1) + 0..3 of the block, lowest first: the four
//  registers of an m16n8k32 A fragment, if the columns of a block are taken in
//  that order (any order serves a sum, if both operands share it).  The same
//  words, two codes at a time, are the A fragments of two m16n8k16 steps.
//    byte offset = ((((tile * KC + stage) * 8 + strip) * 4 + block) * 32 + lane) * 16 + 4 j,   KC = K_PAD/128
//
//  Token codes, widened to fp16 for the tensor-memory kernel: [M][K_PAD] in
//  the same order of K.  Of the eight columns 8 cq + 0..7 of a block, pair i
//  (columns 8 cq + 2 i, + 1) is word 4 i + cq of the block's 16 words: k16 step
//  i >> 1, fragment registers 2 (i & 1) and its neighbour.
//
//  Scales: fp32 [N_PAD], zero on padding rows.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "archead.h"

struct archead_int8_weight {
  int device = 0;
  int sm_count = 0;
  int64_t N = 0, N_pad = 0;
  int K = 0, K_pad = 0;
  uint8_t *codes = nullptr;
  float *scales = nullptr;
  int *err = nullptr;
  int clusters[2][4] = {};  // of 2^i blocks of the split tensor-memory kernels (64, 128 tokens) that run at once
  void *ws = nullptr;
  size_t ws_bytes = 0;
  bool ws_captured = false;  // a captured call holds addresses of ws: it is kept until the weight goes
  struct Kept {
    void *ws;
    Kept *next;
  } *kept = nullptr;
  int64_t reserved_tokens = 0;  // every AUTO call of up to so many fits
  int64_t owned_bytes = 0;
  int64_t wait_budget = 0;
};

namespace archead {

constexpr int kI8Strip = 16;  // channels per strip
constexpr int kI8Block = 32;  // K per block
constexpr int kI8PadN = 128, kI8PadK = 128;  // a tile's channels, a stage's K
constexpr int kI8MaxK = (1 << 17) - 1;

// Output rows: y[m][n] at y + (m * ld + n) elements.
struct I8Out {
  void *y;
  int64_t ld;
  int dtype;  // archead_dtype
};

cudaError_t launch_int8_layout(const archead_int8_weight *w, const int8_t *codes, cudaStream_t s);

// Quantisation of M rows of K elements.  Codes go to rows of ldc codes, of
// which [K, k_fill) are set to zero; wide: to rows of k_fill widened codes
// (k_fill a multiple of 128).
cudaError_t launch_int8_quantize(const void *x, int dtype, int64_t M, int64_t K, int64_t ldx, void *codes, bool wide,
                                 int64_t ldc, int64_t k_fill, float *scales, cudaStream_t s);
// Token codes [M][K] into rows of K_pad codes (wide: widened), zero beyond K.
cudaError_t launch_int8_pad(const int8_t *codes, int64_t M, int K, int K_pad, void *out, bool wide, cudaStream_t s);
// Warp-level kernel.  The tokens are activations of type `dtype`, which it
// quantises (x_scales NULL; int8_decode_quantizes), or codes; rows ldx elements
// apart.  More tokens than fit take more launches.  If not even
// eight tokens' codes fit into shared memory, the codes have to be padded rows.
cudaError_t launch_int8_decode(const archead_int8_weight *w, const void *x, int dtype, int64_t ldx,
                               const float *x_scales, int64_t M, I8Out out, cudaStream_t s);
// Most activations that every block quantises for itself (4 tokens of 4096:
// 6.5 us for 4096 channels, 7.6 with a launch of its own; 8 tokens: 8.7 and 7.4).
constexpr int64_t kI8FusedQuantize = 16384;
bool int8_decode_quantizes(int64_t M, int K, int K_pad);
bool int8_decode_fits(int64_t M, int K_pad);  // all M tokens in one launch

// Tensor-memory kernel: how a product of M tokens is cut.
struct I8GemmPlan {
  int NT = 0, nt = 0, ks_log2 = 0;
  int64_t num_mt = 0, units = 0;
};
cudaError_t int8_gemm_room(archead_int8_weight *w);  // fills w->clusters
I8GemmPlan int8_gemm_plan(const archead_int8_weight *w, int64_t M);
// x: widened token codes [M][K_pad].
cudaError_t launch_int8_gemm(const archead_int8_weight *w, const I8GemmPlan &f, const uint16_t *x,
                             const float *x_scales, int64_t M, I8Out out, cudaStream_t s);

}  // namespace archead
