// Internal definitions of the INT8 product (int8_*.cu): the weight handle,
// its device layout and the kernel launchers.
//
//  Codes, "fragment-native".  The channels (N padded with zero rows to N_PAD,
//  a multiple of 128) are cut into strips of 16, K (padded with zero codes to
//  K_PAD, a multiple of 128) into blocks of 32.  Block (strip, kb) is 512
//  bytes: [lane 0..31][word j 0..3] of 32-bit words, a strip's blocks following
//  one another.  Word j of lane (gq = lane/4, cq = lane%4) holds row 16 strip +
//  gq + 8 (j & 1), columns 32 kb + 8 cq + 4 (j >> 1) + 0..3, lowest first: the
//  four registers of an m16n8k32 A fragment, if the columns of a block are
//  taken in that order (any order serves a sum, if both operands share it).
//  The same words, two codes at a time, are the A fragments of two m16n8k16
//  steps.
//    byte offset = ((strip * KB + kb) * 32 + lane) * 16 + 4 j,   KB = K_PAD/32
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
  void *ws = nullptr;
  size_t ws_bytes = 0;
  int64_t owned_bytes = 0;
  int64_t wait_budget = 0;
};

namespace archead {

constexpr int kI8Strip = 16;        // channels per strip
constexpr int kI8Block = 32;        // K per block
constexpr int kI8BlockBytes = 512;  // codes of a block
constexpr int kI8PadN = 128, kI8PadK = 128;
constexpr int kI8MaxK = (1 << 17) - 1;

// Output rows: y[m][n] at y + (m * ld + n) elements.
struct I8Out {
  void *y;
  int64_t ld;
  int dtype;  // archead_dtype
};

cudaError_t launch_int8_layout(const archead_int8_weight *w, const int8_t *codes, cudaStream_t s);

// Quantisation of M rows of K elements.  Codes go to rows of ldc bytes, of
// which [K, k_fill) are set to zero.
cudaError_t launch_int8_quantize(const void *x, int dtype, int64_t M, int64_t K, int64_t ldx, int8_t *codes,
                                 int64_t ldc, int64_t k_fill, float *scales, cudaStream_t s);
// Token codes [M][K] into rows of K_pad bytes, zero beyond K.
cudaError_t launch_int8_pad(const int8_t *codes, int64_t M, int K, int K_pad, int8_t *out, cudaStream_t s);
// Product of padded token codes with the weight.
cudaError_t launch_int8_product(const archead_int8_weight *w, const int8_t *x, const float *x_scales, int64_t M,
                                I8Out out, cudaStream_t s);

}  // namespace archead
