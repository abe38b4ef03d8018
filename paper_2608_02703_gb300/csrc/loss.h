// Internal definitions of the dense head's cross entropy and its gradient
// (linear_ce.cu, linear_ce_rows.cu, loss_api.cu).
//
// Tokens that count (a target, and in the gradient a factor that is not zero) are
// gathered to the front, so that the products do no work for the others and what
// stands in them reaches no sum.  How many there are is known on the device only:
// header->count.  With one tile of tokens, where no work would be saved, they stay
// where they are if x's rows start on 16 bytes: the logits' products need not wait
// for the gathering then (count is the number of tokens, and zeros stand in the copy of x
// for those that do not count).
//
// The vocabulary is cut into tiles of 256 rows; the gradient takes them in pieces of
// some tiles, of which it holds G (tokens x piece, 16 bits) in scratch.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "archead.h"

namespace archead {

constexpr int kCeTile = 256;    // tokens, vocabulary rows or columns of a unit
constexpr int kCeStep = 64;     // of the summed dimension a stage
constexpr int kCeParts = 2;     // partial sums of exponentials a tile and token

struct CeHeader {
  int count;              // tokens that count
  float scale, unscale;   // a power of two that the factors are held times, and its inverse
};

// Places in a loss's scratch.
struct CeScratch {
  CeHeader *header;
  int *place;       // [tokens] row of a token among those that count, or -1
  int *target;      // [rows] target, or -1 where it is not a vocabulary row
  float *lse;       // [rows]
  float *factor;    // [rows] grad_ce times header->scale
  float *rest;      // [rows] what rounding took of G at the target (G in one part)
  uint16_t *x;      // panels of 64 columns: [x_pitch / 64][rows][64]
  float2 *part;     // [CeParts][rows]
  float *tlogit;    // [rows]
  uint16_t *G;      // panels of 64 columns of a piece: [tiles * 4][rows][64]
  float *dx;        // [splits][rows][dx_pitch]
};

}  // namespace archead

struct archead_loss {
  int device = 0;
  int sm_count = 0;
  int clusters = 0;  // pairs of blocks that run at once
  int64_t max_tokens = 0, max_vocab = 0, max_hidden = 0;
  bool gradient = false;
  void *ws = nullptr;
  int64_t ws_bytes = 0, g_bytes = 0, dx_bytes = 0;
  archead::CeScratch at{};
  int *err = nullptr;
  int64_t wait_budget = 0;
};

namespace archead {

struct CeRowsParams {
  const void *x;
  const int32_t *targets;
  const float *lse, *grad;  // NULL: the loss alone
  int32_t ignore;
  int64_t M, ldx, V, rows;
  int d, x_pitch, rows_per_block;
  int half;          // the gradient's copy of x stands there again from row 32 on, where it is 32 (see ce_half)
  bool direct;       // one tile of tokens, whose logits are computed from x as it lies: every token keeps its row
  CeScratch at;
};
cudaError_t launch_ce_gather(const CeRowsParams &p, cudaStream_t s);

// Partial sums of a token: by tile of the vocabulary or, where all tokens that count are in one tile, by
// pair of blocks.
struct CeParts {
  int by_tile, by_pair;
};
// The most partial sums of all tokens together (units of fewer than 256 columns, 64 at least, are taken where there
// are at most four of 256 for each pair).
inline int64_t ce_most_parts(int64_t rows, int64_t tiles, int64_t clusters) {
  const int64_t by_tile = kCeParts * rows * tiles, small = kCeParts * kCeTile * 16 * clusters;
  return by_tile > small ? by_tile : small;
}

struct CeFinishParams {
  const int32_t *targets;
  float *ce, *lse;  // lse may be NULL
  int32_t ignore;
  int64_t M, V;
  CeParts parts;
  int64_t rows;  // pitch of the partial sums
  CeScratch at;
  int *err;
};
cudaError_t launch_ce_finish(const CeFinishParams &p, cudaStream_t s);

struct CeDxParams {
  void *dx;
  const void *w;
  int64_t M, ld, ldw, rows;
  int d, pitch, splits;
  int half;  // see CeCall
  bool fp16, vec;
  CeScratch at;
};
cudaError_t launch_ce_dx(const CeDxParams &p, cudaStream_t s);

// What the products' kernels are given (linear_ce.cu).
struct CeCall {
  const archead_loss *loss;
  const void *x, *w;
  int64_t ldx;
  bool direct;   // (see CeRowsParams)
  bool fp16;
  int64_t M, V, d, ldw;
  int64_t rows;  // M rounded up to tiles
  int x_pitch;
  void *dw;      // NULL: not wanted
  int64_t lddw;
  int accumulate;
  bool want_dx;
  int half;      // rows of G's first part, where it has two (see ce_half), else 0
  int splits, dx_pitch;
};
// Up to 64 tokens G is held in two parts of 16 bits, the value and what its rounding took, which is as good as 32 bits:
// the second has the rows behind the first, which a block's half of A has room for, so that the products with W are the
// same and dW takes one more step of 64 rows (up to 32 tokens none).  4 tokens x 4096 x 512, loss and gradients 26.9 ->
// 27.8 us, 64 x 262144 x 2560 900 -> 940; with G in 16 bits dx and dW stood at 1.4 times what their own rounding leaves.
// More tokens would take twice the MMAs, which bound those calls: there G is rounded to 16 bits.  Half of what a row of G
// weighs stands at its target; what rounding took there goes into dx by itself, as a multiple of the target's row of W (M d
// products).
inline int ce_half(int64_t M) { return M <= 32 ? 32 : M <= 64 ? 64 : 0; }
int64_t ce_piece_tiles(const archead_loss *l, const CeCall &c);  // tiles of a piece
int ce_dx_splits(const archead_loss *l, int64_t M, int64_t V, int64_t d, bool want_dw);
cudaError_t ce_clusters(int *clusters);  // pairs of blocks that the current device runs at once
cudaError_t launch_ce_logits(const CeCall &c, CeParts *parts, cudaStream_t s);
cudaError_t launch_ce_gradient(const CeCall &c, cudaStream_t s);

// Tensor map of 16-bit elements [rows][cols], rows `pitch` elements apart: box 64
// columns x box_rows, 128-byte swizzle, zeros out of bounds.
bool make_tma_map_16(CUtensorMap *map, const void *base, int64_t rows, int64_t cols, int64_t pitch, int box_rows);
// The same of fp32 [rows][cols]: box 32 columns x box_rows.
bool make_tma_map_f32(CUtensorMap *map, const void *base, int64_t rows, int64_t cols, int box_rows);

}  // namespace archead
