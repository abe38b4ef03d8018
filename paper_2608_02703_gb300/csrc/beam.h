// Internal definitions of beam search (beam_*.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "archead.h"

struct archead_beam {
  int device = 0;
  int sm_count = 0;
  int64_t max_rows = 0, max_vocab = 0;
  int max_out = 0;
  void *ws = nullptr;
};

namespace archead {

// A row of logits is cut into slices (a block each) of segments; a slice leaves
// (m, sum of exp(l - m)), a segment its largest logit.
struct SelectParams {
  const void *logits;
  int64_t ld;
  int rows, beams, vocab, n;
  const float *scores;
  const uint8_t *ended;  // may be NULL
  int32_t end_token;
  int segments, slices, slice_segments;
  bool vec;         // rows start on 16 bytes
  int *counters;    // [batch] blocks that have finished, zero between calls
  float2 *part;     // [rows][slices]
  float *tops;      // [rows][segments]
  float *out_scores;
  int32_t *out_parents, *out_tokens;
};

// Scratch of the largest selection; its counters, which come first, start as zeros.
size_t beam_scratch_bytes(int64_t max_rows, int64_t max_vocab, int sm_count);
size_t beam_counter_bytes(int64_t max_rows);

cudaError_t launch_beam_select(SelectParams p, int dtype, void *ws, int64_t max_rows, int sm_count, cudaStream_t s);

// Division of numbers below 2^31 by a constant d: q = (n m) >> (31 + l), with l =
// ceil(log2 d) and m = floor(2^(31 + l) / d) + 1 < 2^32 (m = 0: d is 1).
struct Divisor {
  uint32_t d, m, shift;
};

constexpr int kReorderStates = 48;  // states of one launch
struct ReorderState {
  const char *src;
  char *dst;
  int64_t outer_stride, row_stride, inner_stride;
  uint32_t total;      // vectors of one row, below 2^31
  Divisor chunk, per;  // vectors of a chunk, of all inner chunks
  int width;           // bytes of a vector
  int first_tile;      // tiles of the states before this one
};
struct ReorderParams {
  ReorderState st[kReorderStates];
  const int32_t *parents;
  int64_t batch;
  int beams, count, tiles, place;
};
cudaError_t launch_beam_reorder(const ReorderParams &p, cudaStream_t s);
int reorder_vector_bytes(int beams);  // most bytes a thread moves of each row
int reorder_tile();                   // vectors of a row that a block moves

}  // namespace archead
