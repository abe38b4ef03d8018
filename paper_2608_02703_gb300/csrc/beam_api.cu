// C entry points of beam search (include/archead.h): argument checks and launches.
#include <algorithm>
#include <new>

#include "beam.h"
#include "status.h"

using namespace archead;

namespace {

// The largest power of two up to 16 that divides v.
int64_t low_bits(int64_t v) { return v == 0 ? 16 : std::min<int64_t>(v & -v, 16); }

Divisor divisor(uint32_t d) {
  if (d == 1) return {1, 0, 0};
  uint32_t l = 0;
  while (((uint64_t)1 << l) < d) ++l;
  return {d, (uint32_t)(((uint64_t)1 << (31 + l)) / d + 1), l - 1};
}

// Launches of a reordering, filled state by state.  In place and into another
// buffer are launches of their own.
struct Reordering {
  ReorderParams p;
  int64_t tiles = 0;
  cudaStream_t stream;
  cudaError_t failed = cudaSuccess;

  void flush() {
    if (p.count > 0 && failed == cudaSuccess) {
      p.tiles = (int)tiles;
      failed = launch_beam_reorder(p, stream);
    }
    p.count = 0;
    tiles = 0;
  }

  // `bytes` of each of outer x inner chunks; states whose vectors of a row pass
  // 2^31 in parts.
  void add(const char *src, char *dst, int64_t outer, int64_t inner, int64_t bytes, const archead_beam_state &a,
           int64_t width) {
    const int64_t chunk = bytes / width;
    if ((__int128)outer * inner * chunk >= (int64_t)1 << 31) {
      const auto both = [&](int64_t step, int64_t o0, int64_t i0, int64_t b0, int64_t o1, int64_t i1, int64_t b1) {
        add(src, dst, o0, i0, b0, a, width);
        add(src + step, dst + step, o1, i1, b1, a, width);
      };
      if (outer > 1) return both(outer / 2 * a.outer_stride, outer / 2, inner, bytes, outer - outer / 2, inner, bytes);
      if (inner > 1) return both(inner / 2 * a.inner_stride, 1, inner / 2, bytes, 1, inner - inner / 2, bytes);
      const int64_t half = chunk / 2 * width;
      return both(half, 1, 1, half, 1, 1, bytes - half);
    }
    const int64_t total = outer * inner * chunk, n = (total + reorder_tile() - 1) / reorder_tile();
    const int place = dst == src;
    if (p.count == kReorderStates || tiles + n > 0x7fffffff || (p.count > 0 && p.place != place)) flush();
    ReorderState &st = p.st[p.count++];
    st.src = src;
    st.dst = dst;
    st.outer_stride = a.outer_stride;
    st.row_stride = a.row_stride;
    st.inner_stride = a.inner_stride;
    st.total = (uint32_t)total;
    st.chunk = divisor((uint32_t)chunk);
    st.per = divisor((uint32_t)(inner * chunk));
    st.width = (int)width;
    st.first_tile = (int)tiles;
    p.place = place;
    tiles += n;
  }
};

}  // namespace

extern "C" {

archead_status archead_beam_create(int64_t max_rows, int64_t max_vocab, int max_out, archead_beam **out) {
  if (!out) return ARCHEAD_ERR_INVALID_ARG;
  *out = nullptr;
  if (max_rows < 1 || max_vocab < 1 || max_out < 1 || max_out > ARCHEAD_BEAM_MAX_OUT) return ARCHEAD_ERR_INVALID_ARG;
  if (max_rows > 1 << 20 || max_vocab > 1 << 30) return ARCHEAD_ERR_UNSUPPORTED;
  archead_beam *b = new (std::nothrow) archead_beam();
  if (!b) return ARCHEAD_ERR_OOM;
  b->max_rows = max_rows;
  b->max_vocab = max_vocab;
  b->max_out = max_out;
  cudaError_t e = cudaGetDevice(&b->device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&b->sm_count, cudaDevAttrMultiProcessorCount, b->device);
  if (e == cudaSuccess) e = cudaMalloc(&b->ws, beam_scratch_bytes(max_rows, max_vocab, b->sm_count));
  // (In a stream of its own, waited for: any stream may use the handle first.)
  cudaStream_t s = nullptr;
  if (e == cudaSuccess) e = cudaStreamCreateWithFlags(&s, cudaStreamNonBlocking);
  if (e == cudaSuccess) e = cudaMemsetAsync(b->ws, 0, beam_counter_bytes(max_rows), s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (s) cudaStreamDestroy(s);
  if (e != cudaSuccess) {
    const archead_status st = status_of(e);
    if (b->ws) cudaFree(b->ws);
    delete b;
    return st;
  }
  *out = b;
  return ARCHEAD_OK;
}

void archead_beam_destroy(archead_beam *b) {
  if (!b) return;
  cudaSetDevice(b->device);
  cudaDeviceSynchronize();
  cudaFree(b->ws);
  delete b;
}

archead_status archead_beam_select(archead_beam *beam, const void *logits, archead_dtype dtype, int64_t batch,
                                   int beams, int64_t vocab, int64_t ld, const float *scores, const uint8_t *ended,
                                   int32_t end_token, int n_out, float *out_scores, int32_t *out_parents,
                                   int32_t *out_tokens, void *stream) {
  if (!beam || !is_dtype(dtype) || batch < 0 || beams < 1 || beams > ARCHEAD_BEAM_MAX_BEAMS || vocab < 1 ||
      ld < vocab || n_out < 1)
    return ARCHEAD_ERR_INVALID_ARG;
  if (batch == 0) return ARCHEAD_OK;
  if (!logits || !scores || !out_scores || !out_parents || !out_tokens || !is_aligned(logits, dtype_bytes(dtype)) ||
      !is_aligned(scores, 4) || !is_aligned(out_scores, 4) || !is_aligned(out_parents, 4) || !is_aligned(out_tokens, 4))
    return ARCHEAD_ERR_INVALID_ARG;
  if (batch > beam->max_rows / beams || vocab > beam->max_vocab || n_out > beam->max_out) {
    set_last_error_message("the selection is larger than its scratch was created for");
    return ARCHEAD_ERR_UNSUPPORTED;
  }
  AH_TRY(cudaSetDevice(beam->device));
  SelectParams p{};
  p.logits = logits;
  p.ld = ld;
  p.rows = (int)(batch * beams);
  p.beams = beams;
  p.vocab = (int)vocab;
  p.n = n_out;
  p.scores = scores;
  p.ended = ended;
  p.end_token = end_token;
  p.out_scores = out_scores;
  p.out_parents = out_parents;
  p.out_tokens = out_tokens;
  AH_TRY(launch_beam_select(p, dtype, beam->ws, beam->max_rows, beam->sm_count, static_cast<cudaStream_t>(stream)));
  return ARCHEAD_OK;
}

archead_status archead_beam_reorder(const archead_beam_state *states, int count, const int32_t *parents, int64_t batch,
                                    int beams, int64_t length, void *stream) {
  if (count < 0 || batch < 0 || beams < 1 || beams > ARCHEAD_BEAM_MAX_BEAMS || length < 0)
    return ARCHEAD_ERR_INVALID_ARG;
  if (count == 0 || batch == 0) return ARCHEAD_OK;
  if (!states || !parents || !is_aligned(parents, 4)) return ARCHEAD_ERR_INVALID_ARG;
  if (batch > (int64_t)1 << 30) return ARCHEAD_ERR_UNSUPPORTED;
  const int64_t rows = batch * beams;
  // Every state is checked before the first is moved.
  for (int i = 0; i < count; ++i) {
    const archead_beam_state &a = states[i];
    if (a.outer < 0 || a.inner < 0 || a.bytes < 0 || a.bytes_per_position < 0 || a.outer_stride < 0 ||
        a.row_stride < 0 || a.inner_stride < 0 || a.inner > 0x7fffffff)
      return ARCHEAD_ERR_INVALID_ARG;
    int64_t all;
    if (__builtin_mul_overflow(a.outer, a.inner, &all)) return ARCHEAD_ERR_INVALID_ARG;
    constexpr int64_t kMost = (int64_t)1 << 46;  // keeps the products below in 64 bits
    if (a.bytes > kMost || a.bytes_per_position > kMost / std::max<int64_t>(length, 1)) return ARCHEAD_ERR_INVALID_ARG;
    const int64_t bytes = a.bytes + length * a.bytes_per_position;
    if (__builtin_mul_overflow(all, bytes, &all)) return ARCHEAD_ERR_INVALID_ARG;
    if (all == 0) continue;
    if (!a.data || a.out == a.data) return ARCHEAD_ERR_INVALID_ARG;
    if ((a.outer > 1 && bytes > a.outer_stride) || (rows > 1 && bytes > a.row_stride) ||
        (a.inner > 1 && bytes > a.inner_stride))
      return ARCHEAD_ERR_INVALID_ARG;
  }
  const int most = reorder_vector_bytes(beams);
  Reordering r;
  r.p.parents = parents;
  r.p.batch = batch;
  r.p.beams = beams;
  r.p.count = 0;
  r.stream = static_cast<cudaStream_t>(stream);
  for (int i = 0; i < count; ++i) {
    const archead_beam_state &a = states[i];
    const int64_t bytes = a.bytes + length * a.bytes_per_position;
    if (bytes == 0 || a.outer == 0 || a.inner == 0) continue;
    char *src = static_cast<char *>(a.data), *dst = a.out ? static_cast<char *>(a.out) : src;
    const int64_t width = std::min<int64_t>(
        {(int64_t)most, low_bits((int64_t)(intptr_t)src), low_bits((int64_t)(intptr_t)dst), low_bits(bytes),
         a.outer > 1 ? low_bits(a.outer_stride) : 16, rows > 1 ? low_bits(a.row_stride) : 16,
         a.inner > 1 ? low_bits(a.inner_stride) : 16});
    r.add(src, dst, a.outer, a.inner, bytes, a, width);
  }
  r.flush();
  return status_of(r.failed);
}

}  // extern "C"
