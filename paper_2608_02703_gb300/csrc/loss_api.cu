// C entry points of the dense head's cross entropy (include/archead.h): argument
// checks, the scratch handle, kernel sequencing.
#include <algorithm>
#include <new>

#include "device.cuh"
#include "internal.h"
#include "loss.h"
#include "status.h"

using namespace archead;

namespace {

constexpr int64_t kPieceBytes = (int64_t)256 << 20;  // of G, the gradient's piece
constexpr int64_t kMaxTokens = 1 << 20, kMaxVocab = 1 << 24, kMaxHidden = 1 << 16;

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

size_t take(size_t &off, int64_t bytes) {
  const size_t o = off;
  off += (size_t)up(bytes, 1024);
  return o;
}

// Scratch of the largest call.
void lay_out(archead_loss *l, char *base, size_t *bytes) {
  const int64_t tokens = l->max_tokens, rows = up(tokens, kCeTile), tiles = up(l->max_vocab, kCeTile) / kCeTile;
  size_t off = 0;
  const auto place = [&](auto *&p, int64_t n) {
    const size_t o = take(off, n);
    if (base) p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(base + o);
  };
  CeScratch &a = l->at;
  place(a.header, sizeof(CeHeader));
  place(a.place, 4 * tokens);
  place(a.target, 4 * rows);
  place(a.lse, 4 * rows);
  place(a.factor, 4 * rows);
  place(a.tlogit, 4 * rows);
  if (l->gradient) place(a.rest, 4 * rows);
  place(a.x, 2 * rows * up(l->max_hidden, kCeStep));
  place(a.part, (int64_t)sizeof(float2) * ce_most_parts(rows, tiles, l->clusters));
  if (l->gradient) {
    place(a.G, l->g_bytes);
    place(a.dx, l->dx_bytes);
  }
  *bytes = off;
}

archead_status refuse(const char *why) {
  set_last_error_message(why);
  return ARCHEAD_ERR_UNSUPPORTED;
}

bool rows16(const void *p, int64_t ld) { return is_aligned(p, 16) && ld % 8 == 0; }

// What both entries take.
struct Call {
  const void *x, *w;
  int dtype;
  int64_t M, V, d, ldx, ldw;
  const int32_t *targets;
};

archead_status check(const archead_loss *l, const Call &c) {
  if (!l || c.M < 0 || c.V < 1 || c.d < 1 || !is_dtype(c.dtype) || c.ldx < c.d || c.ldw < c.d)
    return ARCHEAD_ERR_INVALID_ARG;
  if (c.dtype == ARCHEAD_DTYPE_FP32) return refuse("x and w in bf16 or fp16 are wanted");
  if (c.M > 0 && (!c.x || !c.targets || !is_aligned(c.x, 2) || !is_aligned(c.targets, 4))) return ARCHEAD_ERR_INVALID_ARG;
  if (c.M > l->max_tokens || c.V > l->max_vocab || c.d > l->max_hidden)
    return refuse("the call is larger than its scratch was created for");
  return ARCHEAD_OK;
}

archead_status check_weight(const void *w, int64_t ldw) {
  if (!w || !is_aligned(w, 2)) return ARCHEAD_ERR_INVALID_ARG;
  if (!rows16(w, ldw)) return refuse("the weight's rows have to start on 16 bytes");
  return ARCHEAD_OK;
}

bool reads_directly(const Call &c) { return c.M <= kCeTile && rows16(c.x, c.ldx); }

CeCall products(const archead_loss *l, const Call &c) {
  CeCall p{};
  p.loss = l;
  p.x = c.x;
  p.w = c.w;
  p.ldx = c.ldx;
  p.direct = reads_directly(c);
  p.fp16 = c.dtype == ARCHEAD_DTYPE_FP16;
  p.M = c.M;
  p.V = c.V;
  p.d = c.d;
  p.ldw = c.ldw;
  p.rows = up(c.M, kCeTile);
  p.x_pitch = (int)up(c.d, kCeStep);
  return p;
}

CeRowsParams gathering(const archead_loss *l, const Call &c, int32_t ignore, const float *lse, const float *grad) {
  CeRowsParams p{};
  p.x = c.x;
  p.targets = c.targets;
  p.lse = lse;
  p.grad = grad;
  p.ignore = ignore;
  p.M = c.M;
  p.ldx = c.ldx;
  p.V = c.V;
  p.d = (int)c.d;
  p.x_pitch = (int)up(c.d, kCeStep);
  p.rows = up(c.M, kCeTile);
  p.direct = reads_directly(c);
  p.half = grad ? ce_half(c.M) : 0;
  p.at = l->at;
  return p;
}

}  // namespace

extern "C" {

archead_status archead_loss_create(int64_t max_tokens, int64_t max_vocab, int64_t max_hidden, int gradient,
                                   archead_loss **out) {
  if (!out) return ARCHEAD_ERR_INVALID_ARG;
  *out = nullptr;
  if (max_tokens < 1 || max_vocab < 1 || max_hidden < 1 || (gradient != 0 && gradient != 1))
    return ARCHEAD_ERR_INVALID_ARG;
  if (max_tokens > kMaxTokens || max_vocab > kMaxVocab || max_hidden > kMaxHidden)
    return refuse("more than 2^20 tokens, a vocabulary of 2^24 or rows of 2^16 elements");
  archead_loss *l = new (std::nothrow) archead_loss();
  if (!l) return ARCHEAD_ERR_OOM;
  l->max_tokens = max_tokens;
  l->max_vocab = max_vocab;
  l->max_hidden = max_hidden;
  l->gradient = gradient != 0;
  l->wait_budget = kDefaultWaitBudget;
  const auto build = [&]() -> cudaError_t {
    cudaError_t e = cudaGetDevice(&l->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&l->sm_count, cudaDevAttrMultiProcessorCount, l->device);
    if (e == cudaSuccess) e = ce_clusters(&l->clusters);
    if (e != cudaSuccess) return e;
    if (l->gradient) {
      const int64_t rows = up(max_tokens, kCeTile), wide = up(max_hidden, kCeTile);
      l->g_bytes = std::min(up(max_vocab, kCeTile) * rows * 2, std::max(kPieceBytes, rows * kCeTile * 2));
      // (splits take at most two units a pair: see ce_dx_splits)
      l->dx_bytes = 4 * kCeTile * kCeTile * std::max<int64_t>(2 * l->clusters, rows / kCeTile * (wide / kCeTile));
    }
    size_t bytes = 0;
    lay_out(l, nullptr, &bytes);
    if ((e = cudaMalloc(&l->ws, bytes)) != cudaSuccess) return e;
    l->ws_bytes = (int64_t)bytes;
    lay_out(l, static_cast<char *>(l->ws), &bytes);
    if ((e = cudaMalloc(&l->err, 16)) != cudaSuccess) return e;
    // (In a stream of its own, waited for: any stream may use the handle first.)
    cudaStream_t s = nullptr;
    if ((e = cudaStreamCreateWithFlags(&s, cudaStreamNonBlocking)) != cudaSuccess) return e;
    e = cudaMemsetAsync(l->err, 0, 16, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    cudaStreamDestroy(s);
    return e;
  };
  const cudaError_t e = build();
  if (e != cudaSuccess) {
    const archead_status st = status_of(e);
    if (l->ws) cudaFree(l->ws);
    if (l->err) cudaFree(l->err);
    delete l;
    return st;
  }
  *out = l;
  return ARCHEAD_OK;
}

void archead_loss_destroy(archead_loss *l) {
  if (!l) return;
  cudaSetDevice(l->device);
  cudaDeviceSynchronize();
  cudaFree(l->ws);
  cudaFree(l->err);
  delete l;
}

int64_t archead_loss_device_bytes(const archead_loss *l) { return l ? l->ws_bytes + 16 : -1; }

archead_status archead_linear_ce(archead_loss *loss, const void *x, const void *w, archead_dtype dtype, int64_t M,
                                 int64_t V, int64_t d, int64_t ldx, int64_t ldw, const int32_t *targets,
                                 int32_t ignore_index, float *ce, float *lse, void *stream) {
  const Call c{x, w, dtype, M, V, d, ldx, ldw, targets};
  archead_status st = check(loss, c);
  if (st != ARCHEAD_OK) return st;
  if (M == 0) return ARCHEAD_OK;
  if (!ce || !is_aligned(ce, 4) || !is_aligned(lse, 4) || ce == lse) return ARCHEAD_ERR_INVALID_ARG;
  if ((st = check_weight(w, ldw)) != ARCHEAD_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  AH_TRY(cudaSetDevice(loss->device));
  AH_TRY(launch_ce_gather(gathering(loss, c, ignore_index, nullptr, nullptr), s));
  const CeCall p = products(loss, c);
  CeFinishParams f{};
  AH_TRY(launch_ce_logits(p, &f.parts, s));
  f.targets = targets;
  f.ce = ce;
  f.lse = lse;
  f.ignore = ignore_index;
  f.M = M;
  f.V = V;
  f.rows = p.rows;
  f.at = loss->at;
  f.err = loss->err;
  AH_TRY(launch_ce_finish(f, s));
  return ARCHEAD_OK;
}

archead_status archead_linear_ce_backward(archead_loss *loss, const void *x, const void *w, archead_dtype dtype,
                                          int64_t M, int64_t V, int64_t d, int64_t ldx, int64_t ldw,
                                          const int32_t *targets, int32_t ignore_index, const float *lse,
                                          const float *grad_ce, void *dx, int64_t lddx, void *dw, int64_t lddw,
                                          int accumulate, void *stream) {
  const Call c{x, w, dtype, M, V, d, ldx, ldw, targets};
  archead_status st = check(loss, c);
  if (st != ARCHEAD_OK) return st;
  if ((accumulate != 0 && accumulate != 1) || (!dx && !dw && M > 0) || (dx && lddx < d) || (dw && lddw < d) ||
      !is_aligned(dx, 2) || !is_aligned(dw, 2) || (dw && (dw == w || dw == dx)) || (dx && dx == x && lddx != ldx))
    return ARCHEAD_ERR_INVALID_ARG;
  if (M > 0 && (!lse || !grad_ce || !is_aligned(lse, 4) || !is_aligned(grad_ce, 4))) return ARCHEAD_ERR_INVALID_ARG;
  if (!loss->gradient) return refuse("the scratch was created for the loss alone");
  if (dw && !rows16(dw, lddw)) return refuse("the rows of the weight's gradient have to start on 16 bytes");
  if (M == 0 && (!dw || accumulate)) return ARCHEAD_OK;
  if (M > 0 && (st = check_weight(w, ldw)) != ARCHEAD_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  AH_TRY(cudaSetDevice(loss->device));
  if (M == 0) {  // a sum of nothing
    AH_TRY(cudaMemset2DAsync(dw, (size_t)lddw * 2, 0, (size_t)d * 2, (size_t)V, s));
    return ARCHEAD_OK;
  }
  AH_TRY(launch_ce_gather(gathering(loss, c, ignore_index, lse, grad_ce), s));
  CeCall p = products(loss, c);
  p.dw = dw;
  p.lddw = lddw;
  p.accumulate = accumulate;
  p.want_dx = dx != nullptr;
  p.half = ce_half(M);
  p.splits = ce_dx_splits(loss, M, V, d, dw != nullptr);
  p.dx_pitch = (int)up(d, kCeTile);
  AH_TRY(launch_ce_gradient(p, s));
  if (dx) {
    CeDxParams f{};
    f.dx = dx;
    f.w = w;
    f.ldw = ldw;
    f.M = M;
    f.ld = lddx;
    f.rows = p.rows;
    f.d = (int)d;
    f.pitch = p.dx_pitch;
    f.splits = p.splits;
    f.fp16 = p.fp16;
    f.half = p.half;
    f.at = loss->at;
    AH_TRY(launch_ce_dx(f, s));
  }
  return ARCHEAD_OK;
}

archead_status archead_loss_sync_status(archead_loss *l, void *stream) {
  if (!l) return ARCHEAD_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  AH_TRY(cudaSetDevice(l->device));
  int word = 0;
  AH_TRY(take_error_word(l->err, s, &word));
  if (word & kErrLayout) return refuse("a kernel found its shared-memory window misaligned for its TMA layout and skipped its work");
  if (word & kErrWaitTimeout) return ARCHEAD_ERR_DEVICE_TIMEOUT;
  return word & kErrTargetRange ? ARCHEAD_ERR_TARGET_RANGE : ARCHEAD_OK;
}

archead_status archead_loss_set_wait_budget(archead_loss *l, int64_t cycles) {
  if (!l || cycles <= 0) return ARCHEAD_ERR_INVALID_ARG;
  l->wait_budget = cycles;
  return ARCHEAD_OK;
}

}  // extern "C"
