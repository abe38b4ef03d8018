// C entry points of the INT8 product (include/archead.h): argument checks, the
// weight handle and its workspace, kernel sequencing.
#include <algorithm>
#include <new>

#include "device.cuh"
#include "int8.h"
#include "internal.h"
#include "status.h"

using namespace archead;

namespace {

constexpr int kReserveTokens = 64;  // a new weight's workspace

// A call's kernel and its place in the workspace.
struct Plan {
  bool gemm = false, direct = false;
  I8GemmPlan g;
  size_t x_off = 0, scale_off = 0, total = 0;
};

size_t take(size_t &off, size_t bytes) {
  const size_t o = off;
  off += (bytes + 255) / 256 * 256;
  return o;
}

// What a call is given: activations, or codes.
enum Given { kActivations, kCodes };

// Whether the warp-level kernel takes what it is given as it is.
bool takes_directly(const archead_int8_weight *w, int64_t M, Given given) {
  return given == kActivations ? int8_decode_quantizes(M, w->K, w->K_pad) : int8_decode_fits(1, w->K_pad);
}

// AUTO takes the warp-level kernel up to 8 tokens, where its integer sums are
// exact (the tensor-memory kernel's are up to 2^24; 8 tokens of 16384 x 4096 14.1 us,
// with that one 12.4, of 4096 x 4096 7.3 and 7.6), and up to 16 where the weight
// is small: a second eight tokens cost its MMAs as much again, the tensor-memory
// kernel costs its start.  16 activations of 4096 x 512 4.6 us against 5.6, of
// 2048 x 2048, which take a launch more, 6.2 against 6.5, of 4096 x 2048 7.5 and
// 6.6, codes 5.7 and 6.4; 24 tokens of 4096 x 512 6.4 and 5.5.
bool auto_decodes(const archead_int8_weight *w, int64_t M, Given given) {
  if (M <= 8) return true;
  const int64_t most = (int64_t)(takes_directly(w, M, given) ? 8 : 4) << 20;
  return M <= 16 && int8_decode_fits(M, w->K_pad) && w->N_pad * w->K_pad <= most;
}

Plan plan(const archead_int8_weight *w, int64_t M, Given given, archead_path path) {
  Plan p;
  p.gemm = path == ARCHEAD_PATH_PREFILL || (path == ARCHEAD_PATH_AUTO && !auto_decodes(w, M, given));
  p.direct = !p.gemm && takes_directly(w, M, given);
  if (!p.direct) p.x_off = take(p.total, (size_t)M * w->K_pad * (p.gemm ? 2 : 1));
  if (!p.direct && given == kActivations) p.scale_off = take(p.total, (size_t)M * sizeof(float));
  if (p.gemm) p.g = int8_gemm_plan(w, M);
  return p;
}

// The most that AUTO needs for up to M tokens: what it needs for M, or for the
// most tokens that the warp-level kernel does not take as they are.
size_t room_for(const archead_int8_weight *w, int64_t M) {
  size_t most = plan(w, M, kActivations, ARCHEAD_PATH_AUTO).total;
  for (int64_t m : {8, 16})
    if (m < M) most = std::max(most, plan(w, m, kActivations, ARCHEAD_PATH_AUTO).total);
  return most;
}

// Growing synchronises the device: a call made earlier on another stream may
// still use the old buffer.  One that a captured call was given stays: its graph
// may run again.  The next is then at least twice as large, so that what is kept is
// never more than what is in use.
cudaError_t grow_workspace(archead_int8_weight *w, size_t bytes) {
  cudaError_t e = cudaDeviceSynchronize();
  if (e != cudaSuccess) return e;
  if (w->ws && w->ws_captured) {
    archead_int8_weight::Kept *k = new (std::nothrow) archead_int8_weight::Kept{w->ws, w->kept};
    if (!k) return cudaErrorMemoryAllocation;
    w->kept = k;
    bytes = std::max(bytes, 2 * w->ws_bytes);
  } else if (w->ws) {
    cudaFree(w->ws);
    w->owned_bytes -= (int64_t)w->ws_bytes;
  }
  w->ws = nullptr;
  w->ws_bytes = 0;
  w->ws_captured = false;
  w->reserved_tokens = 0;
  void *ws = nullptr;
  if ((e = cudaMalloc(&ws, bytes)) != cudaSuccess) return e;
  w->ws = ws;
  w->ws_bytes = bytes;
  w->owned_bytes += (int64_t)bytes;
  return cudaSuccess;
}

// Room for a call that needs `bytes`, and for every AUTO call of fewer tokens.
archead_status ensure_workspace(archead_int8_weight *w, size_t bytes, int64_t M, cudaStream_t s) {
  const bool captured = is_capturing(s);
  if (captured && bytes <= w->ws_bytes) w->ws_captured = true;
  if (bytes <= w->ws_bytes && M <= w->reserved_tokens) return ARCHEAD_OK;
  int64_t tokens = w->reserved_tokens;
  if (M > tokens && !captured) {
    tokens = std::max<int64_t>(M, kReserveTokens);  // (a growth that failed left nothing)
    bytes = std::max(bytes, room_for(w, tokens));
  }
  if (bytes <= w->ws_bytes) {
    w->reserved_tokens = tokens;
    return ARCHEAD_OK;
  }
  if (captured) {
    set_last_error_message("the workspace cannot grow while the stream is captured: call once with as many tokens before");
    return ARCHEAD_ERR_UNSUPPORTED;
  }
  const cudaError_t e = grow_workspace(w, bytes);
  if (e == cudaSuccess) w->reserved_tokens = tokens;
  return status_of(e);
}

template <typename T>
T *at(const archead_int8_weight *w, size_t off) {
  return reinterpret_cast<T *>(static_cast<char *>(w->ws) + off);
}

// The product of token codes that have been laid out in the workspace.
archead_status run_product(archead_int8_weight *w, const Plan &p, const float *x_scales, int64_t M, I8Out out,
                           cudaStream_t s) {
  if (p.gemm)
    return status_of(launch_int8_gemm(w, p.g, at<uint16_t>(w, p.x_off), x_scales, M, out, s));
  return status_of(launch_int8_decode(w, at<int8_t>(w, p.x_off), 0, w->K_pad, x_scales, M, out, s));
}

void free_weight(archead_int8_weight *w) {
  for (void *b : {(void *)w->codes, (void *)w->scales, (void *)w->err, w->ws})
    if (b) cudaFree(b);
  while (w->kept) {
    archead_int8_weight::Kept *k = w->kept;
    w->kept = k->next;
    cudaFree(k->ws);
    delete k;
  }
  delete w;
}

archead_status check_product(const archead_int8_weight *w, const void *x, int64_t M, const void *y, int out_dtype,
                             int64_t ldy) {
  if (!w || M < 0 || !is_dtype(out_dtype) || ldy < w->N) return ARCHEAD_ERR_INVALID_ARG;
  if (M == 0) return ARCHEAD_OK;
  if (!x || !y || !is_aligned(x, 16) || !is_aligned(y, 16)) return ARCHEAD_ERR_INVALID_ARG;
  if (M > (int64_t)1 << 30) return ARCHEAD_ERR_UNSUPPORTED;
  return ARCHEAD_OK;
}

}  // namespace

extern "C" {

archead_status archead_int8_weight_create(const int8_t *codes, const float *scales, int64_t N, int64_t K, void *stream,
                                          archead_int8_weight **out) {
  if (!out) return ARCHEAD_ERR_INVALID_ARG;
  *out = nullptr;
  if (!codes || !scales || N < 1 || K < 1) return ARCHEAD_ERR_INVALID_ARG;
  if (K > kI8MaxK || N > ((int64_t)1 << 31) - 256) return ARCHEAD_ERR_UNSUPPORTED;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  archead_int8_weight *w = new (std::nothrow) archead_int8_weight();
  if (!w) return ARCHEAD_ERR_OOM;
  int8_t *staged = nullptr;
  const auto build = [&]() -> cudaError_t {
    cudaError_t e = cudaGetDevice(&w->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&w->sm_count, cudaDevAttrMultiProcessorCount, w->device);
    if (e != cudaSuccess) return e;
    w->N = N;
    w->K = (int)K;
    w->N_pad = (N + kI8PadN - 1) / kI8PadN * kI8PadN;
    w->K_pad = (int)((K + kI8PadK - 1) / kI8PadK * kI8PadK);
    w->wait_budget = kDefaultWaitBudget;
    if ((e = int8_gemm_room(w)) != cudaSuccess) return e;
    const size_t code_bytes = (size_t)w->N_pad * w->K_pad, scale_bytes = (size_t)w->N_pad * sizeof(float);
    if ((e = cudaMalloc(&w->codes, code_bytes)) != cudaSuccess) return e;
    if ((e = cudaMalloc(&w->scales, scale_bytes)) != cudaSuccess) return e;
    if ((e = cudaMalloc(&w->err, 16)) != cudaSuccess) return e;
    w->owned_bytes = (int64_t)(code_bytes + scale_bytes + 16);
    if ((e = grow_workspace(w, room_for(w, kReserveTokens))) != cudaSuccess) return e;
    w->reserved_tokens = kReserveTokens;
    if ((e = cudaMemsetAsync(w->err, 0, 16, s)) != cudaSuccess) return e;
    if ((e = cudaMemsetAsync(w->scales, 0, scale_bytes, s)) != cudaSuccess) return e;
    if ((e = cudaMemcpyAsync(w->scales, scales, (size_t)N * sizeof(float), cudaMemcpyDefault, s)) != cudaSuccess)
      return e;
    // Codes in this device's memory are re-tiled from where they are.
    const int8_t *src = codes;
    cudaPointerAttributes attr{};
    const bool known = cudaPointerGetAttributes(&attr, codes) == cudaSuccess;
    cudaGetLastError();
    if (!known || attr.type != cudaMemoryTypeDevice || attr.device != w->device) {
      if ((e = cudaMalloc(&staged, (size_t)(N * K))) != cudaSuccess) return e;
      if ((e = cudaMemcpyAsync(staged, codes, (size_t)(N * K), cudaMemcpyDefault, s)) != cudaSuccess) return e;
      src = staged;
    }
    if ((e = launch_int8_layout(w, src, s)) != cudaSuccess) return e;
    return cudaStreamSynchronize(s);
  };
  const cudaError_t e = build();
  if (staged) cudaFree(staged);
  if (e != cudaSuccess) {
    const archead_status st = status_of(e);
    free_weight(w);
    return st;
  }
  *out = w;
  return ARCHEAD_OK;
}

void archead_int8_weight_destroy(archead_int8_weight *w) {
  if (!w) return;
  cudaSetDevice(w->device);
  cudaDeviceSynchronize();
  free_weight(w);
}

int64_t archead_int8_device_bytes(const archead_int8_weight *w) { return w ? w->owned_bytes : -1; }

archead_status archead_int8_quantize_tokens(const void *x, archead_dtype dtype, int64_t M, int64_t K, int64_t ldx,
                                            int8_t *codes, float *scales, void *stream) {
  if (M < 0 || K < 1 || ldx < K || !is_dtype(dtype)) return ARCHEAD_ERR_INVALID_ARG;
  if (M == 0) return ARCHEAD_OK;
  if (!x || !codes || !scales || !is_aligned(x, dtype_bytes(dtype)) || !is_aligned(codes, 16) ||
      !is_aligned(scales, 16))
    return ARCHEAD_ERR_INVALID_ARG;
  if (M > (int64_t)1 << 30 || K > (int64_t)1 << 30) return ARCHEAD_ERR_UNSUPPORTED;
  AH_TRY(launch_int8_quantize(x, dtype, M, K, ldx, codes, false, K, K, scales, static_cast<cudaStream_t>(stream)));
  return ARCHEAD_OK;
}

archead_status archead_int8_matmul_path(archead_int8_weight *w, const int8_t *x_codes, const float *x_scales,
                                        int64_t M, void *y, archead_dtype out_dtype, int64_t ldy, archead_path path,
                                        void *stream) {
  archead_status st = check_product(w, x_codes, M, y, out_dtype, ldy);
  if (st != ARCHEAD_OK || M == 0) return st;
  if (!x_scales || !is_aligned(x_scales, 16)) return ARCHEAD_ERR_INVALID_ARG;
  if (path != ARCHEAD_PATH_AUTO && path != ARCHEAD_PATH_DECODE && path != ARCHEAD_PATH_PREFILL)
    return ARCHEAD_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  AH_TRY(cudaSetDevice(w->device));
  const Plan p = plan(w, M, kCodes, path);
  if (p.direct) return status_of(launch_int8_decode(w, x_codes, 0, w->K, x_scales, M, {y, ldy, out_dtype}, s));
  if ((st = ensure_workspace(w, p.total, M, s)) != ARCHEAD_OK) return st;
  AH_TRY(launch_int8_pad(x_codes, M, w->K, w->K_pad, at<void>(w, p.x_off), p.gemm, s));
  return run_product(w, p, x_scales, M, {y, ldy, out_dtype}, s);
}

archead_status archead_int8_matmul(archead_int8_weight *w, const int8_t *x_codes, const float *x_scales, int64_t M,
                                   void *y, archead_dtype out_dtype, int64_t ldy, void *stream) {
  return archead_int8_matmul_path(w, x_codes, x_scales, M, y, out_dtype, ldy, ARCHEAD_PATH_AUTO, stream);
}

archead_status archead_int8_linear(archead_int8_weight *w, const void *x, archead_dtype x_dtype, int64_t M,
                                   int64_t ldx, void *y, archead_dtype out_dtype, int64_t ldy, void *stream) {
  archead_status st = check_product(w, x, M, y, out_dtype, ldy);
  if (st != ARCHEAD_OK) return st;
  if (!is_dtype(x_dtype) || ldx < w->K) return ARCHEAD_ERR_INVALID_ARG;
  if (M == 0) return ARCHEAD_OK;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  AH_TRY(cudaSetDevice(w->device));
  const Plan p = plan(w, M, kActivations, ARCHEAD_PATH_AUTO);
  if (p.direct) return status_of(launch_int8_decode(w, x, x_dtype, ldx, nullptr, M, {y, ldy, out_dtype}, s));
  if ((st = ensure_workspace(w, p.total, M, s)) != ARCHEAD_OK) return st;
  float *scales = at<float>(w, p.scale_off);
  AH_TRY(launch_int8_quantize(x, x_dtype, M, w->K, ldx, at<void>(w, p.x_off), p.gemm, w->K_pad, w->K_pad, scales, s));
  return run_product(w, p, scales, M, {y, ldy, out_dtype}, s);
}

archead_status archead_int8_sync_status(archead_int8_weight *w, void *stream) {
  if (!w) return ARCHEAD_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  AH_TRY(cudaSetDevice(w->device));
  int word = 0;
  AH_TRY(take_error_word(w->err, s, &word));
  if (word & kErrLayout) {
    set_last_error_message("a kernel found its shared-memory window misaligned for its TMA layout and skipped its work");
    return ARCHEAD_ERR_UNSUPPORTED;
  }
  return word & kErrWaitTimeout ? ARCHEAD_ERR_DEVICE_TIMEOUT : ARCHEAD_OK;
}

archead_status archead_int8_set_wait_budget(archead_int8_weight *w, int64_t cycles) {
  if (!w || cycles <= 0) return ARCHEAD_ERR_INVALID_ARG;
  w->wait_budget = cycles;
  return ARCHEAD_OK;
}

}  // extern "C"
