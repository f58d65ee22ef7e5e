// C ABI of the operators of a fine-tuning step (8-bit frozen weights, cross entropy
// without logits, dropout without a mask): argument validation and dispatch.  Every
// check runs before the first HIP call, so an invalid call launches nothing and
// leaves its outputs untouched.
#include <cmath>
#include <stdint.h>
#include <string.h>

#include "lora_linear.h"
#include "lora_train.hpp"

namespace {

constexpr int64_t kMaxDim = int64_t(1) << 22;       // m, n, k of the 8-bit calls each at most 4M
constexpr int64_t kMaxElems = int64_t(1) << 30;     // any one matrix of theirs, and X of the loss
constexpr int64_t kMaxRows = int64_t(1) << 20;      // rows of the loss
constexpr int64_t kMaxVocab = int64_t(1) << 20;     // columns of its logits
constexpr int64_t kMaxHidden = int64_t(1) << 16;    // width of its rows
constexpr int64_t kMaxCount = int64_t(1) << 35;     // elements of a dropout call: a thread per 16, fewer than 2^32 of them

struct Range {
  uintptr_t lo, hi;  // [lo, hi)
};

Range span(const void* p, uint64_t bytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  return Range{a, p ? a + (uintptr_t)bytes : a};
}

bool aligned(const void* p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool aligned16(const void* p) { return aligned(p, 16); }
bool aligned4(const void* p) { return aligned(p, 4); }

// True if an output overlaps an input or another output.  Empty ranges
// (arguments that a call does without) overlap nothing.
bool any_alias(const Range* out, int n_out, const Range* in, int n_in) {
  auto overlap = [](const Range& x, const Range& y) {
    return x.lo < x.hi && y.lo < y.hi && x.lo < y.hi && y.lo < x.hi;
  };
  for (int i = 0; i < n_out; ++i) {
    for (int j = 0; j < n_in; ++j)
      if (overlap(out[i], in[j])) return true;
    for (int j = i + 1; j < n_out; ++j)
      if (overlap(out[i], out[j])) return true;
  }
  return false;
}

// An error that an earlier HIP call left on the thread is reported before
// anything is enqueued, and left pending for the caller to read.
bool hip_error_pending() { return hipPeekAtLastError() != hipSuccess; }
lora_status status_of(hipError_t e) { return e == hipSuccess ? LORA_OK : LORA_ERR_HIP; }
hipStream_t stream_of(void* s) { return reinterpret_cast<hipStream_t>(s); }

lora_status check_matrix(int64_t rows, int64_t k) {
  if (rows < 1 || k < 8 || k % 8 != 0) return LORA_ERR_SHAPE;
  if (rows > kMaxDim || k > kMaxDim || rows * ((k + 127) / 128 * 128) > kMaxElems) return LORA_ERR_UNSUPPORTED;
  return LORA_OK;
}

lora_status check_blocks(int64_t rows, int64_t k, int block_rows) {
  if (block_rows != 1 && block_rows != 128) return LORA_ERR_SHAPE;
  return check_matrix(rows, k);
}

lora_status check_linear(int64_t m, int64_t n, int64_t k) {
  if (n < 8 || n % 8 != 0) return LORA_ERR_SHAPE;
  lora_status st = check_matrix(m, k);
  if (st == LORA_OK) st = check_matrix(n, k);
  if (st == LORA_OK) st = check_matrix(m, n);
  return st;
}

lora_status check_xent(int64_t rows, int64_t vocab, int64_t k) {
  if (rows < 1 || vocab < 1 || k < 8 || k % 8 != 0) return LORA_ERR_SHAPE;
  if (rows > kMaxRows || vocab > kMaxVocab || k > kMaxHidden || rows * k > kMaxElems) return LORA_ERR_UNSUPPORTED;
  return LORA_OK;
}

// What both directions of the 8-bit layer check: A [m, c] times the weight into out [m, o].
lora_status check_fp8_call(const lora_bf16* A, const uint8_t* Wc, const uint8_t* Ws, lora_bf16* out, void* ws,
                           size_t ws_bytes, size_t need, int64_t m, int64_t c, int64_t o, int64_t n, int64_t k) {
  if (!aligned16(A) || !aligned16(Wc) || !aligned16(Ws) || !aligned16(out)) return LORA_ERR_ALIGN;
  if (!ws || ws_bytes < need) return LORA_ERR_WORKSPACE;
  if (!aligned16(ws)) return LORA_ERR_ALIGN;
  const Range in[3] = {span(A, (uint64_t)(m * c) * 2), span(Wc, lora::fp8_codes_bytes(n, k)),
                       span(Ws, lora::fp8_scales_bytes(n, k, 128))};
  const Range outs[2] = {span(out, (uint64_t)(m * o) * 2), span(ws, need)};
  return any_alias(outs, 2, in, 3) ? LORA_ERR_ALIAS : LORA_OK;
}

}  // namespace

extern "C" {

size_t lora_fp8_codes_size(int64_t rows, int64_t k) {
  return check_matrix(rows, k) == LORA_OK ? lora::fp8_codes_bytes(rows, k) : 0;
}

size_t lora_fp8_scales_size(int64_t rows, int64_t k, int block_rows) {
  return check_blocks(rows, k, block_rows) == LORA_OK ? lora::fp8_scales_bytes(rows, k, block_rows) : 0;
}

lora_status lora_fp8_quantize(const lora_bf16* X, uint8_t* codes, uint8_t* scales, int64_t rows, int64_t k,
                              int block_rows, void* stream) {
  if (!X || !codes || !scales) return LORA_ERR_NULL;
  const lora_status st = check_blocks(rows, k, block_rows);
  if (st != LORA_OK) return st;
  if (!aligned16(X) || !aligned16(codes) || !aligned16(scales)) return LORA_ERR_ALIGN;
  const Range in[1] = {span(X, (uint64_t)(rows * k) * 2)};
  const Range out[2] = {span(codes, lora::fp8_codes_bytes(rows, k)),
                        span(scales, lora::fp8_scales_bytes(rows, k, block_rows))};
  if (any_alias(out, 2, in, 1)) return LORA_ERR_ALIAS;
  if (hip_error_pending()) return LORA_ERR_HIP;
  return status_of(lora::launch_fp8_quantize(lora::Fp8QuantArgs{X, codes, scales, rows, k, block_rows}, stream_of(stream)));
}

lora_status lora_fp8_dequantize(const uint8_t* codes, const uint8_t* scales, lora_bf16* X, int64_t rows, int64_t k,
                                int block_rows, void* stream) {
  if (!codes || !scales || !X) return LORA_ERR_NULL;
  const lora_status st = check_blocks(rows, k, block_rows);
  if (st != LORA_OK) return st;
  if (!aligned16(X) || !aligned16(codes) || !aligned16(scales)) return LORA_ERR_ALIGN;
  const Range in[2] = {span(codes, lora::fp8_codes_bytes(rows, k)),
                       span(scales, lora::fp8_scales_bytes(rows, k, block_rows))};
  const Range out[1] = {span(X, (uint64_t)(rows * k) * 2)};
  if (any_alias(out, 1, in, 2)) return LORA_ERR_ALIAS;
  if (hip_error_pending()) return LORA_ERR_HIP;
  return status_of(lora::launch_fp8_dequantize(codes, scales, X, rows, k, block_rows, stream_of(stream)));
}

size_t lora_linear_fp8_fwd_workspace_size(int64_t m, int64_t n, int64_t k) {
  if (check_linear(m, n, k) != LORA_OK) return 0;
  return lora::bytes_up_to(m, [&](int64_t rows) { return lora::fp8_fwd_layout(rows, n, k).total; });
}

size_t lora_linear_fp8_bwd_workspace_size(int64_t m, int64_t n, int64_t k) {
  if (check_linear(m, n, k) != LORA_OK) return 0;
  return lora::bytes_up_to(m, [&](int64_t rows) { return lora::fp8_bwd_layout(rows, n, k).total; });
}

lora_status lora_linear_fp8_fwd(const lora_bf16* X, const uint8_t* W_codes, const uint8_t* W_scales, lora_bf16* Y,
                                void* workspace, size_t workspace_bytes, int64_t m, int64_t n, int64_t k,
                                void* stream) {
  if (!X || !W_codes || !W_scales || !Y) return LORA_ERR_NULL;
  lora_status st = check_linear(m, n, k);
  if (st == LORA_OK)
    st = check_fp8_call(X, W_codes, W_scales, Y, workspace, workspace_bytes, lora::fp8_fwd_layout(m, n, k).total, m, k, n,
                        n, k);
  if (st != LORA_OK) return st;
  if (hip_error_pending()) return LORA_ERR_HIP;
  return status_of(lora::launch_fp8_fwd(lora::Fp8Args{X, W_codes, W_scales, Y, static_cast<char*>(workspace), m, n, k},
                                        stream_of(stream)));
}

lora_status lora_linear_fp8_bwd(const lora_bf16* dY, const uint8_t* W_codes, const uint8_t* W_scales, lora_bf16* dX,
                                void* workspace, size_t workspace_bytes, int64_t m, int64_t n, int64_t k,
                                void* stream) {
  if (!dY || !W_codes || !W_scales || !dX) return LORA_ERR_NULL;
  lora_status st = check_linear(m, n, k);
  if (st == LORA_OK)
    st = check_fp8_call(dY, W_codes, W_scales, dX, workspace, workspace_bytes, lora::fp8_bwd_layout(m, n, k).total, m, n,
                        k, n, k);
  if (st != LORA_OK) return st;
  if (hip_error_pending()) return LORA_ERR_HIP;
  return status_of(lora::launch_fp8_bwd(lora::Fp8Args{dY, W_codes, W_scales, dX, static_cast<char*>(workspace), m, n, k},
                                        stream_of(stream)));
}

lora_status lora_dropout(const void* X, const void* residual, void* Y, lora_dtype type, int64_t count, uint64_t seed,
                         uint64_t offset, float p, void* stream) {
  int dtype;   // a C caller may pass any int as the type: its bits are read as one
  static_assert(sizeof(lora_dtype) == sizeof(int), "lora_dtype is int-sized");
  memcpy(&dtype, &type, sizeof dtype);
  if (!X || !Y) return LORA_ERR_NULL;
  if (dtype != LORA_BF16 && dtype != LORA_F32) return LORA_ERR_UNSUPPORTED;
  if (count < 1) return LORA_ERR_SHAPE;
  if (count > kMaxCount) return LORA_ERR_UNSUPPORTED;
  if (!(p >= 0.0f && p < 1.0f)) return LORA_ERR_SHAPE;
  if (!aligned16(X) || !aligned16(residual) || !aligned16(Y)) return LORA_ERR_ALIGN;
  const uint64_t bytes = (uint64_t)count * (dtype == LORA_F32 ? 4 : 2);
  const Range out[1] = {span(Y, bytes)};
  const Range in[2] = {span(X, X == Y ? 0 : bytes), span(residual, residual == Y ? 0 : bytes)};   // in place is allowed
  if (any_alias(out, 1, in, 2)) return LORA_ERR_ALIAS;
  if (hip_error_pending()) return LORA_ERR_HIP;
  return status_of(lora::launch_dropout(
      lora::DropoutArgs{X, residual, Y, dtype == LORA_F32, count, seed, offset,
                        (uint32_t)std::floor((1.0 - (double)p) * 65536.0 + 0.5), (float)(1.0 / (1.0 - (double)p))},
      stream_of(stream)));
}

size_t lora_linear_xent_workspace_size(int64_t rows, int64_t vocab, int64_t k, int dx, int dw) {
  if (check_xent(rows, vocab, k) != LORA_OK) return 0;
  return lora::bytes_up_to(rows, [&](int64_t r) { return lora::xent_layout(r, vocab, k, dx != 0, dw != 0).total; });
}

}  // extern "C"

namespace {

// Checks that the three loss calls share; null pointers are arguments a call does without.
lora_status check_xent_call(const lora::XentArgs& a, void* ws, size_t ws_bytes) {
  const lora_status st = check_xent(a.rows, a.vocab, a.k);
  if (st != LORA_OK) return st;
  if (!aligned16(a.X) || !aligned16(a.W) || !aligned16(a.dX) || !aligned16(a.dW) || !aligned4(a.labels) ||
      !aligned4(a.dloss) || !aligned4(a.loss) || !aligned4(a.saved))
    return LORA_ERR_ALIGN;
  const size_t need = lora::xent_layout(a.rows, a.vocab, a.k, a.dX != nullptr, a.dW != nullptr).total;
  if (!ws || ws_bytes < need) return LORA_ERR_WORKSPACE;
  if (!aligned16(ws)) return LORA_ERR_ALIGN;
  return LORA_OK;
}

lora_status check_xent_alias(const lora::XentArgs& a, void* ws, bool saved_is_output) {
  const uint64_t x = (uint64_t)(a.rows * a.k) * 2, w = (uint64_t)a.vocab * a.k * 2, r = (uint64_t)a.rows * 4;
  const size_t need = lora::xent_layout(a.rows, a.vocab, a.k, a.dX != nullptr, a.dW != nullptr).total;
  const Range saved = span(a.saved, 2 * r), none{0, 0};
  const Range in[5] = {span(a.X, x), span(a.W, w), span(a.labels, r), span(a.dloss, r), saved_is_output ? none : saved};
  const Range out[5] = {span(a.loss, r), span(a.dX, x), span(a.dW, w), span(ws, need), saved_is_output ? saved : none};
  return any_alias(out, 5, in, 5) ? LORA_ERR_ALIAS : LORA_OK;
}

}  // namespace

extern "C" {

lora_status lora_linear_xent_fwd(const lora_bf16* X, const lora_bf16* W, const int32_t* labels, float* loss, float* saved,
                                 void* workspace, size_t workspace_bytes, int64_t rows, int64_t vocab, int64_t k,
                                 void* stream) {
  if (!X || !W || !labels || !loss) return LORA_ERR_NULL;
  const lora::XentArgs a{X, W, labels, nullptr, loss, saved, nullptr, nullptr, static_cast<char*>(workspace), rows, vocab, k};
  lora_status st = check_xent_call(a, workspace, workspace_bytes);
  if (st == LORA_OK) st = check_xent_alias(a, workspace, true);
  if (st != LORA_OK) return st;
  if (hip_error_pending()) return LORA_ERR_HIP;
  return status_of(lora::launch_xent_fwd(a, stream_of(stream)));
}

lora_status lora_linear_xent_bwd(const lora_bf16* X, const lora_bf16* W, const int32_t* labels, const float* saved,
                                 const float* dloss, lora_bf16* dX, lora_bf16* dW, void* workspace,
                                 size_t workspace_bytes, int64_t rows, int64_t vocab, int64_t k, void* stream) {
  if (!X || !W || !labels || !saved || !dloss || (!dX && !dW)) return LORA_ERR_NULL;
  const lora::XentArgs a{X, W, labels, dloss, nullptr, const_cast<float*>(saved), dX, dW, static_cast<char*>(workspace),
                         rows, vocab, k};
  lora_status st = check_xent_call(a, workspace, workspace_bytes);
  if (st == LORA_OK) st = check_xent_alias(a, workspace, false);
  if (st != LORA_OK) return st;
  if (hip_error_pending()) return LORA_ERR_HIP;
  return status_of(lora::launch_xent_bwd(a, stream_of(stream)));
}

lora_status lora_linear_xent_step(const lora_bf16* X, const lora_bf16* W, const int32_t* labels, const float* dloss,
                                  float* loss, lora_bf16* dX, lora_bf16* dW, void* workspace, size_t workspace_bytes,
                                  int64_t rows, int64_t vocab, int64_t k, void* stream) {
  if (!X || !W || !labels || !dloss || !loss || (!dX && !dW)) return LORA_ERR_NULL;
  const lora::XentArgs a{X, W, labels, dloss, loss, nullptr, dX, dW, static_cast<char*>(workspace), rows, vocab, k};
  lora_status st = check_xent_call(a, workspace, workspace_bytes);
  if (st == LORA_OK) st = check_xent_alias(a, workspace, true);
  if (st != LORA_OK) return st;
  if (hip_error_pending()) return LORA_ERR_HIP;
  return status_of(lora::launch_xent_step(a, stream_of(stream)));
}

}  // extern "C"
