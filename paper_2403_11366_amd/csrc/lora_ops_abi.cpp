// C ABI of the operators around the layer's output (4-bit weights, token log
// probabilities, distillation): argument validation and dispatch.  Every check
// runs before the first HIP call, so an invalid call launches nothing and
// leaves its outputs untouched.
#include <cmath>
#include <stdint.h>
#include <string.h>

#include "lora_linear.h"
#include "lora_ops.hpp"

namespace {

constexpr int64_t kMaxDim = int64_t(1) << 22;       // m, n, k of the 4-bit calls each at most 4M
constexpr int64_t kMaxElems = int64_t(1) << 30;     // any one matrix of theirs at most 2^30 elements
constexpr int64_t kMaxRows = int64_t(1) << 21;      // rows of logits
constexpr int64_t kMaxVocab = int64_t(1) << 20;     // their columns
constexpr int64_t kMaxLogits = int64_t(1) << 34;    // rows x row pitch
// Temperatures: 1/T and log2(e)/T are finite from the smallest normal number on (an
// infinite one times a row's maximum less itself is NaN); the distillation's T^2
// and its inverse are normal numbers between these two.
constexpr float kMinTemperature = 0x1p-126f;
constexpr float kMinDistillTemperature = 0x1p-63f, kMaxDistillTemperature = 0x1p63f;

struct Range {
  uintptr_t lo, hi;  // [lo, hi)
};

Range span(const void* p, uint64_t bytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  return Range{a, a + (uintptr_t)bytes};
}

bool aligned(const void* p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool aligned16(const void* p) { return aligned(p, 16); }
bool aligned4(const void* p) { return aligned(p, 4); }
// A C caller may pass any int as the type: its bits are read as an int (loading
// a lora_dtype that holds a value past the enumerators is undefined in C++).
int code_of(const lora_dtype* dtype) {
  static_assert(sizeof(lora_dtype) == sizeof(int), "lora_dtype is int-sized");
  int code;
  memcpy(&code, dtype, sizeof code);
  return code;
}

unsigned elem_bytes(int dtype) { return dtype == LORA_F32 ? 4 : 2; }

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

lora_status check_matrix(int64_t rows, int64_t k) {
  if (rows < 1 || k < 8 || k % 8 != 0) return LORA_ERR_SHAPE;
  if (rows > kMaxDim || k > kMaxDim || rows * ((k + 255) / 256 * 256) > kMaxElems) return LORA_ERR_UNSUPPORTED;
  return LORA_OK;
}

lora_status check_linear(int64_t m, int64_t n, int64_t k) {
  if (n < 8 || n % 8 != 0) return LORA_ERR_SHAPE;
  lora_status st = check_matrix(m, k);
  if (st == LORA_OK) st = check_matrix(n, k);
  if (st != LORA_OK) return st;
  return m * n > kMaxElems ? LORA_ERR_UNSUPPORTED : LORA_OK;
}

lora_status check_logits(int64_t rows, int64_t vocab, int64_t ld, int64_t top) {
  if (rows < 1 || vocab < 1 || ld < vocab || top < 0 || top > vocab) return LORA_ERR_SHAPE;
  if (rows > kMaxRows || vocab > kMaxVocab || ld > kMaxLogits / rows || top > lora::kMaxTop)
    return LORA_ERR_UNSUPPORTED;
  return LORA_OK;
}

// Bytes from the first row's start to the last row's end.
uint64_t logits_bytes(int64_t rows, int64_t vocab, int64_t ld, int dtype) {
  return (uint64_t)((rows - 1) * ld + vocab) * elem_bytes(dtype);
}

// Checks that the three distillation calls share.
lora_status check_distill(const void* logits, int dtype, int64_t ld, const int32_t* ids, const float* teacher,
                          const int32_t* labels, float tau, float w, int64_t rows, int64_t vocab, int64_t top) {
  if (!logits || !ids || !teacher) return LORA_ERR_NULL;
  if (dtype != LORA_BF16 && dtype != LORA_F32) return LORA_ERR_UNSUPPORTED;
  lora_status st = check_logits(rows, vocab, ld, top < vocab ? top : vocab);
  if (st != LORA_OK) return st;
  if (top < 1) return LORA_ERR_SHAPE;
  if (top > lora::kMaxTop) return LORA_ERR_UNSUPPORTED;
  if (!(tau >= kMinDistillTemperature && tau <= kMaxDistillTemperature) || !(w >= 0.0f && w <= 1.0f)) return LORA_ERR_SHAPE;
  if (!labels && w != 1.0f) return LORA_ERR_NULL;
  if (!aligned(logits, elem_bytes(dtype)) || !aligned4(ids) || !aligned4(teacher) || !aligned4(labels))
    return LORA_ERR_ALIGN;
  return LORA_OK;
}

lora::DistillArgs distill_args(const void* logits, int dtype, int64_t ld, const int32_t* ids,
                               const float* teacher, const int32_t* labels, float tau, float w, int64_t rows,
                               int64_t vocab, int64_t top) {
  lora::DistillArgs a{};
  a.logits = logits;
  a.f32 = dtype == LORA_F32;
  a.ld = ld;
  a.ids = ids;
  a.teacher = teacher;
  a.labels = labels;
  a.tau = tau;
  a.w = w;
  a.rows = rows;
  a.vocab = (int)vocab;
  a.top = (int)top;
  return a;
}

}  // namespace

extern "C" {

size_t lora_mx4_codes_size(int64_t rows, int64_t k) {
  return check_matrix(rows, k) == LORA_OK ? lora::mx4_codes_bytes(rows, k) : 0;
}

size_t lora_mx4_scales_size(int64_t rows, int64_t k) {
  return check_matrix(rows, k) == LORA_OK ? lora::mx4_scales_bytes(rows, k) : 0;
}

lora_status lora_mx4_quantize(const lora_bf16* X, uint8_t* codes, uint8_t* scales, int64_t rows, int64_t k,
                              void* stream) {
  if (!X || !codes || !scales) return LORA_ERR_NULL;
  const lora_status st = check_matrix(rows, k);
  if (st != LORA_OK) return st;
  if (!aligned16(X) || !aligned16(codes) || !aligned16(scales)) return LORA_ERR_ALIGN;
  const Range in[1] = {span(X, (uint64_t)(rows * k) * 2)};
  const Range out[2] = {span(codes, lora::mx4_codes_bytes(rows, k)), span(scales, lora::mx4_scales_bytes(rows, k))};
  if (any_alias(out, 2, in, 1)) return LORA_ERR_ALIAS;
  if (hip_error_pending()) return LORA_ERR_HIP;
  return status_of(lora::launch_mx4_quantize(lora::Mx4QuantArgs{X, codes, scales, rows, k},
                                             reinterpret_cast<hipStream_t>(stream)));
}

lora_status lora_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, lora_bf16* X, int64_t rows, int64_t k,
                                void* stream) {
  if (!codes || !scales || !X) return LORA_ERR_NULL;
  const lora_status st = check_matrix(rows, k);
  if (st != LORA_OK) return st;
  if (!aligned16(X) || !aligned16(codes) || !aligned16(scales)) return LORA_ERR_ALIGN;
  const Range in[2] = {span(codes, lora::mx4_codes_bytes(rows, k)), span(scales, lora::mx4_scales_bytes(rows, k))};
  const Range out[1] = {span(X, (uint64_t)(rows * k) * 2)};
  if (any_alias(out, 1, in, 2)) return LORA_ERR_ALIAS;
  if (hip_error_pending()) return LORA_ERR_HIP;
  return status_of(lora::launch_mx4_dequantize(codes, scales, X, rows, k, reinterpret_cast<hipStream_t>(stream)));
}

size_t lora_linear_mx4_fwd_workspace_size(int64_t m, int64_t n, int64_t k) {
  return check_linear(m, n, k) == LORA_OK ? lora::mx4_fwd_layout(m, n, k).total : 0;
}

lora_status lora_linear_mx4_fwd(const lora_bf16* X, const uint8_t* W_codes, const uint8_t* W_scales, lora_bf16* Y,
                                void* workspace, size_t workspace_bytes, int64_t m, int64_t n, int64_t k,
                                void* stream) {
  if (!X || !W_codes || !W_scales || !Y) return LORA_ERR_NULL;
  const lora_status st = check_linear(m, n, k);
  if (st != LORA_OK) return st;
  if (!aligned16(X) || !aligned16(W_codes) || !aligned16(W_scales) || !aligned16(Y)) return LORA_ERR_ALIGN;
  const size_t need = lora::mx4_fwd_layout(m, n, k).total;
  if (!workspace || workspace_bytes < need) return LORA_ERR_WORKSPACE;
  if (!aligned16(workspace)) return LORA_ERR_ALIGN;
  const Range in[3] = {span(X, (uint64_t)(m * k) * 2), span(W_codes, lora::mx4_codes_bytes(n, k)),
                       span(W_scales, lora::mx4_scales_bytes(n, k))};
  const Range out[2] = {span(Y, (uint64_t)(m * n) * 2), span(workspace, need)};
  if (any_alias(out, 2, in, 3)) return LORA_ERR_ALIAS;
  if (hip_error_pending()) return LORA_ERR_HIP;
  return status_of(lora::launch_mx4_fwd(lora::Mx4FwdArgs{X, W_codes, W_scales, Y, static_cast<char*>(workspace), m, n, k},
                                        reinterpret_cast<hipStream_t>(stream)));
}

size_t lora_token_logprobs_workspace_size(int64_t rows, int64_t vocab, int64_t top) {
  if (check_logits(rows, vocab, vocab, top) != LORA_OK) return 0;
  return lora::logprobs_workspace(rows, vocab, top);
}

lora_status lora_token_logprobs(const void* logits, lora_dtype type, int64_t ld, const int32_t* tokens,
                                float temperature, float* logp, float* entropy, int32_t* top_ids, float* top_logp,
                                void* workspace, size_t workspace_bytes, int64_t rows, int64_t vocab, int64_t top,
                                void* stream) {
  const int dtype = code_of(&type);
  if (!logits || !entropy || (tokens != nullptr) != (logp != nullptr)) return LORA_ERR_NULL;
  if (dtype != LORA_BF16 && dtype != LORA_F32) return LORA_ERR_UNSUPPORTED;
  const lora_status st = check_logits(rows, vocab, ld, top);
  if (st != LORA_OK) return st;
  if (top > 0 && (!top_ids || !top_logp)) return LORA_ERR_NULL;
  if (!(temperature >= kMinTemperature && temperature < INFINITY)) return LORA_ERR_SHAPE;
  if (!aligned(logits, elem_bytes(dtype)) || !aligned4(tokens) || !aligned4(logp) || !aligned4(entropy) ||
      (top > 0 && (!aligned4(top_ids) || !aligned4(top_logp))))
    return LORA_ERR_ALIGN;
  const size_t need = lora::logprobs_workspace(rows, vocab, top);
  if (!workspace || workspace_bytes < need) return LORA_ERR_WORKSPACE;
  if (!aligned16(workspace)) return LORA_ERR_ALIGN;
  const uint64_t per_row = (uint64_t)rows * 4, lists = per_row * (uint64_t)top;
  const Range in[2] = {span(logits, logits_bytes(rows, vocab, ld, dtype)), span(tokens, tokens ? per_row : 0)};
  const Range out[5] = {span(logp, logp ? per_row : 0), span(entropy, per_row), span(top_ids, lists),
                        span(top_logp, lists), span(workspace, need)};
  if (any_alias(out, 5, in, 2)) return LORA_ERR_ALIAS;
  lora::LogprobArgs a{logits, dtype == LORA_F32, ld, tokens, 1.0f / temperature, logp, entropy,
                      top_ids, top_logp, static_cast<char*>(workspace), rows, (int)vocab, (int)top};
  if (hip_error_pending()) return LORA_ERR_HIP;
  return status_of(lora::launch_token_logprobs(a, reinterpret_cast<hipStream_t>(stream)));
}

lora_status lora_distill_fwd(const void* logits, lora_dtype type, int64_t ld, const int32_t* teacher_ids,
                             const float* teacher_logits, const int32_t* labels, float temperature, float soft_weight,
                             float* loss, float* saved, int64_t rows, int64_t vocab, int64_t top, void* stream) {
  const int dtype = code_of(&type);
  const lora_status st = check_distill(logits, dtype, ld, teacher_ids, teacher_logits, labels, temperature,
                                       soft_weight, rows, vocab, top);
  if (st != LORA_OK) return st;
  if (!loss || !saved) return LORA_ERR_NULL;
  if (!aligned4(loss) || !aligned16(saved)) return LORA_ERR_ALIGN;
  const uint64_t per_row = (uint64_t)rows * 4, lists = per_row * (uint64_t)top;
  const Range in[4] = {span(logits, logits_bytes(rows, vocab, ld, dtype)), span(teacher_ids, lists),
                       span(teacher_logits, lists), span(labels, labels ? per_row : 0)};
  const Range out[2] = {span(loss, per_row), span(saved, per_row * 4)};
  if (any_alias(out, 2, in, 4)) return LORA_ERR_ALIAS;
  lora::DistillArgs a =
      distill_args(logits, dtype, ld, teacher_ids, teacher_logits, labels, temperature, soft_weight, rows, vocab, top);
  a.loss = loss;
  a.saved = saved;
  if (hip_error_pending()) return LORA_ERR_HIP;
  return status_of(lora::launch_distill_fwd(a, reinterpret_cast<hipStream_t>(stream)));
}

lora_status lora_distill_bwd(const void* logits, lora_dtype type, int64_t ld, const int32_t* teacher_ids,
                             const float* teacher_logits, const int32_t* labels, float temperature, float soft_weight,
                             const float* saved, const float* dloss, void* dlogits, int64_t rows, int64_t vocab,
                             int64_t top, void* stream) {
  const int dtype = code_of(&type);
  const lora_status st = check_distill(logits, dtype, ld, teacher_ids, teacher_logits, labels, temperature,
                                       soft_weight, rows, vocab, top);
  if (st != LORA_OK) return st;
  if (!saved || !dloss || !dlogits) return LORA_ERR_NULL;
  if (!aligned16(saved) || !aligned4(dloss) || !aligned(dlogits, elem_bytes(dtype))) return LORA_ERR_ALIGN;
  const uint64_t per_row = (uint64_t)rows * 4, lists = per_row * (uint64_t)top;
  const uint64_t whole = logits_bytes(rows, vocab, ld, dtype);
  const Range in[6] = {span(teacher_ids, lists), span(teacher_logits, lists), span(labels, labels ? per_row : 0),
                       span(saved, per_row * 4), span(dloss, per_row),
                       span(logits, dlogits == logits ? 0 : whole)};   // in place is allowed, a shifted overlap is not
  const Range out[1] = {span(dlogits, whole)};
  if (any_alias(out, 1, in, 6)) return LORA_ERR_ALIAS;
  lora::DistillArgs a =
      distill_args(logits, dtype, ld, teacher_ids, teacher_logits, labels, temperature, soft_weight, rows, vocab, top);
  a.saved = const_cast<float*>(saved);
  a.dloss = dloss;
  a.dlogits = dlogits;
  if (hip_error_pending()) return LORA_ERR_HIP;
  return status_of(lora::launch_distill_bwd(a, reinterpret_cast<hipStream_t>(stream)));
}

lora_status lora_distill_step(const void* logits, lora_dtype type, int64_t ld, const int32_t* teacher_ids,
                              const float* teacher_logits, const int32_t* labels, float temperature, float soft_weight,
                              const float* dloss, float* loss, void* dlogits, int64_t rows, int64_t vocab, int64_t top,
                              void* stream) {
  const int dtype = code_of(&type);
  const lora_status st = check_distill(logits, dtype, ld, teacher_ids, teacher_logits, labels, temperature,
                                       soft_weight, rows, vocab, top);
  if (st != LORA_OK) return st;
  if (!dloss || !loss || !dlogits) return LORA_ERR_NULL;
  if (!aligned4(dloss) || !aligned4(loss) || !aligned(dlogits, elem_bytes(dtype))) return LORA_ERR_ALIGN;
  const uint64_t per_row = (uint64_t)rows * 4, lists = per_row * (uint64_t)top;
  const uint64_t whole = logits_bytes(rows, vocab, ld, dtype);
  const Range in[5] = {span(teacher_ids, lists), span(teacher_logits, lists), span(labels, labels ? per_row : 0),
                       span(dloss, per_row), span(logits, dlogits == logits ? 0 : whole)};
  const Range out[2] = {span(loss, per_row), span(dlogits, whole)};
  if (any_alias(out, 2, in, 5)) return LORA_ERR_ALIAS;
  const Range z[1] = {span(logits, whole)};
  if (any_alias(out, 1, z, 1)) return LORA_ERR_ALIAS;   // the loss apart from the logits, also in place
  lora::DistillArgs a =
      distill_args(logits, dtype, ld, teacher_ids, teacher_logits, labels, temperature, soft_weight, rows, vocab, top);
  a.loss = loss;
  a.dloss = dloss;
  a.dlogits = dlogits;
  if (hip_error_pending()) return LORA_ERR_HIP;
  return status_of(lora::launch_distill_step(a, reinterpret_cast<hipStream_t>(stream)));
}

}  // extern "C"
