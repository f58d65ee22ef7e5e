// Internal interface of the operators around the layer's output between the C
// ABI (lora_ops_abi.cpp: argument checks) and their kernels: 4-bit weights
// (lora_mx4.hip), token log probabilities and distillation (lora_logits.hip).
// Shapes here have already been validated; the launch rules stand here, so that
// lora_linear_plan() reports the launches that the entry points make.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lora {

constexpr int kMaxTop = 128;   // alternatives of a row, and entries of a teacher's list

// ---- rows of logits ----------------------------------------------------------
// A row is walked in chunks of 16 bytes (8 bf16 or 4 fp32 values): the whole
// ones that start at a 16-byte boundary, and single elements before and after.
// One workgroup takes a row; `threads` x `keep` chunks fit its registers, keep =
// 0 reads the row again in every pass.
struct RowShape {
  int threads, keep;
};

// The smallest workgroup whose registers hold the row, up to 64 of a thread's
// 128 registers (1024 threads).
inline RowShape row_shape(int64_t vocab, int elem) {
  const int64_t chunks = (vocab * elem + 15) / 16;
  if (chunks <= 1024) return RowShape{256, 4};
  if (chunks <= 2048) return RowShape{256, 8};
  if (chunks <= 4096) return RowShape{512, 8};
  if (chunks <= 8192) return RowShape{1024, 8};
  if (chunks <= 16384) return RowShape{1024, 16};
  return RowShape{1024, 0};
}

struct LogprobArgs {
  const void* logits;
  bool f32;
  int64_t ld;
  const int32_t* tokens;   // or none
  float itau;              // 1 / temperature
  float *logp, *entropy;
  int32_t* top_ids;
  float* top_logp;
  char* ws;
  int64_t rows;
  int vocab, top;
};

inline size_t logprobs_workspace(int64_t rows, int64_t vocab, int64_t top) {
  (void)rows;
  (void)vocab;
  (void)top;
  return 256;
}

struct DistillArgs {
  const void* logits;
  bool f32;
  int64_t ld;
  const int32_t* ids;      // teacher's list [rows, top]
  const float* teacher;    // its logits
  const int32_t* labels;   // or none (soft_weight 1)
  float tau, w;            // temperature, weight of the soft term
  float *loss, *saved;
  const float* dloss;
  void* dlogits;
  int64_t rows;
  int vocab, top;
};

// Columns of one workgroup of the gradient that reads what the forward saved.
constexpr int kGradThreads = 256, kGradKeep = 8;
inline int grad_parts(int64_t vocab, int elem) {
  const int64_t chunks = (vocab * elem + 15) / 16;
  return (int)((chunks + kGradThreads * kGradKeep - 1) / (kGradThreads * kGradKeep));
}

hipError_t launch_token_logprobs(const LogprobArgs& a, hipStream_t st);
hipError_t launch_distill_fwd(const DistillArgs& a, hipStream_t st);
hipError_t launch_distill_bwd(const DistillArgs& a, hipStream_t st);
hipError_t launch_distill_step(const DistillArgs& a, hipStream_t st);

// ---- 4-bit weights -----------------------------------------------------------
// Microscaled 4 bits: rows of 32-column blocks, a byte of scale each.  A row's
// codes take 128 bytes per 256 columns; scales stand in cells of 512 bytes, one
// per 64 rows and 256 columns (mx4_scale_offset).
inline int64_t mx4_slabs(int64_t k) { return (k + 255) / 256; }        // 256-column slabs of a row
inline int64_t mx4_groups(int64_t rows) { return (rows + 63) / 64; }   // 64-row groups
inline size_t mx4_codes_bytes(int64_t rows, int64_t k) { return (size_t)(rows * mx4_slabs(k) * 128); }
inline size_t mx4_scales_bytes(int64_t rows, int64_t k) { return (size_t)(mx4_groups(rows) * mx4_slabs(k) * 512); }

struct Mx4QuantArgs {
  const uint16_t* X;
  uint8_t *codes, *scales;
  int64_t rows, k;
};

struct Mx4FwdArgs {
  const uint16_t* X;
  const uint8_t *Wc, *Ws;
  uint16_t* Y;
  char* ws;
  int64_t m, n, k;
};

// Workspace of the 4-bit forward: X's codes and scales.
struct Mx4Layout {
  size_t xc, xs, total;
};
inline Mx4Layout mx4_fwd_layout(int64_t m, int64_t n, int64_t k) {
  (void)n;
  Mx4Layout L;
  L.xc = 0;
  L.xs = (mx4_codes_bytes(m, k) + 255) / 256 * 256;
  L.total = L.xs + (mx4_scales_bytes(m, k) + 255) / 256 * 256;
  return L;
}

hipError_t launch_mx4_quantize(const Mx4QuantArgs& a, hipStream_t st);
hipError_t launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, uint16_t* X, int64_t rows, int64_t k,
                                 hipStream_t st);
hipError_t launch_mx4_fwd(const Mx4FwdArgs& a, hipStream_t st);

}  // namespace lora
