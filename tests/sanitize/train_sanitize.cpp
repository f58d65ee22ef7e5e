// Memory- and UB-checking driver for the C ABI of the operators of a fine-tuning step
// and for their launch rules, built with the address and undefined-behaviour
// sanitizers on the host by tests/test_train_plan.py.  It runs without a GPU: every
// entry-point call below is invalid and must be rejected, with the expected status,
// before any HIP call.  Device pointers are fake addresses that validation never reads.
//
// With arguments "fwd" or "bwd" and m n k m n k ... it prints the kernel kind of each
// 8-bit call, with "xent" and rows vocab k ... those of the loss.
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "lora_linear.h"
#include "lora_train.hpp"

static int failures = 0;

#define EXPECT(call, want)                                                                      \
  do {                                                                                          \
    const long got_ = (long)(call);                                                             \
    if (got_ != (long)(want)) {                                                                 \
      fprintf(stderr, "line %d: %s returned %ld, expected %ld\n", __LINE__, #call, got_, (long)(want)); \
      ++failures;                                                                               \
    }                                                                                           \
  } while (0)
#define HOLDS(cond, a, b, c)                                                                    \
  do {                                                                                          \
    if (!(cond)) {                                                                              \
      fprintf(stderr, "line %d: %s: %ld %ld %ld\n", __LINE__, #cond, (long)(a), (long)(b), (long)(c)); \
      ++failures;                                                                               \
    }                                                                                           \
  } while (0)

template <typename T>
static T* dev(int i, uintptr_t off = 0) {
  return reinterpret_cast<T*>((uintptr_t(1) << 50) + uintptr_t(i) * (uintptr_t(1) << 44) + off);
}

static void refusals() {
  lora_bf16 *x = dev<lora_bf16>(0), *y = dev<lora_bf16>(3), *w = dev<lora_bf16>(4), *dw = dev<lora_bf16>(5);
  uint8_t *c = dev<uint8_t>(1), *s = dev<uint8_t>(2);
  void* ws = dev<void>(6);
  float *f = dev<float>(7), *g = dev<float>(8), *h = dev<float>(9);
  int32_t* t = dev<int32_t>(10);
  const int64_t top = INT64_MAX, low = INT64_MIN;
  const size_t much = size_t(1) << 43;
  EXPECT(lora_fp8_quantize(x, c, s, top, top - 7, 128, nullptr), LORA_ERR_UNSUPPORTED);
  EXPECT(lora_fp8_quantize(x, c, s, low, 8, 1, nullptr), LORA_ERR_SHAPE);
  EXPECT(lora_fp8_quantize(x, c, s, 8, 8, INT32_MIN, nullptr), LORA_ERR_SHAPE);
  EXPECT(lora_fp8_dequantize(c, s, dev<lora_bf16>(0, 2), 8, 8, 1, nullptr), LORA_ERR_ALIGN);
  EXPECT(lora_fp8_codes_size(top, top), 0);
  EXPECT(lora_fp8_scales_size(low, 8, 1), 0);
  EXPECT(lora_linear_fp8_fwd_workspace_size(top, 8, 8), 0);
  EXPECT(lora_linear_fp8_bwd_workspace_size(8, low, 8), 0);
  EXPECT(lora_linear_fp8_fwd(x, c, s, y, ws, much, top, top - 7, 8, nullptr), LORA_ERR_UNSUPPORTED);
  EXPECT(lora_linear_fp8_fwd(x, c, s, y, ws, 8, 8, 8, 8, nullptr), LORA_ERR_WORKSPACE);
  EXPECT(lora_linear_fp8_bwd(x, c, s, x, ws, much, 8, 8, 8, nullptr), LORA_ERR_ALIAS);
  EXPECT(lora_dropout(x, nullptr, y, (lora_dtype)9, 8, 1, 2, 0.5f, nullptr), LORA_ERR_UNSUPPORTED);
  EXPECT(lora_dropout(x, nullptr, y, LORA_F32, low, 1, 2, 0.5f, nullptr), LORA_ERR_SHAPE);
  EXPECT(lora_dropout(x, nullptr, y, LORA_F32, top, 1, 2, 0.5f, nullptr), LORA_ERR_UNSUPPORTED);
  EXPECT(lora_dropout(x, x, dev<float>(0, 16), LORA_F32, 8, 1, 2, 0.5f, nullptr), LORA_ERR_ALIAS);
  EXPECT(lora_linear_xent_workspace_size(top, top, top, 1, 1), 0);
  EXPECT(lora_linear_xent_workspace_size(8, low, 8, 1, 1), 0);
  EXPECT(lora_linear_xent_fwd(x, w, t, f, g, ws, much, top, 8, 8, nullptr), LORA_ERR_UNSUPPORTED);
  EXPECT(lora_linear_xent_fwd(x, w, t, f, f, ws, much, 8, 8, 8, nullptr), LORA_ERR_ALIAS);
  EXPECT(lora_linear_xent_bwd(x, w, t, g, h, nullptr, nullptr, ws, much, 8, 8, 8, nullptr), LORA_ERR_NULL);
  EXPECT(lora_linear_xent_bwd(x, w, t, g, h, y, y, ws, much, 8, 8, 8, nullptr), LORA_ERR_ALIAS);
  EXPECT(lora_linear_xent_step(x, w, t, h, f, y, dw, ws, 0, 8, 8, 8, nullptr), LORA_ERR_WORKSPACE);
  EXPECT(lora_linear_xent_step(x, w, t, h, f, w, nullptr, ws, much, 8, 8, 8, nullptr), LORA_ERR_ALIAS);
}

// Every kernel's assumptions on the shapes that its rule gives it.
static int plans() {
  using namespace lora;
  int checked = 0;
  const int64_t ms[] = {1, 2, 7, 16, 17, 32, 33, 64, 100, 128, 129, 500, 1025, 4096, 20000, 1 << 20};
  for (int64_t m : ms)
    for (int64_t n : {8, 64, 200, 1032, 4096, 11008, 32000, 128256, 1 << 20})
      for (int64_t k : {8, 264, 1000, 4096, 8192, 16392, 1 << 17}) {
        if (lora_linear_fp8_fwd_workspace_size(m, n, k) == 0) continue;
        const Fp8Plan f = plan_fp8_fwd(m, n, k), b = plan_fp8_bwd(m, n, k);
        const Fp8Layout lf = fp8_fwd_layout(m, n, k), lb = fp8_bwd_layout(m, n, k);
        HOLDS(f.grid >= 1 && f.grid < (int64_t(1) << 31) && f.splits >= 1, m, n, k);
        HOLDS(b.grid >= 1 && b.grid < (int64_t(1) << 31), m, n, k);
        HOLDS(b.splits >= 1 && b.splits <= fp8_blocks(n), m, n, k);   // no part of a contraction is empty
        if (f.kind <= FP8_TOKEN_2) HOLDS(m <= kFp8TokenRows && fp8_token_lds(m, k) <= 160 * 1024 && m * fp8_blocks(k) * 16 < (1 << 19), m, n, k);
        if (f.kind == FP8_FEW_1) HOLDS(m <= 16 && f.block == 512, m, n, k);
        if (f.kind == FP8_FEW_2) HOLDS(m <= 32 && f.block == 512, m, n, k);
        HOLDS(f.splits == 1 || f.kind == FP8_64x128_DEEP, m, n, k);   // the join's tiles have 64 rows
        HOLDS(b.splits == 1 || b.kind == FP8_BACK_64x256, m, n, k);
        HOLDS(f.splits <= fp8_blocks(k), m, n, k);
        HOLDS(lf.scales >= fp8_codes_bytes(m, k) && lf.sums >= lf.scales + fp8_scales_bytes(m, k, 1), m, n, k);
        HOLDS(lb.scales >= fp8_codes_bytes(m, n) && lb.sums >= lb.scales + fp8_scales_bytes(m, n, 1), m, n, k);
        HOLDS(lf.total >= lf.sums + (f.splits > 1 ? (size_t)f.grid * 64 * 128 * 4 : 0), m, n, k);
        HOLDS(lb.total >= lb.sums + (b.splits > 1 ? (size_t)b.grid * 64 * 256 * 4 : 0), m, n, k);
        // what the tiles' 32-bit offsets reach: 256 rows of codes, a stage's scales
        HOLDS(fp8_blocks(k) * 128 * 256 < (int64_t(1) << 31) && fp8_blocks(n) * 128 * 256 < (int64_t(1) << 31), m, n, k);
        HOLDS((int64_t)fp8_scales_bytes(m, k, 1) < (int64_t(1) << 31) && (int64_t)fp8_scales_bytes(m, n, 1) < (int64_t(1) << 31), m, n, k);
        ++checked;
      }
  for (int64_t rows : {1, 5, 16, 64, 65, 128, 129, 256, 500, 1500, 2049, 4096, 8192, 100000, 1 << 20})
    for (int64_t vocab : {1, 2, 127, 129, 1000, 8003, 32000, 50021, 131072, 1 << 20})
      for (int64_t k : {8, 72, 512, 4096, 5120, 8200, 1 << 16}) {
        if (lora_linear_xent_workspace_size(rows, vocab, k, 0, 0) == 0) continue;
        const XentPlan p = plan_xent(rows, vocab, k);
        HOLDS((int64_t)p.tiles_m * p.tile_m >= rows && p.rows_pad >= (int64_t)p.tiles_m * p.tile_m && p.rows_pad % p.tile_m == 0, rows, vocab, k);
        HOLDS(p.rows_pad >= (int64_t)p.grad_tiles_m * p.grad_m && (int64_t)p.grad_tiles_m * p.grad_m >= rows, rows, vocab, k);
        HOLDS((int64_t)p.vtiles * p.tile_n >= vocab && (int64_t)(p.vtiles - 1) * p.tile_n < vocab, rows, vocab, k);
        HOLDS((int64_t)p.pieces * p.piece_tiles >= p.vtiles && (int64_t)(p.pieces - 1) * p.piece_tiles < p.vtiles, rows, vocab, k);
        HOLDS(p.piece == (int64_t)p.piece_tiles * p.tile_n && p.piece % 64 == 0 && p.stages * 64 == p.piece, rows, vocab, k);
        HOLDS((int64_t)p.tiles_m * p.vtiles < (int64_t(1) << 31) && (int64_t)p.grad_tiles_m * p.tiles_k * p.splits < (int64_t(1) << 28), rows, vocab, k);
        HOLDS(p.splits >= 1, rows, vocab, k);
        for (int64_t sp = 0; p.local && sp < p.splits; ++sp) {   // the tiles of logits that a part of the contraction meets
          const int64_t s0 = p.stages * sp / p.splits, s1 = p.stages * (sp + 1) / p.splits, per = p.tile_n / 64;
          HOLDS(s1 <= s0 || (s1 - 1) / per - s0 / per + 1 <= local_tiles(p.grad_m), rows, vocab, k);
        }
        // what the tiles' 32-bit offsets reach: 256 rows of each operand
        HOLDS(p.piece * 2 * p.tile_m < (int64_t(1) << 31) && p.rows_pad * 2 * 256 < (int64_t(1) << 31) && k * 2 * 256 < (int64_t(1) << 31), rows, vocab, k);
        size_t last = 0;
        for (int d = 0; d < 4; ++d) {
          const XentLayout L = xent_layout(rows, vocab, k, d & 1, d >> 1);
          HOLDS(L.ref - L.coef >= (size_t)p.rows_pad * 8 && L.best - L.ref >= (size_t)p.rows_pad * 8 && L.parts - L.best >= (size_t)p.rows_pad * 8 && L.parts <= L.piece && L.piece <= L.turned && L.turned <= L.known && L.known <= L.sums && L.sums <= L.saved && L.saved <= L.total, rows, vocab, k);
          HOLDS(L.piece - L.parts >= (size_t)(p.vtiles * p.rows_pad * 8), rows, vocab, k);
          if (d) HOLDS(L.turned - L.piece >= (size_t)(p.rows_pad * p.piece * 2), rows, vocab, k);
          if (d & 2) HOLDS(L.known - L.turned >= (size_t)(p.rows_pad * p.piece * 2) && L.sums - L.known >= (size_t)(rows * k * 2) && L.total - L.saved >= (size_t)(rows * 8), rows, vocab, k);
          if (d & 1) HOLDS(L.saved - L.sums >= (size_t)p.splits * p.grad_tiles_m * p.grad_m * p.tiles_k * 256 * 4, rows, vocab, k);
          if (d != 2) HOLDS(L.total >= last, rows, vocab, k);   // a call with fewer outputs needs no more
          last = d == 2 ? last : L.total;
          ++checked;
        }
      }
  return checked;
}

int main(int argc, char** argv) {
  if (argc > 1) {
    for (int i = 2; i + 2 < argc; i += 3) {
      const int64_t m = atoll(argv[i]), n = atoll(argv[i + 1]), k = atoll(argv[i + 2]);
      if (strcmp(argv[1], "xent") == 0) {   // rows, vocab, k: its kernels, and whether there are parts to join and pieces
        const lora::XentPlan p = lora::plan_xent(m, n, k);
        printf("logits%d grad%d join%d pieces%d local%d dw%d\n", p.kind, p.grad_kind, p.splits > 1 ? p.grad_kind : -1, p.pieces > 1, p.local ? p.grad_kind : -1, p.dw_kind);
        continue;
      }
      const lora::Fp8Plan p = strcmp(argv[1], "fwd") == 0 ? lora::plan_fp8_fwd(m, n, k) : lora::plan_fp8_bwd(m, n, k);
      printf("%d%s\n", p.kind, p.splits > 1 ? "s" : "");
    }
    return 0;
  }
  refusals();
  const int n = plans();
  if (failures) return 1;
  printf("operators' sanitizer driver: ok, plans checked: %d\n", n);
  return 0;
}
