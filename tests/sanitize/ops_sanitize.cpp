// Memory- and UB-checking driver for the C ABI of the operators around the
// layer's output and for their launch rules, built with the address and
// undefined-behaviour sanitizers on the host by tests/test_ops_plan.py.  It runs
// without a GPU: every entry-point call below is invalid and must be rejected,
// with the expected status, before any HIP call.  Device pointers are fake
// addresses that validation never reads.
//
// With arguments m n k m n k ... it prints the kernel kind of each 4-bit forward.
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "lora_linear.h"
#include "lora_ops.hpp"

static int failures = 0;

#define EXPECT(call, want)                                                                      \
  do {                                                                                          \
    const long got_ = (long)(call);                                                             \
    if (got_ != (long)(want)) {                                                                 \
      fprintf(stderr, "line %d: %s returned %ld, expected %ld\n", __LINE__, #call, got_, (long)(want)); \
      ++failures;                                                                               \
    }                                                                                           \
  } while (0)
#define HOLDS(cond, ...)                          \
  do {                                            \
    if (!(cond)) {                                \
      fprintf(stderr, "line %d: %s: ", __LINE__, #cond); \
      fprintf(stderr, __VA_ARGS__);               \
      fprintf(stderr, "\n");                      \
      ++failures;                                 \
    }                                             \
  } while (0)

template <typename T>
static T* dev(int i, uintptr_t off = 0) {
  return reinterpret_cast<T*>((uintptr_t(1) << 40) + uintptr_t(i) * (uintptr_t(1) << 36) + off);
}

static void refusals() {
  lora_bf16 *x = dev<lora_bf16>(0), *y = dev<lora_bf16>(3);
  uint8_t *c = dev<uint8_t>(1), *s = dev<uint8_t>(2);
  const int64_t top64 = INT64_MAX, low64 = INT64_MIN;
  EXPECT(lora_mx4_quantize(x, nullptr, s, 8, 8, nullptr), LORA_ERR_NULL);
  EXPECT(lora_mx4_quantize(x, c, s, 8, 12, nullptr), LORA_ERR_SHAPE);
  EXPECT(lora_mx4_quantize(x, c, s, top64, top64 - 7, nullptr), LORA_ERR_UNSUPPORTED);
  EXPECT(lora_mx4_quantize(x, c, s, low64, 8, nullptr), LORA_ERR_SHAPE);
  EXPECT(lora_mx4_dequantize(c, s, dev<lora_bf16>(0, 2), 8, 8, nullptr), LORA_ERR_ALIGN);
  EXPECT(lora_linear_mx4_fwd(x, c, s, y, dev<void>(4), 0, 8, 8, 8, nullptr), LORA_ERR_WORKSPACE);
  EXPECT(lora_linear_mx4_fwd(x, c, s, y, dev<void>(4), 1 << 30, top64, 8, 8, nullptr), LORA_ERR_UNSUPPORTED);
  EXPECT(lora_linear_mx4_fwd(x, c, s, x, dev<void>(4), 1 << 30, 8, 8, 8, nullptr), LORA_ERR_ALIAS);
  EXPECT(lora_mx4_codes_size(top64, top64), 0);
  EXPECT(lora_mx4_scales_size(low64, 8), 0);
  EXPECT(lora_linear_mx4_fwd_workspace_size(8, top64, 8), 0);
  float *f = dev<float>(5), *g = dev<float>(6), *h = dev<float>(9), *q = dev<float>(10);
  int32_t *t = dev<int32_t>(7), *ids = dev<int32_t>(8);
  EXPECT(lora_token_logprobs(x, LORA_BF16, 100, t, 1.f, f, nullptr, ids, h, dev<void>(4), 1 << 20, 8, 100, 4, nullptr), LORA_ERR_NULL);
  EXPECT(lora_token_logprobs(x, LORA_BF16, top64, t, 1.f, f, g, ids, h, dev<void>(4), 1 << 20, 8, 100, 4, nullptr), LORA_ERR_UNSUPPORTED);
  EXPECT(lora_token_logprobs(x, LORA_BF16, 99, t, 1.f, f, g, ids, h, dev<void>(4), 1 << 20, 8, 100, 4, nullptr), LORA_ERR_SHAPE);
  EXPECT(lora_token_logprobs(x, LORA_BF16, 100, t, 1.f, f, g, ids, h, dev<void>(4), 8, 8, 100, 4, nullptr), LORA_ERR_WORKSPACE);
  EXPECT(lora_token_logprobs(x, (lora_dtype)7, 100, t, 1.f, f, g, ids, h, dev<void>(4), 1 << 20, 8, 100, 4, nullptr), LORA_ERR_UNSUPPORTED);
  EXPECT(lora_token_logprobs_workspace_size(top64, top64, top64), 0);
  EXPECT(lora_token_logprobs_workspace_size(low64, 100, 4), 0);
  EXPECT(lora_distill_fwd(x, LORA_F32, 100, ids, f, nullptr, 1.f, 0.5f, g, h, 8, 100, 4, nullptr), LORA_ERR_NULL);
  EXPECT(lora_distill_fwd(x, LORA_F32, 100, ids, f, t, 0.f, 0.5f, g, h, 8, 100, 4, nullptr), LORA_ERR_SHAPE);
  EXPECT(lora_distill_bwd(x, LORA_F32, 100, ids, f, t, 1.f, 0.5f, h, g, dev<float>(0, 16), 8, 100, 4, nullptr), LORA_ERR_ALIAS);
  EXPECT(lora_distill_step(x, LORA_F32, 100, ids, f, t, 1.f, 2.f, g, h, q, 8, 100, 4, nullptr), LORA_ERR_SHAPE);
  EXPECT(lora_distill_step(x, LORA_F32, 100, ids, f, t, 1.f, 0.5f, g, h, q, 8, 100, 129, nullptr), LORA_ERR_UNSUPPORTED);
}

// Every kernel's assumptions on the shapes that its rule gives it.
static int plans() {
  using namespace lora;
  int checked = 0;
  for (int64_t m : {1, 2, 7, 16, 17, 32, 33, 100, 500, 1025, 4096, 20000, 1 << 20})
    for (int64_t n : {8, 64, 200, 1032, 4096, 11008, 32000, 128256, 1 << 20})
      for (int64_t k : {8, 264, 1000, 4096, 8192, 16392, 1 << 17}) {
        if (m * k > (1 << 30) || n * k > (1 << 30) || m * n > (1 << 30)) continue;
        const Mx4Plan p = plan_mx4_fwd(m, n, k);
        HOLDS(p.grid >= 1 && p.grid < (int64_t(1) << 31) && p.grid == (int64_t)p.tiles_m * p.tiles_n, "%ld %ld %ld", (long)m, (long)n, (long)k);
        HOLDS(p.block >= 64 && p.block <= 1024, "%d", p.block);
        if (p.kind <= MX4_TOKEN_2) HOLDS(m <= kTokenRows && mx4_token_lds(mx4_slabs(k)) <= 160 * 1024, "%ld %ld", (long)m, (long)k);
        if (p.kind == MX4_FEW_1) HOLDS(m <= 16, "%ld", (long)m);
        if (p.kind == MX4_FEW_2) HOLDS(m <= 32, "%ld", (long)m);
        const Mx4Layout L = mx4_fwd_layout(m, n, k);
        HOLDS(L.total >= mx4_codes_bytes(m, k) + mx4_scales_bytes(m, k) && L.total == lora_linear_mx4_fwd_workspace_size(m, n, k), "%zu", L.total);
        ++checked;
      }
  for (int elem : {2, 4})
    for (int64_t vocab = 1; vocab <= 1 << 20; vocab += 1 + vocab / 3)
      for (int64_t head = 0; head < 16 / elem && head <= vocab; ++head) {
        const int64_t chunks = (vocab - head) * elem / 16, units = (chunks + kUnitBytes / 16 - 1) / (kUnitBytes / 16);
        HOLDS(units + 1 <= score_units(vocab, elem) && score_units(vocab, elem) <= kMaxUnits, "%ld", (long)vocab);
        const RowShape s = row_shape(vocab, elem);
        HOLDS(s.keep == 0 || chunks <= (int64_t)s.threads * s.keep, "%ld", (long)vocab);
        HOLDS((int64_t)grad_parts(vocab, elem) * kGradThreads * kGradKeep >= chunks, "%ld", (long)vocab);
        for (int64_t rows : {1, 3, 16, 100, 256, 257, 768, 769, 5000, 1 << 21}) {
          for (int least : {1, 4})
            if (read_threads(rows, vocab, elem, least) == 256) HOLDS(units + 1 <= kSmallUnits, "%ld %ld", (long)rows, (long)vocab);
          for (int64_t top : {0, 1, 5, 50, 128}) {
            if (top > vocab) continue;
            const int parts = score_parts(rows, vocab, elem, top);
            HOLDS(parts >= 1 && parts * top <= kMaxKeys && rows * parts <= std::max<int64_t>(256, rows), "%ld %ld", (long)rows, (long)vocab);
            // each part holds `top` values or more
            if (parts > 1) HOLDS(units / parts >= 15, "%ld units in %d parts", (long)units, parts);
            if (parts > 1) {
              char* base = dev<char>(1);
              const ScoreParts w(base, rows, vocab, elem, parts, top);
              HOLDS((size_t)(reinterpret_cast<char*>(w.units) - base) + sizeof(Unit) * rows * w.units_ld <= lora_token_logprobs_workspace_size(rows, vocab, top), "%ld %ld", (long)rows, (long)vocab);
            }
            HOLDS(lora_token_logprobs_workspace_size(rows, vocab, top) > 0 || rows * vocab > (int64_t(1) << 34), "%ld %ld", (long)rows, (long)vocab);
            ++checked;
          }
        }
      }
  return checked;
}

int main(int argc, char** argv) {
  if (argc > 1) {
    for (int i = 1; i + 2 < argc; i += 3)
      printf("%d\n", (int)lora::plan_mx4_fwd(atoll(argv[i]), atoll(argv[i + 1]), atoll(argv[i + 2])).kind);
    return 0;
  }
  refusals();
  const int n = plans();
  if (failures) return 1;
  printf("operators' sanitizer driver: ok, plans checked: %d\n", n);
  return 0;
}
