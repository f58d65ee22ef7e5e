// Dropout whose mask is drawn again wherever it is needed:
//   Y = residual + keep X / (1 - p),
// element e of the tensor in row-major order kept iff its draw, the 16 bits e % 16
// of the Philox4x64-10 block at counter offset + e / 16 (lora_mask.hip, whose
// packed masks hold the same bits), is below floor((1 - p) 2^16 + 1/2).  The
// gradient is the same call on dY without the residual.
//
// A thread makes the 16 elements of a block.
#include "lora_device.hpp"
#include "lora_philox.hpp"
#include "lora_train.hpp"

namespace lora {

template <bool F32>
__device__ __forceinline__ float load_elem(const void* p, int64_t i) {
  if constexpr (F32) return static_cast<const float*>(p)[i];
  else return bf16_to_f32(static_cast<const u16*>(p)[i]);
}

// X, residual and Y may be the same tensor: a thread has read its elements before it
// writes them.
template <bool F32, bool RES>
__global__ __launch_bounds__(256) void lora_dropout_kernel(const void* X, const void* R, void* Y, int64_t count,
                                                           uint64_t seed, uint64_t offset, uint32_t thr, float scale) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, e0 = 16 * t;
  if (e0 >= count) return;
  constexpr int W = F32 ? 4 : 2;   // 16-byte loads of 16 elements
  int4v x[W], r[W];
  const bool whole = e0 + 16 <= count;
  if (whole) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      x[i] = static_cast<const int4v*>(X)[W * t + i];
      if constexpr (RES) r[i] = static_cast<const int4v*>(R)[W * t + i];
    }
  }
  uint64_t c[4] = {0ull, 0ull, 0ull, 0ull};
  if (thr < 65536u) philox_block(seed, offset, (uint64_t)t, c);   // (p = 0 keeps every draw)
  auto value = [&](int e, float xv, float rv) LORA_INLINE {
    const float y = philox_draw(c, e) < thr ? xv * scale : 0.0f;
    return RES ? y + rv : y;
  };
  if (whole) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      int4v o;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        if constexpr (F32) {
          o[h] = __builtin_bit_cast(int, value(4 * i + h, __builtin_bit_cast(float, (int)x[i][h]),
                                               RES ? __builtin_bit_cast(float, (int)r[i][h]) : 0.0f));
        } else {
          const uint32_t xw = (uint32_t)x[i][h], rw = RES ? (uint32_t)r[i][h] : 0u;
          const float lo = value(8 * i + 2 * h, bf16_to_f32((u16)xw), bf16_to_f32((u16)rw));
          const float hi = value(8 * i + 2 * h + 1, bf16_to_f32((u16)(xw >> 16)), bf16_to_f32((u16)(rw >> 16)));
          o[h] = (int)((uint32_t)f32_to_bf16(lo) | ((uint32_t)f32_to_bf16(hi) << 16));
        }
      }
      static_cast<int4v*>(Y)[W * t + i] = o;
    }
  } else {
    for (int e = 0; e0 + e < count; ++e) {
      const uint32_t draw = (uint32_t)((e < 8 ? (e < 4 ? c[0] : c[1]) : (e < 12 ? c[2] : c[3])) >> (16 * (e & 3))) & 0xFFFFu;
      float y = draw < thr ? load_elem<F32>(X, e0 + e) * scale : 0.0f;
      if constexpr (RES) y += load_elem<F32>(R, e0 + e);
      if constexpr (F32) static_cast<float*>(Y)[e0 + e] = y;
      else static_cast<u16*>(Y)[e0 + e] = f32_to_bf16(y);
    }
  }
}

template <bool F32, bool RES>
static hipError_t run_dropout(const DropoutArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((lora_dropout_kernel<F32, RES>), dim3((unsigned)cdiv(cdiv(a.count, 16), 256)), dim3(256), 0, st, a.X,
                     a.residual, a.Y, a.count, a.seed, a.offset, a.thr, a.scale);
  return hipGetLastError();
}

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t st) {
  if (a.f32) return a.residual ? run_dropout<true, true>(a, st) : run_dropout<true, false>(a, st);
  return a.residual ? run_dropout<false, true>(a, st) : run_dropout<false, false>(a, st);
}

}  // namespace lora
