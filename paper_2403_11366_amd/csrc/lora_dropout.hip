// Dropout whose mask is drawn again wherever it is needed:
//   Y = residual + keep X / (1 - p),
// element e of the tensor in row-major order kept iff its draw, the 16 bits e % 16
// of the Philox4x64-10 block at counter offset + e / 16 (lora_mask.hip, whose
// packed masks hold the same bits), is below floor((1 - p) 2^16 + 1/2).  The
// gradient is the same call on dY without the residual.
//
// A thread draws a block.  bf16: it takes the block's 32 bytes.  fp32: its 64 bytes
// would leave lanes' loads 64 bytes apart; through LDS each lane gets the draws of four
// 16-byte pieces instead, a load of the wave's being one run of 1 KiB (8192 x 4096: 60.8
// -> 46.7 us, with a residual 82 -> 71; bf16 gained nothing from it).  Bounded by
// memory where there is much of it -- 8192 x 4096 bf16 with a residual 35.8 us, 5.6 TB/s
// -- the ten rounds of 64-bit products hiding behind it; else by the launch (129 x 4099
// 2.9 us of the kernel's, 6.1 with its call).
#include "lora_device.hpp"
#include "lora_philox.hpp"
#include "lora_train.hpp"

namespace lora {

// X, residual and Y may be the same tensor: a thread has read its elements before it
// writes them.
template <bool RES>
__global__ __launch_bounds__(256) void lora_dropout_kernel(const u16* X, const u16* R, u16* Y, int64_t count, uint64_t seed,
                                                           uint64_t offset, uint32_t thr, float scale) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, e0 = 16 * t;
  if (e0 >= count) return;
  int4v x[2], r[2];
  const bool whole = e0 + 16 <= count;
  if (whole) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[i] = reinterpret_cast<const int4v*>(X)[2 * t + i];
      if constexpr (RES) r[i] = reinterpret_cast<const int4v*>(R)[2 * t + i];
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
    for (int i = 0; i < 2; ++i) {
      int4v o;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const uint32_t xw = (uint32_t)x[i][h], rw = RES ? (uint32_t)r[i][h] : 0u;
        const float lo = value(8 * i + 2 * h, bf16_to_f32((u16)xw), bf16_to_f32((u16)rw));
        const float hi = value(8 * i + 2 * h + 1, bf16_to_f32((u16)(xw >> 16)), bf16_to_f32((u16)(rw >> 16)));
        o[h] = (int)((uint32_t)f32_to_bf16(lo) | ((uint32_t)f32_to_bf16(hi) << 16));
      }
      reinterpret_cast<int4v*>(Y)[2 * t + i] = o;
    }
  } else {
    for (int e = 0; e0 + e < count; ++e) {
      const uint32_t draw = (uint32_t)((e < 8 ? (e < 4 ? c[0] : c[1]) : (e < 12 ? c[2] : c[3])) >> (16 * (e & 3))) & 0xFFFFu;
      float y = draw < thr ? bf16_to_f32(X[e0 + e]) * scale : 0.0f;
      if constexpr (RES) y += bf16_to_f32(R[e0 + e]);
      Y[e0 + e] = f32_to_bf16(y);
    }
  }
}

// fp32, four draws a word of a block: word w of the wave's 256 is its 16-byte piece w's.
template <bool RES>
__global__ __launch_bounds__(256) void lora_dropout_f32_kernel(const float* X, const float* R, float* Y, int64_t count,
                                                               uint64_t seed, uint64_t offset, uint32_t thr, float scale) {
  __shared__ __attribute__((aligned(16))) uint64_t lds[4][256];
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
  const int64_t first = (int64_t)blockIdx.x * 4096 + wave * 1024, left = count - first;   // the wave's elements
  const float *x = X + first, *r = RES ? R + first : nullptr;
  float* y = Y + first;
  const bool whole = left >= 1024;   // of all but the tensor's last wave
  floatx4 xv[4], rv[4];
  if (whole) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      xv[j] = reinterpret_cast<const floatx4*>(x)[64 * j + lane];
      if constexpr (RES) rv[j] = reinterpret_cast<const floatx4*>(r)[64 * j + lane];
    }
  }
  uint64_t c[4] = {0ull, 0ull, 0ull, 0ull};
  if (thr < 65536u) philox_block(seed, offset, (uint64_t)blockIdx.x * 256 + threadIdx.x, c);
#pragma unroll
  for (int i = 0; i < 4; ++i) lds[wave][4 * lane + i] = c[i];
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");   // the wave's own, in order
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
  for (int j = 0; j < 4; ++j) c[j] = lds[wave][64 * j + lane];
  auto value = [&](int e, float xe, float re) LORA_INLINE {
    const float v = philox_draw(c, e) < thr ? xe * scale : 0.0f;
    return RES ? v + re : v;
  };
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    floatx4 o;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const int e = 256 * j + 4 * lane + h;
      if (whole) o[h] = value(4 * j + h, xv[j][h], RES ? rv[j][h] : 0.0f);
      else if (e < left) y[e] = value(4 * j + h, x[e], RES ? r[e] : 0.0f);
    }
    if (whole) reinterpret_cast<floatx4*>(y)[64 * j + lane] = o;
  }
}

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)cdiv(cdiv(a.count, 16), 256));
  auto run = [&](auto kernel, auto type) {
    using T = decltype(type);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, static_cast<const T*>(a.X), static_cast<const T*>(a.residual),
                       static_cast<T*>(a.Y), a.count, a.seed, a.offset, a.thr, a.scale);
    return hipGetLastError();
  };
  if (a.f32) return a.residual ? run(lora_dropout_f32_kernel<true>, float{}) : run(lora_dropout_f32_kernel<false>, float{});
  return a.residual ? run(lora_dropout_kernel<true>, u16{}) : run(lora_dropout_kernel<false>, u16{});
}

}  // namespace lora
