// Microscaled 4-bit matrices: quantisation, its inverse, and the linear layer
// Y = Q(X) Q(W)^T on the matrix cores' scaled 4-bit products.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes 16 rows of A and 16 of B over 128 k
// in 4 bits and a scale byte per row and 32 k.  With c = l % 16, g = l / 16,
// lane l holds row c, k = 32 g .. + 31 (16 bytes), and that block's scale; the
// result holds column c (B's row), rows 4 g .. 4 g + 3 (A's).  A row of 64 bytes
// so feeds the same product time as 32 bf16 k, and the operands of a 256-column
// slab (128 bytes a row) take two products.
#include <type_traits>

#include "lora_device.hpp"
#include "lora_ops.hpp"
#include "lora_plan.hpp"

namespace lora {

typedef int int8v __attribute__((ext_vector_type(8)));

// acc += A B^T over one 128-wide step; SA and SB pick the scale byte of sa and sb.
template <int SA, int SB>
__device__ __forceinline__ floatx4 mfma_mx4(int4v a, int4v b, floatx4 acc, int sa, int sb) {
  const int8v A{a[0], a[1], a[2], a[3], 0, 0, 0, 0}, B{b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, acc, 4, 4, SA, sa, SB, sb);
}

// Scale byte of a row's block within its cell; bytes of 32-row-block b of
// four rows 16 apart follow each other.
__device__ __forceinline__ int mx4_scale_offset(int row, int block) {
  return (block & 3) * 128 + (row & 15) * 8 + ((row >> 4) & 3) * 2 + ((block >> 2) & 1);
}

// ---------------------------------------------------------------------------
// Quantisation.  A workgroup takes a cell of scales, 64 rows x 256 columns: four
// lanes a block, each 8 columns.  Reads 2 bytes and writes 0.53 a column; bound
// by HBM.
__global__ __launch_bounds__(256) void lora_mx4_quantize_kernel(const u16* __restrict__ X, uint8_t* __restrict__ codes,
                                                                uint8_t* __restrict__ scales, int rows, int k,
                                                                int slabs, int groups) {
  __shared__ __attribute__((aligned(16))) uint8_t cell[512];
  const int slab = (int)blockIdx.x % slabs, grp = (int)blockIdx.x / slabs;
  const int tid = threadIdx.x, piece = tid & 31, col = slab * 256 + 8 * piece;
  const bool inside = col < k;
  int4v x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = grp * 64 + (tid >> 5) + 8 * i;
    x[i] = inside && row < rows ? *reinterpret_cast<const int4v*>(X + (size_t)row * k + col) : int4v{0, 0, 0, 0};
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int lrow = (tid >> 5) + 8 * i, row = grp * 64 + lrow;
    uint32_t top = 0;   // the largest magnitude's bits
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const uint32_t w = (uint32_t)x[i][h] & 0x7FFF7FFFu;
      top = max(top, max(w & 0xFFFFu, w >> 16));
    }
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const int field = (int)(top >> 7);
    const bool nan = field == 255;
    const int scale = nan ? 255 : max(field - 2, 0);
    // x 2^(127 - scale) is exact; the conversion rounds to nearest even and saturates
    const float up = __builtin_bit_cast(float, (uint32_t)(254 - scale) << 23);
    uint32_t out = 0;
    if (!nan) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = bf16_to_f32((u16)((uint32_t)x[i][e >> 1] >> (16 * (e & 1)))) * up;
      out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, y[0], y[1], 1.0f, 0);
      out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, y[2], y[3], 1.0f, 1);
      out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, y[4], y[5], 1.0f, 2);
      out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, y[6], y[7], 1.0f, 3);
    }
    const int block = slab * 8 + (piece >> 2);
    if ((piece & 3) == 0) cell[mx4_scale_offset(lrow, block)] = (uint8_t)(row < rows && block * 32 < k ? scale : 0);
    if (row < rows) *reinterpret_cast<uint32_t*>(codes + ((size_t)row * slabs + slab) * 128 + piece * 4) = out;
  }
  __syncthreads();
  if (tid < 32)
    reinterpret_cast<int4v*>(scales + ((size_t)slab * groups + grp) * 512)[tid] = reinterpret_cast<const int4v*>(cell)[tid];
}

// The values of codes and scales: a lane takes 8 columns.
__global__ __launch_bounds__(256) void lora_mx4_dequantize_kernel(const uint8_t* __restrict__ codes,
                                                                  const uint8_t* __restrict__ scales,
                                                                  u16* __restrict__ X, int rows, int k, int slabs,
                                                                  int groups) {
  const int slab = (int)blockIdx.x % slabs, grp = (int)blockIdx.x / slabs;
  const int tid = threadIdx.x, piece = tid & 31, col = slab * 256 + 8 * piece, block = slab * 8 + (piece >> 2);
  if (col >= k) return;
  const uint8_t* cell = scales + ((size_t)slab * groups + grp) * 512;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int lrow = (tid >> 5) + 8 * i, row = grp * 64 + lrow;
    if (row >= rows) continue;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + ((size_t)row * slabs + slab) * 128 + piece * 4);
    const int s = cell[mx4_scale_offset(lrow, block)];
    // 2^(s - 127); s = 0 is a subnormal, 255 NaN
    const uint32_t bits = s == 0 ? 0x00400000u : (s == 255 ? 0x7FC00000u : (uint32_t)s << 23);
    const float unit = __builtin_bit_cast(float, bits);
    const auto p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
    const auto p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
    const float y[8] = {p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
    int4v o;
#pragma unroll
    for (int h = 0; h < 4; ++h)
      o[h] = (int)((uint32_t)f32_to_bf16(y[2 * h] * unit) | ((uint32_t)f32_to_bf16(y[2 * h + 1] * unit) << 16));
    *reinterpret_cast<int4v*>(X + (size_t)row * k + col) = o;
  }
}

// ---------------------------------------------------------------------------
// Y = Q(X) Q(W)^T straight from memory: a workgroup forms 16 features x 16 TG
// tokens, its four waves taking the slabs in turn; their sums are added in wave
// order through LDS.
template <int TG>
__global__ __launch_bounds__(256) void lora_mx4_direct_kernel(const uint8_t* __restrict__ Xc,
                                                              const uint8_t* __restrict__ Xs,
                                                              const uint8_t* __restrict__ Wc,
                                                              const uint8_t* __restrict__ Ws, u16* __restrict__ Y, int m,
                                                              int n, int slabs, int tiles_n) {
  __shared__ floatx4 part[4][TG][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int g = lane >> 4, c = lane & 15;
  const int n0 = (int)(blockIdx.x % (unsigned)tiles_n) * 16, m0 = (int)(blockIdx.x / (unsigned)tiles_n) * 16 * TG;
  const int gw = (n + 63) / 64, gx = (m + 63) / 64;
  const int wrow = min(n0 + c, n - 1);
  const uint8_t* wp = Wc + (size_t)wrow * slabs * 128 + 16 * g;
  const uint8_t* wsp = Ws + (size_t)(wrow >> 6) * 512 + mx4_scale_offset(wrow, g);
  const uint8_t *xp[TG], *xsp[TG];
#pragma unroll
  for (int t = 0; t < TG; ++t) {
    const int row = min(m0 + 16 * t + c, m - 1);
    xp[t] = Xc + (size_t)row * slabs * 128 + 16 * g;
    xsp[t] = Xs + (size_t)(row >> 6) * 512 + mx4_scale_offset(row, g);
  }
  floatx4 acc[TG];
#pragma unroll
  for (int t = 0; t < TG; ++t) acc[t] = floatx4{0.f, 0.f, 0.f, 0.f};
  for (int s = wave; s < slabs; s += 4) {
    const int4v w0 = *reinterpret_cast<const int4v*>(wp + (size_t)s * 128);
    const int4v w1 = *reinterpret_cast<const int4v*>(wp + (size_t)s * 128 + 64);
    const int ws = *reinterpret_cast<const u16*>(wsp + (size_t)s * gw * 512);
#pragma unroll
    for (int t = 0; t < TG; ++t) {
      const int4v x0 = *reinterpret_cast<const int4v*>(xp[t] + (size_t)s * 128);
      const int4v x1 = *reinterpret_cast<const int4v*>(xp[t] + (size_t)s * 128 + 64);
      const int xs = *reinterpret_cast<const u16*>(xsp[t] + (size_t)s * gx * 512);
      acc[t] = mfma_mx4<0, 0>(w0, x0, acc[t], ws, xs);
      acc[t] = mfma_mx4<1, 1>(w1, x1, acc[t], ws, xs);
    }
  }
#pragma unroll
  for (int t = 0; t < TG; ++t) part[wave][t][lane] = acc[t];
  __syncthreads();
  for (int t = wave; t < TG; t += 4) {
    const floatx4 v = ((part[0][t][lane] + part[1][t][lane]) + part[2][t][lane]) + part[3][t][lane];
    const int row = m0 + 16 * t + c, col = n0 + 4 * g;
    if (row < m && col < n) {
      const uint32_t lo = (uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16);
      const uint32_t hi = (uint32_t)f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16);
      *reinterpret_cast<uint2*>(Y + (size_t)row * n + col) = uint2{lo, hi};
    }
  }
}

// ---------------------------------------------------------------------------
// 256 x 256 tiles: eight waves of 128 tokens x 64 features, two slabs in LDS,
// copied from memory straight into LDS (one 16-byte chunk a lane, the swizzle
// applied to the global addresses).
//
// A slab is two 128-wide steps.  A wave holds a step's fragments in registers
// and, as soon as the four products of a token fragment are issued, reads that
// fragment of the next step into its place; the feature fragments have a second
// set.  So no wave waits for LDS at a step's start.  The one barrier of a slab
// stands between its steps: every wave has read the whole slab, whose place the
// second step fills with the slab after next, and the next slab has landed.
//
// The scales go straight to registers, three 8-byte loads a wave and slab (64 of
// its tokens, the other 64, its features), a slab ahead of their use; they are
// issued after that slab's copies, so three loads may be under way when the
// copies are waited for.
template <typename F, int... I>
__device__ __forceinline__ void each_const(std::integer_sequence<int, I...>, F&& f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void unrolled(F&& f) {
  each_const(std::make_integer_sequence<int, N>{}, f);
}

__global__ __launch_bounds__(512) void lora_mx4_big_kernel(const uint8_t* __restrict__ Xc,
                                                           const uint8_t* __restrict__ Xs,
                                                           const uint8_t* __restrict__ Wc,
                                                           const uint8_t* __restrict__ Ws, u16* __restrict__ Y, int m,
                                                           int n, int slabs, int tiles_m, int tiles_n) {
  constexpr int BM = 256, BN = 256, STAGE = (BM + BN) * 128;
  __shared__ __attribute__((aligned(1024))) char smem[2 * STAGE];
  int tm, tn;
  tile_coords(tiles_m, tiles_n, 8, (int)blockIdx.x, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int wm = wave >> 2, wn = wave & 3;
  const int g = lane >> 4, c16 = lane & 15;

  const uint32_t rowbytes = (uint32_t)slabs * 128;
  const __amdgpu_buffer_rsrc_t rsX = make_rsrc(Xc + (size_t)m0 * rowbytes, (uint64_t)min(BM, m - m0) * rowbytes);
  const __amdgpu_buffer_rsrc_t rsW = make_rsrc(Wc + (size_t)n0 * rowbytes, (uint64_t)min(BN, n - n0) * rowbytes);
  // scales from the wave's first cell on (cells past the matrix: another's, or zeros past the end)
  const int gx = (m + 63) / 64, gw = (n + 63) / 64, cx = m0 / 64 + 2 * wm, cw = n0 / 64 + wn;
  const __amdgpu_buffer_rsrc_t rsXs = make_rsrc(Xs, (uint64_t)gx * slabs * 512);
  const __amdgpu_buffer_rsrc_t rsWs = make_rsrc(Ws, (uint64_t)gw * slabs * 512);
  const uint32_t cell = (uint32_t)(g * 128 + c16 * 8);

  floatx4 acc[4][8];           // 16 x 16 fragments: [features 16 a ..][tokens 16 b ..] of the wave's 64 x 128
#pragma unroll
  for (int a = 0; a < 4; ++a)
#pragma unroll
    for (int b = 0; b < 8; ++b) acc[a][b] = floatx4{0.f, 0.f, 0.f, 0.f};
  int4v fw[2][4], fx[8];         // W fragments of both steps, X fragments of the current one
  uint2 sx[2], sw, sx1[2], sw1;  // scales of this slab (two token cells, the feature cell) and the next

  // a wave copies 8 rows of X and of W per instruction, four of each a slab
  const int l8 = lane >> 3, crow = 8 * wave;
  const uint32_t kcol = (uint32_t)(((lane & 7) ^ kc_swz(crow + l8)) << 4);
  const uint32_t coff = (uint32_t)(crow + l8) * rowbytes + kcol;
  auto copy = [&](int kb, int i) LORA_INLINE {
    char* sb = smem + (kb & 1) * STAGE + (crow + 64 * i) * 128;
    dma16(rsX, coff + (uint32_t)(64 * i) * rowbytes, (uint32_t)kb * 128, sb);
    dma16(rsW, coff + (uint32_t)(64 * i) * rowbytes, (uint32_t)kb * 128, sb + BM * 128);
  };
  auto load_scales = [&](int kb) LORA_INLINE {   // three loads, in this place
    __builtin_amdgcn_sched_barrier(0);
    sx1[0] = buf_load8(rsXs, ((uint32_t)kb * gx + cx) * 512 + cell);
    sx1[1] = buf_load8(rsXs, ((uint32_t)kb * gx + cx + 1) * 512 + cell);
    sw1 = buf_load8(rsWs, ((uint32_t)kb * gw + cw) * 512 + cell);
    __builtin_amdgcn_sched_barrier(0);
  };
  const uint32_t fbase = kc_offset(c16, g);      // (rows 16 apart swizzle alike; step 1: chunk 4 further)
  auto read_x = [&](int kb, int step, int b) LORA_INLINE {
    const char* xs = smem + (kb & 1) * STAGE + wm * 128 * 128;
    fx[b] = *reinterpret_cast<const int4v*>(xs + (fbase ^ (step << 6)) + 16 * 128 * b);
  };
  auto read_w = [&](int kb, int step) LORA_INLINE {
    const char* ws = smem + (kb & 1) * STAGE + (BM + wn * 64) * 128;
#pragma unroll
    for (int a = 0; a < 4; ++a)
      fw[step][a] = *reinterpret_cast<const int4v*>(ws + (fbase ^ (step << 6)) + 16 * 128 * a);
  };
  // products of a step; after each token fragment's four, f(its index)
  auto products = [&](auto stepc, auto&& f) LORA_INLINE {
    constexpr int S = decltype(stepc)::value;
    unrolled<8>([&](auto bc) LORA_INLINE {
      constexpr int B = decltype(bc)::value;
      const int sb = (int)((B >> 1) & 1 ? sx[B >> 2].y : sx[B >> 2].x);
      unrolled<4>([&](auto ac) LORA_INLINE {
        constexpr int A = decltype(ac)::value;
        const int sa = (int)(A >> 1 ? sw.y : sw.x);
        acc[A][B] = mfma_mx4<2 * (A & 1) + S, 2 * (B & 1) + S>(fw[S][A], fx[B], acc[A][B], sa, sb);
      });
      __builtin_amdgcn_sched_barrier(0);
      f(B);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  using I2 = std::integral_constant<int, 2>;
  auto slab = [&](int kb, auto mode) LORA_INLINE {   // 0: steady, 1: the last but one, 2: the last
    constexpr int MODE = decltype(mode)::value;
    sx[0] = sx1[0];
    sx[1] = sx1[1];
    sw = sw1;
    if constexpr (MODE < 2) load_scales(kb + 1);
    products(I0{}, [&](int b) LORA_INLINE {
      if (b == 1) read_w(kb, 1);
      read_x(kb, 1, b);
    });
    if constexpr (MODE < 2) {
      copy_barrier<3>();   // every wave has read this slab, and the next one has landed
      read_w(kb + 1, 0);
    }
    products(I1{}, [&](int b) LORA_INLINE {
      if constexpr (MODE == 0)
        if (b < 4) copy(kb + 2, b);
      if constexpr (MODE < 2) read_x(kb + 1, 0, b);
    });
  };
  load_scales(0);
#pragma unroll
  for (int i = 0; i < 4; ++i) copy(0, i);
  if (slabs > 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) copy(1, i);
    copy_barrier<8>();
  } else {
    copy_barrier<0>();
  }
  read_w(0, 0);
#pragma unroll
  for (int b = 0; b < 8; ++b) read_x(0, 0, b);
  int kb = 0;
  for (; kb + 2 < slabs; ++kb) slab(kb, I0{});
  if (slabs > 1) slab(kb++, I1{});
  slab(kb, I2{});

  // Y: each wave's blocks of 32 tokens x 64 features through a region of LDS of its own
  constexpr int OUT = out16_bytes<4, 2>();
  static_assert(8 * OUT <= 2 * STAGE, "output staging");
  __syncthreads();
  const int j0 = n0 + wn * 64;
#pragma unroll
  for (int fi = 0; fi < 4; ++fi) {
    const int i0 = m0 + wm * 128 + 32 * fi;
    floatx4 v[4][2];
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      v[a][0] = acc[a][2 * fi];
      v[a][1] = acc[a][2 * fi + 1];
    }
    store_out16<4, 2>(v, smem + wave * OUT, Y + (size_t)i0 * n + j0, (size_t)n, m - i0, n - j0, lane);
  }
}

hipError_t launch_mx4_quantize(const Mx4QuantArgs& a, hipStream_t st) {
  const int slabs = (int)mx4_slabs(a.k), groups = (int)mx4_groups(a.rows);
  hipLaunchKernelGGL(lora_mx4_quantize_kernel, dim3((unsigned)(slabs * groups)), dim3(256), 0, st, a.X, a.codes, a.scales,
                     (int)a.rows, (int)a.k, slabs, groups);
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, uint16_t* X, int64_t rows, int64_t k,
                                 hipStream_t st) {
  const int slabs = (int)mx4_slabs(k), groups = (int)mx4_groups(rows);
  hipLaunchKernelGGL(lora_mx4_dequantize_kernel, dim3((unsigned)(slabs * groups)), dim3(256), 0, st, codes, scales, X,
                     (int)rows, (int)k, slabs, groups);
  return hipGetLastError();
}

hipError_t launch_mx4_fwd(const Mx4FwdArgs& a, hipStream_t st) {
  const Mx4Layout L = mx4_fwd_layout(a.m, a.n, a.k);
  uint8_t* xc = reinterpret_cast<uint8_t*>(a.ws + L.xc);
  uint8_t* xs = reinterpret_cast<uint8_t*>(a.ws + L.xs);
  const hipError_t e = launch_mx4_quantize(Mx4QuantArgs{a.X, xc, xs, a.m, a.k}, st);
  if (e != hipSuccess) return e;
  if (a.m > 64) {
    const int tm = (int)((a.m + 255) / 256), tn = (int)((a.n + 255) / 256);
    hipLaunchKernelGGL(lora_mx4_big_kernel, dim3((unsigned)(tm * tn)), dim3(512), 0, st, xc, xs, a.Wc, a.Ws, a.Y,
                       (int)a.m, (int)a.n, (int)mx4_slabs(a.k), tm, tn);
    return hipGetLastError();
  }
  constexpr int TG = 4;
  const int tiles_n = (int)((a.n + 15) / 16);
  const int64_t tiles_m = (a.m + 16 * TG - 1) / (16 * TG);
  hipLaunchKernelGGL((lora_mx4_direct_kernel<TG>), dim3((unsigned)(tiles_m * tiles_n)), dim3(256), 0, st, xc, xs, a.Wc,
                     a.Ws, a.Y, (int)a.m, (int)a.n, (int)mx4_slabs(a.k), tiles_n);
  return hipGetLastError();
}

}  // namespace lora
