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
typedef int int2v __attribute__((ext_vector_type(2)));

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

// Eight columns of a block that four neighbouring lanes hold: their codes and the
// block's scale byte.
__device__ __forceinline__ uint32_t quantise_piece(const int4v& x, int& scale) {
  uint32_t top = 0;   // the largest magnitude's bits
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const uint32_t w = (uint32_t)x[h] & 0x7FFF7FFFu;
    top = max(top, max(w & 0xFFFFu, w >> 16));
  }
  top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xf, 0xf, true));   // lane ^ 1
  top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xf, 0xf, true));   // lane ^ 2
  const int field = (int)(top >> 7);
  const bool nan = field == 255;
  scale = nan ? 255 : max(field - 2, 0);
  // x 2^(127 - scale) is exact; the conversion rounds to nearest even and saturates
  const float up = __builtin_bit_cast(float, (uint32_t)(nan ? 0 : 254 - scale) << 23);
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = bf16_to_f32((u16)((uint32_t)x[e >> 1] >> (16 * (e & 1)))) * up;
  uint32_t out = 0;
  out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, y[0], y[1], 1.0f, 0);
  out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, y[2], y[3], 1.0f, 1);
  out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, y[4], y[5], 1.0f, 2);
  out = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(out, y[6], y[7], 1.0f, 3);
  return nan ? 0u : out;
}

// ---------------------------------------------------------------------------
// Quantisation.  A workgroup takes 16 rows x 256 columns, a quarter of a cell of
// scales: four rows and those 16, 32 and 48 after them, whose scales stand
// together.  Four lanes a block, each 8 columns.  Reads 2 bytes and writes 0.53 a
// column; bound by HBM: 11008 x 4096 in 21 us, 5.4 TB/s, run after run (30.6 with
// workgroups of whole cells, whose 2752 leave the last third of the run half empty);
// 26 right behind the inverse, whose stores are still on their way to memory.
__global__ __launch_bounds__(256) void lora_mx4_quantize_kernel(const u16* __restrict__ X, uint8_t* __restrict__ codes,
                                                                uint8_t* __restrict__ scales, int rows, int k,
                                                                int slabs, int groups) {
  __shared__ __attribute__((aligned(16))) uint8_t cell[128];   // [block & 3][32]
  const int slab = (int)blockIdx.x % slabs, quarter = (int)blockIdx.x / slabs, grp = quarter >> 2;
  const int tid = threadIdx.x, piece = tid & 31, col = slab * 256 + 8 * piece;
  const bool inside = col < k;
  int4v x[2];
  int lrow[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = (tid >> 5) + 8 * i;
    lrow[i] = 4 * (quarter & 3) + (r & 3) + 16 * (r >> 2);
    const int row = grp * 64 + lrow[i];
    x[i] = inside && row < rows ? *reinterpret_cast<const int4v*>(X + (size_t)row * k + col) : int4v{0, 0, 0, 0};
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = grp * 64 + lrow[i];
    int scale;
    const uint32_t out = quantise_piece(x[i], scale);
    const int block = slab * 8 + (piece >> 2), at = mx4_scale_offset(lrow[i], block);
    if ((piece & 3) == 0) cell[(at >> 7) * 32 + (at & 31)] = (uint8_t)(row < rows && block * 32 < k ? scale : 0);
    if (row < rows) *reinterpret_cast<uint32_t*>(codes + ((size_t)row * slabs + slab) * 128 + piece * 4) = out;
  }
  __syncthreads();
  if (tid < 32)
    *reinterpret_cast<uint32_t*>(scales + ((size_t)slab * groups + grp) * 512 + (tid >> 3) * 128 + (quarter & 3) * 32 +
                                 (tid & 7) * 4) = reinterpret_cast<const uint32_t*>(cell)[tid];
}

// The values of codes and scales: a lane takes 8 columns of two rows, a workgroup
// 16 rows x 256 columns.  Bound by HBM: 11008 x 4096 in 25 us, 4.5 TB/s, run after
// run; 18 right behind the quantisation, with codes still in the caches.
__global__ __launch_bounds__(256) void lora_mx4_dequantize_kernel(const uint8_t* __restrict__ codes,
                                                                  const uint8_t* __restrict__ scales,
                                                                  u16* __restrict__ X, int rows, int k, int slabs,
                                                                  int groups) {
  const int slab = (int)blockIdx.x % slabs, r0 = (int)blockIdx.x / slabs * 16, grp = r0 >> 6;
  const int tid = threadIdx.x, piece = tid & 31, col = slab * 256 + 8 * piece, block = slab * 8 + (piece >> 2);
  if (col >= k) return;
  const uint8_t* cell = scales + ((size_t)slab * groups + grp) * 512;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = r0 + (tid >> 5) + 8 * i;
    if (row >= rows) continue;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + ((size_t)row * slabs + slab) * 128 + piece * 4);
    const int s = cell[mx4_scale_offset(row & 63, block)];
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
// Few tokens: a workgroup forms 16 FG features x 16 TG tokens with its eight
// waves on different slabs, straight from memory without a barrier until the
// waves' sums are added, in wave order, through LDS.  A lane loads the 16 bytes
// of codes that it multiplies; each wave has the next slab's loads in flight
// under the current one's products.  Bound by the latency of a wave's few slabs:
// 128 x 4096 x 4096 9.8 us, 11.4 on 64 x 128 tiles (the quantisation, 2.5, apart).
template <int TG, int FG>
__global__ __launch_bounds__(512) void lora_mx4_few_kernel(const uint8_t* __restrict__ Xc,
                                                           const uint8_t* __restrict__ Xs,
                                                           const uint8_t* __restrict__ Wc,
                                                           const uint8_t* __restrict__ Ws, u16* __restrict__ Y, int m,
                                                           int n, int slabs, int tiles_m, int tiles_n) {
  constexpr int NW = 8, FR = TG * FG;
  constexpr int RND = FR < 8 ? FR : 8;   // fragments summed per round
  __shared__ floatx4 part[NW][RND][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int g = lane >> 4, c = lane & 15;
  int tm, tn;
  tile_coords(tiles_m, tiles_n, 8, (int)blockIdx.x, tm, tn);
  const int m0 = tm * 16 * TG, n0 = tn * 16 * FG;
  const int gw = (n + 63) / 64, gx = (m + 63) / 64;
  const uint8_t *wp[FG], *wsp[FG], *xp[TG], *xsp[TG];   // rows past the matrix: its last one, not stored
#pragma unroll
  for (int f = 0; f < FG; ++f) {
    const int row = min(n0 + 16 * f + c, n - 1);
    wp[f] = Wc + (size_t)row * slabs * 128 + 16 * g;
    wsp[f] = Ws + (size_t)(row >> 6) * 512 + mx4_scale_offset(row, g);
  }
#pragma unroll
  for (int t = 0; t < TG; ++t) {
    const int row = min(m0 + 16 * t + c, m - 1);
    xp[t] = Xc + (size_t)row * slabs * 128 + 16 * g;
    xsp[t] = Xs + (size_t)(row >> 6) * 512 + mx4_scale_offset(row, g);
  }
  floatx4 acc[FG][TG];
#pragma unroll
  for (int f = 0; f < FG; ++f)
#pragma unroll
    for (int t = 0; t < TG; ++t) acc[f][t] = floatx4{0.f, 0.f, 0.f, 0.f};

  struct Slab {
    int4v w[FG][2], x[TG][2];
    int ws[FG], xs[TG];
  };
  auto load = [&](Slab& b, int s) LORA_INLINE {
#pragma unroll
    for (int f = 0; f < FG; ++f) {
      b.w[f][0] = *reinterpret_cast<const int4v*>(wp[f] + (size_t)s * 128);
      b.w[f][1] = *reinterpret_cast<const int4v*>(wp[f] + (size_t)s * 128 + 64);
      b.ws[f] = *reinterpret_cast<const u16*>(wsp[f] + (size_t)s * gw * 512);
    }
#pragma unroll
    for (int t = 0; t < TG; ++t) {
      b.x[t][0] = *reinterpret_cast<const int4v*>(xp[t] + (size_t)s * 128);
      b.x[t][1] = *reinterpret_cast<const int4v*>(xp[t] + (size_t)s * 128 + 64);
      b.xs[t] = *reinterpret_cast<const u16*>(xsp[t] + (size_t)s * gx * 512);
    }
  };
  auto multiply = [&](Slab& b) LORA_INLINE {
#pragma unroll
    for (int t = 0; t < TG; ++t)
#pragma unroll
      for (int f = 0; f < FG; ++f) {
        acc[f][t] = mfma_mx4<0, 0>(b.w[f][0], b.x[t][0], acc[f][t], b.ws[f], b.xs[t]);
        acc[f][t] = mfma_mx4<1, 1>(b.w[f][1], b.x[t][1], acc[f][t], b.ws[f], b.xs[t]);
      }
  };
  Slab b0, b1;
  int s = wave;
  if (s < slabs) load(b0, s);
  for (; s < slabs; s += 2 * NW) {
    if (s + NW < slabs) load(b1, s + NW);
    multiply(b0);
    if (s + NW >= slabs) break;
    if (s + 2 * NW < slabs) load(b0, s + 2 * NW);
    multiply(b1);
  }
#pragma unroll
  for (int e0 = 0; e0 < FR; e0 += RND) {
    if (e0) __syncthreads();
#pragma unroll
    for (int e = 0; e < RND; ++e) part[wave][e][lane] = acc[(e0 + e) % FG][(e0 + e) / FG];
    __syncthreads();
    if (wave < RND) {
      floatx4 v = part[0][wave][lane];
#pragma unroll
      for (int w = 1; w < NW; ++w) v += part[w][wave][lane];
      const int e = e0 + wave, f = e % FG, t = e / FG;
      const int row = m0 + 16 * t + c, col = n0 + 16 * f + 4 * g;
      if (row < m && col < n) {
        const uint32_t lo = (uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16);
        const uint32_t hi = (uint32_t)f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16);
        *reinterpret_cast<uint2*>(Y + (size_t)row * n + col) = uint2{lo, hi};
      }
    }
  }
}

// At most 16 tokens: one launch.  Every workgroup quantises X into LDS, as the
// fragments that its waves multiply; its first loads of W are under way
// meanwhile.  A group of 16 features is formed by KS waves that share its slabs,
// four slabs' loads of W ahead; their sums are added in wave order.  Bound by
// launch and load latency: 1 x 4096 x 4096 in 4.3 us, 2.1 TB/s of W (with X quantised
// by a launch of its own 2.5 and 4.0).
template <int KS>
__global__ __launch_bounds__(512) void lora_mx4_token_kernel(const u16* __restrict__ X, const uint8_t* __restrict__ Wc,
                                                             const uint8_t* __restrict__ Ws, u16* __restrict__ Y, int m,
                                                             int n, int k, int slabs) {
  constexpr int NW = 8, D = 4;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  int4v* frag = reinterpret_cast<int4v*>(smem);                        // [slab][step][lane]
  u16* xscale = reinterpret_cast<u16*>(smem + (size_t)slabs * 2048);   // [slab][lane]: both steps' bytes
  floatx4* part = reinterpret_cast<floatx4*>(smem + (size_t)slabs * 2176);   // [wave][lane]
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int g = lane >> 4, c = lane & 15;
  const int grp = (int)blockIdx.x * (NW / KS) + wave / KS, ks = wave % KS;
  const int n0 = grp * 16, gw = (n + 63) / 64;
  const int wrow = min(n0 + c, n - 1);   // rows past the matrix: its last one, not stored
  const uint8_t* wp = Wc + (size_t)wrow * slabs * 128 + 16 * g;
  const uint8_t* wsp = Ws + (size_t)(wrow >> 6) * 512 + mx4_scale_offset(wrow, g);
  int4v w[D][2];
  int ws[D];
  auto load = [&](int j, int s) LORA_INLINE {
    w[j][0] = *reinterpret_cast<const int4v*>(wp + (size_t)s * 128);
    w[j][1] = *reinterpret_cast<const int4v*>(wp + (size_t)s * 128 + 64);
    ws[j] = *reinterpret_cast<const u16*>(wsp + (size_t)s * gw * 512);
  };
#pragma unroll
  for (int j = 0; j < D; ++j)
    if (ks + KS * j < slabs) load(j, ks + KS * j);

  // X: four lanes a block of 32 columns.  The places of tokens past m stay as they
  // are: a token's codes and scales enter its own column of the products alone, and
  // those columns are not stored.
  constexpr int U = 8;   // pieces of a thread whose loads are under way together
  const int pieces = slabs * 32, total = m * pieces;
  const float inv = 1.0f / (float)pieces;
  for (int e0 = tid; e0 < total; e0 += 512 * U) {
    int4v x[U];
    int row[U], piece[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = e0 + 512 * u;
      row[u] = (int)(((float)e + 0.5f) * inv);   // (below 2^19: at least 0.5 / pieces from a whole number)
      piece[u] = e - row[u] * pieces;
      x[u] = e < total && 8 * piece[u] < k ? *reinterpret_cast<const int4v*>(X + (size_t)row[u] * k + 8 * piece[u])
                                           : int4v{0, 0, 0, 0};
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (e0 - tid + 512 * u >= total) break;   // (whole waves: total is a multiple of 32, blocks of four lanes)
      int scale;
      const uint32_t out = quantise_piece(x[u], scale);
      const int slab = piece[u] >> 5, step = (piece[u] >> 4) & 1, at = ((piece[u] >> 2) & 3) * 16 + row[u];
      if (e0 + 512 * u < total) {
        reinterpret_cast<uint32_t*>(&frag[(slab * 2 + step) * 64 + at])[piece[u] & 3] = out;
        if ((piece[u] & 3) == 0) reinterpret_cast<uint8_t*>(&xscale[slab * 64 + at])[step] = (uint8_t)scale;
      }
    }
  }
  __syncthreads();
  floatx4 acc{0.f, 0.f, 0.f, 0.f};
  for (int s0 = ks; s0 < slabs; s0 += KS * D) {
#pragma unroll
    for (int j = 0; j < D; ++j) {
      const int s = s0 + KS * j;
      if (s < slabs) {
        const int xs = xscale[s * 64 + lane];
        acc = mfma_mx4<0, 0>(w[j][0], frag[s * 128 + lane], acc, ws[j], xs);
        acc = mfma_mx4<1, 1>(w[j][1], frag[s * 128 + 64 + lane], acc, ws[j], xs);
        if (s + KS * D < slabs) load(j, s + KS * D);
      }
    }
  }
  if constexpr (KS > 1) {
    part[wave * 64 + lane] = acc;
    __syncthreads();
    if (ks != 0) return;
#pragma unroll
    for (int q = 1; q < KS; ++q) acc += part[(wave + q) * 64 + lane];
  }
  const int col = n0 + 4 * g;
  if (c < m && col < n) {
    const uint32_t lo = (uint32_t)f32_to_bf16(acc[0]) | ((uint32_t)f32_to_bf16(acc[1]) << 16);
    const uint32_t hi = (uint32_t)f32_to_bf16(acc[2]) | ((uint32_t)f32_to_bf16(acc[3]) << 16);
    *reinterpret_cast<uint2*>(Y + (size_t)c * n + col) = uint2{lo, hi};
  }
}

// ---------------------------------------------------------------------------
// Tiles of BM tokens x BN features by WM x WN waves, NS slabs in LDS, copied from
// memory straight into LDS (one 16-byte chunk a lane, the swizzle applied to the
// global addresses).  256 x 256, eight waves of 128 x 64: two slabs; the smaller
// ones, for outputs that do not fill the compute units with those: three (128 x
// 128: four), so that a slab's copies have two slabs' products or more to land.
//
// 256 x 256: 4096 x 11008 x 4096 in 95 to 97 us, 3.8 to 3.9 PFLOP/s, the matrix
// cores busy 45% of the cycles at a clock of 2.0 to 2.1 GHz.  The same launch on
// zeros, which run at the full 2.4 GHz, takes 83 us with 43% to 44% busy: the clock is
// worth an eighth, the rest is the loop's, where a slab's LDS reads and copies (256
// KiB, 2048 cycles at 128 bytes) are as long as its products.  A persistent form
// that begins the next tile under the last one's end took 104; waves of a row
// taking turns at the products, instead of the fragments read in place, 100 to 106.
// 256 x 128: 1531 x 4104 x 3208 in 18 us, one round of 198 workgroups with 13
// serial slabs, of which each has 1408 cycles of LDS to 1024 of products, and the
// tile's beginning and end.  64 x 128: 24 x 32000 x 4096 in 13 to 14 us, 5.0 to 5.4
// TB/s, bound by HBM.
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

template <int BM, int BN, int WM, int WN, int NS>
__global__ __launch_bounds__(64 * WM * WN) void lora_mx4_kernel(
    const uint8_t* __restrict__ Xc, const uint8_t* __restrict__ Xs, const uint8_t* __restrict__ Wc,
    const uint8_t* __restrict__ Ws, u16* __restrict__ Y, int m, int n, int slabs, int tiles_m, int tiles_n) {
  constexpr int NW = WM * WN;
  constexpr int XCELLS = BM / 64, CELLS = XCELLS + BN / 64;   // cells of scales
  constexpr int TM = BM / WM, TN = BN / WN;          // tokens, features per wave
  constexpr int FB = TM / 16, FA = TN / 16;          // their fragments
  constexpr int SX = TM / 64;                        // cells of a wave's tokens
  // copies of a wave and slab: 8 rows of X or W each, or half a cell
  // With two stages nothing is copied further ahead than a slab, and the scales go
  // straight to registers (SL loads); through LDS they cost the 256 x 256 tile 5%.
  constexpr bool SREG = NS == 2;
  constexpr int SL = SREG ? SX + 1 : 0;
  constexpr int CX = BM / 8 / NW, CW = BN / 8 / NW, CS = SREG ? 0 : (2 * CELLS + NW - 1) / NW, C = CX + CW + CS;
  constexpr int SOFF = (BM + BN) * 128, STAGE = SOFF + CS * NW * 256;
  constexpr int CPB = (C + FB - 1) / FB;             // of them after each token fragment's products
  static_assert(TM % 64 == 0 && TN == 64 && BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "tile shape");
  static_assert(NS >= 2 && (NS - 1) * C < 64, "copies in flight fit the wait counter");
  constexpr int OUT = out16_bytes<FA, 2>();
  static_assert(NW * OUT <= NS * STAGE && NS * STAGE <= 160 * 1024, "LDS");
  __shared__ __attribute__((aligned(1024))) char smem[NS * STAGE];
  int tm, tn;
  tile_coords(tiles_m, tiles_n, 8, (int)blockIdx.x, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int g = lane >> 4, c16 = lane & 15;

  const uint32_t rowbytes = (uint32_t)slabs * 128;
  const __amdgpu_buffer_rsrc_t rsX = make_rsrc(Xc + (size_t)m0 * rowbytes, (uint64_t)min(BM, m - m0) * rowbytes);
  const __amdgpu_buffer_rsrc_t rsW = make_rsrc(Wc + (size_t)n0 * rowbytes, (uint64_t)min(BN, n - n0) * rowbytes);
  const int gx = (m + 63) / 64, gw = (n + 63) / 64;
  const __amdgpu_buffer_rsrc_t rsXs = make_rsrc(Xs, (uint64_t)gx * slabs * 512);
  const __amdgpu_buffer_rsrc_t rsWs = make_rsrc(Ws, (uint64_t)gw * slabs * 512);

  floatx4 acc[FA][FB];           // 16 x 16 fragments: [features 16 a ..][tokens 16 b ..] of the wave's tile
#pragma unroll
  for (int a = 0; a < FA; ++a)
#pragma unroll
    for (int b = 0; b < FB; ++b) acc[a][b] = floatx4{0.f, 0.f, 0.f, 0.f};
  int4v fw[2][FA], fx[FB];       // W fragments of both steps, X fragments of the current one
  int2v sx[SX], sw, sx1[SX], sw1;   // scales of this slab (the token cells, the feature cell) and the next

  const int l8 = lane >> 3, crow = 8 * wave;
  const uint32_t kcol = (uint32_t)(((lane & 7) ^ kc_swz(crow + l8)) << 4);
  const uint32_t coff = (uint32_t)(crow + l8) * rowbytes + kcol;
  // the wave's half cells (uniform): their matrix, first cell and cells per slab
  __amdgpu_buffer_rsrc_t rsS[CS + 1];
  uint32_t sat[CS + 1], sstep[CS + 1], slane[CS + 1];   // (a cell past the matrix: zeros)
#pragma unroll
  for (int i = 0; i < CS; ++i) {
    const int h = wave * CS + i, cl = h >> 1;
    const bool isx = cl < XCELLS;
    rsS[i] = isx ? rsXs : rsWs;
    const Mx4Cell at = cl < CELLS ? mx4_cell(isx ? m0 / 64 + cl : n0 / 64 + cl - XCELLS, isx ? gx : gw) : Mx4Cell{0u, 0u, kMx4None};
    sat[i] = at.first + (h & 1) * 256;
    sstep[i] = at.step;
    slane[i] = (uint32_t)lane * 4 | at.none;
  }
  // copy i of a slab into the stage at `stage`; past the last slab zeros, so that
  // the counts below hold
  auto copy = [&](const Mx4Slab& s, int i, int stage) LORA_INLINE {
    char* sb = smem + stage;
    if (i < CX) {
      dma16(rsX, (coff + (uint32_t)(8 * NW * i) * rowbytes) | s.none, s.kb * 128, sb + (crow + 8 * NW * i) * 128);
    } else if (i < CX + CW) {
      const int r = 8 * NW * (i - CX);
      dma16(rsW, (coff + (uint32_t)r * rowbytes) | s.none, s.kb * 128, sb + (BM + crow + r) * 128);
    } else {
      const int c = i - CX - CW;
      dma4(rsS[c], slane[c] | s.none, sat[c] + s.kb * sstep[c], sb + SOFF + (wave * CS + c) * 256);
    }
  };
  const uint32_t fbase = kc_offset(c16, g);      // (rows 16 apart swizzle alike; step 1: chunk 4 further)
  const uint32_t cell = (uint32_t)(g * 128 + c16 * 8);
  auto read_x = [&](int stage, int step, int b) LORA_INLINE {
    fx[b] = *reinterpret_cast<const int4v*>(smem + stage + wm * TM * 128 + (fbase ^ (step << 6)) + 16 * 128 * b);
  };
  auto read_w = [&](int stage, int step) LORA_INLINE {
#pragma unroll
    for (int a = 0; a < FA; ++a)
      fw[step][a] =
          *reinterpret_cast<const int4v*>(smem + stage + (BM + wn * TN) * 128 + (fbase ^ (step << 6)) + 16 * 128 * a);
  };
  auto read_scales = [&](int stage) LORA_INLINE {
    const char* sc = smem + stage + SOFF + cell;
#pragma unroll
    for (int i = 0; i < SX; ++i) sx1[i] = *reinterpret_cast<const int2v*>(sc + (wm * SX + i) * 512);
    sw1 = *reinterpret_cast<const int2v*>(sc + (XCELLS + wn) * 512);
  };
  auto load_scales = [&](int kb) LORA_INLINE {   // SL loads, in this place (cells past the matrix: another's, or zeros past the end)
    const uint32_t cx = (uint32_t)kb * gx + m0 / 64 + SX * wm, cw = (uint32_t)kb * gw + n0 / 64 + wn;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < SX; ++i) sx1[i] = __builtin_bit_cast(int2v, buf_load8(rsXs, (cx + i) * 512 + cell));
    sw1 = __builtin_bit_cast(int2v, buf_load8(rsWs, cw * 512 + cell));
    __builtin_amdgcn_sched_barrier(0);
  };
  // products of a step; after each token fragment's, f(its index)
  auto products = [&](auto stepc, auto&& f) LORA_INLINE {
    constexpr int S = decltype(stepc)::value;
    unrolled<FB>([&](auto bc) LORA_INLINE {
      constexpr int B = decltype(bc)::value;
      const int sb = (int)((B >> 1) & 1 ? sx[B >> 2].y : sx[B >> 2].x);
      unrolled<FA>([&](auto ac) LORA_INLINE {
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
  auto first_step = [&](int here, int next) LORA_INLINE {   // next: the slab whose scales to load
#pragma unroll
    for (int i = 0; i < SX; ++i) sx[i] = sx1[i];
    sw = sw1;
    if (SREG && next >= 0) load_scales(next);
    products(I0{}, [&](int b) LORA_INLINE {
      if (b == 1) read_w(here, 1);
      read_x(here, 1, b);
    });
  };
  if constexpr (SREG) load_scales(0);
#pragma unroll
  for (int j = 0; j < NS; ++j)
#pragma unroll
    for (int i = 0; i < C; ++i) copy(mx4_slab(j, slabs), i, j * STAGE);
  copy_barrier<(NS - 1) * C>();
  int here = 0;
  if constexpr (!SREG) read_scales(here);
  read_w(here, 0);
#pragma unroll
  for (int b = 0; b < FB; ++b) read_x(here, 0, b);
  for (int kb = 0; kb + 1 < slabs; ++kb) {   // (no branch inside, or the compiler moves the products)
    const int there = here + STAGE == NS * STAGE ? 0 : here + STAGE;
    first_step(here, kb + 1);
    copy_barrier<(NS - 2) * C + SL>();   // every wave has read this slab, and the next one has landed
    if constexpr (!SREG) read_scales(there);
    read_w(there, 0);
    const Mx4Slab later = mx4_slab(kb + NS, slabs);
    products(I1{}, [&](int b) LORA_INLINE {
#pragma unroll
      for (int i = 0; i < CPB; ++i)
        if (CPB * b + i < C) copy(later, CPB * b + i, here);
      read_x(there, 0, b);
    });
    here = there;
  }
  first_step(here, -1);
  products(I1{}, [](int) {});
  copy_barrier<0>();   // the trailing copies (zeros) have landed before the LDS is used again

  // Y: each wave's blocks of 32 tokens x 64 features through a region of LDS of its own
  const int j0 = n0 + wn * TN;
#pragma unroll
  for (int fi = 0; fi < FB / 2; ++fi) {
    const int i0 = m0 + wm * TM + 32 * fi;
    floatx4 v[FA][2];
#pragma unroll
    for (int a = 0; a < FA; ++a) {
      v[a][0] = acc[a][2 * fi];
      v[a][1] = acc[a][2 * fi + 1];
    }
    store_out16<FA, 2>(v, smem + wave * OUT, Y + (size_t)i0 * n + j0, (size_t)n, m - i0, n - j0, lane);
  }
}

hipError_t launch_mx4_quantize(const Mx4QuantArgs& a, hipStream_t st) {
  const int slabs = (int)mx4_slabs(a.k), groups = (int)mx4_groups(a.rows);
  hipLaunchKernelGGL(lora_mx4_quantize_kernel, dim3((unsigned)(slabs * groups * 4)), dim3(256), 0, st, a.X, a.codes, a.scales,
                     (int)a.rows, (int)a.k, slabs, groups);
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, uint16_t* X, int64_t rows, int64_t k,
                                 hipStream_t st) {
  const int slabs = (int)mx4_slabs(k), groups = (int)mx4_groups(rows);
  hipLaunchKernelGGL(lora_mx4_dequantize_kernel, dim3((unsigned)(slabs * groups * 4)), dim3(256), 0, st, codes, scales, X,
                     (int)rows, (int)k, slabs, groups);
  return hipGetLastError();
}

template <int BM, int BN, int WM, int WN, int NS>
static hipError_t launch_tile(const Mx4Plan& p, const Mx4FwdArgs& a, const uint8_t* xc, const uint8_t* xs,
                              hipStream_t st) {
  hipLaunchKernelGGL((lora_mx4_kernel<BM, BN, WM, WN, NS>), dim3((unsigned)p.grid), dim3((unsigned)p.block), 0, st, xc,
                     xs, a.Wc, a.Ws, a.Y, (int)a.m, (int)a.n, (int)mx4_slabs(a.k), p.tiles_m, p.tiles_n);
  return hipGetLastError();
}
template <int TG, int FG>
static hipError_t launch_few(const Mx4Plan& p, const Mx4FwdArgs& a, const uint8_t* xc, const uint8_t* xs,
                             hipStream_t st) {
  hipLaunchKernelGGL((lora_mx4_few_kernel<TG, FG>), dim3((unsigned)p.grid), dim3((unsigned)p.block), 0, st, xc, xs, a.Wc,
                     a.Ws, a.Y, (int)a.m, (int)a.n, (int)mx4_slabs(a.k), p.tiles_m, p.tiles_n);
  return hipGetLastError();
}
template <int KS>
static hipError_t launch_token(const Mx4Plan& p, const Mx4FwdArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((lora_mx4_token_kernel<KS>), dim3((unsigned)p.grid), dim3((unsigned)p.block),
                     mx4_token_lds(mx4_slabs(a.k)), st, a.X, a.Wc, a.Ws, a.Y, (int)a.m, (int)a.n, (int)a.k,
                     (int)mx4_slabs(a.k));
  return hipGetLastError();
}

hipError_t launch_mx4_fwd(const Mx4FwdArgs& a, hipStream_t st) {
  const Mx4Plan p = plan_mx4_fwd(a.m, a.n, a.k);
  if (p.kind == MX4_TOKEN_8) return launch_token<8>(p, a, st);
  if (p.kind == MX4_TOKEN_2) return launch_token<2>(p, a, st);
  const Mx4Layout L = mx4_fwd_layout(a.m, a.n, a.k);
  uint8_t* xc = reinterpret_cast<uint8_t*>(a.ws + L.xc);
  uint8_t* xs = reinterpret_cast<uint8_t*>(a.ws + L.xs);
  const hipError_t e = launch_mx4_quantize(Mx4QuantArgs{a.X, xc, xs, a.m, a.k}, st);
  if (e != hipSuccess) return e;
  switch (p.kind) {
    case MX4_FEW_1: return launch_few<1, 1>(p, a, xc, xs, st);
    case MX4_FEW_2: return launch_few<2, 1>(p, a, xc, xs, st);
    case MX4_FEW_4: return launch_few<4, 2>(p, a, xc, xs, st);
    case MX4_64x128: return launch_tile<64, 128, 1, 2, 3>(p, a, xc, xs, st);
    case MX4_128x128: return launch_tile<128, 128, 2, 2, 4>(p, a, xc, xs, st);
    case MX4_256x128: return launch_tile<256, 128, 4, 2, 3>(p, a, xc, xs, st);
    default: return launch_tile<256, 256, 2, 4, 2>(p, a, xc, xs, st);
  }
}

}  // namespace lora
