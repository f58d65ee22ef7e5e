// Matrices in 8-bit floating point (e4m3) with a scale 2^(s - 127) for each block of
// 128: quantisation, its inverse, and the products of a frozen weight W [n, k],
//   Y = Q(X) Q(W)^T,   dX = Q(dY) Q(W),
// on the matrix cores' scaled 8-bit products (lora_gemm.hpp).  A weight's blocks are
// 128 x 128, so that its scale is one number for a product of either direction;
// activations have one per row.
#include "lora_device.hpp"
#include "lora_gemm.hpp"
#include "lora_train.hpp"

namespace lora {

// The scale byte of a block from its largest magnitude's bf16 bits: the smallest s
// with magnitude <= 448 2^(s - 127) (448 = 1.75 2^8: 1.75 has bits 0x60 after the
// exponent), at least 0; 255 where the block holds a NaN or an infinity.
__device__ __forceinline__ int fp8_scale(uint32_t top) {
  const int field = (int)(top >> 7);
  return field == 255 ? 255 : max(field - 8 + ((top & 0x7Fu) > 0x60u ? 1 : 0), 0);
}
__device__ __forceinline__ uint32_t top_of(const int4v& x) {
  uint32_t top = 0;
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const uint32_t w = (uint32_t)x[h] & 0x7FFF7FFFu;
    top = max(top, max(w & 0xFFFFu, w >> 16));
  }
  return top;
}
// The largest of a value over 16 neighbouring lanes.
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xf, 0xf, true));    // lane ^ 1
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xf, 0xf, true));    // lane ^ 2
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true));   // 7 - lane of 8
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xf, 0xf, true));   // 15 - lane of 16
}
// Eight bf16 values' codes under a scale.  The division by the scale is exact (below
// 2^-126 it is scaled up), the conversion rounds to nearest even and finds no value
// beyond 448.
__device__ __forceinline__ int2w fp8_codes(const int4v& x, int scale) {
  const float up = __builtin_bit_cast(float, (uint32_t)(scale == 255 ? 0 : 254 - scale) << 23);
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = bf16_to_f32((u16)((uint32_t)x[e >> 1] >> (16 * (e & 1)))) * up;
  int2w o{0, 0};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h], y[4 * h + 1], 0, false);
    o[h] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h + 2], y[4 * h + 3], w, true);
  }
  return scale == 255 ? int2w{0, 0} : o;
}
__device__ __forceinline__ int fp8_row_scale_at(int row, int block, int cells) {
  return (block * cells + (row >> 6)) * 64 + (row & 15) * 4 + ((row >> 4) & 3);
}

// Activations: 16 lanes a row's block, 8 columns each; a thread takes rows 16 apart,
// whose scales are a word.  A workgroup: four blocks of the rows of a quarter cell
// (its rows 4 q .. 4 q + 3, and those 16, 32 and 48 after them).  Bounded by memory: a
// value is read once, held in registers while the block's largest is found by four
// exchanges between lanes, and its byte written; 4096 x 4096 9.6 us (5.2 TB/s), 16384 x
// 4096 36 us (5.6 TB/s), 32 x 4096 2.8 us, what a launch of a few waves takes.
__global__ __launch_bounds__(256) void lora_fp8_quantize_rows_kernel(const u16* __restrict__ X,
                                                                     uint8_t* __restrict__ codes,
                                                                     uint8_t* __restrict__ scales, int rows, int k,
                                                                     int blocks, int cells) {
  const int groups = (blocks + 3) / 4, bg = (int)blockIdx.x % groups, rest = (int)blockIdx.x / groups;
  const int cell = rest >> 2, tid = threadIdx.x, lane16 = tid & 15;
  const int b = bg * 4 + ((tid >> 4) & 3), r16 = 4 * (rest & 3) + (tid >> 6), col = b * 128 + 8 * lane16;
  if (b >= blocks) return;   // (16 lanes alike)
  int4v x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = cell * 64 + r16 + 16 * i;
    x[i] = row < rows && col < k ? *reinterpret_cast<const int4v*>(X + (size_t)row * k + col) : int4v{0, 0, 0, 0};
  }
  uint32_t word = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = cell * 64 + r16 + 16 * i, s = fp8_scale(max16(top_of(x[i])));
    if (row >= rows) continue;
    word |= (uint32_t)s << (8 * i);
    *reinterpret_cast<int2w*>(codes + ((size_t)row * blocks + b) * 128 + 8 * lane16) = fp8_codes(x[i], s);
  }
  if (lane16 == 0) *reinterpret_cast<uint32_t*>(scales + fp8_row_scale_at(cell * 64 + r16, b, cells)) = word;
}

// A weight: a workgroup a block of 128 x 128, all 64 values of a thread in registers, so
// that the block's largest and its codes take one read.  11008 x 4096 21.3 us (6.3
// TB/s).
__global__ __launch_bounds__(256) void lora_fp8_quantize_block_kernel(const u16* __restrict__ X,
                                                                      uint8_t* __restrict__ codes,
                                                                      uint8_t* __restrict__ scales, int rows, int k,
                                                                      int blocks) {
  __shared__ uint32_t tops[4];
  const int b = (int)blockIdx.x % blocks, r0 = (int)blockIdx.x / blocks * 128;
  const int tid = threadIdx.x, j = tid & 15, col = b * 128 + 8 * j;
  int4v x[8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = r0 + (tid >> 4) + 16 * i;
    x[i] = row < rows && col < k ? *reinterpret_cast<const int4v*>(X + (size_t)row * k + col) : int4v{0, 0, 0, 0};
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, top_of(x[i]));
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
  if ((tid & 63) == 0) tops[tid >> 6] = top;
  __syncthreads();
  const int s = fp8_scale(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
  if (tid == 0) scales[blockIdx.x] = (uint8_t)s;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = r0 + (tid >> 4) + 16 * i;
    if (row < rows) *reinterpret_cast<int2w*>(codes + ((size_t)row * blocks + b) * 128 + 8 * j) = fp8_codes(x[i], s);
  }
}

// The values of codes and scales: a lane takes 8 columns.  The product with a power of
// two and the result's bf16 are exact from 2^-126 on (4 significant bits).  11008 x 4096 21.5 us (6.3
// TB/s).
template <bool ROWS>
__global__ __launch_bounds__(256) void lora_fp8_dequantize_kernel(const uint8_t* __restrict__ codes,
                                                                  const uint8_t* __restrict__ scales,
                                                                  u16* __restrict__ X, int rows, int k, int blocks,
                                                                  int cells) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int per = k / 8, row = (int)(e / per), piece = (int)(e - (int64_t)row * per);
  if (row >= rows) return;
  const int b = piece >> 4;
  const int2w w = *reinterpret_cast<const int2w*>(codes + (size_t)row * blocks * 128 + 8 * piece);
  const int s = scales[ROWS ? fp8_row_scale_at(row, b, cells) : (row >> 7) * blocks + b];
  // 2^(s - 127); s = 0 is a subnormal, 255 NaN
  const uint32_t bits = s == 0 ? 0x00400000u : (s == 255 ? 0x7FC00000u : (uint32_t)s << 23);
  const float unit = __builtin_bit_cast(float, bits);
  int4v o;
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const auto v = h & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(w[h >> 1], true) : __builtin_amdgcn_cvt_pk_f32_fp8(w[h >> 1], false);
    o[h] = (int)((uint32_t)f32_to_bf16(v[0] * unit) | ((uint32_t)f32_to_bf16(v[1] * unit) << 16));
  }
  *reinterpret_cast<int4v*>(X + (size_t)row * k + 8 * piece) = o;
}

struct Fp8Product {
  const uint8_t *Ac, *As, *Wc, *Ws;
  u16* out;
  float* sums;
  int m, n, k, tiles_m, tiles_n, splits;
};

// ---------------------------------------------------------------------------
// Few tokens: a workgroup forms 16 features x 16 TG tokens with its eight waves on
// different stages, straight from memory without a barrier until the waves' sums are
// added, in wave order, through LDS.  A lane loads the two 16-byte chunks of codes
// that it multiplies; each wave has D stages' loads under way.  Bounded by W's bytes:
// 16 x 4096 x 4096 10.6 us a call with the quantisation of X (17 MB, 3.3 us at a copy's
// rate; two launches alone 5 to 6), 32 x 11008 x 4096 16.2 us (45 MB, 8.9).
// From about 32 tokens on tiles in LDS, which read a token's codes once and not once per
// group of features, take less.
template <int TG, int D>
__global__ __launch_bounds__(512) void lora_fp8_few_kernel(Fp8Product p) {
  constexpr int NW = 8;
  static_assert(TG <= NW, "a wave adds a fragment's sums");
  __shared__ floatx4 part[NW][TG][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int g = lane >> 4, c = lane & 15;
  int tm, tn;
  tile_coords(p.tiles_m, p.tiles_n, 8, (int)blockIdx.x, tm, tn);
  const int m0 = tm * 16 * TG, n0 = tn * 16, stages = (p.k + 127) / 128, cells = (p.m + 63) / 64;
  // rows past the matrix: its last one, not stored
  const uint8_t* wp = p.Wc + (size_t)min(n0 + c, p.n - 1) * stages * 128 + 16 * g;
  const uint8_t *xp[TG], *xsp[TG];
#pragma unroll
  for (int t = 0; t < TG; ++t) {
    const int row = min(m0 + 16 * t + c, p.m - 1);
    xp[t] = p.Ac + (size_t)row * stages * 128 + 16 * g;
    xsp[t] = p.As + fp8_row_scale_at(row, 0, cells);
  }
  const uint8_t* wsp = p.Ws + (size_t)(n0 / 128) * stages;   // (16 features share a block)
  floatx4 acc[1][TG];
#pragma unroll
  for (int t = 0; t < TG; ++t) acc[0][t] = floatx4{0.f, 0.f, 0.f, 0.f};
  Frag w[D], x[D][TG];
  int ws[D], xs[D][TG];
  auto load = [&](int j, int s) LORA_INLINE {
    w[j].lo = *reinterpret_cast<const int4v*>(wp + (size_t)s * 128);
    w[j].hi = *reinterpret_cast<const int4v*>(wp + (size_t)s * 128 + 64);
    ws[j] = wsp[s];
#pragma unroll
    for (int t = 0; t < TG; ++t) {
      x[j][t].lo = *reinterpret_cast<const int4v*>(xp[t] + (size_t)s * 128);
      x[j][t].hi = *reinterpret_cast<const int4v*>(xp[t] + (size_t)s * 128 + 64);
      xs[j][t] = xsp[t][(size_t)s * cells * 64];
    }
  };
#pragma unroll
  for (int j = 0; j < D; ++j)
    if (wave + NW * j < stages) load(j, wave + NW * j);
  for (int s0 = wave; s0 < stages; s0 += NW * D) {
#pragma unroll
    for (int j = 0; j < D; ++j) {
      const int s = s0 + NW * j;
      if (s >= stages) break;
#pragma unroll
      for (int t = 0; t < TG; ++t) acc[0][t] = stage_product<Fp8, 0>(w[j], x[j][t], acc[0][t], ws[j], xs[j][t]);
      if (s + NW * D < stages) load(j, s + NW * D);
    }
  }
  formed(acc);
#pragma unroll
  for (int t = 0; t < TG; ++t) part[wave][t][lane] = acc[0][t];
  __syncthreads();
  if (wave < TG) {
    floatx4 v = part[0][wave][lane];
#pragma unroll
    for (int q = 1; q < NW; ++q) v += part[q][wave][lane];
    const int row = m0 + 16 * wave + c, col = n0 + 4 * g;
    if (row < p.m && col < p.n) *reinterpret_cast<uint2*>(p.out + (size_t)row * p.n + col) = bf16x4(v);
  }
}

// Very few values of X: one launch.  Every workgroup quantises X into LDS; its first
// loads of W are under way meanwhile.  A group of 16 features is formed by KS waves
// that share its stages, D stages' loads of W ahead; their sums are added in wave
// order.  X (at most 32 KiB, in L2) is quantised again by each workgroup, which
// takes less than the launch that would do it once (2.8 us by itself): 1 x 4096 x 4096 5.0
// us (3.4 TB/s of W; its start and its end, where few loads are under way, are the rest),
// 1 x 32000 x 4096 20 us (6.5 TB/s).
template <int KS, int D>
__global__ __launch_bounds__(512) void lora_fp8_token_kernel(Fp8Product p, const u16* __restrict__ X) {
  constexpr int NW = 8;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int stages = (p.k + 127) / 128, m = p.m;
  char* xc = smem;                                              // [stage][token] rows of 128 bytes, swizzled by the token
  uint8_t* xs = reinterpret_cast<uint8_t*>(smem + (size_t)stages * m * 128);   // [stage][token]
  floatx4* part = reinterpret_cast<floatx4*>(smem + (size_t)((stages * m * 129 + 15) & ~15));   // [wave][lane]
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int g = lane >> 4, c = lane & 15;
  const int grp = (int)blockIdx.x * (NW / KS) + wave / KS, ks = wave % KS, n0 = grp * 16;
  const uint8_t* wp = p.Wc + (size_t)min(n0 + c, p.n - 1) * stages * 128 + 16 * g;   // rows past the matrix: its last one, not stored
  const uint8_t* wsp = p.Ws + (size_t)(min(n0, p.n - 1) / 128) * stages;
  Frag w[D];
  int ws[D];
  auto load = [&](int j, int s) LORA_INLINE {
    w[j].lo = *reinterpret_cast<const int4v*>(wp + (size_t)s * 128);
    w[j].hi = *reinterpret_cast<const int4v*>(wp + (size_t)s * 128 + 64);
    ws[j] = wsp[s];
  };
#pragma unroll
  for (int j = 0; j < D; ++j)
    if (ks + KS * j < stages) load(j, ks + KS * j);

  // X: 16 lanes a token's block.
  const int pieces = stages * 16, total = m * pieces;
  const float inv = 1.0f / (float)pieces;
  for (int e0 = tid; e0 - tid < total; e0 += 512 * 4) {
    int4v x[4];
    int row[4], piece[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int e = e0 + 512 * u;
      row[u] = (int)(((float)e + 0.5f) * inv);   // (below 2^19: at least 0.5 / pieces from a whole number)
      piece[u] = e - row[u] * pieces;
      x[u] = e < total && 8 * piece[u] < p.k ? *reinterpret_cast<const int4v*>(X + (size_t)row[u] * p.k + 8 * piece[u])
                                             : int4v{0, 0, 0, 0};
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (e0 - tid + 512 * u >= total) break;   // (whole blocks of 16 lanes: total is a multiple of 16)
      const int scale = fp8_scale(max16(top_of(x[u])));
      const int2w codes = fp8_codes(x[u], scale);
      if (e0 + 512 * u < total) {
        const int s = piece[u] >> 4, j = piece[u] & 15, at = s * m + row[u];
        *reinterpret_cast<int2w*>(xc + at * 128 + (((j >> 1) ^ kc_swz(row[u])) << 4) + (j & 1) * 8) = codes;
        if (j == 0) xs[at] = (uint8_t)scale;
      }
    }
  }
  __syncthreads();
  floatx4 acc{0.f, 0.f, 0.f, 0.f};
  const int tok = min(c, m - 1);   // (columns past the tokens: the last one's, not stored)
  const char* xr = xc + tok * 128 + ((g ^ kc_swz(tok)) << 4);
  const char* xh = xc + tok * 128 + (((4 + g) ^ kc_swz(tok)) << 4);
  for (int s0 = ks; s0 < stages; s0 += KS * D) {
#pragma unroll
    for (int j = 0; j < D; ++j) {
      const int s = s0 + KS * j;
      if (s < stages) {
        const Frag x{*reinterpret_cast<const int4v*>(xr + s * m * 128), *reinterpret_cast<const int4v*>(xh + s * m * 128)};
        acc = stage_product<Fp8, 0>(w[j], x, acc, ws[j], (int)xs[s * m + tok]);
        if (s + KS * D < stages) load(j, s + KS * D);
      }
    }
  }
  asm volatile("" : "+v"(acc));
  if constexpr (KS > 1) {
    part[wave * 64 + lane] = acc;
    __syncthreads();
    if (ks != 0) return;
#pragma unroll
    for (int q = 1; q < KS; ++q) acc += part[(wave + q) * 64 + lane];
  }
  const int col = n0 + 4 * g;
  if (c < m && col < p.n) *reinterpret_cast<uint2*>(p.out + (size_t)c * p.n + col) = bf16x4(acc);
}

// A tile's part of a split product: its rows of BN sums, [split][tile][row][column].
template <class Core, int BN>
__device__ __forceinline__ void store_sums(const typename Core::Acc& acc, float* to) {
  constexpr int FA = std::extent_v<typename Core::Acc, 0>, FB = std::extent_v<typename Core::Acc, 1>;
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
#pragma unroll
  for (int b = 0; b < FB; ++b)
#pragma unroll
    for (int a = 0; a < FA; ++a)
      *reinterpret_cast<floatx4*>(to + (Core::row0(wave) + 16 * b + (lane & 15)) * BN + Core::col(wave, a) +
                                  4 * (lane >> 4)) = acc[a][b];
}

// A tile of Y, or of its sum over a part of k.  Bounded by the matrix cores where tiles of 256 x 256 fill the card: 4096 x
// 11008 x 4096 147 to 150 us (2.5 PFLOP/s; the matrix cores multiply in 71% of the busy
// compute units' cycles, and 688 tiles are 2.7 rounds of 256, 3 in time); below that by
// how copies into LDS, reads from it and products overlap within one workgroup, about 0.6
// us each of a 256 x 128 tile's stage of 0.6 (few workgroups) to 0.9 us: 1531 x 4104 x
// 3208 24.4 us.  LDS has no conflicts to speak of (3% of its cycles); XCD-aware tile order
// (tile_coords): the 256 x 256 example reads 312 MB from memory and its last-level cache,
// 62 without any repetition.
template <class Core, int BM, int BN, int NT, bool SPLIT>
__global__ __launch_bounds__(NT) void lora_fp8_fwd_kernel(Fp8Product p) {
  __shared__ __attribute__((aligned(1024))) char smem[Core::SMEM];
  int tm, tn, split = 0;
  if constexpr (SPLIT) split = (int)blockIdx.x / (p.tiles_m * p.tiles_n);
  tile_coords(p.tiles_m, p.tiles_n, 8, (int)blockIdx.x - split * p.tiles_m * p.tiles_n, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN, blocks = (p.k + 127) / 128, nb = (p.n + 127) / 128, cells = (p.m + 63) / 64;
  int s0 = 0, s1 = blocks;   // the workgroup's stages; operands and scales begin at s0
  if constexpr (SPLIT) {
    s0 = (int)((int64_t)blocks * split / p.splits);
    s1 = (int)((int64_t)blocks * (split + 1) / p.splits);
  }
  const uint32_t row = (uint32_t)blocks * 128, skip = (uint32_t)s0 * 128;
  const NtTile t{make_rsrc(p.Ac + (size_t)m0 * row + skip, (uint64_t)min(BM, p.m - m0) * row - skip),
                 make_rsrc(p.Wc + (size_t)n0 * row + skip, (uint64_t)min(BN, p.n - n0) * row - skip), row, row,
                 row - skip, s1 - s0};
  const Scales sc{p.As + (size_t)s0 * cells * 64, p.Ws, cells, n0 / 128 * blocks + s0, 1, blocks, nb - n0 / 128};
  typename Core::Acc acc;
  Core::run(t, sc, m0, smem, acc);
  if constexpr (SPLIT)
    store_sums<Core, BN>(acc, p.sums + ((size_t)split * p.tiles_m * p.tiles_n + (size_t)tm * p.tiles_n + tn) * BM * BN);
  else
    store_tile<Core, BM, BN, NT>(acc, smem, p.out + (size_t)m0 * p.n + n0, (size_t)p.n, p.m - m0, p.n - n0);
}

// A tile of dX, or of its sum over a part of n.  W stands as the forward reads it (its rows
// along k), so LDS reads turn it.  1024 x 4096 x 11008 47 to 49 us (172 tiles of 256 x 256
// on 256 compute units; 68% of the busy ones' cycles multiply), 2048 x 4096 x 4096 34.5 us.
template <class Core, int BM, int NT>
__global__ __launch_bounds__(NT) void lora_fp8_bwd_kernel(Fp8Product p) {
  __shared__ __attribute__((aligned(1024))) char smem[Core::SMEM];
  int tm, tn;
  const int tiles = p.tiles_m * p.tiles_n, split = (int)blockIdx.x / tiles;
  tile_coords(p.tiles_m, p.tiles_n, 8, (int)blockIdx.x - split * tiles, tm, tn);
  const int m0 = tm * BM, l0 = tn * 256, stages = (p.n + 127) / 128, kb = (p.k + 127) / 128;
  const uint32_t arow = (uint32_t)stages * 128, brow = (uint32_t)kb * 128;
  const NnTile t{make_rsrc(p.Ac + (size_t)m0 * arow, (uint64_t)min(BM, p.m - m0) * arow), arow,
                 reinterpret_cast<const char*>(p.Wc) + l0, brow, (uint64_t)p.n * brow - l0, stages};
  const Scales sc{p.As, p.Ws, (p.m + 63) / 64, l0 / 128, kb, 1, kb - l0 / 128};
  typename Core::Acc acc;
  const int s0 = (int)((int64_t)stages * split / p.splits), s1 = (int)((int64_t)stages * (split + 1) / p.splits);
  Core::run(t, sc, m0, s0, s1, smem, acc);
  if (p.splits == 1) {
    store_tile<Core, BM, 256, NT>(acc, smem, p.out + (size_t)m0 * p.k + l0, (size_t)p.k, p.m - m0, p.k - l0);
  } else {
    store_sums<Core, 256>(acc, p.sums + ((size_t)split * tiles + (size_t)tm * p.tiles_n + tn) * BM * 256);
  }
}

// The sum of a split product's parts, in their order (the result does not depend on who
// comes first): 4 columns a thread, from the last-level cache where the parts still are.
// Tiles of 64 x BN; out has m rows of n.
template <int BN>
__global__ __launch_bounds__(256) void lora_fp8_join_kernel(const float* __restrict__ sums, u16* __restrict__ out, int m,
                                                            int n, int tiles_n, int tiles, int splits) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int per = n / 4, row = (int)(e / per), col = 4 * (int)(e - (int64_t)row * per);
  if (row >= m) return;
  const float* from = sums + ((size_t)(row / 64) * tiles_n + col / BN) * 64 * BN + (row & 63) * BN + col % BN;
  floatx4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < splits; ++s) v += *reinterpret_cast<const floatx4*>(from + (size_t)s * tiles * 64 * BN);
  *reinterpret_cast<uint2*>(out + (size_t)row * n + col) = bf16x4(v);
}

hipError_t launch_fp8_quantize(const Fp8QuantArgs& a, hipStream_t st) {
  const int blocks = (int)fp8_blocks(a.k), cells = (int)fp8_cells(a.rows);
  if (a.block_rows == 1)
    hipLaunchKernelGGL(lora_fp8_quantize_rows_kernel, dim3((unsigned)(cells * 4 * (int)cdiv(blocks, 4))), dim3(256), 0, st, a.X, a.codes, a.scales, (int)a.rows, (int)a.k, blocks, cells);
  else
    hipLaunchKernelGGL(lora_fp8_quantize_block_kernel, dim3((unsigned)(cdiv(a.rows, 128) * blocks)), dim3(256), 0, st,
                       a.X, a.codes, a.scales, (int)a.rows, (int)a.k, blocks);
  return hipGetLastError();
}

hipError_t launch_fp8_dequantize(const uint8_t* codes, const uint8_t* scales, uint16_t* X, int64_t rows, int64_t k,
                                 int block_rows, hipStream_t st) {
  const dim3 grid((unsigned)cdiv(rows * (k / 8), 256));
  if (block_rows == 1)
    hipLaunchKernelGGL((lora_fp8_dequantize_kernel<true>), grid, dim3(256), 0, st, codes, scales, X, (int)rows, (int)k,
                       (int)fp8_blocks(k), (int)fp8_cells(rows));
  else
    hipLaunchKernelGGL((lora_fp8_dequantize_kernel<false>), grid, dim3(256), 0, st, codes, scales, X, (int)rows, (int)k,
                       (int)fp8_blocks(k), (int)fp8_cells(rows));
  return hipGetLastError();
}

static hipError_t quantise_input(const Fp8Args& a, int64_t cols, const Fp8Layout& L, hipStream_t st) {
  return launch_fp8_quantize(Fp8QuantArgs{a.A, reinterpret_cast<uint8_t*>(a.ws + L.codes),
                                          reinterpret_cast<uint8_t*>(a.ws + L.scales), a.m, cols, 1}, st);
}
static Fp8Product product_of(const Fp8Args& a, const Fp8Layout& L, const Fp8Plan& p) {
  return Fp8Product{reinterpret_cast<uint8_t*>(a.ws + L.codes), reinterpret_cast<uint8_t*>(a.ws + L.scales), a.Wc, a.Ws,
                    a.out, reinterpret_cast<float*>(a.ws + L.sums), (int)a.m, (int)a.n, (int)a.k, p.tiles_m, p.tiles_n,
                    p.splits};
}

template <class Core, int BM, int BN, int NT>
static hipError_t run_fwd_tile(const Fp8Plan& p, const Fp8Product& q, hipStream_t st) {
  hipLaunchKernelGGL((lora_fp8_fwd_kernel<Core, BM, BN, NT, false>), dim3((unsigned)p.grid), dim3(NT), 0, st, q);
  return hipGetLastError();
}
template <int BN>
static hipError_t run_join(const Fp8Plan& p, const Fp8Product& q, int cols, hipStream_t st) {
  hipLaunchKernelGGL((lora_fp8_join_kernel<BN>), dim3((unsigned)cdiv((int64_t)q.m * (cols / 4), 256)), dim3(256), 0, st, q.sums,
                     q.out, q.m, cols, p.tiles_n, p.tiles_m * p.tiles_n, p.splits);
  return hipGetLastError();
}
template <int TG, int D>
static hipError_t run_few(const Fp8Plan& p, const Fp8Product& q, hipStream_t st) {
  hipLaunchKernelGGL((lora_fp8_few_kernel<TG, D>), dim3((unsigned)p.grid), dim3(512), 0, st, q);
  return hipGetLastError();
}
template <int KS>
static hipError_t run_token(const Fp8Plan& p, const Fp8Product& q, const Fp8Args& a, hipStream_t st) {
  hipLaunchKernelGGL((lora_fp8_token_kernel<KS, 4>), dim3((unsigned)p.grid), dim3(512), fp8_token_lds(a.m, a.k), st, q, a.A);
  return hipGetLastError();
}

hipError_t launch_fp8_fwd(const Fp8Args& a, hipStream_t st) {
  const Fp8Layout L = fp8_fwd_layout(a.m, a.n, a.k);
  const Fp8Plan p = plan_fp8_fwd(a.m, a.n, a.k);
  const Fp8Product q = product_of(a, L, p);
  if (p.kind == FP8_TOKEN_8) return run_token<8>(p, q, a, st);
  if (p.kind == FP8_TOKEN_2) return run_token<2>(p, q, a, st);
  const hipError_t e = quantise_input(a, a.k, L, st);
  if (e != hipSuccess) return e;
  switch (p.kind) {
    case FP8_FEW_1: return run_few<1, 4>(p, q, st);
    case FP8_FEW_2: return run_few<2, 2>(p, q, st);
    case FP8_64x64: return run_fwd_tile<NtCore<Fp8, 64, 64, 1, 4, 4, false>, 64, 64, 256>(p, q, st);
    case FP8_64x128: return run_fwd_tile<NtCore<Fp8, 64, 128, 1, 4, 3, false>, 64, 128, 256>(p, q, st);
    case FP8_64x128_DEEP: {
      using Core = NtCore<Fp8, 64, 128, 1, 4, 4, false>;
      if (p.splits == 1) return run_fwd_tile<Core, 64, 128, 256>(p, q, st);
      hipLaunchKernelGGL((lora_fp8_fwd_kernel<Core, 64, 128, 256, true>), dim3((unsigned)p.grid), dim3(256), 0, st, q);
      const hipError_t f = hipGetLastError();
      return f == hipSuccess ? run_join<128>(p, q, (int)a.n, st) : f;
    }
    case FP8_128x128: return run_fwd_tile<NtCore<Fp8, 128, 128, 2, 4, 3, false>, 128, 128, 512>(p, q, st);
    case FP8_256x128: return run_fwd_tile<NtCore<Fp8, 256, 128, 4, 2, 3, false>, 256, 128, 512>(p, q, st);
    default: return run_fwd_tile<NtBig<Fp8, false>, 256, 256, 512>(p, q, st);
  }
}

template <class Core, int BM, int NT>
static hipError_t run_bwd_tile(const Fp8Plan& p, const Fp8Product& q, hipStream_t st) {
  hipLaunchKernelGGL((lora_fp8_bwd_kernel<Core, BM, NT>), dim3((unsigned)p.grid), dim3(NT), 0, st, q);
  return hipGetLastError();
}

hipError_t launch_fp8_bwd(const Fp8Args& a, hipStream_t st) {
  const Fp8Layout L = fp8_bwd_layout(a.m, a.n, a.k);
  hipError_t e = quantise_input(a, a.n, L, st);
  if (e != hipSuccess) return e;
  const Fp8Plan p = plan_fp8_bwd(a.m, a.n, a.k);
  const Fp8Product q = product_of(a, L, p);
  switch (p.kind) {
    case FP8_BACK_64x256: e = run_bwd_tile<NnCore<Fp8, 64, 256, 1, 4, 3>, 64, 256>(p, q, st); break;
    case FP8_BACK_128x256: e = run_bwd_tile<NnCore<Fp8, 128, 256, 2, 4, 3>, 128, 512>(p, q, st); break;
    default: e = run_bwd_tile<NnBig<Fp8>, 256, 512>(p, q, st); break;
  }
  return e != hipSuccess || p.splits == 1 ? e : run_join<256>(p, q, (int)a.k, st);
}

}  // namespace lora
