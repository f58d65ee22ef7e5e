// Cross entropy of an output layer without its logits: for z = X W^T [rows, vocab]
// and each row's label y,
//   loss = log sum_v e^z_v - z_y,   G = dloss (softmax(z) - [v = y]),
//   dX = G W,   dW = G^T X.
//
// The logits exist as the sums of a tile alone.  The forward leaves of a tile the
// maximum and the sum of exponentials of each row, which a small kernel joins.  The
// gradient needs G as the operand of a second product, so the vocabulary is walked
// in pieces whose G (or exponentials) stand in a buffer in bf16.
//
// One call for loss and dX (lora_xent_step without dW) forms the logits once: a
// piece's exponentials are taken against a reference r of each row instead of its
// normaliser, sum_v 2^(z_v log2 e - r) W_v is carried from piece to piece in fp32,
// and divided at the end.  r is 0 until a piece's largest logit is more than 64
// above it or, in the first piece, more than 40 below it (in powers of two; bf16 and
// fp32 hold 2^126): then the tiles of those rows are formed again against the
// maximum, and what is carried is scaled.  So any logits come out right, and
// ordinary ones at the price of two products.  A gradient of W needs the normaliser
// in front of its sum over rows: with dW the forward runs first, and the logits are
// formed again.
//
// The label's own gradient, softmax - 1, is taken as less the sum of all others', so
// that a row sure of its label keeps its digits; the label is left out of the
// sums and of the operand of the one-pass form, and joins at the end.
//
// Exponents are in powers of two: v_exp_f32 of fma(z, log2 e, -r).
#include "lora_device.hpp"
#include "lora_gemm.hpp"
#include "lora_train.hpp"

namespace lora {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -1e30f;   // below any logit that counts

struct Part {   // of a row's logits in a tile: largest (times log2 e), sum of powers
  float m, s;
};

enum XentMode { XENT_STATS, XENT_PIECE, XENT_GRAD };

struct XentLogits {
  const u16 *X, *W;
  const int32_t* labels;
  XentRow* row;
  const float* saved;   // XENT_GRAD: of the forward
  const float* dloss;
  Part* parts;          // [tile of this launch][rows_pad]
  const int32_t* flags; // XENT_PIECE, the tiles formed again: of the row tiles
  int only;             // ... those whose flag has this value (0: all)
  u16 *piece, *turned;  // [rows_pad][piece], [piece][rows_pad]
  int rows, vocab, k, tiles_m, tiles_n, tile0;
  int64_t rows_pad, piece_cols;
};

template <class Core, int BM, int BN, int NT, int MODE>
__global__ __launch_bounds__(NT) void lora_xent_logits_kernel(XentLogits p) {
  constexpr int FA = sizeof(typename Core::Acc) / sizeof(floatx4[sizeof(typename Core::Acc{}[0]) / sizeof(floatx4)]);
  constexpr int FB = sizeof(typename Core::Acc{}[0]) / sizeof(floatx4);
  constexpr int NW = NT / 64, TM = 16 * FB, WN = NW / (BM / TM);
  constexpr int SMEM = Core::SMEM > BM * BN * 2 ? Core::SMEM : BM * BN * 2;
  __shared__ __attribute__((aligned(1024))) char smem[SMEM];
  __shared__ Part joined[WN][BM];
  __shared__ int label[BM];
  __shared__ float ref[BM], scale[BM], own[BM];
  int tm, tn;
  tile_coords(p.tiles_m, p.tiles_n, 8, (int)blockIdx.x, tm, tn);
  if (MODE == XENT_PIECE && p.only && p.flags[tm] != p.only) return;
  const int m0 = tm * BM, n0 = (p.tile0 + tn) * BN, tid = threadIdx.x;
  for (int i = tid; i < BM; i += NT) {   // (read behind the core's barriers)
    const int row = m0 + i, y = row < p.rows ? p.labels[row] : -1;
    const bool known = y >= 0 && y < p.vocab;
    label[i] = known ? y : -1;
    if (MODE == XENT_PIECE) ref[i] = p.row[row].ref;
    if (MODE == XENT_GRAD) {
      const float d = known ? p.dloss[row] : 0.0f;
      ref[i] = known ? p.saved[2 * row] : 0.0f;
      scale[i] = d;
      own[i] = known ? -d * p.saved[2 * row + 1] : 0.0f;
    }
  }
  const uint32_t rowb = (uint32_t)p.k * 2;
  const NtTile t{make_rsrc(p.X + (size_t)m0 * p.k, (uint64_t)min(BM, p.rows - m0) * rowb),
                 make_rsrc(p.W + (size_t)n0 * p.k, (uint64_t)min(BN, p.vocab - n0) * rowb), rowb, rowb, rowb, (p.k + 63) / 64};
  typename Core::Acc acc;
  Core::run(t, Scales{}, m0, smem, acc);
  __syncthreads();

  const int lane = lane_fresh(), wave = uniform(tid >> 6), g = lane >> 4, c16 = lane & 15;
  const int r0 = Core::row0(wave), wn = wave % WN;
#pragma unroll
  for (int b = 0; b < FB; ++b) {
    const int i = r0 + 16 * b + c16, y = label[i];
    if constexpr (MODE != XENT_GRAD) {
      float top = -INFINITY;
#pragma unroll
      for (int a = 0; a < FA; ++a)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int col = n0 + Core::col(wave, a) + 4 * g + q;
          const float z = acc[a][b][q];
          if (col == y) p.row[m0 + i].zy = z;
          if (col < p.vocab && col != y) top = fmaxf(top, z);
        }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      top = fmaxf(top * kLog2e, kLowest);
      const float r = MODE == XENT_STATS ? top : ref[i];
      float sum = 0.0f;
#pragma unroll
      for (int a = 0; a < FA; ++a)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int col = n0 + Core::col(wave, a) + 4 * g + q;
          const float e = __builtin_amdgcn_exp2f(fmaf(acc[a][b][q], kLog2e, -r));
          const float v = col < p.vocab && col != y ? e : 0.0f;
          sum += v;
          if (MODE == XENT_PIECE) acc[a][b][q] = v;
        }
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (g == 0) joined[wn][i] = Part{top, sum};
    } else {
      const float r = ref[i], d = scale[i], o = own[i];
#pragma unroll
      for (int a = 0; a < FA; ++a)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int col = n0 + Core::col(wave, a) + 4 * g + q;
          const float v = d * __builtin_amdgcn_exp2f(fmaf(acc[a][b][q], kLog2e, -r));
          acc[a][b][q] = y < 0 || col >= p.vocab ? 0.0f : (col == y ? o : v);
        }
    }
  }
  // The tile as bf16 rows in LDS, 16-byte chunks swizzled by the row.
  constexpr int CH = BN / 8;
  if constexpr (MODE != XENT_STATS) {
#pragma unroll
    for (int b = 0; b < FB; ++b)
#pragma unroll
      for (int a = 0; a < FA; ++a) {
        const int row = r0 + 16 * b + c16, col = Core::col(wave, a) + 4 * g;
        const floatx4 v = acc[a][b];
        *reinterpret_cast<uint2*>(smem + row * (BN * 2) + (((col >> 3) ^ (row & (CH - 1))) << 4) + (col & 7) * 2) =
            uint2{(uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16),
                  (uint32_t)f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16)};
      }
  }
  __syncthreads();
  if constexpr (MODE != XENT_GRAD) {
    for (int i = tid; i < BM; i += NT) {
      Part v = joined[0][i];
#pragma unroll
      for (int w = 1; w < WN; ++w) {
        const Part u = joined[w][i];
        if (MODE == XENT_STATS) {
          const float m = fmaxf(v.m, u.m);
          v.s = v.s * __builtin_amdgcn_exp2f(v.m - m) + u.s * __builtin_amdgcn_exp2f(u.m - m);
          v.m = m;
        } else {
          v.s += u.s;
          v.m = fmaxf(v.m, u.m);
        }
      }
      p.parts[(size_t)tn * p.rows_pad + m0 + i] = v;
    }
  }
  if constexpr (MODE != XENT_STATS) {
    const size_t c0 = (size_t)tn * BN;
    for (int e = tid; e < BM * CH; e += NT) {
      const int row = e / CH, ch = e % CH;
      *reinterpret_cast<int4v*>(p.piece + (size_t)(m0 + row) * p.piece_cols + c0 + 8 * ch) =
          *reinterpret_cast<const int4v*>(smem + row * (BN * 2) + ((ch ^ (row & (CH - 1))) << 4));
    }
    if (MODE == XENT_GRAD && p.turned) {
      for (int e = tid; e < BN * BM / 8; e += NT) {   // 8 rows of a column; 8 neighbours a column's 64 rows
        const int rb = e & 7, rest = e >> 3, col = rest % BN, r = 64 * (rest / BN) + 8 * rb;
        int4v v;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          uint32_t w = 0;
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int row = r + 2 * h + q;
            w |= (uint32_t)*reinterpret_cast<const u16*>(smem + row * (BN * 2) + (((col >> 3) ^ (row & (CH - 1))) << 4) +
                                                         (col & 7) * 2) << (16 * q);
          }
          v[h] = (int)w;
        }
        *reinterpret_cast<int4v*>(p.turned + (c0 + col) * p.rows_pad + m0 + r) = v;
      }
    }
  }
}

// ---- a row's numbers -----------------------------------------------------------
// 16 rows x 16 threads each: max and sum over `tiles` parts of 16 rows; thread (row,
// 0) receives them.  STATS: every part has its own reference.
template <bool STATS>
__device__ __forceinline__ Part join_parts(const Part* parts, int tiles, int64_t rows_pad, int row, Part* lds) {
  const int tid = threadIdx.x, r = tid & 15;
  Part v{kLowest, 0.0f};
  auto add = [&](Part u) LORA_INLINE {
    const float m = fmaxf(v.m, u.m);
    v.s = STATS ? v.s * __builtin_amdgcn_exp2f(v.m - m) + u.s * __builtin_amdgcn_exp2f(u.m - m) : v.s + u.s;
    v.m = m;
  };
  for (int t = tid >> 4; t < tiles; t += 16) add(parts[(size_t)t * rows_pad + row]);
  __syncthreads();
  lds[tid] = v;
  __syncthreads();
  if (tid < 16)
    for (int j = 1; j < 16; ++j) add(lds[16 * j + r]);
  return v;
}

// Loss, and what the gradient needs, from the sum of all others' powers against ref
// and the label's logit.
struct RowEnd {
  float loss, lse, rest;   // lse in powers of two; rest = 1 - p_label
  float c1, c2;            // 1 / sum and - rest, against ref
};
__device__ __forceinline__ RowEnd row_end(float ref, float others, float zy, bool known) {
  RowEnd e;
  const float dy = known ? fmaf(zy, kLog2e, -ref) : -INFINITY, up = fmaxf(dy, 0.0f);   // (NaN: 0, and dy below)
  const float down = __builtin_amdgcn_exp2f(-up), rest = others * down;
  const float ey = known ? __builtin_amdgcn_exp2f(dy - up) : 0.0f, sum = rest + ey;
  const float bad = sum < INFINITY ? 0.0f : NAN;   // a NaN or an infinity among the logits
  e.loss = known ? (ey > rest ? log1pf(rest / ey) : kLn2 * (log2f(sum) - (dy - up))) + bad : 0.0f;
  e.lse = (up > 0.0f ? zy * kLog2e : ref) + log2f(sum) + bad;
  e.rest = known ? rest / sum + bad : 0.0f;
  e.c1 = known ? down / sum + bad : 0.0f;
  e.c2 = -e.rest;
  return e;
}

__global__ __launch_bounds__(256) void lora_xent_fwd_rows_kernel(const Part* __restrict__ parts,
                                                                 const XentRow* __restrict__ rowv,
                                                                 const int32_t* __restrict__ labels,
                                                                 float* __restrict__ loss, float* __restrict__ saved,
                                                                 int rows, int vocab, int tiles, int64_t rows_pad) {
  __shared__ Part lds[256];
  const int row = (int)blockIdx.x * 16 + ((int)threadIdx.x & 15);
  const Part v = join_parts<true>(parts, tiles, rows_pad, row, lds);
  if (threadIdx.x >= 16 || row >= rows) return;
  const int y = labels[row];
  const bool known = y >= 0 && y < vocab;
  const RowEnd e = row_end(v.m, v.s, known ? rowv[row].zy : 0.0f, known);
  loss[row] = e.loss;
  if (saved) {
    saved[2 * row] = e.lse;
    saved[2 * row + 1] = e.rest;
  }
}

__global__ __launch_bounds__(256) void lora_xent_begin_kernel(XentRow* row, int64_t rows_pad, int32_t* flags, int tiles_m) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < rows_pad) row[i] = XentRow{0.0f, 0.0f, kLowest, 1.0f, 0.0f, 0.0f, 0.0f, 0};
  if (i < tiles_m) flags[i] = 0;
}

// After a piece's tiles: the rows whose reference does not serve, and the others'
// sums.  `before`: the piece before's parts.
__global__ __launch_bounds__(256) void lora_xent_update_kernel(const Part* __restrict__ now, const Part* __restrict__ before,
                                                               XentRow* rowv, int32_t* flags, int tiles, int tiles_before,
                                                               int64_t rows_pad, int rows, int tile_m, int piece) {
  __shared__ Part lds[256];
  const int row = (int)blockIdx.x * 16 + ((int)threadIdx.x & 15);
  XentRow v = rowv[row];
  Part late{0.0f, 0.0f};
  if (tiles_before) late = join_parts<false>(before, tiles_before, rows_pad, row, lds);
  const Part p = join_parts<false>(now, tiles, rows_pad, row, lds);
  if (threadIdx.x >= 16) return;
  if (v.redo) v.sum += late.s;
  v.best = fmaxf(v.best, p.m);
  const bool low = piece == 0 && p.m < v.ref - 40.0f && p.m > kLowest;
  v.redo = row < rows && ((p.m > v.ref + 64.0f && p.m < INFINITY) || low);
  v.alpha = 1.0f;
  if (v.redo) {
    const float ref = ceilf(p.m);
    if (piece > 0) v.alpha = __builtin_amdgcn_exp2f(v.ref - ref);   // (below 1; nothing to scale in the first piece)
    v.sum *= v.alpha;
    v.ref = ref;
    flags[row / tile_m] = piece + 1;   // (every writer the same value)
  } else {
    v.sum += p.s;
  }
  rowv[row] = v;
}

__global__ __launch_bounds__(256) void lora_xent_end_kernel(const Part* __restrict__ last, XentRow* rowv,
                                                            const int32_t* __restrict__ labels,
                                                            const float* __restrict__ dloss, float* __restrict__ loss,
                                                            int rows, int vocab, int tiles, int64_t rows_pad) {
  __shared__ Part lds[256];
  const int row = (int)blockIdx.x * 16 + ((int)threadIdx.x & 15);
  const Part p = join_parts<false>(last, tiles, rows_pad, row, lds);
  if (threadIdx.x >= 16 || row >= rows) return;
  const XentRow v = rowv[row];
  const int y = labels[row];
  const bool known = y >= 0 && y < vocab;
  const RowEnd e = row_end(v.ref, v.redo ? v.sum + p.s : v.sum, v.zy, known);
  loss[row] = e.loss;
  rowv[row].c1 = known ? dloss[row] * e.c1 : 0.0f;
  rowv[row].c2 = known ? dloss[row] * e.c2 : 0.0f;
}

// ---- the second product ----------------------------------------------------------
struct XentGrad {
  const u16 *A, *B;     // A: [rows of the output][a_cols], B: [contraction][k]
  float* sums;          // [split][tile][fragment][thread][4], or
  u16* out;             // the product itself, bf16 rows of k
  const XentRow* row;   // their alpha scales the sums so far (or none)
  bool first;           // no sums so far
  int64_t a_cols, b_rows;
  int m, k, stages, tiles_m, tiles_n, splits;
};

template <class Core, int BM, int NT>
__global__ __launch_bounds__(NT) void lora_xent_grad_kernel(XentGrad p) {
  constexpr int FA = sizeof(typename Core::Acc) / sizeof(floatx4[sizeof(typename Core::Acc{}[0]) / sizeof(floatx4)]);
  constexpr int FB = sizeof(typename Core::Acc{}[0]) / sizeof(floatx4);
  __shared__ __attribute__((aligned(1024))) char smem[Core::SMEM];
  const int tiles = p.tiles_m * p.tiles_n, split = (int)blockIdx.x / tiles;
  int tm, tn;
  tile_coords(p.tiles_m, p.tiles_n, 8, (int)blockIdx.x - split * tiles, tm, tn);
  const int m0 = tm * BM, l0 = tn * 256;
  const uint32_t arow = (uint32_t)p.a_cols * 2, brow = (uint32_t)p.k * 2;
  const NnTile t{make_rsrc(p.A + (size_t)m0 * p.a_cols, (uint64_t)min(BM, p.m - m0) * arow), arow,
                 reinterpret_cast<const char*>(p.B + l0), brow, (uint64_t)p.b_rows * brow - (uint64_t)l0 * 2, p.stages};
  typename Core::Acc acc;
  const int s0 = (int)((int64_t)p.stages * split / p.splits), s1 = (int)((int64_t)p.stages * (split + 1) / p.splits);
  Core::run(t, Scales{}, m0, s0, s1, smem, acc);
  const int lane = lane_fresh(), wave = uniform((int)threadIdx.x >> 6), g = lane >> 4, c16 = lane & 15;
  if (p.sums) {
    floatx4* to = reinterpret_cast<floatx4*>(p.sums) + ((size_t)split * tiles + (size_t)tm * p.tiles_n + tn) * (FA * FB * NT) + threadIdx.x;
#pragma unroll
    for (int b = 0; b < FB; ++b) {
      const float alpha = p.row ? p.row[m0 + Core::row0(wave) + 16 * b + c16].alpha : 1.0f;
#pragma unroll
      for (int a = 0; a < FA; ++a) {
        floatx4 v = acc[a][b];
        if (!p.first) v += to[(a * FB + b) * NT] * alpha;
        to[(a * FB + b) * NT] = v;
      }
    }
  } else {
#pragma unroll
    for (int b = 0; b < FB; ++b) {
      const int row = m0 + Core::row0(wave) + 16 * b + c16;
#pragma unroll
      for (int a = 0; a < FA; ++a) {
        const int col = l0 + Core::col(wave, a) + 4 * g;
        const floatx4 v = acc[a][b];
        if (row < p.m && col < p.k)
          *reinterpret_cast<uint2*>(p.out + (size_t)row * p.k + col) =
              uint2{(uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16),
                    (uint32_t)f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16)};
      }
    }
  }
}

// The sums of all splits, in their order, as dX: with the rows' numbers c1 sum + c2 W_y,
// without them as they are.  A workgroup takes a tile's 4 fragments.
template <class Core, int BM, int NT>
__global__ __launch_bounds__(NT) void lora_xent_join_kernel(const float* __restrict__ sums, const XentRow* __restrict__ rowv,
                                                            const int32_t* __restrict__ labels, const u16* __restrict__ W,
                                                            u16* __restrict__ dX, int rows, int vocab, int k, int tiles_n,
                                                            int tiles, int splits) {
  constexpr int FA = sizeof(typename Core::Acc) / sizeof(floatx4[sizeof(typename Core::Acc{}[0]) / sizeof(floatx4)]);
  constexpr int FB = sizeof(typename Core::Acc{}[0]) / sizeof(floatx4);
  constexpr int PER = FA * FB / 4;
  const int tile = (int)blockIdx.x / PER, f0 = (int)blockIdx.x % PER * 4;
  const int m0 = tile / tiles_n * BM, l0 = tile % tiles_n * 256;
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), g = lane >> 4, c16 = lane & 15;
  for (int f = f0; f < f0 + 4; ++f) {
    const int a = f % FA, b = f / FA;
    const int row = m0 + Core::row0(wave) + 16 * b + c16, col = l0 + Core::col(wave, a) + 4 * g;
    const floatx4* from = reinterpret_cast<const floatx4*>(sums) + (size_t)tile * (FA * FB * NT) + (a * FB + b) * NT + threadIdx.x;
    floatx4 v{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < splits; ++s) v += from[(size_t)s * tiles * (FA * FB * NT)];
    if (row >= rows || col >= k) continue;
    if (rowv) {
      const int y = labels[row];
      const bool known = y >= 0 && y < vocab;
      const float c1 = rowv[row].c1, c2 = rowv[row].c2;
      const uint2 w = *reinterpret_cast<const uint2*>(W + (size_t)(known ? y : 0) * k + col);
      v[0] = known ? c1 * v[0] + c2 * bf16_to_f32((u16)w.x) : 0.0f;
      v[1] = known ? c1 * v[1] + c2 * bf16_to_f32((u16)(w.x >> 16)) : 0.0f;
      v[2] = known ? c1 * v[2] + c2 * bf16_to_f32((u16)w.y) : 0.0f;
      v[3] = known ? c1 * v[3] + c2 * bf16_to_f32((u16)(w.y >> 16)) : 0.0f;
    }
    *reinterpret_cast<uint2*>(dX + (size_t)row * k + col) =
        uint2{(uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16),
              (uint32_t)f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16)};
  }
}

// ---- launches ----------------------------------------------------------------------
using GradBig = NnBig<Bf16>;
using GradSmall = NnCore<Bf16, 64, 256, 4, 3>;

template <int MODE, bool TAIL>
static hipError_t run_logits_of(const XentPlan& p, const XentLogits& q, hipStream_t st) {
  const dim3 grid((unsigned)(q.tiles_m * q.tiles_n));
  if (p.big)
    hipLaunchKernelGGL((lora_xent_logits_kernel<NtBig<Bf16, TAIL>, 256, 256, 512, MODE>), grid, dim3(512), 0, st, q);
  else
    hipLaunchKernelGGL((lora_xent_logits_kernel<NtCore<Bf16, 64, 128, 1, 4, 3, TAIL>, 64, 128, 256, MODE>), grid,
                       dim3(256), 0, st, q);
  return hipGetLastError();
}
template <int MODE>
static hipError_t run_logits(const XentPlan& p, const XentLogits& q, hipStream_t st) {
  return q.k % 64 ? run_logits_of<MODE, true>(p, q, st) : run_logits_of<MODE, false>(p, q, st);
}
static hipError_t run_grad(bool big, const XentGrad& q, hipStream_t st) {
  const dim3 grid((unsigned)(q.tiles_m * q.tiles_n * q.splits));
  if (big) hipLaunchKernelGGL((lora_xent_grad_kernel<GradBig, 256, 512>), grid, dim3(512), 0, st, q);
  else hipLaunchKernelGGL((lora_xent_grad_kernel<GradSmall, 64, 256>), grid, dim3(256), 0, st, q);
  return hipGetLastError();
}
static hipError_t run_join(const XentPlan& p, const XentArgs& a, const XentLayout& L, bool step, hipStream_t st) {
  const int tiles = p.tiles_m * p.tiles_k;
  const float* sums = reinterpret_cast<const float*>(a.ws + L.sums);
  const XentRow* row = step ? reinterpret_cast<const XentRow*>(a.ws + L.rows) : nullptr;
  if (p.big)
    hipLaunchKernelGGL((lora_xent_join_kernel<GradBig, 256, 512>), dim3((unsigned)(tiles * 8)), dim3(512), 0, st, sums, row,
                       a.labels, a.W, a.dX, (int)a.rows, (int)a.vocab, (int)a.k, p.tiles_k, tiles, p.splits);
  else
    hipLaunchKernelGGL((lora_xent_join_kernel<GradSmall, 64, 256>), dim3((unsigned)(tiles * 4)), dim3(256), 0, st, sums, row,
                       a.labels, a.W, a.dX, (int)a.rows, (int)a.vocab, (int)a.k, p.tiles_k, tiles, p.splits);
  return hipGetLastError();
}

static XentLogits logits_of(const XentArgs& a, const XentPlan& p, const XentLayout& L) {
  XentLogits q{};
  q.X = a.X; q.W = a.W; q.labels = a.labels;
  q.row = reinterpret_cast<XentRow*>(a.ws + L.rows);
  q.dloss = a.dloss;
  q.parts = reinterpret_cast<Part*>(a.ws + L.parts);
  q.flags = reinterpret_cast<int32_t*>(a.ws + L.flags);
  q.piece = reinterpret_cast<u16*>(a.ws + L.piece);
  q.rows = (int)a.rows; q.vocab = (int)a.vocab; q.k = (int)a.k;
  q.tiles_m = p.tiles_m; q.tiles_n = p.vtiles;
  q.rows_pad = p.rows_pad; q.piece_cols = p.piece;
  return q;
}
// dX's part of piece i, from its buffer.
static XentGrad piece_grad(const XentArgs& a, const XentPlan& p, const XentLayout& L, int i) {
  XentGrad g{};
  const int64_t v0 = i * p.piece;
  g.A = reinterpret_cast<const u16*>(a.ws + L.piece);
  g.B = a.W + v0 * a.k;
  g.sums = reinterpret_cast<float*>(a.ws + L.sums);
  g.first = i == 0;
  g.a_cols = p.piece;
  g.b_rows = std::min(p.piece, a.vocab - v0);
  g.m = (int)p.rows_pad; g.k = (int)a.k;
  g.stages = (int)cdiv(g.b_rows, 64);
  g.tiles_m = p.tiles_m; g.tiles_n = p.tiles_k; g.splits = p.splits;   // (in a short last piece some have nothing but their scaling to do)
  return g;
}

#define LORA_TRY(call)                     \
  do {                                     \
    const hipError_t e_ = (call);          \
    if (e_ != hipSuccess) return e_;       \
  } while (0)

static hipError_t forward(const XentArgs& a, const XentLayout& L, float* saved, hipStream_t st) {
  const XentPlan p = plan_xent(a.rows, a.vocab, a.k);
  const XentLogits q = logits_of(a, p, L);
  LORA_TRY(run_logits<XENT_STATS>(p, q, st));
  hipLaunchKernelGGL(lora_xent_fwd_rows_kernel, dim3((unsigned)cdiv(a.rows, 16)), dim3(256), 0, st, q.parts, q.row, a.labels,
                     a.loss, saved, (int)a.rows, (int)a.vocab, p.vtiles, p.rows_pad);
  return hipGetLastError();
}

static hipError_t backward(const XentArgs& a, const XentLayout& L, const float* saved, hipStream_t st) {
  const XentPlan p = plan_xent(a.rows, a.vocab, a.k);
  XentLogits q = logits_of(a, p, L);
  q.saved = saved;
  q.turned = a.dW ? reinterpret_cast<u16*>(a.ws + L.turned) : nullptr;
  for (int i = 0; i < p.pieces; ++i) {
    q.tile0 = i * p.piece_tiles;
    q.tiles_n = std::min(p.piece_tiles, p.vtiles - q.tile0);
    LORA_TRY(run_logits<XENT_GRAD>(p, q, st));
    if (a.dX) LORA_TRY(run_grad(p.big, piece_grad(a, p, L, i), st));
    if (a.dW) {
      const int64_t v0 = i * p.piece, cols = std::min(p.piece, a.vocab - v0);
      XentGrad g{};
      g.A = q.turned; g.B = a.X; g.out = a.dW + v0 * a.k;
      g.a_cols = p.rows_pad; g.b_rows = a.rows;
      g.m = (int)cols; g.k = (int)a.k;
      g.stages = (int)(p.rows_pad / 64);
      g.tiles_m = (int)cdiv(cols, 256); g.tiles_n = p.tiles_k; g.splits = 1;
      LORA_TRY(run_grad(true, g, st));
    }
  }
  return a.dX ? run_join(p, a, L, false, st) : hipSuccess;
}

hipError_t launch_xent_fwd(const XentArgs& a, hipStream_t st) {
  return forward(a, xent_layout(a.rows, a.vocab, a.k, false, false), a.saved, st);
}

hipError_t launch_xent_bwd(const XentArgs& a, hipStream_t st) {
  return backward(a, xent_layout(a.rows, a.vocab, a.k, a.dX != nullptr, a.dW != nullptr), a.saved, st);
}

hipError_t launch_xent_step(const XentArgs& a, hipStream_t st) {
  const XentLayout L = xent_layout(a.rows, a.vocab, a.k, a.dX != nullptr, a.dW != nullptr);
  if (a.dW) {
    float* saved = reinterpret_cast<float*>(a.ws + L.saved);
    LORA_TRY(forward(a, L, saved, st));
    return backward(a, L, saved, st);
  }
  const XentPlan p = plan_xent(a.rows, a.vocab, a.k);
  XentLogits q = logits_of(a, p, L);
  Part* parts[2] = {q.parts, q.parts + (size_t)p.piece_tiles * p.rows_pad};
  int32_t* flags = reinterpret_cast<int32_t*>(a.ws + L.flags);
  hipLaunchKernelGGL(lora_xent_begin_kernel, dim3((unsigned)cdiv(p.rows_pad, 256)), dim3(256), 0, st, q.row, p.rows_pad,
                     flags, p.tiles_m);
  LORA_TRY(hipGetLastError());
  int tiles_before = 0;
  for (int i = 0; i < p.pieces; ++i) {
    q.tile0 = i * p.piece_tiles;
    q.tiles_n = std::min(p.piece_tiles, p.vtiles - q.tile0);
    q.parts = parts[i & 1];
    q.only = 0;
    LORA_TRY(run_logits<XENT_PIECE>(p, q, st));
    hipLaunchKernelGGL(lora_xent_update_kernel, dim3((unsigned)(p.rows_pad / 16)), dim3(256), 0, st, q.parts,
                       parts[(i + 1) & 1], q.row, flags, q.tiles_n, tiles_before, p.rows_pad, (int)a.rows, p.tile_m, i);
    LORA_TRY(hipGetLastError());
    q.only = i + 1;
    LORA_TRY(run_logits<XENT_PIECE>(p, q, st));
    tiles_before = q.tiles_n;
    XentGrad g = piece_grad(a, p, L, i);
    g.row = q.row;
    LORA_TRY(run_grad(p.big, g, st));
  }
  hipLaunchKernelGGL(lora_xent_end_kernel, dim3((unsigned)cdiv(a.rows, 16)), dim3(256), 0, st, q.parts, q.row, a.labels,
                     a.dloss, a.loss, (int)a.rows, (int)a.vocab, tiles_before, p.rows_pad);
  LORA_TRY(hipGetLastError());
  return run_join(p, a, L, true, st);
}

}  // namespace lora
