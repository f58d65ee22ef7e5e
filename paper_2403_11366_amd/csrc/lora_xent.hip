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
// normaliser, sum_v e^(z_v - r) W_v is carried from piece to piece in fp32,
// and divided at the end.  r is 0 until a piece's largest logit is more than 44
// above it or, in the first piece, more than 28 below it (e^44 is 2^63, e^-28 2^-40;
// bf16 and fp32 hold 2^126): then the tiles of those rows are formed again against the
// maximum, and what is carried is scaled.  (A piece whose logits all have probability 0 in
// a row leaves the next one that row's first.)  So any logits come out right, and
// ordinary ones at the price of two products and, for each piece, of a launch that
// finds nothing to do (4 us).  For few rows, whose piece is the whole vocabulary, that
// launch and the references' are saved: a tile's powers are taken against its own
// largest, rounded up to a power of two, and the second product, which knows the row's
// by then, subtracts the difference from their exponents where it reads them.  A
// gradient of W needs the normaliser in front of its sum over rows: with dW the forward
// runs first, and the logits are formed again.
//
// The label's own gradient, softmax - 1, is taken as less the sum of all others', so
// that a row sure of its label keeps its digits; the label is left out of the
// sums and of the operand of the one-pass form, and joins at the end.  In the other
// form what its bf16 loses is added to dX's and dW's sums: with few rows that is the
// largest error of dW by far (1500 x 50021: error against 64 bits 0.0022 -> 0.0017 of the
// result, the plain form's).
//
// References are logits, and a power is v_exp_f32 of (z - r) log2 e: the difference first,
// so that a logit that is its own reference has the power 1 however large it is.  (A
// reference in rounded powers of two is off by 2^-24 of itself, and from 1e9 on that is
// more than fp32's exponents: a masked tile at -1e10 made its row's sum infinite.)
//
// What bounds it: with many rows the two (with dW four) products, on the matrix cores --
// loss and dX of 4096 rows, vocabulary 32000, k 4096 in 1.58 ms, the two products alone
// 1.56 ms at the rate of a library's product of that size; a piece's logits 200 us, its
// part of dX 204 us, 75% of the busy compute units' cycles multiplying.  With few rows the
// bytes of W, read once for the logits and once for dX: 37 rows 124 us, of which the two
// reads of 262 MB take 42 and 50 us (6.3 and 5.2 TB/s).  A second reading from the
// last-level cache was tried, in pieces that fit it: a launch for each piece cost more
// than the cache's rate gave.
#include "lora_device.hpp"
#include "lora_gemm.hpp"
#include "lora_train.hpp"

namespace lora {

constexpr float kLog2e = 1.44269504088896340736f, kLog2eLow = 1.925963033500e-8f;   // log2 e = their sum
constexpr float kLowest = -3.4028234663852886e38f;   // the lowest finite logit
constexpr float kNone = -INFINITY;                   // the largest of no logits

struct Part {   // of a row's logits in a tile: reference, sum of powers against it
  float m, s;
};
__device__ __forceinline__ float power(float z, float ref) { return __builtin_amdgcn_exp2f((z - ref) * kLog2e); }

// References of a tile's own (XENT_LOCAL): the power of two next to e^top, so that a tile's
// powers differ from another's by a whole exponent.  2^(t log2 e + c): from 2^28 on, where
// different logits lie 46 powers and more apart, e^top itself.
struct Whole {
  float t, c;
};
__device__ __forceinline__ Whole whole_power(float top) {
  return fabsf(top) < 268435456.0f ? Whole{0.0f, ceilf(top * kLog2e)} : Whole{top, 0.0f};
}
// log2 of e^top over that reference: about -1 .. 0.
__device__ __forceinline__ float past_whole(float top) {
  const Whole w = whole_power(top);
  return fmaf(top - w.t, kLog2e, -w.c) + (top - w.t) * kLog2eLow;
}
// By how many powers of two the reference of m is above that of top, m >= top.
__device__ __forceinline__ float powers_above(float m, float top) {
  const Whole a = whole_power(m), b = whole_power(top);
  return ceilf(fmaf(a.t - b.t, kLog2e, a.c - b.c));
}

// What a row's backward reads: log sum e^z and 1 - p of its label.  From 2^16 on, where the
// logarithm's spacing shows in e^(z - it), instead the largest logit but the label's, and
// 1 - p and what powers against that logit are multiplied by, each as bf16 and apart by
// the sign (1 - p has none).
struct Saved {
  float ref, scale, rest;
};
__device__ __forceinline__ void save_row(float* to, float lse, const Saved& wide) {
  const bool far = fabsf(lse) >= 65536.0f;
  const uint32_t both = 0x80000000u | (uint32_t)f32_to_bf16(wide.rest) << 16 | f32_to_bf16(wide.scale);
  to[0] = far ? wide.ref : lse;
  to[1] = far ? __builtin_bit_cast(float, both) : wide.rest;
}
__device__ __forceinline__ Saved saved_row(const float* at) {
  const uint32_t b = __builtin_bit_cast(uint32_t, at[1]);
  if (!(b >> 31)) return Saved{at[0], 1.0f, at[1]};
  return Saved{at[0], bf16_to_f32((u16)b), bf16_to_f32((u16)(b >> 16 & 0x7FFFu))};
}

enum XentMode { XENT_STATS, XENT_PIECE, XENT_AGAIN, XENT_LOCAL, XENT_GRAD };

struct XentLogits {
  const u16 *X, *W;
  const int32_t* labels;
  float* ref;            // [rows_pad] of this piece; XENT_AGAIN writes the next one's behind it
  float* ref_next;
  uint32_t* best;        // [rows_pad] of this piece
  uint32_t* best_next;
  const float* saved;    // XENT_GRAD: of the forward
  const float* dloss;
  float* coef;           // XENT_GRAD of the first piece: [rows_pad][2], written (or none)
  Part* parts;           // [tile][rows_pad]
  u16 *piece, *turned;   // [rows_pad][piece], [piece][rows_pad]
  int rows, vocab, k, tiles_m, tiles_n, tile0;
  int64_t rows_pad, piece_cols;
};

// Floats as unsigned numbers of the same order (for a maximum whose order of arrival
// does not matter); NaNs do not reach it.
__device__ __forceinline__ uint32_t ordered(float f) {
  const uint32_t b = __builtin_bit_cast(uint32_t, f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t u) {
  return __builtin_bit_cast(float, u & 0x80000000u ? u & 0x7FFFFFFFu : ~u);
}
// The reference that serves a row whose largest logit in a piece is `best`.  A row that
// has met no finite logit has the reference kNoLogit, a 0 apart by its sign: its
// sums are 0, so that it may still move down.
constexpr float kNoLogit = -0.0f;
__device__ __forceinline__ float served_by(float ref, float best) {
  const bool none = __builtin_bit_cast(uint32_t, ref) == 0x80000000u, some = best > kNone;
  const bool high = best > ref + 44.0f && best < INFINITY, low = none && some && best < -28.0f;
  return high || low ? best : (none && some ? 0.0f : ref);
}

// One tile of logits: the product's sums are what the epilogue works on, in registers;
// exponentials (or G) leave through LDS in whole row pieces.
template <class Core, int BM, int BN, int NT, int MODE>
struct XentTile {
  static constexpr int FA = std::extent_v<typename Core::Acc, 0>, FB = std::extent_v<typename Core::Acc, 1>;
  static constexpr int NW = NT / 64, TM = 16 * FB, WN = NW / (BM / TM);
  static constexpr int SMEM = Core::SMEM > BM * BN * 2 ? Core::SMEM : BM * BN * 2;
  static constexpr bool EXPS = MODE == XENT_PIECE || MODE == XENT_AGAIN || MODE == XENT_LOCAL;   // powers against ref
  struct Lds {
    char stages[SMEM];
    Part joined[WN][BM];
    int label[BM];       // or -1
    float ref[BM], scale[BM], own[BM];
  };

  static __device__ __forceinline__ void run(const XentLogits& p, int tm, int tn, Lds& lds) {
    const int m0 = tm * BM, n0 = (p.tile0 + tn) * BN;
    const uint32_t rowb = (uint32_t)p.k * 2;
    const NtTile t{make_rsrc(p.X + (size_t)m0 * p.k, (uint64_t)min(BM, p.rows - m0) * rowb),
                   make_rsrc(p.W + (size_t)n0 * p.k, (uint64_t)min(BN, p.vocab - n0) * rowb), rowb, rowb, rowb,
                   (p.k + 63) / 64};
    typename Core::Acc acc;
    Core::run(t, Scales{}, m0, lds.stages, acc);
    __syncthreads();
    const int lane = lane_fresh(), tid = threadIdx.x, wave = uniform(tid >> 6), g = lane >> 4, c16 = lane & 15;
    const int r0 = Core::row0(wave), wn = wave % WN, c0 = n0 + Core::col(wave, 0);
    // Few waves see a label among their 16 FA columns, and few tiles the vocabulary's end.
    auto largest = [&](auto bc, auto plain) LORA_INLINE {   // of a lane's logits of a row but the label's
      constexpr int b = decltype(bc)::value;
      const int i = r0 + 16 * b + c16, y = lds.label[i];
      float top = -INFINITY;
#pragma unroll
      for (int a = 0; a < FA; ++a)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float z = acc[a][b][q];
          if constexpr (decltype(plain)::value) {
            top = fmaxf(top, z);
          } else {
            const int col = n0 + Core::col(wave, a) + 4 * g + q;
            if (col < p.vocab && col != y) top = fmaxf(top, z);
          }
        }
      return top;
    };
    auto rows_of = [&](auto bc, auto plain) LORA_INLINE {
      constexpr int b = decltype(bc)::value;
      constexpr bool PLAIN = decltype(plain)::value;
      const int i = r0 + 16 * b + c16, y = lds.label[i];
      float r = MODE == XENT_STATS ? 0.0f : lds.ref[i];
      if constexpr (MODE != XENT_GRAD) {
        float top = kNone;
        if constexpr (MODE == XENT_STATS || MODE == XENT_PIECE) {
          top = largest(bc, plain);
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          if (MODE == XENT_STATS) r = top = fmaxf(top, kLowest);
        }
        const float past = MODE == XENT_LOCAL ? past_whole(r) : 0.0f;
        float sum = 0.0f;
#pragma unroll
        for (int a = 0; a < FA; ++a)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float v = MODE == XENT_LOCAL ? __builtin_amdgcn_exp2f(fmaf(acc[a][b][q] - r, kLog2e, past)) : power(acc[a][b][q], r);
            if constexpr (!PLAIN) {
              const int col = n0 + Core::col(wave, a) + 4 * g + q;
              v = col < p.vocab && col != y ? v : 0.0f;
            }
            sum += v;
            if (EXPS) acc[a][b][q] = v;
          }
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (g == 0) lds.joined[wn][i] = Part{top, sum};
      } else {
        const float d = lds.scale[i], o = lds.own[i];
#pragma unroll
        for (int a = 0; a < FA; ++a)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float v = d * power(acc[a][b][q], r);
            v = y < 0 ? 0.0f : v;
            if constexpr (!PLAIN) {
              const int col = n0 + Core::col(wave, a) + 4 * g + q;
              v = y < 0 || col >= p.vocab ? 0.0f : (col == y ? o : v);
            }
            acc[a][b][q] = v;
          }
      }
    };
    const bool inside = n0 + BN <= p.vocab;
    auto is_plain = [&](int b) LORA_INLINE {
      return inside && !__any((unsigned)(lds.label[r0 + 16 * b + c16] - c0) < (unsigned)(16 * FA));
    };
    if constexpr (MODE == XENT_LOCAL) {   // the tile's own references
      each_of<FB>([&](auto bc) LORA_INLINE {
        float top;
        if (is_plain(decltype(bc)::value)) top = largest(bc, std::true_type{});
        else top = largest(bc, std::false_type{});
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (g == 0) lds.joined[wn][r0 + 16 * decltype(bc)::value + c16].m = top;
      });
      __syncthreads();
      for (int i = tid; i < BM; i += NT) {
        float top = lds.joined[0][i].m;
#pragma unroll
        for (int w = 1; w < WN; ++w) top = fmaxf(top, lds.joined[w][i].m);
        lds.ref[i] = fmaxf(top, kLowest);
      }
      __syncthreads();
    }
    each_of<FB>([&](auto bc) LORA_INLINE {
      if (is_plain(decltype(bc)::value)) rows_of(bc, std::true_type{});
      else rows_of(bc, std::false_type{});
    });
    if constexpr (MODE != XENT_STATS) tile_to_lds<Core, BN>(acc, lds.stages);
    __syncthreads();
    if constexpr (MODE != XENT_GRAD) {
      for (int i = tid; i < BM; i += NT) {
        Part v = lds.joined[0][i];
#pragma unroll
        for (int w = 1; w < WN; ++w) {
          const Part u = lds.joined[w][i];
          const float m = fmaxf(v.m, u.m);
          v.s = MODE == XENT_STATS ? v.s * power(v.m, m) + u.s * power(u.m, m) : v.s + u.s;
          v.m = m;
        }
        if (MODE == XENT_PIECE && v.m > kNone) atomicMax(p.best + m0 + i, ordered(v.m));
        if (EXPS) v.m = lds.ref[i];
        if (MODE == XENT_LOCAL) v.s *= __builtin_amdgcn_exp2f(-past_whole(v.m));
        if (v.s == 0.0f) v.m = kLowest;   // no power: its reference does not count
        p.parts[(size_t)(p.tile0 + tn) * p.rows_pad + m0 + i] = v;
      }
    }
    if constexpr (MODE != XENT_STATS) {
      const size_t at = (size_t)tn * BN;
      lds_to_rows<BM, BN, NT>(lds.stages, p.piece + (size_t)m0 * p.piece_cols + at, (size_t)p.piece_cols, BM, BN);
      if (MODE == XENT_GRAD && p.turned) {
        // A wave turns 32 rows x 16 columns at a time: 16 lanes read 4 rows x 16 columns, lane i
        // receives column i's, and two such reads are 8 rows of it.
        constexpr int BLOCKS = (BM / 32) * (BN / 16);
        static_assert(BLOCKS % NW == 0, "whole waves");
        const int e4 = c16 >> 2, q4 = c16 & 3;
#pragma unroll 4
        for (int i = 0; i < BLOCKS / NW; ++i) {
          const int blk = wave + NW * i, r = 32 * (blk / (BN / 16)) + 8 * g, col = 16 * (blk % (BN / 16));
          const int ch = (col >> 3) + (q4 >> 1);
          int2w lo, hi;
          read_tr_asm<Bf16, 0>(lo, lds_addr(lds.stages) + tile_at<BN>(r + e4, ch) + (q4 & 1) * 8);
          read_tr_asm<Bf16, 0>(hi, lds_addr(lds.stages) + tile_at<BN>(r + 4 + e4, ch) + (q4 & 1) * 8);
          asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(lo), "+v"(hi));
          *reinterpret_cast<int4v*>(p.turned + (at + col + c16) * p.rows_pad + m0 + r) = int4v{lo.x, lo.y, hi.x, hi.y};
        }
      }
    }
  }
};

// Workgroups of XENT_AGAIN walk the tiles: those whose rows' references served have
// nothing to do but, in the first column of tiles, to hand them on.
template <class Core, int BM, int BN, int NT, int MODE>
__global__ __launch_bounds__(NT) void lora_xent_logits_kernel(XentLogits p) {
  using Tile = XentTile<Core, BM, BN, NT, MODE>;
  __shared__ __attribute__((aligned(1024))) typename Tile::Lds lds;
  const int tiles = p.tiles_m * p.tiles_n, tid = threadIdx.x;
  for (int tile = blockIdx.x; tile < tiles; tile += MODE == XENT_AGAIN ? (int)gridDim.x : tiles) {
    int tm, tn;
    tile_coords(p.tiles_m, p.tiles_n, 8, tile, tm, tn);
    bool again = false;
    if (MODE == XENT_AGAIN) __syncthreads();   // the tile before is done with the LDS
    for (int i = tid; i < BM; i += NT) {       // (read behind the core's barriers)
      const int row = tm * BM + i, y = row < p.rows ? p.labels[row] : -1;
      const bool known = y >= 0 && y < p.vocab;
      lds.label[i] = known ? y : -1;
      if (MODE == XENT_PIECE) lds.ref[i] = p.ref[row];
      if (MODE == XENT_AGAIN) {
        const float old = p.ref[row], ref = row < p.rows ? served_by(old, from_ordered(p.best[row])) : old;
        again = again || ref != old;
        lds.ref[i] = ref;
        if (tn == 0) {
          p.ref_next[row] = ref;
          p.best_next[row] = ordered(kNone);
        }
      }
      if (MODE == XENT_GRAD) {
        const Saved row_of = known ? saved_row(p.saved + 2 * row) : Saved{0.0f, 0.0f, 0.0f};
        const float d = known ? p.dloss[row] : 0.0f;
        lds.ref[i] = row_of.ref;
        lds.scale[i] = d * row_of.scale;
        const float o = known ? -d * row_of.rest : 0.0f;
        lds.own[i] = o;
        if (p.coef && tn == 0) {   // for dX and dW: what the label's entry of G loses as bf16
          p.coef[2 * row] = 1.0f;
          p.coef[2 * row + 1] = o - bf16_to_f32(f32_to_bf16(o));
        }
      }
    }
    if (MODE == XENT_AGAIN && !__syncthreads_or(again)) continue;
    Tile::run(p, tm, tn, lds);
  }
}

// ---- a row's numbers -----------------------------------------------------------
// Loss, and what the gradient needs, from the sum of all others' powers against ref
// and the label's logit.  That logit's error is the loss's (all others' even out in their
// sum), so it comes here as a sum in fp64 and the logarithms are taken there too: with
// the tile's fp32 sum the loss of 7 x 2000 x 5120 was off by 1.9e-6 (rms), now by 5e-7,
// at 0.3% (4096 x 32000 x 4096) to 4% (37 rows) of the call's time.
struct RowEnd {
  float loss, lse, rest;   // rest = 1 - p_label
  float c1;                // 1 / sum, against ref
};
__device__ __forceinline__ RowEnd row_end(float ref, float others, double zy, bool known) {
  RowEnd e;
  if (!(fabs(zy) <= 3.4028234663852886e38)) zy = (double)(float)zy;   // infinite as a logit is
  const double dy = known ? (zy - (double)ref) * 1.4426950408889634074 : -(double)INFINITY, up = fmax(dy, 0.0);   // (NaN: 0, and dy below)
  const double whole = floor(up);
  const float down = up < 1000.0 ? ldexpf(__builtin_amdgcn_exp2f((float)(whole - up)), -(int)whole) : 0.0f, rest = others * down;
  const float ey = known ? __builtin_amdgcn_exp2f((float)(dy - up)) : 0.0f, sum = rest + ey;
  const float bad = sum < INFINITY ? 0.0f : NAN;   // a NaN or an infinity among the logits
  const double log = log2((double)sum);
  e.loss = known ? (ey > rest ? log1pf(rest / ey) : (float)(0.69314718055994530942 * (log - (dy - up)))) + bad : 0.0f;
  e.lse = (float)((double)ref + 0.69314718055994530942 * (up + log)) + bad;
  e.rest = known ? rest / sum + bad : 0.0f;
  e.c1 = known ? down / sum + bad : 0.0f;
  return e;
}

// Joins the tiles' parts of 4 rows, 64 threads a row, in a fixed order, and forms the
// label's logit in fp64 (a row of X, a row of W).  The
// forward keeps what Saved says in `saved` (or nowhere), the one-pass call c1 and c2 in
// `coef` and, with tiles' own references, the largest tile's logit in `ref` (else none).
constexpr int kRowsPer = 4;
__global__ __launch_bounds__(256) void lora_xent_rows_kernel(const Part* __restrict__ parts, const u16* __restrict__ X,
                                                             const u16* __restrict__ W, const int32_t* __restrict__ labels,
                                                             const float* __restrict__ dloss, float* __restrict__ loss,
                                                             float* __restrict__ saved, float* __restrict__ coef,
                                                             float* __restrict__ ref, int rows, int vocab, int k, int tiles,
                                                             int64_t rows_pad) {
  constexpr int RB = kRowsPer, PER = 256 / RB;
  __shared__ Part lds[256];
  __shared__ double dots[256];
  const int tid = threadIdx.x, r = tid % RB, row = (int)blockIdx.x * RB + r;   // below rows_pad
  const int y = row < rows ? labels[row] : -1;
  const bool known = y >= 0 && y < vocab;
  Part u[4];
  auto load = [&](int t) LORA_INLINE {
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = t + j * PER < tiles ? parts[(size_t)(t + j * PER) * rows_pad + row] : Part{kLowest, 0.0f};
  };
  load(tid / RB);     // (under way during the product)
  double dot = 0.0;   // the label's logit
  if (known) {
    const u16 *x = X + (size_t)row * k, *w = W + (size_t)y * k;
#pragma unroll 4
    for (int c = tid / RB * 8; c < k; c += 8 * PER) {
      const int4v xv = *reinterpret_cast<const int4v*>(x + c), wv = *reinterpret_cast<const int4v*>(w + c);
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        dot = fma((double)bf16_to_f32((u16)xv[h]), (double)bf16_to_f32((u16)wv[h]), dot);
        dot = fma((double)bf16_to_f32((u16)((uint32_t)xv[h] >> 16)), (double)bf16_to_f32((u16)((uint32_t)wv[h] >> 16)), dot);
      }
    }
  }
  Part v{kLowest, 0.0f};
  auto add = [&](Part u) LORA_INLINE {
    const float m = fmaxf(v.m, u.m);
    v.s = v.s * power(v.m, m) + u.s * power(u.m, m);
    v.m = m;
  };
  for (int t = tid / RB; t < tiles; t += 4 * PER) {
#pragma unroll
    for (int j = 0; j < 4; ++j) add(u[j]);
    load(t + 4 * PER);
  }
#pragma unroll
  for (int d = PER / 2; d > 0; d >>= 1) {   // halves of the row's threads
    __syncthreads();
    lds[tid] = v;
    dots[tid] = dot;
    __syncthreads();
    if (tid / RB < d) {
      add(lds[tid + d * RB]);
      dot += dots[tid + d * RB];
    }
  }
  if (tid >= RB) return;
  if (ref) ref[row] = v.m;
  if (row >= rows) return;
  const RowEnd e = row_end(v.m, v.s, dot, known);
  loss[row] = e.loss;
  if (saved) save_row(saved + 2 * row, e.lse, Saved{v.m, e.c1, e.rest});
  if (coef) {
    const float d = known ? dloss[row] : 0.0f, c1 = ref ? e.c1 * __builtin_amdgcn_exp2f(-past_whole(v.m)) : e.c1;
    coef[2 * row] = known ? d * c1 : 0.0f;
    coef[2 * row + 1] = known ? -d * e.rest : 0.0f;
  }
}

__global__ __launch_bounds__(256) void lora_xent_begin_kernel(float* ref, uint32_t* best, int64_t rows_pad) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= rows_pad) return;
  ref[i] = kNoLogit;
  best[i] = ordered(kNone);
}

// X for dW: rows without a label are 0 there, whatever they hold (G is, and its product
// with a NaN would not be).
__global__ __launch_bounds__(256) void lora_xent_known_kernel(const u16* __restrict__ X, const int32_t* __restrict__ labels,
                                                              u16* __restrict__ out, int64_t chunks, int per, int vocab) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= chunks) return;
  const int y = labels[e / per];
  const int4v v = reinterpret_cast<const int4v*>(X)[e];
  reinterpret_cast<int4v*>(out)[e] = y >= 0 && y < vocab ? v : int4v{0, 0, 0, 0};
}

// ---- the second product ----------------------------------------------------------
struct XentGrad {
  const u16 *A, *B;        // A: [rows of the output][a_cols], B: [contraction][k]
  float* sums;             // [split][tile][fragment][thread][4]: what pieces carry
  bool first, last;        // no sums so far; the result is stored (one split)
  const float *ref_old, *ref;   // the rows' references before and in this piece (or none)
  const Part* parts;       // local references: [tile][rows_pad], tiles of 2^tile_log stages
  int tile_log;
  int64_t rows_pad;
  const float* coef;       // out = coef[0] sum + coef[1] W_label, 0 without a label (or none: the sum);
                           // of dW: coef[1] is what the label's entry of G lost
  int label0;              // of dW: the output's first row is this label's
  const int32_t* labels;
  const u16* W;
  u16* out;                // bf16 rows of k
  int64_t a_cols, b_rows;
  int m, rows, vocab, k, stages, tiles_m, tiles_n, splits;
};

// dX of 4 columns of a row from its sum (no branch: rows without a label read W's first).
__device__ __forceinline__ floatx4 with_label(floatx4 v, const float* coef, const int32_t* labels, const u16* W, int row,
                                              int rows, int vocab, int k, int col) {
  const int at = min(row, rows - 1), y = labels[at];
  const bool known = row < rows && y >= 0 && y < vocab;
  const float c1 = coef[2 * at], c2 = coef[2 * at + 1];
  const uint2 w = *reinterpret_cast<const uint2*>(W + (size_t)(known ? y : 0) * k + min(col, k - 4));
  const float u[4] = {bf16_to_f32((u16)w.x), bf16_to_f32((u16)(w.x >> 16)), bf16_to_f32((u16)w.y), bf16_to_f32((u16)(w.y >> 16))};
  floatx4 o;
#pragma unroll
  for (int q = 0; q < 4; ++q) o[q] = known ? c1 * v[q] + c2 * u[q] : 0.0f;
  return o;
}

// dW of a tile: what the labels' entries of G lost when they became bf16, times their
// rows of X, so that a row of W that one label reaches is as exact as its own bf16 (such an
// entry is the largest of its row of G by far, and no sum over rows evens it out).  The
// labels are read by the whole workgroup, 8 a thread; those of the tile's rows are listed
// in an order that does not depend on timing, and 32 of them at a time are a product's
// contraction, with their rests (as bf16, 2^-16 of the entry) in the places of their rows
// and zeros elsewhere (1500 rows, vocabulary 50021, k 2048: 1 to 2% of the backward; 8192
// rows of one label, 32000, 1024: 10%, and 160% with an entry at a time).
template <class Core, int BM, int NT>
__device__ __forceinline__ void add_label_rests(typename Core::Acc& acc, char* smem, const XentGrad& p, int m0, int l0) {
  constexpr int FA = std::extent_v<typename Core::Acc, 0>, FB = std::extent_v<typename Core::Acc, 1>, NW = NT / 64;
  constexpr int U = 8, COUNTS = U * NW;
  static_assert(COUNTS <= 64 && BM <= 256, "a wave's lanes hold all counts; an entry packs its row");
  static_assert(U * NT * 8 + COUNTS * 4 <= Core::SMEM, "the list fits the stages");
  int2w* list = reinterpret_cast<int2w*>(smem);                        // [U NT]: row of X | row of the tile << 20, rest as bf16
  uint32_t* counts = reinterpret_cast<uint32_t*>(smem + U * NT * 8);   // [U][NW]
  const int tid = threadIdx.x, lane = lane_fresh(), wave = uniform(tid >> 6), g = lane >> 4, c16 = lane & 15;
  const int rows = (int)p.b_rows, row0 = Core::row0(wave);
  const uint32_t first = (uint32_t)(p.label0 + m0);
  for (int base = 0; base < rows; base += U * NT) {
    uint32_t at[U];
    uint64_t hits[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = base + u * NT + tid;
      const uint32_t y = i < rows ? (uint32_t)p.labels[i] : ~0u;
      at[u] = y < (uint32_t)p.vocab ? y - first : ~0u;
      hits[u] = __ballot(at[u] < (uint32_t)BM);
    }
    __syncthreads();   // the core's reads, or the list's, are over
    if (lane == 0)
#pragma unroll
      for (int u = 0; u < U; ++u) counts[u * NW + wave] = (uint32_t)__popcll(hits[u]);
    __syncthreads();
    int upto = lane < COUNTS ? (int)counts[lane] : 0;
#pragma unroll
    for (int d = 1; d < COUNTS; d <<= 1) {
      const int below = __shfl_up(upto, d);
      upto += lane >= d ? below : 0;
    }
    const int total = __builtin_amdgcn_readlane(upto, COUNTS - 1);
    if (total == 0) continue;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int before = __builtin_amdgcn_readlane(upto, u * NW + wave) - __popcll(hits[u]);
      if (at[u] < (uint32_t)BM) {
        const int i = base + u * NT + tid;
        const int to = before + __builtin_amdgcn_mbcnt_hi((uint32_t)(hits[u] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hits[u], 0));
        list[to] = int2w{i | (int)at[u] << 20, (int)f32_to_bf16(p.coef[2 * i + 1])};
      }
    }
    __syncthreads();
    for (int e = 0; e < total; e += 32) {   // a lane's entries: e + 8 g .. + 7
      int2w entry[8];
      short8 x[FA];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        entry[j] = list[min(e + 8 * g + j, total - 1)];
        const u16* from = p.B + (size_t)(entry[j].x & 0xFFFFF) * p.k;
#pragma unroll
        for (int a = 0; a < FA; ++a) x[a][j] = (short)from[min(l0 + Core::col(wave, a) + c16, p.k - 1)];
        if (e + 8 * g + j >= total) entry[j].y = 0;
      }
#pragma unroll
      for (int b = 0; b < FB; ++b) {
        short8 r;
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = entry[j].x >> 20 == row0 + 16 * b + c16 ? (short)entry[j].y : (short)0;
#pragma unroll
        for (int a = 0; a < FA; ++a) acc[a][b] = mfma16x16x32(x[a], r, acc[a][b]);
      }
    }
  }
  formed(acc);
}

// What becomes of a tile's sums: carried to the next piece or the join, stored as the
// result of dW, or stored with the label's part as that of dX.
enum XentEnd { XENT_CARRY, XENT_ROWS, XENT_LABEL };

// LOCAL: A's tiles have references of their own (parts), and ref is the row's.
template <class Core, int BM, int NT, int END, bool LOCAL>
__global__ __launch_bounds__(NT) void lora_xent_grad_kernel(XentGrad p) {
  constexpr int FA = std::extent_v<typename Core::Acc, 0>, FB = std::extent_v<typename Core::Acc, 1>;
  constexpr int LT = LOCAL ? local_tiles(BM) : 0;
  __shared__ __attribute__((aligned(1024))) char smem[Core::SMEM + LT * BM * 2];
  const int tiles = p.tiles_m * p.tiles_n, split = (int)blockIdx.x / tiles;
  int tm, tn;
  tile_coords(p.tiles_m, p.tiles_n, 8, (int)blockIdx.x - split * tiles, tm, tn);
  const int m0 = tm * BM, l0 = tn * 256;
  const uint32_t arow = (uint32_t)p.a_cols * 2, brow = (uint32_t)p.k * 2;
  const NnTile t{make_rsrc(p.A + (size_t)m0 * p.a_cols, (uint64_t)min(BM, p.m - m0) * arow), arow,
                 reinterpret_cast<const char*>(p.B + l0), brow, (uint64_t)p.b_rows * brow - (uint64_t)l0 * 2, p.stages};
  typename Core::Acc acc;
  const int s0 = (int)((int64_t)p.stages * split / p.splits), s1 = (int)((int64_t)p.stages * (split + 1) / p.splits);
  if constexpr (LOCAL) {
    u16* table = reinterpret_cast<u16*>(smem + Core::SMEM);   // (read behind the core's barriers)
    const int first = s0 >> p.tile_log, count = s1 > s0 ? ((s1 - 1) >> p.tile_log) - first + 1 : 0;
    for (int i = threadIdx.x; i < min(count, LT) * BM; i += NT) {
      const int row = m0 + i % BM;
      const float d = powers_above(p.ref[row], p.parts[(size_t)(first + i / BM) * p.rows_pad + row].m);
      table[i] = d < 255.0f ? (u16)((int)d << 7) : (u16)(255 << 7);   // (a NaN: 255, and the row's result is one)
    }
    Core::template run<true>(t, Scales{}, m0, s0, s1, smem, acc, Shifts<BM>{table, first, p.tile_log});
  } else {
    Core::run(t, Scales{}, m0, s0, s1, smem, acc);
  }
  const int lane = lane_fresh(), wave = uniform((int)threadIdx.x >> 6), g = lane >> 4, c16 = lane & 15;
  floatx4* to = reinterpret_cast<floatx4*>(p.sums) + ((size_t)split * tiles + (size_t)tm * p.tiles_n + tn) * (FA * FB * NT) + threadIdx.x;
#pragma unroll
  for (int b = 0; b < FB; ++b) {
    const int row = m0 + Core::row0(wave) + 16 * b + c16;
    // (a reference moves down where nothing is carried: 1; and 0 times a masked part's sum, which may be infinite, is 0)
    const float alpha = !LOCAL && !p.first && p.ref ? power(fminf(p.ref_old[row], p.ref[row]), p.ref[row]) : 1.0f;
#pragma unroll
    for (int a = 0; a < FA; ++a) {
      floatx4 v = acc[a][b];
      if (!p.first) {
        const floatx4 carried = to[(a * FB + b) * NT];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] += alpha == 0.0f ? 0.0f : carried[q] * alpha;
      }
      if (END == XENT_CARRY) to[(a * FB + b) * NT] = v;
      if (END == XENT_LABEL) v = with_label(v, p.coef, p.labels, p.W, row, p.rows, p.vocab, p.k, l0 + Core::col(wave, a) + 4 * g);
      acc[a][b] = v;
    }
    __builtin_amdgcn_sched_barrier(0);   // (registers: a row's loads at a time)
  }
  if constexpr (END == XENT_ROWS) add_label_rests<Core, BM, NT>(acc, smem, p, m0, l0);
  if constexpr (END != XENT_CARRY)
    store_tile<Core, BM, 256, NT>(acc, smem, p.out + (size_t)m0 * p.k + l0, (size_t)p.k, p.rows - m0, p.k - l0);
}

// The sums of all splits, in their order, as dX.  A workgroup takes one fragment of
// each thread of a tile (8 parts of 64 x 4096 sums: 4.2 us, mostly the launch's own).
template <class Core, int BM, int NT>
__global__ __launch_bounds__(NT) void lora_xent_join_kernel(XentGrad p) {
  constexpr int FA = std::extent_v<typename Core::Acc, 0>, FB = std::extent_v<typename Core::Acc, 1>;
  const int tile = (int)blockIdx.x / (FA * FB), f = (int)blockIdx.x % (FA * FB), a = f / FB, b = f % FB;
  const int m0 = tile / p.tiles_n * BM, l0 = tile % p.tiles_n * 256;
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), g = lane >> 4, c16 = lane & 15;
  const int row = m0 + Core::row0(wave) + 16 * b + c16, col = l0 + Core::col(wave, a) + 4 * g;
  const size_t step = (size_t)p.tiles_m * p.tiles_n * (FA * FB * NT);
  const floatx4* from = reinterpret_cast<const floatx4*>(p.sums) + (size_t)tile * (FA * FB * NT) + f * NT + threadIdx.x;
  floatx4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = 0; s < p.splits; ++s) v += from[(size_t)s * step];
  if (row >= p.rows || col >= p.k) return;
  if (p.coef) v = with_label(v, p.coef, p.labels, p.W, row, p.rows, p.vocab, p.k, col);
  *reinterpret_cast<uint2*>(p.out + (size_t)row * p.k + col) = bf16x4(v);
}

// ---- launches ----------------------------------------------------------------------
#define LORA_TRY(call)               \
  do {                               \
    const hipError_t e_ = (call);    \
    if (e_ != hipSuccess) return e_; \
  } while (0)

template <int MODE, bool TAIL>
static hipError_t run_logits_of(const XentPlan& p, const XentLogits& q, hipStream_t st) {
  const int tiles = q.tiles_m * q.tiles_n;
  const dim3 grid((unsigned)(MODE == XENT_AGAIN ? std::min(tiles, 256) : tiles));
  switch (p.kind) {
    case XENT_64x128:
      hipLaunchKernelGGL((lora_xent_logits_kernel<NtCore<Bf16, 64, 128, 1, 4, 6, TAIL>, 64, 128, 256, MODE>), grid,
                         dim3(256), 0, st, q);
      break;
    case XENT_128x128:
      hipLaunchKernelGGL((lora_xent_logits_kernel<NtCore<Bf16, 128, 128, 2, 4, 4, TAIL>, 128, 128, 512, MODE>), grid,
                         dim3(512), 0, st, q);
      break;
    case XENT_256x128:
      hipLaunchKernelGGL((lora_xent_logits_kernel<NtCore<Bf16, 256, 128, 4, 2, 3, TAIL>, 256, 128, 512, MODE>), grid,
                         dim3(512), 0, st, q);
      break;
    default:
      hipLaunchKernelGGL((lora_xent_logits_kernel<NtBig<Bf16, TAIL>, 256, 256, 512, MODE>), grid, dim3(512), 0, st, q);
  }
  return hipGetLastError();
}
template <int MODE>
static hipError_t run_logits(const XentPlan& p, const XentLogits& q, hipStream_t st) {
  return q.k % 64 ? run_logits_of<MODE, true>(p, q, st) : run_logits_of<MODE, false>(p, q, st);
}
using Grad64 = NnCore<Bf16, 64, 256, 1, 4, 3>;
using Grad128 = NnCore<Bf16, 128, 256, 2, 4, 3>;
using Grad256 = NnBig<Bf16>;
template <int END>
static hipError_t run_grad_of(int kind, const XentGrad& q, hipStream_t st) {
  const dim3 grid((unsigned)(q.tiles_m * q.tiles_n * q.splits));
  if constexpr (END != XENT_ROWS) {
    if (q.parts) {
      if (kind == XENT_GRAD_64x256)
        hipLaunchKernelGGL((lora_xent_grad_kernel<Grad64, 64, 256, END, true>), grid, dim3(256), 0, st, q);
      else
        hipLaunchKernelGGL((lora_xent_grad_kernel<Grad128, 128, 512, END, true>), grid, dim3(512), 0, st, q);
      return hipGetLastError();
    }
  }
  switch (kind) {
    case XENT_GRAD_64x256: hipLaunchKernelGGL((lora_xent_grad_kernel<Grad64, 64, 256, END, false>), grid, dim3(256), 0, st, q); break;
    case XENT_GRAD_128x256: hipLaunchKernelGGL((lora_xent_grad_kernel<Grad128, 128, 512, END, false>), grid, dim3(512), 0, st, q); break;
    default: hipLaunchKernelGGL((lora_xent_grad_kernel<Grad256, 256, 512, END, false>), grid, dim3(512), 0, st, q);
  }
  return hipGetLastError();
}
static hipError_t run_grad(int kind, const XentGrad& q, hipStream_t st) {
  if (!q.last) return run_grad_of<XENT_CARRY>(kind, q, st);
  return run_grad_of<XENT_LABEL>(kind, q, st);   // (the last piece's has coef)
}
// dW of a piece.
static hipError_t run_rows(int kind, const XentGrad& q, hipStream_t st) { return run_grad_of<XENT_ROWS>(kind, q, st); }
template <class Core, int BM, int NT>
static hipError_t run_join_of(const XentGrad& q, hipStream_t st) {
  constexpr int F = std::extent_v<typename Core::Acc, 0> * std::extent_v<typename Core::Acc, 1>;
  hipLaunchKernelGGL((lora_xent_join_kernel<Core, BM, NT>), dim3((unsigned)(q.tiles_m * q.tiles_n * F)), dim3(NT), 0, st, q);
  return hipGetLastError();
}
static hipError_t run_join(int kind, const XentGrad& q, hipStream_t st) {
  if (kind == XENT_GRAD_64x256) return run_join_of<Grad64, 64, 256>(q, st);
  return kind == XENT_GRAD_128x256 ? run_join_of<Grad128, 128, 512>(q, st) : run_join_of<Grad256, 256, 512>(q, st);
}

struct XentCall {
  const XentArgs& a;
  XentPlan p;
  XentLayout L;
  hipStream_t st;
  template <typename T>
  T* at(size_t offset) const { return reinterpret_cast<T*>(a.ws + offset); }

  XentLogits logits() const {
    XentLogits q{};
    q.X = a.X; q.W = a.W; q.labels = a.labels;
    q.dloss = a.dloss;
    q.parts = at<Part>(L.parts);
    q.piece = at<u16>(L.piece);
    q.rows = (int)a.rows; q.vocab = (int)a.vocab; q.k = (int)a.k;
    q.tiles_m = p.tiles_m; q.tiles_n = p.vtiles;
    q.rows_pad = p.rows_pad; q.piece_cols = p.piece;
    return q;
  }
  void at_piece(XentLogits& q, int i) const {
    q.tile0 = i * p.piece_tiles;
    q.tiles_n = std::min(p.piece_tiles, p.vtiles - q.tile0);
  }
  // dX's part of piece i, from its buffer.
  XentGrad dx(int i) const {
    XentGrad g{};
    const int64_t v0 = i * p.piece;
    g.A = at<u16>(L.piece);
    g.B = a.W + v0 * a.k;
    g.first = i == 0;
    g.last = i + 1 == p.pieces && p.splits == 1;
    g.sums = at<float>(L.sums);
    g.labels = a.labels; g.W = a.W; g.out = a.dX;
    g.a_cols = p.piece;
    g.b_rows = std::min(p.piece, a.vocab - v0);
    g.m = (int)p.rows_pad; g.rows = (int)a.rows; g.vocab = (int)a.vocab; g.k = (int)a.k;
    g.stages = (int)cdiv(g.b_rows, 64);
    g.tiles_m = p.grad_tiles_m; g.tiles_n = p.tiles_k; g.splits = p.splits;   // (some have nothing but their scaling to do in a short last piece)
    return g;
  }
  hipError_t rows(float* saved, float* coef, float* ref) const {
    const Part* parts = at<Part>(L.parts);
    hipLaunchKernelGGL(lora_xent_rows_kernel, dim3((unsigned)cdiv(a.rows, kRowsPer)), dim3(256), 0, st, parts, a.X, a.W,
                       a.labels, a.dloss, a.loss, saved, coef, ref, (int)a.rows, (int)a.vocab, (int)a.k, p.vtiles,
                       p.rows_pad);
    return hipGetLastError();
  }
  hipError_t forward(float* saved) const {
    XentLogits q = logits();
    const int most = (1 << 22) / p.tiles_m;   // (a launch has fewer than 2^32 threads; tiles_m is at most 2^14)
    for (q.tile0 = 0; q.tile0 < p.vtiles; q.tile0 += most) {
      q.tiles_n = std::min(most, p.vtiles - q.tile0);
      LORA_TRY(run_logits<XENT_STATS>(p, q, st));
    }
    return rows(saved, nullptr, nullptr);
  }
  hipError_t backward(const float* saved) const {
    XentLogits q = logits();
    q.saved = saved;
    q.turned = a.dW ? at<u16>(L.turned) : nullptr;
    float* coef = at<float>(L.coef);
    if (a.dW) {
      const int64_t chunks = a.rows * (a.k / 8);
      hipLaunchKernelGGL(lora_xent_known_kernel, dim3((unsigned)cdiv(chunks, 256)), dim3(256), 0, st, a.X, a.labels,
                         at<u16>(L.known), chunks, (int)(a.k / 8), (int)a.vocab);
      LORA_TRY(hipGetLastError());
    }
    for (int i = 0; i < p.pieces; ++i) {
      at_piece(q, i);
      q.coef = i == 0 ? coef : nullptr;
      LORA_TRY(run_logits<XENT_GRAD>(p, q, st));
      if (a.dX) {
        XentGrad g = dx(i);
        g.coef = coef;
        LORA_TRY(run_grad(p.grad_kind, g, st));
      }
      if (a.dW) {
        const int64_t v0 = i * p.piece, cols = std::min(p.piece, a.vocab - v0);
        XentGrad g{};
        g.A = q.turned; g.B = at<u16>(L.known); g.out = a.dW + v0 * a.k;
        g.a_cols = p.rows_pad; g.b_rows = a.rows;
        g.first = g.last = true;
        g.coef = coef; g.labels = a.labels; g.label0 = (int)v0;
        g.m = g.rows = (int)cols; g.vocab = (int)a.vocab; g.k = (int)a.k;
        g.stages = (int)cdiv(a.rows, 64);   // (columns of `turned` that tiles have written)
        g.tiles_m = (int)cdiv(cols, p.dw_m); g.tiles_n = p.tiles_k; g.splits = 1;
        LORA_TRY(run_rows(p.dw_kind, g, st));
      }
    }
    if (!a.dX || p.splits == 1) return hipSuccess;
    XentGrad g = dx(0);
    g.coef = coef;
    return run_join(p.grad_kind, g, st);
  }
  // Loss and dX, the logits formed once.
  hipError_t one_pass() const {
    XentLogits q = logits();
    float* ref[2] = {at<float>(L.ref), at<float>(L.ref) + p.rows_pad};
    uint32_t* best[2] = {at<uint32_t>(L.best), at<uint32_t>(L.best) + p.rows_pad};
    float* coef = at<float>(L.coef);
    if (p.local) {
      at_piece(q, 0);
      LORA_TRY(run_logits<XENT_LOCAL>(p, q, st));
      LORA_TRY(rows(nullptr, coef, ref[0]));
      XentGrad g = dx(0);
      g.coef = coef;
      g.ref = ref[0];
      g.parts = q.parts;
      g.tile_log = p.tile_n == 256 ? 2 : 1;
      g.rows_pad = p.rows_pad;
      LORA_TRY(run_grad(p.grad_kind, g, st));
      return p.splits == 1 ? hipSuccess : run_join(p.grad_kind, g, st);
    }
    hipLaunchKernelGGL(lora_xent_begin_kernel, dim3((unsigned)cdiv(p.rows_pad, 256)), dim3(256), 0, st, ref[0], best[0],
                       p.rows_pad);
    LORA_TRY(hipGetLastError());
    for (int i = 0; i < p.pieces; ++i) {
      at_piece(q, i);
      q.ref = ref[i & 1];
      q.ref_next = ref[(i + 1) & 1];
      q.best = best[i & 1];
      q.best_next = best[(i + 1) & 1];
      LORA_TRY(run_logits<XENT_PIECE>(p, q, st));
      LORA_TRY(run_logits<XENT_AGAIN>(p, q, st));
      XentGrad g = dx(i);
      if (i + 1 == p.pieces) LORA_TRY(rows(nullptr, coef, nullptr));
      if (g.last) g.coef = coef;
      g.ref_old = q.ref;
      g.ref = q.ref_next;
      LORA_TRY(run_grad(p.grad_kind, g, st));
    }
    if (p.splits == 1) return hipSuccess;
    XentGrad g = dx(0);
    g.coef = coef;
    return run_join(p.grad_kind, g, st);
  }
};

static XentCall call_of(const XentArgs& a, hipStream_t st) {
  return XentCall{a, plan_xent(a.rows, a.vocab, a.k), xent_layout(a.rows, a.vocab, a.k, a.dX != nullptr, a.dW != nullptr), st};
}

hipError_t launch_xent_fwd(const XentArgs& a, hipStream_t st) { return call_of(a, st).forward(a.saved); }

hipError_t launch_xent_bwd(const XentArgs& a, hipStream_t st) { return call_of(a, st).backward(a.saved); }

hipError_t launch_xent_step(const XentArgs& a, hipStream_t st) {
  const XentCall c = call_of(a, st);
  if (!a.dW) return c.one_pass();
  float* saved = c.at<float>(c.L.saved);
  LORA_TRY(c.forward(saved));
  return c.backward(saved);
}

}  // namespace lora
