// Internal interface of the operators of a fine-tuning step between the C ABI
// (lora_train_abi.cpp: argument checks) and their kernels: 8-bit frozen weights
// (lora_fp8.hip), cross entropy without logits (lora_xent.hip), dropout without a
// mask (lora_dropout.hip).  Shapes here have already been validated; the launch
// rules stand here, apart from the kernels, so that they can be checked on the host.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace lora {

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t region(size_t bytes) { return (bytes + 255) / 256 * 256; }

// The most bytes that a workspace of 1 to `rows` rows has.  Fewer rows may need more, since
// only few tiles share their contractions, in sums of memory; a caller who keeps one buffer
// for batches of several lengths asks for the longest.  The launch rules know rows by their
// 64s (below 64, what they do without sums), and bytes grow within those: 0.1 to 0.3 us of
// the host's for each 64.
template <class F>
inline size_t bytes_up_to(int64_t rows, F&& bytes) {
  size_t most = 0;
  for (int64_t r = 64; r < rows; r += 64) most = std::max(most, bytes(r));
  return std::max(most, bytes(rows));
}

// ---- dropout -----------------------------------------------------------------
struct DropoutArgs {
  const void *X, *residual;   // residual: or none
  void* Y;
  bool f32;
  int64_t count;
  uint64_t seed, offset;
  uint32_t thr;               // of 2^16 draws, how many keep
  float scale;                // 1 / (1 - p)
};
hipError_t launch_dropout(const DropoutArgs& a, hipStream_t st);

// ---- 8-bit weights -----------------------------------------------------------
// Codes: rows of 128 ceil(k / 128) bytes.  Scales: of a weight one byte per 128 x
// 128 block, of activations one per row and 128 columns, in cells of 64 rows.
inline int64_t fp8_blocks(int64_t k) { return cdiv(k, 128); }
inline int64_t fp8_cells(int64_t rows) { return cdiv(rows, 64); }
inline size_t fp8_codes_bytes(int64_t rows, int64_t k) { return (size_t)(rows * fp8_blocks(k) * 128); }
inline size_t fp8_scales_bytes(int64_t rows, int64_t k, int block_rows) {
  return (size_t)(fp8_blocks(k) * (block_rows == 1 ? 64 * fp8_cells(rows) : cdiv(rows, 128)));
}

struct Fp8QuantArgs {
  const uint16_t* X;
  uint8_t *codes, *scales;
  int64_t rows, k;
  int block_rows;
};
hipError_t launch_fp8_quantize(const Fp8QuantArgs& a, hipStream_t st);
hipError_t launch_fp8_dequantize(const uint8_t* codes, const uint8_t* scales, uint16_t* X, int64_t rows, int64_t k,
                                 int block_rows, hipStream_t st);

// One product of the layer: A (activations, [m, c] in bf16, quantised here) times W.
struct Fp8Args {
  const uint16_t* A;
  const uint8_t *Wc, *Ws;
  uint16_t* out;
  char* ws;
  int64_t m, n, k;   // W is [n, k]
};

// Kernels of the forward: one launch that quantises X on its way for very few values
// of it; else X is quantised before, and the product is formed by waves on different
// stages straight from memory (few tokens) or by tiles staged in LDS.  The backward
// has tiles alone.  Workgroups may share the contractions of tiles of 64 rows.
enum Fp8Kind { FP8_TOKEN_8, FP8_TOKEN_2, FP8_FEW_1, FP8_FEW_2, FP8_64x64, FP8_64x128, FP8_64x128_DEEP, FP8_128x128, FP8_256x128, FP8_256x256 };
enum Fp8BackKind { FP8_BACK_64x256, FP8_BACK_128x256, FP8_BACK_256x256 };

struct Fp8Plan {
  int kind;               // of the forward's or the backward's
  int tiles_m, tiles_n;   // of the output
  int splits;             // workgroups that share a tile's contraction
  int64_t grid;
  int block;
};

// Tiles are chosen by their estimated time in us, launches and the quantisation left
// out: a round of workgroups that fills the compute units takes c + full x stages, one
// of few of them c + light x stages, the last one in between.
//   Forward, fitted to k = 2048 to 11008 (us): 64 x 4096 x 4096 9.3 on 64 x 64 (13 on 64
// x 128, 15.0 from memory), 128 x 11008 x 4096 17.3 on 64 x 128 (21 on 64 x 64, 22 on
// 128 x 128), 1024 x 4096 x 4096 22.4 on 128 x 128 (28
// on 64 x 128, 29 on 256 x 128), 1531 x 4104 x 3208 24.7 on 256 x 128 (33 on 128 x 128,
// 36 on 256 x 256), 4096 x 4096 x 4096 54 on 256 x 256 (63 on 256 x 128).
//   Backward: 200 x 4096 x 4096 23 on 64 x 256, 17 with four workgroups to a tile, 1024
// x 4096 x 4096 27.8 on 64 x 256 (30 on 128 x 256, 43 on 256 x 256), 2048 x 4096 x 4096
// 34.5 on 128 x 256 (53, 47), 1024 x 4096 x 11008 47 on 256 x 256 (60 on 128 x 256).
//   64 x 128 has four stages in LDS where its tiles are at most a compute unit's one, for
// the latency of memory (512 x 4096 x 4096 14.9, with three 17.8), and three where there
// are more, for two workgroups to a unit (64 x 128256 x 4096 114, with four 124).  With
// four, workgroups may share the contractions of few tiles: with X's quantisation 64 x
// 4096 x 11008 32.9 -> 20.1, 128 x 4096 x 11008 32.9 -> 23.8, 64 x 1024 x 8192 18.5 ->
// 13.3.
struct TileCost {
  int kind, bm, bn, block;
  double c, light, full;
};
constexpr TileCost kFp8Tiles[6] = {{FP8_64x64, 64, 64, 256, 1.5, 0.26, 0.29},
                                   {FP8_64x128, 64, 128, 256, 1.8, 0.40, 0.42},
                                   {FP8_64x128_DEEP, 64, 128, 256, 1.8, 0.35, 0.41},
                                   {FP8_128x128, 128, 128, 512, 2.5, 0.42, 0.60},
                                   {FP8_256x128, 256, 128, 512, 4.0, 0.58, 0.90},
                                   {FP8_256x256, 256, 256, 512, 6.0, 1.03, 1.45}};
constexpr TileCost kFp8BackTiles[3] = {{FP8_BACK_64x256, 64, 256, 256, 2.5, 0.62, 0.77},
                                       {FP8_BACK_128x256, 128, 256, 512, 3.5, 0.70, 0.96},
                                       {FP8_BACK_256x256, 256, 256, 512, 6.0, 1.03, 1.65}};
inline double tile_time(const TileCost& t, int64_t grid, double stages) {
  const int64_t rounds = cdiv(grid, 256), last = grid - (rounds - 1) * 256;
  return (double)(rounds - 1) * (t.c + t.full * stages) + t.c + (t.light + (t.full - t.light) * (double)last / 256) * stages;
}
inline Fp8Plan fp8_plan_of(int kind, int64_t rows, int64_t cols, int bm, int bn, int block, int splits) {
  Fp8Plan p;
  p.kind = kind;
  p.tiles_m = (int)cdiv(rows, bm);
  p.tiles_n = (int)cdiv(cols, bn);
  p.splits = splits;
  p.grid = (int64_t)p.tiles_m * p.tiles_n * splits;
  p.block = block;
  return p;
}

// What sharing a tile's contraction costs: the join's launch, the sums in memory.
inline double split_time(const Fp8Plan& p, const TileCost& t) {
  return p.splits > 1 ? 4.5 + (double)p.grid * t.bm * t.bn * 8 / 4.5e6 : 0.0;
}
// The one launch up to 2^14 values of X: each workgroup quantises all of them (1 x 4096
// x 4096 6.2 us against 2.4 + 5.0 in two launches, 4 x 4096 x 4096 7.0 against 2.4 +
// 5.5; 8 x 4096 x 4096 8.5 against 2.4 + 5.8).  Its LDS: X's codes and scales, the waves'
// sums, 27 KB at most.
constexpr int kFp8TokenRows = 16;
inline size_t fp8_token_lds(int64_t m, int64_t k) { return (size_t)((m * fp8_blocks(k) * 129 + 15) / 16 * 16 + 8192); }

inline Fp8Plan plan_fp8_fwd(int64_t m, int64_t n, int64_t k) {
  const int64_t groups = cdiv(n, 16);
  if (m <= kFp8TokenRows && m * k <= (1 << 14)) {
    // eight waves share a group of 16 features up to 1024 groups, else two (us: 1 x 11008
    // x 4096 10.9 and 12.3, 1 x 32000 x 4096 22.7 and 20.4, 1 x 4096 x 11008 12.4 and 27)
    const bool eight = groups <= 1024;
    return fp8_plan_of(eight ? FP8_TOKEN_8 : FP8_TOKEN_2, m, n, kFp8TokenRows, eight ? 16 : 64, 512, 1);
  }
  const double s = (double)fp8_blocks(k);
  Fp8Plan best{};
  double least = 1e30;
  auto consider = [&](const Fp8Plan& p, double t) {
    if (t < least) {
      least = t;
      best = p;
    }
  };
  for (const TileCost& t : kFp8Tiles) {
    const int64_t tiles = cdiv(m, t.bm) * cdiv(n, t.bn);
    if (t.kind == FP8_64x128_DEEP) {   // one workgroup to a compute unit
      for (int64_t splits = 1; splits <= std::min<int64_t>(256 / tiles, std::max<int64_t>(1, (int64_t)s / 4)); ++splits) {
        const Fp8Plan p = fp8_plan_of(t.kind, m, n, t.bm, t.bn, t.block, (int)splits);
        consider(p, tile_time(t, p.grid, (double)cdiv((int64_t)s, splits)) + split_time(p, t));
      }
    } else {
      consider(fp8_plan_of(t.kind, m, n, t.bm, t.bn, t.block, 1), tile_time(t, tiles, s));
    }
  }
  if (m <= 16) {
    const Fp8Plan p = fp8_plan_of(FP8_FEW_1, m, n, 16, 16, 512, 1);
    consider(p, 2.0 + 0.12 * s * std::max(1.0, (double)p.grid / 256));
  } else if (m <= 32) {
    const Fp8Plan p = fp8_plan_of(FP8_FEW_2, m, n, 32, 16, 512, 1);
    consider(p, 2.0 + 0.19 * s * std::max(1.0, (double)p.grid / 256));
  }
  return best;
}

// Up to 256 workgroups may share the contractions of few tiles, 4 stages to each or
// more; what that costs is the join's launch and the sums in memory.
inline Fp8Plan plan_fp8_bwd(int64_t m, int64_t n, int64_t k) {
  const int64_t stages = fp8_blocks(n);
  Fp8Plan best{};
  double least = 1e30;
  for (const TileCost& t : kFp8BackTiles) {
    const int64_t tiles = cdiv(m, t.bm) * cdiv(k, t.bn);
    const int64_t most = t.kind == FP8_BACK_64x256 ? std::max<int64_t>(1, std::min<int64_t>(256 / tiles, stages / 4)) : 1;
    for (int64_t splits = 1; splits <= most; ++splits) {
      const Fp8Plan p = fp8_plan_of(t.kind, m, k, t.bm, t.bn, t.block, (int)splits);
      const double time = tile_time(t, p.grid, (double)cdiv(stages, splits)) + split_time(p, t);
      if (time < least) {
        least = time;
        best = p;
      }
    }
  }
  return best;
}
struct Fp8Layout {
  size_t codes, scales, sums, total;
};
inline Fp8Layout fp8_fwd_layout(int64_t m, int64_t n, int64_t k) {
  Fp8Layout L;
  L.codes = 0;
  L.scales = region(fp8_codes_bytes(m, k));
  L.sums = L.scales + region(fp8_scales_bytes(m, k, 1));
  const Fp8Plan p = plan_fp8_fwd(m, n, k);
  L.total = L.sums + (p.splits > 1 ? (size_t)p.grid * 64 * 128 * 4 : 0);
  return L;
}
inline Fp8Layout fp8_bwd_layout(int64_t m, int64_t n, int64_t k) {
  Fp8Layout L;
  L.codes = 0;
  L.scales = region(fp8_codes_bytes(m, n));
  L.sums = L.scales + region(fp8_scales_bytes(m, n, 1));
  const Fp8Plan p = plan_fp8_bwd(m, n, k);
  L.total = L.sums + (p.splits > 1 ? (size_t)p.grid * 64 * 256 * 4 : 0);
  return L;
}
hipError_t launch_fp8_fwd(const Fp8Args& a, hipStream_t st);
hipError_t launch_fp8_bwd(const Fp8Args& a, hipStream_t st);

// ---- cross entropy without logits --------------------------------------------
struct XentArgs {
  const uint16_t *X, *W;
  const int32_t* labels;
  const float* dloss;
  float *loss, *saved;      // saved: [rows][2], or none
  uint16_t *dX, *dW;        // or none
  char* ws;
  int64_t rows, vocab, k;
};

// The logits' tiles and those of dX, by estimated time (TileCost above; a stage of 64
// bf16 columns moves as much as one of 128 8-bit ones).  Measured, rows x vocabulary x k:
// the loss alone (us) 300 x 4000 x 1024 13.0 on 64 x 128 (14.3 on 128 x 128, 20, 31), 37
// x 32000 x 4096 43 on 64 x 128 (50 on 256 x 128), 200 x 32000 x 4096 61 on 256 x 128
// (74 on 128 x 128, 82 on 256 x 256, 103 on 64 x 128), 1024 x 32000 x 4096 197 on 256 x
// 256 (230 on 256 x 128).  Loss with dX: 200 x 32000 x 4096 172 on 64 x 256 shared by
// four workgroups (176 on 128 x 256, 216 on 256 x 256, 383 unshared), 512 x 32003 x 4096
// 249 on 256 x 256 shared by eight (262 on 128 x 256 by four, 311 on 64 x 256).  dW of a
// piece: with its gradient of 8192 x 32000 x 1024, whose pieces are 64 tiles of 256 x 256,
// the two-call backward takes 1670 us on 64 x 256 and 2270 on 256 x 256.
enum XentTileKind { XENT_64x128, XENT_128x128, XENT_256x128, XENT_256x256 };
enum XentGradKind { XENT_GRAD_64x256, XENT_GRAD_128x256, XENT_GRAD_256x256 };
constexpr TileCost kXentTiles[4] = {{XENT_64x128, 64, 128, 256, 3.0, 0.45, 0.62},
                                    {XENT_128x128, 128, 128, 512, 5.0, 0.45, 0.60},
                                    {XENT_256x128, 256, 128, 512, 7.0, 0.65, 0.90},
                                    {XENT_256x256, 256, 256, 512, 11.0, 1.03, 1.35}};
constexpr TileCost kXentGradTiles[3] = {{XENT_GRAD_64x256, 64, 256, 256, 2.5, 0.66, 0.77},
                                        {XENT_GRAD_128x256, 128, 256, 512, 4.5, 0.72, 0.88},
                                        {XENT_GRAD_256x256, 256, 256, 512, 6.0, 1.03, 1.45}};

// The vocabulary is walked in pieces: the exponentials (or gradients) of a piece's
// logits in bf16 are the operand of the next product.  A piece's buffer is at most
// 64 MiB (and a tile's width at least), so that it is still in the last-level cache
// when it is read; of those widths the one whose tiles fill whole rounds of 256
// workgroups.
constexpr int64_t kPieceElems = int64_t(1) << 25;
struct XentPlan {
  int kind, tile_m, tile_n;    // of the logits' tiles
  int grad_kind, grad_m;       // of dX's
  int tiles_m, grad_tiles_m;
  int vtiles, piece_tiles, pieces;   // tiles of the vocabulary, of a piece
  int64_t rows_pad, piece;     // padded rows, columns of a piece (its row pitch)
  int tiles_k, splits;         // column tiles of dX, parts of a piece that workgroups share
  int dw_kind, dw_m;           // a piece's dW: XentGradKind, its rows
  int64_t stages;              // 64-column stages of a piece
  bool local;                  // the one-pass call takes a tile's powers against the tile's own largest
};
// Tiles of logits whose references a workgroup of dX holds in LDS: 64 rows' 256 in 32
// KiB, 128 rows' 40 in 10 KiB beside its stages.
constexpr int local_tiles(int grad_m) { return grad_m == 64 ? 256 : 40; }
inline XentPlan xent_plan_of(const TileCost& t, int64_t rows, int64_t vocab) {
  XentPlan p{};
  p.kind = t.kind;
  p.tile_m = t.bm;
  p.tile_n = t.bn;
  p.tiles_m = (int)cdiv(rows, t.bm);
  p.vtiles = (int)cdiv(vocab, t.bn);
  int64_t most = std::max<int64_t>(1, kPieceElems / (cdiv(rows, 256) * 256) / t.bn);
  if (most >= p.vtiles) {
    most = p.vtiles;
  } else {
    const int64_t rounds = (most * p.tiles_m + p.tiles_m - 1) / 256;
    if (rounds > 0) most = std::min(most, std::max<int64_t>(1, rounds * 256 / p.tiles_m));
  }
  p.piece_tiles = (int)most;
  p.pieces = (int)cdiv(p.vtiles, most);
  p.piece = most * t.bn;
  p.stages = p.piece / 64;
  return p;
}
inline XentPlan plan_xent(int64_t rows, int64_t vocab, int64_t k) {
  const double kstages = (double)cdiv(k, 64);
  XentPlan p{};
  double least = 1e30;
  for (const TileCost& t : kXentTiles) {
    const XentPlan q = xent_plan_of(t, rows, vocab);
    const double time = (q.pieces - 1) * tile_time(t, (int64_t)q.tiles_m * q.piece_tiles, kstages) +
                        tile_time(t, (int64_t)q.tiles_m * (q.vtiles - (int64_t)(q.pieces - 1) * q.piece_tiles), kstages);
    if (time < least) {
      least = time;
      p = q;
    }
  }
  p.tiles_k = (int)cdiv(k, 256);
  least = 1e30;
  for (const TileCost& t : kXentGradTiles) {
    const int64_t tm = cdiv(rows, t.bm), tiles = tm * p.tiles_k;
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(256 / tiles, p.stages / 8));
    for (int64_t splits = 1; splits <= most; ++splits) {
      // (W's columns come from memory at 5.5 TB/s, whoever reads them first)
      double time = std::max(tile_time(t, tiles * splits, (double)cdiv(p.stages, splits)), (double)(p.piece * k) * 2 / 5.5e6) +
                    (double)(tiles * splits) * t.bm * 256 * 8 * (p.pieces > 1) / 4.5e6;
      if (splits > 1) time += (4.5 + (double)(tiles * splits) * t.bm * 256 * 8 / 4.5e6) / p.pieces;
      if (time < least) {
        least = time;
        p.grad_kind = t.kind;
        p.grad_m = t.bm;
        p.grad_tiles_m = (int)tm;
        p.splits = (int)splits;
      }
    }
  }
  least = 1e30;
  for (const TileCost& t : kXentGradTiles) {
    const double time = tile_time(t, cdiv(std::min(p.piece, vocab), t.bm) * p.tiles_k, (double)cdiv(rows, 64));
    if (time < least) {
      least = time;
      p.dw_kind = t.kind;
      p.dw_m = t.bm;
    }
  }
  p.local = p.pieces == 1 && p.grad_kind != XENT_GRAD_256x256 &&
            cdiv(p.stages, p.splits) / (p.tile_n / 64) + 2 <= local_tiles(p.grad_m);
  const int64_t pad = std::max(p.tile_m, p.grad_m);
  p.rows_pad = cdiv(rows, pad) * pad;
  return p;
}
// Regions of the workspace.
struct XentLayout {
  size_t coef;     // [rows_pad][2] dX = c1 sum_v e_v W_v + c2 W_label
  size_t ref;      // [2][rows_pad] references of the exponentials, of a piece and the next
  size_t best;     // [2][rows_pad] a piece's largest logits
  size_t parts;    // [tile][rows_pad] reference and sum of each tile's rows
  size_t piece;    // [rows_pad][piece] exponentials or gradients of a piece
  size_t turned;   // [piece][rows_pad] the latter turned, for dW
  size_t known;    // [rows][k] X, zero in rows without a label, for dW
  size_t sums;     // [split][tile] fp32 sums of dX
  size_t saved;    // of the forward, in a call that runs both
  size_t total;
};
inline XentLayout xent_layout(int64_t rows, int64_t vocab, int64_t k, bool dx, bool dw) {
  const XentPlan p = plan_xent(rows, vocab, k);
  XentLayout L;
  L.coef = 0;
  L.ref = L.coef + region((size_t)p.rows_pad * 8);
  L.best = L.ref + region((size_t)p.rows_pad * 8);
  L.parts = L.best + region((size_t)p.rows_pad * 8);
  L.piece = L.parts + region((size_t)p.vtiles * p.rows_pad * 8);
  L.turned = L.piece + (dx || dw ? region((size_t)(p.rows_pad * p.piece) * 2) : 0);
  L.known = L.turned + (dw ? region((size_t)(p.rows_pad * p.piece) * 2) : 0);
  L.sums = L.known + (dw ? region((size_t)(rows * k) * 2) : 0);
  L.saved = L.sums + (dx ? region((size_t)p.splits * p.grad_tiles_m * p.tiles_k * p.grad_m * 256 * 4) : 0);
  L.total = L.saved + (dw ? region((size_t)rows * 8) : 0);
  return L;
}
hipError_t launch_xent_fwd(const XentArgs& a, hipStream_t st);
hipError_t launch_xent_bwd(const XentArgs& a, hipStream_t st);
hipError_t launch_xent_step(const XentArgs& a, hipStream_t st);

}  // namespace lora
