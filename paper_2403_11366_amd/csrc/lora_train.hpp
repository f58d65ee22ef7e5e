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

enum Fp8Kind { FP8_SMALL, FP8_BIG };
struct Fp8Plan {
  Fp8Kind kind;
  int tiles_m, tiles_n, splits;
  int64_t grid;
};
inline Fp8Plan plan_fp8_fwd(int64_t m, int64_t n, int64_t k) {
  (void)k;
  Fp8Plan p;
  p.kind = cdiv(m, 256) * cdiv(n, 256) >= 128 ? FP8_BIG : FP8_SMALL;
  p.tiles_m = (int)cdiv(m, p.kind == FP8_BIG ? 256 : 64);
  p.tiles_n = (int)cdiv(n, p.kind == FP8_BIG ? 256 : 128);
  p.splits = 1;
  p.grid = (int64_t)p.tiles_m * p.tiles_n;
  return p;
}
inline Fp8Plan plan_fp8_bwd(int64_t m, int64_t n, int64_t k) {
  Fp8Plan p;
  p.kind = cdiv(m, 256) * cdiv(k, 256) >= 128 ? FP8_BIG : FP8_SMALL;
  p.tiles_m = (int)cdiv(m, p.kind == FP8_BIG ? 256 : 64);
  p.tiles_n = (int)cdiv(k, 256);
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
  p.splits = p.kind == FP8_BIG ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(256 / tiles, fp8_blocks(n)));
  p.grid = tiles * p.splits;
  return p;
}
struct Fp8Layout {
  size_t codes, scales, sums, total;
};
inline Fp8Layout fp8_fwd_layout(int64_t m, int64_t n, int64_t k) {
  (void)n;
  Fp8Layout L;
  L.codes = 0;
  L.scales = region(fp8_codes_bytes(m, k));
  L.sums = L.total = L.scales + region(fp8_scales_bytes(m, k, 1));
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

// Few rows take tiles of 64 rows (128 columns of logits, 256 of gradients), others
// 256 x 256.
//
// The vocabulary is walked in pieces: the exponentials (or gradients) of a piece's
// logits in bf16 are the operand of the next product.  A piece's buffer is at most
// 64 MiB (and a tile's width at least), so that it is still in the last-level cache
// when it is read; of those widths the one whose tiles fill whole rounds of 256
// workgroups.
constexpr int64_t kPieceElems = int64_t(1) << 25;
struct XentPlan {
  bool big;
  int tile_m, tile_n;          // of the logits' tiles
  int tiles_m;
  int vtiles, piece_tiles, pieces;   // tiles of the vocabulary, of a piece
  int64_t rows_pad, piece;     // padded rows, columns of a piece (its row pitch)
  int tiles_k, splits;         // column tiles of dX, parts of a piece that workgroups share
  int64_t stages;              // 64-column stages of a piece
};
inline XentPlan plan_xent(int64_t rows, int64_t vocab, int64_t k) {
  XentPlan p;
  p.big = rows > 128;
  p.tile_m = p.big ? 256 : 64;
  p.tile_n = p.big ? 256 : 128;
  p.tiles_m = (int)cdiv(rows, p.tile_m);
  p.rows_pad = (int64_t)p.tiles_m * p.tile_m;
  p.vtiles = (int)cdiv(vocab, p.tile_n);
  int64_t most = std::max<int64_t>(1, kPieceElems / p.rows_pad / p.tile_n);
  if (most >= p.vtiles) most = p.vtiles;
  else {
    const int64_t rounds = (most * p.tiles_m + p.tiles_m - 1) / 256;
    if (rounds > 0) most = std::min(most, std::max<int64_t>(1, rounds * 256 / p.tiles_m));
  }
  p.piece_tiles = (int)most;
  p.pieces = (int)cdiv(p.vtiles, most);
  p.piece = most * p.tile_n;
  p.stages = p.piece / 64;
  p.tiles_k = (int)cdiv(k, 256);
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_k;
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(256 / tiles, p.stages / 8));
  return p;
}
// Regions of the workspace.
struct XentLayout {
  size_t zy;       // [rows_pad] the labels' logits
  size_t coef;     // [rows_pad][2] dX = c1 sum_v e_v W_v + c2 W_label
  size_t ref;      // [2][rows_pad] references of the exponentials, of a piece and the next
  size_t best;     // [2][rows_pad] a piece's largest logits
  size_t parts;    // [tile][rows_pad] reference and sum of each tile's rows
  size_t piece;    // [rows_pad][piece] exponentials or gradients of a piece
  size_t turned;   // [piece][rows_pad] the latter turned, for dW
  size_t sums;     // [split][tile] fp32 sums of dX
  size_t saved;    // of the forward, in a call that runs both
  size_t total;
};
inline XentLayout xent_layout(int64_t rows, int64_t vocab, int64_t k, bool dx, bool dw) {
  const XentPlan p = plan_xent(rows, vocab, k);
  XentLayout L;
  L.zy = 0;
  L.coef = L.zy + region((size_t)p.rows_pad * 4);
  L.ref = L.coef + region((size_t)p.rows_pad * 8);
  L.best = L.ref + region((size_t)p.rows_pad * 8);
  L.parts = L.best + region((size_t)p.rows_pad * 8);
  L.piece = L.parts + region((size_t)p.vtiles * p.rows_pad * 8);
  L.turned = L.piece + (dx || dw ? region((size_t)(p.rows_pad * p.piece) * 2) : 0);
  L.sums = L.turned + (dw ? region((size_t)(p.rows_pad * p.piece) * 2) : 0);
  L.saved = L.sums + (dx ? region((size_t)p.splits * p.tiles_m * p.tiles_k * p.tile_m * 256 * 4) : 0);
  L.total = L.saved + (dw ? region((size_t)rows * 8) : 0);
  return L;
}
hipError_t launch_xent_fwd(const XentArgs& a, hipStream_t st);
hipError_t launch_xent_bwd(const XentArgs& a, hipStream_t st);
hipError_t launch_xent_step(const XentArgs& a, hipStream_t st);

}  // namespace lora
