// Internal interface of the operators around the layer's output between the C
// ABI (lora_ops_abi.cpp: argument checks) and their kernels: 4-bit weights
// (lora_mx4.hip), token log probabilities and distillation (lora_logits.hip).
// Shapes here have already been validated; the launch rules stand here, apart from
// the kernels, so that they can be checked on the host.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace lora {

constexpr int kMaxTop = 128;   // alternatives of a row, and entries of a teacher's list

// ---- rows of logits ----------------------------------------------------------
// A row is walked in chunks of 16 bytes (8 bf16 or 4 fp32 values): the whole
// ones that start at a 16-byte boundary, and single elements before and after.
//
// The distillation step keeps a row in the registers of one workgroup: `threads`
// x `keep` chunks; keep = 0 reads the row again for the gradient.
struct RowShape {
  int threads, keep;
};

// Four chunks a thread, with which it can hold the exponentials too, up to 1024
// threads; then up to 16, 64 of a thread's 128 registers (512 x 131072 bf16 66 us, 79
// read twice).
inline RowShape row_shape(int64_t vocab, int elem) {
  const int64_t chunks = (vocab * elem + 15) / 16;
  if (chunks <= 1024) return RowShape{256, 4};
  if (chunks <= 2048) return RowShape{512, 4};
  if (chunks <= 4096) return RowShape{1024, 4};
  if (chunks <= 8192) return RowShape{1024, 8};
  if (chunks <= 16384) return RowShape{1024, 16};
  return RowShape{1024, 0};
}

// Units of 4 KiB of a row (and one for its ends), each with three fp32 sums.
constexpr int kUnitBytes = 4096;
constexpr int kMaxUnits = 1026;      // of 2^20 fp32 values
constexpr int kSmallUnits = 33;      // of the rows that 256 threads take
inline int64_t score_units(int64_t vocab, int elem) { return (vocab * elem + kUnitBytes - 1) / kUnitBytes + 1; }

// Threads to a row in the calls that only read it; a row's results do not depend
// on them.  Up to one row a compute unit takes 1024 threads each (256 x 32000 bf16
// with 20 alternatives: 9.6 us, 10.0 with 512 threads, 11.7 with 256; 300 rows: 15.2,
// 12.4, 13.0).  Otherwise a wave is to have units to load while others reduce, but
// not so many that few rows leave the chip empty: the forward's waves more than
// one unit (4096 x 32000 bf16: 52 us with 512 threads, 55 with 256; 8192 x 8000: 40
// and 33), those of the log probabilities, where a row's threads wait for its
// selection, more than four (4096 x 32000 with 20 alternatives: 65 and 61).  Up to
// three rows a compute unit the chip has room for 512 anyway (512 x 32000: log
// probabilities 13.2 and 14.2, forward 9.8 and 10.2; 768 rows: 16.3 and 16.2, 12.3
// and 12.1; 900: 19.8 and 18.5, 14.1 and 13.8; rows of 8000 do not tell up to there).
inline int read_threads(int64_t rows, int64_t vocab, int elem, int least_units) {
  if (rows <= 256) return 1024;
  return rows <= 768 || score_units(vocab, elem) > std::min(8 * least_units, kSmallUnits) ? 512 : 256;
}

struct LogprobArgs {
  const void* logits;
  bool f32;
  int64_t ld;
  const int32_t* tokens;   // or none
  float itau;              // 1 / temperature
  float *logp, *entropy;
  int32_t* top_ids;
  float* top_logp;
  char* ws;
  int64_t rows;
  int vocab, top;
};

// Parts of a row: workgroups of at least 16 units (one to a wave), as many as 256
// together, with at most kMaxKeys top values to join.
constexpr int kMaxKeys = 512;
inline int score_parts(int64_t rows, int64_t vocab, int elem, int64_t top) {
  const int64_t most = std::min<int64_t>(256 / rows, (score_units(vocab, elem) - 1) / 16);
  return (int)std::max<int64_t>(1, top > 0 ? std::min<int64_t>(most, kMaxKeys / top) : most);
}
struct Unit {
  float m, s, a;   // maximum, and two sums against it
};
struct ScoreParts {   // the workspace of a split call
  uint64_t* keys;     // [rows, parts, top]
  Unit* units;        // [rows, units_ld]
  int64_t units_ld;
  ScoreParts(char* ws, int64_t rows, int64_t vocab, int elem, int parts, int64_t top)
      : keys(reinterpret_cast<uint64_t*>(ws)),
        units(reinterpret_cast<Unit*>(ws + rows * parts * top * 8)),
        units_ld(score_units(vocab, elem)) {}
};
// (for fp32 logits, which have more of both; never 0)
inline size_t logprobs_workspace(int64_t rows, int64_t vocab, int64_t top) {
  const int parts = score_parts(rows, vocab, 4, top);
  return parts == 1 ? 256 : (size_t)rows * (score_units(vocab, 4) * sizeof(Unit) + 8 * parts * top);
}

struct DistillArgs {
  const void* logits;
  bool f32;
  int64_t ld;
  const int32_t* ids;      // teacher's list [rows, top]
  const float* teacher;    // its logits
  const int32_t* labels;   // or none (soft_weight 1)
  float tau, w;            // temperature, weight of the soft term
  float *loss, *saved;
  const float* dloss;
  void* dlogits;
  int64_t rows;
  int vocab, top;
};

// Columns of one workgroup of the gradient that reads what the forward saved.
constexpr int kGradThreads = 256, kGradKeep = 8;
inline int grad_parts(int64_t vocab, int elem) {
  const int64_t chunks = (vocab * elem + 15) / 16;
  return (int)((chunks + kGradThreads * kGradKeep - 1) / (kGradThreads * kGradKeep));
}

hipError_t launch_token_logprobs(const LogprobArgs& a, hipStream_t st);
hipError_t launch_distill_fwd(const DistillArgs& a, hipStream_t st);
hipError_t launch_distill_bwd(const DistillArgs& a, hipStream_t st);
hipError_t launch_distill_step(const DistillArgs& a, hipStream_t st);

// ---- 4-bit weights -----------------------------------------------------------
// Microscaled 4 bits: rows of 32-column blocks, a byte of scale each.  A row's
// codes take 128 bytes per 256 columns; scales stand in cells of 512 bytes, one
// per 64 rows and 256 columns (mx4_scale_offset).
inline int64_t mx4_slabs(int64_t k) { return (k + 255) / 256; }        // 256-column slabs of a row
inline int64_t mx4_groups(int64_t rows) { return (rows + 63) / 64; }   // 64-row groups
inline size_t mx4_codes_bytes(int64_t rows, int64_t k) { return (size_t)(rows * mx4_slabs(k) * 128); }
inline size_t mx4_scales_bytes(int64_t rows, int64_t k) { return (size_t)(mx4_groups(rows) * mx4_slabs(k) * 512); }

struct Mx4QuantArgs {
  const uint16_t* X;
  uint8_t *codes, *scales;
  int64_t rows, k;
};

struct Mx4FwdArgs {
  const uint16_t* X;
  const uint8_t *Wc, *Ws;
  uint16_t* Y;
  char* ws;
  int64_t m, n, k;
};

// Kernel of the 4-bit forward.  One launch that quantises X on its way for very
// few values of X; else X is quantised before, and the product is formed by
// waves on different slabs straight from memory (few tokens) or by tiles staged
// in LDS.
enum Mx4Kind {
  MX4_TOKEN_8, MX4_TOKEN_2, MX4_FEW_1, MX4_FEW_2, MX4_FEW_4, MX4_64x128, MX4_128x128, MX4_256x128, MX4_256x256
};

struct Mx4Plan {
  Mx4Kind kind;
  int tiles_m, tiles_n;   // of the output
  int64_t grid;           // workgroups
  int block;
};

// LDS of the one launch: X's fragments and scales, the waves' sums.
constexpr int kTokenRows = 16;
inline size_t mx4_token_lds(int64_t slabs) { return (size_t)slabs * 2176 + 8192; }

// The one launch up to 2^15 values of X: each workgroup quantises all of them
// (8 x 4096 x 4096 6.1 us against 2.5 + 4.3 in two launches, 16 x 4096 x 4096 8.6
// against 2.5 + 4.7; 1 x 4096 x 4096 4.3 against 2.5 + 4.0).
//
// The others by their estimated time in us, launches and the quantisation left
// out.  A round of workgroups that fills the compute units takes c + full x slabs
// and a round of few of them c + light x slabs (the card is then short of
// neither power nor memory); the last one lies between.  Fitted to k = 512 to
// 16384: 4096 x 4096 x 4096 36 us on 256 x 256 (47 on 256 x 128), 2048 x 4096 x
// 4096 23 on 256 x 128 (28 on 256 x 256 and on 128 x 128), 1024 x 4096 x 4096 15 on
// 128 x 128 (16 on 64 x 128, 20 on 256 x 128), 512 x 4096 x 4096 12 on 64 x 128 (13
// on 128 x 128), 128 x 4096 x 4096 9.8 from memory (11.4 on 64 x 128).
struct Mx4Tile {
  Mx4Kind kind;
  int bm, bn, per_cu, block;
  double c, light, full;
};
constexpr Mx4Tile kMx4Tiles[4] = {{MX4_256x256, 256, 256, 1, 512, 6.0, 1.37, 1.85},
                                  {MX4_256x128, 256, 128, 1, 512, 5.0, 0.75, 1.2},
                                  {MX4_128x128, 128, 128, 1, 256, 2.2, 0.6, 0.78},
                                  {MX4_64x128, 64, 128, 2, 128, 1.5, 0.5, 0.93}};

inline Mx4Plan mx4_plan_of(Mx4Kind kind, int64_t m, int64_t n, int bm, int bn, int block) {
  Mx4Plan p;
  p.kind = kind;
  p.tiles_m = (int)((m + bm - 1) / bm);
  p.tiles_n = (int)((n + bn - 1) / bn);
  p.grid = (int64_t)p.tiles_m * p.tiles_n;
  p.block = block;
  return p;
}

inline Mx4Plan plan_mx4_fwd(int64_t m, int64_t n, int64_t k) {
  const int64_t slabs = mx4_slabs(k), groups = (n + 15) / 16;
  if (m <= kTokenRows && m * k <= (1 << 15) && mx4_token_lds(slabs) <= 160 * 1024) {
    // eight waves share a group of 16 features up to 512 groups, of more than eight
    // tokens (which each workgroup quantises) up to 256, else two.  Eight and two, us:
    // 1 x 4096 x 4096 4.5, 7.0; 1 x 8192 x 4096 5.8, 7.2; 1 x 16384 x 4096 10.8, 9.1;
    // 1 x 4096 x 13824 (one workgroup to a compute unit's LDS) 8.7, 18.0; 1 x 8192 x
    // 13824 17.5, 20.5; 1 x 11008 x 13824 24.0, 21.5; 8 x 8192 x 4096 9.2, 9.0; 16 x
    // 4096 x 2048 5.7, 6.7; 16 x 5120 x 2048 7.8, 6.7
    const bool eight = groups <= (m <= 8 ? 512 : 256);
    return mx4_plan_of(eight ? MX4_TOKEN_8 : MX4_TOKEN_2, 1, n, 1, eight ? 16 : 64, 512);
  }
  Mx4Plan best{};
  double best_time = 1e30;
  auto consider = [&](const Mx4Plan& p, double t) {
    if (t < best_time) {
      best_time = t;
      best = p;
    }
  };
  const double s = (double)slabs;
  for (const Mx4Tile& t : kMx4Tiles) {
    const Mx4Plan p = mx4_plan_of(t.kind, m, n, t.bm, t.bn, t.block);
    const int64_t cap = 256 * t.per_cu, rounds = (p.grid + cap - 1) / cap, last = p.grid - (rounds - 1) * cap;
    const double part = t.per_cu == 1 ? (double)last / 256 : (last > 256 ? 1.0 : 0.0);
    consider(p, (double)(rounds - 1) * (t.c + t.full * s) + t.c + (t.light + (t.full - t.light) * part) * s);
  }
  // from memory: by the rounds of 256 workgroups, shared where several fit a compute unit
  if (m <= 16) {
    const Mx4Plan p = mx4_plan_of(MX4_FEW_1, m, n, 16, 16, 512);
    consider(p, 1.0 + 0.15 * s * (p.grid > 256 ? (double)p.grid / 256 : 1.0));
  } else if (m <= 32) {
    const Mx4Plan p = mx4_plan_of(MX4_FEW_2, m, n, 32, 16, 512);
    consider(p, 1.0 + 0.19 * s * (p.grid > 256 ? (double)p.grid / 256 : 1.0));
  } else {
    const Mx4Plan p = mx4_plan_of(MX4_FEW_4, m, n, 64, 32, 512);
    consider(p, (double)((p.grid + 255) / 256) * (2.3 + 0.39 * s));
  }
  return best;
}

// What a tile's copies read.  A copy's address is a scalar offset, the same for
// the wave, and a lane offset.  The lanes' alone is sure to be compared with the
// operand's size, or with that size less the scalar offset: what lies past the
// operand has a lane offset past any operand and a scalar offset inside it.
constexpr uint32_t kMx4None = 0x80000000u;
struct Mx4Slab {
  uint32_t kb, none;           // the slab of the scalar offset; kMx4None or 0, for the lanes
};
__host__ __device__ inline Mx4Slab mx4_slab(int kb, int slabs) {
  return kb < slabs ? Mx4Slab{(uint32_t)kb, 0u} : Mx4Slab{0u, kMx4None};
}
struct Mx4Cell {
  uint32_t first, step, none;  // byte of a cell of scales in slab 0, bytes from slab to slab; as above
};
__host__ __device__ inline Mx4Cell mx4_cell(int cell, int cells) {
  return cell < cells ? Mx4Cell{(uint32_t)cell * 512, (uint32_t)cells * 512, 0u} : Mx4Cell{0u, 0u, kMx4None};
}

// Workspace of the 4-bit forward: X's codes and scales.
struct Mx4Layout {
  size_t xc, xs, total;
};
inline Mx4Layout mx4_fwd_layout(int64_t m, int64_t n, int64_t k) {
  (void)n;
  Mx4Layout L;
  L.xc = 0;
  L.xs = (mx4_codes_bytes(m, k) + 255) / 256 * 256;
  L.total = L.xs + (mx4_scales_bytes(m, k) + 255) / 256 * 256;
  return L;
}

hipError_t launch_mx4_quantize(const Mx4QuantArgs& a, hipStream_t st);
hipError_t launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, uint16_t* X, int64_t rows, int64_t k,
                                 hipStream_t st);
hipError_t launch_mx4_fwd(const Mx4FwdArgs& a, hipStream_t st);

}  // namespace lora
