// Matrix product cores shared by the 8-bit linear layer (lora_fp8.hip) and the
// cross entropy without logits (lora_xent.hip): output tiles of BM rows x BN
// columns whose sums stay in registers, for an epilogue of the caller's.
//
//   nt_*:  C = A B^T, both operands' rows contiguous along the contraction
//   nn_*:  C = A B,   A as above, B's rows contiguous along the columns
//
// A stage is 128 bytes of contraction of every k-contiguous row: 64 bf16 or 128
// 8-bit elements.  Lane l (g = l / 16, c = l % 16) multiplies chunks g and g + 4 of
// 16 bytes of a row's eight: two 16x16x32 bf16 products, or one 16x16x128 product
// of 8 bits.  The order in which a product's contraction stands in the registers
// is free as long as both operands agree on it, so both types share addresses,
// copies and reads; the 8-bit ones' scales cover a whole stage (blocks of 128), so
// they do not depend on it either.  (The 8-bit instruction adds the 16 products of a
// chunk after cutting each, towards zero, to a multiple of 2^-13 of the largest one's
// power of two -- a product has 8 significant bits, so only those below 2^-7 of the
// largest lose any -- and chunks in fp32: measured by products that cancel.  On normal
// values that is far below the result's rounding to bf16.)  Products are formed transposed (B as the A
// operand), so a lane's sums are 4 consecutive columns of one row:
//   acc[a][b] of lane l: row 16 b + c of the wave's, columns 4 g .. 4 g + 3 of
//   fragment a.
#pragma once

#include <type_traits>
#include <utility>

#include "lora_device.hpp"

namespace lora {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef int int2w __attribute__((ext_vector_type(2)));

template <typename F, int... I>
__device__ __forceinline__ void each_index(std::integer_sequence<int, I...>, F&& f) {
  (f(std::integral_constant<int, I>{}), ...);
}
// f(0), ..., f(N - 1) with compile-time arguments.
template <int N, typename F>
__device__ __forceinline__ void each_of(F&& f) {
  each_index(std::make_integer_sequence<int, N>{}, f);
}

struct Bf16 {
  static constexpr int BYTES = 2, KS = 64;   // of an element; elements of a stage
  static constexpr bool SCALED = false;
};
struct Fp8 {   // e4m3
  static constexpr int BYTES = 1, KS = 128;
  static constexpr bool SCALED = true;
};

__device__ __forceinline__ uint2 bf16x4(const floatx4& v) {
  return uint2{(uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16),
               (uint32_t)f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16)};
}

struct Frag {   // of 16 rows (or columns) x a stage
  int4v lo, hi;
};

// The sums are formed here, and not where a caller's branch on a lane's row or column
// first uses them: a product reads registers (the scales among them) of lanes that
// such a branch has switched off.
template <int FA, int FB>
__device__ __forceinline__ void formed(floatx4 (&acc)[FA][FB]) {
#pragma unroll
  for (int a = 0; a < FA; ++a)
#pragma unroll
    for (int b = 0; b < FB; ++b) asm volatile("" : "+v"(acc[a][b]));
}

// acc += A B^T of a stage; SB picks the byte of sb (the rows' scales), sa is the
// columns'.
template <class E, int SB>
__device__ __forceinline__ floatx4 stage_product(const Frag& a, const Frag& b, floatx4 acc, int sa, int sb) {
  if constexpr (E::SCALED) {
    const int8v A{a.lo[0], a.lo[1], a.lo[2], a.lo[3], a.hi[0], a.hi[1], a.hi[2], a.hi[3]};
    const int8v B{b.lo[0], b.lo[1], b.lo[2], b.lo[3], b.hi[0], b.hi[1], b.hi[2], b.hi[3]};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, acc, 0, 0, 0, sa, SB, sb);
  } else {
    acc = mfma16x16x32(__builtin_bit_cast(short8, a.lo), __builtin_bit_cast(short8, b.lo), acc);
    return mfma16x16x32(__builtin_bit_cast(short8, a.hi), __builtin_bit_cast(short8, b.hi), acc);
  }
}

// Scales of 8-bit operands.  A's (activations): a word per 16-row position of a
// 64-row cell, cells [stage][cells]; B's (a weight): one byte per 128 x 128 block.
struct Scales {
  const uint8_t* a;
  const uint8_t* b;
  int cells;      // 64-row cells of A
  int b_first;    // B: byte of (this tile's first column block, stage 0)
  int b_step;     // from stage to stage
  int b_col;      // from column block to column block
  int b_cols;     // column blocks from this tile's first on (clamped to)
};

// A lane's offset in a stage's scales of A: words of `count` cells from `first` on,
// past them and past the operand kOOB.
__device__ __forceinline__ uint32_t scale_words(const Scales& s, int first, int count, int lane) {
  return lane < 16 * count && first + (lane >> 4) < s.cells ? (uint32_t)first * 64 + 4 * lane : kOOB;
}

// A tile's operands.
struct NtTile {
  __amdgpu_buffer_rsrc_t a, b;    // from the tile's first row, and column, on
  uint32_t a_row, b_row;          // bytes of a row
  uint32_t kbytes;                // of them to contract
  int stages;
};
struct NnTile {
  __amdgpu_buffer_rsrc_t a;       // from the tile's first row on
  uint32_t a_row;
  const char* b;                  // column of the tile's first, row 0 of the contraction
  uint32_t b_row;
  uint64_t b_bytes;               // from b to the operand's end
  int stages;
};
// B's rows from the current stage on: what is left of the operand (past its end
// nothing, and copies of zeros).
struct NnRows {
  const char* at;
  uint64_t left;
  uint32_t step;   // bytes of a stage's rows
  __device__ __forceinline__ void start(const NnTile& t, int stage, int ks) {
    step = t.b_row * (uint32_t)ks;
    const uint64_t skip = (uint64_t)stage * step;
    left = t.b_bytes > skip ? t.b_bytes - skip : 0;
    at = t.b + (left ? skip : 0);
  }
  __device__ __forceinline__ void next() {
    at += step;
    left = left > step ? left - step : 0;
  }
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t rows() const { return make_rsrc(at, left); }
};

// The weight's scale bytes of up to 64 stages in one register, a stage to a lane
// (with two column blocks a stage: 32 stages, two lanes each).
template <int COLS>
struct BScales {
  int lanes = 0, base = 0;
  static constexpr int SPAN = 64 / COLS;
  __device__ __forceinline__ void load(const Scales& s, int col, int kb, int stages, int lane) {
    base = kb;
    const int st = min(kb + lane / COLS, stages - 1), cb = min(col + lane % COLS, s.b_cols - 1);
    lanes = s.b[(size_t)s.b_first + (size_t)st * s.b_step + (size_t)cb * s.b_col];
    asm volatile("" : "+v"(lanes));   // waited for here, once, and not at every use
  }
  __device__ __forceinline__ int at(int kb, int col) const {
    return __builtin_amdgcn_readlane(lanes, (kb - base) * COLS + col);
  }
};

// ---------------------------------------------------------------------------
// C = A B^T, BM x BN by WM x WN waves, NS stages of LDS copied from memory straight
// into LDS, one barrier a stage, fragments read a stage ahead.
//
// A compute unit often holds one such workgroup, a wave to a SIMD, and then the wave's
// own instructions bound a stage: the loop is unrolled over the stages' places, whose
// addresses are constants, and copies past the end take the last stage again (nobody
// reads them) instead of a condition each.  Copies and LDS reads are issued between the
// products, a few behind each row fragment's: issued ahead of them all they took 0.1 us
// more of a stage (8 bits, 256 x 128: 0.58 to 0.90 us against 0.77 to 1.00; 1531 x 4104
// x 3208 27.5 -> 24.2 us), since the wave's first product waited for its last issue.
template <class E, int BM, int BN, int WM, int WN, int NS, bool TAIL>
struct NtCore {
  static constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN, FA = TN / 16, FB = TM / 16;
  static constexpr int CX = BM / 8 / NW, CB = BN / 8 / NW, CS = E::SCALED ? 1 : 0, C = CX + CB + CS;
  static constexpr int SOFF = (BM + BN) * 128, STAGE = SOFF + CS * NW * 256, SMEM = NS * STAGE;
  static_assert(TM % 64 == 0 && TN % 16 == 0 && BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && NS * C < 64, "tile");
  typedef floatx4 Acc[FA][FB];
  static __device__ __forceinline__ int row0(int wave) { return wave / WN * TM; }
  static __device__ __forceinline__ int col(int wave, int a) { return wave % WN * TN + 16 * a; }

  static __device__ __forceinline__ void run(const NtTile& t, const Scales& sc, int m0, char* smem, Acc& acc) {
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int wm = wave / WN, wn = wave % WN, g = lane >> 4, c16 = lane & 15, l8 = lane >> 3;
#pragma unroll
    for (int a = 0; a < FA; ++a)
#pragma unroll
      for (int b = 0; b < FB; ++b) acc[a][b] = floatx4{0.f, 0.f, 0.f, 0.f};
    const int crow = 8 * wave;
    const uint32_t kcol = (uint32_t)(((lane & 7) ^ kc_swz(crow + l8)) << 4);
    uint32_t aoff[CX], boff[CB], soff = kOOB;
#pragma unroll
    for (int i = 0; i < CX; ++i) aoff[i] = (uint32_t)(crow + l8 + 8 * NW * i) * t.a_row + kcol;
#pragma unroll
    for (int i = 0; i < CB; ++i) boff[i] = (uint32_t)(crow + l8 + 8 * NW * i) * t.b_row + kcol;
    __amdgpu_buffer_rsrc_t rsS = t.a;
    BScales<1> bs;
    const int bcol = wn * TN / 128;
    const uint32_t sstep = E::SCALED ? (uint32_t)sc.cells * 64 : 0;
    if constexpr (E::SCALED) {
      rsS = make_rsrc(sc.a, (uint64_t)sstep * t.stages);
      soff = scale_words(sc, m0 / 64 + wm * (TM / 64), TM / 64, lane);
      bs.load(sc, bcol, 0, t.stages, lane);
    }
    const uint32_t last = (uint32_t)(t.stages - 1) * 128, slast = (uint32_t)(t.stages - 1) * sstep;
    uint32_t at = 0, sat = 0;   // of the next stage to copy
    char* const mine = smem + crow * 128;
    // The q-th copy of the wave's C of a stage; the last one moves on to the next stage.
    auto copy_one = [&](auto place, auto qc) LORA_INLINE {
      constexpr int Q = decltype(qc)::value, O = decltype(place)::value * STAGE;
      const bool out = TAIL && at + kcol >= t.kbytes;
      if constexpr (Q < CX) {
        dma16(t.a, out ? kOOB : aoff[Q], at, mine + O + 8 * NW * Q * 128);
      } else if constexpr (Q < CX + CB) {
        dma16(t.b, out ? kOOB : boff[Q - CX], at, mine + O + (BM + 8 * NW * (Q - CX)) * 128);
      } else {
        dma4(rsS, soff, sat, smem + O + SOFF + wave * 256);
        sat = min(sat + sstep, slast);
      }
      if constexpr (Q == C - 1) at = min(at + 128, last);
    };
    auto copy = [&](auto place) LORA_INLINE { each_of<C>([&](auto q) LORA_INLINE { copy_one(place, q); }); };
    Frag fa[2][FA], fb[2][FB];   // of this stage and the next
    int sa[2] = {}, sw[2][TM / 64] = {};
    // Rows 16 apart swizzle alike, and the second chunk is 4 further.
    const uint32_t f0 = kc_offset(c16, g), f1 = f0 ^ 64;
    const char *a0 = smem + (BM + wn * TN) * 128 + f0, *a1 = smem + (BM + wn * TN) * 128 + f1;
    const char *b0 = smem + wm * TM * 128 + f0, *b1 = smem + wm * TM * 128 + f1;
    const char* s0 = smem + SOFF + wave * 256 + c16 * 4;
    int O = 0;   // of the place that is read
    auto read_scales = [&](int kb, auto set) LORA_INLINE {
      constexpr int S = decltype(set)::value;
      if constexpr (E::SCALED) {
        sa[S] = bs.at(kb, 0);
#pragma unroll
        for (int i = 0; i < TM / 64; ++i) sw[S][i] = *reinterpret_cast<const int*>(s0 + O + i * 64);
      }
    };
    auto read_one = [&](auto set, auto qc) LORA_INLINE {   // fragment q of the FA + FB
      constexpr int S = decltype(set)::value, Q = decltype(qc)::value;
      if constexpr (Q < FA)
        fa[S][Q] = Frag{*reinterpret_cast<const int4v*>(a0 + O + 2048 * Q), *reinterpret_cast<const int4v*>(a1 + O + 2048 * Q)};
      else
        fb[S][Q - FA] = Frag{*reinterpret_cast<const int4v*>(b0 + O + 2048 * (Q - FA)),
                             *reinterpret_cast<const int4v*>(b1 + O + 2048 * (Q - FA))};
    };
    auto set_place = [&](auto place) LORA_INLINE {
      O = decltype(place)::value * STAGE;
      // Addresses beyond the reads' own offsets are formed here where a wave's sums need the
      // registers that keeping them for every place takes.
      if (SMEM > 65536 && FA * FB >= 16) asm volatile("" : "+s"(O));
    };
    // A stage's products; behind each row fragment's, f(its index).
    auto multiply = [&](auto set, auto&& f) LORA_INLINE {
      constexpr int S = decltype(set)::value;
      each_of<FB>([&](auto bc) LORA_INLINE {
        constexpr int B = decltype(bc)::value;
#pragma unroll
        for (int a = 0; a < FA; ++a)
          acc[a][B] = stage_product<E, B & 3>(fa[S][a], fb[S][B], acc[a][B], sa[S], sw[S][B >> 2]);
        __builtin_amdgcn_sched_barrier(0);
        f(bc);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    each_of<NS>([&](auto j) LORA_INLINE { copy(j); });
    copy_barrier<(NS - 1) * C>();
    {
      using I0 = std::integral_constant<int, 0>;
      set_place(I0{});
      read_scales(0, I0{});
      each_of<FA + FB>([&](auto q) LORA_INLINE { read_one(I0{}, q); });
    }
    constexpr int U = NS % 2 ? 2 * NS : NS;
    for (int k0 = 0; k0 < t.stages; k0 += U) {
      if constexpr (E::SCALED)
        if (k0 + U - bs.base >= bs.SPAN) bs.load(sc, bcol, k0, t.stages, lane);   // (U and the next stage's)
      each_of<U>([&](auto jc) LORA_INLINE {
        constexpr int J = decltype(jc)::value;
        // The next stage has landed, and every wave has read this one, whose place is
        // filled again.  The products come first; copies and the next stage's reads are
        // issued between them.
        if (J == 0 || k0 + J < t.stages) {
          using Next = std::integral_constant<int, (J + 1) & 1>;
          copy_barrier<(NS - 2) * C>();
          __builtin_amdgcn_sched_barrier(0);
          multiply(std::integral_constant<int, J & 1>{}, [&](auto bc) LORA_INLINE {
            constexpr int B = decltype(bc)::value;
            if constexpr (B == 0) {
              set_place(std::integral_constant<int, (J + 1) % NS>{});
              read_scales(k0 + J + 1, Next{});
            }
            each_of<FA + FB>([&](auto q) LORA_INLINE {
              if constexpr (decltype(q)::value * FB / (FA + FB) == B) read_one(Next{}, q);
            });
            each_of<C>([&](auto q) LORA_INLINE {
              if constexpr (decltype(q)::value * FB / C == B) copy_one(std::integral_constant<int, J % NS>{}, q);
            });
          });
        }
      });
    }
    formed(acc);
    copy_barrier<0>();   // the trailing copies have landed before the LDS is used again
  }
};

// ---------------------------------------------------------------------------
// LDS reads that transpose, for operands whose rows run along the columns.  16
// bits: 16 lanes take 4 rows x 16 columns, 8 bits: 8 rows x 16 columns, and lane i
// receives column i.
template <class E, int OFF>
__device__ __forceinline__ void read_tr_asm(int2w& d, uint32_t addr) {
  if constexpr (E::BYTES == 1)
    asm volatile("ds_read_b64_tr_b8 %0, %1 offset:%2" : "=v"(d) : "v"(addr), "i"(OFF));
  else
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(d) : "v"(addr), "i"(OFF));
}

// Swizzle of the 8-bit rows of 128 bytes: the 16 rows that a half wave reads (8 of
// one g, 8 of the next) fall into different banks.
__device__ __forceinline__ int mc8_swz(int row) { return ((row >> 1) & 3) + 4 * ((row >> 4) & 1); }

// The places of a stage of B, in panels of 128 columns: rows of 256 bytes (bf16,
// 64 rows) or 128 bytes (8 bits, 128 rows), 16 KiB a panel.
template <class E>
struct Panel {
  static constexpr int ROW = 128 * E::BYTES, CHUNKS = ROW / 16, RPC = 64 / CHUNKS;   // rows per copy of 1 KiB
  static __device__ __forceinline__ int swz(int row) { return E::BYTES == 1 ? mc8_swz(row) : mc16_swz(row); }
  // Address of the first read of the fragment at column chunk `chunk` (of 16 columns);
  // the others are 1024, 8192 and 9216 bytes further (registers in that order).
  static __device__ __forceinline__ uint32_t read_at(int frag, int lane) {
    const int g = lane >> 4, j = lane & 15;
    if constexpr (E::BYTES == 1) {
      const int row = 16 * g + (j >> 1);
      return (uint32_t)(row * ROW + ((frag ^ swz(row)) << 4) + (j & 1) * 8);
    } else {
      const int row = 8 * g + (j >> 2), q = j & 3;
      return (uint32_t)(row * ROW + (((2 * frag + (q >> 1)) ^ swz(row)) << 4) + (q & 1) * 8);
    }
  }
};

// bf16 values of at most 1, not negative, times 2^-(shift / 128): below 2^-126 nearly
// or quite 0.
__device__ __forceinline__ int4v scaled_down(int4v v, uint32_t shift) {
  typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
  const ushort2v by{(unsigned short)shift, (unsigned short)shift};
#pragma unroll
  for (int h = 0; h < 4; ++h)
    v[h] = __builtin_bit_cast(int, __builtin_elementwise_sub_sat(__builtin_bit_cast(ushort2v, (int)v[h]), by));
  return v;
}
// Powers of two that a core's A is multiplied by where it is read: a number per row and
// 2^log stages.
template <int ROWS>
struct Shifts {
  const u16* table;   // [stages from `first` on, >> log][ROWS] in LDS
  int first, log;
  __device__ __forceinline__ uint32_t at(int stage, int row) const { return table[((stage >> log) - first) * ROWS + row]; }
};

// C = A B, BM x BN (BN 256) by WM x WN waves, NS stages, issued as in NtCore (8 bits,
// 2048 x 4096 x 4096 on 128 x 256: 36.8 -> 34.4 us).
template <class E, int BM, int BN, int WM, int WN, int NS>
struct NnCore {
  static constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN, FA = TN / 16, FB = TM / 16;
  static constexpr int CX = BM / 8 / NW, CB = BN * 128 / 1024 / NW, CS = E::SCALED ? 1 : 0, C = CX + CB + CS;
  static constexpr int SOFF = (BM + BN) * 128, STAGE = SOFF + CS * NW * 256, SMEM = NS * STAGE;
  static_assert(TM == 64 && BN % 128 == 0 && TN % 16 == 0 && 128 % TN == 0 && NS * C < 64, "tile");
  typedef floatx4 Acc[FA][FB];
  static __device__ __forceinline__ int row0(int wave) { return wave / WN * TM; }
  static __device__ __forceinline__ int col(int wave, int a) { return wave % WN * TN + 16 * a; }

  // stages [s0, s1) of the contraction
  template <bool SHIFT = false>
  static __device__ __forceinline__ void run(const NnTile& t, const Scales& sc, int m0, int s0, int s1, char* smem,
                                             Acc& acc, const Shifts<BM>& shifts = {}) {
    using P = Panel<E>;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int wm = wave / WN, wn = wave % WN, g = lane >> 4, c16 = lane & 15, l8 = lane >> 3;
#pragma unroll
    for (int a = 0; a < FA; ++a)
#pragma unroll
      for (int b = 0; b < FB; ++b) acc[a][b] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (s1 <= s0) return;
    const int crow = 8 * wave;
    const uint32_t kcol = (uint32_t)(((lane & 7) ^ kc_swz(crow + l8)) << 4);
    uint32_t aoff[CX], boff[CB], soff = kOOB;
#pragma unroll
    for (int i = 0; i < CX; ++i) aoff[i] = (uint32_t)(crow + l8 + 8 * NW * i) * t.a_row + kcol;
#pragma unroll
    for (int i = 0; i < CB; ++i) {
      const int q = wave + NW * i, p = q >> 4, row = (q & 15) * P::RPC + lane / P::CHUNKS;   // 16 copies a panel
      boff[i] = (uint32_t)row * t.b_row + (uint32_t)(p * P::ROW + 16 * (lane % P::CHUNKS ^ P::swz(row)));
    }
    __amdgpu_buffer_rsrc_t rsS = t.a;
    BScales<1> bs;
    const int bcol = wn * TN / 128;
    const uint32_t sstep = E::SCALED ? (uint32_t)sc.cells * 64 : 0;
    if constexpr (E::SCALED) {
      rsS = make_rsrc(sc.a, (uint64_t)sstep * t.stages);
      soff = scale_words(sc, m0 / 64 + wm, 1, lane);
      bs.load(sc, bcol, s0, t.stages, lane);
    }
    const uint32_t last = (uint32_t)(s1 - 1) * 128, slast = (uint32_t)(s1 - 1) * sstep;
    uint32_t at = (uint32_t)s0 * 128, sat = (uint32_t)s0 * sstep;   // of the next stage to copy
    NnRows rows;
    rows.start(t, s0, E::KS);
    __amdgpu_buffer_rsrc_t rs = t.a;   // B's rows of the stage being copied
    auto copy_one = [&](auto place, auto qc) LORA_INLINE {   // as in NtCore
      constexpr int Q = decltype(qc)::value;
      char* sb = smem + decltype(place)::value * STAGE;
      if constexpr (Q == 0) rs = rows.rows();
      if constexpr (Q < CX) {
        dma16(t.a, aoff[Q], at, sb + (crow + 8 * NW * Q) * 128);
      } else if constexpr (Q < CX + CB) {
        dma16(rs, boff[Q - CX], 0, sb + BM * 128 + (wave + NW * (Q - CX)) * 1024);
      } else {
        dma4(rsS, soff, sat, sb + SOFF + wave * 256);
        sat = min(sat + sstep, slast);
      }
      if constexpr (Q == C - 1) {
        at = min(at + 128, last);
        rows.next();
      }
    };
    auto copy = [&](auto place) LORA_INLINE { each_of<C>([&](auto q) LORA_INLINE { copy_one(place, q); }); };
    uint32_t wa[FA];
#pragma unroll
    for (int a = 0; a < FA; ++a) {
      const int f = (wn * TN + 16 * a) / 16;
      wa[a] = lds_addr(smem + BM * 128 + (f >> 3) * 16384) + P::read_at(f & 7, lane);
    }
    Frag fb[2][FB];              // of this stage and the next
    int2w w[2][FA][4];
    int sa[2] = {}, sw[2] = {};
    uint32_t down[2][FB];
    static_assert(FA == 4, "the wait's operands");
    const uint32_t f0 = kc_offset(c16, g), f1 = f0 ^ 64;
    const char *b0 = smem + wm * TM * 128 + f0, *b1 = smem + wm * TM * 128 + f1;
    auto read_scales = [&](int kb, auto place, auto set) LORA_INLINE {
      constexpr int S = decltype(set)::value, O = decltype(place)::value * STAGE;
      if constexpr (E::SCALED) {
        sa[S] = bs.at(kb, 0);
        sw[S] = *reinterpret_cast<const int*>(smem + O + SOFF + wave * 256 + c16 * 4);
      }
      if constexpr (SHIFT)
#pragma unroll
        for (int b = 0; b < FB; ++b) down[S][b] = shifts.at(min(kb, s1 - 1), wm * TM + 16 * b + c16);
    };
    auto read_one = [&](auto place, auto set, auto qc) LORA_INLINE {   // fragment q of the FB + FA
      constexpr int S = decltype(set)::value, O = decltype(place)::value * STAGE, Q = decltype(qc)::value;
      if constexpr (Q < FB) {
        fb[S][Q] = Frag{*reinterpret_cast<const int4v*>(b0 + O + 2048 * Q), *reinterpret_cast<const int4v*>(b1 + O + 2048 * Q)};
      } else {
        const uint32_t from = wa[Q - FB] + (uint32_t)O;
        read_tr_asm<E, 0>(w[S][Q - FB][0], from);
        read_tr_asm<E, 1024>(w[S][Q - FB][1], from);
        read_tr_asm<E, 8192>(w[S][Q - FB][2], from);
        read_tr_asm<E, 9216>(w[S][Q - FB][3], from);
      }
    };
    auto arrived = [&](auto set) LORA_INLINE {   // (before any branch)
      constexpr int S = decltype(set)::value;
      asm volatile("s_waitcnt lgkmcnt(0)"
                   : "+v"(w[S][0][0]), "+v"(w[S][0][1]), "+v"(w[S][0][2]), "+v"(w[S][0][3]), "+v"(w[S][1][0]),
                     "+v"(w[S][1][1]), "+v"(w[S][1][2]), "+v"(w[S][1][3]), "+v"(w[S][2][0]), "+v"(w[S][2][1]),
                     "+v"(w[S][2][2]), "+v"(w[S][2][3]), "+v"(w[S][3][0]), "+v"(w[S][3][1]), "+v"(w[S][3][2]),
                     "+v"(w[S][3][3]));
      __builtin_amdgcn_sched_barrier(0);
    };
    auto multiply = [&](auto set, auto&& issue) LORA_INLINE {
      constexpr int S = decltype(set)::value;
      each_of<FB>([&](auto bc) LORA_INLINE {
        constexpr int B = decltype(bc)::value;
        if constexpr (SHIFT) fb[S][B] = Frag{scaled_down(fb[S][B].lo, down[S][B]), scaled_down(fb[S][B].hi, down[S][B])};
#pragma unroll
        for (int a = 0; a < FA; ++a) {
          Frag f;
          f.lo = int4v{w[S][a][0].x, w[S][a][0].y, w[S][a][1].x, w[S][a][1].y};
          f.hi = int4v{w[S][a][2].x, w[S][a][2].y, w[S][a][3].x, w[S][a][3].y};
          acc[a][B] = stage_product<E, B & 3>(f, fb[S][B], acc[a][B], sa[S], sw[S]);
        }
        __builtin_amdgcn_sched_barrier(0);
        issue(bc);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    using I0 = std::integral_constant<int, 0>;
    each_of<NS>([&](auto j) LORA_INLINE { copy(j); });
    copy_barrier<(NS - 1) * C>();
    read_scales(s0, I0{}, I0{});
    each_of<FA + FB>([&](auto q) LORA_INLINE { read_one(I0{}, I0{}, q); });
    arrived(I0{});
    constexpr int U = NS % 2 ? 2 * NS : NS;
    for (int k0 = s0; k0 < s1; k0 += U) {
      if constexpr (E::SCALED)
        if (k0 + U - bs.base >= bs.SPAN) bs.load(sc, bcol, k0, t.stages, lane);
      each_of<U>([&](auto jc) LORA_INLINE {   // as in NtCore
        constexpr int J = decltype(jc)::value;
        using Next = std::integral_constant<int, (J + 1) & 1>;
        if (J == 0 || k0 + J < s1) {
          copy_barrier<(NS - 2) * C>();
          __builtin_amdgcn_sched_barrier(0);
          multiply(std::integral_constant<int, J & 1>{}, [&](auto bc) LORA_INLINE {
            constexpr int B = decltype(bc)::value;
            using From = std::integral_constant<int, (J + 1) % NS>;
            if constexpr (B == 0) read_scales(k0 + J + 1, From{}, Next{});
            each_of<FA + FB>([&](auto q) LORA_INLINE {
              if constexpr (decltype(q)::value * FB / (FA + FB) == B) read_one(From{}, Next{}, q);
            });
            each_of<C>([&](auto q) LORA_INLINE {
              if constexpr (decltype(q)::value * FB / C == B) copy_one(std::integral_constant<int, J % NS>{}, q);
            });
          });
          arrived(Next{});
        }
      });
    }
    formed(acc);
    copy_barrier<0>();
  }
};

// ---------------------------------------------------------------------------
// The 256 x 256 tiles: eight waves in two rows of 128 x 64, two stages in LDS.  The
// wave rows take turns: waves w and w + 4 share a SIMD, and while one multiplies,
// the other reads its next fragments and issues copies; a workgroup barrier ends
// each slot, and the second row runs one slot behind.  A stage is four phases, each
// a slot of reads and a slot of products: (B half 0, A half 0), (B 1, A 0), (B 0, A
// 1), (B 1, A 1), reading A half 0, B half 1, A half 1 and the next stage's B half
// 0.  Every wave waits for its reads before the barrier that ends its read slot, so
// the quarter of a stage read in phase P is free from the read slots of phase P + 1
// on, which refill it for the stage after next.  The reads before the first slot
// are closed the same way, by a barrier of all eight waves before the second row's
// extra one.
//
// Copies of a wave in issue order: B half 0 (2), its rows' scales (S: 1 with 8 bits,
// else 0) and A half 0 (2), B half 1 (2), A half 1 (2).  A phase's read slot waits
// for the quarter read in the next phase; the newer ones may be under way.
template <int N>
using Count = std::integral_constant<int, N>;
constexpr int kBigStage = 512 * 128;   // bytes of a stage

// Runs the phases: F has read_a(kb, half), read_b(kb, Count<half>), copy_a, copy_b
// (kb, half), wait_b(Count<half>) (-1: no fragments pass through the wait) and
// products(hb, ha).
template <int S, class F>
__device__ __forceinline__ void big_phases(F& f, int stages, int wm) {
  auto slot_end = [&]() LORA_INLINE {
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto ready = [&](auto left, auto half) LORA_INLINE {
    __builtin_amdgcn_sched_barrier(0);
    f.wait_b(half);
    wait_vmcnt<decltype(left)::value>();
    slot_end();
  };
  auto multiply = [&](auto hb, auto ha) LORA_INLINE {
    f.products(hb, ha);
    __builtin_amdgcn_sched_barrier(0);
    slot_end();
  };
  using N1 = Count<-1>;
  using I0 = Count<0>;
  using I1 = Count<1>;
  auto stage = [&](int kb, auto mode) LORA_INLINE {   // 0: steady, 1: the last but one, 2: the last
    constexpr int MODE = decltype(mode)::value;
    f.read_a(kb, 0);
    if constexpr (MODE == 0) { f.copy_b(kb + 2, 0); ready(Count<12 + S>{}, N1{}); }
    else if constexpr (MODE == 1) ready(Count<10 + S>{}, N1{});
    else ready(Count<2>{}, N1{});
    multiply(I0{}, I0{});
    f.read_b(kb, I1{});
    if constexpr (MODE == 0) { f.copy_a(kb + 2, 0); ready(Count<12 + 2 * S>{}, I1{}); }
    else if constexpr (MODE == 1) ready(Count<8 + S>{}, I1{});
    else ready(I0{}, I1{});
    multiply(I1{}, I0{});
    f.read_a(kb, 1);
    if constexpr (MODE == 0) { f.copy_b(kb + 2, 1); ready(Count<12 + 2 * S>{}, N1{}); }
    else if constexpr (MODE == 1) ready(Count<6 + S>{}, N1{});
    else ready(I0{}, N1{});
    multiply(I0{}, I1{});
    if constexpr (MODE < 2) f.read_b(kb + 1, I0{});
    if constexpr (MODE == 0) { f.copy_a(kb + 2, 1); ready(Count<12 + S>{}, I0{}); }
    else if constexpr (MODE == 1) ready(Count<4>{}, I0{});
    else ready(I0{}, N1{});
    multiply(I1{}, I1{});
  };
  auto fill = [&](int kb) LORA_INLINE { f.copy_b(kb, 0); f.copy_a(kb, 0); f.copy_b(kb, 1); f.copy_a(kb, 1); };
  fill(0);
  if (stages > 1) {
    fill(1);
    wait_vmcnt<12 + S>();
  } else {
    wait_vmcnt<0>();
  }
  slot_end();
  f.read_b(0, I0{});
  __builtin_amdgcn_sched_barrier(0);
  f.wait_b(I0{});
  slot_end();                    // every wave has read the quarter that the first read slot refills
  if (wm == 1) slot_end();       // the second wave row runs one slot behind
  int kb = 0;
  for (; kb + 2 < stages; ++kb) {
    f.reload(kb);
    stage(kb, I0{});
  }
  f.reload_end(kb);
  if (stages > 1) stage(kb++, I1{});
  stage(kb, Count<2>{});
  if (wm == 0) slot_end();
}

template <class E>
struct BigBase {
  static constexpr int CS = E::SCALED ? 1 : 0;
  static constexpr int SMEM = 2 * kBigStage + CS * 2 * 8 * 256;
  typedef floatx4 Acc[4][8];
  static __device__ __forceinline__ int row0(int wave) { return (wave >> 2) * 128; }
};

template <class E, bool TAIL>
struct NtBig : BigBase<E> {
  static __device__ __forceinline__ int col(int wave, int a) { return (wave & 3) * 64 + 16 * a; }

  struct Loop {
    const NtTile& t;
    const Scales& sc;
    floatx4 (&acc)[4][8];
    char* smem;
    __amdgpu_buffer_rsrc_t rsS;
    int wm, wn, g, c16, lane, wave, bcol;
    uint32_t aoff, boff, kcol, soff;
    int arow, brow;                  // this wave's first tile row of a copy
    Frag fb[2][2], fa[4];            // B halves, the current A half
    int sw[2], sa;
    BScales<1> bs;

    __device__ __forceinline__ void reload(int kb) {
      if constexpr (E::SCALED)
        if (kb - bs.base == bs.SPAN) bs.load(sc, bcol, kb, t.stages, lane);
    }
    __device__ __forceinline__ void reload_end(int kb) {
      if constexpr (E::SCALED) bs.load(sc, bcol, kb, t.stages, lane);
    }
    __device__ __forceinline__ void copy_a(int kb, int h) {
      char* sb = smem + (kb & 1) * kBigStage + arow * 128 + h * 8192;
      if constexpr (E::SCALED)
        if (h == 0)
          dma4(rsS, soff, (uint32_t)kb * sc.cells * 64, smem + 2 * kBigStage + ((kb & 1) * 8 + wave) * 256);
      const bool ok = !TAIL || (uint32_t)kb * 128 + kcol < t.kbytes;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        dma16(t.a, ok ? aoff + (uint32_t)(64 * h + 128 * i) * t.a_row : kOOB, (uint32_t)kb * 128, sb + i * 16384);
    }
    __device__ __forceinline__ void copy_b(int kb, int h) {
      char* sb = smem + (kb & 1) * kBigStage + 256 * 128 + brow * 128 + h * 4096;
      const bool ok = !TAIL || (uint32_t)kb * 128 + kcol < t.kbytes;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        dma16(t.b, ok ? boff + (uint32_t)(32 * h + 128 * i) * t.b_row : kOOB, (uint32_t)kb * 128, sb + i * 16384);
    }
    __device__ __forceinline__ void read_a(int kb, int h) {
      const char* As = smem + (kb & 1) * kBigStage;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        fa[b].lo = __builtin_bit_cast(int4v, kc_read(As, wm * 128 + 64 * h + 16 * b + c16, g));
        fa[b].hi = __builtin_bit_cast(int4v, kc_read(As, wm * 128 + 64 * h + 16 * b + c16, 4 + g));
      }
      if constexpr (E::SCALED)
        if (h == 0) {
          const char* ss = smem + 2 * kBigStage + ((kb & 1) * 8 + wave) * 256 + c16 * 4;
          sw[0] = *reinterpret_cast<const int*>(ss);
          sw[1] = *reinterpret_cast<const int*>(ss + 64);
          sa = bs.at(kb, 0);
        }
    }
    template <int H>
    __device__ __forceinline__ void read_b(int kb, Count<H>) {
      const char* Bs = smem + (kb & 1) * kBigStage + 256 * 128;
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        fb[H][a].lo = __builtin_bit_cast(int4v, kc_read(Bs, wn * 64 + 32 * H + 16 * a + c16, g));
        fb[H][a].hi = __builtin_bit_cast(int4v, kc_read(Bs, wn * 64 + 32 * H + 16 * a + c16, 4 + g));
      }
    }
    template <int H>
    __device__ __forceinline__ void wait_b(Count<H>) { wait_lgkm0(); }
    template <int HB, int HA>
    __device__ __forceinline__ void products(Count<HB>, Count<HA>) {
      each_of<4>([&](auto bc) LORA_INLINE {
        constexpr int B = decltype(bc)::value;
#pragma unroll
        for (int a = 0; a < 2; ++a)
          acc[2 * HB + a][4 * HA + B] = stage_product<E, B>(fb[HB][a], fa[B], acc[2 * HB + a][4 * HA + B], sa, sw[HA]);
      });
    }
  };

  static __device__ __forceinline__ void run(const NtTile& t, const Scales& sc, int m0, char* smem,
                                             floatx4 (&acc)[4][8]) {
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
      for (int b = 0; b < 8; ++b) acc[a][b] = floatx4{0.f, 0.f, 0.f, 0.f};
    Loop f{t, sc, acc, smem, t.a, wave >> 2, wave & 3, lane >> 4, lane & 15, lane, wave, (wave & 3) >> 1};
    const int l8 = lane >> 3;
    f.arow = 8 * wave;
    f.brow = 64 * (wave >> 2) + 8 * (wave & 3);
    f.kcol = (uint32_t)(((lane & 7) ^ kc_swz(f.arow + l8)) << 4);
    f.aoff = (uint32_t)(f.arow + l8) * t.a_row + f.kcol;
    f.boff = (uint32_t)(f.brow + l8) * t.b_row + f.kcol;
    if constexpr (E::SCALED) {
      f.rsS = make_rsrc(sc.a, (uint64_t)sc.cells * t.stages * 64);
      f.soff = scale_words(sc, m0 / 64 + 2 * f.wm, 2, lane);
      f.bs.load(sc, f.bcol, 0, t.stages, lane);
    }
    big_phases<BigBase<E>::CS>(f, t.stages, f.wm);
    formed(acc);
  }
};

// B's panels of 128 columns are its halves: wave column wn takes columns 32 wn ..
// + 31 of both.
template <class E>
struct NnBig : BigBase<E> {
  static __device__ __forceinline__ int col(int wave, int a) { return 128 * (a >> 1) + 32 * (wave & 3) + 16 * (a & 1); }

  struct Loop {
    using P = Panel<E>;
    const NnTile& t;
    const Scales& sc;
    floatx4 (&acc)[4][8];
    char* smem;
    __amdgpu_buffer_rsrc_t rsS;
    int wm, wn, g, c16, lane, wave, s0;   // s0: the first stage of the contraction
    uint32_t aoff, boff[2], soff;
    uint32_t wa[2];
    NnRows rows;
    Frag fa[4];
    int2w w[2][2][4];                // B halves: [half][fragment][read]
    int sw[2], sa[2];
    BScales<2> bs;

    __device__ __forceinline__ void reload(int kb) {
      if constexpr (E::SCALED)
        if (s0 + kb - bs.base == bs.SPAN) bs.load(sc, 0, s0 + kb, t.stages, lane);
    }
    __device__ __forceinline__ void reload_end(int kb) {
      if constexpr (E::SCALED) bs.load(sc, 0, s0 + kb, t.stages, lane);
    }
    __device__ __forceinline__ void copy_a(int kb, int h) {
      char* sb = smem + (kb & 1) * kBigStage + wave * 1024 + h * 8192;
      if constexpr (E::SCALED)
        if (h == 0)
          dma4(rsS, soff, (uint32_t)(s0 + kb) * sc.cells * 64, smem + 2 * kBigStage + ((kb & 1) * 8 + wave) * 256);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        dma16(t.a, aoff + (uint32_t)(64 * h + 128 * i) * t.a_row, (uint32_t)(s0 + kb) * 128, sb + i * 16384);
    }
    __device__ __forceinline__ void copy_b(int kb, int h) {
      char* sb = smem + (kb & 1) * kBigStage + 256 * 128 + h * 16384 + wave * 1024;
      const __amdgpu_buffer_rsrc_t rs = rows.rows();   // (a stage's halves are copied in order, stage by stage)
#pragma unroll
      for (int i = 0; i < 2; ++i) dma16(rs, boff[i] + (uint32_t)(h * P::ROW), 0, sb + i * 8192);
      if (h == 1) rows.next();
    }
    __device__ __forceinline__ void read_a(int kb, int h) {
      const char* As = smem + (kb & 1) * kBigStage;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        fa[b].lo = __builtin_bit_cast(int4v, kc_read(As, wm * 128 + 64 * h + 16 * b + c16, g));
        fa[b].hi = __builtin_bit_cast(int4v, kc_read(As, wm * 128 + 64 * h + 16 * b + c16, 4 + g));
      }
      if constexpr (E::SCALED)
        if (h == 0) {
          const char* ss = smem + 2 * kBigStage + ((kb & 1) * 8 + wave) * 256 + c16 * 4;
          sw[0] = *reinterpret_cast<const int*>(ss);
          sw[1] = *reinterpret_cast<const int*>(ss + 64);
          sa[0] = bs.at(s0 + kb, 0);
          sa[1] = bs.at(s0 + kb, 1);
        }
    }
    template <int H>
    __device__ __forceinline__ void read_b(int kb, Count<H>) {
      const uint32_t o = (uint32_t)((kb & 1) * kBigStage);
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        read_tr_asm<E, H * 16384>(w[H][a][0], wa[a] + o);
        read_tr_asm<E, H * 16384 + 1024>(w[H][a][1], wa[a] + o);
        read_tr_asm<E, H * 16384 + 8192>(w[H][a][2], wa[a] + o);
        read_tr_asm<E, H * 16384 + 9216>(w[H][a][3], wa[a] + o);
      }
    }
    // The B fragments pass through the wait, so that their products stay behind it.
    template <int H>
    __device__ __forceinline__ void wait_b(Count<H>) {
      if constexpr (H >= 0)
        asm volatile("s_waitcnt lgkmcnt(0)"
                     : "+v"(w[H][0][0]), "+v"(w[H][0][1]), "+v"(w[H][0][2]), "+v"(w[H][0][3]), "+v"(w[H][1][0]),
                       "+v"(w[H][1][1]), "+v"(w[H][1][2]), "+v"(w[H][1][3]));
      else
        wait_lgkm0();
    }
    template <int HB, int HA>
    __device__ __forceinline__ void products(Count<HB>, Count<HA>) {
      each_of<4>([&](auto bc) LORA_INLINE {
        constexpr int B = decltype(bc)::value;
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          Frag f;
          f.lo = int4v{w[HB][a][0].x, w[HB][a][0].y, w[HB][a][1].x, w[HB][a][1].y};
          f.hi = int4v{w[HB][a][2].x, w[HB][a][2].y, w[HB][a][3].x, w[HB][a][3].y};
          acc[2 * HB + a][4 * HA + B] = stage_product<E, B>(f, fa[B], acc[2 * HB + a][4 * HA + B], sa[HB], sw[HA]);
        }
      });
    }
  };

  // stages [s0, s1)
  static __device__ __forceinline__ void run(const NnTile& t, const Scales& sc, int m0, int s0, int s1, char* smem,
                                             floatx4 (&acc)[4][8]) {
    using P = Panel<E>;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
      for (int b = 0; b < 8; ++b) acc[a][b] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (s1 <= s0) return;
    Loop f{t, sc, acc, smem, t.a, wave >> 2, wave & 3, lane >> 4, lane & 15, lane, wave, s0};
    const int ar = 8 * wave + (lane >> 3), br = P::RPC * wave + lane / P::CHUNKS;
    f.aoff = (uint32_t)ar * t.a_row + (uint32_t)(((lane & 7) ^ kc_swz(ar)) << 4);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      f.boff[i] = (uint32_t)(br + 8 * P::RPC * i) * t.b_row + (uint32_t)((lane % P::CHUNKS ^ P::swz(br)) << 4);
    f.rows.start(t, s0, E::KS);
#pragma unroll
    for (int a = 0; a < 2; ++a) f.wa[a] = lds_addr(smem + 256 * 128) + P::read_at(2 * f.wn + a, lane);
    if constexpr (E::SCALED) {
      f.rsS = make_rsrc(sc.a, (uint64_t)sc.cells * t.stages * 64);
      f.soff = scale_words(sc, m0 / 64 + 2 * f.wm, 2, lane);
      f.bs.load(sc, 0, s0, t.stages, lane);
    }
    big_phases<BigBase<E>::CS>(f, s1 - s0, f.wm);
    formed(acc);
  }
};

// ---------------------------------------------------------------------------
// A tile as bf16 rows in LDS (BM x BN x 2 bytes), 16-byte chunks swizzled by the row,
// so that it leaves in whole row pieces.
template <int BN>
__device__ __forceinline__ uint32_t tile_at(int row, int chunk) {
  return (uint32_t)(row * (BN * 2) + ((chunk ^ (row & (BN / 8 - 1))) << 4));
}
template <class Core, int BN>
__device__ __forceinline__ void tile_to_lds(const typename Core::Acc& acc, char* smem) {
  constexpr int FA = std::extent_v<typename Core::Acc, 0>, FB = std::extent_v<typename Core::Acc, 1>;
  const int lane = lane_fresh(), wave = uniform((int)threadIdx.x >> 6), g = lane >> 4, c16 = lane & 15;
#pragma unroll
  for (int b = 0; b < FB; ++b)
#pragma unroll
    for (int a = 0; a < FA; ++a) {
      const int row = Core::row0(wave) + 16 * b + c16, col = Core::col(wave, a) + 4 * g;
      *reinterpret_cast<uint2*>(smem + tile_at<BN>(row, col >> 3) + (col & 7) * 2) = bf16x4(acc[a][b]);
    }
}
// Rows >= nrows and columns >= ncols (a multiple of 8) are not written.
template <int BM, int BN, int NT>
__device__ __forceinline__ void lds_to_rows(const char* smem, u16* dst, size_t ld, int nrows, int ncols) {
  constexpr int CH = BN / 8, STEP = NT / CH;   // rows of a step
  static_assert(NT % CH == 0 && BM % STEP == 0, "whole steps");
  const int ch = (int)threadIdx.x % CH, r = (int)threadIdx.x / CH;
  if (8 * ch >= ncols) return;
#pragma unroll 8
  for (int i = 0; i < BM; i += STEP)
    if (r + i < nrows)
      *reinterpret_cast<int4v*>(dst + (size_t)(r + i) * ld + 8 * ch) = *reinterpret_cast<const int4v*>(smem + tile_at<BN>(r + i, ch));
}
// The tile of a core that has run, stored from its LDS.
template <class Core, int BM, int BN, int NT>
__device__ __forceinline__ void store_tile(const typename Core::Acc& acc, char* smem, u16* dst, size_t ld, int nrows,
                                           int ncols) {
  static_assert(BM * BN * 2 <= Core::SMEM, "the tile fits the stages");
  __syncthreads();   // every wave is past its last reads
  tile_to_lds<Core, BN>(acc, smem);
  __syncthreads();
  lds_to_rows<BM, BN, NT>(smem, dst, ld, nrows, ncols);
}

}  // namespace lora
