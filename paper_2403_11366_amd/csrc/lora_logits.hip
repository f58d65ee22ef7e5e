// Operators on rows of logits z [rows, vocab]:
//   * log probability of each row's token, entropy, and the top alternatives of
//     softmax(z / tau);
//   * distillation from a teacher's top logits, its loss and its gradient.
//
// Both are bound by reading z (and writing its gradient) once.  Sums, maxima and
// softmax statistics are fp32.  The calls that only read take a row in units of
// 4 KiB: one wave finds a unit's maximum and its sums against that maximum, and a
// row's units are joined in their order, so a row's results do not depend on how
// many waves or workgroups share it.
//
// Exponentials are taken to base 2, of y = (z - max z) log2(e) / tau; with S =
// sum 2^y, log softmax = (z - max z) / tau - ln S (not from y: the difference of
// a row's maximum and the type's lowest value fits fp32, its multiple need not).
// The maximum is subtracted before the scale is applied, so that rows of the
// lowest value do not overflow; a row without a value above -inf subtracts 0 and
// has S = 0, and one that holds a NaN or +inf has S = NaN.
#include <algorithm>
#include <type_traits>

#include "lora_device.hpp"
#include "lora_ops.hpp"
#include "lora_plan.hpp"

namespace lora {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kNegInf = -__builtin_inff();
constexpr int kUnitChunks = 256;   // chunks of a unit: four to a lane

typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// 16-byte chunks of a row.
template <typename T>
struct Chunk;
template <>
struct Chunk<u16> {
  static constexpr int CH = 8;
  static constexpr int kFill = (int)0xFF80FF80;   // -inf in both halves
  static __device__ __forceinline__ float get(const int4v& v, int e) {
    const uint32_t w = (uint32_t)v[e >> 1];
    return __builtin_bit_cast(float, e & 1 ? w & 0xFFFF0000u : w << 16);
  }
  static __device__ __forceinline__ float one(u16 x) { return bf16_to_f32(x); }
  static __device__ __forceinline__ int4v pack(const float (&x)[8]) {
    int4v v;
#pragma unroll
    for (int h = 0; h < 4; ++h)
      v[h] = __builtin_bit_cast(int, __builtin_convertvector((f32x2_t{x[2 * h], x[2 * h + 1]}), bf16x2_t));
    return v;
  }
  static __device__ __forceinline__ u16 pack1(float x) { return f32_to_bf16(x); }
};
template <>
struct Chunk<float> {
  static constexpr int CH = 4;
  static constexpr int kFill = (int)0xFF800000;
  static __device__ __forceinline__ float get(const int4v& v, int e) {
    const int w = v[e];   // (a bit cast of the element itself takes the first one)
    return __builtin_bit_cast(float, w);
  }
  static __device__ __forceinline__ float one(float x) { return x; }
  static __device__ __forceinline__ int4v pack(const float (&x)[4]) {
    int4v v;
#pragma unroll
    for (int h = 0; h < 4; ++h) v[h] = __builtin_bit_cast(int, x[h]);
    return v;
  }
  static __device__ __forceinline__ float pack1(float x) { return x; }
};

// A row: single elements to its first 16-byte boundary, whole chunks, single
// elements after them.  The singles go to threads 0 .. head-1 and CH .. CH+tail-1.
template <typename T>
struct Row {
  static constexpr int CH = Chunk<T>::CH;
  const T* p;          // the row
  int head, chunks;    // single elements before the first chunk, whole chunks
  int tail0;           // the first element after the chunks

  __device__ __forceinline__ Row(const T* row, int vocab) : p(row) {
    const int off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    head = min(off ? CH - off : 0, vocab);
    chunks = (vocab - head) / CH;
    tail0 = head + chunks * CH;
  }
  __device__ __forceinline__ int units() const { return (chunks + kUnitChunks - 1) / kUnitChunks; }
  __device__ __forceinline__ int4v at(int c) const {
    return *reinterpret_cast<const int4v*>(p + head + (size_t)c * CH);
  }
  // this thread's single element, -1: none
  __device__ __forceinline__ int edge(int vocab) const {
    const int tid = threadIdx.x;
    return tid < head ? tid : (tid >= CH && tid - CH < vocab - tail0 ? tail0 + tid - CH : -1);
  }
  // as stored: nothing waits for the load before the value is formed
  __device__ __forceinline__ T raw(int index) const { return index >= 0 ? p[index] : Chunk<T>::pack1(kNegInf); }
  __device__ __forceinline__ float value(int index) const { return index >= 0 ? Chunk<T>::one(p[index]) : kNegInf; }
  static __device__ __forceinline__ int4v fill() {
    return int4v{Chunk<T>::kFill, Chunk<T>::kFill, Chunk<T>::kFill, Chunk<T>::kFill};
  }
};

// A chunk of the gradient: whole where its row lies like the logits' in 16 bytes,
// else value by value.
template <typename T>
__device__ __forceinline__ void put(T* p, const float (&x)[Chunk<T>::CH], bool whole) {
  if (whole) {
    *reinterpret_cast<int4v*>(p) = Chunk<T>::pack(x);
  } else {
#pragma unroll
    for (int e = 0; e < Chunk<T>::CH; ++e) p[e] = Chunk<T>::pack1(x[e]);
  }
}
template <typename T>
__device__ __forceinline__ bool lies_alike(const T* a, const T* b) {
  return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15) == 0;
}

// Over a wave, uniform: lane 15 of each row of 16 collects its row by shifts, then
// lane 63 the four rows (six steps in the vector unit, none through LDS).
template <typename F>
__device__ __forceinline__ float wave_reduce(float x, float none, F&& f) {
  auto step = [&](auto ctrl, auto rows) LORA_INLINE {
    const int y = __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, x),
                                              decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
    x = f(x, __builtin_bit_cast(float, y));
  };
  using std::integral_constant;
  constexpr integral_constant<int, 0xf> all{};
  step(integral_constant<int, 0x111>{}, all);   // row_shr 1, 2, 4, 8
  step(integral_constant<int, 0x112>{}, all);
  step(integral_constant<int, 0x114>{}, all);
  step(integral_constant<int, 0x118>{}, all);
  step(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});   // lane 15 to the next row
  step(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});   // lane 31 to rows 2 and 3
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ __forceinline__ float wave_max(float x) {
  return wave_reduce(x, kNegInf, [](float a, float b) LORA_INLINE { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_sum(float x) {
  return wave_reduce(x, 0.f, [](float a, float b) LORA_INLINE { return a + b; });
}

// Maximum (NaN left out) and sums over the workgroup, the same on every thread;
// `box` holds NT / 64 floats per value.  Each call takes a box of its own.
template <int NT>
__device__ __forceinline__ float block_max(float x, float* box) {
  x = wave_max(x);
  if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = x;
  __syncthreads();
  return wave_max((threadIdx.x & 63) < NT / 64 ? box[threadIdx.x & 63] : kNegInf);
}
template <int NT>
__device__ __forceinline__ float2 block_sum2(float a, float b, float2* box) {
  a = wave_sum(a);
  b = wave_sum(b);
  if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = float2{a, b};
  __syncthreads();
  const float2 r = (threadIdx.x & 63) < NT / 64 ? box[threadIdx.x & 63] : float2{0.f, 0.f};
  return float2{wave_sum(r.x), wave_sum(r.y)};
}

__device__ __forceinline__ float exp2_hw(float y) { return __builtin_amdgcn_exp2f(y); }

// What is subtracted for a row's maximum: 0 where no value is above -inf.
__device__ __forceinline__ float shift_of(float m) { return m == kNegInf ? 0.f : m; }

// ---------------------------------------------------------------------------
// Units of a row.  `Term` forms a value's exponential and a second sum:
// Term::add(d, s, a) with d = z - shift, and Term::moved(d, s, a) moves both sums
// to a shift that is larger by -d.
// The units first .. last-1 of a row, unit u to box[u - first]; `wave` of `waves`.
// seen(i, m): the lane's own maximum of its i-th unit.
template <typename T, typename Term, typename Seen>
__device__ __forceinline__ void row_units(const Row<T>& row, int first, int last, int wave, int waves, const Term& term,
                                          Unit* box, Seen&& seen) {
  constexpr int CH = Chunk<T>::CH, U = kUnitChunks / 64;
  const int lane = threadIdx.x & 63;
  for (int u = first + wave, it = 0; u < last; u += waves, ++it) {
    int4v v[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int c = u * kUnitChunks + i * 64 + lane;
      v[i] = c < row.chunks ? row.at(c) : Row<T>::fill();
    }
    float m = kNegInf;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int e = 0; e < CH; ++e) m = fmaxf(m, Chunk<T>::get(v[i], e));
    seen(it, m);
    m = wave_max(m);
    const float shift = shift_of(m);
    float s = 0.f, a = 0.f;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int e = 0; e < CH; ++e) term.add(Chunk<T>::get(v[i], e) - shift, s, a);
    s = wave_sum(s);
    a = wave_sum(a);
    if (lane == 0) box[u - first] = Unit{m, s, a};
  }
}

// The row's single elements as a unit, by the first wave.
template <typename Term>
__device__ __forceinline__ void edge_unit(float x, const Term& term, Unit* box) {
  const float m = wave_max(x);
  float s = 0.f, a = 0.f;
  term.add(x - shift_of(m), s, a);
  s = wave_sum(s);
  a = wave_sum(a);
  if ((threadIdx.x & 63) == 0) *box = Unit{m, s, a};
}

// n units as one, uniform, by each wave that asks.
template <typename Term>
__device__ __forceinline__ Unit join_units(const Unit* box, int n, const Term& term) {
  const int lane = threadIdx.x & 63;
  float m = kNegInf;
  for (int i = lane; i < n; i += 64) m = fmaxf(m, box[i].m);
  m = wave_max(m);
  const float shift = shift_of(m);
  float s = 0.f, a = 0.f;
  for (int i = lane; i < n; i += 64) {
    Unit u = box[i];
    term.moved(u.m - shift, u.s, u.a);
    s += u.s;
    a += u.a;
  }
  return Unit{m, wave_sum(s), wave_sum(a)};
}

// ---------------------------------------------------------------------------
// Log probabilities, entropy (second sum: 2^y y) and the top alternatives.
//
// The top values are found without sorting or a second pass: the top-th largest
// of the threads' own maxima is at most the top-th largest value, so only the
// few threads whose maximum reaches it (the owners) hold values to look at.  A
// lower bound of it comes from one wave's bisection over maxima of groups of threads.  The
// owners' chunks are read again, four lanes an owner; the values at or above
// the bound go into an LDS list and are ranked against each other by value and
// index.  Where more values tie than the list holds (a constant row, or one with
// fewer than `top` values above -inf, where -inf ties), the exact top-th value is
// found by counting over the row, four bits a pass, and its lowest columns by
// counting on from the row's start: 6 passes over a bf16 row and 10 over an fp32
// one, an element a load.
//
// Few rows of many units are split over workgroups: each leaves its units and
// its own top values in the workspace, and a second launch joins them.
//
// Bound by HBM, and by the selection's latency at a row's end where few other rows
// cover it: 4096 x 32000 bf16 55 us (4.7 TB/s) without alternatives, 60 with 20;
// 777 x 50021 fp32 33 and, with 64, 41; one row of 32000 4.0 and, with 20, 7.4;
// one of 131072 fp32 with 20, split, 7.6 and 4.6 to join (17 in one workgroup).
// Reading all chunks of an owning thread again, instead of one unit's, fetched
// more lines than the row has (777 x 50021: 52).  By counting, with ten columns
// above -inf: 4096 x 32000 837 us, 777 x 50021 755, one row of 32000 89, one of
// 131072 fp32 110 and 5; constant rows take as long.

struct EntropyTerm {
  float scale;   // log2(e) / tau
  __device__ __forceinline__ void add(float d, float& s, float& a) const {
    const float y = d * scale, e = exp2_hw(y);
    s += e;
    a = fmaf(e, fmaxf(y, -1e4f), a);   // (0 for e = 0 at y = -inf)
  }
  __device__ __forceinline__ void moved(float d, float& s, float& a) const {
    const float y = fmaxf(d * scale, -1e4f), f = exp2_hw(y);
    a = f * fmaf(y, s, a);
    s *= f;
  }
};

// Whole numbers in the order of the values; -0 as 0 and NaN as -inf.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x != x ? kNegInf : x + 0.f);
  return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
// The value of an order (a NaN's: -inf).
__device__ __forceinline__ float value_of(uint32_t o) {
  return __builtin_bit_cast(float, o ^ (o >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}
constexpr int kCandidates = 512;
constexpr int kOwners = 512;
constexpr int kSeen = 8;        // places of a thread for the maxima of its units

template <int NT>
struct TopShared {
  uint32_t maxima[NT];          // the threads' maxima in order_of form, 0: no value
  uint64_t cand[kCandidates];   // order above ~index: larger is earlier
  uint16_t seen[kSeen * NT];    // their upper halves, unit by unit (wide rows: 2^by units a place)
  int owner[kOwners];           // places of `seen` that reach the bound
  uint32_t bound;
  int count, owners;
  int part[2][16][NT / 64];
};

// A bound that at least `top` of 64 x G groups' maxima reach and not many more
// (0: fewer groups hold a value).  One wave; bisection over the maxima's range,
// ten times and on while over twice as many reach it.  A lane has its own groups:
// its places in every wave (of every fourth wave).
template <int G, int NT>
__device__ __forceinline__ uint32_t top_bound(const uint32_t* maxima, int top) {
  uint32_t o[G], hi = 0, lo = 0xFFFFFFFFu;
  int reach = 0;
#pragma unroll
  for (int q = 0; q < G; ++q) {
    o[q] = 0;
#pragma unroll
    for (int j = q; j < NT / 64; j += G) o[q] = max(o[q], maxima[(threadIdx.x & 63) + 64 * j]);
    hi = max(hi, o[q]);
    lo = min(lo, o[q] ? o[q] : 0xFFFFFFFFu);
    reach += __popcll(__ballot(o[q] != 0));
  }
  if (reach < top) return 0;
#pragma unroll
  for (int q = 32; q > 0; q >>= 1) {
    hi = max(hi, (uint32_t)__shfl_xor((int)hi, q));
    lo = min(lo, (uint32_t)__shfl_xor((int)lo, q));
  }
  for (int it = 0; (it < 10 || reach > 2 * top + 16) && lo < hi; ++it) {
    const uint32_t mid = lo + (hi - lo) / 2 + 1;
    int n = 0;
#pragma unroll
    for (int q = 0; q < G; ++q) n += __popcll(__ballot(o[q] >= mid));
    if (n >= top) {
      lo = mid;
      reach = n;
    } else {
      hi = mid - 1;
    }
  }
  return lo;
}
// (64 groups hold about 1.4 top values at or above the bound for a top of half as many)
template <int NT>
__device__ __forceinline__ uint32_t top_bound(const uint32_t* maxima, int top) {
  const uint32_t t = top <= 32 ? top_bound<1, NT>(maxima, top) : 0u;
  return t ? t : top_bound<4, NT>(maxima, top);
}

template <int NT>
__device__ __forceinline__ void push(TopShared<NT>& sh, uint32_t order, int index) {
  const int at = atomicAdd(&sh.count, 1);
  if (at < kCandidates) sh.cand[at] = (uint64_t)order << 32 | (uint32_t)~index;
}

// N counts over the workgroup, the same on every thread; calls alternate between
// two boxes (`turn`).
template <int NT, int N>
__device__ __forceinline__ void block_counts(int (&n)[N], int (*part)[16][NT / 64], int& turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
#pragma unroll
    for (int q = 32; q > 0; q >>= 1) n[i] += __shfl_xor(n[i], q);
    if ((threadIdx.x & 63) == 0) part[turn][i][threadIdx.x >> 6] = n[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    n[i] = 0;
    for (int w = 0; w < NT / 64; ++w) n[i] += part[turn][i][w];
  }
  turn ^= 1;
}

// The candidates where the list does not hold all values at or above the bound.
// (columns col0 .. col1-1)
template <typename T, int NT>
__device__ __forceinline__ void select_by_counting(const T* p, int col0, int col1, int top, TopShared<NT>& sh) {
  const int tid = threadIdx.x;
  int turn = 0;
  uint32_t kth = 0;          // the top-th largest value's order
  // (a bf16 value's lower 16 bits are all its sign's)
  for (int bit = 28; bit >= (sizeof(T) == 2 ? 16 : 0); bit -= 4) {
    int n[15];
#pragma unroll
    for (int j = 0; j < 15; ++j) n[j] = 0;
    for (int i = col0 + tid; i < col1; i += NT) {
      const uint32_t o = order_of(Chunk<T>::one(p[i]));
#pragma unroll
      for (int j = 0; j < 15; ++j) n[j] += o >= (kth | (uint32_t)(j + 1) << bit);
    }
    block_counts<NT, 15>(n, sh.part, turn);
    uint32_t digit = 0;
#pragma unroll
    for (int j = 0; j < 15; ++j) digit += n[j] >= top;
    kth |= digit << bit;
  }
  if (sizeof(T) == 2 && !(kth >> 31)) kth |= 0xFFFFu;
  if (tid == 0) sh.count = 0;
  int above[1] = {0};
  for (int i = col0 + tid; i < col1; i += NT) above[0] += order_of(Chunk<T>::one(p[i])) > kth;
  block_counts<NT, 1>(above, sh.part, turn);   // (its barrier also publishes count = 0)
  for (int i = col0 + tid; i < col1; i += NT) {
    const uint32_t o = order_of(Chunk<T>::one(p[i]));
    if (o > kth) push<NT>(sh, o, i);
  }
  // the first top - above ties: blocks of NT columns from the first
  int need = top - above[0];
  for (int i0 = col0; need > 0 && i0 < col1; i0 += NT) {
    const int i = i0 + tid;
    const bool tie = i < col1 && order_of(Chunk<T>::one(p[i])) == kth;
    const uint64_t lanes = __ballot(tie);
    if ((tid & 63) == 0) sh.part[turn][0][tid >> 6] = __popcll(lanes);
    __syncthreads();
    int before = __popcll(lanes & ((1ull << (tid & 63)) - 1)), all = 0;
    for (int w = 0; w < NT / 64; ++w) {
      before += w < (tid >> 6) ? sh.part[turn][0][w] : 0;
      all += sh.part[turn][0][w];
    }
    if (tie && before < need) push<NT>(sh, kth, i);
    need -= all;
    turn ^= 1;
  }
  __syncthreads();
}

// The values at or above sh.bound of units first .. last-1 and of the single
// elements given (`edge` -1: none), among columns col0 .. col1-1, in sh.cand; at
// least `top`.  After the barrier that publishes sh.bound, sh.count = 0 and
// sh.owners = 0.
template <typename T, int NT>
__device__ __forceinline__ void select_top(const Row<T>& row, int first, int last, int by, int col0, int col1, int edge,
                                           int top, TopShared<NT>& sh) {
  constexpr int CH = Chunk<T>::CH, kWaves = NT / 64, U = kUnitChunks / 64;
  const int tid = threadIdx.x;
  const uint32_t bound = sh.bound;
  for (int i = 0; i < kSeen && (first + (i << by) * kWaves + (tid >> 6)) < last; ++i)
    if (sh.seen[i * NT + tid] >= bound >> 16) {
      const int at = atomicAdd(&sh.owners, 1);
      if (at < kOwners) sh.owner[at] = i * NT + tid;
    }
  if (edge >= 0) {
    const uint32_t o = order_of(row.value(edge));
    if (o >= bound) push<NT>(sh, o, edge);
  }
  __syncthreads();
  const int owners = sh.owners;
  // (a NaN passes the comparison, and ranks with -inf)
  const float least = bound ? value_of(bound) : kNegInf;
  if (owners <= kOwners)
    for (int q = tid / U; q < owners; q += NT / U) {
      const int place = sh.owner[q], t = place % NT;
      for (int k = 0; k < 1 << by; ++k) {
        const int u = first + ((place / NT << by) + k) * kWaves + (t >> 6);
        const int c = u * kUnitChunks + (t & 63) + tid % U * 64;
        if (u >= last || c >= row.chunks) break;
        const int4v v = row.at(c);
        uint32_t in = 0;
#pragma unroll
        for (int e = 0; e < CH; ++e) in |= !(Chunk<T>::get(v, e) < least) ? 1u << e : 0u;
        for (; in; in &= in - 1) {
          const int e = __builtin_ctz(in), h = e / (CH / 4);
          int4v x;
          x[0] = h < 2 ? (h == 0 ? v[0] : v[1]) : (h == 2 ? v[2] : v[3]);
          push<NT>(sh, order_of(CH == 4 || !(e & 1) ? Chunk<T>::get(x, 0) : Chunk<T>::get(x, 1)), row.head + c * CH + e);
        }
      }
    }
  __syncthreads();
  if (owners > kOwners || sh.count > kCandidates) {   // (uniform)
    __syncthreads();                                  // everyone has read sh.count
    select_by_counting<T, NT>(row.p, col0, col1, top, sh);
  }
}

// What a row's results are formed from.
struct ScoreRow {
  float shift, itau, lns;
  bool empty;
  __device__ __forceinline__ ScoreRow(const Unit& u, float itau_)
      : shift(shift_of(u.m)), itau(itau_), lns(logf(u.s)), empty(u.s == 0.f) {}
  __device__ __forceinline__ float logp(float x) const { return empty ? kNegInf : (x - shift) * itau - lns; }
};

// Log probability of the token and entropy, by one thread.
template <typename T>
__device__ __forceinline__ void put_scores(const Row<T>& row, const ScoreRow& sc, const Unit& u, const int32_t* tokens,
                                           int64_t r, float* logp, float* entropy, int vocab) {
  entropy[r] = sc.empty ? 0.f : sc.lns - u.a / u.s * kLn2;
  if (tokens) {
    const int token = tokens[r];
    logp[r] = (uint32_t)token >= (uint32_t)vocab ? 0.f : sc.logp(row.value(token));
  }
}

// Place of a key (order above ~index) among n.
__device__ __forceinline__ int rank_of(uint64_t mine, const uint64_t* keys, int n) {
  int rank = 0;
  for (int j = 0; j < n; ++j) rank += keys[j] > mine;
  return rank;
}

// One workgroup to a row, or to one of its `parts` (the row's results are then
// the second launch's).
template <typename T, int NT, bool SPLIT>
__global__ __launch_bounds__(NT) void lora_logprobs_kernel(const T* __restrict__ logits, int64_t ld,
                                                           const int32_t* __restrict__ tokens, float itau,
                                                           float* __restrict__ logp, float* __restrict__ entropy,
                                                           int32_t* __restrict__ top_ids, float* __restrict__ top_logp,
                                                           int vocab, int top, int parts, ScoreParts ws) {
  __shared__ TopShared<NT> sh;
  __shared__ Unit box[SPLIT ? 1 : (NT == 256 ? kSmallUnits : kMaxUnits)];
  const int64_t r = SPLIT ? blockIdx.x / (unsigned)parts : blockIdx.x;
  const int part = SPLIT ? (int)(blockIdx.x - (unsigned)r * (unsigned)parts) : 0;
  const int tid = threadIdx.x;
  const Row<T> row(logits + r * ld, vocab);
  const int units = row.units();
  const int first = SPLIT ? (int)((int64_t)units * part / parts) : 0;
  const int last = SPLIT ? (int)((int64_t)units * (part + 1) / parts) : units;
  const EntropyTerm term{kLog2e * itau};
  int edge = row.edge(vocab);
  const float xe = row.value(edge);
  Unit* out = SPLIT ? ws.units + r * ws.units_ld : box;
  int by = 0;
  while ((last - first - 1) / (NT / 64) >> by >= kSeen) ++by;
  float own = kNegInf, place = kNegInf;
  row_units(row, first, last, uniform(tid >> 6), NT / 64, term, out + first, [&](int i, float m) LORA_INLINE {
    if (top == 0) return;
    own = fmaxf(own, m);
    place = (i & ((1 << by) - 1)) == 0 ? m : fmaxf(place, m);
    sh.seen[(i >> by) * NT + tid] = (uint16_t)(order_of(place) >> 16);
  });
  if (part == 0 && tid < 64) edge_unit(xe, term, out + units);
  if (top > 0) {   // 0 for the threads without a chunk
    sh.maxima[tid] = (first + (tid >> 6)) * kUnitChunks + (tid & 63) < min(row.chunks, last * kUnitChunks) ? order_of(own) : 0u;
    if (tid == 0) sh.count = sh.owners = 0;
  }
  __syncthreads();
  if (top > 0 && tid < 64) {
    const uint32_t t = top_bound<NT>(sh.maxima, top);
    if (tid == 0) sh.bound = t;
  }
  if constexpr (SPLIT) {
    if (top == 0) return;
    const int col0 = part == 0 ? 0 : row.head + first * kUnitChunks * Chunk<T>::CH;
    const int col1 = part == parts - 1 ? vocab : row.head + last * kUnitChunks * Chunk<T>::CH;
    if (edge < col0 || edge >= col1) edge = -1;
    __syncthreads();
    select_top<T, NT>(row, first, last, by, col0, col1, edge, top, sh);
    const int n = sh.count;
    uint64_t* keys = ws.keys + (r * parts + part) * top;
    for (int c = tid; c < n; c += NT) {
      const int rank = rank_of(sh.cand[c], sh.cand, n);
      if (rank < top) keys[rank] = sh.cand[c];
    }
  } else {
    const Unit u = join_units(box, units + 1, term);
    const ScoreRow sc(u, itau);
    if (tid == 0) put_scores(row, sc, u, tokens, r, logp, entropy, vocab);
    if (top == 0) return;
    __syncthreads();
    select_top<T, NT>(row, 0, units, by, 0, vocab, edge, top, sh);
    const int n = sh.count;
    for (int c = tid; c < n; c += NT) {
      const uint64_t mine = sh.cand[c];
      const int rank = rank_of(mine, sh.cand, n);
      if (rank < top) {
        top_ids[r * top + rank] = (int)~(uint32_t)mine;
        top_logp[r * top + rank] = sc.logp(value_of((uint32_t)(mine >> 32)));
      }
    }
  }
}

// The rows of a split call from their parts.
template <typename T>
__global__ __launch_bounds__(kMaxKeys) void lora_logprobs_join_kernel(
    const T* __restrict__ logits, int64_t ld, const int32_t* __restrict__ tokens, float itau, float* __restrict__ logp,
    float* __restrict__ entropy, int32_t* __restrict__ top_ids, float* __restrict__ top_logp, int vocab, int top,
    int parts, ScoreParts ws) {
  __shared__ uint64_t keys[kMaxKeys];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x, n = parts * top;
  const Row<T> row(logits + r * ld, vocab);
  const EntropyTerm term{kLog2e * itau};
  const uint64_t mine = tid < n ? ws.keys[r * n + tid] : 0;
  keys[tid] = mine;
  const Unit u = join_units(ws.units + r * ws.units_ld, row.units() + 1, term);
  const ScoreRow sc(u, itau);
  if (tid == 0) put_scores(row, sc, u, tokens, r, logp, entropy, vocab);
  __syncthreads();
  if (tid < n) {
    const int rank = rank_of(mine, keys, n);
    if (rank < top) {
      top_ids[r * top + rank] = (int)~(uint32_t)mine;
      top_logp[r * top + rank] = sc.logp(value_of((uint32_t)(mine >> 32)));
    }
  }
}

// ---------------------------------------------------------------------------
// Distillation.  With the teacher's list (id_k, t_k), p = softmax(t / tau) over
// the list's entries with an id in the vocabulary, q = softmax(z / tau) and the
// label y,
//   loss = w tau^2 sum_k p_k (log p_k - log q_{id_k}) - (1 - w) log softmax(z)_y,
//   dz_j = g ( w tau (q_j sum p - sum_{k: id_k = j} p_k) + (1 - w) (softmax(z)_j - [j = y]) ).
// A row without entries has no soft term, one without a label no hard term; a
// row of logits without a value above -inf has loss and gradient 0.

// What the rows' special columns need: the teacher's list and the label as entry `top`.
struct ListShared {
  int id[kMaxTop + 1];
  float p[kMaxTop + 1];    // p_k (the label's: 0)
  float mass;              // sum of p: 1, 0 without entries
  float entropy;           // sum p ln p
};

// A row's list and label as the first wave's lanes hold them: entries lane and
// lane + 64, as loaded (nothing waits for the loads here).
struct ListIn {
  int id[2], label;
  float t[2];
};
__device__ __forceinline__ ListIn list_in(const int32_t* ids, const float* t, const int32_t* label, int top) {
  const int lane = threadIdx.x & 63;
  ListIn in;
  in.label = label ? *label : -1;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int k = lane + 64 * h;
    in.id[h] = k < top ? ids[k] : -1;
    in.t[h] = k < top ? t[k] : kNegInf;
  }
  return in;
}

// One wave forms p and leaves it in sh (before a barrier of the caller); ids
// outside the vocabulary are none (-1).
__device__ __forceinline__ void teacher_list(ListIn in, float scale, int vocab, int top, ListShared& sh) {
  const int lane = threadIdx.x & 63;
  if ((uint32_t)in.label >= (uint32_t)vocab) in.label = -1;
#pragma unroll
  for (int h = 0; h < 2; ++h)
    if ((uint32_t)in.id[h] >= (uint32_t)vocab) in.id[h] = -1;
  float y[2], e[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) y[h] = in.id[h] >= 0 ? in.t[h] : kNegInf;
  const float shift = shift_of(wave_max(fmaxf(y[0], y[1])));
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    y[h] = (y[h] - shift) * scale;
    e[h] = exp2_hw(y[h]);
  }
  const float sum = wave_sum(e[0] + e[1]);
  const float lnsum = logf(sum), inv = sum == 0.f ? 0.f : 1.f / sum;
  float plogp = 0.f;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float p = e[h] * inv;
    if (!(p == 0.f)) plogp = fmaf(p, y[h] * kLn2 - lnsum, plogp);
    if (lane + 64 * h < top) {
      sh.id[lane + 64 * h] = in.id[h];
      sh.p[lane + 64 * h] = p;
    }
  }
  plogp = wave_sum(plogp);
  if (lane == 0) {
    sh.id[top] = in.label;
    sh.p[top] = 0.f;
    sh.mass = sum == 0.f ? 0.f : sum * inv;   // NaN where the list holds one
    sh.entropy = plogp;
  }
}

// Loss of a row by one wave from the logarithms of both softmaxes' sums; x(k) is
// entry k's logit.  The soft term's sum is taken over z - max z, before the
// temperature: divided by one below 1, the type's lowest value (a banned column
// that the teacher lists) would pass fp32's range where the loss does not.
template <typename X>
__device__ __forceinline__ float row_loss(const ListShared& sh, X&& x, int top, float tau, float w, float shift,
                                          float lnsoft, float lnhard) {
  const int lane = threadIdx.x & 63;
  float cross = 0.f;       // sum p (z - max z)
  if (w > 0.f)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = lane + 64 * h;
      if (k < top && sh.id[k] >= 0) {
        const float p = sh.p[k];
        if (!(p == 0.f)) cross = fmaf(p, x(k) - shift, cross);
      }
    }
  cross = wave_sum(cross);
  // (without entries: no soft term, whatever the row's sum)
  float loss = w > 0.f && sh.mass != 0.f ? w * tau * (tau * fmaf(sh.mass, lnsoft, sh.entropy) - cross) : 0.f;
  if (w < 1.f && sh.id[top] >= 0)
    loss += (1.f - w) * (lnhard - (x(top) - shift));
  return loss;
}

// How the two softmaxes' exponentials of an element are formed from u = 2^((z -
// max z) scale): one where the temperature is 1 or a term has no weight, a power
// of u at temperatures 2 and 4, else an exponential of its own (4096 x 32000
// bf16: the step takes 99 to 101 us at temperatures 1, 2 and 4, 137 at 3).
enum Hard { HARD_SAME, HARD_SQUARE, HARD_FOURTH, HARD_OWN };
__host__ __device__ __forceinline__ Hard hard_of(float tau, float w) {
  if (tau == 1.f || w == 1.f || w == 0.f) return HARD_SAME;
  return tau == 2.f ? HARD_SQUARE : (tau == 4.f ? HARD_FOURTH : HARD_OWN);
}
// log2(e) over the temperature of u.
__device__ __forceinline__ float scale_of(float tau, float w) { return w == 0.f ? kLog2e : kLog2e / tau; }

template <int H>
__device__ __forceinline__ float hard_exp(float u, float d) {
  if constexpr (H == HARD_SAME) return u;
  if constexpr (H == HARD_SQUARE) return u * u;
  if constexpr (H == HARD_FOURTH) return (u * u) * (u * u);
  return exp2_hw(d * kLog2e);
}

template <typename F>
__host__ __device__ __forceinline__ void with_hard(Hard h, F&& f) {
  switch (h) {
    case HARD_SAME: f(std::integral_constant<int, HARD_SAME>{}); break;
    case HARD_SQUARE: f(std::integral_constant<int, HARD_SQUARE>{}); break;
    case HARD_FOURTH: f(std::integral_constant<int, HARD_FOURTH>{}); break;
    default: f(std::integral_constant<int, HARD_OWN>{}); break;
  }
}

// Gradient factors of a row: dz = fs u + fh (the hard term's exponential) away
// from the listed columns.
struct GradRow {
  float shift, scale, fs, fh;
  template <int H>
  __device__ __forceinline__ float of_exp(float u) const {
    if constexpr (H == HARD_SQUARE) return u * fmaf(fh, u, fs);
    if constexpr (H == HARD_FOURTH) return u * fmaf(fh, u * (u * u), fs);
    return fs * u;
  }
  template <int H>
  __device__ __forceinline__ float dense(float x) const {
    const float d = x - shift, u = exp2_hw(d * scale);
    if constexpr (H == HARD_OWN) return fmaf(fh, exp2_hw(d * kLog2e), fs * u);
    return of_exp<H>(u);
  }
};

// From the sums of both exponentials (an empty row: both infinite).
__device__ __forceinline__ GradRow grad_row(const ListShared& sh, int top, float g, float tau, float w, float shift,
                                            float soft, float hard) {
  const bool label = sh.id[top] >= 0;
  GradRow r{shift, scale_of(tau, w), w > 0.f ? g * w * tau * sh.mass / soft : 0.f,
            w < 1.f && label ? g * (1.f - w) / hard : 0.f};
  if (hard_of(tau, w) == HARD_SAME) r.fs += r.fh;
  return r;
}

// The teacher's probability of a column (entries with one id add up).
__device__ __forceinline__ float listed_p(const ListShared& sh, int id, int top) {
  float p = 0.f;
#pragma unroll 4
  for (int j = 0; j < top; ++j) p += sh.id[j] == id ? sh.p[j] : 0.f;
  return p;
}
// dz of a listed column whose logit is x (entries with one id all get its whole value).
template <int H>
__device__ __forceinline__ float listed_grad(const ListShared& sh, int id, float p, float x, int top, float g, float tau,
                                             float w, const GradRow& gr) {
  float d = gr.template dense<H>(x);
  if (w > 0.f) d -= g * w * tau * p;
  if (sh.id[top] == id) d -= g * (1.f - w);
  return d;
}

// The listed columns of a row, chained to the threads that store their chunks: a
// column's own gradient follows its dense one from the same thread, in its program
// order, so no barrier waits for the stores.
template <int NT>
struct ListChain {
  float x[kMaxTop + 1];         // the entries' logits
  int next[kMaxTop + 1];        // a thread's entries, -1: end
  int first[NT];
  // (thread `owner` of the workgroup stores the column; all `first` are -1 before)
  __device__ __forceinline__ void link(int k, int owner) { next[k] = atomicExch(&first[owner], k); }
  template <int H, typename T>
  __device__ __forceinline__ void put(T* dz, const ListShared& list, int top, bool empty, float g, float tau, float w,
                                      const GradRow& gr) const {
    const int k0 = first[threadIdx.x];
    for (int k = k0; k >= 0; k = next[k]) {
      const int id = list.id[k];
      float p = 0.f;      // (the sum of two is the same in either order, the list has that of more)
      int same = 0;
      for (int j = k0; j >= 0; j = next[j])
        if (list.id[j] == id) {
          p += list.p[j];
          ++same;
        }
      if (same > 2) p = listed_p(list, id, top);
      dz[id] = Chunk<T>::pack1(empty ? 0.f : listed_grad<H>(list, id, p, x[k], top, g, tau, w, gr));
    }
  }
};

// First sum: the exponential at the temperature; second: the hard term's.
template <int H>
struct DistillTerm {
  float scale;
  __device__ __forceinline__ void add(float d, float& s, float& a) const {
    const float u = exp2_hw(d * scale);
    s += u;
    if constexpr (H != HARD_SAME) a += hard_exp<H>(u, d);
  }
  __device__ __forceinline__ void moved(float d, float& s, float& a) const {
    const float u = exp2_hw(d * scale);
    s *= u;
    if constexpr (H != HARD_SAME) a *= hard_exp<H>(u, d);
  }
};

// Both sums of a row and its maximum, the same on every wave.
template <int H, int NT, typename T>
__device__ __forceinline__ Unit row_sums(const Row<T>& row, float xe, float scale, Unit* box) {
  const DistillTerm<H> term{scale};
  const int units = row.units();
  row_units(row, 0, units, uniform((int)threadIdx.x >> 6), NT / 64, term, box, [](int, float) LORA_INLINE {});
  if (threadIdx.x < 64) edge_unit(xe, term, box + units);
  __syncthreads();
  Unit u = join_units(box, units + 1, term);
  if constexpr (H == HARD_SAME) u.a = u.s;
  return u;
}

// The loss of every row, and what the gradient needs.  Bound by HBM: 4096 x 32000
// bf16 in 50 us, 5.2 TB/s; 301 x 131071 fp32 in 34, 4.6 TB/s (301 workgroups on 256
// compute units); 75 and 49 right behind a gradient that is still on its way to
// memory.  A unit's loads ahead of the last one's sums were slower (53 us, 49
// without in the same run): other waves cover the loads.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void lora_distill_fwd_kernel(const T* __restrict__ logits, int64_t ld,
                                                              const int32_t* __restrict__ ids,
                                                              const float* __restrict__ teacher,
                                                              const int32_t* __restrict__ labels, float tau, float w,
                                                              float* __restrict__ loss, float4* __restrict__ saved,
                                                              int vocab, int top) {
  __shared__ ListShared list;
  __shared__ Unit box[kMaxUnits];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x;
  const Row<T> row(logits + r * ld, vocab);
  if (tid < 64) teacher_list(list_in(ids + r * top, teacher + r * top, labels ? labels + r : nullptr, top), kLog2e / tau, vocab, top, list);
  const float xe = row.value(row.edge(vocab));
  Unit sum;
  with_hard(hard_of(tau, w), [&](auto hc) LORA_INLINE {
    sum = row_sums<decltype(hc)::value, NT>(row, xe, scale_of(tau, w), box);
  });
  if (tid < 64) {
    const bool empty = sum.s == 0.f;
    const float shift = shift_of(sum.m), inf = __builtin_inff();
    const float l = row_loss(list, [&](int k) LORA_INLINE { return row.value(list.id[k]); }, top, tau, w, shift, logf(sum.s), logf(sum.a));
    if (tid == 0) {
      loss[r] = empty ? 0.f : l;
      // an empty row's sums are taken as infinite: every probability is 0
      saved[r] = float4{shift, empty ? inf : sum.s, empty ? inf : sum.a, 0.f};
    }
  }
}

// The gradient from what the forward saved: workgroups of kGradThreads x
// kGradKeep chunks of a row.  Bound by HBM: 4096 x 32000 bf16 with a list of 64 in
// 103 us, 301 x 131071 fp32 in 60, 5.1 to 5.3 TB/s read and written, run after run;
// 86 and 51 right behind the forward, with logits still in the caches (116 and 66,
// against 107 and 60 in the same run, with the listed columns' logits looked up
// once the list was made).  Registers for seven waves a SIMD: eight spill two.
template <typename T, int H>
__global__ __launch_bounds__(kGradThreads, 7) void lora_distill_bwd_kernel(
    const T* logits, int64_t ld, const int32_t* __restrict__ ids, const float* __restrict__ teacher,
    const int32_t* __restrict__ labels, float tau, float w, const float4* __restrict__ saved,
    const float* __restrict__ dloss, T* dlogits, int vocab, int top, int parts) {
  constexpr int CH = Chunk<T>::CH, NT = kGradThreads;
  __shared__ ListShared list;
  __shared__ ListChain<NT> chain;
  const int64_t r = blockIdx.x / (unsigned)parts;
  const int part = (int)(blockIdx.x - (unsigned)r * (unsigned)parts), tid = threadIdx.x;
  const T* z = logits + r * ld;
  T* dz = dlogits + r * ld;
  const bool alike = lies_alike<T>(logits, dlogits);
  const Row<T> row(z, vocab);
  // this workgroup's chunks and columns (the single elements before the first
  // chunk belong to the first workgroup, those after the last to the last)
  const bool last = part == parts - 1;
  const int c0 = min(row.chunks, part * (NT * kGradKeep)), c1 = last ? row.chunks : min(row.chunks, c0 + NT * kGradKeep);
  const int col0 = part == 0 ? 0 : row.head + c0 * CH, col1 = last ? vocab : row.head + c1 * CH;
  // the entries' columns, by a thread each, ahead of the list that the first wave
  // makes of them: their logits come with the row
  const int mine = tid < top ? ids[r * top + tid] : (tid == top && labels ? labels[r] : -1);
  int4v v[kGradKeep];
#pragma unroll
  for (int i = 0; i < kGradKeep; ++i) {
    const int c = c0 + tid + i * NT;
    if (c < c1) v[i] = row.at(c);
  }
  chain.first[tid] = -1;
  const bool fixes = mine >= col0 && mine < col1;
  const T xl = row.raw(fixes ? mine : -1);
  int edge = row.edge(vocab);
  if (edge < col0 || edge >= col1) edge = -1;
  const float xe = row.value(edge);
  if (tid < 64) teacher_list(list_in(ids + r * top, teacher + r * top, labels ? labels + r : nullptr, top), kLog2e / tau, vocab, top, list);
  const float4 sv = saved[r];
  const float g = dloss[r];
  __syncthreads();
  const GradRow gr = grad_row(list, top, g, tau, w, sv.x, sv.y, sv.z);
  if (fixes) {
    chain.x[tid] = Chunk<T>::one(xl);
    chain.link(tid, mine < row.head ? mine : (mine >= row.tail0 ? CH + mine - row.tail0 : ((mine - row.head) / CH - c0) % NT));
  }
  __syncthreads();   // the listed columns are read: dlogits may be the logits
#pragma unroll
  for (int i = 0; i < kGradKeep; ++i) {
    const int c = c0 + tid + i * NT;
    if (c < c1) {
      float x[CH];
#pragma unroll
      for (int e = 0; e < CH; ++e) x[e] = gr.template dense<H>(Chunk<T>::get(v[i], e));
      put<T>(dz + row.head + (size_t)c * CH, x, alike);
    }
    __builtin_amdgcn_sched_barrier(0);   // one chunk's values at a time
  }
  if (edge >= 0) dz[edge] = Chunk<T>::pack1(gr.template dense<H>(xe));
  chain.template put<H>(dz, list, top, sv.y == __builtin_inff(), g, tau, w, gr);
}

// Loss and gradient in one pass over the logits.  A workgroup keeps a row in
// registers and takes row after row.  With the row's exponentials held (four
// chunks, from the sums to the gradient), a chunk's place takes the
// next row's as soon as the chunk is summed, else once its gradient is on its
// way; so the next row arrives under this row's arithmetic and stores.  The
// listed columns' gradients are stored by the thread that stored their chunk (a
// chain of entries per thread in LDS), in its program order, so no barrier waits
// for the stores; two LDS copies alternate, so that none waits for the row's end.
// Chunks are loaded and stored through buffer resources of the row's whole
// chunks: those past it are neither read nor stored.  Bound by HBM: 4096 x 32000 bf16 with a
// list of 64 in 99 us, 5.3 TB/s, a copy's rate (124 with the exponentials formed
// again and the loads behind the stores).
template <int NT>
struct StepShared {
  ListShared list;
  ListChain<NT> chain;
  float mbox[NT / 64];
  float2 sbox[NT / 64];
};

__device__ __forceinline__ const void* uniform_ptr(const void* p) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = (uint32_t)uniform((int)(uint32_t)a), hi = (uint32_t)uniform((int)(a >> 32));
  return reinterpret_cast<const void*>((uint64_t)hi << 32 | lo);
}

template <typename T, int NT, int KEEP, int H, bool ALIKE>
__global__ __launch_bounds__(NT) void lora_distill_step_kernel(const T* logits, int64_t ld,
                                                               const int32_t* __restrict__ ids,
                                                               const float* __restrict__ teacher,
                                                               const int32_t* __restrict__ labels, float tau, float w,
                                                               const float* __restrict__ dloss,
                                                               float* __restrict__ loss, T* dlogits, int rows,
                                                               int vocab, int top) {
  constexpr int CH = Chunk<T>::CH;
  __shared__ StepShared<NT> both[2];
  const int tid = threadIdx.x;
  const float scale = scale_of(tau, w);
  int64_t r = blockIdx.x;
  Row<T> row(logits + r * ld, vocab);
  int4v v[KEEP];
  __amdgpu_buffer_rsrc_t rs = make_rsrc(uniform_ptr(row.p + row.head), (uint64_t)uniform(row.chunks) * 16);
  auto load = [&](int i) LORA_INLINE {
    // (the whole offset in the lane's register, where it is compared with the row's size)
    return __builtin_bit_cast(int4v, __builtin_amdgcn_raw_buffer_load_b128(rs, (tid + i * NT) * 16, 0, 0));
  };
  auto past = [&](int i, int chunks) LORA_INLINE {   // -inf in the chunks past the row
    if ((i + 1) * NT > chunks)
      if (tid >= chunks - i * NT) v[i] = Row<T>::fill();
  };
  constexpr bool kHold = KEEP == 4 && H != HARD_OWN;
  float held[kHold ? KEEP : 1][CH];
#pragma unroll
  for (int i = 0; i < KEEP; ++i) v[i] = load(i);
  ListIn in = list_in(ids + r * top, teacher + r * top, labels ? labels + r : nullptr, top);
  T xe_in = row.raw(row.edge(vocab));
  float g = dloss[r];
  for (int turn = 0;; turn ^= 1) {
    StepShared<NT>& sh = both[turn];
    T* dz = dlogits + r * ld;
    if (tid < 64) teacher_list(in, kLog2e / tau, vocab, top, sh.list);
    sh.chain.first[tid] = -1;
    const float xe = Chunk<T>::one(xe_in);
    float m = xe;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      past(i, row.chunks);
#pragma unroll
      for (int e = 0; e < CH; ++e) m = fmaxf(m, Chunk<T>::get(v[i], e));
      __builtin_amdgcn_sched_barrier(0);
    }
    m = block_max<NT>(m, sh.mbox);
    const float shift = shift_of(m);
    // the entries' columns: chained to the threads that store them
    const int mine = tid <= top ? sh.list.id[tid] : -1;
    const T xl = row.raw(mine);
    if (mine >= 0) {
      const int owner = mine < row.head ? mine : (mine >= row.tail0 ? CH + mine - row.tail0 : (mine - row.head) / CH % NT);
      sh.chain.link(tid, owner);
    }
    // the next row
    const int64_t rn = r + gridDim.x;
    const bool more = rn < rows;
    const int64_t rl = more ? rn : r;
    const Row<T> next(logits + rl * ld, vocab);
    rs = make_rsrc(uniform_ptr(next.p + next.head), more ? (uint64_t)uniform(next.chunks) * 16 : 0);
    const ListIn in_next = list_in(ids + rl * top, teacher + rl * top, labels ? labels + rl : nullptr, top);
    const T xe_next = next.raw(next.edge(vocab));
    const float g_next = dloss[rl];
    float soft = 0.f, hard = 0.f;
    auto add = [&](float x) LORA_INLINE {
      const float d = x - shift, u = exp2_hw(d * scale);
      soft += u;
      if constexpr (H != HARD_SAME) hard += hard_exp<H>(u, d);
      return u;
    };
#pragma unroll
    for (int i = 0; i < KEEP; ++i) asm volatile("" : "+v"(v[i]));   // values are formed anew instead of being kept
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
#pragma unroll
      for (int e = 0; e < CH; ++e) {
        const float u = add(Chunk<T>::get(v[i], e));
        if constexpr (kHold) held[i][e] = u;
      }
      if constexpr (kHold) v[i] = load(i);
      __builtin_amdgcn_sched_barrier(0);
    }
    add(xe);
    if constexpr (H == HARD_SAME) hard = soft;
    if (mine >= 0) sh.chain.x[tid] = Chunk<T>::one(xl);   // (from here on dlogits may be written over the logits)
    const float2 sum = block_sum2<NT>(soft, hard, sh.sbox);
    const bool empty = sum.x == 0.f;
    const float inf = __builtin_inff();
    const GradRow gr = grad_row(sh.list, top, g, tau, w, shift, empty ? inf : sum.x, empty ? inf : sum.y);
    // (a row that lies differently may start between two words)
    const int off = ALIKE ? 0 : (int)(reinterpret_cast<uintptr_t>(dz + row.head) & 3);
    const __amdgpu_buffer_rsrc_t rd = make_rsrc(uniform_ptr(reinterpret_cast<char*>(dz + row.head) - off),
                                                (uint64_t)uniform(row.chunks) * 16 + uniform(off));
    if constexpr (!kHold) {
#pragma unroll
      for (int i = 0; i < KEEP; ++i) asm volatile("" : "+v"(v[i]));
    }
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      float x[CH];
#pragma unroll
      for (int e = 0; e < CH; ++e)
        x[e] = kHold ? gr.template of_exp<H>(held[kHold ? i : 0][e]) : gr.template dense<H>(Chunk<T>::get(v[i], e));
      // (the whole offset in the lane's register: with a part of it in a scalar one,
      // an instruction right after the store that overwrote the data's first
      // register had its value stored, and the compiler only keeps the two apart
      // without it)
      const int at = (tid + i * NT) * 16;
      if constexpr (ALIKE) {
        typedef unsigned u4 __attribute__((ext_vector_type(4)));
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, Chunk<T>::pack(x)), rd, at, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < CH; ++e) {
          if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(Chunk<T>::pack1(x[e]), rd, at + off + 2 * e, 0, 0);
          else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, x[e]), rd, at + off + 4 * e, 0, 0);
        }
      }
      if constexpr (!kHold) v[i] = load(i);
      __builtin_amdgcn_sched_barrier(0);
    }
    const int edge = row.edge(vocab);
    if (edge >= 0) dz[edge] = Chunk<T>::pack1(gr.template dense<H>(xe));
    sh.chain.template put<H>(dz, sh.list, top, empty, g, tau, w, gr);
    if (tid < 64) {
      const float l = row_loss(sh.list, [&](int k) LORA_INLINE { return sh.chain.x[k]; }, top, tau, w, shift, logf(sum.x), logf(sum.y));
      if (tid == 0) loss[r] = empty ? 0.f : l;
    }
    if (!more) break;
    r = rn;
    row = next;
    in = in_next;
    xe_in = xe_next;
    g = g_next;
  }
}

// Rows wider than a workgroup's registers: the row is read again for the gradient
// (301 x 131071 fp32 120 us; its passes follow each other in a workgroup, so it
// takes what the forward and the backward take together or somewhat more).
template <typename T, int NT>
__global__ __launch_bounds__(NT) void lora_distill_wide_kernel(const T* logits, int64_t ld,
                                                               const int32_t* __restrict__ ids,
                                                               const float* __restrict__ teacher,
                                                               const int32_t* __restrict__ labels, float tau, float w,
                                                               const float* __restrict__ dloss,
                                                               float* __restrict__ loss, T* dlogits, int vocab,
                                                               int top) {
  constexpr int CH = Chunk<T>::CH, U = 8;
  __shared__ ListShared list;
  __shared__ ListChain<NT> chain;
  __shared__ Unit box[kMaxUnits];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x;
  T* dz = dlogits + r * ld;
  const bool alike = lies_alike<T>(logits, dlogits);
  const Row<T> row(logits + r * ld, vocab);
  chain.first[tid] = -1;
  const float g = dloss[r];
  if (tid < 64) teacher_list(list_in(ids + r * top, teacher + r * top, labels ? labels + r : nullptr, top), kLog2e / tau, vocab, top, list);
  const int edge = row.edge(vocab);
  const float xe = row.value(edge);
  with_hard(hard_of(tau, w), [&](auto hc) LORA_INLINE {
    constexpr int H = decltype(hc)::value;
    const Unit sum = row_sums<H, NT>(row, xe, scale_of(tau, w), box);
    const bool empty = sum.s == 0.f;
    const float shift = shift_of(sum.m), inf = __builtin_inff();
    if (tid < 64) {
      const float l = row_loss(list, [&](int k) LORA_INLINE { return row.value(list.id[k]); }, top, tau, w, shift, logf(sum.s), logf(sum.a));
      if (tid == 0) loss[r] = empty ? 0.f : l;
    }
    const GradRow gr = grad_row(list, top, g, tau, w, shift, empty ? inf : sum.s, empty ? inf : sum.a);
    const int mine = tid <= top ? list.id[tid] : -1;
    if (mine >= 0) {
      chain.x[tid] = row.value(mine);
      chain.link(tid, mine < row.head ? mine : (mine >= row.tail0 ? CH + mine - row.tail0 : (mine - row.head) / CH % NT));
    }
    __syncthreads();   // the listed columns are read: dlogits may be the logits
    for (int c0 = tid; c0 < row.chunks; c0 += NT * U) {
      int4v v[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c0 + NT * u < row.chunks) v[u] = row.at(c0 + NT * u);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c0 + NT * u < row.chunks) {
          float x[CH];
#pragma unroll
          for (int e = 0; e < CH; ++e) x[e] = gr.template dense<H>(Chunk<T>::get(v[u], e));
          put<T>(dz + row.head + (size_t)(c0 + NT * u) * CH, x, alike);
        }
    }
    if (edge >= 0) dz[edge] = Chunk<T>::pack1(gr.template dense<H>(xe));
    chain.template put<H>(dz, list, top, empty, g, tau, w, gr);
  });
}

// f(threads, chunks kept) for a row of the step.
template <typename F>
static hipError_t with_row(const RowShape& s, F&& f) {
  using std::integral_constant;
  if (s.keep == 16) return f(integral_constant<int, 1024>{}, integral_constant<int, 16>{});
  if (s.keep == 8) return f(integral_constant<int, 1024>{}, integral_constant<int, 8>{});
  if (s.threads == 256) return f(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  if (s.threads == 512) return f(integral_constant<int, 512>{}, integral_constant<int, 4>{});
  return f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}

template <typename F>
static hipError_t with_type(bool f32, F&& f) {
  return f32 ? f(float{}) : f(u16{});
}

hipError_t launch_token_logprobs(const LogprobArgs& a, hipStream_t st) {
  return with_type(a.f32, [&](auto t) {
    using T = decltype(t);
    const int parts = score_parts(a.rows, a.vocab, sizeof(T), a.top);
    const ScoreParts ws(a.ws, a.rows, a.vocab, sizeof(T), parts, a.top);
    auto launch = [&](auto kernel, int threads, int64_t grid) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(threads), 0, st, static_cast<const T*>(a.logits), a.ld,
                         a.tokens, a.itau, a.logp, a.entropy, a.top_ids, a.top_logp, a.vocab, a.top, parts, ws);
      return hipGetLastError();
    };
    if (parts > 1) {
      const hipError_t e = launch(lora_logprobs_kernel<T, 1024, true>, 1024, a.rows * parts);
      return e != hipSuccess ? e : launch(lora_logprobs_join_kernel<T>, kMaxKeys, a.rows);
    }
    return with_int<256, 512, 1024>(read_threads(a.rows, a.vocab, sizeof(T), 4), [&](auto nt) {
      return launch(lora_logprobs_kernel<T, decltype(nt)::value, false>, decltype(nt)::value, a.rows);
    });
  });
}

hipError_t launch_distill_fwd(const DistillArgs& a, hipStream_t st) {
  return with_type(a.f32, [&](auto t) {
    using T = decltype(t);
    return with_int<256, 512, 1024>(read_threads(a.rows, a.vocab, sizeof(T), 1), [&](auto nt) {
      constexpr int NT = decltype(nt)::value;
      hipLaunchKernelGGL((lora_distill_fwd_kernel<T, NT>), dim3((unsigned)a.rows), dim3(NT), 0, st,
                         static_cast<const T*>(a.logits), a.ld, a.ids, a.teacher, a.labels, a.tau, a.w, a.loss,
                         reinterpret_cast<float4*>(a.saved), a.vocab, a.top);
      return hipGetLastError();
    });
  });
}

hipError_t launch_distill_bwd(const DistillArgs& a, hipStream_t st) {
  return with_type(a.f32, [&](auto t) {
    using T = decltype(t);
    const int parts = grad_parts(a.vocab, sizeof(T));
    with_hard(hard_of(a.tau, a.w), [&](auto hc) {
      hipLaunchKernelGGL((lora_distill_bwd_kernel<T, decltype(hc)::value>), dim3((unsigned)(a.rows * parts)),
                         dim3(kGradThreads), 0, st, static_cast<const T*>(a.logits), a.ld, a.ids, a.teacher, a.labels,
                         a.tau, a.w, reinterpret_cast<const float4*>(a.saved), a.dloss, static_cast<T*>(a.dlogits),
                         a.vocab, a.top, parts);
    });
    return hipGetLastError();
  });
}

hipError_t launch_distill_step(const DistillArgs& a, hipStream_t st) {
  return with_type(a.f32, [&](auto t) {
    using T = decltype(t);
    // (a gradient that lies differently in 16 bytes is stored value by value)
    const bool alike = ((reinterpret_cast<uintptr_t>(a.logits) ^ reinterpret_cast<uintptr_t>(a.dlogits)) & 15) == 0;
    if (row_shape(a.vocab, sizeof(T)).keep == 0) {
      constexpr int NT = 512;
      hipLaunchKernelGGL((lora_distill_wide_kernel<T, NT>), dim3((unsigned)a.rows), dim3(NT), 0, st,
                         static_cast<const T*>(a.logits), a.ld, a.ids, a.teacher, a.labels, a.tau, a.w, a.dloss, a.loss,
                         static_cast<T*>(a.dlogits), a.vocab, a.top);
      return hipGetLastError();
    }
    return with_row(row_shape(a.vocab, sizeof(T)), [&](auto nt, auto keep) {
      constexpr int NT = decltype(nt)::value, KEEP = decltype(keep)::value;
      const int64_t grid = std::min<int64_t>(a.rows, 256 * (1024 / NT));
      with_hard(hard_of(a.tau, a.w), [&](auto hc) {
        constexpr int H = decltype(hc)::value;
        const auto kernel = alike ? lora_distill_step_kernel<T, NT, KEEP, H, true> : lora_distill_step_kernel<T, NT, KEEP, H, false>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(NT), 0, st, static_cast<const T*>(a.logits), a.ld, a.ids,
                           a.teacher, a.labels, a.tau, a.w, a.dloss, a.loss, static_cast<T*>(a.dlogits), (int)a.rows,
                           a.vocab, a.top);
      });
      return hipGetLastError();
    });
  });
}

}  // namespace lora
