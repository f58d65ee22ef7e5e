// Operators on rows of logits z [rows, vocab]:
//   * log probability of each row's token, entropy, and the top alternatives of
//     softmax(z / tau);
//   * distillation from a teacher's top logits, its loss and its gradient.
//
// Both are bound by reading z (and writing its gradient) once.  One workgroup
// takes a row and keeps it in registers between the pass for the maximum, the
// one for the sums and the one that writes or selects, so that HBM sees each
// value once; rows too wide for that are read again in each pass.  Sums,
// maxima and softmax statistics are fp32 in a fixed order.
//
// Exponentials are taken to base 2, of y = (z - max z) log2(e) / tau; with S =
// sum 2^y, log softmax = (z - max z) / tau - ln S (not from y: the difference of
// a row's maximum and the type's lowest value fits fp32, its multiple need not).
// The maximum is subtracted before the scale is applied, so that rows of the
// lowest value do not overflow; a row without a value above -inf subtracts 0 and has S = 0, and one
// that holds a NaN or +inf has S = NaN.
#include <type_traits>

#include "lora_device.hpp"
#include "lora_ops.hpp"
#include "lora_plan.hpp"

namespace lora {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kNegInf = -__builtin_inff();

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
      v[h] = (int)((uint32_t)f32_to_bf16(x[2 * h]) | ((uint32_t)f32_to_bf16(x[2 * h + 1]) << 16));
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

// A thread's share of a row: chunks tid, tid + NT, ... and at most one of the
// single elements at the row's ends (threads 0 .. head-1 and CH .. CH+tail-1).
// With KEEP > 0 the chunks stay in registers after load(); those past the row
// hold -inf.
template <typename T, int NT, int KEEP>
struct Row {
  static constexpr int CH = Chunk<T>::CH;
  const T* p;          // the row
  int head, chunks;    // single elements before the first chunk, whole chunks
  int edge;            // this thread's single element, -1: none
  float xe;            // its value, -inf without one
  int4v v[KEEP > 0 ? KEEP : 1];

  // Without `first` (`last`) the single elements before (after) the chunks are left out.
  __device__ __forceinline__ void open(const T* row, int vocab, bool first = true, bool last = true) {
    p = row;
    const int off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    head = min(off ? CH - off : 0, vocab);
    chunks = (vocab - head) / CH;
    const int tid = threadIdx.x, tail0 = head + chunks * CH;
    edge = first && tid < head ? tid : (last && tid >= CH && tid - CH < vocab - tail0 ? tail0 + tid - CH : -1);
    xe = edge >= 0 ? Chunk<T>::one(row[edge]) : kNegInf;
    if constexpr (KEEP > 0) {
#pragma unroll
      for (int i = 0; i < KEEP; ++i) {
        const int c = tid + i * NT;
        v[i] = c < chunks ? at(c) : int4v{Chunk<T>::kFill, Chunk<T>::kFill, Chunk<T>::kFill, Chunk<T>::kFill};
      }
    }
  }
  __device__ __forceinline__ int4v at(int c) const {
    return *reinterpret_cast<const int4v*>(p + head + (size_t)c * CH);
  }
  // f(chunk's values, its first element's index); without registers for the
  // chunks past the row f is not called.
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
    if constexpr (KEEP > 0) {
      int at0 = head + (int)threadIdx.x * CH;
      asm volatile("" : "+v"(at0));   // indices are formed in each pass, not kept
#pragma unroll
      for (int i = 0; i < KEEP; ++i) {
        f(v[i], at0 + i * (NT * CH));
        __builtin_amdgcn_sched_barrier(0);   // one chunk's values at a time
      }
    } else {
      for (int c = threadIdx.x; c < chunks; c += NT) f(at(c), head + c * CH);
    }
  }
  // Between two passes over kept chunks: their fp32 values are formed anew
  // instead of being kept (twice the registers of bf16 chunks).
  __device__ __forceinline__ void reread() {
    if constexpr (KEEP > 0) {
#pragma unroll
      for (int i = 0; i < KEEP; ++i) asm volatile("" : "+v"(v[i]));
    }
  }
  __device__ __forceinline__ bool whole(int index) const { return index < head + chunks * CH; }
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

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) x = fmaxf(x, __shfl_xor(x, s));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) x += __shfl_xor(x, s);
  return x;
}

// Maximum (NaN left out) and sums over the workgroup, the same on every thread;
// `box` holds NT / 64 floats per value.  Each call takes a box of its own.
template <int NT>
__device__ __forceinline__ float block_max(float x, float* box) {
  x = wave_max(x);
  if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = x;
  __syncthreads();
  float r = box[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) r = fmaxf(r, box[w]);
  return r;
}
template <int NT>
__device__ __forceinline__ float2 block_sum2(float a, float b, float2* box) {
  a = wave_sum(a);
  b = wave_sum(b);
  if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = float2{a, b};
  __syncthreads();
  float2 r = box[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) {
    r.x += box[w].x;
    r.y += box[w].y;
  }
  return r;
}

__device__ __forceinline__ float exp2_hw(float y) { return __builtin_amdgcn_exp2f(y); }

// What is subtracted for a row's maximum: 0 where no value is above -inf.
__device__ __forceinline__ float shift_of(float m) { return m == kNegInf ? 0.f : m; }

// ---------------------------------------------------------------------------
// Log probabilities, entropy and the top alternatives.
//
// The top values are found without sorting: the top-th largest of the threads'
// own maxima is at most the top-th largest value, so the values at or above it
// hold the answer.  It is looked for on the upper 16 bits of the values'
// ordered form by one wave (16 counts over ballots) while the others form the
// sums.  The values at or above it, a few times `top` where values are spread,
// go into an LDS list and are ranked against each other by value and index.
// Where more values tie than the list holds (a constant row), the exact
// top-th value and the index up to which its ties count are found by counting.

// Whole numbers in the order of the values; -0 as 0 and NaN as -inf.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x != x ? kNegInf : x + 0.f);
  return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return __builtin_bit_cast(float, o ^ (o >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}
constexpr uint32_t kOrderNegInf = 0x007FFFFFu;
constexpr int kCandidates = 1024;

template <int NT>
struct TopShared {
  uint32_t maxima[NT];
  uint64_t cand[kCandidates];   // order above ~index: larger is earlier
  uint32_t threshold;           // upper 16 bits
  int count;
  int part[2][NT / 64];
};

// The count over the workgroup of what every thread counted; calls alternate
// between two boxes (`turn`).
template <int NT>
__device__ __forceinline__ int block_count(int n, int (*part)[NT / 64], int& turn) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) n += __shfl_xor(n, s);
  if ((threadIdx.x & 63) == 0) part[turn][threadIdx.x >> 6] = n;
  __syncthreads();
  int r = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) r += part[turn][w];
  turn ^= 1;
  return r;
}

// The largest t with at least `top` of the threads' maxima at or above t in
// their upper 16 bits (0: fewer threads than `top` hold a value).  One wave.
template <int NT>
__device__ __forceinline__ uint32_t top_threshold(const uint32_t* maxima, int top) {
  uint32_t o[NT / 64], t = 0;
#pragma unroll
  for (int j = 0; j < NT / 64; ++j) o[j] = maxima[(threadIdx.x & 63) + 64 * j] >> 16;
  for (uint32_t bit = 0x8000u; bit; bit >>= 1) {
    int n = 0;
#pragma unroll
    for (int j = 0; j < NT / 64; ++j) n += __popcll(__ballot(o[j] >= (t | bit)));
    if (n >= top) t |= bit;
  }
  return t;
}

template <int NT>
__device__ __forceinline__ void push(TopShared<NT>& sh, uint32_t order, int index) {
  const int at = atomicAdd(&sh.count, 1);
  if (at < kCandidates) sh.cand[at] = (uint64_t)order << 32 | (uint32_t)~index;
}

// After the barrier that publishes sh.threshold and sh.count = 0.
template <typename T, int NT, int KEEP>
__device__ __forceinline__ void select_top(Row<T, NT, KEEP>& row, float own_max, int vocab, int top, float shift,
                                           float itau, float lns, bool empty, TopShared<NT>& sh, int32_t* ids,
                                           float* lps) {
  constexpr int CH = Chunk<T>::CH;
  const uint32_t t16 = sh.threshold;
  const bool all = t16 <= (kOrderNegInf >> 16);     // -inf or NaN among the top: every value is a candidate
  const float bar = value_of(t16 << 16);
  if (all || own_max >= bar) {
    row.reread();
    row.each([&](const int4v& v, int at) LORA_INLINE {
      if (!row.whole(at)) return;
#pragma unroll
      for (int e = 0; e < CH; ++e) {
        const float x = Chunk<T>::get(v, e);
        if (all || x >= bar) push<NT>(sh, order_of(x), at + e);
      }
    });
    if (row.edge >= 0 && (all || row.xe >= bar)) push<NT>(sh, order_of(row.xe), row.edge);
  }
  __syncthreads();
  int n = sh.count;
  if (n > kCandidates) {
    int turn = 0;
    auto count = [&](auto&& pred) LORA_INLINE {
      int c = 0;
      row.reread();
      row.each([&](const int4v& v, int at) LORA_INLINE {
        if (!row.whole(at)) return;
#pragma unroll
        for (int e = 0; e < CH; ++e) c += pred(order_of(Chunk<T>::get(v, e)), at + e);
      });
      if (row.edge >= 0) c += pred(order_of(row.xe), row.edge);
      return block_count<NT>(c, sh.part, turn);
    };
    uint32_t kth = 0;          // the top-th largest value's order
    for (uint32_t bit = 0x80000000u; bit; bit >>= 1)
      if (count([&](uint32_t o, int) { return o >= (kth | bit); }) >= top) kth |= bit;
    const int above = count([&](uint32_t o, int) { return o > kth; });
    int last = 0;              // the largest index bound with fewer than top - above ties below it
    for (int bit = 1 << 22; bit; bit >>= 1)
      if (count([&](uint32_t o, int i) { return o == kth && i < (last | bit); }) < top - above) last |= bit;
    __syncthreads();           // everyone has read sh.count
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    auto take = [&](float x, int i) LORA_INLINE {
      const uint32_t o = order_of(x);
      if (o > kth || (o == kth && i <= last)) push<NT>(sh, o, i);
    };
    row.reread();
    row.each([&](const int4v& v, int at) LORA_INLINE {
      if (!row.whole(at)) return;
#pragma unroll
      for (int e = 0; e < CH; ++e) take(Chunk<T>::get(v, e), at + e);
    });
    if (row.edge >= 0) take(row.xe, row.edge);
    __syncthreads();
    n = sh.count;
  }
  for (int c = threadIdx.x; c < n; c += NT) {
    const uint64_t mine = sh.cand[c];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += sh.cand[j] > mine;
    if (rank < top) {
      const int index = (int)~(uint32_t)mine;
      ids[rank] = index;
      const float x = Chunk<T>::one(row.p[index]);
      lps[rank] = empty ? kNegInf : (x - shift) * itau - lns;
    }
  }
}

template <typename T, int NT, int KEEP>
__global__ __launch_bounds__(NT) void lora_logprobs_kernel(const T* __restrict__ logits, int64_t ld,
                                                           const int32_t* __restrict__ tokens, float itau,
                                                           float* __restrict__ logp, float* __restrict__ entropy,
                                                           int32_t* __restrict__ top_ids, float* __restrict__ top_logp,
                                                           int vocab, int top) {
  constexpr int CH = Chunk<T>::CH;
  __shared__ TopShared<NT> sh;
  __shared__ float mbox[NT / 64];
  __shared__ float2 sbox[NT / 64];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x;
  const float scale = kLog2e * itau;
  Row<T, NT, KEEP> row;
  row.open(logits + r * ld, vocab);

  float own = row.xe;
  row.each([&](const int4v& v, int) LORA_INLINE {
#pragma unroll
    for (int e = 0; e < CH; ++e) own = fmaxf(own, Chunk<T>::get(v, e));
  });
  if (top > 0) {   // 0 for the threads without a value
    sh.maxima[tid] = row.edge >= 0 || tid < row.chunks ? order_of(own) : 0u;
    if (tid == 0) sh.count = 0;
  }
  const float m = block_max<NT>(own, mbox);
  const float shift = shift_of(m);
  if (top > 0 && tid < 64) {
    const uint32_t t = top_threshold<NT>(sh.maxima, top);
    if (tid == 0) sh.threshold = t;
  }
  float s = 0.f, a = 0.f;
  auto add = [&](float x) LORA_INLINE {
    const float y = (x - shift) * scale, e = exp2_hw(y);
    s += e;
    a = fmaf(e, fmaxf(y, -1e4f), a);   // (0 for e = 0 at y = -inf)
  };
  row.reread();
  row.each([&](const int4v& v, int) LORA_INLINE {
#pragma unroll
    for (int e = 0; e < CH; ++e) add(Chunk<T>::get(v, e));
  });
  add(row.xe);
  const float2 sum = block_sum2<NT>(s, a, sbox);
  const float lns = logf(sum.x);
  const bool empty = sum.x == 0.f;
  if (tid == 0) {
    entropy[r] = empty ? 0.f : lns - sum.y / sum.x * kLn2;
    if (tokens) {
      const int t = tokens[r];
      float lp = 0.f;
      if ((uint32_t)t < (uint32_t)vocab)
        lp = empty ? kNegInf : (Chunk<T>::one(row.p[t]) - shift) * itau - lns;
      logp[r] = lp;
    }
  }
  if (top > 0)
    select_top<T, NT, KEEP>(row, own, vocab, top, shift, itau, lns, empty, sh, top_ids + r * top, top_logp + r * top);
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

// One wave forms p and leaves it in sh (before a barrier of the caller).
__device__ __forceinline__ void teacher_list(const int32_t* ids, const float* t, const int32_t* label, float scale,
                                             int vocab, int top, ListShared& sh) {
  const int lane = threadIdx.x & 63;
  int id[2];
  float y[2], e[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int k = lane + 64 * h;
    id[h] = k < top ? ids[k] : -1;
    if ((uint32_t)id[h] >= (uint32_t)vocab) id[h] = -1;
    y[h] = id[h] >= 0 ? t[k] : kNegInf;
  }
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
      sh.id[lane + 64 * h] = id[h];
      sh.p[lane + 64 * h] = p;
    }
  }
  plogp = wave_sum(plogp);
  if (lane == 0) {
    const int y0 = label ? *label : -1;
    sh.id[top] = (uint32_t)y0 < (uint32_t)vocab ? y0 : -1;
    sh.p[top] = 0.f;
    sh.mass = sum == 0.f ? 0.f : sum * inv;   // NaN where the list holds one
    sh.entropy = plogp;
  }
}

// Loss of a row by one wave from the logarithms of both softmaxes' sums.
template <typename T>
__device__ __forceinline__ float row_loss(const T* row, const ListShared& sh, int top, float tau, float w, float shift,
                                          float lnsoft, float lnhard) {
  const int lane = threadIdx.x & 63;
  const float itau = 1.f / tau;
  float cross = 0.f;       // sum p ln q
  if (w > 0.f)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = lane + 64 * h;
      if (k < top && sh.id[k] >= 0) {
        const float p = sh.p[k];
        if (!(p == 0.f)) cross = fmaf(p, (Chunk<T>::one(row[sh.id[k]]) - shift) * itau - lnsoft, cross);
      }
    }
  cross = wave_sum(cross);
  float loss = w > 0.f ? w * tau * tau * (sh.entropy - cross) : 0.f;
  if (w < 1.f && sh.id[top] >= 0)
    loss += (1.f - w) * (lnhard - (Chunk<T>::one(row[sh.id[top]]) - shift));
  return loss;
}

// Gradient factors of a row: dz = fs 2^((z - shift) scale + bs) + fh 2^((z -
// shift) log2e + bh) away from the listed columns.
struct GradRow {
  float shift, scale, fs, bs, fh, bh;
  __device__ __forceinline__ float dense(float x) const {
    const float d = x - shift;
    float g = 0.f;
    if (fs != 0.f) g = fs * exp2_hw(fmaf(d, scale, bs));
    if (fh != 0.f) g = fmaf(fh, exp2_hw(fmaf(d, kLog2e, bh)), g);
    return g;
  }
};

// dz of listed column k (entries with one id all get its whole value).
template <typename T>
__device__ __forceinline__ float listed_grad(const T* row, const ListShared& sh, int k, int top, float g, float tau,
                                             float w, const GradRow& gr) {
  const int id = sh.id[k];
  float p = 0.f;
  for (int j = 0; j < top; ++j) p += sh.id[j] == id ? sh.p[j] : 0.f;
  float d = gr.dense(Chunk<T>::one(row[id])) - g * w * tau * p;
  if (sh.id[top] == id) d -= g * (1.f - w);
  return d;
}

// The loss of every row: one pass with a running maximum per thread.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void lora_distill_fwd_kernel(const T* __restrict__ logits, int64_t ld,
                                                              const int32_t* __restrict__ ids,
                                                              const float* __restrict__ teacher,
                                                              const int32_t* __restrict__ labels, float tau, float w,
                                                              float* __restrict__ loss, float4* __restrict__ saved,
                                                              int vocab, int top) {
  constexpr int CH = Chunk<T>::CH;
  __shared__ ListShared list;
  __shared__ float mbox[NT / 64];
  __shared__ float2 sbox[NT / 64];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x;
  const float scale = kLog2e / tau;
  Row<T, NT, 0> row;
  row.open(logits + r * ld, vocab);
  if (tid < 64) teacher_list(ids + r * top, teacher + r * top, labels ? labels + r : nullptr, scale, vocab, top, list);
  float m = row.xe, shift = shift_of(m), soft = exp2_hw((row.xe - shift) * scale), hard = exp2_hw((row.xe - shift) * kLog2e);
  row.each([&](const int4v& v, int) LORA_INLINE {
    float cm = Chunk<T>::get(v, 0);
#pragma unroll
    for (int e = 1; e < CH; ++e) cm = fmaxf(cm, Chunk<T>::get(v, e));
    if (cm > m) {
      const float d = m - cm;
      soft *= exp2_hw(d * scale);
      hard *= exp2_hw(d * kLog2e);
      m = cm;
      shift = cm;
    }
#pragma unroll
    for (int e = 0; e < CH; ++e) {
      const float d = Chunk<T>::get(v, e) - shift;
      soft += exp2_hw(d * scale);
      hard += exp2_hw(d * kLog2e);
    }
  });
  const float mr = block_max<NT>(m, mbox);
  shift = shift_of(mr);
  const float2 sum = block_sum2<NT>(soft * exp2_hw((m - shift) * scale), hard * exp2_hw((m - shift) * kLog2e), sbox);
  if (tid < 64) {
    const bool empty = sum.x == 0.f;
    const float l = row_loss(row.p, list, top, tau, w, shift, logf(sum.x), logf(sum.y));
    if (tid == 0) {
      loss[r] = empty ? 0.f : l;
      // an empty row's sums are taken as infinite: every probability is 0
      saved[r] = float4{shift, empty ? __builtin_inff() : log2f(sum.x), empty ? __builtin_inff() : log2f(sum.y), 0.f};
    }
  }
}

// The gradient from what the forward saved: workgroups of kGradThreads x
// kGradKeep chunks of a row.
template <typename T>
__global__ __launch_bounds__(kGradThreads) void lora_distill_bwd_kernel(
    const T* logits, int64_t ld, const int32_t* __restrict__ ids, const float* __restrict__ teacher,
    const int32_t* __restrict__ labels, float tau, float w, const float4* __restrict__ saved,
    const float* __restrict__ dloss, T* dlogits, int vocab, int top, int parts) {
  constexpr int CH = Chunk<T>::CH, NT = kGradThreads;
  __shared__ ListShared list;
  const int64_t r = blockIdx.x / (unsigned)parts;
  const int part = (int)(blockIdx.x - (unsigned)r * (unsigned)parts), tid = threadIdx.x;
  const float scale = kLog2e / tau;
  const T* z = logits + r * ld;
  T* dz = dlogits + r * ld;
  const bool alike = lies_alike<T>(logits, dlogits);
  if (tid < 64) teacher_list(ids + r * top, teacher + r * top, labels ? labels + r : nullptr, scale, vocab, top, list);
  Row<T, NT, 0> row;
  row.open(z, vocab, part == 0, part == parts - 1);
  // this workgroup's chunks and columns (the single elements before the first
  // chunk belong to the first workgroup, those after the last to the last)
  const int c0 = part * (NT * kGradKeep), c1 = part == parts - 1 ? row.chunks : min(row.chunks, c0 + NT * kGradKeep);
  const int col0 = part == 0 ? 0 : row.head + c0 * CH;
  const int col1 = part == parts - 1 ? vocab : row.head + c1 * CH;
  int4v v[kGradKeep];
#pragma unroll
  for (int i = 0; i < kGradKeep; ++i) {
    const int c = c0 + tid + i * NT;
    if (c < c1) v[i] = row.at(c);
  }
  const float4 sv = saved[r];
  const float g = dloss[r];
  const bool empty = sv.y == __builtin_inff();
  __syncthreads();
  GradRow gr{sv.x, scale, w > 0.f && !empty ? g * w * tau * list.mass : 0.f, -sv.y,
             w < 1.f && !empty && list.id[top] >= 0 ? g * (1.f - w) : 0.f, -sv.z};
  float fix = 0.f;
  const int mine = tid <= top ? list.id[tid] : -1;
  const bool fixes = mine >= col0 && mine < col1;
  if (fixes && !empty) fix = listed_grad(z, list, tid, top, g, tau, w, gr);
  __syncthreads();   // the listed columns are read: dlogits may be the logits
#pragma unroll
  for (int i = 0; i < kGradKeep; ++i) {
    const int c = c0 + tid + i * NT;
    if (c < c1) {
      float x[CH];
#pragma unroll
      for (int e = 0; e < CH; ++e) x[e] = gr.dense(Chunk<T>::get(v[i], e));
      put<T>(dz + row.head + (size_t)c * CH, x, alike);
    }
  }
  if (row.edge >= 0) dz[row.edge] = Chunk<T>::pack1(gr.dense(row.xe));
  __syncthreads();   // the listed columns over the dense values
  if (fixes) dz[mine] = Chunk<T>::pack1(fix);
}

// Loss and gradient of a row in one pass over it.
template <typename T, int NT, int KEEP>
__global__ __launch_bounds__(NT) void lora_distill_step_kernel(const T* logits, int64_t ld,
                                                               const int32_t* __restrict__ ids,
                                                               const float* __restrict__ teacher,
                                                               const int32_t* __restrict__ labels, float tau, float w,
                                                               const float* __restrict__ dloss,
                                                               float* __restrict__ loss, T* dlogits, int vocab,
                                                               int top) {
  constexpr int CH = Chunk<T>::CH;
  __shared__ ListShared list;
  __shared__ float mbox[NT / 64];
  __shared__ float2 sbox[NT / 64];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x;
  const float scale = kLog2e / tau;
  T* dz = dlogits + r * ld;
  const bool alike = lies_alike<T>(logits, dlogits);
  Row<T, NT, KEEP> row;
  row.open(logits + r * ld, vocab);
  if (tid < 64) teacher_list(ids + r * top, teacher + r * top, labels ? labels + r : nullptr, scale, vocab, top, list);
  const float g = dloss[r];
  float m = row.xe;
  row.each([&](const int4v& v, int) LORA_INLINE {
#pragma unroll
    for (int e = 0; e < CH; ++e) m = fmaxf(m, Chunk<T>::get(v, e));
  });
  m = block_max<NT>(m, mbox);
  const float shift = shift_of(m);
  float soft = 0.f, hard = 0.f;
  auto add = [&](float x) LORA_INLINE {
    const float d = x - shift;
    soft += exp2_hw(d * scale);
    hard += exp2_hw(d * kLog2e);
  };
  row.reread();
  row.each([&](const int4v& v, int) LORA_INLINE {
#pragma unroll
    for (int e = 0; e < CH; ++e) add(Chunk<T>::get(v, e));
  });
  add(row.xe);
  const float2 sum = block_sum2<NT>(soft, hard, sbox);
  const bool empty = sum.x == 0.f;
  if (tid < 64) {
    const float l = row_loss(row.p, list, top, tau, w, shift, logf(sum.x), logf(sum.y));
    if (tid == 0) loss[r] = empty ? 0.f : l;
  }
  GradRow gr{shift, scale, w > 0.f && !empty ? g * w * tau * list.mass / sum.x : 0.f, 0.f,
             w < 1.f && !empty && list.id[top] >= 0 ? g * (1.f - w) / sum.y : 0.f, 0.f};
  float fix = 0.f;
  const int mine = tid <= top ? list.id[tid] : -1;
  if (mine >= 0 && !empty) fix = listed_grad(row.p, list, tid, top, g, tau, w, gr);
  __syncthreads();   // the listed columns are read: dlogits may be the logits
  row.reread();
  row.each([&](const int4v& v, int at) LORA_INLINE {
    if (!row.whole(at)) return;
    float x[CH];
#pragma unroll
    for (int e = 0; e < CH; ++e) x[e] = gr.dense(Chunk<T>::get(v, e));
    put<T>(dz + at, x, alike);
  });
  if (row.edge >= 0) dz[row.edge] = Chunk<T>::pack1(gr.dense(row.xe));
  __syncthreads();   // the listed columns over the dense values
  if (mine >= 0) dz[mine] = Chunk<T>::pack1(fix);
}

// f(threads, chunks kept) for the row's shape.
template <typename F>
static hipError_t with_row(int64_t vocab, int elem, F&& f) {
  using std::integral_constant;
  const RowShape s = row_shape(vocab, elem);
  if (s.threads == 256 && s.keep == 4) return f(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  if (s.threads == 256) return f(integral_constant<int, 256>{}, integral_constant<int, 8>{});
  if (s.threads == 512) return f(integral_constant<int, 512>{}, integral_constant<int, 8>{});
  if (s.keep == 8) return f(integral_constant<int, 1024>{}, integral_constant<int, 8>{});
  if (s.keep == 16) return f(integral_constant<int, 1024>{}, integral_constant<int, 16>{});
  return f(integral_constant<int, 1024>{}, integral_constant<int, 0>{});
}

template <typename F>
static hipError_t with_type(bool f32, F&& f) {
  return f32 ? f(float{}) : f(u16{});
}

hipError_t launch_token_logprobs(const LogprobArgs& a, hipStream_t st) {
  return with_type(a.f32, [&](auto t) {
    using T = decltype(t);
    return with_row(a.vocab, sizeof(T), [&](auto nt, auto keep) {
      constexpr int NT = decltype(nt)::value, KEEP = decltype(keep)::value;
      hipLaunchKernelGGL((lora_logprobs_kernel<T, NT, KEEP>), dim3((unsigned)a.rows), dim3(NT), 0, st,
                         static_cast<const T*>(a.logits), a.ld, a.tokens, a.itau, a.logp, a.entropy, a.top_ids,
                         a.top_logp, a.vocab, a.top);
      return hipGetLastError();
    });
  });
}

hipError_t launch_distill_fwd(const DistillArgs& a, hipStream_t st) {
  return with_type(a.f32, [&](auto t) {
    using T = decltype(t);
    constexpr int NT = 512;
    hipLaunchKernelGGL((lora_distill_fwd_kernel<T, NT>), dim3((unsigned)a.rows), dim3(NT), 0, st,
                       static_cast<const T*>(a.logits), a.ld, a.ids, a.teacher, a.labels, a.tau, a.w, a.loss,
                       reinterpret_cast<float4*>(a.saved), a.vocab, a.top);
    return hipGetLastError();
  });
}

hipError_t launch_distill_bwd(const DistillArgs& a, hipStream_t st) {
  return with_type(a.f32, [&](auto t) {
    using T = decltype(t);
    const int parts = grad_parts(a.vocab, sizeof(T));
    hipLaunchKernelGGL((lora_distill_bwd_kernel<T>), dim3((unsigned)(a.rows * parts)), dim3(kGradThreads), 0, st,
                       static_cast<const T*>(a.logits), a.ld, a.ids, a.teacher, a.labels, a.tau, a.w,
                       reinterpret_cast<const float4*>(a.saved), a.dloss, static_cast<T*>(a.dlogits), a.vocab, a.top,
                       parts);
    return hipGetLastError();
  });
}

hipError_t launch_distill_step(const DistillArgs& a, hipStream_t st) {
  return with_type(a.f32, [&](auto t) {
    using T = decltype(t);
    return with_row(a.vocab, sizeof(T), [&](auto nt, auto keep) {
      constexpr int NT = decltype(nt)::value, KEEP = decltype(keep)::value;
      hipLaunchKernelGGL((lora_distill_step_kernel<T, NT, KEEP>), dim3((unsigned)a.rows), dim3(NT), 0, st,
                         static_cast<const T*>(a.logits), a.ld, a.ids, a.teacher, a.labels, a.tau, a.w, a.dloss, a.loss,
                         static_cast<T*>(a.dlogits), a.vocab, a.top);
      return hipGetLastError();
    });
  });
}

}  // namespace lora
