// One block of the counter-based generator Philox4x64-10 (Salmon, Moraes, Dror and
// Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011), as lora_mask.hip
// describes it, and how its draws keep elements.
#pragma once

#include <stdint.h>

namespace lora {

// The 128-bit product of two 64-bit words from four 32 x 32 -> 64 products,
// each with a 32-bit addend (v_mad_u64_u32), none of which can overflow:
// the low word is lo32(a_l b_l) + 2^32 lo32(v), the high word
// a_h b_h + hi32(u) + hi32(v), with u = a_l b_h + hi32(a_l b_l) and
// v = a_h b_l + lo32(u).
__device__ __forceinline__ void mulhilo64(uint64_t a, uint64_t b, uint64_t& hi, uint64_t& lo) {
  const uint32_t al = (uint32_t)a, ah = (uint32_t)(a >> 32), bl = (uint32_t)b, bh = (uint32_t)(b >> 32);
  const uint64_t t = (uint64_t)al * bl;
  const uint64_t u = (uint64_t)al * bh + (t >> 32);
  const uint64_t v = (uint64_t)ah * bl + (uint32_t)u;
  lo = (uint32_t)t | (v << 32);
  hi = (uint64_t)ah * bh + (u >> 32) + (v >> 32);
}

__device__ __forceinline__ void philox4x64_10(uint64_t (&c)[4], uint64_t k0, uint64_t k1) {
  constexpr uint64_t M0 = 0xD2E7470EE14C6C93ull, M1 = 0xCA5A826395121157ull;   // round multipliers
  constexpr uint64_t W0 = 0x9E3779B97F4A7C15ull, W1 = 0xBB67AE8584CAA73Bull;   // key increments
#pragma unroll
  for (int rnd = 0; rnd < 10; ++rnd) {
    uint64_t hi0, lo0, hi1, lo1;
    mulhilo64(M0, c[0], hi0, lo0);
    mulhilo64(M1, c[2], hi1, lo1);
    const uint64_t n0 = hi1 ^ c[1] ^ k0, n2 = hi0 ^ c[3] ^ k1;
    c[0] = n0;
    c[1] = lo1;
    c[2] = n2;
    c[3] = lo0;
    k0 += W0;
    k1 += W1;
  }
}

// The block at offset + t (a 128-bit counter) under the key (seed, 0).
__device__ __forceinline__ void philox_block(uint64_t seed, uint64_t offset, uint64_t t, uint64_t (&c)[4]) {
  c[0] = offset + t;
  c[1] = c[0] < offset ? 1ull : 0ull;
  c[2] = c[3] = 0ull;
  philox4x64_10(c, seed, 0ull);
}

// The 16-bit draw of element e of a block's sixteen.
__device__ __forceinline__ uint32_t philox_draw(const uint64_t (&c)[4], int e) {
  return (uint32_t)(c[e >> 2] >> (16 * (e & 3))) & 0xFFFFu;
}

}  // namespace lora
