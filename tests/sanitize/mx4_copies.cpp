// What the 4-bit tiles copy into LDS, address by address, for ragged shapes: every
// lane of every copy either lies past its operand by its lane offset alone (and so
// reads nothing) or stays inside it with its scalar offset; and no scalar offset
// passes the operand's size, so that the size less the scalar offset, which the
// hardware may compare the lane's with, does not wrap.  Host only; built with the
// sanitizers by tests/test_mx4_copies.py.
#include <stdint.h>
#include <stdio.h>

#include "lora_ops.hpp"

using namespace lora;

static long copies = 0, outside = 0;

static void one(const char* what, uint64_t lane, uint64_t scalar, uint64_t bytes, uint64_t size, long m, long n, long k) {
  ++copies;
  const bool none = lane >= size, inside = lane + scalar + bytes <= size;
  if ((none || inside) && scalar <= size) return;
  if (outside++ < 10)
    fprintf(stderr, "%ld x %ld x %ld: %s at lane %lu + scalar %lu of %lu bytes\n", m, n, k, what, (unsigned long)lane,
            (unsigned long)scalar, (unsigned long)size);
}

// Copies of a tile of bm x bn by nw waves, `stages` slabs ahead: 8 rows of X or W
// each, or half a cell of scales where those go through LDS.
static void tile(int bm, int bn, int nw, int stages, bool lds_scales, int m, int n, int k, int m0, int n0) {
  const int slabs = (int)mx4_slabs(k), gx = (int)mx4_groups(m), gw = (int)mx4_groups(n);
  const uint64_t row = (uint64_t)slabs * 128;
  const uint64_t xsize = (uint64_t)(m - m0 < bm ? m - m0 : bm) * row, wsize = (uint64_t)(n - n0 < bn ? n - n0 : bn) * row;
  const int xcells = bm / 64, cells = xcells + bn / 64, per = lds_scales ? (2 * cells + nw - 1) / nw : 0;
  for (int kb = 0; kb < slabs + stages; ++kb) {
    const Mx4Slab s = mx4_slab(kb, slabs);
    for (int r = 0; r < bm; ++r) one("X", (uint32_t)(r * row) | s.none, s.kb * 128, 128, xsize, m, n, k);
    for (int r = 0; r < bn; ++r) one("W", (uint32_t)(r * row) | s.none, s.kb * 128, 128, wsize, m, n, k);
    for (int h = 0; h < per * nw; ++h) {
      const int c = h >> 1;
      const bool isx = c < xcells;
      const Mx4Cell at = c < cells ? mx4_cell(isx ? m0 / 64 + c : n0 / 64 + c - xcells, isx ? gx : gw) : Mx4Cell{0, 0, kMx4None};
      one(isx ? "X's scales" : "W's scales", (at.none | s.none), at.first + s.kb * at.step + (h & 1) * 256, 256,
          (uint64_t)(isx ? gx : gw) * slabs * 512, m, n, k);
    }
  }
}

int main() {
  const struct {
    int bm, bn, nw, stages;
    bool lds_scales;
  } tiles[4] = {{256, 256, 8, 2, false}, {256, 128, 8, 3, true}, {128, 128, 4, 4, true}, {64, 128, 2, 3, true}};
  for (const auto& t : tiles)
    for (int m : {1, 17, 63, 64, 65, 128, 129, 200, 256, 257, 321, 511})
      for (int n : {8, 64, 72, 128, 136, 200, 256, 264, 392})
        for (int k : {8, 256, 264, 776, 1032})
          for (int m0 = 0; m0 < m; m0 += t.bm)
            for (int n0 = 0; n0 < n; n0 += t.bn) tile(t.bm, t.bn, t.nw, t.stages, t.lds_scales, m, n, k, m0, n0);
  printf("copies %ld, outside %ld\n", copies, outside);
  return outside != 0;
}
