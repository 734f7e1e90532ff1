// fade_op_rules.h — how the operators cut their work: rules on sizes alone, as plain C++ (host tests compile them by themselves).
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace fade_op {

struct GradPlan {
  int passes, bits, items;      // digits; elements per thread of a tile of 256 threads
  uint32_t n, vocab, tiles;
  int shift, strips;            // 2^shift lanes on a strip of columns, 8 each
  uint32_t piece, pieces;       // sorted positions summed by one group of lanes
  size_t keys[2], pos[2], hist, total, flags, part, bytes;
};
constexpr int MAX_DIGITS = 1024;

inline int lanes_shift(size_t width, int most) {  // lanes for a row of this width: the least power of two that covers it, at most 2^most
  int s = 2;
  while (s < most && ((size_t)8 << s) < width) ++s;
  return s;
}
inline GradPlan grad_plan(size_t n, size_t vocab, size_t width) {
  GradPlan p{};
  int bits = 1;
  while (((size_t)1 << bits) < vocab) ++bits;
  p.passes = bits <= 10 ? 1 : 2;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.n = (uint32_t)n;
  p.vocab = (uint32_t)vocab;
  p.items = n <= ((size_t)1 << 17) ? 4 : 16;
  p.tiles = n ? (uint32_t)((n + 256 * p.items - 1) / (256 * p.items)) : 1;
  p.shift = lanes_shift(width, 6);
  p.strips = (int)((width + ((size_t)8 << p.shift) - 1) / ((size_t)8 << p.shift));
  p.piece = 32;
  p.pieces = (uint32_t)((n + p.piece - 1) / p.piece);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 15) & ~(size_t)15;
    return here;
  };
  for (int i = 0; i < p.passes; ++i) {
    p.keys[i] = take(4 * n);
    p.pos[i] = take(4 * n);
  }
  p.hist = take((size_t)4 * p.tiles << p.bits);
  p.total = take(4 * (MAX_DIGITS + 4));  // the digits' counts, then how many positions have a token at all
  p.flags = take(vocab);
  p.part = take((size_t)2 * p.pieces * 4 * ((width + 7) & ~(size_t)7));
  p.bytes = at;
  return p;
}

constexpr int WT = 128;  // tile of a weight gradient: WT x WT on four wavefronts
struct WgradPlan {
  int tiles_m, tiles_n, units, ranges, per;
};
// Ranges of the rows: as many as fill the chip where the tiles do not, and so many that no fp32 sum runs over more than 16384 products' worth
// of rows (4096 where three terms each are added).
inline WgradPlan wgrad_plan(size_t rows, size_t K, size_t N, bool f32) {
  WgradPlan p{};
  p.tiles_m = (int)((K + WT - 1) / WT);
  p.tiles_n = (int)((N + WT - 1) / WT);
  p.units = (int)((rows + 63) / 64);
  const size_t tiles = (size_t)p.tiles_m * p.tiles_n, chain = f32 ? 64 : 256;
  size_t r = tiles >= 512 ? 1 : 512 / tiles;
  if (r > (size_t)p.units) r = p.units;
  if (r < (p.units + chain - 1) / chain) r = (p.units + chain - 1) / chain;
  r = r < 1 ? 1 : r > 1024 ? 1024 : r;
  p.per = (int)((p.units + r - 1) / r);
  p.ranges = p.per ? (p.units + p.per - 1) / p.per : 1;
  return p;
}

// Lanes for a row: 8 columns each, from 16 to a workgroup of 1024; two steps of 8 columns above 8192.
struct JoinShape {
  int L, V, groups;
};
inline JoinShape join_shape(size_t width) {
  int L = 16;
  while (L < 1024 && (size_t)L * 8 < width) L *= 2;
  return {L, (size_t)L * 8 < width ? 2 : 1, L >= 256 ? 1 : 256 / L};
}
inline int grad_blocks(size_t rows, size_t width) {
  const JoinShape sh = join_shape(width);
  const size_t need = (rows + sh.groups - 1) / sh.groups, most = sh.L >= 512 ? 256 : 512;
  return (int)(need < most ? need : most);
}

}  // namespace fade_op
