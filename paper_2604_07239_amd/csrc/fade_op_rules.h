// fade_op_rules.h — how the operators cut their work: rules on sizes alone, as plain C++ (host tests compile them by themselves).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <initializer_list>

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

// The weight gradient K x N over `rows` rows: tiles of the result, and equal ranges of the rows (units of 64) whose sums are added up behind it.
struct WgradPlan {
  bool large;  // tiles of 256 x 256 (fp32 dy: 256 x 128), one workgroup of eight wavefronts per compute unit; else 128 x 128
  int tiles_m, tiles_n, units, ranges, per;
};
inline WgradPlan wgrad_plan(size_t rows, size_t K, size_t N, bool f32) {
  const size_t units = (rows + 63) / 64, chain = f32 ? 64 : 256;  // units that one fp32 sum may run over
  WgradPlan best{};
  double least = 0;
  for (const bool large : {true, false}) {
    const size_t bm = large ? 256 : 128, bn = large && !f32 ? 256 : 128, tm = (K + bm - 1) / bm, tn = (N + bn - 1) / bn, tiles = tm * tn;
    for (size_t want = 1; want <= 1024 && (want == 1 || want <= units); want += want < 8 ? 1 : want / 4) {
      const size_t per = (units + want - 1) / want, r = per ? (units + per - 1) / per : 1;  // no range is empty
      if (per > chain && want + want / 4 <= 1024) continue;
      // cost in microseconds
      const size_t at_once = 256 * (large || f32 ? 1 : 2), rounds = (tiles * r + at_once - 1) / at_once;
      const double unit = (large ? (f32 ? 2.7 : 1.8) : (f32 ? 1.4 : 1.0)), add = r > 1 ? 3.0 + (double)(r + r + 1) * K * N * 4 / 4e6 : 0.0;
      const double cost = rounds * (per * unit + 3.0) + add;
      if (least == 0 || cost < least) {
        least = cost;
        best = WgradPlan{large, (int)tm, (int)tn, (int)units, (int)r, (int)per};
      }
      if (tiles * r > 4 * 256 && per <= chain) break;
    }
  }
  return best;
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
