// fade_op_rules.h — how the operators cut their work: rules on sizes alone, as plain C++ (host tests compile them by themselves).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <initializer_list>

namespace fade_op {

// Workgroups of 256 for rows, `groups` at a time: one for each, up to 2^20 of them (a launch may have
// 2^32 lanes); the kernels go on in strides.
inline uint32_t row_blocks(size_t rows, int groups) {
  const size_t need = (rows + groups - 1) / groups;
  return (uint32_t)(need < ((size_t)1 << 20) ? need : (size_t)1 << 20);
}

struct GradPlan {
  int passes, bits;             // digits
  uint32_t n, vocab, tiles;
  int shift, strips;            // 2^shift lanes on a strip of columns, 8 each
  uint32_t piece, pieces;       // sorted positions summed by one group of lanes, at most 60
  uint32_t share;               // pieces that a workgroup looks over for runs to join, at most 16
  uint32_t clear_rows;          // of the gradient that a wavefront clears at a turn: a power of two, at least its groups of lanes
  uint32_t range;               // one-launch sort: tokens of the vocabulary per workgroup; 0: radix passes
  int range_bits;
  size_t keys[2], pos[2], hist, total, flags, ends, part, bytes;
};
constexpr int MAX_DIGITS = 1024, SORT_ITEMS = 4;  // elements per thread of a tile of 256 threads
constexpr int RANGE_TOKENS = 256;              // of a workgroup of the one-launch sort, at most

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
  p.tiles = n ? (uint32_t)((n + 256 * SORT_ITEMS - 1) / (256 * SORT_ITEMS)) : 1;
  // Every workgroup of the one-launch sort reads all the tokens, and the one with the frequent ones ranks most of them: up to 8192 of them by 512 workgroups, or
  // 16384 where a range has so few tokens that ranking them takes few comparisons. One launch | radix passes, us: 4096 of 32000 5.6 | 17; 16384 of 256 10.8 | 14;
  // 32768 of 65536 39 | 25.
  p.range = (uint32_t)((vocab + 255) / 256);
  if (p.range > RANGE_TOKENS) p.range = RANGE_TOKENS;
  if (n > (p.range <= 16 ? 16384 : 8192) || n * ((vocab + p.range - 1) / p.range) > (size_t)1 << 22) p.range = 0;
  while (((uint32_t)1 << p.range_bits) < p.range) ++p.range_bits;
  p.shift = lanes_shift(width, 6);
  p.clear_rows = 64;
  while (p.clear_rows > (64u >> p.shift) && vocab / p.clear_rows < 2048) p.clear_rows /= 2;
  p.strips = (int)((width + ((size_t)8 << p.shift) - 1) / ((size_t)8 << p.shift));
  // as many pieces as there are wavefronts for, but none so short that the partial sums at their borders cost more than the rows between
  const size_t want = n * p.strips >> (6 - p.shift);
  p.piece = (uint32_t)(want >= (size_t)1 << 18 ? 60 : want >= (size_t)1 << 16 ? 32 : want >= (size_t)1 << 15 ? 16 : 8);
  p.pieces = (uint32_t)((n + p.piece - 1) / p.piece);
  const size_t looks = ((size_t)p.pieces * p.strips + 1023) / 1024;
  p.share = looks > 16 ? 16 : looks < 1 ? 1 : (uint32_t)looks;
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
  p.ends = take(4 * vocab);
  p.part = take((size_t)2 * p.pieces * 4 * ((width + 7) & ~(size_t)7));
  p.bytes = at;
  return p;
}

// The weight gradient K x N over `rows` rows: tiles of the result, and equal ranges of the rows (units of 64) whose sums are added up behind it.
// Of tile sizes and counts of ranges the cheapest by a model of what was measured, in us: 256 x 256 tiles (fp32 dy: 256 x 128) take 1.85 (2.75) a unit with one
// workgroup per compute unit, 128 x 128 tiles 0.72 (1.6), or 1.45 with two of them; the first loads and the last stores 10 and 4; sums leave at 5.5 MB/us, and
// the launch that adds several takes 4.5 more. Measured in turn, the rule's choice | others: 16384 rows, 4096 x 2048, bf16 256 (large, 2) | 392 (large, 1), 349 (small, 1);
// 4096 rows, 1024 x 1024 26 (small, 4) | 33 (2), 27 (8), 33 (large, 8); 512 rows, 512 x 512 8.9 (small, 1) | 9.3 (2), 14.7 (large, 4); fp32, 16384 rows,
// 2048 x 2048 351 (large, 4, as many as the limit below asks for) | 342 (large, 2), 403 (small, 1); 1500 rows, 512 x 1000 19.2 (small, 8) | 18.0 (6), 18.9 (4),
// 22.6 (large, 8).
// A sum over thousands of rows in one fp32 accumulator drifts with its length: no range is longer than 16384 rows, 4096 with fp32 dy's three products a
// row, until there are 1024 ranges.
struct WgradPlan {
  bool large;
  int tiles_m, tiles_n, units, ranges, per;  // units of 64 rows; units in one range
};
inline WgradPlan wgrad_plan(size_t rows, size_t K, size_t N, bool f32) {
  const size_t units = (rows + 63) / 64, chain = f32 ? 64 : 256;
  WgradPlan best{};
  double least = 0;
  for (const bool large : {true, false}) {
    const size_t bm = large ? 256 : 128, bn = large && !f32 ? 256 : 128, tm = (K + bm - 1) / bm, tn = (N + bn - 1) / bn, tiles = tm * tn;
    for (size_t want = 1; want <= 1024 && (want == 1 || want <= units); want += want < 8 ? 1 : want / 4) {
      const size_t per = (units + want - 1) / want, r = per ? (units + per - 1) / per : 1;  // no range is empty
      if (per > chain && want + want / 4 <= 1024) continue;
      const bool pair = !large && !f32 && tiles * r > 256;
      const double unit = large ? (f32 ? 2.75 : 1.85) : f32 ? 1.6 : pair ? 1.45 : 0.72, bytes = 4.0 * K * N;
      const size_t rounds = (tiles * r + (pair ? 511 : 255)) / (pair ? 512 : 256);
      const double cost = (large ? 10.0 : 4.0) + rounds * per * unit + r * bytes / 5.5e6 + (r > 1 ? 4.5 + (r + 1) * bytes / 5.5e6 : 0.0);
      if (least == 0 || cost < least) {
        least = cost;
        best = WgradPlan{large, (int)tm, (int)tn, (int)units, (int)r, (int)per};
      }
      if (tiles * r > 1024 && per <= chain) break;  // more ranges only add sums
    }
  }
  return best;
}

// Lanes for a row of the join, 8 columns each, and the rows a workgroup has at a time.
struct JoinShape {
  int lanes, groups;
};
inline JoinShape join_shape(size_t width) {
  int lanes = 16;
  while ((size_t)lanes * 8 < width) lanes *= 2;
  return {lanes, lanes >= 256 ? 1 : 256 / lanes};
}
// Workgroups that take rows in turn. The gradient's keep their columns' sums in registers over all their rows, so that they are two per compute unit (one of
// 512 lanes and more). (As many fewer as give all of them equal turns: 1500 x 777 in 17.4 us instead of 14.4.)
inline int turn_blocks(size_t rows, int groups, size_t most) {
  const size_t need = (rows + groups - 1) / groups;
  return (int)(need < most ? need : most);
}
inline int grad_blocks(size_t rows, size_t width) {
  const JoinShape sh = join_shape(width);
  return turn_blocks(rows, sh.groups, sh.lanes >= 512 ? 256 : 512);
}

}  // namespace fade_op
