// fade_embed.hip — embedding lookup with scaling, and its gradient by sorted tokens (gfx950).
//
// Forward: y[i] = scale * E[t_i], one pass over the output, whose bytes bound it: 20011 tokens, width 1000, fp32 table, bf16 rows 15.4 us.
// Gradient: G[v] = scale * sum of dy[i] over t_i = v. Atomics would add the rows of a token in any order, and the result would
// differ from run to run; a decoder that repeats an encoder's training would leave it. So the positions are sorted by token first
// (stable, hence ascending in every token's run) and cut into pieces of equal length, each summed in order by one group of lanes. The sort moves a
// few words a token, the sums read dy once and write G once. 32768 tokens of 65536, width 2048, bf16: sort 25 us, sums 130 to 145 (671 MB at 4.6 to 5.2 TB/s: the
// memory bounds them), long runs 9. 262144 bytes, width 64, fp32: sort 16, sums 14 (67 MB), long runs 11: there launches and dependent loads are most of it.
// Tried and slower: no sort, but a table of the vocabulary in LDS for each wavefront, which adds its rows to it in order (96 us instead of 43: LDS takes 150 ns for 64
// float additions, and tables of 64 KB leave two wavefronts a compute unit to wait for them).
#include "../../include/fade.h"
#include "fade_op_rules.h"
#include "fade_ops.h"

namespace {
using namespace fade_op;

constexpr uint32_t NO_TOKEN = 0xffffffffu;
__device__ __forceinline__ uint32_t token_at(const OpTokens &t, size_t i, uint32_t vocab) {
  if (t.type == FADE_TOKEN_U8) {
    const uint32_t v = static_cast<const uint8_t *>(t.p)[i];
    return v < vocab ? v : NO_TOKEN;
  }
  if (t.type == FADE_TOKEN_I32) {
    const uint32_t v = static_cast<const uint32_t *>(t.p)[i];  // a negative one is past every vocabulary
    return v < vocab ? v : NO_TOKEN;
  }
  const uint64_t v = static_cast<const uint64_t *>(t.p)[i];
  return v < vocab ? (uint32_t)v : NO_TOKEN;
}

// 2^shift lanes on a row, 8 columns each
template <typename TT, typename TO>
__global__ __launch_bounds__(256) void embed_kernel(OpTokens t, size_t n, const TT *table, size_t table_ld, uint32_t vocab, int width, float scale,
                                                    TO *out, size_t out_ld, int shift) {
  for (size_t row = (size_t)blockIdx.x * (256 >> shift) + (threadIdx.x >> shift); row < n; row += (size_t)gridDim.x * (256 >> shift)) {
    const uint32_t v = token_at(t, row, vocab);
    for (int c = (threadIdx.x & ((1 << shift) - 1)) * 8; c < width; c += 8 << shift) {
      float x[8];
      OpRaw<TT> in;
      if (v != NO_TOKEN) in.load(table + v * table_ld + c, width - c, c);
      else in.zero();
      in.fix(width - c, c);
      in.get(x);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = v != NO_TOKEN ? x[k] * scale : 0.0f;
      OpRaw<TO> o;
      o.put(x);
      o.store(out + row * out_ld + c, width - c);
    }
  }
}

// ---------------------------------------------------------------------------------------------------
// The sort: least significant digit first, one or two passes of up to 10 bits. A workgroup counts the digits of its tile, a wavefront per
// digit adds the counts of the tiles in front, and the tiles' elements go to their places, in order.
// ---------------------------------------------------------------------------------------------------
// counts of the tile's digits; the first pass reads the tokens themselves and clears the flags of the tokens that occur
template <bool FIRST>
__global__ __launch_bounds__(256) void sort_count_kernel(OpTokens t, GradPlan p, const uint32_t *keys, const uint32_t *total, uint32_t *hist,
                                                         uint8_t *flags, int low) {
  __shared__ uint32_t count[MAX_DIGITS];
  const uint32_t digits = 1u << p.bits;
  for (uint32_t d = threadIdx.x; d < digits; d += 256) count[d] = 0;
  __syncthreads();
  const uint32_t n = FIRST ? p.n : total[MAX_DIGITS];
  const size_t begin = (size_t)blockIdx.x * (256 * SORT_ITEMS);
  uint32_t k[SORT_ITEMS];
#pragma unroll
  for (int i = 0; i < SORT_ITEMS; ++i) {
    const size_t at = begin + i * 256 + threadIdx.x;
    k[i] = at >= n ? NO_TOKEN : FIRST ? token_at(t, at, p.vocab) : keys[at];
  }
#pragma unroll
  for (int i = 0; i < SORT_ITEMS; ++i)
    if (k[i] != NO_TOKEN) atomicAdd(&count[(k[i] >> low) & (digits - 1)], 1u);
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < digits; d += 256) hist[(size_t)d * p.tiles + blockIdx.x] = count[d];
  if (FIRST) {
    uint4 *f = reinterpret_cast<uint4 *>(flags);
    const size_t words = ((size_t)p.vocab + 15) / 16;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < words; i += (size_t)gridDim.x * 256) f[i] = make_uint4(0, 0, 0, 0);
  }
}
// a wavefront per digit: counts of a tile -> counts of the tiles in front of it, and the digit's total
__global__ __launch_bounds__(256) void sort_scan_kernel(GradPlan p, uint32_t *hist, uint32_t *total) {
  const uint32_t d = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (d >= 1u << p.bits) return;
  uint32_t *h = hist + (size_t)d * p.tiles;
  uint32_t sum = 0;
  for (uint32_t i = 0; i < p.tiles; i += 64) {
    const uint32_t v = i + lane < p.tiles ? h[i + lane] : 0;
    const uint32_t upto = fade_lanes_scan(v);
    if (i + lane < p.tiles) h[i + lane] = sum + upto - v;
    sum += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
  }
  if (lane == 0) total[d] = sum;
}
// Every element to its place: the digits in front, the same digit in the tiles in front, in the wavefronts in front, and in front
// in its own wavefront, whose 64 elements at a time compare their digits bit by bit (ballots).
template <bool FIRST, bool LAST>
__global__ __launch_bounds__(256) void sort_place_kernel(OpTokens t, GradPlan p, const uint32_t *keys, const uint32_t *pos, const uint32_t *hist,
                                                         uint32_t *total, uint32_t *keys_out, uint32_t *pos_out, uint8_t *flags, int low) {
  __shared__ uint32_t count[4][MAX_DIGITS];  // per wavefront, then where its first element of the digit goes
  __shared__ uint32_t wave_sum[4];
  const uint32_t digits = 1u << p.bits;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, per = (int)((digits + 255) / 256);  // digits per thread, at most 4
  // everything that has to come from memory, at once
  const uint32_t n = FIRST ? p.n : total[MAX_DIGITS];
  const size_t begin = (size_t)blockIdx.x * (256 * SORT_ITEMS) + (size_t)wave * (64 * SORT_ITEMS);
  uint32_t key[SORT_ITEMS], at_pos[SORT_ITEMS], rank[SORT_ITEMS], all[4], front[4];
#pragma unroll
  for (int i = 0; i < SORT_ITEMS; ++i) {
    const size_t at = begin + i * 64 + lane;
    key[i] = NO_TOKEN;
    at_pos[i] = (uint32_t)at;
    if (at < n) {
      key[i] = FIRST ? token_at(t, at, p.vocab) : keys[at];
      if (!FIRST) at_pos[i] = pos[at];
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t d = tid * per + j;
    const bool in = j < per && d < digits;
    all[j] = in ? total[d] : 0;
    front[j] = in ? hist[(size_t)d * p.tiles + blockIdx.x] : 0;
  }
  for (uint32_t d = tid; d < digits; d += 256)
#pragma unroll
    for (int w = 0; w < 4; ++w) count[w][d] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < SORT_ITEMS; ++i) {
    const bool in = key[i] != NO_TOKEN;
    const uint32_t d = (key[i] >> low) & (digits - 1);
    uint64_t same = __ballot(in);
    for (int b = 0; b < p.bits; ++b) {
      const bool one = (d >> b) & 1;
      const uint64_t m = __ballot(one);
      same &= one ? m : ~m;
    }
    const uint64_t below = same & (((uint64_t)1 << lane) - 1);
    rank[i] = 0;
    if (in) rank[i] = count[wave][d] + (uint32_t)__popcll(below);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (in && below == 0) count[wave][d] += (uint32_t)__popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  // digits in front: an exclusive scan of the totals
  uint32_t sum = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) sum += all[j];
  const uint32_t upto = fade_lanes_scan(sum);
  if (lane == 63) wave_sum[wave] = upto;
  __syncthreads();
  uint32_t before = upto - sum;
  for (int w = 0; w < wave; ++w) before += wave_sum[w];
  if (FIRST && blockIdx.x == 0 && tid == 255) total[MAX_DIGITS] = before + sum;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t d = tid * per + j;
    if (j >= per || d >= digits) break;
    uint32_t to = before + front[j];
    before += all[j];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t c = count[w][d];
      count[w][d] = to;
      to += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < SORT_ITEMS; ++i)
    if (key[i] != NO_TOKEN) {
      const uint32_t to = count[wave][(key[i] >> low) & (digits - 1)] + rank[i];
      keys_out[to] = key[i];
      pos_out[to] = at_pos[i];
      if (LAST) flags[key[i]] = 1;
    }
}

// The sort in one launch, for up to 16384 tokens: every workgroup reads all of them, keeps those of its own range of the vocabulary, and knows how many
// lie in front of the range without asking another. Its wavefronts take consecutive parts of the tokens, 64 at a time, STEPS times; what each has
// counted of a token in front gives the places. They are taken in LDS, and the range leaves in order: half of a text's tokens are in the first range,
// and one compute unit's scattered stores of them took 30 us. The radix passes above are six launches of some four microseconds each there.
template <int STEPS>
__global__ __launch_bounds__(1024) void sort_ranges_kernel(OpTokens t, GradPlan p, uint32_t *total, uint32_t *keys_out, uint32_t *pos_out, uint8_t *flags) {
  __shared__ uint32_t count[16][RANGE_TOKENS];  // per wavefront, then where its first position of the token goes
  __shared__ uint32_t front[16], scans[16], total_here[1];
  extern __shared__ uint32_t sorted[];  // [n]: position and, above 16 bits, token of the range
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t low = blockIdx.x * p.range, span = p.vocab - low < p.range ? p.vocab - low : p.range;
  for (uint32_t d = tid; d < 16 * RANGE_TOKENS; d += 1024) count[d / RANGE_TOKENS][d % RANGE_TOKENS] = 0;
  uint32_t key[STEPS], rank[STEPS], below_range = 0;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const uint32_t at = (uint32_t)(wave * STEPS + i) * 64 + lane;
    key[i] = at < p.n ? token_at(t, at, p.vocab) : NO_TOKEN;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    below_range += key[i] < low ? 1 : 0;
    const uint32_t d = key[i] - low;
    const bool in = key[i] >= low && d < span;  // NO_TOKEN is past every range
    uint64_t same = __ballot(in);
    rank[i] = NO_TOKEN;
    if (!same) continue;
    for (int b = 0; b < p.range_bits; ++b) {
      const bool one = (d >> b) & 1;
      const uint64_t m = __ballot(one);
      same &= one ? m : ~m;
    }
    const uint64_t before = same & (((uint64_t)1 << lane) - 1);
    if (in) rank[i] = count[wave][d] + (uint32_t)__popcll(before);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (in && before == 0) count[wave][d] += (uint32_t)__popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  below_range = fade_lanes_sum(below_range);
  if (lane == 0) front[wave] = below_range;
  __syncthreads();
  // a thread per token: its positions, the tokens in front, and the range's start
  uint32_t mine = 0, start = 0;
  if (tid < RANGE_TOKENS)
    for (int w = 0; w < 16; ++w) mine += count[w][tid];
  const uint32_t upto = fade_lanes_scan(mine);
  if (lane == 63) scans[wave] = upto;
  __syncthreads();
  for (int w = 0; w < 16; ++w) start += front[w];
  const uint32_t first = start;
  start = 0;  // from here on within the range
  for (int w = 0; w < wave; ++w) start += scans[w];
  start += upto - mine;
  if (tid < RANGE_TOKENS) {
    if (tid < (int)span) flags[low + tid] = mine != 0;
    if (tid == RANGE_TOKENS - 1) total_here[0] = start + mine;
    for (int w = 0; w < 16; ++w) {
      const uint32_t c = count[w][tid];
      count[w][tid] = start;
      start += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < STEPS; ++i)
    if (rank[i] != NO_TOKEN) sorted[count[wave][key[i] - low] + rank[i]] = (uint32_t)(wave * STEPS + i) * 64 + lane | (key[i] - low) << 16;
  __syncthreads();
  const uint32_t have = total_here[0];
  if (tid == 0 && blockIdx.x == gridDim.x - 1) total[MAX_DIGITS] = first + have;
  for (uint32_t i = tid; i < have; i += 1024) {
    const uint32_t v = sorted[i];
    keys_out[first + i] = low + (v >> 16);
    pos_out[first + i] = v & 0xffffu;
  }
}

// ---------------------------------------------------------------------------------------------------
// The sums
// ---------------------------------------------------------------------------------------------------
struct SumArgs {
  const uint32_t *keys, *pos, *total;
  const uint8_t *flags;  // tokens that occur
  uint32_t clears;       // workgroups that write the rows of the others
  uint32_t *ends;        // of a token whose run reaches past the next piece: the piece it ends in
  const void *dout;
  size_t dout_ld;
  float scale;
  float *grad;
  size_t grad_ld;
  float *part;   // [pieces][2][part_ld]: a run that came from the piece in front; one that starts here and goes on
  int width, part_ld;
  uint32_t share;  // pieces per workgroup of the join, at most 16
  bool accumulate;
};
__device__ __forceinline__ void grad_put(const SumArgs &a, uint32_t v, int c, float x[8]) {
  float *dst = a.grad + v * a.grad_ld + c;
  OpRaw<float> o;
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] *= a.scale;
  if (a.accumulate) {
    float old[8];
    o.load(dst, a.width - c, c);
    o.fix(a.width - c, c);
    o.get(old);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] += old[k];
  }
  o.put(x);
  o.store(dst, a.width - c);
}
// Pieces of the sorted positions, one group of lanes each for a strip of columns. A run (the positions of one token) belongs to the piece it starts in, which
// follows it into the next piece if it ends there; a longer one leaves the sums of its parts to grad_join_kernel.
// FULL: a group of lanes is a wavefront; its positions and keys come with a few loads and go round as scalars.
// The first workgroups write zeros into the rows of tokens that do not occur, which is bounded by the memory's writes; the others wait for reads, and the two
// share the chip.
template <typename T, bool FULL> __global__ __launch_bounds__(256) void grad_sum_kernel(GradPlan p, SumArgs a) {
  const uint32_t lane = threadIdx.x & 63;
  if (blockIdx.x < a.clears) {  // p.clear_rows rows of the table per wavefront and turn
    const op_f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    const int lanes = 1 << p.shift, first = (threadIdx.x & (lanes - 1)) * 4, rows = 64 >> p.shift, mine = (int)lane >> p.shift;
    for (uint32_t v0 = (blockIdx.x * 4 + (threadIdx.x >> 6)) * p.clear_rows; v0 < p.vocab; v0 += a.clears * 4 * p.clear_rows) {
      const uint64_t absent = __ballot(lane < p.clear_rows && v0 + lane < p.vocab && !a.flags[v0 + lane]);
      for (int r = 0; r < (int)p.clear_rows; r += rows) {
        if (!(absent >> (r + mine) & 1)) continue;
        float *dst = a.grad + (size_t)(v0 + r + mine) * a.grad_ld;
        int c = first;
        for (; c + 4 <= a.width; c += lanes * 4) *reinterpret_cast<op_f32x4 *>(dst + c) = zero;
        for (int k = c; k < a.width && k < c + 4; ++k) dst[k] = 0.0f;
      }
    }
    return;
  }
  uint32_t g = (blockIdx.x - a.clears) * (256 >> p.shift) + (threadIdx.x >> p.shift);
  if constexpr (FULL) g = __builtin_amdgcn_readfirstlane(g);
  const uint32_t piece = g / p.strips, P = p.piece;
  const int c = ((g - piece * p.strips) << (p.shift + 3)) + (threadIdx.x & ((1 << p.shift) - 1)) * 8;
  const uint32_t n = a.total[MAX_DIGITS];
  const size_t first = (size_t)piece * P;
  if (first >= n || (!FULL && c >= a.width)) return;
  const uint32_t begin = (uint32_t)first, end = n - begin < P ? n : begin + P, last = n - 1;
  auto inside = [&](uint32_t i) { return i < last ? i : last; };
  // FULL: lane i has the i-th position of the piece and of the next one (at most 60 of them), and the keys at the borders
  uint32_t my_key = 0, my_pos = 0, next_key = 0, next_pos = 0;
  if constexpr (FULL) {
    const uint32_t at = inside(begin + (lane < P ? lane : P - 1)), next = inside(end + lane);
    my_key = a.keys[lane == 63 ? (begin > 0 ? begin - 1 : 0) : lane == 62 ? (begin > P ? begin - P - 1 : 0) : at];
    my_pos = a.pos[at];
    next_key = a.keys[next];
    next_pos = a.pos[next];
  }
  auto lane_of = [](uint32_t v, uint32_t i) { return (uint32_t)__builtin_amdgcn_readlane((int)v, (int)i); };
  auto key_at = [&](uint32_t i) { return FULL ? lane_of(my_key, i - begin) : a.keys[i]; };
  const uint32_t before = FULL ? lane_of(my_key, 63) : a.keys[begin > 0 ? begin - 1 : 0], far_before = FULL ? lane_of(my_key, 62) : a.keys[begin > P ? begin - P - 1 : 0];
  const uint32_t behind = FULL ? lane_of(next_key, 0) : a.keys[inside(end)], far_behind = FULL ? lane_of(next_key, P) : a.keys[inside(end + P)];
  const uint32_t last_key = key_at(end - 1);
  uint32_t cur = key_at(begin);
  bool came = begin > 0 && before == cur;
  const bool goes = end < n && behind == last_key;                                  // the last run does not end here
  const bool far = goes && end + P < n && far_behind == last_key;                   // nor in the next piece
  const bool from_far = came && begin > P && far_before == cur;                     // the first run does not start in the piece in front
  float acc[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  auto part = [&](int which, bool ended) {
    if (ended && c == 0) a.ends[cur] = piece;
    if (c >= a.width) return;
    OpRaw<float> o;
    o.put(acc);
    o.store(a.part + ((size_t)piece * 2 + which) * a.part_ld + c, 8);
  };
  constexpr uint32_t AHEAD = 8;  // rows on their way at a time
  const T *src = static_cast<const T *>(a.dout) + (c < a.width ? c : 0);
  const int left = c < a.width ? a.width - c : 8;
  uint32_t i = begin;
  if (came && !from_far && !(goes && last_key == cur)) {  // the piece in front follows its run to the end
    if constexpr (FULL) {
      const uint64_t other = __ballot(my_key != cur && lane < end - begin);
      i = other ? begin + (uint32_t)__builtin_ctzll(other) : end;
    } else {
      while (i < end && a.keys[i] == cur) ++i;
    }
    if (i == end) return;
    cur = key_at(i);
    came = false;
  }
  for (; i < end; i += AHEAD) {
    uint32_t key[AHEAD];
    OpRaw<T> row[AHEAD];
#pragma unroll
    for (uint32_t j = 0; j < AHEAD; ++j) {
      const uint32_t at = i + j < end ? i + j : end - 1;
      key[j] = key_at(at);
      row[j].load(src + (FULL ? lane_of(my_pos, at - begin) : a.pos[at]) * a.dout_ld, left, c);
    }
#pragma unroll
    for (uint32_t j = 0; j < AHEAD; ++j) {
      if (i + j >= end) break;
      if (key[j] != cur) {
        if (came) part(0, true);
        else if (c < a.width) grad_put(a, cur, c, acc);
        cur = key[j];
        came = false;
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[k] = 0.0f;
      }
      float x[8];
      row[j].fix(left, c);
      row[j].get(x);
#pragma unroll
      for (int k = 0; k < 8; ++k) acc[k] += x[k];
    }
  }
  if (came || far) {
    part(came ? 0 : 1, came && !goes);
    return;
  }
  if (goes) {  // into the next piece
    uint32_t stop = end;
    if constexpr (FULL) {
      const uint64_t other = __ballot(next_key != cur || end + lane >= n);
      stop = other ? end + (uint32_t)__builtin_ctzll(other) : end + 64;
    } else {
      while (stop < n && a.keys[stop] == cur) ++stop;
    }
    for (i = end; i < stop; i += AHEAD) {
      OpRaw<T> row[AHEAD];
#pragma unroll
      for (uint32_t j = 0; j < AHEAD; ++j) {
        const uint32_t at = i + j < stop ? i + j : stop - 1;
        row[j].load(src + (FULL ? lane_of(next_pos, at - end) : a.pos[at]) * a.dout_ld, left, c);
      }
#pragma unroll
      for (uint32_t j = 0; j < AHEAD; ++j) {
        if (i + j >= stop) break;
        float x[8];
        row[j].fix(left, c);
        row[j].get(x);
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[k] += x[k];
      }
    }
  }
  if (c < a.width) grad_put(a, cur, c, acc);
}
// The runs that reach past the next piece: the workgroup of the pieces they start in adds their parts, its groups of lanes in equal ranges of the pieces
// in between. A few pieces per workgroup; hardly any has such a run.
constexpr int JOIN_THREADS = 512;  // 262144 bytes: 11 us; of four parts on their way at a time, 13 with 512, 15 with 1024, 19 with 256 (16 parts: 13)
__global__ __launch_bounds__(JOIN_THREADS) void grad_join_kernel(GradPlan p, SumArgs a) {
  __shared__ __align__(16) float sums[JOIN_THREADS][8];
  constexpr uint32_t AHEAD = 8;
  const uint32_t block = blockIdx.x / p.strips, P = p.piece;
  const int strip = (int)(blockIdx.x - block * p.strips), group = threadIdx.x >> p.shift, groups = JOIN_THREADS >> p.shift;
  const int lane = threadIdx.x & ((1 << p.shift) - 1), c = (strip << (p.shift + 3)) + lane * 8;
  const uint32_t n = a.total[MAX_DIGITS];
  uint32_t key = 0;
  bool owner = false;
  {
    const size_t first = ((size_t)block * a.share + (threadIdx.x & 15)) * P, next = first + P;
    if ((threadIdx.x & 15) < a.share && next + P < n) {
      key = a.keys[next - 1];
      const uint32_t k0 = a.keys[first > 0 ? first - 1 : 0], k1 = a.keys[first], k2 = a.keys[next], k3 = a.keys[next + P];
      owner = k2 == key && k3 == key && !(k1 == key && first > 0 && k0 == key);
    }
  }
  for (uint32_t owners = (uint32_t)__ballot(owner) & 0xffffu; owners; owners &= owners - 1) {  // the same in every wavefront
    const uint32_t at_owner = (uint32_t)__builtin_ctz(owners), piece = block * a.share + at_owner;
    const uint32_t v = (uint32_t)__builtin_amdgcn_readlane((int)key, (int)at_owner);
    const uint32_t last = a.ends[v], count = last - piece, per = (count + groups - 1) / groups;
    float acc[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t from = piece + 1 + group * per, to = from + per < last + 1 ? from + per : last + 1;
    if (c < a.width) {
      if (group == 0) {
        OpRaw<float> o;
        o.load(a.part + ((size_t)piece * 2 + 1) * a.part_ld + c, 8);
        o.get(acc);
      }
      // several parts on their way together; past the last one it comes again, for nothing
      const float *src = a.part + c;
      const size_t step = (size_t)2 * a.part_ld;
      for (uint32_t i = from; i < to; i += AHEAD) {
        OpRaw<float> o[AHEAD];
#pragma unroll
        for (uint32_t j = 0; j < AHEAD; ++j) o[j].load(src + (i + j < to ? i + j : to - 1) * step, 8);
#pragma unroll
        for (uint32_t j = 0; j < AHEAD; ++j) {
          float x[8];
          o[j].get(x);
#pragma unroll
          for (int k = 0; k < 8; ++k) acc[k] += i + j < to ? x[k] : 0.0f;
        }
      }
    }
    // groups of one wavefront by exchanges, widest first, then the wavefronts in order
    const auto plus = [](float a, float b) { return a + b; };
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (p.shift <= 5) acc[k] = fade_level<32>(acc[k], plus);
      if (p.shift <= 4) acc[k] = fade_level<16>(acc[k], plus);
      if (p.shift <= 3) acc[k] = fade_level<8>(acc[k], plus);
      if (p.shift <= 2) acc[k] = fade_level<4>(acc[k], plus);
    }
    f32x4 *mine = reinterpret_cast<f32x4 *>(sums[threadIdx.x]);
    mine[0] = f32x4{acc[0], acc[1], acc[2], acc[3]};
    mine[1] = f32x4{acc[4], acc[5], acc[6], acc[7]};
    __syncthreads();
    if (group == 0 && c < a.width) {
      for (int w = 1; w < JOIN_THREADS / 64; ++w)
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[k] += sums[w * 64 + lane][k];
      grad_put(a, v, c, acc);
    }
    __syncthreads();
  }
}

}  // namespace

hipError_t fade_embed_launch(const OpTokens &t, size_t n, const OpMat &table, size_t vocab, size_t width, float scale, const OpMat &out, hipStream_t s) {
  const int shift = lanes_shift(width, 8), rows = 256 >> shift;
  const dim3 grid(row_blocks(n, rows));
  auto go = [&](auto *in, auto *to) {
    typedef std::remove_const_t<std::remove_pointer_t<decltype(in)>> TT;
    typedef std::remove_pointer_t<decltype(to)> TO;
    hipLaunchKernelGGL((embed_kernel<TT, TO>), grid, dim3(256), 0, s, t, n, in, table.ld, (uint32_t)vocab, (int)width, scale, to, out.ld, shift);
  };
  const float *tf = static_cast<const float *>(table.p);
  const bf16_t *tb = static_cast<const bf16_t *>(table.p);
  float *of = static_cast<float *>(const_cast<void *>(out.p));
  bf16_t *ob = static_cast<bf16_t *>(const_cast<void *>(out.p));
  if (table.f32 && out.f32) go(tf, of);
  else if (table.f32) go(tf, ob);
  else if (out.f32) go(tb, of);
  else go(tb, ob);
  return hipGetLastError();
}

size_t fade_embed_grad_bytes(size_t n, size_t vocab, size_t width) {
  const GradPlan p = grad_plan(n, vocab, width);
  return (size_t)p.pieces * p.strips > 0x7fffffff ? 0 : p.bytes;
}

hipError_t fade_embed_grad_launch(const OpTokens &t, size_t n, const OpMat &dout, float scale, float *grad, size_t grad_ld, size_t vocab, size_t width,
                                  bool accumulate, void *work, hipStream_t s) {
  const GradPlan p = grad_plan(n, vocab, width);
  uint8_t *w = static_cast<uint8_t *>(work);
  auto words = [&](size_t at) { return reinterpret_cast<uint32_t *>(w + at); };
  uint32_t *hist = words(p.hist), *total = words(p.total), *k0 = words(p.keys[0]), *p0 = words(p.pos[0]), *k1 = words(p.keys[1]), *p1 = words(p.pos[1]);
  uint8_t *flags = w + p.flags;
  const dim3 tiles(p.tiles), scans(((1u << p.bits) + 3) / 4), b(256);
  if (n == 0 && accumulate) return hipSuccess;
  if (p.range) {
    const dim3 ranges((p.vocab + p.range - 1) / p.range);
    auto *f = n <= 4096 ? sort_ranges_kernel<4> : n <= 8192 ? sort_ranges_kernel<8> : sort_ranges_kernel<16>;
    const size_t lds = (4 * n + 15) & ~(size_t)15;
    if (lds > 32 * 1024) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(f), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(f, ranges, dim3(1024), lds, s, t, p, total, k0, p0, flags);
  } else {
    hipLaunchKernelGGL(sort_count_kernel<true>, tiles, b, 0, s, t, p, nullptr, nullptr, hist, flags, 0);
    hipLaunchKernelGGL(sort_scan_kernel, scans, b, 0, s, p, hist, total);
    if (p.passes == 1) {
      hipLaunchKernelGGL((sort_place_kernel<true, true>), tiles, b, 0, s, t, p, nullptr, nullptr, hist, total, k0, p0, flags, 0);
    } else {
      hipLaunchKernelGGL((sort_place_kernel<true, false>), tiles, b, 0, s, t, p, nullptr, nullptr, hist, total, k1, p1, flags, 0);
      hipLaunchKernelGGL(sort_count_kernel<false>, tiles, b, 0, s, t, p, k1, total, hist, flags, p.bits);
      hipLaunchKernelGGL(sort_scan_kernel, scans, b, 0, s, p, hist, total);
      hipLaunchKernelGGL((sort_place_kernel<false, true>), tiles, b, 0, s, t, p, k1, p1, hist, total, k0, p0, flags, p.bits);
    }
  }
  const uint32_t groups = 256 >> p.shift, turns = (uint32_t)((vocab + 4 * p.clear_rows - 1) / (4 * p.clear_rows)), clears = accumulate ? 0 : turns < 512 ? turns : 512;
  const SumArgs a{k0, p0, total, flags, clears, words(p.ends), dout.p, dout.ld, scale, grad, grad_ld, reinterpret_cast<float *>(w + p.part), (int)width, (int)((width + 7) & ~(size_t)7),
                  p.share, accumulate};
  const dim3 sums(clears + (uint32_t)(((size_t)p.pieces * p.strips + groups - 1) / groups));
  auto *sum = dout.f32 ? (p.shift == 6 ? grad_sum_kernel<float, true> : grad_sum_kernel<float, false>)
                       : (p.shift == 6 ? grad_sum_kernel<bf16_t, true> : grad_sum_kernel<bf16_t, false>);
  hipLaunchKernelGGL(sum, sums, b, 0, s, p, a);
  if (p.pieces > 2)
    hipLaunchKernelGGL(grad_join_kernel, dim3((p.pieces + a.share - 1) / a.share * (uint32_t)p.strips), dim3(JOIN_THREADS), 0, s, p, a);
  return hipGetLastError();
}
