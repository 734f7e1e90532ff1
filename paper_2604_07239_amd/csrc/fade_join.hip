// fade_join.hip — the join of a block with the residual stream: z = N_u(u), h = lam r + sigma(g) z, n = N_n(h), and its gradient (gfx950).
//
// A row stays in the registers of the L lanes that own it (8 columns per lane), so each pass reads its operands once and writes its
// results once, whatever norms and gate there are; the bytes bound it: 16384 x 2048, fp32 stream, bf16 branch 89 us forward (470 MB, 5.2 TB/s); bf16 103 us backward
// (537 MB). The backward pass forms the statistics again instead of reading saved ones, from the operands themselves or from 8-bit checkpoints of them
// (8192 x 4096: 120 us, 440 MB: there the two exchanges a row are as long as its bytes).
// LayerNorm's variance is the mean of the squares of centred values: the difference of E[x^2] and mean^2 loses what a large mean covers.
// Parameter gradients are sums over the rows: a workgroup keeps its columns' sums in registers over all its rows and leaves one partial sum per column,
// which a second kernel adds in order (4 to 5 us). No atomics.
// With 8 columns a lane, what a row costs once (exchanges, reciprocals) is half of the vector instructions: sums by DPP shifts, one exchange for several of them and v_rsq
// took the gradient of 16384 x 2048 from 142 to 103 us. Rows of 1024 lanes (4097 to 8192 columns) have 128 registers a lane, and their gradient
// spills 44 to 72 of them: 4096 x 8192, bf16 100 us forward (with three checkpoints 127), 286 backward, 245 from checkpoints.
// Tried and no faster: two rows on their way instead of one (118 | 118), LDS sums on rows of 512 lanes (118 | 203).
#include <type_traits>

#include "../../include/fade.h"
#include "fade_op_rules.h"
#include "fade_ops.h"

namespace {
using namespace fade_op;

constexpr int most(int a, int b) { return a > b ? a : b; }

// Sum over the L lanes of a row in this wavefront: 64 lanes by shifts inside the rows of 16 and broadcasts of their last lanes (one add each) into lane 63,
// fewer lanes by a butterfly.
template <int L> __device__ __forceinline__ float wave_total(float v) {
  if constexpr (L < 64) return fade_lanes_sum<L>(v);
  auto add = [&](auto ctrl, auto rows) { v += __builtin_bit_cast(float, fade_dpp<decltype(ctrl)::value, decltype(rows)::value>(fade_bits(v))); };
  typedef std::integral_constant<int, 0xf> All;
  add(std::integral_constant<int, 0x111>{}, All{});
  add(std::integral_constant<int, 0x112>{}, All{});
  add(std::integral_constant<int, 0x114>{}, All{});
  add(std::integral_constant<int, 0x118>{}, All{});
  add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
  add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane((int)fade_bits(v), 63));
}
// s / n from a reciprocal good to an ulp: the remainder's quotient makes up for it (a row of equal values has exactly that mean)
__device__ __forceinline__ float quotient(float s, float n, float inv) {
  const float q = s * inv;
  return fmaf(fmaf(-n, q, s), inv, q);
}
// What the L lanes of a row know together. Above a wavefront its values pass through LDS: one barrier for four of them, in two places in turn (a wavefront may be
// one exchange ahead of another, never two).
template <int L> struct RowSums {
  static constexpr int W = L >= 64 ? L / 64 : 1, GROUPS = L >= 256 ? 1 : 256 / L;  // wavefronts of a row; rows of a workgroup
  typedef float Lds[2][GROUPS][4][W];
  Lds &lds;
  int group, wave, width, place = 0;
  float inv = 1.0f / (float)width;
  float mine = W > 1 ? fmaxf(columns(wave), 1.0f) : (float)width, inv_mine = 1.0f / mine, theirs = columns(threadIdx.x % W);  // theirs: the wavefront's that this lane reads
  __device__ __forceinline__ float columns(int w) const {  // of the row's w-th wavefront
    const int have = width - w * 512, span = (L < 64 ? L : 64) * 8;
    return (float)(have < 0 ? 0 : have > span ? span : have);
  }
  // in: this wavefront's values; out: in lane i those of the row's (i % W)-th wavefront
  template <int N> __device__ __forceinline__ void exchange(float (&v)[N]) {
    if constexpr (W > 1) {
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) lds[place][group][i][wave] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = lds[place][group][i][threadIdx.x % W];
      place ^= 1;
    }
  }
  __device__ __forceinline__ float over_waves(float v) const {  // sum of what exchange() left in the lanes
    auto add = [](float a, float b) { return a + b; };
    if constexpr (W >= 16) v = fade_level<8>(v, add);
    if constexpr (W >= 8) v = fade_level<4>(v, add);
    if constexpr (W >= 4) v = fade_level<2>(v, add);
    if constexpr (W >= 2) v = fade_level<1>(v, add);
    return v;
  }
  // A row's statistics in two parts: this wavefront's mean m (LayerNorm, else 0) and sum q of squared distances from it; and, of what exchange() left of
  // them, the row's mean and 1 / sigma: no difference of large squares anywhere.
  template <bool WHOLE> __device__ __forceinline__ void part(int norm, const float (&x)[8], int left, float &m, float &q) const {
    m = 0.0f;
    q = 0.0f;
    if (norm == FADE_NORM_LAYER) {
      float s = 0.0f;
#pragma unroll
      for (int k = 0; k < 8; ++k) s += x[k];  // columns that do not exist hold zeros
      m = quotient(wave_total<L>(s), mine, inv_mine);
      if (WHOLE || left >= 8 || left <= 0) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float d = x[k] - m;
          q = fmaf(d, d, q);
        }
        q = left > 0 ? q : 0.0f;
      } else {
#pragma unroll
        for (int k = 0; k < 7; ++k) {
          const float d = x[k] - m;
          if (k < left) q = fmaf(d, d, q);
        }
      }
    } else if (norm == FADE_NORM_RMS) {
#pragma unroll
      for (int k = 0; k < 8; ++k) q = fmaf(x[k], x[k], q);
    }
    q = wave_total<L>(q);
  }
  __device__ __forceinline__ void whole(int norm, float m, float q, float eps, float &mean, float &rstd) const {
    mean = W > 1 ? quotient(over_waves(m * theirs), (float)width, inv) : m;
    const float d = m - mean, sq = over_waves(W > 1 ? fmaf(d * theirs, d, q) : q);  // in this order: d^2 may be past fp32 where a wavefront has no columns
    rstd = norm == FADE_NORM_NONE ? 1.0f : __builtin_amdgcn_rsqf(fmaf(sq, inv, eps));  // good to an ulp
  }
};
// The factor of (x - mean) where a row is normalised: 1 / sigma. Columns that do not exist hold x = 0 there, and where mean / sigma is past fp32 they would put an infinity, and
// their parameters' zeros a NaN, into the row's sums. Such a row is level, its variance far below the square of mean's last place, so that every x - mean is zero
// and any factor right: zero. A NaN stays one.
__device__ __forceinline__ float factor(float rstd, float mean) { return fabsf(mean) * rstd > 1e38f ? 0.0f : rstd; }

// 8 columns of a parameter; `otherwise` where there is none, zeros past the row's end
__device__ __forceinline__ void param8(const float *p, float otherwise, int c, int left, float x[8]) {
  if (left <= 0 || !p) {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = k < left ? otherwise : 0.0f;
  } else {
    OpRaw<float> r;
    r.load(p + c, left, c);
    r.fix(left, c);
    r.get(x);
  }
}
// A parameter's columns of this lane: held in registers over all the rows, or, on rows of 1024 lanes, whose workgroup has 128 registers a lane, fetched
// from the caches at each use.
template <bool HELD> struct Param {
  const float *p;
  float otherwise, held[HELD ? 8 : 1];
  int c, left;
  __device__ __forceinline__ Param(const float *p_, float o, int c_, int left_) : p(p_), otherwise(o), c(c_), left(left_) {
    if constexpr (HELD) param8(p, otherwise, c, left, held);
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    if constexpr (HELD) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = held[k];
    } else {
      param8(p, otherwise, c, left, x);
    }
  }
};
// sigma(x) = 1 / (1 + exp(-x)); fade_sigmoid's reciprocal is the hardware's, good to an ulp
__device__ __forceinline__ float sigma(float x) { return fade_sigmoid(x); }

template <int L> struct Lane {  // the same row for a whole wavefront is known to be one: addresses of rows are scalar then
  int group, lane, c, left;
  __device__ __forceinline__ Lane(int width) {
    group = L >= 256 ? 0 : L >= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / L) : threadIdx.x / L;
    lane = threadIdx.x % L;
    c = lane * 8;
    left = width - c;
  }
  __device__ __forceinline__ int wave() const { return L > 64 ? __builtin_amdgcn_readfirstlane(lane / 64) : 0; }
};
// 8 columns that have arrived, in their places (rows of whole pieces: there they are)
template <bool WHOLE, int L, typename R> __device__ __forceinline__ R &arrived(R &raw, const Lane<L> &l) {
  if constexpr (!WHOLE) raw.fix(l.left, l.c);
  return raw;
}
// how many of 8 columns to move: all of them on rows of whole pieces
template <bool WHOLE> __device__ __forceinline__ int op_left(int left) { return WHOLE ? 8 : left; }

__device__ __forceinline__ void keep_row(uint8_t *keep, int rows, int width, size_t row, bool in, const float (&x)[8], int c) {
  const int groups = (width + 31) / 32;
  uint32_t exp;
  const uint2 w = op_keep_pack(x, exp);
  if (in && c < groups * 32) {
    *reinterpret_cast<uint2 *>(keep + row * groups * 32 + c) = w;
    if ((threadIdx.x & 3) == 0) keep[(size_t)rows * groups * 32 + row * groups + (c >> 5)] = (uint8_t)exp;
  }
}

// A workgroup takes rows in strides of the grid. The next rows' operands are on their way while it works on these, and u's statistics of the next rows pass
// through the same exchange as h's of these: one barrier a row. WHOLE: the width is a multiple of 8. KEEP: it can write checkpoints; rows of 1024 lanes have a kernel without
// them, whose registers then hold all of a lane's values (4096 x 8192: fp32 196 us with their code, 163 without; bf16 101, 99).
template <int L, typename TS, typename TB, bool WHOLE, bool KEEP = true> __global__ __launch_bounds__(most(L, 256)) void join_kernel(JoinArgs a) {
  typedef RowSums<L> Sums;
  typedef Param<(L <= 512)> P;
  __shared__ __align__(16) typename Sums::Lds lds;
  const Lane<L> l(a.width);
  Sums rs{lds, l.group, l.wave(), a.width};
  const P gu(a.gamma_u, 1.0f, l.c, l.left), bu(a.beta_u, 0.0f, l.c, l.left), gn(a.gamma_n, 1.0f, l.c, l.left), bn(a.beta_n, 0.0f, l.c, l.left),
      lam(a.lam_count == 1 ? nullptr : a.lam, a.lam_count == 1 ? a.lam[0] : 1.0f, l.c, l.left);
  OpRaw<TS> raw_r;
  OpRaw<TB> raw_u, raw_g;
  raw_r.zero(); raw_u.zero(); raw_g.zero();  // and so they stay in lanes past the row's end
  auto load = [&](size_t row) {              // past the last row: that one again
    if (row >= (size_t)a.rows) row = a.rows - 1;
    if (l.left > 0) {
      const int left = op_left<WHOLE>(l.left);
      raw_r.load(static_cast<const TS *>(a.r) + row * a.r_ld + l.c, left, l.c);
      raw_u.load(static_cast<const TB *>(a.u) + row * a.u_ld + l.c, left, l.c);
      if (a.g) raw_g.load(static_cast<const TB *>(a.g) + row * a.g_ld + l.c, left, l.c);
    }
  };
  const bool has_n = a.n || (KEEP && a.keep_n);
  const int norm_n = has_n ? a.norm_n : FADE_NORM_NONE;
  uint32_t base = blockIdx.x * Sums::GROUPS;
  float x[8], mean_u, rstd_u;
  load(base + l.group);
  arrived<WHOLE>(raw_u, l).get(x);
  {
    float v[2];
    rs.template part<WHOLE>(a.norm_u, x, l.left, v[0], v[1]);
    if (a.norm_u != FADE_NORM_NONE) rs.exchange(v);
    rs.whole(a.norm_u, v[0], v[1], a.eps, mean_u, rstd_u);
  }
  for (; base < (uint32_t)a.rows; base += gridDim.x * Sums::GROUPS) {
    const size_t row = base + l.group;
    const bool in = Sums::GROUPS == 1 || row < (size_t)a.rows;  // the workgroup's barriers are for all its rows
    float h[8], g[8], p[8], q[8];
    arrived<WHOLE>(raw_r, l).get(h); arrived<WHOLE>(raw_g, l).get(g);
    load(row + gridDim.x * Sums::GROUPS);
    if (KEEP && a.keep_r) keep_row(a.keep_r, a.rows, a.width, row, in, h, l.c);
    if (KEEP && a.keep_u) keep_row(a.keep_u, a.rows, a.width, row, in, x, l.c);
    if (KEEP && a.keep_g) keep_row(a.keep_g, a.rows, a.width, row, in, g, l.c);
    if (a.norm_u != FADE_NORM_NONE) {
      const float by = factor(rstd_u, mean_u);
      gu.get(p); bu.get(q);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = fmaf((x[k] - mean_u) * by, p[k], q[k]);
    }
    lam.get(p);
#pragma unroll
    for (int k = 0; k < 8; ++k) h[k] = fmaf(p[k], h[k], a.g ? sigma(g[k]) * x[k] : x[k]);
    if (in && l.left > 0) {
      OpRaw<TS> o;
      o.put(h);
      o.store(static_cast<TS *>(a.h) + row * a.h_ld + l.c, op_left<WHOLE>(l.left));
    }
    float v[4], mean, rstd;
    rs.template part<WHOLE>(norm_n, h, l.left, v[0], v[1]);
    arrived<WHOLE>(raw_u, l).get(x);
    rs.template part<WHOLE>(a.norm_u, x, l.left, v[2], v[3]);
    rs.exchange(v);
    rs.whole(norm_n, v[0], v[1], a.eps, mean, rstd);
    rs.whole(a.norm_u, v[2], v[3], a.eps, mean_u, rstd_u);
    if (!has_n) continue;
    if (norm_n != FADE_NORM_NONE) {
      const float by = factor(rstd, mean);
      gn.get(p); bn.get(q);
#pragma unroll
      for (int k = 0; k < 8; ++k) h[k] = fmaf((h[k] - mean) * by, p[k], q[k]);
    }
    OpRaw<TB> o;
    o.put(h);
    if (a.n && in && l.left > 0) o.store(static_cast<TB *>(a.n) + row * a.n_ld + l.c, op_left<WHOLE>(l.left));
    if (KEEP && a.keep_n) {
      o.get(h);  // a checkpoint of n is one of the values as rounded
      keep_row(a.keep_n, a.rows, a.width, row, in, h, l.c);
    }
  }
}

// ---------------------------------------------------------------------------------------------------
// The gradient
// ---------------------------------------------------------------------------------------------------
// partial sums of the parameters' gradients: [workgroup][5][width rounded up to 8]; one value of lam: its sum at the first column
enum { PART_GU = 0, PART_BU, PART_GN, PART_BN, PART_LAM, PARTS };
__host__ __device__ inline size_t part_width(int width) { return (size_t)((width + 7) / 8 * 8); }

template <typename T> struct SavedRaw {  // 8 columns of a saved operand: as it was
  OpRaw<T> v;
  __device__ __forceinline__ void zero() { v.zero(); }
  __device__ __forceinline__ void load(const void *p, size_t ld, int, int, size_t row, int c, int left) { v.load(static_cast<const T *>(p) + row * ld + c, left, c); }
  __device__ __forceinline__ void fix(int left, int c) { v.fix(left, c); }
  __device__ __forceinline__ void get(float x[8]) const { v.get(x); }
};
struct SavedKeep {  // or from its checkpoint
  uint2 q;
  uint32_t e;
  __device__ __forceinline__ void zero() { q = make_uint2(0, 0); e = 0; }
  __device__ __forceinline__ void load(const void *p, size_t, int rows, int width, size_t row, int c, int) {
    const int groups = (width + 31) / 32;
    const uint8_t *k = static_cast<const uint8_t *>(p);
    q = *reinterpret_cast<const uint2 *>(k + row * groups * 32 + c);
    e = k[(size_t)rows * groups * 32 + row * groups + (c >> 5)];
  }
  __device__ __forceinline__ void fix(int, int) {}
  __device__ __forceinline__ void get(float x[8]) const { op_keep_unpack(q, op_keep_unit(e), x); }
};

// A lane's sums over its rows, 8 columns of a parameter: in registers; on rows of 1024 lanes those of the norms' parameters in LDS (128 KB: a row's bytes take
// the memory longer than these sums take LDS).
template <int L> struct Sums8 {
  static constexpr bool LDS = L > 512;
  float reg[LDS ? 1 : PARTS][8];
  f32x4 *lds;  // [4][2][L]
  __device__ __forceinline__ void clear(unsigned char *mem) {
    lds = reinterpret_cast<f32x4 *>(mem) + threadIdx.x;
#pragma unroll
    for (int p = 0; p < (LDS ? 1 : PARTS); ++p)
#pragma unroll
      for (int k = 0; k < 8; ++k) reg[p][k] = 0.0f;
    if constexpr (LDS)
#pragma unroll
      for (int i = 0; i < 8; ++i) lds[i * L] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  template <int P, typename F> __device__ __forceinline__ void update(F &&f) {  // f(sum, column)
    if constexpr (LDS && P != PART_LAM) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x4 v = lds[(P * 2 + h) * L];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = f(v[k], h * 4 + k);
        lds[(P * 2 + h) * L] = v;
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) reg[LDS ? 0 : P][k] = f(reg[LDS ? 0 : P][k], k);
    }
  }
};
template <int L, typename TS, typename TB, bool KEPT, bool WHOLE> __global__ __launch_bounds__(most(L, 256)) void join_grad_kernel(JoinArgs a) {
  typedef RowSums<L> Sums;
  typedef Param<(L <= 512)> P;
  typedef std::conditional_t<KEPT, SavedKeep, SavedRaw<TS>> RawS;
  typedef std::conditional_t<KEPT, SavedKeep, SavedRaw<TB>> RawB;
  constexpr int GROUPS = Sums::GROUPS;
  __shared__ __align__(16) typename Sums::Lds lds;
  __shared__ __align__(16) float fold[GROUPS > 1 ? 256 * 8 : 4];
  const Lane<L> l(a.width);
  Sums rs{lds, l.group, l.wave(), a.width};
  const P gu(a.gamma_u, 1.0f, l.c, l.left), bu(a.beta_u, 0.0f, l.c, l.left), gn(a.gamma_n, 1.0f, l.c, l.left),
      lam(a.lam_count == 1 ? nullptr : a.lam, a.lam_count == 1 ? a.lam[0] : 1.0f, l.c, l.left);
  extern __shared__ __align__(16) unsigned char dynamic[];
  Sums8<L> part;
  part.clear(dynamic);
  const void *src_r = KEPT ? a.keep_r : a.r, *src_u = KEPT ? a.keep_u : a.u, *src_g = KEPT ? a.keep_g : a.g;
  RawS raw_r;
  RawB raw_u, raw_g;
  OpRaw<TS> raw_dh;
  OpRaw<TB> raw_dn;
  auto none = [&] { raw_r.zero(); raw_u.zero(); raw_g.zero(); raw_dh.zero(); raw_dn.zero(); };
  none();  // and so they stay in lanes past the row's end
  auto load = [&](size_t row) {  // past the last row: that one again
    if (row >= (size_t)a.rows) row = a.rows - 1;
    if (l.left > 0) {
      const int left = op_left<WHOLE>(l.left);
      raw_r.load(src_r, a.r_ld, a.rows, a.width, row, l.c, left);
      raw_u.load(src_u, a.u_ld, a.rows, a.width, row, l.c, left);
      if (src_g) raw_g.load(src_g, a.g_ld, a.rows, a.width, row, l.c, left);
      if (a.dh) raw_dh.load(static_cast<const TS *>(a.dh) + row * a.dh_ld + l.c, left, l.c);
      if (a.dn) raw_dn.load(static_cast<const TB *>(a.dn) + row * a.dn_ld + l.c, left, l.c);
    }
  };
  // Two exchanges a row: h's statistics with the sums of N_n's gradient, and the sums of N_u's with u's statistics of the next row.
  uint32_t base = blockIdx.x * GROUPS;
  float uhat[8], mean_u, rstd_u;
  load(base + l.group);
  arrived<WHOLE>(raw_u, l).get(uhat);
  {
    float v[2];
    rs.template part<WHOLE>(a.norm_u, uhat, l.left, v[0], v[1]);
    rs.exchange(v);
    rs.whole(a.norm_u, v[0], v[1], a.eps, mean_u, rstd_u);
  }
  for (; base < (uint32_t)a.rows; base += gridDim.x * GROUPS) {
    const size_t row = base + l.group;
    const bool in = GROUPS == 1 || row < (size_t)a.rows;
    // forward again: uhat, z, sigma(g), h
    float z[8], sg[8], r[8], t[8], e[8], w[8];
    arrived<WHOLE>(raw_r, l).get(r); arrived<WHOLE>(raw_g, l).get(sg); arrived<WHOLE>(raw_dh, l).get(t); arrived<WHOLE>(raw_dn, l).get(e);
    load(row + gridDim.x * GROUPS);
    if (!in) {  // a row that is not there adds zeros; its statistics are the last row's, and nothing times them is to be anything else
#pragma unroll
      for (int k = 0; k < 8; ++k) r[k] = sg[k] = t[k] = e[k] = uhat[k] = 0.0f;
      mean_u = rstd_u = 0.0f;
    }
    if (a.norm_u != FADE_NORM_NONE) {
      const float by = factor(rstd_u, mean_u);
      float q[8];
      gu.get(w); bu.get(q);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        uhat[k] = (uhat[k] - mean_u) * by;
        z[k] = fmaf(uhat[k], w[k], q[k]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) z[k] = uhat[k];
    }
    if (src_g)
#pragma unroll
      for (int k = 0; k < 8; ++k) sg[k] = sigma(sg[k]);
    else
#pragma unroll
      for (int k = 0; k < 8; ++k) sg[k] = 1.0f;
    // t = dh + N_n'(dn)
    if (a.dn && a.norm_n != FADE_NORM_NONE) {
      float h[8], v[4], mean, rstd;
      lam.get(w);
#pragma unroll
      for (int k = 0; k < 8; ++k) h[k] = fmaf(w[k], r[k], sg[k] * z[k]);
      rs.template part<WHOLE>(a.norm_n, h, l.left, v[0], v[1]);
      part.template update<PART_BN>([&](float s, int k) { return s + e[k]; });
      gn.get(w);
      const float m = v[0];
      float e0 = 0.0f, e1 = 0.0f;  // sums of e = dn gamma and of e times h's distance from the wavefront's mean
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float f = e[k] * w[k];
        e0 += f;
        e1 = fmaf(f, h[k] - m, e1);
      }
      v[2] = wave_total<L>(e0);
      v[3] = wave_total<L>(e1);
      rs.exchange(v);
      rs.whole(a.norm_n, v[0], v[1], a.eps, mean, rstd);
      const float along = rs.over_waves(fmaf(v[0] - mean, v[2], v[3])) * rstd * rs.inv, level = a.norm_n == FADE_NORM_LAYER ? rs.over_waves(v[2]) * rs.inv : 0.0f;
      const float by = factor(rstd, mean);
#pragma unroll
      for (int k = 0; k < 8; ++k) h[k] = (h[k] - mean) * by;
      part.template update<PART_GN>([&](float s, int k) { return fmaf(e[k], h[k], s); });
#pragma unroll
      for (int k = 0; k < 8; ++k) t[k] = fmaf(rstd, fmaf(-h[k], along, fmaf(e[k], w[k], -level)), t[k]);
    } else if (a.dn) {
#pragma unroll
      for (int k = 0; k < 8; ++k) t[k] += e[k];
    }
    // through the join
    lam.get(w);
    part.template update<PART_LAM>([&](float s, int k) { return fmaf(t[k], r[k], s); });
#pragma unroll
    for (int k = 0; k < 8; ++k) r[k] = w[k] * t[k];
    const bool store = in && l.left > 0;
    if (a.dr && store) {
      OpRaw<TS> o;
      o.put(r);
      o.store(static_cast<TS *>(a.dr) + row * a.dr_ld + l.c, op_left<WHOLE>(l.left));
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      t[k] *= sg[k];
      sg[k] = t[k] * z[k] * (1.0f - sg[k]);
    }
    if (a.dg && store) {
      OpRaw<TB> o;
      o.put(sg);
      o.store(static_cast<TB *>(a.dg) + row * a.dg_ld + l.c, op_left<WHOLE>(l.left));
    }
    // du = N_u'(dz)
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f}, rstd = rstd_u, x[8];
    if (a.norm_u != FADE_NORM_NONE) {
      gu.get(w);
      part.template update<PART_GU>([&](float s, int k) { return fmaf(t[k], uhat[k], s); });
      part.template update<PART_BU>([&](float s, int k) { return s + t[k]; });
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        t[k] *= w[k];
        v[0] += t[k];
        v[1] = fmaf(t[k], uhat[k], v[1]);
      }
      v[0] = wave_total<L>(v[0]);
      v[1] = wave_total<L>(v[1]);
    }
    arrived<WHOLE>(raw_u, l).get(x);
    rs.template part<WHOLE>(a.norm_u, x, l.left, v[2], v[3]);
    rs.exchange(v);
    rs.whole(a.norm_u, v[2], v[3], a.eps, mean_u, rstd_u);
    if (a.norm_u != FADE_NORM_NONE) {
      const float level = a.norm_u == FADE_NORM_LAYER ? rs.over_waves(v[0]) * rs.inv : 0.0f, along = rs.over_waves(v[1]) * rs.inv;
#pragma unroll
      for (int k = 0; k < 8; ++k) t[k] = rstd * fmaf(-uhat[k], along, t[k] - level);
    }
    if (a.du && store) {
      OpRaw<TB> o;
      o.put(t);
      o.store(static_cast<TB *>(a.du) + row * a.du_ld + l.c, op_left<WHOLE>(l.left));
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) uhat[k] = x[k];
  }
  // the workgroup's sums over its rows, its groups' in order
  if (a.lam_count == 1) {
    float s[1] = {0.0f};
    part.template update<PART_LAM>([&](float v, int) { s[0] += v; return v; });
    s[0] = wave_total<L>(s[0]);
    rs.exchange(s);
    s[0] = rs.over_waves(s[0]);
    part.template update<PART_LAM>([&](float, int) { return s[0]; });
  }
  float *dst = a.work + (size_t)blockIdx.x * PARTS * part_width(a.width);
  auto leave = [&](auto p_c) {
    constexpr int p = decltype(p_c)::value;
    float x[8];
    part.template update<p>([&](float v, int k) { x[k] = v; return v; });
    if constexpr (GROUPS > 1) {
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 8; ++k) fold[(l.group * 8 + k) * L + l.lane] = x[k];
      __syncthreads();
      if (l.group == 0)
        for (int g = 1; g < GROUPS; ++g)
#pragma unroll
          for (int k = 0; k < 8; ++k) x[k] += fold[(g * 8 + k) * L + l.lane];
    }
    if (l.group == 0 && l.left > 0) {
      OpRaw<float> o;
      o.put(x);
      o.store(dst + p * part_width(a.width) + l.c, 8);
    }
  };
  leave(std::integral_constant<int, PART_GU>{});
  leave(std::integral_constant<int, PART_BU>{});
  leave(std::integral_constant<int, PART_GN>{});
  leave(std::integral_constant<int, PART_BN>{});
  leave(std::integral_constant<int, PART_LAM>{});
}

// The workgroups' partial sums, in order: 64 columns of one parameter a workgroup, four a lane, 64 slices of the partial sums side by side, then the slices in four
// ranges.
__global__ __launch_bounds__(1024) void join_finish_kernel(JoinArgs a, int blocks) {
  __shared__ float sums[64][68], four[4][64];
  const int p = blockIdx.y, width = p == PART_LAM && a.lam_count == 1 ? 1 : a.width;
  float *dst = p == PART_GU ? a.d_gamma_u : p == PART_BU ? a.d_beta_u : p == PART_GN ? a.d_gamma_n : p == PART_BN ? a.d_beta_n : a.d_lam;
  const int c0 = blockIdx.x * 64, slice = threadIdx.x >> 4, quad = (threadIdx.x & 15) * 4, per = (blocks + 63) / 64;
  if (!dst || c0 >= width) return;
  const size_t w = part_width(a.width);
  f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
  if (c0 + quad < (int)w) {
    const float *src = a.work + p * w + c0 + quad;
    const int end = (slice + 1) * per < blocks ? (slice + 1) * per : blocks;
#pragma unroll 8
    for (int b = slice * per; b < end; ++b) s += *reinterpret_cast<const f32x4 *>(src + (size_t)b * PARTS * w);
  }
  *reinterpret_cast<f32x4 *>(&sums[slice][quad]) = s;
  __syncthreads();
  if (threadIdx.x < 256) {
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += sums[threadIdx.x / 64 * 16 + i][threadIdx.x & 63];
    four[threadIdx.x >> 6][threadIdx.x & 63] = v;
  }
  __syncthreads();
  const int c = c0 + threadIdx.x;
  if (threadIdx.x < 64 && c < width) {
    const float v = ((four[0][threadIdx.x] + four[1][threadIdx.x]) + four[2][threadIdx.x]) + four[3][threadIdx.x];
    dst[c] = a.accumulate ? dst[c] + v : v;
  }
}

template <typename F> hipError_t with_lanes(int lanes, F &&f) {
  switch (lanes) {
    case 16: f(std::integral_constant<int, 16>{}); break;
    case 32: f(std::integral_constant<int, 32>{}); break;
    case 64: f(std::integral_constant<int, 64>{}); break;
    case 128: f(std::integral_constant<int, 128>{}); break;
    case 256: f(std::integral_constant<int, 256>{}); break;
    case 512: f(std::integral_constant<int, 512>{}); break;
    default: f(std::integral_constant<int, 1024>{}); break;
  }
  return hipGetLastError();
}
template <typename F> hipError_t with_types(const JoinArgs &a, F &&f) {
  if (a.branch_f32) return f(float{}, float{});
  if (a.stream_f32) return f(float{}, bf16_t{});
  return f(bf16_t{}, bf16_t{});
}

}  // namespace

hipError_t fade_join_launch(const JoinArgs &a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  const JoinShape sh = join_shape(a.width);
  const int blocks = turn_blocks(a.rows, sh.groups, 2048);
  return with_types(a, [&](auto st, auto br) {
    return with_lanes(sh.lanes, [&](auto l) {
      constexpr int L = decltype(l)::value;
      typedef decltype(st) TS;
      typedef decltype(br) TB;
      constexpr bool SPARE = L <= 512;  // registers for the checkpoints whether they are wanted or not
      const bool whole = a.width % 8 == 0, keep = a.keep_r || a.keep_u || a.keep_g || a.keep_n;
      auto *f = SPARE || keep ? (whole ? join_kernel<L, TS, TB, true> : join_kernel<L, TS, TB, false>)
                              : (whole ? join_kernel<L, TS, TB, true, SPARE> : join_kernel<L, TS, TB, false, SPARE>);
      hipLaunchKernelGGL(f, dim3(blocks), dim3(most(L, 256)), 0, s, a);
    });
  });
}
size_t fade_join_grad_bytes(size_t rows, size_t width) {
  const size_t blocks = grad_blocks(rows, width);
  return 4 * (blocks ? blocks : 1) * PARTS * part_width((int)width);
}
hipError_t fade_join_grad_launch(const JoinArgs &a, hipStream_t s) {
  if (a.rows == 0 && a.accumulate) return hipSuccess;  // not even a zero is added: it would make a positive zero of a negative one
  const JoinShape sh = join_shape(a.width);
  const int blocks = grad_blocks(a.rows, a.width);
  if (blocks) {
    const hipError_t e = with_types(a, [&](auto st, auto br) {
      return with_lanes(sh.lanes, [&](auto l) {
        constexpr int L = decltype(l)::value;
        typedef decltype(st) TS;
        typedef decltype(br) TB;
        const bool whole = a.width % 8 == 0;
        auto *f = a.kept ? (whole ? join_grad_kernel<L, TS, TB, true, true> : join_grad_kernel<L, TS, TB, true, false>)
                         : (whole ? join_grad_kernel<L, TS, TB, false, true> : join_grad_kernel<L, TS, TB, false, false>);
        constexpr int LDS = Sums8<L>::LDS ? 8 * L * 16 : 0;
        if (LDS) (void)hipFuncSetAttribute(reinterpret_cast<const void *>(f), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
        hipLaunchKernelGGL(f, dim3(blocks), dim3(most(L, 256)), LDS, s, a);
      });
    });
    if (e != hipSuccess) return e;
  }
  if (a.d_gamma_u || a.d_beta_u || a.d_gamma_n || a.d_beta_n || a.d_lam)
    hipLaunchKernelGGL(join_finish_kernel, dim3((a.width + 63) / 64, PARTS), dim3(1024), 0, s, a, blocks);
  return hipGetLastError();
}
