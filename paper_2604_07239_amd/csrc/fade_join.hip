// fade_join.hip — the join of a block with the residual stream: z = N_u(u), h = lam r + sigma(g) z, n = N_n(h), and its gradient (gfx950).
//
// A row stays in the registers of the L lanes that own it (8 columns per lane and step), so each pass reads its operands once and writes its
// results once, whatever norms and gate there are; the bytes bound it. The backward pass forms the statistics again instead of reading
// saved ones, from the operands themselves or from 8-bit checkpoints of them.
// LayerNorm's variance is the mean of the squares of centred values: the difference of E[x^2] and mean^2 loses what a large mean covers.
// Parameter gradients are sums over the rows: a workgroup keeps its columns' sums in registers over all its rows and leaves one partial sum per column,
// which a second kernel adds in order. No atomics.
#include "../../include/fade.h"
#include "fade_op_rules.h"
#include "fade_ops.h"

namespace {
using namespace fade_op;

constexpr int most(int a, int b) { return a > b ? a : b; }

// Sums over the L lanes of a row, the same value in each of them. Above a wavefront through LDS: one barrier a sum, in two places in turn
// (a wavefront may be one sum ahead of another, never two).
template <int L> struct RowSums {
  static constexpr int W = L / 64, GROUPS = L >= 256 ? 1 : 256 / L;  // wavefronts of a row; rows of a workgroup
  float (*lds)[GROUPS][W > 0 ? W : 1][4];                            // [2]
  int place = 0, group, wave;
  template <int N> __device__ __forceinline__ void sum(float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = fade_lanes_sum<(L < 64 ? L : 64)>(v[i]);
    if constexpr (W > 1) {
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) lds[place][group][wave][i] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) v[i] += lds[place][group][w][i];
      }
      place ^= 1;
    }
  }
  // mean and sum of squared distances from it, of `mine` values in this wavefront and C in the row: centred on the wavefront's mean, then moved to the row's
  template <typename F> __device__ __forceinline__ void moments(float s, float mine, float C, float &mean, float &sq, F &&centred) {
    s = fade_lanes_sum<(L < 64 ? L : 64)>(s);
    mean = mine > 0.0f ? s / mine : 0.0f;
    sq = fade_lanes_sum<(L < 64 ? L : 64)>(centred(mean));
    if constexpr (W > 1) {
      if ((threadIdx.x & 63) == 0) {
        float *p = lds[place][group][wave];
        p[0] = mean; p[1] = sq; p[2] = mine; p[3] = s;
      }
      __syncthreads();
      float all = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) all += lds[place][group][w][3];
      mean = all / C;
      sq = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float d = lds[place][group][w][0] - mean;
        sq += fmaf(lds[place][group][w][2] * d, d, lds[place][group][w][1]);
      }
      place ^= 1;
    }
  }
};

// statistics of a row's values x: mean (0 unless LayerNorm) and 1 / sigma
template <int V, int L> __device__ __forceinline__ void row_stats(RowSums<L> &rs, int norm, const float (&x)[V][8], const int (&left)[V], float mine, float C,
                                                                  float eps, float &mean, float &rstd) {
  float sq;
  if (norm == FADE_NORM_LAYER) {
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int k = 0; k < 8; ++k) s += x[v][k];  // columns that do not exist hold zeros
    rs.moments(s, mine, C, mean, sq, [&](float m) {
      float q = 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float d = k < left[v] ? x[v][k] - m : 0.0f;
          q = fmaf(d, d, q);
        }
      return q;
    });
  } else {
    float q[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int k = 0; k < 8; ++k) q[0] = fmaf(x[v][k], x[v][k], q[0]);
    rs.sum(q);
    mean = 0.0f;
    sq = q[0];
  }
  rstd = 1.0f / sqrtf(sq / C + eps);
}

// 8 columns of a parameter; `otherwise` where there is none, zeros past the row's end
__device__ __forceinline__ void param8(const float *p, float otherwise, int c, int left, float x[8]) {
  if (left <= 0 || !p) {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = k < left ? otherwise : 0.0f;
  } else {
    OpRaw<float> r;
    r.load(p + c, left);
    r.get(x);
  }
}
// sigma(x) = 1 / (1 + exp(-x)); fade_sigmoid's reciprocal is the hardware's, good to an ulp
__device__ __forceinline__ float sigma(float x) { return fade_sigmoid(x); }

template <int L, int V> struct Lanes {
  int group, lane, c[V], left[V];
  float mine;  // columns of this wavefront (of this row where a wavefront holds several)
  __device__ __forceinline__ Lanes(int width) {
    group = threadIdx.x / L;
    lane = threadIdx.x % L;
    int n = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      c[v] = (v * L + lane) * 8;
      left[v] = width - c[v];
      const int first = (v * L + (L > 64 ? lane / 64 * 64 : 0)) * 8, have = width - first, span = (L < 64 ? L : 64) * 8;
      n += have < 0 ? 0 : have > span ? span : have;
    }
    mine = (float)n;
  }
};

template <int V> __device__ __forceinline__ void keep_row(uint8_t *keep, int rows, int width, size_t row, bool in, const float (&x)[V][8], const int (&c)[V]) {
  const int groups = (width + 31) / 32;
  uint8_t *q = keep + row * groups * 32, *e = keep + (size_t)rows * groups * 32 + row * groups;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    uint32_t exp;
    const uint2 w = op_keep_pack(x[v], exp);
    if (in && c[v] < groups * 32) {
      *reinterpret_cast<uint2 *>(q + c[v]) = w;
      if ((threadIdx.x & 3) == 0) e[c[v] >> 5] = (uint8_t)exp;
    }
  }
}

template <int L, int V, typename TS, typename TB> __global__ __launch_bounds__(most(L, 256)) void join_kernel(JoinArgs a) {
  typedef RowSums<L> Sums;
  __shared__ float lds[2][Sums::GROUPS][Sums::W > 0 ? Sums::W : 1][4];
  const Lanes<L, V> l(a.width);
  Sums rs{lds, 0, l.group, l.lane / 64};
  float gu[V][8], bu[V][8], gn[V][8], bn[V][8], lam[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    param8(a.gamma_u, 1.0f, l.c[v], l.left[v], gu[v]);
    param8(a.beta_u, 0.0f, l.c[v], l.left[v], bu[v]);
    param8(a.gamma_n, 1.0f, l.c[v], l.left[v], gn[v]);
    param8(a.beta_n, 0.0f, l.c[v], l.left[v], bn[v]);
    param8(a.lam_count == 1 ? nullptr : a.lam, a.lam_count == 1 ? a.lam[0] : 1.0f, l.c[v], l.left[v], lam[v]);
  }
  const float C = (float)a.width;
  for (uint32_t base = blockIdx.x * Sums::GROUPS; base < (uint32_t)a.rows; base += gridDim.x * Sums::GROUPS) {
    const bool in = base + l.group < (uint32_t)a.rows;  // the workgroup's barriers are for all its rows
    const size_t row = in ? base + l.group : a.rows - 1;
    OpRaw<TS> raw_r[V];
    OpRaw<TB> raw_u[V], raw_g[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      raw_r[v].zero(); raw_u[v].zero(); raw_g[v].zero();
      if (l.left[v] > 0) {
        raw_r[v].load(static_cast<const TS *>(a.r) + row * a.r_ld + l.c[v], l.left[v]);
        raw_u[v].load(static_cast<const TB *>(a.u) + row * a.u_ld + l.c[v], l.left[v]);
        if (a.g) raw_g[v].load(static_cast<const TB *>(a.g) + row * a.g_ld + l.c[v], l.left[v]);
      }
    }
    float x[V][8], h[V][8], g[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) { raw_u[v].get(x[v]); raw_r[v].get(h[v]); raw_g[v].get(g[v]); }
    if (a.keep_r) keep_row<V>(a.keep_r, a.rows, a.width, row, in, h, l.c);
    if (a.keep_u) keep_row<V>(a.keep_u, a.rows, a.width, row, in, x, l.c);
    if (a.keep_g) keep_row<V>(a.keep_g, a.rows, a.width, row, in, g, l.c);
    if (a.norm_u != FADE_NORM_NONE) {
      float mean, rstd;
      row_stats<V>(rs, a.norm_u, x, l.left, l.mine, C, a.eps, mean, rstd);
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int k = 0; k < 8; ++k) x[v][k] = fmaf((x[v][k] - mean) * rstd, gu[v][k], bu[v][k]);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
      for (int k = 0; k < 8; ++k) h[v][k] = fmaf(lam[v][k], h[v][k], a.g ? sigma(g[v][k]) * x[v][k] : x[v][k]);
      OpRaw<TS> o;
      o.put(h[v]);
      if (in && l.left[v] > 0) o.store(static_cast<TS *>(a.h) + row * a.h_ld + l.c[v], l.left[v]);
    }
    if (!a.n && !a.keep_n) continue;
    if (a.norm_n != FADE_NORM_NONE) {
      float mean, rstd;
      row_stats<V>(rs, a.norm_n, h, l.left, l.mine, C, a.eps, mean, rstd);
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int k = 0; k < 8; ++k) h[v][k] = fmaf((h[v][k] - mean) * rstd, gn[v][k], bn[v][k]);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      OpRaw<TB> o;
      o.put(h[v]);
      if (a.n && in && l.left[v] > 0) o.store(static_cast<TB *>(a.n) + row * a.n_ld + l.c[v], l.left[v]);
      o.get(h[v]);  // a checkpoint of n is one of the values as rounded
    }
    if (a.keep_n) keep_row<V>(a.keep_n, a.rows, a.width, row, in, h, l.c);
  }
}

// ---------------------------------------------------------------------------------------------------
// The gradient
// ---------------------------------------------------------------------------------------------------
// partial sums of the parameters' gradients: [workgroup][5][width rounded up to 8]
enum { PART_GU = 0, PART_BU, PART_GN, PART_BN, PART_LAM, PARTS };
__host__ __device__ inline size_t part_width(int width) { return (size_t)((width + 7) / 8 * 8); }

template <typename T> struct SavedRaw {  // 8 columns of a saved operand: as it was
  OpRaw<T> v;
  __device__ __forceinline__ void zero() { v.zero(); }
  __device__ __forceinline__ void load(const void *p, size_t ld, int, int, size_t row, int c, int left) { v.load(static_cast<const T *>(p) + row * ld + c, left); }
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
  __device__ __forceinline__ void get(float x[8]) const { op_keep_unpack(q, op_keep_unit(e), x); }
};

template <int L, int V, typename TS, typename TB, bool KEPT> __global__ __launch_bounds__(most(L, 256)) void join_grad_kernel(JoinArgs a) {
  typedef RowSums<L> Sums;
  typedef std::conditional_t<KEPT, SavedKeep, SavedRaw<TS>> RawS;
  typedef std::conditional_t<KEPT, SavedKeep, SavedRaw<TB>> RawB;
  constexpr int GROUPS = Sums::GROUPS;
  __shared__ float lds[2][GROUPS][Sums::W > 0 ? Sums::W : 1][4];
  __shared__ __align__(16) float fold[GROUPS > 1 ? 256 * 8 * V : 4];
  const Lanes<L, V> l(a.width);
  Sums rs{lds, 0, l.group, l.lane / 64};
  float gu[V][8], bu[V][8], gn[V][8], lam[V][8], part[PARTS][V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    param8(a.gamma_u, 1.0f, l.c[v], l.left[v], gu[v]);
    param8(a.beta_u, 0.0f, l.c[v], l.left[v], bu[v]);
    param8(a.gamma_n, 1.0f, l.c[v], l.left[v], gn[v]);
    param8(a.lam_count == 1 ? nullptr : a.lam, a.lam_count == 1 ? a.lam[0] : 1.0f, l.c[v], l.left[v], lam[v]);
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int p = 0; p < PARTS; ++p) part[p][v][k] = 0.0f;
  }
  const float C = (float)a.width, inv = 1.0f / C;
  const void *src_r = KEPT ? a.keep_r : a.r, *src_u = KEPT ? a.keep_u : a.u, *src_g = KEPT ? a.keep_g : a.g;
  for (uint32_t base = blockIdx.x * GROUPS; base < (uint32_t)a.rows; base += gridDim.x * GROUPS) {
    const bool in = base + l.group < (uint32_t)a.rows;
    const size_t row = base + l.group;
    RawS raw_r[V];
    RawB raw_u[V], raw_g[V];
    OpRaw<TS> raw_dh[V];
    OpRaw<TB> raw_dn[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      raw_r[v].zero(); raw_u[v].zero(); raw_g[v].zero(); raw_dh[v].zero(); raw_dn[v].zero();
      if (in && l.left[v] > 0) {
        raw_r[v].load(src_r, a.r_ld, a.rows, a.width, row, l.c[v], l.left[v]);
        raw_u[v].load(src_u, a.u_ld, a.rows, a.width, row, l.c[v], l.left[v]);
        if (src_g) raw_g[v].load(src_g, a.g_ld, a.rows, a.width, row, l.c[v], l.left[v]);
        if (a.dh) raw_dh[v].load(static_cast<const TS *>(a.dh) + row * a.dh_ld + l.c[v], l.left[v]);
        if (a.dn) raw_dn[v].load(static_cast<const TB *>(a.dn) + row * a.dn_ld + l.c[v], l.left[v]);
      }
    }
    // forward again: uhat, z, sigma(g), h
    float uhat[V][8], z[V][8], sg[V][8], r[V][8], t[V][8], rstd_u = 1.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      raw_u[v].get(uhat[v]);
      raw_r[v].get(r[v]);
      raw_g[v].get(sg[v]);
      raw_dh[v].get(t[v]);
    }
    if (a.norm_u != FADE_NORM_NONE) {
      float mean;
      row_stats<V>(rs, a.norm_u, uhat, l.left, l.mine, C, a.eps, mean, rstd_u);
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          uhat[v][k] = (uhat[v][k] - mean) * rstd_u;
          z[v][k] = fmaf(uhat[v][k], gu[v][k], bu[v][k]);
        }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int k = 0; k < 8; ++k) z[v][k] = uhat[v][k];
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int k = 0; k < 8; ++k) sg[v][k] = src_g ? sigma(sg[v][k]) : 1.0f;
    // t = dh + N_n'(dn)
    if (a.dn) {
      if (a.norm_n != FADE_NORM_NONE) {
        float h[V][8], mean, rstd, s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int k = 0; k < 8; ++k) h[v][k] = fmaf(lam[v][k], r[v][k], sg[v][k] * z[v][k]);
        row_stats<V>(rs, a.norm_n, h, l.left, l.mine, C, a.eps, mean, rstd);
        float e[V][8];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          raw_dn[v].get(e[v]);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            h[v][k] = (h[v][k] - mean) * rstd;
            part[PART_GN][v][k] = fmaf(e[v][k], h[v][k], part[PART_GN][v][k]);
            part[PART_BN][v][k] += e[v][k];
            e[v][k] *= gn[v][k];
            s[0] += e[v][k];
            s[1] = fmaf(e[v][k], h[v][k], s[1]);
          }
        }
        rs.sum(s);
        const float level = a.norm_n == FADE_NORM_LAYER ? s[0] * inv : 0.0f, along = s[1] * inv;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int k = 0; k < 8; ++k) t[v][k] = fmaf(rstd, fmaf(-h[v][k], along, e[v][k] - level), t[v][k]);
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float e[8];
          raw_dn[v].get(e);
#pragma unroll
          for (int k = 0; k < 8; ++k) t[v][k] += e[k];
        }
      }
    }
    // through the join
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        part[PART_LAM][v][k] = fmaf(t[v][k], r[v][k], part[PART_LAM][v][k]);
        x[k] = lam[v][k] * t[v][k];
      }
      if (a.dr && in && l.left[v] > 0) {
        OpRaw<TS> o;
        o.put(x);
        o.store(static_cast<TS *>(a.dr) + row * a.dr_ld + l.c[v], l.left[v]);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float dz = t[v][k] * sg[v][k];
        x[k] = dz * z[v][k] * (1.0f - sg[v][k]);
        t[v][k] = dz;
      }
      if (a.dg && in && l.left[v] > 0) {
        OpRaw<TB> o;
        o.put(x);
        o.store(static_cast<TB *>(a.dg) + row * a.dg_ld + l.c[v], l.left[v]);
      }
    }
    // du = N_u'(dz)
    if (a.norm_u != FADE_NORM_NONE) {
      float s[2] = {0.0f, 0.0f};
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          part[PART_GU][v][k] = fmaf(t[v][k], uhat[v][k], part[PART_GU][v][k]);
          part[PART_BU][v][k] += t[v][k];
          t[v][k] *= gu[v][k];
          s[0] += t[v][k];
          s[1] = fmaf(t[v][k], uhat[v][k], s[1]);
        }
      rs.sum(s);
      const float level = a.norm_u == FADE_NORM_LAYER ? s[0] * inv : 0.0f, along = s[1] * inv;
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int k = 0; k < 8; ++k) t[v][k] = rstd_u * fmaf(-uhat[v][k], along, t[v][k] - level);
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (a.du && in && l.left[v] > 0) {
        OpRaw<TB> o;
        o.put(t[v]);
        o.store(static_cast<TB *>(a.du) + row * a.du_ld + l.c[v], l.left[v]);
      }
  }
  // the workgroup's sums over its rows, its groups' in order
  float *dst = a.work + (size_t)blockIdx.x * PARTS * part_width(a.width);
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    if constexpr (GROUPS > 1) {
      __syncthreads();
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int k = 0; k < 8; ++k) fold[((v * GROUPS + l.group) * 8 + k) * L + l.lane] = part[p][v][k];
      __syncthreads();
      if (l.group == 0)
        for (int g = 1; g < GROUPS; ++g)
#pragma unroll
          for (int v = 0; v < V; ++v)
#pragma unroll
            for (int k = 0; k < 8; ++k) part[p][v][k] += fold[((v * GROUPS + g) * 8 + k) * L + l.lane];
    }
    if (l.group == 0)
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (l.left[v] > 0) {
          OpRaw<float> o;
          o.put(part[p][v]);
          o.store(dst + p * part_width(a.width) + l.c[v], 8);
        }
  }
}

// The workgroups' partial sums, in order: 16 slices of them side by side per column, then the slices.
// One value of lam: its column sums are added up as well, by the one workgroup that has them all.
__global__ __launch_bounds__(1024) void join_finish_kernel(JoinArgs a, int blocks) {
  __shared__ float sums[16][65];
  const int p = blockIdx.y;
  float *dst = p == PART_GU ? a.d_gamma_u : p == PART_BU ? a.d_beta_u : p == PART_GN ? a.d_gamma_n : p == PART_BN ? a.d_beta_n : a.d_lam;
  if (!dst) return;
  const bool one = p == PART_LAM && a.lam_count == 1;
  if (one && blockIdx.x > 0) return;
  const int slice = threadIdx.x >> 6, lane = threadIdx.x & 63, per = (blocks + 15) / 16;
  const size_t w = part_width(a.width);
  float total = 0.0f;
  for (int c0 = blockIdx.x * 64; c0 < a.width; c0 += one ? 64 : a.width) {
    float s = 0.0f;
    const int c = c0 + lane;
    if (c < a.width)
      for (int b = slice * per; b < (slice + 1) * per && b < blocks; ++b) s += a.work[((size_t)b * PARTS + p) * w + c];
    __syncthreads();
    sums[slice][lane] = s;
    __syncthreads();
    if (slice == 0) {
      s = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) s += sums[i][lane];
      if (one) total += s;
      else if (c < a.width) dst[c] = a.accumulate ? dst[c] + s : s;
    }
  }
  if (one && slice == 0) {
    total = fade_lanes_sum(total);
    if (lane == 0) dst[0] = a.accumulate ? dst[0] + total : total;
  }
}

template <typename F> hipError_t with_shape(const JoinShape &sh, F &&f) {
  if (sh.V == 2) f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
  else switch (sh.L) {
    case 16: f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{}); break;
    case 32: f(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{}); break;
    case 64: f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{}); break;
    case 128: f(std::integral_constant<int, 128>{}, std::integral_constant<int, 1>{}); break;
    case 256: f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{}); break;
    case 512: f(std::integral_constant<int, 512>{}, std::integral_constant<int, 1>{}); break;
    default: f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{}); break;
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
  const int need = (a.rows + sh.groups - 1) / sh.groups, blocks = need < 2048 ? need : 2048;
  return with_types(a, [&](auto st, auto br) {
    return with_shape(sh, [&](auto l, auto v) {
      constexpr int L = decltype(l)::value, V = decltype(v)::value;
      hipLaunchKernelGGL((join_kernel<L, V, decltype(st), decltype(br)>), dim3(blocks), dim3(most(L, 256)), 0, s, a);
    });
  });
}
size_t fade_join_grad_bytes(size_t rows, size_t width) {
  const size_t blocks = grad_blocks(rows, width);
  return 4 * (blocks ? blocks : 1) * PARTS * part_width((int)width);
}
hipError_t fade_join_grad_launch(const JoinArgs &a, hipStream_t s) {
  const JoinShape sh = join_shape(a.width);
  const int blocks = grad_blocks(a.rows, a.width);
  if (blocks) {
    const hipError_t e = with_types(a, [&](auto st, auto br) {
      return with_shape(sh, [&](auto l, auto v) {
        constexpr int L = decltype(l)::value, V = decltype(v)::value;
        typedef decltype(st) TS;
        typedef decltype(br) TB;
        if (a.kept) hipLaunchKernelGGL((join_grad_kernel<L, V, TS, TB, true>), dim3(blocks), dim3(most(L, 256)), 0, s, a);
        else hipLaunchKernelGGL((join_grad_kernel<L, V, TS, TB, false>), dim3(blocks), dim3(most(L, 256)), 0, s, a);
      });
    });
    if (e != hipSuccess) return e;
  }
  if (a.d_gamma_u || a.d_beta_u || a.d_gamma_n || a.d_beta_n || a.d_lam)
    hipLaunchKernelGGL(join_finish_kernel, dim3((a.width + 63) / 64, PARTS), dim3(1024), 0, s, a, blocks);
  return hipGetLastError();
}
