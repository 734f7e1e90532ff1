// fade_keep.hip — activations kept in 8 bits between the passes, and the weight gradient from them (gfx950).
//
// A group of 32 columns shares a power of two, so what a checkpoint stands for is exact in bf16, and a product with it runs on the bf16 matrix
// cores with nothing rounded but the fp32 sums. Writing and reading are one pass over the data, bounded by its bytes. The weight gradient dW = x^T dy contracts over the rows: the
// row-major tiles of both operands are turned on their way out of LDS (ds_read_b64_tr_b16), x is widened to bf16 on its way in.
// An fp32 dy goes in as three bf16 terms, each the leading 8 bits of what the ones before left: 24 bits, so that they add up to it.
#include <type_traits>

#include "../../include/fade.h"
#include "fade_op_rules.h"
#include "fade_ops.h"

namespace {
using namespace fade_op;

template <typename T>
__global__ __launch_bounds__(256) void keep_kernel(const T *x, size_t ld, int width, OpKeep k, int shift) {
  const size_t row = (size_t)blockIdx.x * (256 >> shift) + (threadIdx.x >> shift);
  if (row >= k.rows) return;
  uint8_t *q = k.p + row * k.groups * 32, *e = k.p + k.rows * k.groups * 32 + row * k.groups;
  for (int c = (threadIdx.x & ((1 << shift) - 1)) * 8; c < k.groups * 32; c += 8 << shift) {
    float v[8];
    OpRaw<T> in;
    if (c < width) in.load(x + row * ld + c, width - c);
    else in.zero();
    in.get(v);
    uint32_t exp;
    const uint2 w = op_keep_pack(v, exp);
    *reinterpret_cast<uint2 *>(q + c) = w;
    if ((threadIdx.x & 3) == 0) e[c >> 5] = (uint8_t)exp;
  }
}
template <typename T>
__global__ __launch_bounds__(256) void keep_read_kernel(OpKeep k, int width, T *out, size_t ld, int shift) {
  const size_t row = (size_t)blockIdx.x * (256 >> shift) + (threadIdx.x >> shift);
  if (row >= k.rows) return;
  const uint8_t *q = k.p + row * k.groups * 32, *e = k.p + k.rows * k.groups * 32 + row * k.groups;
  for (int c = (threadIdx.x & ((1 << shift) - 1)) * 8; c < width; c += 8 << shift) {
    float v[8];
    op_keep_unpack(*reinterpret_cast<const uint2 *>(q + c), op_keep_unit(e[c >> 5]), v);
    OpRaw<T> o;
    o.put(v);
    o.store(out + row * ld + c, width - c);
  }
}

// ---------------------------------------------------------------------------------------------------
// dW[K][N] = sum over rows of x[row][k] * dy[row][n]
// ---------------------------------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(4))) short i16x4;
typedef __attribute__((ext_vector_type(8))) short i16x8;
struct WgradArgs {
  OpKeep x;
  const void *dy;
  size_t dy_ld;
  int K, N, tiles_m, tiles_n, ranges, units, per;  // units of 64 rows; units in one range
  float *out;                                       // the gradient, or the ranges' sums [range][K][N]
  size_t out_ld;
  bool add;
};

__device__ __forceinline__ i16x4 wg_turn(const uint8_t *lds) {  // gfx950's transposing read: see the address pattern below
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)lds);
}

// fp32 as the leading 8 bits, the next 8, the last 8: cut, not rounded, so that nothing overflows and the rest is exact
__device__ __forceinline__ void wg_split(float v, uint32_t &hi, uint32_t &mid, uint32_t &lo) {
  hi = __builtin_bit_cast(uint32_t, v) & 0xffff0000u;
  float rest = v - __builtin_bit_cast(float, hi);
  if (fabsf(v) == __builtin_inff()) rest = 0.0f;  // an infinity is its first term alone; a NaN stays one in the second
  mid = __builtin_bit_cast(uint32_t, rest) & 0xffff0000u;
  lo = __builtin_bit_cast(uint32_t, rest - __builtin_bit_cast(float, mid));
}
__device__ __forceinline__ uint32_t wg_upper(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }  // upper halves, a's first
__device__ __forceinline__ bf16x8 wg_widen(uint32_t lo, uint32_t hi, float unit) {
  float v[8];
  op_keep_unpack(make_uint2(lo, hi), unit, v);
  bf16x8 b;
#pragma unroll
  for (int k = 0; k < 8; ++k) b[k] = (bf16_t)v[k];
  return b;
}

// WM x WN wavefronts, each TM x TN tiles of 32 x 32. Units of 64 rows pass through two places in LDS: while the matrix cores work on one, the
// next is on its way through the registers (x has to be widened, an fp32 dy split, on the way) into the other; one barrier a unit.
template <int WM, int WN, int TM, int TN, bool F32> __global__ __launch_bounds__(WM *WN * 64, 1) void keep_grad_kernel(WgradArgs g) {
  constexpr int BM = WM * TM * 32, BN = WN * TN * 32, NT = WM * WN * 64, PLANES = F32 ? 3 : 1;
  constexpr int A_BYTES = 64 * BM * 2, B_BYTES = 64 * BN * 2, PLACE = A_BYTES + PLANES * B_BYTES;
  constexpr int QA = 64 * BM / 16 / NT, QB = 64 * BN / 8 / NT;  // 16 columns of x, 8 of dy: pieces per thread and unit
  extern __shared__ __align__(16) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave / WN, wn = wave % WN;

  // Consecutive workgroups go to the 8 XCDs in turn; each XCD takes one run of the tiles, four rows of tiles wide, so that the operands' columns that
  // it reads at a time are few and stay in its L2.
  const int total = g.tiles_m * g.tiles_n * g.ranges, xcd = blockIdx.x & 7, q8 = total >> 3, r8 = total & 7;
  const int at = xcd * q8 + (xcd < r8 ? xcd : r8) + (blockIdx.x >> 3);
  const int tiles = g.tiles_m * g.tiles_n, range = at / tiles, tile = at - range * tiles;
  const int band = tile / (4 * g.tiles_n), in_band = tile - band * 4 * g.tiles_n, high = g.tiles_m - band * 4 < 4 ? g.tiles_m - band * 4 : 4;
  const int m0 = (band * 4 + in_band % high) * BM, n0 = in_band / high * BN;
  const int u0 = range * g.per, u1 = u0 + g.per < g.units ? u0 + g.per : g.units;

  // a row of a unit is pieces of 16 bytes; piece p of row r lies at p ^ 4 (r % 4): four rows of a column block in four quarters of the banks
  auto piece_at = [](int pitch, int r, int p) { return r * pitch + ((p ^ ((r & 3) << 2)) << 4); };
  // transposing reads: in each group of 16 lanes, lane s supplies the address of row s / 4, columns 4 (s % 4) .. + 3 of a 4 x 16 block, and
  // lane i receives column i with the block's 4 rows in order; two such loads make the 8 rows of a lane's column
  const int s16 = lane & 15, r0 = (lane >> 5) * 8 + (s16 >> 2), mh = (lane >> 4) & 1;
  auto turned = [&](const uint8_t *base, int pitch, int t, int ks) {
    const uint8_t *src = base + piece_at(pitch, ks * 16 + r0, t * 4 + 2 * mh + ((s16 & 3) >> 1)) + (s16 & 1) * 8;
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(wg_turn(src), wg_turn(src + 4 * pitch), 0, 1, 2, 3, 4, 5, 6, 7));
  };

  const size_t pitch = (size_t)g.x.groups * 32;
  const uint8_t *exps = g.x.p + g.x.rows * pitch;
  typedef std::conditional_t<F32, float, bf16_t> TD;
  const TD *dy = static_cast<const TD *>(g.dy);
  // this thread's pieces. Columns that do not exist read column 0: what they bring reaches only results that do not exist.
  int xr[QA], xc[QA], yr[QB], yc[QB];
#pragma unroll
  for (int i = 0; i < QA; ++i) {
    xr[i] = (tid + i * NT) / (BM / 16);
    xc[i] = (tid + i * NT) % (BM / 16);
  }
#pragma unroll
  for (int i = 0; i < QB; ++i) {
    yr[i] = (tid + i * NT) / (BN / 8);
    yc[i] = (tid + i * NT) % (BN / 8);
  }
  uint4 qx[QA];
  uint32_t ex[QA];
  OpRaw<TD> qy[QB];
  // The last unit, whose rows may end and whose last piece of dy may reach past the matrix, is loaded with every access checked. In the others a piece that
  // starts in a row ends in the next one at the latest (rows of 8 columns or more), which exists.
  auto load = [&](int u) {
    if (u + 1 < g.units && g.N >= 8) {
#pragma unroll
      for (int i = 0; i < QA; ++i) {
        const size_t row = (size_t)u * 64 + xr[i], c = (size_t)(m0 + xc[i] * 16) < pitch ? m0 + xc[i] * 16 : 0;
        qx[i] = *reinterpret_cast<const uint4 *>(g.x.p + row * pitch + c);
        ex[i] = exps[row * g.x.groups + (c >> 5)];
      }
#pragma unroll
      for (int i = 0; i < QB; ++i) {
        const size_t row = (size_t)u * 64 + yr[i], c = n0 + yc[i] * 8 < g.N ? n0 + yc[i] * 8 : 0;
        qy[i].load(dy + row * g.dy_ld + c, 8);
      }
    } else {
#pragma unroll
      for (int i = 0; i < QA; ++i) {
        const size_t row = (size_t)u * 64 + xr[i], c = m0 + xc[i] * 16;
        qx[i] = make_uint4(0, 0, 0, 0);
        ex[i] = 0;
        if (row < g.x.rows && c < pitch) {
          qx[i] = *reinterpret_cast<const uint4 *>(g.x.p + row * pitch + c);
          ex[i] = exps[row * g.x.groups + (c >> 5)];
        }
      }
#pragma unroll
      for (int i = 0; i < QB; ++i) {
        const size_t row = (size_t)u * 64 + yr[i];
        const int c = n0 + yc[i] * 8;
        qy[i].zero();
        if (row < g.x.rows && c < g.N) qy[i].load(dy + row * g.dy_ld + c, g.N - c);
      }
    }
  };
  auto store = [&](uint8_t *to) {
#pragma unroll
    for (int i = 0; i < QA; ++i) {
      const float unit = op_keep_unit(ex[i]);
      *reinterpret_cast<bf16x8 *>(to + piece_at(BM * 2, xr[i], xc[i] * 2)) = wg_widen(qx[i].x, qx[i].y, unit);
      *reinterpret_cast<bf16x8 *>(to + piece_at(BM * 2, xr[i], xc[i] * 2 + 1)) = wg_widen(qx[i].z, qx[i].w, unit);
    }
#pragma unroll
    for (int i = 0; i < QB; ++i) {
      uint8_t *dst = to + A_BYTES + piece_at(BN * 2, yr[i], yc[i]);
      if constexpr (F32) {
        float v[8];
        qy[i].get(v);
        uint32_t w[3][8];
#pragma unroll
        for (int k = 0; k < 8; ++k) wg_split(v[k], w[0][k], w[1][k], w[2][k]);
#pragma unroll
        for (int t = 0; t < 3; ++t)
          *reinterpret_cast<uint4 *>(dst + t * B_BYTES) = make_uint4(wg_upper(w[t][0], w[t][1]), wg_upper(w[t][2], w[t][3]), wg_upper(w[t][4], w[t][5]),
                                                                     wg_upper(w[t][6], w[t][7]));
      } else {
        *reinterpret_cast<uint4 *>(dst) = make_uint4(qy[i].v[0], qy[i].v[1], qy[i].v[2], qy[i].v[3]);
      }
    }
  };
  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
  auto multiply = [&](const uint8_t *from, int ks) {
    bf16x8 a[TM], b[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) a[i] = turned(from, BM * 2, wm * TM + i, ks);
#pragma unroll
    for (int t = PLANES - 1; t >= 0; --t) {  // the smallest terms first
#pragma unroll
      for (int j = 0; j < TN; ++j) b[j] = turned(from + A_BYTES + t * B_BYTES, BN * 2, wn * TN + j, ks);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[j], acc[i][j], 0, 0, 0);
    }
  };

  if (u0 < u1) {
    load(u0);
    store(smem);
    __syncthreads();
    for (int u = u0; u < u1; ++u) {
      uint8_t *here = smem + ((u - u0) & 1) * PLACE, *next = smem + ((u - u0 + 1) & 1) * PLACE;
      if (u + 1 < u1) load(u + 1);
      multiply(here, 0);
      multiply(here, 1);
      multiply(here, 2);
      if (u + 1 < u1) store(next);
      multiply(here, 3);
      __syncthreads();
    }
  }
  // a lane holds a column of each 32 x 32 tile: runs of 128 bytes
  float *out = g.out + (size_t)range * g.K * g.out_ld;
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int n = n0 + (wn * TN + j) * 32 + (lane & 31);
      if (n >= g.N) continue;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int m = m0 + (wm * TM + i) * 32 + (e >> 2) * 8 + (lane >> 5) * 4 + (e & 3);
        if (m >= g.K) continue;
        float *dst = out + (size_t)m * g.out_ld + n;
        *dst = g.add ? *dst + acc[i][j][e] : acc[i][j][e];
      }
    }
}
// the ranges' sums, added in their order
__global__ __launch_bounds__(256) void keep_grad_add_kernel(const float *part, int ranges, int K, int N, float *grad, size_t ld, bool add) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x, count = (size_t)K * N;
  if (i >= count) return;
  float s = 0.0f;
  for (int r = 0; r < ranges; ++r) s += part[(size_t)r * count + i];
  float *dst = grad + i / N * ld + i % N;
  *dst = add ? *dst + s : s;
}

}  // namespace

hipError_t fade_keep_launch(const OpMat &x, size_t width, const OpKeep &k, hipStream_t s) {
  const int shift = lanes_shift(width, 8), rows = 256 >> shift;
  const dim3 grid((uint32_t)((k.rows + rows - 1) / rows));
  if (x.f32) hipLaunchKernelGGL(keep_kernel<float>, grid, dim3(256), 0, s, static_cast<const float *>(x.p), x.ld, (int)width, k, shift);
  else hipLaunchKernelGGL(keep_kernel<bf16_t>, grid, dim3(256), 0, s, static_cast<const bf16_t *>(x.p), x.ld, (int)width, k, shift);
  return hipGetLastError();
}
hipError_t fade_keep_read_launch(const OpKeep &k, size_t width, const OpMat &out, hipStream_t s) {
  const int shift = lanes_shift(width, 8), rows = 256 >> shift;
  const dim3 grid((uint32_t)((k.rows + rows - 1) / rows));
  void *p = const_cast<void *>(out.p);
  if (out.f32) hipLaunchKernelGGL(keep_read_kernel<float>, grid, dim3(256), 0, s, k, (int)width, static_cast<float *>(p), out.ld, shift);
  else hipLaunchKernelGGL(keep_read_kernel<bf16_t>, grid, dim3(256), 0, s, k, (int)width, static_cast<bf16_t *>(p), out.ld, shift);
  return hipGetLastError();
}

size_t fade_keep_grad_bytes(size_t rows, size_t in_width, size_t out_width) {
  size_t most = 0;
  for (const bool f32 : {false, true}) {
    const WgradPlan p = wgrad_plan(rows, in_width, out_width, f32);
    const size_t bytes = p.ranges > 1 ? 4 * (size_t)p.ranges * in_width * out_width : 0;
    most = bytes > most ? bytes : most;
  }
  return most;
}
template <int WM, int WN, int TM, int TN, bool F32> static hipError_t wgrad_go(const WgradArgs &g, hipStream_t s) {
  constexpr int BM = WM * TM * 32, BN = WN * TN * 32, LDS = 2 * (64 * BM * 2 + (F32 ? 3 : 1) * 64 * BN * 2);
  static_assert(LDS <= 160 * 1024, "LDS");
  const void *f = reinterpret_cast<const void *>(keep_grad_kernel<WM, WN, TM, TN, F32>);
  if constexpr (LDS > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((keep_grad_kernel<WM, WN, TM, TN, F32>), dim3((uint32_t)((size_t)g.tiles_m * g.tiles_n * g.ranges)), dim3(WM * WN * 64), LDS, s, g);
  return hipGetLastError();
}
hipError_t fade_keep_grad_launch(const OpKeep &k, size_t in_width, const OpMat &dy, size_t out_width, float *grad, size_t grad_ld, bool accumulate,
                                 void *work, hipStream_t s) {
  const WgradPlan p = wgrad_plan(k.rows, in_width, out_width, dy.f32);
  const bool parts = p.ranges > 1;
  const WgradArgs g{k, dy.p, dy.ld, (int)in_width, (int)out_width, p.tiles_m, p.tiles_n, p.ranges, p.units, p.per, parts ? static_cast<float *>(work) : grad,
                    parts ? out_width : grad_ld, !parts && accumulate};
  const hipError_t e = dy.f32 ? (p.large ? wgrad_go<4, 2, 2, 2, true>(g, s) : wgrad_go<2, 2, 2, 2, true>(g, s))
                              : (p.large ? wgrad_go<2, 4, 4, 2, false>(g, s) : wgrad_go<2, 2, 2, 2, false>(g, s));
  if (e != hipSuccess) return e;
  if (parts)
    hipLaunchKernelGGL(keep_grad_add_kernel, dim3((uint32_t)((in_width * out_width + 255) / 256)), dim3(256), 0, s, static_cast<const float *>(work),
                       p.ranges, (int)in_width, (int)out_width, grad, grad_ld, accumulate);
  return hipGetLastError();
}
