// fade_keep.hip — activations kept in 8 bits between the passes, and the weight gradient from them (gfx950).
//
// A group of 32 columns shares a power of two, so what a checkpoint stands for is exact in bf16, and a product with it runs on the bf16 matrix
// cores with nothing rounded but the fp32 sums. Writing and reading are one pass over the data, bounded by its bytes. The weight gradient dW = x^T dy contracts over the rows: the
// row-major tiles of both operands are turned on their way out of LDS (ds_read_b64_tr_b16), x is widened to bf16 on its way in.
// An fp32 dy goes in as three bf16 terms, each the leading 8 bits of what the ones before left: 24 bits, so that they add up to it.
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
  int K, N, tiles_n, units, per;  // units of 64 rows; units in one range
  float *out;                     // the gradient, or the ranges' sums [range][K][N]
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

template <bool F32>
__global__ __launch_bounds__(256) void keep_grad_kernel(WgradArgs g) {
  constexpr int PLANES = F32 ? 3 : 1, UNIT = 64 * WT * 2;
  __shared__ __align__(16) uint8_t smem[(1 + PLANES) * UNIT];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1;
  const int m0 = (int)(blockIdx.x / g.tiles_n) * WT, n0 = (int)(blockIdx.x % g.tiles_n) * WT;
  const int range = blockIdx.y, u0 = range * g.per, u1 = u0 + g.per < g.units ? u0 + g.per : g.units;
  const size_t pitch = (size_t)g.x.groups * 32;
  const uint8_t *exps = g.x.p + g.x.rows * pitch;

  // a row of a tile is 16 pieces of 16 bytes; piece p of row r lies at p ^ 4 (r % 4): four rows of a column block in four quarters of the banks
  auto piece_at = [](int r, int p) { return r * (WT * 2) + ((p ^ ((r & 3) << 2)) << 4); };
  // transposing reads: in each group of 16 lanes, lane s supplies the address of row s / 4, columns 4 (s % 4) .. + 3 of a 4 x 16 block, and
  // lane i receives column i with the block's 4 rows in order; two such loads make the 8 rows of a lane's column
  const int s16 = lane & 15, r0 = (lane >> 5) * 8 + (s16 >> 2), mh = (lane >> 4) & 1;
  auto turned = [&](const uint8_t *base, int tile, int ks) {
    const int r = ks * 16 + r0, p = tile * 4 + 2 * mh + ((s16 & 3) >> 1);
    const uint8_t *at = base + piece_at(r, p) + (s16 & 1) * 8;
    const i16x4 lo = wg_turn(at), hi = wg_turn(at + 4 * WT * 2);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

  for (int u = u0; u < u1; ++u) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {  // x: 16 columns of a row at a time
      const int r = (tid >> 3) + i * 32, c = (tid & 7) * 16;
      const size_t row = (size_t)u * 64 + r;
      uint4 q = make_uint4(0, 0, 0, 0);
      float unit = 0.0f;
      if (row < g.x.rows && (size_t)(m0 + c) < pitch) {
        q = *reinterpret_cast<const uint4 *>(g.x.p + row * pitch + m0 + c);
        unit = op_keep_unit(exps[row * g.x.groups + ((m0 + c) >> 5)]);
      }
      float v[8];
      bf16x8 b;
      op_keep_unpack(make_uint2(q.x, q.y), unit, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) b[k] = (bf16_t)v[k];
      *reinterpret_cast<bf16x8 *>(smem + piece_at(r, (tid & 7) * 2)) = b;
      op_keep_unpack(make_uint2(q.z, q.w), unit, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) b[k] = (bf16_t)v[k];
      *reinterpret_cast<bf16x8 *>(smem + piece_at(r, (tid & 7) * 2 + 1)) = b;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // dy: 8 columns at a time
      const int r = (tid >> 4) + i * 16, p = tid & 15, n = n0 + p * 8;
      const size_t row = (size_t)u * 64 + r;
      const bool in = row < g.x.rows && n < g.N;
      uint8_t *at = smem + UNIT + piece_at(r, p);
      if constexpr (F32) {
        OpRaw<float> raw;
        raw.zero();
        if (in) raw.load(static_cast<const float *>(g.dy) + row * g.dy_ld + n, g.N - n);
        float v[8];
        raw.get(v);
        uint32_t w[3][8];
#pragma unroll
        for (int k = 0; k < 8; ++k) wg_split(v[k], w[0][k], w[1][k], w[2][k]);
#pragma unroll
        for (int t = 0; t < 3; ++t)
          *reinterpret_cast<uint4 *>(at + t * UNIT) = make_uint4(w[t][0] >> 16 | (w[t][1] & 0xffff0000u), w[t][2] >> 16 | (w[t][3] & 0xffff0000u),
                                                                 w[t][4] >> 16 | (w[t][5] & 0xffff0000u), w[t][6] >> 16 | (w[t][7] & 0xffff0000u));
      } else {
        OpRaw<bf16_t> raw;
        raw.zero();
        if (in) raw.load(static_cast<const bf16_t *>(g.dy) + row * g.dy_ld + n, g.N - n);
        *reinterpret_cast<uint4 *>(at) = make_uint4(raw.v[0], raw.v[1], raw.v[2], raw.v[3]);
      }
    }
    __syncthreads();
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      bf16x8 a[2], b[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) a[i] = turned(smem, wm * 2 + i, ks);
#pragma unroll
      for (int t = PLANES - 1; t >= 0; --t) {
#pragma unroll
        for (int j = 0; j < 2; ++j) b[j] = turned(smem + (1 + t) * UNIT, wn * 2 + j, ks);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[j], acc[i][j], 0, 0, 0);
      }
    }
  }
  // a lane holds a column of each 32 x 32 tile: runs of 128 bytes
  float *out = g.out + (size_t)range * g.K * g.out_ld;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int n = n0 + (wn * 2 + j) * 32 + (lane & 31);
      if (n >= g.N) continue;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int m = m0 + (wm * 2 + i) * 32 + (e >> 2) * 8 + (lane >> 5) * 4 + (e & 3);
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
hipError_t fade_keep_grad_launch(const OpKeep &k, size_t in_width, const OpMat &dy, size_t out_width, float *grad, size_t grad_ld, bool accumulate,
                                 void *work, hipStream_t s) {
  const WgradPlan p = wgrad_plan(k.rows, in_width, out_width, dy.f32);
  const bool parts = p.ranges > 1;
  WgradArgs g{k, dy.p, dy.ld, (int)in_width, (int)out_width, p.tiles_n, p.units, p.per, parts ? static_cast<float *>(work) : grad,
              parts ? out_width : grad_ld, !parts && accumulate};
  const dim3 grid((uint32_t)((size_t)p.tiles_m * p.tiles_n), (uint32_t)p.ranges);
  if (dy.f32) hipLaunchKernelGGL(keep_grad_kernel<true>, grid, dim3(256), 0, s, g);
  else hipLaunchKernelGGL(keep_grad_kernel<false>, grid, dim3(256), 0, s, g);
  if (parts)
    hipLaunchKernelGGL(keep_grad_add_kernel, dim3((uint32_t)((in_width * out_width + 255) / 256)), dim3(256), 0, s, static_cast<const float *>(work),
                       p.ranges, (int)in_width, (int)out_width, grad, grad_ld, accumulate);
  return hipGetLastError();
}
