// fade_keep.hip — activations kept in 8 bits between the passes, and the weight gradient from them (gfx950).
//
// A group of 32 columns shares a power of two, so what a checkpoint stands for is exact in bf16, and a product with it runs on the bf16 matrix
// cores with nothing rounded but the fp32 sums. Writing and reading are one pass over the data, bounded by its bytes: 16384 x 4096, bf16, 46 and 30 us, 39 and 29 at best (203 MB each).
// The weight gradient dW = x^T dy contracts over the rows: the row-major tiles of both operands are turned on their way out of LDS (ds_read_b64_tr_b16), x is widened
// to bf16 on its way in. An fp32 dy goes in as three bf16 terms, each the leading 8 bits of what the ones before left: 24 bits, so that they add up to it
// (three products at the bf16 rate: 16384 rows, 2048 x 2048 351 us with the sum of four ranges, 1.17 PFLOP/s of matrix work; a library's fp32 product of that size takes 900).
#include <type_traits>

#include "../../include/fade.h"
#include "fade_op_rules.h"
#include "fade_ops.h"

namespace {
using namespace fade_op;

template <typename T>
__global__ __launch_bounds__(256) void keep_kernel(const T *x, size_t ld, int width, OpKeep k, int shift) {
  for (size_t row = (size_t)blockIdx.x * (256 >> shift) + (threadIdx.x >> shift); row < k.rows; row += (size_t)gridDim.x * (256 >> shift)) {
    uint8_t *q = k.p + row * k.groups * 32, *e = k.p + k.rows * k.groups * 32 + row * k.groups;
    for (int c = (threadIdx.x & ((1 << shift) - 1)) * 8; c < k.groups * 32; c += 8 << shift) {  // a quad's lanes together
      float v[8];
      OpRaw<T> in;
      if (c < width) in.load(x + row * ld + c, width - c, c);
      else in.zero();
      in.fix(width - c, c);
      in.get(v);
      uint32_t exp;
      const uint2 w = op_keep_pack(v, exp);
      *reinterpret_cast<uint2 *>(q + c) = w;
      if ((threadIdx.x & 3) == 0) e[c >> 5] = (uint8_t)exp;
    }
  }
}
template <typename T>
__global__ __launch_bounds__(256) void keep_read_kernel(OpKeep k, int width, T *out, size_t ld, int shift) {
  for (size_t row = (size_t)blockIdx.x * (256 >> shift) + (threadIdx.x >> shift); row < k.rows; row += (size_t)gridDim.x * (256 >> shift)) {
    const uint8_t *q = k.p + row * k.groups * 32, *e = k.p + k.rows * k.groups * 32 + row * k.groups;
    for (int c = (threadIdx.x & ((1 << shift) - 1)) * 8; c < width; c += 8 << shift) {
      float v[8];
      op_keep_unpack(*reinterpret_cast<const uint2 *>(q + c), op_keep_unit(e[c >> 5]), v);
      OpRaw<T> o;
      o.put(v);
      o.store(out + row * ld + c, width - c);
    }
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

// fp32 as the leading 8 bits, the next 8, the last 8: cut, not rounded, so that nothing overflows and the rest is exact (of numbers below 2^-110 down to
// 2^-133, bf16's smallest, which the matrix cores do not flush)
__device__ __forceinline__ void wg_split(float v, uint32_t &hi, uint32_t &mid, uint32_t &lo) {
  hi = __builtin_bit_cast(uint32_t, v) & 0xffff0000u;
  float rest = v - __builtin_bit_cast(float, hi);
  if (fabsf(v) == __builtin_inff()) rest = 0.0f;  // an infinity is its first term alone; a NaN stays one in the second
  mid = __builtin_bit_cast(uint32_t, rest) & 0xffff0000u;
  lo = __builtin_bit_cast(uint32_t, rest - __builtin_bit_cast(float, mid));
}
__device__ __forceinline__ uint32_t wg_upper(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }  // upper halves, a's first
__device__ __forceinline__ bf16x8 wg_widen(uint32_t lo, uint32_t hi, uint32_t e) {  // 8 bytes of a checkpoint as bf16, exactly
  float v[8];
  op_keep_unpack(make_uint2(lo, hi), op_keep_unit(e), v);
  bf16x8 b;
#pragma unroll
  for (int k = 0; k < 8; ++k) b[k] = (bf16_t)v[k];
  return b;
}

// MM matrix instructions, between them evenly RD reads of LDS, WR writes and VA vector instructions, as the compiler is told to order them
template <int MM, int RD, int WR, int VA, int K = 0> __device__ __forceinline__ void wg_pace() {
  if constexpr (K < MM) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if constexpr (RD * (K + 1) / MM > RD * K / MM) __builtin_amdgcn_sched_group_barrier(0x100, RD * (K + 1) / MM - RD * K / MM, 0);
    if constexpr (VA * (K + 1) / MM > VA * K / MM) __builtin_amdgcn_sched_group_barrier(0x002, VA * (K + 1) / MM - VA * K / MM, 0);
    if constexpr (WR * (K + 1) / MM > WR * K / MM) __builtin_amdgcn_sched_group_barrier(0x200, WR * (K + 1) / MM - WR * K / MM, 0);
    wg_pace<MM, RD, WR, VA, K + 1>();
  }
}
// WM x WN wavefronts, each TM x TN tiles of 32 x 32. Units of 64 rows pass through two places in LDS: while the matrix cores work on one, the
// next is on its way through the registers (x has to be widened, an fp32 dy split, on the way) into the other; one barrier a unit. Loads are a unit ahead of the
// stores into LDS, operand reads a step of 16 rows ahead of the matrix instructions. 256 x 256 tiles: 1.9 us a unit and compute unit at 1.12 PFLOP/s (the library's
// bf16 product 1.22); the matrix cores are busy 53 % of the cycles, LDS 40 %, the vector ALU 33 %, at the clock that this power leaves. Tried and no
// faster: four wavefronts of 128 x 128 (340 us instead of 260 at 16384 rows, 4096 x 2048), all of a unit's stores at one step, 128 x 256 tiles without ranges (300).
template <int WM, int WN, int TM, int TN, bool F32> __global__ __launch_bounds__(WM * WN * 64, 1) void keep_grad_kernel(WgradArgs g) {
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
  typedef std::conditional_t<F32, float, bf16_t> TD;
  // This thread's pieces: where they go in a place, and where the unit's come from, as an offset from the unit's first row; its pieces are XS (YS) rows
  // apart, multiples of 4, so the others follow from the first. Columns that do not exist read column 0: what they bring reaches only results that do not exist.
  constexpr int XS = NT / (BM / 16), YS = NT / (BN / 8);
  static_assert(XS % 4 == 0 && YS % 4 == 0, "the permutation of a piece's row");
  const int xr = tid / (BM / 16), xc = tid % (BM / 16), xcol = m0 + xc * 16 < (int)pitch ? m0 + xc * 16 : 0;
  const int yr = tid / (BN / 8), yc = n0 + tid % (BN / 8) * 8, ycol = yc < g.N ? yc : 0;
  const int x_at = piece_at(BM * 2, xr, xc * 2), y_at = A_BYTES + piece_at(BN * 2, yr, tid % (BN / 8));
  const uint32_t x_off = (uint32_t)xr * (uint32_t)pitch + xcol, e_off = (uint32_t)xr * g.x.groups + (xcol >> 5);
  const uint32_t y_off = (uint32_t)yr * (uint32_t)g.dy_ld + ycol;
  const uint8_t *x_row = g.x.p + (size_t)u0 * 64 * pitch, *e_row = g.x.p + g.x.rows * pitch + (size_t)u0 * 64 * g.x.groups;
  const TD *y_row = static_cast<const TD *>(g.dy) + (size_t)u0 * 64 * g.dy_ld;
  uint4 qx[QA];
  uint32_t ex[QA];
  OpRaw<TD> qy[QB];
  // The last unit, whose rows may end and whose last piece of dy may reach past the matrix, is loaded with every access checked. In the others a piece that
  // starts in a row ends in the next one at the latest (rows of 8 columns or more), which exists.
  auto load = [&](int u) {  // units in order
    if (u + 1 < g.units && g.N >= 8) {
#pragma unroll
      for (int i = 0; i < QA; ++i) {
        qx[i] = *reinterpret_cast<const uint4 *>(x_row + i * XS * pitch + x_off);
        ex[i] = (e_row + (size_t)i * XS * g.x.groups)[e_off];
      }
#pragma unroll
      for (int i = 0; i < QB; ++i) qy[i].load(y_row + i * YS * g.dy_ld + y_off, 8);
    } else {
      const int left = (int)(g.x.rows - (size_t)u * 64 < 64 ? g.x.rows - (size_t)u * 64 : 64);
#pragma unroll
      for (int i = 0; i < QA; ++i) {
        qx[i] = make_uint4(0, 0, 0, 0);
        ex[i] = 0;
        if (xr + i * XS < left) {
          qx[i] = *reinterpret_cast<const uint4 *>(x_row + i * XS * pitch + x_off);
          ex[i] = (e_row + (size_t)i * XS * g.x.groups)[e_off];
        }
      }
#pragma unroll
      for (int i = 0; i < QB; ++i) {
        qy[i].zero();
        if (yr + i * YS < left && yc < g.N) qy[i].load(y_row + i * YS * g.dy_ld + y_off, g.N - yc);
      }
    }
    x_row += pitch * 64;
    e_row += (size_t)g.x.groups * 64;
    y_row += g.dy_ld * 64;
  };
  // what has been loaded, into a place: a quarter at each step (bf16), or all of it at the third (fp32, whose splitting the compiler spreads better by itself)
  auto store = [&](uint8_t *to, int quarter) {
    if (F32 && quarter != 2) return;
#pragma unroll
    for (int h = 0; h < 2 * QA; ++h)
      if (F32 || h * 4 / (2 * QA) == quarter) {  // an even piece's neighbour is its neighbour after the permutation too
        uint32_t lo = h % 2 ? qx[h / 2].z : qx[h / 2].x, hi = h % 2 ? qx[h / 2].w : qx[h / 2].y;
        if constexpr (!F32) asm volatile("" : "+v"(lo), "+v"(hi));  // its quarter's work stays among its quarter's matrix instructions
        *reinterpret_cast<bf16x8 *>(to + x_at + h / 2 * XS * BM * 2 + h % 2 * 16) = wg_widen(lo, hi, ex[h / 2]);
      }
#pragma unroll
    for (int i = 0; i < QB; ++i)
      if (F32 || i * 4 / QB == quarter) {
        if constexpr (F32) {
          float v[8];
          qy[i].get(v);
          uint32_t w[3][8];
#pragma unroll
          for (int k = 0; k < 8; ++k) wg_split(v[k], w[0][k], w[1][k], w[2][k]);
#pragma unroll
          for (int t = 0; t < 3; ++t)
            *reinterpret_cast<uint4 *>(to + y_at + i * YS * BN * 2 + t * B_BYTES) = make_uint4(wg_upper(w[t][0], w[t][1]), wg_upper(w[t][2], w[t][3]),
                                                                                wg_upper(w[t][4], w[t][5]), wg_upper(w[t][6], w[t][7]));
        } else {
          *reinterpret_cast<uint4 *>(to + y_at + i * YS * BN * 2) = make_uint4(qy[i].v[0], qy[i].v[1], qy[i].v[2], qy[i].v[3]);
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
  // operands of one step of 16 rows, read a step ahead of the matrix instructions
  bf16x8 a[2][TM], b[2][PLANES][TN];
  auto read = [&](int buf, const uint8_t *from, int ks) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int t = PLANES - 1; t >= 0; --t) b[buf][t][j] = turned(from + A_BYTES + t * B_BYTES, BN * 2, wn * TN + j, ks);
#pragma unroll
    for (int i = 0; i < TM; ++i) a[buf][i] = turned(from, BM * 2, wm * TM + i, ks);
  };
  auto multiply = [&](int buf) {
#pragma unroll
    for (int t = PLANES - 1; t >= 0; --t)  // the smallest terms first
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[buf][i], b[buf][t][j], acc[i][j], 0, 0, 0);
  };
  // a step's matrix instructions, and between them the next step's reads and a quarter of the next unit's way into LDS
  constexpr int MM = PLANES * TM * TN, RD = 2 * (TM + PLANES * TN), WR = F32 ? 0 : QA / 2 + QB / 4, VA = F32 ? 0 : QA / 2 * 24;
  auto hand_over = [] {  // this wavefront's LDS accesses are done; then everybody's
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  if (u0 < u1) {
    uint8_t *here = smem, *next = smem + PLACE;
    load(u0);
#pragma unroll
    for (int k = 0; k < 4; ++k) store(here, k);
    if (u0 + 1 < u1) load(u0 + 1);
    hand_over();
    read(0, here, 0);
    for (int u = u0; u + 1 < u1; ++u) {
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        __builtin_amdgcn_sched_barrier(0);
        read((k + 1) & 1, here, k + 1);
        store(next, k);
        multiply(k & 1);
        if (!F32 || k < 2) wg_pace<MM, RD, WR, VA>();
      }
      __builtin_amdgcn_sched_barrier(0);
      store(next, 3);
      if (u + 2 < u1) load(u + 2);
      hand_over();
      read(0, next, 0);
      multiply(1);
      wg_pace<MM, RD, 0, 0>();
      uint8_t *t = here;
      here = next;
      next = t;
    }
    read(1, here, 1);
    multiply(0);
    read(0, here, 2);
    multiply(1);
    read(1, here, 3);
    multiply(0);
    multiply(1);
  }
  // a lane holds a column of each 32 x 32 tile: runs of 128 bytes
  float *out = g.out + (size_t)range * g.K * g.out_ld;
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int n = n0 + (wn * TN + j) * 32 + (lane & 31), m = m0 + (wm * TM + i) * 32 + (lane >> 5) * 4;
      if (n >= g.N) continue;
      float *dst = out + (size_t)m * g.out_ld + n;
      const auto row = [](int e) { return (e >> 2) * 8 + (e & 3); };
      if (g.add) {  // all of what is there at once
        float old[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) old[e] = m + row(e) < g.K ? dst[(size_t)row(e) * g.out_ld] : 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] += old[e];
      }
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (m + row(e) < g.K) dst[(size_t)row(e) * g.out_ld] = acc[i][j][e];
    }
}
// The ranges' sums, added in their order, V pieces of four values per thread: a gradient without gaps between its rows is one run of values; else a
// workgroup takes 1024 V columns of a row.
template <int V>
__global__ __launch_bounds__(256) void keep_grad_add_kernel(const float *part, int ranges, size_t count, int N, int blocks_n, float *grad, size_t ld, bool add) {
  size_t row = 0, first = (size_t)blockIdx.x * (1024 * V), have = count;
  if (blocks_n) {
    row = blockIdx.x / blocks_n;
    first = (blockIdx.x - row * blocks_n) * (1024 * V);
    have = N;
  }
  const float *src = part + row * N + first;
  float *dst = grad + row * ld + first;
  const int left = have - first < 1024 * V ? (int)(have - first) : 1024 * V, at = threadIdx.x * 4;
  op_f32x4 s[V];
#pragma unroll
  for (int k = 0; k < V; ++k) s[k] = op_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  constexpr int AHEAD = 8 / V;  // ranges whose loads are on their way together
  if (at + (V - 1) * 1024 + 4 <= left) {
#pragma unroll AHEAD
    for (int r = 0; r < ranges; ++r, src += count)
#pragma unroll
      for (int k = 0; k < V; ++k) s[k] += *reinterpret_cast<const op_f32x4 *>(src + at + k * 1024);
  } else {  // what does not exist is the block's first value again, and not stored
#pragma unroll AHEAD
    for (int r = 0; r < ranges; ++r, src += count)
#pragma unroll
      for (int k = 0; k < V; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[k][i] += src[at + k * 1024 + i < left ? at + k * 1024 + i : 0];
  }
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const int c = at + k * 1024;
    if (c + 4 <= left) {
      op_f32x4 *to = reinterpret_cast<op_f32x4 *>(dst + c);
      *to = add ? *to + s[k] : s[k];
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (c + i < left) dst[c + i] = add ? dst[c + i] + s[k][i] : s[k][i];
    }
  }
}

}  // namespace

hipError_t fade_keep_launch(const OpMat &x, size_t width, const OpKeep &k, hipStream_t s) {
  const int shift = lanes_shift(width, 8), rows = 256 >> shift;
  const dim3 grid(row_blocks(k.rows, rows));
  if (x.f32) hipLaunchKernelGGL(keep_kernel<float>, grid, dim3(256), 0, s, static_cast<const float *>(x.p), x.ld, (int)width, k, shift);
  else hipLaunchKernelGGL(keep_kernel<bf16_t>, grid, dim3(256), 0, s, static_cast<const bf16_t *>(x.p), x.ld, (int)width, k, shift);
  return hipGetLastError();
}
hipError_t fade_keep_read_launch(const OpKeep &k, size_t width, const OpMat &out, hipStream_t s) {
  const int shift = lanes_shift(width, 8), rows = 256 >> shift;
  const dim3 grid(row_blocks(k.rows, rows));
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
  if (k.rows == 0 && accumulate) return hipSuccess;  // not even a zero is added: it would make a positive zero of a negative one
  const WgradPlan p = wgrad_plan(k.rows, in_width, out_width, dy.f32);
  const bool parts = p.ranges > 1;
  const WgradArgs g{k, dy.p, dy.ld, (int)in_width, (int)out_width, p.tiles_m, p.tiles_n, p.ranges, p.units, p.per, parts ? static_cast<float *>(work) : grad,
                    parts ? out_width : grad_ld, !parts && accumulate};
  const hipError_t e = dy.f32 ? (p.large ? wgrad_go<4, 2, 2, 2, true>(g, s) : wgrad_go<2, 4, 2, 1, true>(g, s))
                              : (p.large ? wgrad_go<2, 4, 4, 2, false>(g, s) : wgrad_go<2, 4, 2, 1, false>(g, s));
  if (e != hipSuccess) return e;
  if (parts) {
    const size_t count = in_width * out_width;
    const bool gaps = grad_ld != out_width, four = count >= (size_t)1 << 22;  // pieces enough for every compute unit
    const size_t block = four ? 4096 : 1024, wide = (out_width + block - 1) / block;
    const dim3 grid((uint32_t)(gaps ? in_width * wide : (count + block - 1) / block));
    auto *f = four ? keep_grad_add_kernel<4> : keep_grad_add_kernel<1>;
    hipLaunchKernelGGL(f, grid, dim3(256), 0, s, static_cast<const float *>(work), p.ranges, count, (int)out_width, gaps ? (int)wide : 0, grad, grad_ld, accumulate);
  }
  return hipGetLastError();
}
