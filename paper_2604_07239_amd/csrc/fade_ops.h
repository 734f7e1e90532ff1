// fade_ops.h — the operators around a program's own model: launchers, and what their kernels share (internal to the library).
#pragma once
#include "fade_dev.h"

// rows of `ld` elements; f32 says which type
struct OpMat {
  const void *p;
  size_t ld;
  bool f32;
};
struct OpTokens {
  const void *p;
  int type;  // FADE_TOKEN_*
};
struct OpKeep {  // a checkpoint: bytes [rows][32 groups], exponents [rows][groups]
  uint8_t *p;
  size_t rows;
  int groups;
};

hipError_t fade_embed_launch(const OpTokens &t, size_t n, const OpMat &table, size_t vocab, size_t width, float scale, const OpMat &out, hipStream_t s);
size_t fade_embed_grad_bytes(size_t n, size_t vocab, size_t width);
hipError_t fade_embed_grad_launch(const OpTokens &t, size_t n, const OpMat &dout, float scale, float *grad, size_t grad_ld, size_t vocab, size_t width,
                                  bool accumulate, void *work, hipStream_t s);

hipError_t fade_keep_launch(const OpMat &x, size_t width, const OpKeep &k, hipStream_t s);
hipError_t fade_keep_read_launch(const OpKeep &k, size_t width, const OpMat &out, hipStream_t s);
size_t fade_keep_grad_bytes(size_t rows, size_t in_width, size_t out_width);
hipError_t fade_keep_grad_launch(const OpKeep &k, size_t in_width, const OpMat &dy, size_t out_width, float *grad, size_t grad_ld, bool accumulate,
                                 void *work, hipStream_t s);

struct JoinArgs {  // the C ABI's fade_join_args, checked; no pointer that is not used
  int rows, width, norm_u, norm_n;
  float eps;
  int lam_count;
  bool accumulate;
  bool stream_f32, branch_f32, kept;
  const float *lam, *gamma_u, *beta_u, *gamma_n, *beta_n;
  const void *r, *u, *g;
  size_t r_ld, u_ld, g_ld;
  void *h, *n;
  size_t h_ld, n_ld;
  uint8_t *keep_r, *keep_u, *keep_g, *keep_n;
  const void *dh, *dn;
  size_t dh_ld, dn_ld;
  void *dr, *du, *dg;
  size_t dr_ld, du_ld, dg_ld;
  float *d_lam, *d_gamma_u, *d_beta_u, *d_gamma_n, *d_beta_n;
  float *work;
};
size_t fade_join_grad_bytes(size_t rows, size_t width);
hipError_t fade_join_launch(const JoinArgs &a, hipStream_t s);
hipError_t fade_join_grad_launch(const JoinArgs &a, hipStream_t s);

// ---------------------------------------------------------------------------------------------------
// 8 neighbouring elements of a row. Rows of any width and ld: the 16-byte accesses may start at any element (gfx950 takes
// global accesses of 16 bytes on any address in one instruction), so there is one path for all strides. The last columns of a row that is no whole number
// of pieces: the 8 that end with the row are loaded, which fix() moves to their places once they are there (a join of 8000 x 1001 whose last columns came
// one by one took 31 us, this way 23, 8000 x 1008 17.5); rows of fewer than 8 columns, and stores, go one by one.
// ---------------------------------------------------------------------------------------------------
typedef uint32_t op_u32x4 __attribute__((ext_vector_type(4), aligned(2)));
typedef float op_f32x4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T> struct OpRaw;  // 8 elements as they are in memory
template <> struct OpRaw<bf16_t> {
  op_u32x4 v;
  __device__ __forceinline__ void zero() { v = op_u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ void load(const bf16_t *p, int left, int c = 0) {  // left >= 1: how many of the 8 exist; c: the column p stands at
    if (left >= 8 || c >= 8) {
      v = *reinterpret_cast<const op_u32x4 *>(p - (left >= 8 ? 0 : 8 - left));
    } else {
      uint32_t w[4] = {0, 0, 0, 0};
      const uint16_t *q = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < left) w[i >> 1] |= (uint32_t)q[i] << ((i & 1) * 16);
      v = op_u32x4{w[0], w[1], w[2], w[3]};
    }
  }
  __device__ __forceinline__ void fix(int left, int c) {  // what load(.., left, c) brought, in its places
    if (left >= 8 || left <= 0 || c < 8) return;
    const int s = 8 - left;
    if (s & 4) v = op_u32x4{v[2], v[3], 0, 0};
    if (s & 2) v = op_u32x4{v[1], v[2], v[3], 0};
    if (s & 1) v = op_u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
  }
  __device__ __forceinline__ void get(float x[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __builtin_bit_cast(float, v[i] << 16);
      x[2 * i + 1] = __builtin_bit_cast(float, v[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void put(const float x[8]) {  // to the nearest, ties to even
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (bf16_t)x[i];
    v = __builtin_bit_cast(op_u32x4, r);
  }
  __device__ __forceinline__ void store(bf16_t *p, int left) const {
    if (left >= 8) {
      *reinterpret_cast<op_u32x4 *>(p) = v;
    } else {
      uint16_t *q = reinterpret_cast<uint16_t *>(p);
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < left) q[i] = (uint16_t)(v[i >> 1] >> ((i & 1) * 16));
    }
  }
};
template <> struct OpRaw<float> {
  op_f32x4 a, b;
  __device__ __forceinline__ void zero() { a = b = op_f32x4{0.0f, 0.0f, 0.0f, 0.0f}; }
  __device__ __forceinline__ void load(const float *p, int left, int c = 0) {
    if (left >= 8 || c >= 8) {
      p -= left >= 8 ? 0 : 8 - left;
      a = *reinterpret_cast<const op_f32x4 *>(p);
      b = *reinterpret_cast<const op_f32x4 *>(p + 4);
    } else {
      float w[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < left) w[i] = p[i];
      a = op_f32x4{w[0], w[1], w[2], w[3]};
      b = op_f32x4{w[4], w[5], w[6], w[7]};
    }
  }
  __device__ __forceinline__ void fix(int left, int c) {
    if (left >= 8 || left <= 0 || c < 8) return;
    const int s = 8 - left;
    if (s & 4) { a = b; b = op_f32x4{0.0f, 0.0f, 0.0f, 0.0f}; }
    if (s & 2) { a = op_f32x4{a[2], a[3], b[0], b[1]}; b = op_f32x4{b[2], b[3], 0.0f, 0.0f}; }
    if (s & 1) { a = op_f32x4{a[1], a[2], a[3], b[0]}; b = op_f32x4{b[1], b[2], b[3], 0.0f}; }
  }
  __device__ __forceinline__ void get(float x[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
  }
  __device__ __forceinline__ void put(const float x[8]) {
    a = op_f32x4{x[0], x[1], x[2], x[3]};
    b = op_f32x4{x[4], x[5], x[6], x[7]};
  }
  __device__ __forceinline__ void store(float *p, int left) const {
    if (left >= 8) {
      *reinterpret_cast<op_f32x4 *>(p) = a;
      *reinterpret_cast<op_f32x4 *>(p + 4) = b;
    } else {
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < left) p[i] = i < 4 ? a[i] : b[i - 4];
    }
  }
};

// ---------------------------------------------------------------------------------------------------
// 8-bit checkpoints: a group of 32 columns is four lanes of 8 columns each, neighbours inside a quad.
// ---------------------------------------------------------------------------------------------------
// Exponent byte e + 127 of a group from the bits of its largest magnitude: with top = m 2^k, 127 = 1.984375 * 2^6, the least e is k - 6, or k - 5
// where m > 1.984375 (mantissa bits over 0x7e0000), 121 at most; 255: an infinity or NaN is among them.
constexpr uint32_t OP_KEEP_EXP_MAX = 121 + 127;
__device__ __forceinline__ uint32_t op_keep_exp(uint32_t top) {
  const int k = (int)(top >> 23);
  const int e = k - 6 + ((top & 0x7fffffu) > 0x7e0000u ? 1 : 0);
  return k == 255 ? 255u : (uint32_t)min(max(e, 1), (int)OP_KEEP_EXP_MAX);
}
// 2^e of an exponent byte; 255 gives an infinity: 0 * infinity is the NaN such a group reads back as (its bytes are zeros)
__device__ __forceinline__ float op_keep_unit(uint32_t e) { return __builtin_bit_cast(float, e << 23); }
__device__ __forceinline__ uint32_t op_quad_max(uint32_t v) {  // over the four lanes of a quad
  uint32_t o = fade_dpp<0xB1>(v);
  v = v > o ? v : o;
  o = fade_dpp<0x4E>(v);
  return v > o ? v : o;
}
// The 8 bytes of this lane's columns and the group's exponent byte. Every lane of the quad takes part; columns that do not exist hold zeros.
// x 2^-e + 1.5 * 2^23 is rounded to a whole number, ties to even, whose two's complement is in its low bits: one instruction a value, and one that keeps it within 127
// where the exponent is at its end (for all groups: a branch for those alone took registers that cost the join one of four wavefronts: 149 us instead of 139 at 9000 x 4095).
__device__ __forceinline__ uint2 op_keep_pack(const float x[8], uint32_t &e) {
  // bits of magnitudes are in the magnitudes' order, infinities and NaNs on top
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t m = __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffffu;
    top = m > top ? m : top;
  }
  e = op_keep_exp(op_quad_max(top));
  if (e == 255) return make_uint2(0, 0);
  const float inv = __builtin_bit_cast(float, (254u - e) << 23);
  uint32_t q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_fmed3f(fmaf(x[i], inv, 12582912.0f), 12582912.0f - 127.0f, 12582912.0f + 127.0f));
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t a = __builtin_amdgcn_perm(q[4 * i + 1], q[4 * i], 0x0c0c0400u), b = __builtin_amdgcn_perm(q[4 * i + 3], q[4 * i + 2], 0x0c0c0400u);
    w[i] = a | b << 16;
  }
  return make_uint2(w[0], w[1]);
}
// A byte of a word is converted with its sign in one instruction (SDWA), then scaled. An infinite unit gives NaNs.
__device__ __forceinline__ void op_keep_unpack(const uint2 q, float unit, float x[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)(int8_t)((i < 4 ? q.x : q.y) >> ((i & 3) * 8)) * unit;
}
