// fade_op_checks.h — what the entry points of the operators ask of their arguments, as plain C++ (host tests compile it by itself).
// Each function gives NULL, or what is wrong; nothing here needs a device.
#pragma once
#include <cfloat>
#include <cmath>
#include <initializer_list>
#include <stdint.h>

#include "../../include/fade.h"

namespace fade_op {

constexpr size_t ROWS = 0x7fffffff, WIDTH = (size_t)1 << 20, VOCAB = (size_t)1 << 20, GRAD_WIDTH = 65536, GRAD_LD = (size_t)1 << 22, JOIN_WIDTH = 8192;

inline bool type(uint32_t t) { return t == FADE_F32 || t == FADE_BF16; }
inline bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
// a matrix of `rows` rows: there (unless it has no rows), on whole elements, its rows not on top of one another
inline bool matrix(const void *p, uint32_t t, size_t rows, size_t width, size_t ld) {
  return rows == 0 || (p && type(t) && aligned(p, t == FADE_F32 ? 4 : 2) && ld >= width && ld <= SIZE_MAX / 8 / rows);
}
inline bool tokens(const void *p, int t, size_t n) { return n == 0 || (p && aligned(p, t == FADE_TOKEN_U8 ? 1 : t == FADE_TOKEN_I32 ? 4 : 8)); }
inline bool keep(const void *p, size_t rows) { return rows == 0 || (p && aligned(p, 16)); }
inline bool work(const void *p, size_t have, size_t need) { return p && aligned(p, 16) && have >= need; }
inline bool embed_sizes(size_t n, size_t vocab, size_t width) { return n <= ROWS && vocab > 0 && vocab <= VOCAB && width > 0 && width <= WIDTH; }
inline bool keep_sizes(size_t rows, size_t width) { return rows <= ROWS && width > 0 && width <= WIDTH; }
inline bool grad_sizes(size_t rows, size_t k, size_t n) { return rows <= ROWS && k > 0 && k <= GRAD_WIDTH && n > 0 && n <= GRAD_WIDTH; }
inline bool join_sizes(size_t rows, size_t width) { return rows <= ROWS && width > 0 && width <= JOIN_WIDTH; }

inline const char *embed(const void *tok, int tok_type, size_t n, const void *table, int table_type, size_t table_ld, size_t vocab, size_t width, const void *out,
                         int out_type, size_t out_ld) {
  if (!embed_sizes(n, vocab, width)) return "n, vocab or width out of range";
  if (tok_type < FADE_TOKEN_U8 || tok_type > FADE_TOKEN_I64 || !type(table_type) || !type(out_type)) return "unknown type";
  if (!tokens(tok, tok_type, n)) return "tokens";
  if (n && !matrix(table, table_type, vocab, width, table_ld)) return "table";
  return matrix(out, out_type, n, width, out_ld) ? nullptr : "out";
}
inline const char *embed_grad(const void *tok, int tok_type, size_t n, const void *dout, int dout_type, size_t dout_ld, const float *grad, size_t grad_ld, size_t vocab,
                              size_t width, const void *w, size_t have, size_t need) {
  if (!embed_sizes(n, vocab, width) || need == 0) return "n, vocab or width out of range";
  if (tok_type < FADE_TOKEN_U8 || tok_type > FADE_TOKEN_I64 || !type(dout_type)) return "unknown type";
  if (!tokens(tok, tok_type, n)) return "tokens";
  if (!matrix(dout, dout_type, n, width, dout_ld)) return "dout";
  if (!matrix(grad, FADE_F32, vocab, width, grad_ld)) return "grad";
  return work(w, have, need) ? nullptr : "workspace missing, too small or not aligned to 16 bytes";
}
inline const char *checkpoint(const void *x, int x_type, size_t ld, size_t rows, size_t width, const void *k) {  // either direction
  if (!keep_sizes(rows, width)) return "rows or width out of range";
  if (!type(x_type)) return "unknown type";
  if (!matrix(x, x_type, rows, width, ld)) return "matrix";
  return keep(k, rows) ? nullptr : "checkpoint missing or not aligned to 16 bytes";
}
inline const char *weight_grad(const void *k, size_t rows, size_t in_width, const void *dy, int dy_type, size_t dy_ld, size_t out_width, const float *grad,
                               size_t grad_ld, const void *w, size_t have, size_t need) {
  if (!grad_sizes(rows, in_width, out_width) || need == 0) return "rows or widths out of range";
  if (!type(dy_type)) return "unknown type";
  if (!keep(k, rows)) return "checkpoint missing or not aligned to 16 bytes";
  if (!matrix(dy, dy_type, rows, out_width, dy_ld) || dy_ld > GRAD_LD) return "dy";
  if (!matrix(grad, FADE_F32, in_width, out_width, grad_ld)) return "grad";
  return work(w, have, need) ? nullptr : "workspace missing, too small or not aligned to 16 bytes";
}

// what both directions of the join ask for
inline const char *join_model(const fade_join_args *a, bool grad) {
  if (!a || a->struct_size != sizeof(fade_join_args)) return "arguments or their struct_size";
  if (!join_sizes(a->rows, a->width)) return "rows or width out of range";
  if (a->norm_u > FADE_NORM_RMS || a->norm_n > FADE_NORM_RMS) return "unknown norm";
  if (!type(a->stream_type) || !type(a->branch_type) || (a->branch_type == FADE_F32 && a->stream_type == FADE_BF16)) return "types";
  if (!(a->eps == 0.0f || a->eps >= FLT_MIN) || !std::isfinite(a->eps)) return "eps";  // 1 / sqrt takes a subnormal number for zero
  if (a->lam_count != 0 && a->lam_count != 1 && a->lam_count != a->width) return "lam has neither one value nor one per column";
  if ((a->lam_count != 0) != (a->lam != nullptr)) return "lam and lam_count";
  if (a->norm_u == FADE_NORM_NONE && (a->gamma_u || a->beta_u)) return "parameters of a norm of u that is none";
  if (a->norm_n == FADE_NORM_NONE && (a->gamma_n || a->beta_n)) return "parameters of a norm of h that is none";
  for (const float *p : {a->lam, a->gamma_u, a->beta_u, a->gamma_n, a->beta_n})
    if (!aligned(p, 4)) return "alignment of a parameter";
  for (const void *k : {a->keep_r, a->keep_u, a->keep_g, a->keep_n})
    if (!aligned(k, 16)) return "a checkpoint is not aligned to 16 bytes";
  if (grad && a->keep_u) {
    if (a->r || a->u || a->g) return "operands both as they were and as checkpoints";
    return a->keep_r || a->rows == 0 ? nullptr : "keep_r is missing";
  }
  if (grad && (a->keep_r || a->keep_g)) return "keep_u is missing";
  if (!matrix(a->r, a->stream_type, a->rows, a->width, a->r_ld)) return "r";
  if (!matrix(a->u, a->branch_type, a->rows, a->width, a->u_ld)) return "u";
  return !a->g || matrix(a->g, a->branch_type, a->rows, a->width, a->g_ld) ? nullptr : "g";
}
inline const char *join(const fade_join_args *a) {
  if (const char *why = join_model(a, false)) return why;
  if (!matrix(a->h, a->stream_type, a->rows, a->width, a->h_ld)) return "h";
  if (a->n && !matrix(a->n, a->branch_type, a->rows, a->width, a->n_ld)) return "n";
  if (a->h == a->r && a->rows > 1 && a->h_ld != a->r_ld) return "h on top of r with another ld";
  return a->keep_g && !a->g ? "a checkpoint of g without g" : nullptr;
}
inline const char *join_grad(const fade_join_args *a, size_t need) {
  if (const char *why = join_model(a, true)) return why;
  if (a->rows && !a->dh && !a->dn) return "neither dh nor dn";
  if (a->dh && !matrix(a->dh, a->stream_type, a->rows, a->width, a->dh_ld)) return "dh";
  if (a->dn && !matrix(a->dn, a->branch_type, a->rows, a->width, a->dn_ld)) return "dn";
  if (a->dr && !matrix(a->dr, a->stream_type, a->rows, a->width, a->dr_ld)) return "dr";
  if (a->du && !matrix(a->du, a->branch_type, a->rows, a->width, a->du_ld)) return "du";
  if (a->dg && !matrix(a->dg, a->branch_type, a->rows, a->width, a->dg_ld)) return "dg";
  if (a->dg && !a->g && !a->keep_g) return "dg without a gate";
  if ((a->dr && a->dr == a->dh && a->rows > 1 && a->dr_ld != a->dh_ld) || (a->du && a->du == a->dn && a->rows > 1 && a->du_ld != a->dn_ld))
    return "a gradient on top of another with another ld";
  if (a->d_lam && !a->lam) return "d_lam without lam";
  if (a->norm_u == FADE_NORM_NONE && (a->d_gamma_u || a->d_beta_u)) return "gradients of a norm of u that is none";
  if (a->norm_n == FADE_NORM_NONE && (a->d_gamma_n || a->d_beta_n)) return "gradients of a norm of h that is none";
  for (const float *p : {a->d_lam, a->d_gamma_u, a->d_beta_u, a->d_gamma_n, a->d_beta_n})
    if (!aligned(p, 4)) return "alignment of a parameter's gradient";
  return work(a->work, a->work_bytes, need) ? nullptr : "workspace missing, too small or not aligned to 16 bytes";
}

}  // namespace fade_op
