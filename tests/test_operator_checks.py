"""What the operators' entry points refuse, and the rules that cut their work, compiled for the host: no device is needed. A call that
one of these checks refuses enqueues nothing."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(text, tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(text)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2604_07239_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


CHECKS = """
#include <stdio.h>
#include <string.h>
#include <functional>
#include "fade_op_checks.h"
static int wrong = 0;
#define OK(x) do { const char *w = (x); if (w) { printf("line %d refused: %s\\n", __LINE__, w); ++wrong; } } while (0)
#define NO(x) do { if (!(x)) { printf("line %d not refused\\n", __LINE__); ++wrong; } } while (0)
using namespace fade_op;
int main() {
  alignas(64) static char mem[4096];
  char *p = mem;
  const float *f = (const float *)mem;
  // embedding: tokens, table, out
  OK(embed(p, FADE_TOKEN_U8, 5, p, FADE_BF16, 8, 10, 8, p, FADE_F32, 8));
  OK(embed(p + 1, FADE_TOKEN_U8, 5, p + 2, FADE_BF16, 9, 10, 8, p + 4, FADE_F32, 8));
  OK(embed(NULL, FADE_TOKEN_I64, 0, NULL, FADE_BF16, 8, 10, 8, NULL, FADE_F32, 8));
  NO(embed(NULL, FADE_TOKEN_U8, 5, p, FADE_BF16, 8, 10, 8, p, FADE_F32, 8));
  NO(embed(p, FADE_TOKEN_U8, 5, NULL, FADE_BF16, 8, 10, 8, p, FADE_F32, 8));
  NO(embed(p, FADE_TOKEN_U8, 5, p, FADE_BF16, 8, 10, 8, NULL, FADE_F32, 8));
  NO(embed(p, 3, 5, p, FADE_BF16, 8, 10, 8, p, FADE_F32, 8));
  NO(embed(p, -1, 5, p, FADE_BF16, 8, 10, 8, p, FADE_F32, 8));
  NO(embed(p, FADE_TOKEN_U8, 5, p, 2, 8, 10, 8, p, FADE_F32, 8));
  NO(embed(p, FADE_TOKEN_U8, 5, p, FADE_BF16, 8, 10, 8, p, 7, 8));
  NO(embed(p, FADE_TOKEN_U8, 5, p, FADE_BF16, 7, 10, 8, p, FADE_F32, 8));
  NO(embed(p, FADE_TOKEN_U8, 5, p, FADE_BF16, 8, 10, 8, p, FADE_F32, 7));
  NO(embed(p, FADE_TOKEN_U8, 5, p, FADE_BF16, 8, 10, 8, p + 2, FADE_F32, 8));
  NO(embed(p, FADE_TOKEN_U8, 5, p + 1, FADE_BF16, 8, 10, 8, p, FADE_F32, 8));
  NO(embed(p + 2, FADE_TOKEN_I32, 5, p, FADE_BF16, 8, 10, 8, p, FADE_F32, 8));
  NO(embed(p + 4, FADE_TOKEN_I64, 5, p, FADE_BF16, 8, 10, 8, p, FADE_F32, 8));
  NO(embed(p, FADE_TOKEN_U8, (size_t)1 << 31, p, FADE_BF16, 8, 10, 8, p, FADE_F32, 8));
  NO(embed(p, FADE_TOKEN_U8, 5, p, FADE_BF16, 8, 0, 8, p, FADE_F32, 8));
  NO(embed(p, FADE_TOKEN_U8, 5, p, FADE_BF16, 8, ((size_t)1 << 20) + 1, 8, p, FADE_F32, 8));
  NO(embed(p, FADE_TOKEN_U8, 5, p, FADE_BF16, 8, 10, 0, p, FADE_F32, 8));
  NO(embed(p, FADE_TOKEN_U8, 5, p, FADE_BF16, (size_t)1 << 62, 10, 8, p, FADE_F32, 8));
  // its gradient
  OK(embed_grad(p, FADE_TOKEN_I32, 5, p, FADE_BF16, 8, f, 8, 10, 8, p, 100, 100));
  OK(embed_grad(NULL, FADE_TOKEN_I32, 0, NULL, FADE_BF16, 8, f, 8, 10, 8, p, 100, 100));
  NO(embed_grad(p, FADE_TOKEN_I32, 5, p, FADE_BF16, 8, NULL, 8, 10, 8, p, 100, 100));
  NO(embed_grad(p, FADE_TOKEN_I32, 5, NULL, FADE_BF16, 8, f, 8, 10, 8, p, 100, 100));
  NO(embed_grad(p, FADE_TOKEN_I32, 5, p, FADE_BF16, 8, f, 7, 10, 8, p, 100, 100));
  NO(embed_grad(p, FADE_TOKEN_I32, 5, p, FADE_BF16, 8, f, 8, 10, 8, p, 99, 100));
  NO(embed_grad(p, FADE_TOKEN_I32, 5, p, FADE_BF16, 8, f, 8, 10, 8, NULL, 100, 100));
  NO(embed_grad(p, FADE_TOKEN_I32, 5, p, FADE_BF16, 8, f, 8, 10, 8, p + 8, 100, 100));
  NO(embed_grad(p, FADE_TOKEN_I32, 5, p, FADE_BF16, 8, f, 8, 10, 8, p, 100, 0));
  // checkpoints
  OK(checkpoint(p + 2, FADE_BF16, 33, 4, 33, p + 16));
  OK(checkpoint(NULL, FADE_BF16, 33, 0, 33, NULL));
  NO(checkpoint(p, FADE_BF16, 33, 4, 33, p + 8));
  NO(checkpoint(p, FADE_BF16, 32, 4, 33, p));
  NO(checkpoint(p, FADE_BF16, 33, 4, 33, NULL));
  NO(checkpoint(p, 2, 33, 4, 33, p));
  NO(checkpoint(p, FADE_BF16, 33, 4, 0, p));
  OK(weight_grad(p, 4, 33, p, FADE_F32, 5, 5, f, 5, p, 16, 16));
  OK(weight_grad(NULL, 0, 33, NULL, FADE_F32, 5, 5, f, 5, p, 16, 16));
  NO(weight_grad(NULL, 4, 33, p, FADE_F32, 5, 5, f, 5, p, 16, 16));
  NO(weight_grad(p, 4, 33, p, FADE_F32, 4, 5, f, 5, p, 16, 16));
  NO(weight_grad(p, 4, 33, p, FADE_F32, 5, 5, f, 4, p, 16, 16));
  NO(weight_grad(p, 4, 33, p, FADE_F32, 5, 5, NULL, 5, p, 16, 16));
  NO(weight_grad(p, 4, 33, p, FADE_F32, 5, 5, f, 5, p, 15, 16));
  NO(weight_grad(p, 4, 65537, p, FADE_F32, 5, 5, f, 5, p, 16, 16));
  NO(weight_grad(p, 4, 33, p, 9, 5, 5, f, 5, p, 16, 16));
  // join
  fade_join_args a;
  memset(&a, 0, sizeof a);
  a.struct_size = sizeof a;
  a.rows = 3; a.width = 40; a.stream_type = FADE_F32; a.branch_type = FADE_BF16; a.norm_u = FADE_NORM_LAYER; a.norm_n = FADE_NORM_RMS;
  a.r = p; a.u = p; a.g = p; a.r_ld = a.u_ld = a.g_ld = a.h_ld = a.n_ld = a.dh_ld = a.dn_ld = a.dr_ld = a.du_ld = a.dg_ld = 40;
  a.h = p + 512; a.n = p + 1024; a.lam = f; a.lam_count = 40; a.gamma_u = a.beta_u = a.gamma_n = a.beta_n = f;
  const fade_join_args good = a;
  auto with = [&](std::function<void(fade_join_args &)> change, bool grad = false) {
    a = good;
    if (grad) { a.dh = p; a.dn = p; a.work = p; a.work_bytes = 64; }
    change(a);
    return grad ? join_grad(&a, 64) : join(&a);
  };
  typedef fade_join_args &A;
  OK(with([](A) {}));
  OK(with([](A a) { a.g = NULL; a.n = NULL; a.lam = NULL; a.lam_count = 0; a.beta_u = NULL; }));
  OK(with([](A a) { a.rows = 0; a.r = a.u = a.h = NULL; }));
  OK(with([&](A a) { a.h = p; }));
  NO(join(NULL));
  NO(with([](A a) { a.struct_size--; }));
  NO(with([](A a) { a.width = 0; }));
  NO(with([](A a) { a.width = 8193; }));
  NO(with([](A a) { a.rows = (size_t)1 << 31; }));
  NO(with([](A a) { a.norm_u = 3; }));
  NO(with([](A a) { a.norm_n = 3; }));
  NO(with([](A a) { a.norm_u = FADE_NORM_NONE; }));
  NO(with([](A a) { a.norm_n = FADE_NORM_NONE; }));
  NO(with([](A a) { a.stream_type = FADE_BF16; a.branch_type = FADE_F32; }));
  NO(with([](A a) { a.stream_type = 2; }));
  NO(with([](A a) { a.eps = -1; }));
  NO(with([](A a) { a.eps = NAN; }));
  NO(with([](A a) { a.eps = INFINITY; }));
  NO(with([](A a) { a.lam_count = 39; }));
  NO(with([](A a) { a.lam_count = 0; }));
  NO(with([](A a) { a.lam = NULL; }));
  NO(with([&](A a) { a.gamma_u = (const float *)(p + 2); }));
  NO(with([](A a) { a.r = NULL; }));
  NO(with([](A a) { a.u = NULL; }));
  NO(with([](A a) { a.h = NULL; }));
  NO(with([](A a) { a.r_ld = 39; }));
  NO(with([](A a) { a.u_ld = 39; }));
  NO(with([](A a) { a.g_ld = 39; }));
  NO(with([](A a) { a.h_ld = 39; }));
  NO(with([](A a) { a.n_ld = 39; }));
  NO(with([&](A a) { a.r = p + 2; }));
  NO(with([&](A a) { a.u = p + 1; }));
  NO(with([&](A a) { a.h = p; a.h_ld = 41; }));
  NO(with([&](A a) { a.keep_u = p + 8; }));
  NO(with([&](A a) { a.g = NULL; a.keep_g = p; }));
  OK(with([](A) {}, true));
  OK(with([](A a) { a.dn = NULL; }, true));
  OK(with([](A a) { a.dh = NULL; }, true));
  OK(with([&](A a) { a.r = a.u = a.g = NULL; a.keep_r = a.keep_u = p; }, true));
  OK(with([](A a) { a.rows = 0; a.r = a.u = a.g = NULL; a.dh = a.dn = NULL; }, true));
  NO(with([](A a) { a.dh = a.dn = NULL; }, true));
  NO(with([&](A a) { a.keep_u = p; }, true));
  NO(with([&](A a) { a.r = a.u = a.g = NULL; a.keep_u = p; }, true));
  NO(with([&](A a) { a.keep_r = p; }, true));
  NO(with([&](A a) { a.keep_g = p; }, true));
  NO(with([](A a) { a.dh_ld = 39; }, true));
  NO(with([](A a) { a.dn_ld = 39; }, true));
  NO(with([&](A a) { a.dr = p; a.dr_ld = 39; }, true));
  NO(with([&](A a) { a.du = p; a.du_ld = 39; }, true));
  NO(with([&](A a) { a.dg = p; a.dg_ld = 39; }, true));
  NO(with([&](A a) { a.dg = p; a.g = NULL; }, true));
  NO(with([&](A a) { a.dr = p; a.dr_ld = 41; }, true));  // dh, with another ld
  NO(with([&](A a) { a.du = p; a.du_ld = 41; }, true));
  NO(with([&](A a) { a.lam = NULL; a.lam_count = 0; a.d_lam = (float *)p; }, true));
  NO(with([&](A a) { a.norm_u = FADE_NORM_NONE; a.gamma_u = a.beta_u = NULL; a.d_gamma_u = (float *)p; }, true));
  NO(with([&](A a) { a.norm_n = FADE_NORM_NONE; a.gamma_n = a.beta_n = NULL; a.d_beta_n = (float *)p; }, true));
  NO(with([&](A a) { a.d_beta_u = (float *)(p + 2); }, true));
  NO(with([](A a) { a.work = NULL; }, true));
  NO(with([](A a) { a.work_bytes = 63; }, true));
  NO(with([&](A a) { a.work = p + 4; }, true));
  return wrong != 0;
}
"""


def test_what_the_calls_refuse(tmp_path):
    _run(CHECKS, tmp_path)


RULES = """
#include <stdio.h>
#include <initializer_list>
#include "fade_op_rules.h"
using namespace fade_op;
#define WANT(x) do { if (!(x)) { printf("line %d: %s\\n", __LINE__, #x); return 1; } } while (0)
int main() {
  for (size_t n : {(size_t)0, (size_t)1, (size_t)31, (size_t)32, (size_t)33, (size_t)1025, (size_t)131072, (size_t)131073, (size_t)5000001, (size_t)0x7fffffff})
    for (size_t vocab : {(size_t)1, (size_t)2, (size_t)256, (size_t)1024, (size_t)1025, (size_t)50021, (size_t)1 << 20})
      for (size_t width : {(size_t)1, (size_t)32, (size_t)33, (size_t)512, (size_t)513, (size_t)4096}) {
        const GradPlan p = grad_plan(n, vocab, width);
        // the digits cover every token, the tiles and pieces every position, the lanes every column, and no region of the workspace another
        WANT(p.passes * p.bits <= 20 && ((size_t)1 << (p.passes * p.bits)) >= vocab && (1 << p.bits) <= MAX_DIGITS);
        WANT((size_t)p.tiles * 256 * SORT_ITEMS >= n && p.tiles >= 1);
        WANT((size_t)p.pieces * p.piece >= n);
        WANT(((size_t)p.strips * 8 << p.shift) >= width && p.shift >= 2 && p.shift <= 6);
        size_t at = 0;
        for (int i = 0; i < p.passes; ++i) {
          WANT(p.keys[i] >= at && p.keys[i] % 16 == 0);
          WANT(p.pos[i] >= p.keys[i] + 4 * n && p.pos[i] % 16 == 0);
          at = p.pos[i] + 4 * n;
        }
        WANT(p.hist >= at && p.total >= p.hist + ((size_t)4 * p.tiles << p.bits));
        WANT(p.flags >= p.total + 4 * (MAX_DIGITS + 1) && p.flags % 16 == 0);
        WANT(p.ends >= p.flags + (vocab + 15) / 16 * 16 && p.part >= p.ends + 4 * vocab && p.part % 16 == 0);
        WANT(p.piece >= 1 && p.piece <= 60 && p.share >= 1 && p.share <= 16);
        WANT(p.clear_rows >= (64u >> p.shift) && p.clear_rows <= 64 && 64 % p.clear_rows == 0);
        WANT(p.range == 0 || (n <= 16384 && p.range <= RANGE_TOKENS && (1u << p.range_bits) >= p.range));
        WANT(p.bytes >= p.part + (size_t)2 * p.pieces * 4 * ((width + 7) / 8 * 8));
      }
  for (int groups : {1, 2, 64}) WANT(row_blocks(1, groups) == 1 && (size_t)row_blocks(0x7fffffff, groups) * 256 < (size_t)1 << 32 && row_blocks(1000, groups) == (uint32_t)((1000 + groups - 1) / groups));
  for (size_t rows : {(size_t)0, (size_t)1, (size_t)64, (size_t)65, (size_t)1500, (size_t)16384, (size_t)100001, (size_t)0x7fffffff})
    for (size_t K : {(size_t)1, (size_t)128, (size_t)129, (size_t)4096, (size_t)65536})
      for (size_t N : {(size_t)1, (size_t)1000, (size_t)2048, (size_t)65536})
        for (bool f32 : {false, true}) {
          const WgradPlan p = wgrad_plan(rows, K, N, f32);
          WANT((size_t)p.units * 64 >= rows && p.ranges >= 1 && p.ranges <= 1024);
          WANT((long long)p.ranges * p.per >= p.units);
          WANT(p.units == 0 || (long long)(p.ranges - 1) * p.per < p.units);  // no range is empty
        }
  for (size_t width = 1; width <= 8192; width += width < 300 ? 1 : 97) {
    const JoinShape s = join_shape(width);
    WANT((size_t)s.lanes * 8 >= width && s.lanes >= 16 && s.lanes <= 1024 && s.groups >= 1);
    for (size_t rows : {(size_t)0, (size_t)1, (size_t)100, (size_t)0x7fffffff}) {
      const int b = grad_blocks(rows, width);
      WANT(b >= 0 && b <= 1024 && (rows == 0 || b >= 1) && (size_t)b * s.groups < rows + s.groups);
    }
  }
  return 0;
}
"""


def test_rules_cover_the_work_and_stay_inside_the_workspace(tmp_path):
    _run(RULES, tmp_path)


def test_arguments_and_sizes_as_the_library_sees_them():
    import paper_2604_07239_amd as fa
    L = fa.lib()
    assert C.sizeof(fa.JoinArgs) == 336
    assert L.fade_checkpoint_nbytes(3, 33) == 3 * 2 * 33
    assert L.fade_checkpoint_nbytes(0, 33) == 0 and L.fade_checkpoint_nbytes(3, 0) == 0 and L.fade_checkpoint_nbytes(3, (1 << 20) + 1) == 0
    assert L.fade_embed_grad_work(1 << 31, 10, 8) == 0 and L.fade_embed_grad_work(5, 0, 8) == 0 and L.fade_embed_grad_work(0, 10, 8) > 0
    assert L.fade_join_grad_work(5, 8193) == 0 and L.fade_join_grad_work(0, 8) > 0
    assert L.fade_checkpoint_weight_grad_work(5, 65537, 8) == 0 and L.fade_checkpoint_weight_grad_work(0, 8, 8) >= 16
    # without a context nothing else is looked at
    assert L.fade_embed(None, None, 0, 0, None, 0, 0, 0, 0, 1.0, None, 0, 0) == -1
    assert L.fade_embed_grad(None, None, 0, 0, None, 0, 0, 1.0, None, 0, 0, 0, 0, None, 0) == -1
    assert L.fade_checkpoint(None, None, 0, 0, 0, 0, None) == -1 and L.fade_checkpoint_read(None, None, 0, 0, None, 0, 0) == -1
    assert L.fade_checkpoint_weight_grad(None, None, 0, 0, None, 0, 0, 0, None, 0, 0, None, 0) == -1
    assert L.fade_join(None, None) == -1 and L.fade_join_grad(None, None) == -1


class _Ctx:
    """The binding's own checks, without a device: a context that no call may reach."""

    def __new__(cls):
        import paper_2604_07239_amd as fa
        g = fa.Fade.__new__(fa.Fade)
        g.cfg, g.L, g.h, g.device = fa.make_config(16, 32, 16, 128), fa.lib(), None, 0
        return g


@pytest.mark.parametrize("call", ["embed", "embed_grad", "checkpoint", "checkpoint_read", "checkpoint_weight_grad", "join", "join_grad"])
def test_the_binding_refuses_tensors_that_are_not_on_the_device(call):
    import torch

    import paper_2604_07239_amd as fa
    x, t, b = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32), torch.zeros(4096, dtype=torch.uint8)
    args = {"embed": (t, x, x), "embed_grad": (t, x, x, b), "checkpoint": (x, b), "checkpoint_read": (b, x), "checkpoint_weight_grad": (b, x, x, b),
            "join": (x, x), "join_grad": (x, x, b)}[call]
    with pytest.raises(fa.FadeError) as e:
        getattr(_Ctx(), call)(*args, **({"r": x, "u": x} if call.startswith("join") else {}))
    assert e.value.code == -1


EPS = """
#include <stdio.h>
#include <string.h>
#include "fade_op_checks.h"
int main() {
  alignas(64) static char mem[64];
  fade_join_args a;
  memset(&a, 0, sizeof a);
  a.struct_size = sizeof a;
  a.rows = 1; a.width = 8; a.r = a.u = mem; a.h = mem + 32; a.r_ld = a.u_ld = a.h_ld = 8;
  for (const float eps : {0.0f, 1e-5f, FLT_MIN}) {
    a.eps = eps;
    if (const char *why = fade_op::join(&a)) return printf("%g refused: %s\\n", eps, why), 1;
  }
  for (const float eps : {FLT_MIN / 2, 1e-45f}) {
    a.eps = eps;
    if (!fade_op::join(&a)) return printf("%g not refused\\n", eps), 1;
  }
  return 0;
}
"""


def test_an_eps_that_the_reciprocal_root_takes_for_zero_is_refused(tmp_path):
    """1 / sqrt of a subnormal number is infinite on the device: a row of equal values would become NaN instead of zeros."""
    _run(EPS, tmp_path)


@pytest.mark.parametrize("shape", [(4,), (2, 3, 8)])
def test_gradients_that_are_no_matrix_are_refused(shape):
    torch = pytest.importorskip("torch")
    import paper_2604_07239_amd as fa
    ctx = object.__new__(fa.Fade)
    ctx.h, ctx.device = None, 0
    for dh, dn in ((torch.zeros(shape), None), (None, torch.zeros(shape))):
        with pytest.raises(fa.FadeError):
            ctx.join_grad(dh, dn, None)
