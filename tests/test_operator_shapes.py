"""The sizes that the GPU tests of several turns and of large tiles run are what they are meant to be, and the bars of the join's gradients let no
wrong one through. No device is needed."""
import os
import subprocess

import numpy as np
import pytest
import torch

from join_reference import MODELS, STEPS, TYPES, backward, forward, model, rows_wrong, sums_wrong
from operator_shapes import JOIN_TURNS, WEIGHT_GRADS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PLANS = """
#include <stdio.h>
#include <stdlib.h>
#include "fade_op_rules.h"
using namespace fade_op;
int main(int argc, char **argv) {
  for (int i = 1; i + 3 < argc; i += 4) {
    const size_t rows = atoll(argv[i]), a = atoll(argv[i + 1]), b = atoll(argv[i + 2]);
    if (argv[i + 3][0] == 'j') {
      const JoinShape s = join_shape(a);
      printf("%d %d %d %d\\n", s.lanes, s.groups, turn_blocks(rows, s.groups, 2048), grad_blocks(rows, a));
    } else {
      const WgradPlan p = wgrad_plan(rows, a, b, argv[i + 3][0] == 'f');
      printf("%d %d %d\\n", p.large, p.ranges, p.per);
    }
  }
}
"""


def _plans(tmp_path, what):
    src, exe = tmp_path / "p.cpp", tmp_path / "p"
    src.write_text(PLANS)
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2604_07239_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe), *(str(x) for w in what for x in w)], capture_output=True, text=True, check=True).stdout
    return [tuple(int(x) for x in line.split()) for line in out.splitlines()]


def test_joins_of_several_turns(tmp_path):
    seen = set()
    for (rows, C, _), (lanes, groups, there, back) in zip(JOIN_TURNS, _plans(tmp_path, [(r, C, 0, "j") for r, C, _ in JOIN_TURNS])):
        assert rows > there * groups and rows > 2 * back * groups  # two turns forward, three backward
        assert rows % (there * groups) and rows % (back * groups)  # the last one of some workgroups only
        seen |= {lanes, (lanes >= 512, C % 8 == 0)}
    assert seen >= {16, 32, 64, 128, 256, 512, 1024, (False, False), (False, True), (True, False), (True, True)}


def test_weight_gradients_of_large_tiles(tmp_path):
    plans = _plans(tmp_path, [(r, K, N, "f" if t == "float32" else "b") for r, K, N, t, *_ in WEIGHT_GRADS])
    seen = set()
    for (rows, K, N, t, accumulate, pad, _, large, ranges, add), (l, r, _) in zip(WEIGHT_GRADS, plans):
        assert (bool(l), r) == (large, ranges) and add == (0 if r == 1 else 4 if K * N >= 1 << 22 else 1)
        seen |= {(large, t, r > 1), (t, add), (large, accumulate), (add, pad > 0)}
        assert rows % 64
    assert seen >= {(True, t, r) for t in ("float32", "bfloat16") for r in (False, True)} | {(t, a) for t in ("float32", "bfloat16") for a in (0, 1, 4)}
    assert seen >= {(True, True), (True, False), (4, True), (4, False), (1, True), (1, False)}


def test_the_plans_whose_times_the_rules_quote(tmp_path):
    """Rows, in, out, type of dy: large tiles, ranges. A change of the rule that moves one of these asks for new figures beside it."""
    quoted = {(16384, 4096, 2048, "b"): (1, 2), (4096, 1024, 1024, "b"): (0, 4), (512, 512, 512, "b"): (0, 1), (16384, 2048, 2048, "f"): (1, 4), (1500, 512, 1000, "f"): (0, 8)}
    assert [(large, ranges) for large, ranges, _ in _plans(tmp_path, quoted)] == list(quoted.values())


@pytest.mark.parametrize("i", range(len(MODELS)))
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("rows,C", [(700, 60), (61, 777), (2500, 24)])
def test_the_bars_let_no_wrong_gradient_through(i, types, rows, C):
    """Zeros, the other sign, 1 % too much, a row that is lost: planted in the 64-bit values."""
    norm_u, norm_n, gate, lam = MODELS[i]
    rng = np.random.default_rng(i)
    p = model(rng, C, gate, lam, norm_u, norm_n, lambda x: torch.from_numpy(x))
    r, u, g, dh, dn = (torch.from_numpy(rng.standard_normal((rows, C))) for _ in range(5))
    g = g if gate else None
    f = forward(r, u, g, p, norm_u, norm_n)
    values, params = backward(r, u, g, p, norm_u, norm_n, 0.1 * dh, 0.1 * dn)
    values = {"h": (f["h"], f["m_h"]), "n": (f["n"], f["m_n"]), **values}
    types = dict(zip(("stream", "branch"), TYPES[types]))
    for k, (want, made) in values.items():
        t = types["stream" if k in ("h", "dr") else "branch"]
        bf16 = t == torch.bfloat16
        assert rows_wrong(want.to(t).double(), want, made, STEPS[k], bf16) == 0, k  # rounded as a kernel's are
        for wrong in (torch.zeros_like(want), -want, 1.01 * want, want.roll(1, 0)):
            assert rows_wrong(wrong.to(t).double(), want, made, STEPS[k], bf16) == rows, k
        one = want.clone()
        one[rows // 2] *= 0.99
        assert rows_wrong(one.to(t).double(), want, made, STEPS[k], bf16) == 1, k
        one[rows // 2] = float("nan")
        assert rows_wrong(one, want, made, STEPS[k], bf16) == 1, k
    for k, (terms, made) in params.items():
        want = terms.sum().reshape(1) if k == "d_lam" and lam == "scalar" else terms.sum(0)
        lost = terms[rows // 2].sum().reshape(1) if want.numel() == 1 else terms[rows // 2]
        for start in (0.0, 0.25):
            assert sums_wrong((want + start).float().double(), terms, made, start) is None, k
            for wrong in (torch.zeros_like(want), -want, 0.99 * want, 1.01 * want, want - lost, want + lost, want * float("nan")):
                assert sums_wrong((wrong + start).float().double(), terms, made, start), k
