"""The join where a workgroup takes several turns of rows: the next rows' operands on their way, u's statistics passed on through the shared exchange, its two places in
turn, and parameter gradients summed over the turns; against 64-bit values, row by row and element by element."""
import numpy as np
import pytest

from gpu_helpers import need_gpu
from join_reference import MODELS, STEPS, TYPES, backward, forward, model, rows_wrong, sums_wrong
from operator_helpers import context
from operator_shapes import JOIN_TURNS

pytestmark = pytest.mark.gpu


def _operands(torch, rows, C, types, gate, seed):
    """r, u, g, dh and dn; magnitudes differ from row to row, so that no row passes for another."""
    st, br = TYPES[types]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    size = torch.exp(0.5 * torch.randn((rows, 1), device="cuda", generator=gen))
    mk = lambda t, a, b=0.0: ((torch.randn((rows, C), device="cuda", generator=gen) * a + b) * size).to(t)  # noqa: E731
    return mk(st, 2.0, 0.1), mk(br, 1.0, 0.3), mk(br, 1.0) if gate else None, mk(st, 0.1), mk(br, 0.1)


def _double(x):
    return None if x is None else x.double()


@pytest.mark.parametrize("shape", range(len(JOIN_TURNS)))
@pytest.mark.parametrize("second", [0, 3])
def test_forward(shape, second):
    torch = need_gpu()
    rows, C, types = JOIN_TURNS[shape]
    norm_u, norm_n, gate, lam = MODELS[(shape + second) % len(MODELS)]
    r, u, g, _, _ = _operands(torch, rows, C, types, gate, shape)
    p = model(np.random.default_rng(shape), C, gate, lam, norm_u, norm_n, lambda x: torch.from_numpy(x.astype(np.float32)).cuda())
    c = context()
    h, n = torch.full_like(r, 9.0), torch.full_like(u, 9.0)
    keep, back = [torch.empty(c.checkpoint_nbytes(rows, C), dtype=torch.uint8, device="cuda") for _ in range(8)], {}
    names = ["keep_r", "keep_u", "keep_n"] + (["keep_g"] if gate else [])
    torch.cuda.synchronize()
    c.join(h, n, r=r, u=u, g=g, norm_u=norm_u, norm_n=norm_n, **dict(zip(names, keep)), **p)
    torch.cuda.synchronize()
    f = forward(_double(r), _double(u), _double(g), {k: v.double() for k, v in p.items()}, norm_u, norm_n)
    for k, got in (("h", h), ("n", n)):
        assert rows_wrong(got.double(), f[k], f["m_" + k], STEPS[k], got.dtype == torch.bfloat16) == 0, k
    # the checkpoints are those of a pass of its own over the same values
    for name, k in zip(names, keep):
        c.checkpoint({"keep_r": r, "keep_u": u, "keep_g": g, "keep_n": n}[name], keep[4])
        torch.cuda.synchronize()
        assert torch.equal(k, keep[4]), name
    # a row is the same bits by itself, and over r
    one_h, one_n = torch.empty_like(h[:1]), torch.empty_like(n[:1])
    for i in (0, rows // 2, rows - 2, rows - 1):
        c.join(one_h, one_n, r=r[i:i + 1], u=u[i:i + 1], g=None if g is None else g[i:i + 1], norm_u=norm_u, norm_n=norm_n, **p)
        torch.cuda.synchronize()
        assert torch.equal(one_h[0], h[i]) and torch.equal(one_n[0], n[i]), i
    n2 = torch.full_like(u, 9.0)
    torch.cuda.synchronize()
    c.join(r, n2, r=r, u=u, g=g, norm_u=norm_u, norm_n=norm_n, **p)
    torch.cuda.synchronize()
    assert torch.equal(r, h) and torch.equal(n2, n)
    c.close()


@pytest.mark.parametrize("shape", range(len(JOIN_TURNS)))
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("second", [0, 3])
def test_backward(shape, kept, second):
    torch = need_gpu()
    rows, C, types = JOIN_TURNS[shape]
    norm_u, norm_n, gate, lam = MODELS[(shape + second) % len(MODELS)]
    r, u, g, dh, dn = _operands(torch, rows, C, types, gate, 100 + shape)
    p = model(np.random.default_rng(shape), C, gate, lam, norm_u, norm_n, lambda x: torch.from_numpy(x.astype(np.float32)).cuda())
    c = context()
    operands = {k: v for k, v in (("r", r), ("u", u), ("g", g)) if v is not None}
    if kept:  # what a checkpoint stands for is tested to the bit where it is written
        buf = {}
        for k, x in operands.items():
            buf["keep_" + k] = torch.empty(c.checkpoint_nbytes(rows, C), dtype=torch.uint8, device="cuda")
            torch.cuda.synchronize()
            c.checkpoint(x, buf["keep_" + k])
            c.checkpoint_read(buf["keep_" + k], x)
        operands = buf
    work = torch.full((c.join_grad_work(rows, C),), 0xFF, dtype=torch.uint8, device="cuda")  # NaNs
    accumulate = (shape + second) % 2 == 1

    def grads(dh, dn, dr, du):
        out = {"dr": dr, "du": du, **({"dg": torch.full_like(u, 5.0)} if gate else {})}
        out.update({"d_" + k: torch.full_like(v, 0.25) for k, v in p.items()})
        torch.cuda.synchronize()
        c.join_grad(dh, dn, work, norm_u=norm_u, norm_n=norm_n, accumulate=accumulate, **operands, **p, **out)
        torch.cuda.synchronize()
        return out

    out = grads(dh, dn, torch.full_like(r, 5.0), torch.full_like(u, 5.0))
    values, params = backward(_double(r), _double(u), _double(g), {k: v.double() for k, v in p.items()}, norm_u, norm_n, dh.double(), dn.double())
    for k, (want, made) in values.items():
        assert rows_wrong(out[k].double(), want, made, STEPS[k], out[k].dtype == torch.bfloat16) == 0, k
    for k, (terms, made) in params.items():
        assert sums_wrong(out[k].double(), terms, made, 0.25 if accumulate else 0.0) is None, k
    # the same bits again, and over dh and dn
    again = grads(dh, dn, dh, dn)
    assert all(torch.equal(out[k], again[k]) for k in out)
    c.close()
