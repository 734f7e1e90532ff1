"""Values and sizes at the ends of what the operators are given."""
import numpy as np
import pytest

from gpu_helpers import need_gpu
from join_reference import STEPS, backward, forward, rows_wrong, sums_wrong
from operator_helpers import U, context, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_the_largest_values_come_back_finite(dtype):
    """Above 127 * 2^121 the exponent stays at 121 and the byte at 127: with 122 the largest values would round to 64 * 2^122, which is infinite in fp32. They
    are off by at most 2^121 this way, half a step of 2^122."""
    torch = need_gpu()
    T = getattr(torch, dtype)
    most, limit = torch.finfo(T).max, 127 * 2.0 ** 121
    tops = [most, -most, limit, -limit, limit * (1 + torch.finfo(T).eps), 3.3e38, 63.5 * 2.0 ** 122, 2.0 ** 127]
    x = torch.randn((len(tops), 70), device="cuda") * 2.0 ** 125
    for i, v in enumerate(tops):
        x[i, ::5] = v
    x[0] = -most  # a mask's row
    x = x.to(T)
    g = context()
    keep, y = torch.empty(g.checkpoint_nbytes(len(tops), 70), dtype=torch.uint8, device="cuda"), torch.empty_like(x)
    torch.cuda.synchronize()
    g.checkpoint(x, keep)
    g.checkpoint_read(keep, y)
    torch.cuda.synchronize()
    v = np.zeros((len(tops), 96))
    v[:, :70] = f64(x)
    v = v.reshape(len(tops), 3, 32)
    finite = np.isfinite(v).all(2)  # in bf16 the fifth of them, 127 * 129 / 128 * 2^121 = 127.99 * 2^121, is nearer to 2^128 than to 127.5 * 2^121: infinite
    assert finite.all() or (dtype == "bfloat16" and (finite == (np.arange(len(tops)) != 4)[:, None]).all())
    v = np.where(finite[:, :, None], v, 0.0)
    with np.errstate(divide="ignore"):
        e = np.clip(np.ceil(np.log2(np.abs(v).max(2) / 127)), -126, 121)
    q = np.clip(np.rint(v / np.exp2(e)[:, :, None]), -127, 127)
    e[~finite] = 128
    host = keep.cpu().numpy()
    np.testing.assert_array_equal(host[:q.size].view(np.int8), q.reshape(-1))
    np.testing.assert_array_equal(host[q.size:], e.reshape(-1).astype(int) + 127)
    want = np.where(finite[:, :, None], q * np.exp2(e)[:, :, None], np.nan).reshape(len(tops), -1)[:, :70]
    np.testing.assert_array_equal(f64(y), want)
    whole = finite.all(1)
    assert np.isfinite(f64(y)[whole]).all() and (np.abs(want - f64(x)) <= 2.0 ** 121)[whole].all()
    # and so do the join's checkpoints of the same values, and products with them
    other = torch.empty_like(keep)
    torch.cuda.synchronize()
    g.join(torch.empty_like(x), None, r=x, u=torch.zeros_like(x), norm_u="none", norm_n="none", keep_r=other)
    grad, work = torch.empty((70, 3), device="cuda"), torch.empty(g.checkpoint_weight_grad_work(len(tops), 70, 3), dtype=torch.uint8, device="cuda")
    dy = torch.full((len(tops), 3), 2.0 ** -9, device="cuda").to(T)
    torch.cuda.synchronize()
    g.checkpoint_weight_grad(keep, dy, grad, work)
    torch.cuda.synchronize()
    assert torch.equal(other, keep)
    bound = 32 * U * np.abs(want).sum(0)[:, None] * 2.0 ** -9  # eight exact products, three terms of a dy each
    total = want.sum(0)[:, None] * 2.0 ** -9
    assert ((np.abs(f64(grad) - total) <= bound) | (np.isnan(total) & np.isnan(f64(grad)))).all()
    g.close()


def _level(torch, rows, C, at, seed, of, level, gamma):
    """Operands of which row `at` of u or of r (and so of h) is `level` throughout, whose distance from its mean is zero, and the same with zeros there, for a norm that
    takes the mean away the same operands; eps is so small that level / sigma is near the end of fp32 or past it."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r, u, g, dh, dn = (torch.randn((rows, C), device="cuda", generator=gen) for _ in range(5))
    p = {k: 1.0 + 0.1 * torch.randn(C, device="cuda", generator=gen) for k in ("gamma_u", "beta_u", "gamma_n", "beta_n")}
    p["lam"] = torch.full((1,), 2.0, device="cuda")
    if of == "u":
        u[at] = level
        p["gamma_u"] *= gamma
        plain = (r, u.clone())
        plain[1][at] = 0.0
    else:
        g = None
        p = {k: p[k] for k in ("gamma_n", "beta_n", "lam")}
        r[at], u[at] = level, 0.0
        dn, dh = 1e-7 * dn, 0.1 * dh
        plain = (r.clone(), u)
        plain[0][at] = 0.0
    return r, u, g, p, dh, dn, plain


def _check_level(rows, C, at, of, level=2.0 ** 114, gamma=1.0):
    torch = need_gpu()
    eps, c = 1e-12, context()
    r, u, g, p, dh, dn, plain = _level(torch, rows, C, at, C, of, level, gamma)
    norm_u = "layer" if of == "u" else "none"
    h, n = torch.empty_like(r), torch.empty_like(r)
    keep = [torch.empty(c.checkpoint_nbytes(rows, C), dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    c.join(h, n, r=r, u=u, g=g, norm_u=norm_u, norm_n="layer", eps=eps, keep_n=keep[0], **p)
    c.checkpoint(n, keep[1])
    torch.cuda.synchronize()
    p64, g64 = {k: v.double() for k, v in p.items()}, None if g is None else g.double()
    f = forward(plain[0].double(), plain[1].double(), g64, p64, norm_u, "layer", eps)
    assert rows_wrong(n.double(), f["n"], f["m_n"], STEPS["n"], False) == 0
    if of == "u":
        assert rows_wrong(h.double(), f["h"], f["m_h"], STEPS["h"], False) == 0
    assert torch.equal(*keep)
    out = {k: torch.empty_like(r) for k in ("dr", "du") + (("dg",) if of == "u" else ())}
    out.update({"d_" + k: torch.empty_like(v) for k, v in p.items()})
    work = torch.empty(c.join_grad_work(rows, C), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    c.join_grad(dh, dn, work, r=r, u=u, g=g, norm_u=norm_u, norm_n="layer", eps=eps, **p, **out)
    torch.cuda.synchronize()
    values, params = backward(plain[0].double(), plain[1].double(), g64, p64, norm_u, "layer", dh.double(), dn.double(), eps)
    if of == "r":  # the only one in which the row's level is
        t, m = (x / 2.0 for x in values["dr"])
        params["d_lam"] = (t * r.double(), m * r.double().abs())
    for k, (want, made) in values.items():
        assert rows_wrong(out[k].double(), want, made, STEPS[k], False) == 0, k
    for k, (terms, made) in params.items():
        assert sums_wrong(out[k].double(), terms, made) is None, k
    c.close()


@pytest.mark.parametrize("of", ["u", "r"])
@pytest.mark.parametrize("rows,C,at", [(64, 31, 5), (64, 40, 5), (16, 777, 5), (2, 8000, 1)])
def test_a_level_row_far_from_zero(rows, C, at, of):
    """Its normalised values are zeros; those of columns that do not exist, behind the width up to the lanes of a row, may be nothing else."""
    _check_level(rows, C, at, of)


@pytest.mark.parametrize("of", ["u", "r"])
@pytest.mark.parametrize("rows,C,at", [(3, 1500, 1), (2, 3000, 1), (2, 7000, 0)])
def test_a_level_row_where_wavefronts_of_the_row_have_no_columns(rows, C, at, of):
    """A wavefront without columns has nothing to add to the row's variance, however far its mean of nothing is from the row's."""
    _check_level(rows, C, at, of)


@pytest.mark.parametrize("level,gamma", [(2.0 ** 114, 1.0), (2.0 ** 106, 16.0)])
@pytest.mark.parametrize("rows,C,at", [(3, 128, 2), (3, 512, 2), (18, 100, 17)])
def test_a_level_row_at_the_end_of_a_batch(rows, C, at, level, gamma):
    """The rows that a workgroup has beside the last one, and that do not exist, add nothing to the parameters' gradients: with the last row's statistics their zeros would be
    2^106 / sigma = 8e37 away from its mean, and gamma past fp32."""
    _check_level(rows, C, at, "u", level, gamma)


def test_a_batch_of_no_rows_leaves_sums_alone_to_the_bit():
    """Added to a negative zero, a sum of nothing would make it a positive one."""
    torch = need_gpu()
    c = context()
    none, gamma = torch.zeros((0, 40), device="cuda"), torch.ones(40, device="cuda")
    d, grad = torch.full((40,), -0.0, device="cuda"), torch.full((40, 9), -0.0, device="cuda")
    work = torch.empty(max(c.join_grad_work(0, 40), c.checkpoint_weight_grad_work(0, 40, 9)), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    c.join_grad(none, none, work, r=none, u=none, gamma_u=gamma, d_gamma_u=d, accumulate=True)
    c.checkpoint_weight_grad(torch.zeros(0, dtype=torch.uint8, device="cuda"), none[:, :9], grad, work, accumulate=True)
    torch.cuda.synchronize()
    assert bool(torch.signbit(d).all()) and bool(torch.signbit(grad).all())
    c.close()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,K,N,low", [(70, 40, 300, 18), (70, 40, 300, -1), (517, 4090, 4090, 18), (517, 4090, 4090, -1)])
def test_weight_gradient_of_the_smallest_values(rows, K, N, low, dtype):
    """The matrix cores take subnormal bf16 as it is, and give subnormal fp32. Of an fp32 dy they get three bf16 terms: all of it from 2^-110 on, whose last bit is bf16's smallest number, 2^-133,
    below that all but less than 2^-133."""
    torch = need_gpu()
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.zeros((rows, K), device="cuda")
    x[7] = torch.exp2(torch.randint(low, low + 4, (K,), device="cuda", generator=gen).float())
    e = torch.randint(-149, -100, (rows, N), device="cuda", generator=gen).double()
    dy = (torch.exp2(e) * (1 + torch.rand((rows, N), device="cuda", generator=gen).double())).float().to(getattr(torch, dtype))
    c = context()
    keep = torch.empty(c.checkpoint_nbytes(rows, K), dtype=torch.uint8, device="cuda")
    grad = torch.zeros((K, N), device="cuda")
    work = torch.zeros(c.checkpoint_weight_grad_work(rows, K, N), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    c.checkpoint(x, keep)
    c.checkpoint_weight_grad(keep, dy, grad, work)
    torch.cuda.synchronize()
    err = (grad.double() - x[7].double()[:, None] * dy[7].double()[None]).abs() / x[7].double()[:, None]
    if dtype == "bfloat16":
        assert bool((err == 0).all())
    else:
        assert bool((err[:, dy[7].double() >= 2.0 ** -110] == 0).all()) and bool((err < 2.0 ** -133).all())
    c.close()
