"""The weight gradient from checkpoints on each of its tiles, and the launches that add ranges, against 64-bit products on the device."""
import pytest

from gpu_helpers import need_gpu
from operator_helpers import U, context
from operator_shapes import WEIGHT_GRADS

pytestmark = pytest.mark.gpu


def _place(torch, x, pad, shift):
    """x with `pad` elements behind each row and `shift` in front of the first; they hold NaN, which may reach nothing."""
    rows, width = x.shape
    flat = torch.full((rows * (width + pad) + shift + 8,), float("nan"), dtype=x.dtype, device="cuda")
    view = flat[shift:shift + rows * (width + pad)].view(rows, width + pad)[:, :width]
    view.copy_(x)
    return view, flat


def _keep(torch, c, x):
    """x's checkpoint, and the values it stands for (to the bit, as tested where it is written)"""
    keep, values = torch.empty(c.checkpoint_nbytes(*x.shape), dtype=torch.uint8, device="cuda"), torch.empty_like(x)
    torch.cuda.synchronize()
    c.checkpoint(x, keep)
    c.checkpoint_read(keep, values)
    torch.cuda.synchronize()
    return keep, values


def _run(torch, c, keep, dy, grad, accumulate=False):
    work = torch.full((c.checkpoint_weight_grad_work(dy.shape[0], *grad.shape),), 0xFF, dtype=torch.uint8, device="cuda")  # NaNs
    torch.cuda.synchronize()
    c.checkpoint_weight_grad(keep, dy, grad, work, accumulate=accumulate)
    torch.cuda.synchronize()


@pytest.mark.parametrize("rows,K,N,dtype,accumulate,pad,shift,large,ranges,add", WEIGHT_GRADS)
def test_against_the_product(rows, K, N, dtype, accumulate, pad, shift, large, ranges, add):
    torch = need_gpu()
    gen = torch.Generator(device="cuda").manual_seed(rows + K)
    mk = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    c = context()
    keep, x = _keep(torch, c, mk(rows, K) * torch.exp(mk(1, K)))
    dy, _ = _place(torch, (mk(rows, N) * torch.exp(mk(rows, 1))).to(getattr(torch, dtype)), pad, shift)
    before = mk(K, N)
    grad, flat = _place(torch, before, pad, shift)
    _run(torch, c, keep, dy, grad, accumulate)
    got = grad.double()
    x, d = x.double().t().contiguous(), dy.double()
    want, size, square = x @ d, x.abs() @ d.abs(), (x * x) @ (d * d)
    start = before.double() if accumulate else torch.zeros_like(want)
    # exact products, three for an fp32 dy; each addition of a range's chain (at most its rows' terms) and of the ranges rounds, on the matrix cores
    # perhaps by cutting: a whole step, 2 u; the last one, with what was there, half a step
    chain = (3 if dtype == "float32" else 1) * min(rows, (rows + 63) // 64 // ranges * 64 + 64) + ranges
    err = (got - want - start).abs()
    assert bool((err <= chain * 2 * U * size + 2 * U * start.abs()).all())
    # and as roundings of any sign add up: their root, with a margin of four
    assert float(err.norm() / ((square.sqrt() + start.abs()).norm())) <= 4 * 2 * U * chain ** 0.5
    # a row, a column, a tile's edge for themselves
    for at in ((0, slice(None)), (K - 1, slice(None)), (slice(None), 0), (slice(None), N - 1)):
        assert float(err[at].norm() / (square.sqrt() + start.abs())[at].norm()) <= 4 * 2 * U * chain ** 0.5, at
    grad.fill_(float("nan"))
    assert bool(flat.isnan().all())  # nothing between the rows was written
    c.close()


@pytest.mark.parametrize("rows,K,N", [(1, 1, 1), (70, 40, 50), (1500, 512, 1000), (517, 4090, 4090), (3001, 2050, 2056), (16300, 1020, 1015)])
def test_an_fp32_dy_keeps_all_of_its_bits(rows, K, N):
    """One row of x is not zero, and holds powers of two: the gradient is that row times dy's, to the bit."""
    torch = need_gpu()
    gen = torch.Generator(device="cuda").manual_seed(K)
    at = rows * 2 // 3
    x = torch.zeros((rows, K), device="cuda")
    x[at] = torch.exp2(torch.randint(-1, 3, (K,), device="cuda", generator=gen).float()) * (torch.randint(0, 2, (K,), device="cuda", generator=gen) * 2 - 1)
    dy = torch.randn((rows, N), device="cuda", generator=gen) * torch.exp(4 * torch.randn((rows, N), device="cuda", generator=gen))
    # a whole significand: the lowest bit set, as three terms in 8 bits each have to show
    dy = (dy.view(torch.int32) | 1).view(torch.float32)
    c = context()
    keep, values = _keep(torch, c, x)
    assert torch.equal(values, x)
    grad = torch.full((K, N), 7.0, device="cuda")
    _run(torch, c, keep, dy, grad)
    assert torch.equal(grad, x[at][:, None] * dy[at][None, :])
    c.close()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,K,N", [(517, 4090, 4090), (3001, 2050, 2056)])
def test_values_that_are_not_finite_on_large_tiles(rows, K, N, dtype):
    torch = need_gpu()
    gen = torch.Generator(device="cuda").manual_seed(7)
    x, dy = (torch.randn((rows, k), device="cuda", generator=gen) for k in (K, N))
    x[3], x[4] = 0.0, 2.0
    x[rows - 1, 5] = float("inf")  # a group of 32 columns that reads back as NaN
    dy[4, 7], dy[5, N - 1], dy[3, 13], dy[4, 300] = float("inf"), float("nan"), float("inf"), 3.3e38
    dy[rows - 1, 17] = 0.0
    c = context()
    keep, _ = _keep(torch, c, x)
    grad = torch.zeros((K, N), device="cuda")
    _run(torch, c, keep, dy.to(getattr(torch, dtype)), grad)
    nan = torch.zeros((K, N), dtype=torch.bool, device="cuda")
    nan[:32] = True
    nan[:, 13] = nan[:, N - 1] = True  # infinity times zero; NaN
    assert torch.equal(grad.isnan(), nan)
    inf = torch.zeros_like(nan)
    inf[32:, 7] = inf[32:, 300] = True  # the latter's products of 6.6e38 are past the type
    assert torch.equal(grad.isinf(), inf)
    c.close()
