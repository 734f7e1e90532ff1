"""8-bit activation checkpoints against their definition, to the bit, and the weight gradient from them."""
import numpy as np
import pytest

from gpu_helpers import need_gpu
from operator_helpers import U, context, f64, guards_untouched, keep64, place

pytestmark = pytest.mark.gpu


def _values(rng, rows, width):
    """Groups of very different size, among them zeros, values on a border of the exponent, ties, and the smallest and largest there are."""
    x = rng.standard_normal((rows, width)) * np.exp(4 * rng.standard_normal((rows, 1))) * np.exp(rng.standard_normal((1, width)))
    x = x.astype(np.float32)
    for i, v in enumerate([0.0, 127.0, 127.25, 126.5, 1.984375, 1.9843752, 2.0 ** -126, 2.0 ** -140, 3.3e38, -3.3e38, 0.5, -0.0]):
        if i < rows:
            x[i] = 0.0
            x[i, ::3] = v
            x[i, 1::7] = v / 254  # half a step, or near it
    return x


@pytest.mark.parametrize("rows,width,dtype,pad,shift", [(1, 1, "float32", 0, 0), (13, 31, "bfloat16", 1, 1), (40, 32, "float32", 0, 0), (17, 33, "bfloat16", 0, 0),
                                                        (100, 777, "float32", 3, 3), (33, 1024, "bfloat16", 8, 1), (3, 5000, "float32", 0, 0)])
def test_bytes_and_values_are_the_definitions(rows, width, dtype, pad, shift):
    torch = need_gpu()
    T = getattr(torch, dtype)
    x, _ = place(torch, _values(np.random.default_rng(rows), rows, width), T, pad, shift)
    g = context()
    n = g.checkpoint_nbytes(rows, width)
    buf = torch.full((n + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    g.checkpoint(x, buf[:n])
    torch.cuda.synchronize()
    q, e, values = keep64(f64(x))
    host = buf.cpu().numpy()
    np.testing.assert_array_equal(host[:q.size].view(np.int8).reshape(q.shape), q)
    np.testing.assert_array_equal(host[q.size:n].reshape(e.shape), e)
    assert (host[n:] == 0xA5).all()
    for O in (torch.float32, torch.bfloat16):
        y, flat = place(torch, np.zeros((rows, width)), O, pad, shift)
        g.checkpoint_read(buf[:n], y)
        torch.cuda.synchronize()
        np.testing.assert_array_equal(f64(y), values)  # 7 bits and a power of two: exact in either type
        assert guards_untouched(torch, flat, rows, width, pad, shift)
    g.close()


def test_a_value_is_off_by_half_a_step_of_its_group():
    x = np.random.default_rng(2).standard_normal((50, 320)).astype(np.float32)
    _, _, v = keep64(x.astype(np.float64))
    top = np.abs(x).reshape(50, 10, 32).max(2).repeat(32, 1)
    assert (np.abs(v - x) <= top / 127).all()  # a step is at most top / 63.5


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_groups_with_an_infinity_or_nan_read_back_as_nan(dtype):
    torch = need_gpu()
    x = torch.randn((4, 100), device="cuda").to(getattr(torch, dtype))
    x[0, 5], x[1, 40], x[2, 99] = float("nan"), float("inf"), -float("inf")
    g = context()
    keep, y = torch.empty(g.checkpoint_nbytes(4, 100), dtype=torch.uint8, device="cuda"), torch.empty((4, 100), device="cuda")
    g.checkpoint(x, keep)
    g.checkpoint_read(keep, y)
    torch.cuda.synchronize()
    want = np.zeros((4, 100), bool)
    want[0, :32] = want[1, 32:64] = want[2, 96:] = True
    np.testing.assert_array_equal(np.isnan(f64(y)), want)
    g.close()


@pytest.mark.parametrize("rows,K,N,dtype,accumulate,pad,shift", [
    (1, 1, 1, "float32", False, 0, 0), (1, 40, 130, "bfloat16", True, 0, 0), (63, 33, 7, "float32", False, 3, 1), (64, 128, 128, "bfloat16", False, 0, 0),
    (65, 129, 127, "bfloat16", False, 1, 1), (200, 300, 77, "float32", True, 0, 0), (1000, 256, 512, "bfloat16", False, 8, 0), (1500, 260, 264, "float32", False, 0, 0),
    (4099, 96, 520, "bfloat16", True, 0, 0), (130, 1100, 1030, "bfloat16", False, 0, 0), (5000, 512, 256, "float32", False, 0, 0),
    (20000, 64, 72, "bfloat16", False, 0, 0)])
def test_weight_gradient(rows, K, N, dtype, accumulate, pad, shift):
    torch = need_gpu()
    rng = np.random.default_rng(rows + K)
    x = (rng.standard_normal((rows, K)) * np.exp(rng.standard_normal((1, K)))).astype(np.float32)
    dy, _ = place(torch, rng.standard_normal((rows, N)) * np.exp(rng.standard_normal((rows, 1))), getattr(torch, dtype), pad, shift)
    before = rng.standard_normal((K, N)).astype(np.float32)
    grad, flat = place(torch, before, torch.float32, pad, shift)
    g = context()
    keep = torch.empty(g.checkpoint_nbytes(rows, K), dtype=torch.uint8, device="cuda")
    work = torch.full((g.checkpoint_weight_grad_work(rows, K, N),), 0xFF, dtype=torch.uint8, device="cuda")  # NaNs
    g.checkpoint(torch.from_numpy(x).cuda(), keep)
    g.checkpoint_weight_grad(keep, dy, grad, work, accumulate=accumulate)
    torch.cuda.synchronize()
    _, _, v = keep64(x.astype(np.float64))
    want, size, d = torch.from_numpy(v).T @ torch.from_numpy(f64(dy)), np.abs(v).T @ np.abs(f64(dy)), before if accumulate else 0.0
    # exact products (three for an fp32 dy); each addition of the chain of at most 3 rows terms and of the ranges' sums rounds, on the matrix cores perhaps
    # by cutting: a whole step, 2 u
    bound = (3 * rows + 1100) * 2 * U * size + 2 * U * np.abs(d)
    err = np.abs(f64(grad) - (want.numpy() + d))
    assert (err <= bound).all(), (err - bound).max()
    # and as sums of roundings of any sign add up: their root, with a margin of four
    rel = np.linalg.norm(err) / np.linalg.norm(np.sqrt((v * v).T @ (f64(dy) ** 2)) + np.abs(d))
    assert rel <= 4 * 2 * U * np.sqrt(3 * rows + 1100), rel
    assert guards_untouched(torch, flat, K, N, pad, shift)
    g.close()


def test_weight_gradient_of_no_rows():
    torch = need_gpu()
    g = context()
    none, grad = torch.zeros((0, 9), device="cuda"), torch.ones((40, 9), device="cuda")
    keep, work = torch.zeros(0, dtype=torch.uint8, device="cuda"), torch.zeros(g.checkpoint_weight_grad_work(0, 40, 9), dtype=torch.uint8, device="cuda")
    g.checkpoint_weight_grad(keep, none, grad, work, accumulate=True)
    torch.cuda.synchronize()
    assert (grad == 1).all()
    g.checkpoint_weight_grad(keep, none, grad, work)
    torch.cuda.synchronize()
    assert (grad == 0).all()
    g.close()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_values_that_are_not_finite_go_where_the_products_take_them(dtype):
    torch = need_gpu()
    rng = np.random.default_rng(1)
    x, dy = rng.standard_normal((70, 40)).astype(np.float32), rng.standard_normal((70, 50)).astype(np.float32)
    x[3] = 0.0
    x[4] = 2.0
    dy[4, 7], dy[5, 11], dy[3, 13], dy[4, 17] = np.inf, np.nan, np.inf, 3.4e38
    d = torch.from_numpy(dy).cuda().to(getattr(torch, dtype))
    g = context()
    keep = torch.empty(g.checkpoint_nbytes(70, 40), dtype=torch.uint8, device="cuda")
    grad, work = torch.empty((40, 50), device="cuda"), torch.empty(g.checkpoint_weight_grad_work(70, 40, 50), dtype=torch.uint8, device="cuda")
    g.checkpoint(torch.from_numpy(x).cuda(), keep)
    g.checkpoint_weight_grad(keep, d, grad, work)
    torch.cuda.synchronize()
    got = f64(grad)
    assert (got[:, 7] == np.inf).all() and np.isnan(got[:, 11]).all() and np.isnan(got[:, 13]).all() and (got[:, 17] == np.inf).all()
    assert np.isfinite(np.delete(got, [7, 11, 13, 17], 1)).all()
    g.close()
