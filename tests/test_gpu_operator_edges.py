"""Values and sizes at the ends of what the operators are given."""
import numpy as np
import pytest

from gpu_helpers import need_gpu
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
