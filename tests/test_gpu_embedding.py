"""Embedding lookup with scaling and its gradient by sorted tokens against their definitions."""
import numpy as np
import pytest

from gpu_helpers import need_gpu
from operator_helpers import U, context, f64, guards_untouched, place

pytestmark = pytest.mark.gpu
TOKENS = {"u8": np.uint8, "i32": np.int32, "i64": np.int64}


def _tokens(rng, n, vocab, kind, outside=False):
    t = rng.integers(0, min(vocab, 256) if kind == "u8" else vocab, n)
    if outside and n:
        t[rng.random(n) < 0.2] = 255 if kind == "u8" else -1
        if kind == "i64":
            t[rng.random(n) < 0.1] = (1 << 40) + 1  # its low word is a token of most vocabularies
        if kind == "i32":
            t[rng.random(n) < 0.1] = vocab
    return t.astype(TOKENS[kind])


@pytest.mark.parametrize("n,vocab,width,token,table,out,pad,shift", [
    (1, 256, 32, "u8", "float32", "float32", 0, 0), (16, 256, 1, "i32", "bfloat16", "float32", 0, 0), (33, 7, 7, "i64", "float32", "bfloat16", 3, 1),
    (257, 1000, 33, "i32", "bfloat16", "bfloat16", 1, 3), (1000, 1, 1000, "u8", "float32", "float32", 0, 0),
    (130, 5000, 2056, "i64", "bfloat16", "float32", 8, 1), (5, 9, 20000, "i32", "float32", "bfloat16", 0, 0)])
def test_lookup_is_the_rounded_product(n, vocab, width, token, table, out, pad, shift):
    torch = need_gpu()
    rng = np.random.default_rng(n + width)
    T, O = getattr(torch, table), getattr(torch, out)
    e, _ = place(torch, rng.standard_normal((vocab, width)), T, pad, shift)
    t = _tokens(rng, n, vocab, token, outside=True)
    y, flat = place(torch, np.zeros((n, width)), O, pad, shift)
    g = context()
    g.embed(torch.from_numpy(t).cuda(), e, y, scale=1.7)
    torch.cuda.synchronize()
    inside = (t.astype(np.int64) >= 0) & (t.astype(np.int64) < vocab)
    want = torch.zeros((n, width), device="cuda")
    want[torch.from_numpy(inside).cuda()] = e.float()[torch.from_numpy(t.astype(np.int64)[inside]).cuda()] * 1.7
    assert torch.equal(y, want.to(O))
    assert guards_untouched(torch, flat, n, width, pad, shift)
    g.close()


def test_nothing_is_done_for_no_tokens():
    torch = need_gpu()
    g = context()
    empty = torch.zeros(0, dtype=torch.int32, device="cuda")
    e, none = torch.ones((5, 8), device="cuda"), torch.zeros((0, 8), device="cuda")
    g.embed(empty, e, none)
    grad, work = torch.ones((5, 8), device="cuda"), torch.zeros(g.embed_grad_work(0, 5, 8), dtype=torch.uint8, device="cuda")
    g.embed_grad(empty, none, grad, work, accumulate=True)
    torch.cuda.synchronize()
    assert (grad == 1).all()
    g.embed_grad(empty, none, grad, work)
    torch.cuda.synchronize()
    assert (grad == 0).all()
    g.close()


def _check_grad(torch, g, t, dy, vocab, scale, accumulate, pad=0, shift=0, dtype="float32"):
    n, width = dy.shape
    d, _ = place(torch, dy, getattr(torch, dtype), pad, shift)
    rng = np.random.default_rng(1)
    before = rng.standard_normal((vocab, width)).astype(np.float32)
    grad, flat = place(torch, before, torch.float32, pad, shift)
    work = torch.full((g.embed_grad_work(n, vocab, width),), 0xA5, dtype=torch.uint8, device="cuda")
    g.embed_grad(torch.from_numpy(t).cuda(), d, grad, work, scale=scale, accumulate=accumulate)
    torch.cuda.synchronize()
    got, d64 = f64(grad), f64(d)
    t64 = t.astype(np.int64)
    inside = (t64 >= 0) & (t64 < vocab)
    want, size, count = np.zeros((vocab, width)), np.zeros((vocab, width)), np.zeros((vocab, 1))
    np.add.at(want, t64[inside], d64[inside])
    np.add.at(size, t64[inside], np.abs(d64[inside]))
    np.add.at(count, t64[inside], 1)
    want, size = want * scale, size * abs(scale)
    # the sum, its product with the scale (fp32 itself: half a step), and the sum with what was there
    bound = (count + 2) * U * size + (2 * U * (np.abs(before) + np.abs(want)) if accumulate else 0)
    if accumulate:
        want = want + before
        np.testing.assert_array_equal(got[count[:, 0] == 0], before[count[:, 0] == 0])
    assert (np.abs(got - want) <= bound).all(), np.abs(got - want).max()
    assert guards_untouched(torch, flat, vocab, width, pad, shift)
    return grad.clone()


@pytest.mark.parametrize("n,vocab,width,token,dtype,accumulate,pad,shift", [
    (1, 256, 32, "u8", "float32", False, 0, 0), (1, 70000, 8, "i32", "float32", True, 0, 0), (31, 3, 1, "i64", "bfloat16", False, 0, 0),
    (32, 1, 33, "i32", "float32", False, 2, 1), (33, 2, 7, "u8", "bfloat16", True, 1, 3), (1000, 1023, 64, "i32", "float32", False, 0, 0),
    (1025, 1024, 100, "i64", "bfloat16", False, 4, 1), (2049, 1025, 520, "i32", "float32", True, 0, 0), (5000, 7, 129, "u8", "bfloat16", False, 0, 0),
    (4097, 50021, 40, "i64", "float32", False, 0, 0), (300, 1 << 20, 4, "i32", "bfloat16", False, 0, 0), (140000, 300, 16, "i32", "bfloat16", False, 0, 0),
    (70, 11, 5000, "i32", "float32", False, 0, 0), (4096, 30000, 24, "i64", "float32", False, 0, 0), (8192, 60000, 24, "i32", "bfloat16", True, 0, 0),
    (8193, 60000, 24, "i32", "float32", False, 0, 0), (16384, 256, 40, "u8", "bfloat16", False, 0, 0), (16385, 256, 40, "u8", "float32", False, 0, 0),
    (20011, 50021, 17, "i64", "bfloat16", True, 1, 1), (9000, 1 << 20, 8, "i32", "float32", False, 0, 0)])
def test_gradient_against_the_sum(n, vocab, width, token, dtype, accumulate, pad, shift):
    torch = need_gpu()
    rng = np.random.default_rng(n + vocab)
    g = context()
    _check_grad(torch, g, _tokens(rng, n, vocab, token, outside=True), rng.standard_normal((n, width)), vocab, 0.7, accumulate, pad, shift, dtype)
    g.close()


@pytest.mark.parametrize("width", [72, 600])
@pytest.mark.parametrize("case", ["one token", "all different", "none inside", "two runs", "borders"])
def test_gradient_of_extreme_runs(case, width):
    torch = need_gpu()
    n, vocab = 6001, 7000
    t = {"one token": np.full(n, 4321), "all different": np.random.default_rng(3).permutation(vocab)[:n], "none inside": np.full(n, -5),
         "two runs": np.where(np.arange(n) % 2 == 0, 17, 6999), "borders": np.arange(n) // 32}[case].astype(np.int32)
    g = context()
    _check_grad(torch, g, t, np.random.default_rng(4).standard_normal((n, width)), vocab, 3.0, False)
    g.close()


def test_gradient_is_the_same_bits_every_time_and_on_every_context():
    torch = need_gpu()
    rng = np.random.default_rng(8)
    t, dy = np.minimum(rng.geometric(0.02, 50000), 400).astype(np.int32), rng.standard_normal((50000, 48))
    a, b = context(), context()
    first = _check_grad(torch, a, t, dy, 512, 1.0, False)
    for g in (a, b, a):
        assert torch.equal(first, _check_grad(torch, g, t, dy, 512, 1.0, False))
    a.close()
    b.close()


def test_padding_may_hold_anything():
    """NaN and infinities in the rows of tokens outside the table reach nothing."""
    torch = need_gpu()
    rng = np.random.default_rng(5)
    t = _tokens(rng, 500, 40, "i32", outside=True)
    dy = rng.standard_normal((500, 24)).astype(np.float32)
    clean = dy.copy()
    dy[(t < 0) | (t >= 40)] = np.array([np.nan, np.inf, -np.inf] * 8)
    clean[(t < 0) | (t >= 40)] = 0
    g = context()
    got = []
    for d in (dy, clean):
        grad, work = torch.empty((40, 24), device="cuda"), torch.empty(g.embed_grad_work(500, 40, 24), dtype=torch.uint8, device="cuda")
        g.embed_grad(torch.from_numpy(t).cuda(), torch.from_numpy(d).cuda(), grad, work)
        torch.cuda.synchronize()
        got.append(grad)
    assert torch.equal(got[0], got[1])
    g.close()


@pytest.mark.parametrize("n,vocab,width,dtype", [(70001, 3000, 600, "bfloat16"), (140000, 700, 1024, "bfloat16"), (300000, 256, 64, "float32"), (33000, 200000, 520, "float32")])
def test_gradient_of_large_batches(n, vocab, width, dtype):
    """Pieces of every length, against 64-bit sums on the device; tokens as frequent as in a text, so that runs of every length cross every border."""
    torch = need_gpu()
    rng = np.random.default_rng(n)
    t = torch.from_numpy(np.minimum(np.exp(rng.random(n) * np.log(vocab + 1)).astype(np.int64) - 1, vocab - 1)).cuda()
    d = torch.randn((n, width), device="cuda").to(getattr(torch, dtype))
    g = context()
    grad, work = torch.full((vocab, width), 7.0, device="cuda"), torch.full((g.embed_grad_work(n, vocab, width),), 0xA5, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    g.embed_grad(t, d, grad, work, scale=0.5)
    torch.cuda.synchronize()
    want = torch.zeros((vocab, width), dtype=torch.float64, device="cuda").index_add_(0, t, d.double()) * 0.5
    size = torch.zeros((vocab, width), dtype=torch.float64, device="cuda").index_add_(0, t, d.double().abs()) * 0.5
    count = torch.bincount(t, minlength=vocab)[:, None]
    assert ((grad.double() - want).abs() <= (count + 2) * U * size).all()
    g.close()


def test_more_rows_than_a_launch_has_workgroups():
    """2^24 + 5 rows of 1032 columns (35 GB): the rows behind those that one workgroup each takes first."""
    torch = need_gpu()
    n, width = (1 << 24) + 5, 1032
    g = context()
    table = torch.randn((3, width), device="cuda").bfloat16()
    t = torch.zeros(n, dtype=torch.uint8, device="cuda")
    t[-7:] = 2
    t[n // 2] = 1
    out = torch.empty((n, width), dtype=torch.bfloat16, device="cuda")
    keep = torch.empty(g.checkpoint_nbytes(n, width), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    g.embed(t, table, out)
    g.checkpoint(out, keep)
    torch.cuda.synchronize()
    for at, v in ((0, 0), (n // 2, 1), (n // 2 + 1, 0), (n - 8, 0), (n - 7, 2), (n - 1, 2)):
        assert torch.equal(out[at], table[v]), at
    back = torch.empty((3, width), dtype=torch.bfloat16, device="cuda")
    small = torch.empty(g.checkpoint_nbytes(3, width), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    g.checkpoint(table, small)
    g.checkpoint_read(small, back)
    g.checkpoint_read(keep, out)
    torch.cuda.synchronize()
    for at, v in ((0, 0), (n // 2, 1), (n - 1, 2)):
        assert torch.equal(out[at], back[v]), at
    g.close()
