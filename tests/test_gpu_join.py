"""The join of a block with the residual stream, forward and backward, against its definition in 64 bits and against differences.

Bars. fp32: a row's statistics are sums of C terms (pairwise in 64 lanes of 8 terms each: at most 18 additions in a chain), a value passes some twenty
roundings more, sigma's exponential and reciprocal are good to a few units in the last place: 64 u, relative to the largest magnitude that went into the
value, which for a normalised value is the input's distance from zero in units of sigma. bf16 outputs add half a step of bf16."""
import numpy as np
import pytest

from gpu_helpers import need_gpu
from operator_helpers import BF16_HALF_STEP, U, context, f64, guards_untouched, join64, join_grad64, keep64, place

pytestmark = pytest.mark.gpu
F32_BAR = 64 * U
TYPES = {"f32": ("float32", "float32"), "mixed": ("float32", "bfloat16"), "bf16": ("bfloat16", "bfloat16")}


def _inputs(rng, rows, C, gate, lam, norm_u, norm_n, mean=0.3):
    p = {}
    if lam:
        p["lam"] = (1.0 + 0.3 * rng.standard_normal(C if lam == "vector" else 1)).astype(np.float32)
    for k, norm in (("u", norm_u), ("n", norm_n)):
        if norm != "none":
            p["gamma_" + k] = (1.0 + 0.3 * rng.standard_normal(C)).astype(np.float32)
            p["beta_" + k] = (0.2 * rng.standard_normal(C)).astype(np.float32)
    r, u = 2 * rng.standard_normal((rows, C)) + 0.1, rng.standard_normal((rows, C)) + mean
    return r, u, rng.standard_normal((rows, C)) * 2 if gate else None, p


def _close(got, want, scale, bf16, what):
    """|got - want| within the fp32 bar of `scale` (per row or the whole), and half a bf16 step of the value"""
    bar = F32_BAR * scale + (BF16_HALF_STEP * np.abs(want) if bf16 else 0)
    bad = np.abs(got - want) > bar
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, worst {np.max(np.abs(got - want) / bar):.1f} bars"


def _size(x):  # a row's largest magnitude, at least 1
    return np.maximum(np.abs(x).max(1, keepdims=True), 1.0)


def _vectors(torch, p):
    return {k: torch.from_numpy(v).cuda() for k, v in p.items()}


SHAPES = [(1, 1, "f32"), (5, 8, "bf16"), (3, 31, "f32"), (40, 32, "mixed"), (130, 128, "bf16"), (17, 129, "mixed"), (9, 264, "f32"), (33, 500, "bf16"), (7, 777, "f32"),
          (20, 1024, "bf16"), (6, 2048, "mixed"), (3, 2051, "bf16"), (5, 4096, "bf16"), (2, 4100, "f32"), (3, 8192, "mixed"), (2, 8000, "bf16"), (3, 8192, "f32"),
          (2, 8191, "bf16")]
MODELS = [("layer", "layer", True, "vector"), ("rms", "rms", True, "scalar"), ("none", "layer", False, None), ("layer", "none", True, None), ("none", "none", False, "vector"),
          ("rms", "layer", False, "scalar")]


@pytest.mark.parametrize("i,shape", enumerate(SHAPES))
@pytest.mark.parametrize("model", MODELS[:3])
def test_forward(i, shape, model):
    torch = need_gpu()
    rows, C, types = shape
    model = model if i % 2 == 0 else MODELS[3 + MODELS.index(model)]
    norm_u, norm_n, gate, lam = model
    st, br = (getattr(torch, t) for t in TYPES[types])
    pad, shift = (0, 0) if i % 3 == 0 else (i % 5, i % 4)
    r, u, g, p = _inputs(np.random.default_rng(i), rows, C, gate, lam, norm_u, norm_n)
    (r, _), (u, _) = place(torch, r, st, pad, shift), place(torch, u, br, pad, shift)
    g = place(torch, g, br, pad, shift)[0] if gate else None
    (h, fh), (n, fn) = place(torch, np.zeros((rows, C)), st, pad, shift), place(torch, np.zeros((rows, C)), br, pad, shift)
    c = context()
    keep = {k: torch.full((c.checkpoint_nbytes(rows, C) + 16,), 0xA5, dtype=torch.uint8, device="cuda") for k in ("keep_r", "keep_u", "keep_n") + (("keep_g",) if gate else ())}
    c.join(h, n, r=r, u=u, g=g, norm_u=norm_u, norm_n=norm_n, **_vectors(torch, p), **{k: v[:-16] for k, v in keep.items()})
    torch.cuda.synchronize()
    f = join64(f64(r), f64(u), f64(g) if gate else None, p, norm_u, norm_n)
    # what a value of z and h was made of; n divides it by h's sigma
    made = _size(f64(r)) * 2 + _size(f["uhat"]) * 2 * (1 + np.abs(f64(u)).max(1, keepdims=True) * f["urstd"])
    _close(f64(h), f["h"], made, st == torch.bfloat16, "h")
    _close(f64(n), f["n"], 2 * (made * f["rstd"] if norm_n != "none" else made) + _size(f["n"]), br == torch.bfloat16, "n")
    assert guards_untouched(torch, fh, rows, C, pad, shift) and guards_untouched(torch, fn, rows, C, pad, shift)
    # the checkpoints are those of the operands, and of n as it was rounded
    for k, of in (("keep_r", r), ("keep_u", u), ("keep_g", g), ("keep_n", n)):
        if k in keep:
            q, e, _ = keep64(f64(of))
            host = keep[k].cpu().numpy()
            np.testing.assert_array_equal(host[:q.size].view(np.int8), q.reshape(-1), err_msg=k)
            np.testing.assert_array_equal(host[q.size:q.size + e.size], e.reshape(-1), err_msg=k)
            assert (host[q.size + e.size:] == 0xA5).all()
    c.close()


def _grads(torch, c, rows, C, st, br, operands, dh, dn, p, norm_u, norm_n, gate, accumulate=False, start=0.0, **more):
    out = {"dr": torch.full((rows, C), 5.0, dtype=st, device="cuda"), "du": torch.full((rows, C), 5.0, dtype=br, device="cuda")}
    if gate:
        out["dg"] = torch.full((rows, C), 5.0, dtype=br, device="cuda")
    for k, v in p.items():
        out["d_" + k] = torch.full((v.size,), start, device="cuda")
    work = torch.full((c.join_grad_work(rows, C),), 0xFF, dtype=torch.uint8, device="cuda")
    c.join_grad(dh, dn, work, norm_u=norm_u, norm_n=norm_n, accumulate=accumulate, **operands, **out, **_vectors(torch, p), **more)
    torch.cuda.synchronize()
    return out


def _check_grads(out, r, u, g, p, norm_u, norm_n, dh, dn, st16, br16, start=0.0):
    w = join_grad64(r, u, g, p, norm_u, norm_n, dh, dn)
    f = join64(r, u, g, p, norm_u, norm_n)
    # a gradient is made of dh and of dn in units of h's sigma, with the sums over the row; statistics and uhat carry the operands' own errors
    err_u = 1 + np.abs(u).max(1, keepdims=True) * f["urstd"]
    err_h = 1 + (np.abs(r).max(1, keepdims=True) + _size(f["uhat"]) * 2 * err_u) * f["rstd"]
    t = (0 if dh is None else np.abs(dh).max(1, keepdims=True)) + (0 if dn is None else np.abs(dn).max(1, keepdims=True) * 2 * f["rstd"] * _size(f["hat"]) * err_h * 2)
    scale_z = _size(f["z"]) * err_u
    _close(out["dr"], w["dr"], 2 * t, st16, "dr")
    _close(out["du"], w["du"], 4 * t * f["urstd"] * _size(f["uhat"]) * err_u, br16, "du")
    if g is not None:
        _close(out["dg"], w["dg"], t * scale_z, br16, "dg")
    rows = r.shape[0]
    long = 1 + rows / 64  # the sum over the rows: their terms' errors, and as many additions
    for k, made in (("d_gamma_n", None if dn is None else np.abs(dn).max() * (_size(f["hat"]) * err_h).max()), ("d_beta_n", None if dn is None else np.abs(dn).max()),
                    ("d_gamma_u", (t * _size(f["uhat"]) * err_u).max()), ("d_beta_u", t.max()), ("d_lam", (t * np.abs(r).max(1, keepdims=True)).max())):
        if k in out:
            terms = rows * (r.shape[1] if k == "d_lam" and out[k].size == 1 else 1)
            made = 0.0 if made is None else made
            _close(out[k] - start, w[k], (made * long * terms + abs(start)) * np.ones(1), False, k)


@pytest.mark.parametrize("i,shape", enumerate(SHAPES + [(1030, 24, "f32"), (2100, 100, "bf16"), (700, 1000, "mixed")]))
@pytest.mark.parametrize("model", MODELS[:3])
@pytest.mark.parametrize("kept", [False, True])
def test_backward(i, shape, model, kept):
    torch = need_gpu()
    rows, C, types = shape
    model = model if i % 2 == 0 else MODELS[3 + MODELS.index(model)]
    norm_u, norm_n, gate, lam = model
    st, br = (getattr(torch, t) for t in TYPES[types])
    rng = np.random.default_rng(i + 50)
    r, u, g, p = _inputs(rng, rows, C, gate, lam, norm_u, norm_n)
    pad, shift = (0, 0) if i % 3 == 0 else (i % 5, i % 4)
    place_ = lambda x, t: None if x is None else place(torch, x, t, pad, shift)[0]  # noqa: E731
    r, u, g, dh, dn = place_(r, st), place_(u, br), place_(g, br), place_(0.1 * rng.standard_normal((rows, C)), st), place_(0.1 * rng.standard_normal((rows, C)), br)
    c = context()
    operands = {"r": r, "u": u, "g": g}
    values = [f64(x) if x is not None else None for x in (r, u, g)]
    if kept:
        values = [None if x is None else keep64(x)[2] for x in values]
        buf = {}
        for k, x in operands.items():
            if x is not None:
                buf["keep_" + k] = torch.empty(c.checkpoint_nbytes(rows, C), dtype=torch.uint8, device="cuda")
                c.checkpoint(x, buf["keep_" + k])
        operands = buf
    accumulate, start = (True, 0.25) if i % 2 else (False, 7.0)
    out = _grads(torch, c, rows, C, st, br, operands, dh, dn, p, norm_u, norm_n, gate, accumulate, start)
    _check_grads({k: f64(v) for k, v in out.items()}, *values, p, norm_u, norm_n, f64(dh), f64(dn), st == torch.bfloat16, br == torch.bfloat16, start if accumulate else 0.0)
    again = _grads(torch, c, rows, C, st, br, operands, dh, dn, p, norm_u, norm_n, gate, accumulate, start)
    assert all(torch.equal(out[k], again[k]) for k in out)  # the same bits
    c.close()


@pytest.mark.parametrize("missing", ["dh", "dn"])
def test_backward_of_one_output(missing):
    torch = need_gpu()
    rows, C = 21, 200
    rng = np.random.default_rng(3)
    r, u, g, p = _inputs(rng, rows, C, True, "scalar", "layer", "rms")
    dev = {k: torch.from_numpy(v.astype(np.float32)).cuda() for k, v in (("r", r), ("u", u), ("g", g))}
    d = rng.standard_normal((rows, C)).astype(np.float32)
    dh, dn = (None, d) if missing == "dh" else (d, None)
    c = context()
    out = _grads(torch, c, rows, C, torch.float32, torch.float32, dev, *(None if x is None else torch.from_numpy(x).cuda() for x in (dh, dn)), p, "layer", "rms", True)
    _check_grads({k: f64(v) for k, v in out.items()}, *(f64(dev[k]) for k in "rug"), p, "layer", "rms", dh, dn, False, False)
    c.close()


def test_backward_against_differences():
    """The definition's gradient is the derivative of its forward pass (64 bits, central differences of step 1e-5: error 1e-10 of third derivatives), and
    the kernel's is the definition's (above)."""
    rng = np.random.default_rng(4)
    for norm_u, norm_n, gate, lam in MODELS:
        r, u, g, p = _inputs(rng, 3, 10, gate, lam, norm_u, norm_n)
        p = {k: v.astype(np.float64) for k, v in p.items()}
        dh, dn = rng.standard_normal((3, 10)), rng.standard_normal((3, 10))

        def loss():
            f = join64(r, u, g, p, norm_u, norm_n)
            return (f["h"] * dh).sum() + (f["n"] * dn).sum()

        w = join_grad64(r, u, g, p, norm_u, norm_n, dh, dn)
        for x, d in [(r, w["dr"]), (u, w["du"])] + ([(g, w["dg"])] if gate else []) + [(p[k], w["d_" + k]) for k in p]:
            for at in np.ndindex(x.shape):
                was = x[at]
                x[at] = was + 1e-5
                up = loss()
                x[at] = was - 1e-5
                down = loss()
                x[at] = was
                assert abs((up - down) / 2e-5 - d[at]) <= 1e-6 * max(1.0, abs(d[at]))


@pytest.mark.parametrize("norm", ["layer", "rms"])
def test_rows_without_variance_and_far_from_zero(norm):
    """A constant row's normalised values are zeros (layer); a mean of a thousand sigma costs the digits that the input itself has lost, no more."""
    torch = need_gpu()
    rows, C = 4, 640
    rng = np.random.default_rng(6)
    u = 1e-3 * rng.standard_normal((rows, C)) + np.array([[0.0], [3.0], [1000.0], [-1.0]])
    u[1] = 3.0
    r = np.zeros((rows, C))
    r[0] = 0.5
    dev = {k: torch.from_numpy(v.astype(np.float32)).cuda() for k, v in (("r", r), ("u", u))}
    h, n = torch.empty((rows, C), device="cuda"), torch.empty((rows, C), device="cuda")
    c = context()
    c.join(h, n, norm_u=norm, norm_n="none", **dev)
    torch.cuda.synchronize()
    f = join64(f64(dev["r"]), f64(dev["u"]), None, {}, norm, "none")
    if norm == "layer":
        assert (f64(h)[1] == 0).all()
    made = 2 + _size(f["uhat"]) + np.abs(u).max(1, keepdims=True) * f["urstd"]
    _close(f64(h), f["h"], made, False, "h")
    assert torch.equal(n, h)  # no norm: n is h
    c.close()


def test_in_place():
    """h over r, dr over dh and du over dn are the same bits as with buffers of their own."""
    torch = need_gpu()
    rows, C = 37, 1500
    rng = np.random.default_rng(7)
    r, u, g, p = _inputs(rng, rows, C, True, "vector", "layer", "layer")
    r, u, g, dh, dn = (torch.from_numpy(x.astype(np.float32)).cuda().bfloat16() for x in (r, u, g, rng.standard_normal((rows, C)), rng.standard_normal((rows, C))))
    c = context()
    v = _vectors(torch, p)
    h, n = torch.empty_like(r), torch.empty_like(r)
    c.join(h, n, r=r, u=u, g=g, **v)
    torch.cuda.synchronize()
    r2 = r.clone()
    c.join(r2, n, r=r2, u=u, g=g, **v)
    torch.cuda.synchronize()
    assert torch.equal(r2, h)
    work = torch.empty(c.join_grad_work(rows, C), dtype=torch.uint8, device="cuda")
    dr, du = torch.empty_like(r), torch.empty_like(r)
    c.join_grad(dh, dn, work, r=r, u=u, g=g, dr=dr, du=du, **v)
    torch.cuda.synchronize()
    dh2, dn2 = dh.clone(), dn.clone()
    c.join_grad(dh2, dn2, work, r=r, u=u, g=g, dr=dh2, du=dn2, **v)
    torch.cuda.synchronize()
    assert torch.equal(dh2, dr) and torch.equal(dn2, du)
    c.close()


def test_a_row_does_not_depend_on_its_batch():
    torch = need_gpu()
    C = 1111
    rng = np.random.default_rng(9)
    r, u, g, p = _inputs(rng, 600, C, True, "vector", "layer", "rms")
    r, u, g = (torch.from_numpy(x.astype(np.float32)).cuda() for x in (r, u, g))
    c = context()
    v = _vectors(torch, p)
    h, n = torch.empty_like(r), torch.empty_like(r)
    c.join(h, n, r=r, u=u, g=g, norm_n="rms", **v)
    one_h, one_n = torch.empty((1, C), device="cuda"), torch.empty((1, C), device="cuda")
    for i in (0, 1, 299, 599):
        torch.cuda.synchronize()
        c.join(one_h, one_n, r=r[i:i + 1], u=u[i:i + 1], g=g[i:i + 1], norm_n="rms", **v)
        torch.cuda.synchronize()
        assert torch.equal(one_h[0], h[i]) and torch.equal(one_n[0], n[i])
    c.close()


def test_no_rows():
    torch = need_gpu()
    c = context()
    none = torch.zeros((0, 40), device="cuda")
    gamma = torch.ones(40, device="cuda")
    c.join(none, none.clone(), r=none, u=none, gamma_u=gamma)
    work = torch.empty(c.join_grad_work(0, 40), dtype=torch.uint8, device="cuda")
    for accumulate, want in ((True, 3.0), (False, 0.0)):
        d = torch.full((40,), 3.0, device="cuda")
        c.join_grad(none, none, work, r=none, u=none, gamma_u=gamma, d_gamma_u=d, accumulate=accumulate)
        torch.cuda.synchronize()
        assert (d == want).all()
    c.close()


def test_refusals_leave_the_outputs_alone():
    torch = need_gpu()
    import paper_2604_07239_amd as fa
    c = context()
    x = torch.zeros((4, 40), device="cuda")
    h = torch.full((4, 40), 9.0, device="cuda")
    bad = [dict(norm_u="batch"), dict(u=x[:, :39]), dict(u=x.t()), dict(u=x.double()), dict(r=x.cpu()), dict(lam=torch.ones(3, device="cuda")),
           dict(gamma_u=torch.ones(41, device="cuda")), dict(norm_u="none", gamma_u=torch.ones(40, device="cuda")), dict(eps=-1.0),
           dict(keep_u=torch.zeros(10, dtype=torch.uint8, device="cuda")), dict(u=x.bfloat16(), g=x), dict(r=x.bfloat16(), u=x),
           dict(keep_g=torch.zeros(1000, dtype=torch.uint8, device="cuda"))]
    for over in bad:
        with pytest.raises(fa.FadeError) as e:
            c.join(h, None, **{"r": x, "u": x, **over})
        assert e.value.code == -1, over
    work = torch.zeros(c.join_grad_work(4, 40), dtype=torch.uint8, device="cuda")
    for over in (dict(work=work[:-16]), dict(work=work[8:]), dict(dh=None, dn=None), dict(keep_r=work), dict(dg=h), dict(d_lam=h[0, :1])):
        with pytest.raises(fa.FadeError) as e:
            c.join_grad(**{"dh": x, "dn": x, "work": work, "r": x, "u": x, "dr": h, **over})
        assert e.value.code == -1, over
    torch.cuda.synchronize()
    assert (h == 9.0).all()
    c.close()
