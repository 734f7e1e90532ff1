"""The join and its gradient in 64 bits, on whatever device the operands are, and bars on what a kernel in fp32 makes of them. Written from the definitions.

u = 2^-24 is half a step of fp32. A row's bar is a norm over its columns: roundings of any sign add up as the root of their number, each at most u / sqrt(3) of the magnitudes that
went into the value, with a margin of four. h: the 18 additions of a statistic, its root (1 ulp), six roundings of the normalised value and as many of sigma and the sum,
some 30: sqrt(30 / 3) u = 3.2 u, bar 16 u (a gate adds |g| u to sigma, 1.6 u where g is normal with a spread of 2). n goes through as many again, on values that carry h's errors: 32 u.
What both statistics enter has twice that, 64 u, and du, with u's sums on top, 128 u. bf16 outputs add half a step of bf16 of the value.
A parameter's gradient sums terms over the rows: element by element 512 u of the terms' magnitudes (256 u a term at worst, and the additions of its chain, at most 60 and one a turn);
and, as errors of different rows have any sign, as a norm over all its elements 64 u of the root of the terms' squares and of the sums: a term's roundings, some 40
of at most u / sqrt(3) each, are 4 u of the magnitudes, those of the additions 3 u, hardware functions that err to one side 8 u of the sum; four times that."""
import torch

U = 2.0 ** -24
BF16_HALF_STEP = 2.0 ** -8


def _norm(x, kind, gamma, beta, eps):
    """value, normalised value, 1 / sigma, and the magnitudes that went into the normalised one"""
    if kind == "none":
        return x, x, torch.ones_like(x[:, :1]), x.abs()
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    rstd = 1.0 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    hat = (x - mean) * rstd
    return hat * (1.0 if gamma is None else gamma) + (0.0 if beta is None else beta), hat, rstd, (x.abs() + x.abs().mean(1, keepdim=True)) * rstd + hat.abs()


def _abs(v, otherwise):
    return otherwise if v is None else v.abs()


def forward(r, u, g, p, norm_u, norm_n, eps=1e-5):
    """h and n with their magnitudes, and what the backward pass needs again"""
    z, uhat, urstd, m_uhat = _norm(u, norm_u, p.get("gamma_u"), p.get("beta_u"), eps)
    m_z = m_uhat * _abs(p.get("gamma_u"), 1.0) + _abs(p.get("beta_u"), 0.0)
    s = torch.ones_like(u) if g is None else torch.sigmoid(g)
    lam = 1.0 if p.get("lam") is None else p["lam"]
    h = lam * r + s * z
    m_h = (lam * r).abs() + s * m_z
    n, hat, rstd, m_hat = _norm(h, norm_n, p.get("gamma_n"), p.get("beta_n"), eps)
    m_hat = m_hat + (m_h + m_h.mean(1, keepdim=True)) * rstd
    m_n = m_hat * _abs(p.get("gamma_n"), 1.0) + _abs(p.get("beta_n"), 0.0)
    return dict(h=h, n=n, m_h=m_h, m_n=m_n, z=z, m_z=m_z, uhat=uhat, m_uhat=m_uhat, urstd=urstd, s=s, hat=hat, m_hat=m_hat, rstd=rstd)


def _norm_grad(d, m_d, kind, hat, m_hat, rstd):
    if kind == "none":
        return d, m_d
    mean = lambda x: x.mean(1, keepdim=True)  # noqa: E731
    layer = kind == "layer"
    return rstd * (d - (mean(d) if layer else 0.0) - hat * mean(d * hat)), rstd * (m_d + (mean(m_d) if layer else 0.0) + m_hat * mean(m_d * m_hat))


def backward(r, u, g, p, norm_u, norm_n, dh, dn, eps=1e-5):
    """{name: (value, magnitudes)} of dr, du, dg and {name: (terms [rows][C], their magnitudes)} of the parameters"""
    f = forward(r, u, g, p, norm_u, norm_n, eps)
    gn, gu, lam = p.get("gamma_n"), p.get("gamma_u"), p.get("lam")
    e, m_e = _norm_grad(dn * (1.0 if gn is None else gn), dn.abs() * _abs(gn, 1.0), norm_n, f["hat"], f["m_hat"], f["rstd"])
    t, m_t = dh + e, dh.abs() + m_e
    dz, m_dz = t * f["s"], m_t * f["s"]
    out = {"dr": (t * (1.0 if lam is None else lam), m_t * _abs(lam, 1.0)),
           "du": _norm_grad(dz * (1.0 if gu is None else gu), m_dz * _abs(gu, 1.0), norm_u, f["uhat"], f["m_uhat"], f["urstd"])}
    if g is not None:
        out["dg"] = (dz * f["z"] * (1.0 - f["s"]), m_dz * f["m_z"])
    terms = {"lam": (t * r, m_t * r.abs()), "gamma_u": (dz * f["uhat"], m_dz * f["m_uhat"]), "beta_u": (dz, m_dz), "gamma_n": (dn * f["hat"], dn.abs() * f["m_hat"]),
             "beta_n": (dn, dn.abs())}
    return out, {"d_" + k: terms[k] for k in p}


def rows_wrong(got, want, made, steps, bf16):
    """How many rows are further from `want` than their bar."""
    bar = steps * U * made.norm(dim=1) + (BF16_HALF_STEP * want.norm(dim=1) if bf16 else 0.0)
    return int((~((got - want).norm(dim=1) <= bar)).sum())  # what is no number is wrong


def sums_wrong(got, terms, made, start=0.0):
    """What is wrong with a parameter's gradient that was added to `start`: None if nothing is."""
    one = got.numel() == 1 and terms.shape[1] > 1
    over = (0, 1) if one else (0,)
    want, size, square = (x.sum(over).reshape(-1) for x in (terms, made, made ** 2))
    err = (got - start - want).abs()
    if not bool((err <= 512 * U * size + 2 * U * (abs(start) + want.abs())).all()):
        return f"an element, {float((err / (512 * U * size)).max()):.2f} bars"
    bar = 64 * U * (square.sqrt().norm() + want.norm()) + 2 * U * abs(start) * want.numel() ** 0.5
    return None if bool(err.norm() <= bar) else f"the norm, {float(err.norm() / bar):.2f} bars"


def model(rng, C, gate, lam, norm_u, norm_n, make):
    """Parameters; `make` turns a numpy array into a tensor."""
    p = {}
    if lam:
        p["lam"] = make(1.0 + 0.3 * rng.standard_normal(C if lam == "vector" else 1))
    for k, norm in (("u", norm_u), ("n", norm_n)):
        if norm != "none":
            p["gamma_" + k] = make(1.0 + 0.3 * rng.standard_normal(C))
            p["beta_" + k] = make(0.2 * rng.standard_normal(C))
    return p


MODELS = [("layer", "layer", True, "vector"), ("rms", "rms", True, "scalar"), ("none", "layer", False, None), ("layer", "none", True, None),
          ("none", "none", False, "vector"), ("rms", "layer", False, "scalar")]
TYPES = {"f32": (torch.float32, torch.float32), "mixed": (torch.float32, torch.bfloat16), "bf16": (torch.bfloat16, torch.bfloat16)}
STEPS = {"h": 16, "n": 32, "dr": 64, "dg": 64, "du": 128}
