"""Plain 64-bit forms of the operators around a program's own model, and their inputs. Written from the definitions; no code of the library.

Error bounds: u = 2^-24 is half a step of fp32. A sum of m terms in any order is off by at most (m - 1) u times the sum of their magnitudes
(to first order); a value rounded to bf16 by at most 2^-8 of itself."""
import numpy as np

U = 2.0 ** -24
BF16_HALF_STEP = 2.0 ** -8


def context(stream=None):
    import paper_2604_07239_amd as fa
    return fa.Fade(fa.make_config(16, 32, 16, 128, dtype=fa.F32, hip_stream=stream))


def place(torch, x, dtype, pad=0, shift=0):
    """x on the device as `dtype` with `pad` guard elements behind each row and `shift` in front of the first; the guards hold 777."""
    rows, width = x.shape
    flat = torch.full((rows * (width + pad) + shift + 8,), 777.0, dtype=dtype, device="cuda")
    view = flat[shift:shift + rows * (width + pad)].view(rows, width + pad)
    view[:, :width] = torch.as_tensor(np.ascontiguousarray(x), device="cuda").to(dtype)
    return view[:, :width], flat


def guards_untouched(torch, flat, rows, width, pad, shift):
    left = flat.clone()
    left[shift:shift + rows * (width + pad)].view(rows, width + pad)[:, :width] = 777.0
    return bool((left == 777.0).all())


def f64(t):
    return t.detach().double().cpu().numpy()


# -- checkpoints ---------------------------------------------------------------------------------------
def keep64(x):
    """(bytes q [rows][32 G], exponents [rows][G], values [rows][width]) of a checkpoint, group by group from the definition."""
    rows, width = x.shape
    G = (width + 31) // 32
    v = np.zeros((rows, G, 32))
    v.reshape(rows, -1)[:, :width] = x
    q, e = np.zeros((rows, G, 32), np.int8), np.zeros((rows, G), np.int64)
    finite = np.isfinite(v).all(2)
    top = np.where(finite, np.abs(np.where(np.isfinite(v), v, 0)).max(2), 0.0)
    e[:] = -126
    while True:  # the least exponent that reaches the largest value
        short = top > 127.0 * np.exp2(e.astype(np.float64))
        if not short.any():
            break
        e[short] += 1
    unit = np.exp2(e.astype(np.float64))[:, :, None]
    q[:] = np.where(finite[:, :, None], np.rint(np.where(np.isfinite(v), v, 0) / unit), 0)
    values = np.where(finite[:, :, None], q * unit, np.nan).reshape(rows, -1)[:, :width]
    return q.reshape(rows, -1), np.where(finite, e + 127, 255).astype(np.uint8), values


# -- join ----------------------------------------------------------------------------------------------
def norm64(x, kind, gamma, beta, eps):
    if kind == "none":
        return x, x, np.ones((x.shape[0], 1))
    c = x - x.mean(1, keepdims=True) if kind == "layer" else x
    rstd = 1.0 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    hat = c * rstd
    return hat * (1.0 if gamma is None else gamma) + (0.0 if beta is None else beta), hat, rstd


def norm_grad64(dy, kind, hat, rstd, gamma):
    if kind == "none":
        return dy
    d = dy * (1.0 if gamma is None else gamma)
    return rstd * (d - (d.mean(1, keepdims=True) if kind == "layer" else 0.0) - hat * (d * hat).mean(1, keepdims=True))


def join64(r, u, g, p, norm_u, norm_n, eps=1e-5):
    z, uhat, urstd = norm64(u, norm_u, p.get("gamma_u"), p.get("beta_u"), eps)
    s = 1.0 / (1.0 + np.exp(-g)) if g is not None else np.ones_like(u)
    h = (1.0 if p.get("lam") is None else p["lam"]) * r + s * z
    n, hat, rstd = norm64(h, norm_n, p.get("gamma_n"), p.get("beta_n"), eps)
    return dict(z=z, uhat=uhat, urstd=urstd, s=s, h=h, n=n, hat=hat, rstd=rstd)


def join_grad64(r, u, g, p, norm_u, norm_n, dh, dn, eps=1e-5):
    f = join64(r, u, g, p, norm_u, norm_n, eps)
    dh = np.zeros_like(r) if dh is None else dh
    dn = np.zeros_like(r) if dn is None else dn
    t = dh + norm_grad64(dn, norm_n, f["hat"], f["rstd"], p.get("gamma_n"))
    dz = t * f["s"]
    lam = p.get("lam")
    return {"dr": t * (1.0 if lam is None else lam), "dg": dz * f["z"] * (1.0 - f["s"]), "du": norm_grad64(dz, norm_u, f["uhat"], f["urstd"], p.get("gamma_u")),
            "d_lam": None if lam is None else (t * r).sum(0) if lam.size > 1 or r.shape[1] == 1 else np.array([(t * r).sum()]),
            "d_gamma_u": (dz * f["uhat"]).sum(0), "d_beta_u": dz.sum(0), "d_gamma_n": (dn * f["hat"]).sum(0), "d_beta_n": dn.sum(0)}
