"""The operators around a program's own model, as a list of measurable cases: the embedding and its gradient, the join of a
block (norm, gate and scaled residual, with the norm in front of the next block), and activations kept in 8 bits for the backward pass.

Kinds of case, each one call (or the pair that is used together) of `paper_2604_07239_amd.Fade`:
  embed         tokens -> scaled rows of a table
  embed-grad    the table's gradient from the gradient of those rows
  join          h = lam * r + sigma(g) * norm(u) and n = norm(h)
  join-grad     its gradients, from the operands as they were, or from 8-bit checkpoints of them
  join-train    both, with the operands kept in 8 bits in between
  checkpoint    activations to 8 bits and back
  weight-grad   a matrix's gradient from its input's checkpoint and its output's gradient

A token that is none of the table's (padding) reads zeros and adds to no row.
"""
import math

import torch

own = False
_ctx = None

F32, BF16 = torch.float32, torch.bfloat16
TYPES = {"f32": F32, "bf16": BF16}
TOKENS = {"u8": torch.uint8, "i32": torch.int32, "i64": torch.int64}
EPS = 1e-5


def listed():
    return [
        # the next byte of 16 streams into an fp32 model: nothing but latency
        dict(name="embed-bytes-b16", kind="embed", n=16, V=256, C=32, token="u8", table="f32", out="f32"),
        # a batch of word pieces, vocabulary and width of no round size
        dict(name="embed-pieces", kind="embed", n=20011, V=50021, C=1000, token="i32", table="f32", out="bf16"),
        # bytes of 1024 streams, 256 of each: a small table in which every row is hit a thousand times, the blank far more often
        dict(name="embed-grad-bytes", kind="embed-grad", n=262144, V=256, C=64, token="u8", dy="f32", accumulate=False),
        # a large vocabulary of which a batch meets a part: the dense gradient is most of it
        dict(name="embed-grad-pieces", kind="embed-grad", n=32768, V=65536, C=2048, token="i64", dy="bf16", accumulate=False),
        # one token of a served model through one block's end
        dict(name="join-one-row", kind="join", rows=1, C=1024, stream="bf16", branch="bf16", norm_u="layer", norm_n="layer", gate=True, lam="vector"),
        # the ends of the blocks of a training batch: an fp32 residual stream, bf16 branches
        dict(name="join-rows", kind="join", rows=16384, C=2048, stream="f32", branch="bf16", norm_u="layer", norm_n="layer", gate=True, lam="scalar"),
        # an odd width in fp32, no gate: the plain norm after and before
        dict(name="join-grad-odd", kind="join-grad", rows=1500, C=777, stream="f32", branch="f32", norm_u="rms", norm_n="rms", gate=False, lam="vector",
             kept=False),
        # backward through a block's end of that batch from the operands themselves
        dict(name="join-grad-rows", kind="join-grad", rows=16384, C=2048, stream="bf16", branch="bf16", norm_u="layer", norm_n="layer", gate=True,
             lam="vector", kept=False),
        # forward and backward with nothing but 8-bit checkpoints in between, at a wide model
        dict(name="join-train-wide", kind="join-train", rows=8192, C=4096, stream="bf16", branch="bf16", norm_u="rms", norm_n="rms", gate=True,
             lam="scalar", kept=True),
        # a batch's activations kept and read back
        dict(name="checkpoint-rows", kind="checkpoint", rows=16384, C=4096, dtype="bf16"),
        # weight gradient of a small fp32 model on a ragged batch
        dict(name="weight-grad-odd", kind="weight-grad", rows=1500, K=512, N=1000, dy="f32", accumulate=False),
        # weight gradient of a wide bf16 model on a large batch
        dict(name="weight-grad-rows", kind="weight-grad", rows=16384, K=4096, N=2048, dy="bf16", accumulate=False),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high):
    """Most widths of models are multiples of 64; one in three here is any number."""
    w = _log_int(rng, low, high)
    return w if rng.random() < 0.34 else max(64, (w + 32) // 64 * 64)


def draw(rng):
    kind = rng.choice(["embed", "embed-grad", "embed-grad", "join", "join-grad", "join-train", "checkpoint", "weight-grad", "weight-grad"])
    if kind in ("embed", "embed-grad"):
        token = rng.choice(["u8", "i32", "i64"])
        C = _width(rng, 32, 4096)
        c = dict(kind=kind, n=_log_int(rng, 1, min(262144, (1 << 25) // C)), V=256 if token == "u8" else _log_int(rng, 256, min(131072, (1 << 27) // C)), C=C,
                 token=token)
        if kind == "embed":
            return dict(c, table=rng.choice(["f32", "bf16"]), out=rng.choice(["f32", "bf16"]))
        return dict(c, dy=rng.choice(["f32", "bf16"]), accumulate=rng.random() < 0.5)
    if kind == "checkpoint":
        C = _width(rng, 16, 8192)
        return dict(kind=kind, rows=_log_int(rng, 1, (1 << 26) // C), C=C, dtype=rng.choice(["f32", "bf16"]))
    if kind == "weight-grad":
        K, N = _width(rng, 32, 4096), _width(rng, 32, 4096)
        return dict(kind=kind, rows=_log_int(rng, 1, min(65536, (1 << 36) // (K * N))), K=K, N=N, dy=rng.choice(["f32", "bf16"]), accumulate=rng.random() < 0.5)
    stream, branch = rng.choice([("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
    C = _width(rng, 32, 8192)
    c = dict(kind=kind, rows=_log_int(rng, 1, (1 << 24) // C), C=C, stream=stream, branch=branch, norm_u=rng.choice(["none", "layer", "rms"]),
             norm_n=rng.choice(["layer", "rms"]), gate=rng.random() < 0.6, lam=rng.choice(["one", "scalar", "vector"]))
    if kind != "join":
        c["kept"] = kind == "join-train" or rng.random() < 0.5
    return c


def _groups(C):
    return (C + 31) // 32


def _keep(x):
    """The 8-bit checkpoint of x [rows][C]: signed bytes [rows][32 G], then one exponent byte for each group of 32 columns [rows][G]."""
    rows, C = x.shape
    G = _groups(C)
    v = torch.zeros((rows, G, 32), device=x.device)
    v.view(rows, G * 32)[:, :C] = x.float()
    top = v.abs().amax(2)
    bits = top.view(torch.int32)
    # least e with top <= 127 * 2^e: 127 is 1.984375 * 2^6
    e = ((bits >> 23) - 6 + ((bits & 0x7FFFFF) > 0x7E0000).int()).clamp(min=1)
    q = torch.round(v * ((254 - e) << 23).view(F32)[:, :, None]).to(torch.int8)
    return torch.cat([q.view(torch.uint8).reshape(-1), e.to(torch.uint8).reshape(-1)])


def _kept(keep, rows, C):
    """The values a checkpoint stands for, in 32 bits."""
    G = _groups(C)
    q = keep[:rows * G * 32].view(torch.int8).view(rows, G, 32).float()
    e = keep[rows * G * 32:].int().view(rows, G, 1)
    return (q * (e << 23).view(F32)).view(rows, G * 32)[:, :C]


def _tokens(case, g):
    # frequencies fall with the rank as in a text: the first tokens are met again and again; two in a hundred are padding
    u = torch.rand(case["n"], device="cuda", generator=g, dtype=torch.float64)
    t = torch.clamp(torch.exp(u * math.log(case["V"] + 1)).long() - 1, 0, case["V"] - 1)
    if case["token"] != "u8":
        t[torch.rand(case["n"], device="cuda", generator=g) < 0.02] = -1
    return t.to(TOKENS[case["token"]])


def prepare(case, seed):
    kind = case["kind"]
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0, dtype=F32):
        return (torch.randn(shape, device="cuda", generator=g) * std + mean).to(dtype)

    def empty(*shape, dtype=F32):
        return torch.empty(shape, device="cuda", dtype=dtype)

    s = dict(case=case)
    if kind in ("embed", "embed-grad"):
        n, V, C = case["n"], case["V"], case["C"]
        s["tokens"], s["scale"] = _tokens(case, g), math.sqrt(C)
        if kind == "embed":
            s["table"] = normal(V, C, std=0.02, dtype=TYPES[case["table"]])
            s["out"] = empty(n, C, dtype=TYPES[case["out"]])
        else:
            s["dy"] = normal(n, C, std=1e-2, dtype=TYPES[case["dy"]])
            s["grad"] = normal(V, C, std=1e-2) if case["accumulate"] else empty(V, C)
            # what the sums are added to: a pass leaves the buffer as it found it, so that it can be repeated
            s["before"] = s["grad"].clone() if case["accumulate"] else None
        return s
    rows = case["rows"]
    if kind == "checkpoint":
        C, t = case["C"], TYPES[case["dtype"]]
        # channels of very different size, as activations have them
        s["x"] = (normal(rows, C) * torch.exp(normal(C))).to(t)
        s["keep"] = empty(rows * _groups(C) * 33, dtype=torch.uint8)
        s["out"] = empty(rows, C, dtype=t)
        return s
    if kind == "weight-grad":
        K, N = case["K"], case["N"]
        s["keep"] = _keep(normal(rows, K) * torch.exp(0.5 * normal(K)))
        s["dy"] = normal(rows, N, std=1e-2, dtype=TYPES[case["dy"]])
        s["grad"] = normal(K, N, std=1e-1) if case["accumulate"] else empty(K, N)
        s["before"] = s["grad"].clone() if case["accumulate"] else None
        return s
    C, st, br = case["C"], TYPES[case["stream"]], TYPES[case["branch"]]
    s["r"] = normal(rows, C, std=2.0, mean=0.1, dtype=st)
    s["u"] = normal(rows, C, std=0.7, mean=0.2, dtype=br)
    s["g"] = normal(rows, C, dtype=br) if case["gate"] else None
    s["lam"] = None if case["lam"] == "one" else normal(1 if case["lam"] == "scalar" else C, std=0.1, mean=0.9)
    for norm, of in (("norm_u", "u"), ("norm_n", "n")):
        s["gamma_" + of] = normal(C, std=0.2, mean=1.0) if case[norm] != "none" else None
        s["beta_" + of] = normal(C, std=0.1) if case[norm] == "layer" else None
    if kind != "join-grad":
        s["h"], s["n"] = empty(rows, C, dtype=st), empty(rows, C, dtype=br)
    if kind != "join":
        s["dh"], s["dn"] = normal(rows, C, std=1e-2, dtype=st), normal(rows, C, std=1e-2, dtype=br)
        s["dr"], s["du"] = empty(rows, C, dtype=st), empty(rows, C, dtype=br)
        s["dg"] = empty(rows, C, dtype=br) if case["gate"] else None
        for k in ("lam", "gamma_u", "beta_u", "gamma_n", "beta_n"):
            s["d_" + k] = None if s[k] is None else torch.empty_like(s[k])
        if kind == "join-train":
            for k in ("r", "u", "g"):
                s["keep_" + k] = empty(rows * _groups(C) * 33, dtype=torch.uint8) if s[k] is not None else None
        elif case["kept"]:
            for k in ("r", "u", "g"):
                s["keep_" + k] = _keep(s[k]) if s[k] is not None else None
                s[k] = None  # nothing else is left of them
    return s


def _norm(x, kind, gamma, beta):
    """(norm(x), normalised x, 1 / sigma)"""
    if kind == "none":
        return x, x, None
    c = x - x.mean(1, keepdim=True) if kind == "layer" else x
    rstd = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
    hat = c * rstd
    y = hat * gamma
    return (y if beta is None else y + beta), hat, rstd


def _norm_grad(dy, kind, hat, rstd, gamma):
    if kind == "none":
        return dy
    d = dy * gamma
    a = d - hat * (d * hat).mean(1, keepdim=True)
    if kind == "layer":
        a = a - d.mean(1, keepdim=True)
    return a * rstd


def _join_parts(case, r, u, g, s):
    z, uhat, urstd = _norm(u, case["norm_u"], s["gamma_u"], s["beta_u"])
    sg = 1.0 / (1.0 + torch.exp(-g)) if g is not None else None
    h = (r if s["lam"] is None else s["lam"] * r) + (z if sg is None else sg * z)
    return z, uhat, urstd, sg, h


def _join_grad(case, r, u, g, s):
    z, uhat, urstd, sg, h = _join_parts(case, r, u, g, s)
    _, hat, rstd = _norm(h, case["norm_n"], s["gamma_n"], s["beta_n"])
    dn = s["dn"].float()
    t = s["dh"].float() + _norm_grad(dn, case["norm_n"], hat, rstd, s["gamma_n"])
    dz = t if sg is None else t * sg
    out = {"dr": (t if s["lam"] is None else s["lam"] * t).to(TYPES[case["stream"]]),
           "du": _norm_grad(dz, case["norm_u"], uhat, urstd, s["gamma_u"]).to(TYPES[case["branch"]]), "d_gamma_n": (dn * hat).sum(0)}
    if sg is not None:
        out["dg"] = (t * z * sg * (1.0 - sg)).to(TYPES[case["branch"]])
    if s["lam"] is not None:
        out["d_lam"] = (t * r).sum(0) if case["lam"] == "vector" else (t * r).sum().reshape(1)
    if s["beta_n"] is not None:
        out["d_beta_n"] = dn.sum(0)
    if s["gamma_u"] is not None:
        out["d_gamma_u"] = (dz * uhat).sum(0)
    if s["beta_u"] is not None:
        out["d_beta_u"] = dz.sum(0)
    return out


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind in ("embed", "embed-grad"):
        t = s["tokens"].long()
        inside = (t >= 0) & (t < case["V"])
        t = torch.where(inside, t, torch.zeros_like(t))
        if kind == "embed":
            return (s["table"][t].float() * s["scale"] * inside[:, None]).to(TYPES[case["out"]])
        grad = torch.zeros((case["V"], case["C"]), device="cuda")
        grad.index_add_(0, t, s["dy"].float() * inside[:, None])
        grad *= s["scale"]
        return grad if s["before"] is None else grad.add_(s["before"])
    if kind == "checkpoint":
        return _kept(_keep(s["x"]), case["rows"], case["C"]).to(TYPES[case["dtype"]])
    if kind == "weight-grad":
        grad = _kept(s["keep"], case["rows"], case["K"]).t() @ s["dy"].float()
        return grad if s["before"] is None else grad.add_(s["before"])
    if kind == "join-grad":
        if case["kept"]:
            r, u, g = (_kept(s["keep_" + k], case["rows"], case["C"]) if s["keep_" + k] is not None else None for k in ("r", "u", "g"))
        else:
            r, u, g = (s[k].float() if s[k] is not None else None for k in ("r", "u", "g"))
        return _join_grad(case, r, u, g, s)
    r, u, g = (s[k].float() if s[k] is not None else None for k in ("r", "u", "g"))
    h = _join_parts(case, r, u, g, s)[4]
    out = {"h": h.to(TYPES[case["stream"]]), "n": _norm(h, case["norm_n"], s["gamma_n"], s["beta_n"])[0].to(TYPES[case["branch"]])}
    if kind == "join-train":
        r, u, g = (_kept(_keep(s[k]), case["rows"], case["C"]) if s[k] is not None else None for k in ("r", "u", "g"))
        out |= _join_grad(case, r, u, g, s)
    return out


def _context():
    """A program keeps one context, on the stream of its other work (1 is HIP's name for the default one, where torch works); these calls
    need no weights in it."""
    global _ctx
    if _ctx is None:
        import paper_2604_07239_amd as fade
        _ctx = fade.Fade(fade.make_config(16, 32, 16, 128, dtype=fade.F32, hip_stream=1))
    return _ctx


def _work_of(s, nbytes):
    """The workspace a call asks for, allocated once and kept beside the state's other buffers."""
    w = s.get("work")
    if w is None:
        w = s["work"] = torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")
    return w


def _own(s):
    case, ctx = s["case"], _context()
    kind = case["kind"]
    if kind == "embed":
        ctx.embed(s["tokens"], s["table"], s["out"], scale=s["scale"])
        return s["out"]
    if kind == "embed-grad":
        work = s.get("work")
        if work is None:
            work = _work_of(s, ctx.embed_grad_work(case["n"], case["V"], case["C"]))
        if s["before"] is not None:
            s["grad"].copy_(s["before"])
        ctx.embed_grad(s["tokens"], s["dy"], s["grad"], work, scale=s["scale"], accumulate=case["accumulate"])
        return s["grad"]
    if kind == "checkpoint":
        ctx.checkpoint(s["x"], s["keep"])
        ctx.checkpoint_read(s["keep"], s["out"])
        return s["out"]
    if kind == "weight-grad":
        work = s.get("work")
        if work is None:
            work = _work_of(s, ctx.checkpoint_weight_grad_work(case["rows"], case["K"], case["N"]))
        if s["before"] is not None:
            s["grad"].copy_(s["before"])
        ctx.checkpoint_weight_grad(s["keep"], s["dy"], s["grad"], work, accumulate=case["accumulate"])
        return s["grad"]
    model = dict(norm_u=case["norm_u"], norm_n=case["norm_n"], eps=EPS, lam=s["lam"], gamma_u=s["gamma_u"], beta_u=s["beta_u"], gamma_n=s["gamma_n"],
                 beta_n=s["beta_n"])
    out = {}
    if kind != "join-grad":
        kept = {k: s[k] for k in ("keep_r", "keep_u", "keep_g")} if kind == "join-train" else {}
        ctx.join(s["h"], s["n"], r=s["r"], u=s["u"], g=s["g"], **kept, **model)
        out = {"h": s["h"], "n": s["n"]}
    if kind != "join":
        work = s.get("work")
        if work is None:
            work = _work_of(s, ctx.join_grad_work(case["rows"], case["C"]))
        kept = {k: s[k] for k in ("keep_r", "keep_u", "keep_g")} if case["kept"] else {k: s[k] for k in ("r", "u", "g")}
        grads = {k: s[k] for k in ("dr", "du", "dg", "d_lam", "d_gamma_u", "d_beta_u", "d_gamma_n", "d_beta_n")}
        ctx.join_grad(s["dh"], s["dn"], work, **kept, **grads, **model)
        out |= {k: v for k, v in grads.items() if v is not None}
    return out


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    kind = case["kind"]
    size = {"f32": 4, "bf16": 2, "u8": 1, "i32": 4, "i64": 8}
    if kind in ("embed", "embed-grad"):
        n, V, C = case["n"], case["V"], case["C"]
        met = min(n, V)
        if kind == "embed":
            return {"bytes": n * size[case["token"]] + C * (met * size[case["table"]] + n * size[case["out"]]), "flops": n * C}
        # written whole, or, added to what is there, read and written
        return {"bytes": n * size[case["token"]] + n * C * size[case["dy"]] + V * C * (8 if case["accumulate"] else 4), "flops": n * C}
    rows = case["rows"]
    if kind == "checkpoint":
        C = case["C"]
        return {"bytes": rows * (2 * C * size[case["dtype"]] + 2 * 33 * _groups(C)), "flops": 4 * rows * C}
    if kind == "weight-grad":
        K, N = case["K"], case["N"]
        return {"bytes": rows * (33 * _groups(K) + N * size[case["dy"]]) + K * N * (8 if case["accumulate"] else 4), "flops": 2 * rows * K * N}
    C, st, br = case["C"], size[case["stream"]], size[case["branch"]]
    inputs = [st, br] + ([br] if case["gate"] else [])
    total = flops = 0
    if kind != "join-grad":
        total += rows * C * (sum(inputs) + st + br)
        flops += 30 * rows * C
        if kind == "join-train":
            total += len(inputs) * rows * 33 * _groups(C)
    if kind != "join":
        total += len(inputs) * rows * 33 * _groups(C) if case["kept"] else rows * C * sum(inputs)
        total += rows * C * (st + br + sum(inputs))
        flops += 60 * rows * C
    return {"bytes": total, "flops": flops}


def _norm64(x, kind, gamma, beta):
    """Value and the map from the value's gradient to (x's gradient, gamma's, beta's), from the definition."""
    if kind == "none":
        return x, lambda d: (d, None, None)
    C = x.shape[1]
    mu = x.sum(1, keepdim=True) / C if kind == "layer" else torch.zeros_like(x[:, :1])
    var = torch.square(x - mu).sum(1, keepdim=True) / C
    sigma = torch.sqrt(var + EPS)
    hat = (x - mu) / sigma

    def back(d):
        e = d * gamma
        along = (e * hat).sum(1, keepdim=True) / C
        level = e.sum(1, keepdim=True) / C if kind == "layer" else 0.0
        return (e - level - hat * along) / sigma, (d * hat).sum(0), d.sum(0)

    return hat * gamma + (0.0 if beta is None else beta), back


def _value64(keep, rows, C):
    G = _groups(C)
    q = keep[:rows * G * 32].reshape(rows, G, 32).to(torch.float64)
    q = torch.where(q >= 128, q - 256, q)
    e = keep[rows * G * 32:].reshape(rows, G, 1).to(torch.float64) - 127
    return torch.reshape(q * torch.exp2(e), (rows, G * 32))[:, :C]


def _rounded64(x):
    """What is left of x in 8 bits, by the definition: groups of 32 columns, each to whole multiples of the least power of two that
    reaches its largest value in 127 of them."""
    rows, C = x.shape
    out = torch.empty((rows, C), dtype=torch.float64, device=x.device)
    for c in range(0, C, 32):
        v = x[:, c:c + 32].to(torch.float64)
        top = v.abs().amax(1, keepdim=True)
        e = torch.ceil(torch.log2(torch.clamp(top, min=2.0 ** -130) / 127))
        e = torch.where(top > 127 * torch.exp2(e), e + 1, e)
        e = torch.where(top <= 127 * torch.exp2(e - 1), e - 1, e)
        unit = torch.exp2(torch.clamp(e, min=-126))
        out[:, c:c + 32] = torch.round(v / unit) * unit
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("embed", "embed-grad"):
        t = s["tokens"].to(torch.int64)
        at = torch.nonzero((t >= 0) & (t < case["V"])).flatten()
        if kind == "embed":
            out = torch.zeros((case["n"], case["C"]), dtype=torch.float64, device="cuda")
            out[at] = s["table"].to(torch.float64)[t[at]] * s["scale"]
            return out
        out = torch.zeros((case["V"], case["C"]), dtype=torch.float64, device="cuda")
        out.index_add_(0, t[at], s["dy"][at].to(torch.float64), alpha=s["scale"])
        return out if s["before"] is None else out + s["before"]
    if kind == "checkpoint":
        return _rounded64(s["x"])
    if kind == "weight-grad":
        x = _value64(s["keep"], case["rows"], case["K"])
        out = torch.mm(x.t().contiguous(), s["dy"].to(torch.float64))
        return out if s["before"] is None else out + s["before"]
    p = {k: None if s[k] is None else s[k].to(torch.float64) for k in ("lam", "gamma_u", "beta_u", "gamma_n", "beta_n")}

    def forward(r, u, g):
        z, back_u = _norm64(u, case["norm_u"], p["gamma_u"], p["beta_u"])
        gate = torch.ones_like(u) if g is None else torch.sigmoid(g)
        h = r * (1.0 if p["lam"] is None else p["lam"]) + gate * z
        n, back_n = _norm64(h, case["norm_n"], p["gamma_n"], p["beta_n"])
        return h, n, z, gate, back_u, back_n

    out = {}
    if kind != "join-grad":
        h, n = forward(*(None if s[k] is None else s[k].to(torch.float64) for k in ("r", "u", "g")))[:2]
        out = {"h": h, "n": n}
    if kind != "join":
        if kind == "join-train":
            r, u, g = (None if s[k] is None else _rounded64(s[k]) for k in ("r", "u", "g"))
        elif case["kept"]:
            r, u, g = (None if s["keep_" + k] is None else _value64(s["keep_" + k], case["rows"], case["C"]) for k in ("r", "u", "g"))
        else:
            r, u, g = (None if s[k] is None else s[k].to(torch.float64) for k in ("r", "u", "g"))
        _, _, z, gate, back_u, back_n = forward(r, u, g)
        through, d_gamma_n, d_beta_n = back_n(s["dn"].to(torch.float64))
        t = s["dh"].to(torch.float64) + through
        du, d_gamma_u, d_beta_u = back_u(gate * t)
        out |= {"dr": t * (1.0 if p["lam"] is None else p["lam"]), "du": du}
        if g is not None:
            out["dg"] = t * z * gate * (1.0 - gate)
        if case["lam"] != "one":
            out["d_lam"] = (t * r).sum(0) if case["lam"] == "vector" else (t * r).sum().reshape(1)
        for k, v in (("gamma_u", d_gamma_u), ("beta_u", d_beta_u), ("gamma_n", d_gamma_n), ("beta_n", d_beta_n)):
            if p[k] is not None:
                out["d_" + k] = v
    return out
