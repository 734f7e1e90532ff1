"""The operators as a program with its own model uses them: together, on the program's stream, captured into graphs, and around the coder."""
import numpy as np
import pytest

from gpu_helpers import need_gpu
from operator_helpers import U, context, f64, join64, join_grad64, keep64

pytestmark = pytest.mark.gpu


class _Block:
    """Embedding, one block (two products and a gate), its join, a head: a byte model of a program's own, its products torch's, fp32."""

    def __init__(self, torch, c, n, C, seed):
        self.torch, self.c, self.n, self.C = torch, c, n, C
        gen = torch.Generator(device="cuda").manual_seed(seed)
        mk = lambda *s, std=0.2: torch.randn(s, device="cuda", generator=gen) * std  # noqa: E731
        self.w = {"E": mk(256, C), "W": mk(C, C), "G": mk(C, C), "H": mk(C, 256), "lam": 1 + mk(C), "gamma_u": 1 + mk(C), "beta_u": mk(C), "gamma_n": 1 + mk(C), "beta_n": mk(C)}
        self.grad = {k: torch.zeros_like(v) for k, v in self.w.items()}
        e = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
        b = lambda k: torch.empty(k, dtype=torch.uint8, device="cuda")  # noqa: E731
        self.x, self.h, self.y, self.dx, self.du, self.dg = (e(n, C) for _ in range(6))
        self.keep = {k: b(c.checkpoint_nbytes(n, C)) for k in ("r", "u", "g", "n")}
        self.work = b(max(c.embed_grad_work(n, 256, C), c.join_grad_work(n, C), c.checkpoint_weight_grad_work(n, C, C), c.checkpoint_weight_grad_work(n, C, 256)))

    def model(self):
        return {k: self.w[k] for k in ("lam", "gamma_u", "beta_u", "gamma_n", "beta_n")}

    def forward(self, tokens):
        c, w = self.c, self.w
        c.embed(tokens, w["E"], self.x, scale=2.0)
        u, g = self.x @ w["W"], self.x @ w["G"]
        c.join(self.h, self.y, r=self.x, u=u, g=g, **{"keep_" + k: v for k, v in self.keep.items()}, **self.model())
        return self.torch.softmax(self.y @ w["H"], 1)

    def backward(self, tokens, dlogits):
        """All gradients, with nothing of the forward pass left but its checkpoints."""
        c, w, d = self.c, self.w, self.grad
        dy = dlogits @ w["H"].t()
        c.checkpoint_weight_grad(self.keep["n"], dlogits, d["H"], self.work)
        c.join_grad(None, dy, self.work, **{"keep_" + k: self.keep[k] for k in "rug"}, **self.model(), dr=self.dx, du=self.du, dg=self.dg,
                    **{"d_" + k: d[k] for k in ("lam", "gamma_u", "beta_u", "gamma_n", "beta_n")})
        c.checkpoint_weight_grad(self.keep["r"], self.du, d["W"], self.work)  # r is the products' input too
        c.checkpoint_weight_grad(self.keep["r"], self.dg, d["G"], self.work)
        dx = self.dx + self.du @ w["W"].t() + self.dg @ w["G"].t()
        c.embed_grad(tokens, dx, d["E"], self.work, scale=2.0)
        return d


def test_a_training_step_from_checkpoints():
    torch = need_gpu()
    n, C = 700, 96
    s = torch.cuda.Stream()
    c = context(s.cuda_stream)
    with torch.cuda.stream(s):
        m = _Block(torch, c, n, C, 1)
        rng = np.random.default_rng(2)
        tokens = torch.from_numpy(rng.integers(0, 200, n, dtype=np.uint8)).cuda()
        target = torch.from_numpy(rng.integers(0, 256, n)).cuda()
        probs = m.forward(tokens)
        dlogits = (probs - torch.nn.functional.one_hot(target, 256).float()) / n
        d = {k: f64(v) for k, v in m.backward(tokens, dlogits).items()}
    s.synchronize()
    # the same in 64 bits; every operand that the backward pass takes is what its checkpoint stands for
    w = {k: f64(v) for k, v in m.w.items()}
    t = tokens.cpu().numpy()
    x = w["E"][t] * 2.0
    u, g = x @ w["W"], x @ w["G"]
    f = join64(x, u, g, w, "layer", "layer")
    kept = {k: keep64(v.astype(np.float32).astype(np.float64))[2] for k, v in (("r", x), ("u", u), ("g", g), ("n", f["n"]))}
    dl = f64(dlogits)
    dy = dl @ w["H"].T
    j = join_grad64(kept["r"], kept["u"], kept["g"], w, "layer", "layer", None, dy)
    want = {"H": kept["n"].T @ dl, "W": kept["r"].T @ j["du"], "G": kept["r"].T @ j["dg"], **{k: j["d_" + k] for k in ("lam", "gamma_u", "beta_u", "gamma_n", "beta_n")}}
    dx = j["dr"] + j["du"] @ w["W"].T + j["dg"] @ w["G"].T
    want["E"] = np.zeros((256, C))
    np.add.at(want["E"], t, 2.0 * dx)
    # fp32 throughout, but a value near a border of its checkpoint's steps may round the other way: 1e-5 of them (fp32 error 1e-6 over a step of 1/100) by
    # a step of 1 / 127 of their group's largest value, as a norm sqrt(1e-5) / 127 = 2.5e-5 beside fp32's own 1e-6; four times that
    for k, v in want.items():
        assert np.linalg.norm(d[k] - v) <= 1e-4 * np.linalg.norm(v), k
    # and the gradient without checkpoints is near: an operand in 8 bits is off by 1 / 254 of its group's largest value at most
    j = join_grad64(x, u, g, w, "layer", "layer", None, dy)
    assert np.linalg.norm(d["W"] - x.T @ j["du"]) <= 0.05 * np.linalg.norm(d["W"])
    c.close()


def test_two_programs_train_alike_to_the_bit():
    """What an adapting codec needs: the decoder's model repeats the encoder's steps, so a payload coded with its tables decodes."""
    torch = need_gpu()
    n, C, lr = 64, 64, 0.5
    data = np.random.default_rng(1).integers(97, 101, (12, n), dtype=np.uint8)

    def models():
        c = context()
        m = _Block(torch, c, n, C, 7)
        freq = torch.zeros((n, 256), dtype=torch.int16, device="cuda")
        return c, m, freq

    def step(c, m, freq, prev):  # tables of the next byte of n streams
        probs = m.forward(prev)
        c.quantize(probs, freq)
        return probs

    def learn(m, prev, probs, target):
        dlogits = (probs - torch.nn.functional.one_hot(target.long(), 256).float()) / n
        torch.cuda.synchronize()
        for k, v in m.backward(prev, dlogits).items():
            m.w[k] -= lr * v
        torch.cuda.synchronize()

    c, m, freq = models()
    tables, prev = [], torch.zeros(n, dtype=torch.uint8, device="cuda")
    for row in data:
        torch.cuda.synchronize()
        probs = step(c, m, freq, prev)
        tables.append(freq.clone())
        target = torch.from_numpy(row).cuda()
        learn(m, prev, probs, target)
        prev = target
    cap = 4 * len(data) + 16
    out, ln = torch.zeros((n, cap), dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    c.coder_encode_tables(torch.stack(tables), torch.from_numpy(data).cuda(), len(data), n, out, cap, ln)
    c.close()
    # the decoder has the payload and its own copy of the model: it learns from what it decodes and has to arrive at the same tables
    c, m, freq = models()
    prev, mine = torch.zeros(n, dtype=torch.uint8, device="cuda"), []
    back = torch.zeros((len(data), n), dtype=torch.uint8, device="cuda")
    for i, row in enumerate(data):
        torch.cuda.synchronize()
        probs = step(c, m, freq, prev)
        mine.append(freq.clone())
        assert torch.equal(mine[i], tables[i]), i
        c.coder_decode_tables(torch.stack(mine), i + 1, n, out, cap, ln, back[:i + 1])
        target = back[i].clone()
        learn(m, prev, probs, target)
        prev = target
    np.testing.assert_array_equal(back.cpu().numpy(), data)
    c.close()


def test_calls_wait_for_the_stream_they_are_given():
    """Operands that another kernel of the same stream has yet to write."""
    torch = need_gpu()
    s = torch.cuda.Stream()
    c = context(s.cuda_stream)
    x = torch.zeros((300, 512), device="cuda")
    keep, y = torch.zeros(c.checkpoint_nbytes(300, 512), dtype=torch.uint8, device="cuda"), torch.zeros((300, 512), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(50_000_000)
        x.fill_(2.0)
        c.checkpoint(x, keep)
        c.checkpoint_read(keep, y)
        assert not s.query()  # nothing waited for
        z = y + 1
    s.synchronize()
    assert (z == 3.0).all()
    c.close()


def test_captured_calls_replay_as_they_ran():
    torch = need_gpu()
    n, C, V = 3000, 200, 5000
    s = torch.cuda.Stream()
    c = context(s.cuda_stream)
    rng = np.random.default_rng(3)
    with torch.cuda.stream(s):
        tokens = torch.from_numpy(rng.integers(0, V, n)).cuda()
        table, g, dh, dn = (torch.randn(k, C, device="cuda") for k in (V, n, n, n))
        gamma = torch.rand(C, device="cuda") + 0.5
        bufs = {k: torch.empty((n, C), device="cuda") for k in ("x", "h", "n", "dr", "du", "dg")}
        grad, dw, dgamma = torch.empty((V, C), device="cuda"), torch.empty((C, C), device="cuda"), torch.empty(C, device="cuda")
        keep = [torch.empty(c.checkpoint_nbytes(n, C), dtype=torch.uint8, device="cuda") for _ in range(4)]
        work = [torch.empty(k, dtype=torch.uint8, device="cuda") for k in (c.embed_grad_work(n, V, C), c.join_grad_work(n, C), c.checkpoint_weight_grad_work(n, C, C))]

        def all_of_it():
            c.embed(tokens, table, bufs["x"])
            c.join(bufs["h"], bufs["n"], r=bufs["x"], u=bufs["x"], g=g, gamma_u=gamma, keep_r=keep[0], keep_u=keep[1], keep_g=keep[2], keep_n=keep[3])
            c.join_grad(dh, dn, work[1], keep_r=keep[0], keep_u=keep[1], keep_g=keep[2], gamma_u=gamma, dr=bufs["dr"], du=bufs["du"], dg=bufs["dg"], d_gamma_u=dgamma)
            c.checkpoint_weight_grad(keep[3], bufs["du"], dw, work[2])
            c.embed_grad(tokens, bufs["dr"], grad, work[0])

        results = lambda: [t.clone() for t in (*bufs.values(), grad, dw, dgamma, *keep)]  # noqa: E731
        graph = torch.cuda.CUDAGraph()
        s.synchronize()
        with torch.cuda.graph(graph, stream=s):
            all_of_it()
        for i in range(4):  # new inputs every time, eager work and waits in between
            tokens.copy_(torch.from_numpy(rng.integers(0, V, n)))
            dh.normal_()
            g.normal_()
            all_of_it()
            want = results()
            s.synchronize()
            for t in (*bufs.values(), grad, dw, dgamma, *keep, *work):
                t.fill_(0)
            graph.replay()
            got = results()
            s.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, got)), i
    c.close()


def test_two_graphs_with_workspaces_of_their_own_run_side_by_side():
    """Two programs on two streams, captured, replayed together many times: what each computes is what it computes alone."""
    torch = need_gpu()
    n, C, V = 5000, 264, 900
    rng = np.random.default_rng(6)
    programs = []
    for k in range(2):
        s = torch.cuda.Stream()
        c = context(s.cuda_stream)
        with torch.cuda.stream(s):
            tokens = torch.from_numpy(rng.integers(0, V, n).astype(np.int32)).cuda()
            d, u = torch.randn((n, C), device="cuda"), torch.randn((n, C), device="cuda")
            gamma, keep = torch.rand(C, device="cuda") + 0.5, torch.empty(c.checkpoint_nbytes(n, C), dtype=torch.uint8, device="cuda")
            grad, dw, du, dgamma = torch.empty((V, C), device="cuda"), torch.empty((C, C), device="cuda"), torch.empty((n, C), device="cuda"), torch.empty(C, device="cuda")
            work = [torch.empty(b, dtype=torch.uint8, device="cuda") for b in (c.embed_grad_work(n, V, C), c.join_grad_work(n, C), c.checkpoint_weight_grad_work(n, C, C))]

        def calls(c=c, tokens=tokens, d=d, u=u, gamma=gamma, keep=keep, grad=grad, dw=dw, du=du, dgamma=dgamma, work=work):
            c.checkpoint(u, keep)
            c.join_grad(d, d, work[1], r=u, u=u, gamma_u=gamma, du=du, d_gamma_u=dgamma)
            c.checkpoint_weight_grad(keep, du, dw, work[2])
            c.embed_grad(tokens, du, grad, work[0])

        s.synchronize()
        with torch.cuda.stream(s):
            calls()
        s.synchronize()
        want = [t.clone() for t in (grad, dw, du, dgamma)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            calls()
        programs.append((s, c, graph, (grad, dw, du, dgamma), want))
    torch.cuda.synchronize()
    for _ in range(20):
        for s, _, graph, _, _ in programs:
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for _, c, _, got, want in programs:
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        c.close()


def test_a_context_on_the_default_stream():
    """hip_stream 1 is HIP's name for the default stream: calls and a program's other work there follow one another without waits."""
    torch = need_gpu()
    c = context(1)
    x, keep = torch.zeros((300, 512), device="cuda"), torch.zeros(context(1).checkpoint_nbytes(300, 512), dtype=torch.uint8, device="cuda")
    y = torch.zeros_like(x)
    for i in range(20):
        x.fill_(float(i))
        c.checkpoint(x, keep)
        c.checkpoint_read(keep, y)
        x.fill_(-1.0)
        assert (y == float(i)).all()
    c.close()


def test_the_current_device_and_errors_are_left_alone():
    torch = need_gpu()
    import paper_2604_07239_amd as fa
    c = context()
    x = torch.zeros((2, 8), device="cuda")
    with pytest.raises(fa.FadeError):
        c.embed(torch.zeros(3, dtype=torch.int32, device="cuda"), x, x)
    assert torch.cuda.current_device() == 0
    c.checkpoint(x, torch.zeros(c.checkpoint_nbytes(2, 8), dtype=torch.uint8, device="cuda"))  # the context goes on
    torch.cuda.synchronize()
    c.close()


def test_rows_past_two_to_the_31st_element():
    """Offsets of more than 32 bits: 2^21 + 5 rows of 1040 columns with a row pitch of 2080 (bf16, 8.7 GB): the last rows are right."""
    torch = need_gpu()
    rows, C, ld = (1 << 21) + 5, 1040, 2080
    c = context()
    flat = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    x = flat.view(rows, ld)[:, :C]
    x.fill_(1.0)
    x[-5:] = torch.randn((5, C), device="cuda").bfloat16()
    keep = torch.empty(c.checkpoint_nbytes(rows, C), dtype=torch.uint8, device="cuda")
    c.checkpoint(x, keep)
    tail = x[-5:].clone()
    torch.cuda.synchronize()
    c.checkpoint_read(keep, x)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(f64(x[-5:]), keep64(f64(tail))[2])
    # a join over them, in place, without norms: h = r + u
    x.fill_(1.0)
    torch.cuda.synchronize()
    c.join(x, None, r=x, u=torch.ones((rows, C), dtype=torch.bfloat16, device="cuda"), norm_u="none", norm_n="none")
    torch.cuda.synchronize()
    assert (x[-5:] == 2.0).all() and (x[:5] == 2.0).all() and (x[rows // 2] == 2.0).all()
    # and the last rows of a table
    del keep
    table = flat[:(1 << 20) * ld].view(1 << 20, ld)
    table[-1] = 3.0
    out = torch.empty((4, ld), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    c.embed(torch.full((4,), (1 << 20) - 1, dtype=torch.int32, device="cuda"), table, out)
    torch.cuda.synchronize()
    assert (out == 3.0).all()
    c.close()


def test_sums_are_fp32():
    """Two to the 24th tokens of one row: a running fp32 sum of ones stops at 2^24, sums of pieces do not."""
    torch = need_gpu()
    n = (1 << 24) + 4096
    c = context()
    t, d = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.ones((n, 4), dtype=torch.bfloat16, device="cuda")
    grad, work = torch.empty((2, 4), device="cuda"), torch.empty(c.embed_grad_work(n, 2, 4), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    c.embed_grad(t, d, grad, work)
    torch.cuda.synchronize()
    assert (grad[0] == n).all() and (grad[1] == 0).all()
    assert U * 2 ** 24 == 1.0
    c.close()
