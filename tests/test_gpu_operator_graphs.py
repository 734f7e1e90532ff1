"""Graphs of the operators at the sizes where a launch needs more than 64 KB of LDS, or sorts in several passes: two programs captured on two streams, replayed side by side over new
inputs into cleared outputs, with eager work in between."""
import pytest

from gpu_helpers import need_gpu
from operator_helpers import context

pytestmark = pytest.mark.gpu


class _Program:
    def __init__(self, torch, seed, n, V, C, rows, K, N, dtype):
        self.torch, self.s = torch, torch.cuda.Stream()
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        c = self.c = context(self.s.cuda_stream)
        mk = lambda *s, t=dtype: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
        b = lambda k: mk(k, t=torch.uint8)  # noqa: E731
        self.tokens, self.V = mk(n, t=torch.int32), V
        self.inputs = {"d": mk(n, C), "r": mk(rows, K), "u": mk(rows, K), "g": mk(rows, K), "dh": mk(rows, K), "dn": mk(rows, K), "dy": mk(rows, N)}
        self.p = {k: torch.rand(K, device="cuda", generator=self.gen) + 0.5 for k in ("lam", "gamma_u", "beta_u", "gamma_n", "beta_n")}
        self.out = {"table": mk(V, C, t=torch.float32), "h": mk(rows, K), "n": mk(rows, K), "dr": mk(rows, K), "du": mk(rows, K), "dg": mk(rows, K), "dw": mk(K, N, t=torch.float32)}
        self.out.update({"d_" + k: mk(K, t=torch.float32) for k in self.p})
        self.keep = [b(c.checkpoint_nbytes(rows, K)) for _ in range(4)]
        self.work = [b(c.embed_grad_work(n, V, C)), b(c.join_grad_work(rows, K)), b(c.checkpoint_weight_grad_work(rows, K, N))]

    def calls(self):
        c, i, o, k = self.c, self.inputs, self.out, self.keep
        c.embed_grad(self.tokens, i["d"], o["table"], self.work[0])
        c.join(o["h"], o["n"], r=i["r"], u=i["u"], g=i["g"], keep_r=k[0], keep_u=k[1], keep_g=k[2], keep_n=k[3], **self.p)
        c.join_grad(i["dh"], i["dn"], self.work[1], keep_r=k[0], keep_u=k[1], keep_g=k[2], **self.p, **{x: o[x] for x in o if x[0] == "d" and x != "dw"})
        c.checkpoint_weight_grad(k[3], i["dy"], o["dw"], self.work[2])

    def renew(self):
        self.tokens.random_(-1, self.V, generator=self.gen)
        for x in self.inputs.values():
            x.normal_(generator=self.gen)

    def clear(self):
        for x in (*self.out.values(), *self.keep, *self.work):
            x.fill_(99)

    def results(self):
        return {k: v.clone() for k, v in (*self.out.items(), *enumerate(self.keep))}


def test_two_programs_side_by_side():
    torch = need_gpu()
    programs = [_Program(torch, 1, 20000, 3000, 264, 3001, 2050, 2056, torch.float32), _Program(torch, 2, 9000, 40000, 40, 517, 5000, 4090, torch.bfloat16)]
    torch.cuda.synchronize()
    for p in programs:
        with torch.cuda.stream(p.s):
            p.renew()
            p.calls()
        p.s.synchronize()
        p.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(p.graph, stream=p.s):
            p.calls()
    for i in range(4):
        for p in programs:
            with torch.cuda.stream(p.s):
                p.renew()
                p.calls()
                p.want = p.results()
                p.clear()
        torch.cuda.synchronize()
        for p in programs:
            with torch.cuda.stream(p.s):
                p.graph.replay()
        for p in programs:
            with torch.cuda.stream(p.s):
                got = p.results()
            p.s.synchronize()
            for k, want in p.want.items():
                assert torch.equal(got[k], want), (i, k)
                assert not bool((want == 99).all()), k
    for p in programs:
        p.c.close()
