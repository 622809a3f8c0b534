"""The operators at either end of a step on two streams at once, and two captured graphs that share a workspace, replayed in turn: every result is the one
of a call by itself, bit for bit (sums have a fixed order, and nothing is kept between calls)."""
import pytest
import torch

from paper_2502_02406_amd import binding as B

pytestmark = pytest.mark.gpu


class Job:
    """Lookup, distillation, both sequence losses and all gradients, on buffers of its own (but for a workspace that it is given)."""

    def __init__(self, n, E, V, K, seed, ws=None):
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).cuda()
        f32 = lambda *s: torch.empty(s, device="cuda")
        self.S = 3
        self.w = rnd(V, E) * 0.1
        self.tokens = torch.randint(-1, V, (n,), generator=g).cuda()
        self.ids = torch.randint(-1, V, (n, K), generator=g).cuda()
        self.teacher = torch.randn((n, K), generator=g).cuda()
        self.d = torch.rand(n, generator=g).cuda()
        self.first = torch.tensor([0] + sorted(torch.randint(n, (2 * self.S - 1,), generator=g).tolist()) + [n], device="cuda")
        self.adv = torch.randn(2 * self.S, generator=g).cuda()
        self.x, self.dx, self.dw = rnd(n, E), rnd(n, E), torch.empty_like(self.w)
        self.loss, self.lse, self.ln_p = f32(n), f32(n), f32(n, K)
        self.pair, self.answer, self.d_pair, self.d_answer = f32(self.S), f32(2 * self.S), f32(n), f32(n)
        self.stats, self.ones = f32(2 * self.S, 3), torch.ones(2 * self.S, device="cuda")
        self.ws = torch.empty(self.room(n, E, V, K), dtype=torch.uint8, device="cuda") if ws is None else ws

    @staticmethod
    def room(n, E, V, K):
        return max(B.lvx_distil_workspace_bytes(n, E, V, K, B.LVX_BF16), B.lvx_embed_workspace_bytes(n, E, V), B.lvx_preference_workspace_bytes(n, 3),
                   B.lvx_policy_workspace_bytes(n, 6))

    def run(self):
        S = self.S
        B.lvx_embed_fwd(self.w, self.tokens, self.x, 2.0)
        B.lvx_distil_fwd(self.x, self.w, self.ids, self.teacher, self.loss, self.lse, self.ln_p, self.ws, 2.0)
        B.lvx_preference(self.loss, self.d, self.tokens, self.first, self.pair, None, self.ones[:S], self.d_pair, self.ws)
        B.lvx_policy(self.loss, self.loss, self.d, self.adv, self.tokens, self.first, self.answer, self.stats, self.ones, self.d_answer, self.ws, beta=0.1)
        B.lvx_distil_bwd(self.x, self.w, self.ids, self.teacher, self.lse, self.ln_p, self.d_answer, self.dx, self.dw, self.ws, 2.0)
        B.lvx_embed_bwd(self.dx, self.tokens, self.dw, self.ws, 2.0, accumulate=True)

    def results(self):
        return [self.x, self.loss, self.lse, self.ln_p, self.pair, self.answer, self.stats, self.d_pair, self.d_answer, self.dx, self.dw]

    def clear(self):
        for t in self.results():
            t.fill_(float("nan"))


SIZES = [(700, 256, 5000, 12), (40000, 64, 900, 5)]


def alone(jobs):
    want = []
    for j in jobs:
        j.run()
        torch.cuda.synchronize()
        want.append([t.clone() for t in j.results()])
        assert all(t.isfinite().all() for t in want[-1])
        j.clear()
    torch.cuda.synchronize()
    return want


def same(job, want):
    return all(torch.equal(a, b) for a, b in zip(job.results(), want))


def test_two_streams():
    jobs = [Job(*s, seed=i) for i, s in enumerate(SIZES)]
    want = alone(jobs)
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(4):
        for j, s in zip(jobs, streams):
            with torch.cuda.stream(s):
                j.run()
    torch.cuda.synchronize()
    assert all(same(j, w) for j, w in zip(jobs, want))


def test_two_graphs_with_one_workspace():
    ws = torch.empty(max(Job.room(*s) for s in SIZES), dtype=torch.uint8, device="cuda")
    jobs = [Job(*s, seed=10 + i, ws=ws) for i, s in enumerate(SIZES)]
    want = alone(jobs)
    graphs = []
    for j in jobs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            j.run()
    for i in (0, 1, 1, 0, 1, 0):
        jobs[i].clear()
        graphs[i].replay()
        torch.cuda.synchronize()
        assert same(jobs[i], want[i]), i
        jobs[1 - i].run()                                    # eager work between the replays
        torch.cuda.synchronize()
        assert same(jobs[1 - i], want[1 - i]), i
