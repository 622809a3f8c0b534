"""The norms' gradients and the cross entropy on two streams at once, and two captured graphs that share a workspace, replayed in turn: every
result is the one of a call by itself, bit for bit (sums have a fixed order, and nothing is kept between calls)."""
import pytest
import torch

from paper_2502_02406_amd import binding as B

pytestmark = pytest.mark.gpu


class Job:
    """Norm with packing, loss, both gradients, on buffers of its own (but for a workspace that it is given)."""

    def __init__(self, n, E, V, seed, ws=None):
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).cuda()
        self.x, self.w, self.gamma, self.beta = rnd(n, E), rnd(V, E) * 0.1, rnd(E), rnd(E)
        self.labels = torch.randint(-1, V, (n,), generator=g).cuda()
        self.d = torch.rand(n, generator=g).cuda()
        self.packed = B.Packed(n, E)
        self.y, self.dy, self.dx, self.dw = torch.empty_like(self.x), torch.empty_like(self.x), torch.empty_like(self.x), torch.empty_like(self.w)
        self.stats = torch.empty((n, 2), device="cuda")
        self.loss, self.lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        self.dparam = torch.empty((2, E), device="cuda")
        self.ws = torch.empty(self.room(n, E, V), dtype=torch.uint8, device="cuda") if ws is None else ws

    @staticmethod
    def room(n, E, V):
        return max(B.lvx_xent_workspace_bytes(n, E, V, B.LVX_BF16), B.lvx_norm_workspace_bytes(n, E))

    def run(self):
        B.lvx_norm_fwd(self.x, self.gamma, self.beta, self.y, self.stats, packed=self.packed)
        B.lvx_xent_fwd(self.y, self.w, self.labels, self.loss, self.lse, self.ws)
        B.lvx_xent_bwd(self.y, self.w, self.labels, self.lse, self.d, self.dy, self.dw, self.ws)
        self.dparam.zero_()
        B.lvx_norm_bwd(None, self.gamma, self.stats, self.dy, self.dx, self.dparam[0], self.dparam[1], self.ws, packed=self.packed)

    def results(self):
        return [self.loss, self.lse, self.dx, self.dw, self.dparam, self.y]

    def clear(self):
        for t in self.results():
            t.fill_(float("nan"))


SIZES = [(700, 256, 5000), (2100, 128, 900)]


def alone(jobs):
    want = []
    for j in jobs:
        j.run()
        torch.cuda.synchronize()
        want.append([t.clone() for t in j.results()])
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
