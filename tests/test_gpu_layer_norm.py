"""The operators around the layer as a training step uses them, together: the norms of the token features before the projections, their
8-bit checkpoint, and the loss at the end (RecomputeLayer with norm and packed, LossHead), against float64."""
import numpy as np
import pytest
import torch

from paper_2502_02406_amd import binding as B
from paper_2502_02406_amd import workloads as W

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def norm64(x, gamma, beta, kind):
    mu = x.mean(-1, keepdim=True) if kind == "layer" else 0.0
    y = (x - mu) / torch.sqrt(((x - mu) ** 2).mean(-1, keepdim=True) + EPS) * gamma
    return y if beta is None else y + beta


def unpacked(p):
    x = torch.empty(p.shape, dtype=torch.float32, device="cuda")
    B.lvx_unpack(p, x)
    return x.double().cpu()


class Step:
    """One training step: h = x + attention(norm(x), norm(y)), loss = cross entropy of norm(h), and all gradients."""

    def __init__(self, dtype, kind, packed, n_blocks, Sq=96, Skv=512, Hq=4, Hkv=2, D=64, V=777, seed=0):
        from paper_2502_02406_amd.blockloop import LossHead, Norm, RecomputeLayer
        E = Hq * D
        self.E, self.V, self.Sq, self.kind, self.packed = E, V, Sq, kind, packed
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *s, std=1.0: (torch.randn(s, generator=g) * std).to(DT[dtype]).cuda()
        self.x, self.y = rnd(1, Sq, E), rnd(1, Skv, E, std=2.0)
        self.wq, self.wkv, self.w = rnd(Hq * D, E, std=E ** -0.5), rnd(2 * Hkv * D, E, std=E ** -0.5), rnd(V, E, std=E ** -0.5)
        self.norms = [Norm((1.0 + rnd(E, std=0.2)).to(DT[dtype]), rnd(E, std=0.2) if kind == "layer" else None) for _ in range(3)]
        self.labels = torch.randint(V, (Sq,), generator=g).cuda()
        self.labels[::5] = -100
        self.d_loss = torch.full((Sq,), 1.0 / int((self.labels >= 0).sum()), device="cuda")
        self.layer = RecomputeLayer(1, Sq, Skv, E, Hq, Hkv, D, DT[dtype], n_blocks, norm=kind, packed=packed, eps=EPS)
        self.head = LossHead(Sq, E, V, DT[dtype], norm=kind, packed=packed, eps=EPS)
        self.dims = (Sq, Skv, Hq, Hkv, D)

    def run(self):
        nx, ny, nh = self.norms
        o, lse = self.layer.forward(self.x, self.y, self.wq, self.wkv, nx, ny)
        self.kv = self.layer.k.clone(), self.layer.v.clone()
        self.h = (self.x + o.transpose(1, 2).reshape(self.x.shape)).contiguous()
        loss = self.head.forward(self.h, self.w, self.labels, nh)
        dh, dw, *dnh = self.head.backward(None if self.packed else self.h, self.w, self.labels, self.d_loss, nh)
        d_o = dh.view(1, self.Sq, o.shape[1], o.shape[3]).transpose(1, 2).contiguous()
        keep = (None, None) if self.packed else (self.x, self.y)
        dx, dy, dwq, dwkv, *dn = self.layer.backward(*keep, self.wq, self.wkv, o, lse, d_o, nx, ny)
        names = ("loss", "dh", "dw", "dgh", "dbh", "dx", "dy", "dwq", "dwkv", "dgx", "dbx", "dgy", "dby")
        return {n: t for n, t in zip(names, (loss, dh, dw, *dnh, dx, dy, dwq, dwkv, *dn)) if t is not None}

    def reference(self):
        """float64 autograd of the definitions.  What is packed is a leaf of its own, with the values that it stands for (the rounding is
        passed over); h likewise."""
        Sq, Skv, Hq, Hkv, D = self.dims
        d64 = lambda t: t.double().cpu()
        leaf = lambda t: t.clone().requires_grad_(True)
        x, y = (leaf(unpacked(f.packed) if self.packed else d64(t)[0]) for f, t in ((self.layer.fx, self.x), (self.layer.fy, self.y)))
        wq, wkv, w = leaf(d64(self.wq)), leaf(d64(self.wkv)), leaf(d64(self.w))
        gb = [(leaf(d64(n.gamma)), leaf(d64(n.beta)) if n.beta is not None else None) for n in self.norms]
        q = (norm64(x, *gb[0], self.kind) @ wq.T).view(Sq, Hq, D).transpose(0, 1)
        kv = (norm64(y, *gb[1], self.kind) @ wkv.T).view(Skv, 2, Hkv, D)
        k, v = (kv[:, i].transpose(0, 1).repeat_interleave(Hq // Hkv, 0) for i in (0, 1))
        o = torch.softmax(q @ k.transpose(1, 2) / D ** 0.5, -1) @ v
        h0 = d64(self.x)[0] + o.transpose(0, 1).reshape(Sq, self.E)
        h = leaf(unpacked(self.head.f.packed) if self.packed else h0.detach())
        z = norm64(h, *gb[2], self.kind) @ w.T
        lab = self.labels.cpu()
        on = lab >= 0
        loss = torch.where(on, torch.logsumexp(z, 1) - z.gather(1, lab.clamp(min=0)[:, None])[:, 0], 0.0)
        (loss * d64(self.d_loss)).sum().backward()
        (h0 * h.grad).sum().backward()
        out = dict(loss=loss.detach(), dh=h.grad, dw=w.grad, dx=x.grad, dy=y.grad, dwq=wq.grad, dwkv=wkv.grad)
        for name, (g, b) in zip(("x", "y", "h"), gb):
            out["dg" + name] = g.grad
            if b is not None:
                out["db" + name] = b.grad
        return out


@pytest.mark.parametrize("dtype,kind,packed,n_blocks", [("f32", "layer", False, 2), ("f32", "rms", True, 1), ("f32", "layer", True, 4),
                                                        ("bf16", "layer", False, 1), ("bf16", "rms", True, 2), ("bf16", "layer", True, 4)])
def test_step_against_autograd(dtype, kind, packed, n_blocks):
    """float32: sums of up to 777 terms at every stage, a few 2^-24 sqrt(777) of a result's size each, some ten stages: 1e-5 of it, with
    room 1e-4.  bf16: every stage rounds to 2^-8 of a value at most, 2^-9 on average, and ten stages one behind the other
    give 1e-2 of a result's size; the layer's own tests take 2e-2 and so does this one, 3e-2 behind both layer and head."""
    # (bf16 projections need E % 256 == 0 on the matrix cores)
    s = Step(dtype, kind, packed, n_blocks, seed=n_blocks)
    got, ref = s.run(), s.reference()
    torch.cuda.synchronize()
    assert set(got) == set(ref)
    for name, t in got.items():
        r = ref[name].reshape(t.shape).numpy()
        g = t.double().cpu().numpy()
        assert np.isfinite(g).all(), name
        err = np.linalg.norm(g - r) / np.linalg.norm(r)
        assert err <= (1e-4 if dtype == "f32" else 3e-2), f"{name}: {err}"


@pytest.mark.parametrize("kind", [None, "layer", "rms"])
def test_what_is_made_again_is_what_was_used(kind):
    """K, V of the backward pass, from the packed tokens alone, are the forward pass's bit for bit."""
    from paper_2502_02406_amd.blockloop import Norm, RecomputeLayer
    Sq, Skv, E, Hq, Hkv, D = 70, 300, 256, 4, 2, 128
    inp = W.projection_inputs(1, Skv, E, 2 * Hkv * D, "bf16", seed=3)
    y, wkv = inp["x"].cuda(), inp["w"].cuda()
    inp = W.projection_inputs(1, Sq, E, Hq * D, "bf16", seed=4)
    x, wq = inp["x"].cuda(), inp["w"].cuda()
    norm = Norm(torch.full((E,), 1.25, dtype=x.dtype, device="cuda"), torch.full((E,), 0.5, dtype=x.dtype, device="cuda")) if kind else None
    layer = RecomputeLayer(1, Sq, Skv, E, Hq, Hkv, D, torch.bfloat16, norm=kind, packed=True)
    args = (norm, norm) if kind else ()
    o, lse = layer.forward(x, y, wq, wkv, *args)
    o, lse, q, k, v = o.clone(), lse.clone(), layer.q.clone(), layer.k.clone(), layer.v.clone()
    for t in (layer.q, layer.k, layer.v):
        t.fill_(7.0)
    out = layer.backward(None, None, wq, wkv, o, lse, torch.ones_like(o), *args)
    assert torch.equal(layer.q, q) and torch.equal(layer.k, k) and torch.equal(layer.v, v)
    assert len(out) == (4 if kind is None else 8) and all(t.isfinite().all() for t in out)
    # without packing, the values that the checkpoint stands for as inputs: the same results
    plain = RecomputeLayer(1, Sq, Skv, E, Hq, Hkv, D, torch.bfloat16, norm=kind)
    ux, uy = unpacked(layer.fx.packed).to(x.dtype).cuda().view(x.shape), unpacked(layer.fy.packed).to(x.dtype).cuda().view(y.shape)
    o2, lse2 = plain.forward(ux, uy, wq, wkv, *args)
    assert torch.equal(o2, o) and torch.equal(lse2, lse)
    for a, b in zip(plain.backward(ux, uy, wq, wkv, o2, lse2, torch.ones_like(o2), *args), out):
        assert torch.equal(a, b)


def test_refusals():
    from paper_2502_02406_amd.blockloop import LossHead, Norm, RecomputeLayer
    x = torch.zeros((1, 64, 256), dtype=torch.bfloat16, device="cuda")
    w = torch.zeros((256, 256), dtype=torch.bfloat16, device="cuda")
    norm = Norm(torch.ones(256, dtype=torch.bfloat16, device="cuda"))
    layer = RecomputeLayer(1, 64, 64, 256, 2, 1, 128, torch.bfloat16, norm="layer")
    with pytest.raises(ValueError):
        layer.forward(x, x, w, w)                                # no weights for the norm
    with pytest.raises(ValueError):
        layer.backward(None, None, w, w, None, None, None, norm, norm)       # nothing was packed
    with pytest.raises(ValueError):
        RecomputeLayer(1, 64, 64, 256, 2, 1, 128, torch.bfloat16, norm="batch")
    with pytest.raises(ValueError):
        RecomputeLayer(1, 64, 64, 256, 2, 1, 128, torch.bfloat16).forward(x, x, w, w, norm, norm)
    head = LossHead(64, 256, 300, torch.bfloat16)
    labels = torch.zeros(64, dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError):
        head.forward(x[:, :32], torch.zeros((300, 256), dtype=torch.bfloat16, device="cuda"), labels)
    with pytest.raises(ValueError):
        head.backward(None, torch.zeros((300, 256), dtype=torch.bfloat16, device="cuda"), labels, torch.zeros(64, device="cuda"))
    with pytest.raises(B.LvxError):
        LossHead(64, 100, 300, torch.bfloat16)


def test_step_replays_from_a_graph():
    s = Step("bf16", "layer", True, 2, seed=9)
    want = {n: t.clone() for n, t in s.run().items()}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = s.run()
    for i in range(3):
        for t in got.values():
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n, t in got.items():
            assert torch.equal(t, want[n]), f"replay {i}: {n}"
        again = s.run()                                          # eager work between the replays
        assert all(torch.equal(again[n], want[n]) for n in want)


@pytest.mark.parametrize("kind,packed", [("layer", True), ("rms", False), (None, True)])
def test_two_batches_are_two_layers(kind, packed):
    """float32, the bound of test_step_against_autograd on either side: each batch's results are a layer's of its own, and the weights' gradients
    add up."""
    from paper_2502_02406_amd.blockloop import Norm, RecomputeLayer
    Sq, Skv, E, Hq, Hkv, D = 40, 130, 96, 3, 1, 64
    g = torch.Generator().manual_seed(21)
    rnd = lambda *s, std=1.0: (torch.randn(s, generator=g) * std).cuda()
    x, y, wq, wkv, d_o = rnd(2, Sq, E), rnd(2, Skv, E), rnd(Hq * D, E, std=E ** -0.5), rnd(2 * Hkv * D, E, std=E ** -0.5), rnd(2, Hq, Sq, D)
    norms = [Norm(1.0 + rnd(E, std=0.2), rnd(E, std=0.2) if kind == "layer" else None) for _ in range(2)] if kind else []

    def run(b, e):
        layer = RecomputeLayer(e - b, Sq, Skv, E, Hq, Hkv, D, torch.float32, norm=kind, packed=packed)
        xb, yb = x[b:e].contiguous(), y[b:e].contiguous()
        o, lse = layer.forward(xb, yb, wq, wkv, *norms)
        keep = (None, None) if packed else (xb, yb)
        return [o.clone(), lse.clone()] + [t if t is None else t.clone() for t in layer.backward(*keep, wq, wkv, o, lse, d_o[b:e].contiguous(), *norms)]

    both, one, two = run(0, 2), run(0, 1), run(1, 2)
    torch.cuda.synchronize()
    for i, (t, a, b) in enumerate(zip(both, one, two)):
        if t is None:
            assert a is None and b is None
            continue
        r = (torch.cat([a, b]) if i < 4 else a + b).double()
        assert t.shape == r.shape and torch.linalg.norm(t.double() - r) <= 2e-4 * torch.linalg.norm(r), i
