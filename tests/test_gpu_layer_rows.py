"""RecomputeLayer on windows of wider tensors: the values are a contiguous copy's bit for bit wherever it takes them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,packed", [(None, False), ("layer", False), ("rms", True), (None, True)])
def test_windows_of_wider_tensors(kind, packed):
    from paper_2502_02406_amd.blockloop import Norm, RecomputeLayer
    Sq, Skv, E, Hq, Hkv, D = 64, 512, 256, 4, 2, 64
    g = torch.Generator().manual_seed(6)
    rnd = lambda *s, std=1.0: (torch.randn(s, generator=g) * std).bfloat16().cuda()
    wide = lambda t: torch.cat([t, torch.full_like(t[..., :16], float("nan"))], -1)[..., :E]
    x, y, wq, wkv, d_o = rnd(1, Sq, E), rnd(1, Skv, E), rnd(Hq * D, E, std=E ** -0.5), rnd(2 * Hkv * D, E, std=E ** -0.5), rnd(1, Hq, Sq, D)
    norms = [Norm(rnd(E)) for _ in range(2)] if kind else []
    results = []
    for f in (lambda t: t, wide):
        layer = RecomputeLayer(1, Sq, Skv, E, Hq, Hkv, D, torch.bfloat16, 2, norm=kind, packed=packed)
        o, lse = layer.forward(f(x), f(y), wq, wkv, *norms)
        out = [o.clone(), lse.clone()]
        layer.dx.fill_(7.0)
        layer.dy.fill_(7.0)
        if not packed and f is wide:
            for a, b in ((wide(x), y), (x, wide(y))):
                with pytest.raises(ValueError):
                    layer.backward(a, b, wq, wkv, o, lse, d_o, *norms)
            assert (layer.dx == 7.0).all() and (layer.dy == 7.0).all()
        else:
            keep = (None, None) if packed else (x, y)
            out += [t.clone() for t in layer.backward(*keep, wq, wkv, o, lse, d_o, *norms) if t is not None]
        results.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*results)) and (not packed or len(results[0]) == len(results[1]))


def test_one_token_out_of_a_wider_tensor():
    """A single token's stride says nothing: contiguous as torch counts, and taken by both passes."""
    from paper_2502_02406_amd.blockloop import RecomputeLayer
    Skv, E, Hq, Hkv, D = 128, 256, 4, 2, 64
    g = torch.Generator().manual_seed(7)
    rnd = lambda *s, std=1.0: (torch.randn(s, generator=g) * std).bfloat16().cuda()
    x, y, wq, wkv, d_o = rnd(1, 9, E + 8)[:, 4:5, :E], rnd(1, Skv, E), rnd(Hq * D, E, std=0.06), rnd(2 * Hkv * D, E, std=0.06), rnd(1, Hq, 1, D)
    layer = RecomputeLayer(1, 1, Skv, E, Hq, Hkv, D, torch.bfloat16)
    results = []
    for t in (x, x.clone(memory_format=torch.contiguous_format).view(1, 1, E)):
        o, lse = layer.forward(t, y, wq, wkv)
        o, lse = o.clone(), lse.clone()
        results.append([o, lse] + [r.clone() for r in layer.backward(t, y, wq, wkv, o, lse, d_o)])
    assert all(torch.equal(a, b) for a, b in zip(*results))
