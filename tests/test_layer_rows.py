"""Token features whose rows do not follow each other (a window of a wider tensor) in RecomputeLayer, with the library replaced by a recorder (no
GPU needed): the forward pass reads them, the backward pass writes gradients of its own layout and refuses them before it launches anything."""
import pytest
import torch

from paper_2502_02406_amd import binding as B
from paper_2502_02406_amd import blockloop
from test_blockloop import Dev, lib  # noqa: F401

E, SQ, SKV = 128, 64, 256


@pytest.fixture
def calls(lib, monkeypatch):  # noqa: F811
    out = []
    for name in ("lvx_xattn_project", "lvx_xattn_project_bwd", "lvx_xattn_fwd", "lvx_xattn_fwd_merge", "lvx_xattn_fwd_merge_last", "lvx_xattn_bwd_visit",
                 "lvx_norm_fwd", "lvx_norm_bwd", "lvx_pack", "lvx_unpack"):
        monkeypatch.setattr(B, name, lambda *a, _n=name, **k: out.append((_n, a, k)))
    monkeypatch.setattr(B, "lvx_norm_workspace_bytes", lambda n, e: 256)
    return out


def layer_of(norm, packed):
    layer = blockloop.RecomputeLayer(1, SQ, SKV, E, 4, 2, 64, torch.bfloat16, 2, device="cpu", norm=norm, packed=packed)
    layer.q = Dev(layer.q)
    return layer


def tokens(S, pad=0, longer=0):
    return torch.zeros((1, S + longer, E + pad), dtype=torch.bfloat16)[:, :S, :E]


def grads():
    return torch.zeros((1, 4, SQ, 64), dtype=torch.bfloat16), torch.zeros(1, 4, SQ), torch.zeros((1, 4, SQ, 64), dtype=torch.bfloat16)


def weights(norm):
    return () if norm is None else (blockloop.Norm(torch.ones(E, dtype=torch.bfloat16)),) * 2


@pytest.mark.parametrize("norm", [None, "layer", "rms"])
@pytest.mark.parametrize("wide", ["x", "y"])
def test_wide_rows_are_refused_before_the_backward_pass_starts(calls, norm, wide):
    layer = layer_of(norm, False)
    x, y = tokens(SQ, 8 if wide == "x" else 0), tokens(SKV, 8 if wide == "y" else 0)
    layer.forward(x, y, None, None, *weights(norm))
    assert calls                                                 # (reading them is no trouble)
    calls.clear()
    with pytest.raises(ValueError, match=f"{wide} "):
        layer.backward(x, y, None, None, *grads(), *weights(norm))
    assert not calls


@pytest.mark.parametrize("norm", [None, "layer"])
def test_packed_features_do_not_ask_how_the_tokens_lay(calls, norm):
    layer = layer_of(norm, True)
    x, y = tokens(SQ, 8), tokens(SKV, 8)
    layer.forward(x, y, None, None, *weights(norm))
    layer.backward(None, None, None, None, *grads(), *weights(norm))


@pytest.mark.parametrize("norm,packed", [(None, False), ("layer", False), (None, True), ("rms", True)])
def test_gradients_are_written_where_they_belong(calls, norm, packed):
    """dx of a block's projection is that block of dy, by address and strides (x and y out of longer tensors: a single batch's stride says nothing)."""
    layer = layer_of(norm, packed)
    x, y = tokens(SQ, longer=3), tokens(SKV, longer=5)
    layer.forward(x, y, None, None, *weights(norm))
    calls.clear()
    keep = (None, None) if packed else (x, y)
    layer.backward(*keep, None, None, *grads(), *weights(norm))
    dx = [k["dx"] for n, a, k in calls if n == "lvx_xattn_project_bwd"]
    assert len(dx) == 3
    for t, whole, first, rows in zip(dx, (layer.dy, layer.dy, layer.dx), (0, SKV // 2, 0), (SKV // 2, SKV // 2, SQ)):
        assert t.data_ptr() == whole.data_ptr() + 2 * first * E and t.shape == (1, rows, E) and t.stride()[1:] == (E, 1)


def project_bwd(x, dx):
    d_out, w = Dev(torch.zeros(x.shape[0], 2, x.shape[1], 64, dtype=torch.bfloat16)), torch.zeros(128, E, dtype=torch.bfloat16)
    B.lvx_xattn_project_bwd(Dev(x), w, [d_out], dx=Dev(dx))


def test_the_projection_compares_the_rows_of_dx_with_those_of_x(lib):  # noqa: F811
    x = torch.zeros((1, 6, E), dtype=torch.bfloat16)
    project_bwd(x, torch.zeros((1, 9, E), dtype=torch.bfloat16)[:, 2:8])       # a single batch's stride says nothing
    assert len(lib.calls) == 1
    two = torch.zeros((2, 6, E), dtype=torch.bfloat16)
    for a, b in ((x, torch.zeros((1, 6, E + 8), dtype=torch.bfloat16)[:, :, :E]), (torch.zeros((1, 6, E + 8), dtype=torch.bfloat16)[:, :, :E], x),
                 (x, x.transpose(1, 2).contiguous().transpose(1, 2)), (two, torch.zeros((2, 9, E), dtype=torch.bfloat16)[:, :6]), (x, x[:, :5])):
        with pytest.raises(AssertionError):
            project_bwd(a, b)
    assert len(lib.calls) == 1
