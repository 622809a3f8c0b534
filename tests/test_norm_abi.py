"""Host-side checks of the norms and of the packed form that need no GPU: refusals before anything is launched, workspace
sizes, and the binding's own checks."""
import ctypes as C

import pytest
import torch

from paper_2502_02406_amd import binding as B
from test_abi import FAKE, lib  # noqa: F401


def norm(**kw):
    p = B.lvx_norm(100, 256, 0, 256, 256, 1e-5)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def fwd(lib, p, dtype=B.LVX_BF16, x=FAKE, packed=None, gamma=FAKE, beta=FAKE, y=FAKE, stats=FAKE):
    return lib.lvx_norm_fwd(C.byref(p) if p is not None else None, dtype, x, C.byref(packed) if packed is not None else None, gamma, beta, y,
                            stats, None)


def bwd(lib, p, dtype=B.LVX_BF16, x=FAKE, packed=None, gamma=FAKE, stats=FAKE, dy=FAKE, dx=FAKE, dgamma=FAKE, dbeta=FAKE, ws=FAKE, n=1 << 40):
    return lib.lvx_norm_bwd(C.byref(p) if p is not None else None, dtype, x, C.byref(packed) if packed is not None else None, gamma, stats, dy,
                            dx, dgamma, dbeta, ws, n, None)


def test_norm_fwd_refusals(lib):  # noqa: F811
    assert fwd(lib, None) == -1
    assert fwd(lib, norm(), x=None) == -1                        # neither x nor packed
    assert fwd(lib, norm(), packed=B.lvx_packed(FAKE, None)) == -1
    assert fwd(lib, norm(), gamma=None) == -1 and fwd(lib, norm(), y=None) == -1 and fwd(lib, norm(), stats=None) == -1
    assert fwd(lib, norm(), dtype=5) == -3
    assert fwd(lib, norm(n=0)) == -2 and fwd(lib, norm(E=0)) == -2 and fwd(lib, norm(n=1 << 31)) == -2
    assert fwd(lib, norm(eps=0.0)) == -2 and fwd(lib, norm(eps=float("nan"))) == -2
    assert fwd(lib, norm(x_ss=255)) == -4 and fwd(lib, norm(y_ss=255)) == -4
    assert fwd(lib, norm(), x=FAKE + 1) == -4 and fwd(lib, norm(), y=FAKE + 1) == -4 and fwd(lib, norm(), beta=FAKE + 1) == -4
    assert fwd(lib, norm(), dtype=B.LVX_F32, x=FAKE + 2) == -4
    assert fwd(lib, norm(), stats=FAKE + 2) == -4
    assert fwd(lib, norm(x_ss=264)) == -4                        # y is x, with other strides


def test_norm_bwd_refusals(lib):  # noqa: F811
    pk = B.lvx_packed(FAKE, FAKE)
    assert bwd(lib, None) == -1
    assert bwd(lib, norm(), x=None) == -1
    assert bwd(lib, norm(), packed=pk) == -2                     # both
    assert bwd(lib, norm(), x=None, packed=B.lvx_packed(None, FAKE)) == -1
    assert bwd(lib, norm(), dx=None, dgamma=None, dbeta=None) == -1
    assert bwd(lib, norm(), stats=None) == -1 and bwd(lib, norm(), dy=None) == -1 and bwd(lib, norm(), gamma=None) == -1
    assert bwd(lib, norm(), ws=None) == -6 and bwd(lib, norm(), ws=FAKE + 16) == -6
    assert bwd(lib, norm(), n=B.lvx_norm_workspace_bytes(100, 256) - 1) == -6
    assert bwd(lib, norm(), dx=FAKE + 1) == -4 and bwd(lib, norm(), dgamma=FAKE + 2) == -4 and bwd(lib, norm(), dbeta=FAKE + 2) == -4
    assert bwd(lib, norm(x_ss=264)) == -4 and bwd(lib, norm(y_ss=264)) == -4       # dx is dy, with other strides
    assert bwd(lib, norm(x_ss=8)) == -4 and bwd(lib, norm(n=-1)) == -2 and bwd(lib, norm(), dtype=2) == -3


def test_pack_refusals(lib):  # noqa: F811
    pk = B.lvx_packed(FAKE, FAKE)
    for f in (lambda n, E, ss, dt, x, p: lib.lvx_pack(n, E, ss, dt, x, C.byref(p) if p is not None else None, None),
              lambda n, E, ss, dt, x, p: lib.lvx_unpack(n, E, ss, dt, C.byref(p) if p is not None else None, x, None)):
        assert f(4, 64, 64, B.LVX_BF16, None, pk) == -1
        assert f(4, 64, 64, B.LVX_BF16, FAKE, None) == -1
        assert f(4, 64, 64, B.LVX_BF16, FAKE, B.lvx_packed(FAKE, None)) == -1
        assert f(4, 64, 64, 3, FAKE, pk) == -3
        assert f(0, 64, 64, B.LVX_BF16, FAKE, pk) == -2 and f(4, -1, 64, B.LVX_BF16, FAKE, pk) == -2
        assert f(4, 64, 63, B.LVX_BF16, FAKE, pk) == -4 and f(4, 64, 64, B.LVX_F32, FAKE + 2, pk) == -4


def test_norm_workspace_serves_fewer(lib):  # noqa: F811
    assert B.lvx_norm_workspace_bytes(0, 64) == 0 and B.lvx_norm_workspace_bytes(64, 0) == 0
    for E in (1, 33, 512, 1000, 1024, 1032, 2048, 4096, 4104, 8192, 9000, 16384, 20000):
        sizes = [B.lvx_norm_workspace_bytes(n, E) for n in (1, 2, 15, 16, 17, 100, 4000, 4097, 100000, 1 << 30)]
        assert sizes == sorted(sizes) and sizes[0] >= 8 * E and sizes[-1] % 256 == 0
    for n in (1, 100, 4000, 100000):
        sizes = [B.lvx_norm_workspace_bytes(n, E) for E in range(1, 20000, 37)]
        assert sizes == sorted(sizes), n


def test_binding_checks():
    x, g, y = torch.zeros(4, 64), torch.zeros(64), torch.zeros(4, 64)
    with pytest.raises(RuntimeError):                            # host tensors
        B.lvx_norm_fwd(x, g, g, y, torch.zeros(4, 2))
    with pytest.raises(RuntimeError):
        B.lvx_pack(x, B.Packed(4, 64, device="cpu"))
    with pytest.raises(ValueError):
        B.lvx_norm_fwd(None, g, g, y, torch.zeros(4, 2))
    with pytest.raises(ValueError):
        B.lvx_norm_bwd(x, g, torch.zeros(4, 2), y, packed=B.Packed(4, 64, device="cpu"))
    with pytest.raises(ValueError):
        B.lvx_norm_bwd(x, g, torch.zeros(4, 2), y)
    s = B._norm_struct("t", x, y, g, torch.zeros(4, 2), False, 1e-5)
    assert (s.n, s.E, s.x_ss, s.y_ss) == (4, 64, 64, 64)
    with pytest.raises(ValueError):
        B._norm_struct("t", x, y, g[:63], torch.zeros(4, 2), False, 1e-5)
    with pytest.raises(ValueError):
        B._norm_struct("t", x[:3], y, g, torch.zeros(4, 2), False, 1e-5)
    with pytest.raises(ValueError):
        B._norm_struct("t", x, y, g, torch.zeros(4), False, 1e-5)
    w = torch.zeros(2, 6, 96)
    assert B._token_rows(w[:, :, :64], "x") == (12, 64, 96)
    assert B._token_rows(w[:, :1, :64], "x") == (2, 64, 6 * 96)
    assert B._token_rows(w[1:, 2:5, :], "x") == (3, 96, 96)
    with pytest.raises(ValueError):
        B._token_rows(w[:, :4], "x")                             # batches that do not follow each other
    with pytest.raises(ValueError):
        B._token_rows(w.transpose(1, 2), "x")
    with pytest.raises(ValueError):
        B._token_rows(torch.zeros(5), "x")
    assert B.Packed(5, 33, device="cpu").rows(1, 3).shape == (2, 33)
