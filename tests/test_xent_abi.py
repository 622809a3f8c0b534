"""Host-side checks of the cross entropy against a vocabulary that need no GPU: refusals before anything is launched and workspaces."""
import ctypes as C

import pytest
import torch

from paper_2502_02406_amd import binding as B
from test_abi import FAKE, lib  # noqa: F401


def prob(**kw):
    p = B.lvx_xent(100, 1000, 256, 256)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def fwd(lib, p, dtype=B.LVX_BF16, x=FAKE, w=FAKE, labels=FAKE, loss=FAKE, lse=FAKE, ws=FAKE, n=1 << 40):
    return lib.lvx_xent_fwd(C.byref(p) if p is not None else None, dtype, x, w, labels, loss, lse, ws, n, None)


def bwd(lib, p, dtype=B.LVX_BF16, x=FAKE, w=FAKE, labels=FAKE, lse=FAKE, d=FAKE, dx=FAKE * 2, dw=FAKE, ws=FAKE, n=1 << 40):
    return lib.lvx_xent_bwd(C.byref(p) if p is not None else None, dtype, x, w, labels, lse, d, dx, dw, ws, n, None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_shared_refusals(lib, call):  # noqa: F811
    assert call(lib, None) == -1
    for name in ("x", "w", "labels", "lse"):
        assert call(lib, prob(), **{name: None}) == -1
    assert call(lib, prob(n=0)) == -2 and call(lib, prob(V=0)) == -2 and call(lib, prob(E=0)) == -2
    assert call(lib, prob(), dtype=4) == -3
    assert call(lib, prob(E=200)) == -7                          # E % 64 on the matrix cores
    assert call(lib, prob(x_ss=255)) == -4 and call(lib, prob(x_ss=260)) == -4
    assert call(lib, prob(n=1 << 20, x_ss=4096)) == -4           # n * x_ss past 2^31
    assert call(lib, prob(), x=FAKE + 8) == -4 and call(lib, prob(), w=FAKE + 8) == -4
    assert call(lib, prob(), labels=FAKE + 4) == -4 and call(lib, prob(), lse=FAKE + 2) == -4
    assert call(lib, prob(E=200, x_ss=201), dtype=B.LVX_F32, x=FAKE + 2) == -4
    assert call(lib, prob(), ws=None) == -6 and call(lib, prob(), ws=FAKE + 16) == -6 and call(lib, prob(), n=4096) == -6


def test_own_refusals(lib):  # noqa: F811
    assert fwd(lib, prob(), loss=None) == -1
    assert bwd(lib, prob(), d=None) == -1 and bwd(lib, prob(), dx=None, dw=None) == -1
    assert bwd(lib, prob(), dx=FAKE) == -4                       # dx is x
    assert bwd(lib, prob(), dx=FAKE * 2 + 8) == -4 and bwd(lib, prob(), dw=FAKE + 8) == -4


def test_workspace(lib):  # noqa: F811
    size = B.lvx_xent_workspace_bytes
    assert size(0, 256, 1000, B.LVX_BF16) == 0 and size(10, 200, 1000, B.LVX_BF16) == 0 and size(10, 200, 1000, 7) == 0
    assert size(10, 200, 1000, B.LVX_F32) > 0 and size(10, 256, 1000, B.LVX_BF16) % 256 == 0
    # one for more tokens, features or entries is taken for fewer (refused calls return before a launch: -6; taken ones would launch, so the
    # smallest room that a call takes is asked for through its refusal below it)
    def smallest(n, E, V, dt):
        p = prob(n=n, E=E, V=V, x_ss=E)
        el, Mp = (4 if dt == B.LVX_F32 else 2), (n + 255) // 256 * 256
        up = lambda x: (x + 255) // 256 * 256
        edge = 256 if dt == B.LVX_BF16 else 64 if n <= 64 or -(-n // 128) * -(-E // 128) * max(1, min(64, V // 256)) < 256 else 128
        rows = 128 if dt == B.LVX_BF16 and n <= 128 else edge
        tiles = -(-n // rows) * -(-E // edge)
        need = 256 + 2 * up(4 * n) + up(8 * n) + max(tiles, min(64 * tiles, 512)) * rows * edge * 4 + 320 * Mp * el   # lists, sums of dx, 256 columns and 64 between
        assert bwd(lib, p, dtype=dt, n=need - 1) == -6
        return need
    for dt in (B.LVX_BF16, B.LVX_F32):
        for n, E, V in ((2304, 4096, 256), (5000, 1024, 50000), (300, 512, 5003), (16, 64, 1)):
            room = size(n, E, V, dt)
            for n2, E2, V2 in ((n, E, V), (2048 if n > 2048 else n, E, V), (1, E, V), (n // 2, 64, V), (n, 64, 1), (n - 1, E, (V + 1) // 2)):
                assert smallest(n2, E2, V2, dt) <= room, (n2, E2, V2)


def test_binding_checks():
    x, w, lab, f, ws = torch.zeros(4, 64), torch.zeros(9, 64), torch.zeros(4, dtype=torch.int64), torch.zeros(4), torch.zeros(9)
    s = B._xent_struct("t", x, w, lab, (f, f), ws)
    assert (s.n, s.V, s.E, s.x_ss) == (4, 9, 64, 64)
    for bad in (dict(w=w[:, :32]), dict(w=w.bfloat16()), dict(labels=lab.int()), dict(labels=lab[:3]), dict(per_token=(f, f[:3])),
                dict(per_token=(f.double(),)), dict(workspace=torch.zeros(4, 4).t())):
        with pytest.raises(ValueError):
            B._xent_struct("t", **{**dict(x=x, w=w, labels=lab, per_token=(f,), workspace=ws), **bad})
    with pytest.raises(RuntimeError):
        B.lvx_xent_fwd(x, w, lab, f, f, ws)
    with pytest.raises(ValueError):
        B.lvx_xent_bwd(x, w, lab, f, f, workspace=ws)
