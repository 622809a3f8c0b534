"""Host-side checks of the distillation that need no GPU: refusals before anything is launched and workspaces."""
import ctypes as C
import random

import pytest
import torch

from paper_2502_02406_amd import binding as B
from test_abi import FAKE, lib  # noqa: F401


def prob(**kw):
    p = B.lvx_distil(100, 1000, 256, 16, 256, 2.0)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def fwd(lib, p, dtype=B.LVX_BF16, x=FAKE, w=FAKE, ids=FAKE, teacher=FAKE, td=B.LVX_F32, loss=FAKE, lse=FAKE, ln_p=FAKE, ws=FAKE, n=1 << 40):
    return lib.lvx_distil_fwd(C.byref(p) if p is not None else None, dtype, x, w, ids, teacher, td, loss, lse, ln_p, ws, n, None)


def bwd(lib, p, dtype=B.LVX_BF16, x=FAKE, w=FAKE, ids=FAKE, teacher=FAKE, td=B.LVX_F32, lse=FAKE, ln_p=FAKE, d=FAKE, dx=FAKE * 2, dw=FAKE, ws=FAKE, n=1 << 40):
    return lib.lvx_distil_bwd(C.byref(p) if p is not None else None, dtype, x, w, ids, teacher, td, lse, ln_p, d, dx, dw, ws, n, None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_shared_refusals(lib, call):  # noqa: F811
    assert call(lib, None) == -1
    for name in ("x", "w", "ids", "teacher", "lse", "ln_p"):
        assert call(lib, prob(), **{name: None}) == -1, name
    assert call(lib, prob(n=0)) == -2 and call(lib, prob(V=0)) == -2 and call(lib, prob(E=0)) == -2 and call(lib, prob(K=0)) == -2
    assert call(lib, prob(K=1025)) == -7 and call(lib, prob(E=200)) == -7
    for T in (0.0, -1.0, float("nan"), float("inf"), 1e-45, 4e-39):
        assert call(lib, prob(temperature=T)) == -2, T
    assert call(lib, prob(), dtype=4) == -3 and call(lib, prob(), td=2) == -3
    assert call(lib, prob(x_ss=255)) == -4 and call(lib, prob(x_ss=260)) == -4 and call(lib, prob(n=1 << 20, x_ss=4096)) == -4
    assert call(lib, prob(), x=FAKE + 8) == -4 and call(lib, prob(), w=FAKE + 8) == -4 and call(lib, prob(), ids=FAKE + 4) == -4
    for name in ("teacher", "lse", "ln_p"):
        assert call(lib, prob(), **{name: FAKE + 2}) == -4, name
    assert call(lib, prob(), td=B.LVX_BF16, teacher=FAKE + 1) == -4
    assert call(lib, prob(), ws=None) == -6 and call(lib, prob(), ws=FAKE + 16) == -6 and call(lib, prob(), n=4096) == -6


def test_own_refusals(lib):  # noqa: F811
    assert fwd(lib, prob(), loss=None) == -1
    assert bwd(lib, prob(), d=None) == -1 and bwd(lib, prob(), dx=None, dw=None) == -1
    assert bwd(lib, prob(), dx=FAKE) == -4 and bwd(lib, prob(), dx=FAKE * 2 + 8) == -4 and bwd(lib, prob(), dw=FAKE + 8) == -4


@pytest.mark.parametrize("dtype", [B.LVX_BF16, B.LVX_F32])
def test_more_never_takes_less(lib, dtype):  # noqa: F811
    size, rng = B.lvx_distil_workspace_bytes, random.Random(1)
    assert size(0, 64, 9, 1, dtype) == 0 and size(9, 64, 9, 0, dtype) == 0 and size(9, 64, 9, 1025, dtype) == 0 and size(9, 64, 9, 1, 7) == 0
    assert size(9, 64, 9, 1, dtype) % 256 == 0 and size(9, 64, 9, 1, dtype) > B.lvx_xent_workspace_bytes(9, 64, 9, dtype)
    log = lambda top: int(round(2.0 ** rng.uniform(0.0, top)))
    for _ in range(20000):
        n, E, V, K = log(17), 64 * log(7), log(19), log(10)
        n2, E2, V2, K2 = (rng.choice((k, max(1, k - rng.randrange(300)), max(1, k // rng.choice((2, 3, 7))), rng.randint(1, k))) for k in (n, E // 64, V, K))
        assert size(n2, 64 * E2, V2, K2, dtype) <= size(n, E, V, K, dtype), ((n2, 64 * E2, V2, K2), (n, E, V, K))


def test_binding_checks():
    x, w, ids, f, ws = torch.zeros(4, 64), torch.zeros(9, 64), torch.zeros(4, 3, dtype=torch.int64), torch.zeros(4), torch.zeros(9)
    t = torch.zeros(4, 3)
    good = dict(x=x, w=w, ids=ids, teacher=t, ln_p=t, per_token=(f,), workspace=ws, temperature=2.0)
    s = B._distil_struct("t", **good)
    assert (s.n, s.V, s.E, s.K, s.x_ss, s.temperature) == (4, 9, 64, 3, 64, 2.0)
    for bad in (dict(w=w[:, :32]), dict(w=w.bfloat16()), dict(ids=ids.int()), dict(ids=ids[:3]), dict(ids=ids[:, :2]), dict(ids=ids.flatten()), dict(teacher=t[:, :2]),
                dict(teacher=torch.zeros(3, 4).t()), dict(ln_p=t.double()), dict(per_token=(f, f[:3])), dict(workspace=torch.zeros(4, 4).t())):
        with pytest.raises(ValueError):
            B._distil_struct("t", **{**good, **bad})
    with pytest.raises(RuntimeError):
        B.lvx_distil_fwd(x, w, ids, t, f, f, t, ws)
    with pytest.raises(ValueError):
        B.lvx_distil_bwd(x, w, ids, t, f, t, f, workspace=ws)
