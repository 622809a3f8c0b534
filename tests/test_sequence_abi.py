"""Host-side checks of the losses of sequences that need no GPU: refusals before anything is launched and workspaces."""
import ctypes as C
import random

import pytest
import torch

from paper_2502_02406_amd import binding as B
from test_abi import FAKE, lib  # noqa: F401


def pref(**kw):
    p = B.lvx_pref(100, 4, 0, 0.1, 0.0)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def clip(**kw):
    p = B.lvx_clip(100, 4, 1, 0, 0.2, 0.2, 0.1)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def preference(lib, p, nll=FAKE, ref=FAKE, labels=FAKE, first=FAKE, loss=FAKE, margin=FAKE, d_loss=FAKE, d_nll=FAKE, ws=FAKE, n=1 << 40):
    return lib.lvx_preference(C.byref(p) if p is not None else None, nll, ref, labels, first, loss, margin, d_loss, d_nll, ws, n, None)


def policy(lib, p, nll=FAKE, old=FAKE, ref=FAKE, adv=FAKE, labels=FAKE, first=FAKE, loss=FAKE, stats=FAKE, d_loss=FAKE, d_nll=FAKE, ws=FAKE, n=1 << 40):
    return lib.lvx_policy(C.byref(p) if p is not None else None, nll, old, ref, adv, labels, first, loss, stats, d_loss, d_nll, ws, n, None)


@pytest.mark.parametrize("call,make", [(preference, pref), (policy, clip)])
def test_shared_refusals(lib, call, make):  # noqa: F811
    assert call(lib, None) == -1
    for name in ("nll", "labels", "first", "loss", "d_loss", "d_nll"):
        assert call(lib, make(), **{name: None}) == -1, name
    for bad in (dict(n=0), dict(S=0), dict(n=(1 << 30) + 1), dict(S=(1 << 21) + 1), dict(beta=-1.0), dict(beta=float("nan")), dict(beta=float("inf"))):
        assert call(lib, make(**bad)) == -2, bad
    for name in ("nll", "ref", "loss", "d_loss", "d_nll"):
        assert call(lib, make(), **{name: FAKE + 2}) == -4, name
    for name in ("labels", "first"):
        assert call(lib, make(), **{name: FAKE + 4}) == -4, name
    assert call(lib, make(), ws=None) == -6 and call(lib, make(), ws=FAKE + 16) == -6 and call(lib, make(), n=255) == -6


def test_own_refusals(lib):  # noqa: F811
    assert preference(lib, pref(form=3)) == -7 and preference(lib, pref(form=-1)) == -7 and preference(lib, pref(form=1, smoothing=0.1)) == -7
    assert preference(lib, pref(beta=0.0)) == -2 and preference(lib, pref(smoothing=1.5)) == -2 and preference(lib, pref(smoothing=float("nan"))) == -2
    assert preference(lib, pref(), margin=FAKE + 2) == -4
    assert policy(lib, clip(), old=None) == -1 and policy(lib, clip(), adv=None) == -1 and policy(lib, clip(), ref=None) == -1
    assert policy(lib, clip(clip_low=-0.1)) == -2 and policy(lib, clip(clip_high=float("nan"))) == -2
    assert policy(lib, clip(), stats=FAKE + 2) == -4 and policy(lib, clip(), old=FAKE + 2) == -4


@pytest.mark.parametrize("size", ["lvx_preference_workspace_bytes", "lvx_policy_workspace_bytes"])
def test_workspace(lib, size):  # noqa: F811
    size, rng = getattr(B, size), random.Random(2)
    assert size(0, 1) == 0 and size(1, 0) == 0 and size(1, 1) > 0 and size(1, 1) % 256 == 0
    for _ in range(3000):
        n, S = rng.randint(1, 1 << 20), rng.randint(1, 5000)
        assert size(rng.randint(1, n), rng.randint(1, S)) <= size(n, S)


def test_binding_checks():
    n, S = 10, 2
    f, i = torch.zeros(n), torch.zeros(n, dtype=torch.int64)
    first, one, ws = torch.arange(2 * S + 1), torch.zeros(S), torch.zeros(64)
    good = dict(where="t", tokens=(f, None), per_sequence=(one,), labels=i, first=first, d_loss=one, d_nll=f, workspace=ws, pairs=True)
    assert B._sequences(**good) == (n, S)
    for bad in (dict(labels=i.int()), dict(labels=i[::2]), dict(first=first.int()), dict(first=first.view(1, -1)), dict(first=first[:4]), dict(first=first[:1]),
                dict(d_loss=None), dict(tokens=(f[:3],)), dict(tokens=(f.double(),)), dict(per_sequence=(f,)), dict(d_nll=f[:4]),
                dict(workspace=torch.zeros(4, 4).t())):
        with pytest.raises(ValueError):
            B._sequences(**{**good, **bad})
    with pytest.raises(ValueError):
        B.lvx_preference(f, f, i, first, one)
    with pytest.raises(ValueError):
        B.lvx_policy(f, f, f, one, i, first, one)
    with pytest.raises(RuntimeError):
        B.lvx_preference(f, f, i, first, one, workspace=ws)
    with pytest.raises(RuntimeError):
        B.lvx_policy(f, f, f, one, i, first, one, workspace=ws)
