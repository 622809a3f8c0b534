"""Host-side checks of the embedding lookup that need no GPU: refusals before anything is launched and workspaces."""
import ctypes as C
import random

import pytest
import torch

from paper_2502_02406_amd import binding as B
from test_abi import FAKE, lib  # noqa: F401

FAR = FAKE + (1 << 40)


def prob(**kw):
    p = B.lvx_embed(100, 1000, 256, 1.0, 256)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def fwd(lib, p, dtype=B.LVX_BF16, table=FAKE, ids=FAKE, rows=FAR):
    return lib.lvx_embed_fwd(C.byref(p) if p is not None else None, dtype, table, ids, rows, None)


def bwd(lib, p, dtype=B.LVX_BF16, table=FAKE, ids=FAKE, rows=FAR, ws=FAKE, n=1 << 40):
    return lib.lvx_embed_bwd(C.byref(p) if p is not None else None, dtype, rows, ids, table, 0, ws, n, None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_refusals(lib, call):  # noqa: F811
    assert call(lib, None) == -1
    for name in ("table", "ids", "rows"):
        assert call(lib, prob(), **{name: None}) == -1
    assert call(lib, prob(), dtype=4) == -3
    for bad in (dict(n=0), dict(V=0), dict(E=0), dict(n=1 << 29), dict(V=1 << 29), dict(E=1 << 21)):
        assert call(lib, prob(**bad)) == -2, bad
    assert call(lib, prob(y_ss=255)) == -4 and call(lib, prob(y_ss=1 << 50)) == -4
    assert call(lib, prob(), rows=FAR + 1) == -4 and call(lib, prob(), table=FAKE + 1) == -4 and call(lib, prob(), ids=FAKE + 4) == -4
    assert call(lib, prob(), dtype=B.LVX_F32, rows=FAR + 2) == -4
    # rows and table in each other: the first and the last element, a window beside it
    size = 1000 * 256 * 2
    assert call(lib, prob(), rows=FAKE) == -4 and call(lib, prob(), rows=FAKE + size - 2) == -4
    assert call(lib, prob(n=3, y_ss=10000), rows=FAKE - 2 * 20000) == -4 and call(lib, prob(n=1), rows=FAKE - 510) == -4


def test_workspace_refusals(lib):  # noqa: F811
    need = B.lvx_embed_workspace_bytes(100, 256, 1000)
    assert need > 0 and need % 256 == 0
    assert bwd(lib, prob(), ws=None) == -6 and bwd(lib, prob(), ws=FAKE + 16) == -6 and bwd(lib, prob(), n=need - 1) == -6
    assert B.lvx_embed_workspace_bytes(0, 1, 1) == 0 and B.lvx_embed_workspace_bytes(1, 0, 1) == 0 and B.lvx_embed_workspace_bytes(1, 1, 1 << 29) == 0


def test_more_never_takes_less(lib):  # noqa: F811
    size, rng = B.lvx_embed_workspace_bytes, random.Random(3)
    log = lambda top: int(round(2.0 ** rng.uniform(0.0, top)))
    for _ in range(20000):
        n, E, V = log(20), log(14), log(20)
        n2, E2, V2 = (rng.choice((k, max(1, k - rng.randrange(300)), max(1, k // rng.choice((2, 3, 7))), rng.randint(1, k))) for k in (n, E, V))
        assert size(n2, E2, V2) <= size(n, E, V), ((n2, E2, V2), (n, E, V))


def test_binding_checks():
    table, ids, y = torch.zeros(9, 64), torch.zeros(4, dtype=torch.int64), torch.zeros(4, 64)
    p = B._embed_struct("t", table, ids, y, 0.5)
    assert (p.n, p.V, p.E, p.scale, p.y_ss) == (4, 9, 64, 0.5, 64)
    p = B._embed_struct("t", table, ids, torch.zeros(4, 80)[:, 8:72], 1.0)
    assert p.y_ss == 80
    for bad in (dict(table=table[:, :32]), dict(table=table.bfloat16()), dict(table=table.t()), dict(ids=ids.int()), dict(ids=ids[:3]),
                dict(ids=torch.zeros(8, dtype=torch.int64)[::2]), dict(y=torch.zeros(64, 4).t())):
        with pytest.raises(ValueError):
            B._embed_struct("t", **{**dict(table=table, ids=ids, y=y, scale=1.0), **bad})
    with pytest.raises(RuntimeError):
        B.lvx_embed_fwd(table, ids, y)
    with pytest.raises(RuntimeError):
        B.lvx_embed_bwd(y, ids, table, torch.zeros(1))
