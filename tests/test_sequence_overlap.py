"""A preference loss refuses to write over what it still reads (no GPU needed: every call here ends before anything is launched)."""
import ctypes as C

import pytest

from paper_2502_02406_amd import binding as B
from test_abi import FAKE, lib  # noqa: F401

FAR = 1 << 16


def call(lib, **kw):  # noqa: F811
    p = B.lvx_pref(100, 4, 0, 0.1, 0.0)
    at = {k: FAKE + i * FAR for i, k in enumerate(("nll", "ref", "labels", "first", "loss", "margin", "d_loss", "d_nll"))}
    at.update({k: None if v is None else at["d_loss"] + v for k, v in kw.items()})
    return lib.lvx_preference(C.byref(p), *at.values(), FAKE + 64 * FAR, 1 << 40, None)


@pytest.mark.parametrize("name", ["loss", "margin"])
@pytest.mark.parametrize("by", [0, 4, 12, -4, -12])
def test_losses_and_margins_where_d_loss_lies(lib, name, by):  # noqa: F811
    assert call(lib, **{name: by}) == -4
    assert call(lib, **{name: by, "margin" if name == "loss" else "loss": 16}) == -4       # (one beside it is none)
