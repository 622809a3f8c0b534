"""The loss's gradients may not lie in what they are made from, or in each other: dw of a piece of the vocabulary is written before dx reads that
piece of w.  Refused before anything is launched (no GPU needed); what lies beside the operands is taken (tests/test_gpu_xent_apart.py)."""
import ctypes as C

import pytest

from paper_2502_02406_amd import binding as B
from test_abi import lib  # noqa: F401

N, V, E = 100, 1000, 256
X, W, DX, DW, REST = (i << 30 for i in range(1, 6))      # far apart; never dereferenced


def bwd(lib, dtype=B.LVX_BF16, x=X, w=W, dx=DX, dw=DW, x_ss=E, V=V):  # noqa: F811
    p = B.lvx_xent(N, V, E, x_ss)
    return lib.lvx_xent_bwd(C.byref(p), dtype, x, w, REST, REST + (1 << 20), REST + (2 << 20), dx, dw, REST + (1 << 28), 1 << 40, None)


@pytest.mark.parametrize("dtype,el", [(B.LVX_BF16, 2), (B.LVX_F32, 4)])
def test_gradients_in_the_operands(lib, dtype, el):  # noqa: F811
    rows, vocab, row = N * E * el, V * E * el, E * el
    assert bwd(lib, dtype, dx=X) == -4                           # dx is x
    assert bwd(lib, dtype, dw=W) == -4                           # dw is w
    assert bwd(lib, dtype, dx=W) == -4 and bwd(lib, dtype, dw=X) == -4 and bwd(lib, dtype, dx=DW) == -4
    # ... in part, from either side
    assert bwd(lib, dtype, dw=W + vocab - 16) == -4 and bwd(lib, dtype, dw=W - vocab + 16) == -4
    assert bwd(lib, dtype, dx=X + rows - 16) == -4 and bwd(lib, dtype, dx=X - rows + 16) == -4
    assert bwd(lib, dtype, dx=W + vocab - 16) == -4 and bwd(lib, dtype, dx=W - rows + 16) == -4
    assert bwd(lib, dtype, dw=X + rows - 16) == -4 and bwd(lib, dtype, dx=DW + vocab - 16) == -4
    # ... with dw or dx left out
    assert bwd(lib, dtype, dx=None, dw=W) == -4 and bwd(lib, dtype, dw=None, dx=W + 16) == -4
    # windows of one wider tensor: features that overlap, rows that do
    assert bwd(lib, dtype, x_ss=3 * E, dx=X + row - 16) == -4 and bwd(lib, dtype, x_ss=3 * E, dx=X + 3 * row) == -4
    assert bwd(lib, dtype, x_ss=3 * E, dx=X - 3 * row * (N - 1) + 16) == -4 and bwd(lib, dtype, x_ss=3 * E, dx=X + 2 * row + 16) == -4
    # a short vocabulary's gradient inside one row of a wider tensor's x
    assert bwd(lib, dtype, x_ss=9 * E, V=1, dw=X + 9 * row * 5 + 16) == -4 and bwd(lib, dtype, x_ss=9 * E, V=2, dw=X + 9 * row * 5 - row - 16) == -4
