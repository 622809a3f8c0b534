"""The loss's gradients beside their operands in one tensor: bit for bit what they are in tensors of their own."""
import pytest
import torch

from paper_2502_02406_amd import binding as B
from test_gpu_xent import inputs, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,n,E,V", [("bf16", 70, 128, 300), ("bf16", 300, 64, 700), ("f32", 70, 36, 300)])
def test_gradients_beside_their_operands(dtype, n, E, V):
    x, w, labels, d = inputs(n, E, V, dtype, 51)
    loss, lse, dx, dw = run(x, w, labels, d)
    wide = torch.full((n, 3 * E), 5.0, dtype=x.dtype, device="cuda")          # x, dx, and what nobody touches
    wide[:, :E] = x
    both = torch.full((2 * V, E), 5.0, dtype=x.dtype, device="cuda")          # dw in front of w
    both[V:] = w
    ws = torch.empty(B.lvx_xent_workspace_bytes(n, E, V, B.dtype_code(x.dtype)), dtype=torch.uint8, device="cuda")
    B.lvx_xent_bwd(wide[:, :E], both[V:], labels, lse, d, wide[:, E:2 * E], both[:V], ws)
    assert torch.equal(wide[:, E:2 * E], dx) and torch.equal(both[:V], dw)
    assert (wide[:, 2 * E:] == 5.0).all() and torch.equal(both[V:], w)
    assert torch.equal(wide[:, :E].nan_to_num(9.0), x.nan_to_num(9.0))
    with pytest.raises(B.LvxError):
        B.lvx_xent_bwd(x, w, labels, lse, d, None, w, ws)
    with pytest.raises(B.LvxError):
        B.lvx_xent_bwd(x, w, labels, lse, d, x, None, ws)
    torch.cuda.synchronize()
    assert torch.equal(both[V:], w)
