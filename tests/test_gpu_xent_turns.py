"""The cross entropy where workgroups take several tiles one after the other, in each of its products, against float64.  Inputs, tolerances and
their derivation as in test_gpu_xent.py; the long float32 case takes its reference on the GPU, in float64 as well."""
import pytest
import torch

from paper_2502_02406_amd import binding as B
from test_gpu_xent import check, inputs, reference, run

pytestmark = pytest.mark.gpu


# more than 256 tiles of 256 x 256 or 128 x 256 on a chip of 256 compute units: of logits and of dw; of dx; of both with few features
@pytest.mark.parametrize("n,E,V", [(1030, 1280, 16500), (6300, 3840, 300), (2100, 64, 9001)])
def test_bf16_tiles_in_turn(n, E, V):
    print(f"[xent] bf16 {n}x{E} V={V}", flush=True)
    args = inputs(n, E, V, "bf16", n + V)
    got = run(*args)
    ref, tol = reference(*args, "bf16")
    check(got, ref, tol, f"{n}x{E}x{V}")
    assert all(torch.equal(a, b) for a, b in zip(got, run(*args))), "not repeatable"


def test_f32_tiles_in_turn():
    """More tiles and rows than a launch has workgroups.  A logit: 8 products; errors as in test_gpu_xent.py with E = 8 and the largest values of
    the case in place of every token's."""
    n, E, V = 70000, 8, 4100
    x, w, labels, d = inputs(n, E, V, "f32", 5)
    loss, lse, dx, dw = run(x, w, labels, d)
    on = labels >= 0
    u = 2.0 ** -24
    w64, dw64, tol_w = w.double(), torch.zeros(V, E, dtype=torch.float64, device="cuda"), torch.zeros(V, E, dtype=torch.float64, device="cuda")
    assert not loss[~on].any() and not lse[~on].any() and not dx[~on].any()
    for part in on.nonzero()[:, 0].split(10000):
        x64, d64, lab = x[part].double(), d[part].double(), labels[part, None]
        z = x64 @ w64.T
        ref = torch.logsumexp(z, 1)
        zl = z.gather(1, lab)[:, 0]
        p = torch.exp(z - ref[:, None])
        g = p.scatter_add(1, lab, torch.full_like(zl, -1.0)[:, None]) * d64[:, None]
        ez = (E / 2 + 16) * u * (x64.abs() @ w64.abs().T)
        e_lse = ez.max(1).values + (V / 4096 + 200 + 4 * (ref.abs() + z.abs().max(1).values)) * u
        assert ((lse[part] - ref).abs() <= 1.02 * e_lse).all()
        assert ((loss[part] - (ref - zl)).abs() <= 1.02 * (e_lse + ez.gather(1, lab)[:, 0] + 2 * u * (ref.abs() + zl.abs()))).all()
        eg = p * d64.abs()[:, None] * (ez + e_lse[:, None] + (8 + 4 * (ref.abs()[:, None] + z.abs())) * u) + 2 * u * g.abs()
        assert ((dx[part] - g @ w64).abs() <= 1.02 * (eg @ w64.abs() + (V / 2 + 64) * u * (g.abs() @ w64.abs()))).all()
        dw64 += g.T @ x64
        tol_w += eg.T @ x64.abs() + (n / 2 + 64) * u * (g.abs().T @ x64.abs())
    assert ((dw - dw64).abs() <= 1.02 * tol_w).all()


# few tiles of dw and many tokens: its contraction is cut into parts
@pytest.mark.parametrize("dtype,n,E,V,ignored", [("bf16", 5000, 64, 300, 0.3), ("bf16", 3000, 320, 1000, 0.0), ("bf16", 1280, 64, 1, 0.5), ("bf16", 2000, 64, 129, 0.999),
                                                 ("f32", 3000, 40, 200, 0.3), ("f32", 1030, 67, 130, 0.0), ("f32", 1500, 3, 1, 0.9)])
def test_dw_in_parts(dtype, n, E, V, ignored):
    print(f"[xent] {dtype} {n}x{E} V={V}", flush=True)
    args = inputs(n, E, V, dtype, n + V, ignored=ignored)
    got = run(*args)
    ref, tol = reference(*args, dtype)
    check(got, ref, tol, f"{dtype} {n}x{E}x{V}")
    assert all(torch.equal(a, b) for a, b in zip(got, run(*args))), "not repeatable"
    assert torch.equal(run(*args, dx=False)[3], got[3])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dw_in_parts_piece_by_piece(dtype):
    """Room for pieces of 256 entries and, with one byte too few for them and with enough, for the parts of dw."""
    n, E, V = 3000, 64, 700
    args = inputs(n, E, V, dtype, 8)
    ref, tol = reference(*args, dtype)
    f32 = dtype == "f32"
    up = lambda v: (v + 255) // 256 * 256
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    edge = 64 if f32 and -(-n // 128) * -(-E // 128) * max(1, min(64, V // 256)) < cus else 128 if f32 else 256
    tiles = -(-n // edge) * -(-E // edge)
    least = 256 + 2 * up(4 * n) + up(8 * n) + max(tiles, min(64 * tiles, 2 * cus)) * edge * edge * 4 + 320 * up(n) * (4 if f32 else 2)
    dw_tiles = 4 if f32 else 2
    room = min(64, (-(-n // 64)) // 4, cus // 8 * 8 // dw_tiles) * dw_tiles * (64 * 64 if f32 else 128 * 256) * 4
    assert room < 256 * up(n) * (4 if f32 else 2) or least + room <= B.lvx_xent_workspace_bytes(n, E, V, B.dtype_code(args[0].dtype))
    for ws in (least, least + room - 1, least + room):
        check(run(*args, ws_bytes=ws), ref, tol, f"{ws - least} bytes for parts")


@pytest.mark.parametrize("dtype,n,E,V", [("bf16", 2000, 64, 129), ("f32", 1500, 40, 200), ("f32", 20, 40, 200), ("bf16", 200, 128, 300)])
def test_no_labels(dtype, n, E, V):
    """Nothing to do, in each form of the products: zeros."""
    x, w, labels, d = inputs(n, E, V, dtype, 3)
    loss, lse, dx, dw = run(x, w, torch.full_like(labels, -1), d)
    assert not loss.any() and not lse.any() and not dx.any() and not dw.any()


def test_f32_few_tokens_of_a_long_vocabulary():
    """More workgroups than one side of a launch takes.  The loss of 2 tokens of 2 features; errors as in test_gpu_xent.py."""
    n, E, V = 2, 2, 32 * 16384 + 77
    x, w, labels, d = inputs(n, E, V, "f32", 6, ignored=0.0)
    labels[1] = V - 1
    loss, lse, dx, dw = run(x, w, labels, d)
    z = x.double() @ w.double().T
    ref = torch.logsumexp(z, 1)
    u = 2.0 ** -24
    ez = 17 * u * (x.double().abs() @ w.double().abs().T)
    e_lse = ez.max(1).values + (V / 4096 + 200 + 4 * (ref.abs() + z.abs().max(1).values)) * u
    zl = z.gather(1, labels[:, None])[:, 0]
    assert ((lse - ref).abs() <= 1.02 * e_lse).all()
    assert ((loss - (ref - zl)).abs() <= 1.02 * (e_lse + ez.gather(1, labels[:, None])[:, 0] + 2 * u * (ref.abs() + zl.abs()))).all()
    p = torch.exp(z - ref[:, None])
    g = p.scatter_add(1, labels[:, None], torch.full_like(zl, -1.0)[:, None]) * d.double()[:, None]
    eg = p * d.double().abs()[:, None] * (ez + e_lse[:, None] + (8 + 4 * (ref.abs()[:, None] + z.abs())) * u) + 2 * u * g.abs()
    assert ((dx - g @ w.double()).abs() <= 1.02 * (eg @ w.double().abs() + (V / 2 + 64) * u * (g.abs() @ w.double().abs()))).all()
    assert ((dw - g.T @ x.double()).abs() <= 1.02 * (eg.T @ x.double().abs() + 65 * u * (g.abs().T @ x.double().abs()))).all()


@pytest.mark.parametrize("dtype,n", [("bf16", 20), ("bf16", 64), ("f32", 32)])
def test_labels_outside_among_few_tokens(dtype, n):
    x, w, labels, d = inputs(n, 64, 300, dtype, 19, ignored=0.0)
    ref, tol = reference(x, w, labels, d, dtype)
    far = labels.clone()
    far[3], far[5], far[7], far[n - 1] = 300, 1 << 40, -(1 << 40), -1
    loss, lse, dx, dw = run(x, w, far, d)
    bad, off = torch.zeros(n, dtype=torch.bool), torch.zeros(n, dtype=torch.bool)
    bad[[3, 5]] = True
    off[[7, n - 1]] = True
    assert loss.cpu().isnan().equal(bad) and lse.cpu().isnan().equal(bad) and dw.isnan().all()
    assert dx.cpu()[bad].isnan().all() and not loss.cpu()[off].any() and not lse.cpu()[off].any() and not dx.cpu()[off].any()
    good = ~(bad | off)
    for name, t in (("loss", loss), ("lse", lse), ("dx", dx)):
        err = (t.double().cpu()[good] - torch.from_numpy(ref[name])[good]).abs()
        assert (err <= 1.02 * torch.from_numpy(tol[name])[good] + 1e-30).all(), name


@pytest.mark.parametrize("dtype,n,E", [("bf16", 20, 64), ("bf16", 50, 192), ("bf16", 64, 1024), ("f32", 20, 40), ("bf16", 150, 64)])
def test_few_tokens_piece_by_piece(dtype, n, E):
    """Pieces of 2048 entries, of which the last has one: parts of dx without anything to add."""
    V = 4097
    args = inputs(n, E, V, dtype, 23, pad=8)
    ref, tol = reference(*args, dtype)
    check(run(*args), ref, tol, "whole")
    f32 = dtype == "f32"
    up = lambda v: (v + 255) // 256 * 256
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    edge = 64 if f32 else 256
    rows = 64 if f32 else 128 if n <= 128 else 256
    tiles = -(-n // rows) * -(-E // edge)
    ws = 256 + 2 * up(4 * n) + up(8 * n) + max(tiles, min(64 * tiles, 2 * cus)) * rows * edge * 4 + (2048 + 64) * up(n) * (4 if f32 else 2)
    check(run(*args, ws_bytes=ws), ref, tol, "pieces of 2048")


@pytest.mark.parametrize("n,E,V", [(70, 36, 300), (10, 33, 500), (1400, 64, 100)])
def test_f32_at_any_address(n, E, V):
    args = inputs(n, E, V, "f32", 41)
    ref, tol = reference(*args, "f32")
    off = lambda t: torch.cat([t.new_zeros(1), t.reshape(-1)])[1:].view(t.shape)          # 4 bytes behind an allocation's start
    x, w, labels, d = (off(t.contiguous()) for t in args)
    assert x.data_ptr() % 16 == 4 and w.data_ptr() % 16 == 4
    loss, lse, dx, dw = (off(torch.full(s, 5.0, device="cuda")) for s in ((n,), (n,), (n, E), (V, E)))
    ws = torch.empty(B.lvx_xent_workspace_bytes(n, E, V, B.LVX_F32), dtype=torch.uint8, device="cuda")
    B.lvx_xent_fwd(x, w, labels, loss, lse, ws)
    B.lvx_xent_bwd(x, w, labels, lse, d, dx, dw, ws)
    check((loss, lse, dx, dw), ref, tol, f"{n}x{E}x{V}")
