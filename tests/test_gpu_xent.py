"""Softmax cross entropy against a vocabulary and its gradients through the C ABI, against float64.

Tolerances, from the arithmetic.  A logit is a float32 sum of E exact (bf16) or rounded (float32) products in chains of at most E / 2, so
with A = sum |x| |w| it is off by ez = (E / 2 + 16) 2^-24 A.  The sum of exponentials adds V terms in chains of at most 64 + V / 4096
joined by chains of 32, each exponential off by a few 2^-24 and by its argument's rounding, 2^-23 times the argument:
    e_lse = max ez + (V / 4096 + 200 + 4 (|lse| + max |z|)) 2^-24,     e_loss = e_lse + ez(label) + 2^-23 (|lse| + |z|).
g = (p - [label]) d is off by eg = p d (ez + e_lse + (8 + 4 (|lse| + |z|)) 2^-24) + 2^-23 |g|, in bf16 by another half step of its
rounding, 2^-8 |g|.  dx = g w: eg |w| + (V / 2 + 64) 2^-24 |g| |w| (pieces and parts included) and the half step of its own rounding;
dw = g^T x likewise with n."""
import numpy as np
import pytest
import torch

from paper_2502_02406_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def inputs(n, E, V, dtype, seed, pad=0, ignored=0.3):
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((n + 1, E + pad), float("nan"), dtype=DT[dtype])
    buf[:n, :E] = torch.randn((n, E), generator=g).to(DT[dtype])
    w = (torch.randn((V, E), generator=g) * (2.0 / E ** 0.5)).to(DT[dtype])
    labels = torch.randint(V, (n,), generator=g)
    drop = torch.rand(n, generator=g) < ignored
    drop[0] = False
    labels[drop] = torch.where(torch.rand(n, generator=g) < 0.5, -100, -1)[drop]
    buf[:n][drop] = float("nan")                          # what a token without a label holds reaches nothing
    d = torch.randn(n, generator=g) / n
    d[drop] = float("nan")
    return buf.cuda()[:n, :E], w.cuda(), labels.cuda(), d.cuda()


def run(x, w, labels, d, ws_bytes=None, dx=True, dw=True):
    n, E = x.shape
    V = w.shape[0]
    code = B.dtype_code(x.dtype)
    ws = torch.full((B.lvx_xent_workspace_bytes(n, E, V, code),), 255, dtype=torch.uint8, device="cuda")
    loss, lse = torch.full((n,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    B.lvx_xent_fwd(x, w, labels, loss, lse, ws)
    ws.fill_(255)
    gx = torch.full((n + 1, x.stride(0) if n > 1 else E), 5.0, dtype=x.dtype, device="cuda")
    gw = torch.full((V + 1, E), 5.0, dtype=x.dtype, device="cuda")
    B.lvx_xent_bwd(x, w, labels, lse, d, gx[:n, :E] if dx else None, gw[:V] if dw else None, ws[:ws_bytes])
    torch.cuda.synchronize()
    assert (gx[n:] == 5.0).all() and (gx[:, E:] == 5.0).all() and (gw[V:] == 5.0).all()
    return loss, lse, gx[:n, :E], gw[:V]


def reference(x, w, labels, d, dtype):
    on = (labels >= 0).cpu().numpy()
    xs, ws_, lab, ds = x.double().cpu().numpy()[on], w.double().cpu().numpy(), labels.cpu().numpy()[on], d.double().cpu().numpy()[on]
    n, E, V, rows = x.shape[0], x.shape[1], w.shape[0], np.arange(on.sum())
    z, A = xs @ ws_.T, np.abs(xs) @ np.abs(ws_).T
    top = z.max(1, keepdims=True)
    lse = np.log(np.exp(z - top).sum(1)) + top[:, 0]
    p = np.exp(z - lse[:, None])
    g = p.copy()
    g[rows, lab] -= 1.0
    g *= ds[:, None]
    u, half = 2.0 ** -24, 2.0 ** -8 if dtype == "bf16" else 0.0
    ez = (E / 2 + 16) * u * A
    e_lse = ez.max(1) + (V / 4096 + 200 + 4 * (np.abs(lse) + np.abs(z).max(1))) * u
    zl = z[rows, lab]
    eg = p * np.abs(ds)[:, None] * (ez + e_lse[:, None] + (8 + 4 * (np.abs(lse)[:, None] + np.abs(z))) * u) + (half + 2 * u) * np.abs(g)
    dx, dw = g @ ws_, g.T @ xs
    full = lambda v, shape: np.zeros(shape)
    out, tol = {}, {}
    for name, v, e, shape in (("loss", lse - zl, e_lse + ez[rows, lab] + 2 * u * (np.abs(lse) + np.abs(zl)), (n,)), ("lse", lse, e_lse, (n,)),
                              ("dx", dx, eg @ np.abs(ws_) + (V / 2 + 64) * u * (np.abs(g) @ np.abs(ws_)) + half * np.abs(dx), (n, E))):
        out[name], tol[name] = np.zeros(shape), np.zeros(shape)
        out[name][on], tol[name][on] = v, e
    out["dw"] = dw
    tol["dw"] = eg.T @ np.abs(xs) + (n / 2 + 64) * u * (np.abs(g).T @ np.abs(xs)) + half * np.abs(dw)
    return out, tol


def check(got, ref, tol, tag):
    for name, t in zip(("loss", "lse", "dx", "dw"), got):
        v = t.double().cpu().numpy()
        assert np.isfinite(v).all(), f"{tag} {name}: not finite"
        worst = (np.abs(v - ref[name]) / (tol[name] * 1.02 + 1e-30)).max()
        assert worst <= 1.0, f"{tag} {name}: off by {worst:.3g} of the bound"


BF16 = [(1, 64, 1, 0), (1, 64, 2, 0), (3, 64, 100, 8), (64, 128, 256, 0), (65, 64, 257, 0), (128, 192, 1000, 64), (129, 64, 511, 0), (200, 320, 777, 8),
        (300, 512, 3001, 0), (257, 1024, 300, 0), (16, 256, 9000, 0), (33, 640, 1111, 0), (64, 128, 40000, 8), (128, 192, 700, 0), (100, 640, 1111, 8), (100, 2048, 900, 0), (70, 2048, 16500, 0), (300, 256, 20001, 0), (2, 64, 33000, 0), (700, 256, 20001, 0), (1300, 64, 129, 0)]
F32 = [(1, 1, 1, 0), (5, 33, 7, 3), (130, 100, 129, 0), (64, 64, 500, 0), (200, 257, 333, 1), (300, 40, 9000, 0), (1, 512, 3000, 0), (31, 130, 1000, 0), (33, 96, 700, 0), (64, 2048, 300, 0), (20, 29, 3001, 3)]


@pytest.mark.parametrize("dtype,n,E,V,pad", [("bf16",) + s for s in BF16] + [("f32",) + s for s in F32])
def test_loss_and_gradients(dtype, n, E, V, pad):
    print(f"[xent] {dtype} {n}x{E} V={V}", flush=True)
    args = inputs(n, E, V, dtype, n + E + V, pad)
    got = run(*args)
    ref, tol = reference(*args, dtype)
    check(got, ref, tol, f"{dtype} {n}x{E}x{V}")
    off = (args[2] < 0).cpu()
    assert (got[0].cpu()[off] == 0).all() and (got[1].cpu()[off] == 0).all() and (got[2].cpu()[off] == 0).all()
    again = run(*args)
    assert all(torch.equal(a, b) for a, b in zip(got, again)), "not repeatable"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_workspace_and_parts_left_out(dtype):
    n, E, V = 300, 192, 1500
    args = inputs(n, E, V, dtype, 4)
    ref, tol = reference(*args, dtype)
    el, Mp = (2 if dtype == "bf16" else 4), 512
    up = lambda v: (v + 255) // 256 * 256
    edge = 64 if dtype == "f32" else 256
    tiles = -(-n // edge) * -(-E // edge)
    least = 256 + 2 * up(4 * n) + up(8 * n) + max(tiles, min(64 * tiles, 2 * torch.cuda.get_device_properties(0).multi_processor_count)) * edge * edge * 4 + 320 * Mp * el
    check(run(*args, ws_bytes=least), ref, tol, "pieces of 256")
    with pytest.raises(B.LvxError):
        run(*args, ws_bytes=least - 256)
    whole = run(*args)
    assert torch.equal(run(*args, dw=False)[2], whole[2]) and torch.equal(run(*args, dx=False)[3], whole[3])
    room = B.lvx_xent_workspace_bytes(1300, 512, 2000, B.dtype_code(DT[dtype]))
    ws = torch.empty(room, dtype=torch.uint8, device="cuda")
    loss, lse, dx, dw = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty((n, E), dtype=DT[dtype], device="cuda"), torch.empty_like(args[1])
    B.lvx_xent_fwd(*args[:3], loss, lse, ws)
    B.lvx_xent_bwd(*args[:3], lse, args[3], dx, dw, ws)
    check((loss, lse, dx, dw), ref, tol, "a larger problem's workspace")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_labels_and_labels_outside(dtype):
    x, w, labels, d = inputs(70, 64, 300, dtype, 9, ignored=0.0)
    none = torch.full_like(labels, -100)
    loss, lse, dx, dw = run(x, w, none, d)
    assert not loss.any() and not lse.any() and not dx.any() and not dw.any()
    far = labels.clone()
    far[3], far[5] = 300, 1 << 40
    far[7] = -(1 << 40)
    loss, lse, dx, dw = run(x, w, far, d)
    bad = torch.zeros(70, dtype=torch.bool)
    bad[[3, 5]] = True
    assert loss.cpu().isnan().equal(bad) and lse.cpu().isnan().equal(bad)
    assert dx.cpu()[bad].isnan().all() and dx.cpu()[~bad].isfinite().all() and dw.isnan().all()
    assert loss[7] == 0 and not dx[7].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extreme_logits(dtype):
    """Logits of +-300 beside small ones, a token whose logits are all the same, one with a NaN feature."""
    n, E, V = 40, 64, 500
    x, w, labels, d = inputs(n, E, V, dtype, 12, ignored=0.0)
    x[1] *= 60.0
    x[2] = 0.0
    ref, tol = reference(x, w, labels, d, dtype)
    check(run(x, w, labels, d), ref, tol, "extreme")
    assert abs(ref["lse"][2] - np.log(V)) < 1e-12
    x[4, 5] = float("nan")
    loss, lse, dx, dw = run(x, w, labels, d)
    assert loss.isnan().sum() == 1 and lse[4].isnan() and dx[4].isnan().all() and dx[[i for i in range(n) if i != 4]].isfinite().all()


def test_gradient_by_differences():
    """float64 central differences of sum(loss d) through the definition."""
    x, w, labels, d = inputs(4, 6, 5, "f32", 2, ignored=0.0)
    labels[2] = -1
    _, _, dx, dw = run(x, w, labels, d)
    x64, w64, lab, d64 = x.double().cpu().numpy(), w.double().cpu().numpy(), labels.cpu().numpy(), d.double().cpu().numpy()

    def total(xv, wv):
        z = xv @ wv.T
        return sum(d64[i] * (np.log(np.exp(z[i]).sum()) - z[i, lab[i]]) for i in range(4) if lab[i] >= 0)

    h = 1e-5
    for arr, got in ((x64, dx), (w64, dw)):
        for i in range(arr.shape[0]):
            for e in range(6):
                keep = arr[i, e]
                arr[i, e] = keep + h
                up = total(x64, w64)
                arr[i, e] = keep - h
                dn = total(x64, w64)
                arr[i, e] = keep
                # (h^2 / 6 of a third derivative of about 10, 1e-16 * 10 / 1e-5 of cancellation, float32's 1e-6)
                assert abs((up - dn) / (2 * h) - float(got[i, e])) <= 1e-5


def test_on_another_stream_and_in_a_graph():
    n, E, V = 260, 128, 9000
    x, w, labels, d = inputs(n, E, V, "bf16", 31)
    x.nan_to_num_(0.0)
    d.nan_to_num_(0.003)
    ws = torch.empty(B.lvx_xent_workspace_bytes(n, E, V, B.LVX_BF16), dtype=torch.uint8, device="cuda")
    out = [torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty((n, E), dtype=x.dtype, device="cuda"), torch.empty_like(w)]

    def step():
        B.lvx_xent_fwd(x, w, labels, out[0], out[1], ws)
        B.lvx_xent_bwd(x, w, labels, out[1], d, out[2], out[3], ws)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in out]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for t in out:
            t.fill_(7.0)
        step()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    first_labels = labels.clone()
    for i in range(3):
        labels.copy_(first_labels.roll(i * 17))             # other tokens have labels, and another number of them
        labels[: 40 * i] = -1
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in out]
        for t in out:
            t.fill_(3.0)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, replayed)), i
