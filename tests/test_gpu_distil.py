"""Distillation from a teacher's top logits through the C ABI, against float64.

Tolerances, from the arithmetic, with those of the cross entropy's logits: a logit is off by ez = (E / 2 + 16) 2^-24 A, A = sum |x| |w|.  All in units of
1 / T: e_lse = max ez + (V / 4096 + 200 + 4 (|lse| + max |z|)) 2^-24, an entry's e_p = ez + e_lse + 2^-23 (|z| + |lse| + |ln p|).  ln q comes from logits
divided by T (2^-24 of each), their differences and a sum of K exponentials: e_q = (2 |t| + 2 max |t| + 4 |ln q| + K / 16 + 32) 2^-24, and q is off by
q e_q, so the loss by sum q (e_p + e_q + (e_q + 2^-23 (K / 32 + 8)) |ln q - ln p|).
g = (p - q) d / T: p by p (ez + e_lse + (8 + 4 (|lse| + |z|)) 2^-24), at the teacher's entries by p (e_p + 8 2^-24 (1 + |ln p|)) + q (e_q + K 2^-24); times d, with
2^-22 of it for the factors, in bf16 another half step of g's rounding, 2^-8 |g|.  dx = g w: eg |w| + (V / 2 + 64) 2^-24 |g| |w| and the half
step of its own rounding; dw = g^T x likewise with n."""
import numpy as np
import pytest
import torch

from paper_2502_02406_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
NAN = float("nan")


def inputs(n, E, V, K, dtype, seed, teacher="f32", pad=0, ignored=0.3, twice=False):
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((n + 1, E + pad), NAN, dtype=DT[dtype])
    buf[:n, :E] = torch.randn((n, E), generator=g).to(DT[dtype])
    w = (torch.randn((V, E), generator=g) * (2.0 / E ** 0.5)).to(DT[dtype])
    if twice or K > V:
        ids = torch.randint(min(V, 5), (n, K), generator=g)                # ids that come more than once
    else:
        ids = torch.rand((n, min(V, 20 * K)), generator=g).argsort(1)[:, :K] * (V // min(V, 20 * K))
    t = (torch.randn((n, K), generator=g) * 3.0).to(DT[teacher])
    gone = torch.rand((n, K), generator=g) < 0.2                        # entries that are not there, and some with q = 0
    gone[:, 0] = False
    ids[gone] = -7
    t[gone] = NAN
    t[(torch.rand((n, K), generator=g) < 0.1) & (torch.arange(K) > 0) & ~gone] = -float("inf")
    drop = torch.rand(n, generator=g) < ignored
    drop[0] = False
    ids[drop] = -100
    t[drop] = NAN
    none = drop.clone()
    none[: n // 2] = False                                           # without a probability instead of without an entry
    ids[none] = 0
    t[none] = -float("inf")
    buf[:n][drop] = NAN
    d = torch.randn(n, generator=g) / n
    d[drop] = NAN
    return buf.cuda()[:n, :E], w.cuda(), ids.cuda(), t.cuda(), d.cuda()


def run(x, w, ids, t, d, T, ws_bytes=None, dx=True, dw=True):
    n, E = x.shape
    (V, K), code = (w.shape[0], ids.shape[1]), B.dtype_code(x.dtype)
    ws = torch.full((B.lvx_distil_workspace_bytes(n, E, V, K, code),), 255, dtype=torch.uint8, device="cuda")
    loss, lse, ln_p = (torch.full(s, 7.0, device="cuda") for s in ((n,), (n,), (n, K)))
    B.lvx_distil_fwd(x, w, ids, t, loss, lse, ln_p, ws, T)
    ws.fill_(255)
    gx = torch.full((n + 1, x.stride(0) if n > 1 else E), 5.0, dtype=x.dtype, device="cuda")
    gw = torch.full((V + 1, E), 5.0, dtype=x.dtype, device="cuda")
    B.lvx_distil_bwd(x, w, ids, t, lse, ln_p, d, gx[:n, :E] if dx else None, gw[:V] if dw else None, ws[:ws_bytes], T)
    torch.cuda.synchronize()
    assert (gx[n:] == 5.0).all() and (gx[:, E:] == 5.0).all() and (gw[V:] == 5.0).all()
    return loss, lse, ln_p, gx[:n, :E], gw[:V]


def reference(x, w, ids, t, d, T, dtype):
    ids, tt = ids.cpu().numpy(), t.double().cpu().numpy()
    T = float(np.float32(T))
    there = (ids >= 0) & (tt != -np.inf)
    on = there.any(1)
    xs, W, I, D = x.double().cpu().numpy()[on], w.double().cpu().numpy(), ids[on], d.double().cpu().numpy()[on]
    th, tq = ids[on] >= 0, np.where(ids[on] >= 0, tt[on], -np.inf) / T
    n, K, V, E = ids.shape[0], ids.shape[1], W.shape[0], xs.shape[1]
    u, half = 2.0 ** -24, 2.0 ** -8 if dtype == "bf16" else 0.0
    z, ez = xs @ W.T / T, (E / 2 + 16) * u * (np.abs(xs) @ np.abs(W).T) / T
    top = z.max(1, keepdims=True)
    lse = np.log(np.exp(z - top).sum(1)) + top[:, 0]
    mt = tq.max(1, keepdims=True)
    ln_q = tq - mt - np.log(np.exp(tq - mt).sum(1, keepdims=True))
    q = np.exp(ln_q)
    rows = np.arange(len(I))[:, None]
    at = np.where(th, I, 0)
    ze, eze = z[rows, at], ez[rows, at]
    ln_p = np.where(th, ze - lse[:, None], 0.0)
    lq = np.where(q > 0, ln_q, 0.0)
    gap = np.where(q > 0, lq - ln_p, 0.0)
    loss = (q * gap).sum(1)
    L = np.abs(lse)[:, None]
    e_lse = ez.max(1) + (V / 4096 + 200 + 4 * (np.abs(lse) + np.abs(z).max(1))) * u
    e_p = eze + e_lse[:, None] + 2 * u * (np.abs(ze) + L + np.abs(ln_p))
    tf = np.where(q > 0, np.abs(tq), 0.0)
    e_q = (2 * tf + 2 * np.abs(mt) + 4 * np.abs(lq) + K / 16 + 32) * u
    e_loss = (q * (e_p + e_q + (e_q + 2 * u * (K / 32 + 8)) * np.abs(gap))).sum(1) + u * np.abs(loss)
    p = np.exp(z - lse[:, None])
    hot, e_hot = np.zeros_like(z), np.zeros_like(z)
    np.add.at(hot, (rows, at), np.where(th, q, 0.0))
    np.add.at(e_hot, (rows, at), np.where(th, q * (e_q + K * u), 0.0))
    e = p * (ez + e_lse[:, None] + (8 + 4 * (L + np.abs(z))) * u)
    ee = p[rows, at] * (e_p + 8 * u * (1 + np.abs(ln_p)))
    for k in range(K):
        r = np.nonzero(th[:, k])[0]
        e[r, at[r, k]] = np.maximum(e[r, at[r, k]], ee[r, k])
    s = np.abs(D)[:, None] / T
    g = (p - hot) * D[:, None] / T
    eg = (e + e_hot) * s + (half + 4 * u) * np.abs(g)
    dx, dw, aw, ax = g @ W, g.T @ xs, np.abs(W), np.abs(xs)
    out, tol = {}, {}
    for name, v, er, shape in (("loss", loss, e_loss, (n,)), ("lse", lse, e_lse, (n,)), ("ln_p", ln_p, e_p, (n, K)),
                               ("dx", dx, eg @ aw + (V / 2 + 64) * u * (np.abs(g) @ aw) + half * np.abs(dx), (n, E))):
        out[name], tol[name] = np.zeros(shape), np.zeros(shape)
        out[name][on], tol[name][on] = v, er
    out["dw"], tol["dw"] = dw, eg.T @ ax + (n / 2 + 64) * u * (np.abs(g).T @ ax) + half * np.abs(dw)
    return out, tol, on


def check(got, ref, tol, tag):
    for name, t in zip(("loss", "lse", "ln_p", "dx", "dw"), got):
        v = t.double().cpu().numpy()
        assert np.array_equal(np.isfinite(v), np.isfinite(ref[name])), f"{tag} {name}: not finite"
        with np.errstate(invalid="ignore"):
            off = np.where(np.isfinite(v), np.abs(v - ref[name]), 0.0)
        worst = (off / (tol[name] * 1.02 + 1e-30)).max()
        assert worst <= 1.0, f"{tag} {name}: off by {worst:.3g} of the bound"


# (bf16: each of the product's forms: few tokens listed by every wave, 64 x 128 and 128 x 128 tiles, 128 and 256 rows; float32: 32 tokens, 64 and 128 tiles)
BF16 = [(1, 64, 1, 1, 0), (1, 64, 300, 1, 0), (3, 64, 100, 8, 8), (64, 128, 256, 17, 0), (33, 640, 1111, 64, 0), (20, 64, 40000, 100, 8), (65, 64, 257, 3, 0),
        (129, 64, 511, 65, 0), (300, 512, 3001, 20, 0), (100, 2048, 16500, 16, 0), (300, 256, 20001, 64, 0), (700, 256, 20001, 5, 64), (1300, 64, 129, 30, 0),
        (2500, 64, 20001, 33, 0), (2000, 320, 9000, 64, 0), (70, 64, 1000, 1000, 0), (1100, 128, 1000, 128, 0)]
F32 = [(1, 1, 1, 1, 0), (5, 33, 7, 7, 3), (20, 29, 3001, 50, 3), (32, 64, 500, 5, 0), (33, 96, 700, 40, 0), (200, 257, 333, 100, 1), (300, 40, 9000, 16, 0),
       (700, 20, 30000, 8, 0)]


@pytest.mark.parametrize("dtype,n,E,V,K,pad", [("bf16",) + s for s in BF16] + [("f32",) + s for s in F32])
def test_loss_and_gradients(dtype, n, E, V, K, pad):
    teacher, T = ("bf16", 0.7) if (n + V) % 2 else ("f32", 2.0)
    print(f"[distil] {dtype} {n}x{E} V={V} K={K} teacher {teacher} T {T}", flush=True)
    args = inputs(n, E, V, K, dtype, n + E + V, teacher, pad)
    got = run(*args, T)
    ref, tol, on = reference(*args, T, dtype)
    check(got, ref, tol, f"{dtype} {n}x{E}x{V}, {K}")
    off = torch.from_numpy(~on)
    assert all((t.cpu()[off] == 0).all() for t in got[:4])
    again = run(*args, T)
    assert all(torch.equal(a, b) for a, b in zip(got, again)), "not repeatable"


@pytest.mark.parametrize("dtype,n", [("bf16", 40), ("bf16", 200), ("bf16", 1500), ("f32", 20), ("f32", 150)])
def test_ids_that_come_more_than_once(dtype, n):
    args = inputs(n, 64, 700, 12, dtype, 5, twice=True)
    ref, tol, _ = reference(*args, 1.0, dtype)
    check(run(*args, 1.0), ref, tol, "twice")


@pytest.mark.parametrize("dtype,n,K", [("bf16", 64, 8), ("bf16", 64, 9), ("bf16", 65, 8), ("bf16", 33, 1), ("bf16", 768, 8), ("bf16", 769, 8), ("bf16", 1024, 6), ("bf16", 1025, 2),
                                       ("f32", 32, 8), ("f32", 33, 8), ("f32", 32, 9), ("f32", 1024, 5)])
def test_few_entries(dtype, n, K):
    """Where the ways of few entries begin and end, with ids that come more than once, and with half of the tokens or none taking part."""
    args = inputs(n, 64, 333, K, dtype, n + K, twice=True)
    ref, tol, on = reference(*args, 0.5, dtype)
    got = run(*args, 0.5)
    check(got, ref, tol, "few")
    assert all(torch.equal(a, b) for a, b in zip(got, run(*args, 0.5)))
    x, w, ids, t, d = args
    t = t.clone()
    t[: n // 2] = -float("inf")
    ref, tol, on = reference(x, w, ids, t, d, 0.5, dtype)
    got = run(x, w, ids, t, d, 0.5)
    check(got, ref, tol, "behind others")
    assert not any(v[: n // 2].any() for v in got[:4])
    t[:] = -float("inf")
    assert not any(v.any() for v in run(x, w, ids, t, d, 0.5))


@pytest.mark.parametrize("dtype,n", [("bf16", 70), ("bf16", 300), ("f32", 30), ("f32", 100)])
def test_a_whole_teacher(dtype, n):
    """All entries of the vocabulary are known, in any order: the divergence of two whole softmaxes."""
    V = 200
    x, w, ids, t, d = inputs(n, 64, V, 1, dtype, 7, ignored=0.0)
    g = torch.Generator().manual_seed(1)
    ids = torch.rand((n, V), generator=g).argsort(1).cuda()
    t = torch.randn((n, V), generator=g).cuda()
    ref, tol, _ = reference(x, w, ids, t, d, 1.5, dtype)
    check(run(x, w, ids, t, d, 1.5), ref, tol, "whole")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_workspace_and_parts_left_out(dtype):
    n, E, V, K, T = 300, 192, 1500, 9, 1.0
    args = inputs(n, E, V, K, dtype, 4)
    ref, tol, _ = reference(*args, T, dtype)
    el, Mp = (2 if dtype == "bf16" else 4), 512
    up = lambda v: (v + 255) // 256 * 256
    edge = 64 if dtype == "f32" else 256
    tiles = -(-n // edge) * -(-E // edge)
    least = 2 * up(8 * n) + 256 + 2 * up(4 * n) + up(8 * n) + max(tiles, min(64 * tiles, 2 * torch.cuda.get_device_properties(0).multi_processor_count)) * edge * edge * 4 + 320 * Mp * el
    check(run(*args, T, ws_bytes=least), ref, tol, "pieces of 256")
    with pytest.raises(B.LvxError):
        run(*args, T, ws_bytes=least - 256)
    whole = run(*args, T)
    assert torch.equal(run(*args, T, dw=False)[3], whole[3]) and torch.equal(run(*args, T, dx=False)[4], whole[4])
    ws = torch.empty(B.lvx_distil_workspace_bytes(1300, 512, 2000, 20, B.dtype_code(DT[dtype])), dtype=torch.uint8, device="cuda")
    loss, lse, ln_p = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty((n, K), device="cuda")
    dx, dw = torch.empty((n, E), dtype=DT[dtype], device="cuda"), torch.empty_like(args[1])
    B.lvx_distil_fwd(*args[:4], loss, lse, ln_p, ws, T)
    B.lvx_distil_bwd(*args[:4], lse, ln_p, args[4], dx, dw, ws, T)
    check((loss, lse, ln_p, dx, dw), ref, tol, "a larger problem's workspace")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,K", [(32768, 8), (32769, 8), (131072, 2), (131073, 2)])
def test_few_entries_of_a_long_vocabulary(dtype, V, K):
    args = inputs(20, 64, V, K, dtype, 3)
    ref, tol, _ = reference(*args, 1.0, dtype)
    check(run(*args, 1.0), ref, tol, "long")


@pytest.mark.parametrize("dtype,n,K", [("bf16", 40, 4), ("bf16", 40, 20), ("f32", 20, 4), ("bf16", 200, 5)])
def test_few_entries_in_pieces_of_the_vocabulary(dtype, n, K):
    """The least workspace that the backward pass takes (found by what it refuses, before any launch): the entries are handed to several pieces."""
    args = inputs(n, 128, 1500, K, dtype, 12, twice=True)
    ref, tol, _ = reference(*args, 1.5, dtype)
    low, high = 0, B.lvx_distil_workspace_bytes(n, 128, 1500, K, B.dtype_code(DT[dtype])) // 256
    while high - low > 1:
        mid = (low + high) // 2
        try:
            run(*args, 1.5, ws_bytes=mid * 256)
            high = mid
        except B.LvxError:
            low = mid
    check(run(*args, 1.5, ws_bytes=high * 256), ref, tol, f"{high * 256} bytes")


@pytest.mark.parametrize("dtype,n", [("bf16", 70), ("bf16", 30), ("f32", 70), ("f32", 20)])
def test_nothing_to_learn_and_ids_outside(dtype, n):
    x, w, ids, t, d = inputs(n, 64, 300, 4, dtype, 9, ignored=0.0)
    t.nan_to_num_(0.0, neginf=-1.0)
    none = torch.full_like(ids, -100)
    assert not any(o.any() for o in run(x, w, none, t, d, 1.0))
    far = ids.clone()
    far[3, 2], far[5, 0] = 300, 1 << 40
    far[7] = -(1 << 40)
    loss, lse, ln_p, dx, dw = run(x, w, far, t, d, 1.0)
    bad = torch.zeros(n, dtype=torch.bool)
    bad[[3, 5]] = True
    assert loss.cpu().isnan().equal(bad) and lse.cpu().isnan().equal(bad)
    assert dx.cpu()[bad].isnan().all() and dx.cpu()[~bad].isfinite().all() and dw.isnan().all()
    assert loss[7] == 0 and not dx[7].any() and not ln_p[7].any()
    for value in (NAN, float("inf")):
        t2 = t.clone()
        t2[4, 1] = value
        ids2 = ids.clone()
        ids2[4, 1] = 17
        loss, lse, ln_p, dx, dw = run(x, w, ids2, t2, d, 1.0)
        assert loss.isnan().sum() == 1 and loss[4].isnan() and lse.isfinite().all() and ln_p.isfinite().all()
        assert dx[4].isnan().all() and dx[[i for i in range(n) if i != 4]].isfinite().all()


def test_gradient_by_differences():
    """Central differences in float64 of sum(loss d) through the definition: h^2 / 6 of a third derivative of about 10, h = 1e-5, 1e-16 * 10 / h of
    cancellation, float32's 1e-6."""
    T = 0.8
    x, w, ids, t, d = inputs(4, 6, 9, 3, "f32", 2, ignored=0.0)
    ids[2] = -1
    _, _, _, dx, dw = run(x, w, ids, t, d, T)
    x64, w64, I, tt, d64 = x.double().cpu().numpy(), w.double().cpu().numpy(), ids.cpu().numpy(), t.double().cpu().numpy(), d.double().cpu().numpy()
    T = float(np.float32(T))

    def total(xv, wv):
        s = 0.0
        for i in range(4):
            at = [k for k in range(3) if I[i, k] >= 0 and tt[i, k] > -np.inf]
            if at:
                z, q = xv[i] @ wv.T / T, np.exp(tt[i, at] / T)
                q /= q.sum()
                s += d64[i] * (q * (np.log(q) - (z[I[i, at]] - np.log(np.exp(z).sum())))).sum()
        return s

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
                assert abs((up - dn) / (2 * h) - float(got[i, e])) <= 1e-5


@pytest.mark.parametrize("n", [50, 260])
def test_batches_other_stream_and_graph(n):
    E, V, K, T = 128, 9000, 16, 2.0
    x, w, ids, t, d = inputs(n, E, V, K, "bf16", 31, ignored=0.0)
    x, ids, t = x.reshape(2, n // 2, E), ids.view(2, n // 2, K), t.nan_to_num(0.0, neginf=-2.0).view(2, n // 2, K)
    ws = torch.empty(B.lvx_distil_workspace_bytes(n, E, V, K, B.LVX_BF16), dtype=torch.uint8, device="cuda")
    out = [torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty((n, K), device="cuda"), torch.empty_like(x), torch.empty_like(w)]

    def step():
        B.lvx_distil_fwd(x, w, ids, t, out[0], out[1], out[2], ws, T)
        B.lvx_distil_bwd(x, w, ids, t, out[1], out[2], d, out[3], out[4], ws, T)

    step()
    torch.cuda.synchronize()
    want = [o.clone() for o in out]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for o in out:
            o.fill_(7.0)
        step()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    base = ids.clone()
    for i in range(3):
        ids.copy_(base.roll(i * 3, 1))
        ids[:, : 10 * i] = -1
        graph.replay()
        torch.cuda.synchronize()
        replayed = [o.clone() for o in out]
        for o in out:
            o.fill_(3.0)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, replayed)), i
