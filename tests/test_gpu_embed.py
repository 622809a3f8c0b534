"""Embedding lookup and its gradient through the C ABI, against float64.

Tolerances, from the arithmetic.  y: one float32 product, 2^-24 |y|, and (bf16) half a step of its rounding, 2^-8 |y|.  d_table[v]: however the
c tokens of a row are grouped, a sum of theirs is off by at most c 2^-24 A with A = sum |d_y|; times the scale (2^-24 of it), added to what
is there (2^-24), and rounded."""
import numpy as np
import pytest
import torch

from paper_2502_02406_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def inputs(n, E, V, dtype, seed, pad=0, off=0, ignored=0.2, ids=None):
    """Rows `off` elements behind an aligned address, E + pad apart; NaN in the gaps and where the id is negative."""
    g = torch.Generator().manual_seed(seed)
    table = torch.randn(V * E + off, generator=g).to(DT[dtype]).cuda()[off:].view(V, E)
    if ids is None:
        rank = torch.exp(torch.rand(n, generator=g) * np.log(V + 1)).long().clamp(1, V) - 1          # words are as frequent as their rank is low
        ids = torch.randperm(V, generator=g)[rank]
        ids[torch.rand(n, generator=g) < ignored] = -1
    dy = torch.full((n * (E + pad) + off,), float("nan"), dtype=DT[dtype])[off:].view(n, E + pad)
    dy[:, :E] = torch.randn((n, E), generator=g).to(DT[dtype])
    dy[ids < 0] = float("nan")
    store = torch.empty(n * (E + pad) + off, dtype=DT[dtype], device="cuda")[off:].view(n, E + pad)
    store.copy_(dy)
    return table, ids.cuda(), store[:, :E]


def run(table, ids, dy, scale, pad=0, off=0, old=None):
    n, (V, E) = ids.numel(), table.shape
    y = torch.full((n * (E + pad) + off + 9,), 5.0, dtype=table.dtype, device="cuda")
    rows = y[off:off + n * (E + pad)].view(n, E + pad)
    B.lvx_embed_fwd(table, ids, rows[:, :E], scale)
    d = torch.full((V * E + off + 9,), 5.0, dtype=table.dtype, device="cuda")
    dt = d[off:off + V * E].view(V, E)
    if old is not None:
        dt.copy_(old)
    ws = torch.full((B.lvx_embed_workspace_bytes(n, E, V),), 255, dtype=torch.uint8, device="cuda")
    B.lvx_embed_bwd(dy, ids, dt, ws, scale, accumulate=old is not None)
    torch.cuda.synchronize()
    for buf, size in ((y, n * (E + pad)), (d, V * E)):
        assert (buf[:off] == 5.0).all() and (buf[off + size:] == 5.0).all()
    assert (rows[:, E:] == 5.0).all()
    return rows[:, :E], dt


def check(table, ids, dy, scale, y, dt, old=None):
    half = 2.0 ** -8 if table.dtype == torch.bfloat16 else U
    t, i, g = table.double().cpu().numpy(), ids.cpu().numpy(), dy.double().cpu().numpy()
    s = float(np.float32(scale))
    on = (i >= 0) & (i < len(t))
    want = np.zeros(g.shape)
    want[on] = t[i[on]] * s
    got = y.double().cpu().numpy()
    inside = i < len(t)
    assert (np.abs(got - want)[inside] <= (half + U) * np.abs(want)[inside]).all()
    assert np.isnan(got[~inside]).all()
    d, A, c = np.zeros(t.shape), np.zeros(t.shape), np.zeros(len(t))
    np.add.at(d, i[on], g[on])
    np.add.at(A, i[on], np.abs(g[on]))
    np.add.at(c, i[on], 1.0)
    want = d * s + (old.double().cpu().numpy() if old is not None else 0.0)
    tol = ((c[:, None] + 2) * U * A * abs(s) + 2 * U * np.abs(want)) * (1 + half) + half * np.abs(want)
    got = dt.double().cpu().numpy()
    worst = np.abs(got - want) - tol
    assert (worst <= 0).all(), f"off by {worst.max():.3g} more than the bound"
    if old is not None:
        assert torch.equal(dt[torch.from_numpy(c == 0).cuda()], old[torch.from_numpy(c == 0).cuda()]), "rows without tokens have changed"


SIZES = [(1, 1, 1), (1, 4096, 100), (3, 7, 5), (64, 64, 1000), (65, 129, 1), (700, 1001, 300), (2000, 512, 33000), (8192, 64, 1025), (8193, 40, 50021),
         (20000, 8, 131072), (10000, 2056, 7), (9000, 16, (1 << 20) + 5), (12289, 520, 1024), (40000, 24, 300), (5000, 40, 9), (1025, 16, 2), (7000, 24, 200000), (1024, 8, 5000), (16, 256, 3), (17, 40, 2), (256, 16, 900), (257, 16, 900),
         (3000, 8, (1 << 21) + 3), (32768, 16, 4000), (32769, 16, 4000), (30000, 8, 2), (15000, 8, (1 << 20) + 7)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,E,V", SIZES)
def test_lookup_and_gradient(dtype, n, E, V):
    for pad, off, add in ((0, 0, False), (5, 1, True), (8, 0, True)):
        print(f"[embed] {dtype} {n}x{E} V={V} pad {pad} off {off} add {add}", flush=True)
        args = inputs(n, E, V, dtype, n + E + V, pad, off)
        old = torch.randn((V, E), generator=torch.Generator().manual_seed(1)).to(DT[dtype]).cuda() if add else None
        y, dt = run(*args, 0.3, pad, off, old)
        check(*args, 0.3, y, dt, old)
        y2, dt2 = run(*args, 0.3, pad, off, old)
        assert torch.equal(y, y2) and torch.equal(dt, dt2), "not repeatable"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [9, 200, 300, 3000, 8192, 30000])
@pytest.mark.parametrize("which", ["none", "same", "two", "outside", "last"])
def test_few_ids(dtype, n, which):
    """All tokens padding, one id for all, two that alternate, ids outside the table, the table's last row among others."""
    E, V = 72, 3000
    k = torch.arange(n)
    ids = {"none": torch.full((n,), -100), "same": torch.full((n,), 1234), "two": torch.where(k % 3 == 0, 2999, 0),
           "outside": torch.where(k % 2 == 0, k % V, torch.where(k % 4 == 1, V, 1 << 40)), "last": torch.where(k == n - 1, V - 1, k % 5)}[which]
    args = inputs(n, E, V, dtype, 5, ids=ids)
    y, dt = run(*args, 2.0)
    check(*args, 2.0, y, dt)
    old = torch.ones((V, E), dtype=DT[dtype], device="cuda")
    y, dt = run(*args, 2.0, old=old)
    check(*args, 2.0, y, dt, old)


def test_gradient_by_differences():
    """Central differences in float64 of sum(y c) through the definition; the gradient is linear, so they are exact up to 1e-9."""
    g = torch.Generator().manual_seed(1)
    n, E, V = 9, 5, 4
    ids = torch.tensor([0, 3, -1, 3, 3, 2, 0, -7, 2])
    c = torch.randn((n, E), generator=g)
    dt = torch.empty((V, E), device="cuda")
    ws = torch.empty(B.lvx_embed_workspace_bytes(n, E, V), dtype=torch.uint8, device="cuda")
    B.lvx_embed_bwd(c.cuda(), ids.cuda(), dt, ws, 0.5)
    t = torch.randn((V, E), generator=g, dtype=torch.float64)

    def total(table):
        return sum(float((0.5 * table[i] * c[k].double()).sum()) for k, i in enumerate(ids.tolist()) if i >= 0)

    for v in range(V):
        for e in range(E):
            up, dn = t.clone(), t.clone()
            up[v, e] += 0.25
            dn[v, e] -= 0.25
            assert abs((total(up) - total(dn)) / 0.5 - float(dt[v, e])) <= 1e-5


@pytest.mark.parametrize("n", [200, 9000])
def test_batches_other_stream_and_graph(n):
    """[B, S, E] rows, a workspace for more, another stream, and a captured call that is replayed on other ids."""
    E, V = 136, 5000
    table, ids, dy = inputs(n, E, V, "bf16", 3)
    ids = ids.view(2, n // 2)
    dy = dy.reshape(2, n // 2, E).nan_to_num(0.0)
    y, dt = torch.empty_like(dy), torch.empty_like(table)
    ws = torch.empty(B.lvx_embed_workspace_bytes(2 * n, 2 * E, 2 * V), dtype=torch.uint8, device="cuda")

    def step():
        B.lvx_embed_fwd(table, ids, y, 1.5)
        B.lvx_embed_bwd(dy, ids, dt, ws, 1.5)

    step()
    torch.cuda.synchronize()
    check(table, ids.flatten(), dy.view(n, E), 1.5, y.view(n, E), dt)
    want = y.clone(), dt.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y.fill_(7.0), dt.fill_(7.0)
        step()
    s.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(dt, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    base = ids.clone()
    for i in range(3):
        ids.copy_((base * (i + 3)) % V)
        ids[:, : 30 * i] = -1
        graph.replay()
        torch.cuda.synchronize()
        replayed = y.clone(), dt.clone()
        y.fill_(3.0), dt.fill_(3.0)
        step()
        torch.cuda.synchronize()
        assert torch.equal(y, replayed[0]) and torch.equal(dt, replayed[1]), i
        check(table, ids.flatten(), dy.view(n, E), 1.5, y.view(n, E), dt)


def test_refused_overlap():
    t = torch.zeros((64, 64), device="cuda")
    ids = torch.zeros(8, dtype=torch.int64, device="cuda")
    ws = torch.empty(B.lvx_embed_workspace_bytes(8, 64, 64), dtype=torch.uint8, device="cuda")
    with pytest.raises(B.LvxError):
        B.lvx_embed_fwd(t, ids, t[8:16])
    with pytest.raises(B.LvxError):
        B.lvx_embed_bwd(t[:8], ids, t, ws)


@pytest.mark.parametrize("times,E", [(1, 8), (1, 300), (7, 24), (18, 8), (40, 16)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ids_of_so_many_chunks(dtype, times, E):
    """Sorted tokens are summed four at a time here: ids of as many tokens as end before, at and behind the edges of 1 to 65 such chunks and of 32 of them, in
    several orders."""
    g = torch.Generator().manual_seed(times + E)
    counts = [4 * k + d for k in (1, 2, 31, 32, 33, 63, 64, 65) for d in (-1, 0, 1)] + [1, 2, 3, 4, 128, 128, 256]
    counts = torch.tensor(counts)
    per_id = torch.cat([counts[torch.randperm(len(counts), generator=g)] for _ in range(times)])
    V = len(per_id)
    ids = torch.repeat_interleave(torch.arange(V), per_id)
    ids = ids[torch.randperm(len(ids), generator=g)]
    table, ids, dy = inputs(len(ids), E, V, dtype, times, ids=ids)
    old = torch.randn((V, E), generator=g).to(DT[dtype]).cuda()
    for there in (None, old):
        y, dt = run(table, ids, dy, 0.5, old=there)
        check(table, ids, dy, 0.5, y, dt, there)
        assert torch.equal(dt, run(table, ids, dy, 0.5, old=there)[1])


@pytest.mark.parametrize("n,E,V,share", [(131072, 64, 5000, 1.0), (70000, 24, 900, 0.7), (20000, 40, 50, 0.5), (9000, 520, 9000, 0.9), (3000, 8, 7, 0.95)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_id_that_most_tokens_have(dtype, n, E, V, share):
    """Its sums go over whole groups of chunks, which begin and end anywhere; other ids stand in front of it and behind."""
    g = torch.Generator().manual_seed(n)
    for hot in (0, V // 2, V - 1):
        ids = torch.where(torch.rand(n, generator=g) < share, hot, torch.randint(V, (n,), generator=g))
        args = inputs(n, E, V, dtype, 5, ids=ids)
        y, dt = run(*args, 0.5)
        check(*args, 0.5, y, dt)
        old = torch.ones((V, E), dtype=DT[dtype], device="cuda")
        y, dt = run(*args, 0.5, old=old)
        check(*args, 0.5, y, dt, old)


def test_offsets_that_pass_32_bits():
    """A table of more than 2^32 elements and rows of y so far apart that theirs pass 2^32 too: the last rows, ids that few and that many tokens have."""
    V, E, n = 530000, 8192, 1200
    far = (1 << 32) // 1000
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(V - 300, V, (n,), generator=g, device="cuda")
    ids[::3] = V - 1
    ids[1::7] = 5
    table = torch.empty((V, E), dtype=torch.bfloat16, device="cuda")
    for rows in (table[:10], table[V - 300:]):
        rows.normal_(generator=g)
    y = torch.empty((n, far), dtype=torch.bfloat16, device="cuda")
    B.lvx_embed_fwd(table, ids, y[:, :E], 0.25)
    assert torch.equal(y[:, :E], table[ids] * 0.25)               # (a power of two)
    grad = torch.full_like(table, 3.0)
    ws = torch.empty(B.lvx_embed_workspace_bytes(n, E, V), dtype=torch.uint8, device="cuda")
    B.lvx_embed_bwd(y[:, :E], ids, grad, ws, 1.0)
    want = torch.zeros((V, 4), dtype=torch.float64, device="cuda").index_add_(0, ids, y[:, E - 4:E].double())
    size = torch.zeros((V, 4), dtype=torch.float64, device="cuda").index_add_(0, ids, y[:, E - 4:E].double().abs())
    tol = (n * U * size) * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
    assert ((grad[:, E - 4:].double() - want).abs() <= tol).all()
    some = torch.zeros(V, dtype=torch.bool, device="cuda")
    some[ids] = True
    assert not any(grad[r:r + 50000][~some[r:r + 50000]].any() for r in range(0, V, 50000))
