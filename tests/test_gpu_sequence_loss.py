"""Preference and policy losses through the C ABI, against their definitions in float64.

Tolerances, from the arithmetic.  Everything is float64 up to one rounding of each result, 2^-24 of it, and for a policy's mean gradient three (the
token's, that of 1 / count, their product).  Float64 leaves of a sum of c terms of size A in all at most c 2^-53 A: eD below, with 2^-48 for
the functions; of a margin this goes through the loss with |loss'| at most beta (1 + ..) or 2 |m - 1 / (2 beta)|, and into the gradient
with loss'' at most beta^2 or 2."""
import math

import numpy as np
import pytest
import torch

from paper_2502_02406_amd import binding as B

pytestmark = pytest.mark.gpu
U, D = 2.0 ** -24, 2.0 ** -48
NAN = float("nan")


def sequences(n, count, seed, kind):
    g = np.random.default_rng(seed)
    if kind == "even":
        return [n * i // count for i in range(count + 1)]
    if kind == "gaps":                              # tokens in front of the first sequence and behind the last one
        cuts = np.sort(g.integers(n // 10, n - n // 10 + 1, count + 1))
        return cuts.tolist()
    return [0] + np.sort(g.integers(0, n + 1, count - 1)).tolist() + [n]


def inputs(n, count, seed, kind="any", masked=0.3, adv=None):
    g = torch.Generator().manual_seed(seed)
    first = sequences(n, count, seed, kind)
    nll = -torch.log(torch.rand(n, generator=g).clamp(min=1e-6))
    s = {"nll": nll, "ref": nll + 0.2 * torch.randn(n, generator=g), "old": nll + 0.3 * torch.randn(n, generator=g),
         "labels": torch.randint(1000, (n,), generator=g), "adv": torch.randn(adv or count, generator=g)}
    off = torch.rand(n, generator=g) < masked
    if n > 4:
        off[first[1]:first[2] if count > 1 else 0] = True             # a sequence without a label
    s["labels"][off] = torch.where(torch.rand(n, generator=g) < 0.5, -100, -1)[off]
    for name in ("nll", "ref", "old") + (("adv",) if adv == n else ()):
        s[name][off] = NAN                                         # what a token without a label holds reaches nothing
    s["first"] = torch.tensor(first)
    return {k: v.cuda() for k, v in s.items()}


def host(s):
    return {k: v.double().cpu().numpy() if v.is_floating_point() else v.cpu().numpy() for k, v in s.items()}


def spans(s, n):
    f = np.clip(s["first"], 0, n)
    return [(a, max(a, b)) for a, b in zip(f, f[1:])]


def pref_reference(s, n, S, d, form, beta, smooth):
    on = s["labels"] >= 0
    more = np.where(on, np.nan_to_num(s["ref"]) - np.nan_to_num(s["nll"]), 0.0)
    sp = spans(s, n)
    tot, A = np.array([more[a:b].sum() for a, b in sp]), np.array([np.abs(more[a:b]).sum() * (b - a + 64) for a, b in sp]) * 2.0 ** -53
    m, eD = tot[:S] - tot[S:], A[:S] + A[S:] + 2.0 ** -52 * np.abs(tot[:S])
    h = beta * m
    if form == "logistic":
        soft = lambda x: np.logaddexp(0.0, x)
        loss, sig = (1 - smooth) * soft(-h) + smooth * soft(h), np.array([1 / (1 + math.exp(-x)) if x > 0 else math.exp(x) / (1 + math.exp(x)) for x in h])
        slope, by, curve = beta * (sig - (1 - smooth)), beta, beta ** 2
    elif form == "hinge":
        loss, slope, by, curve = np.maximum(0.0, 1 - h), np.where(h < 1, -beta, 0.0), beta, 0.0
    else:
        loss, slope, by, curve = (m - 0.5 / beta) ** 2, 2 * (m - 0.5 / beta), 2 * np.abs(m - 0.5 / beta), 2.0
    grad, tg = np.full(n, NAN), np.zeros(n)
    e = (curve * eD + D * (np.abs(slope) + beta)) * np.abs(d)
    for i, (a, b) in enumerate(sp):
        sign = -1.0 if i >= S else 1.0
        grad[a:b] = np.where(on[a:b], -sign * slope[i % S] * d[i % S], 0.0)
        tg[a:b] = U * np.abs(grad[a:b]) + e[i % S]
    return (loss, m, grad), (U * np.abs(loss) + by * eD + D * (np.abs(loss) + 1), U * np.abs(m) + eD, tg)


def policy_reference(s, n, S, d, lo, hi, beta, mean):
    loss, stats, grad, tg, tl = np.zeros(S), np.zeros((S, 3)), np.full(n, NAN), np.zeros(n), np.zeros(S)
    for i, (a, b) in enumerate(spans(s, n)):
        at = a + np.nonzero(s["labels"][a:b] >= 0)[0]
        grad[a:b] = 0.0
        c = len(at)
        if c == 0:
            continue
        adv = s["adv"][at] if len(s["adv"]) != S else np.full(c, s["adv"][i])
        r = np.exp(s["old"][at] - s["nll"][at])
        free, held = r * adv, np.clip(r, 1 - lo, 1 + hi) * adv
        l, g, kl = -np.minimum(free, held), np.where(free <= held, free, 0.0), np.zeros(c)
        if beta > 0:
            dd = s["nll"][at] - s["ref"][at]
            kl = np.expm1(dd) - dd
            l, g = l + beta * kl, g + beta * np.expm1(dd)
        over = c if mean else 1
        loss[i], stats[i] = l.sum() / over, (c, (free > held).mean(), kl.mean())
        grad[at] = g * d[i] / over
        tl[i] = (D + c * 2.0 ** -53) * np.abs(l).sum() / over
        tg[at] = (3 if mean else 1) * U * np.abs(grad[at]) + D * (np.abs(free) + beta * np.exp(np.abs(s["nll"][at] - s["ref"][at]))) * abs(d[i]) / over + 2.0 ** -148
    tl += U * np.abs(loss)
    return (loss, stats, grad), (tl, U * np.abs(stats) + 1e-12, tg)


def compare(got, want, tol, tag):
    for k, (g, w, t) in enumerate(zip(got, want, tol)):
        v = g.double().cpu().numpy()
        rest = np.isnan(w)
        assert (v[rest] == 7.0).all(), f"{tag} output {k}: written where no sequence is"
        bad = np.abs(v - w)[~rest] - t[~rest] * 1.01 if t.shape == w.shape else np.abs(v - w)[~rest] - t
        assert (bad <= 0).all(), f"{tag} output {k}: off by {bad.max():.3g} more than the bound"


def run_pref(s, S, d, in_place=False, **kw):
    n = s["labels"].numel()
    loss, margin = torch.full((S,), 7.0, device="cuda"), torch.full((S,), 7.0, device="cuda")
    ws = torch.full((B.lvx_preference_workspace_bytes(n, S),), 255, dtype=torch.uint8, device="cuda")
    nll = s["nll"].clone()
    grad = nll if in_place else torch.full((n,), 7.0, device="cuda")
    B.lvx_preference(nll, s["ref"], s["labels"], s["first"], loss, margin, d, grad, ws, **kw)
    torch.cuda.synchronize()
    return loss, margin, grad


def run_policy(s, S, d, in_place=False, **kw):
    n = s["labels"].numel()
    loss, stats = torch.full((S,), 7.0, device="cuda"), torch.full((S, 3), 7.0, device="cuda")
    ws = torch.full((B.lvx_policy_workspace_bytes(n, S),), 255, dtype=torch.uint8, device="cuda")
    nll = s["nll"].clone()
    grad = nll if in_place else torch.full((n,), 7.0, device="cuda")
    B.lvx_policy(nll, s["old"], s["ref"], s["adv"], s["labels"], s["first"], loss, stats, d, grad, ws, **kw)
    torch.cuda.synchronize()
    return loss, stats, grad


SIZES = [(2, 1, "even"), (1, 1, "any"), (100, 3, "any"), (513, 1, "even"), (3000, 700, "any"), (32768, 5, "gaps"), (32769, 5, "gaps"), (40000, 3000, "any"),
         (200001, 2, "any"), (100000, 64, "gaps"), (65536, 8, "even"), (33000, 300, "any")]


@pytest.mark.parametrize("n,S,kind", SIZES)
@pytest.mark.parametrize("form,beta,smooth", [("logistic", 0.1, 0.0), ("logistic", 0.5, 0.1), ("hinge", 0.3, 0.0), ("square", 0.2, 0.0)])
def test_preference(n, S, kind, form, beta, smooth):
    print(f"[preference] {n} tokens, {S} pairs, {kind}, {form}", flush=True)
    s = inputs(n, 2 * S, n + S, kind)
    d = torch.randn(S, generator=torch.Generator().manual_seed(S)).cuda()
    got = run_pref(s, S, d, form=form, beta=beta, smoothing=smooth)
    want, tol = pref_reference(host(s), n, S, d.double().cpu().numpy(), form, beta, smooth)
    compare(got, want, tol, "preference")
    assert all(torch.equal(a, b) for a, b in zip(got, run_pref(s, S, d, form=form, beta=beta, smoothing=smooth))), "not repeatable"


@pytest.mark.parametrize("n,S,kind", SIZES)
@pytest.mark.parametrize("mean,per_token,beta", [(True, False, 0.04), (False, True, 0.2), (True, True, 0.0), (False, False, 0.0)])
def test_policy(n, S, kind, mean, per_token, beta):
    print(f"[policy] {n} tokens, {S} sequences, {kind}, mean {mean}, per token {per_token}, beta {beta}", flush=True)
    s = inputs(n, S, n + S, kind, adv=n if per_token and n != S else None)
    d = torch.randn(S, generator=torch.Generator().manual_seed(S)).cuda()
    kw = dict(clip=(0.2, 0.28), beta=beta, mean=mean)
    got = run_policy(s, S, d, **kw)
    want, tol = policy_reference(host(s), n, S, d.double().cpu().numpy(), 0.2, 0.28, beta, mean)
    compare(got, want, tol, "policy")
    assert all(torch.equal(a, b) for a, b in zip(got, run_policy(s, S, d, **kw))), "not repeatable"


@pytest.mark.parametrize("n", [80, 33000])
def test_gradient_of_sure_pairs(n):
    """One labelled token a sequence, margins from -80 to 80 without a rounding: the gradient of a pair that is nearly certain is exp(-h), with one rounding
    to float32 (2^-24) and a few of float64."""
    S = 40
    h = torch.linspace(-80, 80, S).round()
    z = lambda: torch.zeros(n, device="cuda")
    s = {"nll": z(), "ref": z(), "labels": torch.full((n,), -1, device="cuda"), "first": torch.arange(2 * S + 1, device="cuda") * (n // (2 * S))}
    at = s["first"][:S]
    s["labels"][at], s["labels"][s["first"][S:-1]] = 1, 1
    s["ref"][at] = h.cuda()
    loss, margin, grad = run_pref(s, S, torch.ones(S, device="cuda"), form="logistic", beta=1.0)
    want = np.exp(-np.logaddexp(0.0, h.double().numpy()))
    assert torch.equal(margin.cpu(), h)
    for rows, sign in ((at, 1.0), (s["first"][S:-1], -1.0)):
        assert (np.abs(grad[rows].double().cpu().numpy() - sign * want) <= want * (2.0 ** -24 + 2.0 ** -48)).all()
    assert (np.abs(loss.double().cpu().numpy() - np.logaddexp(0.0, -h.double().numpy())) <= np.logaddexp(0.0, -h.double().numpy()) * (2.0 ** -24 + 2.0 ** -48)).all()


@pytest.mark.parametrize("n", [3000, 50000])
def test_in_place_loss_alone_and_no_reference(n):
    S = 6
    s = inputs(n, 2 * S, 3, "any", masked=0.1)
    d = torch.rand(S, device="cuda")
    a, b = run_pref(s, S, d), run_pref(s, S, d, in_place=True)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    ws = torch.empty(B.lvx_preference_workspace_bytes(2 * n, 3 * S), dtype=torch.uint8, device="cuda")
    loss = torch.empty(S, device="cuda")
    B.lvx_preference(s["nll"], s["ref"], s["labels"], s["first"], loss, workspace=ws)
    assert torch.equal(loss, a[0])
    zero, none = dict(s, ref=torch.zeros_like(s["nll"])), dict(s, ref=None)
    assert all(torch.equal(x, y) for x, y in zip(run_pref(zero, S, d), run_pref(none, S, d)))
    s = inputs(n, S, 4, "any", masked=0.1)
    for mean in (True, False):
        a, b = run_policy(s, S, d, beta=0.1, mean=mean), run_policy(s, S, d, in_place=True, beta=0.1, mean=mean)
        assert all(torch.equal(x, y) for x, y in zip(a, b))
        loss = torch.empty(S, device="cuda")
        B.lvx_policy(s["nll"], s["old"], s["ref"], s["adv"], s["labels"], s["first"], loss, workspace=ws, beta=0.1, mean=mean)
        assert torch.equal(loss, a[0])


@pytest.mark.parametrize("n", [600, 40000])
def test_bounds_outside_the_tensors(n):
    """Sequences that begin before the first token, end behind the last, or end before they begin."""
    s = inputs(n, 4, 8, "even", masked=0.1)
    s["first"] = torch.tensor([-5, n // 3, n // 3, n // 2, n + 100], device="cuda")
    d = torch.rand(2, device="cuda")
    want, tol = pref_reference(host(s), n, 2, d.double().cpu().numpy(), "logistic", 0.1, 0.0)
    compare(run_pref(s, 2, d), want, tol, "outside")
    s["first"] = torch.tensor([1 << 40, -(1 << 40), 7, 3, n], device="cuda")         # (nothing outside is touched; no result is promised)
    run_pref(s, 2, d)
    run_policy(dict(s, adv=torch.ones(4, device="cuda")), 4, torch.rand(4, device="cuda"))


def test_a_nan_that_counts():
    s = inputs(500, 4, 9, "even", masked=0.0)
    s["labels"].fill_(3)
    for name in ("nll", "ref", "old"):
        s[name].nan_to_num_(0.5)
    s["nll"][130] = NAN                            # of the second sequence: the chosen one of pair 1
    d = torch.ones(2, device="cuda")
    for form in B.LVX_PREF_FORMS:
        loss, margin, grad = run_pref(s, 2, d, form=form)
        assert loss.isnan().tolist() == [False, True] and margin.isnan().tolist() == [False, True], form
        assert grad[125:250].isnan().all() and grad[375:].isnan().all() and grad[:125].isfinite().all() and grad[250:375].isfinite().all()
    loss, stats, grad = run_policy(s, 4, torch.ones(4, device="cuda"))
    assert loss.isnan().tolist() == [False, True, False, False] and grad.isnan().sum() == 1


def test_gradients_by_differences():
    """Central differences in float64 through the definitions: h^2 / 6 of third derivatives of about 10, h = 1e-5, 1e-16 * 10 / h of
    cancellation, and float32's 1e-6 of the result."""
    n, S, h = 24, 2, 1e-5
    s = inputs(n, 4, 5, "even", masked=0.2)
    d = torch.tensor([0.7, -1.3], device="cuda")
    hs, hd = host(s), d.double().cpu().numpy()
    for form in B.LVX_PREF_FORMS:
        grad = run_pref(s, S, d, form=form, beta=0.3)[2].cpu().numpy()
        for t in range(n):
            if hs["labels"][t] >= 0:
                total = [0.0, 0.0]
                for k, step in enumerate((h, -h)):
                    moved = dict(hs, nll=hs["nll"].copy())
                    moved["nll"][t] += step
                    total[k] = (pref_reference(moved, n, S, hd, form, 0.3, 0.0)[0][0] * hd).sum()
                assert abs((total[0] - total[1]) / (2 * h) - grad[t]) <= 2e-6 * (1 + abs(grad[t])), (form, t)
    s = inputs(n, S, 6, "even", masked=0.2)
    hs = host(s)
    for mean in (True, False):
        grad = run_policy(s, S, d, beta=0.3, mean=mean)[2].cpu().numpy()
        for t in range(n):
            if hs["labels"][t] >= 0:
                total = [0.0, 0.0]
                for k, step in enumerate((h, -h)):
                    moved = dict(hs, nll=hs["nll"].copy())
                    moved["nll"][t] += step
                    total[k] = (policy_reference(moved, n, S, hd, 0.2, 0.2, 0.3, mean)[0][0] * hd).sum()
                assert abs((total[0] - total[1]) / (2 * h) - grad[t]) <= 2e-6 * (1 + abs(grad[t])), (mean, t)


@pytest.mark.parametrize("n", [2000, 70000])
def test_other_stream_and_graph(n):
    S = 5
    s, t = inputs(n, 2 * S, 1, "any"), inputs(n, S, 2, "any")
    d = torch.rand(S, device="cuda")
    ws = torch.empty(max(B.lvx_preference_workspace_bytes(n, S), B.lvx_policy_workspace_bytes(n, S)), dtype=torch.uint8, device="cuda")
    out = [torch.empty(k, device="cuda") for k in (S, S, n, S, 3 * S, n)]

    def step():
        B.lvx_preference(s["nll"], s["ref"], s["labels"], s["first"], out[0], out[1], d, out[2], ws)
        B.lvx_policy(t["nll"], t["old"], t["ref"], t["adv"], t["labels"], t["first"], out[3], out[4], d, out[5], ws, beta=0.1)

    step()
    torch.cuda.synchronize()
    want = [x.clone() for x in out]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for x in out:
            x.fill_(7.0)
        step()
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    labels, first = s["labels"].clone(), s["first"].clone()
    for i in range(3):
        s["labels"].copy_(labels)
        s["labels"][: 400 * i] = -1
        s["first"].copy_(first)
        s["first"][1:-1] = first[1:-1] // (i + 1)                   # other sequences, of other lengths
        graph.replay()
        torch.cuda.synchronize()
        replayed = [x.clone() for x in out]
        for x in out:
            x.fill_(3.0)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, replayed)), i
