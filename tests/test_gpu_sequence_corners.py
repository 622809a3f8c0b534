"""Losses of sequences where two readings of a call, infinities or roundings meet: against the definitions in float64."""
import math

import numpy as np
import pytest
import torch

from paper_2502_02406_amd import binding as B
from test_gpu_sequence_loss import D, U, compare, host, inputs, policy_reference, pref_reference, run_policy, run_pref

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("n,first", [(3, [0, 2, 2, 3]), (3, [0, 0, 1, 3]), (5000, None), (40000, None)])
@pytest.mark.parametrize("per_token", [True, False])
@pytest.mark.parametrize("mean", [True, False])
def test_as_many_sequences_as_tokens(n, first, per_token, mean):
    """An advantage a token and one a sequence are as many: which of them they are is said."""
    s = inputs(n, n, 11, "any", masked=0.0, adv=n)
    for name in ("nll", "ref", "old", "adv"):
        s[name].nan_to_num_(0.5)
    if first is not None:
        s["first"] = torch.tensor(first, device="cuda")
        s["labels"].fill_(3)
    d = torch.randn(n, generator=torch.Generator().manual_seed(n)).cuda()
    h, hd = host(s), d.double().cpu().numpy()
    if per_token:
        h["adv"] = np.append(h["adv"], 0.0)          # (one more, by which policy_reference knows them)
    want, tol = policy_reference(h, n, n, hd, 0.2, 0.2, 0.1, mean)
    compare(run_policy(s, n, d, beta=0.1, mean=mean, per_token=per_token), want, tol, "as many")
    with pytest.raises(ValueError):
        run_policy(s, n, d, beta=0.1, mean=mean)


def test_advantages_through_the_sequence_loss():
    from paper_2502_02406_amd.blockloop import SequenceLoss
    s = inputs(3, 3, 5, "even", masked=0.0)
    s.update(first=torch.tensor([0, 2, 2, 3], device="cuda"), labels=torch.ones(3, dtype=torch.int64, device="cuda"), adv=torch.tensor([1.0, -2.0, 3.0], device="cuda"))
    for name in ("nll", "ref", "old"):
        s[name] = torch.ones(3, device="cuda")       # (ratios of 1: a token's loss is its advantage with the other sign)
    seq = SequenceLoss(3, 3)
    call = lambda **kw: seq.policy(s["nll"], s["old"], None, s["adv"], s["labels"], s["first"], mean=False, **kw)[0].tolist()
    assert call(per_token=True) == [1.0, 0.0, -3.0] and call(per_token=False) == [-2.0, 0.0, -3.0]
    with pytest.raises(ValueError):
        call()


def pairs_of_one(n, S, nll):
    """S pairs of one labelled token a sequence, among n tokens: (inputs, the chosen ones' places, the rejected ones')."""
    z = lambda: torch.zeros(n, device="cuda")
    s = {"nll": z(), "ref": z(), "labels": torch.full((n,), -1, device="cuda"), "first": torch.arange(2 * S + 1, device="cuda") * (n // (2 * S))}
    c, r = s["first"][:S], s["first"][S:-1]
    s["labels"][c] = s["labels"][r] = 1
    s["nll"][c], s["nll"][r] = nll[0].cuda(), nll[1].cuda()
    return s, c, r


@pytest.mark.parametrize("n", [80, 40000])
@pytest.mark.parametrize("form,smooth", [("logistic", 0.0), ("logistic", 0.25), ("logistic", 1.0), ("hinge", 0.0)])
def test_an_answer_without_likelihood(n, form, smooth):
    """A margin of +infinity (the rejected one's nll is), or -infinity: a part of the loss that counts for nothing adds nothing, whatever it would be, and the slope is
    that of the loss far out.  All values are exact in float32."""
    beta = 0.5
    s, c, r = pairs_of_one(n, 3, torch.tensor([[1.0, INF, 2.0], [INF, 1.0, 2.0]]))
    loss, margin, grad = run_pref(s, 3, torch.tensor([1.0, 1.0, 0.0], device="cuda"), form=form, beta=beta, smoothing=smooth)
    assert margin.tolist() == [INF, -INF, 0.0]
    if form == "hinge":
        want, slope = [0.0, INF], [0.0, -beta]
    else:
        want = [INF if smooth > 0 else 0.0, INF if smooth < 1 else 0.0]
        slope = [beta * smooth, -beta * (1 - smooth)]
    assert loss.tolist()[:2] == want
    assert grad[c].tolist()[:2] == [-x for x in slope] and grad[r].tolist()[:2] == slope


@pytest.mark.parametrize("n", [40, 40000])
@pytest.mark.parametrize("mean", [True, False])
def test_a_token_that_the_reference_rules_out(n, mean):
    """ref = +infinity: the divergence is infinite, its slope exp(-infinity) - 1 = -1, and no other token's gradient is touched.  Also far out, where d is finite."""
    beta, S = 0.25, 2
    z = lambda x: torch.full((n,), x, device="cuda")
    s = {"nll": z(1.0), "old": z(1.0), "ref": z(1.0), "labels": z(1.0).long(), "adv": torch.zeros(S, device="cuda"), "first": torch.tensor([0, 8, 16], device="cuda")}
    s["ref"][3], s["ref"][11] = INF, 1e30
    loss, stats, grad = run_policy(s, S, torch.full((S,), 8.0 if mean else 1.0, device="cuda"), beta=beta, mean=mean)
    want = torch.zeros(16)
    want[3] = want[11] = -beta
    assert loss[0].item() == INF and stats[0, 2].item() == INF and loss[1].item() == pytest.approx(0.25e30 / (8 if mean else 1), rel=2 * U)
    assert torch.equal(grad[:16].cpu(), want) and (grad[16:] == 7.0).all()


@pytest.mark.parametrize("count", [7, 120, 1000])
@pytest.mark.parametrize("S", [25, 300])
def test_a_means_gradient_is_rounded_twice(S, count):
    """Once as the token's and once by the number of tokens, 2^-24 each; the rest is float64, as in policy_reference.  (300 sequences of 120 tokens and more: two launches.)"""
    n = S * count
    print(f"[mean] {S} sequences of {count} tokens", flush=True)
    s = inputs(n, S, count, "even", masked=0.0)
    for name in ("nll", "ref", "old"):
        s[name].nan_to_num_(0.5)
    s["labels"].fill_(3)
    d = torch.randn(S, generator=torch.Generator().manual_seed(S)).cuda()
    got = run_policy(s, S, d, beta=0.2)
    h = host(s)
    want, (tl, ts, _) = policy_reference(h, n, S, d.double().cpu().numpy(), 0.2, 0.2, 0.2, True)
    size = np.exp(h["old"] - h["nll"]) * np.abs(np.repeat(h["adv"], count)) + 0.2 * np.exp(np.abs(h["nll"] - h["ref"]))
    of_it = np.repeat(np.abs(d.double().cpu().numpy()), count) / count
    compare(got, want, (tl, ts, (2 * U * np.abs(want[2]) + D * size * of_it + 2.0 ** -148) / 1.01), "mean")      # (compare allows a hundredth more)


def many_tokens(n):
    g = torch.Generator(device="cuda").manual_seed(n)
    s = {"nll": torch.rand(n, generator=g, device="cuda"), "labels": torch.randint(-2, 9, (n,), generator=g, device="cuda")}
    s["ref"] = s["nll"] + 0.01 * torch.randn(n, generator=g, device="cuda")
    s["old"] = s["nll"] + 0.2 * torch.randn(n, generator=g, device="cuda")
    return s


@pytest.mark.parametrize("op", ["preference", "policy"])
def test_time_goes_with_the_tokens_not_with_their_square(op):
    """2^27 tokens in two sequences, and in 16384 of them: the same bytes and arithmetic, so no more than four times the time."""
    n, times = 1 << 27, {}
    s = many_tokens(n)
    d_nll = torch.empty(n, device="cuda")
    for count in (2, 16384):
        first = torch.arange(count + 1, device="cuda") * (n // count)
        S = count // 2 if op == "preference" else count
        loss, one = torch.empty(S, device="cuda"), torch.ones(S, device="cuda")
        ws = torch.empty(max(B.lvx_preference_workspace_bytes(n, S), B.lvx_policy_workspace_bytes(n, S)), dtype=torch.uint8, device="cuda")
        took = []
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            if op == "preference":
                B.lvx_preference(s["nll"], s["ref"], s["labels"], first, loss, None, one, d_nll, ws)
            else:
                B.lvx_policy(s["nll"], s["old"], s["ref"], one, s["labels"], first, loss, None, one, d_nll, ws, beta=0.1)
            b.record()
            torch.cuda.synchronize()
            took.append(a.elapsed_time(b))
        times[count] = min(took[1:])
    print(f"[long] {op}: ms {times}", flush=True)
    assert times[2] <= 4 * times[16384], times


@pytest.mark.parametrize("n,S,kind", [((1 << 24) - 1, 2, "any"), (1 << 24, 1, "even"), ((1 << 24) + 777, 3, "gaps"), ((1 << 24) + 1025, 3000, "any")])
def test_sums_of_long_sequences(n, S, kind):
    print(f"[long] {n} tokens, {S}, {kind}", flush=True)
    d = torch.randn(S, generator=torch.Generator().manual_seed(S)).cuda()
    hd = d.double().cpu().numpy()
    s = inputs(n, 2 * S, n + S, kind)
    got = run_pref(s, S, d, beta=0.01)
    compare(got, *pref_reference(host(s), n, S, hd, "logistic", 0.01, 0.0), "preference")
    assert all(torch.equal(a, b) for a, b in zip(got, run_pref(s, S, d, beta=0.01))), "not repeatable"
    s = inputs(n, S, n + S, kind)
    for mean in (True, False):
        got = run_policy(s, S, d, beta=0.1, mean=mean)
        compare(got, *policy_reference(host(s), n, S, hd, 0.2, 0.2, 0.1, mean), "policy")
        assert all(torch.equal(a, b) for a, b in zip(got, run_policy(s, S, d, beta=0.1, mean=mean))), "not repeatable"
