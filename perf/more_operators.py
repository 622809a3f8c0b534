"""Operators of a training step at either end of the cross-attention layer: from token ids to features and back, and the
losses that are more than a label's cross entropy.

A case is a dict of plain values:

  kind     "embed"   n ids to rows of a table [V, E], scaled; train: and the table's gradient.  The share `ignored` of the
                     tokens is padding (a negative id).  tied: the gradient is added to one that is there already, that of the
                     same table as a vocabulary's weights; otherwise it is overwritten
           "distil"  divergence of the student's softmax of n tokens x E features against a vocabulary [V, E] from a
                     teacher's, of which K logits a token are known, both at a temperature; train: and the gradients of features
                     and weights.  The share `ignored` of the tokens takes no part
           "pref"    preference loss of S pairs of sequences, n tokens in all, from the tokens' negative log likelihoods under
                     the policy and under a reference, and its gradient
           "policy"  clipped policy loss of S sequences, n tokens in all, with a divergence from a reference
                     (beta > 0), and its gradient; the advantages belong to sequences or (per_token) to tokens
  dtype    "bf16" or "f32"; teacher: the type of the teacher's logits
  pad      features between one token's row and the next (a window of a wider tensor)

`listed` holds one case for each kind of use, `draw` gives others of the same ranges.
"""
from __future__ import annotations

import math

import torch

own = False

SCALE = 0.125          # of looked-up rows
BETA = 0.1             # of preferences
CLIP = (0.2, 0.28)     # a ratio's room below and above 1


def _embed(n, E, V, *, dtype="bf16", train=True, ignored=0.0, tied=False, pad=0):
    return dict(kind="embed", n=n, E=E, V=V, dtype=dtype, train=train, ignored=ignored, tied=tied, pad=pad)


def _distil(n, E, V, K, *, dtype="bf16", teacher="f32", temperature=1.0, train=True, ignored=0.0):
    return dict(kind="distil", n=n, E=E, V=V, K=K, dtype=dtype, teacher=teacher, temperature=temperature, train=train, ignored=ignored)


def _pref(S, n, *, form="logistic", smoothing=0.0, prompt=0.3, uneven=False):
    return dict(kind="pref", S=S, n=n, form=form, smoothing=smoothing, prompt=prompt, uneven=uneven)


def _policy(S, n, *, beta=0.04, mean=True, per_token=False, prompt=0.3, uneven=False):
    return dict(kind="policy", S=S, n=n, beta=beta, mean=mean, per_token=per_token, prompt=prompt, uneven=uneven)


def listed():
    return [
        # serving, the features of one generated token (launch and latency)
        dict(_embed(1, 4096, 32768, train=False), name="embed_token"),
        # training, the text rows of the benchmark's workload
        dict(_embed(2048, 4096, 32768), name="embed_text"),
        # training, the longest text side against a very large vocabulary
        dict(_embed(65536, 4096, 131072), name="embed_long"),
        # the Video-MME text length, padded, an odd width inside a wider float32 tensor, a table that the loss uses too
        dict(_embed(5514, 1001, 50021, dtype="f32", ignored=0.1, tied=True, pad=6), name="embed_odd_f32"),
        # scoring 16 tokens against a teacher (the vocabulary's weights are read once)
        dict(_distil(16, 4096, 32768, 16, train=False), name="distil_score"),
        # training, the text rows of the benchmark's workload
        dict(_distil(2048, 4096, 32768, 64, temperature=2.0), name="distil_text"),
        # training, an odd vocabulary and a narrow model; most tokens are a prompt; a teacher's logits kept in 16 bits
        dict(_distil(5514, 1024, 50021, 20, teacher="bf16", ignored=0.6), name="distil_prompt"),
        # the exact check in float32
        dict(_distil(300, 512, 5003, 8, dtype="f32", temperature=0.5, ignored=0.1), name="distil_f32"),
        # one pair of short answers (launch and latency)
        dict(_pref(1, 512), name="pref_pair"),
        # a batch of 64 pairs, labels that may be wrong
        dict(_pref(64, 131072, smoothing=0.1, uneven=True), name="pref_batch"),
        # 512 sampled answers, an advantage each, mean over an answer's tokens
        dict(_policy(512, 524288, uneven=True), name="policy_group"),
        # eight very long answers, an advantage a token, sum over all tokens
        dict(_policy(8, 1048576, mean=False, per_token=True), name="policy_long"),
    ]


# ---- further cases --------------------------------------------------------------------------

_MOST_ROWS = 65536 * 4096                   # "embed_long"
_MOST_TABLE = 131072 * 4096
_MOST_PRODUCT = 2048 * 4096 * 32768         # "distil_text"


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size in [lo, hi], even over its logarithm: a power of two, a multiple of 64, or any number."""
    n = _log(rng, lo, hi)
    how = rng.randrange(4)
    if how == 0:
        n = 1 << round(math.log2(n))
    elif how == 1:
        n = (n + 63) // 64 * 64
    return max(lo, min(hi, n))


def draw(rng):
    kind = rng.choice(("embed", "embed", "embed", "distil", "distil", "distil", "pref", "policy"))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    if kind == "embed":
        E = _size(rng, 64, 8192)
        V = _size(rng, 1000, min(131072, _MOST_TABLE // E // (2 if dtype == "f32" else 1)))
        n = _size(rng, 1, min(131072, _MOST_ROWS // E // (2 if dtype == "f32" else 1)))
        return _embed(n, E, V, dtype=dtype, train=rng.random() < 0.75, ignored=rng.choice((0.0, 0.0, 0.1, 0.7)),
                      tied=rng.random() < 0.3, pad=rng.choice((0, 0, 8, rng.randint(1, 50))))
    if kind == "distil":
        E = 64 * _log(rng, 2, 64)
        V = _size(rng, 1000, 131072)
        most = _MOST_PRODUCT / (E * V) if dtype == "bf16" else (1 << 32) / (E * V)
        n = _size(rng, 1, max(1, min(8192, int(most))))
        return _distil(n, E, V, _log(rng, 1, 128), dtype=dtype, teacher=rng.choice(("f32", "bf16")),
                       temperature=rng.choice((1.0, 1.0, 2.0, 4.0, 0.7)), train=rng.random() < 0.7,
                       ignored=rng.choice((0.0, 0.0, 0.1, 0.5, 0.9)))
    S = _size(rng, 1, 512)
    n = min(1 << 20, max(2 * S, S * _log(rng, 2, 16384)))
    prompt, uneven = rng.choice((0.0, 0.1, 0.5, 0.9)), rng.random() < 0.7
    if kind == "pref":
        form = rng.choice(("logistic", "logistic", "hinge", "square"))
        return _pref(S, n, form=form, smoothing=rng.choice((0.0, 0.1)) if form == "logistic" else 0.0, prompt=prompt, uneven=uneven)
    return _policy(S, n, beta=rng.choice((0.0, 0.04, 0.2)), mean=rng.random() < 0.6, per_token=rng.random() < 0.4, prompt=prompt,
                   uneven=uneven)


# ---- one case -------------------------------------------------------------------------------

def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _sequences(case, seed):
    """Where the case's sequences start, and the end of the last one: lengths alike, or anything from nothing on."""
    count = case["S"] * (2 if case["kind"] == "pref" else 1)
    if not case["uneven"]:
        return [case["n"] * i // count for i in range(count + 1)]
    g = torch.Generator()
    g.manual_seed(seed)
    cuts = torch.randint(case["n"] + 1, (count - 1,), generator=g).sort().values.tolist()
    return [0] + cuts + [case["n"]]


def _inputs(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device="cuda") * std

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    def wide(rows, cols, dt, std, pad=0):
        # (drawn in place, some rows at a time: no second copy of a large tensor in float32)
        out = torch.zeros((rows, cols + pad), dtype=dt, device="cuda")[:, :cols]
        for part in out.split(8192):
            part.copy_(normal(part.shape[0], cols, std=std))
        return out

    if c["kind"] == "embed":
        dt, n, E, V = _dtype(c["dtype"]), c["n"], c["E"], c["V"]
        # (words are as frequent as their rank is low, and lie anywhere in the table)
        rank = torch.exp(uniform(n) * math.log(V)).long().clamp(max=V) - 1
        ids = torch.randperm(V, generator=g, device="cuda")[rank]
        ids[1:][uniform(n - 1) < c["ignored"]] = -1
        s = {"table": wide(V, E, dt, 1.0), "ids": ids}
        if c["train"]:
            s["d_y"] = wide(n, E, dt, 0.05, c["pad"])
            if c["tied"]:
                s["dw"] = wide(V, E, dt, 0.01)
        return s
    if c["kind"] == "distil":
        dt, n, E, V, K = _dtype(c["dtype"]), c["n"], c["E"], c["V"], c["K"]
        s = {"x": wide(n, E, dt, 1.0), "w": wide(V, E, dt, 2.0 / E ** 0.5)}
        # (a token's entries differ from each other, like those that a selection of the largest gives)
        step = (uniform(n, 1) * (V // K)).long().clamp(min=1)
        s["ids"] = (torch.randint(V, (n, 1), generator=g, device="cuda") + step * torch.arange(K, device="cuda")) % V
        s["teacher"] = normal(n, K, std=3.0).sort(1, descending=True).values.to(_dtype(c["teacher"]))
        # (the student has learned something of it)
        s["x"] += (1.5 * s["w"][s["ids"][:, 0]].float() + 0.7 * s["w"][s["ids"][:, -1]].float()).to(dt)
        off = torch.cat((torch.zeros(1, dtype=torch.bool, device="cuda"), uniform(n - 1) < c["ignored"]))
        s["ids"][off] = -1
        s["d_loss"] = torch.full((n,), 1.0, device="cuda") / (~off).sum()
        return s
    n = c["n"]
    first = _sequences(c, seed)
    s = {"first": torch.tensor(first, device="cuda"), "nll": -torch.log(uniform(n).clamp(min=1e-6))}
    s["labels"] = torch.randint(32768, (n,), generator=g, device="cuda")
    s["labels"][uniform(n) < c["prompt"]] = -100
    s["ref"] = (s["nll"] + normal(n, std=0.2)).abs()
    if c["kind"] == "policy":
        s["old"] = (s["nll"] + normal(n, std=0.1)).abs()
        s["adv"] = normal(n if c["per_token"] else c["S"])
    for name in ("nll", "ref", "old"):
        if name in s:
            s[name][s["labels"] < 0] = 0.0
    # (the mean over pairs or answers, or over all tokens)
    over = c["S"] if c["kind"] == "pref" or c["mean"] else n
    s["d_loss"] = torch.full((c["S"],), 1.0 / over, device="cuda")
    return s


def prepare(case, seed):
    return dict(_inputs(case, seed), case=case)


def _plain_embed(s):
    c, ids = s["case"], s["ids"]
    on = ids >= 0
    y = (s["table"][ids.clamp(min=0)].float() * SCALE * on.unsqueeze(1)).to(s["table"].dtype)
    if not c["train"]:
        return y
    d = s["dw"].float() if c["tied"] else torch.zeros((c["V"], c["E"]), device="cuda")
    at = torch.nonzero(on).squeeze(1)
    d.index_add_(0, ids[at], s["d_y"][at].float() * SCALE)
    return y, d.to(s["table"].dtype)


def _plain_distil(s):
    c, ids, T = s["case"], s["ids"], s["case"]["temperature"]
    dt = _dtype(c["dtype"])
    x, w, t = s["x"].float(), s["w"].float(), s["teacher"].float() / T
    on = ids[:, :1] >= 0
    at = ids.clamp(min=0)
    t = t - t.amax(1, keepdim=True)
    ln_q = t - torch.log(torch.exp(t).sum(1, keepdim=True))
    q = torch.exp(ln_q)
    z = (x @ w.t()) / T
    top = z.amax(1, keepdim=True)
    lse = torch.log(torch.exp(z - top).sum(1, keepdim=True)) + top
    ln_p = torch.where(on, z.gather(1, at) - lse, 0.0)
    loss = torch.where(on.squeeze(1), (q * (ln_q - ln_p)).sum(1), 0.0)
    out = loss, torch.where(on, lse, 0.0).squeeze(1), ln_p
    if not c["train"]:
        return out
    g = torch.exp(z - lse)
    g.scatter_add_(1, at, -q)
    g *= (s["d_loss"] / T).unsqueeze(1) * on
    return out + ((g @ w).to(dt), (g.t() @ x).to(dt))


def _numbered(s, count):
    """The sequence of every token."""
    return torch.repeat_interleave(torch.arange(count, device="cuda"), s["first"][1:] - s["first"][:-1], output_size=s["case"]["n"])


def _sums(s, values):
    """Sums of the rows of values over every sequence, as differences of running sums."""
    run = torch.nn.functional.pad(torch.cumsum(values, -1), (1, 0))
    return run[..., s["first"][1:]] - run[..., s["first"][:-1]]


def _plain_pref(s):
    c, on = s["case"], s["labels"] >= 0
    S = c["S"]
    seq = _numbered(s, 2 * S)
    # (sums over long sequences, of which a difference is taken)
    total = _sums(s, torch.where(on, s["ref"].double() - s["nll"].double(), 0.0))
    margin = total[:S] - total[S:]
    h = BETA * margin
    if c["form"] == "logistic":
        a, e = c["smoothing"], torch.exp(-h.abs())
        soft = torch.log1p(e)
        loss = (1.0 - a) * (soft + (-h).clamp(min=0.0)) + a * (soft + h.clamp(min=0.0))
        slope = BETA * (torch.where(h >= 0.0, 1.0 / (1.0 + e), e / (1.0 + e)) - (1.0 - a))
    elif c["form"] == "hinge":
        loss = (1.0 - h).clamp(min=0.0)
        slope = torch.where(h < 1.0, -BETA, 0.0)
    else:
        loss = (margin - 0.5 / BETA) ** 2
        slope = 2.0 * (margin - 0.5 / BETA)
    slope = slope * s["d_loss"]
    d_nll = torch.where(on, torch.cat((-slope, slope))[seq], 0.0)
    return loss.float(), margin.float(), d_nll.float()


def _plain_policy(s):
    c, on = s["case"], s["labels"] >= 0
    S, beta = c["S"], c["beta"]
    seq = _numbered(s, S)
    # (a ratio next to its bound is on one side or the other)
    gone = s["old"].double() - s["nll"].double()
    ratio = torch.exp(gone)
    adv = (s["adv"] if c["per_token"] else s["adv"][seq]).double()
    clipped = torch.where(adv > 0.0, ratio > 1.0 + CLIP[1], (ratio < 1.0 - CLIP[0]) & (adv < 0.0))
    held = torch.where(clipped, ratio.clamp(1.0 - CLIP[0], 1.0 + CLIP[1]), ratio)
    loss, slope = -held * adv, torch.where(clipped, 0.0, ratio * adv)
    kl = torch.zeros_like(loss)
    if beta > 0.0:
        d = s["nll"].double() - s["ref"].double()
        kl = torch.expm1(d) - d
        loss, slope = loss + beta * kl, slope + beta * torch.expm1(d)
    total = _sums(s, torch.where(on, torch.stack((loss, torch.ones_like(loss), clipped.double(), kl)), 0.0))
    count = total[1].clamp(min=1.0)
    share = 1.0 / count if c["mean"] else torch.ones_like(count)
    d_nll = torch.where(on, slope * (s["d_loss"] * share)[seq], 0.0)
    stats = torch.stack((total[1], total[2] / count, total[3] / count), 1)
    return (total[0] * share).float(), stats.float(), d_nll.float()


def _own(s):
    from paper_2502_02406_amd import binding as B

    c = s["case"]
    if "buffers" not in s:                   # what a program keeps from step to step
        f32 = dict(dtype=torch.float32, device="cuda")
        b = s["buffers"] = {}

        def workspace(nbytes):
            return torch.empty(nbytes, dtype=torch.uint8, device="cuda")

        if c["kind"] == "embed":
            b["y"] = torch.empty((c["n"], c["E"]), dtype=s["table"].dtype, device="cuda")
            if c["train"]:
                b["d_table"] = torch.empty_like(s["table"])
                b["ws"] = workspace(B.lvx_embed_workspace_bytes(c["n"], c["E"], c["V"]))
        elif c["kind"] == "distil":
            b["loss"], b["lse"] = torch.empty(c["n"], **f32), torch.empty(c["n"], **f32)
            b["top"] = torch.empty((c["n"], c["K"]), **f32)
            b["ws"] = workspace(B.lvx_distil_workspace_bytes(c["n"], c["E"], c["V"], c["K"], B.dtype_code(s["x"].dtype)))
            if c["train"]:
                b["dx"], b["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
        else:
            b["loss"], b["d_nll"] = torch.empty(c["S"], **f32), torch.empty(c["n"], **f32)
            b["margin"], b["stats"] = torch.empty(c["S"], **f32), torch.empty((c["S"], 3), **f32)
            size = B.lvx_preference_workspace_bytes if c["kind"] == "pref" else B.lvx_policy_workspace_bytes
            b["ws"] = workspace(size(c["n"], c["S"]))
    b = s["buffers"]
    if c["kind"] == "embed":
        B.lvx_embed_fwd(s["table"], s["ids"], b["y"], scale=SCALE)
        if not c["train"]:
            return b["y"]
        # (what the plain form adds to: a float32 gradient itself, a copy of a bf16 one)
        d_table = s["dw"] if c["tied"] and c["dtype"] == "f32" else b["d_table"].copy_(s["dw"]) if c["tied"] else b["d_table"]
        B.lvx_embed_bwd(s["d_y"], s["ids"], d_table, b["ws"], scale=SCALE, accumulate=c["tied"])
        return b["y"], d_table
    if c["kind"] == "distil":
        T = c["temperature"]
        B.lvx_distil_fwd(s["x"], s["w"], s["ids"], s["teacher"], b["loss"], b["lse"], b["top"], b["ws"], temperature=T)
        if not c["train"]:
            return b["loss"], b["lse"], b["top"]
        B.lvx_distil_bwd(s["x"], s["w"], s["ids"], s["teacher"], b["lse"], b["top"], s["d_loss"], b["dx"], b["dw"], b["ws"], temperature=T)
        return b["loss"], b["lse"], b["top"], b["dx"], b["dw"]
    if c["kind"] == "pref":
        B.lvx_preference(s["nll"], s["ref"], s["labels"], s["first"], b["loss"], b["margin"], s["d_loss"], b["d_nll"], b["ws"],
                         form=c["form"], beta=BETA, smoothing=c["smoothing"])
        return b["loss"], b["margin"], b["d_nll"]
    B.lvx_policy(s["nll"], s["old"], s["ref"] if c["beta"] > 0.0 else None, s["adv"], s["labels"], s["first"], b["loss"], b["stats"],
                 s["d_loss"], b["d_nll"], b["ws"], clip=CLIP, beta=c["beta"], mean=c["mean"])
    return b["loss"], b["stats"], b["d_nll"]


_PLAIN = {"embed": _plain_embed, "distil": _plain_distil, "pref": _plain_pref, "policy": _plain_policy}


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["kind"]](state)


def work(case):
    """Each input read once and each output written once.  Of a table, the rows that may be asked for, or (its gradient) all; of a
    vocabulary's products one for the loss and one for each gradient."""
    c = case
    if c["kind"] == "embed":
        e = 4 if c["dtype"] == "f32" else 2
        n, E, V = c["n"], c["E"], c["V"]
        m = n - int(n * c["ignored"])
        fwd = (min(m, V) + n) * E * e + 8 * n
        bwd = m * E * e + 8 * n + V * E * e * (2 if c["tied"] else 1)
        return {"bytes": fwd + (bwd if c["train"] else 0), "flops": (3.0 if c["train"] else 1.0) * m * E}
    if c["kind"] == "distil":
        e, t = (4 if c["dtype"] == "f32" else 2), (4 if c["teacher"] == "f32" else 2)
        n, E, V, K = c["n"], c["E"], c["V"], c["K"]
        m = n - int(n * c["ignored"])
        fwd = (m + V) * E * e + m * K * (8 + t + 4) + 8 * n
        bwd = 2 * (m + V) * E * e + m * K * (8 + t + 4) + 8 * n
        return {"bytes": fwd + (bwd if c["train"] else 0), "flops": (6.0 if c["train"] else 2.0) * m * V * E}
    n, S = c["n"], c["S"]
    if c["kind"] == "pref":
        return {"bytes": n * (4 + 4 + 8 + 4) + S * 28, "flops": 4.0 * n}
    return {"bytes": n * (4 + 4 + 8 + 4 + (4 if c["beta"] > 0.0 else 0) + (4 if c["per_token"] else 0)) + S * 32, "flops": 30.0 * n}


# ---- the definitions in float64 -------------------------------------------------------------

def _exact_embed(c, s):
    table, ids = s["table"].double(), s["ids"]
    y = torch.zeros((c["n"], c["E"]), dtype=torch.float64, device="cuda")
    words = torch.nonzero(ids >= 0).squeeze(1)
    y[words] = table[ids[words]] * SCALE
    if not c["train"]:
        return y
    # a row's gradient is the sum over where its id stands: the tokens in the order of their ids, a difference of running sums
    d = s["dw"].double() if c["tied"] else torch.zeros_like(table)
    order = words[torch.argsort(ids[words], stable=True)]
    found, times = torch.unique_consecutive(ids[order], return_counts=True)
    last = torch.cumsum(times, 0)
    for cols in torch.arange(c["E"], device="cuda").split(512):
        run = torch.cumsum(s["d_y"][order][:, cols].double(), 0)
        upto = run[last - 1]
        upto[1:] -= run[last[:-1] - 1]
        at = (found.unsqueeze(1), cols.unsqueeze(0))
        d[at] = d[at] + upto * SCALE
    return y, d


def _exact_distil(c, s):
    x, w, T = s["x"].double(), s["w"].double(), c["temperature"]
    n, K = c["n"], c["K"]
    loss, lse, dx = torch.zeros_like(x[:, 0]), torch.zeros_like(x[:, 0]), torch.zeros_like(x)
    ln_p = torch.zeros((n, K), dtype=torch.float64, device="cuda")
    dw = torch.zeros_like(w) if c["train"] else None
    for at in torch.nonzero(s["ids"][:, 0] >= 0).squeeze(1).split(512):
        xs, ids = x[at], s["ids"][at]
        z = (xs @ w.t()) / T
        ln = torch.log_softmax(z, 1)
        ln_q = torch.log_softmax(s["teacher"][at].double() / T, 1)
        lse[at] = torch.logsumexp(z, 1)
        ln_p[at] = torch.gather(ln, 1, ids)
        loss[at] = ((ln_q - ln_p[at]) * torch.exp(ln_q)).sum(1)
        if c["train"]:
            want = torch.zeros_like(z).scatter_(1, ids, torch.exp(ln_q))
            back = (torch.exp(ln) - want) * (s["d_loss"][at].double() / T)[:, None]
            dx[at] = back @ w
            dw += back.t().contiguous() @ xs
    return (loss, lse, ln_p, dx, dw) if c["train"] else (loss, lse, ln_p)


def _exact_pref(c, s):
    first, S = s["first"].tolist(), c["S"]
    on = (s["labels"] >= 0).double()
    d_nll = torch.zeros(c["n"], dtype=torch.float64, device="cuda")
    # the logarithm of what a sequence's likelihood has grown by
    grown = torch.stack([((s["ref"][a:b].double() - s["nll"][a:b].double()) * on[a:b]).sum() for a, b in zip(first, first[1:])])
    margin = (grown[:S] - grown[S:]).detach().requires_grad_()
    if c["form"] == "logistic":
        a = c["smoothing"]
        loss = -(1.0 - a) * torch.nn.functional.logsigmoid(BETA * margin) - a * torch.nn.functional.logsigmoid(-BETA * margin)
    elif c["form"] == "hinge":
        loss = torch.relu(1.0 - BETA * margin)
    else:
        loss = (margin - 1.0 / (2.0 * BETA)) ** 2
    slope, = torch.autograd.grad(loss, margin, s["d_loss"].double())
    for i, (a, b) in enumerate(zip(first, first[1:])):
        d_nll[a:b] = on[a:b] * (-slope[i] if i < S else slope[i - S])
    return loss.detach(), margin.detach(), d_nll


def _exact_policy(c, s):
    first, S, beta = s["first"].tolist(), c["S"], c["beta"]
    losses, stats = [], []
    d_nll = torch.zeros(c["n"], dtype=torch.float64, device="cuda")
    for i, (a, b) in enumerate(zip(first, first[1:])):
        at = a + torch.nonzero(s["labels"][a:b] >= 0).squeeze(1)
        count = len(at)
        if count == 0:
            losses.append(torch.zeros((), dtype=torch.float64, device="cuda"))
            stats.append(torch.zeros(3, dtype=torch.float64, device="cuda"))
            continue
        ln_p, ln_old = -s["nll"][at].double(), -s["old"][at].double()
        ratio = torch.exp(ln_p - ln_old)
        adv = s["adv"][at].double() if c["per_token"] else s["adv"][i].double().expand(count)
        free, bound = ratio * adv, ratio.clamp(1.0 - CLIP[0], 1.0 + CLIP[1]) * adv
        loss, slope = -torch.minimum(free, bound), torch.where(free <= bound, -free, 0.0)      # by ln_p
        kl = torch.zeros_like(loss)
        if beta > 0.0:
            behind = -s["ref"][at].double() - ln_p
            kl = torch.expm1(behind) - behind
            loss, slope = loss + beta * kl, slope - beta * torch.expm1(behind)
        over = count if c["mean"] else 1
        losses.append(loss.sum() / over)
        stats.append(torch.stack((torch.tensor(float(count), dtype=torch.float64, device="cuda"), (free > bound).double().mean(), kl.mean())))
        d_nll[at] = -slope * s["d_loss"][i].double() / over
    return torch.stack(losses), torch.stack(stats), d_nll


def exact(case, seed):
    """The definitions in float64."""
    return {"embed": _exact_embed, "distil": _exact_distil, "pref": _exact_pref, "policy": _exact_policy}[case["kind"]](case, _inputs(case, seed))
