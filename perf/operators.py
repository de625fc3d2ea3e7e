"""The operators of a training step, and what they are measured on.

A model over the hop stack learns two kinds of parameters: a table of embedding rows (one per word, category or node) that
stands in for features, and the weight matrices of its layers.  Four operators carry their step:

  lookup  out[i, :] = scale * table[token[i], :], zero where token[i] names no row;
  grad    its gradient: grad[v, :] = scale * (sum of up[i, :] over all i with token[i] = v), rows without a token zero;
  orth    a matrix G's update direction by Newton-Schulz products:  X = G / (|G|_F + eps), then, as often as asked for,
          A = X X^T,  X <- a X + (b A + c A A) X  (on the transpose where G has more rows than columns);
  muon    the whole step of a weight matrix around it:  M <- mu M + G,  U = G + mu M,
          W <- (1 - lr wd) W - lr orth(U).

listed() names the standing cases, draw(rng) gives another case of the same ranges, prepare(case, seed) makes what a
program has in hand before the call, run(state) is one pass: through the library's entry points where `own` is true, else
through elementary tensor operations in 32 bits.  exact(case, seed) is the result in 64 bits, work(case) what a pass cannot do without.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TORCH_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}
BYTES = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
COEFF = (3.4445, -4.7750, 2.0315)  # a, b, c of a Newton-Schulz step
EPS = 1e-7
LR, MU, DECAY = 0.02, 0.95, 0.01


def listed():
    return [
        # the rows of one mini-batch of nodes out of a table with a row per node: the smallest call
        dict(name="lookup_batch", kind="lookup", N=4_096, V=169_343, d=128, dtype="f32", out="f32", index="i32",
             ids="uniform", absent=0.0, scale=1.0),
        # the features of all nodes of a graph from the word each stands for, stored in bf16 for the hops; some have none
        dict(name="lookup_words_bf16", kind="lookup", N=507_001, V=32_768, d=100, dtype="f32", out="bf16", index="i64",
             ids="zipf", absent=0.05, scale=10.0),
        # a large batch from a table that no cache holds
        dict(name="lookup_large", kind="lookup", N=2_450_000, V=2_450_000, d=256, dtype="bf16", out="bf16", index="i32",
             ids="uniform", absent=0.0, scale=16.0),
        # the gradient of one mini-batch's rows
        dict(name="grad_batch", kind="grad", N=4_096, V=10_000, d=128, dtype="f32", out="f32", index="i32",
             ids="uniform", absent=0.0, scale=1.0),
        # every node has one of a few categories: thousands of rows meet in each, odd columns
        dict(name="grad_categories", kind="grad", N=169_343, V=47, d=47, dtype="f32", out="f32", index="i32",
             ids="zipf", absent=0.0, scale=1.0),
        # words of a graph's nodes, gradients stored in bf16, the table in fp32
        dict(name="grad_words_bf16", kind="grad", N=507_001, V=32_768, d=100, dtype="bf16", out="f32", index="i64",
             ids="zipf", absent=0.05, scale=10.0),
        # a row per node, as many tokens as rows: nothing is shared, both sides are read and written from memory
        dict(name="grad_large", kind="grad", N=2_450_000, V=2_450_000, d=100, dtype="f32", out="f32", index="i32",
             ids="uniform", absent=0.0, scale=1.0),
        # the hidden layers of a model over the stack
        dict(name="orth_hidden", kind="orth", rows=256, cols=256, count=2, dtype="f32", steps=5),
        # the first layer on 602 features: tall, odd, in bf16
        dict(name="orth_features_bf16", kind="orth", rows=602, cols=256, count=1, dtype="bf16", steps=5),
        # a large square matrix
        dict(name="orth_large", kind="orth", rows=4096, cols=4096, count=1, dtype="f32", steps=5),
        # the output layer of a model: the smallest step
        dict(name="muon_classes", kind="muon", rows=256, cols=40, count=1, dtype="f32", steps=5),
        # two layers of a wide model at once, gradients in bf16
        dict(name="muon_wide_bf16", kind="muon", rows=1024, cols=4096, count=2, dtype="bf16", steps=5),
    ]


def draw(rng):
    """One more case of the ranges above.  Sizes are spread over their logarithms."""
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["lookup", "lookup", "grad", "grad", "grad", "orth", "orth", "muon"])
    if kind in ("lookup", "grad"):
        d = rng.choice([64, 100, 128, 256, size(16, 640), size(16, 640)])
        return dict(kind=kind, N=min(size(500, 2_450_000), 600_000_000 // d), V=min(size(40, 2_450_000), 240_000_000 // d), d=d,
                    dtype=rng.choice(["f32", "bf16"]), out=rng.choice(["f32", "f32", "bf16"]), index=rng.choice(["i32", "i64"]),
                    ids=rng.choice(["uniform", "zipf"]), absent=rng.choice([0.0, 0.0, 0.05, 0.3]), scale=rng.choice([1.0, 16.0]))
    rows, cols = size(16, 4096), size(16, 4096)
    if rng.random() < 0.25:
        cols = rows
    count = rng.choice([1, 1, 2, 4])
    while count > 1 and count * min(rows, cols) ** 2 * max(rows, cols) > 4096 ** 3:
        count //= 2
    return dict(kind=kind, rows=rows, cols=cols, count=count, dtype=rng.choice(["f32", "bf16"]), steps=5)


# ---- inputs ----------------------------------------------------------------------------------------

ZIPF = 1.05  # a word's share falls with this power of its rank


def _shares(c):
    """The probability of every row of the table, by rank."""
    w = np.arange(1, c["V"] + 1, dtype=np.float64) ** -(ZIPF if c["ids"] == "zipf" else 0.0)
    return w / w.sum()


def _tokens(c, gen):
    N, V = c["N"], c["V"]
    if c["ids"] == "uniform":
        t = torch.randint(V, (N,), generator=gen, device="cuda")
    else:  # ranks by their shares, then names without an order
        edge = torch.from_numpy(np.cumsum(_shares(c))).cuda()
        t = torch.searchsorted(edge, torch.rand(N, generator=gen, device="cuda", dtype=torch.float64)).clamp_(max=V - 1)
        t = torch.randperm(V, generator=gen, device="cuda")[t]
    if c["absent"]:
        t.masked_fill_(torch.rand(N, generator=gen, device="cuda") < c["absent"], -1)
    return t.to(TORCH_TYPE[c["index"]])


def _gradient(c, gen):
    """Gradients of weight matrices: a few strong directions (those of the batch's errors) over a floor of noise."""
    n, r, s = c["count"], c["rows"], c["cols"]
    k = max(1, min(r, s) // 8)
    left = torch.randn(n, r, k, generator=gen, device="cuda") * torch.arange(1, k + 1, device="cuda") ** -0.5
    right = torch.randn(n, k, s, generator=gen, device="cuda")
    return 1e-3 * (left @ right + 0.2 * torch.randn(n, r, s, generator=gen, device="cuda"))


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if c["kind"] == "lookup":
        return dict(c=c, tokens=_tokens(c, gen), table=torch.randn(c["V"], c["d"], generator=gen, device="cuda").to(TORCH_TYPE[c["dtype"]]))
    if c["kind"] == "grad":
        up = torch.randn(c["N"], c["d"], generator=gen, device="cuda") * 1e-2
        return dict(c=c, tokens=_tokens(c, gen), up=up.to(TORCH_TYPE[c["dtype"]]))
    G = _gradient(c, gen).to(TORCH_TYPE[c["dtype"]])
    if c["kind"] == "orth":
        return dict(c=c, G=G)
    return dict(c=c, G=G, M=5 * _gradient(c, gen), W=torch.randn(G.shape, generator=gen, device="cuda") / math.sqrt(c["rows"]))


# ---- one pass --------------------------------------------------------------------------------------

def run(state):
    c = state["c"]
    if own:
        return _run_own(c, state)
    if c["kind"] == "lookup":
        tokens = state["tokens"].long()
        known = (tokens >= 0) & (tokens < c["V"])
        rows = state["table"][tokens.clamp(0, c["V"] - 1)].float() * c["scale"]
        return torch.where(known[:, None], rows, torch.zeros_like(rows)).to(TORCH_TYPE[c["out"]])
    if c["kind"] == "grad":
        tokens = state["tokens"].long()
        tokens = torch.where((tokens >= 0) & (tokens < c["V"]), tokens, c["V"])  # (one row more takes what belongs to none)
        sums = torch.zeros(c["V"] + 1, c["d"], device=tokens.device).index_add_(0, tokens, state["up"].float())
        return (sums[:-1] * c["scale"]).to(TORCH_TYPE[c["out"]])
    if c["kind"] == "orth":
        return _newton_schulz(state["G"].float(), c["steps"]).to(state["G"].dtype)
    M = MU * state["M"] + state["G"].float()
    O = _newton_schulz(state["G"].float() + MU * M, c["steps"])
    return {"W": (1 - LR * DECAY) * state["W"] - LR * O, "M": M}


def _newton_schulz(G, steps):
    a, b, c = COEFF
    X = G / (torch.sqrt((G * G).sum(dim=(-2, -1), keepdim=True)) + EPS)
    tall = X.shape[-2] > X.shape[-1]
    if tall:
        X = X.transpose(-2, -1).contiguous()
    for _ in range(steps):
        A = X @ X.transpose(-2, -1).contiguous()
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.transpose(-2, -1).contiguous() if tall else X


def _run_own(c, state):
    import paper_2207_12000_amd as gp
    if c["kind"] == "lookup":
        return gp.embedding_tensors(state["table"], state["tokens"], scale=c["scale"], out_dtype=TORCH_TYPE[c["out"]])
    if c["kind"] == "grad":
        return gp.embedding_grad_tensors(state["tokens"], state["up"], c["V"], scale=c["scale"], out_dtype=TORCH_TYPE[c["out"]])
    if c["kind"] == "orth":
        return gp.orthogonalize_tensors(state["G"], steps=c["steps"], coeff=COEFF, eps=EPS)
    W, M = torch.empty_like(state["W"]), torch.empty_like(state["M"])
    gp.muon_step_tensors(state["W"], state["M"], state["G"], lr=LR, momentum=MU, weight_decay=DECAY, nesterov=True,
                         steps=c["steps"], coeff=COEFF, eps=EPS, W_out=W, M_out=M)
    return {"W": W, "M": M}


# ---- the same from the definitions, in 64 bits -------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["kind"] in ("lookup", "grad"):
        tokens = s["tokens"].long()
        named = torch.nonzero((tokens >= 0) & (tokens < c["V"])).flatten()
        if c["kind"] == "lookup":
            out = torch.zeros(c["N"], c["d"], dtype=torch.float64, device=tokens.device)
            out[named] = s["table"].double()[tokens[named]] * float(c["scale"])
            return out
        # every token's rows next to one another, running sums by halving steps inside them
        order = named[torch.sort(tokens[named], stable=True).indices]
        tok, rows = tokens[order], s["up"].double()[order]
        while True:  # pairs of neighbours of one token become one row, until none are left
            if tok.numel() < 2:
                break
            new = torch.ones_like(tok, dtype=torch.bool)
            new[1:] = tok[1:] != tok[:-1]
            if bool(new.all()):
                break
            first = torch.nonzero(new).flatten()
            place = torch.arange(tok.numel(), device=tok.device) - first[torch.cumsum(new, 0) - 1]
            keep = torch.nonzero(place % 2 == 0).flatten()
            follows = keep + 1
            paired = (follows < tok.numel()) & (place[follows.clamp(max=tok.numel() - 1)] % 2 == 1)
            merged = rows[keep]
            merged[paired] += rows[follows[paired]]
            tok, rows = tok[keep], merged
        out = torch.zeros(c["V"], c["d"], dtype=torch.float64, device=tokens.device)
        out[tok] = rows * float(c["scale"])
        return out
    G = s["G"].double()
    if c["kind"] == "orth":
        return torch.stack([_polynomial(g, c["steps"]) for g in G])
    M = MU * s["M"].double() + G
    O = torch.stack([_polynomial(u, c["steps"]) for u in G + MU * M])
    return {"W": s["W"].double() - LR * DECAY * s["W"].double() - LR * O, "M": M}


def _polynomial(G, steps):
    """Newton-Schulz steps of one matrix in 64 bits, from the side of its shorter dimension."""
    a, b, c = COEFF
    one = torch.eye(min(G.shape), dtype=G.dtype, device=G.device)
    X = G / (G.pow(2).sum().sqrt() + EPS)
    for _ in range(steps):
        if G.shape[0] <= G.shape[1]:
            S = X.mm(X.t())
            X = (a * one + S.mm(b * one + c * S)).mm(X)
        else:
            S = X.t().mm(X)
            X = X.mm(a * one + S.mm(b * one + c * S))
    return X


# ---- what a pass cannot do without -------------------------------------------------------------------

def work(case):
    c = dict(case)
    if c["kind"] in ("lookup", "grad"):
        N, V, d = c["N"], c["V"], c["d"]
        named = N * (1 - c["absent"])
        if c["kind"] == "grad":  # the rows of tokens that name one, the whole table's gradient
            return {"bytes": int(N * BYTES[c["index"]] + named * d * BYTES[c["dtype"]] + V * d * BYTES[c["out"]]), "flops": int(named * d)}
        distinct = float(-np.expm1(named * np.log1p(-np.minimum(_shares(c), 1 - 1e-12))).sum())  # rows expected to be named
        return {"bytes": int(N * BYTES[c["index"]] + distinct * d * BYTES[c["dtype"]] + N * d * BYTES[c["out"]]), "flops": int(named * d)}
    m, n = sorted((c["rows"], c["cols"]))
    elements = c["count"] * m * n
    # a step: X X^T and A A are symmetric, half of each will do; then B X
    flops = c["count"] * c["steps"] * (3 * m * m * n + m ** 3)
    if c["kind"] == "orth":
        return {"bytes": 2 * elements * BYTES[c["dtype"]], "flops": flops}
    return {"bytes": elements * (BYTES[c["dtype"]] + 16), "flops": flops}
