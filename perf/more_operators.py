"""What a model over the hop stack normalises, answers with and learns from, and what these operators are measured on.

  norm         y = (x - m) r w + b  row by row,  m = mean(x),  r = 1 / sqrt(mean((x - m)^2) + eps);  (m, r) are kept for
  norm_grad    h = (x - m) r,  u = w g:  dx = r (u - mean(u) - h mean(u h)),  dw = sum over rows of g h,  db = sum of g;
  answer       z = s x,  log p = z - log(sum exp z):  log p of one named class a row (0 where none is named), the entropy
               -sum p log p, and the k largest classes with their log p (ties go to the lower class);
  answer_grad  dx_j = s (g1 ([j = named] - p_j) - g2 p_j (log p_j + entropy)), g1 and g2 the gradients of log p and entropy;
  distill      a teacher names K classes a row and their logits v (an entry outside the classes is none):
               q = softmax(v / T),  loss = T^2 sum q (log q - log p),  p = softmax(x / T) over all classes, and at once
               dx_j = g T (p_j - sum of q over the entries that name j), where asked for.

listed() names the standing cases, draw(rng) gives another case of the same ranges, prepare(case, seed) makes what a
program has in hand before the call, run(state) is one pass: through the library's entry points where `own` is true, else
through elementary tensor operations in 32 bits.  exact(case, seed) is the result in 64 bits, work(case) what a pass cannot do without.
"""
from __future__ import annotations

import math

import torch

own = False

TORCH_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}
BYTES = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
EPS = 1e-5


def listed():
    return [
        # the features of one mini-batch of nodes: the smallest call
        dict(name="norm_batch", kind="norm", N=4_096, d=128, dtype="f32"),
        # the features of all nodes of a graph, stored in bf16, rows of 200 bytes
        dict(name="norm_nodes_bf16", kind="norm", N=507_001, d=100, dtype="bf16"),
        # the first layer's gradient of a mini-batch: the smallest backward pass, where weights' sums have few rows
        dict(name="norm_grad_batch", kind="norm_grad", N=1_000, d=256, dtype="f32"),
        # all nodes of a graph with wide features, whose rows end inside a line of memory
        dict(name="norm_grad_nodes", kind="norm_grad", N=232_965, d=602, dtype="f32"),
        # the wide hidden layer of a large batch
        dict(name="norm_grad_wide_bf16", kind="norm_grad", N=16_384, d=4_096, dtype="bf16"),
        # what a classifier says of all nodes of a graph, five alternatives each
        dict(name="answer_nodes", kind="answer", N=169_343, C=40, k=5, dtype="f32", index="i64", scale=1.0, absent=0.3, hidden=0.0),
        # one masked word out of a table of them, some ruled out: a single row
        dict(name="answer_one_word", kind="answer", N=1, C=391_000, k=20, dtype="f32", index="i64", scale=0.7, absent=0.0, hidden=0.1),
        # the words of a large batch, logits stored in bf16, where equal ones are common
        dict(name="answer_words_bf16", kind="answer", N=4_096, C=32_768, k=8, dtype="bf16", index="i32", scale=1.0, absent=0.1, hidden=0.0),
        # the gradient of a node classifier's logits from its labels, few of which are known, and its entropy
        dict(name="answer_grad_nodes", kind="answer_grad", N=2_450_000, C=47, dtype="f32", index="i64", scale=1.0, absent=0.9),
        # one mini-batch of a small model that learns from a larger one's five best: loss and gradient
        dict(name="distill_batch", kind="distill", N=1_000, C=172, K=5, dtype="f32", index="i32", T=2.0, absent=0.0, grad=True),
        # all nodes of a graph
        dict(name="distill_nodes", kind="distill", N=507_001, C=47, K=8, dtype="f32", index="i32", T=4.0, absent=0.1, grad=True),
        # words: a long list of a teacher's, in bf16
        dict(name="distill_words_bf16", kind="distill", N=4_096, C=32_768, K=32, dtype="bf16", index="i64", T=1.0, absent=0.0, grad=True),
    ]


def draw(rng):
    """One more case of the ranges above.  Sizes are spread over their logarithms."""
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["norm", "norm_grad", "norm_grad", "answer", "answer", "answer_grad", "distill", "distill"])
    dtype, index = rng.choice(["f32", "bf16"]), rng.choice(["i32", "i64"])
    if kind in ("norm", "norm_grad"):
        d = rng.choice([64, 100, 128, 256, 602, size(8, 8_192), size(8, 8_192)])
        return dict(kind=kind, N=min(size(8, 2_450_000), 140_000_000 // d), d=d, dtype=dtype)
    C = rng.choice([40, 47, 172, size(2, 400_000), size(2, 400_000)])
    N = min(size(1, 2_450_000), 134_000_000 // C)
    absent = rng.choice([0.0, 0.1, 0.5])
    if kind == "answer":
        return dict(kind=kind, N=N, C=C, k=min(C, rng.choice([0, 1, 5, 8, 20, 64])), dtype=dtype, index=index, scale=rng.choice([1.0, 0.7]),
                    absent=absent, hidden=rng.choice([0.0, 0.1]))
    if kind == "answer_grad":
        return dict(kind=kind, N=N, C=C, dtype=dtype, index=index, scale=rng.choice([1.0, 0.7]), absent=absent)
    return dict(kind=kind, N=N, C=C, K=min(C, rng.choice([1, 5, 8, 32, 64])), dtype=dtype, index=index, T=rng.choice([1.0, 2.0, 4.0]),
                absent=absent, grad=rng.random() < 0.7)


# ---- inputs ----------------------------------------------------------------------------------------

def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _row_stats(x):
    x = x.double()
    m = x.mean(1)
    return torch.stack([m, 1 / torch.sqrt(((x - m[:, None]) ** 2).mean(1) + EPS)], 1).float()


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if c["kind"] in ("norm", "norm_grad"):
        # every column has a scale of its own, every row an offset
        x = (_normal(gen, c["N"], c["d"]) * (0.5 + torch.rand(c["d"], generator=gen, device="cuda")) + _normal(gen, c["N"], 1)).to(TORCH_TYPE[c["dtype"]])
        s = dict(c=c, x=x, w=1 + 0.2 * _normal(gen, c["d"]), b=0.1 * _normal(gen, c["d"]))
        if c["kind"] == "norm_grad":
            s["g"] = (1e-2 * _normal(gen, c["N"], c["d"])).to(x.dtype)
            s["stats"] = _row_stats(x)
        return s
    N, C = c["N"], c["C"]
    x = (3 * _normal(gen, N, C)).to(TORCH_TYPE[c["dtype"]])
    if c["kind"] == "distill":
        # the teacher's classes: K different ones a row, best first, which the student is for as well, to a degree
        K = c["K"]
        first = torch.randint(C, (N, 1), generator=gen, device="cuda")
        classes = (first + torch.arange(K, device="cuda") * (C // K)) % C
        logits = (2 * _normal(gen, N, K)).sort(1, descending=True).values + 4
        x.scatter_add_(1, classes, (0.8 * logits).to(x.dtype))
        if c["absent"]:  # shorter lists, and nodes without one
            keep = (torch.rand(N, 1, generator=gen, device="cuda") * (1 + c["absent"]) * K).floor()
            classes.masked_fill_(torch.arange(K, device="cuda") >= keep, -1)
        return dict(c=c, x=x, classes=classes.to(TORCH_TYPE[c["index"]]), logits=logits.to(x.dtype),
                    g=torch.full((N,), 1 / N, device="cuda") * (1 + 0.5 * torch.rand(N, generator=gen, device="cuda")))
    tokens = torch.randint(C, (N,), generator=gen, device="cuda")
    if c.get("hidden"):
        x.masked_fill_(torch.rand(1, C, generator=gen, device="cuda") < c["hidden"], -math.inf)
        x[:, 0] = 1.0  # (one is always left)
    if c["absent"]:
        tokens.masked_fill_(torch.rand(N, generator=gen, device="cuda") < c["absent"], -1)
    s = dict(c=c, x=x, tokens=tokens.to(TORCH_TYPE[c["index"]]))
    if c["kind"] == "answer_grad":
        part = max(1, (1 << 25) // C)
        kept = [_kept(x[i:i + part], c["scale"]) for i in range(0, N, part)]
        s["stats"], s["entropy"] = torch.cat([a for a, _ in kept]), torch.cat([b for _, b in kept])
        s["g1"], s["g2"] = -(0.5 + torch.rand(N, generator=gen, device="cuda")) / N, 0.1 * _normal(gen, N) / N
    return s


def _kept(x, scale):
    """What the answers of these rows leave for their gradient: (the largest logit, the log of the sum behind it), and the entropy."""
    x = x.double()
    top = x.max(1).values
    z = (x - top[:, None]) * scale
    e = z.exp()
    total = e.sum(1)
    return torch.stack([top, total.log()], 1).float(), (total.log() - (e * z).sum(1) / total).float()


# ---- one pass --------------------------------------------------------------------------------------

def run(state):
    c = state["c"]
    if own:
        return _run_own(c, state)
    x = state["x"].float()
    if c["kind"] == "norm":
        m = x.mean(1, keepdim=True)
        x = x - m
        r = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
        return {"y": (x * r * state["w"] + state["b"]).to(state["x"].dtype), "stats": torch.cat([m, r], 1)}
    if c["kind"] == "norm_grad":
        m, r = state["stats"][:, :1], state["stats"][:, 1:]
        g = state["g"].float()
        h = (x - m) * r
        u = g * state["w"]
        dx = r * (u - u.mean(1, keepdim=True) - h * (u * h).mean(1, keepdim=True))
        return {"x_grad": dx.to(state["x"].dtype), "weight_grad": (g * h).sum(0), "bias_grad": g.sum(0)}
    if c["kind"] == "answer":
        top = x.max(1, keepdim=True).values
        z = (x - top) * c["scale"]
        e = torch.exp(z)
        total = e.sum(1, keepdim=True)
        log_total = torch.log(total)
        tokens = state["tokens"].long()
        named = (tokens >= 0) & (tokens < c["C"])
        logp = torch.where(named, (z.gather(1, tokens.clamp(0, c["C"] - 1)[:, None]) - log_total)[:, 0], 0.0)
        entropy = (log_total - (e * z.clamp(min=-1e4)).sum(1, keepdim=True) / total)[:, 0]
        out = {"logp": logp, "entropy": entropy}
        if c["k"]:
            # logits as whole numbers of the same order, the class below them: no two are equal
            bits = (x + 0.0).view(torch.int32).long()
            order = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF)) * (1 << 20) + (c["C"] - 1 - torch.arange(c["C"], device=x.device))
            order = torch.topk(order, c["k"], dim=1).values
            classes = c["C"] - 1 - (order & ((1 << 20) - 1))
            top_logp = z.gather(1, classes) - log_total
            out["top_logp"] = top_logp
            out["top_index"] = torch.where(torch.isinf(top_logp), -1, classes).int()
        return out
    if c["kind"] == "answer_grad":
        logp = (x - state["stats"][:, :1]) * c["scale"] - state["stats"][:, 1:]
        p = torch.exp(logp)
        tokens = state["tokens"].long()
        named = (tokens >= 0) & (tokens < c["C"])
        g1 = torch.where(named, state["g1"], 0.0)[:, None]
        dx = -g1 * p - state["g2"][:, None] * p * (logp + state["entropy"][:, None])
        dx.scatter_add_(1, tokens.clamp(0, c["C"] - 1)[:, None], g1)
        return (dx * c["scale"]).to(state["x"].dtype)
    T = c["T"]
    classes = state["classes"].long()
    named = (classes >= 0) & (classes < c["C"])
    v = torch.where(named, state["logits"].float() / T, -math.inf)
    v = v - v.max(1, keepdim=True).values.clamp(min=-3e38)
    e = torch.exp(v)
    total = e.sum(1, keepdim=True)
    some = total > 0
    q = torch.where(some, e / total, 0.0)
    z = (x - x.max(1, keepdim=True).values) / T
    logp = z - torch.log(torch.exp(z).sum(1, keepdim=True))
    at = classes.clamp(0, c["C"] - 1)
    terms = torch.where(named, q * (v - torch.log(total) - logp.gather(1, at)), 0.0)
    out = {"loss": T * T * terms.sum(1)}
    if c["grad"]:
        dx = torch.where(some, torch.exp(logp), 0.0).scatter_add_(1, at, -q)
        out["grad"] = (dx * (T * state["g"][:, None])).to(state["x"].dtype)
    return out


def _run_own(c, s):
    import paper_2207_12000_amd as gp
    if c["kind"] == "norm":
        stats = torch.empty(c["N"], 2, device=s["x"].device)
        return {"y": gp.layer_norm_tensors(s["x"], s["w"], s["b"], eps=EPS, stats=stats), "stats": stats}
    if c["kind"] == "norm_grad":
        x_grad, weight_grad, bias_grad = gp.layer_norm_grad_tensors(s["g"], s["x"], s["stats"], s["w"])
        return {"x_grad": x_grad, "weight_grad": weight_grad, "bias_grad": bias_grad}
    if c["kind"] == "answer":
        a = gp.log_probs_tensors(s["x"], s["tokens"], scale=c["scale"], top=c["k"])
        out = {"logp": a.logp, "entropy": a.entropy}
        return {**out, "top_logp": a.top_logp, "top_index": a.top_index} if c["k"] else out
    if c["kind"] == "answer_grad":
        return gp.log_probs_grad_tensors(s["x"], s["tokens"], s["stats"], scale=c["scale"], entropy=s["entropy"], grad_logp=s["g1"], grad_entropy=s["g2"])
    if not c["grad"]:
        return {"loss": gp.distill_tensors(s["x"], s["classes"], s["logits"], temperature=c["T"])}
    loss, grad = gp.distill_tensors(s["x"], s["classes"], s["logits"], temperature=c["T"], grad_loss=s["g"])
    return {"loss": loss, "grad": grad}


# ---- the same from the definitions, in 64 bits -------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["kind"] in ("norm", "norm_grad"):
        wide = {k: s[k].double() for k in ("x", "w", "b", "g", "stats") if k in s}
        part, got = max(1, (1 << 26) // c["d"]), []
        for i in range(0, c["N"], part):
            x = wide["x"][i:i + part]
            if c["kind"] == "norm":
                var, m = torch.var_mean(x, 1, correction=0)
                r = (var + EPS).pow(-0.5)
                got.append(((x - m[:, None]) * r[:, None] * wide["w"] + wide["b"], torch.stack([m, r], 1)))
                continue
            m, r = wide["stats"][i:i + part].unbind(1)
            g = wide["g"][i:i + part]
            h = torch.addcmul((-m * r)[:, None], x, r[:, None])
            # dx = r (I - 1 1^T / d - h h^T / d) W g
            u = g.mul(wide["w"])
            dx = u - (u.sum(1) / c["d"]).unsqueeze(1)
            dx = (dx - h * ((h * u).sum(1) / c["d"]).unsqueeze(1)) * r[:, None]
            got.append((dx, g.mul(h).sum(0), g.sum(0)))
        if c["kind"] == "norm":
            return {"y": torch.cat([a for a, _ in got]), "stats": torch.cat([b for _, b in got])}
        return {"x_grad": torch.cat([a for a, _, _ in got]), "weight_grad": sum(b for _, b, _ in got), "bias_grad": sum(b for _, _, b in got)}
    part = max(1, (1 << 26) // c["C"])
    rows = [_exact_rows(c, {k: v[i:i + part] for k, v in s.items() if k != "c"}) for i in range(0, c["N"], part)]
    if not isinstance(rows[0], dict):
        return torch.cat(rows)
    return {k: None if rows[0][k] is None else torch.cat([r[k] for r in rows]) for k in rows[0]}


def _exact_rows(c, s):
    C = c["C"]
    x = s["x"].double()
    if c["kind"] == "answer":
        logp = torch.log_softmax(x * c["scale"], 1)
        named = (s["tokens"] >= 0).nonzero().flatten()
        got = torch.zeros(x.shape[0], dtype=x.dtype, device=x.device)
        got[named] = logp[named, s["tokens"][named].long()]
        out = {"logp": got, "entropy": torch.special.entr(logp.exp()).sum(1)}
        if c["k"]:
            out["top_logp"], out["top_index"] = torch.topk(logp, c["k"], dim=1).values, None
        return out
    if c["kind"] == "answer_grad":
        logp = (x - s["stats"][:, :1].double()) * c["scale"] - s["stats"][:, 1:].double()
        mine = torch.zeros_like(x)
        named = (s["tokens"] >= 0).nonzero().flatten()
        mine[named, s["tokens"][named].long()] = 1.0
        by_logp = torch.zeros_like(x)
        by_logp[named] = mine[named] - logp[named].exp()
        by_entropy = -logp.exp() * (logp + s["entropy"].double()[:, None])
        return c["scale"] * (s["g1"].double()[:, None] * by_logp + s["g2"].double()[:, None] * by_entropy)
    T = float(c["T"])
    known = s["classes"] >= 0
    some = known.any(1)
    logq = torch.log_softmax((s["logits"].double() / T).masked_fill(~known, -math.inf), 1)
    q = torch.where(known, logq.exp(), torch.zeros_like(logq))
    logp = torch.log_softmax(x / T, 1)
    at = torch.where(known, s["classes"].long(), torch.zeros_like(s["classes"], dtype=torch.long))
    gap = torch.where(known, logq - logp.gather(1, at), torch.zeros_like(logq))
    out = {"loss": T * T * (q * gap).sum(1)}
    if c["grad"]:
        full = torch.zeros_like(x).scatter_add_(1, at, q)
        out["grad"] = torch.where(some[:, None], (logp.exp() - full) * (T * s["g"].double())[:, None], torch.zeros_like(x))
    return out


# ---- what a pass cannot do without -------------------------------------------------------------------

def work(case):
    c = dict(case)
    size, N = BYTES[c["dtype"]], c["N"]
    if c["kind"] == "norm":
        return {"bytes": 2 * N * c["d"] * size + 8 * N + 8 * c["d"], "flops": 8 * N * c["d"]}
    if c["kind"] == "norm_grad":
        return {"bytes": 3 * N * c["d"] * size + 8 * N + 12 * c["d"], "flops": 15 * N * c["d"]}
    cells = N * c["C"]
    if c["kind"] == "answer":
        return {"bytes": cells * size + N * (BYTES[c["index"]] + 8 + 8 * c["k"]), "flops": 6 * cells}
    if c["kind"] == "answer_grad":
        return {"bytes": 2 * cells * size + N * (BYTES[c["index"]] + 20), "flops": 8 * cells}
    listed_bytes = N * c["K"] * (BYTES[c["index"]] + size) + 4 * N
    if not c["grad"]:
        return {"bytes": cells * size + listed_bytes, "flops": 4 * cells}
    return {"bytes": 2 * cells * size + listed_bytes + 4 * N, "flops": 7 * cells}
