"""Tensors to write that share memory with what a call reads are refused, seen without a GPU: by then a call has only its tensors' places to go by."""
import random

import pytest

import paper_2207_12000_amd as gp


def places(t):
    """The bytes that a tensor's elements take."""
    import numpy as np
    at = np.array([0])
    for n, step in zip(t.shape, t.stride()):
        at = (at[:, None] + np.arange(n) * step).ravel()
    size = t.element_size()
    return {int(t.data_ptr() + size * a + b) for a in at for b in range(size)}


def test_overlap_is_that_of_the_elements():
    import torch
    rng = random.Random(0)
    flat = torch.zeros(400, dtype=torch.int32)
    seen = [0, 0, 0]
    for _ in range(4000):
        ts = []
        step = rng.randint(1, 12)
        for _ in range(2):
            if rng.random() < 0.2:
                step = rng.randint(1, 12)
            base = flat.view(torch.int16) if rng.random() < 0.3 else flat
            d, N = rng.randint(0, step), rng.randint(0, 6)
            ts.append(base.as_strided((N, d), (step * 4 // base.element_size(), 1), rng.randint(0, 80)))
        a, b = ts
        real = bool(places(a) & places(b))
        said = gp._overlap(a, b)
        assert said == gp._overlap(b, a)
        rows = [gp._memory(t) for t in ts]
        if rows[0][3] > 1 and rows[1][3] > 1 and rows[0][1] != rows[1][1]:
            assert said or not real  # (of two distances: not told apart where they lie between each other's ends)
        else:
            assert said == real, (rows, real)
        seen[real + (said and not real) * 2] += 1
    assert min(seen[:2]) > 500


def tensors():
    import torch
    flat = torch.zeros(8 * 40)
    buffer = flat.view(8, 40)
    x, beside = buffer[:4, :11], buffer[:4, 11:22]
    return dict(flat=flat, x=x, beside=beside, behind=buffer[4:, :11], within=buffer[:4, 5:16], later=buffer[1:5, :11], stats=torch.zeros(4, 2), tokens=torch.zeros(4, dtype=torch.int32),
                at=torch.zeros(4, 3, dtype=torch.int32), v=torch.zeros(4, 3), g=torch.zeros(4), w=torch.zeros(11), b=torch.zeros(11), up=torch.zeros(4, 11))


REFUSED = {
    "layer_norm": lambda t, o: gp.layer_norm_tensors(t["x"], t["w"], t["b"], out=o),
    "layer_norm_grad": lambda t, o: gp.layer_norm_grad_tensors(t["up"], t["x"], t["stats"], t["w"], x_grad=o),
    "layer_norm_grad of that": lambda t, o: gp.layer_norm_grad_tensors(t["x"], t["up"], t["stats"], t["w"], x_grad=o),
    "log_probs_grad": lambda t, o: gp.log_probs_grad_tensors(t["x"], t["tokens"], t["stats"], grad_logp=t["g"], out=o),
    "distill": lambda t, o: gp.distill_tensors(t["x"], t["at"], t["v"], grad_loss=t["g"], out=o),
    "distill_grad": lambda t, o: gp.distill_grad_tensors(t["x"], t["at"], t["v"], t["stats"], t["g"], out=o),
}


@pytest.mark.parametrize("name", REFUSED)
def test_rows_to_write_over_the_rows_that_are_read(name):
    t = tensors()
    for where in ("within", "later"):
        with pytest.raises(ValueError, match="overlap"):
            REFUSED[name](t, t[where])
    with pytest.raises(ValueError, match="on the GPU" if "layer_norm" in name else "overlap"):
        REFUSED[name](t, t["x"])
    for where in ("beside", "behind"):
        with pytest.raises(ValueError, match="on the GPU"):
            REFUSED[name](t, t[where])


def test_other_tensors_to_write_over_what_is_read_or_written():
    import torch
    t = tensors()
    x, up, stats, w, b, tokens, g, at, v = (t[k] for k in ("x", "up", "stats", "w", "b", "tokens", "g", "at", "v"))
    one = t["flat"][:11]
    wide = torch.zeros(4, 11)
    same_memory = wide.view(torch.bfloat16)[:, :11]
    few, square = torch.zeros(1, 11), torch.zeros(4, 4)
    rows = torch.zeros(4, 11)
    for call in (lambda: gp.layer_norm_tensors(x[:1], one, out=one[None]), lambda: gp.layer_norm_tensors(few, w, b, out=b[None]), lambda: gp.layer_norm_tensors(wide, out=same_memory),
                 lambda: gp.layer_norm_tensors(rows[:3], out=rows[1:]),
                 lambda: gp.layer_norm_grad_tensors(up[:1].expand(4, 11), rows, stats, x_grad=up),  # one row that stands for all, in the rows to write
                 lambda: gp.layer_norm_grad_tensors(up[:1], few, stats[:1], w, x_grad=w[None]),
                 lambda: gp.layer_norm_grad_tensors(up, x, stats, w, weight_grad=x[0]), lambda: gp.layer_norm_grad_tensors(up, x, stats, w, bias_grad=up[3]),
                 lambda: gp.layer_norm_grad_tensors(up, x, stats, w, bias_grad=b, weight_grad=b), lambda: gp.layer_norm_grad_tensors(up, x, stats, w, x_grad=rows, bias_grad=rows[2]),
                 lambda: gp.layer_norm_grad_tensors(up[:, :2], x[:, :2].contiguous(), stats, weight_grad=stats[1]),
                 lambda: gp.log_probs_grad_tensors(square, tokens, stats, grad_logp=g, out=square),
                 lambda: gp.log_probs_grad_tensors(x[:, :4], tokens, stats, grad_logp=square[0], out=square),
                 lambda: gp.log_probs_grad_tensors(x[:, :2], tokens, stats, grad_logp=g, out=stats), lambda: gp.log_probs_grad_tensors(x[:, :1], tokens, stats, entropy=g, grad_entropy=g[:1], out=g[:, None]),
                 lambda: gp.log_probs_grad_tensors(x[:, :1], tokens, stats, grad_logp=w[:4], out=tokens.view(torch.float32)[:, None]),
                 lambda: gp.distill_tensors(x[:, :3], at, v, grad_loss=g, out=v), lambda: gp.distill_tensors(x[:, :3], at, v, grad_loss=g, out=at.view(torch.float32)),
                 lambda: gp.distill_tensors(x[:, :2], at, v, grad_loss=g, out=stats, stats=stats), lambda: gp.distill_grad_tensors(x[:, :2], at, v, stats, g, out=stats),
                 lambda: gp.distill_grad_tensors(x[:, :1], at, v, stats, g, out=g[:, None])):
        with pytest.raises(ValueError, match="overlap"):
            call()


def test_an_empty_call_overlaps_nothing():
    import torch
    x = torch.zeros(0, 8)
    with pytest.raises(ValueError, match="on the GPU"):
        gp.log_probs_grad_tensors(x, torch.zeros(0, dtype=torch.int32), torch.zeros(0, 2), grad_logp=torch.zeros(1), out=x)


@pytest.mark.parametrize("over", ["weight", "bias", "both halves"])
def test_gradients_written_over_the_weight_leave_the_call_a_copy_of_it(monkeypatch, over):
    """Of few rows the workgroups that write the weight's gradient run beside those that read the weight: the call gets other memory to read it from."""
    import contextlib

    import torch
    calls = []
    monkeypatch.setattr(gp, "_on_stream", lambda tensor, stream: contextlib.nullcontext(0))
    monkeypatch.setattr(gp, "gp_layer_norm_grad_workspace", lambda N, d: 0)
    monkeypatch.setattr(gp, "gp_layer_norm_grad", lambda *a: calls.append((a, weights(a[9], a[7]))))

    def weights(address, d):
        import ctypes
        return list((ctypes.c_float * d).from_address(address))

    x, stats = torch.randn(4, 8), torch.ones(4, 2)
    flat = torch.arange(24.0)
    w = flat[8:16]
    dw, db = {"weight": (w, None), "bias": (None, w), "both halves": (flat[4:12], flat[12:20])}[over]
    for accumulate in (False, True):
        gp.layer_norm_grad_tensors(x, x.clone(), stats, w, weight_grad=torch.zeros(8) if dw is None else dw, bias_grad=torch.zeros(8) if db is None else db, accumulate=accumulate)
    gp.layer_norm_grad_tensors(x, x.clone(), stats, w)
    for args, held in calls[:2]:
        assert held == list(range(8, 16))
        start = args[9]
        for to in (args[13], args[14]):
            assert to + 32 <= start or start + 32 <= to
        if dw is not None:
            assert args[13] == dw.data_ptr()
        if db is not None:
            assert args[14] == db.data_ptr()
    assert calls[2][0][9] == w.data_ptr()
