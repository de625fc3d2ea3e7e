"""Layer norm and its gradients on the GPU against their definitions in 64 bits.

Tolerances, u = 2^-24.  A sum over a row is added up by lanes of at most 32 elements, then in at most 10 steps: 50 u of the terms' magnitudes at most, with what
the terms themselves were rounded by.  So the mean is off by e = 50 u mean|x|, x - m by e + u |x - m|, the sum of squares by 52 u and 2 e / sigma of itself,
r by half of that and three roundings.  With h = (x - m) r:  |w| (r e (1 + |h|) + 40 u |h|) + 2 u (|h w| + |b|), and the rounding of what is written (half a step of
its type: 2^-24, 2^-8).  Gradients take mean and r as given: h is off by 3 u |h|, the two means by 58 u of the terms'.  A sum over N rows is of at most
N / 64 + 44 terms one after another: as many u of the terms' magnitudes.
"""
import numpy as np
import pytest

import paper_2207_12000_amd as gp
from oracle import answers

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


def types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}


def half_step(t):
    import torch
    return torch.finfo(t.dtype).eps / 2


def padded(rows, cols, ld, dtype, skew=0, fill=float("nan")):
    """A (rows, cols) view with rows ld elements apart, `skew` elements into its memory; the rest is `fill`."""
    import torch
    flat = torch.full((rows * ld + skew + 64,), fill, dtype=dtype, device="cuda")
    return flat, flat[skew:skew + rows * ld].view(rows, ld)[:, :cols]


def wide(t):
    return t.detach().double().cpu().numpy()


def bits(t):
    import torch
    return t.detach().contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32).clone()


def inputs(N, d, dtype, pad=0, skew=0, seed=0, offset=3.0):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000 + N + d)
    _, x = padded(N, d, d + pad, types()[dtype], skew)
    x.copy_(torch.randn(N, d, generator=gen, device="cuda") * torch.rand(N, 1, generator=gen, device="cuda") + offset * torch.randn(N, 1, generator=gen, device="cuda"))
    return gen, x


def check_forward(y, stats, x, w, b, eps):
    X, W, B = wide(x), 1.0 if w is None else wide(w), 0.0 if b is None else wide(b)
    eps = float(np.float32(eps))
    want, s = answers.layer_norm(X, W, B, eps)
    r = s[:, 1:]
    h = (X - s[:, :1]) * r
    e = 50 * U * np.abs(X).mean(1, keepdims=True)
    bound = np.abs(W) * (r * e * (1 + np.abs(h)) + 40 * U * np.abs(h)) + 2 * U * (np.abs(h * W) + np.abs(B)) + half_step(y) * np.abs(want) + 1e-37
    assert (np.abs(wide(y) - want) <= bound).all(), f"worst {np.max(np.abs(wide(y) - want) / bound):.2f} of the bound"
    if stats is not None:
        off = np.abs(wide(stats) - s)
        assert (off[:, :1] <= e + U * np.abs(s[:, :1]) + 1e-37).all() and (off[:, 1:] <= r * (e * r + 40 * U)).all()


def check_backward(got, g, x, stats, w, before=None):
    G, X, S, W = wide(g), wide(x), wide(stats), 1.0 if w is None else wide(w)
    dx, dw, db = answers.layer_norm_grad(G, X, S, W)
    h, u, r = (X - S[:, :1]) * S[:, 1:], G * W, S[:, 1:]
    mean = lambda a: np.abs(a).mean(1, keepdims=True)  # noqa: E731
    # u, the means, h times its mean, each taken from the other: roundings of every term
    parts = 6 * np.abs(u) + 60 * mean(u) + 66 * np.abs(h) * mean(u * h)
    terms = X.shape[0] / 64 + 44
    bounds = [U * r * parts, terms * U * np.abs(G * h).sum(0), terms * U * np.abs(G).sum(0)]
    for k, (a, want, bound) in enumerate(zip(got, (dx, dw, db), bounds)):
        if a is None:
            continue
        if before is not None and k:
            want, bound = want + before[k - 1], bound + U * np.abs(before[k - 1])
        bound = bound + half_step(a) * np.abs(want) + 1e-37
        off = np.abs(wide(a) - want)
        assert (off <= bound).all(), f"output {k}: worst {np.nanmax(off / bound):.2f} of the bound"


# every team: rows below a vector, all widths of teams up to what 1,024 lanes hold, and longer ones; few rows, and more than one round of workgroups
SIZES = [(1, 1, 0, 0), (5, 2, 1, 1), (3, 3, 0, 1), (9, 4, 0, 0), (17, 7, 2, 1), (64, 8, 0, 0), (100, 9, 3, 1), (1, 33, 0, 0), (257, 47, 0, 1), (1000, 64, 0, 0),
         (4096, 128, 0, 0), (70_001, 100, 0, 0), (40_000, 129, 7, 3), (3001, 256, 0, 0), (1234, 602, 6, 0), (35, 1000, 1, 1), (300, 1025, 0, 0), (129, 2051, 0, 1),
         (77, 4096, 0, 0), (600, 5000, 8, 0), (11, 8192, 0, 0), (1100, 9001, 0, 0), (5, 16384, 0, 0), (3, 16385, 0, 1), (2, 32768, 0, 0), (70, 33_001, 3, 0)]


@pytest.mark.parametrize("kinds", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("N,d,pad,skew", SIZES)
def test_forward_and_backward(N, d, pad, skew, kinds):
    import torch
    ty = types()
    gen, x = inputs(N, d, kinds[0], pad, skew)
    for params in ("f32", "bf16", None):
        w = b = None
        if params:
            w, b = (torch.randn(d, generator=gen, device="cuda").to(ty[params]) for _ in range(2))
        flat, y = padded(N, d, d + 2 * pad, ty[kinds[1]], skew, fill=7.0)
        stats = torch.full((N, 2), float("nan"), device="cuda")
        assert gp.layer_norm_tensors(x, w, b, eps=1e-3, out=y, stats=stats) is y
        check_forward(y, stats, x, w, b, 1e-3)
        _, g = padded(N, d, d + pad, ty[kinds[1]], skew)
        g.copy_(torch.randn(N, d, generator=gen, device="cuda"))
        gflat, xg = padded(N, d, d + 2 * pad, ty[kinds[0]], skew, fill=7.0)
        got = gp.layer_norm_grad_tensors(g, x, stats, w, x_grad=xg, weight_dtype=ty[params] if params else None)
        assert got[0] is xg and got[1].dtype == got[2].dtype == (ty[params] if params else torch.float32)
        check_backward(got, g, x, stats, w)
        for f, t in ((flat, y), (gflat, xg)):  # between the rows, before and behind them: untouched
            t.fill_(7.0)
            assert bool((f == 7.0).all())


def test_parts_of_what_can_be_asked_for():
    import torch
    for N, d in ((300, 100), (40, 17_000)):
        gen, x = inputs(N, d, "f32")
        w, b = torch.randn(d, generator=gen, device="cuda"), torch.randn(d, generator=gen, device="cuda")
        g = torch.randn(N, d, generator=gen, device="cuda")
        stats = torch.empty(N, 2, device="cuda")
        y = gp.layer_norm_tensors(x, w, b, stats=stats)
        assert torch.equal(y, gp.layer_norm_tensors(x, w, b))
        check_forward(gp.layer_norm_tensors(x, w), None, x, w, None, 1e-5)
        check_forward(gp.layer_norm_tensors(x, None, b), None, x, None, b, 1e-5)
        full = gp.layer_norm_grad_tensors(g, x, stats, w)
        for leave in range(1, 8):
            part = gp.layer_norm_grad_tensors(g, x, stats, w, *(False if leave >> k & 1 else None for k in range(3)))
            for k in range(3):
                assert part[k] is None if leave >> k & 1 else torch.equal(part[k], full[k])
        # added to what is there, and one row that stands for all
        before = [torch.randn(d, generator=gen, device="cuda") for _ in range(2)]
        held = [t.clone() for t in before]
        gp.layer_norm_grad_tensors(g, x, stats, w, False, *held, accumulate=True)
        check_backward([None] + held, g, x, stats, w, [wide(t) for t in before])
        one = g[:1].expand(N, d)
        got = gp.layer_norm_grad_tensors(one, x, stats, w)
        assert all(torch.equal(p, q) for p, q in zip(got, gp.layer_norm_grad_tensors(one.contiguous(), x, stats, w)))
        # in place
        z = x.clone()
        assert gp.layer_norm_tensors(z, w, b, out=z) is z and torch.equal(z, y)
        for over in ("x", "grad"):
            X, G = x.clone(), g.clone()
            got = gp.layer_norm_grad_tensors(G, X, stats, w, x_grad=X if over == "x" else G)
            assert all(torch.equal(p, q) for p, q in zip(got, full))


def test_no_rows():
    import torch
    x, stats, w = torch.empty(0, 12, device="cuda"), torch.empty(0, 2, device="cuda"), torch.ones(12, device="cuda")
    assert gp.layer_norm_tensors(x, w).shape == (0, 12)
    _, dw, db = gp.layer_norm_grad_tensors(x, x, stats, w)
    assert torch.equal(dw, torch.zeros(12, device="cuda")) and torch.equal(db, dw)
    dw.fill_(3.0)
    gp.layer_norm_grad_tensors(x, x, stats, w, False, dw, False, accumulate=True)
    assert torch.equal(dw, torch.full((12,), 3.0, device="cuda"))


@pytest.mark.parametrize("d", [100, 5000, 40_000])
def test_rows_far_from_zero_constant_rows_and_rows_that_are_no_numbers(d):
    import torch
    gen, x = inputs(8, d, "f32", offset=0.0)
    x[0] += 4096.0
    x[1] = -7.25
    x[2, d // 2] = float("inf")
    x[3, d - 1] = float("nan")
    x[4] *= 1e16
    x[5] *= 1e-18
    w, b = torch.randn(d, generator=gen, device="cuda"), torch.randn(d, generator=gen, device="cuda")
    stats = torch.empty(8, 2, device="cuda")
    y = gp.layer_norm_tensors(x, w, b, stats=stats)
    fine = [0, 1, 4, 5, 6, 7]
    check_forward(y[fine], stats[fine], x[fine], w, b, 1e-5)
    # a constant row: x - m is at most 50 u |x|, the mean of that is off by 50 u of it: 2500 u^2 * 7.25 = 6.5e-11 are left, times r = 316 and |w| < 5
    assert bool(((y[1] - b).abs() <= 1.1e-7 + U * b.abs()).all()) and bool(y[2:4].isnan().all())
    g = torch.randn(8, d, generator=gen, device="cuda")
    dx, dw, db = gp.layer_norm_grad_tensors(g, x, stats, w)
    check_backward((dx[fine], None, None), g[fine], x[fine], stats[fine], w)
    assert bool(dx[2:4].isnan().all()) and bool(dw.isnan().all())
    check_backward((None, None, db), g, torch.zeros_like(x), torch.ones_like(stats), w)


def test_past_32_bit_offsets():
    import torch
    N, d = 17_000_003, 260  # 4.4e9 elements of bf16
    x = torch.empty(N, d, dtype=torch.bfloat16, device="cuda")
    x[:, 0], x[:, 1:] = 1.0, 0.0
    rows = torch.tensor([0, 9_000_001, 16_500_000, N - 1], device="cuda")
    x[rows] = torch.randn(4, d, device="cuda").bfloat16()
    stats = torch.empty(N, 2, device="cuda")
    few, fewstats = x[rows], torch.empty(4, 2, device="cuda")
    gp.layer_norm_tensors(x, out=x, stats=stats)
    want = gp.layer_norm_tensors(few, stats=fewstats)
    check_forward(x[rows], stats[rows], few, None, None, 1e-5)
    check_forward(want, fewstats, few, None, None, 1e-5)


def test_the_same_bits_in_a_graph_on_another_stream_and_with_a_kept_workspace():
    import torch
    for N, d in ((5000, 100), (700, 4100), (30, 17_000)):
        gen, x = inputs(N, d, "bf16")
        g = torch.randn(N, d, generator=gen, device="cuda").bfloat16()
        w, b = torch.randn(d, generator=gen, device="cuda"), torch.randn(d, generator=gen, device="cuda")
        stats, y, dx = torch.empty(N, 2, device="cuda"), torch.empty_like(x), torch.empty_like(x)
        dw, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
        ws = torch.empty(gp.gp_layer_norm_grad_workspace(N, d) + 256, dtype=torch.uint8, device="cuda")

        def both(stream=None):
            gp.layer_norm_tensors(x, w, b, out=y, stats=stats, stream=stream)
            gp.layer_norm_grad_tensors(g, x, stats, w, dx, dw, db, workspace=ws, stream=stream)

        both()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            both()
        side = torch.cuda.Stream()
        for turn in range(4):
            x.add_(0.5)
            g.mul_(-1.25)
            both()
            want = [bits(t) for t in (stats, y, dx, dw, db)]
            for t in (stats, y, dx, dw, db):
                t.zero_()
            torch.cuda.synchronize()
            if turn == 3:
                both(side.cuda_stream)
                side.synchronize()
            else:
                graph.replay()
                torch.cuda.synchronize()
            assert all(torch.equal(p, bits(t)) for p, t in zip(want, (stats, y, dx, dw, db)))


def test_automatic_differentiation():
    import torch
    gen = torch.Generator(device="cuda").manual_seed(3)
    for shape in ((50, 33), (4, 5, 16), (20,)):
        x = torch.randn(shape, generator=gen, device="cuda", requires_grad=True)
        w = torch.randn(shape[-1], generator=gen, device="cuda", requires_grad=True)
        b = torch.randn(shape[-1], generator=gen, device="cuda", requires_grad=True)
        up = torch.randn(shape, generator=gen, device="cuda")
        y = gp.layer_norm_tensors(x, w, b)
        assert y.shape == x.shape and y.requires_grad
        y.backward(up)
        stats = torch.tensor(answers.layer_norm(wide(x).reshape(-1, shape[-1]))[1], dtype=torch.float32, device="cuda")
        rows = lambda t: t.detach().reshape(-1, shape[-1])  # noqa: E731
        N = rows(x).shape[0]
        # (the statistics that the forward pass kept are the definition's to the bounds above; 1e-5 of the largest covers what that changes here)
        dx, dw, db = answers.layer_norm_grad(wide(rows(up)), wide(rows(x)), wide(stats), wide(w))
        for got, want in ((rows(x.grad), dx), (w.grad, dw), (b.grad, db)):
            assert np.abs(wide(got) - want).max() <= 1e-5 * np.abs(want).max()
        # a sum's gradient is one number, expanded; a weight alone; no bias
        x2 = x.detach()
        gp.layer_norm_tensors(x2, w, None).sum().backward()
        _, dw2, _ = answers.layer_norm_grad(np.ones((N, shape[-1])), wide(rows(x)), wide(stats), wide(w))
        assert np.abs(wide(w.grad) - dw - dw2).max() <= 1e-5 * (np.abs(dw).max() + np.abs(dw2).max() + N ** 0.5)
    before = w._version
    gp.layer_norm_grad_tensors(up, x.detach(), torch.ones(1, 2, device="cuda"), w.detach(), weight_grad=w.detach())
    assert w._version > before
    with torch.no_grad():
        assert not gp.layer_norm_tensors(x, w).requires_grad


def test_a_followed_call_is_not_captured():
    import torch
    x = torch.randn(4, 8, device="cuda", requires_grad=True)
    out = torch.empty(4, 8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(ValueError, match="captured"):
            gp.layer_norm_tensors(x)
        with torch.no_grad():
            gp.layer_norm_tensors(x, out=out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, gp.layer_norm_tensors(x.detach()))
