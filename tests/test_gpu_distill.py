"""The loss against a teacher's best logits and its gradient on the GPU against their definitions in 64 bits.

Tolerances, u = 2^-24: log p as in the tests of log probabilities.  Of at most 64 entries v / T, with w their distance from the largest: log q is off by
(4 |w| + 80 + 4 |log sum|) u, q by as much of itself and 4 u.  The loss is T^2 sum q (log q - log p): q's share of every difference, the differences' own
errors, and 70 u of the terms.  The gradient g T (p - q): the errors of p and q, 6 u of both, and 2^-126 (a smaller p is 0).
"""
import numpy as np
import pytest

import paper_2207_12000_amd as gp
from oracle import answers
from test_gpu_layer_norm import U, bits, half_step, padded, types, wide
from test_gpu_log_probs import logp_bound, logits_of, same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


def check(loss, grad, x, at, v, T, g):
    X, A, V = wide(x), at.cpu().numpy(), wide(v)
    N, C = X.shape
    K = A.shape[1]
    T = float(np.float32(T))
    G = None if g is None else np.broadcast_to(wide(g), (N,))
    want, wants = answers.distill(X, A, V, T, G)
    lp, offp = answers.log_softmax(X / T), logp_bound(X, 1 / T)
    named = (A >= 0) & (A < C) & ~np.isneginf(V)
    with np.errstate(all="ignore"):
        w = np.where(named, V / T, -np.inf)
        top = w.max(1, keepdims=True)
        w = np.where(named, w - np.where(np.isneginf(top), 0.0, top), 0.0)
        total = np.where(named, np.exp(w), 0.0).sum(1, keepdims=True)
        logs = np.abs(np.log(np.where(total > 0, total, 1.0)))
        q = np.where(named, np.exp(w) / np.where(total > 0, total, 1.0), 0.0)
        offq = U * (4 * np.abs(w) + 84 + 4 * logs)
        c = np.where(named, A, 0)
        lpa, offa = np.take_along_axis(lp, c, 1), np.take_along_axis(offp, c, 1)
        gap = np.where(q > 0, np.abs(w - np.log(np.where(total > 0, total, 1.0)) - lpa), 0.0)
        bound = T * T * (q * (gap * (offq + 74 * U) + offq + offa)).sum(1)
    if loss is not None:
        same(loss, want, bound + 1e-37)
    if grad is not None:
        p = np.exp(lp)
        q_of, offq_of = np.zeros((N, C)), np.zeros((N, C))
        for k in range(K):
            np.add.at(q_of, (np.arange(N), c[:, k]), q[:, k])
            np.add.at(offq_of, (np.arange(N), c[:, k]), (q * (offq + 8 * U))[:, k])
        b = np.abs(G)[:, None] * T * (p * (offp + 8 * U) + offq_of + 6 * U * (p + q_of) + 2.0 ** -126) + half_step(grad) * np.abs(wants) + 1e-37
        off = np.abs(wide(grad) - wants)
        assert (off <= b).all(), f"worst {np.max(off / b):.2f} of the bound"


def teacher_of(gen, N, C, K, dtype, distinct=True, pad=0, skew=0):
    """Some entries are none, some rows have none; the same class twice where not distinct."""
    import torch
    at = torch.randint(0, C, (N, K), generator=gen, device="cuda")
    if distinct and K <= C:
        at = (at[:, :1] + torch.arange(K, device="cuda") * (C // K)) % C
    hide = torch.rand(N, K, generator=gen, device="cuda") < 0.2
    at = torch.where(hide, torch.where(torch.rand(N, K, generator=gen, device="cuda") < 0.5, -1, C + 3), at)
    at[:: 5] = -1
    _, v = padded(N, K, K + pad, types()[dtype], skew)
    v.copy_(2 * torch.randn(N, K, generator=gen, device="cuda") - 4)
    return at, v


SIZES = [(1, 1, 0, 0), (9, 2, 1, 1), (300, 3, 0, 1), (65, 7, 0, 0), (5000, 13, 0, 1), (3000, 40, 0, 0), (20_000, 47, 0, 0), (999, 64, 3, 1), (4001, 100, 0, 0), (2500, 172, 0, 0),
         (1000, 333, 1, 3), (40, 500, 0, 0), (700, 512, 0, 1), (300, 1000, 0, 0), (200, 1025, 5, 1), (90, 2047, 0, 0), (60, 3001, 0, 1), (50, 8192, 0, 0), (33, 8193, 0, 1),
         (12, 32_768, 0, 0), (7, 32_771, 1, 1), (3, 100_003, 0, 0), (1, 16_384, 0, 0), (600, 3300, 0, 0), (257, 33_003, 1, 1), (2048, 1501, 1, 1), (2050, 4095, 0, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,C,pad,skew", SIZES)
def test_loss_and_gradient(N, C, pad, skew, dtype):
    import torch
    gen, x, _ = logits_of(N, C, dtype, pad, skew)
    for K, T, index, teacher, distinct in ((1, 1.0, torch.int32, "f32", True), (5, 2.0, torch.int64, "bf16", True), (8, 4.0, torch.int32, "f32", False), (13, 0.5, torch.int64, "f32", False),
                                           (64, 1.0, torch.int32, "bf16", True)):
        if K > 4 * C:
            continue
        at, v = teacher_of(gen, N, C, K, teacher, distinct, pad, skew)
        g = torch.randn(N, generator=gen, device="cuda")
        flat, out = padded(N, C, C + 2 * pad, x.dtype, skew, fill=7.0)
        stats = torch.empty(N, 2, device="cuda")
        atp = padded(N, K, K + 2 * pad, index, skew, fill=-7)[1]
        atp.copy_(at)
        loss, grad = gp.distill_tensors(x, atp, v, T, grad_loss=g, out=out, stats=stats)
        assert grad is out and loss.dtype == torch.float32
        check(loss, grad, x, at, v, T, g)
        assert bool((loss[:: 5] == 0).all()) and not bool(grad[:: 5].any())
        alone = gp.distill_tensors(x, atp, v, T)
        check(alone, None, x, at, v, T, None)
        check(None, gp.distill_grad_tensors(x, atp, v, stats, g[:1], T), x, at, v, T, g[:1])
        out.fill_(7.0)
        assert bool((flat == 7.0).all())


@pytest.mark.parametrize("C", [5, 47, 700, 5000, 100_000])
def test_students_and_teachers_with_classes_ruled_out(C):
    import torch
    inf = float("inf")
    gen, x, _ = logits_of(8, C, "f32")
    at = torch.tensor([[0, C - 1, 2]] * 8, device="cuda")
    v = torch.randn(8, 3, generator=gen, device="cuda")
    x[0, 1] = -inf                # the student has it at 0, the teacher does not name it
    x[1, 0] = -inf                # the teacher does: a loss of +inf
    x[2] = -inf                   # nothing left
    v[3, 1] = -inf                # no entry
    v[4] = -inf                   # none at all
    v[5] = torch.finfo(torch.float32).min  # all equal
    x[6] = torch.finfo(torch.float32).min
    x[7] += 20_000.0
    v[7] -= 30_000.0
    g = torch.ones(8, device="cuda")
    loss, grad = gp.distill_tensors(x, at, v, 1.0, grad_loss=g)
    assert loss[1].item() == loss[2].item() == inf and loss[4].item() == 0 and not bool(grad[4].any())
    fine = [0, 3, 4, 5, 6, 7]
    check(loss[fine], grad[fine], x[fine], at[fine], v[fine], 1.0, g[fine])
    check(None, grad[:3], x[:3], at[:3], v[:3], 1.0, g[:3])
    # no numbers, in one row: the others are left alone
    x2 = x.clone()
    x2[0, 3] = float("nan")
    x2[7, 3] = inf
    v2 = v.clone()
    v2[5, 0] = float("nan")
    again, grad2 = gp.distill_tensors(x2, at, v2, 1.0, grad_loss=g)
    assert bool(again[[0, 5, 7]].isnan().all()) and torch.equal(again[[3, 4, 6]], loss[[3, 4, 6]]) and torch.equal(grad2[[1, 2, 3, 4, 6]], grad[[1, 2, 3, 4, 6]])


def test_a_teacher_that_is_the_student_and_the_same_class_many_times():
    import torch
    for C in (40, 900):
        gen, x, _ = logits_of(50, C, "f32")
        k = min(C, 64)
        a = gp.log_probs_tensors(x, top=k, scale=0.5)
        assert bool((a.top_index >= 0).all())
        loss, grad = gp.distill_tensors(x, a.top_index, x.gather(1, a.top_index.long()), 2.0, grad_loss=torch.ones(1, device="cuda"))
        check(loss, grad, x, a.top_index, x.gather(1, a.top_index.long()), 2.0, torch.ones(1, device="cuda"))
        if C <= 64:  # all classes are named: no loss, no gradient
            assert float(loss.abs().max()) < 1e-4 and float(grad.abs().max()) < 1e-5
        at = torch.full((50, 64), C - 1, device="cuda")
        v = torch.randn(50, 64, generator=gen, device="cuda")
        loss, grad = gp.distill_tensors(x, at, v, 1.0, grad_loss=torch.ones(1, device="cuda"))
        check(loss, grad, x, at, v, 1.0, torch.ones(1, device="cuda"))


def test_automatic_differentiation():
    import torch
    gen = torch.Generator(device="cuda").manual_seed(9)
    for shape in ((60, 47), (3, 4, 500), (700,)):
        x = torch.randn(shape, generator=gen, device="cuda", requires_grad=True)
        at = torch.randint(0, shape[-1], shape[:-1] + (6,), generator=gen, device="cuda")
        v = torch.randn(shape[:-1] + (6,), generator=gen, device="cuda")
        loss = gp.distill_tensors(x, at, v, 3.0)
        assert loss.shape == shape[:-1] and loss.requires_grad
        loss.mean().backward()
        rows = lambda t: t.detach().reshape(-1, t.shape[-1])  # noqa: E731
        N = rows(x).shape[0]
        check(loss.reshape(-1), x.grad.reshape(N, -1), rows(x), rows(at), rows(v), 3.0, torch.full((N,), 1 / N, device="cuda"))


def test_the_same_bits_in_a_graph_on_another_stream_and_with_kept_workspaces():
    import torch
    for N, C, K in ((3000, 47, 8), (40, 3000, 32), (2, 60_000, 8)):
        gen, x, _ = logits_of(N, C, "bf16")
        at, v = teacher_of(gen, N, C, K, "bf16", distinct=False)
        stats, out, loss = torch.empty(N, 2, device="cuda"), torch.empty_like(x), torch.empty(N, device="cuda")
        g = torch.ones(1, device="cuda")
        ws = torch.empty(gp.gp_distill_workspace(N, C) + 256, dtype=torch.uint8, device="cuda")

        def both(stream, fused):
            gp.gp_distill(x.data_ptr(), C, gp.GP_BF16, N, C, at.data_ptr(), K, gp.GP_I64, v.data_ptr(), v.stride(0) if N > 1 else K, gp.GP_BF16, K, 2.0, loss.data_ptr(),
                          None if fused else stats.data_ptr(), g.data_ptr(), 0, out.data_ptr() if fused else None, C, ws.data_ptr(), ws.numel(), stream)
            if not fused:
                gp.gp_distill_grad(x.data_ptr(), C, gp.GP_BF16, N, C, at.data_ptr(), K, gp.GP_I64, v.data_ptr(), v.stride(0), gp.GP_BF16, K, 2.0, stats.data_ptr(), g.data_ptr(), 0,
                                   out.data_ptr(), C, stream)

        for fused in (False, True):
            both(torch.cuda.current_stream().cuda_stream, fused)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                both(torch.cuda.current_stream().cuda_stream, fused)
            side = torch.cuda.Stream()
            for turn in range(4):
                x.mul_(-0.9)
                both(torch.cuda.current_stream().cuda_stream, fused)
                want = [bits(t) for t in (loss, out)]
                check(loss, out, x, at, v, 2.0, g)
                loss.zero_(), out.zero_()
                torch.cuda.synchronize()
                if turn == 3:
                    both(side.cuda_stream, fused)
                    side.synchronize()
                else:
                    graph.replay()
                    torch.cuda.synchronize()
                assert all(torch.equal(p, bits(t)) for p, t in zip(want, (loss, out)))
