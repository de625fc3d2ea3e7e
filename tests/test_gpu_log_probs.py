"""Log probabilities, entropies, alternatives and their gradient on the GPU against their definitions in 64 bits.

Tolerances, u = 2^-24.  With z = s (x - m), a term exp(z) is off by (4 |z| + 2) u of itself, and a sum of them by at most 32 additions in a lane, 10 steps among
lanes and, for rows in parts, N_parts / 64 + 6 more: 64 u with what else happens to it (parts of up to 800 columns' groups: 80 u).  With Z the mean of |z| under p, the log of
the sum is off by (80 + 4 Z + 4 |log|) u, log p by 4 u |z| more.  The entropy is log(sum) - weighted / sum: (160 + 170 Z + 4 mean(z^2) + 4 Z^2 + 4 |log| + 2 H) u.  The order
of alternatives is that of the logits as they are stored: exact.  Gradients take what the forward pass kept as given to those bounds; a p below
2^-126, the least normal number, is 0: off by as much.  What is written in bf16 is
off by 2^-8 of itself besides.
"""
import numpy as np
import pytest

import paper_2207_12000_amd as gp
from oracle import answers
from test_gpu_layer_norm import U, bits, half_step, padded, types, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


def spread(x, scale):
    """z, p, the mean of |z| under p, that of z^2, and the log of the sum, of every row; rows without a number left out of account."""
    s = float(np.float32(scale))
    m = x.max(1, keepdims=True)
    m = np.where(np.isneginf(m), 0.0, m)
    with np.errstate(divide="ignore", invalid="ignore"):
        z = s * (x - m)
        e = np.exp(z)
        total = e.sum(1, keepdims=True)
        p = np.where(total > 0, e / np.where(total > 0, total, 1), 0.0)
        finite = np.where(np.isneginf(z), 0.0, z)
        return z, p, (p * np.abs(finite)).sum(1), (p * finite ** 2).sum(1), np.where(total > 0, np.abs(np.log(np.where(total > 0, total, 1))), 0.0)[:, 0]


def logp_bound(x, scale):
    """Of log p, for every element (that of -inf is exact)."""
    z, _, Z, _, l = spread(x, scale)
    return U * (84 + 4 * Z + 4 * l)[:, None] + 6 * U * np.where(np.isneginf(z), 0.0, np.abs(z))


def same(got, want, bound):
    """Equal infinities and NaN, and finite numbers within the bound."""
    got = wide(got)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)])
    off = np.abs(got[fine] - want[fine])
    bound = np.broadcast_to(bound, want.shape)[fine]
    assert (off <= bound).all(), f"worst {np.max(off / bound):.2f} of the bound"


def check(a, logits, tokens, scale, k):
    x = wide(logits)
    logp, entropy, index, top = answers.log_probs(x, None if tokens is None else tokens.cpu().numpy(), scale, k)
    _, _, Z, Z2, l = spread(x, scale)
    every = logp_bound(x, scale)
    if tokens is not None:
        t = tokens.cpu().numpy()
        named = (t >= 0) & (t < x.shape[1])
        same(a.logp, logp, np.where(named, every[np.arange(len(t)), np.where(named, t, 0)], 0.0))
    same(a.entropy, entropy, U * (160 + 170 * Z + 4 * Z2 + 4 * Z ** 2 + 4 * l + 2 * np.abs(entropy)))
    if k:
        assert np.array_equal(a.top_index.cpu().numpy(), index)
        same(a.top_logp, top, np.where(index >= 0, np.take_along_axis(every, np.maximum(index, 0), 1), 0.0))


def logits_of(N, C, dtype, pad=0, skew=0, seed=0, hide=0.0):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed + 7 * N + C)
    _, x = padded(N, C, C + pad, types()[dtype], skew)
    x.copy_(3 * torch.randn(N, C, generator=gen, device="cuda"))
    if hide:
        x.masked_fill_(torch.rand(N, C, generator=gen, device="cuda") < hide, -float("inf"))
    tokens = torch.randint(-2, C + 2, (N,), generator=gen, device="cuda")
    return gen, x, tokens


# every team (4 to 64 lanes, 256, 1,024), rows below a vector, parts, odd widths
SIZES = [(1, 1, 0, 0), (9, 2, 1, 1), (300, 3, 0, 1), (65, 7, 0, 0), (17, 8, 0, 0), (5000, 13, 0, 1), (20_000, 16, 0, 0), (3000, 40, 0, 0), (70_000, 47, 0, 0), (999, 64, 3, 1),
         (4001, 100, 0, 0), (2500, 172, 0, 0), (2000, 333, 1, 3), (40, 500, 0, 0), (700, 512, 0, 1), (300, 1000, 0, 0), (200, 1025, 5, 1), (90, 2047, 0, 0), (60, 3001, 0, 1),
         (50, 8192, 0, 0), (33, 8193, 0, 1), (20, 20_001, 0, 0), (12, 32_768, 0, 0), (7, 32_771, 1, 1), (3, 100_003, 0, 0), (1, 16_384, 0, 0), (1, 391_000, 0, 0), (600, 33_000, 0, 0),
         (2048, 1501, 1, 1), (2050, 4095, 0, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,C,pad,skew", SIZES)
def test_answers(N, C, pad, skew, dtype):
    import torch
    _, x, tokens = logits_of(N, C, dtype, pad, skew, hide=0.1 if N % 2 else 0.0)
    for k, scale, index in ((0, 1.0, torch.int32), (1, 0.37, torch.int64), (2, 2.5, torch.int64), (5, 1.0, torch.int32), (8, 1.0, torch.int64), (9, 1.0, torch.int64), (20, 0.7, torch.int32),
                            (64, 1.0, torch.int64)):
        if N * C > 3_000_000 and k not in (5, 20):
            continue
        a = gp.log_probs_tensors(x, tokens.to(index), scale=scale, top=k)
        assert a.logp.dtype == a.entropy.dtype == torch.float32 and (a.top_index is None) == (k == 0)
        check(a, x, tokens, scale, k)


@pytest.mark.parametrize("C", [5, 47, 130, 700, 5000, 33_000, 100_000])
def test_equal_logits_ruled_out_classes_and_rows_that_are_no_numbers(C):
    import torch
    inf, nan, lowest = float("inf"), float("nan"), torch.finfo(torch.float32).min
    _, x, tokens = logits_of(16, C, "f32")
    x[0] = 2.0                                    # all equal
    x[1] = -inf                                   # nothing left
    x[2] = lowest                                 # the type's lowest instead: all equal
    x[3] = lowest
    x[3, C // 2] = 1.0                            # one class among the lowest
    x[4] = -inf
    x[4, C - 1] = -5.0                            # one class alone
    x[5] = -inf
    x[5, ::3] = x[6, ::3]                         # every third
    x[7] = torch.where(torch.arange(C, device="cuda") % 2 == 0, 0.0, -0.0)
    x[8, C // 3] = inf
    x[9, C - 1] = nan
    x[10, 0] = nan
    x[10, C // 2] = -nan
    x[11] = torch.arange(C, device="cuda") / C    # ascending, descending
    x[12] = -torch.arange(C, device="cuda") / C
    x[13] = 0.0
    x[13, :: max(C // 70, 1)] = 3.0               # many of the largest
    x[14] = 1e30 * x[14]
    x[15] = 30_000.0 + 0.01 * x[15]
    tokens[:] = torch.tensor([0, 1, C - 1, C // 2, C - 1, 0, -1, 3, C // 3, 0, C // 2, C, 0, 1, 2, 4], device="cuda")
    for k in (0, 3, 8, 40, 64):
        a = gp.log_probs_tensors(x, tokens, top=k)
        with np.errstate(all="ignore"):
            check(a, x, tokens, 1.0, k)
    a = gp.log_probs_tensors(x[1:2].bfloat16(), tokens[1:2], top=2)
    assert a.logp.item() == -inf and a.entropy.item() == 0 and a.top_index.tolist() == [[-1, -1]] and a.top_logp.tolist() == [[-inf, -inf]]


@pytest.mark.parametrize("C,period", [(700, 64), (2000, 256), (8192, 1024), (32_768, 4096), (32_768, 1024), (120_000, 4096)])
def test_alternatives_that_all_lie_with_one_lane(C, period):
    """The largest logits a team's stride apart, so that one lane or group of lanes holds them all, and more of them than a list has room for."""
    import torch
    gen, x, _ = logits_of(3, C, "f32")
    for width in (4, 16, 64):
        y = x.clone()
        at = (torch.arange(C, device="cuda") % period) < width
        y[:, at] += 50.0
        for k in (8, 33, 64):
            check(gp.log_probs_tensors(y, top=k), y, None, 1.0, k)
            check(gp.log_probs_tensors(y.bfloat16(), top=k), y.bfloat16(), None, 1.0, k)


@pytest.mark.parametrize("C", [47, 700, 33_000])
def test_tiny_and_negative_logits_keep_their_order(C):
    import torch
    gen, x, _ = logits_of(6, C, "f32")
    x[0] *= 1e-40                     # below the type's normal numbers
    x[1] = -x[1].abs() * 1e-40
    x[2] = -x[2].abs() - 1
    x[3] = -1e30 * x[3].abs() - 1e30
    x[4] = -x[4].abs()
    x[4, ::2] = -0.0
    for y in (x, x.bfloat16()):
        for k in (8, 40):
            check(gp.log_probs_tensors(y, top=k), y, None, 1.0, k)


def gradient(x, tokens, scale, g1, g2):
    return answers.log_probs_grad(x, tokens, scale, g1, g2)


def check_gradient(got, logits, tokens, scale, g1, g2):
    x, s = wide(logits), float(np.float32(scale))
    N, C = x.shape
    wants = gradient(x, tokens.cpu().numpy(), scale, None if g1 is None else wide(g1), None if g2 is None else wide(g2))
    lp = answers.log_softmax(x * s)
    _, p, Z, Z2, l = spread(x, scale)
    every = logp_bound(x, scale) + 8 * U * np.where(np.isneginf(lp), 0.0, np.abs(lp))  # of log p; so also p's relative error
    H = -np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0).sum(1)
    offH = (U * (160 + 170 * Z + 4 * Z2 + 4 * Z ** 2 + 4 * l + 2 * np.abs(H)))[:, None]
    a1 = 0.0 if g1 is None else np.broadcast_to(np.abs(wide(g1)), (N,))[:, None]
    a2 = 0.0 if g2 is None else np.broadcast_to(np.abs(wide(g2)), (N,))[:, None]
    t = tokens.cpu().numpy()[:, None]
    named = (t >= 0) & (t < C)
    a1 = a1 * named
    size = np.abs(np.where(p > 0, lp, 0.0)) + H[:, None]
    bound = s * (a1 * (p * (every + 4 * U) + 4 * U * (np.arange(C) == t)) + a2 * p * (size * (every + 8 * U) + every + offH) + 2.0 ** -126 * (a1 + a2 * size)) + half_step(got) * np.abs(wants) + 1e-37
    off = np.abs(wide(got) - wants)
    assert (off <= bound).all(), f"worst {np.max(off / bound):.2f} of the bound"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,C,pad,skew", [s for s in SIZES if s[0] * s[1] <= 3_500_000])
def test_gradient(N, C, pad, skew, dtype):
    import torch
    gen, x, tokens = logits_of(N, C, dtype, pad, skew, hide=0.1 if N % 2 else 0.0)
    x[:, 0] = 0.5  # (one class is left in every row)
    g1, g2 = torch.randn(N, generator=gen, device="cuda"), torch.randn(N, generator=gen, device="cuda")
    for scale, a, b, index in ((1.0, g1, None, torch.int32), (0.37, None, g2, torch.int64), (2.0, g1, g2, torch.int64), (1.0, g1[:1], g2[0].expand(N), torch.int32)):
        stats = torch.empty(N, 2, device="cuda")
        got = gp.log_probs_tensors(x, tokens.to(index), scale=scale, stats=stats)
        flat, out = padded(N, C, C + 2 * pad, x.dtype, skew, fill=7.0)
        assert gp.log_probs_grad_tensors(x, tokens.to(index), stats, scale, got.entropy, a, b, out=out) is out
        check_gradient(out, x, tokens, scale, a, b)
        out.fill_(7.0)
        assert bool((flat == 7.0).all())


def test_gradient_of_rows_with_nothing_left_and_by_differences():
    import torch
    x = torch.full((3, 50), -float("inf"), device="cuda")
    x[1] = torch.randn(50, device="cuda")
    x[2, 7] = 4.0
    tokens = torch.tensor([0, 3, 7], device="cuda")
    stats = torch.empty(3, 2, device="cuda")
    a = gp.log_probs_tensors(x, tokens, stats=stats)
    g = gp.log_probs_grad_tensors(x, tokens, stats, 1.0, a.entropy, torch.ones(1, device="cuda"), torch.ones(1, device="cuda"))
    assert g[0].tolist() == [1.0] + [0.0] * 49 and bool(g[2].abs().max() <= 1e-6)
    # differences of what the library itself returns: 2^-24 of values of about 5 over a step of 2^-4, and the third derivative
    step = 2.0 ** -4
    for j in (0, 3, 49):
        up, down = x[1:2].clone(), x[1:2].clone()
        up[0, j] += step
        down[0, j] -= step
        p, q = gp.log_probs_tensors(up, tokens[1:2]), gp.log_probs_tensors(down, tokens[1:2])
        want = ((p.logp + p.entropy) - (q.logp + q.entropy)).item() / (2 * step)
        assert abs(want - g[1, j].item()) <= 2e-3


def test_automatic_differentiation():
    import torch
    gen = torch.Generator(device="cuda").manual_seed(5)
    for shape in ((60, 47), (3, 4, 500), (700,)):
        x = torch.randn(shape, generator=gen, device="cuda", requires_grad=True)
        tokens = torch.randint(0, shape[-1], shape[:-1], generator=gen, device="cuda")
        a = gp.log_probs_tensors(x, tokens, scale=0.5, top=3)
        assert a.logp.shape == tokens.shape and a.top_index.shape == shape[:-1] + (3,) and a.logp.requires_grad and not a.top_logp.requires_grad
        (a.entropy.sum() - 2 * a.logp.mean()).backward()
        rows, t = x.detach().reshape(-1, shape[-1]), tokens.reshape(-1)
        N = rows.shape[0]
        check_gradient(x.grad.reshape(N, -1), rows, t, 0.5, torch.full((N,), -2 / N, device="cuda"), torch.ones(N, device="cuda"))
        x.grad = None
        gp.log_probs_tensors(x, tokens).logp.sum().backward()
        check_gradient(x.grad.reshape(N, -1), rows, t, 1.0, torch.ones(N, device="cuda"), None)
    assert gp.log_probs_tensors(x.detach(), None, entropy=False, top=1).logp is None


def test_past_32_bit_offsets_and_no_rows():
    import torch
    N, C = 26_000, 170_000  # 4.4e9 elements of bf16
    x = torch.zeros(N, C, dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 13_000, 25_999], device="cuda")
    x[rows] = (3 * torch.randn(3, C, device="cuda")).bfloat16()
    tokens = torch.full((N,), C - 1, device="cuda")
    stats = torch.empty(N, 2, device="cuda")
    a = gp.log_probs_tensors(x, tokens, top=4, stats=stats)
    check(gp.LogProbs(*(t[rows] for t in a)), x[rows], tokens[rows], 1.0, 4)
    one = torch.ones(1, device="cuda")
    few = gp.log_probs_grad_tensors(x[rows], tokens[rows], stats[rows], grad_logp=one)
    big = gp.log_probs_grad_tensors(x, tokens, stats, grad_logp=one)
    assert torch.equal(big[rows], few) and bool((big[1, : C - 1] == big[1, 0]).all())
    del big, x
    a = gp.log_probs_tensors(torch.empty(0, 9, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"), top=2)
    assert a.logp.shape == a.entropy.shape == (0,) and a.top_index.shape == (0, 2)


def test_the_same_bits_in_a_graph_on_another_stream_and_with_kept_workspaces():
    import torch
    for N, C, k in ((3000, 47, 5), (40, 3000, 20), (2, 60_000, 8)):
        _, x, tokens = logits_of(N, C, "f32")
        stats, out = torch.empty(N, 2, device="cuda"), torch.empty_like(x)
        g = torch.ones(1, device="cuda")
        ws = torch.empty(gp.gp_log_probs_workspace(N, C, k) + 256, dtype=torch.uint8, device="cuda")
        logp, entropy = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
        index, top = torch.empty(N, k, dtype=torch.int32, device="cuda"), torch.empty(N, k, device="cuda")

        def both(stream):
            gp.gp_log_probs(x.data_ptr(), C, gp.GP_F32, N, C, tokens.data_ptr(), gp.GP_I64, 1.0, logp.data_ptr(), entropy.data_ptr(), k, index.data_ptr(), top.data_ptr(),
                            stats.data_ptr(), ws.data_ptr(), ws.numel(), stream)
            gp.gp_log_probs_grad(x.data_ptr(), C, gp.GP_F32, N, C, tokens.data_ptr(), gp.GP_I64, 1.0, stats.data_ptr(), entropy.data_ptr(), g.data_ptr(), 0, g.data_ptr(), 0,
                                 out.data_ptr(), C, stream)

        both(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            both(torch.cuda.current_stream().cuda_stream)
        side = torch.cuda.Stream()
        outs = (logp, entropy, index, top, stats, out)
        for turn in range(4):
            x.mul_(-0.9)
            both(torch.cuda.current_stream().cuda_stream)
            want = [bits(t) for t in outs]
            check(gp.LogProbs(logp, entropy, index, top), x, tokens, 1.0, k)
            for t in outs:
                t.zero_()
            torch.cuda.synchronize()
            if turn == 3:
                both(side.cuda_stream)
                side.synchronize()
            else:
                graph.replay()
                torch.cuda.synchronize()
            assert all(torch.equal(p, bits(t)) for p, t in zip(want, outs))
