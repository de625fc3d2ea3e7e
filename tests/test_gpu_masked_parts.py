"""Entropies, log probabilities and gradients on the GPU of rows of which whole stretches are ruled out, by -inf or by the type's lowest value, at scales
that take the distance to them beyond fp32; against the definitions in 64 bits.

Tolerances, u = 2^-24, Z the mean of |z| under p, z = s (x - m).  A term exp(z) is off by (5 + 4 |z|) u of itself.  A lane adds up at most 64 of them, then 6
steps among its wavefront, 4 among wavefronts, 2 of a row's parts and 6 among those, and two factors exp(distance of two bases) of (3 + 4 |z|) u each: the sum is off
by (63 + 18 + 6 + 5) u < 100 u and 12 Z u of itself, its log by as much and 4 u |log|, log p by 6 u |z| more.  The entropy is log(sum) - weighted / sum, where the
weighted sum's terms are off as the sum's are, twice with the division: (100 + 12 Z + 4 |log| + 220 Z + 12 mean(z^2) + 12 Z^2 + 2 H) u.  A log p beyond fp32's range is -inf.
Gradients: p is off by what log p is and 8 u |log p|, and 2^-126 (what is below the least normal number is 0); bf16 is off by 2^-8 of itself besides.
"""
import numpy as np
import pytest

import paper_2207_12000_amd as gp
from oracle import answers
from test_gpu_layer_norm import U, half_step, types, wide
from test_gpu_log_probs import same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


def rows(C, dtype, gen):
    """(rows, a class of each that is not masked, or is as good as any)"""
    import torch
    inf, lowest = float("inf"), torch.finfo(types()[dtype]).min
    x = 3 * torch.randn(9, C, generator=gen, device="cuda")
    j = torch.arange(C, device="cuda")
    x[0] = lowest
    x[1] = torch.where(j < C // 2, -inf, lowest)
    x[2] = torch.where(j < C - C // 4, -inf, lowest)
    x[3, C // 3:] = lowest
    x[4, : C - 9] = lowest
    x[4, : C // 2] = -inf
    x[5] = lowest
    x[5, C // 2] = 1.0
    x[6] = torch.where(j % 7 == 0, -1e38, lowest)
    x[7] = torch.where((j // 64) % 2 == 0, x[7], lowest)
    return x.to(types()[dtype]), torch.tensor([0, C - 1, C - 1, 0, C - 1, C // 2, 7, 1, C // 3], device="cuda")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,times", [(47, 1), (700, 1), (700, 256), (5000, 1), (33_000, 1), (33_000, 60), (100_000, 1), (391_000, 1)])
def test_whole_stretches_ruled_out(C, times, dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(C)
    x, tokens = rows(C, dtype, gen)
    n = len(tokens)
    X, t = wide(x), tokens.cpu().numpy()
    g1, g2 = torch.randn(n, generator=gen, device="cuda"), torch.randn(n, generator=gen, device="cuda")
    for scale in (0.7, 1.25, 2.5, 1e4):
        s = float(np.float32(scale))
        many, names = x.repeat(times, 1), tokens.repeat(times)
        stats = torch.empty(n * times, 2, device="cuda")
        a = gp.log_probs_tensors(many, names, scale=scale, top=3, stats=stats)
        grad = gp.log_probs_grad_tensors(many, names, stats, scale, a.entropy, g1.repeat(times), g2.repeat(times))
        for got in (a.logp, a.entropy, a.top_index, a.top_logp, grad):  # the same rows have the same answers
            again = got.reshape(times, n, -1)
            assert torch.equal(again, again[:1].expand_as(again))
        with np.errstate(all="ignore"):
            logp, entropy, index, top = answers.log_probs(X, t, scale, 3)
            want = answers.log_probs_grad(X, t, scale, wide(g1), wide(g2))
            lp = answers.log_softmax(X * s)
            z = s * (X - X.max(1, keepdims=True))
            p = np.exp(lp)
            near = np.where(p > 0, z, 0.0)
            Z, Z2 = (p * -near).sum(1), (p * near ** 2).sum(1)
            log_sum = np.abs(np.log(np.exp(z).sum(1)))
            every = U * ((104 + 12 * Z + 4 * log_sum)[:, None] + 6 * np.abs(near))
            off_entropy = U * (100 + 232 * Z + 12 * Z2 + 12 * Z ** 2 + 4 * log_sum + 2 * entropy)
            top = np.where(top < -3.4028236e38, -np.inf, top)
            each = every + 6 * U * np.where(p > 0, 0.0, np.minimum(np.abs(z), 3.5e38))  # (of log p where p is 0, too)
            same(a.logp[:n], logp, each[np.arange(n), t])
            same(a.entropy[:n], entropy, off_entropy)
            assert np.array_equal(a.top_index[:n].cpu().numpy(), index)
            same(a.top_logp[:n], top, np.where(index >= 0, np.take_along_axis(each, np.maximum(index, 0), 1), 0.0))
            size = np.abs(np.where(p > 0, lp, 0.0))
            off_p = p * (every + 8 * U * size + 4 * U)
            a1, a2 = np.abs(wide(g1))[:, None], np.abs(wide(g2))[:, None]
            part = size + entropy[:, None]
            bound = s * (a1 * (off_p + 4 * U * (np.arange(C) == t[:, None])) + a2 * (part * (off_p + 8 * U * p) + p * (every + off_entropy[:, None])) + 2.0 ** -126 * (a1 + a2 * part))
            bound += half_step(grad) * np.abs(want) + 1e-37
            off = np.abs(wide(grad[:n]) - want)
            assert (off <= bound).all(), f"worst {np.nanmax(off / bound):.2f} of the bound"
