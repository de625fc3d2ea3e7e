"""Rows that hold very large logits beside the type's lowest value: a class as far from the largest as fp32 does not hold has the log p that it has, as long as that is a number.

Bounds, u = 2^-24: all p but the largest logits' are 0, so the sum is their number, exact up to 2^24, its log off by 2 u of itself; z = s (x - m) by 3 u of itself, log p by u more.
The loss is T q (T (log q + log sum) - (x - m)): q off by what its exponential and its sum are, (4 |w| + 80 + 4 |log|) u as in the tests of distillation, below 200 u here, and 8 u."""
import numpy as np
import pytest

import paper_2207_12000_amd as gp
from test_gpu_layer_norm import U, types, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [5, 47, 300, 900, 5000, 33_000, 100_000])
def test_distances_beyond_fp32(C, dtype):
    import torch
    from oracle import answers
    ty = types()[dtype]
    top, lowest = torch.finfo(ty).max, torch.finfo(ty).min
    x = torch.full((4, C), lowest, device="cuda", dtype=ty)
    x[0, 2] = top
    x[1, 1:4] = 3e37
    x[2, :] = 0.0
    x[2, 0], x[2, C - 1] = lowest, top
    x[3, C - 2:] = 1e38
    tokens = torch.tensor([1, 0, 0, 2], device="cuda")
    X, t = wide(x), tokens.cpu().numpy()
    with np.errstate(all="ignore"):
        for scale in (1e-3, 0.25, 0.7):
            a = gp.log_probs_tensors(x, tokens, scale=scale, top=5)
            logp, entropy, index, best = answers.log_probs(X, t, scale, 5)
            for got, want in ((a.logp, logp), (a.top_logp, best)):
                assert np.isfinite(want).any() and (np.abs(want[np.isfinite(want)]) < 3.4e38).any()
                want = np.where(want < -3.4028235e38, -np.inf, want)
                got = wide(got)
                fine = np.isfinite(want)
                assert np.array_equal(got[~fine], want[~fine]) and (np.abs(got - want)[fine] <= 6 * U * np.abs(want)[fine] + 1e-30).all()
            assert np.array_equal(a.top_index.cpu().numpy(), index) and (np.abs(wide(a.entropy) - entropy) <= 6 * U * entropy).all()
        at = torch.tensor([[0, 1, 2], [0, 4, 1], [0, 1, C - 1], [0, 1, C - 1]], device="cuda")
        v = torch.tensor([[0.3, -0.5, 1.0], [0.1, 0.2, -1.0], [1.0, 0.0, 0.5], [-2.0, -2.0, 1.0]], device="cuda")
        for T in (0.1, 0.25):
            loss, grad = gp.distill_tensors(x, at, v, T, grad_loss=torch.ones(1, device="cuda"))
            want, wants = answers.distill(X, at.cpu().numpy(), wide(v), T, np.ones(4))
            assert np.isfinite(want).all() and (np.abs(wide(loss) - want) <= 208 * U * np.abs(want)).all()
            assert (np.abs(wide(grad) - wants) <= 208 * U * T + np.abs(wants) * 2.0 ** -8 * (dtype == "bf16")).all()
