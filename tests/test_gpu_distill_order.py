"""Entries of a teacher's list that name one class are added up in their order, whichever kernel a row goes to.

With the named classes' logits at -inf, a temperature and a gradient of the loss of 1, a class's gradient is 0 less its entries' probabilities: those of a list
of different classes are the probabilities themselves, and a list that names one class for all gives the sum that fp32 makes of them one after another, exactly.
"""
import numpy as np
import pytest

import paper_2207_12000_amd as gp

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


@pytest.mark.parametrize("N", [3, 5000])
@pytest.mark.parametrize("C,K", [(3, 2), (12, 8), (20, 16), (40, 32), (47, 8), (80, 64), (130, 64), (300, 33), (512, 64), (700, 64), (3000, 40), (70_000, 64)])
def test_entries_of_one_class_are_added_up_in_order(N, C, K):
    import torch
    if N * C > 40_000_000:
        N = 700
    gen = torch.Generator(device="cuda").manual_seed(C + K)
    x = torch.randn(N, C, generator=gen, device="cuda")
    x[:, :K] = -float("inf")
    v = 4 * torch.randn(N, K, generator=gen, device="cuda")
    each = torch.rand(N, K, generator=gen, device="cuda").argsort(1).int()
    one = torch.ones(1, device="cuda")
    _, grad = gp.distill_tensors(x, each, v, grad_loss=one)
    q = -grad.gather(1, each.long()).cpu().numpy()
    assert (q > 0).all() and len({float(n) for n in q[0]}) > K // 2
    want = np.zeros(N, dtype=np.float32)
    for k in range(K):
        want = want + q[:, k]
    stats = torch.empty(N, 2, device="cuda")
    for at in (each[:, :1].expand(N, K).contiguous(), torch.full_like(each, K - 1)):
        _, grad = gp.distill_tensors(x, at, v, grad_loss=one)
        gp.distill_tensors(x, at, v, stats=stats)
        again = gp.distill_grad_tensors(x, at, v, stats, one)
        for got in (grad, again):
            assert np.array_equal(-got.gather(1, at[:, :1].long())[:, 0].cpu().numpy(), want)
