"""A teacher that names classes which the student has at its type's lowest value: the loss is as large as it is, at temperatures below 1 too, where (logit - largest) / T is
beyond fp32 though T^2 times it is not.  Bounds: those of the other tests of distillation."""
import numpy as np
import pytest

import paper_2207_12000_amd as gp
from test_gpu_distill import check
from test_gpu_layer_norm import types, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [5, 40, 300, 900, 5000, 33_000, 100_000])
def test_named_classes_at_the_lowest_value(C, dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(C)
    ty = types()[dtype]
    lowest = torch.finfo(ty).min
    x = torch.randn(6, C, generator=gen, device="cuda")
    x[0, :3] = lowest
    x[1, 1] = lowest
    x[2, 2:] = lowest
    x[3] = lowest
    x[4, : C // 2] = lowest
    x = x.to(ty)
    at = torch.tensor([[0, 1, 2], [0, 1, 2], [0, 1, 4], [0, 3, 1], [C - 1, 0, -1], [0, 1, C - 1]], device="cuda")
    v = torch.randn(6, 3, generator=gen, device="cuda")
    g = torch.randn(6, generator=gen, device="cuda")
    for T in (0.25, 0.5, 0.9):
        loss, grad = gp.distill_tensors(x, at, v, T, grad_loss=g)
        want = wide(loss)
        assert np.isfinite(want).all()
        with np.errstate(all="ignore"):
            check(loss, grad, x, at, v, T, g)
