"""Layer norm of rows at the ends of what fp32 holds: rows that are no numbers, rows whose squares or sums are beyond it, and rows far from zero."""
import numpy as np
import pytest

import paper_2207_12000_amd as gp
from test_gpu_layer_norm import types

pytestmark = pytest.mark.gpu

# a lane to a row's vector, part of a wavefront, a wavefront, workgroups of each size, rows beyond the registers
WIDTHS = [1, 3, 9, 47, 100, 300, 1000, 1501, 5000, 9001, 16_384, 32_768, 40_000]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_statistics_of_rows_that_are_no_numbers_are_none(d, dtype):
    import torch
    inf, nan = float("inf"), float("nan")
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn(7, d, generator=gen, device="cuda").to(types()[dtype])
    x[0, d // 2], x[1, 0], x[2, d - 1], x[3, d // 3] = inf, -inf, nan, -nan
    x[4, :] = inf
    stats = torch.empty(7, 2, device="cuda")
    y = gp.layer_norm_tensors(x, stats=stats)
    assert bool(stats[:5, 1].isnan().all()) and not bool(stats[:5, 0].isfinite().any()) and bool(y[:5].isnan().all())
    assert bool(stats[5:].isfinite().all()) and bool(y[5:].isfinite().all())
    want = gp.layer_norm_tensors(x[5:].contiguous(), stats=torch.empty(2, 2, device="cuda"))
    assert torch.equal(y[5:], want)
