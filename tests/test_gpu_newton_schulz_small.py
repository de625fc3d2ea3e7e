"""Newton-Schulz directions of matrices with a short side: sums of few terms, in which dropped bits do not average out.

The bar: 33 bits are more than fp32's 24, so what is left are fp32 roundings, of another order and number than those of fp32 steps.  An emulation puts the
error at up to 1.25 of theirs (geometric mean over matrices), and that of 22 bits at up to 2; the bar is 1.4.
"""
import numpy as np
import pytest

import paper_2207_12000_amd as gp
from test_gpu_newton_schulz import errors, inputs, steps

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


@pytest.mark.parametrize("kind", ["normal", "gradient"])
@pytest.mark.parametrize("shape", [(1, 7), (7, 1), (2, 2), (3, 5), (4, 4), (8, 8), (40, 8), (16, 16), (16, 40), (32, 32), (31, 256), (256, 17)])
def test_short_sides_are_as_near_as_fp32(shape, kind):
    G = inputs(shape, 256, kind)
    exact = steps(G.double())
    mean = lambda X: float(errors(X, exact).clamp_min(1e-12).log().mean().exp())  # noqa: E731
    assert mean(gp.orthogonalize_tensors(G)) <= 1.4 * mean(steps(G))
