"""How near Newton-Schulz steps have to be, and that the bar tells 22 bits from fewer.

The bar.  Operands of 22 bits are rounded four times as coarsely as those of fp32, and the steps stretch both alike: at most four times the error that fp32
steps leave on the same matrices, as the median over a batch.  What a kernel leaves when one of its part products is lost, or all second parts
are, lies beyond it; that is shown here, by emulation.  tests/test_gpu_newton_schulz.py holds the kernels to it.
"""
import numpy as np
import pytest

from newton_schulz_parts import in_64_bits, in_fp32, mistakes, relative_errors, steps_in_parts

TIMES_FP32 = 4.0


def matrices(shape, kind, count=16, seed=0):
    """Normal ones, or a few strong directions over a floor of noise."""
    rng = np.random.default_rng(seed)
    if kind == "normal":
        return rng.normal(size=(count,) + shape).astype(np.float32)
    k = max(1, min(shape) // 8)
    return (1e-3 * (rng.normal(size=(count, shape[0], k)) @ rng.normal(size=(count, k, shape[1])) + 0.2 * rng.normal(size=(count,) + shape))).astype(np.float32)


@pytest.mark.parametrize("kind", ["normal", "gradient"])
@pytest.mark.parametrize("shape", [(1, 7), (2, 2), (5, 3), (16, 16), (16, 40), (63, 65), (64, 64), (40, 256), (256, 40), (70, 90), (100, 300), (128, 128)])
def test_the_bar_for_a_step_s_last_products_in_one_launch(shape, kind):
    check_bar(shape, kind, True)


@pytest.mark.parametrize("kind", ["normal", "gradient"])
@pytest.mark.parametrize("shape", [(130, 257), (300, 140), (200, 200)])
def test_the_bar_for_products_of_their_own(shape, kind):
    check_bar(shape, kind, False)


def check_bar(shape, kind, panel):
    G = matrices(shape, kind)
    exact = in_64_bits(G)
    bar = TIMES_FP32 * np.median(relative_errors(in_fp32(G), exact))
    assert np.median(relative_errors(steps_in_parts(G, panel), exact)) <= bar
    assert np.median(relative_errors(steps_in_parts(G, panel, parts=1), exact)) > bar
    for lost in mistakes(panel):
        assert np.median(relative_errors(steps_in_parts(G, panel, lost), exact)) > bar, lost
