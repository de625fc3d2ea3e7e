"""Newton-Schulz directions and the Muon step on the GPU, at every kernel and tile: as near to 64 bits as operands of 22 bits allow.

The bar is that of tests/test_newton_schulz_bits.py: four times the error that fp32 steps leave on the same matrices (the median over a batch), which a
kernel that has lost one of its part products does not meet.  tests/test_training_launches.py checks, without a GPU, that the shapes reach what they are for.
"""
import numpy as np
import pytest

import paper_2207_12000_amd as gp
from oracle import training
from test_gpu_training import padded, same_bits, types
from test_newton_schulz_bits import TIMES_FP32, matrices

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


# rows, cols, matrices: one launch (up to 32, 48 and 64 on the shorter side) ...
SMALL = [(1, 1, 16), (1, 7, 16), (7, 1, 16), (2, 2, 16), (16, 16, 16), (17, 30, 16), (256, 32, 16), (40, 256, 16), (256, 40, 16), (64, 64, 16), (65, 63, 16), (63, 256, 16)]
# ... a launch for a step's last two products (up to 64 and 128) ...
PANELS = [(1, 300, 16), (63, 257, 16), (257, 63, 16), (70, 90, 16), (100, 1023, 4), (1023, 100, 4), (128, 128, 16)]
# ... tiles of 32, by one workgroup and by several ...
THIRTY_TWOS = [(131, 257, 4), (257, 131, 4), (256, 256, 2), (130, 1030, 1), (1030, 130, 1)]
# ... and of 64, 128, 128 x 256, 192 and 256
TILES = [(150, 2101, 1), (2101, 150, 1), (511, 1001, 2), (203, 3205, 4), (3205, 203, 4), (301, 4801, 4), (4801, 301, 4), (703, 2815, 4), (2815, 703, 4), (401, 6401, 4),
         (6401, 401, 4)]
SHAPES = SMALL + PANELS + THIRTY_TWOS + TILES


def inputs(shape, count, kind, seed=0):
    import torch
    return torch.from_numpy(matrices(shape, kind, count, seed)).cuda()


def steps(U):
    """The definition, in U's own type: fp64, or fp32 throughout."""
    a, b, c = (float(np.float32(x)) for x in training.COEFF)
    X = U / (U.pow(2).sum(dim=(1, 2), keepdim=True).sqrt() + 1e-7)
    tall = X.shape[1] > X.shape[2]
    if tall:
        X = X.transpose(1, 2).contiguous()
    for _ in range(5):
        S = X @ X.transpose(1, 2).contiguous()
        X = a * X + (b * S + c * (S @ S)) @ X
    return X.transpose(1, 2).contiguous() if tall else X


def errors(X, exact):
    return (X.double() - exact).flatten(1).norm(dim=1) / exact.flatten(1).norm(dim=1)


@pytest.mark.parametrize("kind", ["normal", "gradient"])
@pytest.mark.parametrize("rows,cols,count", SHAPES)
def test_directions_are_as_near_as_22_bits_allow(rows, cols, count, kind):
    G = inputs((rows, cols), count, kind)
    exact = steps(G.double())
    got = gp.orthogonalize_tensors(G)
    assert float(errors(got, exact).median()) <= TIMES_FP32 * float(errors(steps(G), exact).median())
    assert same_bits(got, gp.orthogonalize_tensors(G))


@pytest.mark.parametrize("rows,cols,count", SHAPES)
def test_a_bf16_direction_is_the_fp32_one_rounded_once(rows, cols, count):
    G = inputs((rows, cols), count, "gradient").bfloat16()
    assert same_bits(gp.orthogonalize_tensors(G), gp.orthogonalize_tensors(G.float()).bfloat16())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("rows,cols,count", SHAPES)
def test_muon_steps(rows, cols, count, nesterov, dtype):
    """M: two roundings.  W: the direction's bar (the fp32 steps start from their own U), times lr, and three roundings."""
    import torch
    lr, mu, wd = (float(np.float32(x)) for x in (0.02, 0.95, 0.1))
    G = inputs((rows, cols), count, "gradient").to(types()[dtype])
    M0 = 5 * inputs((rows, cols), count, "gradient", 1)
    W0 = inputs((rows, cols), count, "normal", 2) / rows ** 0.5

    def strided(values, pad, skew):   # matrices in rows of their own length, from an odd address; NaN beside them
        flat, all_rows = padded(count * rows, cols, cols + pad, torch.float32, skew)
        view = all_rows.unflatten(0, (count, rows))
        view.copy_(values)
        return flat, view

    w_flat, W = strided(W0, 3, 1)
    m_flat, M = strided(M0, 5, 2)
    gp.muon_step_tensors(W, M, G, lr, mu, wd, nesterov)
    assert int(w_flat.isnan().sum()) == w_flat.numel() - W.numel() and int(m_flat.isnan().sum()) == m_flat.numel() - M.numel()
    W2, M2 = gp.muon_step_tensors(W0, M0, G, lr, mu, wd, nesterov, W_out=torch.empty_like(W0), M_out=torch.empty_like(M0))
    assert same_bits(W, W2) and same_bits(M, M2)

    m, g = M0.double(), G.double()
    want_M = mu * m + g
    assert bool(((M2.double() - want_M).abs() <= 2.0 ** -23 * ((mu * m).abs() + g.abs())).all())
    exact = steps(g + mu * want_M if nesterov else want_M)
    M32 = mu * M0 + G.float()
    near = TIMES_FP32 * float(errors(steps(G.float() + mu * M32 if nesterov else M32), exact).median())
    want_W = (1 - lr * wd) * W0.double() - lr * exact
    norm = lambda x: x.flatten(1).norm(dim=1)  # noqa: E731
    over = norm(W2.double() - want_W) - 3 * 2.0 ** -24 * (norm(W0.double()) + lr * norm(exact))
    assert float((over / (lr * norm(exact))).median()) <= near
