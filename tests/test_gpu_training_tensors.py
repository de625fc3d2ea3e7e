"""The training operators' calls on torch tensors: shapes, and what automatic differentiation sees of them."""
import pytest

import paper_2207_12000_amd as gp

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


@pytest.mark.parametrize("shape", [(), (1,), (5,), (1, 4), (2, 3), (2, 1, 3), (0,), (2, 0)])
def test_gradient_takes_what_the_lookup_returns(shape):
    """tokens of any number of dimensions, none included."""
    import torch
    table = torch.randn(7, 3, device="cuda")
    tokens = torch.randint(0, 7, shape, device="cuda")
    rows = gp.embedding_tensors(table, tokens)
    assert rows.shape == shape + (3,) and torch.equal(rows, table[tokens])
    got = gp.embedding_grad_tensors(tokens, torch.ones_like(rows), 7)
    assert torch.equal(got, torch.bincount(tokens.flatten(), minlength=7).float()[:, None].expand(7, 3))
    for bad in (torch.ones(shape + (3, 3), device="cuda"), torch.ones((), device="cuda"), torch.ones((8, 3), device="cuda")):
        with pytest.raises(ValueError):
            gp.embedding_grad_tensors(tokens, bad, 7)
