"""A row of a teacher without an entry that counts has no loss and no gradient, whatever the gradient of its loss is."""
import pytest

import paper_2207_12000_amd as gp

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [5, 47, 300, 900, 5000, 70_000])
def test_rows_without_an_entry_take_no_part(C, dtype):
    import torch
    inf, nan = float("inf"), float("nan")
    gen = torch.Generator(device="cuda").manual_seed(C)
    x = torch.randn(6, C, generator=gen, device="cuda").to(torch.float32 if dtype == "f32" else torch.bfloat16)
    at = torch.tensor([[1, 2, 3], [1, 1, 4], [-1, C, -7], [0, -1, 3], [4, 3, 2], [2, 2, 2]], device="cuda")
    v = torch.tensor([[-inf, -inf, -inf], [-inf, -inf, -inf], [1.0, 2.0, 3.0], [-inf, 5.0, -inf], [1.0, 2.0, -inf], [-inf, -inf, -inf]], device="cuda")
    plain = gp.distill_tensors(x, at, v, 2.0, grad_loss=torch.ones(6, device="cuda"))
    g = torch.tensor([inf, nan, -inf, inf, 1.0, nan], device="cuda")
    stats = torch.empty(6, 2, device="cuda")
    loss, grad = gp.distill_tensors(x, at, v, 2.0, grad_loss=g, stats=stats)
    again = gp.distill_grad_tensors(x, at, v, stats, g, 2.0)
    assert loss[[0, 1, 2, 3, 5]].tolist() == [0.0] * 5 and loss[4].item() == plain[0][4].item() > 0
    for got in (grad, again):
        assert not bool(got[[0, 1, 2, 3, 5]].any()) and not bool(got.isnan().any())
    assert torch.equal(grad[4], plain[1][4])
