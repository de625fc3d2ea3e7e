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


def test_what_is_written_in_place_is_seen_by_automatic_differentiation():
    """A backward pass that kept a matrix which a call has written since is an error, not a wrong gradient."""
    import torch
    def square(n=6):
        return torch.randn(n, n, device="cuda")
    W, M, out, grad = (square().requires_grad_() for _ in range(4))
    tokens = torch.randint(0, 6, (6,), device="cuda")
    spare = square(), square()
    for kept, write in ((W, lambda: gp.muon_step_tensors(W, M, square(), 0.1)), (M, lambda: gp.muon_step_tensors(W, M, square(), 0.1)),
                        (out, lambda: gp.muon_step_tensors(*spare, square(), 0.1, W_out=out, M_out=grad)),
                        (out, lambda: gp.orthogonalize_tensors(square(), out=out)), (out, lambda: gp.embedding_tensors(square(), tokens, out=out)),
                        (grad, lambda: gp.embedding_grad_tensors(tokens, square(), 6, out=grad)),
                        (grad, lambda: gp.embedding_grad_tensors(tokens, square(), 6, out=grad, accumulate=True))):
        y = square().requires_grad_() @ kept
        write()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
    before = [t._version for t in (W, M, out, grad, *spare)]
    gp.embedding_tensors(out.detach(), tokens), gp.embedding_grad_tensors(tokens, grad.detach(), 6), gp.orthogonalize_tensors(out.detach())
    gp.muon_step_tensors(*spare, square(), 0.1, W_out=square(), M_out=square())
    assert [t._version for t in (W, M, out, grad, *spare)] == before   # what is only read keeps its version


@pytest.mark.parametrize("types", [("float32", "float32"), ("bfloat16", "float32"), ("float32", "bfloat16")])
@pytest.mark.parametrize("shape", [(), (40,), (5, 8), (0,)])
def test_a_lookup_of_learned_rows_has_their_gradient(shape, types):
    """Whole numbers, so that sums in any order are equal: against indexing, through gradients of several layouts."""
    import torch
    dtype, out_dtype = (getattr(torch, t) for t in types)
    gen = torch.Generator(device="cuda").manual_seed(0)
    tokens = torch.randint(0, 7, shape, generator=gen, device="cuda")
    weight = torch.randint(-3, 4, shape + (6,), generator=gen, device="cuda").float()
    start = torch.randint(-8, 9, (7, 6), generator=gen, device="cuda").to(dtype)
    turned = lambda y: y.flatten(0, -2).t() if y.dim() > 1 else y  # noqa: E731
    for loss in (lambda y: (y * weight).sum(), lambda y: y.sum(), lambda y: (y.sum(-1) * weight[..., 0]).sum(),
                 lambda y: (turned(y) * turned(weight)).sum(), lambda y: (y.sum(0) * weight[:1].sum(0)).sum() if y.dim() > 1 else y.sum()):
        table, same = start.clone().requires_grad_(), start.clone().float().requires_grad_()
        rows = gp.embedding_tensors(table, tokens, scale=2.0, out_dtype=out_dtype)
        assert rows.requires_grad and rows.dtype == out_dtype and rows.shape == shape + (6,)
        loss(rows.float()).backward()
        loss((2.0 * same[tokens])).backward()
        assert table.grad.dtype == dtype and torch.equal(table.grad.float(), same.grad)


def test_a_lookup_outside_automatic_differentiation_is_as_it_was():
    import torch
    table, tokens = torch.randn(5, 4, device="cuda").requires_grad_(), torch.tensor([3, -1, 0], device="cuda")
    with torch.no_grad():
        assert not gp.embedding_tensors(table, tokens).requires_grad
    out = torch.empty(3, 4, device="cuda")
    assert gp.embedding_tensors(table, tokens, out=out) is out and not out.requires_grad
    assert torch.equal(out, gp.embedding_tensors(table, tokens).detach()) and torch.equal(out, gp.embedding_tensors(table.detach(), tokens))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    rows = gp.embedding_tensors(table, tokens, stream=side.cuda_stream)
    side.synchronize()
    rows.sum().backward()
    assert torch.equal(table.grad, torch.tensor([1.0, 0.0, 0.0, 1.0, 0.0], device="cuda")[:, None].expand(5, 4))
    with pytest.raises(ValueError):
        gp.embedding_tensors(table[0], tokens)
    with pytest.raises(ValueError):
        gp.embedding_tensors(table, tokens.float())
