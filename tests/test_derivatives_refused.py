"""What automatic differentiation cannot follow is refused, not dropped: tangents of forward mode, and traces that would keep a result's memory alone."""
import pytest

import paper_2207_12000_amd as gp


def calls():
    import torch
    f, v, w = torch.randn(4, 8), torch.randn(8), torch.randn(4, 3)
    at, t = torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    s, g = torch.zeros(4, 2), torch.zeros(4, 8)
    return [(lambda x: gp.layer_norm_tensors(x, v, v), f), (lambda x: gp.layer_norm_tensors(f, x), v), (lambda x: gp.layer_norm_tensors(f, None, x), v),
            (lambda x: gp.layer_norm_tensors(f, x, out=g, stats=s), v), (lambda x: gp.log_probs_tensors(x, t, top=2), f), (lambda x: gp.log_probs_tensors(x, stats=s), f),
            (lambda x: gp.distill_tensors(x, at, w), f), (lambda x: gp.distill_tensors(x, at, w, grad_loss=v[:1]), f), (lambda x: gp.distill_tensors(f, at, x), w),
            (lambda x: gp.embedding_tensors(x, t), f)]


@pytest.mark.parametrize("i", range(len(calls())))
def test_tangents_are_refused(i):
    import torch
    from torch.autograd import forward_ad
    call, x = calls()[i]
    with forward_ad.dual_level():
        with pytest.raises(ValueError, match="forward-mode"):
            call(forward_ad.make_dual(x, torch.ones_like(x)))
        with pytest.raises(ValueError, match="on the GPU"):  # a level alone is none of the call's business
            call(x)


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("i", range(len(calls())))
def test_traces_are_refused(i, grad):
    import torch
    call, x = calls()[i]
    with pytest.raises(ValueError, match="torch.jit.trace"):
        torch.jit.trace(call, (x.requires_grad_(grad),), check_trace=False)


def test_transforms_of_functions_are_refused():
    import torch
    call, x = calls()[0]
    for transform in (torch.func.vmap(lambda r: call(r[None])), torch.func.grad(lambda r: call(r).sum()), lambda r: torch.func.jvp(call, (r,), (r,))):
        with pytest.raises((ValueError, RuntimeError)):
            transform(x)
