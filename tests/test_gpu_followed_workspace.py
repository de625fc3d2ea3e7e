"""A caller's workspace is the one that is used where automatic differentiation follows a call, too."""
import pytest

import paper_2207_12000_amd as gp

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


@pytest.mark.parametrize("which", ["log_probs", "distill"])
def test_the_workspace_that_is_given_is_used(which):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(0)
    N, C = 2, 60_000
    x = torch.randn(N, C, generator=gen, device="cuda", requires_grad=True)
    tokens = torch.tensor([5, 59_999], device="cuda")
    at, v = torch.randint(0, C, (N, 4), generator=gen, device="cuda"), torch.randn(N, 4, generator=gen, device="cuda")

    def call(ws):
        x.grad = None
        if which == "log_probs":
            a = gp.log_probs_tensors(x, tokens, top=3, workspace=ws)
            (a.logp.sum() + 0.5 * a.entropy.sum()).backward()
            return a.logp.detach(), a.entropy.detach(), a.top_logp, a.top_index, x.grad
        loss = gp.distill_tensors(x, at, v, 2.0, workspace=ws)
        loss.sum().backward()
        return loss.detach(), x.grad

    need = gp.gp_log_probs_workspace(N, C, 3) if which == "log_probs" else gp.gp_distill_workspace(N, C)
    assert need > 0
    want = call(None)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    got = call(ws)
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and bool(ws.any())
    with pytest.raises(gp.GpError):
        call(ws[: need - 256])
    with pytest.raises(ValueError):
        call(ws.view(torch.int32))
