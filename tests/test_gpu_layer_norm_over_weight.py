"""Layer norm's gradients of weight and bias written over the weight itself, with few rows and many, and in place of x: as if into other memory."""
import pytest

import paper_2207_12000_amd as gp

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d", [(1, 20), (50, 33), (1000, 256), (1024, 1024), (3000, 100), (4, 17_000)])
def test_over_the_weight(N, d, dtype):
    import torch
    ty = torch.float32 if dtype == "f32" else torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(N + d)
    x, g, w = (torch.randn(*s, generator=gen, device="cuda").to(ty) for s in ((N, d), (N, d), (d,)))
    stats = torch.empty(N, 2, device="cuda")
    gp.layer_norm_tensors(x, w, stats=stats)
    want = gp.layer_norm_grad_tensors(g, x, stats, w)
    for x_grad in ("new", "x", "grad"):
        for which in (0, 1):
            X, G, W, other = x.clone(), g.clone(), w.clone(), torch.empty_like(w)
            before = W._version
            got = gp.layer_norm_grad_tensors(G, X, stats, W, x_grad={"new": None, "x": X, "grad": G}[x_grad], weight_grad=(W, other)[which], bias_grad=(other, W)[which])
            assert all(torch.equal(p, q) for p, q in zip(got, want)) and W._version > before
            X, G, W = x.clone(), g.clone(), w.clone()
            held = torch.ones_like(w)
            clean = gp.layer_norm_grad_tensors(g, x, stats, w, weight_grad=w.clone(), bias_grad=held.clone(), accumulate=True)
            got = gp.layer_norm_grad_tensors(G, X, stats, W, x_grad={"new": None, "x": X, "grad": G}[x_grad], weight_grad=W, bias_grad=held, accumulate=True)
            assert all(torch.equal(p, q) for p, q in zip(got, clean))
