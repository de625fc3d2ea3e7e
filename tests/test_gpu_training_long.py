"""The gradient of embedding rows on the way that long lists take (sorted tokens, tiles, joins): more than 4,096 tokens.

Tolerances are those of tests/test_gpu_training.py.  What the sizes below reach is checked without a GPU in
tests/test_training_launches.py.
"""
import numpy as np
import pytest

import paper_2207_12000_amd as gp
from test_gpu_training import check_gradient, padded, same_bits, tokens_of, types

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


KINDS = [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")]

# N, V, d, pad, skew: places by counting (up to 8,192 tokens), then sorts of 4 and of 16 entries per thread; V with one, two and three digits
SHAPES = [(4097, 41, 1, 0, 1), (5003, 900, 47, 1, 1), (5000, 90_000, 130, 3, 1), (4500, 40, 602, 1, 1), (8193, 600, 5, 1, 1), (20_011, 3000, 100, 4, 0),
          (20_011, 500_000, 9, 2, 3), (9001, 4_200_000, 3, 1, 1), (2 ** 20 + 77, 50_000, 6, 1, 1)]


@pytest.mark.parametrize("index", ["i32", "i64"])
@pytest.mark.parametrize("kinds", KINDS)
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("N,V,d,pad,skew", SHAPES)
def test_types_and_strides(N, V, d, pad, skew, kinds, accumulate, index):
    import torch
    ty = types()
    rng = np.random.default_rng(d)
    tokens = torch.from_numpy(tokens_of("hot", N, V - 3, rng)).to(ty[index]).cuda()   # (the last rows have no token)
    tokens[::13] = -1
    if index == "i64":
        tokens[::17] += 2 ** 32   # (no row either)
    _, up = padded(N, d, d + pad, ty[kinds[0]], skew)
    up.copy_(torch.from_numpy(rng.normal(size=(N, d)).astype(np.float32)))
    flat, out = padded(V, d, d + 2 * pad, ty[kinds[1]], skew, fill=0.25)
    ws = torch.full((gp.gp_embedding_grad_workspace(N, V, d),), 255, dtype=torch.uint8, device="cuda")
    gp.embedding_grad_tensors(tokens, up, V, scale=2.0, out=out, accumulate=accumulate, workspace=ws)
    check_gradient(out, tokens, up, V, 2.0, before=0.25 if accumulate else None)
    first = out.clone()
    flat[skew:skew + V * (d + 2 * pad)].view(V, -1)[:, :d] = 0.25
    assert bool((flat == 0.25).all())                                                 # nothing beside the rows was written
    gp.embedding_grad_tensors(tokens, up, V, scale=2.0, out=out, accumulate=accumulate)
    assert same_bits(out, first)


@pytest.mark.parametrize("kinds", KINDS)
@pytest.mark.parametrize("N,V,d", [(6000, 500, 36), (20_000, 300_000, 36), (150_000, 47, 47)])
def test_replays(N, V, d, kinds):
    import torch
    ty = types()
    tokens, up = torch.empty(N, dtype=torch.int32, device="cuda"), torch.empty(N, d, dtype=ty[kinds[0]], device="cuda")
    out = torch.empty(V, d, dtype=ty[kinds[1]], device="cuda")
    ws = torch.empty(gp.gp_embedding_grad_workspace(N, V, d), dtype=torch.uint8, device="cuda")

    def call():
        gp.embedding_grad_tensors(tokens, up, V, out=out, workspace=ws)

    def fill(seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        tokens.copy_(torch.randint(-1, V if seed % 2 else 4, (N,), generator=gen, device="cuda"))
        up.copy_(torch.randn(N, d, generator=gen, device="cuda"))
        out.fill_(float("nan"))

    fill(0)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(1, 5):
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        out.fill_(float("nan"))
        call()
        torch.cuda.synchronize()
        assert same_bits(replayed, out)
        check_gradient(out, tokens, up, V, 1.0)


@pytest.mark.parametrize("kinds", KINDS)
def test_one_gradient_row_for_all_tokens(kinds):
    import torch
    ty = types()
    rng = np.random.default_rng(15)
    tokens = torch.from_numpy(rng.integers(-1, 2000, 20_000)).cuda()
    up = torch.from_numpy(rng.normal(size=(1, 37))).to(ty[kinds[0]]).cuda().expand(20_000, 37)
    check_gradient(gp.embedding_grad_tensors(tokens, up, 2000, out_dtype=ty[kinds[1]]), tokens, up, 2000, 1.0)


def test_a_row_with_infinity_or_nan_stays_alone():
    import torch
    N, V, d = 9000, 700, 9
    tokens = (torch.arange(N, device="cuda") % (V + 1)).to(torch.int32)   # (V names no row)
    up = torch.ones(N, d, device="cuda")
    up[3, 2], up[V + 1 + 5, 4], up[V] = float("inf"), float("nan"), float("nan")
    want = torch.bincount(tokens.long(), minlength=V + 1)[:V].float()[:, None].repeat(1, d)
    want[3, 2], want[5, 4] = float("inf"), float("nan")
    assert torch.allclose(gp.embedding_grad_tensors(tokens, up, V), want, rtol=0, atol=0, equal_nan=True)


def gaps_of(limit, first, last, seed):
    """Named rows with gaps of around `limit` rows between them, some of none and some far longer, so that they begin and end on every side of the
    multiples of `limit`; `first` rows before and `last` rows behind.  Tokens (more than 4,096 of them) and V: for gaps of 32, a table of more than 16 rows
    per token, for 256 of fewer."""
    rng = np.random.default_rng(seed)
    count, often = (4500, 1) if limit == 32 else (3000, 30)
    usual = [limit - 2, limit - 1, limit, limit + 1, limit + 2, 2 * limit - 1, 2 * limit, 2 * limit + 1]
    gaps = rng.choice(usual + [0, 1, 7 * limit + 5], size=count - 1, p=[0.11] * 8 + [0.04] * 3)
    named = first + np.concatenate([[0], np.cumsum(gaps + 1)])
    V = int(named[-1]) + 1 + last
    tokens = rng.permutation(np.repeat(named, often))
    assert len(tokens) > 4096 and (V > 16 * len(tokens)) == (limit == 32)
    return named, tokens, V, float(often)


GAPS = [(limit, first, last) for limit in (32, 256) for first in (0, 1, limit - 1, limit, limit + 1, 3 * limit + 2) for last in (0, 1, limit, limit + 1, 5 * limit)]


@pytest.mark.parametrize("limit,first,last", GAPS)
def test_rows_in_gaps_around_their_limits_are_zero(limit, first, last):
    """Gaps of up to 32 rows, or 256 where the table has at most 16 rows per token, are written beside the run behind them, longer ones by wavefronts
    of another launch."""
    import torch
    named, tokens, V, often = gaps_of(limit, first, last, 64 * limit + first + 7 * last)
    d = 5
    tokens = torch.from_numpy(tokens).to(torch.int32).cuda()
    for dtype, pad, skew in ((torch.float32, 0, 0), (torch.bfloat16, 2, 1), (torch.float32, 3, 3)):
        flat, out = padded(V, d, d + pad, dtype, skew, fill=0.25)
        out.fill_(float("nan"))
        gp.embedding_grad_tensors(tokens, torch.ones(tokens.numel(), d, device="cuda", dtype=dtype), V, out=out)
        want = torch.zeros(V, d, device="cuda", dtype=dtype)
        want[torch.from_numpy(named).cuda()] = often
        assert torch.equal(out, want)
        out.fill_(0.25)
        assert bool((flat == 0.25).all())
