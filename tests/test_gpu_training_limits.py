"""Training operators at sizes where a launch's workgroups no longer cover the work in one go."""
import pytest

import paper_2207_12000_amd as gp

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu(gpu_or_skip):
    yield


def test_lookup_of_more_rows_than_the_workgroups_take_at_once():
    """2^20 workgroups of 1024 rows each, and some: every row of out is written, the last ones in a second round."""
    import torch
    N, V = 2 ** 30 + 12_345, 1009
    table = torch.randn(V, 1, device="cuda").bfloat16()
    tokens = torch.arange(N, dtype=torch.int32, device="cuda").remainder_(V + 1)   # (V names no row)
    out = torch.full((N, 1), float("nan"), dtype=torch.bfloat16, device="cuda")
    gp.embedding_tensors(table, tokens, out=out)
    rows = torch.cat([table, torch.zeros(1, 1, dtype=torch.bfloat16, device="cuda")]).flatten()
    for first in range(0, N, 1 << 27):
        assert torch.equal(out[first:first + (1 << 27), 0], rows[tokens[first:first + (1 << 27)].long()])


@pytest.mark.parametrize("N", [5000, 9000])
def test_gaps_of_a_table_longer_than_the_workgroups_take_at_once(N):
    """2^20 workgroups of four wavefronts of 32 rows, and some: every row of the gradient is written, those behind in a second round."""
    import torch
    V = 2 ** 27 + 1_000_003
    place = torch.randint(0, V, (N,), device="cuda")
    place[:4] = torch.tensor([0, 2 ** 27 - 1, 2 ** 27 + 40, V - 500_000], device="cuda")
    place = place.unique()
    tokens = place[torch.randint(0, place.numel(), (N,), device="cuda")]
    up = torch.ones(N, 1, dtype=torch.bfloat16, device="cuda")
    out = torch.full((V, 1), float("nan"), dtype=torch.bfloat16, device="cuda")
    gp.embedding_grad_tensors(tokens.to(torch.int32), up, V, out=out)
    named, count = tokens.unique(return_counts=True)
    assert torch.equal(out[named, 0], count.bfloat16())
    assert int(torch.count_nonzero(out)) == named.numel()      # (NaN would count)
