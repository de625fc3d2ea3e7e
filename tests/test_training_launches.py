"""What the training operators launch, seen without a GPU (tests/launches.py): sizes that the runtime takes, kernels that shapes reach."""
import re
import shutil

import pytest

import paper_2207_12000_amd as gp
from launches import launches

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not found")

P = 4096  # stands for an address


def lookup(**kw):
    a = dict(table_ptr=P, ldt=8, dtype=gp.GP_F32, V=10, d=8, tokens_ptr=P, index=gp.GP_I32, N=4, scale=1.0, out_ptr=P, ldo=8,
             out_dtype=gp.GP_F32)
    return "gp_embedding", {**a, **kw}


def grad(**kw):
    a = dict(tokens_ptr=P, index=gp.GP_I32, N=4, grad_ptr=P, ldg=8, dtype=gp.GP_F32, d=8, scale=1.0, V=10, table_grad_ptr=P, ldt=8,
             out_dtype=gp.GP_F32, accumulate=False, workspace_ptr=P, workspace_bytes=1 << 50)
    return "gp_embedding_grad", {**a, **kw}


def check_sizes(result):
    """hipLaunchKernel takes fewer than 2^32 threads in each dimension, 1024 to a workgroup."""
    assert result["status"] == gp.GP_OK and result["launches"]
    for l in result["launches"]:
        assert all(0 < g * b < 1 << 32 for g, b in zip(l["grid"], l["block"])), l
        assert l["block"][0] * l["block"][1] * l["block"][2] <= 1024, l


@pytest.mark.parametrize("N", [1, 2 ** 30, 2 ** 34 - 1024, 2 ** 34 + 5, 2 ** 45])
@pytest.mark.parametrize("d", [1, 8])
def test_lookups_of_any_length_can_be_launched(N, d):
    for dtype in (gp.GP_F32, gp.GP_BF16):
        check_sizes(launches([lookup(N=N, d=d, dtype=dtype, out_dtype=dtype)])[0])


@pytest.mark.parametrize("N", [0, 4097, 100_000, 2 ** 27, 2 ** 31 - 1])
@pytest.mark.parametrize("V", [1, 2 ** 28, 2 ** 31 - 4000, 2 ** 31 - 1])
def test_gradients_of_any_table_can_be_launched(N, V):
    for dtype in (gp.GP_F32, gp.GP_BF16):
        check_sizes(launches([grad(N=N, V=V, d=1, dtype=dtype, out_dtype=dtype)])[0])
