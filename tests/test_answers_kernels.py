"""The kernels that rows of logits go to hold what they are given: elements of the logits' own type, and as many as the longest part of a row has.
Seen without a GPU (tests/launches.py)."""
import re
import shutil

import pytest

import paper_2207_12000_amd as gp
from launches import launches
from test_answers_launches import answer, distill

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not found")


@pytest.mark.parametrize("dtype", [gp.GP_F32, gp.GP_BF16])
def test_long_rows_are_read_as_they_are_stored_and_held_whole(dtype):
    letter, vec = ("f", 4) if dtype == gp.GP_F32 else ("t", 8)
    widths = sorted({*range(1100, 140_000, 4111), *(k * 32_768 + s for k in (1, 2, 3, 4, 8, 12, 13, 4095, 8192) for s in (-1, 0, 1) if k * 32_768 + s <= 2 ** 28), 50_257, 100_003, 2 ** 28})
    calls = [f(N, C, 5, dtype, **kw) for C in widths for N in (1, 3, 256, 600, 5000) for f, kw in ((answer, {}), (distill, {}), (distill, dict(grad_ptr=0)))]
    for (name, kw), result in zip(calls, launches(calls)):
        assert result["status"] == gp.GP_OK
        for l in result["launches"]:
            if "_rows" not in l["kernel"]:
                continue
            of, v, held, lanes = re.search(r"gp_(?:answer|distill)_rowsI([ft])Li(\d+)ELi(\d+)ELi(\d+)E", l["kernel"]).groups()
            v, held, lanes = int(v), int(held), int(lanes)
            assert of == letter and v == vec, (name, kw["N"], kw["C"], l)
            teams = l["block"][0] // lanes
            if l["grid"][0] < 1 << 20 and kw["N"] % teams == 0:
                parts = l["grid"][0] * teams // kw["N"]
                assert -(-(-(-kw["C"] // v)) // parts) <= held * lanes, (name, kw["N"], kw["C"], l)
