"""What the training operators launch, seen without a GPU (tests/launches.py): sizes that the runtime takes, kernels that shapes reach."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2207_12000_amd as gp
from launches import launches
from test_kernel_registers import READELF, code_objects

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


def orth(rows, cols, count=1, **kw):
    a = dict(G_ptr=P, ldg=cols, stride_g=rows * cols, dtype=gp.GP_F32, rows=rows, cols=cols, count=count, steps=2, coeff=None, eps=1e-7, out_ptr=P,
             ldo=cols, stride_o=rows * cols, workspace_ptr=P, workspace_bytes=1 << 60)
    return "gp_orthogonalize", {**a, **kw}


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


@pytest.fixture(scope="module")
def own_lds(tmp_path_factory):
    """The LDS that a kernel has by itself, in bytes, by its name."""
    if not os.path.exists(READELF):
        pytest.skip("llvm-readelf not found")
    found = {}
    for i, code in enumerate(code_objects()):
        path = tmp_path_factory.mktemp("co") / f"{i}.co"
        path.write_bytes(code)
        notes = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True, check=True).stdout
        for entry in re.split(r"\n  - \.agpr_count", notes)[1:]:
            found[re.search(r"\.name:\s+(\S+)", entry).group(1)] = int(re.search(r"\.group_segment_fixed_size:\s+(\d+)", entry).group(1))
    return found


def test_lds_beyond_64_kb_is_asked_for(own_lds):
    """A kernel has 64 KB, its own and what the launch adds together; the launch's part of more than that needs the runtime's leave."""
    calls = [orth(*shape) for shape in ((16, 16), (40, 256), (64, 64), (100, 1000), (300, 300), (704, 2000), (768, 768), (1024, 1024), (1536, 1536),
                                        (2048, 2048), (4096, 4096), (4096, 1024))] + [orth(1024, 4096, 2), orth(4096, 1024, 2)]
    calls += [grad(N=N, V=V, d=d, ldg=d, ldt=d, dtype=dtype) for N, V, d in ((4096, 1000, 128), (4096, 1000, 3), (9000, 60, 16), (20_000, 100_000, 16), (2_000_000, 3_000_000, 16))
              for dtype in (gp.GP_F32, gp.GP_BF16)]
    large = 0
    for result in launches(calls):
        check_sizes(result)
        for l in result["launches"]:
            total = own_lds[l["kernel"]] + l["lds"]
            assert total <= 160 * 1024 and (total <= 64 * 1024 or l["lds_asked"] >= l["lds"]), (l, own_lds[l["kernel"]])
            large += total > 64 * 1024
    assert large


def test_an_allocation_that_fails_is_an_error_of_the_call():
    """Timed launches are noted in memory of the library's own; without any, a call says so, and the process lives on."""
    W = dict(W_ptr=P, W_out_ptr=P, ldw=8, stride_w=80, M_ptr=P, M_out_ptr=P, ldm=8, stride_m=80, G_ptr=P, ldg=8, stride_g=80, dtype=gp.GP_F32, rows=10,
             cols=8, count=2, lr=0.1, momentum=0.9, weight_decay=0.0, nesterov=True, steps=5, coeff=None, eps=1e-7, workspace_ptr=P, workspace_bytes=1 << 30)
    calls = [lookup(), grad(), grad(N=0), grad(N=5000), orth(8, 8), ("gp_muon_step", W)]
    for name, kw in calls:
        failed, after = launches([(name, {**kw, "no_memory": True}), (name, kw)])
        assert failed["status"] == gp.GP_ERR_OOM_HOST and after["status"] == gp.GP_OK, name


def kernels(result):
    """The names of what was launched, in order."""
    assert result["status"] == gp.GP_OK
    return [re.search(r"gp_(?:token|sum|join|zero|ns|embedding)\w*?(?=I[A-Z]|E[A-Z]|I[ft]|E[v]|ENS)", l["kernel"]).group(0) for l in result["launches"]]


def test_shapes_of_long_lists_reach_what_they_are_for():
    from test_gpu_training_long import SHAPES
    ways = set()
    for (N, V, d, _, _), result in zip(SHAPES, launches([grad(N=N, V=V, d=d, ldg=d, ldt=d) for N, V, d, _, _ in SHAPES])):
        seen = kernels(result)
        assert seen[-2:] == ["gp_sum_tiles", "gp_join_tiles"] and "gp_sum_short" not in seen, (N, V, seen)
        items = {int(m) for l in result["launches"] for m in re.findall(r"gp_token_countILi(\d+)E", l["kernel"])}
        ways.add(("rank",) if "gp_token_rank" in seen else (seen.count("gp_token_scatter"), *items))
    assert {("rank",), (1, 4), (2, 4), (3, 4), (2, 16)} <= ways


def test_gaps_of_long_lists_reach_both_ways_of_writing_them():
    from test_gpu_training_long import GAPS, gaps_of
    sizes = []
    for limit, first, last in GAPS:
        named, tokens, V, _ = gaps_of(limit, first, last, 64 * limit + first + 7 * last)
        inside = named[1:] - named[:-1] - 1
        assert (inside > limit).any() and ((inside <= limit) & (inside >= limit - 2)).any()
        assert {int(x) % limit for x in named} == set(range(limit))   # (first rows of gaps on all sides of a wavefront's rows)
        sizes.append((len(tokens), V))
    for result in launches([grad(N=N, V=V, d=5) for N, V in sizes]):
        assert kernels(result)[-2:] == ["gp_sum_tiles", "gp_join_tiles"]


def test_newton_schulz_shapes_reach_every_kernel():
    from test_gpu_newton_schulz import PANELS, SHAPES, SMALL, THIRTY_TWOS, TILES

    def seen(shapes, name):
        return {re.search(name, l["kernel"]).group(1) for result in launches([orth(*s, dtype=d) for s in shapes for d in (gp.GP_F32, gp.GP_BF16)])
                for l in result["launches"] if re.search(name, l["kernel"])}

    types = ("f", "t")
    assert seen(SMALL, r"gp_ns_(tiny)") == {"tiny"} and seen(SHAPES[len(SMALL):], r"gp_ns_(tiny)") == set()
    assert seen(SMALL, r"gp_ns_tinyILi(.*)EEvNS") == {f"{b}E{t}{o}" for b in (1, 2, 3, 4) for t, o in (("f", "f"), ("t", "t"))}
    assert seen(PANELS, r"gp_ns_panelILi(.*)EEEvNS") == {f"{m}E{t}Lb{last}" for m in (64, 128) for t, last in (("f", 0), ("f", 1), ("t", 1))}
    assert seen(THIRTY_TWOS, r"gp_ns_product_smallI(.*)EEEvNS") == {"fLb0ELb0", "fLb0ELb1", "fLb1ELb0", "tLb1ELb0"}
    wide, tall = {(64, 64), (128, 128), (128, 256), (192, 192), (256, 256)}, {(256, 128)}
    last = {f"{m}ELi{n}E{t}" for m, n in wide | tall for t in types}
    assert {re.sub(r"E(Li\dE){3}", "E", x) for x in seen(TILES, r"gp_ns_productILi(\S*)Lb1EEEvNS")} == last
    assert {re.sub(r"E(Li\dE){3}", "E", x) for x in seen(TILES, r"gp_ns_productILi(\S*)Lb0EEEvNS")} == {f"{m}ELi{n}Ef" for m, n in wide}
    assert seen(SHAPES, r"gp_ns_normsILi(\d+)") == {"256", "1024"}


def test_muon_shapes_reach_every_kernel_that_writes_weights():
    """The same cuts, whatever U is made of."""
    from test_gpu_newton_schulz import SHAPES
    calls = []
    for rows, cols, count in SHAPES:
        calls.append(("gp_muon_step", dict(W_ptr=P, W_out_ptr=P, ldw=cols, stride_w=rows * cols, M_ptr=P, M_out_ptr=P, ldm=cols, stride_m=rows * cols, G_ptr=P,
                                           ldg=cols, stride_g=rows * cols, dtype=gp.GP_BF16, rows=rows, cols=cols, count=count, lr=0.1, momentum=0.9,
                                           weight_decay=0.0, nesterov=True, steps=2, coeff=None, eps=1e-7, workspace_ptr=P, workspace_bytes=1 << 60)))
    with_weights = launches(calls)
    plain = launches([orth(*s) for s in SHAPES])
    products = lambda result: [l["kernel"] for l in result["launches"] if "gp_ns_product" in l["kernel"] or "gp_ns_panel" in l["kernel"]]  # noqa: E731
    assert [products(a) for a in with_weights] == [products(b) for b in plain]
