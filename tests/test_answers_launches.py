"""What layer norm, log probabilities and distillation launch, seen without a GPU (tests/launches.py): sizes that the runtime takes, kernels that shapes
reach, LDS, and errors in place of exceptions."""
import shutil

import pytest

import paper_2207_12000_amd as gp
from launches import launches
from test_training_launches import check_sizes

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not found")

P = 4096  # stands for an address
TYPES = (gp.GP_F32, gp.GP_BF16)


def norm(N, d, dtype=gp.GP_F32, **kw):
    return "gp_layer_norm", {**dict(x_ptr=P, ldx=d, dtype=dtype, N=N, d=d, weight_ptr=P, bias_ptr=P, weight_dtype=gp.GP_F32, eps=1e-5, y_ptr=2 * P, ldy=d, out_dtype=dtype,
                                    stats_ptr=P), **kw}


def norm_grad(N, d, dtype=gp.GP_F32, **kw):
    return "gp_layer_norm_grad", {**dict(grad_ptr=P, ldg=d, grad_dtype=dtype, x_ptr=2 * P, ldx=d, dtype=dtype, N=N, d=d, stats_ptr=P, weight_ptr=P, weight_dtype=gp.GP_F32,
                                         x_grad_ptr=3 * P, ldxg=d, weight_grad_ptr=P, bias_grad_ptr=P, accumulate=False, workspace_ptr=P, workspace_bytes=1 << 62), **kw}


def answer(N, C, k, dtype=gp.GP_F32, **kw):
    return "gp_log_probs", {**dict(logits_ptr=P, ld=C, dtype=dtype, N=N, C=C, tokens_ptr=P, index=gp.GP_I64, scale=1.0, logp_ptr=P, entropy_ptr=P, k=k, top_index_ptr=P,
                                   top_logp_ptr=P, stats_ptr=P, workspace_ptr=P, workspace_bytes=1 << 62), **kw}


def answer_grad(N, C, dtype=gp.GP_F32):
    return "gp_log_probs_grad", dict(logits_ptr=P, ld=C, dtype=dtype, N=N, C=C, tokens_ptr=P, index=gp.GP_I64, scale=1.0, stats_ptr=P, entropy_ptr=P, grad_logp_ptr=P,
                                     stride_logp=0, grad_entropy_ptr=P, stride_entropy=0, grad_ptr=P, ldg=C)


def distill(N, C, K, dtype=gp.GP_F32, **kw):
    return "gp_distill", {**dict(logits_ptr=P, ld=C, dtype=dtype, N=N, C=C, teacher_index_ptr=P, ldi=K, index=gp.GP_I64, teacher_logits_ptr=P, ldt=K, teacher_dtype=gp.GP_F32,
                                 K=K, temperature=1.0, loss_ptr=P, stats_ptr=P, grad_loss_ptr=P, stride_loss=0, grad_ptr=P, ldg=C, workspace_ptr=P,
                                 workspace_bytes=1 << 62), **kw}


ROWS = [1, 1000, 2 ** 22, 2 ** 36, 2 ** 40]


@pytest.mark.parametrize("dtype", TYPES)
def test_any_number_of_rows_can_be_launched(dtype):
    calls = [norm(N, d, dtype) for N in ROWS for d in (1, 100, 5000, 40_000)] + [norm_grad(N, d, dtype) for N in ROWS for d in (1, 100, 5000, 40_000, 2 ** 31 - 1)]
    calls += [answer(N, C, k, dtype) for N in ROWS for C in (1, 47, 3000, 100_000) for k in (0, 5, 64)] + [answer_grad(N, C, dtype) for N in ROWS for C in (1, 47, 100_000)]
    calls += [distill(N, C, K, dtype) for N in ROWS for C in (1, 47, 3000, 100_000) for K in (1, 8, 64)]
    for result in launches(calls):
        check_sizes(result)


@pytest.mark.parametrize("dtype", TYPES)
def test_every_width_and_number_of_places_has_a_kernel(dtype):
    widths = sorted({*range(1, 140), *(2 ** i + s for i in range(7, 17) for s in (-1, 0, 1)), 172, 300, 602, 30_000, 100_003, 2 ** 28})
    calls = [answer(N, C, k, dtype) for C in widths for k in (0, 1, 2, 3, 4, 5, 8, 9, 16, 17, 32, 33, 64) for N in (3, 10 ** 7)]
    calls += [distill(N, C, K, dtype) for C in widths for K in (1, 2, 3, 5, 8, 9, 16, 17, 32, 33, 64) for N in (3, 10 ** 7)]
    calls += [f(N, d, dtype) for d in widths for N in (3, 3000, 10 ** 7) for f in (norm, norm_grad)]
    for (name, kw), result in zip(calls, launches(calls)):
        assert result["status"] == gp.GP_OK and result["launches"], (name, kw)
        check_sizes(result)


def test_what_a_call_launches():
    names = {"short": ["gp_answer_short"], "rows": ["gp_answer_rows"], "parts": ["gp_answer_rows", "gp_answer_join"]}
    for call, want in ((answer(5000, 47, 5), "short"), (answer(5000, 512, 8), "short"), (answer(5000, 257, 20), "rows"), (answer(5000, 129, 33), "rows"), (answer(5000, 128, 64), "short"),
                       (answer(4096, 32_768, 8, gp.GP_BF16), "rows"), (answer(4096, 32_769, 8, gp.GP_BF16), "parts"), (answer(1, 391_000, 20), "parts"), (answer(3, 2000, 0), "rows")):
        seen = [l["kernel"] for l in launches([call])[0]["launches"]]
        assert len(seen) == len(names[want]) and all(n in s for n, s in zip(names[want], seen)), (call, seen)
    for call, want in ((distill(5000, 47, 8), ["gp_distill_short"]), (distill(5000, 600, 8), ["gp_distill_rows"]), (distill(4, 100_000, 8), ["gp_answer_rows", "gp_distill_join", "gp_distill_rows"]),
                       (distill(4, 100_000, 8, grad_ptr=0), ["gp_answer_rows", "gp_distill_join"]), (norm(100, 50_000), ["gp_norm_long"]), (norm_grad(1000, 100), ["gp_norm_grad_rows"]),
                       (norm_grad(1025, 100), ["gp_norm_grad_rows", "gp_norm_grad_join"]), (norm_grad(1025, 100, weight_grad_ptr=0, bias_grad_ptr=0), ["gp_norm_grad_rows"]),
                       # what the columns' workgroups read is written by the rows': one after the other
                       (norm_grad(1000, 100, x_grad_ptr=P), ["gp_norm_grad_rows"] * 2), (norm_grad(1000, 100, x_grad_ptr=2 * P), ["gp_norm_grad_rows"] * 2),
                       (norm_grad(10, 20_000), ["gp_norm_grad_means", "gp_norm_grad_columns", "gp_norm_grad_join"])):
        seen = [l["kernel"] for l in launches([call])[0]["launches"]]
        assert len(seen) == len(want) and all(n in s for n, s in zip(want, seen)), (call, seen)


def test_lds_beyond_64_kb_is_asked_for():
    for dtype in TYPES:
        for d in (100, 600, 1000, 2000, 4000):
            for l in launches([norm_grad(100_000, d, dtype)])[0]["launches"]:
                if "norm_grad_rows" in l["kernel"] and l["lds"] > 32 * 1024:
                    assert l["lds_asked"] >= l["lds"], l


def test_an_allocation_that_fails_is_an_error():
    for call in (norm(10, 100), norm_grad(10, 100), answer(10, 100, 5), answer(1, 100_000, 5), answer_grad(10, 100), distill(10, 100, 5), distill(1, 100_000, 5)):
        name, kw = call
        assert launches([(name, {**kw, "no_memory": True})])[0]["status"] == gp.GP_ERR_OOM_HOST
