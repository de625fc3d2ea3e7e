"""Host logic of layer norm, log probabilities and distillation: what is rejected before anything touches a GPU, workspace sizes, and the oracle's own
pins (hand cases and differences)."""
import numpy as np
import pytest

import paper_2207_12000_amd as gp
from oracle import answers

BAD, NO = gp.GP_ERR_INVALID_ARG, gp.GP_ERR_UNSUPPORTED
P = 4096  # stands for an address


def norm(**kw):
    a = dict(x_ptr=P, ldx=8, dtype=gp.GP_F32, N=4, d=8, weight_ptr=P, bias_ptr=P, weight_dtype=gp.GP_F32, eps=1e-5, y_ptr=P, ldy=8, out_dtype=gp.GP_F32)
    gp.gp_layer_norm(**{**a, **kw})


def norm_grad(**kw):
    a = dict(grad_ptr=P, ldg=8, grad_dtype=gp.GP_F32, x_ptr=P, ldx=8, dtype=gp.GP_F32, N=4, d=8, stats_ptr=P, weight_ptr=P, weight_dtype=gp.GP_F32,
             x_grad_ptr=P, ldxg=8, weight_grad_ptr=P, bias_grad_ptr=P, accumulate=False, workspace_ptr=P, workspace_bytes=1 << 40)
    gp.gp_layer_norm_grad(**{**a, **kw})


def answer(**kw):
    a = dict(logits_ptr=P, ld=8, dtype=gp.GP_F32, N=4, C=8, tokens_ptr=P, index=gp.GP_I32, scale=1.0, logp_ptr=P, entropy_ptr=P, k=2, top_index_ptr=P,
             top_logp_ptr=P, stats_ptr=P, workspace_ptr=P, workspace_bytes=1 << 40)
    gp.gp_log_probs(**{**a, **kw})


def answer_grad(**kw):
    a = dict(logits_ptr=P, ld=8, dtype=gp.GP_F32, N=4, C=8, tokens_ptr=P, index=gp.GP_I32, scale=1.0, stats_ptr=P, entropy_ptr=P, grad_logp_ptr=P,
             stride_logp=1, grad_entropy_ptr=P, stride_entropy=1, grad_ptr=P, ldg=8)
    gp.gp_log_probs_grad(**{**a, **kw})


TEACHER = dict(logits_ptr=P, ld=8, dtype=gp.GP_F32, N=4, C=8, teacher_index_ptr=P, ldi=3, index=gp.GP_I32, teacher_logits_ptr=P, ldt=3,
               teacher_dtype=gp.GP_F32, K=3, temperature=1.0, grad_loss_ptr=P, stride_loss=1, grad_ptr=P, ldg=8)


def distill(**kw):
    gp.gp_distill(**{**TEACHER, "loss_ptr": P, "stats_ptr": P, "workspace_ptr": P, "workspace_bytes": 1 << 40, **kw})


def distill_grad(**kw):
    gp.gp_distill_grad(**{**TEACHER, "stats_ptr": P, **kw})


NAN = float("nan")
LONG = dict(N=2, C=1 << 20, ld=1 << 20)
REFUSED = [
    (norm, dict(x_ptr=0), BAD), (norm, dict(y_ptr=0), BAD), (norm, dict(dtype=2), BAD), (norm, dict(out_dtype=-1), BAD), (norm, dict(weight_dtype=5), BAD),
    (norm, dict(N=-1), BAD), (norm, dict(d=0), BAD), (norm, dict(ldx=7), BAD), (norm, dict(ldy=7), BAD), (norm, dict(eps=0.0), BAD), (norm, dict(eps=-1.0), BAD),
    (norm, dict(eps=NAN), BAD), (norm, dict(eps=float("inf")), BAD),
    (norm_grad, dict(grad_ptr=0), BAD), (norm_grad, dict(x_ptr=0), BAD), (norm_grad, dict(stats_ptr=0), BAD), (norm_grad, dict(dtype=9), BAD),
    (norm_grad, dict(grad_dtype=2), BAD), (norm_grad, dict(weight_dtype=2), BAD), (norm_grad, dict(N=-1), BAD), (norm_grad, dict(d=0), BAD),
    (norm_grad, dict(ldg=7), BAD), (norm_grad, dict(ldx=7), BAD), (norm_grad, dict(ldxg=7), BAD), (norm_grad, dict(N=5000, workspace_ptr=0), BAD),
    (norm_grad, dict(N=5000, workspace_ptr=P + 16), BAD), (norm_grad, dict(N=5000, workspace_bytes=gp.gp_layer_norm_grad_workspace(5000, 8) - 1), BAD),
    (norm_grad, dict(N=(1 << 40) + 1), NO),
    (norm_grad, dict(d=16385, ldx=16385, ldg=16385, ldxg=16385, weight_grad_ptr=0, bias_grad_ptr=0, workspace_ptr=0), BAD),
    (answer, dict(logits_ptr=0), BAD), (answer, dict(tokens_ptr=0), BAD), (answer, dict(top_index_ptr=0), BAD), (answer, dict(top_logp_ptr=0), BAD),
    (answer, dict(dtype=2), BAD), (answer, dict(index=3), BAD), (answer, dict(N=-1), BAD), (answer, dict(C=0), BAD), (answer, dict(ld=7), BAD),
    (answer, dict(scale=0.0), BAD), (answer, dict(scale=-1.0), BAD), (answer, dict(scale=NAN), BAD), (answer, dict(scale=float("inf")), BAD),
    (answer, dict(k=-1), BAD), (answer, dict(k=65), NO), (answer, dict(N=(1 << 40) + 1), NO), (answer, dict(C=(1 << 28) + 1, ld=1 << 29), NO),
    (answer, dict(**LONG, workspace_ptr=0), BAD), (answer, dict(**LONG, workspace_ptr=P + 8), BAD),
    (answer, dict(**LONG, workspace_bytes=gp.gp_log_probs_workspace(2, 1 << 20, 2) - 1), BAD),
    (answer_grad, dict(logits_ptr=0), BAD), (answer_grad, dict(tokens_ptr=0), BAD), (answer_grad, dict(stats_ptr=0), BAD), (answer_grad, dict(entropy_ptr=0), BAD),
    (answer_grad, dict(grad_ptr=0), BAD), (answer_grad, dict(dtype=2), BAD), (answer_grad, dict(index=-1), BAD), (answer_grad, dict(N=-1), BAD),
    (answer_grad, dict(C=0), BAD), (answer_grad, dict(ld=7), BAD), (answer_grad, dict(ldg=7), BAD), (answer_grad, dict(stride_logp=2), BAD),
    (answer_grad, dict(stride_entropy=-1), BAD), (answer_grad, dict(scale=0.0), BAD), (answer_grad, dict(C=1 << 28, ld=1 << 28, ldg=1 << 28, N=1 << 40), gp.GP_ERR_OVERFLOW),
]
for call in (distill, distill_grad):
    REFUSED += [(call, dict(logits_ptr=0), BAD), (call, dict(teacher_index_ptr=0), BAD), (call, dict(teacher_logits_ptr=0), BAD), (call, dict(grad_loss_ptr=0), BAD),
                (call, dict(dtype=2), BAD), (call, dict(teacher_dtype=2), BAD), (call, dict(index=2), BAD), (call, dict(N=-1), BAD), (call, dict(C=0), BAD),
                (call, dict(ld=7), BAD), (call, dict(ldg=7), BAD), (call, dict(ldi=2), BAD), (call, dict(ldt=2), BAD), (call, dict(K=0), BAD),
                (call, dict(K=65, ldi=65, ldt=65), NO), (call, dict(temperature=0.0), BAD), (call, dict(temperature=NAN), BAD), (call, dict(temperature=1e16), BAD), (call, dict(stride_loss=2), BAD),
                (call, dict(N=(1 << 40) + 1), NO), (call, dict(C=(1 << 28) + 1, ld=1 << 29, ldg=1 << 29), NO)]
REFUSED += [(distill, dict(**LONG, ldg=1 << 20, workspace_ptr=0), BAD), (distill, dict(**LONG, ldg=1 << 20, workspace_bytes=gp.gp_distill_workspace(2, 1 << 20) - 1), BAD),
            (distill_grad, dict(stats_ptr=0), BAD), (distill_grad, dict(grad_ptr=0), BAD)]


@pytest.mark.parametrize("call,kw,status", REFUSED)
def test_rejected_arguments(call, kw, status):
    with pytest.raises(gp.GpError) as e:
        call(**kw)
    assert e.value.status == status
    assert gp.gp_last_error()


def test_empty_calls_touch_nothing():
    norm(N=0, x_ptr=0, y_ptr=0, weight_ptr=0, bias_ptr=0)
    norm_grad(N=0, grad_ptr=0, x_ptr=0, stats_ptr=0, x_grad_ptr=0, weight_grad_ptr=0, bias_grad_ptr=0, workspace_ptr=0, workspace_bytes=0)
    norm_grad(N=0, grad_ptr=0, x_ptr=0, stats_ptr=0, accumulate=True, workspace_ptr=0, workspace_bytes=0)
    norm_grad(x_grad_ptr=0, weight_grad_ptr=0, bias_grad_ptr=0)
    answer(N=0, logits_ptr=0, tokens_ptr=0, logp_ptr=0, workspace_ptr=0, workspace_bytes=0)
    answer(logp_ptr=0, entropy_ptr=0, k=0, stats_ptr=0)
    answer_grad(N=0, logits_ptr=0, stats_ptr=0, grad_ptr=0)
    distill(N=0, logits_ptr=0, teacher_index_ptr=0, teacher_logits_ptr=0, workspace_ptr=0, workspace_bytes=0)
    distill(loss_ptr=0, stats_ptr=0, grad_ptr=0)
    distill_grad(N=0, logits_ptr=0, stats_ptr=0, grad_ptr=0)


def test_workspace_sizes():
    assert gp.gp_layer_norm_grad_workspace(0, 8) == gp.gp_log_probs_workspace(0, 1 << 20, 5) == gp.gp_distill_workspace(0, 1 << 20) == 0
    assert gp.gp_log_probs_workspace(4096, 32768, 64) == gp.gp_distill_workspace(1, 1000) == 0
    for bad in ((-1, 8), ((1 << 40) + 1, 8), (4, 0)):
        assert gp.gp_layer_norm_grad_workspace(*bad) == -1
    for bad in ((-1, 8, 1), ((1 << 40) + 1, 8, 1), (4, 0, 1), (4, (1 << 28) + 1, 1), (4, 8, -1), (4, 8, 65)):
        assert gp.gp_log_probs_workspace(*bad) == -1
    for bad in ((-1, 8), ((1 << 40) + 1, 8), (4, 0), (4, (1 << 28) + 1)):
        assert gp.gp_distill_workspace(*bad) == -1
    assert gp.gp_layer_norm_grad_workspace(4, 8) == 0 < gp.gp_layer_norm_grad_workspace(5000, 8) and gp.gp_layer_norm_grad_workspace(4, 17_000) > 0
    assert 0 < gp.gp_log_probs_workspace(1 << 40, 1 << 28, 64) < 1 << 63
    assert gp.gp_log_probs_workspace(1, 1 << 20, 0) < gp.gp_log_probs_workspace(1, 1 << 20, 1)


def test_tensors_must_be_on_the_gpu_and_of_matching_shapes():
    import torch
    f, v, s, t = torch.zeros(4, 8), torch.zeros(8), torch.zeros(4, 2), torch.zeros(4, dtype=torch.int32)
    at, g = torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4)
    of = torch.zeros(4, 3)
    for bad in (lambda: gp.layer_norm_tensors(f), lambda: gp.layer_norm_tensors(f.double()), lambda: gp.layer_norm_tensors(f.t()), lambda: gp.layer_norm_tensors(f, v[:7]),
                lambda: gp.layer_norm_tensors(f, v, v.bfloat16()), lambda: gp.layer_norm_tensors(f, v.double()), lambda: gp.layer_norm_tensors(f, f),
                lambda: gp.layer_norm_tensors(f, out=torch.zeros(3, 8)), lambda: gp.layer_norm_tensors(f, stats=s[:3]), lambda: gp.layer_norm_tensors(f, stats=s.double()),
                lambda: gp.layer_norm_tensors(torch.zeros(2, 8, 4).transpose(1, 2)), lambda: gp.layer_norm_tensors(torch.zeros(())),
                lambda: gp.layer_norm_grad_tensors(f, f, s), lambda: gp.layer_norm_grad_tensors(f, f[:3], s[:3]), lambda: gp.layer_norm_grad_tensors(f, f, None),
                lambda: gp.layer_norm_grad_tensors(f, f, s[:3]), lambda: gp.layer_norm_grad_tensors(f, f, s, accumulate=True),
                lambda: gp.layer_norm_grad_tensors(f, f, s, v, weight_grad=v.bfloat16()), lambda: gp.layer_norm_grad_tensors(f, f, s, x_grad=f[:3]),
                lambda: gp.layer_norm_grad_tensors(f, f, s, x_grad=f.bfloat16()), lambda: gp.layer_norm_grad_tensors(f, f, s, bias_grad=v[:7]),
                lambda: gp.log_probs_tensors(f), lambda: gp.log_probs_tensors(f, t[:3]), lambda: gp.log_probs_tensors(f, t.float()), lambda: gp.log_probs_tensors(f, top=-1),
                lambda: gp.log_probs_tensors(f.half()), lambda: gp.log_probs_tensors(f, stats=s[:3]), lambda: gp.log_probs_tensors(f.t()),
                lambda: gp.log_probs_grad_tensors(f, t, s, grad_logp=g), lambda: gp.log_probs_grad_tensors(f, t, None, grad_logp=g),
                lambda: gp.log_probs_grad_tensors(f, None, s, grad_logp=g), lambda: gp.log_probs_grad_tensors(f, t, s, grad_entropy=g),
                lambda: gp.log_probs_grad_tensors(f, t, s, entropy=g[:3], grad_entropy=g), lambda: gp.log_probs_grad_tensors(f, t, s, entropy=g[:1], grad_entropy=g),
                lambda: gp.log_probs_grad_tensors(f, t, s, grad_logp=g.double()), lambda: gp.log_probs_grad_tensors(f, t, s, grad_logp=torch.zeros(8)[::2]),
                lambda: gp.log_probs_grad_tensors(f, t, s, grad_logp=g[:3]), lambda: gp.log_probs_grad_tensors(f, t, s, grad_logp=g, out=f[:3]),
                lambda: gp.distill_tensors(f, at, of), lambda: gp.distill_tensors(f, at, of[:, :2]), lambda: gp.distill_tensors(f, at[:3], of[:3]),
                lambda: gp.distill_tensors(f, at.float(), of), lambda: gp.distill_tensors(f, at, of.double()), lambda: gp.distill_tensors(f, at, of, out=f.clone()),
                lambda: gp.distill_tensors(f, at, of, grad_loss=g[:3]), lambda: gp.distill_tensors(f, at, of, grad_loss=g, out=f.bfloat16()),
                lambda: gp.distill_grad_tensors(f, at, of, s, g), lambda: gp.distill_grad_tensors(f, at, of, None, g), lambda: gp.distill_grad_tensors(f, at, of, s, None),
                lambda: gp.log_probs_tensors(f.clone().requires_grad_(), t), lambda: gp.distill_tensors(f.clone().requires_grad_(), at, of),
                lambda: gp.layer_norm_tensors(f, v.clone().requires_grad_()), lambda: gp.log_probs_tensors(f.clone().requires_grad_(), t, stream=1), lambda: gp.distill_tensors(f.clone().requires_grad_(), at, of, stream=1),
                lambda: gp.layer_norm_tensors(f.clone().requires_grad_(), stream=1)):
        with pytest.raises(ValueError):
            bad()


# ---- the oracle's pins -----------------------------------------------------------------------------------

def differences(f, x, up, step=1e-5):
    grad = np.zeros_like(x)
    for at in np.ndindex(*x.shape):
        h = np.zeros_like(x)
        h[at] = step
        grad[at] = ((f(x + h) - f(x - h)) * up).sum() / (2 * step)
    return grad


def test_oracle_layer_norm_by_hand():
    y, stats = answers.layer_norm([[1.0, 3.0], [5.0, 5.0]], np.array([2.0, 1.0]), np.array([0.5, 0.0]), eps=3.0)
    assert np.allclose(stats, [[2, 0.5], [5, 3 ** -0.5]]) and np.allclose(y, [[-0.5, 0.5], [0.5, 0.0]])


def test_oracle_layer_norm_gradients_agree_with_differences():
    rng = np.random.default_rng(0)
    x, w, b, up = rng.normal(size=(4, 5)), rng.normal(size=5), rng.normal(size=5), rng.normal(size=(4, 5))
    stats = answers.layer_norm(x, w, b)[1]
    dx, dw, db = answers.layer_norm_grad(up, x, stats, w)
    assert np.allclose(dx, differences(lambda v: answers.layer_norm(v, w, b)[0], x, up), atol=1e-7)
    assert np.allclose(dw, differences(lambda v: answers.layer_norm(x, v, b)[0], w, up), atol=1e-7)
    assert np.allclose(db, differences(lambda v: answers.layer_norm(x, w, v)[0], b, up), atol=1e-7)


def test_oracle_log_probs_by_hand():
    x = np.array([[0.0, np.log(3.0)], [-np.inf, 2.0], [-np.inf, -np.inf], [1.0, 1.0]])
    logp, entropy, index, top = answers.log_probs(x, [0, 0, 1, 5], k=3)
    assert np.allclose(logp[:1], np.log(0.25)) and np.isneginf(logp[1:3]).all() and logp[3] == 0
    assert np.allclose(entropy, [np.log(4) - 0.75 * np.log(3), 0, 0, np.log(2)])
    assert np.array_equal(index, [[1, 0, -1], [1, -1, -1], [-1, -1, -1], [0, 1, -1]])
    assert np.allclose(top[0, :2], np.log([0.75, 0.25])) and top[1, 0] == 0 and np.isneginf(top[2]).all()


def test_oracle_log_probs_gradient_agrees_with_differences():
    rng = np.random.default_rng(1)
    x, tokens = rng.normal(size=(5, 6)), np.array([0, 5, -1, 2, 6])
    g1, g2 = rng.normal(size=5), rng.normal(size=5)
    got = answers.log_probs_grad(x, tokens, 0.5, g1, g2)

    def both(v):
        logp, entropy, _, _ = answers.log_probs(v, tokens, 0.5)
        return logp * g1 + entropy * g2

    want = differences(both, x, 1.0)
    assert np.allclose(got, want, atol=1e-7)


def test_oracle_distill_by_hand_and_by_differences():
    # two entries of equal logits: q = 1/2 each, over a uniform student of four classes: log(1/2) - log(1/4)
    loss, _ = answers.distill(np.zeros((2, 4)), np.array([[1, 3, -1], [-1, 9, -1]]), np.zeros((2, 3)), 2.0)
    assert np.allclose(loss, [4 * np.log(2.0), 0])
    rng = np.random.default_rng(2)
    x, index, v, g = rng.normal(size=(4, 6)), np.array([[0, 1, 2], [3, 3, -1], [5, 0, 5], [-1, -1, -1]]), rng.normal(size=(4, 3)), rng.normal(size=4)
    got = answers.distill(x, index, v, 1.5, g)[1]
    assert np.allclose(got, differences(lambda z: answers.distill(z, index, v, 1.5)[0], x, g), atol=1e-7)
    assert np.array_equal(got[3], np.zeros(6))
