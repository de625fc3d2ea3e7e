"""Host logic of the training operators: what is rejected before anything touches a GPU, workspace sizes, and the oracle's own pins."""
import numpy as np
import pytest

import paper_2207_12000_amd as gp
from oracle import training

BAD, NO = gp.GP_ERR_INVALID_ARG, gp.GP_ERR_UNSUPPORTED
P = 4096  # stands for an address


def lookup(**kw):
    a = dict(table_ptr=P, ldt=8, dtype=gp.GP_F32, V=10, d=8, tokens_ptr=P, index=gp.GP_I32, N=4, scale=1.0, out_ptr=P, ldo=8,
             out_dtype=gp.GP_F32)
    a.update(kw)
    gp.gp_embedding(**a)


def grad(**kw):
    a = dict(tokens_ptr=P, index=gp.GP_I32, N=4, grad_ptr=P, ldg=8, dtype=gp.GP_F32, d=8, scale=1.0, V=10, table_grad_ptr=P, ldt=8,
             out_dtype=gp.GP_F32, accumulate=False, workspace_ptr=P, workspace_bytes=1 << 30)
    a.update(kw)
    gp.gp_embedding_grad(**a)


def orth(**kw):
    a = dict(G_ptr=P, ldg=8, stride_g=80, dtype=gp.GP_F32, rows=10, cols=8, count=2, steps=5, coeff=None, eps=1e-7, out_ptr=P, ldo=8,
             stride_o=80, workspace_ptr=P, workspace_bytes=1 << 30)
    a.update(kw)
    gp.gp_orthogonalize(**a)


def muon(**kw):
    a = dict(W_ptr=P, W_out_ptr=P, ldw=8, stride_w=80, M_ptr=P, M_out_ptr=P, ldm=8, stride_m=80, G_ptr=P, ldg=8, stride_g=80,
             dtype=gp.GP_F32, rows=10, cols=8, count=2, lr=0.1, momentum=0.9, weight_decay=0.0, nesterov=True, steps=5, coeff=None,
             eps=1e-7, workspace_ptr=P, workspace_bytes=1 << 30)
    a.update(kw)
    gp.gp_muon_step(**a)


@pytest.mark.parametrize("call,kw,status", [
    (lookup, dict(table_ptr=0), BAD), (lookup, dict(tokens_ptr=0), BAD), (lookup, dict(out_ptr=0), BAD), (lookup, dict(dtype=2), BAD),
    (lookup, dict(out_dtype=-1), BAD), (lookup, dict(index=2), BAD), (lookup, dict(V=0), BAD), (lookup, dict(d=0), BAD),
    (lookup, dict(N=-1), BAD), (lookup, dict(ldt=7), BAD), (lookup, dict(ldo=7), BAD),
    (lookup, dict(N=1 << 61), gp.GP_ERR_OVERFLOW),
    (grad, dict(tokens_ptr=0), BAD), (grad, dict(grad_ptr=0), BAD), (grad, dict(table_grad_ptr=0), BAD), (grad, dict(dtype=2), BAD),
    (grad, dict(out_dtype=7), BAD), (grad, dict(index=-1), BAD), (grad, dict(V=0), BAD), (grad, dict(d=0), BAD), (grad, dict(N=-1), BAD),
    (grad, dict(ldg=7), BAD), (grad, dict(ldt=7), BAD), (grad, dict(workspace_ptr=0), BAD), (grad, dict(workspace_ptr=P + 16), BAD),
    (grad, dict(workspace_bytes=gp.gp_embedding_grad_workspace(4, 10, 8) - 1), BAD), (grad, dict(N=1 << 31), NO), (grad, dict(V=1 << 31), NO),
    (orth, dict(G_ptr=0), BAD), (orth, dict(out_ptr=0), BAD), (orth, dict(dtype=2), BAD), (orth, dict(rows=-1), BAD), (orth, dict(cols=-1), BAD),
    (orth, dict(count=-1), BAD), (orth, dict(ldg=7), BAD), (orth, dict(ldo=7), BAD), (orth, dict(stride_o=79), BAD), (orth, dict(stride_o=0), BAD),
    (orth, dict(steps=0), BAD), (orth, dict(steps=33), BAD), (orth, dict(eps=-1.0), BAD), (orth, dict(eps=float("nan")), BAD),
    (orth, dict(coeff=[100.0, 0.0, 0.0]), BAD), (orth, dict(coeff=[float("nan"), 0.0, 0.0]), BAD), (orth, dict(workspace_ptr=0), BAD),
    (orth, dict(workspace_ptr=P + 128), BAD), (orth, dict(workspace_bytes=gp.gp_orthogonalize_workspace(10, 8, 2) - 1), BAD),
    (orth, dict(rows=(1 << 20) + 1), NO), (orth, dict(cols=(1 << 20) + 1, ldg=1 << 21, ldo=1 << 21), NO), (orth, dict(count=65536), NO),
    (muon, dict(W_ptr=0), BAD), (muon, dict(W_out_ptr=0), BAD), (muon, dict(M_ptr=0), BAD), (muon, dict(M_out_ptr=0), BAD),
    (muon, dict(G_ptr=0), BAD), (muon, dict(dtype=2), BAD), (muon, dict(ldw=7), BAD), (muon, dict(ldm=7), BAD), (muon, dict(ldg=7), BAD),
    (muon, dict(stride_w=79), BAD), (muon, dict(stride_m=10), BAD), (muon, dict(steps=0), BAD), (muon, dict(workspace_bytes=100), BAD),
    (muon, dict(count=65536), NO),
])
def test_rejected_arguments(call, kw, status):
    with pytest.raises(gp.GpError) as e:
        call(**kw)
    assert e.value.status == status
    assert gp.gp_last_error()


def test_empty_calls_touch_nothing():
    lookup(N=0, table_ptr=0, tokens_ptr=0, out_ptr=0)
    for empty in (dict(rows=0), dict(cols=0), dict(count=0)):
        orth(**empty, G_ptr=0, out_ptr=0, workspace_ptr=0, workspace_bytes=0)
        muon(**empty, W_ptr=0, W_out_ptr=0, M_ptr=0, M_out_ptr=0, G_ptr=0, workspace_ptr=0, workspace_bytes=0)


def test_workspace_sizes():
    assert gp.gp_embedding_grad_workspace(0, 10, 8) == 0
    assert gp.gp_orthogonalize_workspace(0, 10, 1) == gp.gp_orthogonalize_workspace(10, 10, 0) == 0
    for bad in ((-1, 10, 8), (1 << 31, 10, 8), (4, 0, 8), (4, 1 << 31, 8), (4, 10, 0)):
        assert gp.gp_embedding_grad_workspace(*bad) == -1
    for bad in ((-1, 1, 1), (1, -1, 1), (1, 1, -1), ((1 << 20) + 1, 1, 1), (1, (1 << 20) + 1, 1), (1, 1, 65536)):
        assert gp.gp_orthogonalize_workspace(*bad) == -1
    assert gp.gp_orthogonalize_workspace(300, 70, 1) == gp.gp_orthogonalize_workspace(70, 300, 1)
    assert gp.gp_orthogonalize_workspace(1 << 20, 1 << 20, 65535) > 0


def test_coefficients_come_as_three_or_three_per_step():
    for coeff in ([1.0, 2.0], [[1.0, 0.0, 0.0]] * 4, [[1.0, 0.0]] * 5):
        with pytest.raises(ValueError):
            orth(coeff=coeff)


def test_tensors_must_be_on_the_gpu_and_of_matching_shapes():
    import torch
    f = torch.zeros(4, 8)
    t = torch.zeros(4, dtype=torch.int32)
    for bad in (lambda: gp.embedding_tensors(f, t), lambda: gp.embedding_tensors(f.double(), t), lambda: gp.embedding_tensors(f, t.float()),
                lambda: gp.embedding_tensors(f.t(), t), lambda: gp.embedding_tensors(f, t[::2]), lambda: gp.embedding_tensors(f[0], t),
                lambda: gp.embedding_tensors(f, t, out=torch.zeros(3, 8)), lambda: gp.embedding_grad_tensors(t, f, 10),
                lambda: gp.embedding_grad_tensors(t, f[:3], 10), lambda: gp.embedding_grad_tensors(t, f, 10, accumulate=True),
                lambda: gp.embedding_grad_tensors(t, f, 10, out=torch.zeros(9, 8)), lambda: gp.orthogonalize_tensors(f),
                lambda: gp.orthogonalize_tensors(f[0]), lambda: gp.orthogonalize_tensors(f, out=torch.zeros(8, 4)),
                lambda: gp.muon_step_tensors(f, f, torch.zeros(8, 4), 0.1), lambda: gp.muon_step_tensors(f.bfloat16(), f, f, 0.1),
                lambda: gp.muon_step_tensors(f, f, f, 0.1)):
        with pytest.raises(ValueError):
            bad()


# ---- the oracle's pins -----------------------------------------------------------------------------------

def test_oracle_embedding_by_hand():
    table = np.array([[1.0, 2.0], [3.0, 4.0]])
    tokens = np.array([1, -1, 0, 1, 2])
    assert np.array_equal(training.embedding(table, tokens, 2.0), [[6, 8], [0, 0], [2, 4], [6, 8], [0, 0]])
    up = np.array([[1.0, 10.0], [2.0, 20.0], [3.0, 30.0], [4.0, 40.0], [5.0, 50.0]])
    g, size, terms = training.embedding_grad(tokens, -up, 2, 2.0)
    assert np.array_equal(g, [[-6, -60], [-10, -100]]) and np.array_equal(size, -g) and np.array_equal(terms, [1, 2])


def test_oracle_gradient_agrees_with_differences():
    rng = np.random.default_rng(1)
    table, tokens, up = rng.normal(size=(5, 3)), rng.integers(-1, 6, 20), rng.normal(size=(20, 3))
    g = training.embedding_grad(tokens, up, 5, 0.7)[0]
    for v, c in np.ndindex(5, 3):
        h = np.zeros_like(table)
        h[v, c] = 1e-6
        diff = ((training.embedding(table + h, tokens, 0.7) - training.embedding(table - h, tokens, 0.7)) * up).sum() / 2e-6
        assert abs(diff - g[v, c]) < 1e-7


@pytest.mark.parametrize("shape", [(3, 5), (5, 3), (4, 4), (1, 6)])
def test_oracle_steps_act_on_singular_values_alone(shape):
    G = np.random.default_rng(2).normal(size=shape)
    U, s, Vt = np.linalg.svd(G, full_matrices=False)
    s = s / (np.sqrt((s * s).sum()) + 1e-7)
    for a, b, c in [training.COEFF] * 3:
        s = a * s + b * s ** 3 + c * s ** 5
    assert np.allclose(training.newton_schulz(G, 3)[-1], (U * s) @ Vt, atol=1e-12)


def test_oracle_muon_step_by_hand():
    # one element: U = 2 + 0.5 * 2.5 = 3.25, its direction after one step of (1, 0, 0) is 3.25 / (3.25 + 0.75)
    W, M = training.muon_step([[10.0]], [[1.0]], [[2.0]], 0.1, momentum=0.5, weight_decay=0.2, steps=1, coeff=(1, 0, 0), eps=0.75)
    assert np.allclose(M, 2.5) and np.allclose(W, 0.98 * 10 - 0.1 * 3.25 / 4)
    W, _ = training.muon_step([[10.0]], [[1.0]], [[2.0]], 0.1, momentum=0.5, nesterov=False, steps=1, coeff=(1, 0, 0), eps=0.0)
    assert np.allclose(W, 9.9)
