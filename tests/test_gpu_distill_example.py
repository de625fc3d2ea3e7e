"""Layer norm, log probabilities and distillation together with the operators around them, as examples/distill_words.py uses them: its gradients
against automatic differentiation in fp64, the same model by the library's own differentiable calls, and a run."""
import importlib.util
import os
import sys

import numpy as np
import pytest

import paper_2207_12000_amd as gp

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example(gpu_or_skip):
    folder = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples")
    sys.path.insert(0, folder)
    try:
        spec = importlib.util.spec_from_file_location("distill_words", os.path.join(folder, "distill_words.py"))
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
    finally:
        sys.path.remove(folder)
    return module


def test_gradients_agree_with_automatic_differentiation(example):
    """fp32 sums of at most a few hundred terms, through seven hops, a norm, a layer and back: 2e-5 of a gradient's norm."""
    import torch
    nodes, classes = 300, 11
    rng = np.random.default_rng(0)
    src, dst, label, word, words = example.train_words.graph_of(nodes, classes, rng)
    student = example.Student(words, 20, classes)
    gen = torch.Generator(device="cuda").manual_seed(2)
    student.w += 0.2 * torch.randn(20, generator=gen, device="cuda")
    student.b += 0.2 * torch.randn(20, generator=gen, device="cuda")
    best = gp.log_probs_tensors(3 * torch.randn(nodes, classes, generator=gen, device="cuda"), top=4)
    known = torch.from_numpy(np.where(rng.random(nodes) < 0.3, label, -1)).cuda()
    word_d = torch.from_numpy(word).cuda()
    with gp.gp_plan_blocks(src, dst, nodes, 512, gp.GP_SYMMETRISE | gp.GP_ADD_SELF_LOOPS) as plan:
        got = student.gradients(plan, word_d, known, best.top_index, best.top_logp)
        S = np.zeros((nodes, nodes))
        S[np.repeat(np.arange(nodes), np.diff(plan.rowptr)), plan.col] = 1.0
        # the same loss by calls that automatic differentiation follows: the logits' gradient, through the norm
        Z, _, _, _ = student.logits(plan, word_d)
        Z, w, b = Z.requires_grad_(), student.w.clone().requires_grad_(), student.b.clone().requires_grad_()
        W = student.W.clone().requires_grad_()
        X = gp.layer_norm_tensors(Z, w, b) @ W
        soft, hard = gp.distill_tensors(X, best.top_index, best.top_logp, student.temperature), gp.log_probs_tensors(X, known).logp
        followed = soft.mean() - hard.sum() / (known >= 0).sum()
        followed.backward()
    assert abs(float(followed.detach()) - float(got[0])) < 1e-5
    for mine, theirs in zip(got[2:], (w.grad, b.grad, W.grad)):
        assert float((mine - theirs).norm()) <= 2e-5 * float(theirs.norm())
    deg = S.sum(1)
    S = torch.from_numpy(S / np.sqrt(deg[:, None] * deg[None, :]))
    table = student.features.table.double().cpu().requires_grad_()
    w, b, W = (t.double().cpu().requires_grad_() for t in (student.w, student.b, student.W))
    exists = torch.from_numpy(word >= 0)
    hop = torch.where(exists[:, None], student.features.scale * table[torch.from_numpy(word).long().clamp(min=0)], torch.zeros(1, dtype=torch.float64))
    Z = 0.0
    for c in student.features.coeff:
        Z, hop = Z + float(np.float32(c)) * hop, S @ hop
    X = torch.nn.functional.layer_norm(Z, (20,), w, b, 1e-5) @ W
    T = student.temperature
    q = torch.softmax(best.top_logp.double().cpu() / T, 1)
    logp = torch.log_softmax(X / T, 1).gather(1, best.top_index.long().cpu())
    rows = known.cpu() >= 0
    want = (T * T * (q * (q.log() - logp)).sum(1)).mean() + torch.nn.functional.cross_entropy(X[rows], known.cpu()[rows])
    want.backward()
    assert abs(float(got[0]) - float(want.detach())) < 1e-5
    for mine, ref in zip(got[1:], (table.grad, w.grad, b.grad, W.grad)):
        assert float((mine.double().cpu() - ref).norm()) <= 2e-5 * float(ref.norm())


def test_a_run(example):
    losses, accuracy, agreement = example.train(nodes=3000, steps=12, classes=8)
    assert len(losses) == 12 and np.isfinite(losses).all() and 0 <= accuracy <= 1 and 0 <= agreement <= 1
