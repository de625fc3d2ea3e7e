"""The training operators together, as examples/train_words.py uses them: its gradients against automatic differentiation in fp64, and
a short run that learns."""
import importlib.util
import os

import numpy as np
import pytest

import paper_2207_12000_amd as gp

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example(gpu_or_skip):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_words.py")
    spec = importlib.util.spec_from_file_location("train_words", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_gradients_agree_with_automatic_differentiation(example):
    """fp32 sums of at most a few hundred terms, through seven hops, two layers and back: 1e-5 of a gradient's norm."""
    import torch
    nodes, classes = 300, 5
    rng = np.random.default_rng(0)
    src, dst, label, word, words = example.graph_of(nodes, classes, rng)
    model = example.Model(words, 20, 24, classes)
    rows = torch.arange(0, nodes, 2, device="cuda")
    with gp.gp_plan_blocks(src, dst, nodes, 512, gp.GP_SYMMETRISE | gp.GP_ADD_SELF_LOOPS) as plan:
        loss, table_grad, grads = model.gradients(plan, torch.from_numpy(word).cuda(), torch.from_numpy(label).cuda(), rows)
        S = np.zeros((nodes, nodes))
        S[np.repeat(np.arange(nodes), np.diff(plan.rowptr)), plan.col] = 1.0
        deg = S.sum(1)
    S = torch.from_numpy(S / np.sqrt(deg[:, None] * deg[None, :]))
    table = model.table.double().cpu().requires_grad_()
    W = [w.double().cpu().requires_grad_() for w in model.W]
    known = torch.from_numpy(word >= 0)
    X = torch.where(known[:, None], model.scale * table[torch.from_numpy(word).long().clamp(min=0)], torch.zeros(1, dtype=torch.float64))
    Z, hop = 0.0, X
    for c in model.coeff:
        Z, hop = Z + float(np.float32(c)) * hop, S @ hop
    logits = (torch.relu(Z @ W[0]) @ W[1])[rows.cpu()]
    want = torch.nn.functional.cross_entropy(logits, torch.from_numpy(label)[rows.cpu()])
    want.backward()
    assert abs(float(loss) - float(want.detach())) < 1e-5
    for got, ref in zip([table_grad] + grads, [table.grad] + [w.grad for w in W]):
        assert float((got.double().cpu() - ref).norm()) <= 1e-5 * float(ref.norm())


def test_a_short_run_learns(example):
    losses, accuracy = example.train(nodes=4000, steps=25, classes=8)
    assert losses[-1] < 0.5 * losses[0] and accuracy > 0.6     # (guessing: an eighth)
