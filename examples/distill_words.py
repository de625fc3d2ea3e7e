"""Trains a small node classifier from a larger one's best answers, over features that are learned.

The teacher is the classifier of train_words.py.  Once trained it answers for every node with its few best classes and their log
probabilities (gp_log_probs); that list is all the student sees of it.  The student has a table of its own and one layer over normalised features:

    Z = sum_k gamma_k S^k (s * table[word])      gp_embedding, gp_propagate_combine
    Y = layer_norm(Z) * w + b                    gp_layer_norm
    X = Y W                                      logits
    loss = mean over all nodes of the distillation loss + mean over labelled nodes of -log p[label]

with the loss's gradient from gp_distill and gp_log_probs_grad, the norm's from gp_layer_norm_grad, the filter's from itself, the table's from
gp_embedding_grad, and gp_muon_step for W.

    python examples/distill_words.py [--nodes 20000] [--steps 40]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path[:0] = [os.path.dirname(os.path.abspath(__file__)), os.path.dirname(os.path.dirname(os.path.abspath(__file__)))]
import paper_2207_12000_amd as gp  # noqa: E402
import train_words  # noqa: E402


class Student:
    """Table, norm and one layer, and what a step keeps."""

    def __init__(self, words: int, d: int, classes: int, temperature: float = 2.0, seed: int = 1):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.features = train_words.Model(words, d, 1, classes, seed=seed)  # (its table and its filter)
        self.w, self.b = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")
        self.W = torch.randn(d, classes, generator=gen, device="cuda") / d ** 0.5
        self.M = torch.zeros_like(self.W)
        self.temperature = temperature

    def logits(self, plan, word):
        Z = self.features.features(plan, word)
        stats = torch.empty(Z.shape[0], 2, device=Z.device)
        Y = gp.layer_norm_tensors(Z, self.w, self.b, stats=stats)
        return Z, stats, Y, Y @ self.W

    def gradients(self, plan, word, known, best, best_logp):
        """The loss, and its gradients: of the table, the norm's weight and bias, and W.  known: every node's label, -1 where there is none."""
        Z, stats, Y, X = self.logits(plan, word)
        N, labelled = X.shape[0], (known >= 0).sum().float()
        soft, dX = gp.distill_tensors(X, best, best_logp, self.temperature, grad_loss=torch.full((1,), 1 / N, device=X.device))
        kept = torch.empty(N, 2, device=X.device)
        hard = gp.log_probs_tensors(X, known, entropy=False, stats=kept).logp
        dX += gp.log_probs_grad_tensors(X, known, kept, grad_logp=(-1 / labelled).reshape(1))
        loss = soft.mean() - hard.sum() / labelled
        dZ, dw, db = gp.layer_norm_grad_tensors(dX @ self.W.t(), Z, stats, self.w)
        table_grad = gp.embedding_grad_tensors(word, self.features.filtered(plan, dZ), self.features.table.shape[0], scale=self.features.scale)
        return loss, table_grad, dw, db, Y.t() @ dX

    def step(self, plan, word, known, best, best_logp, lr: float):
        loss, table_grad, dw, db, dW = self.gradients(plan, word, known, best, best_logp)
        table = self.features.table
        table -= lr * table_grad / (table_grad.norm() + 1e-12) * table.norm()
        self.w -= lr * dw
        self.b -= lr * db
        gp.muon_step_tensors(self.W, self.M, dW, lr=lr, momentum=0.9, weight_decay=0.01)
        return loss


def train(nodes: int = 20_000, steps: int = 40, d: int = 32, classes: int = 16, entries: int = 4, seed: int = 0, report=None):
    """(losses, accuracy on nodes without a label, how many of the student's answers are the teacher's)."""
    rng = np.random.default_rng(seed)
    src, dst, label, word, words = train_words.graph_of(nodes, classes, rng)
    label, word = torch.from_numpy(label).cuda(), torch.from_numpy(word).cuda()
    order = torch.from_numpy(rng.permutation(nodes)).cuda()
    rows, held = order[:nodes // 2], order[nodes // 2:]
    known = torch.full_like(label, -1)
    known[rows] = label[rows]
    teacher, student = train_words.Model(words, 64, 128, classes, seed=seed), Student(words, d, classes, seed=seed + 1)
    losses = []
    with gp.gp_plan_blocks(src, dst, nodes, 1 << 20, gp.GP_SYMMETRISE | gp.GP_ADD_SELF_LOOPS) as plan:
        for i in range(steps):
            teacher.step(plan, word, label, rows, lr=0.1 * (1 - i / steps), table_lr=0.1 * (1 - i / steps))
        H = gp.lc_forward_tensors(teacher.features(plan, word)[None], None, [1.0], teacher.W)
        answers = gp.log_probs_tensors(H, top=entries, entropy=False)
        for i in range(steps):
            losses.append(float(student.step(plan, word, known, answers.top_index, answers.top_logp, lr=0.1 * (1 - i / steps))))
            if report:
                report(i, losses[-1])
        said = gp.log_probs_tensors(student.logits(plan, word)[3], top=1, entropy=False).top_index[:, 0]
    return losses, float((said == label)[held].float().mean()), float((said == answers.top_index[:, 0]).float().mean())


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--nodes", type=int, default=20_000)
    ap.add_argument("--steps", type=int, default=40)
    args = ap.parse_args()
    history, accuracy, agreement = train(args.nodes, args.steps, report=lambda i, loss: print(f"step {i:3d}  loss {loss:.4f}", flush=True))
    print(f"accuracy on nodes without a label {accuracy:.3f}, answers that are the teacher's {agreement:.3f}")
