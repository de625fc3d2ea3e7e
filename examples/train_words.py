"""Trains a node classifier whose features are learned: every node of a graph stands for a word, a table holds one row per word.

    X = s * table[word]                 gp_embedding
    Z = sum_k gamma_k S^k X             gp_propagate_combine (Personalized PageRank over the symmetric operator S)
    H = relu(Z W1) W2,  Y = softmax(H)

and backwards: dZ from the two layers, dX = the same filter of dZ (S is symmetric, so the filter is its own transpose), the table's
gradient from the sorted words (gp_embedding_grad), a step along it for the table and an orthogonalised one for each weight matrix
(gp_muon_step).  The accuracy is that of the library's own forward pass (gp_lc_forward).  The graph is synthetic: communities are the
classes, and a node's word says little about its class on its own.

    python examples/train_words.py [--nodes 20000] [--steps 40]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2207_12000_amd as gp  # noqa: E402


def graph_of(nodes: int, classes: int, rng):
    """Edges mostly inside communities; labels; words that name the class in two of five draws, else none in particular."""
    label = rng.integers(0, classes, nodes)
    order = np.argsort(label, kind="stable")
    first = np.searchsorted(label[order], np.arange(classes + 1))
    m = 8 * nodes
    src = rng.integers(0, nodes, m)
    size = np.maximum(first[label[src] + 1] - first[label[src]], 1)
    dst = np.where(rng.random(m) < 0.7, order[first[label[src]] + (rng.random(m) * size).astype(np.int64)], rng.integers(0, nodes, m))
    words = 50 * classes
    word = np.where(rng.random(nodes) < 0.4, label * 50 + rng.integers(0, 50, nodes), rng.integers(0, words, nodes))
    word[rng.random(nodes) < 0.05] = -1  # some nodes have none
    return src.astype(np.int32), dst.astype(np.int32), label, word.astype(np.int32), words


class Model:
    """Table, weights, and what a step keeps: momenta, and the scratch of the calls."""

    def __init__(self, words: int, d: int, hidden: int, classes: int, hops: int = 6, alpha: float = 0.15, seed: int = 0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.scale = d ** 0.5
        self.coeff = [alpha * (1 - alpha) ** k for k in range(hops)] + [(1 - alpha) ** hops]
        self.table = torch.randn(words, d, generator=gen, device="cuda") / d
        self.W = [torch.randn(d, hidden, generator=gen, device="cuda") / d ** 0.5, torch.randn(hidden, classes, generator=gen, device="cuda") / hidden ** 0.5]
        self.M = [torch.zeros_like(w) for w in self.W]
        self.scratch = [torch.empty(max(gp.gp_orthogonalize_workspace(*w.shape), 1), dtype=torch.uint8, device="cuda") for w in self.W]

    def filtered(self, plan, X):
        out = torch.empty_like(X)
        gp.gp_propagate_combine(plan, X.data_ptr(), X.stride(0), X.shape[1], gp.GP_F32, gp.GP_AGG_SYM, len(self.coeff) - 1, self.coeff,
                                out.data_ptr(), out.stride(0), torch.cuda.current_stream().cuda_stream)
        return out

    def features(self, plan, word):
        return self.filtered(plan, gp.embedding_tensors(self.table, word, scale=self.scale))

    def gradients(self, plan, word, label, rows):
        """Mean cross entropy over `rows`, and its gradients: of the table and of every weight matrix."""
        Z = self.features(plan, word)
        A = torch.relu(Z @ self.W[0])
        logits = (A @ self.W[1])[rows]
        logp = logits - torch.logsumexp(logits, 1, keepdim=True)
        loss = -logp.gather(1, label[rows, None]).mean()
        dH = torch.zeros(Z.shape[0], logits.shape[1], device="cuda")
        dH[rows] = (logp.exp() - torch.nn.functional.one_hot(label[rows], logits.shape[1])) / rows.numel()
        dA = (dH @ self.W[1].t()) * (A > 0)
        dX = self.filtered(plan, dA @ self.W[0].t())
        table_grad = gp.embedding_grad_tensors(word, dX, self.table.shape[0], scale=self.scale)
        return loss, table_grad, [Z.t() @ dA, A.t() @ dH]

    def step(self, plan, word, label, rows, lr: float, table_lr: float):
        loss, table_grad, grads = self.gradients(plan, word, label, rows)
        self.table -= table_lr * table_grad / (table_grad.norm() + 1e-12) * self.table.norm()
        for w, m, g, ws in zip(self.W, self.M, grads, self.scratch):
            gp.muon_step_tensors(w, m, g, lr=lr, momentum=0.9, weight_decay=0.01, workspace=ws)
        return loss

    def answers(self, plan, word):
        """The predicted label matrix of all nodes, by the library's forward pass."""
        H = gp.lc_forward_tensors(self.features(plan, word)[None], None, [1.0], self.W)
        gp.gp_lc_softmax(H.data_ptr(), H.shape[0], H.shape[1], H.stride(0), torch.cuda.current_stream().cuda_stream)
        return H


def train(nodes: int = 20_000, steps: int = 40, d: int = 64, hidden: int = 128, classes: int = 16, seed: int = 0, report=None):
    """(losses, accuracy on the nodes that were not trained on)."""
    rng = np.random.default_rng(seed)
    src, dst, label, word, words = graph_of(nodes, classes, rng)
    model = Model(words, d, hidden, classes, seed=seed)
    label, word = torch.from_numpy(label).cuda(), torch.from_numpy(word).cuda()
    known = torch.from_numpy(rng.permutation(nodes)).cuda()
    rows, held = known[:nodes // 2], known[nodes // 2:]
    losses = []
    with gp.gp_plan_blocks(src, dst, nodes, 1 << 20, gp.GP_SYMMETRISE | gp.GP_ADD_SELF_LOOPS) as plan:
        for i in range(steps):
            losses.append(float(model.step(plan, word, label, rows, lr=0.1 * (1 - i / steps), table_lr=0.1 * (1 - i / steps))))
            if report:
                report(i, losses[-1])
        accuracy = float((model.answers(plan, word).argmax(1) == label)[held].float().mean())
    return losses, accuracy


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--nodes", type=int, default=20_000)
    ap.add_argument("--steps", type=int, default=40)
    args = ap.parse_args()
    history, accuracy = train(args.nodes, args.steps, report=lambda i, loss: print(f"step {i:3d}  loss {loss:.4f}", flush=True))
    print(f"accuracy on held-out nodes {accuracy:.3f}")
