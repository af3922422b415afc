"""A student of propagated labels: texts as vertices, a kNN-like graph, labels propagated from a few of them, and a classifier that learns
them and labels texts the graph has never held.

    python examples/student.py [--items 20000] [--steps 300] [--bits 8]

Synthetic texts: every class has its own frequent words.  The graph joins texts of the same class more often than others
(``workloads.sbm``).  One process, one GPU.  ``DynLP.get_labels`` returns the soft rows that ``head_loss`` takes: here as numpy arrays, as the graph is one of these (a
context made with ``device_ptrs=True`` takes and returns tensors on the GPU).
"""
import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

import paper_2604_06596_amd as P
import workloads as W


def make_texts(true_class, classes, words, mean_len, seed):
    """ids, offsets, weights (as of TF-IDF: rare words weigh more, every text has length one)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = len(true_class)
    length = 1 + (2 * mean_len * torch.rand(n, generator=g, device="cuda")).long()
    offsets = torch.zeros(n + 1, dtype=torch.int64, device="cuda")
    torch.cumsum(length, 0, out=offsets[1:])
    item = torch.repeat_interleave(torch.arange(n, device="cuda"), length)
    count = len(item)
    common = torch.floor(10 * torch.exp(torch.rand(count, generator=g, device="cuda") * math.log(words / 10 + 1)) - 10).long().clamp(0, words - 1)
    own = words // 2 + true_class[item] + classes * (torch.rand(count, generator=g, device="cuda") ** 2 * (words // 2 // classes - 1)).long()
    ids = torch.where(torch.rand(count, generator=g, device="cuda") < 0.25, own, common)
    weights = torch.log1p(ids.float() / 10.0) + 0.1
    norm = torch.zeros(n, device="cuda").index_add_(0, item, weights * weights).sqrt()
    return ids.to(torch.int32), offsets, weights / norm[item]


class Student:
    """A table of token rows and a head of one row per class, in bfloat16 with float32 parameters behind them."""

    def __init__(self, words, dim, classes, bits, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.params = [0.05 * torch.randn(words, dim, generator=g, device="cuda"),
                       torch.zeros(classes, dim, device="cuda"), torch.zeros(classes, device="cuda")]
        self.table, self.weight = (p.to(torch.bfloat16) for p in self.params[:2])
        self.bias = self.params[2].clone()
        self.states = [P.adamw_state(p, bits) for p in self.params]
        self.steps = 0

    def labels(self, ids, offsets, weights):
        return P.head_labels(P.embed(self.table, ids, offsets, weights), self.weight, self.bias)

    def learn(self, ids, offsets, weights, soft, row_weight, lr):
        """One step; returns the rows' losses."""
        h = P.embed(self.table, ids, offsets, weights)
        loss, dh, dweight, dbias = P.head_loss(h, self.weight, self.bias, soft, row_weight=row_weight, grad_scale=1.0 / len(h))
        dtable = P.embed_grad(dh, ids, len(self.table), offsets, weights)
        self.steps += 1
        P.adamw_step(self.params, [dtable, dweight, dbias], self.states, step=self.steps, lr=lr, weight_decay=[1e-4, 1e-4, 0.0],
                     copies=[self.table, self.weight, self.bias])
        return loss


def run(items=20000, steps=300, bits=8, words=20000, dim=64, classes=10, verbose=True):
    """Returns (agreement of the propagated, and of the student's, labels of unseen texts with the truth, first and last mean loss)."""
    graph = W.sbm(items, classes, 16.0, 60.0, 0.1, 3)
    with P.DynLP(graph.n, graph.row_ptr, graph.col, graph.w, classes, graph.seed_vertex, graph.seed_class) as d:
        d.static_solve(1e-5, 2000)
        soft, hard = d.get_labels()
    soft = torch.from_numpy(soft).cuda()
    true_class = torch.from_numpy(np.asarray(graph.true_class)).cuda().long()
    unseen_class = torch.arange(5000, device="cuda") % classes
    texts, unseen = make_texts(true_class, classes, words, 20.0, 1), make_texts(unseen_class, classes, words, 20.0, 2)
    # a row that propagation is unsure of (near 1/C everywhere) counts for little
    sure = ((soft.max(1).values - 1.0 / classes) / (1.0 - 1.0 / classes)).clamp(0.0, 1.0)
    student = Student(words, dim, classes, bits, 5)
    first = last = None
    for k in range(steps):
        loss = student.learn(*texts, soft, sure, 0.01)
        if k in (0, steps - 1):
            first, last = (float(loss.mean()) if k == 0 else first), float(loss.mean())
            if verbose:
                print(f"step {k}: mean loss {last:.4f}")
    propagated = float((torch.from_numpy(hard).cuda() == true_class).float().mean())
    learned = float((student.labels(*unseen)[1] == unseen_class).float().mean())
    if verbose:
        print(f"propagated labels agree with the truth on {propagated:.3f} of the graph, the student's on {learned:.3f} of unseen texts")
    return propagated, learned, first, last


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--items", type=int, default=20000)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args()
    run(a.items, a.steps, a.bits)
