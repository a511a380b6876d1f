"""The vocabulary operators together, as a training step of a language model with a tied table uses them: lookup, dropout, loss over the
vocabulary, its gradient, dropout's, the lookup's into the same table; eagerly, replayed as a CUDA graph that draws new masks, and with a
table that changes between the steps."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import vocab_oracle as orc
from paper_2107_05377_b200 import binding as mt

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HALF = 2.0 ** -8       # half a step of bf16, relative
SEED, P = 1234567890123, 0.1


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


class Step:
    """What the step keeps, and the step: x = dropout(scale E[ids]), loss(x E^T + b, labels), and the gradients of E and b."""

    def __init__(self, tokens, vocab, hidden, masked):
        gen = torch.Generator().manual_seed(tokens)
        self.table = (torch.randn(vocab, hidden, generator=gen) * 1.5 / hidden ** 0.5).bfloat16().cuda()
        self.bias = (torch.randn(vocab, generator=gen) * 0.1).bfloat16().cuda()
        self.scale = float(hidden) ** 0.5 * 0.5
        ids = torch.randint(0, vocab, (tokens,), generator=gen, dtype=torch.int32)
        ids[::9] = -1                                    # padding
        ids[1::4] = vocab // 2                           # a word that comes often
        labels = torch.where(torch.rand(tokens, generator=gen) < masked, torch.randint(0, vocab, (tokens,), generator=gen), -1).int()
        labels[ids < 0] = -1
        self.ids, self.labels = ids.cuda(), labels.cuda()
        self.weight = torch.full((tokens,), 1.0 / max(1, int((labels >= 0).sum()))).cuda()
        new = lambda *shape, dtype=torch.bfloat16: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
        self.x0, self.x, self.dx, self.dx0 = (new(tokens, hidden) for _ in range(4))
        self.dtable, self.dbias = new(vocab, hidden), new(vocab, dtype=torch.float32)
        self.loss, self.lse = new(tokens, dtype=torch.float32), new(tokens, dtype=torch.float32)
        sizes = [mt.mt_kernel_embedding_grad_workspace(tokens, vocab, hidden), mt.mt_kernel_vocab_loss_workspace(tokens, vocab, hidden),
                 mt.mt_kernel_vocab_loss_grad_workspace(tokens, vocab, hidden)]
        self.ws = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")   # one after the other on a stream: one workspace for all
        self.number = torch.zeros(1, dtype=torch.int64, device="cuda")

    def run(self):
        mt.mt_kernel_embedding_lookup(self.ids, self.table, self.x0, self.scale)
        mt.mt_kernel_dropout(self.x0, self.x, P, SEED, counter_dev=self.number)
        mt.mt_kernel_vocab_loss(self.x, self.table, self.bias, self.labels, self.loss, self.lse, self.ws)
        mt.mt_kernel_vocab_loss_grad(self.x, self.table, self.bias, self.labels, self.lse, self.weight, self.dx, self.dtable, self.dbias, self.ws)
        mt.mt_kernel_dropout(self.dx, self.dx0, P, SEED, counter_dev=self.number)
        mt.mt_kernel_embedding_grad(self.ids, self.dx0, self.dtable, self.ws, self.scale, accumulate=True)
        self.number += 1

    def check(self, number):
        """Against the formula in 64 bits at the hidden states that the step has stored."""
        ids, labels = self.ids.cpu().numpy(), self.labels.cpu().numpy()
        w, b, weight = f64(self.table), f64(self.bias), f64(self.weight)
        keep = orc.dropout_keep(*self.x.shape, P, SEED, number)
        factor = 1.0 / (1.0 - orc.dropout_threshold(P) / 65536.0)
        want = orc.embedding_lookup(ids, w, float(np.float32(self.scale))) * keep * factor
        x = f64(self.x)
        assert (np.abs(x - want) <= 2.05 * HALF * np.abs(want)).all()       # two roundings to bf16, some to fp32
        loss, lse = orc.vocab_loss(x, w, b, labels)
        z = (x.shape[1] + 2) * 2.0 ** -23 * (np.abs(x) @ np.abs(w).max(axis=0) + np.abs(b).max())   # of a logit: a step per addition
        assert (np.abs(f64(self.loss) - loss) <= 2 * z + 2.0 ** -15).all()
        # the gradients and, beside them, how far roundings can move them
        dx, dw, db = orc.vocab_loss_grad(x, w, b, labels, weight)
        g = np.zeros((len(x), len(w)))
        p = np.zeros_like(g)
        for at, label, logits, total in orc._softmax_rows(x, w, b, labels):
            p[at] = np.exp(logits - total[:, None]) * weight[at][:, None]
            g[at] = p[at]
            g[at, label] -= weight[at]
        off = p * (2.1 * z + 2.0 ** -17)[:, None] + 2.0 ** -22 * np.abs(g)
        off_g = off + HALF * (np.abs(g) + off)
        sums = 2.0 ** -22 * (len(w) + 40)
        off_dx = off_g @ np.abs(w) + sums * (np.abs(g) @ np.abs(w))
        off_dx += HALF * (np.abs(dx) + off_dx)
        dx0 = dx * keep * factor
        off_dx0 = off_dx * keep * factor
        off_dx0 += HALF * (np.abs(dx0) + off_dx0)
        scale = float(np.float32(self.scale))
        de, size, count = orc.embedding_grad(ids, dx0, len(w), scale)
        off_de = orc.embedding_grad(ids, off_dx0, len(w), scale)[0] + (count[:, None] + 2) * 2.0 ** -23 * size
        off_dw = off_g.T @ np.abs(x) + (len(x) + 2) * 2.0 ** -22 * (np.abs(g).T @ np.abs(x))
        off_dw += HALF * (np.abs(dw) + off_dw)
        want, off_all = dw + de, off_dw + off_de
        off_all += HALF * (np.abs(want) + off_all)
        assert (np.abs(f64(self.dtable) - want) <= off_all + 1e-30).all()
        assert (np.abs(f64(self.dbias) - db) <= off.sum(axis=0) + (len(x) + 2) * 2.0 ** -23 * np.abs(g).sum(axis=0) + 1e-30).all()


@pytest.mark.parametrize("tokens,vocab,hidden,masked", [(5, 40, 64, 1.0), (90, 700, 200, 0.5), (700, 3001, 128, 0.15), (4500, 2000, 64, 0.4)])
def test_step(tokens, vocab, hidden, masked):
    s = Step(tokens, vocab, hidden, masked)
    for turn in range(2):
        s.run()
        torch.cuda.synchronize()
        s.check(turn)
        s.table.copy_((s.table.float() - 2.0 * s.dtable.float()).bfloat16())       # (the next step sees the new table)


@pytest.mark.parametrize("tokens", [60, 2100])
def test_replayed_steps(tokens):
    s = Step(tokens, 900, 72, 0.5)
    s.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for turn in range(1, 4):
        for t in (s.x0, s.x, s.dx, s.dx0, s.dtable, s.dbias, s.loss, s.lse):
            t.fill_(float("nan"))
        s.ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        s.check(turn)


def test_two_graphs_side_by_side():
    """Captured apart, each with a workspace of its own, replayed at the same time."""
    steps, graphs, streams = [Step(500, 900, 72, 0.5), Step(110, 900, 72, 0.9)], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in steps:
        s.run()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            s.run()
    torch.cuda.synchronize()
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for s in steps:
        s.check(3)


def test_first_calls_of_a_process_may_be_captured():
    code = ("import torch, sys; sys.path[:0] = [%r, %r]; from test_gpu_vocab_step import Step; s = Step(300, 900, 72, 0.5); t = Step(60, 900, 72, 0.5)\n"
            "torch.cuda.synchronize(); g = torch.cuda.CUDAGraph()\n"
            "with torch.cuda.graph(g):\n    s.run(); t.run()\n"
            "g.replay(); torch.cuda.synchronize(); s.check(0); t.check(0); print('captured')" % (ROOT, os.path.join(ROOT, "tests")))
    out = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT, timeout=300)
    assert out.returncode == 0 and "captured" in out.stdout, out.stderr[-2000:]


def test_first_calls_of_a_process_with_a_sort_may_be_captured():
    """Token lists that one CTA and that a cluster of sixteen sorts, whose launch asks the device what fits."""
    code = ("import torch, sys; sys.path[:0] = [%r, %r]; from test_gpu_vocab_step import Step; s = Step(1500, 900, 72, 0.5); t = Step(6000, 900, 72, 0.3)\n"
            "torch.cuda.synchronize(); g = torch.cuda.CUDAGraph()\n"
            "with torch.cuda.graph(g):\n    t.run(); s.run()\n"
            "g.replay(); torch.cuda.synchronize(); s.check(0); t.check(0); print('captured')" % (ROOT, os.path.join(ROOT, "tests")))
    out = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT, timeout=300)
    assert out.returncode == 0 and "captured" in out.stdout, out.stderr[-2000:]
