"""Gradients of the loss whose vocabulary is taken in four and more pieces: buffers of g used again, dx added to over many launches,
pieces that are wider where fewer rows have a label, up to 128 of them, none.  Checked on the GPU against the definition in 64 bits."""
import pytest
import torch

from gpu_util import captured_kernels
from paper_2107_05377_b200 import binding as mt

pytestmark = pytest.mark.gpu

BF16, F32 = 2.0 ** -8, 2.0 ** -24       # half a step, relative


class Case:
    def __init__(self, rows, vocab, hidden, labelled, seed=0):
        gen = torch.Generator("cuda").manual_seed(seed + rows + labelled)
        new = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
        self.rows, self.vocab, self.hidden = rows, vocab, hidden
        self.w, self.x = (new(vocab, hidden) * 1.5 / hidden ** 0.5).bfloat16(), new(rows, hidden).bfloat16()
        self.b, self.weight = (new(vocab) * 0.3).bfloat16(), (0.5 + torch.rand(rows, device="cuda", generator=gen)) / rows
        self.labels = torch.randint(0, vocab, (rows,), device="cuda", generator=gen, dtype=torch.int32)
        away = torch.randperm(rows, device="cuda", generator=gen)[labelled:]
        self.labels[away] = -1
        self.x[away] = float("nan")
        self.lse = torch.zeros(rows, device="cuda")
        for at, z in self.logits():
            self.lse[at] = torch.logsumexp(z, 1).float()
        self.old = ((new(vocab, hidden) * 1e-4).bfloat16(), new(vocab) * 1e-4)

    def logits(self):
        """Rows with a label, up to 1024 at a time, and their logits in 64 bits."""
        for at in torch.nonzero(self.labels >= 0)[:, 0].split(1024):
            yield at, torch.addmm(self.b.double(), self.x[at].double(), self.w.double().T)

    def workspace(self):
        return torch.full((mt.mt_kernel_vocab_loss_grad_workspace(self.rows, self.vocab, self.hidden),), 0xFF, dtype=torch.uint8, device="cuda")

    def outputs(self, want=(True, True, True)):
        out = [torch.full((self.rows, self.hidden), float("nan"), dtype=torch.bfloat16, device="cuda"), self.old[0].clone(), self.old[1].clone()]
        return [t if on else None for t, on in zip(out, want)]

    def run(self, out, ws, accumulate=False, status=None):
        mt.mt_kernel_vocab_loss_grad(self.x, self.w, self.b, self.labels, self.lse, self.weight, *out, ws, accumulate, status)

    def check(self, out, accumulate=False):
        x_all, w = torch.nan_to_num(self.x.double()), self.w.double()
        n = int((self.labels >= 0).sum())
        z_size = x_all.abs() @ w.abs().max(0).values + self.b.double().abs().max()
        dx, dx_off, dx_size = (torch.zeros(self.rows, self.hidden, dtype=torch.float64, device="cuda") for _ in range(3))
        dw, dw_off, dw_size = (torch.zeros_like(w) for _ in range(3))
        db, db_off, db_size = (torch.zeros(self.vocab, dtype=torch.float64, device="cuda") for _ in range(3))
        for at, z in self.logits():
            row, label, weight = torch.arange(len(at), device="cuda"), self.labels[at].long(), self.weight[at].double()[:, None]
            p = torch.exp(z - self.lse[at].double()[:, None]) * weight
            g = p.clone()
            g[row, label] -= weight[:, 0]
            # of a probability, relative: a step per addition of its logit, the exponent's rounding, the exponential
            off = (self.hidden + 2) * 2 * F32 * z_size[at] + 8 * F32 * (self.lse[at].double().abs() + 1) + 2.0 ** -20
            dg = p * off[:, None] * 1.02 + 4 * F32 * (g.abs() + p)
            dgr = dg + BF16 * (g.abs() + dg)               # after the rounding of g
            dx[at], dx_off[at], dx_size[at] = g @ w, dgr @ w.abs(), (g.abs() + dgr) @ w.abs()
            x = x_all[at]
            dw += g.T @ x
            dw_off += dgr.T @ x.abs()
            dw_size += (g.abs() + dgr).T @ x.abs()
            db += g.sum(0)
            db_off += dg.sum(0)
            db_size += (g.abs() + dg).sum(0)
        if accumulate:
            dw, db = dw + self.old[0].double(), db + self.old[1].double()
        bounds = (dx_off + (self.vocab + 40) * 2 * F32 * dx_size, dw_off + (n + 2) * 2 * F32 * dw_size, db_off + (n + 2) * F32 * db_size)
        for name, got, want, bound, half in zip("xwb", out, (dx, dw, db), bounds, (BF16, BF16, 2 * F32)):
            if got is not None:
                off = (got.double() - want).abs() - (bound + half * (want.abs() + bound) + 1e-37 * self.rows)
                assert not off.isnan().any() and float(off.max()) <= 0.0, f"gradient of {name}"


# (8192 rows: four pieces, up to four times as wide; 32768 rows: five, up to eight times)
SIZES = [(8192, 30522, 16, n) for n in (8192, 4097, 4096, 2049, 600, 128, 1)] + [(32768, 9001, 24, n) for n in (32768, 16384, 8193, 8192, 4000, 100, 0)]


def pieces(rows):
    return 4 if rows == 8192 else 5


@pytest.mark.parametrize("rows,vocab,hidden,labelled", SIZES)
def test_gradients(rows, vocab, hidden, labelled):
    c = Case(rows, vocab, hidden, labelled)
    out, ws, status = c.outputs(), c.workspace(), torch.zeros(1, dtype=torch.int32, device="cuda")
    c.run(out, ws, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    c.check(out)


@pytest.mark.parametrize("rows,vocab", [(8192, 30522), (32768, 9001)])
def test_the_sizes_above_are_taken_in_pieces(rows, vocab):
    c = Case(rows, vocab, 16, 50)
    out, ws = c.outputs(), c.workspace()
    names = [name for name, _, _ in captured_kernels(lambda: c.run(out, ws))]
    assert sum("vocab_loss_pair" in name for name in names) == pieces(rows) + 1


@pytest.mark.parametrize("rows,vocab,hidden,labelled", [(8192, 30522, 16, 8192), (8192, 30522, 16, 3000), (32768, 9001, 24, 9000), (32768, 9001, 24, 120)])
def test_accumulation(rows, vocab, hidden, labelled):
    c = Case(rows, vocab, hidden, labelled)
    out = c.outputs()
    c.run(out, c.workspace(), accumulate=True)
    torch.cuda.synchronize()
    c.check(out, accumulate=True)


@pytest.mark.parametrize("labelled", [8192, 4000, 90])
@pytest.mark.parametrize("want", [(True, False, False), (False, True, False), (False, False, True), (True, False, True)])
def test_sides_that_are_frozen(labelled, want):
    c = Case(8192, 30522, 16, labelled)
    every, some = c.outputs(), c.outputs(want)
    c.run(every, c.workspace())
    c.run(some, c.workspace())
    torch.cuda.synchronize()
    for got, full in zip(some, every):
        assert got is None or torch.equal(got, full)


def test_equal_bits_on_two_streams_and_replayed():
    """At the same time, each with a workspace of its own; and a graph whose labels change between its replays."""
    c = Case(8192, 30522, 16, 8192)
    first = c.outputs()
    c.run(first, c.workspace())
    torch.cuda.synchronize()
    streams, results = [torch.cuda.Stream(), torch.cuda.Stream()], []
    spaces = [c.workspace() for _ in streams]
    outs = [c.outputs() for _ in streams]
    torch.cuda.synchronize()
    for s, out, ws in zip(streams, outs, spaces):
        with torch.cuda.stream(s):
            c.run(out, ws)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for out in outs for a, b in zip(out, first))
    graph, out = torch.cuda.CUDAGraph(), c.outputs()
    with torch.cuda.graph(graph):
        c.run(out, spaces[0])
    for labelled in (8192, 3000, 128, 0, 8192):
        other = Case(8192, 30522, 16, labelled)
        for name in ("x", "w", "b", "labels", "lse", "weight"):
            getattr(c, name).copy_(getattr(other, name))
        graph.replay()
        torch.cuda.synchronize()
        c.check(out)


@pytest.mark.parametrize("rows", [0, 5, 300])
def test_rows_of_the_table_gigabytes_apart(rows):
    """A stride of more than 2^31 bytes, of the table and of its gradient, with and without rows."""
    vocab, hidden, stride = 2, 24, 2 ** 30 + 8
    w_memory, dw_memory = (torch.zeros(stride + hidden, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c = Case(rows, vocab, hidden, rows)
    w = torch.as_strided(w_memory, (vocab, hidden), (stride, 1))
    w.copy_(c.w)
    c.w = w
    out = c.outputs()
    out[1] = torch.as_strided(dw_memory, (vocab, hidden), (stride, 1))
    out[1].fill_(1.0)
    dw_memory[hidden] = 3.0
    c.run(out, c.workspace())
    torch.cuda.synchronize()
    if rows:
        c.check(out)
    else:
        assert not out[1].any() and not out[2].any()
    assert float(dw_memory[hidden]) == 3.0 and float(dw_memory[hidden + 1:stride].abs().max()) == 0.0
