"""Cross entropy over the vocabulary and its gradients against their definitions in 64 bits: one row to thousands (one tile of rows
to many, one piece of the vocabulary to several), vocabularies of one word to beyond 2^16, widths that are no multiple of a k-block,
rows further apart than they are long, rows without a label that hold NaN, banned words, accumulation, frozen sides, graphs, streams."""
import numpy as np
import pytest
import torch

from oracle import vocab_oracle as orc
from paper_2107_05377_b200 import binding as mt

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8       # half a step of bf16, relative
F32 = 2.0 ** -24


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def matrix(rows, cols, gap, gen, std):
    full = (torch.randn(rows, cols + gap, generator=gen) * std).bfloat16().cuda()
    return full[:, :cols], full


class Case:
    def __init__(self, rows, vocab, hidden, bias=True, ignored=0.0, gap=0, seed=0, std=1.0):
        gen = torch.Generator().manual_seed(seed * 1000003 + rows * 31 + vocab * 7 + hidden)
        self.rows, self.vocab, self.hidden = rows, vocab, hidden
        self.w, _ = matrix(vocab, hidden, gap, gen, 1.5 * std / hidden ** 0.5)
        self.labels = torch.randint(0, vocab, (rows,), generator=gen, dtype=torch.int32)
        self.x, _ = matrix(rows, hidden, gap, gen, 1.0)
        self.x += (3.0 * torch.rand(rows, 1, generator=gen).cuda() * self.w[self.labels.long().cuda()].float()).bfloat16()
        away = torch.rand(rows, generator=gen) < ignored
        self.labels[away] = torch.randint(-100, 0, (int(away.sum()),), generator=gen, dtype=torch.int32)
        self.x[away.cuda()] = float("nan")              # what lies in rows without a label has no influence
        self.b = (torch.randn(vocab, generator=gen) * 0.3).bfloat16().cuda() if bias else None
        self.dloss = (0.5 + torch.rand(rows, generator=gen)) / rows
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.dev_labels, self.dev_dloss = self.labels.cuda(), self.dloss.cuda()

    def exact(self):
        return np.nan_to_num(f64(self.x)), f64(self.w), None if self.b is None else f64(self.b), self.labels.numpy()

    def logit_error(self):
        """Largest error of a logit of every row: products of bf16 numbers are exact in fp32; the sum of `hidden` of them and the
        bias is off by at most a step (the tensor cores may cut off) per addition of a partial sum below the sum of magnitudes."""
        x, w, b, _ = self.exact()
        size = np.abs(x) @ np.abs(w).max(axis=0) + (0.0 if b is None else np.abs(b[b > -1e30]).max(initial=0.0))
        return (self.hidden + 2) * 2 * F32 * size

    def forward(self, stream=None, fill=0xFF):
        ws = torch.full((mt.mt_kernel_vocab_loss_workspace(self.rows, self.vocab, self.hidden),), fill, dtype=torch.uint8, device="cuda")
        loss, lse = (torch.full((self.rows,), float("nan"), device="cuda") for _ in range(2))
        mt.mt_kernel_vocab_loss(self.x, self.w, self.b, self.dev_labels, loss, lse, ws, self.status, stream)
        return loss, lse, ws

    def backward(self, lse, want=(True, True, True), accumulate=False, gap=0, gen=None, dloss=True, fill=0xFF):
        ws = torch.full((mt.mt_kernel_vocab_loss_grad_workspace(self.rows, self.vocab, self.hidden),), fill, dtype=torch.uint8, device="cuda")
        gen = gen or torch.Generator().manual_seed(1)
        dx, dx_all = matrix(self.rows, self.hidden, gap, gen, 1.0)
        dw, dw_all = matrix(self.vocab, self.hidden, gap, gen, 1e-2)
        db = (torch.randn(self.vocab, generator=gen) * 1e-2).cuda()
        out = [t if on else None for t, on in zip((dx, dw, db), want)]
        mt.mt_kernel_vocab_loss_grad(self.x, self.w, self.b, self.dev_labels, lse, self.dev_dloss if dloss else None, *out, ws,
                                     accumulate, self.status)
        return out, (dx_all, dw_all), ws


def check_forward(c, loss, lse):
    want_loss, want_lse = orc.vocab_loss(*c.exact())
    # exponentials: off by 2^-21 relative and by the rounding of an exponent below |z| + |lse|; at most a hundred additions lie on the
    # way of a term to the sum; its logarithm and the last sum are rounded at the size of the results
    z = c.logit_error()
    bound = z + 100 * F32 + 2.0 ** -21 + 8 * F32 * (np.abs(want_lse) + np.abs(want_loss) + 1)
    there = c.labels.numpy() >= 0
    assert np.array_equal(f64(loss)[~there], np.zeros((~there).sum())) and np.array_equal(f64(lse)[~there], np.zeros((~there).sum()))
    assert (np.abs(f64(lse) - want_lse) <= bound)[there].all()
    finite = np.isfinite(want_loss)
    assert (np.abs(f64(loss)[finite] - want_loss[finite]) <= (bound + z)[finite]).all()
    assert (f64(loss)[~finite] == want_loss[~finite]).all()


def check_backward(c, out, lse, old=None, dloss=True):
    x, w, b, labels = c.exact()
    weight = f64(c.dloss) if dloss else np.ones(c.rows)
    want = orc.vocab_loss_grad(x, w, b, labels, weight)
    there = (labels >= 0) & (labels < c.vocab)
    # of a probability, relative: the logit, the lse that was given, the exponent's rounding and the exponential
    off = (c.logit_error() + np.abs(lse - orc.vocab_loss(x, w, b, labels)[1]) + 8 * F32 * (np.abs(lse) + 1) + 2.0 ** -20) * 1.02
    p, g = np.zeros((c.rows, c.vocab)), np.zeros((c.rows, c.vocab))
    for at, label, z, total in orc._softmax_rows(x, w, b, labels):
        p[at] = np.exp(z - total[:, None]) * np.abs(weight[at])[:, None]
        g[at] = np.exp(z - total[:, None])
        g[at, label] -= 1.0
        g[at] *= weight[at][:, None]
    dg = p * off[:, None] + 4 * F32 * np.abs(g)         # error of g before it is rounded
    dgr = dg + BF16 * (np.abs(g) + dg)                  # and after
    n = there.sum()
    size = np.abs(g) + dgr
    bounds = [dgr @ np.abs(w) + (c.vocab + 40) * 2 * F32 * (size @ np.abs(w)), dgr.T @ np.abs(x) + (n + 2) * 2 * F32 * (size.T @ np.abs(x)),
              dg.sum(axis=0) + (n + 2) * F32 * (np.abs(g) + dg).sum(axis=0)]
    for k, (got, exact, bound) in enumerate(zip(out, want, bounds)):
        if got is None:
            continue
        if old is not None and k > 0:
            exact = exact + old[k]
        rounding = (F32 * 2 if k == 2 else BF16) * (np.abs(exact) + bound)
        # (with the smallest normal numbers: exponentials below them count as zero)
        assert (np.abs(f64(got) - exact) <= bound + rounding + 1e-37 * c.rows).all(), f"gradient {k}"
    if out[0] is not None:
        assert np.array_equal(f64(out[0])[~there], np.zeros((int((~there).sum()), c.hidden)))


SIZES = [(1, 1, 8), (1, 50, 64), (3, 257, 72), (20, 30522, 64), (77, 513, 200), (128, 2000, 768), (256, 300, 136), (257, 1000, 64), (300, 4097, 1024),
         (615, 255, 96), (1030, 7000, 40), (2, 131073, 16), (511, 256, 256)]


@pytest.mark.parametrize("rows,vocab,hidden", SIZES)
@pytest.mark.parametrize("bias,ignored,gap", [(True, 0.0, 0), (False, 0.0, 8), (True, 0.6, 24)])
def test_forward(rows, vocab, hidden, bias, ignored, gap):
    c = Case(rows, vocab, hidden, bias, ignored, gap)
    loss, lse, _ = c.forward()
    torch.cuda.synchronize()
    assert int(c.status) == 0
    check_forward(c, loss, lse)


@pytest.mark.parametrize("rows,vocab,hidden", SIZES)
@pytest.mark.parametrize("bias,ignored,gap", [(True, 0.0, 0), (False, 0.0, 8), (True, 0.6, 24)])
def test_gradients(rows, vocab, hidden, bias, ignored, gap):
    c = Case(rows, vocab, hidden, bias, ignored, gap)
    lse = orc.vocab_loss(*c.exact())[1].astype(np.float32)
    out, memory, _ = c.backward(torch.from_numpy(lse).cuda(), gap=gap)
    torch.cuda.synchronize()
    assert int(c.status) == 0
    check_backward(c, out, lse.astype(np.float64))
    if gap:                                             # nothing is written between the rows
        gen = torch.Generator().manual_seed(1)
        for got, (r, k) in zip(memory, ((rows, 1.0), (vocab, 1e-2))):
            assert torch.equal(got[:, hidden:], matrix(r, hidden, gap, gen, k)[1][:, hidden:])


@pytest.mark.parametrize("rows,vocab,hidden,ignored", [(4097, 20000, 24, 0.0), (4200, 16000, 40, 0.3), (2900, 24007, 16, 0.85)])
def test_several_pieces_of_the_vocabulary(rows, vocab, hidden, ignored):
    c = Case(rows, vocab, hidden, True, ignored)
    loss, lse, _ = c.forward()
    check_forward(c, loss, lse)
    out, _, _ = c.backward(lse)
    torch.cuda.synchronize()
    assert int(c.status) == 0
    check_backward(c, out, f64(lse))


@pytest.mark.parametrize("want", [(True, False, False), (False, True, False), (False, False, True), (True, True, False), (False, True, True)])
@pytest.mark.parametrize("rows", [90, 4100])
def test_sides_that_are_frozen(want, rows):
    """A gradient that is not asked for changes no bit of the others."""
    c = Case(rows, 9000, 64, True, 0.2)
    lse = c.forward()[1]
    every, _, _ = c.backward(lse)
    some, _, _ = c.backward(lse, want)
    torch.cuda.synchronize()
    for got, on, full in zip(some, want, every):
        assert got is None if not on else torch.equal(got, full)


@pytest.mark.parametrize("rows,vocab", [(40, 700), (4100, 9001)])
def test_accumulation(rows, vocab):
    c = Case(rows, vocab, 72, True, 0.4)
    lse = c.forward()[1]
    gen = torch.Generator().manual_seed(1)
    old = [None, f64(matrix(rows, 72, 0, gen, 1.0)[0])]
    old = [None, f64(matrix(vocab, 72, 0, gen, 1e-2)[0]), f64(torch.randn(vocab, generator=gen) * 1e-2)]
    out, _, _ = c.backward(lse, accumulate=True)
    torch.cuda.synchronize()
    check_backward(c, out, f64(lse), old)


@pytest.mark.parametrize("rows", [1, 100, 129, 300, 4100])
def test_weights_of_any_sign(rows):
    """Weights below zero, zero (their rows have no gradient), tiny and huge ones."""
    c = Case(rows, 2100, 72, True, 0.1)
    c.dloss[::3] *= -1.0
    c.dloss[1::5] = 0.0
    c.dloss[2::7] *= 1e-12
    c.dloss[4::11] *= 1e6
    c.dev_dloss = c.dloss.cuda()
    lse = c.forward()[1]
    out, _, _ = c.backward(lse)
    torch.cuda.synchronize()
    check_backward(c, out, f64(lse))
    assert not out[0][1::5].any()


@pytest.mark.parametrize("rows,vocab,hidden", [(40, 600, 4096), (300, 513, 2056), (129, 70000, 8), (128, 70000, 8)])
def test_wide_hidden_states_and_long_vocabularies(rows, vocab, hidden):
    c = Case(rows, vocab, hidden, True, 0.2)
    loss, lse, _ = c.forward()
    check_forward(c, loss, lse)
    out, _, _ = c.backward(lse)
    torch.cuda.synchronize()
    check_backward(c, out, f64(lse))


@pytest.mark.parametrize("rows", [77, 900])
def test_the_same_label_everywhere(rows):
    c = Case(rows, 3000, 64, False)
    c.labels[:] = 2999
    c.dev_labels = c.labels.cuda()
    loss, lse, _ = c.forward()
    check_forward(c, loss, lse)
    out, _, _ = c.backward(lse)
    torch.cuda.synchronize()
    check_backward(c, out, f64(lse))


def test_weights_of_one():
    c = Case(33, 500, 64)
    lse = c.forward()[1]
    out, _, _ = c.backward(lse, dloss=False)
    torch.cuda.synchronize()
    check_backward(c, out, f64(lse), dloss=False)


@pytest.mark.parametrize("rows", [5, 300, 4100])
@pytest.mark.parametrize("accumulate", [False, True])
def test_no_row_has_a_label(rows, accumulate):
    c = Case(rows, 9000, 64, True, 2.0)
    loss, lse, _ = c.forward()
    gen = torch.Generator().manual_seed(1)
    matrix(rows, 64, 0, gen, 1.0)
    old = [matrix(c.vocab, 64, 0, gen, 1e-2)[0], (torch.randn(c.vocab, generator=gen) * 1e-2).cuda()]
    out, _, _ = c.backward(lse, accumulate=accumulate)
    torch.cuda.synchronize()
    for t in (loss, lse, out[0]):
        assert torch.equal(t, torch.zeros_like(t))
    for t, before in zip(out[1:], old):
        assert torch.equal(t, before if accumulate else torch.zeros_like(t))


def test_no_rows():
    c = Case(0, 50, 64)
    c.forward()
    out, _, _ = c.backward(torch.zeros(0, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(out[1], torch.zeros_like(out[1])) and torch.equal(out[2], torch.zeros_like(out[2]))


@pytest.mark.parametrize("rows", [30, 700])
def test_labels_outside_the_vocabulary_are_flagged_and_take_no_part(rows):
    c = Case(rows, 600, 64, True, 0.1)
    c.labels[3::7] = 600 + torch.arange(len(c.labels[3::7]), dtype=torch.int32)
    c.labels[4] = 2 ** 31 - 1
    c.dev_labels = c.labels.cuda()
    loss, lse, _ = c.forward()
    torch.cuda.synchronize()
    assert int(c.status) == mt.FLAG_BAD_TOKEN
    c.status.zero_()
    out, _, _ = c.backward(lse)
    torch.cuda.synchronize()
    assert int(c.status) == mt.FLAG_BAD_TOKEN
    bad = c.labels >= 600
    assert not loss[bad.cuda()].any() and not lse[bad.cuda()].any()
    c.labels[bad] = -1
    check_forward(c, loss, lse)
    check_backward(c, out, f64(lse))


@pytest.mark.parametrize("rows", [70, 300, 4100])
def test_banned_words_and_sharp_rows(rows):
    """A bias of -inf; whole tiles of it; logits far apart (one word has all of the probability)."""
    c = Case(rows, 1500, 64, True, 0.0, std=8.0)
    c.b[200:900] = float("-inf")
    c.b[1499] = float("-inf")
    c.labels[c.b.cpu()[c.labels.long()] < -1e30] = 10
    c.labels[:2] = torch.tensor([300, 5])                # the loss of a banned word is infinite
    c.dev_labels = c.labels.cuda()
    loss, lse, _ = c.forward()
    torch.cuda.synchronize()
    assert float(loss[0]) == float("inf")
    check_forward(c, loss, lse)
    out, _, _ = c.backward(lse)
    torch.cuda.synchronize()
    check_backward(c, out, f64(lse))
    assert not out[2][200:300].any() and not out[1][301:900].any()


@pytest.mark.parametrize("rows", [3, 70, 300, 4100])
@pytest.mark.parametrize("left", [0, 40])
def test_words_banned_by_the_lowest_number(rows, left):
    """A bias of bf16's lowest value on all words but `left`: where it is on all, every logit is that value (what x and W add is lost in
    its rounding) and the words are equally likely."""
    c = Case(rows, 1300, 64, True, 0.1)
    lowest = torch.finfo(torch.bfloat16).min
    c.b[left:] = lowest
    if left:
        c.labels = torch.where(c.labels >= 0, c.labels % left, c.labels)
        c.dev_labels = c.labels.cuda()
    loss, lse, _ = c.forward()
    out, _, _ = c.backward(lse)
    torch.cuda.synchronize()
    if left:
        check_forward(c, loss, lse)
        check_backward(c, out, f64(lse))
        assert not out[2][left:].any() and not out[1][left:].any()
        return
    there = (c.labels >= 0).numpy()
    assert (np.abs(f64(loss)[there] - np.log(1300.0)) <= 2.0 ** -18).all() and (f64(lse)[there] == float(lowest)).all()
    # (the lse that the backward pass is given cannot hold the log 1300 above the lowest number: its probabilities are all one, but finite)
    assert torch.isfinite(out[0]).all() and torch.isfinite(out[1]).all() and torch.isfinite(out[2]).all()


def test_gradient_against_differences():
    """The gradient of the call's own loss along a direction, by a difference quotient of the 64-bit loss at the same bf16 points."""
    c = Case(60, 400, 64, True, 0.2)
    lse = c.forward()[1]
    out, _, _ = c.backward(lse)
    x, w, b, labels = c.exact()
    weight, h = f64(c.dloss), 1e-6
    rng = np.random.default_rng(0)
    total = lambda x, w, b: float(weight @ orc.vocab_loss(x, w, b, labels)[0])  # noqa: E731
    for k, got in enumerate(out):
        step = rng.standard_normal((x, w, b)[k].shape)
        args = [[x, w, b], [x, w, b]]
        args[0][k], args[1][k] = (x, w, b)[k] + h * step, (x, w, b)[k] - h * step
        quotient = (total(*args[0]) - total(*args[1])) / (2 * h)
        # g and the result are rounded to bf16: half a step of each term's size, whatever the signs
        grads = [np.abs(v) for v in orc.vocab_loss_grad(x, w, b, labels, weight)]
        slack = 2 * BF16 * float((grads[k] * np.abs(step)).sum()) + (0 if k == 2 else BF16 * spread(c, step, k))
        assert abs(float((f64(got) * step).sum()) - quotient) <= slack + 1e-7


def spread(c, step, k):
    """sum |g| times what a step moves a logit by: what rounding g can move the result by."""
    x, w, b, labels = c.exact()
    g = np.zeros((c.rows, c.vocab))
    for at, label, z, total in orc._softmax_rows(x, w, b, labels):
        g[at] = np.exp(z - total[:, None])
        g[at, label] -= 1.0
    moved = np.abs(step @ w.T) if k == 0 else np.abs(x @ step.T)
    return float((np.abs(g) * f64(c.dloss)[:, None] * moved).sum())


def test_equal_bits_on_any_stream_whatever_the_workspace_held_and_replayed():
    c = Case(4100, 9001, 72, True, 0.3)
    loss, lse, ws = c.forward(fill=0)
    first, _, _ = c.backward(lse, fill=0)
    torch.cuda.synchronize()
    results = []
    for s in (torch.cuda.Stream(), torch.cuda.Stream()):  # at the same time
        with torch.cuda.stream(s):
            results.append((c.forward(stream=s), c.backward(lse)))
    torch.cuda.synchronize()
    for (l1, l2, _), (grads, _, _) in results:
        assert torch.equal(l1, loss) and torch.equal(l2, lse) and all(torch.equal(a, b) for a, b in zip(grads, first))
    graph = torch.cuda.CUDAGraph()
    ws_grad = torch.empty(mt.mt_kernel_vocab_loss_grad_workspace(c.rows, c.vocab, c.hidden), dtype=torch.uint8, device="cuda")
    again = [torch.empty_like(t) for t in (loss, lse, *first)]
    with torch.cuda.graph(graph):
        mt.mt_kernel_vocab_loss(c.x, c.w, c.b, c.dev_labels, again[0], again[1], ws)
        mt.mt_kernel_vocab_loss_grad(c.x, c.w, c.b, c.dev_labels, again[1], c.dev_dloss, *again[2:], ws_grad)
    for turn in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, (loss, lse, *first)))
    c.labels[::2] = 7                                     # other labels, as many rows with one as there are now
    c.x[::2] = 0.25
    c.dev_labels.copy_(c.labels)
    graph.replay()
    torch.cuda.synchronize()
    check_forward(c, again[0], again[1])
    check_backward(c, again[2:], f64(again[1]))


def test_binding_refusals():
    c = Case(4, 30, 16)
    loss, lse, ws = c.forward()
    good = dict(x=c.x, w=c.w, bias=c.b, labels=c.dev_labels, loss=loss, lse=lse, workspace=ws)
    for change in [dict(x=c.x.float()), dict(w=c.w.half()), dict(x=c.x[:, :8]), dict(bias=c.b.float()), dict(bias=c.b[:-1]), dict(labels=c.dev_labels.long()),
                   dict(loss=loss[:3]), dict(lse=lse.double()), dict(workspace=ws[:-256]), dict(workspace=ws[16:]), dict(x=c.x.cpu()),
                   dict(x=torch.zeros(16, 4, dtype=torch.bfloat16, device="cuda").T), dict(x=torch.zeros(4, 20, dtype=torch.bfloat16, device="cuda")[:, 4:]),
                   dict(x=torch.zeros(4, 18, dtype=torch.bfloat16, device="cuda")[:, :16])]:
        with pytest.raises(mt.MTError):
            mt.mt_kernel_vocab_loss(**(good | change))
    out, _, ws = c.backward(lse)
    good = dict(x=c.x, w=c.w, bias=c.b, labels=c.dev_labels, lse=lse, grad_loss=c.dev_dloss, grad_x=out[0], grad_w=out[1], grad_bias=out[2], workspace=ws)
    for change in [dict(grad_x=None, grad_w=None, grad_bias=None), dict(grad_x=out[0].float()), dict(grad_w=out[1][:-1]), dict(grad_bias=out[2].bfloat16()),
                   dict(grad_loss=c.dev_dloss.double()), dict(lse=lse[:2]), dict(workspace=ws[:256]), dict(grad_w=out[1].cpu())]:
        with pytest.raises(mt.MTError):
            mt.mt_kernel_vocab_loss_grad(**(good | change))


def test_what_follows_a_gradient_without_labels_sees_it_whole():
    # no kernel of a call may end before those in front of it: the next call reads the zeros of dW at once
    vocab, hidden, rows = 120000, 1024, 300
    c = Case(rows, vocab, hidden, False, 2.0)
    ws = torch.empty(mt.mt_kernel_vocab_loss_grad_workspace(rows, vocab, hidden), dtype=torch.uint8, device="cuda")
    dx = torch.empty(rows, hidden, dtype=torch.bfloat16, device="cuda")
    dw = torch.empty(vocab, hidden, dtype=torch.bfloat16, device="cuda")
    lse, ids = torch.zeros(rows, device="cuda"), torch.arange(vocab, dtype=torch.int32, device="cuda")
    seen = torch.empty(vocab, hidden, dtype=torch.bfloat16, device="cuda")
    for _ in range(5):
        dw.fill_(1.0)
        seen.fill_(2.0)
        mt.mt_kernel_vocab_loss_grad(c.x, c.w, None, c.dev_labels, lse, None, dx, dw, None, ws)
        mt.mt_kernel_embedding_lookup(ids, dw, seen)
        torch.cuda.synchronize()
        assert not seen.any() and not dx.any()


@pytest.mark.parametrize("rows", [100, 4000])
@pytest.mark.parametrize("hidden", [768, 4096])
def test_logits_are_not_too_small_on_average(rows, hidden):
    """With one word lse is the logit.  The tensor cores cut partial sums off: a logit that grows evenly over hidden / 16 of them would
    lose about 0.27 half steps of itself each time (at most 0.5, half of it on average, and less than half a logit to lose it from)."""
    gen = torch.Generator().manual_seed(hidden)
    w = torch.randn(1, hidden, generator=gen) * 1.5 / hidden ** 0.5
    x = torch.randn(rows, hidden, generator=gen) + w * (3.0 + 3.0 * torch.rand(rows, 1, generator=gen))
    w, x = w.bfloat16().cuda(), x.bfloat16().cuda()
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    ws = torch.empty(mt.mt_kernel_vocab_loss_workspace(rows, 1, hidden), dtype=torch.uint8, device="cuda")
    mt.mt_kernel_vocab_loss(x, w, None, torch.zeros(rows, dtype=torch.int32, device="cuda"), loss, lse, ws)
    torch.cuda.synchronize()
    z = (f64(x) @ f64(w).T)[:, 0]
    assert abs((f64(lse) - z).mean()) <= 0.1 * F32 * hidden / 16 * z.mean()
    assert not loss.any()


@pytest.mark.parametrize("rows,labelled", [(60, 60), (128, 100), (129, 1), (300, 20), (300, 65), (300, 128), (4500, 40), (4500, 127), (9000, 128)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_few_labels_leave_only_the_rounding_of_the_result_in_dw(rows, labelled, accumulate):
    """Up to 128 rows with a label, of however many: a row of dW is little else than one entry of g times a row of x, and g is taken in two
    terms, so that its rounding (2^-8 relative, and 2^-8 of what that left) is no part of the error."""
    vocab, hidden = 2100, 200
    c = Case(rows, vocab, hidden, True, 0.0)
    away = torch.randperm(rows, generator=torch.Generator().manual_seed(rows))[labelled:]
    c.labels[away] = -1
    c.x[away.cuda()] = float("nan")
    c.dev_labels = c.labels.cuda()
    x, w, b, labels = c.exact()
    weight, there = f64(c.dloss), labels >= 0
    _, exact_lse = orc.vocab_loss(x, w, b, labels)
    lse = torch.from_numpy(np.where(there, exact_lse, 0.0)).float().cuda()
    gen = torch.Generator().manual_seed(1)
    matrix(rows, hidden, 0, gen, 1.0)
    old = f64(matrix(vocab, hidden, 0, gen, 1e-2)[0]) if accumulate else 0.0
    out, _, _ = c.backward(lse, accumulate=accumulate)
    torch.cuda.synchronize()
    want = orc.vocab_loss_grad(x, w, b, labels, weight)[1] + old
    z = x[there] @ w.T + b
    p = np.exp(z - exact_lse[there][:, None]) * weight[there][:, None]
    g = p.copy()
    g[np.arange(labelled), labels[there]] -= weight[there]
    off = (c.logit_error()[there] + 9 * F32 * (np.abs(exact_lse[there]) + 1) + 2.0 ** -20) * 1.02
    dg = p * off[:, None] + 4 * F32 * np.abs(g)
    dg += BF16 ** 2 * (np.abs(g) + dg)
    bound = dg.T @ np.abs(x[there]) + (2 * labelled + 2) * 2 * F32 * ((np.abs(g) + dg).T @ np.abs(x[there]))
    assert (np.abs(f64(out[1]) - want) <= bound + BF16 * (np.abs(want) + bound)).all()
