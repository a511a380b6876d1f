"""Logits of the vocabulary operators: what the formula x W^T + b gives, for operands whose sums fp32 holds exactly as for those
where the tensor cores cut partial sums off.  With one word lse is the logit, and a gradient says how far exp(z - lse) is from one."""
import numpy as np
import pytest
import torch

from paper_2107_05377_b200 import binding as mt

pytestmark = pytest.mark.gpu

F32 = 2.0 ** -24       # half a step of fp32, relative


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def forward(x, w, bias=None):
    rows, vocab, hidden = len(x), len(w), x.shape[1]
    loss, lse = (torch.full((rows,), float("nan"), device="cuda") for _ in range(2))
    ws = torch.full((mt.mt_kernel_vocab_loss_workspace(rows, vocab, hidden),), 0xFF, dtype=torch.uint8, device="cuda")
    mt.mt_kernel_vocab_loss(x, w, bias, torch.zeros(rows, dtype=torch.int32, device="cuda"), loss, lse, ws)
    torch.cuda.synchronize()
    return loss, lse


def backward(x, w, lse, weight, bias=None):
    rows, vocab, hidden = len(x), len(w), x.shape[1]
    dx, dw, db = torch.full_like(x, float("nan")), torch.full_like(w, float("nan")), torch.full((vocab,), float("nan"), device="cuda")
    ws = torch.full((mt.mt_kernel_vocab_loss_grad_workspace(rows, vocab, hidden),), 0xFF, dtype=torch.uint8, device="cuda")
    mt.mt_kernel_vocab_loss_grad(x, w, bias, torch.zeros(rows, dtype=torch.int32, device="cuda"), lse, weight, dx, dw, db, ws)
    torch.cuda.synchronize()
    return dx, dw, db


def exact_operands(kind, rows, hidden, gen):
    """bf16 operands of one word whose partial sums are fp32 numbers in any order."""
    if kind == "one term":                               # a product of two bf16 numbers has 16 bits
        x, w = torch.zeros(rows, hidden), torch.randn(1, hidden, generator=gen) * 3.0
        x[torch.arange(rows), torch.randint(0, hidden, (rows,), generator=gen)] = 1.0 + torch.rand(rows, generator=gen)
    elif kind == "integers":                             # at most 16 * 16384 in magnitude
        x, w = (torch.randint(-4, 5, (n, hidden), generator=gen).float() for n in (rows, 1))
    else:                                                # a narrow hidden state in a wide row: zeros behind
        x, w = (torch.randint(-7, 8, (n, hidden), generator=gen) * 2.0 ** -5 for n in (rows, 1))
        x[:, min(40, hidden):] = 0.0
    return x.bfloat16().cuda(), w.bfloat16().cuda()


@pytest.mark.parametrize("rows", [1, 20, 100, 300, 2100])
@pytest.mark.parametrize("hidden", [8, 200, 768, 1000, 16384])
@pytest.mark.parametrize("kind", ["one term", "integers", "narrow"])
def test_sums_that_fp32_holds_are_exact(rows, hidden, kind):
    x, w = exact_operands(kind, rows, hidden, torch.Generator().manual_seed(rows + hidden))
    z = (f64(x) @ f64(w).T)[:, 0]
    loss, lse = forward(x, w)
    assert np.array_equal(f64(lse), z) and not loss.any()
    # weights of powers of two: exp(0) = 1 of them is the weight
    grads = backward(x, w, lse, torch.full((rows,), 2.0 ** -9, device="cuda"))
    assert not any(g.any() for g in grads)


@pytest.mark.parametrize("rows", [100, 3000])
@pytest.mark.parametrize("hidden", [768, 16384])
@pytest.mark.parametrize("where", ["first", "last"])
def test_large_columns_at_either_end(rows, hidden, where):
    """Two columns make most of the logit, the others a hundredth of it.  An instruction of 16 terms cuts off less than a step of the partial
    sum (half of one on average; two where its own terms are aligned first); sums of at most 384 terms are joined rounding to nearest."""
    gen = torch.Generator().manual_seed(hidden + rows)
    x, w = torch.randn(rows, hidden, generator=gen) * 0.5, torch.randn(1, hidden, generator=gen) / hidden ** 0.5
    at = slice(0, 2) if where == "first" else slice(hidden - 2, hidden)
    x[:, at], w[:, at] = 8.0 + torch.rand(rows, 2, generator=gen), 6.0 + torch.rand(1, 2, generator=gen)
    x, w = x.bfloat16().cuda(), w.bfloat16().cuda()
    z = (f64(x) @ f64(w).T)[:, 0]
    off = f64(forward(x, w)[1]) - z
    step = 2 * F32 * np.abs(z).max() * 1.1
    sums = -(-hidden // 192)
    assert np.abs(off).max() <= (2 * 24 + 0.5 * sums + 1) * step
    assert abs(off.mean()) <= (0.5 * 24 + 1) * step


@pytest.mark.parametrize("rows", [100, 4000])
@pytest.mark.parametrize("hidden", [768, 4096])
def test_gradients_are_not_off_on_average(rows, hidden):
    """The gradient of a bias of one word is the sum of weight * (exp(z - lse) - 1): with the exact lse, what the logits are off by."""
    gen = torch.Generator().manual_seed(hidden)
    w = torch.randn(1, hidden, generator=gen) * 1.5 / hidden ** 0.5
    x = torch.randn(rows, hidden, generator=gen) + w * (3.0 + 3.0 * torch.rand(rows, 1, generator=gen))
    w, x = w.bfloat16().cuda(), x.bfloat16().cuda()
    z = (f64(x) @ f64(w).T)[:, 0]
    db = backward(x, w, torch.from_numpy(z).float().cuda(), torch.full((rows,), 1.0 / rows, device="cuda"))[2]
    # (0.27 of half a step per 16 of 384 terms, and a tenth more; the lse is rounded, the exponential off by 2^-22)
    assert abs(float(db)) <= 0.3 * F32 * 24 * z.mean() + F32 * np.abs(z).max() + 2.0 ** -21


@pytest.mark.parametrize("rows", [100, 300])
@pytest.mark.parametrize("weight", [0.7 * 2.0 ** -12, -0.7 * 2.0 ** -12, 3e-12, 7e-25, -7e-25, 7e19])
def test_a_weight_scales_the_gradient_whatever_its_size(rows, weight):
    """Rows sure of their label: weight * (p - 1) with p near 1.  p is off by the exponential's 2^-22 and the product by half a step, so that the
    gradient is off by as much of the weight, however far the weight is from one."""
    x, w = torch.zeros(rows, 8, dtype=torch.bfloat16, device="cuda"), torch.randn(2, 8, device="cuda").bfloat16()
    bias = torch.tensor([0.0, -10.0], device="cuda").bfloat16()
    lse = np.float32(np.log1p(np.exp(-10.0)))
    weight = np.float32(weight)
    db = f64(backward(x, w, torch.full((rows,), float(lse), device="cuda"), torch.full((rows,), float(weight), device="cuda"), bias)[2])
    want = rows * float(weight) * np.array([np.expm1(-float(lse)), np.exp(-10.0 - float(lse))])
    bound = rows * abs(float(weight)) * (2.0 ** -22 + 2.0 ** -23) * np.array([1.0, np.exp(-10.0) * 8]) + (rows + 2) * F32 * np.abs(want)
    assert (np.abs(db - want) <= bound).all()
    # and none at all where the label has all of the probability
    grads = backward(x, w[:1], torch.zeros(rows, device="cuda"), torch.full((rows,), float(weight), device="cuda"), bias[:1])
    assert not any(g.any() for g in grads)
