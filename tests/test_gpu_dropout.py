"""Dropout against its definition in 64 bits: the mask bit for bit, rows of any length and distance, both types, in place, with a
residual, the gradient as the same call, a replayed graph that draws anew."""
import numpy as np
import pytest
import torch

from oracle import vocab_oracle as orc
from paper_2107_05377_b200 import binding as mt

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def matrix(rows, cols, gap, dtype, gen, offset=0):
    full = torch.randn(offset + rows * (cols + gap), generator=gen).to(dtype).cuda()
    return full[offset:].view(rows, cols + gap)[:, :cols], full


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def check(x, y, before, p, seed, counter, residual):
    want = orc.dropout(f64(x) if before is None else before, p, seed, counter, residual)
    got = f64(y)
    kept = want if residual is None else want - residual
    # the factor, the product and the sum in fp32, then the output's type
    bound = np.abs(kept) * 2.02 * 2.0 ** -24 + np.abs(want) * (2.0 ** -24 + 1.01 * HALF_STEP[y.dtype])
    assert (np.abs(got - want) <= bound).all()
    return want


@pytest.mark.parametrize("x_type", ["bf16", "f32"])
@pytest.mark.parametrize("y_type", ["bf16", "f32"])
@pytest.mark.parametrize("with_residual", [False, True])
@pytest.mark.parametrize("rows,cols,gap,offset", [(1, 1, 0, 0), (1, 8, 0, 0), (101, 768, 0, 0), (5, 13, 0, 0), (33, 200, 8, 0), (33, 200, 3, 0),
                                                 (40, 64, 0, 1), (3001, 24, 0, 0), (2, 9000, 0, 0)])
def test_dropout(x_type, y_type, with_residual, rows, cols, gap, offset):
    gen = torch.Generator().manual_seed(rows * 7 + cols)
    x, _ = matrix(rows, cols, gap, TYPES[x_type], gen, offset)
    y, memory = matrix(rows, cols, gap, TYPES[y_type], gen, offset)
    r = matrix(rows, cols, gap, TYPES[y_type], gen, offset)[0] if with_residual else None
    before = memory.clone()
    for p, seed, counter in [(0.1, 0x123456789ABCDEF0, 0xFEDCBA9876543210), (0.5, -1, 1), (0.0, 3, 0), (1.0, 5, 2 ** 63)]:
        mt.mt_kernel_dropout(x, y, p, seed, counter, residual=r)
        torch.cuda.synchronize()
        check(x, y, None, p, seed, counter, None if r is None else f64(r))
    kept = torch.ones(len(memory), dtype=torch.bool)
    kept[offset:].view(rows, cols + gap)[:, :cols] = False
    assert torch.equal(memory.cpu()[kept], before.cpu()[kept])


def test_mask_of_a_bulk_batch():
    """More groups than one round of the grid takes; every element's mask."""
    rows, cols = 9001, 776
    x, y = torch.ones(rows, cols, device="cuda"), torch.empty(rows, cols, device="cuda")
    mt.mt_kernel_dropout(x, y, 0.3, 77, 99)
    assert np.array_equal((y != 0).cpu().numpy(), orc.dropout_keep(rows, cols, 0.3, 77, 99))


@pytest.mark.parametrize("over", ["x", "residual"])
def test_in_place(over):
    gen = torch.Generator().manual_seed(0)
    x, r = (matrix(65, 96, 0, torch.float32, gen)[0] for _ in range(2))
    old_x, old_r = f64(x), f64(r)
    y = x if over == "x" else r
    mt.mt_kernel_dropout(x, y, 0.2, 5, 6, residual=r)
    check(x, y, old_x, 0.2, 5, 6, old_r)


def test_gradient_is_the_same_mask():
    """Of sum(dy * y): the formula's, and the difference quotient of the call itself (the map is linear in x)."""
    x, dy = torch.randn(50, 104, device="cuda"), torch.randn(50, 104, device="cuda")
    y0, y1, dx = (torch.empty_like(x) for _ in range(3))
    mt.mt_kernel_dropout(dy, dx, 0.1, 8, 9)
    step = torch.randn_like(x)
    mt.mt_kernel_dropout(x, y0, 0.1, 8, 9)
    mt.mt_kernel_dropout(x + step, y1, 0.1, 8, 9)
    quotient = ((y1.double() - y0.double()) * dy.double()).sum()
    # every term is off by some roundings of numbers of size |x| + |step|
    bound = 2.0 ** -22 * float(((x.abs() + step.abs()) * dy.abs()).double().sum()) / 0.9
    assert abs(float(quotient - (dx.double() * step.double()).sum())) <= bound


def test_dropped_places_may_hold_anything():
    keep = orc.dropout_keep(64, 72, 0.4, 1, 2)
    x = torch.where(torch.from_numpy(keep), 1.0, float("nan")).cuda()
    x[0, :] = torch.where(torch.from_numpy(keep[0]).cuda(), x[0, :], float("inf"))
    y = torch.empty_like(x)
    mt.mt_kernel_dropout(x, y, 0.4, 1, 2)
    assert torch.isfinite(y).all() and np.array_equal((y != 0).cpu().numpy(), keep)
    mt.mt_kernel_dropout(torch.full_like(x, float("nan")), y, 1.0, 1, 2)
    assert torch.equal(y, torch.zeros_like(y))


def test_replayed_graph_draws_anew():
    x, y, number = torch.ones(31, 64, device="cuda"), torch.empty(31, 64, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mt.mt_kernel_dropout(x, y, 0.5, 21, 2 ** 64 - 2, counter_dev=number)
        number += 1
    for turn in range(4):                             # (the sum of the two counters wraps around on the way)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal((y != 0).cpu().numpy(), orc.dropout_keep(31, 64, 0.5, 21, 2 ** 64 - 2 + turn))


def test_rows_behind_32_bits():
    """More than 2^32 elements, and more than 2^31 bytes between the first row and the last."""
    rows, cols = 4_200_000, 1032
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    mt.mt_kernel_dropout(x, x, 0.1, 4, 5)
    words = np.arange(cols) // 8
    last = orc.philox4x32((words, np.full(cols, rows - 1), np.full(cols, 5), np.zeros(cols)), (4, 0))
    word = np.select([np.arange(cols) % 8 // 2 == i for i in range(4)], last)
    draw = np.where(np.arange(cols) % 2 == 1, word >> np.uint64(16), word & np.uint64(0xFFFF))
    assert np.array_equal((x[-1] != 0).cpu().numpy(), draw >= orc.dropout_threshold(0.1))


def test_binding_refusals():
    x, y = torch.zeros(4, 16, device="cuda"), torch.zeros(4, 16, device="cuda")
    bad = [dict(x=x.half()), dict(y=y[:3]), dict(p=1.5), dict(p=-0.1), dict(p=float("nan")), dict(residual=y.bfloat16()), dict(residual=y[:, :8]),
           dict(x=x.cpu()), dict(counter_dev=torch.zeros(1, dtype=torch.int32, device="cuda")), dict(x=torch.zeros(16, 4, device="cuda").T)]
    for change in bad:
        with pytest.raises(mt.MTError):
            mt.mt_kernel_dropout(**({"x": x, "y": y, "p": 0.1, "seed": 1} | change))
    mt.mt_kernel_dropout(x[:0], y[:0], 0.1, 1)        # nothing to do
