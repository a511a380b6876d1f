"""Refusals of the vocabulary operators and of dropout that need no GPU: every check comes before the first CUDA call."""
import pytest

from paper_2107_05377_b200 import binding, build

INVALID, SHAPE, CUDA, UNSUPPORTED = -1, -2, -6, -7
A = 1 << 20            # stands for a device address; nothing reads it


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


LOOKUP = dict(ids=A, table=A, out=A, tokens=4, vocab=9, hidden=16, table_stride=16, out_stride=16, table_dtype=0, out_dtype=1, scale=1.0,
              status=0, stream=0)
GRAD = dict(ids=A, grad=A, table=A, tokens=4, vocab=9, hidden=16, grad_stride=16, table_stride=16, grad_dtype=0, table_dtype=1, scale=1.0,
            padding=-1, accumulate=0, ws=A, ws_bytes=1 << 20, status=0, stream=0)
DROPOUT = dict(x=A, residual=0, y=A, rows=4, cols=16, x_stride=16, residual_stride=0, y_stride=16, x_dtype=0, y_dtype=1, p=0.1, seed=1, counter=2,
               counter_dev=0, stream=0)


def call(lib, name, base, **change):
    return getattr(lib, name)(*(base | change).values())


@pytest.mark.parametrize("change,want", [
    (dict(table_dtype=2), UNSUPPORTED), (dict(out_dtype=-1), UNSUPPORTED), (dict(tokens=-1), SHAPE), (dict(tokens=(1 << 30) + 1), SHAPE),
    (dict(vocab=0), SHAPE), (dict(hidden=0), SHAPE), (dict(hidden=1 << 21, table_stride=1 << 21, out_stride=1 << 21), SHAPE), (dict(table_stride=15), SHAPE), (dict(out_stride=-16), SHAPE), (dict(ids=0), INVALID),
    (dict(table=0), INVALID), (dict(out=0), INVALID), (dict(ids=A + 2), INVALID), (dict(table=A + 1), INVALID), (dict(out=A + 2), INVALID),
    (dict(tokens=0, ids=0, table=0, out=0), 0)])
def test_lookup(lib, change, want):
    assert call(lib, "mt_kernel_embedding_lookup", LOOKUP, **change) == want


@pytest.mark.parametrize("change,want", [
    (dict(grad_dtype=2), UNSUPPORTED), (dict(table_dtype=7), UNSUPPORTED), (dict(tokens=-1), SHAPE), (dict(tokens=(1 << 30) + 1), SHAPE),
    (dict(vocab=-4), SHAPE), (dict(hidden=0), SHAPE), (dict(grad_stride=8), SHAPE), (dict(table_stride=8), SHAPE), (dict(ids=0), INVALID),
    (dict(grad=0), INVALID), (dict(table=0), INVALID), (dict(ws=0), INVALID), (dict(ws=A + 16), INVALID), (dict(ws_bytes=255), INVALID),
    (dict(grad=A + 1), INVALID), (dict(table=A + 2), INVALID), (dict(tokens=0, accumulate=1, ids=0, grad=0, ws=0), 0)])
def test_gradient(lib, change, want):
    assert call(lib, "mt_kernel_embedding_grad", GRAD, **change) == want


def test_gradient_workspace(lib):
    size = lib.mt_kernel_embedding_grad_workspace
    assert size(-1, 9, 16) == 0 and size(4, 0, 16) == 0 and size(4, 9, 0) == 0 and size((1 << 30) + 1, 9, 16) == 0
    assert size(0, 9, 16) >= 1
    for tokens in (1, 7, 8, 9, 4096, 131072, 1 << 30):
        chunks = size(tokens, 9, 8) - 2 * ((tokens * 8 + 255) // 256 * 256)
        assert chunks % 256 == 0 and chunks > 0
    assert size(1 << 30, 9, 1024) > 1 << 33            # (counted in 64 bits)


@pytest.mark.parametrize("change,want", [
    (dict(x_dtype=2), UNSUPPORTED), (dict(y_dtype=-3), UNSUPPORTED), (dict(p=-0.01), INVALID), (dict(p=1.01), INVALID), (dict(p=float("nan")), INVALID),
    (dict(rows=-1), SHAPE), (dict(cols=-1), SHAPE), (dict(cols=1 << 21, x_stride=1 << 21, y_stride=1 << 21), SHAPE), (dict(x_stride=15), SHAPE), (dict(y_stride=0), SHAPE), (dict(residual=A, residual_stride=4), SHAPE),
    (dict(x=0), INVALID), (dict(y=0), INVALID), (dict(x=A + 1), INVALID), (dict(y=A + 2), INVALID), (dict(residual=A + 2, residual_stride=16), INVALID),
    (dict(counter_dev=A + 4), INVALID), (dict(rows=0, x=0, y=0), 0), (dict(cols=0, x=0, y=0), 0)])
def test_dropout(lib, change, want):
    assert call(lib, "mt_kernel_dropout", DROPOUT, **change) == want


LOSS = dict(x=A, w=A, bias=A, labels=A, loss=A, lse=A, rows=4, vocab=90, hidden=64, x_stride=64, w_stride=64, ws=A, ws_bytes=1 << 24, status=0, stream=0)
LOSS_GRAD = dict(x=A, w=A, bias=A, labels=A, lse=A, grad_loss=A, dx=A, dw=A, db=A, rows=4, vocab=90, hidden=64, x_stride=64, w_stride=64,
                 dx_stride=64, dw_stride=64, accumulate=0, ws=A, ws_bytes=1 << 26, status=0, stream=0)
LOSS_SIZES = [(dict(rows=-1), SHAPE), (dict(rows=(1 << 22) + 1), SHAPE), (dict(vocab=0), SHAPE), (dict(vocab=(1 << 22) + 1), SHAPE), (dict(hidden=0), SHAPE),
              (dict(hidden=60), SHAPE), (dict(hidden=16392, x_stride=16392, w_stride=16392), SHAPE), (dict(x_stride=56), SHAPE), (dict(w_stride=68), SHAPE),
              (dict(x_stride=-64), SHAPE), (dict(x=0), INVALID), (dict(w=0), INVALID), (dict(labels=0), INVALID), (dict(lse=0), INVALID),
              (dict(x=A + 8), INVALID), (dict(w=A + 2), INVALID), (dict(bias=A + 4), INVALID), (dict(labels=A + 1), INVALID), (dict(lse=A + 2), INVALID),
              (dict(ws=0), INVALID), (dict(ws=A + 128), INVALID), (dict(ws_bytes=1000), INVALID)]


@pytest.mark.parametrize("change,want", LOSS_SIZES + [(dict(loss=0), INVALID), (dict(loss=A + 2), INVALID), (dict(rows=0, x=0, labels=0, loss=0, ws=0), 0)])
def test_loss(lib, change, want):
    assert call(lib, "mt_kernel_vocab_loss", LOSS, **change) == want


@pytest.mark.parametrize("change,want", LOSS_SIZES + [
    (dict(dx=0, dw=0, db=0), INVALID), (dict(dx_stride=60), SHAPE), (dict(dw_stride=32), SHAPE), (dict(dx=A + 8), INVALID), (dict(dw=A + 2), INVALID),
    (dict(db=A + 2), INVALID), (dict(grad_loss=A + 2), INVALID), (dict(rows=0, accumulate=1, x=0, ws=0), 0)])
def test_loss_gradient(lib, change, want):
    assert call(lib, "mt_kernel_vocab_loss_grad", LOSS_GRAD, **change) == want


def test_loss_workspaces(lib):
    for size in (lib.mt_kernel_vocab_loss_workspace, lib.mt_kernel_vocab_loss_grad_workspace):
        assert size(-1, 9, 16) == 0 and size(4, 0, 16) == 0 and size(4, 9, 12) == 0 and size(4, 9, 0) == 0
        assert 0 < size(1, 1, 8) <= size(1, 30522, 768) <= size(256, 30522, 768)
    # the logits are not kept: a fraction of their fp32 size, in bf16 pieces
    assert lib.mt_kernel_vocab_loss_grad_workspace(8192, 131072, 1024) < 8192 * 131072 * 4 / 8


@pytest.mark.parametrize("name,base", [("mt_kernel_embedding_lookup", LOOKUP), ("mt_kernel_embedding_grad", GRAD), ("mt_kernel_vocab_loss", LOSS),
                                       ("mt_kernel_vocab_loss_grad", LOSS_GRAD)])
def test_status_words_that_are_not_aligned(lib, name, base):
    for off in (1, 2, 3):
        assert call(lib, name, base, status=A + off) == INVALID
