"""Sizes beyond 32 bits never reach the library cut off: tensors without memory stand for those of more than 2^31 rows."""
import pytest
import torch

from paper_2107_05377_b200 import binding, build

INVALID, SHAPE = -1, -2
BIG = 2 ** 32 + 8          # whose low 32 bits are 8


@pytest.fixture(autouse=True)
def on_no_device(monkeypatch):
    build.build()
    monkeypatch.setattr(binding, "_torch", binding._Torch())
    monkeypatch.setattr(binding, "_begin", lambda where, stream: (binding._torch, -1, 0))


def new(*shape, dtype=torch.bfloat16):
    t = torch.empty(*shape, dtype=dtype, device="meta")
    assert t.get_device() == -1
    return t


def refused(code, call, *args, match=None, **named):
    with pytest.raises(binding.MTError, match=match) as e:
        call(*args, **named)
    assert e.value.code == code


def test_rows_and_columns():
    small, ws, ids = new(8, 1), new(1 << 20, dtype=torch.uint8), new(8, dtype=torch.int32)
    many = new(BIG, dtype=torch.int32)
    for long in (BIG, 2 ** 31):
        refused(SHAPE, binding.mt_kernel_dropout, new(long, 1), new(long, 1), 0.1, 1)
        refused(SHAPE, binding.mt_kernel_dropout, new(1, long), new(1, long), 0.1, 1)
        refused(SHAPE, binding.mt_kernel_embedding_lookup, ids, new(long, 1), small)
        refused(SHAPE, binding.mt_kernel_embedding_grad, ids, small, new(long, 1), ws)
    refused(SHAPE, binding.mt_kernel_embedding_lookup, many, small, new(BIG, 1))
    refused(SHAPE, binding.mt_kernel_embedding_grad, many, new(BIG, 1), small, ws)
    one = new(8, dtype=torch.float32)
    refused(SHAPE, binding.mt_kernel_vocab_loss, new(8, 8), new(BIG, 8), None, ids, one, one, ws)
    refused(SHAPE, binding.mt_kernel_vocab_loss_grad, new(8, 8), new(BIG, 8), None, ids, one, None, new(8, 8), None, None, ws)
    refused(SHAPE, binding.mt_kernel_vocab_loss, new(BIG, 8), new(8, 8), None, many, one, one, ws)


@pytest.mark.parametrize("padding_id", [2 ** 31, 2 ** 32 + 3, -2 ** 31 - 1])
def test_padding_id(padding_id):
    refused(INVALID, binding.mt_kernel_embedding_grad, new(8, dtype=torch.int32), new(8, 8), new(8, 8), new(1 << 20, dtype=torch.uint8),
            padding_id=padding_id, match="padding_id")


@pytest.mark.parametrize("size", [binding.mt_kernel_embedding_grad_workspace, binding.mt_kernel_vocab_loss_workspace,
                                  binding.mt_kernel_vocab_loss_grad_workspace])
def test_workspaces(size):
    assert size(8, 16, 8) > 0
    for sizes in [(BIG, 16, 8), (8, BIG, 8), (8, 16, BIG), (-BIG + 16, 16, 8)]:
        assert size(*sizes) == 0
