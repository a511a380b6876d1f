"""Pins of the 64-bit definitions of the vocabulary operators: known answers of the generator, closed forms, differences."""
import numpy as np
import pytest

from oracle import vocab_oracle as orc


@pytest.mark.parametrize("counter,key,want", [
    # the known answers that are published with the generator: zeros, ones, digits of pi
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator_known_answers(counter, key, want):
    got = orc.philox4x32([np.array([w], dtype=np.uint64) for w in counter], key)
    assert tuple(int(w[0]) for w in got) == want


def test_mask_is_the_half_words_in_order():
    words = orc.philox4x32([np.array([w], dtype=np.uint64) for w in (2, 5, 7, 9)], (3, 4))
    draws = [(int(w[0]) >> shift) & 0xFFFF for w in words for shift in (0, 16)]
    for p in (0.0, 0.25, 0.5, 1.0):
        keep = orc.dropout_keep(6, 24, p, seed=3 | 4 << 32, counter=7 | 9 << 32)
        assert keep[5, 16:24].tolist() == [d >= p * 65536 for d in draws]


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9])
def test_mask_keeps_its_share_and_rows_differ(p):
    keep = orc.dropout_keep(512, 512, p, seed=11, counter=13)
    q = orc.dropout_threshold(p) / 65536.0
    assert abs(keep.mean() - (1 - q)) <= 6 * np.sqrt(q * (1 - q) / keep.size)      # six standard deviations
    if 0 < p < 1:
        assert not np.array_equal(keep[0], keep[1])
        assert not np.array_equal(keep, orc.dropout_keep(512, 512, p, seed=11, counter=14))
        assert not np.array_equal(keep, orc.dropout_keep(512, 512, p, seed=12, counter=13))
        assert np.array_equal(keep[:100, :77], orc.dropout_keep(100, 77, p, seed=11, counter=13))


def test_dropout_forms():
    x, r = np.ones((4, 9)), np.full((4, 9), 5.0)
    assert np.array_equal(orc.dropout(x, 0.0, 1, 2), x)
    assert np.array_equal(orc.dropout(x * np.inf, 1.0, 1, 2, r), r)
    keep = orc.dropout_keep(4, 9, 0.5, 1, 2)
    assert np.array_equal(orc.dropout(x, 0.5, 1, 2, r), np.where(keep, 7.0, 5.0))


def test_lookup_and_its_gradient_are_adjoint():
    rng = np.random.default_rng(0)
    ids = np.array([3, -1, 0, 3, 9, 5, 3])
    table, dy = rng.standard_normal((6, 4)), rng.standard_normal((7, 4))
    out = orc.embedding_lookup(ids, table, 2.0)
    assert np.array_equal(out[1], np.zeros(4)) and np.array_equal(out[4], np.zeros(4)) and np.array_equal(out[3], 2.0 * table[3])
    grad, size, count = orc.embedding_grad(ids, dy, 6, 2.0)
    assert np.isclose((out * dy).sum(), (table * grad).sum())
    assert count.tolist() == [1, 0, 0, 3, 0, 1] and (size >= np.abs(grad) - 1e-12).all()
    assert np.array_equal(orc.embedding_grad(ids, dy, 6, 2.0, padding_id=3)[0][3], np.zeros(4))


def test_loss_closed_forms():
    x, w = np.zeros((2, 3)), np.ones((5, 3))
    loss, lse = orc.vocab_loss(x, w, None, [2, -1])
    assert np.allclose(loss, [np.log(5), 0]) and np.allclose(lse, [np.log(5), 0])
    bias = np.array([0, -np.inf, -np.inf, 0, -np.inf])           # all but two words are banned
    loss, lse = orc.vocab_loss(x, w, bias, [0, 5])
    assert np.allclose(loss, [np.log(2), 0])


def test_loss_gradient_against_differences():
    rng = np.random.default_rng(1)
    x, w, b = rng.standard_normal((4, 3)), rng.standard_normal((7, 3)), rng.standard_normal(7)
    labels, weight = [2, -1, 6, 0], rng.standard_normal(4)
    total = lambda x, w, b: float(weight @ orc.vocab_loss(x, w, b, labels)[0])  # noqa: E731
    grads = orc.vocab_loss_grad(x, w, b, labels, weight)
    h = 1e-5
    for k, array in enumerate((x, w, b)):
        for at in np.ndindex(array.shape):
            moved = [array.copy(), array.copy()]
            moved[0][at] += h
            moved[1][at] -= h
            args = [[x, w, b], [x, w, b]]
            args[0][k], args[1][k] = moved
            assert abs((total(*args[0]) - total(*args[1])) / (2 * h) - grads[k][at]) < 1e-8
    assert np.allclose(grads[2].sum(), 0) and np.array_equal(grads[0][1], np.zeros(3))
