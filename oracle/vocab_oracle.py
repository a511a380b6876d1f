"""Plain definitions, in 64 bits, of the operators at the vocabulary's ends of a language model and of dropout: lookup of rows
and the gradient of the table, the counter-based generator and its mask, softmax cross entropy and its gradients.

Written from the formulas in numpy; shares no code with the package.
"""
import numpy as np

_MASK32 = 0xFFFFFFFF


def philox4x32(counter, key, rounds=10):
    """Philox4x32 of Salmon, Moraes, Dror and Shaw (SC 2011): four counter words and two key words (arrays of integers below
    2^32, of one shape) to four words."""
    c = [np.asarray(w).astype(np.uint64) for w in counter]
    k = [int(w) for w in key]
    for _ in range(rounds):
        first, second = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)      # (both below 2^64)
        c = [(second >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), second & np.uint64(_MASK32),
             (first >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), first & np.uint64(_MASK32)]
        k = [(k[0] + 0x9E3779B9) & _MASK32, (k[1] + 0xBB67AE85) & _MASK32]
    return c


def dropout_threshold(p):
    """p as a multiple of 2^-16, halves to even."""
    return int(round(p * 65536.0))


def dropout_keep(rows, cols, p, seed, counter):
    """keep(r, c): half-word c % 8 of the block of counter (c // 8, r, counter) is at least p * 2^16."""
    r, c = np.meshgrid(np.arange(rows), np.arange(cols), indexing="ij")
    counter &= (1 << 64) - 1
    words = philox4x32((c // 8, r, np.full_like(r, counter & _MASK32), np.full(r.shape, counter >> 32, np.uint64)),
                       (seed & _MASK32, (seed >> 32) & _MASK32))
    word = np.select([c % 8 // 2 == i for i in range(4)], words)
    draw = np.where(c % 2 == 1, word >> np.uint64(16), word & np.uint64(0xFFFF))
    return draw.astype(np.int64) >= dropout_threshold(p)


def dropout(x, p, seed, counter, residual=None):
    t = dropout_threshold(p)
    keep = dropout_keep(x.shape[0], x.shape[1], p, seed, counter)
    y = np.zeros(x.shape)
    if t < 65536:
        y[keep] = x[keep] / (1.0 - t / 65536.0)
    return y if residual is None else residual + y


def embedding_lookup(ids, table, scale=1.0):
    out = np.zeros((len(ids), table.shape[1]))
    for t, i in enumerate(ids):
        if 0 <= i < len(table):
            out[t] = scale * table[i]
    return out


def embedding_grad(ids, grad_out, vocab, scale=1.0, padding_id=-1):
    """The gradient, and the sum of the magnitudes and the number of terms of every row (for bounds on rounding)."""
    total, size, count = np.zeros((vocab, grad_out.shape[1])), np.zeros((vocab, grad_out.shape[1])), np.zeros(vocab, np.int64)
    for t, i in enumerate(ids):
        if 0 <= i < vocab and i != padding_id:
            total[i] += grad_out[t]
            size[i] += np.abs(grad_out[t])
            count[i] += 1
    return scale * total, abs(scale) * size, count


def _softmax_rows(x, w, bias, labels, block=512):
    """For blocks of rows with a label (0 <= label < vocab): the rows, their labels, logits and log-sum-exp."""
    labels = np.asarray(labels)
    rows = np.flatnonzero((labels >= 0) & (labels < len(w)))
    for at in (rows[i:i + block] for i in range(0, len(rows), block)):
        z = x[at] @ w.T + (0.0 if bias is None else bias)
        top = z.max(axis=1)
        yield at, labels[at], z, top + np.log(np.exp(z - top[:, None]).sum(axis=1))


def vocab_loss(x, w, bias, labels):
    """loss and log-sum-exp of every row with a label; zeros elsewhere."""
    loss, lse = np.zeros(len(x)), np.zeros(len(x))
    for at, label, z, total in _softmax_rows(x, w, bias, labels):
        lse[at] = total
        loss[at] = total - z[np.arange(len(at)), label]
    return loss, lse


def vocab_loss_grad(x, w, bias, labels, grad_loss):
    """Gradients of sum_n grad_loss[n] * loss[n] with respect to x, w and bias."""
    dx, dw, db = np.zeros(x.shape), np.zeros(w.shape), np.zeros(len(w))
    for at, label, z, total in _softmax_rows(x, w, bias, labels):
        g = np.exp(z - total[:, None])
        g[np.arange(len(at)), label] -= 1.0
        g *= grad_loss[at][:, None]
        dx[at] = g @ w
        dw += g.T @ x[at]
        db += g.sum(axis=0)
    return dx, dw, db
