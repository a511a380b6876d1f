"""What the speed of the vocabulary operators is measured on: embedding lookup and its gradient, dropout whose mask is never
stored, and softmax cross entropy over the vocabulary with its gradient.

They are the two ends of a language model over the vocabulary, and what lies between its layers while it is trained: the
students that this library serves are fine-tuned with them, and a text is scored by its tokens' probabilities.  ``prepare``
makes what a training step has in hand, ``run`` is one call: with ``own`` false in elementary torch operations, with ``own``
true through the library's entry points.
"""
import math

import numpy as np
import torch

own = False

BF16, F32 = "bfloat16", "float32"
VOCAB = 30522          # the uncased vocabulary of the configurations of this package
MASK_ID = 103          # the token that stands in the masked places of such a vocabulary


def listed():
    cases = {
        # lookup of one query: launch latency
        "lookup_1x128": dict(op="lookup", tokens=128, vocab=VOCAB, hidden=768, table=BF16, out=BF16, absent=0.0, scale=1.0),
        # lookup of a bulk batch of long padded sequences from fp32 master weights, scaled by the root of the width
        "lookup_256x509": dict(op="lookup", tokens=256 * 509, vocab=VOCAB, hidden=1024, table=F32, out=BF16, absent=0.2, scale=32.0),
        # gradient of a handful of tokens into a small table
        "lookup_grad_101": dict(op="lookup_grad", tokens=101, vocab=2000, hidden=1024, grad=BF16, out=F32, absent=0.0, scale=1.0),
        # the headline batch, padded (lengths 16 to 128 of 128): most rows of the table get no gradient
        "lookup_grad_32x128": dict(op="lookup_grad", tokens=32 * 128, vocab=VOCAB, hidden=768, grad=BF16, out=BF16, absent=0.44, scale=1.0),
        # bulk batch of pre-training: an eighth of the tokens are the same one
        "lookup_grad_256x512": dict(op="lookup_grad", tokens=256 * 512, vocab=VOCAB, hidden=1024, grad=BF16, out=F32, absent=0.0, scale=32.0),
        # dropout of one short query's hidden state
        "dropout_101x768": dict(op="dropout", rows=101, cols=768, x=BF16, y=BF16, residual=False, p=0.1, gap=0),
        # dropout before the residual addition of a bulk batch: bf16 projection onto the fp32 residual stream
        "dropout_32768x1024": dict(op="dropout", rows=32768, cols=1024, x=BF16, y=F32, residual=True, p=0.1, gap=0),
        # scoring of one query's masked tokens: the table is read once for 20 rows
        "loss_20": dict(op="loss", rows=20, vocab=VOCAB, hidden=768, bias=True, ignored=0.0, gap=0),
        # scoring of every token of a bulk batch
        "loss_8192": dict(op="loss", rows=8192, vocab=VOCAB, hidden=1024, bias=True, ignored=0.0, gap=0),
        # a small training step on masked tokens that were gathered before
        "loss_grad_77": dict(op="loss_grad", rows=77, vocab=VOCAB, hidden=768, bias=True, ignored=0.0, gap=0),
        # a training step on a batch in place: 15 % of the tokens have a label
        "loss_grad_4096_masked": dict(op="loss_grad", rows=4096, vocab=VOCAB, hidden=768, bias=True, ignored=0.85, gap=0),
        # every token of a bulk batch has a label
        "loss_grad_8192": dict(op="loss_grad", rows=8192, vocab=VOCAB, hidden=1024, bias=False, ignored=0.0, gap=0),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["lookup", "lookup_grad", "dropout", "loss", "loss_grad", "loss_grad"])
    kind = lambda: rng.choice([BF16, F32])  # noqa: E731
    hidden = rng.choice([768, 1024, 8 * rng.randint(8, 128)])
    if op in ("lookup", "lookup_grad"):
        case = dict(op=op, tokens=_log(rng, 1, 130000), vocab=_log(rng, 50, 130000), hidden=hidden,
                    absent=rng.choice([0.0, rng.uniform(0.0, 0.6)]), scale=rng.choice([1.0, math.sqrt(hidden)]))
        return case | (dict(table=kind(), out=kind()) if op == "lookup" else dict(grad=kind(), out=kind()))
    if op == "dropout":
        return dict(op=op, rows=_log(rng, 1, 32768), cols=rng.choice([768, 1024, rng.randint(1, 1024)]), x=kind(), y=kind(),
                    residual=rng.random() < 0.5, p=rng.choice([0.1, 0.1, rng.uniform(0.0, 0.9)]), gap=rng.choice([0, 0, rng.randint(1, 64)]))
    vocab = rng.choice([VOCAB, _log(rng, 50, 130000)])
    rows = _log(rng, 1, min(8192, 8192 * 1024 * VOCAB // (hidden * vocab)))
    return dict(op=op, rows=rows, vocab=vocab, hidden=hidden, bias=rng.random() < 0.5,
                ignored=rng.choice([0.0, 0.85, rng.uniform(0.0, 1.0)]), gap=rng.choice([0, 0, 8 * rng.randint(1, 8)]))


def _type(name):
    return torch.bfloat16 if name == BF16 else torch.float32


def _rows(shape, gap, dtype, gen, std=1.0):
    """A matrix whose rows may lie further apart than they are long."""
    full = torch.randn(shape[0], shape[1] + gap, device="cuda", generator=gen) * std
    return full.to(dtype)[:, :shape[1]]


def _tokens(n, vocab, absent, gen):
    """Token ids as text has them: log-uniform over the vocabulary, an eighth the same token, -1 where a padded batch has none."""
    ids = torch.exp(torch.rand(n, device="cuda", generator=gen, dtype=torch.float64) * math.log(vocab + 1.0)).long() - 1
    ids = ids.clamp(0, vocab - 1)
    if vocab > MASK_ID:
        ids = torch.where(torch.rand(n, device="cuda", generator=gen) < 0.12, MASK_ID, ids)
    return torch.where(torch.rand(n, device="cuda", generator=gen) < absent, -1, ids).int()


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    s, op = dict(case), case["op"]
    if op in ("lookup", "lookup_grad"):
        s["ids"] = _tokens(case["tokens"], case["vocab"], case["absent"], gen)
    if op == "lookup":
        s["weights"] = _rows((case["vocab"], case["hidden"]), 0, _type(case["table"]), gen, 0.02)
        s["result"] = torch.empty(case["tokens"], case["hidden"], dtype=_type(case["out"]), device="cuda")
    elif op == "lookup_grad":
        s["dy"] = _rows((case["tokens"], case["hidden"]), 0, _type(case["grad"]), gen, 1e-3)
        s["result"] = torch.empty(case["vocab"], case["hidden"], dtype=_type(case["out"]), device="cuda")
    elif op == "dropout":
        s["in"] = _rows((case["rows"], case["cols"]), case["gap"], _type(case["x"]), gen)
        s["rest"] = _rows((case["rows"], case["cols"]), case["gap"], _type(case["y"]), gen) if case["residual"] else None
        s["seed"], s["counter"] = (int(v) for v in torch.randint(0, 1 << 62, (2,), device="cuda", generator=gen).tolist())
        s["result"] = torch.empty(case["rows"], case["cols"], dtype=_type(case["y"]), device="cuda")
    else:
        n, vocab, hidden = case["rows"], case["vocab"], case["hidden"]
        s["w"] = _rows((vocab, hidden), case["gap"], torch.bfloat16, gen, 1.5 / math.sqrt(hidden))
        s["b"] = (torch.randn(vocab, device="cuda", generator=gen) * 0.1).bfloat16() if case["bias"] else None
        labels = _tokens(n, vocab, 0.0, gen)
        # hidden states of a model that has learned something: towards their labels' rows
        x = _rows((n, hidden), case["gap"], torch.float32, gen)
        s["x"] = torch.zeros(n, hidden + case["gap"], dtype=torch.bfloat16, device="cuda")[:, :hidden]
        s["x"].copy_(x + 4.0 * torch.rand(n, 1, device="cuda", generator=gen) * s["w"][labels.long()].float())
        at = torch.randperm(n, device="cuda", generator=gen)[:round(case["ignored"] * n)]
        labels[at] = -1
        s["labels"] = labels
        if op == "loss":
            s["result"] = (torch.empty(n, device="cuda"), torch.empty(n, device="cuda"))
        else:
            # the loss is a mean over the rows with a label, each with a weight of its own
            s["dloss"] = (0.5 + torch.rand(n, device="cuda", generator=gen)) / max(1, int((labels >= 0).sum()))
            s["lse"] = torch.empty(n, device="cuda")
            for i in range(0, n, 2048):       # what the forward pass left for the backward pass
                z = s["x"][i:i + 2048].float() @ s["w"].float().T
                s["lse"][i:i + 2048] = torch.logsumexp(z if s["b"] is None else z + s["b"].float(), 1)
            s["lse"][labels < 0] = 0.0
            s["result"] = (torch.empty(n, hidden, dtype=torch.bfloat16, device="cuda"),
                           torch.empty(vocab, hidden, dtype=torch.bfloat16, device="cuda"),
                           torch.empty(vocab, device="cuda") if case["bias"] else None)
    return s


def _lookup(s):
    ids = s["ids"].long()
    rows = s["weights"][ids.clamp(min=0)].float() * s["scale"]
    return torch.where((ids >= 0)[:, None], rows, 0.0).to(_type(s["out"]))


def _lookup_grad(s):
    ids = s["ids"].long()
    rows = torch.where((ids >= 0)[:, None], s["dy"].float(), 0.0)
    total = torch.zeros(s["vocab"], s["hidden"], device="cuda").index_add_(0, ids.clamp(min=0), rows)
    return (total * s["scale"]).to(_type(s["out"]))


def _multiply_wide(a, b):
    """High and low 32 bits of the products of 32-bit numbers held in 64-bit integers: b in two halves of 16 bits."""
    low, high = a * (b & 0xFFFF), a * (b >> 16)
    mid = (low >> 16) + high
    return mid >> 16, ((mid & 0xFFFF) << 16) | (low & 0xFFFF)


def _keep(rows, cols, p, seed, counter):
    """Which elements stay: 16 bits of Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011) each, eight elements of a row to a block."""
    groups = -(-cols // 8)
    c0 = torch.arange(groups, device="cuda").expand(rows, groups)
    c1 = torch.arange(rows, device="cuda")[:, None].expand(rows, groups)
    c2, c3 = (torch.full((1, 1), v, device="cuda") for v in (counter & 0xFFFFFFFF, counter >> 32))
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        high0, low0 = _multiply_wide(c0, 0xD2511F53)
        high1, low1 = _multiply_wide(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = high1 ^ c1 ^ k0, low1, high0 ^ c3 ^ k1, low0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack([c0, c1, c2, c3], -1)
    bits = torch.stack([words & 0xFFFF, words >> 16], -1).reshape(rows, groups * 8)[:, :cols]
    return bits >= round(p * 65536)


def _dropout(s):
    kept = _keep(s["rows"], s["cols"], s["p"], s["seed"], s["counter"])
    y = torch.where(kept, s["in"].float() * (65536.0 / (65536 - round(s["p"] * 65536))), 0.0)
    return (y if s["rest"] is None else y + s["rest"].float()).to(_type(s["y"]))


def _logits(s):
    z = s["x"].float() @ s["w"].float().T
    return z if s["b"] is None else z + s["b"].float()


def _loss(s):
    z, labels = _logits(s), s["labels"].long()
    top = z.max(1, keepdim=True).values
    lse = torch.exp(z - top).sum(1).log() + top[:, 0]
    loss = lse - z.gather(1, labels.clamp(min=0)[:, None])[:, 0]
    return torch.where(labels >= 0, loss, 0.0), torch.where(labels >= 0, lse, 0.0)


def _loss_grad(s):
    labels = s["labels"].long()
    g = torch.exp(_logits(s) - s["lse"][:, None])
    at = labels.clamp(min=0)[:, None]
    g.scatter_(1, at, g.gather(1, at) - 1.0)
    g = torch.where((labels >= 0)[:, None], g * s["dloss"][:, None], 0.0)
    x = torch.where((labels >= 0)[:, None], s["x"].float(), 0.0)
    return (g @ s["w"].float()).bfloat16(), (g.T @ x).bfloat16(), None if s["b"] is None else g.sum(0)


def _workspace(s, size):
    """The scratch memory that a program keeps for a call of these sizes."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _own(s):
    from paper_2107_05377_b200 import binding as mt
    op, result = s["op"], s["result"]
    if op == "lookup":
        mt.mt_kernel_embedding_lookup(s["ids"], s["weights"], result, s["scale"])
    elif op == "lookup_grad":
        ws = s.get("workspace")
        if ws is None:
            ws = _workspace(s, mt.mt_kernel_embedding_grad_workspace(s["tokens"], s["vocab"], s["hidden"]))
        mt.mt_kernel_embedding_grad(s["ids"], s["dy"], result, ws, s["scale"])
    elif op == "dropout":
        mt.mt_kernel_dropout(s["in"], result, s["p"], s["seed"], s["counter"], residual=s["rest"])
    elif op == "loss":
        ws = s.get("workspace")
        if ws is None:
            ws = _workspace(s, mt.mt_kernel_vocab_loss_workspace(s["rows"], s["vocab"], s["hidden"]))
        mt.mt_kernel_vocab_loss(s["x"], s["w"], s["b"], s["labels"], result[0], result[1], ws)
    else:
        ws = s.get("workspace")
        if ws is None:
            ws = _workspace(s, mt.mt_kernel_vocab_loss_grad_workspace(s["rows"], s["vocab"], s["hidden"]))
        mt.mt_kernel_vocab_loss_grad(s["x"], s["w"], s["b"], s["labels"], s["lse"], s["dloss"], *result, ws)
    return result


def run(state):
    if own:
        return _own(state)
    return {"lookup": _lookup, "lookup_grad": _lookup_grad, "dropout": _dropout, "loss": _loss, "loss_grad": _loss_grad}[state["op"]](state)


def work(case):
    size = lambda name: 2 if case[name] == BF16 else 4  # noqa: E731
    op = case["op"]
    if op == "lookup":
        n = case["tokens"]
        touched = min(case["vocab"], n)    # table rows that can be read
        return {"bytes": 4 * n + touched * case["hidden"] * size("table") + n * case["hidden"] * size("out"), "flops": n * case["hidden"]}
    if op == "lookup_grad":
        n = round(case["tokens"] * (1.0 - case["absent"]))
        return {"bytes": 4 * case["tokens"] + n * case["hidden"] * size("grad") + case["vocab"] * case["hidden"] * size("out"),
                "flops": n * case["hidden"]}
    if op == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (size("x") + size("y") * (2 if case["residual"] else 1)), "flops": 2 * n}
    n, vocab, hidden = case["rows"] - round(case["ignored"] * case["rows"]), case["vocab"], case["hidden"]
    read = 2 * hidden * (n + vocab) + 4 * case["rows"] + (2 * vocab if case["bias"] else 0)
    if op == "loss":
        return {"bytes": read + 8 * case["rows"], "flops": 2 * n * vocab * hidden}
    wrote = 2 * hidden * (case["rows"] + vocab) + (4 * vocab if case["bias"] else 0)
    return {"bytes": read + 8 * case["rows"] + wrote, "flops": 6 * n * vocab * hidden}


def _exact_kept(case, seed, counter):
    """The generator once more, in numpy's unsigned 64-bit integers."""
    rows, cols, mask = case["rows"], case["cols"], np.uint64(0xFFFFFFFF)
    groups = (cols + 7) // 8
    shift = np.uint64(32)
    index = np.arange(rows * groups, dtype=np.uint64)
    word = [index % np.uint64(groups), index // np.uint64(groups), np.full_like(index, counter & 0xFFFFFFFF), np.full_like(index, counter >> 32)]
    for turn in range(10):
        key = [np.uint64((part + turn * step) & 0xFFFFFFFF) for part, step in ((seed & 0xFFFFFFFF, 0x9E3779B9), (seed >> 32, 0xBB67AE85))]
        first, second = word[0] * np.uint64(0xD2511F53), word[2] * np.uint64(0xCD9E8D57)
        word = [(second >> shift) ^ word[1] ^ key[0], second & mask, (first >> shift) ^ word[3] ^ key[1], first & mask]
    block = np.stack(word, 1).astype("<u4").view("<u2").reshape(rows, groups * 8)[:, :cols]
    return torch.from_numpy(block.astype(np.int64) >= int(round(case["p"] * 65536))).cuda()


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "lookup":
        padded = torch.cat([s["weights"].double() * case["scale"], torch.zeros(1, case["hidden"], dtype=torch.float64, device="cuda")])
        return padded[s["ids"].long()]          # (id -1: the row of zeros at the end)
    if op == "lookup_grad":
        total = torch.zeros(case["vocab"], case["hidden"], dtype=torch.float64, device="cuda")
        there = s["ids"] >= 0
        total.index_put_((s["ids"][there].long(),), s["dy"][there].double() * case["scale"], accumulate=True)
        return total
    if op == "dropout":
        t = int(round(case["p"] * 65536))
        y = s["in"].double() * _exact_kept(case, s["seed"], s["counter"]).double() / (1.0 - t / 65536.0)
        return y if s["rest"] is None else s["rest"].double() + y
    w = s["w"].double()
    b = torch.zeros(case["vocab"], dtype=torch.float64, device="cuda") if s["b"] is None else s["b"].double()
    with_label = torch.nonzero(s["labels"] >= 0)[:, 0]
    loss, lse = (torch.zeros(case["rows"], dtype=torch.float64, device="cuda") for _ in range(2))
    dx = torch.zeros(case["rows"], case["hidden"], dtype=torch.float64, device="cuda")
    dw, db = torch.zeros_like(w), torch.zeros_like(b)
    for at in with_label.split(1024):
        x, label = s["x"][at].double(), s["labels"][at].long()
        z = torch.addmm(b, x, w.T)
        if op == "loss":
            lse[at] = torch.logsumexp(z, 1)
            loss[at] = lse[at] - z[torch.arange(len(at), device="cuda"), label]
            continue
        # (the forward's result is an input here, in 32 bits)
        g = (z - s["lse"][at].double()[:, None]).exp_()
        g[torch.arange(len(at), device="cuda"), label] -= 1.0
        g *= s["dloss"][at].double()[:, None]
        dx[at] = g @ w
        dw.addmm_(g.T, x)
        db += g.sum(0)
    return (loss, lse) if op == "loss" else (dx, dw, None if s["b"] is None else db)
