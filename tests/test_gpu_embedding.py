"""Lookup of rows and the gradient of the table against their definitions in 64 bits: one token to tens of thousands (one CTA to a
cluster of sixteen sorts them), one row to 2^31 - 1 (one to four sort passes), widths that are no multiple of eight,
rows further apart than they are long, runs of equal ids inside a chunk, over its border and over many chunks."""
import numpy as np
import pytest
import torch

from oracle import vocab_oracle as orc
from paper_2107_05377_b200 import binding as mt

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def matrix(rows, cols, gap, dtype, gen, offset=0):
    """[rows, cols] whose rows are cols + gap apart, `offset` elements behind an allocation's start; and all of its memory."""
    full = torch.randn(offset + rows * (cols + gap), generator=gen).to(dtype).cuda()
    return full[offset:].view(rows, cols + gap)[:, :cols], full


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


@pytest.mark.parametrize("table_type", ["bf16", "f32"])
@pytest.mark.parametrize("out_type", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,hidden,gap,offset", [(1, 1, 8, 0, 0), (3, 50, 7, 0, 0), (129, 2000, 768, 0, 0), (1000, 50, 1024, 24, 0),
                                                           (65, 31, 200, 3, 0), (77, 9, 264, 0, 1), (20000, 30522, 64, 8, 0), (5, 6, 1500, 0, 0)])
def test_lookup(table_type, out_type, tokens, vocab, hidden, gap, offset):
    gen = torch.Generator().manual_seed(tokens + hidden)
    table, _ = matrix(vocab, hidden, gap, TYPES[table_type], gen, offset)
    out, memory = matrix(tokens, hidden, gap, TYPES[out_type], gen, offset)
    before = memory.clone()
    ids = torch.randint(-1, vocab + 1, (tokens,), generator=gen, dtype=torch.int32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    scale = 1.7
    mt.mt_kernel_embedding_lookup(ids.cuda(), table, out, scale, status)
    torch.cuda.synchronize()
    assert int(status) == (mt.FLAG_BAD_TOKEN if bool((ids == vocab).any()) else 0)
    want = orc.embedding_lookup(ids.numpy(), f64(table), float(np.float32(scale)))
    # one product in fp32, one rounding to the output's type
    bound = np.abs(want) * (2.0 ** -24 + HALF_STEP[out.dtype] * (1 + 2.0 ** -24))
    assert (np.abs(f64(out) - want) <= bound).all()
    kept = torch.ones(len(memory), dtype=torch.bool)
    kept[offset:].view(tokens, hidden + gap)[:, :hidden] = False          # between the rows nothing is written
    assert torch.equal(memory.cpu()[kept], before.cpu()[kept])


def grad_case(ids, vocab, hidden, grad_type, out_type, scale=1.0, padding_id=-1, accumulate=False, gap=0, offset=0, seed=0):
    gen = torch.Generator().manual_seed(seed)
    tokens = len(ids)
    dy, _ = matrix(tokens, hidden, gap, grad_type, gen, offset)
    out, memory = matrix(vocab, hidden, gap, out_type, gen, offset)
    before, old = memory.clone(), f64(out)
    away = torch.from_numpy((ids < 0) | (ids >= vocab) | ((ids == padding_id) & (padding_id >= 0)))
    if tokens:
        dy[away.cuda()] = float("nan")                # what has no part is not read
    ws = torch.full((mt.mt_kernel_embedding_grad_workspace(tokens, vocab, hidden),), 0xFF, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dev_ids = torch.from_numpy(ids.astype(np.int32)).cuda()
    mt.mt_kernel_embedding_grad(dev_ids, dy, out, ws, scale, padding_id, accumulate, status)
    torch.cuda.synchronize()
    assert int(status) == (mt.FLAG_BAD_TOKEN if (ids >= vocab).any() else 0)
    scale = float(np.float32(scale))
    values = np.nan_to_num(f64(dy))
    want, size, count = orc.embedding_grad(ids, values, vocab, scale, padding_id)
    # k terms: at most k - 1 additions whatever their order, each off by half an fp32 step of a partial sum that is at most the
    # sum of magnitudes; the scale, and what was there, one more each
    half = 2.0 ** -24
    bound = (count[:, None] + 2) * half * size * 1.01
    if accumulate:
        want = want + old
        bound = bound + half * np.abs(want)
        bound[count == 0] = 0.0
    rounded = np.abs(want) * HALF_STEP[out_type] * 1.01
    if accumulate:
        rounded[count == 0] = 0.0
    if out_type == torch.float32 and not accumulate:
        rounded[:] = 0.0                              # (the scaled sum is an fp32 number already)
    got = f64(out)
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= bound + rounded).all()
    kept = torch.ones(len(memory), dtype=torch.bool)
    kept[offset:].view(vocab, hidden + gap)[:, :hidden] = False
    assert torch.equal(memory.cpu()[kept], before.cpu()[kept])
    return out


def skewed(tokens, vocab, seed, absent=0.1, repeated=0.12):
    rng = np.random.default_rng(seed)
    ids = np.minimum(np.exp(rng.uniform(0, np.log(vocab + 1.0), tokens)).astype(np.int64) - 1, vocab - 1)
    ids[rng.uniform(size=tokens) < repeated] = vocab // 3
    ids[rng.uniform(size=tokens) < absent] = -1
    return ids


@pytest.mark.parametrize("grad_type", ["bf16", "f32"])
@pytest.mark.parametrize("out_type", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,hidden", [(1, 1, 8), (1, 1200000, 8), (2, 3, 1), (33, 7, 200), (101, 2000, 1024), (1025, 513, 72),
                                                 (2049, 30522, 64), (5000, 130001, 40), (20000, 512, 48), (40001, 300000, 24), (700, 100, 1544)])
def test_gradient(grad_type, out_type, tokens, vocab, hidden):
    grad_case(skewed(tokens, vocab, tokens), vocab, hidden, TYPES[grad_type], TYPES[out_type], scale=2.5)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("gap,offset", [(0, 0), (8, 0), (5, 0), (0, 3)])
def test_gradient_strides_padding_and_accumulation(accumulate, gap, offset):
    ids = skewed(3000, 400, 5)
    ids[::17] = 400 + np.arange(len(ids[::17]))       # outside the table: flagged, no part
    grad_case(ids, 400, 104, torch.bfloat16, torch.float32, padding_id=400 // 3, accumulate=accumulate, gap=gap, offset=offset)
    grad_case(ids, 400, 104, torch.bfloat16, torch.bfloat16, accumulate=accumulate, gap=gap, offset=offset)


@pytest.mark.parametrize("tokens", [7, 8, 9, 16, 17, 4096, 60000])
def test_gradient_of_one_id_only(tokens):
    """A run over every chunk; and one of all tokens but the first and the last."""
    grad_case(np.full(tokens, 4), 6, 64, torch.float32, torch.float32)
    ids = np.full(tokens, 4)
    ids[0], ids[-1] = 0, 5
    grad_case(ids, 6, 64, torch.bfloat16, torch.float32)


@pytest.mark.parametrize("hidden", [8, 260, 768, 1288, 2056, 2312])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_few_tokens_by_how_often_an_id_comes(hidden, accumulate):
    """Ids that come once, twice ... ten times, a hundred and some hundred times among each other: rows of one block of columns to more
    than a CTA has warps."""
    ids = np.concatenate([np.full(k, 3 * k) for k in range(1, 11)] + [np.full(100, 40), np.full(513, 41), np.full(100, -1)])
    ids = np.random.default_rng(hidden).permutation(ids)
    grad_case(ids, 45, hidden, torch.bfloat16, torch.float32, accumulate=accumulate, scale=0.5)
    grad_case(ids, 45, hidden, torch.float32, torch.bfloat16, accumulate=accumulate, padding_id=41)


@pytest.mark.parametrize("ids", [np.full(300, -1), np.full(300, 9), np.zeros(0, np.int64)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_without_tokens(ids, accumulate):
    grad_case(ids, 9, 72, torch.bfloat16, torch.float32, accumulate=accumulate)


def test_equal_calls_give_equal_bits_on_any_stream_and_replayed():
    tokens, vocab, hidden = 30000, 30522, 128
    ids = torch.from_numpy(skewed(tokens, vocab, 3).astype(np.int32)).cuda()
    dy = torch.randn(tokens, hidden, device="cuda").bfloat16()
    outs, streams = [], [torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for s in streams:                                 # at the same time, each with a workspace of its own
        with torch.cuda.stream(s):
            ws = torch.empty(mt.mt_kernel_embedding_grad_workspace(tokens, vocab, hidden), dtype=torch.uint8, device="cuda")
            out = torch.full((vocab, hidden), float("nan"), device="cuda")
            mt.mt_kernel_embedding_grad(ids, dy, out, ws, stream=s)
            outs.append((out, ws))
    torch.cuda.synchronize()
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][0], outs[2][0])
    graph, out, ws = torch.cuda.CUDAGraph(), torch.empty_like(outs[0][0]), outs[0][1]
    looked = torch.empty(tokens, hidden, device="cuda")
    with torch.cuda.graph(graph):
        mt.mt_kernel_embedding_grad(ids, dy, out, ws)
        mt.mt_kernel_embedding_lookup(ids, out, looked)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, outs[0][0])
    ids.copy_(torch.from_numpy(skewed(tokens, vocab, 4, absent=0.4).astype(np.int32)))
    graph.replay()
    want = torch.empty_like(out)
    mt.mt_kernel_embedding_grad(ids, dy, want, outs[1][1])
    torch.cuda.synchronize()
    assert torch.equal(out, want) and not torch.equal(out, outs[0][0])
    assert torch.equal(looked, torch.where((ids >= 0)[:, None], want[ids.clamp(min=0).long()], 0.0))


def test_lookup_behind_32_bits():
    """Offsets of more than 2^32 elements: a table of 4.4 billion."""
    vocab, hidden = 4_300_000, 1024
    table = torch.empty(vocab, hidden, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([vocab - 1, 4_200_000, 5], dtype=torch.int32, device="cuda")
    for k, i in enumerate(ids.tolist()):
        table[i] = k + 1.0
    out = torch.empty(3, hidden, device="cuda")
    mt.mt_kernel_embedding_lookup(ids, table, out)
    assert torch.equal(out, torch.arange(1.0, 4.0, device="cuda")[:, None].expand(3, hidden))
    ws = torch.empty(mt.mt_kernel_embedding_grad_workspace(3, vocab, hidden), dtype=torch.uint8, device="cuda")
    mt.mt_kernel_embedding_grad(ids, out, table, ws, accumulate=True)
    for k, i in enumerate(ids.tolist()):
        assert torch.equal(table[i].float(), torch.full((hidden,), 2.0 * (k + 1), device="cuda"))


def test_binding_refusals():
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    table, out = torch.zeros(5, 16, device="cuda"), torch.zeros(4, 16, device="cuda")
    ws = torch.empty(mt.mt_kernel_embedding_grad_workspace(4, 5, 16), dtype=torch.uint8, device="cuda")
    for args in [(ids.long(), table, out), (ids, table.half(), out), (ids, table, out[:3]), (ids, table.cpu(), out),
                 (ids, table, torch.zeros(16, 4, device="cuda").T), (ids, table, out[:, :8])]:
        with pytest.raises(mt.MTError):
            mt.mt_kernel_embedding_lookup(*args)
    for args in [(ids, out, table, ws[:-256]), (ids, out[:, :8], table, ws), (ids, out, table, ws[1:]), (ids.cpu(), out, table, ws)]:
        with pytest.raises(mt.MTError):
            mt.mt_kernel_embedding_grad(*args)


def test_zeros_of_a_table_of_nearly_as_many_rows_as_there_are_ids():
    """Rows counted beyond 32 bits: the step behind the last row of a table of 2^31 - 1 must not come back in front of it."""
    vocab, guard = 2 ** 31 - 1, 1 << 20
    memory = torch.ones(guard + vocab, dtype=torch.bfloat16, device="cuda")
    table = memory[guard:].view(vocab, 1)
    ids = torch.arange(0, 1500, dtype=torch.int64) * 1_400_000
    ids[-3:] = torch.tensor([vocab - 1, vocab - 2, vocab - 4673])
    dy = (1.0 + torch.arange(1500) % 7).bfloat16().cuda()
    ws = torch.empty(mt.mt_kernel_embedding_grad_workspace(1500, vocab, 1), dtype=torch.uint8, device="cuda")
    mt.mt_kernel_embedding_grad(ids.int().cuda(), dy.view(1500, 1), table, ws)
    torch.cuda.synchronize()
    assert bool((memory[:guard] == 1.0).all())
    assert torch.equal(table[ids.cuda(), 0], dy) and int(torch.count_nonzero(table)) == 1500


@pytest.mark.parametrize("tokens,vocab", [(140001, 70000), (300000, 513)])
def test_gradient_of_lists_that_no_warp_holds(tokens, vocab):
    """More than 131072 tokens: a warp of the sort has more of them than its registers hold from the count to their places."""
    grad_case(skewed(tokens, vocab, tokens), vocab, 8, torch.float32, torch.float32)
    grad_case(np.full(tokens, 4), 6, 8, torch.bfloat16, torch.float32)


@pytest.mark.parametrize("tokens", [1025, 1500, 2048, 2049, 30000])
@pytest.mark.parametrize("vocab", [300_000, 2 ** 27 + 5])
@pytest.mark.parametrize("accumulate", [False, True])
def test_sort_in_three_and_four_passes(tokens, vocab, accumulate):
    """Up to 2048 tokens one CTA sorts in place, in shared memory; beyond, a cluster from one list to the other."""
    rng = np.random.default_rng(tokens)
    named = rng.integers(0, vocab, 200)
    ids = np.where(rng.uniform(size=tokens) < 0.5, rng.integers(0, vocab, tokens), named[rng.integers(0, 200, tokens)])
    ids[::50], ids[1::50] = -1, vocab - 1
    dy = torch.from_numpy(rng.integers(-8, 9, tokens)).float().cuda()            # (sums of small integers: exact in any order)
    table = torch.full((vocab, 1), 0.5, device="cuda")
    ws = torch.full((mt.mt_kernel_embedding_grad_workspace(tokens, vocab, 1),), 0xFF, dtype=torch.uint8, device="cuda")
    mt.mt_kernel_embedding_grad(torch.from_numpy(ids.astype(np.int32)).cuda(), dy.view(-1, 1), table, ws, accumulate=accumulate)
    torch.cuda.synchronize()
    there = torch.from_numpy(ids >= 0).cuda()
    want = torch.full((vocab,), 0.5 if accumulate else 0.0, dtype=torch.float64, device="cuda")
    want.index_add_(0, torch.from_numpy(ids).cuda()[there], dy.double()[there])
    assert torch.equal(table[:, 0].double(), want)
