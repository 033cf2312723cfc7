"""sr_embed_grad: no row is lost or counted twice, sums run in the order that is promised, and their chains are as short as the plan makes them.

Whole numbers.  Rows of 1 .. 15 that depend on row and column: every sum of them, in any order, is a whole number below 15 * 2^20 < 2^24, which single
precision holds, so that a row too many or too few changes every column by one at least and nothing is left to a tolerance.

Order.  The sorted list is cut into chunks, eight chunks are a span; a chunk's rows of a token are added one after the other, then the chunks of a span, then the
spans by eight runs of them, then the runs.  Evaluated so in single precision on the host, the sums agree bit for bit.

Chains.  Rows of one sign and one value that is no sum of few powers of two: an addition's rounding goes the same way again and again, and one chain over all
rows is off by far more than the bound that chunk + 8 + ceil(spans / 8) + 8 additions and 3 roundings more give, u = 2^-24 each.
"""
import ctypes

import numpy as np
import pytest
import torch

import paper_2605_05802_amd as sr
from test_decoder_rows import BF16, F16, F32, U, rng, row_plan, some_tokens  # noqa: F401  (row_plan: a fixture)


def whole_rows(n, width, dtype):
    i, c = torch.arange(n, device="cuda")[:, None], torch.arange(width, device="cuda")[None]
    return (((i * 40503 + c * 977) >> 3) % 15 + 1).to(dtype)


def workspace(n, width):
    return torch.empty(sr.embed_grad_workspace(n, width), dtype=torch.uint8, device="cuda")


def sums(d, tokens, vocab):
    t = tokens.long()
    inside = (t >= 0) & (t < vocab)
    return torch.zeros(vocab, d.shape[1], dtype=torch.int64, device="cuda").index_add_(0, t[inside], d[inside].long())


@pytest.mark.gpu
@pytest.mark.parametrize("types", [(BF16, F32), (F32, F32), (F16, F16), (BF16, BF16)])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n,width", [(700, 72), (1024, 8), (1025, 8), (4096, 260), (8192, 72), (8193, 72), (16385, 33), (20001, 1031), (65536, 5), (70001, 64), (100000, 260), (262144, 16),
                                     (1 << 20, 8)])
def test_no_row_is_lost(types, accumulate, n, width):
    T, O = types
    gen = rng(n)
    d = whole_rows(n, width, T)
    for vocab, hot, outside in ((1, 0.0, 0.0), (40, 0.5, 0.05), (40, 0.9, 0.0), (3, 0.0, 0.1), (977, 0.7, 0.0)):
        tokens = some_tokens(gen, n, vocab, hot, outside)
        table = torch.full((vocab, width), 3.0, dtype=O, device="cuda")
        sr.sr_embed_grad(d, tokens, table, workspace(n, width), accumulate=accumulate)
        want = sums(d, tokens, vocab)
        if accumulate:
            named = torch.zeros(vocab, dtype=torch.bool, device="cuda")
            named[tokens[(tokens >= 0) & (tokens < vocab)].long()] = True
            want = torch.where(named[:, None], want + 3, 3)
        # half precision ends at 65504: the rounding of a larger sum is infinity on both sides
        assert torch.equal(table, want.float().to(O))


@pytest.mark.gpu
@pytest.mark.parametrize("n", [8200, 9001, 30011])
@pytest.mark.parametrize("vocab,width", [((1 << 22) + 1, 3), ((1 << 27) - 5, 2), ((1 << 28) + 3, 2), ((1 << 31) - 1, 1)])
def test_tokens_of_vocabularies_that_take_three_passes_of_the_sort(n, vocab, width):
    """23 and 27 bits in digits of eight and nine, 29 and 31 in digits of ten and eleven.  Added to a table whose other rows stay."""
    gen = rng(n + width)
    t = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
    near = torch.tensor([0, 1, vocab - 1, vocab - 2, vocab // 2, 1 << 9, 1 << 18, (1 << 22) - 1], device="cuda")
    t = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.3, near[torch.randint(0, 8, (n,), generator=gen, device="cuda")], t)
    bad = torch.tensor([-1, min(vocab, 2 ** 31 - 1), -2 ** 31], device="cuda")[torch.randint(0, 3, (n,), generator=gen, device="cuda")]
    tokens = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.1, bad, t).int()
    d = whole_rows(n, width, BF16)
    table = torch.ones(vocab, width, dtype=BF16, device="cuda")
    sr.sr_embed_grad(d, tokens, table, workspace(n, width), accumulate=True)
    inside = (tokens >= 0) & (tokens.long() < vocab)
    rows, place = torch.unique(tokens[inside].long(), return_inverse=True)
    want = torch.ones(len(rows), width, dtype=torch.int64, device="cuda").index_add_(0, place, d[inside].long())
    assert torch.equal(table[rows], want.float().to(BF16))
    table[rows] = 1.0
    assert table.min().item() == 1.0 and table.max().item() == 1.0


def in_order(d, tokens, vocab, chunk):
    """The promised order in single precision, for rows of the tokens as numpy arrays."""
    keep = np.flatnonzero((tokens >= 0) & (tokens < vocab))
    order = keep[np.argsort(tokens[keep], kind="stable")]
    t, out = tokens[order], np.zeros((vocab, d.shape[1]), np.float32)

    def chain(rows, start=None):
        s = np.zeros(d.shape[1], np.float32) if start is None else start.copy()
        for r in rows:
            s = s + r
        return s
    for token in np.unique(t):
        a, b = np.searchsorted(t, token), np.searchsorted(t, token, side="right")
        spans = []                                   # of each span: the sums of its chunks, added up
        for s in range(a // (8 * chunk), (b - 1) // (8 * chunk) + 1):
            parts = [chain(d[order[max(a, f):min(b, f + chunk)]]) for f in range(s * 8 * chunk, (s + 1) * 8 * chunk, chunk) if max(a, f) < min(b, f + chunk)]
            spans.append(chain(parts[1:], parts[0]))
        if len(spans) == 1:
            out[token] = spans[0]
            continue
        each = -(-len(spans) // 8)
        runs = [chain(spans[k:k + each]) for k in range(0, len(spans), each)]
        out[token] = chain(runs[1:], runs[0])
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("n,width,vocab,hot", [(8192, 12, 100, 0.3), (8193, 12, 100, 0.3), (9001, 9, 5, 0.0), (20000, 8, 1, 0.0), (20000, 8, 2500, 0.6), (50001, 8, 300000, 0.1)])
def test_sums_in_the_order_that_is_promised(row_plan, n, width, vocab, hot):  # noqa: F811
    gen = rng(n + vocab)
    tokens, d = some_tokens(gen, n, vocab, hot, 0.05), torch.randn(n, width, generator=gen, device="cuda")
    plan = (ctypes.c_longlong * 8)()
    row_plan.grad_plan(n, width, 1, 4, plan)
    table = torch.empty(vocab, width, device="cuda")
    sr.sr_embed_grad(d, tokens, table, workspace(n, width))
    want = in_order(d.cpu().numpy(), tokens.cpu().numpy(), vocab, plan[2])
    assert np.array_equal(table.cpu().numpy(), want)


LONG = [(8193, 8), (20000, 260), (70001, 64), (262144, 16), (100000, 1031), (1 << 20, 8)]
VALUE = np.float32(0.1)


def chain_bound(row_plan, n, width):  # noqa: F811
    plan = (ctypes.c_longlong * 8)()
    row_plan.grad_plan(n, width, 1, 4, plan)
    chunk, spans = plan[2], plan[3]
    m = chunk + 8 + -(-spans // 8) + 8 + 3
    return m * U / (1 - m * U)


@pytest.mark.parametrize("n,width", LONG)
def test_one_chain_over_all_rows_exceeds_the_bound(row_plan, n, width):  # noqa: F811
    """That the bound of the next test can tell."""
    one = np.cumsum(np.full(n, VALUE), dtype=np.float32)[-1]
    assert abs(float(one) - n * float(VALUE)) > 2 * chain_bound(row_plan, n, width) * n * float(VALUE)


@pytest.mark.gpu
@pytest.mark.parametrize("n,width", LONG)
def test_long_sums_have_short_chains(row_plan, n, width):  # noqa: F811
    d = torch.full((n, width), float(VALUE), device="cuda")
    table = torch.empty(1, width, device="cuda")
    sr.sr_embed_grad(d, torch.zeros(n, dtype=torch.int32, device="cuda"), table, workspace(n, width))
    want = n * float(VALUE)
    assert (table.double() - want).abs().max().item() <= chain_bound(row_plan, n, width) * want
