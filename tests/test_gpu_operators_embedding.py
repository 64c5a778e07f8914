"""Embedding lookup and its gradient against the formula."""
import math

import numpy as np
import pytest
import torch

from paper_2010_16248_amd import binding as B
from tests import operators_plain as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF = torch.float32, torch.bfloat16


def _ids(gen, n, vocab, kind, index):
    if kind == "same":
        ids = torch.full((n,), vocab // 2)
    elif kind == "zipf":
        ids = (torch.exp(torch.rand(n, generator=gen, dtype=torch.float64) * math.log(vocab + 1.0)) - 1).long().clamp(0, vocab - 1)
    elif kind == "distinct":
        ids = torch.randperm(vocab, generator=gen)[:n]
    elif kind == "outside":
        ids = torch.randint(-3, vocab + 3, (n,), generator=gen)
        ids[: max(1, n // 3)] = vocab
        if index == torch.int64:
            ids[-1] = 2 ** 40 + 1
    else:
        ids = torch.randint(0, vocab, (n,), generator=gen)
    return ids.to(index).to(DEV)


@pytest.mark.parametrize("tokens,vocab,dim,table,out,index,kind", [
    (1, 1, 1, F32, F32, torch.int64, "uniform"),
    (5, 7, 3, BF, F32, torch.int32, "uniform"),
    (700, 32768, 672, F32, F32, torch.int64, "zipf"),
    (63, 11, 33, F32, BF, torch.int64, "outside"),
    (257, 1000, 1001, BF, BF, torch.int32, "outside"),
    (3, 50, 20001, F32, F32, torch.int32, "uniform"),
    (1025, 129, 8, BF, BF, torch.int64, "same"),
])
def test_lookup_is_the_scaled_row(tokens, vocab, dim, table, out, index, kind):
    print(f"case lookup {tokens} {vocab} {dim} {table} {out} {index} {kind}", flush=True)
    gen = torch.Generator().manual_seed(tokens * 31 + dim)
    ids = _ids(gen, tokens, vocab, kind, index)
    tab = torch.randn(vocab, dim, generator=gen).to(table).to(DEV)
    got = torch.full((tokens, dim), 7.0, dtype=out, device=DEV)
    B.embedding_forward(ids, tab, got, 2.5)
    at = ids.long().cpu()
    known = (at >= 0) & (at < vocab)
    ref = (tab.cpu()[at.clamp(0, vocab - 1)].float() * 2.5 * known[:, None]).to(out)
    assert torch.equal(got.cpu(), ref)


def test_lookup_between_rows_of_larger_buffers_leaves_the_rest():
    gen = torch.Generator().manual_seed(1)
    ids = _ids(gen, 40, 30, "uniform", torch.int64)
    whole = torch.randn(30, 77, generator=gen).to(DEV)
    out = torch.full((40, 90), 3.0, device=DEV)
    B.embedding_forward(ids, whole[:, 5:70], out[:, 1:66])
    assert torch.equal(out[:, 1:66], whole[ids, 5:70])
    assert (out[:, :1] == 3).all() and (out[:, 66:] == 3).all()


@pytest.mark.parametrize("tokens,vocab,dim,kind,grad,index,accumulate", [
    (1, 1, 1, "uniform", F32, torch.int64, False),
    (1, 500, 40, "uniform", BF, torch.int64, False),
    (0, 100, 33, "uniform", F32, torch.int32, False),
    (0, 100, 33, "uniform", F32, torch.int32, True),
    (64, 9, 5, "uniform", F32, torch.int32, False),
    (65, 65, 1001, "distinct", F32, torch.int64, False),
    (2800, 3000, 672, "zipf", F32, torch.int64, False),
    (1000, 200, 100, "outside", BF, torch.int32, False),
    (100, 20, 16, "same", F32, torch.int64, True),
    (8192, 37, 65, "same", F32, torch.int64, False),
    (8192, 1000, 64, "zipf", BF, torch.int32, True),
    (8193, 1000, 64, "zipf", BF, torch.int32, False),      # one token more: ordered by digits
    (20001, 1023, 33, "zipf", F32, torch.int64, False),    # one digit
    (20000, 1024, 33, "outside", F32, torch.int64, False),  # the key of ids outside takes a bit more: two digits
    (40000, 70000, 24, "zipf", F32, torch.int64, True),
    (33333, 2 ** 21, 4, "uniform", BF, torch.int64, False),  # three digits
    (600000, 50, 8, "zipf", F32, torch.int32, False),       # tiles of several steps
])
def test_gradient_is_the_sum_over_equal_tokens(tokens, vocab, dim, kind, grad, index, accumulate):
    print(f"case gradient {tokens} {vocab} {dim} {kind} {grad} {index} {accumulate}", flush=True)
    gen = torch.Generator().manual_seed(tokens * 7 + dim)
    ids = _ids(gen, tokens, vocab, kind, index)
    g = (torch.randn(tokens, dim, generator=gen) * torch.exp(torch.randn(tokens, 1, generator=gen))).to(grad).to(DEV)
    start = torch.randn(vocab, dim, generator=gen).to(DEV)
    table = start.clone()
    B.embedding_backward(ids, g, table, 1.7, accumulate=accumulate)
    scale = float(np.float32(1.7))
    ref, bound = P.embedding_gradient(ids, g, vocab, scale, start if accumulate else None)
    P.assert_within(table, ref, bound, "gradient")
    if accumulate:
        untouched = torch.ones(vocab, dtype=torch.bool, device=DEV)
        inside = ids[(ids >= 0) & (ids < vocab)].long()
        untouched[inside] = False
        assert torch.equal(table[untouched], start[untouched])
    again = start.clone()
    B.embedding_backward(ids, g, again, 1.7, accumulate=accumulate)
    assert torch.equal(again, table), "the same call gave other bits"


def test_gradient_between_rows_of_larger_buffers_leaves_the_rest():
    gen = torch.Generator().manual_seed(2)
    for tokens in (300, 9000):
        ids = _ids(gen, tokens, 40, "uniform", torch.int32)
        g = torch.randn(tokens, 50, generator=gen).to(DEV)
        table = torch.full((40, 64), 3.0, device=DEV)
        B.embedding_backward(ids, g[:, 3:38], table[:, 7:42])
        ref, bound = P.embedding_gradient(ids, g[:, 3:38], 40, 1.0)
        P.assert_within(table[:, 7:42], ref, bound, "gradient")
        assert (table[:, :7] == 3).all() and (table[:, 42:] == 3).all()


def test_infinities_and_nan_stay_in_their_rows():
    ids = torch.tensor([3, 1, 3, 0, 9], device=DEV)      # 9 lies outside
    g = torch.ones(5, 6, device=DEV)
    g[1], g[4] = math.inf, math.nan
    table = torch.empty(5, 6, device=DEV)
    B.embedding_backward(ids, g, table)
    assert table[3].eq(2).all() and table[0].eq(1).all() and table[1].isinf().all() and table[2].eq(0).all() and table[4].eq(0).all()


@pytest.mark.parametrize("tokens,dim", [(4096, 672), (5000, 333), (5000, 16), (4100, 2501), (4096, 9001)])
@pytest.mark.parametrize("table,out", [(F32, F32), (BF, BF), (BF, F32)])
def test_lookup_of_many_tokens(tokens, dim, table, out):
    print(f"case lookup many {tokens} {dim} {table} {out}", flush=True)
    gen = torch.Generator().manual_seed(tokens + dim)
    ids = _ids(gen, tokens, 700, "outside", torch.int64)
    tab = torch.randn(700, dim, generator=gen).to(table).to(DEV)
    got = torch.full((tokens, dim), 7.0, dtype=out, device=DEV)
    B.embedding_forward(ids, tab, got, 2.5)
    known = (ids >= 0) & (ids < 700)
    ref = (tab[ids.clamp(0, 699)].float() * 2.5 * known[:, None]).to(out)
    assert torch.equal(got, ref)


# gradients of more than 128 MiB, which are streamed; runs from one token to a fifth of them all
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("tokens,vocab,dim,grad", [(40001, 5000, 1024, F32), (70000, 3001, 1028, BF), (40000, 40000, 900, F32)])
def test_gradient_of_more_than_the_caches_hold(tokens, vocab, dim, grad, accumulate):
    print(f"case gradient streamed {tokens} {vocab} {dim} {grad} {accumulate}", flush=True)
    gen = torch.Generator().manual_seed(tokens + dim)
    ids = _ids(gen, tokens, vocab, "zipf", torch.int64)
    ids[::97] = vocab + 3
    g = (torch.randn(tokens, dim, generator=gen) * torch.exp(torch.randn(tokens, 1, generator=gen))).to(grad).to(DEV)
    assert g.numel() * g.element_size() > 128 << 20
    start = torch.randn(vocab, dim, generator=gen).to(DEV)
    table = start.clone()
    B.embedding_backward(ids, g, table, 1.7, accumulate=accumulate)
    again = start.clone()
    B.embedding_backward(ids, g, again, 1.7, accumulate=accumulate)
    assert torch.equal(again, table), "the same call gave other bits"
    # the statement of operators_plain.embedding_gradient, on the GPU
    ok, scale = ids < vocab, float(np.float32(1.7))
    zeros = lambda *s: torch.zeros(*s, dtype=torch.float64, device=DEV)
    count = zeros(vocab).index_add_(0, ids[ok], torch.ones_like(ids[ok], dtype=torch.float64))
    ref = zeros(vocab, dim).index_add_(0, ids[ok], g[ok].double()) * scale
    bound = zeros(vocab, dim).index_add_(0, ids[ok], g[ok].double().abs()) * (count[:, None] + 2) * P.U * scale
    if accumulate:
        ref += start.double()
        bound += P.U * ref.abs()
    P.assert_within(table, P.f64(ref), P.f64(bound), "gradient")
