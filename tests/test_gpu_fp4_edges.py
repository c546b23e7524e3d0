"""The 4-bit cache and its attention: counts that are no counts, and splits of many sequences. Definitions and tolerances
are those of test_gpu_fp4.py.
"""
import random

import pytest
import torch

from .test_gpu_fp4 import BF16, DEV, append_reference, attention_case, filled_cache, normal, ops, same_numbers, tokens_of  # noqa: F401

pytestmark = pytest.mark.gpu

LEAST = -2 ** 31


@pytest.mark.parametrize("tokens", [6, 700])          # one token a thread, and four
@pytest.mark.parametrize("count", [[LEAST, LEAST + 1, LEAST + 2], [LEAST + 5, LEAST + 699, LEAST + 702], [-1, 0, LEAST], [LEAST, 3, 2 ** 31 - 1]])
def test_counts_that_are_no_counts(ops, tokens, count):  # noqa: F811
    """A count below 1 is of no token, the least 32-bit numbers among them; one above the tokens is of all."""
    heads, page, dim, batch = 4, 64, 128, 3
    columns = (tokens + 20 + page - 1) // page + 1
    cache = filled_cache(ops, batch * columns, heads, page, dim)
    table = torch.arange(batch * columns, dtype=torch.int32).reshape(batch, columns)
    start, n = torch.tensor([0, 3, 17], dtype=torch.int32), torch.tensor(count, dtype=torch.int32)
    k, v = (normal(i, batch, tokens, heads, dim).to(BF16) for i in (8, 9))
    before = tokens_of(cache)
    want = [append_reference(before[i], (k, v)[i], table, start, n, page) for i in range(2)]
    ops.kv_cache_fp4_append(k.to(DEV), v.to(DEV), *cache, table.to(DEV), start.to(DEV), n.to(DEV))
    for got, w in zip(tokens_of(cache), want):
        assert same_numbers(got, w)
    whole = ops.kv_cache_fp4_read(*cache, table.to(DEV), start.to(DEV), tokens)
    got = ops.kv_cache_fp4_read(*cache, table.to(DEV), start.to(DEV), tokens, n.to(DEV))
    for g, w in zip(got, whole):
        for b in range(batch):
            c = min(max(count[b], 0), tokens)
            assert torch.equal(g[b, :c], w[b, :c]) and not g[b, c:].any() and w[b].any()


@pytest.mark.parametrize("tokens,group,window", [(1, 3, 0), (1, 1, 700), (9, 2, 0), (20, 2, 0), (33, 1, 300)])
@pytest.mark.parametrize("dim", [16, 80, 144])
def test_attention_of_many_sequences_of_unequal_lengths(ops, tokens, group, window, dim):  # noqa: F811
    """More than 256 blocks of few queries: splits of at least 16 steps, many without keys, joined."""
    rng = random.Random(tokens + dim)
    lengths = [rng.choice([0, 1, tokens, 63, rng.randint(1, 400), rng.randint(1, 2100)]) for _ in range(134)] + [2100]
    attention_case(ops, dim, 64 if dim < 100 else 128, 2 if dim == 16 else 1, group, tokens, lengths * (1 if dim == 16 else 2), window=window, seed=dim,
                   count=[min(n, tokens) for n in lengths] * (1 if dim == 16 else 2))
