"""Lengths beyond the page table: tokens that have no place there are seen by no query, of few rows or many, in every step of keys that the kernels take without looking at each key."""
import pytest
import torch

import host_wave
import kv_reference as ref
from paper_2409_17870_amd import binding
from test_kv_bounds import agree, cache, host, rows  # noqa: F401  (host: the fixture)

CASES = [  # page, pages of the table, length, new, window, sinks
    (16, 5, 10000, 100, 60, 96),     # all keys are first tokens, the last step of 32 has a page and none
    (16, 5, 10000, 100, 60, 75),
    (16, 3, 10000, 90, 1, 1000),
    (16, 7, 150, 100, 60, 96),       # some queries have a place
    (16, 5, 10000, 100, 9960, 40),   # the window ends inside the table
    (16, 5, 10000, 100, 0, 0),
    (32, 3, 10000, 100, 60, 128),
    (16, 5, 10000, 5, 60, 96),
    (16, 5, 10000, 1, 60, 96),
]


def inputs(case, dtype):
    ps, width, length, new, window, sinks = case
    codes, scales, table, _ = cache([ps * width], 2, 64, ps, dtype, spare=3)
    unused = [p for p in range(codes.shape[0]) if p not in table[0].tolist()]
    scales[unused] = 0.2   # of pages that are not the sequence's: as large as any, too small to fail a step
    if 0 not in unused:    # one of them is the cache's first
        other = unused[0]
        for t in (codes, scales):
            t[[0, other]] = t[[other, 0]]
        table[table == 0] = other
    return (codes, scales, table), rows(new, 4, 64, dtype), [length], [0, new], window, sinks


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("case", CASES)
def test_on_the_host(host, case, dtype):  # noqa: F811
    c, q, lengths, starts, window, sinks = inputs(case, dtype)
    m = host_wave.Memory()
    got = host.attention(m.copy(q), *[m.copy(t) for t in c], torch.tensor(lengths, dtype=torch.int32), torch.tensor(starts, dtype=torch.int32), window, sinks)
    agree(got, *ref.attention(q, *c, lengths, starts, window, sinks, 64 ** -0.5))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("case", CASES)
def test_on_the_gpu(case, dtype):
    c, q, lengths, starts, window, sinks = inputs(case, dtype)
    on = [torch.tensor(x, dtype=torch.int32).cuda() for x in (lengths, starts)]
    got = binding.apmm_kv_attention(q.cuda(), *[t.cuda() for t in c], *on, window=window, sinks=sinks)
    agree(got, *ref.attention(q, *c, lengths, starts, window, sinks, 64 ** -0.5))
