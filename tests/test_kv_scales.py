"""Attention over value scales of all sizes that bfloat16 has, and with softmax scales of all sizes, on the CPU (host_wave.py) and the GPU against 64 bits."""
import pytest
import torch

import host_wave
import kv_reference as ref
from paper_2409_17870_amd import binding
from test_kv_bounds import agree, cache, host, rows  # noqa: F401  (host: the fixture)

CASES = [(1, 190, 2), (5, 190, 2), (90, 190, 2), (1, 3300, 1), (40, 1100, 1)]  # new tokens, length (the last two are cut in pieces), heads


def inputs(new, length, heads, by, some):
    """Value scales times 2^by, all of them or those of every seventh token behind the first hundred."""
    codes, scales, table, lengths = cache([length], heads, 64, 16, torch.bfloat16, seed=new)
    tokens = torch.arange(length)
    if some:
        tokens = tokens[100::7]
    page, at = table[0].long()[tokens // 16], tokens % 16
    scales[page, :, 1, at] = (scales[page, :, 1, at].float() * 2.0 ** by).bfloat16()
    q = rows(new, 2 * heads, 64, torch.bfloat16, seed=by)
    q[::2] *= 0.25  # broad rows, whose many small weights count
    return q, (codes, scales, table), [length], [0, new]


def want(q, c, lengths, starts):
    return ref.attention(q, *c, lengths, starts, 0, 0, 64 ** -0.5)


@pytest.mark.parametrize("some", [False, True])
@pytest.mark.parametrize("by", [-90, 60, 70, 104, 120, 126])
@pytest.mark.parametrize("new, length, heads", CASES[:3])
def test_on_the_host(host, new, length, heads, by, some):  # noqa: F811
    q, c, lengths, starts = inputs(new, length, heads, by, some)
    m = host_wave.Memory()
    got = host.attention(m.copy(q), *[m.copy(t) for t in c], *[torch.tensor(x, dtype=torch.int32) for x in (lengths, starts)])
    agree(got, *want(q, c, lengths, starts))


@pytest.mark.gpu
@pytest.mark.parametrize("some", [False, True])
@pytest.mark.parametrize("by", [-90, 60, 70, 104, 120, 126])
@pytest.mark.parametrize("new, length, heads", CASES)
def test_on_the_gpu(new, length, heads, by, some):
    q, c, lengths, starts = inputs(new, length, heads, by, some)
    got = binding.apmm_kv_attention(q.cuda(), *[t.cuda() for t in c], *[torch.tensor(x, dtype=torch.int32).cuda() for x in (lengths, starts)])
    agree(got, *want(q, c, lengths, starts))


SOFTMAX = [1.5e-45, 1e-39, 2.0 ** -100, 2.0 ** 110, 3.4e38]


def softmax_inputs(new, dtype, scale):
    """Queries of many sizes; where the scale is large zeros, whose keys all weigh the same."""
    codes, scales, table, _ = cache([130], 2, 64, 16, dtype, seed=7)
    q = rows(new, 4, 64, dtype, seed=8)
    q[1::3] *= 2.0 ** -12
    if dtype == torch.bfloat16:
        q[2::3] *= 2.0 ** -100
    if scale > 1:
        q.zero_()
    return q, (codes, scales, table), [130], [0, new]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("scale", SOFTMAX)
@pytest.mark.parametrize("new", [1, 3, 70])
def test_softmax_scales_on_the_host(host, new, scale, dtype):  # noqa: F811
    q, c, lengths, starts = softmax_inputs(new, dtype, scale)
    m = host_wave.Memory()
    got = host.attention(m.copy(q), *[m.copy(t) for t in c], *[torch.tensor(x, dtype=torch.int32) for x in (lengths, starts)], scale=scale, window=60, sinks=5)
    agree(got, *ref.attention(q, *c, lengths, starts, 60, 5, scale))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("scale", SOFTMAX)
@pytest.mark.parametrize("new", [1, 3, 70])
def test_softmax_scales_on_the_gpu(new, scale, dtype):
    q, c, lengths, starts = softmax_inputs(new, dtype, scale)
    got = binding.apmm_kv_attention(q.cuda(), *[t.cuda() for t in c], *[torch.tensor(x, dtype=torch.int32).cuda() for x in (lengths, starts)], scale=scale, window=60, sinks=5)
    agree(got, *ref.attention(q, *c, lengths, starts, 60, 5, scale))


# value scales of 2^-85 and 2^80 within a row: where the large ones are, of the tokens' numbers
APART = {"later": lambda t, n: t >= n // 2, "earlier": lambda t, n: t < n // 3, "in turn": lambda t, n: t % 2 == 1, "steps in turn": lambda t, n: t // 32 % 2 == 1, "the last": lambda t, n: t == n - 1}


def apart(new, length, heads, where):
    codes, scales, table, _ = cache([length], heads, 64, 16, torch.bfloat16, seed=new)
    t = torch.arange(length)
    by = torch.where(APART[where](t, length), torch.tensor(2.0 ** 80), torch.tensor(2.0 ** -85))
    page, at = table[0].long()[t // 16], t % 16
    scales[page, :, 1, at] = (scales[page, :, 1, at].float() * by[:, None]).bfloat16()
    return rows(new, 2 * heads, 64, torch.bfloat16, seed=3) * 0.25, (codes, scales, table), [length], [0, new]


@pytest.mark.parametrize("window", [0, 7])
@pytest.mark.parametrize("where", list(APART))
@pytest.mark.parametrize("new, length, heads", CASES[:3])
def test_far_apart_on_the_host(host, new, length, heads, where, window):  # noqa: F811
    q, c, lengths, starts = apart(new, length, heads, where)
    m = host_wave.Memory()
    got = host.attention(m.copy(q), *[m.copy(t) for t in c], *[torch.tensor(x, dtype=torch.int32) for x in (lengths, starts)], window=window)
    agree(got, *ref.attention(q, *c, lengths, starts, window, 0, 64 ** -0.5))


@pytest.mark.gpu
@pytest.mark.parametrize("window", [0, 7])
@pytest.mark.parametrize("where", list(APART))
@pytest.mark.parametrize("new, length, heads", CASES)
def test_far_apart_on_the_gpu(new, length, heads, where, window):
    q, c, lengths, starts = apart(new, length, heads, where)
    got = binding.apmm_kv_attention(q.cuda(), *[t.cuda() for t in c], *[torch.tensor(x, dtype=torch.int32).cuda() for x in (lengths, starts)], window=window)
    agree(got, *ref.attention(q, *c, lengths, starts, window, 0, 64 ** -0.5))
