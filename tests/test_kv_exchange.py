"""Lanes of the key/value cache's kernels pass numbers to each other through LDS.  On the CPU (host_wave.py) a lane runs until its wave exchanges something, so that numbers which are
read without a fence behind their writing, or written anew without one behind their reading, are the wrong ones."""
import pytest
import torch

import kv_reference as ref
from test_kv_bounds import agree, cache, host, rows  # noqa: F401  (host: the fixture)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_scales_of_a_step_of_keys(host, dtype):  # noqa: F811
    """Tiles of 32 rows: a lane loads the scale of one key or value and takes those of sixteen."""
    lengths, starts = [100, 40], [0, 70, 110]
    args, q = cache(lengths, 2, 64, 16, dtype), rows(110, 4, 64, dtype)
    got = host.attention(q, *args, torch.tensor(starts, dtype=torch.int32))
    agree(got, *ref.attention(q, *args[:3], lengths, starts, 0, 0, 64 ** -0.5))


def test_codes_of_two_heads(host):  # noqa: F811
    """Heads of 64 channels two to a wave, one after the other through the same place, as calls of 16384 eights of tokens and heads have them; an odd number of heads."""
    heads, tokens = 63, 2100
    assert (tokens // 8 + 2) * heads >= 16384
    k, v = rows(tokens, heads, 64, seed=5), rows(tokens, heads, 64, seed=6)
    args, starts = cache([tokens + 3], heads, 64, 256), torch.tensor([0, tokens], dtype=torch.int32)
    host_args = [t.clone().share_memory_() for t in args]  # the calls run in child processes
    host.write(k, v, *host_args, starts)
    for got, given in zip(host.read(*host_args, tokens, starts), (k, v)):
        assert torch.equal(got, ref.value(*ref.quantise(given)))


def test_pages_of_a_last_step(host):  # noqa: F811
    """A piece whose last step is the first one behind a request for page numbers, and a plain one: no lane is asked for the page of a step before it (host_wave.py ends a run that
    reads a lane which there is not).  Two tokens of 340 heads of 33 queries, 33 steps in one piece; some heads against 64 bits."""
    heads, groups, length = 340, 33, 33 * 32
    args, q, starts = cache([length], heads, 64, 16), rows(2, heads * groups, 64), [0, 2]
    got = host.attention(q, *args, torch.tensor(starts, dtype=torch.int32))
    for h in (0, heads - 1):
        of = slice(h * groups, h * groups + 2)
        c, s = (t[:, h:h + 1] for t in args[:2])
        agree(got[:, of], *ref.attention(q[:, of], c, s, args[2], [length], starts, 0, 0, 64 ** -0.5))
