"""Attention over contexts so long that a workgroup or wave asks for page numbers more than once (32 steps of 32 keys at a time), with pages that are none and steps that are done again at
every place of those 32.  Some rows and heads against 64 bits."""
import pytest
import torch

import kv_reference as ref
from paper_2409_17870_amd import binding
from test_kv_bounds import agree

pytestmark = pytest.mark.gpu

D, PAGE = 64, 16


def long_cache(heads, length, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    pages = -(-length // PAGE)
    codes = torch.randint(0, 256, (pages, heads, 2, PAGE * D // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = (torch.rand((pages, heads, 2, PAGE), generator=g, device="cuda") * 0.2 + 0.01).to(dtype)
    table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)[None]
    return codes, scales, table


def run(heads, length, new, dtype, window, sinks, seed, change):
    codes, scales, table = long_cache(heads, length, dtype, seed)
    change(scales, table)
    q = torch.randn((new, heads, D), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)
    lengths, starts = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([length], [0, new])]
    got = binding.apmm_kv_attention(q, codes, scales, table, lengths, starts, window=window, sinks=sinks)
    for h in (0, heads // 2, heads - 1):
        c, s = codes[:, h:h + 1].cpu(), scales[:, h:h + 1].cpu()
        for row in sorted({0, new // 3, new - 1}):
            agree(got[row:row + 1, h:h + 1], *ref.attention(q[row:row + 1, h:h + 1], c, s, table.cpu(), [length - new + 1 + row], [0, 1], window, sinks, D ** -0.5))


def nothing(scales, table):
    pass


def no_pages(*steps):
    def change(scales, table):
        for i, step in enumerate(s for s in steps if 2 * s + 1 < table.shape[1]):
            table[0, step * 2 + i % 2] = (-1, scales.shape[0], 2 ** 31 - 1)[i % 3]
    return change


def large_keys(every, first):
    """Scores at these steps far above those before, each more than the last ones."""
    def change(scales, table):
        steps = list(range(first, table.shape[1] // 2, every))
        for i, step in enumerate(steps):
            scales[table[0, step * 2].long(), :, 0, 5] = 2.0 + 2.0 * i
    return change


CHANGES = {
    "plain": nothing,
    "no page in the second 32": no_pages(34, 40),
    "no page in the first 32": no_pages(3),
    "no page here and there": no_pages(1, 31, 32, 33, 64, 65, 97, 110, 128),
    "again at 32": large_keys(32, 32),
    "again at 33": large_keys(32, 33),
    "again at 31": large_keys(32, 31),
    "again in every seventh": large_keys(7, 2),
}


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("window, sinks", [(0, 0), (3000, 200)])
@pytest.mark.parametrize("change", list(CHANGES))
def test_tiles(change, window, sinks, dtype):
    """512 heads: two pieces of some 80 steps of the one tile."""
    run(512, 5000, 40, dtype, window, sinks, 1, CHANGES[change])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("change", list(CHANGES))
def test_tiles_uncut(change, dtype):
    """As many tiles as places: 1024 rows of 128 heads see 4000 keys in one piece."""
    run(128, 4000, 1024, dtype, 0, 0, 2, CHANGES[change])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads", [128, 512])
@pytest.mark.parametrize("change", ["plain", "no page here and there", "again in every seventh"])
def test_single_tokens(change, heads, dtype):
    """Eight and four waves, some 40 steps to each of a piece."""
    far = {"no page here and there": no_pages(1, 31, 255, 256, 263, 264, 300, 311, 312, 400, 599)}.get(change, CHANGES[change])
    run(heads, 20011, 1, dtype, 0, 0, 3, far)
