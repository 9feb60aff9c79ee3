"""What lies in lengths, starts and page tables is read on the device: whatever it is, the key/value cache's kernels touch nothing outside of their buffers.  On the CPU, where the kernels run
between pages that cannot be touched (host_wave.py), and on the GPU with NaN behind the workspace."""
import random

import pytest
import torch

import host_wave
from paper_2409_17870_amd import binding
from test_kv import close


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    if not host_wave.available():
        pytest.skip("no clang++")
    return host_wave.Host(host_wave.build(tmp_path_factory.mktemp("kv")))


def cache(lengths, heads, D, ps, dtype=torch.float16, seed=1, width=0, spare=1):
    """Codes, scales, a table whose rows name pages of their own (-1 behind them), lengths."""
    g = torch.Generator().manual_seed(seed)
    pages_of = [-(-n // ps) for n in lengths]
    pages = sum(pages_of) + spare
    codes = torch.randint(0, 256, (pages, heads, 2, ps * D // 2), generator=g, dtype=torch.uint8)
    scales = (torch.rand((pages, heads, 2, ps), generator=g) * 0.2 + 0.01).to(dtype)
    order, table = torch.randperm(pages, generator=g).to(torch.int32), torch.full((len(lengths), max(width, *pages_of, 1)), -1, dtype=torch.int32)
    for b, n in enumerate(pages_of):
        table[b, :n], order = order[:n], order[n:]
    return codes, scales, table, torch.tensor(lengths, dtype=torch.int32)


def rows(tokens, heads, D, dtype=torch.float16, seed=2):
    return torch.randn((tokens, heads, D), generator=torch.Generator().manual_seed(seed)).to(dtype)


def agree(got, want, near):
    """Finite, and as close as test_kv.py asks of its results (a difference that is no number passes its comparison)."""
    assert bool(torch.isfinite(got).all())
    close(torch, got, want, near)


# Sequences whose rows overlap have more tiles (12 + 8 + 1) than the host makes slots for from 12 tokens of 12 sequences; the last one is long and cut.
OVERLAP = dict(lengths=[40] * 4 + [3200] + [40] * 7, starts=[0, 12, 4, 12, 11, 12] + [12] * 7, heads=32, groups=16, D=128, ps=16)


def overlapping():
    c = OVERLAP
    return rows(12, c["heads"] * c["groups"], c["D"]), cache(c["lengths"], c["heads"], c["D"], c["ps"]), torch.tensor(c["starts"], dtype=torch.int32)


def test_pieces_beyond_the_slots(host):
    q, args, starts = overlapping()
    m = host_wave.Memory()
    out = host.attention(m.copy(q), *[m.copy(t) for t in args], m.copy(starts))
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("seed", range(24))
def test_wild_batches(host, seed):
    """Lengths, starts and page numbers of any size and order, for writes, reads and attention of few rows and many."""
    r = random.Random(seed)
    D, heads, groups, ps = r.choice([64, 128]), r.choice([1, 3, 32]), r.choice([1, 2, 16]), r.choice([16, 64])
    sequences, tokens, width = r.choice([1, 2, 6, 12, 70]), r.choice([1, 3, 12, 40]), r.choice([1, 4, 50])

    def wild(most):
        return r.choice([0, 1, -1, most, r.randint(0, most), r.randint(0, most), 2 ** 31 - 1, -2 ** 31, r.randint(-50, most + 50)])
    lengths = [wild(width * ps) if i < 8 else wild(60) for i in range(sequences)]
    starts = [r.choice([(0, tokens)[i % 2], r.randint(0, tokens), wild(tokens)]) for i in range(sequences + 1)]
    dtype = r.choice([torch.float16, torch.bfloat16])
    codes, scales, _, _ = cache([200], heads, D, ps, dtype, seed=seed)
    table = torch.randint(-2, codes.shape[0] + 2, (sequences, width), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
    m = host_wave.Memory()
    args = [m.copy(t) for t in (codes, scales, table, torch.tensor(lengths, dtype=torch.int32))]
    starts = m.copy(torch.tensor(starts, dtype=torch.int32))
    host.attention(m.copy(rows(tokens, heads * groups, D, dtype)), *args, starts, window=r.choice([0, 0, 50]), sinks=7)
    host.write(*[m.copy(rows(tokens, heads, D, dtype, seed=i)) for i in (3, 4)], *args, starts)
    host.read(*args, tokens, starts)


@pytest.mark.gpu
def test_pieces_beyond_the_slots_on_the_gpu():
    """Which of the sequences that share a row writes it last is open, what lies behind the workspace reaches none."""
    q, args, starts = overlapping()
    q, args = q.cuda(), [t.cuda() for t in args]
    need = binding.apmm_kv_attention_workspace_bytes(q.shape[0], q.shape[1], *args)
    assert need > 0
    room = torch.full((need + (64 << 20),), 0xff, dtype=torch.uint8, device="cuda")  # NaN
    out = binding.apmm_kv_attention(q, *args, starts.cuda(), workspace=room[:need])
    assert bool(torch.isfinite(out).all()) and bool((room[need:] == 0xff).all())
