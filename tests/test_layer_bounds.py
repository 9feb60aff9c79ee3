"""Rotary positions and the cache's budget on the CPU, between pages that cannot be touched (host_layers.py): their results in small against 64 bits, and batches whose lengths, starts, page numbers
and positions are anything, of which the kernels touch nothing outside of their buffers."""
import random

import pytest
import torch

import host_layers
import host_wave
import kv_reference as ref
from test_kv_bounds import cache, rows
from test_kv_budget import stay, weights_of
from test_rotary import close, exact


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    if not host_wave.available():
        pytest.skip("no clang++")
    return host_layers.Host(host_layers.build(tmp_path_factory.mktemp("layers")))


class Held:
    """What weights_of asks of a batch."""

    def __init__(self, codes, scales, table, lengths, **more):
        self.codes, self.scales, self.table, self.lengths = codes, scales, table, lengths.tolist()


def frequencies(pairs):
    return 10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)


def guarded(*tensors):
    m = host_wave.Memory()
    return [m.copy(t) for t in tensors]


@pytest.mark.parametrize("D, pairs, interleaved", [(128, 64, 0), (128, 32, 1), (64, 20, 0), (7, 3, 1), (80, 16, 0), (1024, 512, 0)])
def test_rotary(host, D, pairs, interleaved):
    for dtype in (torch.float16, torch.bfloat16):
        x, at, f = rows(5, 3, D, dtype), torch.tensor([0, -7, 100000, 2 ** 31 - 1, 1], dtype=torch.int32), frequencies(pairs)
        y = host.rotary(*guarded(x, at, f), interleaved=interleaved, magnitude=1.5, inverse=1)
        want, near = exact(torch, x, at, f, interleaved, 1.5, True)
        # (the product of position and frequency in 64 bits, as in test_far_positions)
        close(torch, y, want, near + 2 ** 31 * 2.0 ** -50 * 1.5 * (x.double().abs().amax(2, keepdim=True)))


SMALL = [  # D, heads, groups, page, lengths, new, window, sinks
    (64, 2, 2, 16, [100, 0, 7, 33], [1, 1, 1, 1], 0, 0),
    (128, 1, 3, 16, [70, 40], [20, 3], 30, 2),
    (64, 1, 1, 64, [200, 1], [150, 1], 0, 0),
    (128, 1, 16, 16, [2100], [1], 0, 0),
    (64, 1, 2, 16, [700] + [30] * 12, [9] + [0] * 9 + [1] * 3, 300, 3),
    (64, 1, 5, 16, [700] + [30] * 12, [9] + [0] * 9 + [1] * 3, 300, 3),
]


@pytest.mark.parametrize("case", range(len(SMALL)))
def test_weights(host, case):
    D, heads, groups, ps, lengths, new, window, sinks = SMALL[case]
    for dtype in (torch.float16, torch.bfloat16):
        args, starts = cache(lengths, heads, D, ps, dtype), torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32)
        q, w = rows(sum(new), heads * groups, D, dtype), torch.rand((len(lengths), heads, max(lengths) - 3), generator=torch.Generator().manual_seed(case))
        b = Held(*args)
        got = host.weights(*guarded(q, *args, w, starts), window=window, sinks=sinks, decay=0.5)
        want, near = weights_of(torch, b, q, w, starts.tolist(), window, sinks, D ** -0.5, 0.5)
        for i, n in enumerate(lengths):
            n = min(n, w.shape[2])
            assert bool(((got[i, :, :n].double() - want[i, :, :n]).abs() <= near[i, :, :n]).all()) and torch.equal(got[i, :, n:], w[i, :, n:])


@pytest.mark.parametrize("ps, lengths, budget, sinks, recent, width", [(16, [100, 0, 7, 33], 20, 2, 5, 0), (64, [900, 3], 300, 0, 100, 100), (64, [700], 64, 4, 0, 300), (64, [500, 65], 70, 1, 9, 1100), (16, [9000, 5000, 30], 700, 3, 40, 4200),
                                                                        (16, [4097, 8192], 4500, 0, 0, 4200)])
def test_eviction(host, ps, lengths, budget, sinks, recent, width):
    """Tables of all widths that the selection tells apart."""
    heads, D = 2, 64
    codes, scales, table, n = cache(lengths, heads, D, ps, width=width, spare=1 + sum(-(-min(n, budget) // ps) for n in lengths))
    free = [p for p in range(codes.shape[0]) if p not in table.flatten().tolist()]
    to = torch.full((len(lengths), -(-budget // ps)), -1, dtype=torch.int32)
    for i, length in enumerate(lengths):
        for j in range(-(-min(length, budget) // ps)):
            to[i, j] = free.pop()
    w = torch.rand((len(lengths), heads, max(lengths)), generator=torch.Generator().manual_seed(budget))
    w[:, :, ::5] = 0.25
    codes, scales, table, n, w, to = guarded(codes, scales, table, n, w, to)
    kept, weights, left = host.evict(codes, scales, table, n, w, budget, to, sinks=sinks, recent=recent)
    ck, cv = ref.unlayout(codes, ps)
    for i, length in enumerate(lengths):
        for h in range(heads):
            want = stay(torch, w[i, h].tolist(), length, [True] * length, budget, sinks, recent)
            m = len(want)
            assert int(left[i]) == m and kept[i, h].tolist() == want + [-1] * (budget - m) and weights[i, h].tolist() == w[i, h, want].tolist() + [0.0] * (budget - m)
            j, d = torch.tensor(want, dtype=torch.long), torch.arange(m)
            for t in (ck, cv):
                assert torch.equal(t[to[i].long()[d // ps], h, d % ps], t[table[i].long()[j // ps], h, j % ps])


def wild(r, most):
    return r.choice([0, 1, -1, most, r.randint(0, most), r.randint(0, most), 2 ** 31 - 1, -2 ** 31, r.randint(-50, most + 50)])


@pytest.mark.parametrize("seed", range(24))
def test_wild_batches(host, seed):
    r, g = random.Random(seed), torch.Generator().manual_seed(seed)
    D, heads, groups, ps = r.choice([64, 128]), r.choice([1, 3]), r.choice([1, 2, 16]), r.choice([16, 64])
    sequences, tokens, width = r.choice([1, 2, 6, 12, 70]), r.choice([1, 3, 12, 40]), r.choice([1, 4, 50])
    lengths = torch.tensor([wild(r, width * ps) if i < 8 else wild(r, 60) for i in range(sequences)], dtype=torch.int32)
    starts = torch.tensor([r.choice([(0, tokens)[i % 2], r.randint(0, tokens), wild(r, tokens)]) for i in range(sequences + 1)], dtype=torch.int32)
    dtype = r.choice([torch.float16, torch.bfloat16])
    codes, scales, _, _ = cache([200], heads, D, ps, dtype, seed=seed)
    table, to = (torch.randint(-2, codes.shape[0] + 2, (sequences, n), generator=g, dtype=torch.int32) for n in (width, r.choice([1, 3])))
    q, k, v = (rows(tokens, n, D, dtype, seed=i) for i, n in ((3, heads * groups), (4, heads), (5, heads)))
    positions, f = torch.tensor([wild(r, 10 ** 6) for _ in range(tokens)], dtype=torch.int32), frequencies(r.choice([1, 5, D // 4, D // 2]))
    w = torch.rand((sequences, heads, r.choice([1, 30, width * ps])), generator=g)
    codes, scales, table, to, lengths, starts, q, k, v, positions, f, w = guarded(codes, scales, table, to, lengths, starts, q, k, v, positions, f, w)
    args = codes, scales, table, lengths
    host.write_rotary(q, k, v, *args, f, starts, r.choice([None, positions]), interleaved=seed % 2)
    host.weights(q, *args, w, starts, window=r.choice([0, 0, 50]), sinks=7, decay=r.choice([0.0, 1.0]))
    if seed % 3 == 0:  # (a table so wide that several workgroups share a sequence)
        wide = torch.randint(-2, codes.shape[0] + 2, (sequences, 4200), generator=g, dtype=torch.int32)
        lengths = torch.tensor([wild(r, 12000) for _ in range(sequences)], dtype=torch.int32)
        table, lengths = guarded(wide, lengths)
        args, width = (codes, scales, table, lengths), 4200
    if sequences <= 12:
        budget = r.choice([1, 20, 70])
        kept, _, left = host.evict(*args, w, budget, to, sinks=r.choice([0, 1]), recent=r.choice([0, budget - 1]))
        assert bool((left >= 0).all()) and bool((left <= budget).all())
        for i in range(sequences):
            n = int(left[i])
            assert bool((kept[i, :, n:] == -1).all()) and bool((kept[i, :, :n] >= 0).all()) and bool((kept[i, :, :n] < width * ps).all()) and bool((kept[i, :, :n].diff(dim=1) > 0).all())


def test_rows_that_sequences_share(host):
    """More tiles than the host makes slots for (as in test_kv_bounds.py), of few rows and of many."""
    for lengths, starts, groups in (([40] * 4 + [3200] + [40] * 7, [0, 12, 4, 12, 11, 12] + [12] * 7, 16), ([40, 3200, 40, 900], [0, 90, 0, 90, 10], 1)):
        tokens = max(starts)
        args = cache(lengths, 8, 128, 16)
        w = host.weights(*guarded(rows(tokens, 8 * groups, 128), *args, torch.zeros((len(lengths), 8, 3200)), torch.tensor(starts, dtype=torch.int32)))
        assert bool(torch.isfinite(w).all())
