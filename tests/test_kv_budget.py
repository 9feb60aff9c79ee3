"""What attention gives each token of the four-bit cache, and the eviction of the lightest, on the GPU against plain implementations in 64 bits."""
import math

import pytest

import kv_reference as ref
from test_kv import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2409_17870_amd import binding
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    binding.load()
    return torch, binding


def weights_of(torch, b, q, before, starts, window, sinks, scale, decay, table=None, scales=None):
    """weights in 64 bits, and how far sums in 32 bits may be from them."""
    table, scales = b.table if table is None else table, (b.scales if scales is None else scales).cpu()
    ps, pages = scales.shape[3], scales.shape[0]
    ck, _ = ref.unlayout(b.codes, ps)
    k = (2.0 * ck.double() - 15.0) * scales[:, :, 0].double()[..., None]
    H, D = k.shape[1], k.shape[3]
    q = q.cpu().double()
    G = q.shape[1] // H
    out, near = before.cpu().double().clone(), torch.zeros(before.shape, dtype=torch.float64)
    capacity = before.shape[2]
    for i, length in enumerate(b.lengths):
        n = starts[i + 1] - starts[i]
        keys = min(length, table.shape[1] * ps)
        if n == 0 or keys == 0:
            continue
        j = torch.arange(keys)
        page = table[i].long()[j // ps]
        there = (page >= 0) & (page < pages)
        kk = k[page.clamp(0, pages - 1), :, j % ps]                        # keys, heads, D
        p = (length - n + torch.arange(n))[:, None]
        seen = (j[None] <= p) & there[None]
        if window:
            seen &= (j[None] > p - window) | (j[None] < sinks)
        for h in range(H):
            total, off = torch.zeros(keys, dtype=torch.float64), torch.zeros(keys, dtype=torch.float64)
            for g in range(h * G, h * G + G):
                x = scale * q[starts[i]:starts[i + 1], g] @ kk[:, h].t()
                w = torch.softmax(x.masked_fill(~seen, -math.inf), 1).nan_to_num_(0.0) if not bool(torch.isnan(x).any()) else \
                    torch.where(seen, torch.softmax(x.masked_fill(~seen, -math.inf), 1), torch.zeros(()).double())
                # the score: D products and sums, the factors and the exponent's argument to 2^-24 each; the weight follows it in both places, the exponential itself and the row's sum
                d = (D + 8) * 2.0 ** -24 * scale * (q[starts[i]:starts[i + 1], g].abs() @ kk[:, h].abs().t())
                d = torch.where(seen, d, torch.zeros(())).amax(1, keepdim=True)
                off += (w * (2.0 * d + (keys // 16 + 64) * 2.0 ** -24)).sum(0)
                total += w.sum(0)
            m = min(keys, capacity)
            out[i, h, :m] = total[:m] + (decay * out[i, h, :m] if decay else 0.0)
            # a lane's sum: up to 32 tiles' rows one after the other (or 16 rows of few), such sums one after the other, sixteen lanes'
            near[i, h, :m] = off[:m] + (min(n * G, 32 + n * G / 512) + 8) * 2.0 ** -24 * out[i, h, :m].abs() + 1e-30
    return out, near


CASES = [  # D, heads, groups, page, lengths, new, window, sinks
    (128, 1, 1, 16, [1], [1], 0, 0),
    (128, 2, 4, 16, [777, 5, 0, 64], [1, 1, 1, 1], 0, 0),                    # an empty sequence, whose query sees nothing
    (64, 3, 3, 16, [9, 8, 7, 16, 17, 33], [9, 1, 7, 16, 2, 20], 0, 0),
    (128, 2, 1, 64, [130, 64, 1, 0, 200], [130, 3, 1, 2, 17], 0, 0),
    (64, 1, 2, 32, [100] * 70, [1] * 70, 0, 0),                              # more sequences than lanes
    (128, 1, 16, 128, [700, 300], [3, 1], 0, 0),
    (64, 2, 5, 16, [600, 333], [40, 333], 100, 3),
    (128, 1, 2, 16, [1100, 3], [1, 1], 40, 5),
    (64, 1, 1, 256, [1500], [700], 0, 0),
    (128, 1, 1, 16, [520], [520], 16, 0),
    (64, 1, 1, 16, [513], [300], 1, 0),                                      # each query sees itself alone
    (64, 1, 2, 16, [1100] + [30] * 24, [20] + [0] * 20 + [1] * 4, 0, 0),     # no more tokens than sequences, of which one has most
    (128, 2, 4, 16, [100] + [30] * 24, [20] + [0] * 20 + [1] * 4, 40, 3),
    (64, 1, 8, 16, [1100] + [30] * 24, [20] + [0] * 20 + [1] * 4, 0, 0),
    (128, 1, 5, 32, [100, 333] + [30] * 23, [20, 3] + [0] * 20 + [1] * 3, 40, 3),
]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_weights(gpu, case, dtype):
    torch, binding = gpu
    D, heads, groups, ps, lengths, new, window, sinks = CASES[case]
    b = Batch(torch, getattr(torch, dtype), D, heads, groups, ps, lengths, new, seed=case, room=1)
    capacity = b.table.shape[1] * ps + 5
    for decay, scale in ((1.0, None), (0.0, 0.3), (0.9, 1.0 / D)):
        w = torch.rand((len(lengths), heads, capacity), generator=torch.Generator().manual_seed(case)).cuda()
        if decay == 0:
            w.fill_(float("nan"))                                            # is not read
        before = w.clone()
        got = binding.apmm_kv_weights(b.q, *b.args, w, b.starts_gpu, window=window, sinks=sinks, scale=scale, decay=decay)
        assert got is w
        base = before if decay else torch.zeros_like(before)
        want, near = weights_of(torch, b, b.q, base, b.starts, window, sinks, D ** -0.5 if scale is None else scale, decay)
        for i, length in enumerate(lengths):
            if new[i] == 0:                                                  # keeps what is there, the NaN too
                assert torch.equal(torch.nan_to_num(got[i], 7.0), torch.nan_to_num(before[i], 7.0))
                continue
            assert bool(((got[i, :, :length].cpu().double() - want[i, :, :length]).abs() <= near[i, :, :length]).all()), (decay, i)
            assert torch.equal(torch.nan_to_num(got[i, :, length:], 7.0), torch.nan_to_num(before[i, :, length:], 7.0))
            if decay == 0 and length:                                        # each query gives 1 in all
                n = min(new[i], length)
                assert abs(float(got[i, :, :length].double().sum()) - n * heads * groups) <= 1e-4 * n * heads * groups


def test_sums_over_many_rows(gpu):
    """First tokens that every query sees under a window: 65536 rows' weights to one sum, 4096 a lane.  Two steps of 32 and 128 round to 2^-25 of the sum at most at each and so are off by 2^-25 sqrt((32 + 128) / 3) as a
    rule, 2.2e-7; one after the other 4096 would be by 1.1e-6."""
    torch, binding = gpu
    b = Batch(torch, torch.bfloat16, 64, 1, 16, 64, [4096], [4096], seed=16)
    w = binding.apmm_kv_weights(b.q, *b.args, torch.zeros((1, 1, 4096), device="cuda"), b.starts_gpu, window=14, sinks=3, decay=0.0)
    want, near = weights_of(torch, b, b.q, torch.zeros((1, 1, 4096)), b.starts, 14, 3, 64 ** -0.5, 0.0)
    off = (w.cpu().double() - want).abs()
    assert bool((off <= near).all()) and float((off[0, 0, :3] / want[0, 0, :3]).pow(2).mean().sqrt()) < 6e-7


def test_cut_rows_of_long_sequences(gpu):
    """Keys of few rows are cut in pieces and joined: as many tokens as give several, ragged, with and without a window."""
    torch, binding = gpu
    lengths = [9001, 40, 4100, 0, 6000]
    b = Batch(torch, torch.bfloat16, 64, 2, 3, 64, lengths, [1, 1, 1, 1, 1], seed=11)
    for window, sinks in ((0, 0), (5000, 100)):
        w = torch.zeros((5, 2, b.table.shape[1] * 64), device="cuda")
        binding.apmm_kv_weights(b.q, *b.args, w, window=window, sinks=sinks)
        want, near = weights_of(torch, b, b.q, torch.zeros_like(w), b.starts, window, sinks, 64 ** -0.5, 1.0)
        assert bool(((w.cpu().double() - want).abs() <= near).all())
    assert binding.apmm_kv_weights_workspace_bytes(5, 6, *b.args) > 5 * 6 * 8


def test_wide_table(gpu):
    """Few rows whose scores, as far as the table goes, would take more room than is given to them."""
    torch, binding = gpu
    for D, dtype, window in ((64, torch.float16, 0), (128, torch.bfloat16, 300)):
        b = Batch(torch, dtype, D, 2, 2, 16, [1700, 40], [1, 1], seed=15)
        wide = torch.full((2, 1 << 20), -1, dtype=torch.int32)
        wide[:, :b.table.shape[1]] = b.table
        args = [b.args[0], b.args[1], wide.cuda(), b.args[3]]
        assert binding.apmm_kv_weights_workspace_bytes(2, 4, *args) < binding.apmm_kv_weights_workspace_bytes(2, 4, *args[:2], args[2][:, :1 << 18].contiguous(), args[3])
        for a in (b.args, args):
            w = binding.apmm_kv_weights(b.q, *a, torch.ones((2, 2, 1700), device="cuda"), window=window, sinks=5)
            want, near = weights_of(torch, b, b.q, torch.ones((2, 2, 1700)), b.starts, window, 5, D ** -0.5, 1.0)
            assert bool(((w.cpu().double() - want).abs() <= near).all())


def test_capacity_strides_streams_workspace_and_graph(gpu):
    torch, binding = gpu
    lengths, new = [300, 40, 129], [7, 40, 1]
    b = Batch(torch, torch.float16, 128, 2, 2, 16, lengths, new, seed=12)
    wide = torch.full((3, 4, 400), 3.0, device="cuda")
    w = wide[:, 1:3, 11:11 + 100]                                            # tokens from 100 on have none
    binding.apmm_kv_weights(b.q, *b.args, w, b.starts_gpu)
    want, near = weights_of(torch, b, b.q, torch.full((3, 2, 100), 3.0), b.starts, 0, 0, 128 ** -0.5, 1.0)
    assert bool(((w.cpu().double() - want).abs() <= near).all())
    w.fill_(3.0)
    assert bool((wide == 3).all())
    q = b.q.contiguous()
    workspace = torch.empty(binding.apmm_kv_weights_workspace_bytes(b.tokens, 4, *b.args), dtype=torch.uint8, device="cuda")
    want = binding.apmm_kv_weights(q, *b.args, torch.zeros((3, 2, 300), device="cuda"), b.starts_gpu)
    out = torch.zeros_like(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.apmm_kv_weights(q, *b.args, out, b.starts_gpu, decay=0.0, workspace=workspace)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.apmm_kv_weights(q, *b.args, out, b.starts_gpu, decay=0.5, workspace=workspace)
    out.zero_()
    expected = torch.zeros_like(out)
    for _ in range(3):
        q.normal_()
        graph.replay()
        binding.apmm_kv_weights(q, *b.args, expected, b.starts_gpu, decay=0.5)
        assert torch.equal(out, expected)


def test_pages_that_there_are_not_and_scales_that_are_nan(gpu):
    torch, binding = gpu
    lengths, new = [100, 70], [20, 70]
    b = Batch(torch, torch.bfloat16, 64, 2, 2, 16, lengths, new, seed=13)
    table = b.table.clone()
    table[0, 2], table[1, 0] = -1, 10 ** 6
    args = [b.args[0], b.args[1], table.cuda(), b.args[3]]
    w = torch.zeros((2, 2, 112), device="cuda")
    binding.apmm_kv_weights(b.q, *args, w, b.starts_gpu)
    want, near = weights_of(torch, b, b.q, torch.zeros_like(w), b.starts, 0, 0, 64 ** -0.5, 1.0, table=table)
    assert bool(((w.cpu().double() - want).abs() <= near).all())
    assert bool((w[0, :, 32:48] == 0).all()) and bool((w[1, :, :16] == 0).all())
    # one key's scale of one head: every query that sees it gives NaN to what it sees, the others what they gave before
    scales = b.scales.clone()
    scales[int(table[1, 2]), 1, 0, 3] = float("nan")                         # key 35 of the second sequence
    got = torch.zeros_like(w)
    binding.apmm_kv_weights(b.q, b.codes, scales, *args[2:], got, b.starts_gpu)
    assert torch.equal(got[0], w[0]) and torch.equal(got[1, 0], w[1, 0])
    assert bool(torch.isnan(got[1, 1, 16:70]).all()) and bool((got[1, 1, :16] == 0).all()) and bool((got[1, 1, 70:] == 0).all())
    # starts that leave rows out, and a sequence without new tokens, which keeps what it has
    starts = torch.tensor([5, 25, 25], dtype=torch.int32).cuda()
    got = torch.full_like(w, 2.0)
    binding.apmm_kv_weights(b.q, *b.args, got, starts, decay=0.0)
    want, near = weights_of(torch, b, b.q, torch.full_like(w, 2.0), [5, 25, 25], 0, 0, 64 ** -0.5, 0.0)
    assert bool(((got.cpu().double() - want).abs() <= near).all()) and bool((got[1] == 2).all())


def test_rows_with_numbers_that_are_not_finite_leave_others_alone(gpu):
    torch, binding = gpu
    b = Batch(torch, torch.float16, 64, 1, 1, 16, [90, 50], [90, 1], seed=14)
    q = b.q.contiguous()
    w = binding.apmm_kv_weights(q, *b.args, torch.zeros((2, 1, 96), device="cuda"), b.starts_gpu)
    q[40, 0, 3] = float("nan")
    got = binding.apmm_kv_weights(q, *b.args, torch.zeros((2, 1, 96), device="cuda"), b.starts_gpu)
    assert bool(torch.isnan(got[0, 0, :41]).all()) and torch.equal(got[0, 0, 41:], w[0, 0, 41:]) and torch.equal(got[1], w[1])


# ---------------------------------------------------------------- eviction ---
def stay(torch, w, length, eligible, budget, sinks, recent):
    """Places that stay, one by one from the definition."""
    held = [j for j in range(length) if eligible[j] and (j < sinks or j >= length - recent)]
    others = [j for j in range(length) if eligible[j] and not (j < sinks or j >= length - recent)]

    def weight(j):
        if j >= len(w) or math.isnan(w[j]):
            return (0, 0.0)
        return (1, w[j])
    others.sort(key=lambda j: (tuple(-x for x in weight(j)), j))
    return sorted(held + others[:max(0, budget - len(held))])


EVICTIONS = [  # D, heads, page, lengths, budget, sinks, recent
    (128, 1, 16, [1], 1, 0, 0),
    (64, 2, 16, [100, 0, 7, 33], 20, 2, 5),
    (128, 3, 32, [700, 64, 65, 1, 130], 64, 4, 16),
    (64, 1, 64, [3000], 777, 0, 0),
    (128, 2, 16, [2500, 1100], 1001, 10, 991),
    (64, 2, 128, [300] * 66, 8, 8, 0),
    (128, 1, 16, [40, 500], 600, 3, 100),                                     # all stay
]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("kind", ["heavy", "equal", "odd"])
@pytest.mark.parametrize("case", range(len(EVICTIONS)))
def test_eviction(gpu, case, kind, dtype):
    torch, binding = gpu
    D, heads, ps, lengths, budget, sinks, recent = EVICTIONS[case]
    dt = getattr(torch, dtype)
    kept_of = [min(n, budget) for n in lengths]
    b = Batch(torch, dt, D, heads, 1, ps, lengths, [1] * len(lengths), seed=case, spare=sum(-(-n // ps) for n in kept_of) + 2)
    g = torch.Generator().manual_seed(case)
    capacity = b.table.shape[1] * ps
    w = torch.exp(2 * torch.randn((len(lengths), heads, capacity), generator=g))
    if kind == "equal":
        w = torch.randint(0, 3, w.shape, generator=g).float() * torch.where(torch.rand(w.shape, generator=g) < 0.5, -1.0, 1.0)   # zeros of both signs, negative ones
    if kind == "odd":
        w[:, :, 5::7], w[:, :, 3::11], w[:, :, 2::13] = float("nan"), float("inf"), -float("inf")
        w = w[:, :, :max(1, capacity // 2)]                                    # tokens from there on have none
    table = b.table.clone()
    if kind == "odd" and table.shape[1] > 2:
        table[0, 1] = -5                                                       # tokens without a page never stay
    used = set(int(p) for p in b.table.flatten() if p >= 0)
    free = [p for p in range(b.codes.shape[0]) if p not in used]
    to = torch.full((len(lengths), max(1, -(-max(kept_of) // ps))), -1, dtype=torch.int32)
    for i, n in enumerate(kept_of):
        for j in range(-(-n // ps)):
            to[i, j] = free.pop()
    codes, scales = b.codes.clone(), b.scales.clone()
    kept, weights, length = binding.apmm_kv_evict(codes, scales, table.cuda(), b.args[3], w.cuda(), budget, to.cuda(), sinks=sinks, recent=recent)
    (ck, cv), (dk, dv) = ref.unlayout(b.codes, ps), ref.unlayout(codes, ps)
    before, after = b.scales.cpu(), scales.cpu()
    ck, cv, before = ck.clone(), cv.clone(), before.clone()                    # what is to come out
    for i, n in enumerate(lengths):
        eligible = [0 <= int(table[i, j // ps]) < b.codes.shape[0] for j in range(n)]
        for h in range(heads):
            want = stay(torch, w[i, h].tolist(), n, eligible, budget, sinks, recent)
            m = len(want)
            assert int(length[i]) == m
            assert kept[i, h, :m].tolist() == want and bool((kept[i, h, m:] == -1).all()), (i, h)
            ww = torch.tensor([float(w[i, h, j]) if j < w.shape[2] else 0.0 for j in want])
            assert torch.equal(torch.nan_to_num(weights[i, h, :m].cpu(), 123.0, 124.0, 125.0), torch.nan_to_num(ww, 123.0, 124.0, 125.0)) and bool((weights[i, h, m:] == 0).all())
            if m:
                j, d = torch.tensor(want), torch.arange(m)
                page, to_page = table[i].long()[j // ps], to[i].long()[d // ps]
                for t in (ck, cv):
                    t[to_page, h, d % ps] = t[page, h, j % ps]
                before[to_page, h, :, d % ps] = before[page, h, :, j % ps]
    assert torch.equal(dk, ck) and torch.equal(dv, cv)
    assert torch.equal(after.view(torch.int16), before.view(torch.int16))      # (bits: the rest of the cache is as it was)


@pytest.mark.parametrize("L, heads, budget", [(70001, 2, 5003), (17000, 3, 16999), (33000, 1, 4096), (300017, 2, 70001), (1200001, 1, 1), (70001, 260, 100), (20000, 300, 3000)])
def test_long_eviction_equals_a_stable_sort(gpu, L, heads, budget):
    """Sequences of one workgroup to a head and of many, of one chunk of tokens each and of several."""
    torch, binding = gpu
    ps = 16
    g = torch.Generator(device="cuda").manual_seed(1)
    pages = -(-L // ps) + -(-budget // ps)
    codes = torch.empty((pages, heads, 2, ps * 32), device="cuda", dtype=torch.uint8)
    scales = torch.empty((pages, heads, 2, ps), device="cuda", dtype=torch.float16)
    table, to = (torch.arange(a, z, dtype=torch.int32, device="cuda")[None] for a, z in ((0, -(-L // ps)), (-(-L // ps), pages)))
    lengths = torch.tensor([L], dtype=torch.int32, device="cuda")
    for step in (0.0, 0.5, 1e9):                                               # all different, many equal, all equal
        w = torch.exp(2 * torch.randn((1, heads, L), generator=g, device="cuda"))
        if step:
            w = torch.floor(w / step) * step
        sinks, recent = min(4, budget), min(100, max(0, budget - 4))
        kept, weights, length = binding.apmm_kv_evict(codes, scales, table, lengths, w, budget, to, sinks=sinks, recent=recent)
        value = w.clone()
        value[:, :, :sinks] = float("inf")
        if recent:
            value[:, :, -recent:] = float("inf")
        order = torch.sort(value, dim=2, descending=True, stable=True).indices[:, :, :budget].sort(2).values
        assert torch.equal(kept.long(), order) and torch.equal(weights, w.gather(2, order)) and length.tolist() == [budget]


@pytest.mark.parametrize("columns", [13, 4200])                               # of a table for one workgroup to a sequence and head, and for several
def test_graph_and_stream(gpu, columns):
    torch, binding = gpu
    b = Batch(torch, torch.float16, 64, 2, 1, 16, [200, 90], [1, 1], seed=21, spare=20)
    table = torch.full((2, columns), -1, dtype=torch.int32)
    table[:, :b.table.shape[1]] = b.table
    b.args[2] = table.cuda()
    used = set(int(p) for p in b.table.flatten() if p >= 0)
    free = torch.tensor([p for p in range(b.codes.shape[0]) if p not in used][:8], dtype=torch.int32).view(2, 4).cuda()
    w = torch.rand((2, 2, 208), device="cuda")
    out = [x.clone() for x in binding.apmm_kv_evict(*b.args, w, 50, free, recent=10)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        again = binding.apmm_kv_evict(*b.args, w, 50, free, recent=10)
    stream.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(out, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.apmm_kv_evict(*b.args, w, 50, free, recent=10, kept=out[0], to_weights=out[1], to_lengths=out[2])
    for _ in range(3):
        w.uniform_()
        graph.replay()
        cache = b.codes.clone()
        want = binding.apmm_kv_evict(*b.args, w, 50, free, recent=10)
        assert all(torch.equal(x, y) for x, y in zip(out, want)) and torch.equal(cache, b.codes)


def test_generation_within_a_budget(gpu):
    """The operators as they are used: queries and keys turned on their way into the cache, attention, weights, and eviction when the budget is passed; after it attention over what
    stayed is attention over those tokens of the whole cache."""
    torch, binding = gpu
    B, H, G, D, ps, budget, recent = 2, 2, 2, 64, 16, 48, 16
    g = torch.Generator(device="cuda").manual_seed(5)
    codes, scales = binding.apmm_kv_cache(40, ps, H, D)
    tables = [torch.arange(0, 16, dtype=torch.int32, device="cuda").view(B, 8), torch.arange(16, 32, dtype=torch.int32, device="cuda").view(B, 8)]
    f = binding.apmm_rotary_frequencies(D)
    lengths = torch.tensor([70, 64], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 70, 134], dtype=torch.int32, device="cuda")
    weights = torch.zeros((B, H, 128), device="cuda")

    def rows(n):
        return torch.randn((n, H * G + 2 * H, D), generator=g, device="cuda").half().split((H * G, H, H), 1)
    q, k, v = rows(134)
    q = binding.apmm_kv_write_rotary(q, k, v, codes, scales, tables[0], lengths, f, starts)
    binding.apmm_kv_attention(q, codes, scales, tables[0], lengths, starts)
    binding.apmm_kv_weights(q, codes, scales, tables[0], lengths, weights, starts)
    whole_k, whole_v = binding.apmm_kv_read(codes, scales, tables[0], lengths, 134, starts)
    kept, heavy, lengths = binding.apmm_kv_evict(codes, scales, tables[0], lengths, weights, budget, tables[1], recent=recent)
    weights.zero_()
    weights[:, :, :budget] = heavy
    positions = torch.tensor([70, 64], dtype=torch.int32, device="cuda")
    for step in range(3):
        lengths += 1
        q, k, v = rows(B)
        q = binding.apmm_kv_write_rotary(q, k, v, codes, scales, tables[1], lengths, f, positions=positions)
        o = binding.apmm_kv_attention(q, codes, scales, tables[1], lengths)
        binding.apmm_kv_weights(q, codes, scales, tables[1], lengths, weights)
        positions += 1
        now_k, now_v = binding.apmm_kv_read(codes, scales, tables[1], lengths, int(lengths.sum()), torch.tensor([0, budget + step + 1, 2 * (budget + step + 1)], dtype=torch.int32, device="cuda"))
        for b in range(B):
            for h in range(H):
                at = b * (budget + step + 1)
                first = (0, 70)[b]
                kk = torch.cat([whole_k[first + kept[b, h].long(), h], now_k[at + budget:at + budget + step + 1, h]]).double().cpu()
                vv = torch.cat([whole_v[first + kept[b, h].long(), h], now_v[at + budget:at + budget + step + 1, h]]).double().cpu()
                for i in range(h * G, h * G + G):
                    p = torch.softmax(kk @ q[b, i].double().cpu() * D ** -0.5, 0)
                    # keys and values read back are rounded to 2^-11 of themselves, weights of the attention as much, the result once
                    far = 2.0 ** -11 * D ** -0.5 * float((kk.abs() @ q[b, i].double().cpu().abs()).max())
                    assert bool(((o[b, i].double().cpu() - p @ vv).abs() <= (2 * far + 3 * 2.0 ** -11) * (p @ vv.abs()) + 2.0 ** -11 * (p @ vv).abs() + 1e-3 * 2.0 ** -10).all())
    assert bool((weights[:, :, :budget] >= heavy).all()) and bool((weights[:, :, budget:budget + 3] > 0).all())


def test_offsets_beyond_32_bits(gpu):
    """Pages beyond 4 GiB of codes, weights of sequences and heads 2^31 numbers apart and in the order of heads."""
    torch, binding = gpu
    D, heads, ps = 128, 8, 256
    pages = (5 << 30) // (heads * ps * D)
    codes, scales = binding.apmm_kv_cache(pages, ps, heads, D, torch.float16)
    f = binding.apmm_rotary_frequencies(D)
    for new, groups in (([300, 1], 1), ([1, 1], 4)):
        x = Batch(torch, torch.float16, D, heads, groups, ps, [300, 520], new, seed=9, spare=4)
        far = [pages - 1 - 7 * i for i in range(x.scales.shape[0])]
        codes[far], scales[far] = x.codes, x.scales
        where = torch.tensor(far, dtype=torch.int32)
        table = torch.where(x.table >= 0, where[x.table.long()], x.table).cuda()
        args = [codes, scales, table, x.args[3]]
        a, b = (binding.apmm_kv_write_rotary(x.q, x.k, x.v, *to, f, x.starts_gpu) for to in (x.args, args))
        assert torch.equal(a, b) and torch.equal(codes[far], x.codes) and torch.equal(scales[far], x.scales)
        near = binding.apmm_kv_weights(a, *x.args, torch.zeros((2, heads, 700), device="cuda"), x.starts_gpu)
        apart = torch.empty((1 << 31) + (8 << 20), device="cuda").as_strided((2, heads, 700), (1 << 31, 1 << 20, 1)).zero_()
        turned = torch.zeros((heads, 2, 700), device="cuda").transpose(0, 1)
        for w in (apart, turned):
            assert torch.equal(binding.apmm_kv_weights(a, *args, w, x.starts_gpu), near)
        used = set(int(p) for p in x.table.flatten() if p >= 0)
        to = torch.tensor([p for p in range(len(far)) if p not in used][:4], dtype=torch.int32).view(2, 2)
        one, other = binding.apmm_kv_evict(*x.args, near, 400, to.cuda(), recent=9), binding.apmm_kv_evict(*args, apart, 400, where[to.long()].cuda(), recent=9)
        assert all(torch.equal(i, j) for i, j in zip(one, other)) and torch.equal(codes[far], x.codes) and torch.equal(scales[far], x.scales)
        del apart


def test_calls_on_two_streams_at_once(gpu):
    """Each call has its own workspace: calls that overlap give what they give one after the other."""
    torch, binding = gpu
    lengths, new = [4000, 900, 2100], [1, 1, 1]
    b, prompt = Batch(torch, torch.bfloat16, 128, 4, 4, 16, lengths, new, seed=31), Batch(torch, torch.float16, 64, 4, 1, 16, lengths, [300, 900, 40], seed=32)
    codes, scales = torch.randint(0, 16, (1000, 2000), device="cuda", dtype=torch.uint8), torch.rand((1000, 16), device="cuda").half()
    packed, x = binding.apmm_w4_pack(codes, scales, 128), torch.randn((50, 2000), device="cuda").half()
    wide = torch.full((3, 4200), -1, dtype=torch.int32)
    wide[:, :b.table.shape[1]] = b.table
    wide, to = wide.cuda(), torch.full((3, 30), -1, dtype=torch.int32, device="cuda")
    heavy = torch.rand((3, 4, 4000), device="cuda")

    def calls():
        return [binding.apmm_kv_weights(b.q, *b.args, torch.zeros((3, 4, 4000), device="cuda")), binding.apmm_kv_weights(prompt.q, *prompt.args, torch.zeros((3, 4, 4000), device="cuda"), prompt.starts_gpu),
                binding.apmm_w4_gemm(x, packed, 1000, 128), *binding.apmm_kv_evict(b.codes, b.scales, wide, b.args[3], heavy, 400, to, sinks=2, recent=20)]
    want = calls()
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(calls())
    torch.cuda.synchronize()
    assert all(torch.equal(i, j) for some in got for i, j in zip(some, want))
