"""Rotary positions, on the GPU against turns in 64 bits; and on their way into the four-bit cache against the calls one by one."""
import pytest

from test_kv import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2409_17870_amd import binding
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    binding.load()
    return torch, binding


def exact(torch, x, positions, frequencies, interleaved, magnitude, inverse=False):
    """Rows turned in 64 bits, and how far turns in 32 bits may be from it: cosine and sine to 4 units of their last place (2^-23 each) and their product with the magnitude to one, a product and
    a sum to half of one each."""
    x, pairs = x.double(), frequencies.shape[0]
    t = positions.double()[:, None, None] * frequencies.double().cpu()
    c, s = torch.cos(t) * magnitude, torch.sin(t) * magnitude * (-1 if inverse else 1)
    i = torch.arange(pairs)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
    y, near = x.clone(), torch.zeros_like(x)
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    near[..., first] = near[..., second] = 6 * 2.0 ** -23 * magnitude * (a.abs() + b.abs())
    return y, near


def close(torch, got, want, near):
    half, tiny = (2.0 ** -11, 2.0 ** -25) if got.dtype == torch.float16 else (2.0 ** -8, 0.0)
    d = (got.cpu().double() - want).abs()
    bad = ~(d <= near + half * (want.abs() + near) + tiny)
    assert not bool(bad.any()), "%d of %d off, worst %.3g" % (int(bad.sum()), bad.numel(), float(d[bad].max()))


SHAPES = [  # tokens, heads, head_dim, pairs
    (1, 1, 2, 1), (3, 5, 64, 32), (7, 3, 128, 64), (5, 2, 128, 32), (4, 9, 96, 48), (2, 3, 80, 20), (6, 1, 128, 10), (3, 4, 7, 3), (2, 2, 1024, 512), (1500, 3, 64, 16), (2100, 2, 16, 3), (1, 70, 256, 128)]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_rows(gpu, shape, interleaved, dtype):
    torch, binding = gpu
    tokens, heads, D, pairs = shape
    dt = getattr(torch, dtype)
    g = torch.Generator().manual_seed(tokens + D)
    x = torch.randn((tokens, heads, D), generator=g).to(dt)
    at = torch.randint(-5, 1 << 20, (tokens,), generator=g, dtype=torch.int32)
    at[0] = 0
    f = binding.apmm_rotary_frequencies(2 * pairs)
    for inverse, magnitude in ((False, 1.0), (True, 1.25)):
        y = binding.apmm_rotary(x.cuda(), at.cuda(), f, interleaved=interleaved, magnitude=magnitude, inverse=inverse)
        close(torch, y, *exact(torch, x, at, f, interleaved, magnitude, inverse))
        assert torch.equal(y[:, :, 2 * pairs:].cpu(), x[:, :, 2 * pairs:])
    z = x.cuda()
    assert binding.apmm_rotary(z, at.cuda(), f, interleaved=interleaved, magnitude=1.25, inverse=True, out=z) is z and torch.equal(z, y)  # where they lie
    wide = torch.full((tokens, heads + 2, D + 8 + 3), float("nan"), dtype=dt, device="cuda")  # rows at odd addresses
    part = wide[:, 1:1 + heads, 3:3 + D]
    part.copy_(x)
    out = torch.full_like(wide, 5.0)
    binding.apmm_rotary(part, at.cuda(), f, interleaved=interleaved, magnitude=1.25, inverse=True, out=out[:, 1:1 + heads, 3:3 + D])
    assert torch.equal(out[:, 1:1 + heads, 3:3 + D], y)
    out[:, 1:1 + heads, 3:3 + D] = 5.0
    assert bool((out == 5).all())


def test_far_positions(gpu):
    """Frequencies of a radian and less at positions up to 2^31: an angle in 32 bits would be any."""
    torch, binding = gpu
    at = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 16777217, -1], dtype=torch.int32)
    f = torch.tensor([1.0, 0.7, 1e-3, 3.0], dtype=torch.float64).cuda()
    x = torch.randn((5, 2, 8), generator=torch.Generator().manual_seed(1)).half()
    y = binding.apmm_rotary(x.cuda(), at.cuda(), f)
    want, near = exact(torch, x, at, f, False, 1.0)
    # the product in 64 bits: 2^31 * 3 / (2 pi) turns, to 2^-53 of that each in the frequency's quotient and the product, and as much in the reference's
    near += 6.3 * 2.0 ** 30 * 4 * 2.0 ** -53 * (x.double().abs().sum(-1, keepdim=True))
    close(torch, y, want, near)


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(gpu, interleaved):
    """The inverse is the gradient: of the formula's, in 64 bits, by automatic differentiation and by differences."""
    torch, binding = gpu
    g = torch.Generator().manual_seed(2)
    x, dy = (torch.randn((6, 3, 32), generator=g).bfloat16() for _ in range(2))
    at, f = torch.randint(0, 5000, (6,), generator=g, dtype=torch.int32), binding.apmm_rotary_frequencies(24)
    leaf = x.double().requires_grad_()
    y, _ = exact(torch, leaf, at, f, interleaved, 1.5)
    y.backward(dy.double())
    _, near = exact(torch, dy, at, f, interleaved, 1.5)
    got = binding.apmm_rotary(dy.cuda(), at.cuda(), f, interleaved=interleaved, magnitude=1.5, inverse=True)
    close(torch, got, leaf.grad, near)
    v = torch.randn(x.shape, generator=g).double()
    up, down = (exact(torch, x.double() + e * v, at, f, interleaved, 1.5)[0] for e in (1e-4, -1e-4))
    by_difference = ((up - down) / 2e-4 * dy.double()).sum()
    assert abs(float(by_difference - (got.cpu().double() * v).sum())) <= float(((near + 2.0 ** -8 * leaf.grad.abs()) * v.abs()).sum()) + 1e-8


def test_frequencies(gpu):
    torch, binding = gpu
    f = binding.apmm_rotary_frequencies(128, base=5e5, device="cpu")
    assert f.dtype == torch.float64 and f.shape == (64,) and f[0] == 1.0 and abs(float(f[32]) - 5e5 ** -0.5) < 1e-15
    assert torch.equal(binding.apmm_rotary_frequencies(128, base=5e5, factor=4.0, device="cpu"), f / 4)
    g = binding.apmm_rotary_frequencies(128, base=5e5, factor=4.0, original=8192, device="cpu")
    turns = f * 8192 / (2 * 3.141592653589793)
    assert torch.equal(g[turns >= 32], f[turns >= 32]) and torch.allclose(g[turns <= 1], f[turns <= 1] / 4, rtol=1e-15)
    assert bool((g <= f).all()) and bool((g >= f / 4).all()) and bool((g[1:] < g[:-1]).all())


STORES = [  # D, heads, groups, page, lengths, new, pairs, interleaved
    (128, 1, 1, 16, [1], [1], 64, False),
    (128, 8, 4, 16, [777, 5, 0, 16], [1, 1, 1, 1], 64, True),
    (64, 3, 2, 16, [9, 8, 7, 16, 17, 33], [9, 1, 7, 16, 2, 20], 32, False),
    (128, 5, 1, 64, [130, 64, 1, 0, 200], [130, 3, 1, 2, 17], 32, False),   # one sequence without a place for its two tokens
    (64, 2, 3, 32, [100] * 70, [1] * 70, 12, False),                         # pairs that are no eights; more sequences than lanes
    (128, 2, 2, 256, [300, 300], [44, 300], 13, True),
    (64, 32, 1, 16, [1500, 777], [1490, 777], 16, True),
    (64, 32, 1, 16, [1500, 777], [1490, 777], 32, False),
]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("case", range(len(STORES)))
def test_store_is_the_calls_one_by_one(gpu, case, dtype):
    torch, binding = gpu
    D, heads, groups, ps, lengths, new, pairs, interleaved = STORES[case]
    b = Batch(torch, getattr(torch, dtype), D, heads, groups, ps, lengths, new, seed=case)
    f = binding.apmm_rotary_frequencies(2 * pairs)
    g = torch.Generator().manual_seed(case)
    given = torch.randint(0, 100000, (b.tokens,), generator=g, dtype=torch.int32).cuda()
    places = torch.cat([torch.arange(n, dtype=torch.int32) + (length - n) for length, n in zip(lengths, new)]).cuda()
    for at in (given, None):
        one, other = ((b.codes.clone(), b.scales.clone()) for _ in range(2))
        positions = places if at is None else at
        q, k = (binding.apmm_rotary(x, positions, f, interleaved=interleaved, magnitude=1.1) for x in (b.q, b.k))
        binding.apmm_kv_write(k, b.v, *one, *b.args[2:], b.starts_gpu)
        got = binding.apmm_kv_write_rotary(b.q, b.k, b.v, *other, *b.args[2:], f, b.starts_gpu, positions=at, interleaved=interleaved, magnitude=1.1)
        assert torch.equal(got, q)
        assert torch.equal(one[0], other[0]) and torch.equal(one[1], other[1])
    before = b.q.clone()  # queries turned where they lie, and no queries at all
    here = binding.apmm_kv_write_rotary(b.q, b.k, b.v, *other, *b.args[2:], f, b.starts_gpu, interleaved=interleaved, magnitude=1.1, q_out=b.q)
    assert here is b.q and torch.equal(b.q, q) and not torch.equal(before, b.q)
    third = b.codes.clone(), b.scales.clone()
    assert binding.apmm_kv_write_rotary(None, b.k, b.v, *third, *b.args[2:], f, b.starts_gpu, interleaved=interleaved, magnitude=1.1) is None
    assert torch.equal(third[0], one[0]) and torch.equal(third[1], one[1])


def test_store_one_token_each_and_rows_at_odd_addresses(gpu):
    torch, binding = gpu
    b = Batch(torch, torch.float16, 64, 2, 3, 16, [5, 40, 17], [1, 1, 1], seed=3)
    f = binding.apmm_rotary_frequencies(64)
    one, other = ((b.codes.clone(), b.scales.clone()) for _ in range(2))
    q = binding.apmm_kv_write_rotary(b.q, b.k, b.v, *one, *b.args[2:], f)  # without starts: a token each
    wide = torch.zeros((3, 10, 67), dtype=torch.float16, device="cuda")
    wide[:, :, 3:].copy_(torch.cat([b.q, b.k, b.v], 1))
    x = wide[:, :, 3:]
    out = torch.full((3, 6, 65), 9.0, dtype=torch.float16, device="cuda")
    binding.apmm_kv_write_rotary(x[:, :6], x[:, 6:8], x[:, 8:], *other, *b.args[2:], f, b.starts_gpu, q_out=out[:, :, 1:])
    assert torch.equal(out[:, :, 1:], q) and bool((out[:, :, 0] == 9).all())
    assert torch.equal(one[0], other[0]) and torch.equal(one[1], other[1])


def test_rows_of_no_sequence_and_of_no_page_stay(gpu):
    torch, binding = gpu
    b = Batch(torch, torch.bfloat16, 128, 2, 1, 16, [20, 40], [10, 12], seed=4)
    f = binding.apmm_rotary_frequencies(128)
    starts = torch.tensor([2, 9, 9], dtype=torch.int32).cuda()       # rows 2 to 8 are the first sequence's, the second has none
    table = b.args[2].clone()
    table[0, 1] = 10 ** 6                                            # its second page is none
    codes, scales = b.codes.clone(), b.scales.clone()
    out = torch.full(b.q.shape, 3.0, dtype=torch.bfloat16, device="cuda")
    binding.apmm_kv_write_rotary(b.q, b.k, b.v, codes, scales, table, b.args[3], f, starts, q_out=out)
    at = torch.arange(13, 20, dtype=torch.int32, device="cuda")
    assert torch.equal(out[2:9], binding.apmm_rotary(b.q[2:9], at, f)) and bool((out[:2] == 3).all()) and bool((out[9:] == 3).all())
    first = int(table[0, 0])
    for t, before in ((codes, b.codes), (scales, b.scales)):
        changed = (t != before).flatten(1).any(1).nonzero().flatten().tolist()
        assert changed == [first]


def test_graph(gpu):
    torch, binding = gpu
    b = Batch(torch, torch.bfloat16, 128, 4, 2, 16, [33, 7, 100], [1, 1, 1], seed=5)
    f = binding.apmm_rotary_frequencies(128)
    x, (k, v), at = b.q.contiguous(), (b.k.contiguous(), b.v.contiguous()), torch.tensor([5, 6, 7], dtype=torch.int32).cuda()
    q_out, y = torch.zeros_like(x), torch.zeros_like(x)
    codes, scales = b.codes.clone(), b.scales.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.apmm_rotary(x, at, f, out=y)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.apmm_rotary(x, at, f, out=y)
        binding.apmm_kv_write_rotary(x, k, v, codes, scales, *b.args[2:], f, positions=at, q_out=q_out)
    for _ in range(3):
        x.normal_()
        k.normal_()
        at.add_(1000)
        graph.replay()
        want = codes.clone(), scales.clone()
        assert torch.equal(y, binding.apmm_rotary(x, at, f)) and torch.equal(q_out, y)
        binding.apmm_kv_write(binding.apmm_rotary(k, at, f), v, *want, *b.args[2:])
        assert torch.equal(want[0], codes) and torch.equal(want[1], scales)


def test_refusals(gpu):
    torch, binding = gpu
    x, at, f = torch.zeros((3, 2, 64), dtype=torch.float16, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"), binding.apmm_rotary_frequencies(64)
    for bad in (lambda: binding.apmm_rotary(x.float(), at, f), lambda: binding.apmm_rotary(x[:, :, ::2], at, f), lambda: binding.apmm_rotary(x, at.long(), f), lambda: binding.apmm_rotary(x, at[:2], f),
                lambda: binding.apmm_rotary(x, at, f.float()), lambda: binding.apmm_rotary(x, at, f.cpu()), lambda: binding.apmm_rotary(x, at, f, out=x[:2]), lambda: binding.apmm_rotary(x.cpu(), at, f),
                lambda: binding.apmm_rotary(x, at, binding.apmm_rotary_frequencies(66)), lambda: binding.apmm_rotary(x, at, f, magnitude=0.0),
                lambda: binding.apmm_rotary(x, at, f, out=torch.as_strided(x, (3, 2, 64), (128, 32, 1)))):
        with pytest.raises((ValueError, binding.ApmmError)):
            bad()
    with pytest.raises(ValueError):
        binding.apmm_rotary_frequencies(7)


def test_offsets_beyond_32_bits(gpu):
    """Rows so far apart that the last ones begin beyond 2^32 elements."""
    torch, binding = gpu
    x = torch.randn((17, 3, 64), generator=torch.Generator().manual_seed(3)).half().cuda()
    at, f = torch.arange(17, dtype=torch.int32, device="cuda"), binding.apmm_rotary_frequencies(64)
    far = torch.empty((1 << 32) + (1 << 28), dtype=torch.float16, device="cuda").as_strided(x.shape, (1 << 28, 1 << 20, 1))
    far.copy_(x)
    want = binding.apmm_rotary(x, at, f)
    assert torch.equal(binding.apmm_rotary(far, at, f), want) and torch.equal(binding.apmm_rotary(far, at, f, out=far), want)


@pytest.mark.parametrize("interleaved", [False, True])
def test_numbers_that_are_not_finite(gpu, interleaved):
    """An infinity goes where the formula takes it, with the signs of cosine and sine, two of a pair that cancel and NaN give NaN; other pairs do not notice."""
    torch, binding = gpu
    inf, nan = float("inf"), float("nan")
    for dt in (torch.float16, torch.bfloat16):
        x = torch.randn((6, 2, 64), generator=torch.Generator().manual_seed(7)).to(dt)
        at, f = torch.tensor([1, 2, 3, 4, 5, 6], dtype=torch.int32), binding.apmm_rotary_frequencies(64)
        clean = binding.apmm_rotary(x.cuda(), at.cuda(), f, interleaved=interleaved).cpu()
        x[0, 0, 3], x[1, 1, 40], x[2, 0, 10], x[3, 0, 11], x[4, 1, 32], x[4, 1, 33], x[4, 1, 0], x[4, 1, 1] = inf, -inf, nan, inf, inf, -inf, inf, inf
        x[5, 0, 5] = torch.finfo(dt).max
        y = binding.apmm_rotary(x.cuda(), at.cuda(), f, interleaved=interleaved).cpu()
        want, _ = exact(torch, x, at, f, interleaved, 1.0)
        odd = ~torch.isfinite(want)
        assert bool(odd.any()) and torch.equal(torch.nan_to_num(y[odd].double(), 1.0, 2.0, 3.0), torch.nan_to_num(want[odd], 1.0, 2.0, 3.0))
        same = x == x
        partner = torch.ones_like(same)
        for row, head, channel in torch.nonzero(~torch.isfinite(x) | (x == torch.finfo(dt).max)).tolist():
            other = channel ^ 1 if interleaved else channel ^ 32
            partner[row, head, channel] = partner[row, head, other] = False
        assert torch.equal(y[partner], clean[partner])
