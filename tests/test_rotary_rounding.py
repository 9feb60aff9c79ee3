"""Rotary positions where rounding decides: pairs that nearly cancel, numbers next to the middle between two of 16 bits, binary16 numbers below 2^-14, products without a place in 32 bits.  Every
number has to be the pair turned in more than 64 bits, rounded to 32 and then to 16, whichever kernel makes it; on the CPU (host_layers.py) and on the GPU."""
import functools

import numpy as np
import pytest
import torch

import host_layers
import host_wave
from test_kv_bounds import cache, rows

TOKENS, HEADS, PAIRS, D = 4, 6, 32, 64
TYPES = [torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    if not host_wave.available():
        pytest.skip("no clang++")
    return host_layers.Host(host_layers.build(tmp_path_factory.mktemp("layers")))


@pytest.fixture(scope="module")
def gpu():
    from paper_2409_17870_amd import binding
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    binding.load()
    return binding


def turned(a, b, t, magnitude=1.0):
    """(a, b) by the angle t, a product of 64 bits, in the 64 bits of extended precision.  (Of pairs that cancel but for 2^-22 it leaves 2^-42 of the result.)"""
    assert np.finfo(np.longdouble).nmant >= 63
    t, a, b, g = np.asarray(t).astype(np.longdouble), a.astype(np.longdouble), b.astype(np.longdouble), np.longdouble(np.float32(magnitude))
    c, s = np.cos(t) * g, np.sin(t) * g
    return a * c - b * s, b * c + a * s


def rounded(y, dtype):
    with np.errstate(over="ignore"):
        return torch.from_numpy(y.astype(np.float32)).to(dtype)


def sixteen(x, dtype):
    """Numbers of 16 bits, as 64."""
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(dtype).double().numpy()


def near_middle(y, dtype):
    """Within two units of 32 bits of the middle between two numbers of 16."""
    low = 16 if dtype == torch.bfloat16 else 13
    bits = np.asarray(y).astype(np.float32).view(np.uint32).astype(np.int64) & ((1 << low) - 1)
    return np.abs(bits - (1 << (low - 1))) <= 2


def angles(seed):
    r = np.random.RandomState(seed)
    positions, frequencies = r.randint(0, 100000, TOKENS).astype(np.int32), 10000.0 ** (-np.arange(PAIRS) / PAIRS)
    return r, positions, frequencies, positions.astype(np.float64)[:, None] * frequencies


@functools.lru_cache(maxsize=None)
def pairs_of(kind, dtype, seed=5):
    """Positions, frequencies, and pairs (tokens x heads x pairs) of the kind for these angles."""
    r, positions, frequencies, t = angles(seed)
    a, b = np.empty((TOKENS, HEADS, PAIRS)), np.empty((TOKENS, HEADS, PAIRS))
    for i in range(TOKENS):
        for j in range(PAIRS):
            n = 4096 if kind == "cancel" else 200000 if dtype == torch.bfloat16 else 30000
            if kind == "cancel":  # the partner that takes most of it away, in 16 bits
                v = sixteen(r.randn(n), dtype)
                u = sixteen(v * np.tan(t[i, j]), dtype)
                y = np.abs(u * np.cos(t[i, j]) - v * np.sin(t[i, j])) / np.abs(v)
                best = np.argsort(np.where(y > 2.0 ** -22, y, np.inf))[:HEADS]
            else:
                size = 2.0 ** -15 if kind == "subnormal" else 1.0
                u, v = sixteen(r.randn(n) * size, dtype), sixteen(r.randn(n) * size, dtype)
                y = u * np.cos(t[i, j]) - v * np.sin(t[i, j])
                if kind == "subnormal":  # the middles lie at odd multiples of 2^-25
                    best = np.argsort(np.abs(np.mod(y * 2.0 ** 24, 1.0) - 0.5))[:HEADS]
                else:
                    best = np.resize(np.flatnonzero(near_middle(y, dtype)), HEADS)  # (some angles have few)
            a[i, :, j], b[i, :, j] = u[best], v[best]
    return positions, frequencies, a, b, *turned(a, b, t[:, None])


def rows_of(a, b, interleaved, dtype):
    x = np.stack([a, b], -1).reshape(*a.shape[:-1], -1) if interleaved else np.concatenate([a, b], -1)
    return torch.from_numpy(x).float().to(dtype)


def guarded(*tensors):
    m = host_wave.Memory()
    return [m.copy(t) for t in tensors]


def on_host(host, x, positions, frequencies, interleaved, magnitude=1.0):
    """By the kernel of rows alone, of eights and of single numbers, and by the one on the way into the cache."""
    p, f = torch.from_numpy(positions), torch.from_numpy(frequencies)
    wide = torch.zeros((*x.shape[:2], x.shape[2] + 3), dtype=x.dtype)
    wide[:, :, 3:] = x
    n, k = x.shape[0], rows(x.shape[0], 1, D, x.dtype)
    g = guarded(x, p, f, wide)
    yield host.rotary(*g[:3], interleaved=interleaved, magnitude=magnitude)
    yield host.rotary(g[3][:, :, 3:], *g[1:3], interleaved=interleaved, magnitude=magnitude)
    k, starts, *args = guarded(k, torch.tensor([0, n], dtype=torch.int32), *cache([n], 1, D, 16, x.dtype))
    yield host.write_rotary(g[0], k, k, *args, g[2], starts, g[1], interleaved=interleaved, magnitude=magnitude)


def on_gpu(binding, x, positions, frequencies, interleaved, magnitude=1.0):
    x, p, f = x.cuda(), torch.from_numpy(positions).cuda(), torch.from_numpy(frequencies).cuda()
    wide = torch.zeros((*x.shape[:2], x.shape[2] + 3), dtype=x.dtype, device="cuda")
    wide[:, :, 3:] = x
    n = x.shape[0]
    k, starts, args = x[:, :1], torch.tensor([0, n], dtype=torch.int32).cuda(), [t.cuda() for t in cache([n], 1, D, 16, x.dtype)]
    one, other = ([args[0].clone(), args[1].clone()] for _ in range(2))
    yield (y := binding.apmm_rotary(x, p, f, interleaved=interleaved, magnitude=magnitude)).cpu()
    yield binding.apmm_rotary(wide[:, :, 3:], p, f, interleaved=interleaved, magnitude=magnitude).cpu()
    yield binding.apmm_kv_write_rotary(x, k, k, *one, *args[2:], f, starts, positions=p, interleaved=interleaved, magnitude=magnitude).cpu()
    binding.apmm_kv_write(y[:, :1], k, *other, *args[2:], starts)
    assert torch.equal(one[0], other[0]) and torch.equal(one[1].view(torch.int16), other[1].view(torch.int16))


def check(turn, where, kind, dtype, interleaved):
    positions, frequencies, a, b, first, second = pairs_of(kind, dtype)
    want = rows_of(rounded(first, dtype).double().numpy(), rounded(second, dtype).double().numpy(), interleaved, dtype)
    if kind == "cancel":  # half of the pairs at least lose 16 bits and more; none is all gone
        assert np.median(np.abs(first) / np.abs(b)) < 2.0 ** -15 and bool((first != 0).all())
    if kind == "middle":
        assert near_middle(first, dtype).mean() > 0.9
    for y in turn(where, rows_of(a, b, interleaved, dtype), positions, frequencies, interleaved):
        wrong = (y != want).sum()
        assert wrong == 0, "%d of %d are not the exact pair's" % (wrong, want.numel())


KINDS = [("cancel", t) for t in TYPES] + [("middle", t) for t in TYPES] + [("subnormal", torch.float16)]


@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("kind, dtype", KINDS)
def test_pairs_on_the_host(host, kind, dtype, interleaved):
    check(on_host, host, kind, dtype, interleaved)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("kind, dtype", KINDS)
def test_pairs_on_the_gpu(gpu, kind, dtype, interleaved):
    check(on_gpu, gpu, kind, dtype, interleaved)


# Pairs of which one number is near a middle that is not among those of normal numbers: position, frequency, a, b
SMALL = [(1, 2.8041749902067479, 0x09c5, 0x054e), (1, 6.1626298429616133, 0x0d92, 0x02f8), (3103, 10000.0 ** (-6 / 32), None, None)]


def small_pairs():
    for position, frequency, a, b in SMALL:
        a, b = (np.array([v], dtype=np.uint16).view(np.float16).astype(np.float64) for v in (a, b)) if a else (np.array([float.fromhex(v)]) for v in ("0x1.82p-17", "-0x1.8fp-16"))
        yield position, frequency, a, b


def check_small(turn, where, interleaved):
    for position, frequency, a, b in small_pairs():
        positions, frequencies = np.array([position], dtype=np.int32), np.full(PAIRS, frequency)
        first, second = (rounded(v, torch.float16) for v in turned(a, b, position * frequency))
        x = rows_of(np.full((1, 1, PAIRS), a), np.full((1, 1, PAIRS), b), interleaved, torch.float16)
        want = rows_of(np.full((1, 1, PAIRS), first.item()), np.full((1, 1, PAIRS), second.item()), interleaved, torch.float16)
        for y in turn(where, x, positions, frequencies, interleaved):
            assert torch.equal(y, want)


@pytest.mark.parametrize("interleaved", [0, 1])
def test_subnormal_pairs_on_the_host(host, interleaved):
    check_small(on_host, host, interleaved)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [0, 1])
def test_subnormal_pairs_on_the_gpu(gpu, interleaved):
    check_small(on_gpu, gpu, interleaved)


def check_large(turn, where, interleaved):
    """The largest bfloat16 numbers: products, and cosines and sines with the magnitude, of which some have no place in 32 bits where their sum has one, and sums that have none."""
    r, positions, frequencies, t = angles(7)
    a, b = (sixteen(np.ldexp(r.uniform(-1, 1, (TOKENS, HEADS, PAIRS)), 128), torch.bfloat16) for _ in range(2))
    a, b = (np.clip(v, -torch.finfo(torch.bfloat16).max, torch.finfo(torch.bfloat16).max) for v in (a, b))
    for magnitude in (1.0, 1.4375, 3e38):
        if magnitude > 2:
            a, b = (np.where(np.arange(PAIRS) % 4 == 1, v, sixteen(np.ldexp(v, -127), torch.bfloat16)) for v in (a, b))
        first, second = turned(a, b, t[:, None], magnitude)
        want = rows_of(rounded(first, torch.bfloat16).double().numpy(), rounded(second, torch.bfloat16).double().numpy(), interleaved, torch.bfloat16)
        assert 0.02 < torch.isinf(want).float().mean() < 0.9
        for y in turn(where, rows_of(a, b, interleaved, torch.bfloat16), positions, frequencies, interleaved, magnitude):
            assert torch.equal(y, want)


@pytest.mark.parametrize("interleaved", [0, 1])
def test_large_pairs_on_the_host(host, interleaved):
    check_large(on_host, host, interleaved)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [0, 1])
def test_large_pairs_on_the_gpu(gpu, interleaved):
    check_large(on_gpu, gpu, interleaved)


# Pairs of large angles of which a number lies so near the middle between two of 32 bits, next to that of two of 16, that the angle's turns have to be right to 2^-50 of a turn: a, b, position, frequency
LARGE_ANGLES = [
    (torch.float16, -1.76171875, -1.337890625, 1002222, 0.1539926526059492), (torch.float16, 0.42236328125, 1.6083984375, 782958, 0.4216965034285822), (torch.float16, 3.947265625, 2.1015625, 727726, 1.0),
    (torch.float16, 1.4150390625, -1.15625, 755405, 0.7498942093324559), (torch.float16, -0.4384765625, 1.14453125, 972351, 0.042169650342858224),
    (torch.float16, 0.22998046875, -2.4296875, 798727, 0.23713737056616552), (torch.bfloat16, 1.296875, 1.8984375, 727513, 0.4216965034285822)]


def check_large_angles(turn, where, interleaved):
    for dtype, a, b, position, frequency in LARGE_ANGLES:
        positions, frequencies = np.array([position], dtype=np.int32), np.full(PAIRS, frequency)
        first, second = (rounded(v, dtype).item() for v in turned(np.array([a]), np.array([b]), position * frequency))
        x, want = (rows_of(np.full((1, 1, PAIRS), v), np.full((1, 1, PAIRS), w), interleaved, dtype) for v, w in ((a, b), (first, second)))
        for y in turn(where, x, positions, frequencies, interleaved):
            assert torch.equal(y, want)


@pytest.mark.parametrize("interleaved", [0, 1])
def test_large_angles_on_the_host(host, interleaved):
    check_large_angles(on_host, host, interleaved)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [0, 1])
def test_large_angles_on_the_gpu(gpu, interleaved):
    check_large_angles(on_gpu, gpu, interleaved)
