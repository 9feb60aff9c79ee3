"""Codes and scales of rows of any bit patterns, as the definition in exact arithmetic has them, on the CPU (host_wave.py) and the GPU."""
import pytest
import torch

import host_wave
import kv_reference as ref
from paper_2409_17870_amd import binding
from test_kv_bounds import cache, host  # noqa: F401  (host: the fixture)


def patterns(dtype, D, n=400):
    """Random bits (all exponents within a row), numbers around the smallest ones, and the largest beside the smallest of either sign."""
    g = torch.Generator().manual_seed(D)
    info = torch.finfo(dtype)
    bits = torch.randint(-2 ** 15, 2 ** 15, (n, 1, D), generator=g, dtype=torch.int32).to(torch.int16).view(dtype)
    bits[::4] = torch.nan_to_num(bits[::4], nan=1.0, posinf=2.0, neginf=-2.0)
    near = [(torch.randn((40, 1, D), generator=g) * info.smallest_normal * f).to(dtype) for f in (0.01, 1.0, 100.0)]
    apart = (torch.randint(-9, 10, (60, 1, D), generator=g) * info.smallest_normal * info.eps).to(dtype)
    for i in range(60):
        apart[i, 0, i] = info.max * 2.0 ** (-4 * i) if dtype == torch.bfloat16 else info.max * 2.0 ** (-i % 30)
    return torch.cat([bits, *near, apart])


def expect(args, x, y, ps):
    """The cache holds x and y, as exact arithmetic has them."""
    codes, scales, table = (t.cpu() for t in args[:3])
    at = torch.arange(x.shape[0])
    page, at = table[0].long()[at // ps], at % ps
    for i, rows in enumerate((x, y)):
        want_codes, want_scales = ref.quantise(rows)
        got_codes, got_scales = ref.unlayout(codes, ps)[i][page, :, at], scales[page, :, i, at]
        finite = torch.isfinite(want_scales)
        assert torch.equal(torch.isnan(got_scales), ~finite)
        assert torch.equal(got_scales[finite], want_scales[finite]) and torch.equal(got_codes[finite], want_codes[finite])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
def test_on_the_host(host, D, dtype):  # noqa: F811
    x = patterns(dtype, D)
    m, y = host_wave.Memory(), x.flip(0)
    args = [m.copy(t) for t in cache([x.shape[0]], 1, D, 16, dtype)]
    host.write(m.copy(x), m.copy(y), *args, torch.tensor([0, x.shape[0]], dtype=torch.int32))
    expect(args, x, y, 16)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
def test_on_the_gpu(D, dtype):
    x = patterns(dtype, D)
    y, args = x.flip(0), [t.cuda() for t in cache([x.shape[0]], 1, D, 16, dtype)]
    binding.apmm_kv_write(x.cuda(), y.cuda(), *args, torch.tensor([0, x.shape[0]], dtype=torch.int32).cuda())
    expect(args, x, y, 16)
