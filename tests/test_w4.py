"""Products of 16-bit activations with four-bit weights and group scales, on the GPU against sums in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2409_17870_amd import binding
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    binding.load()
    return torch, binding


def weights(torch, N, K, group, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (N, K), generator=g, dtype=torch.uint8)  # (the upper four bits do not count)
    scales = (torch.rand((N, -(-K // group)), generator=g) * 0.1 + 1e-3).to(dtype)
    return codes, scales


def exact(x, codes, scales, group):
    """The product in 64 bits, and how far sums in 32 bits may be from it: of a group's terms one after the other and of the groups and of what workgroups' waves have, each to 2^-24."""
    K = codes.shape[1]
    w = (2.0 * (codes & 15).double() - 15.0) * scales.double().repeat_interleave(group, 1)[:, :K]
    return x.double() @ w.t(), (group + K // group + 32) * 2.0 ** -24 * (x.double().abs() @ w.abs().t())


def close(torch, got, want, near):
    half, tiny = (2.0 ** -11, 2.0 ** -25) if got.dtype == torch.float16 else (2.0 ** -8, 0.0)
    d = (got.cpu().double() - want).abs()
    bad = ~(d <= near + half * (want.abs() + near) + tiny)
    assert not bool(bad.any()), "%d of %d off, worst %.3g" % (int(bad.sum()), bad.numel(), float(d[bad].max()))


SIZES = [(1, 1, 1), (1, 16, 128), (1, 17, 129), (2, 40, 31), (15, 33, 127), (16, 64, 256), (17, 100, 640), (33, 7, 1000), (48, 130, 95), (64, 257, 512), (65, 96, 384), (100, 300, 200),
         (129, 513, 136), (200, 256, 1024), (256, 1000, 64), (300, 48, 2000), (1, 4096, 2048), (7, 1030, 4100), (31, 600, 130), (32, 40, 4096), (20, 50, 4200), (18, 12400, 70)]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M, N, K", SIZES)
def test_product(gpu, M, N, K, group, dtype):
    torch, binding = gpu
    dt = getattr(torch, dtype)
    codes, scales = weights(torch, N, K, group, dt, M + N + K)
    x = torch.randn((M, K), generator=torch.Generator().manual_seed(M * N)).to(dt)
    packed = binding.apmm_w4_pack(codes.cuda(), scales.cuda(), group)
    y = binding.apmm_w4_gemm(x.cuda(), packed, N, group)
    close(torch, y, *exact(x, codes, scales, group))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("M", [1, 5, 40, 150])
def test_every_code_and_input(gpu, M, dtype):
    """Integers small enough that every sum is exact: one input at a time meets every code; any place that is mixed up shows."""
    torch, binding = gpu
    dt, N, K, group = getattr(torch, dtype), 48, 384, 32
    codes = (torch.arange(N)[:, None] * 5 + torch.arange(K)[None] * 3 + torch.arange(K)[None] // 16).to(torch.uint8)
    scales = (2.0 ** (torch.arange(N)[:, None] % 3 - torch.arange(K // group)[None] % 2)).to(dt)
    x = torch.zeros((M, K), dtype=dt)
    for m in range(M):
        x[m, (m * 37 + torch.arange(5) * 71) % K] = torch.tensor([1.0, -2.0, 3.0, 1.0, -1.0]).to(dt)
    y = binding.apmm_w4_gemm(x.cuda(), binding.apmm_w4_pack(codes.cuda(), scales.cuda(), group), N, group)
    want, _ = exact(x, codes, scales, group)
    assert torch.equal(y.cpu(), want.to(dt))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("M", [3, 70, 300])
def test_rows_at_any_place(gpu, M, dtype):
    """x a slice at an odd address with odd rows, y columns of a wider tensor: what lies around stays."""
    torch, binding = gpu
    dt, N, K, group = getattr(torch, dtype), 130, 261, 64
    codes, scales = weights(torch, N, K, group, dt, 3)
    packed = binding.apmm_w4_pack(codes.cuda(), scales.cuda(), group)
    wide = torch.randn((M, K + 10), generator=torch.Generator().manual_seed(4)).to(dt).cuda()
    wide[:, :3] = wide[:, 3 + K:] = float("nan")
    out = torch.full((M, N + 9), 7.0, dtype=dt, device="cuda")
    y = binding.apmm_w4_gemm(wide[:, 3:3 + K], packed, N, group, out=out[:, 5:5 + N])
    assert y.data_ptr() == out[:, 5:].data_ptr()
    close(torch, y, *exact(wide[:, 3:3 + K].cpu(), codes, scales, group))
    assert bool((out[:, :5] == 7).all()) and bool((out[:, 5 + N:] == 7).all())
    same = binding.apmm_w4_gemm(wide[:1, 3:3 + K].expand(M, K), packed, N, group)  # one row for all
    assert torch.equal(same, y[:1].expand(M, N)) or M > 16  # (many rows are summed in another order than few)
    close(torch, same, *exact(wide[:1, 3:3 + K].cpu().expand(M, K), codes, scales, group))


@pytest.mark.parametrize("M", [1, 20, 200])
def test_numbers_that_are_not_finite(gpu, M):
    """A row with an infinity has infinities of the codes' signs, one with NaN is NaN, others do not notice; results beyond the type's range are infinite."""
    torch, binding = gpu
    N, K, group = 32, 256, 128
    for dt in (torch.float16, torch.bfloat16):
        codes, scales = weights(torch, N, K, group, dt, 5)
        packed = binding.apmm_w4_pack(codes.cuda(), scales.cuda(), group)
        x = torch.randn((M, K), generator=torch.Generator().manual_seed(6)).to(dt)
        clean = binding.apmm_w4_gemm(x.cuda(), packed, N, group).cpu()
        x[0, 130] = float("inf")
        if M > 1:
            x[M - 1, 7] = float("nan")
        y = binding.apmm_w4_gemm(x.cuda(), packed, N, group).cpu()
        sign = torch.where((codes[:, 130] & 15) >= 8, 1.0, -1.0)
        assert torch.equal(y[0], (sign * float("inf")).to(dt))
        if M > 1:
            assert bool(torch.isnan(y[M - 1]).all()) and torch.equal(y[1:M - 1], clean[1:M - 1])
        big = torch.full((M, K), torch.finfo(dt).max, dtype=dt)
        y = binding.apmm_w4_gemm(big.cuda(), packed, N, group).cpu()
        want, near = exact(big, codes, scales, group)
        sure = want.abs() - near > torch.finfo(dt).max * (1 + torch.finfo(dt).eps)
        # where no sum of 32 bits may overflow on the way: a group of 128 terms of up to 15 |x| is at most 1.3e8 for binary16, while one term of bfloat16's largest number, 15 * 3.4e38, has
        # no place in 32 bits, so that infinities of both signs meet there
        sure &= (big.double().abs() @ (2.0 * (codes & 15).double() - 15.0).abs().t()) < torch.finfo(torch.float32).max
        assert bool(sure.any()) == (dt == torch.float16) and torch.equal(y[sure], (want[sure].sign() * float("inf")).to(dt))


def test_graph_streams_and_equal_results(gpu):
    torch, binding = gpu
    for M in (1, 16, 40, 200):
        N, K, group = 600, 1000, 64
        codes, scales = weights(torch, N, K, group, torch.bfloat16, 7)
        packed = binding.apmm_w4_pack(codes.cuda(), scales.cuda(), group)
        x = torch.randn((M, K), generator=torch.Generator().manual_seed(8)).bfloat16().cuda()
        want = binding.apmm_w4_gemm(x, packed, N, group)
        out = torch.zeros_like(want)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            assert torch.equal(binding.apmm_w4_gemm(x, packed, N, group), want)
        torch.cuda.current_stream().wait_stream(stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            binding.apmm_w4_gemm(x, packed, N, group, out=out)
        for i in range(4):
            x.normal_()
            graph.replay()
            assert torch.equal(out, binding.apmm_w4_gemm(x, packed, N, group))


def test_workspace(gpu):
    """Shares of the inputs meet in it: of any contents, reused by calls one after the other, as much as the call asks for."""
    torch, binding = gpu
    N, K, group = 520, 4100, 128
    codes, scales = weights(torch, N, K, group, torch.float16, 11)
    packed = binding.apmm_w4_pack(codes.cuda(), scales.cuda(), group)
    for M in (17, 40, 77, 128, 161):
        need = binding.apmm_w4_workspace_bytes(M, N, K, group)
        assert need > 0
        workspace = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        x = torch.randn((M, K), generator=torch.Generator().manual_seed(M)).half()
        y = binding.apmm_w4_gemm(x.cuda(), packed, N, group, workspace=workspace)
        close(torch, y, *exact(x, codes, scales, group))
        assert torch.equal(y, binding.apmm_w4_gemm(x.cuda(), packed, N, group, workspace=workspace))
        with pytest.raises(binding.ApmmError):
            binding.apmm_w4_gemm(x.cuda(), packed, N, group, workspace=workspace[:-1])
    with pytest.raises(ValueError):
        binding.apmm_w4_gemm(x.cuda(), packed, N, group, workspace=workspace.cpu())


def test_wide_calls(gpu):
    """More channels than one dimension of a launch would have as tiles of tokens, and no tokens or channels at all."""
    torch, binding = gpu
    N, K, group, dt = 70000, 40, 32, torch.float16
    codes, scales = weights(torch, N, K, group, dt, 9)
    packed = binding.apmm_w4_pack(codes.cuda(), scales.cuda(), group)
    x = torch.randn((2, K), generator=torch.Generator().manual_seed(1)).to(dt)
    close(torch, binding.apmm_w4_gemm(x.cuda(), packed, N, group), *exact(x, codes, scales, group))
    assert binding.apmm_w4_gemm(x[:0].cuda(), packed, N, group).shape == (0, N)
    empty = binding.apmm_w4_pack(codes[:0].cuda(), scales[:0].cuda(), group)
    assert binding.apmm_w4_gemm(x.cuda(), empty, 0, group).shape == (2, 0)
    codes, scales = weights(torch, 20, K, group, dt, 9)
    x = torch.randn((9000, K), generator=torch.Generator().manual_seed(1)).to(dt)
    close(torch, binding.apmm_w4_gemm(x.cuda(), binding.apmm_w4_pack(codes.cuda(), scales.cuda(), group), 20, group), *exact(x, codes, scales, group))


def test_refusals(gpu):
    torch, binding = gpu
    codes, scales = weights(torch, 32, 128, 64, torch.float16, 1)
    codes, scales = codes.cuda(), scales.cuda()
    packed = binding.apmm_w4_pack(codes, scales, 64)
    x = torch.zeros((4, 128), dtype=torch.float16, device="cuda")
    for bad in (lambda: binding.apmm_w4_pack(codes, scales, 32), lambda: binding.apmm_w4_pack(codes, scales.float(), 64), lambda: binding.apmm_w4_pack(codes.cpu(), scales, 64),
                lambda: binding.apmm_w4_pack(codes, scales, 64, out=packed[:-1]), lambda: binding.apmm_w4_gemm(x.float(), packed, 32, 64), lambda: binding.apmm_w4_gemm(x, packed, 48, 64),
                lambda: binding.apmm_w4_gemm(x.cpu(), packed, 32, 64), lambda: binding.apmm_w4_gemm(x.t(), packed, 32, 64), lambda: binding.apmm_w4_gemm(x[:, ::2], packed, 32, 64),
                lambda: binding.apmm_w4_gemm(x, packed, 32, 64, out=torch.empty((4, 32), device="cuda")), lambda: binding.apmm_w4_gemm(x, packed.cpu(), 32, 64)):
        with pytest.raises((ValueError, binding.ApmmError)):
            bad()
    with pytest.raises(binding.ApmmError):
        binding.apmm_w4_pack(codes, torch.zeros((32, 3), dtype=torch.float16, device="cuda"), 48)


def test_offsets_beyond_32_bits(gpu):
    """Rows of x and y so far apart that the last ones begin beyond 2^32 elements."""
    torch, binding = gpu
    N, K, group = 40, 300, 64
    codes, scales = weights(torch, N, K, group, torch.float16, 12)
    packed = binding.apmm_w4_pack(codes.cuda(), scales.cuda(), group)
    for M, stride in ((9, 1 << 29), (33, 1 << 27), (2100, 1 << 21)):
        x = torch.randn((M, K), generator=torch.Generator().manual_seed(M)).half().cuda()
        far = torch.empty((M - 1) * stride + 512, dtype=torch.float16, device="cuda")
        rows, out = far.as_strided((M, K), (stride, 1)), far[400:].as_strided((M, N), (stride, 1))  # (results behind their row)
        rows.copy_(x)
        assert torch.equal(binding.apmm_w4_gemm(rows, packed, N, group, out=out), binding.apmm_w4_gemm(x, packed, N, group)) and torch.equal(rows, x)
        del far, rows, out
