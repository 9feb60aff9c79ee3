"""Products with four-bit weights on the CPU (host_layers.py), where codes, scales, packed weights, activations, results and workspace lie between pages that cannot be touched and loads to LDS arrive no
sooner than they are waited for: every kernel at the remainders of tokens, channels and inputs, against 64 bits."""
import pytest
import torch

import host_layers
import host_wave
from test_w4 import close, exact, weights


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    if not host_wave.available():
        pytest.skip("no clang++")
    return host_layers.Products(host_layers.build(tmp_path_factory.mktemp("products"), host_layers.PRODUCTS))


def rows(M, K, stride, dtype, seed, aligned):
    """M rows `stride` apart with NaN between, of which the last one ends where memory does; their address a multiple of 16 bytes, or (rows at any address) the end one."""
    n = (M - 1) * stride + K
    before = 0 if aligned else -n % 8
    x = host_wave.Memory().empty((before + n,), dtype).fill_(float("nan"))[before:].as_strided((M, K), (stride, 1))
    return x.copy_(torch.randn((M, K), generator=torch.Generator().manual_seed(seed)).to(dtype))


# M: few tokens by one and two blocks of them; tiles of 1, 2, 3 and 4 blocks.  K: none of an eight, cut eights, cut blocks, whole ones; rings that are filled and not
FEW = [(1, 1, 1), (1, 17, 7), (3, 40, 9), (15, 33, 127), (16, 49, 129), (5, 800, 136), (17, 20, 255), (32, 40, 130), (2, 20, 8200), (31, 1000, 64)]
MANY = [(33, 1, 1), (33, 129, 7), (34, 40, 129), (48, 20, 4200), (65, 130, 1030), (97, 33, 264), (128, 20, 1161), (193, 40, 136), (200, 20, 515), (289, 33, 255), (300, 20, 640),
        (100, 20, 2180), (200, 24, 2176), (290, 16, 2049)]


def call(host, M, N, K, group, dtype, aligned):
    codes, scales = (host_wave.Memory().copy(t) for t in weights(torch, N, K, group, dtype, M + N + K))
    x = rows(M, K, -(-K // 8) * 8 + 8 if aligned else K + 3, dtype, M * N + K, aligned)
    y = host_wave.Memory().empty((M, N), dtype).fill_(float("nan"))
    packed = host.pack(codes, scales, group)
    close(torch, host.gemm(x, packed, N, group, y), *exact(x, codes, scales, group))


@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("M, N, K", FEW)
def test_few_tokens(host, M, N, K, aligned):
    for group, dtype in ((32, torch.float16), (64, torch.bfloat16), (128, torch.float16)):
        call(host, M, N, K, group, dtype, aligned)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("M, N, K", MANY)
def test_many_tokens(host, M, N, K, aligned, group):
    call(host, M, N, K, group, torch.bfloat16 if (M + group // 32) % 2 else torch.float16, aligned)


def test_inputs_are_cut_and_whole(host):
    """The list has both of tiles of every size (of so few channels as many blocks of 32 tokens as 96 tokens more ask for): as many bytes of workspace as shares have results."""
    shares = {(M, N, K): host.lib.apmm_w4_workspace_bytes(M, N, K, 64) // (M * (-(-N // 4) * 4) * 4) for M, N, K in MANY}
    for blocks in (1, 2, 3, 4):
        of = [n for (M, _, _), n in shares.items() if min(4, -(-M // 96)) == blocks]
        assert 0 in of and max(of) > 1
    assert not any(host.lib.apmm_w4_workspace_bytes(M, N, K, 64) for M, N, K in FEW)
