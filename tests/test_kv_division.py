"""Sequences, tiles and heads of the key/value cache's kernels are told apart by a multiplication with a reciprocal (apmm_kv.h): against integer division."""
import subprocess

import pytest
import torch

import host_wave
from paper_2409_17870_amd import binding

PROGRAM = r"""
#include <cstdio>
#include "apmm_kv.h"
int main()
{
    const int most = (1ll << 31) - 1;
    long long wrong = 0;
    for (int d = 1; d <= 1024; ++d) {
        const uint64_t m = apmm::kv_divisor(d);
        auto ask = [&](long long x) {
            if (x < 0 || x > most || apmm::kv_divide((int)x, m) == (int)(x / d)) return;
            if (!wrong++) std::printf("%lld / %d: %d\n", x, d, apmm::kv_divide((int)x, m));
        };
        for (long long x = 0; x < 3 * 1024; ++x) ask(x);
        for (int bit = 10; bit <= 31; ++bit)
            for (long long around : {1ll << bit, (1ll << bit) * d, (1ll << bit) / d * d})
                for (int i = -2; i <= 2; ++i) ask(around + i);
        for (long long x = d; x <= most; x += x / 3 + 1) {
            ask(x / d * d);
            ask(x / d * d - 1);
        }
    }
    std::printf("%lld wrong\n", wrong);
}
"""


def test_quotients(tmp_path):
    if not host_wave.available():
        pytest.skip("no clang++")
    out = subprocess.run([host_wave.build(tmp_path, PROGRAM)], capture_output=True, text=True, check=True).stdout
    assert out == "0 wrong\n", out


@pytest.mark.gpu
def test_more_rows_than_24_bits():
    """A prompt of more than 2^24 tokens whose queries see their own key alone: the results are the values, whichever place a row has, within the rounding of the one weight to 11 bits and of
    both sides to 8 (half a unit each is 2^-8 of the number at most)."""
    tokens, ps = (1 << 24) + 4321, 1 << 20
    codes, scales, table, lengths, starts = long_cache(tokens, ps)
    v = binding.apmm_kv_read(codes, scales, table, lengths, tokens, starts)[1].float()
    q = torch.randn((tokens, 2, 64), device="cuda", dtype=torch.bfloat16)
    out = binding.apmm_kv_attention(q, codes, scales, table, lengths, starts, window=1)
    allowed = v.abs() * (2.0 ** -7 + 2.0 ** -10) + 2.0 ** -15
    for h in range(2):
        assert bool(((out[:, h:h + 1].float() - v).abs() <= allowed).all())


@pytest.mark.gpu
def test_more_eights_than_24_bits():
    """More than 2^27 tokens read back in one call: the last ones as from a call of their own."""
    tokens, ps, last = (1 << 27) + 4321, 1 << 20, 5000
    codes, scales, table, lengths, starts = long_cache(tokens, ps)
    out = [torch.full((tokens, 1, 64), float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    binding.apmm_kv_read(codes, scales, table, lengths, tokens, starts, k_out=out[0], v_out=out[1])
    few = binding.apmm_kv_read(codes, scales, table, lengths, last, torch.tensor([0, last], dtype=torch.int32, device="cuda"))
    for a, b in zip(out, few):
        assert torch.equal(a[-last:], b) and not bool(torch.isnan(a[::997]).any())


def long_cache(tokens, ps):
    """One sequence, one head of 64 channels, random codes and scales, pages in reverse order."""
    g = torch.Generator(device="cuda").manual_seed(3)
    pages = -(-tokens // ps)
    codes = torch.randint(0, 256, (pages, 1, 2, ps * 32), generator=g, device="cuda", dtype=torch.uint8)
    scales = (torch.rand((pages, 1, 2, ps), generator=g, device="cuda") + 0.01).bfloat16()
    table = torch.arange(pages - 1, -1, -1, dtype=torch.int32, device="cuda")[None]
    return codes, scales, table, torch.tensor([tokens], dtype=torch.int32, device="cuda"), torch.tensor([0, tokens], dtype=torch.int32, device="cuda")
