"""Calls of more work than a launch takes (2^32 work items) are refused before it, on the host; the largest ones below are not."""
import subprocess

import pytest

import host_wave
from test_abi import lib  # noqa: F401  (the fixture)
from test_kv_abi import UNSUPPORTED, attention, pair, structs

# sequences, tokens, key/value heads, channels of one, query heads to one: workgroups of writes and reads
WRITES = [(3, (1 << 19) - 8 * 8, 1024, 128), (1, (1 << 29) - 8 * 400, 1, 64), (65536, 65536, 1023, 128), (65536, 65536, 1024, 64)]
TOO_MANY = [(3, 1 << 19, 1024, 128), (1, 1 << 29, 1, 64), (65536, 65536, 1024, 128), (65536, 1 << 21, 1024, 64)]
# of attention: single tokens, tiles
ATTENDED = [(65536, 65536, 255, 128, 1), (1, 1 << 20, 511, 64, 1)]
NOT_ATTENDED = [(65536, 65536, 256, 128, 1), (32768, 32768, 512, 64, 16)]

PROGRAM = r"""
#include <cstdio>
#include "apmm_kv.h"
int main()
{
    long long sequences, tokens, heads, head_dim, groups;
    while (std::scanf("%lld %lld %lld %lld %lld", &sequences, &tokens, &heads, &head_dim, &groups) == 5) {
        apmm::KvArgs a = {};
        a.sequences = sequences; a.tokens = tokens; a.heads = heads; a.head_dim = head_dim; a.page_shift = 4; a.width = 100;
        std::printf("%lld\n", (long long)(groups ? apmm::kv_attention_items(apmm::kv_plan(a, groups, 0, 0), heads) : apmm::kv_store_items(a)));
    }
}
"""


def batch(sequences, tokens, heads, head_dim):
    return dict(kv_heads=heads, head_dim=head_dim), dict(sequences=sequences, tokens=tokens)


@pytest.mark.parametrize("sizes", TOO_MANY)
def test_writes_and_reads_are_refused(lib, sizes):  # noqa: F811
    for fn in (lib.apmm_kv_write, lib.apmm_kv_read):
        assert pair(fn, *batch(*sizes)) == UNSUPPORTED


@pytest.mark.parametrize("sizes", NOT_ATTENDED)
def test_attention_is_refused(lib, sizes):  # noqa: F811
    *sizes, groups = sizes
    c, b = batch(*sizes)
    assert attention(lib, c, b, q_heads=sizes[2] * groups) == UNSUPPORTED
    assert lib.apmm_kv_attention_workspace_bytes(*structs(c, b), sizes[2] * groups) == 0


def test_where_the_line_is(tmp_path):
    if not host_wave.available():
        pytest.skip("no clang++")
    cases = [(*s, 0) for s in WRITES] + ATTENDED, [(*s, 0) for s in TOO_MANY] + NOT_ATTENDED
    path = host_wave.build(tmp_path, PROGRAM)
    for below, some in zip((True, False), cases):
        out = subprocess.run([path], input="".join("%d %d %d %d %d\n" % s for s in some), capture_output=True, text=True, check=True).stdout.split()
        assert len(out) == len(some)
        for s, n in zip(some, out):
            assert (int(n) < 1 << 32) == below, (s, n)
