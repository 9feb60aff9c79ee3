"""How attention calls are cut: the host's rules of sizes on both sides of their lines (apmm_kv_attention.hip), asked on the host."""
import subprocess

import pytest

import host_wave

PROGRAM = r"""
#include <cstdio>
#include "apmm_kv.h"
int main()
{
    long long sequences, tokens, heads, groups, longest, window, sinks;
    while (std::scanf("%lld %lld %lld %lld %lld %lld %lld", &sequences, &tokens, &heads, &groups, &longest, &window, &sinks) == 7) {
        apmm::KvArgs a = {};
        a.sequences = sequences; a.tokens = tokens; a.heads = heads; a.head_dim = 128; a.page_shift = 4; a.width = (longest + 15) / 16;
        const apmm::KvPlan p = apmm::kv_plan(a, groups, window, sinks);
        std::printf("%d %d\n", p.tiles.tile ? p.tiles.target != 0 : -1, p.rows.tile ? p.rows.target != 0 : -1);
    }
}
"""
CASES = [  # sequences, new tokens, heads, groups, longest, window, sinks: whether tiles are cut (None: there are none)
    (1, 4096, 8, 1, 4096, 0, 0, True), (1, 4096, 9, 1, 4096, 0, 0, False), (1, 2000, 32, 1, 2000, 0, 0, False), (1, 500, 64, 1, 8000, 0, 0, True), (1, 500, 72, 1, 8000, 0, 0, False),
    (1, 500, 72, 1, 8000, 4096, 0, False), (1, 500, 64, 1, 8000, 4096, 0, True), (1, 1000, 8, 1, 1000, 0, 0, False),
    (2, 2000, 8, 4, 9000, 2048, 16, False), (2, 1600, 8, 4, 9000, 2048, 16, True),                  # a window of 68 steps: 896 tiles
    (15, 960, 32, 1, 9000, 2048, 0, False), (15, 960, 32, 1, 9000, 4096, 0, True), (25, 1600, 32, 1, 9000, 8192, 0, True),  # of 131 and more: as without
    (61, 3904, 32, 1, 8000, 0, 0, True), (101, 6464, 32, 1, 8000, 0, 0, False), (101, 6464, 32, 1, 8000, 8192, 0, False),
    (2, 2, 8, 4, 9000, 0, 0, None),
]


def test_where_tiles_are_cut(tmp_path):
    if not host_wave.available():
        pytest.skip("no clang++")
    out = subprocess.run([host_wave.build(tmp_path, PROGRAM)], input="".join("%d %d %d %d %d %d %d\n" % c[:7] for c in CASES), capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(out) == len(CASES)
    for c, line in zip(CASES, out):
        assert {"-1": None, "0": False, "1": True}[line.split()[0]] is c[7], (c, line)
