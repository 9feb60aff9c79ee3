"""Host-side checks of the entry points for rotary positions, the cache's budget and four-bit weights with group scales that need no GPU: argument errors come before any launch, sizes, registers of the
kernels."""
import ctypes
import re

import pytest

from test_abi import lib  # noqa: F401  (the fixture)
from test_code_object import code_objects, kernels  # noqa: F401
from test_kv_abi import REFUSED, structs

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 4


def rotation(**change):
    from paper_2409_17870_amd.binding import ApmmRotation
    return ApmmRotation(**{**dict(frequencies=0x8000, pairs=32, interleaved=0, magnitude=1.0), **change})


def rotary(lib, tokens=0, heads=4, head_dim=64, dtype=0, x=0x6000, at=0x9000, r={}, out=0x7000, strides=(256, 64), out_strides=(256, 64)):
    return lib.apmm_rotary(tokens, heads, head_dim, dtype, x, *strides, at, rotation(**r), 0, out, *out_strides, None)


def store(lib, cache={}, batch={}, q_heads=0, at=None, r={}, q=0xa000, q_out=0xb000, k=0x6000, v=0x7000, q_strides=(4096, 128), out_strides=(4096, 128)):
    return lib.apmm_kv_write_rotary(*structs(cache, batch), q_heads, at, rotation(**r), q, *q_strides, q_out, *out_strides, k, 1024, 128, v, 1024, 128, None)


def weigh(lib, cache={}, batch={}, q_heads=32, q=0x6000, w=0x7000, strides=(8192, 1000), capacity=1000, decay=1.0, scale=0.1, window=0, sinks=0, workspace=None, size=0):
    return lib.apmm_kv_weights(*structs(cache, batch), q_heads, q, 4096, 128, w, *strides, capacity, decay, scale, window, sinks, workspace, size, None)


def evict(lib, cache={}, sequences=3, lengths=0x3000, table=0x5000, width=10, w=0x7000, strides=(8192, 1000), capacity=1000, budget=64, sinks=0, recent=0, to=0x5800, to_stride=4, to_width=4,
          to_lengths=0x9000, kept=0xa000, to_weights=0xb000, workspace=None, size=0):
    return lib.apmm_kv_evict(structs(cache)[0], sequences, lengths, table, width, width, w, *strides, capacity, budget, sinks, recent, to, to_stride, to_width, to_lengths, kept, to_weights, workspace,
                             size, None)


@pytest.mark.parametrize("status, cache, batch", REFUSED)
def test_caches_and_batches_that_are_refused(lib, status, cache, batch):  # noqa: F811
    assert store(lib, cache, batch) == status
    assert weigh(lib, cache, batch, q_heads=4 * cache.get("kv_heads", 8)) == status
    if not batch:
        assert evict(lib, cache) == status
    assert lib.apmm_last_error()


def test_rotary(lib):  # noqa: F811
    assert rotary(lib) == OK and rotary(lib, tokens=3, heads=0) == OK
    for status, change in [(INVALID, dict(tokens=-1)), (INVALID, dict(heads=-1)), (INVALID, dict(head_dim=0)), (INVALID, dict(dtype=2)), (UNSUPPORTED, dict(tokens=(1 << 30) + 1)),
                           (UNSUPPORTED, dict(heads=65537)), (UNSUPPORTED, dict(head_dim=1025)), (INVALID, dict(r=dict(pairs=0))), (INVALID, dict(r=dict(pairs=33))), (INVALID, dict(r=dict(frequencies=None))),
                           (INVALID, dict(r=dict(frequencies=0x8004))), (INVALID, dict(r=dict(magnitude=0.0))), (INVALID, dict(r=dict(magnitude=-1.0))), (INVALID, dict(r=dict(magnitude=float("inf")))),
                           (INVALID, dict(r=dict(magnitude=float("nan")))), (INVALID, dict(tokens=3, x=None)), (INVALID, dict(tokens=3, x=0x6001)), (INVALID, dict(tokens=3, out=None)),
                           (INVALID, dict(tokens=3, at=None)), (INVALID, dict(tokens=3, at=0x9002)), (INVALID, dict(tokens=3, out=0x6000, out_strides=(512, 64)))]:
        assert rotary(lib, **change) == status, change
    assert lib.apmm_rotary(0, 1, 64, 0, None, 0, 0, None, None, 0, None, 0, 0, None) == INVALID


def test_store(lib):  # noqa: F811
    assert store(lib, batch=dict(tokens=0)) == OK and store(lib, batch=dict(sequences=0), q_heads=7) == OK
    for status, change in [(INVALID, dict(q_heads=-1)), (UNSUPPORTED, dict(q_heads=2049)), (INVALID, dict(r=dict(pairs=65))), (INVALID, dict(at=0x9001)), (INVALID, dict(k=None)), (INVALID, dict(v=0x7001)),
                           (INVALID, dict(q_heads=8, q=None)), (INVALID, dict(q_heads=8, q_out=None)), (INVALID, dict(q_heads=8, q=0xb000, q_strides=(2048, 128))),
                           (UNSUPPORTED, dict(batch=dict(tokens=1 << 29)))]:
        assert store(lib, **change) == status, change


def test_weights(lib):  # noqa: F811
    assert weigh(lib, batch=dict(tokens=0), q=None) == OK and weigh(lib, batch=dict(sequences=0)) == OK
    for status, change in [(INVALID, dict(q_heads=0)), (INVALID, dict(q_heads=12)), (UNSUPPORTED, dict(q_heads=8 * 1025)), (UNSUPPORTED, dict(batch=dict(tokens=1 << 26))), (INVALID, dict(q=None)),
                           (INVALID, dict(q=0x6001)), (INVALID, dict(w=None)), (INVALID, dict(w=0x7002)), (INVALID, dict(capacity=0)), (INVALID, dict(strides=(8192, 999))), (INVALID, dict(strides=(7999, 1000))),
                           (INVALID, dict(strides=(-1, 1000))), (UNSUPPORTED, dict(capacity=1 << 47)), (INVALID, dict(decay=-0.5)), (INVALID, dict(decay=float("nan"))), (INVALID, dict(decay=float("inf"))),
                           (INVALID, dict(scale=0.0)), (INVALID, dict(scale=float("inf"))), (INVALID, dict(window=-1)), (INVALID, dict(sinks=-1)), (UNSUPPORTED, dict(window=(1 << 30) + 1)),
                           (UNSUPPORTED, dict(batch=dict(sequences=65536, tokens=65536, starts=None, table_width=1 << 26, table_stride=1 << 26), q_heads=8)), (WORKSPACE, {})]:
        assert weigh(lib, **change) == status, change
    need = lib.apmm_kv_weights_workspace_bytes(*structs(), 32)
    # either order of sequences and heads, rows that follow each other or lie apart; 7 or 8 of them one capacity apart do not fit
    s, h = structs()[1].sequences, structs()[0].kv_heads
    for strides in ((h * 1000, 1000), (1000, s * 1000), (5000, 5000 * s), (h * 1234, 1234)):
        assert weigh(lib, strides=strides) == WORKSPACE, strides
    for strides in ((1000, s * 1000 - 1), (1000, 1000), (0, 1000), (1000, 0), (h * 1000 - 1, 1000)):
        assert weigh(lib, strides=strides) == INVALID, strides
    assert weigh(lib, strides=(0, 1000), batch=dict(sequences=1)) == WORKSPACE and weigh(lib, strides=(1000, 0), cache=dict(kv_heads=1), q_heads=4) == WORKSPACE
    assert need >= 7 * 32 * 8 and need % 8 == 0
    assert weigh(lib, workspace=0xc000, size=need - 1) == WORKSPACE and weigh(lib, workspace=0xc008, size=need) == INVALID
    assert lib.apmm_kv_weights_workspace_bytes(*structs(batch=dict(tokens=0)), 32) == 0 and lib.apmm_kv_weights_workspace_bytes(*structs(), 33) == 0
    for tokens in (1, 3, 33, 1000, 100000):                            # whatever lengths the batch has: as much as the queries and 320 MiB
        for sequences in (1, 2, 64, 1000):
            for kv_heads in (1, 8, 32, 1024):
                size = lib.apmm_kv_weights_workspace_bytes(*structs(dict(kv_heads=kv_heads), dict(tokens=tokens, sequences=sequences, table_width=1 << 16, table_stride=1 << 16)), kv_heads * 4)
                assert 0 < size <= (tokens * 4 + 16 * (sequences + 1)) * kv_heads * (256 + 12) + min(tokens, sequences) * kv_heads * 2 * 128 + (320 << 20)


def test_eviction(lib):  # noqa: F811
    assert evict(lib, sequences=0) == OK
    for status, change in [(INVALID, dict(sequences=-1)), (UNSUPPORTED, dict(sequences=65537)), (INVALID, dict(budget=0)), (INVALID, dict(sinks=-1)), (INVALID, dict(recent=-1)), (INVALID, dict(sinks=65)),
                           (INVALID, dict(sinks=30, recent=35)), (UNSUPPORTED, dict(budget=(1 << 30) + 1)), (INVALID, dict(to_width=0)), (INVALID, dict(to_stride=3)),
                           (UNSUPPORTED, dict(to_width=(1 << 26) + 1, to_stride=1 << 27)), (INVALID, dict(lengths=None)), (INVALID, dict(table=None)), (INVALID, dict(w=None)), (INVALID, dict(capacity=0)),
                           (INVALID, dict(to=None)), (INVALID, dict(to_lengths=None)), (INVALID, dict(kept=None)), (INVALID, dict(to_weights=None)), (INVALID, dict(kept=0xa002)),
                           (INVALID, dict(to_lengths=0x3000)), (UNSUPPORTED, dict(budget=1 << 28)), (UNSUPPORTED, dict(sequences=65536, cache=dict(kv_heads=64), budget=1))]:
        assert evict(lib, **change) == status, change
    room, (c, b) = lib.apmm_kv_evict_workspace_bytes, structs()
    assert room(c, 3, 65536 // c.page_size) == 0 and room(c, 0, 1 << 20) == 0 and room(c, -1, 1 << 20) == 0 and room(c, 3, 0) == 0
    width = 65536 // c.page_size + 1
    need = room(c, 3, width)
    assert 3 * c.kv_heads * 3 * 2048 * 4 < need <= 3 * c.kv_heads * (3 * 2048 * 4 + 256 * 8) and room(c, 3, 1 << 26) <= 3 * c.kv_heads * (3 * 2048 * 4 + 256 * 8)
    assert evict(lib, width=width) == WORKSPACE and evict(lib, width=width, workspace=0xc000, size=need - 1) == WORKSPACE and evict(lib, width=width, workspace=0xc008, size=need) == INVALID


def test_w4(lib):  # noqa: F811
    size = lib.apmm_w4_packed_bytes
    assert size(0, 128, 64) == 0 and size(16, 128, 128) == 1024 + 32 and size(1, 1, 32) == 1024 + 4 * 32 and size(17, 129, 64) == 2 * 2 * (1024 + 2 * 32)
    assert size(-1, 128, 64) == size(16, 0, 64) == size(16, 128, 48) == size(1 << 25, 128, 64) == size(16, 1 << 25, 64) == 0

    def pack(codes=0x1000, scales=0x2000, N=16, K=128, group=64, dtype=0, packed=0x3000):
        return lib.apmm_w4_pack(codes, scales, N, K, group, dtype, packed, None)

    def gemm(M=4, N=16, K=128, group=64, dtype=0, x=0x1000, x_stride=128, packed=0x3000, y=0x4000, y_stride=16, workspace=None, size=0):
        return lib.apmm_w4_gemm(M, N, K, group, dtype, x, x_stride, packed, y, y_stride, workspace, size, None)
    assert pack(N=0) == OK and gemm(M=0) == OK and gemm(N=0, y=None) == OK
    for status, change in [(INVALID, dict(N=-1)), (INVALID, dict(K=0)), (INVALID, dict(group=0)), (UNSUPPORTED, dict(group=16)), (UNSUPPORTED, dict(group=256)), (UNSUPPORTED, dict(N=(1 << 24) + 1)),
                           (UNSUPPORTED, dict(K=(1 << 24) + 1)), (INVALID, dict(dtype=2)), (INVALID, dict(packed=None)), (INVALID, dict(packed=0x3008))]:
        assert pack(**change) == status and gemm(**change) == status, change
    assert pack(codes=None) == INVALID and pack(scales=None) == INVALID and pack(scales=0x2001) == INVALID
    for status, change in [(INVALID, dict(M=-1)), (UNSUPPORTED, dict(M=(1 << 20) + 1)), (INVALID, dict(x=None)), (INVALID, dict(x=0x1001)), (INVALID, dict(y=None)), (INVALID, dict(y=0x4001)),
                           (INVALID, dict(y_stride=15)), (INVALID, dict(x_stride=-1)), (UNSUPPORTED, dict(M=1 << 20, N=1 << 24, y_stride=1 << 24))]:
        assert gemm(**change) == status, change


def test_w4_workspace(lib):  # noqa: F811
    need = lib.apmm_w4_workspace_bytes
    assert need(0, 4096, 4096, 64) == need(16, 4096, 4096, 64) == need(4, 0, 4096, 64) == need(64, 4096, 4096, 48) == need(64, 4096, 64, 64) == 0
    size = need(64, 4096, 4096, 64)
    assert size > 0 and size % (64 * 4096 * 4) == 0

    def gemm(workspace, size):
        return lib.apmm_w4_gemm(64, 4096, 4096, 64, 0, 0x1000, 4096, 0x3000, 0x4000, 4096, workspace, size, None)
    assert gemm(None, 0) == gemm(None, size) == gemm(0x8000, size - 1) == WORKSPACE and gemm(0x8008, size) == INVALID
    for M in (17, 100, 1000, 100000, 1 << 20):                         # of a few times the result, whatever the sizes
        for N in (1, 1000, 100000):
            for K in (1, 1000, 100000):
                assert need(M, N, K, 32) <= max(64 * M * (N + 3), 0) and need(M, N, K, 32) <= 512 << 20


def test_structure(lib):  # noqa: F811
    assert ctypes.sizeof(rotation()) == 24


def test_kernels_spill_nothing(kernels):  # noqa: F811
    found = {name: k for name, k in kernels.items() if re.search(r"\d(rotary|kv_rotary|kv_statistics|kv_weights|kv_select|kv_move|w4)\w*_kernel", name)}
    assert len(found) >= 4 + 4 + 8 + 1 + 4 + 1 + 2 + 2 + 12
    assert not [name for name, k in found.items() if k[".vgpr_spill_count"] or k[".private_segment_fixed_size"]]
