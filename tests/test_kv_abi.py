"""Host-side checks of the four-bit cache's entry points that need no GPU: argument errors come before any launch, workspace sizes, registers of the kernels."""
import re

import pytest

from test_abi import lib  # noqa: F401  (the fixture)
from test_code_object import code_objects, kernels  # noqa: F401

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 4
CACHE = dict(codes=0x1000, scales=0x2000, pages=100, page_size=16, kv_heads=8, head_dim=128, dtype=0)
BATCH = dict(sequences=3, tokens=7, lengths=0x3000, starts=0x4000, page_table=0x5000, table_stride=10, table_width=10)


def structs(cache={}, batch={}):
    from paper_2409_17870_amd.binding import ApmmKvBatch, ApmmKvCache
    return ApmmKvCache(**{**CACHE, **cache}), ApmmKvBatch(**{**BATCH, **batch})


def pair(fn, cache={}, batch={}, k=0x6000, v=0x7000):
    return fn(*structs(cache, batch), k, 1024, 128, v, 1024, 128, None)


def attention(lib, cache={}, batch={}, q_heads=32, q=0x6000, out=0x7000, scale=0.1, window=0, sinks=0, workspace=None, size=0):
    return lib.apmm_kv_attention(*structs(cache, batch), q_heads, q, 4096, 128, out, 4096, 128, scale, window, sinks, workspace, size, None)


REFUSED = [
    (INVALID, dict(pages=0), {}), (INVALID, dict(kv_heads=0), {}), (INVALID, dict(page_size=0), {}), (INVALID, dict(dtype=2), {}), (INVALID, dict(dtype=-1), {}),
    (UNSUPPORTED, dict(page_size=8), {}), (UNSUPPORTED, dict(page_size=48), {}), (UNSUPPORTED, dict(page_size=1 << 21), {}), (UNSUPPORTED, dict(head_dim=96), {}),
    (UNSUPPORTED, dict(kv_heads=1025), {}), (UNSUPPORTED, dict(pages=1 << 31), {}),
    (INVALID, dict(codes=None), {}), (INVALID, dict(scales=None), {}), (INVALID, dict(codes=0x1008), {}), (INVALID, dict(scales=0x2008), {}),
    (INVALID, {}, dict(sequences=-1)), (INVALID, {}, dict(tokens=-1)), (UNSUPPORTED, {}, dict(sequences=65537)), (UNSUPPORTED, {}, dict(tokens=(1 << 30) + 1)),
    (INVALID, {}, dict(table_width=0)), (INVALID, {}, dict(table_stride=9)), (UNSUPPORTED, {}, dict(table_width=(1 << 26) + 1, table_stride=1 << 30)),
    (INVALID, {}, dict(lengths=None)), (INVALID, {}, dict(page_table=None)), (INVALID, {}, dict(lengths=0x3002)), (INVALID, {}, dict(starts=0x4001)),
    (INVALID, {}, dict(page_table=0x5002)), (INVALID, {}, dict(starts=None)),  # without starts: a token a sequence
]


@pytest.mark.parametrize("status, cache, batch", REFUSED)
def test_caches_and_batches_that_are_refused(lib, status, cache, batch):  # noqa: F811
    assert pair(lib.apmm_kv_write, cache, batch) == status
    assert pair(lib.apmm_kv_read, cache, batch) == status
    assert attention(lib, cache, batch, q_heads=4 * cache.get("kv_heads", 8)) == status
    assert lib.apmm_last_error()


def test_tensors_that_are_refused(lib):  # noqa: F811
    for fn in (lib.apmm_kv_write, lib.apmm_kv_read):
        for bad in (None, 0x6001):
            assert pair(fn, k=bad) == INVALID and pair(fn, v=bad) == INVALID
        assert pair(fn, batch=dict(tokens=1 << 29)) == UNSUPPORTED     # more workgroups than a launch has
        assert pair(fn, batch=dict(sequences=0)) == OK and pair(fn, batch=dict(tokens=0), k=None, v=None) == OK
    for bad in (None, 0x6001):
        assert attention(lib, q=bad) == INVALID and attention(lib, out=bad) == INVALID
    assert attention(lib, q_heads=0) == INVALID and attention(lib, q_heads=12) == INVALID
    assert attention(lib, q_heads=8 * 1025) == UNSUPPORTED and attention(lib, batch=dict(tokens=1 << 26)) == UNSUPPORTED
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert attention(lib, scale=scale) == INVALID
    assert attention(lib, window=-1) == INVALID and attention(lib, window=4, sinks=-1) == INVALID
    assert attention(lib, window=(1 << 30) + 1) == UNSUPPORTED and attention(lib, window=4, sinks=(1 << 30) + 1) == UNSUPPORTED
    assert attention(lib, batch=dict(sequences=0)) == OK and attention(lib, batch=dict(tokens=0), q=None, out=None) == OK
    assert attention(lib, batch=dict(tokens=0), scale=0.0) == INVALID  # an empty batch's arguments are looked at all the same


def test_workspace(lib):  # noqa: F811
    def need(q_heads=32, cache={}, **batch):
        return lib.apmm_kv_attention_workspace_bytes(*structs(cache, {"table_stride": 1 << 26, **batch}), q_heads)
    assert need(table_width=1) == 0                                    # nothing to cut in 16 keys
    long = need(table_width=1 << 16)
    assert long > 0 and long % 16 == 0
    assert need(table_width=1 << 26) == long                           # depends on whether, not on how far
    assert need(tokens=0, table_width=1 << 16) == 0 and need(sequences=0, table_width=1 << 16) == 0
    assert need(q_heads=33, table_width=1 << 16) == 0 and need(cache=dict(head_dim=80), table_width=1 << 16) == 0  # what the call refuses
    for size, at, status in ((0, None, WORKSPACE), (long, None, WORKSPACE), (long - 1, 0x8000, WORKSPACE), (long, 0x8008, INVALID)):
        assert attention(lib, batch=dict(table_width=1 << 16, table_stride=1 << 16), workspace=at, size=size) == status
    for tokens in (1, 3, 33, 1000, 100000):                            # whatever lengths the batch has: a few hundred MiB at most
        for sequences in (1, 2, 64, 1000):
            for kv_heads in (1, 8, 32, 1024):
                assert need(q_heads=kv_heads * 4, cache=dict(kv_heads=kv_heads), tokens=tokens, sequences=sequences, table_width=1 << 16) <= 512 << 20


def test_kernels_spill_nothing(kernels):  # noqa: F811
    found = {name: k for name, k in kernels.items() if re.search(r"\dkv_(write|read|attention)\w*_kernel", name)}
    assert len(found) == 4 + 4 + 8 + 8 + 4  # head_dim and type; attention of few rows for four and eight waves, of many for pages of 16 and others; the join
    assert not [name for name, k in found.items() if k[".vgpr_spill_count"] or k[".private_segment_fixed_size"]]
    assert all(k[".vgpr_count"] <= 168 for name, k in found.items() if re.search(r"kv_attention_rows_kernelILi\d+ELb\dELi4E", name))  # three workgroups on a compute unit
