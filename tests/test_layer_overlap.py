"""Results that would be written over what the same call still reads: refused before any launch, where both begin at one place."""
import pytest

from test_abi import lib  # noqa: F401  (the fixture)
from test_layer_abi import INVALID, OK, evict, store

SAME = dict(q_heads=8, q=0xa000)


def test_products(lib):  # noqa: F811
    def gemm(y, M=4):
        return lib.apmm_w4_gemm(M, 128, 128, 64, 0, 0x1000, 128, 0x3000, y, 128, None, 0, None)
    assert gemm(0x1000) == INVALID and gemm(0x1000, M=1) == INVALID and gemm(0x1000, M=0) == OK


def test_eviction(lib):  # noqa: F811
    assert evict(lib, to_weights=0x7000) == INVALID and evict(lib, sequences=0, to_weights=0x7000) == OK


@pytest.mark.parametrize("change", [dict(q_out=0x6000), dict(q_out=0x7000)])
def test_queries_over_keys_or_values(lib, change):  # noqa: F811
    assert store(lib, **SAME, **change) == INVALID and store(lib, batch=dict(tokens=0), **SAME, **change) == OK
