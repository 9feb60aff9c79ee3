"""A cache of no channels is refused alike by the calls in C++ and the Python functions that they stand for."""
import pytest
import torch

from paper_2409_17870_amd import binding
from test_call import general, outcome

pytestmark = pytest.mark.gpu


def test_refused_alike():
    codes = torch.zeros((1, 2, 2, 0), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((1, 2, 2, 16), dtype=torch.float16, device="cuda")
    table, one = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    x = torch.zeros((1, 2, 0), dtype=torch.float16, device="cuda")
    for name, args in (("apmm_kv_write", (x, x, codes, scales, table, one)), ("apmm_kv_read", (codes, scales, table, one, 1)), ("apmm_kv_attention", (x, codes, scales, table, one))):
        got, want = outcome(getattr(binding, name), *args), outcome(general(name), *args)
        assert got == want and got[0] == "ValueError", (name, got, want)
