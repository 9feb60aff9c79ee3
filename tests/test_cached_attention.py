"""The example that runs products, cache and attention together, prompts and then single tokens of a graph."""
import importlib.util
import os

import pytest

import kv_reference as ref
from test_kv import close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "cached_attention.py")
    spec = importlib.util.spec_from_file_location("cached_attention", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("sizes", [
    dict(sequences=4, longest=300, steps=20),
    dict(sequences=3, longest=500, steps=7, window=100, sinks=4, hidden=1024, heads=8, kv_heads=2, head_dim=64, page_size=16),
    dict(sequences=1, longest=1, steps=3, hidden=512, heads=4, kv_heads=4, page_size=16),
])
def test_prompts_and_single_tokens(example, sizes):
    """Against attention in 64 bits over the cache's codes, within what kv_reference.py derives."""
    import torch
    checked = []

    def check(part, cache, table, lengths, new, q, o):
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        close(torch, o, *ref.attention(q, *cache, table.cpu(), lengths, starts, part.window, part.sinks, part.head_dim ** -0.5))
        checked.append(sum(new))
    example.serve(check=check, **sizes)
    assert len(checked) == 2 and checked[1] == sizes["sequences"]


def test_command(example, capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["cached_attention.py", "--sequences", "2", "--longest", "90", "--steps", "2", "--window", "40", "--sinks", "2"])
    example.main()
    assert "us a step" in capsys.readouterr().out
