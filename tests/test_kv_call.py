"""The calls of the four-bit cache in C++ (csrc/apmm_call.cpp) against the Python functions that they stand for: the same results and the same errors, plain
arguments without the Python function."""
import inspect

import pytest
import torch

from paper_2409_17870_amd import binding
from test_call import general, outcome

NAMES = ["apmm_kv_write", "apmm_kv_read", "apmm_kv_attention"]


@pytest.mark.parametrize("name", NAMES)
def test_signatures(name):
    assert binding._call is not None
    assert inspect.signature(getattr(binding, name)) == inspect.signature(general(name))


@pytest.mark.parametrize("name, args", [
    ("apmm_kv_write", ()),
    ("apmm_kv_read", (torch.zeros(1, 1, 2, 512, dtype=torch.uint8), torch.zeros(1, 1, 2, 16).half(), None, None, 1)),
    ("apmm_kv_attention", (torch.zeros(1, 1, 64).half(), torch.zeros(1, 1, 2, 512, dtype=torch.uint8), torch.zeros(1, 1, 2, 16).half(), None, None)),
    ("apmm_kv_attention", (1, 2, 3, 4, 5)),
])
def test_refused_alike(name, args):
    binding.load()
    got, want = outcome(getattr(binding, name), *args), outcome(general(name), *args)
    assert isinstance(got, tuple) and got == want


PLAIN, GENERAL = 0, 1


@pytest.mark.gpu
def test_results_and_errors_alike():
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(5)
    H, Hq, D, ps, pages, B = 2, 6, 64, 16, 40, 3
    codes = torch.randint(0, 256, (pages, H, 2, ps * D // 2), generator=g, device=dev, dtype=torch.uint8)
    scales = (torch.rand((pages, H, 2, ps), generator=g, device=dev) * 0.2).half()
    table = torch.arange(30, dtype=torch.int32, device=dev).view(B, 10)
    lengths = torch.tensor([100, 3, 160], dtype=torch.int32, device=dev)
    starts = torch.tensor([0, 5, 6, 20], dtype=torch.int32, device=dev)
    one = torch.randn((B, Hq + 2 * H, D), generator=g, device=dev).half()
    many = torch.randn((20, Hq + 2 * H, D), generator=g, device=dev).half()

    def rows(x):
        return x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]
    q1, k1, v1 = rows(one)
    q, k, v = rows(many)
    c = (codes, scales, table, lengths)
    wide = torch.zeros((B, 100000), dtype=torch.int32, device=dev)
    room = binding.apmm_kv_attention_workspace_bytes(B, Hq, codes, scales, wide, lengths)
    general_of = {name: general(name) for name in NAMES}

    def copy():
        return codes.clone(), scales.clone()
    calls = [
        ("apmm_kv_write", PLAIN, lambda: ((k, v, *copy(), table, lengths, starts), {})),
        ("apmm_kv_write", PLAIN, lambda: ((k1, v1, *copy()), dict(lengths=lengths, page_table=table))),
        ("apmm_kv_write", PLAIN, lambda: ((k1, v1, *copy(), table, lengths, None), {})),
        ("apmm_kv_write", GENERAL, lambda: ((k, v, *copy(), table, lengths), {})),
        ("apmm_kv_write", GENERAL, lambda: ((k1, v1.float(), *copy(), table, lengths), {})),
        ("apmm_kv_write", GENERAL, lambda: ((k1, v1, *copy(), table.long(), lengths), {})),
        ("apmm_kv_write", GENERAL, lambda: ((k1, v1, *copy(), table.t(), lengths), {})),
        ("apmm_kv_read", PLAIN, lambda: ((*c, 20, starts), {})),
        ("apmm_kv_read", PLAIN, lambda: ((*c, B), {})),
        ("apmm_kv_read", PLAIN, lambda: ((*c, 20, starts), dict(k_out=torch.zeros_like(k)))),
        ("apmm_kv_read", PLAIN, lambda: ((*c, 20, starts, torch.zeros_like(k), torch.zeros((20, 3 * H, D), dtype=torch.float16, device=dev)[:, 1:1 + H]), {})),
        ("apmm_kv_read", GENERAL, lambda: ((*c, 20), {})),
        ("apmm_kv_read", GENERAL, lambda: ((*c, 20, starts, torch.zeros_like(k)[:-1]), {})),
        ("apmm_kv_read", GENERAL, lambda: ((codes, scales.float(), table, lengths, 20, starts), {})),
        ("apmm_kv_attention", PLAIN, lambda: ((q, *c, starts), {})),
        ("apmm_kv_attention", PLAIN, lambda: ((q1, *c), {})),
        ("apmm_kv_attention", PLAIN, lambda: ((q, *c, starts), dict(window=9, sinks=2, scale=0.3))),
        ("apmm_kv_attention", PLAIN, lambda: ((q, *c, starts, 9, 2, None, torch.zeros_like(q)), {})),
        ("apmm_kv_attention", PLAIN, lambda: ((q, *c, starts), dict(window=-1))),
        ("apmm_kv_attention", PLAIN, lambda: ((q, *c, starts), dict(scale=0.0))),
        ("apmm_kv_attention", PLAIN, lambda: ((q1[:, :5], *c), {})),
        ("apmm_kv_attention", PLAIN, lambda: ((q1, codes, scales, wide, lengths), {})),
        ("apmm_kv_attention", PLAIN, lambda: ((q1, codes, scales, wide, lengths), dict(workspace=torch.zeros(room, dtype=torch.uint8, device=dev)))),
        ("apmm_kv_attention", PLAIN, lambda: ((q1, codes, scales, wide, lengths), dict(workspace=torch.zeros(room - 1, dtype=torch.uint8, device=dev)))),
        ("apmm_kv_attention", GENERAL, lambda: ((q1, codes, scales, wide, lengths), dict(workspace=torch.zeros(room, dtype=torch.uint8)))),
        ("apmm_kv_attention", GENERAL, lambda: ((q, *c, starts), dict(scale=1))),
        ("apmm_kv_attention", GENERAL, lambda: ((q, *c, starts), dict(window=None))),
        ("apmm_kv_attention", GENERAL, lambda: ((q.bfloat16(), *c, starts), {})),
        ("apmm_kv_attention", GENERAL, lambda: ((q[:, :, ::2], *c, starts), {})),
        ("apmm_kv_attention", PLAIN, lambda: ((many[:0, :Hq], codes, scales, table[:0], lengths[:0]), {})),
    ]
    stream = torch.cuda.Stream()
    for name, route, make in calls:
        results, asked = [], []

        def handed_over(*args, **kw):
            asked.append(name)
            return general_of[name](*args, **kw)
        binding._call.set_general(name, handed_over)
        try:
            for fn in (getattr(binding, name), general_of[name]):
                args, kw = make()
                stream.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(stream):
                    r = outcome(fn, *args, **kw)
                stream.synchronize()
                if name == "apmm_kv_write" and r is None:
                    r = args[2], args[3]
                results.append(r if isinstance(r, tuple) else (r,))
        finally:
            binding._call.set_general(name, binding._general[name])
        assert len(asked) == route, (name, asked, results)
        got, want = results
        assert len(got) == len(want), (name, got, want)
        for s, t in zip(got, want):
            if isinstance(t, torch.Tensor):
                assert type(s) is type(t) and s.dtype == t.dtype and torch.equal(s, t), name
            else:
                assert s == t, (name, s, t)
