"""The calls for rotary positions, the cache's budget and four-bit weights in C++ (csrc/apmm_call.cpp) against the Python functions that they stand for: the same results and the same errors, plain
arguments without the Python function."""
import inspect

import pytest
import torch

from paper_2409_17870_amd import binding
from test_call import general, outcome

NAMES = ["apmm_rotary", "apmm_kv_write_rotary", "apmm_kv_weights", "apmm_kv_evict", "apmm_w4_gemm"]


@pytest.mark.parametrize("name", NAMES)
def test_signatures(name):
    assert binding._call is not None
    assert inspect.signature(getattr(binding, name)) == inspect.signature(general(name))


@pytest.mark.parametrize("name, args", [
    ("apmm_rotary", ()),
    ("apmm_rotary", (torch.zeros(1, 1, 64).half(), torch.zeros(1, dtype=torch.int32), torch.zeros(32, dtype=torch.float64))),
    ("apmm_kv_write_rotary", (1, 2, 3, 4, 5, 6, 7, 8)),
    ("apmm_kv_weights", (torch.zeros(1, 1, 64).half(), torch.zeros(1, 1, 2, 512, dtype=torch.uint8), torch.zeros(1, 1, 2, 16).half(), None, None, None)),
    ("apmm_kv_evict", (None,) * 7),
    ("apmm_w4_gemm", (torch.zeros(1, 64).half(), torch.zeros(5000, dtype=torch.uint8), 16, 64)),
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
    H, Hq, D, ps, pages, B = 2, 6, 64, 16, 60, 3
    codes = torch.randint(0, 256, (pages, H, 2, ps * D // 2), generator=g, device=dev, dtype=torch.uint8)
    scales = (torch.rand((pages, H, 2, ps), generator=g, device=dev) * 0.2).half()
    table, to = torch.arange(30, dtype=torch.int32, device=dev).view(B, 10), torch.arange(30, 60, dtype=torch.int32, device=dev).view(B, 10)
    lengths = torch.tensor([100, 3, 160], dtype=torch.int32, device=dev)
    starts = torch.tensor([0, 5, 6, 20], dtype=torch.int32, device=dev)
    one, many = (torch.randn((n, Hq + 2 * H, D), generator=g, device=dev).half() for n in (B, 20))
    at1, at = (torch.arange(n, dtype=torch.int32, device=dev) for n in (B, 20))
    f = binding.apmm_rotary_frequencies(D)
    w = torch.rand((B, H, 160), generator=g, device=dev)

    def rows(x):
        return x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]
    (q1, k1, v1), (q, k, v) = rows(one), rows(many)
    c = (codes, scales, table, lengths)
    x = torch.randn((40, 256), generator=g, device=dev).half()
    w4 = binding.apmm_w4_pack(torch.randint(0, 16, (48, 256), generator=g, device=dev, dtype=torch.uint8), torch.rand((48, 4), generator=g, device=dev).half(), 64)
    general_of = {name: general(name) for name in NAMES}
    room = binding.apmm_kv_weights_workspace_bytes(20, Hq, *c)
    wide = torch.cat([table, torch.full((B, 4200), -1, dtype=torch.int32, device=dev)], 1)
    more = binding.apmm_kv_evict_workspace_bytes(codes, scales, wide)

    def cache():
        return codes.clone(), scales.clone(), table, lengths

    def space(n, **more):
        return torch.zeros(n, dtype=torch.uint8, **(more or dict(device=dev)))
    calls = [
        ("apmm_rotary", PLAIN, lambda: ((q, at, f), {})),
        ("apmm_rotary", PLAIN, lambda: ((q, at, f, True, 1.5, True, torch.zeros_like(q)), {})),
        ("apmm_rotary", PLAIN, lambda: ((q.bfloat16(), at), dict(frequencies=f[:8], inverse=True))),
        ("apmm_rotary", PLAIN, lambda: ((q, at, f), dict(magnitude=-1.0))),
        ("apmm_rotary", PLAIN, lambda: ((q, at, torch.cat([f, f])), {})),
        ("apmm_rotary", PLAIN, lambda: ((q[:0], at[:0], f), {})),
        ("apmm_rotary", GENERAL, lambda: ((q, at, f), dict(magnitude=1))),
        ("apmm_rotary", GENERAL, lambda: ((q, at, f), dict(interleaved=1))),
        ("apmm_rotary", GENERAL, lambda: ((q.float(), at, f), {})),
        ("apmm_rotary", GENERAL, lambda: ((q, at1, f), {})),
        ("apmm_rotary", GENERAL, lambda: ((q, at, f.float()), {})),
        ("apmm_rotary", GENERAL, lambda: ((q, at, f), dict(out=q1))),
        ("apmm_kv_write_rotary", PLAIN, lambda: ((q, k, v, *cache(), f, starts), {})),
        ("apmm_kv_write_rotary", PLAIN, lambda: ((q, k, v, *cache(), f, starts, at, True, 0.5, torch.zeros_like(q)), {})),
        ("apmm_kv_write_rotary", PLAIN, lambda: ((q1, k1, v1, *cache(), f), dict(positions=at1))),
        ("apmm_kv_write_rotary", PLAIN, lambda: ((q1, k1, v1, *cache(), torch.cat([f, f])), {})),
        ("apmm_kv_write_rotary", GENERAL, lambda: ((None, k1, v1, *cache(), f), {})),
        ("apmm_kv_write_rotary", GENERAL, lambda: ((q, k, v, *cache(), f), {})),
        ("apmm_kv_write_rotary", GENERAL, lambda: ((q, k, v.bfloat16(), *cache(), f, starts), {})),
        ("apmm_kv_write_rotary", GENERAL, lambda: ((q, k, v, *cache(), f, starts, at1), {})),
        ("apmm_kv_weights", PLAIN, lambda: ((q, *c, w.clone(), starts), {})),
        ("apmm_kv_weights", PLAIN, lambda: ((q1, *c, w.clone()), dict(window=9, sinks=2, scale=0.3, decay=0.5))),
        ("apmm_kv_weights", PLAIN, lambda: ((q, *c, w.clone(), starts, 0, 0, None, 0.0, space(room)), {})),
        ("apmm_kv_weights", PLAIN, lambda: ((q, *c, w.clone(), starts), dict(workspace=space(room - 1)))),
        ("apmm_kv_weights", PLAIN, lambda: ((q1, *c, w.clone()), dict(window=-1))),
        ("apmm_kv_weights", PLAIN, lambda: ((q1, *c, w.clone()), dict(decay=-1.0))),
        ("apmm_kv_weights", GENERAL, lambda: ((q1, *c, w.clone()), dict(decay=1))),
        ("apmm_kv_weights", GENERAL, lambda: ((q1, *c, w[:2].clone()), {})),
        ("apmm_kv_weights", GENERAL, lambda: ((q1, *c, w.double()), {})),
        ("apmm_kv_weights", GENERAL, lambda: ((q1, *c, w.clone()), dict(workspace=space(room, device="cpu")))),
        ("apmm_kv_evict", PLAIN, lambda: ((*cache(), w, 50, to), {})),
        ("apmm_kv_evict", PLAIN, lambda: ((*cache(), w, 50, to, 2, 7, torch.zeros((B, H, 50), dtype=torch.int32, device=dev), torch.zeros((B, H, 50), device=dev), torch.zeros_like(lengths)), {})),
        ("apmm_kv_evict", PLAIN, lambda: ((*cache(), w, 50, to), dict(sinks=51))),
        ("apmm_kv_evict", PLAIN, lambda: ((*cache()[:2], wide, lengths, w, 50, to), {})),
        ("apmm_kv_evict", PLAIN, lambda: ((*cache()[:2], wide, lengths, w, 50, to), dict(recent=4, workspace=space(more)))),
        ("apmm_kv_evict", PLAIN, lambda: ((*cache()[:2], wide, lengths, w, 50, to), dict(workspace=space(more - 1)))),
        ("apmm_kv_evict", GENERAL, lambda: ((*cache()[:2], wide, lengths, w, 50, to), dict(workspace=space(more, device="cpu")))),
        ("apmm_kv_evict", GENERAL, lambda: ((*cache(), w, 50, to[:2]), {})),
        ("apmm_kv_evict", GENERAL, lambda: ((*cache(), w, 50, to), dict(kept=torch.zeros((B, H, 49), dtype=torch.int32, device=dev)))),
        ("apmm_kv_evict", GENERAL, lambda: ((*cache(), w.half(), 50, to), {})),
        ("apmm_w4_gemm", PLAIN, lambda: ((x, w4, 48, 64), {})),
        ("apmm_w4_gemm", PLAIN, lambda: ((x[:1], w4, 48, 64), dict(out=torch.zeros((1, 48), dtype=torch.float16, device=dev)))),
        ("apmm_w4_gemm", PLAIN, lambda: ((x, w4, 48, 64, None, space(1 << 20)), {})),
        ("apmm_w4_gemm", PLAIN, lambda: ((x[:0], w4, 48, 64), {})),
        ("apmm_w4_gemm", PLAIN, lambda: ((x, w4, 48, 48), {})),
        ("apmm_w4_gemm", GENERAL, lambda: ((x, w4, 64, 64), {})),
        ("apmm_w4_gemm", GENERAL, lambda: ((x.float(), w4, 48, 64), {})),
        ("apmm_w4_gemm", GENERAL, lambda: ((x, w4, 48, 64), dict(out=torch.zeros((1, 48), dtype=torch.float16, device=dev)))),
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
                r = r if isinstance(r, tuple) else (r,)
                if name in ("apmm_kv_write_rotary", "apmm_kv_evict"):
                    r += args[3:5] if name == "apmm_kv_write_rotary" else args[:2]
                results.append(r)
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
