"""The attention part of a decoder layer with every product on bipolar-INT operands and its keys and values in four bits, as a server runs it: some prompts
of different lengths in one batch, then one new token a sequence at a time from a captured graph.

  python examples/cached_attention.py [--sequences N] [--longest L] [--steps S] [--window W --sinks F]

Random weights and inputs of the sizes of a Llama-2-7B layer (W2A4).  The attention's results are held against ones computed in 32 bits from the keys and
values that apmm_kv_read gives back; those are rounded to 16 bits, the cache's are not, so that large scores differ by some 2^-11 of themselves.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2409_17870_amd import binding


class AttentionPart:
    """q, k and v of one product, the cache, attention, the output product."""

    def __init__(self, hidden=4096, heads=32, kv_heads=32, head_dim=128, p=4, q=2, window=0, sinks=0, device="cuda"):
        self.hidden, self.heads, self.kv_heads, self.head_dim = hidden, heads, kv_heads, head_dim
        self.p, self.q, self.window, self.sinks = p, q, window, sinks
        self.rows = (heads + 2 * kv_heads) * head_dim

        def linear(n, k):
            codes = torch.randint(0, 1 << q, (n, k), dtype=torch.uint8, device=device)
            return binding.apmm_pack_weights(codes, q), (torch.rand(n, device=device) * 2.0 / k ** 0.5).half()
        self.w_qkv, self.s_qkv = linear(self.rows, hidden)
        self.w_out, self.s_out = linear(hidden, heads * head_dim)

    def product(self, x, n, w, w_scale):
        a, a_scale = binding.apmm_quantize_pack_activations(x, self.p)
        return binding.apmm_gemm(x.shape[0], n, x.shape[1], self.p, self.q, a, w, want_i32=False, want_f16=True, w_scale=w_scale, a_scale=a_scale)[1]

    def __call__(self, x, cache, table, lengths, starts=None):
        """x: new tokens x hidden, those of a sequence one after the other; lengths count them.  (result, queries, attention's result)"""
        qkv = self.product(x, self.rows, self.w_qkv, self.s_qkv).view(-1, self.heads + 2 * self.kv_heads, self.head_dim)
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), 1)
        binding.apmm_kv_write(k, v, *cache, table, lengths, starts)
        o = binding.apmm_kv_attention(q, *cache, table, lengths, starts, window=self.window, sinks=self.sinks)
        return self.product(o.view(-1, self.heads * self.head_dim), self.hidden, self.w_out, self.s_out), q, o


def plain_attention(q, k, v, window, sinks):
    """In 32 bits: the last q.shape[0] tokens of a sequence whose keys and values are k and v (tokens x heads x head_dim)."""
    n, length, groups = q.shape[0], k.shape[0], q.shape[1] // k.shape[1]
    k, v = (t.float().repeat_interleave(groups, 1).transpose(0, 1).contiguous() for t in (k, v))
    pos = torch.arange(length - n, length, device=q.device)[:, None]
    key = torch.arange(length, device=q.device)[None]
    seen = key <= pos
    if window:
        seen &= (key > pos - window) | (key < sinks)
    s = torch.matmul(q.float().transpose(0, 1).contiguous(), k.transpose(1, 2).contiguous()) * q.shape[2] ** -0.5
    return torch.matmul(torch.softmax(s.masked_fill(~seen, float("-inf")), -1), v).transpose(0, 1)


def worst(part, cache, table, lengths, new, q, o):
    """Largest difference of o from plain_attention over all sequences, as a share of the largest value."""
    total = sum(lengths)
    starts = torch.tensor([0] + lengths, device=q.device).cumsum(0).int()
    k, v = binding.apmm_kv_read(*cache, table, torch.tensor(lengths, dtype=torch.int32, device=q.device), total, starts)
    off, at, row = 0.0, 0, 0
    for length, n in zip(lengths, new):
        ref = plain_attention(q[row:row + n], k[at:at + length], v[at:at + length], part.window, part.sinks)
        off = max(off, ((o[row:row + n].float() - ref).abs().max() / v[at:at + length].abs().max()).item())
        at, row = at + length, row + n
    return off


def serve(sequences=4, longest=700, steps=32, window=0, sinks=0, page_size=64, hidden=4096, heads=32, kv_heads=32, head_dim=128, seed=0, check=worst):
    """What `check` says of the prompts' attention and of the single tokens', microseconds of a step."""
    torch.manual_seed(seed)
    part = AttentionPart(hidden, heads, kv_heads, head_dim, window=window, sinks=sinks)
    lengths = [max(1, longest - longest * 3 * i // (4 * sequences)) for i in range(sequences)]
    pages = [-(-(n + steps + 1) // page_size) for n in lengths]
    order = torch.randperm(sum(pages)).int()
    table = torch.full((sequences, max(pages)), -1, dtype=torch.int32)
    for i, n in enumerate(pages):
        table[i, :n], order = order[:n], order[n:]
    table = table.cuda()
    cache = binding.apmm_kv_cache(sum(pages), page_size, kv_heads, head_dim)

    # the prompts, of one call
    held = torch.tensor(lengths, dtype=torch.int32).cuda()
    starts = torch.tensor([0] + lengths).cumsum(0).int().cuda()
    x = torch.randn(sum(lengths), hidden, device="cuda").half()
    _, q, o = part(x, cache, table, held, starts)
    of_prompts = check(part, cache, table, lengths, lengths, q, o)

    # single tokens: a step is recorded once, on another stream
    x = torch.randn(sequences, hidden, device="cuda").half()

    def step():
        held.add_(1)
        return part(x, cache, table, held)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, q, o = step()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for i in range(steps):
        if i == 1:  # (the first replay sets the graph up)
            begin.record()
        graph.replay()
        x.copy_(torch.nn.functional.normalize(y.float(), dim=1).mul_(hidden ** 0.5))  # what comes out goes in again
    end.record()
    end.synchronize()
    now = [n + 1 + steps for n in lengths]
    of_steps = check(part, cache, table, now, [1] * sequences, q, o)
    assert held.tolist() == now and bool(torch.isfinite(y).all())
    return of_prompts, of_steps, begin.elapsed_time(end) * 1e3 / (steps - 1) if steps > 1 else float("nan")


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("sequences", 4), ("longest", 700), ("steps", 32), ("window", 0), ("sinks", 0)):
        ap.add_argument("--" + name, type=int, default=default)
    args = ap.parse_args()
    of_prompts, of_steps, us = serve(args.sequences, args.longest, args.steps, args.window, args.sinks)
    print("largest difference from attention in 32 bits, of the largest value: prompts %.2g, single tokens %.2g; %.1f us a step" % (of_prompts, of_steps, us))


if __name__ == "__main__":
    main()
