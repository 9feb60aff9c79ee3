"""Operators around the four-bit key/value cache and the products that feed it, as cases whose time and outputs can be compared
with their plain forms.

Five kinds of cases:

  "product"       ``apmm_w4_gemm``: activations of 16 bits times four-bit weights, codes u of the value 2 u - 15 with a scale for
                  each output channel and ``group`` inputs.
  "rotate"        ``apmm_rotary``: pairs of the first ``rotary`` channels of each head turned by position times frequency; pairs
                  are neighbours (``interleaved``) or lie half of the ``rotary`` channels apart.
  "rotate_store"  ``apmm_kv_write_rotary`` and ``apmm_kv_read``: queries turned, keys turned and quantised into the cache with
                  the values, in one call, and the keys and values that every later reader has of them.
  "weigh"         ``apmm_kv_weights``: what attention of the new tokens gives each cached token, summed over the queries and the
                  query heads of a key/value head, added to what earlier calls gave it (times ``decay``).
  "evict"         ``apmm_kv_evict`` and ``apmm_kv_read``: of each sequence and head the first ``sinks`` tokens, the last
                  ``recent`` and the heaviest others, ``budget`` in all, moved to other pages in their order.

The cache is two tensors, ``codes`` (pages x key/value heads x 2 x page * head_dim / 2 bytes; of the 2 keys, then values) and
``scales`` (pages x key/value heads x 2 x page).  Keys lie token by token, channel c in byte c / 2, even channels in the low four
bits; values in groups of eight tokens: for channels 4 m to 4 m + 3 eight 16-bit words, one a token, channel 4 m + e in bits 4 e
to 4 e + 3.  ``new`` says which tokens of a sequence are new: "one", "all", "some" (the last ``chunk``), "mixed" (a quarter of the
sequences as in "some", the others one); lengths go from ``longest`` down by ``spread``; of ``idle`` batches every fifth sequence
has no tokens.  Queries, keys and values are slices of one fused projection.
"""
import math

import torch

own = False

_BATCH = dict(sequences=1, longest=1, spread=0.0, idle=False, new="all", chunk=1, kv_heads=8, groups=1, head_dim=128, page=16, dtype="f16")


def _case(kind, name=None, **more):
    case = dict(kind=kind, **({} if kind in ("product", "rotate") else _BATCH))
    case.update(more)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # One token through an output projection of the 7B width: the smallest product, where latency counts.
        _case("product", "product_one_token", M=1, N=4096, K=4096, group=128, dtype="f16"),
        # A batch of sixteen single tokens through gate or up: bound by the weights' bytes.
        _case("product", "product_batch", M=16, N=11008, K=4096, group=64, dtype="bf16"),
        # A short ragged batch at the 13B width, odd numbers of tokens and channels, a last group that is cut.
        _case("product", "product_odd", M=77, N=5119, K=13800, group=128, dtype="f16"),
        # A prompt of 2048 tokens through gate or up.
        _case("product", "product_prompt", M=2048, N=11008, K=4096, group=128, dtype="bf16"),
        # A decode step of eight sequences, queries and keys of one projection: latency.
        _case("rotate", "rotate_step", tokens=8, heads=40, head_dim=128, rotary=128, interleaved=True, dtype="bf16", far=100000, scaled=False),
        # A long prompt, frequencies scaled for it.
        _case("rotate", "rotate_prompt", tokens=8192, heads=64, head_dim=128, rotary=128, interleaved=False, dtype="f16", far=1 << 20, scaled=True),
        # A decode step of 32 sequences on its way into the cache, some slots empty.
        _case("rotate_store", "rotate_store_step", sequences=32, longest=4096, spread=0.9, idle=True, new="one", kv_heads=8, groups=4,
              head_dim=128, page=16, dtype="bf16", rotary=128, interleaved=False, scaled=False),
        # Pieces of prompts beside single tokens, part of the head turned.
        _case("rotate_store", "rotate_store_mixed", sequences=13, longest=6001, spread=0.8, new="mixed", chunk=1500, kv_heads=32,
              head_dim=128, page=64, dtype="f16", rotary=64, interleaved=True, scaled=True),
        # Token generation over long contexts: which tokens the new ones look at.
        _case("weigh", "weigh_decode", sequences=8, longest=32768, spread=0.4, new="one", kv_heads=8, groups=4, head_dim=128, page=64,
              dtype="bf16", window=0, sinks=0, decay=1.0),
        # A prompt over its own cache at the 7B width.
        _case("weigh", "weigh_prompt", sequences=1, longest=4096, new="all", kv_heads=32, head_dim=128, page=64, dtype="f16", window=0,
              sinks=0, decay=0.0),
        # A batch of a serving loop after some steps over its budget: ragged, short of it in places.
        _case("evict", "evict_batch", sequences=24, longest=2300, spread=0.6, idle=True, kv_heads=8, head_dim=64, page=16, dtype="f16",
              budget=1000, sinks=4, recent=250),
        # One long prompt cut down to what generation goes on with.
        _case("evict", "evict_long", sequences=1, longest=65001, kv_heads=8, head_dim=128, page=64, dtype="bf16", budget=4096, sinks=4,
              recent=1024),
    ]


# The most that a drawn case may ask for.
_MOST_CACHE = 65001 * 8 * 128          # cached channels of all heads, sequences padded to the longest
_MOST_SCORES = 32 * 4096 * 4096        # queries and keys of all heads, padded likewise
_MOST_STORED = 13 * 1500 * 32 * 128    # new channels, padded likewise
_MOST_PRODUCT = 2048 * 11008 * 4096
_MOST_ROTATED = 8192 * 64 * 128


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["product", "product", "rotate", "rotate_store", "weigh", "weigh", "evict"])
        dtype = rng.choice(["f16", "bf16"])
        if kind == "product":
            sizes = [1024, 2048, 4096, 5120, 11008, 13824]
            case = _case(kind, M=_log_int(rng, 1, 2048), N=rng.choice(sizes + [_log_int(rng, 1, 14000)] * 3),
                         K=rng.choice(sizes + [_log_int(rng, 16, 14000)] * 3), group=rng.choice([32, 64, 128]), dtype=dtype)
            if case["M"] * case["N"] * case["K"] <= _MOST_PRODUCT:
                return case
            continue
        head_dim = rng.choice([64, 128])
        more = dict(interleaved=rng.random() < 0.5, scaled=rng.random() < 0.4, dtype=dtype)
        if kind == "rotate":
            head_dim = rng.choice([64, 80, 96, 128, 256])
            case = _case(kind, tokens=_log_int(rng, 1, 20000), heads=_log_int(rng, 1, 72), head_dim=head_dim,
                         rotary=rng.choice([head_dim, head_dim, head_dim // 2, head_dim // 4]), far=_log_int(rng, 1, 1 << 24), **more)
            if case["tokens"] * case["heads"] * head_dim <= _MOST_ROTATED:
                return case
            continue
        kv_heads, groups = rng.choice([(32, 1), (40, 1), (8, 4), (8, 8), (4, 8), (2, 6), (16, 2), (1, 16), (3, 3)])
        case = _case(kind, sequences=_log_int(rng, 1, 48), longest=_log_int(rng, 1, 65001), spread=round(rng.choice([0.0, rng.random()]), 3),
                     idle=rng.random() < 0.3, new=rng.choice(["one", "one", "all", "some", "mixed"]), chunk=_log_int(rng, 2, 2048),
                     kv_heads=kv_heads, groups=groups, head_dim=head_dim, page=rng.choice([16, 16, 32, 64, 128, 256]), dtype=dtype)
        B, L, most = case["sequences"], case["longest"], max(_new(case))
        if B * L * kv_heads * head_dim > _MOST_CACHE:
            continue
        if kind == "rotate_store":
            case.update(more, rotary=rng.choice([head_dim, head_dim, head_dim // 2]))
            if B * most * kv_heads * groups * head_dim > _MOST_STORED:
                continue
        if kind == "weigh":
            case.update(window=rng.choice([0, 0, _log_int(rng, 1, 4096)]), sinks=rng.choice([0, rng.randint(1, 128)]),
                        decay=rng.choice([0.0, 1.0, 0.9]))
            if B * kv_heads * groups * most * L > _MOST_SCORES:
                continue
        if kind == "evict":
            case.update(new="all", budget=_log_int(rng, 1, 8192))
            case.update(sinks=rng.randint(0, min(16, case["budget"])))
            case.update(recent=rng.randint(0, case["budget"] - case["sinks"]))
        return case


# ------------------------------------------------------------- the batch ----
def _lengths(case):
    out = []
    for b in range(case["sequences"]):
        idle = case["idle"] and b % 5 == 3
        out.append(0 if idle else max(1, int(case["longest"] * (1.0 - case["spread"] * (b * 0.6180339887 % 1.0)))))
    return out


def _new(case):
    out = []
    for b, n in enumerate(_lengths(case)):
        if case["new"] == "all":
            out.append(n)
        elif case["new"] == "one" or (case["new"] == "mixed" and b % 4 != 0):
            out.append(1)
        else:
            out.append(max(1, min(n, case["chunk"])))
    return out


def work(case):
    kind = case["kind"]
    if kind == "product":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": N * K / 2 + 2 * N * -(-K // case["group"]) + 2 * M * (N + K), "flops": 2.0 * M * N * K}
    if kind == "rotate":
        n = case["tokens"] * case["heads"]
        return {"bytes": 4 * n * case["head_dim"] + 4 * case["tokens"], "flops": 3.0 * n * case["rotary"]}
    H, D, G, new = case["kv_heads"], case["head_dim"], case["groups"], sum(_new(case))
    cached, plain = H * (D / 2 + 2), 2 * H * D      # bytes of a token's keys or values
    if kind == "rotate_store":
        return {"bytes": new * (4 * H * G * D + 2 * (plain + cached) + 2 * (plain + cached)), "flops": new * H * (3.0 * (G + 1) * case["rotary"] + 14 * D)}
    if kind == "weigh":
        keys = pairs = 0
        W, S = case["window"], case["sinks"]
        for length, n in zip(_lengths(case), _new(case)):
            for p in range(max(0, length - n), length):
                lo = max(0, p - W + 1) if W else 0
                pairs += p + 1 - lo + min(S, lo)
            if length and n:
                lo = max(0, length - n - W + 1) if W else 0
                keys += length - lo + min(S, lo)
        weights = sum(_lengths(case)) * H * (4 if case["decay"] == 0 else 8)
        return {"bytes": keys * cached + 2 * new * H * G * D + weights, "flops": 2.0 * pairs * H * G * D}
    kept = sum(min(n, case["budget"]) for n in _lengths(case))
    return {"bytes": sum(_lengths(case)) * H * 4 + kept * (8 * H + 2 * 2 * cached + 2 * (cached + plain)), "flops": sum(_lengths(case)) * H * 4.0}


# ---------------------------------------------------------------- inputs ----
_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def _rows(g, shape, dtype):
    """Projections: N(0, 1) with a few heavy channels, as keys have them, and tokens of different size."""
    x = torch.randn(shape, generator=g, device="cuda")
    x[..., 5::37] *= 3.0
    x *= torch.exp(0.3 * torch.randn(shape[:-1] + (1,), generator=g, device="cuda"))
    return x.to(dtype)


def _frequencies(pairs, scaled):
    """Radians a position, in 64 bits: 10000^(-i / pairs); scaled: slow ones (less than a turn in 4096 positions) 8 times slower,
    fast ones (32 turns and more) as they are, a ramp between."""
    f = 10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)
    if scaled:
        keep = ((f * 4096 / (2 * math.pi) - 1) / 31).clamp(0, 1)
        f = f * (keep + (1 - keep) / 8)
    return f.cuda()


def _pages(case, g, lengths, spare):
    """A page table over pages in random order, and how many pages there are."""
    ps = case["page"]
    of = [-(-n // ps) for n in lengths]
    order = torch.randperm(sum(of) + spare, generator=g, device="cuda").to(torch.int32).cpu()
    table = torch.zeros((len(of), max(1, max(of))), dtype=torch.int32)
    at = 0
    for b, n in enumerate(of):
        table[b, :n] = order[at:at + n]
        at += n
    return table.cuda(), order[at:].cuda(), len(order)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype, kind = _TYPES[case["dtype"]], case["kind"]
    if kind == "product":
        M, N, K, group = case["M"], case["N"], case["K"], case["group"]
        codes = torch.randn((N, K), generator=g, device="cuda").mul_(3.0).add_(8.0).floor_().clamp_(0, 15).to(torch.uint8)
        scales = (torch.rand((N, -(-K // group)), generator=g, device="cuda").add_(0.3) / math.sqrt(K) / 6.0).to(dtype)
        s = dict(case=case, x=_rows(g, (M, K), dtype), codes=codes, scales=scales)
        if own:  # weights are laid out once, when a model is loaded
            from paper_2409_17870_amd import binding
            s["packed"] = binding.apmm_w4_pack(codes, scales, group)
        return s
    if kind == "rotate":
        # queries and keys of a fused projection, which holds as many values as keys behind them
        heads = case["heads"]
        x = _rows(g, (case["tokens"], heads + max(1, heads // 4), case["head_dim"]), dtype)[:, :heads]
        at = torch.randint(0, case["far"], (case["tokens"],), generator=g, device="cuda", dtype=torch.int32)
        return dict(case=case, x=x, positions=at, frequencies=_frequencies(case["rotary"] // 2, case["scaled"]),
                    magnitude=1.2079441541679836 if case["scaled"] else 1.0)
    H, G, D, ps = case["kv_heads"], case["groups"], case["head_dim"], case["page"]
    lengths, new = _lengths(case), _new(case)
    kept = [min(n, case["budget"]) for n in lengths] if kind == "evict" else [0] * len(lengths)
    used = [-(-n // ps) for n in kept]
    table, free, pages = _pages(case, g, lengths, sum(used) + 3)
    starts = torch.tensor([0] + new).cumsum(0).int().cuda()
    codes = torch.empty((pages, H, 2, ps * D // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((pages, H, 2, ps), dtype=dtype, device="cuda")
    step = max(1, (1 << 25) // (H * ps * D))
    for p in range(0, pages, step):  # what earlier calls wrote
        n = min(step, pages - p)
        for i in range(2):
            u, s = _quantise(_rows(g, (n, H, ps, D), dtype))
            scales[p:p + n, :, i] = s
            codes[p:p + n, :, i] = _key_bytes(u).flatten(2) if i == 0 else _value_words(u).view(torch.uint8).flatten(2)
    s = dict(case=case, codes=codes, scales=scales, table=table, starts=starts, tokens=sum(new), longest=max(lengths), most=max(new),
             lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    if kind == "rotate_store":
        s.update(frequencies=_frequencies(case["rotary"] // 2, case["scaled"]), magnitude=1.2079441541679836 if case["scaled"] else 1.0)
        x = _rows(g, (s["tokens"], H * G + 2 * H, D), dtype)
        s.update(q=x[:, :H * G], k=x[:, H * G:H * G + H], v=x[:, H * G + H:])
        # places in the cache are not positions where tokens have been evicted: every third sequence has lost 1000 on the way
        lost = 1000 * (torch.arange(len(lengths), device="cuda") % 3 == 1)
        seq = torch.bucketize(torch.arange(s["tokens"], device="cuda"), starts[1:].long(), right=True)
        s["positions"] = (s["lengths"].long()[seq] - starts.long()[seq + 1] + torch.arange(s["tokens"], device="cuda") + lost[seq]).to(torch.int32)
    if kind == "weigh":
        s["q"] = _rows(g, (s["tokens"], H * G + 2 * H, D), dtype)[:, :H * G]
        s["weights"] = torch.exp(2.0 * torch.randn((len(lengths), H, table.shape[1] * ps), generator=g, device="cuda"))
        s["before"] = s["weights"].clone()
    if kind == "evict":
        # heavy tails, and equal ones among the light
        w = torch.exp(2.0 * torch.randn((len(lengths), H, table.shape[1] * ps), generator=g, device="cuda"))
        s["weights"] = torch.where(w < 4.0, torch.round(w * 64.0) / 64.0, w)
        to = torch.zeros((len(lengths), max(1, max(used))), dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(used):
            to[b, :n] = free[at:at + n]
            at += n
        s.update(to_table=to, to_starts=torch.tensor([0] + kept).cumsum(0).int().cuda(), kept=sum(kept))
    return s


# ------------------------------------------------------------ plain forms ---
def _quantise(x):
    """Codes (uint8) and scales of rows x: the largest magnitude / 15 in x's type, the nearest odd multiple, ties upward."""
    x32 = x.float()
    s = (x32.abs().amax(-1) / 15.0).to(x.dtype)
    s32 = s.float().unsqueeze(-1)
    t = torch.where(s32 > 0, x32 / s32, torch.zeros_like(x32))
    return (torch.floor(t * 0.5) + 8.0).clamp_(0, 15).to(torch.uint8), s


def _key_bytes(u):
    """(..., D) codes -> (..., D / 2) bytes."""
    return u[..., 0::2] | (u[..., 1::2] << 4)


def _value_16(u):
    """(..., D) codes of values -> (..., D / 4) 16-bit words."""
    w = u.to(torch.int32)
    w = w[..., 0::4] | (w[..., 1::4] << 4) | (w[..., 2::4] << 8) | (w[..., 3::4] << 12)
    return torch.where(w >= 32768, w - 65536, w).to(torch.int16)


def _value_words(u):
    """(..., tokens, D) codes -> (..., tokens / 8, D / 4, 8) 16-bit words."""
    return _value_16(u).unflatten(-2, (-1, 8)).transpose(-1, -2).contiguous()


def _values(u, s, dtype):
    """What codes and scales stand for, rounded once to dtype; what rounds beyond its largest number becomes that."""
    top = torch.finfo(dtype).max
    return ((2.0 * u.float() - 15.0) * s.float().unsqueeze(-1)).clamp_(-top, top).to(dtype)


def _key_view(s):
    c = s["case"]
    return s["codes"][:, :, 0].unflatten(-1, (c["page"], c["head_dim"] // 2))


def _word_view(s):
    c = s["case"]
    return s["codes"][:, :, 1].view(torch.int16).unflatten(-1, (c["page"] // 8, c["head_dim"] // 4, 8))


def _key_codes(b):
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)


def _value_codes(w):
    w = w.to(torch.int32)
    return torch.stack([w & 15, (w >> 4) & 15, (w >> 8) & 15, (w >> 12) & 15], -1).flatten(-2)


def _places(s, table, lengths, starts, tokens):
    """Sequence, position, page and place in the page of the last starts[b + 1] - starts[b] tokens of each sequence, and whether there is one."""
    ps = s["case"]["page"]
    i = torch.arange(tokens, device="cuda")
    seq = torch.bucketize(i, starts[1:].long(), right=True)
    pos = lengths.long()[seq] - starts.long()[seq + 1] + i
    fine = (pos >= 0) & (pos < table.shape[1] * ps)
    p = pos.clamp(0, table.shape[1] * ps - 1)
    return seq, pos, table[seq, p // ps].long(), p % ps, fine


def _plain_read(s, table, lengths, starts, tokens):
    dtype = s["scales"].dtype
    _, _, page, at, fine = _places(s, table, lengths, starts, tokens)
    none = ~fine[:, None, None]
    return (_values(_key_codes(_key_view(s)[page, :, at]), s["scales"][page, :, 0, at], dtype).masked_fill(none, 0),
            _values(_value_codes(_word_view(s)[page, :, at // 8, :, at % 8]), s["scales"][page, :, 1, at], dtype).masked_fill(none, 0))


def _plain_product(s):
    w = s["codes"].float().mul_(2.0).sub_(15.0)
    w *= s["scales"].float().repeat_interleave(s["case"]["group"], 1)[:, :w.shape[1]]
    return torch.matmul(s["x"].float(), w.t()).to(s["x"].dtype)


def _plain_rotate(s, x):
    """The angle in 64 bits, for far positions; cosine, sine and the turn in 32."""
    c = s["case"]
    half = c["rotary"] // 2
    turn = s["positions"].double()[:, None] * s["frequencies"]
    cos, sin = (f(turn).float()[:, None] * s["magnitude"] for f in (torch.cos, torch.sin))
    y, out = x.float(), x.float().clone()
    if c["interleaved"]:
        a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
        out[..., 0:2 * half:2], out[..., 1:2 * half:2] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = y[..., :half], y[..., half:2 * half]
        out[..., :half], out[..., half:2 * half] = a * cos - b * sin, a * sin + b * cos
    return out.to(x.dtype)


def _plain_store(s):
    _, _, page, at, fine = _places(s, s["table"], s["lengths"], s["starts"], s["tokens"])
    q, k = _plain_rotate(s, s["q"]), _plain_rotate(s, s["k"])
    page, at = page[fine], at[fine]
    uk, sk = _quantise(k[fine])
    uv, sv = _quantise(s["v"][fine])
    s["scales"][page, :, 0, at] = sk
    s["scales"][page, :, 1, at] = sv
    _key_view(s)[page, :, at] = _key_bytes(uk)
    _word_view(s)[page, :, at // 8, :, at % 8] = _value_16(uv)
    return (q,) + _plain_read(s, s["table"], s["lengths"], s["starts"], s["tokens"])


def _plain_weigh(s):
    c, q = s["case"], s["q"]
    H, G, D, ps = c["kv_heads"], c["groups"], c["head_dim"], c["page"]
    B, n, wide = c["sequences"], s["most"], s["table"].shape[1]
    L = wide * ps
    page = s["table"].long()
    k = _key_codes(_key_view(s).transpose(1, 2)[page]).float().mul_(2.0).sub_(15.0)       # B, pages, page, H, D
    k *= s["scales"][:, :, 0].transpose(1, 2)[page].float().unsqueeze(-1)
    k = k.reshape(B, L, H, D).permute(0, 2, 3, 1).contiguous()
    seq, pos, _, _, _ = _places(s, s["table"], s["lengths"], s["starts"], s["tokens"])
    row = torch.arange(s["tokens"], device="cuda") - s["starts"].long()[seq]
    x = torch.zeros((B, n, H, G, D), device="cuda")
    x[seq, row] = q.unflatten(1, (H, G)).float()
    at = torch.full((B, n), -1, dtype=torch.long, device="cuda")
    at[seq, row] = pos
    key = torch.arange(L, device="cuda")
    seen = (key <= at[..., None]) & (key < s["lengths"].long()[:, None, None])            # B, n, L
    if c["window"]:
        seen &= (key > at[..., None] - c["window"]) | (key < c["sinks"])
    x = x.permute(0, 2, 3, 1, 4).reshape(B, H, G * n, D)
    y = torch.matmul(x, k).mul_(1.0 / math.sqrt(D)).view(B, H, G, n, L)
    y.masked_fill_(~seen[:, None, None], float("-inf"))
    top = y.amax(-1, keepdim=True)
    y.sub_(torch.where(top == float("-inf"), torch.zeros_like(top), top)).exp_()
    total = y.sum(-1, keepdim=True)
    y.div_(torch.where(total > 0, total, torch.ones_like(total)))
    there = (key < s["lengths"].long()[:, None])[:, None]
    w = s["weights"]
    more = y.sum((2, 3))
    w.copy_(torch.where(there, more if c["decay"] == 0 else w * c["decay"] + more, w))
    return w


def _plain_evict(s):
    c = s["case"]
    B, H, ps, budget = c["sequences"], c["kv_heads"], c["page"], c["budget"]
    w, length = s["weights"], s["lengths"].long()
    j = torch.arange(w.shape[2], device="cuda")
    there = j < length[:, None]
    held = there & ((j < c["sinks"]) | (j >= length[:, None] - c["recent"]))
    value = torch.where(held[:, None], float("inf"), torch.where(there[:, None], w, float("-inf")))
    order = torch.sort(value, dim=2, descending=True, stable=True).indices[:, :, :budget]
    to = length.clamp(max=budget)
    i = torch.arange(order.shape[2], device="cuda")
    src = torch.sort(torch.where(i < to[:, None, None], order, w.shape[2]), dim=2).values
    kept = torch.full((B, H, budget), -1, dtype=torch.int32, device="cuda")
    weights = torch.zeros((B, H, budget), device="cuda")
    fine = (i < to[:, None, None]).expand_as(src)
    kept[:, :, :len(i)] = torch.where(fine, src, -1).to(torch.int32)
    weights[:, :, :len(i)] = torch.where(fine, w.gather(2, src.clamp(max=w.shape[2] - 1)), 0.0)
    b, h, d = fine.nonzero(as_tuple=True)
    f = src[b, h, d]
    page, at, to_page, to_at = s["table"][b, f // ps].long(), f % ps, s["to_table"][b, d // ps].long(), d % ps
    s["scales"][to_page, h, :, to_at] = s["scales"][page, h, :, at]
    _key_view(s)[to_page, h, to_at] = _key_view(s)[page, h, at]
    _word_view(s)[to_page, h, to_at // 8, :, to_at % 8] = _word_view(s)[page, h, at // 8, :, at % 8]
    to = to.to(torch.int32)
    return (kept, weights, to) + _plain_read(s, s["to_table"], to, s["to_starts"], s["kept"])


# ------------------------------------------------------------------- run ----
def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if kind == "weigh" and c["decay"]:
        s["weights"].copy_(s["before"])  # a pass adds to what earlier calls gave: the same each time
    if own:
        from paper_2409_17870_amd import binding
        if kind == "product":
            return binding.apmm_w4_gemm(s["x"], s["packed"], c["N"], c["group"])
        if kind == "rotate":
            return binding.apmm_rotary(s["x"], s["positions"], s["frequencies"], interleaved=c["interleaved"], magnitude=s["magnitude"])
        if kind == "rotate_store":
            q = binding.apmm_kv_write_rotary(s["q"], s["k"], s["v"], s["codes"], s["scales"], s["table"], s["lengths"], s["frequencies"], s["starts"],
                                             positions=s["positions"], interleaved=c["interleaved"], magnitude=s["magnitude"])
            return (q,) + tuple(binding.apmm_kv_read(s["codes"], s["scales"], s["table"], s["lengths"], s["tokens"], s["starts"]))
        if kind == "weigh":
            return binding.apmm_kv_weights(s["q"], s["codes"], s["scales"], s["table"], s["lengths"], s["weights"], s["starts"],
                                           window=c["window"], sinks=c["sinks"], decay=c["decay"])
        kept, weights, lengths = binding.apmm_kv_evict(s["codes"], s["scales"], s["table"], s["lengths"], s["weights"], c["budget"], s["to_table"],
                                                       sinks=c["sinks"], recent=c["recent"])
        return (kept, weights, lengths) + tuple(binding.apmm_kv_read(s["codes"], s["scales"], s["to_table"], lengths, s["kept"], s["to_starts"]))
    if kind == "product":
        return _plain_product(s)
    if kind == "rotate":
        return _plain_rotate(s, s["x"])
    return {"rotate_store": _plain_store, "weigh": _plain_weigh, "evict": _plain_evict}[kind](s)


# ----------------------------------------------------------------- exact ----
def _turned(s, x):
    """Pairs as complex numbers, turned in 64 bits."""
    c, y = s["case"], x.double()
    r = c["rotary"]
    front = y[..., :r]
    pairs = front.unflatten(-1, (-1, 2)) if c["interleaved"] else front.unflatten(-1, (2, -1)).transpose(-1, -2)
    angle = s["positions"].double()[:, None, None] * s["frequencies"]
    z = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.full_like(angle, s["magnitude"]), angle)
    z = torch.view_as_real(z)
    return torch.cat([z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2), y[..., r:]], -1)


def _grid(x):
    """Values in 64 bits on the grid of each row: s = max |x| / 15 rounded to x's type, odd multiples of s."""
    y = x.double()
    s = (y.abs().amax(-1, keepdim=True) / 15).to(x.dtype).double()
    odd = 2 * torch.floor(y / torch.where(s > 0, s, torch.ones_like(s)) / 2) + 1      # the odd integer above the even one at or below y / s
    return odd.clamp(-15, 15) * s


def _history(s, b, h, t, which):
    """Keys (which = 0) or values (1) of tokens t of sequence b and head h, in 64 bits: tokens x D."""
    c, ps, D = s["case"], s["case"]["page"], s["case"]["head_dim"]
    page, at = s["table"][b, t // ps].long(), t % ps
    d = torch.arange(D, device="cuda")
    if which == 0:
        byte, high = at[:, None] * (D // 2) + d // 2, d % 2 == 1
    else:
        byte, high = ((at[:, None] // 8 * (D // 4) + d // 4) * 8 + at[:, None] % 8) * 2 + d % 4 // 2, d % 4 % 2 == 1
    u = s["codes"][:, h, which][page[:, None], byte]
    u = torch.where(high, torch.div(u, 16, rounding_mode="floor"), u % 16).double()
    return (2 * u - 15) * s["scales"][page, h, which, at].double()[:, None]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "product":
        out = torch.zeros((case["M"], case["N"]), dtype=torch.float64, device="cuda")
        for i in range(0, case["K"], case["group"]):
            u = s["codes"][:, i:i + case["group"]].double()
            out += (s["x"][:, i:i + case["group"]].double() @ (2 * u - 15).t()) * s["scales"][:, i // case["group"]].double()
        return out
    if kind == "rotate":
        return _turned(s, s["x"])
    H, G, D = case["kv_heads"], case["groups"], case["head_dim"]
    lengths, new = _lengths(case), _new(case)
    if kind == "rotate_store":
        placed = torch.cat([torch.arange(n, device="cuda") + (length - n) >= 0 for length, n in zip(lengths, new)])[:, None, None]
        k = _turned(s, s["k"]).to(s["k"].dtype)  # keys are rounded to their type before they are quantised
        return (_turned(s, s["q"]),) + tuple(torch.where(placed, _grid(x), torch.zeros((), dtype=torch.float64, device="cuda")) for x in (k, s["v"]))
    if kind == "weigh":
        out = s["before"].double()
        at = 0
        for b, (length, n) in enumerate(zip(lengths, new)):
            if length:
                p = torch.arange(length - n, length, device="cuda")[:, None]
                j = torch.arange(length, device="cuda")[None]
                hidden = j > p
                if case["window"]:
                    hidden = hidden | ((j <= p - case["window"]) & (j >= case["sinks"]))
                for h in range(H):
                    k = _history(s, b, h, j[0], 0)
                    out[b, h, :length] *= case["decay"]
                    for i in range(h * G, h * G + G):
                        x = s["q"][at:at + n, i].double() @ k.t() / math.sqrt(D)
                        x[hidden] = -math.inf
                        out[b, h, :length] += torch.softmax(x, dim=1).nan_to_num_().sum(0)  # (a query that sees nothing)
            at += n
        return out
    weights = torch.zeros((len(lengths), H, case["budget"]), dtype=torch.float64, device="cuda")
    k, v = (torch.zeros((s["kept"], H, D), dtype=torch.float64, device="cuda") for _ in range(2))
    at = 0
    for b, n in enumerate(lengths):
        m = min(n, case["budget"])
        for h in range(H):
            w = s["weights"][b, h, :n].double()
            first, last = min(case["sinks"], n), max(n - case["recent"], min(case["sinks"], n))
            if m == n:
                t = torch.arange(n, device="cuda")
            else:
                middle = w[first:last]
                rest = m - first - (n - last)
                # the lightest that stays, all above it, and as many of its equals as there is room for, lower places first
                border = torch.kthvalue(middle, len(middle) - rest + 1).values if rest else torch.tensor(math.inf, device="cuda")
                above, equal = middle > border, middle == border
                stays = above | (equal & (equal.long().cumsum(0) <= rest - above.long().sum()))
                t = torch.cat([torch.arange(first, device="cuda"), stays.nonzero()[:, 0] + first, torch.arange(last, n, device="cuda")])
            weights[b, h, :m] = w[t]
            k[at:at + m, h], v[at:at + m, h] = _history(s, b, h, t, 0), _history(s, b, h, t, 1)
        at += m
    return None, weights, None, k, v
